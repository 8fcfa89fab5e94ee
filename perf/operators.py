"""The operators over a paged cache, timed one by one, each with its plain form beside the library's call.

A serving step appends a few tokens to every request of a batch.  Its three operators, in the order of the step:

  tables   block tables, row offsets, positions and slots of the step, from the requests' lengths and the free pages
  append   the new rows' queries and keys rotated to their positions, keys and values stored at their slots of the pages
  attn     attention of the new rows over the pages: every row sees its request's cache and its own chunk up to itself

Page r of a request holds its positions r * page .. r * page + page - 1; pages lie in the cache in no order.  The lengths of a
case's requests follow from the case alone, everything else from the seed.
"""
import functools
import math
import random

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}

GQA4 = dict(q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", rope_base=500000.0)    # the 8B-class layer
GQA7 = dict(q_heads=28, kv_heads=4, head_dim=128, dtype="bf16", rope_base=1000000.0)   # the 7B-class layer with 4 KV heads
GQA8 = dict(q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", rope_base=500000.0)
MHA64 = dict(q_heads=16, kv_heads=8, head_dim=64, dtype="bf16", rope_base=500000.0)    # small models, head_dim 64
TINY32 = dict(q_heads=4, kv_heads=4, head_dim=64, dtype="f32", rope_base=10000.0)      # fp32: verification runs


def _batch(requests, chunked, new, cached, page, lengths):
    """`chunked` of the requests bring new[0] .. new[1] rows, the others one; cached[0] .. cached[1] positions are there already."""
    return dict(requests=requests, chunked=chunked, new_lo=new[0], new_hi=new[1], cached_lo=cached[0], cached_hi=cached[1], page=page, lengths=lengths)


def listed():
    return [
        # The tables of a decoding step of 64 requests: the smallest call of a step, launches and latency.
        dict(name="tables_decode_64", kind="tables", **_batch(64, 0, (1, 1), (100, 16896), 16, 1), padding=0),
        # A full step of 256 requests, 32 of them with a chunk of their prompt, in buffers of fixed size as a captured graph has them.
        dict(name="tables_mixed_256", kind="tables", **_batch(256, 32, (128, 1024), (1, 16896), 32, 2), padding=1000),
        # A decoding step's rows into the pages.
        dict(name="append_decode_64", kind="append", **GQA4, half_layout=False, **_batch(64, 0, (1, 1), (100, 4000), 16, 3)),
        # A prompt's rows of the ordinary request, all at once: streaming.
        dict(name="append_prompt_17k", kind="append", **GQA4, half_layout=False, **_batch(1, 1, (16896, 16896), (0, 0), 64, 4)),
        # Chunks of odd lengths on a small model in the half-split rotary layout.
        dict(name="append_ragged_d64", kind="append", **MHA64, half_layout=True, **_batch(9, 8, (77, 999), (0, 3000), 24, 5)),
        # One request's decoding step: too little work to fill the chip, latency.
        dict(name="attn_one_4k", kind="attn", **GQA4, **_batch(1, 0, (1, 1), (4096, 4096), 16, 6)),
        # A decoding step of a full batch of all lengths: streaming.
        dict(name="attn_decode_64", kind="attn", **GQA4, **_batch(64, 0, (1, 1), (500, 16896), 16, 7)),
        # Drafted tokens of 32 requests verified on a small model, a few rows each, pages of 8.
        dict(name="attn_verify_d64", kind="attn", **MHA64, **_batch(32, 32, (2, 8), (300, 6000), 8, 8)),
        # A chunk of a long prompt behind its first 14k positions: the work of a chunked prefill.
        dict(name="attn_chunk_2k", kind="attn", **GQA4, **_batch(1, 1, (2048, 2048), (14336, 14336), 64, 9)),
        # A prompt of the ordinary length from nothing: the largest product.
        dict(name="attn_prompt_17k", kind="attn", **GQA4, **_batch(1, 1, (16896, 16896), (0, 0), 64, 10)),
        # One chunk beside eight decoding requests, seven query heads per KV head, odd lengths.
        dict(name="attn_mixed_group7", kind="attn", **GQA7, **_batch(9, 1, (777, 777), (1000, 8000), 32, 11)),
        # fp32, ragged chunks: a verification run.
        dict(name="attn_tiny_f32", kind="attn", **TINY32, **_batch(5, 4, (3, 300), (0, 1000), 16, 12)),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], uniform in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng):
    kind = rng.choice(["tables", "append", "append"] + ["attn"] * 7)
    lengths = rng.randrange(1 << 30)
    page = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 128, 256])
    if kind == "tables":
        requests = _spread(rng, 1, 512)
        chunked = rng.choice([0, rng.randint(0, min(requests, 32))])
        return dict(kind=kind, **_batch(requests, chunked, (2, _spread(rng, 2, 1024)), (0, _spread(rng, 1, 16896)), page, lengths), padding=rng.choice([0, rng.randint(1, 2000)]))
    if kind == "append":
        requests = _spread(rng, 1, 64)
        chunked = rng.randint(0, min(requests, 8))
        return dict(kind=kind, **rng.choice([GQA4, GQA7, GQA8, MHA64, TINY32]), half_layout=rng.random() < 0.5,
                    **_batch(requests, chunked, (2, _spread(rng, 2, 1000)), (0, _spread(rng, 1, 3000)), page, lengths))
    layer = rng.choice([GQA4, GQA4, GQA7, GQA8, MHA64, TINY32])
    form = rng.choice(["decode", "decode", "verify", "chunk", "chunk", "prompt", "mixed"])
    small = layer is TINY32
    top = 2000 if small else 16896
    if form == "decode":
        batch = _batch(_spread(rng, 1, 64), 0, (1, 1), (1, _spread(rng, 10, top)), page, lengths)
    elif form == "verify":
        requests = _spread(rng, 1, 32)
        batch = _batch(requests, requests, (2, rng.randint(2, 16)), (0, _spread(rng, 10, top // 2)), page, lengths)
    elif form == "chunk":
        new, cached = _spread(rng, 16, 300 if small else 2048), _spread(rng, 1, top - 2000 if not small else 1000)
        requests = rng.randint(1, 3)
        batch = _batch(requests, requests, (max(1, new // 3), new), (cached // 2, cached), page, lengths)
    elif form == "prompt":
        new = _spread(rng, 5, 600 if small else 8000)
        batch = _batch(1, 1, (new, new), (0, 0), page, lengths)
    else:
        batch = _batch(rng.randint(2, 9), 1, (2, _spread(rng, 10, 300 if small else 777)), (0, _spread(rng, 10, top // 2)), page, lengths)
    return dict(kind=kind, **layer, **batch)


# ---- sizes that follow from a case ----------------------------------------------------------------------------------

def _lengths(case):
    """[(positions cached, new rows)] of the requests; those with a chunk are spread over the batch."""
    rng = random.Random(case["lengths"])
    n = case["requests"]
    chunked = set(rng.sample(range(n), case["chunked"]))
    return [(_spread(rng, case["cached_lo"], case["cached_hi"]), _spread(rng, case["new_lo"], case["new_hi"]) if b in chunked else 1) for b in range(n)]


def _pages(n, page):
    return (n + page - 1) // page


def work(case):
    lens, page = _lengths(case), case["page"]
    rows = sum(n for _, n in lens)
    if case["kind"] == "tables":
        taken = sum(_pages(c + n, page) - _pages(c, page) for c, n in lens)
        there = sum(1 for c, _ in lens if c % page)          # pages that are there already and take new rows
        return {"bytes": 4 * (2 * len(lens) + taken + there + taken + len(lens) + 1 + 2 * (rows + case["padding"]) + 2), "flops": 4 * rows}
    es, d = TORCH[case["dtype"]].itemsize, case["head_dim"]
    q, kv = case["q_heads"] * d, case["kv_heads"] * d
    if case["kind"] == "append":
        return {"bytes": 2 * es * rows * (q + 2 * kv) + 8 * rows, "flops": 3 * rows * (q + kv)}
    seen = sum(c + n for c, n in lens)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in lens)
    return {"bytes": 2 * es * rows * q + 4 * rows * case["q_heads"] + 2 * es * seen * kv + 4 * sum(_pages(c + n, page) + 2 for c, n in lens),
            "flops": 4 * pairs * q}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    lens, page = _lengths(case), case["page"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    n, rows = len(lens), sum(m for _, m in lens)
    cached, new = i32([c for c, _ in lens]), i32([m for _, m in lens])
    before = [_pages(c, page) for c, _ in lens]
    after = [_pages(c + m, page) for c, m in lens]
    width = max(after) + 1
    full = case["kind"] != "tables"
    used = sum(after) if full else sum(before)
    spare = sum(after) - sum(before) + 3
    ids = torch.randperm(used + spare, generator=gen, device="cuda").int()
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    held = i32(after if full else before)
    column = torch.arange(width, device="cuda")
    table[column[None, :] < held[:, None]] = ids[:used]
    st = dict(case=case, cached=cached, new=new, table=table, n=n, rows=rows, page=page, width=width)
    if case["kind"] == "tables":
        st["free"], st["start"] = ids[used:].contiguous(), torch.randint(0, 3, (1,), generator=gen, device="cuda", dtype=torch.int32)
        st["rows"] = rows + case["padding"]
        st["out"] = dict(offsets=torch.empty(n + 1, dtype=torch.int32, device="cuda"), positions=torch.empty(st["rows"], dtype=torch.int32, device="cuda"),
                         slots=torch.empty(st["rows"], dtype=torch.int32, device="cuda"), needed=torch.empty(1, dtype=torch.int32, device="cuda"))
        return st
    t, d, hq, hkv = TORCH[case["dtype"]], case["head_dim"], case["q_heads"], case["kv_heads"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(t)

    st["q"] = normal(rows, hq, d)
    pages = (used + spare, page, hkv, d)
    if case["kind"] == "append":
        request = torch.repeat_interleave(torch.arange(n, device="cuda"), new.long())
        first = torch.cumsum(new.long(), 0) - new
        at = cached[request].long() + torch.arange(rows, device="cuda") - first[request]
        st["positions"] = at.int()
        st["slots"] = (table[request, at // page].long() * page + at % page).int()
        st["k"], st["v"] = normal(rows, hkv, d), normal(rows, hkv, d)
        st["k_pages"], st["v_pages"] = torch.zeros(pages, dtype=t, device="cuda"), torch.zeros(pages, dtype=t, device="cuda")
        st["q_out"] = torch.empty_like(st["q"])
        return st
    st["k_pages"], st["v_pages"] = normal(*pages), normal(*pages)
    # logits of a trained head's spread; the first position of every request stands out
    st["k_pages"].view(-1, hkv, d)[table[:, 0].long() * page] *= 1.5
    st["q"] *= 1.5
    st["max_new"], st["max_seen"] = max(m for _, m in lens), max(c + m for c, m in lens)
    st["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cumsum(new, 0, dtype=torch.int32)])
    st["out"] = torch.empty_like(st["q"])
    st["lse"] = torch.empty((rows, hq), dtype=torch.float32, device="cuda")
    return st


# ---- the operators ------------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context(q_heads, kv_heads, head_dim, dtype, rope_base, half_layout):
    """The library's handle of a layer shape, which a program keeps."""
    from paper_2601_12904_amd import binding as B
    return B.Context(q_heads, kv_heads, head_dim, B.FR_BF16 if dtype == "bf16" else B.FR_F32, rope_base, max_tokens=1024, max_chunks=1, max_question_tokens=1,
                     rope_layout=B.FR_ROPE_HALF if half_layout else B.FR_ROPE_INTERLEAVED)


def _context_of(case):
    c = dict(GQA4, half_layout=False) | case
    return _context(c["q_heads"], c["kv_heads"], c["head_dim"], c["dtype"], c["rope_base"], c["half_layout"])


def run(st):
    return {"tables": _tables, "append": _append, "attn": _attn}[st["case"]["kind"]](st)


def _tables(st):
    o = st["out"]
    if own:
        _context_of(st["case"]).fr_page_tables(st["cached"], st["new"], st["n"], st["page"], st["free"], st["free"].numel(), st["start"], st["table"], st["width"],
                                               st["rows"], o["offsets"], o["positions"], o["slots"], o["needed"])
        return dict(o, table=st["table"])
    page, width, rows, table = st["page"], st["width"], st["rows"], st["table"]
    cached = st["cached"].long()
    offsets = torch.cat([cached.new_zeros(1), torch.cumsum(st["new"], 0)]).clamp(max=rows)
    new = offsets[1:] - offsets[:-1]
    first = torch.clamp((cached + page - 1) // page, max=width)
    last = torch.clamp((cached + new + page - 1) // page, max=width)
    taken = last - first
    begin = torch.cumsum(taken, 0) - taken
    column = torch.arange(width, device="cuda")[None, :]
    source = st["start"].long() + begin[:, None] + column - first[:, None]
    there = source < st["free"].numel()
    page_id = torch.where(there, st["free"][source.clamp(0, st["free"].numel() - 1)], -1)
    table.copy_(torch.where((column >= first[:, None]) & (column < last[:, None]), page_id, table))
    row = torch.arange(rows, device="cuda")
    valid = row < offsets[-1]
    request = torch.searchsorted(offsets[1:], row, right=True).clamp(max=st["n"] - 1)
    position = torch.where(valid, cached[request] + row - offsets[request], 0)
    block = position // page
    at = table[request, block.clamp(max=width - 1)].long()
    slot = torch.where(valid & (block < width) & (at >= 0), at * page + position % page, -1)
    return dict(offsets=offsets.int(), positions=position.int(), slots=slot.int(), needed=taken.sum().int().reshape(1), table=table)


def _rotate(x, positions, case):
    """Rotary embedding of [rows, heads, d] in 32 bits, the angles in 64."""
    d = case["head_dim"]
    theta = case["rope_base"] ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    angle = positions.double()[:, None, None] * theta
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = (x[..., : d // 2].float(), x[..., d // 2:].float()) if case["half_layout"] else (x[..., 0::2].float(), x[..., 1::2].float())
    y = a * cos - b * sin, b * cos + a * sin
    return (torch.cat(y, -1) if case["half_layout"] else torch.stack(y, -1).flatten(-2)).to(x.dtype)


def _append(st):
    case = st["case"]
    if own:
        _context_of(case).fr_paged_append(st["q"], st["k"], st["v"], st["positions"], st["slots"], st["rows"], st["k_pages"], st["v_pages"], st["k_pages"].shape[0],
                                          st["page"], st["q_out"])
        return dict(q=st["q_out"], k_pages=st["k_pages"], v_pages=st["v_pages"])
    slots = st["slots"].long()
    st["k_pages"].flatten(0, 1)[slots] = _rotate(st["k"], st["positions"], case)
    st["v_pages"].flatten(0, 1)[slots] = st["v"]
    return dict(q=_rotate(st["q"], st["positions"], case), k_pages=st["k_pages"], v_pages=st["v_pages"])


def _attn(st):
    case = st["case"]
    if own:
        _context_of(case).fr_paged_attn(st["q"], st["offsets"], st["cached"], st["n"], st["rows"], st["max_new"], st["k_pages"], st["v_pages"], st["k_pages"].shape[0],
                                        st["page"], st["table"], st["width"], st["out"], st["lse"])
        return dict(out=st["out"], lse=st["lse"])
    # requests side by side, padded to the most rows and positions of one of them
    n, page, hq, hkv, d = st["n"], st["page"], case["q_heads"], case["kv_heads"], case["head_dim"]
    group, many, seen = hq // hkv, st["max_new"], st["max_seen"]
    key = torch.arange(seen, device="cuda")
    slot = st["table"][:, key // page].long().clamp(min=0) * page + key % page                     # [n, seen]
    k, v = (p.flatten(0, 1)[slot].float().transpose(1, 2) for p in (st["k_pages"], st["v_pages"]))   # [n, hkv, seen, d]
    i = torch.arange(many, device="cuda")
    row = st["offsets"][:-1, None].long() + i                                                      # [n, many]
    inside = row < st["offsets"][1:, None]
    q = st["q"][row.clamp(max=st["rows"] - 1)].float().view(n, many, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, many * group, d)
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(n, hkv, many, group, seen)
    hidden = key > (st["cached"][:, None] + i)[..., None]                                          # [n, many, seen]
    s.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(n, hkv, many * group, seen), v).view(n, hkv, many, group, d) / total
    lse = (top + total.log()).squeeze(-1)
    o = o.permute(0, 2, 1, 3, 4).reshape(n, many, hq, d)[inside]
    return dict(out=o.to(st["q"].dtype), lse=lse.permute(0, 2, 1, 3).reshape(n, many, hq)[inside])


# ---- the definitions, in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    lens, page = _lengths(case), case["page"]
    if case["kind"] == "tables":
        return None   # whole numbers
    d, hkv, group = case["head_dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    if case["kind"] == "append":
        half = case["half_layout"]
        pair = torch.arange(d // 2, device="cuda")
        one, two = (pair, pair + d // 2) if half else (2 * pair, 2 * pair + 1)
        turn = torch.exp(-2.0 * pair.double() / d * math.log(case["rope_base"]))
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(st["rows"], 1, d // 2).contiguous(), st["positions"].double()[:, None, None] * turn)

        def turned(x):
            w = torch.complex(x[..., one].double(), x[..., two].double()) * z
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            y[..., one], y[..., two] = w.real, w.imag
            return y

        k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
        k, v, slots = turned(st["k"]), st["v"].double(), st["slots"].long()
        k_pages[slots // page, slots % page], v_pages[slots // page, slots % page] = k, v
        return dict(q=turned(st["q"]), k_pages=k_pages, v_pages=v_pages)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, (c, m) in enumerate(lens):
        blocks = st["table"][b, : _pages(c + m, page)].long()
        keys, values = (p[blocks].reshape(-1, hkv, d)[: c + m] for p in (st["k_pages"], st["v_pages"]))
        visible = torch.tril(torch.ones((m, c + m), dtype=torch.bool, device="cuda"), diagonal=c)
        for g in range(hkv):
            kd, vd = keys[:, g].double(), values[:, g].double()
            for h in range(g * group, (g + 1) * group):
                logit = torch.where(visible, st["q"][at: at + m, h].double() @ kd.T / d ** 0.5, -torch.inf)
                weight = torch.softmax(logit, -1)
                out[at: at + m, h] = weight @ vd
                lse[at: at + m, h] = torch.logsumexp(logit, -1)
        at += m
    return dict(out=out, lse=lse)
