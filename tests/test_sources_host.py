"""Every file among the sources is compiled, or is a header that one of them includes."""
import os

from paper_2601_12904_amd import build


def test_no_source_is_left_over():
    files = sorted(os.listdir(build.CSRC))
    text = "".join(open(os.path.join(build.CSRC, f)).read() for f in build.SOURCES)
    headers = [f for f in files if f.endswith(".hpp")]
    text += "".join(open(os.path.join(build.CSRC, f)).read() for f in headers)
    assert [f for f in files if f not in build.SOURCES and f not in headers] == []
    assert [f for f in headers if f'#include "{f}"' not in text] == []
