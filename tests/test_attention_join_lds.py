"""LDS of decode attention's join (csrc/any4_attn_decode.hip): the parts, pairs of floats, begin on 8 bytes behind the factors whatever the
numbers of heads and pieces are, and within what the launch asks for."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_04610_amd", "csrc", "any4_attn_decode.hip")


@pytest.fixture(scope="module")
def text():
    with open(SOURCE) as f:
        return f.read()


def expression(text, pattern):
    """the C expression that `pattern` finds, as Python's"""
    found = re.search(pattern, text)
    assert found, pattern
    return found.group(1).replace("(int)gridDim.x", "blocks").replace("(int)sizeof(float)", "4")


def test_parts_lie_on_eight_bytes_within_the_launch(text):
    body = expression(text, r"int parts_at\(int heads, int pieces\) \{ return (.*?); \}")
    names = {"parts_at": lambda heads, pieces: eval(body, {"heads": heads, "pieces": pieces})}
    parts = expression(text, r"float\* parts = lds \+ (.*?);")
    begins = expression(text, r"int\* begins = reinterpret_cast<int\*>\(lds \+ max\(.*?, (.*)\)\);")
    join = expression(text, r"join = (.*?);")
    for heads in range(1, 17):
        for blocks in (1, 2, 3, 5, 64, 255, 256, 511, 512, 767, 768):
            for pieces in range(1, blocks + 1, max(1, blocks // 40)):
                for waves in (4, 8):
                    where = dict(names, here=heads, heads=heads, most=heads, pieces=pieces, blocks=blocks, THREADS=64 * waves, WAVES=waves)
                    at = eval(parts, where)
                    assert at % 2 == 0 and at >= heads * pieces
                    # the requests' beginnings come behind the parts, and the launch counts both in the same way
                    assert at + 2 * 64 * waves <= eval(begins, where) == eval(join, where)


def test_lds_is_declared_with_the_alignment_of_its_widest_access(text):
    assert re.search(r"extern __shared__ __attribute__\(\(aligned\(16\)\)\) float lds\[\];", text)
