"""csrc/any4_launches.h, compiled for the host: every block of a long grid is launched once, in pieces that HIP takes (fewer than 2^32
threads along an axis), and nothing after a refusal."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_04610_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "any4_launches.h"
int main() {
    long long blocks; int threads, refuse;
    while (scanf("%lld %d %d", &blocks, &threads, &refuse) == 3) {
        int n = 0;
        const int e = any4::launch_blocks((int64_t)blocks, threads, 0, [&](int64_t first, int64_t count) {
            printf("%lld+%lld ", (long long)first, (long long)count);
            return n++ == refuse ? 7 : 0;
        });
        printf("-> %d\n", e);
    }
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="a host compiler is needed")
def test_pieces(tmp_path):
    (tmp_path / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{CSRC}", "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)
    limit = 2 ** 24 - 1                                                     # blocks of 256 threads
    cases = [(b, t, -1) for t in (256, 512) for b in (0, 1, 1000, limit, limit + 1, limit + 2, 2 * limit, 2 * limit + 1, 2 ** 31 - 1)]
    cases += [(2 ** 31 - 1, 256, 0), (2 ** 31 - 1, 256, 2), (5, 256, 0)]
    out = subprocess.run([str(tmp_path / "p")], input="\n".join("%d %d %d" % c for c in cases), capture_output=True, text=True, check=True).stdout
    for (blocks, threads, refuse), line in zip(cases, out.splitlines(), strict=True):
        pieces, code = line.split("->")
        pieces = [tuple(map(int, p.split("+"))) for p in pieces.split()]
        assert all(count > 0 and count * threads < 2 ** 32 for _, count in pieces)
        assert [f for f, _ in pieces] == [sum(c for _, c in pieces[:i]) for i in range(len(pieces))]
        if refuse < 0:
            assert int(code) == 0 and sum(c for _, c in pieces) == blocks
        else:
            assert int(code) == 7 and len(pieces) == refuse + 1
    one = [c for c in zip(cases, out.splitlines()) if c[0] == (limit, 256, -1)]
    assert one[0][1].count("+") == 1


@pytest.mark.parametrize("name", ("any4_kv_cache.hip", "any4_attn_prompt.hip"))
def test_the_kernels_go_through_it(name):
    """each launch of these files stands within launch_blocks() or launch_tokens()"""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert text.count("hipLaunchKernelGGL") == text.count("return launch_blocks(") + text.count("return launch_tokens(") - ("kv_cache" in name)
