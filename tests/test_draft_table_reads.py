"""Host side, no GPU: where chunk attention reads the block table, for every place of every step of a tile, stays within a row's pages, also where the context or the
whole window lies behind the last of them.  A read beyond would change no result, so only the arithmetic can show it."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17133_amd", "csrc")

# a sequence's tiles as chunk.hip goes through them: its steps, and those that are looked up ahead of them; lowest and highest page that is read
CODE = """
#include "chunk_span.h"
extern "C" void pages_read(int context, int fresh, int group, int rows, int step, int tree, int window, int sinks, int page, int max_pages, int there, long long* lowest,
                           long long* highest, long long* counted)
{
    const int cap = there ? page * max_pages : 0;
    *lowest = *highest = *counted = 0;
    for (int tile = 0; tile < (fresh * group + rows - 1) / rows; ++tile) {
        const int j0 = tile * rows / group, last = (tile * rows + rows - 1) / group, j1 = last < fresh - 1 ? last : fresh - 1;
        const bmoe::Span s(context, fresh, j0, j1, tree != 0, window, sinks, cap);
        const int steps = s.n > step ? (s.n + step - 1) / step : 1;
        for (int i = 0; i < (steps + 5) * step; ++i) {
            const long long pos = s.read(i, s.n), at = pos < 0 ? pos : pos / page;
            if (at < *lowest) *lowest = at;
            if (at > *highest) *highest = at;
            if (i < s.n) ++*counted;
        }
    }
}
"""


@pytest.fixture(scope="module")
def pages_read(tmp_path_factory):
    d = tmp_path_factory.mktemp("span")
    (d / "span.cpp").write_text(CODE)
    so = str(d / "span.so")
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-D__host__=", "-D__device__=", "-I", CSRC, str(d / "span.cpp"), "-o", so], check=True)
    f = C.CDLL(so).pages_read

    def call(*args):
        out = [C.c_longlong() for _ in range(3)]
        f(*args, *(C.byref(o) for o in out))
        return [o.value for o in out]
    return call


@pytest.mark.parametrize("tree", [0, 1])
@pytest.mark.parametrize("page,max_pages", [(1, 1), (16, 1), (16, 3), (3, 50)])
def test_within_the_row(pages_read, page, max_pages, tree):
    cap = page * max_pages
    for context in sorted({0, 1, cap - 1, cap, cap + 1, cap + 7, cap + 40, 3 * cap + 100, 1 << 30, 0x7FFE0000}):
        for window in (0, 1, 8, 33, 1 << 29, (1 << 31) - 1):
            for sinks in (0, 1, 5, 1000):
                for fresh, group in ((1, 1), (9, 4), (70, 8)):
                    for there in (0, 1):
                        args = (context, fresh, group, 32, 64, tree, window, sinks, page, max_pages, there)
                        lowest, highest, counted = pages_read(*args)
                        assert lowest == 0 and highest < max_pages, args
                        assert there or counted == 0, args


@pytest.mark.parametrize("tree", [0, 1])
def test_what_is_seen_is_counted(pages_read, tree):
    """Positions that count: of a tile of one token, exactly those it sees; one token, one head."""
    for cap in (16, 64):
        for context in (0, 3, 15, 16, 17, 40, 63, 64, 70, 100):
            for window in (0, 1, 5, 40):
                for sinks in (0, 2, 50):
                    sees = [p for p in range(min(context + 1, cap)) if window == 0 or p > context - window or p < sinks]
                    assert pages_read(context, 1, 1, 32, 64, tree, window, sinks if window else 0, 16, cap // 16, 1)[2] == len(sees), (cap, context, window, sinks)
