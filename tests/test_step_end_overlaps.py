"""Outputs that would lie in other operands' memory, by any byte: refused on the host, without a GPU.  Columns of one
wider matrix are apart."""
import shutil
import subprocess

import pytest
import torch

from paper_2608_05088_gb300 import build, malt
from tests.test_step_end_refusals import BAD, BF16, head

A = 1 << 20         # addresses that nothing reads: every call here fails before a launch
M = 1 << 16


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would be launched")
    build.build()
    return malt.load()


# 8 rows of 64 against 100 entries, bf16: 1 KB of hidden rows, 12800 bytes of table, 32 of labels, weights and losses
PLACES = dict(hidden=A, table=A + M, labels=A + 2 * M, weight=A + 3 * M, loss=A + 4 * M, stats=A + 5 * M, dhidden=A + 6 * M,
              dtable=A + 7 * M, dloss=A + 8 * M, ws=A + 16 * M)
WRITTEN, READ = ("loss", "stats", "dhidden", "dtable", "ws"), ("hidden", "table", "labels", "weight")
SIZE = dict(hidden=1024, table=12800, labels=32, weight=32, loss=32, stats=64, dhidden=1024, dtable=12800, dloss=32)


def call_head(lib, dh_ld=64, dt_ld=64, only=None, rows=8, **kw):
    at = PLACES | kw
    ld = dict(hidden_ld=at.get("h_ld", 64), table_ld=at.get("t_ld", 64))
    h = head(hidden=at["hidden"], table=at["table"], labels=at["labels"], weight=at["weight"], rows=rows, **ld)
    size = lib.malt_head_workspace_bytes(h, 1, 1)
    out = (at["dhidden"], dh_ld, at["dtable"], dt_ld, BF16, 0)
    if only == "gradient":
        return lib.malt_head_backward(h, at["stats"], at["dloss"], *out, at["ws"], size, None)
    if only == "forward":
        return lib.malt_head_forward(h, at["loss"], at["stats"], at["ws"], size, None)
    return lib.malt_head_forward_backward(h, at["loss"], at["stats"], *out, at["ws"], size, None)


def test_head(lib):
    for only, written, read in ((None, WRITTEN, READ), ("forward", ("loss", "stats", "ws"), READ),
                                ("gradient", ("dhidden", "dtable", "ws"), READ + ("stats", "dloss"))):
        size = dict(SIZE, ws=lib.malt_head_workspace_bytes(head(), only != "gradient", only != "forward"))
        for o in written:
            for other in read + written:
                if o != other:
                    for shift in (0, (size[other] - 16) // 256 * 256, -((size[o] - 16) // 256 * 256)):
                        assert call_head(lib, only=only, **{o: PLACES[other] + shift}) == BAD, (only, o, other, shift)


@pytest.mark.parametrize("first", [56, 104, -56, 160 + 40, 160 * 7, -160 * 7 - 56])
def test_head_in_one_matrix(lib, first):
    """dhidden among hidden's rows of 64, 160 apart, over some of their entries."""
    assert call_head(lib, h_ld=160, dh_ld=160, dhidden=PLACES["hidden"] + 2 * first) == BAD
    assert call_head(lib, h_ld=160, dh_ld=200, dhidden=PLACES["hidden"] + 2 * 64) == BAD


SOURCE = r"""
#include "extent.h"
#include <cstdio>
#include <random>
#include <set>
using namespace malt;

int main() {
    std::mt19937 rng(5);
    auto any = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    char* const base = (char*)0x100000;
    int shared = 0, apart = 0;
    for (int i = 0; i < 200000; ++i) {
        const int lds[] = {any(1, 12), any(1, 12)};
        Extent e[2];
        for (int k = 0; k < 2; ++k) {
            const int64_t ld = any(0, 2) ? lds[0] : lds[k];
            e[k] = {base + any(0, 60), any(0, 5), any(0, 8) ? any(1, (int)ld) : ld, ld};
            if (any(0, 5) == 0) e[k] = extent_of(base + any(0, 60), any(0, 30));
        }
        std::set<int64_t> mine;
        for (int64_t r = 0; r < e[0].rows; ++r)
            for (int64_t b = 0; b < e[0].bytes; ++b) mine.insert((int64_t)e[0].p + r * e[0].ld + b);
        bool want = false;
        for (int64_t r = 0; r < e[1].rows; ++r)
            for (int64_t b = 0; b < e[1].bytes; ++b) want |= mine.count((int64_t)e[1].p + r * e[1].ld + b) > 0;
        const bool got = overlap(e[0], e[1]), same = e[0].ld == e[1].ld || e[0].rows <= 1 || e[1].rows <= 1;
        if (got != overlap(e[1], e[0]) || (want && !got) || (same && want != got)) {
            std::printf("%d: %d %d\n", i, want, got);
            return 1;
        }
        ++(want ? shared : apart);
    }
    if (shared < 10000 || apart < 10000 || overlap(Extent{}, {base, 1, 1, 1})) return 2;
    std::puts("fine");
}
"""


def test_overlap_is_that_of_the_bytes(tmp_path):
    """Against sets of bytes; at two strides nothing that overlaps is missed."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "extent.cpp", tmp_path / "extent"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout.strip() == "fine", run.stdout
