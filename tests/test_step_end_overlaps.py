"""Outputs that would lie in other operands' memory, by any byte: refused on the host, without a GPU.  Columns of one
wider matrix are apart."""
import shutil
import subprocess

import pytest
import torch

from paper_2608_05088_gb300 import build, malt
from tests.test_step_end_refusals import BAD, BF16, F32, head, rms, rows

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


# 4 rows of 16 fp32 entries: 256 bytes; a gain of 64, scales of 16
X, S, H, Y, G, C, DG, WS = (A + k * M for k in range(8))


def test_norm(lib):
    """Offsets into an input, and outputs in one another, in the gain and in the scales."""
    def forward(x=X, s=S, h=H, y=Y, gain=G, scales=None, ld=16):
        p, r = rms(gain=gain), lambda at, dtype=F32: rows(data=at, ld=ld, dtype=dtype)
        add = (None, None) if s is None else (r(s), r(h))
        if scales is None:
            return lib.malt_rms_norm_forward(p, r(x), *add, r(y), None)
        return lib.malt_rms_norm_forward_8bit(p, r(x), *add, r(y, malt.MALT_E4M3), scales, 1, None)

    for bad in (dict(y=X + 64), dict(y=X - 64), dict(y=S + 192), dict(h=X + 16), dict(h=S - 240), dict(h=Y), dict(h=Y + 64),
                dict(y=G), dict(h=G - 240), dict(y=X + 4, s=None), dict(x=X, s=X + 64, h=X), dict(y=X + 32, ld=20),
                dict(x=X, y=X + 40, ld=24, s=None)):
        assert forward(**bad) == BAD, bad
    for bad in (dict(scales=X), dict(scales=S + 252), dict(scales=H - 12), dict(scales=Y + 60), dict(scales=G + 60),
                dict(scales=C, y=X + 255), dict(scales=C, y=C), dict(scales=C, h=C)):
        assert forward(**bad) == BAD, bad


def test_norm_gradient(lib):
    need = lib.malt_rms_norm_workspace_bytes(4, 16)

    def backward(dy=X, h=H, dh=S, dx=Y, gain=G, dgain=DG, ws=WS):
        r = lambda at: rows(data=at)
        return lib.malt_rms_norm_backward(rms(gain=gain), r(dy), r(h), r(dh), r(dx), dgain, ws, need, None)

    for bad in (dict(dx=X + 64), dict(dx=H - 240), dict(dx=S + 4), dict(dx=G), dict(dgain=X), dict(dgain=H + 252), dict(dgain=S - 60),
                dict(dgain=Y), dict(dgain=G + 60), dict(dgain=WS + need - 4), dict(ws=X), dict(ws=Y + 240), dict(ws=G - need + 16)):
        assert backward(**bad) == BAD, bad


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
