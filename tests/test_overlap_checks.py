"""Outputs that overlap another buffer of the call are refused (csrc/op_checks.h, compiled for the host): the check itself against
sets of bytes, and every output of the operators on weights in stacks."""
import ctypes as C
import functools
import os
import random
import subprocess
import tempfile

import pytest

from conftest import ROOT
from paper_2303_13775_amd import binding as B

CSRC = os.path.join(ROOT, "paper_2303_13775_amd", "csrc")
_SOURCE = r"""
#include "op_checks.h"
typedef const void *V;
typedef const float *F;
typedef const int32_t *I;
extern "C" int meet(V p, int64_t rows, int64_t width, int64_t stride, V q, int64_t q_rows, int64_t q_width, int64_t q_stride) {
    return op_meet(OpArea{p, rows, width, stride}, OpArea{q, q_rows, q_width, q_stride});
}
extern "C" const char *group_rows(I g, int64_t n, int32_t G, I ptr, I rows) { return op_apart_group_rows(g, n, G, ptr, rows); }
extern "C" const char *fwd(const gsplit_grouped_config *c, V x, int64_t n, int64_t ldx, I ptr, I rows, V w, F b, V y, int64_t ldy) {
    return op_apart_grouped_fwd(c, x, n, ldx, ptr, rows, w, b, y, ldy);
}
extern "C" const char *bwd(const gsplit_grouped_config *c, V x, int64_t n, int64_t ldx, I ptr, I rows, V w, V dy, int64_t lddy, V dx, int64_t lddx,
                           F dw, F db, V work, int64_t bytes) { return op_apart_grouped_bwd(c, x, n, ldx, ptr, rows, w, dy, lddy, dx, lddx, dw, db, work, bytes); }
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "checks.cpp"), os.path.join(d, "checks.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC,
                        "-I", os.path.join(ROOT, "include"), src, "-o", lib], check=True)
        L = C.CDLL(lib)
    vp, i64, i32, cfg = C.c_void_p, C.c_int64, C.c_int32, C.POINTER(B._GroupedConfig)
    for f in (L.group_rows, L.fwd, L.bwd):
        f.restype = C.c_char_p
    L.meet.argtypes = [vp, i64, i64, i64] * 2
    L.group_rows.argtypes = [vp, i64, i32, vp, vp]
    L.fwd.argtypes = [cfg, vp, i64, i64, vp, vp, vp, vp, vp, i64]
    L.bwd.argtypes = [cfg, vp, i64, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, i64]
    return L


def _bytes(at, rows, width, stride):
    return {at + r * stride + c for r in range(rows) for c in range(width)}


def test_areas_meet_where_they_share_a_byte():
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(30_000):
        def area():
            width = rng.randint(1, 9)
            return rng.randint(1, 60), rng.choice([0, 1, 1, 2, 3, 7]), width, width + rng.choice([0, 0, 1, 5, 12])
        a, b = area(), area()
        if rng.random() < 0.5:
            b = b[:2] + (min(b[2], a[3]), a[3])             # the same stride: columns of one buffer
        want = bool(_bytes(*a) & _bytes(*b))
        assert bool(_lib().meet(*a, *b)) == want and bool(_lib().meet(*b, *a)) == want, (a, b)
        seen[want] += 1
    assert min(seen.values()) > 5000


def test_areas_of_any_size():
    m, top = _lib().meet, 2 ** 31 - 1
    half = 2 ** 40
    assert not m(half, top, 2048, 4096, half + 2048, top, 2048, 4096)                   # halves of rows, terabytes
    assert m(half, top, 2049, 4096, half + 2048, top, 2048, 4096)
    assert m(half, top, 2048, 4096, half + 2048 + 4096 * (top - 2), 1, 2049, 2049)      # reaches into the last row
    assert not m(half, top, 2048, 4096, half + 2048 + 4096 * (top - 2), 1, 2048, 2048)
    assert not m(half, top, 2048, 4096, half + 2048, top, 1024, 8192)                   # every second row's other half
    assert not m(None, 5, 4, 4, None, 5, 4, 4) and not m(half, 0, 4, 4, half, 1, 4, 4)
    assert not m(half, top, 4, 2 ** 33, half + 8, top, 4, 2 ** 33 - 4)                  # (there is no such memory)
    assert not m(2 ** 64 - 64, 4, 4, 8, 2 ** 64 - 64, 4, 4, 8) and not m(2 ** 63, 1, 4, 4, half, 3, 4, 4)


GROUPS, N_IN, N_OUT, ROWS = 4, 8, 6, 10
SIZES = dict(x=ROWS * N_IN * 4, y=ROWS * N_OUT * 4, dy=ROWS * N_OUT * 4, dx=ROWS * N_IN * 4, w=GROUPS * N_IN * N_OUT * 4, dw=GROUPS * N_IN * N_OUT * 4,
             b=GROUPS * N_OUT * 4, db=GROUPS * N_OUT * 4, ptr=(GROUPS + 1) * 4, rows=ROWS * 4, group=ROWS * 4, work=256)
CFG = B._GroupedConfig(0, GROUPS, N_IN, N_OUT)


def _rows(group, ptr, rows):
    return _lib().group_rows(group, ROWS, GROUPS, ptr, rows)


def _fwd(x, ptr, rows, w, b, y):
    return _lib().fwd(C.byref(CFG), x, ROWS, N_IN, ptr, rows, w, b, y, N_OUT)


def _bwd(x, ptr, rows, w, dy, dx, dw, db, work):
    return _lib().bwd(C.byref(CFG), x, ROWS, N_IN, ptr, rows, w, dy, N_OUT, dx, N_IN, dw, db, work, SIZES["work"])


CALLS = {_rows: ("group", ("ptr", "rows")), _fwd: ("x ptr rows w b", ("y",)), _bwd: ("x ptr rows w dy", ("dx", "dw", "db", "work"))}


@pytest.mark.parametrize("call", CALLS)
def test_every_output_is_apart_from_everything(call):
    reads, writes = CALLS[call]
    names = [*reads.split(), *writes]
    at, where = 0x10000, {}
    for n in names:             # side by side, without a gap
        where[n] = at
        at += SIZES[n]
    apart = {n: where[n] if n in writes else where[n] - 0x4000 for n in names}
    assert call(**where) is None
    for out in writes:
        for other in names:
            if other == out:
                continue
            lo, hi = where[other], where[other] + SIZES[other]
            for place in (lo, hi - 4, lo - SIZES[out] + 4):         # the same start, its last four bytes, its first
                got = call(**{**where, out: place})
                assert got is not None and b"overlaps" in got, (out, other)
    for a in reads.split():     # what is only read may lie anywhere
        for b in reads.split():
            assert call(**{**apart, a: apart[b]}) is None


def test_what_a_call_is_not_given_overlaps_nothing():
    at = 0x10000
    apart = dict(x=at, ptr=at + 0x1000, rows=at + 0x2000, w=at + 0x3000, dy=at + 0x4000)
    assert _bwd(**apart, dx=at + 0x5000, dw=None, db=None, work=at) is None         # (the working memory is the weight gradients')
    assert _bwd(**apart, dx=None, dw=at + 0x5000, db=None, work=at + 0x6000) is None
    assert _fwd(apart["x"], apart["ptr"], None, apart["w"], None, apart["dy"]) is None
    assert _lib().fwd(C.byref(CFG), at, 0, N_IN, at, at, at, at, at, N_OUT) is None      # no rows
    assert _lib().group_rows(None, 0, GROUPS, at, None) is None
    wide = N_IN + N_OUT         # x and y as columns of one buffer, then a column too far to the left
    assert _lib().fwd(C.byref(CFG), at, ROWS, wide, apart["ptr"], None, apart["w"], None, at + 4 * N_IN, wide) is None
    assert _lib().fwd(C.byref(CFG), at, ROWS, wide, apart["ptr"], None, apart["w"], None, at + 4 * N_IN - 4, wide) is not None
