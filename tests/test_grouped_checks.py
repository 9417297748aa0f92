"""What the operators on weights in stacks refuse (csrc/op_checks.h, compiled for the host), and the rules by which rows and products
are dealt to workgroups (csrc/group_rules.h): every bad argument, and that runs, tiles and slabs cover what they are for."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

import pytest

from conftest import ROOT
from paper_2303_13775_amd import binding as B

CSRC = os.path.join(ROOT, "paper_2303_13775_amd", "csrc")
_SOURCE = r"""
#include "op_checks.h"
#include "group_rules.h"
typedef const void *V;
typedef const float *F;
typedef const int32_t *I;
extern "C" const char *group_rows(I g, int64_t n, int32_t G, I ptr, I rows) { return op_check_group_rows(g, n, G, ptr, rows); }
extern "C" const char *fwd(const gsplit_grouped_config *c, V x, int64_t n, int64_t ldx, I ptr, I rows, V w, F b, V y, int64_t ldy) {
    return op_check_grouped_fwd(c, x, n, ldx, ptr, rows, w, b, y, ldy);
}
extern "C" const char *bwd(const gsplit_grouped_config *c, V x, int64_t n, int64_t ldx, I ptr, I rows, V w, V dy, int64_t lddy, V dx, int64_t lddx,
                           F dw, F db, V work) { return op_check_grouped_bwd(c, x, n, ldx, ptr, rows, w, dy, lddy, dx, lddx, dw, db, work); }
extern "C" void runs(int64_t n, int32_t G, int64_t counters, int n_cu, int64_t *out) {
    const GroupRuns r = group_runs(n, G, counters, n_cu);
    out[0] = r.workgroups; out[1] = r.rows_a_wave;
}
extern "C" int64_t chunk(int64_t n, int64_t tiles, int n_cu) { return group_chunk(n, tiles, n_cu); }
extern "C" int64_t slabs(int64_t n, int64_t chunk) { return group_slabs(n, chunk); }
extern "C" int rows_form(int64_t n, int32_t G, int64_t k, int64_t w, int is_float, int transposed, int granules) {
    return group_rows_form(n, G, k, w, is_float, transposed, granules, 256);
}
extern "C" void weights_form(int64_t n, int32_t G, int64_t k, int64_t w, int is_float, int granules, int64_t *out) {
    const GroupWeights f = group_weights_form(n, G, k, w, is_float, granules, 256);
    out[0] = f.form; out[1] = f.tile; out[2] = f.chunk; out[3] = f.slabs; out[4] = group_most_slabs(n, G, k, w, is_float, 256);
}
extern "C" int64_t row_tiles(int64_t n, int32_t G, int32_t rows) { return group_row_tiles(n, G, rows); }
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "checks.cpp"), os.path.join(d, "checks.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-I", os.path.join(ROOT, "include"),
                        src, "-o", lib], check=True)
        L = C.CDLL(lib)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    for f in (L.group_rows, L.fwd, L.bwd):
        f.restype = C.c_char_p
    cfg = C.POINTER(B._GroupedConfig)
    L.group_rows.argtypes = [vp, i64, i32, vp, vp]
    L.fwd.argtypes = [cfg, vp, i64, i64, vp, vp, vp, vp, vp, i64]
    L.bwd.argtypes = [cfg, vp, i64, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp]
    L.runs.argtypes = [i64, i32, i64, C.c_int, C.POINTER(i64)]
    L.rows_form.argtypes = [i64, i32, i64, i64, C.c_int, C.c_int, C.c_int]
    L.weights_form.argtypes = [i64, i32, i64, i64, C.c_int, C.c_int, C.POINTER(i64)]
    for f, a in ((L.chunk, [i64, i64, C.c_int]), (L.slabs, [i64, i64]), (L.row_tiles, [i64, i32, i32])):
        f.argtypes, f.restype = a, i64
    return L


P = 0x1000          # any aligned address: the checks read none


def _rows(g=P, n=10, G=4, ptr=P, rows=P):
    return _lib().group_rows(g, n, G, ptr, rows)


def _fwd(cfg=(0, 4, 8, 6), x=P, n=10, ldx=8, ptr=P, rows=P, w=P, b=P, y=P, ldy=6):
    return _lib().fwd(None if cfg is None else C.byref(B._GroupedConfig(*cfg)), x, n, ldx, ptr, rows, w, b, y, ldy)


def _bwd(cfg=(0, 4, 8, 6), x=P, n=10, ldx=8, ptr=P, rows=P, w=P, dy=P, lddy=6, dx=P, lddx=8, dw=P, db=P, work=P):
    return _lib().bwd(None if cfg is None else C.byref(B._GroupedConfig(*cfg)), x, n, ldx, ptr, rows, w, dy, lddy, dx, lddx, dw, db, work)


@pytest.mark.parametrize("f, change", [
    (_rows, dict()), (_rows, dict(n=0, g=None, rows=None)), (_rows, dict(G=512)), (_rows, dict(n=2 ** 31 - 1)),
    (_fwd, dict()), (_fwd, dict(rows=None, b=None)), (_fwd, dict(n=0, x=None, y=None, ptr=None, w=None)), (_fwd, dict(ldx=9, ldy=1000)),
    (_fwd, dict(cfg=(1, 1, 1, 1), x=P + 2, y=P + 6, w=P + 2)), (_bwd, dict()), (_bwd, dict(dx=None, lddx=0, w=None)), (_bwd, dict(dw=None, db=None, work=None)),
    (_bwd, dict(db=None)), (_bwd, dict(n=0, x=None, dy=None, dx=None)), (_bwd, dict(dw=None, db=None, x=None))])
def test_accepts(f, change):
    assert f(**change) is None


@pytest.mark.parametrize("f, change, message", [
    (_rows, dict(n=-1), "n_rows"), (_rows, dict(n=2 ** 31), "n_rows"), (_rows, dict(G=0), "n_groups"), (_rows, dict(G=513), "n_groups"),
    (_rows, dict(g=None), "NULL"), (_rows, dict(ptr=None, n=0), "NULL"), (_rows, dict(rows=None), "NULL"), (_rows, dict(g=P + 2), "misaligned"),
    (_rows, dict(ptr=P + 1), "misaligned"), (_rows, dict(rows=P + 2), "misaligned"),
    (_fwd, dict(cfg=None), "config"), (_fwd, dict(cfg=(2, 4, 8, 6)), "dtype"), (_fwd, dict(cfg=(0, 0, 8, 6)), "n_groups"), (_fwd, dict(cfg=(0, 513, 8, 6)), "n_groups"),
    (_fwd, dict(cfg=(0, 4, 0, 6)), "width"), (_fwd, dict(cfg=(0, 4, 8, 2 ** 20 + 1)), "width"), (_fwd, dict(n=-1), "n_rows"), (_fwd, dict(n=2 ** 31), "n_rows"),
    (_fwd, dict(x=None), "NULL"), (_fwd, dict(y=None), "NULL"), (_fwd, dict(w=None), "NULL"), (_fwd, dict(ptr=None), "NULL"), (_fwd, dict(ldx=7), "stride"),
    (_fwd, dict(ldy=5), "stride"), (_fwd, dict(ldy=2 ** 41), "stride"), (_fwd, dict(x=P + 2), "misaligned"), (_fwd, dict(w=P + 1), "misaligned"),
    (_fwd, dict(b=P + 2), "misaligned"), (_fwd, dict(y=P + 1), "misaligned"), (_fwd, dict(rows=P + 2), "misaligned"), (_fwd, dict(cfg=(1, 4, 8, 6), x=P + 1), "misaligned"),
    (_bwd, dict(cfg=None), "config"), (_bwd, dict(dx=None, dw=None, db=None), "nothing"), (_bwd, dict(dw=None), "d_dbias needs"), (_bwd, dict(x=None), "NULL"),
    (_bwd, dict(dy=None), "NULL"), (_bwd, dict(w=None), "NULL"), (_bwd, dict(ptr=None, n=0), "NULL"), (_bwd, dict(lddx=7), "stride"), (_bwd, dict(lddy=5), "stride"),
    (_bwd, dict(work=P + 8), "misaligned"), (_bwd, dict(dw=P + 2), "misaligned"), (_bwd, dict(db=P + 2), "misaligned"), (_bwd, dict(dx=P + 2), "misaligned")])
def test_refuses(f, change, message):
    got = f(**change)
    assert got is not None and message in got.decode()


def test_null_context():
    lib = B.load_library()
    assert lib.gsplit_group_rows(None, None, 0, 1, None, None, None) == -1
    assert lib.gsplit_grouped_linear_fwd(None, None, None, 0, 0, None, None, None, None, None, 0, None) == -1
    assert lib.gsplit_grouped_linear_work(None, None, 0) == -1
    assert lib.gsplit_grouped_linear_bwd(None, None, None, 0, 0, None, None, None, None, 0, None, 0, None, None, None, None) == -1


def test_runs_cover_the_rows_and_fit_the_counters():
    out = (C.c_int64 * 2)()
    for counters in (40960, 512):
        for G in (1, 7, 64, 511, 512):
            for n in (0, 1, 63, 64, 65, 1024, 4096, 4097, 70_001, 10 ** 6, 2 ** 31 - 1):
                _lib().runs(n, G, counters, 256, out)
                wgs, wave = out
                assert wave >= 64 and wave % 64 == 0 and wgs * 16 * wave >= n and (wgs - 1) * 16 * wave < max(n, 1)
                assert wgs == 1 or wgs * G <= counters


def test_chunks_and_slabs_cover_any_groups():
    import random
    rng = random.Random(1)
    for _ in range(2000):
        n, tiles, G = rng.choice([0, 1, 255, 256, 257, 5000, 100_000]), rng.choice([1, 3, 17, 200, 255, 256, 4000]), rng.choice([1, 2, 30, 512])
        chunk = _lib().chunk(n, tiles, 256)
        assert chunk >= 1 and (chunk % 64 == 0 or chunk == max(n, 1))
        cuts = sorted(rng.randint(0, n) for _ in range(G - 1))
        sizes = [b - a for a, b in zip([0] + cuts, cuts + [n])]
        chunks = [-(-s // chunk) for s in sizes]
        assert sum(c for c in chunks if c > 1) <= _lib().slabs(n, chunk)
        assert sum(max(c, 1) for c in chunks) <= n // chunk + G
        assert sum(c > 1 for c in chunks) <= n // chunk
        for rows in (64, 128):
            assert sum(-(-s // rows) for s in sizes) <= _lib().row_tiles(n, G, rows)


CORE, FEW, T128, T64 = range(4)


def _forms(rows, groups, n_in, n_out, is_float, granules):
    out = (C.c_int64 * 5)()
    _lib().weights_form(rows, groups, n_in, n_out, is_float, granules, out)
    f = _lib().rows_form
    return f(rows, groups, n_in, n_out, is_float, 0, granules), f(rows, groups, n_out, n_in, is_float, 1, granules), list(out)


def test_gpu_tests_reach_every_form():
    import test_gpu_grouped as T
    small = [(*shape, kw) for shape in T.SHAPES for kw in (dict(), dict(pad=1, offset=1), dict(pad=8))]
    reached = {True: [set(), set(), set()], False: [set(), set(), set()]}
    for cases, types in ((small + T.LARGE, (True, False)), (T.LARGE_TILES, (False,))):
        for rows, groups, n_in, n_out, kw in cases:
            for is_float in types:
                granules = not is_float and all(x % 8 == 0 for x in (n_in, n_out, kw.get("pad", 0), kw.get("offset", 0)))
                y, dx, w = _forms(rows, groups, n_in, n_out, is_float, granules)
                reached[is_float][0].add(y)
                reached[is_float][1].add(dx)
                reached[is_float][2].add((w[0], w[3] > 0))
    assert reached[True][:2] == [{FEW, T128, T64}] * 2 and reached[False][:2] == [{CORE, FEW, T128, T64}] * 2
    assert reached[True][2] >= {(FEW, False), (T64, False), (T64, True), (T128, True)}
    assert reached[False][2] >= {(FEW, False), (T64, False), (T64, True), (T128, True), (CORE, True)}


def test_working_memory_serves_every_form():
    import random
    rng = random.Random(4)
    for _ in range(3000):
        n, G = rng.choice([0, 1, 300, 4096, 4097, 20_000, 10 ** 6]), rng.choice([1, 3, 64, 512])
        k, w = (rng.choice([1, 8, 47, 64, 65, 128, 256, 1000, 2048, 5000]) for _ in range(2))
        for is_float in (True, False):
            for granules in (True, False):
                if granules and (k % 8 or w % 8 or is_float):
                    continue
                form, tile, chunk, slabs, most = _forms(n, G, k, w, is_float, granules)[2]
                assert slabs <= most and chunk >= 1 and tile == {CORE: 256, FEW: 32, T128: 128, T64: 64}[form]


def test_rows_shorter_than_a_fetch_take_the_form_that_reads_single_elements():
    """The tiles through registers fetch eight elements of a row at once: none of them may get a shorter one."""
    few = 1             # GROUP_FEW
    for k in range(1, 8):
        for n_rows in (1, 300, 70_000, 1 << 30):
            for groups in (1, 16, 512):
                for n in (1, 64, 200, 5000):
                    for is_float in (0, 1):
                        for transposed in (0, 1):
                            assert _lib().rows_form(n_rows, groups, k, n, is_float, transposed, 0) == few
