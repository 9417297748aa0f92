"""What orthogonalisation and the update by orthogonalised momentum refuse (csrc/op_checks.h, compiled for the host), and how matrices are
dealt to launches (csrc/newton_rules.h): every bad argument; every matrix in one launch, within its limits."""
import ctypes as C
import functools
import math
import os
import random
import subprocess
import tempfile

import numpy as np
import pytest

from conftest import ROOT
from paper_2303_13775_amd import binding as B

CSRC = os.path.join(ROOT, "paper_2303_13775_amd", "csrc")
_SOURCE = r"""
#include <vector>
#include "op_checks.h"
#include "newton_rules.h"
extern "C" const char *newton(const gsplit_newton_config *c) { return op_check_newton(c); }
extern "C" const char *matrices(const gsplit_matrix_tensor *t, int64_t n) { return op_check_matrices(t, n); }
extern "C" const char *muon(const gsplit_muon_config *c) { return op_check_muon(c); }
extern "C" const char *muon_tensors(const gsplit_muon_tensor *t, int64_t n) { return op_check_muon_tensors(t, n); }
extern "C" const char *work(const void *p, int64_t bytes) { return op_check_work(p, bytes); }
// rows of: launch, tile, tensor, first, count, mp, np, words
extern "C" int64_t groups(const gsplit_matrix_tensor *t, int64_t n, int64_t *out, int64_t room) {
    int64_t at = 0, launch = 0;
    newton_groups(n, [&](int64_t i) { struct { int64_t count; int32_t rows, cols; } s{t[i].count, t[i].rows, t[i].cols}; return s; },
                  [&](const NewtonStack *in, int k, int tile) {
        for (int j = 0; j < k; ++j, ++at)
            if (at < room) {
                const int64_t row[8] = {launch, tile, in[j].tensor, in[j].first, in[j].size.count, in[j].size.mp, in[j].size.np, newton_words(in[j].size, tile)};
                for (int x = 0; x < 8; ++x) out[8 * at + x] = row[x];
            }
        ++launch;
    });
    return at;
}
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
    for f in (L.newton, L.matrices, L.muon, L.muon_tensors, L.work):
        f.restype = C.c_char_p
    L.newton.argtypes = [C.POINTER(B._NewtonConfig)]
    L.matrices.argtypes = [C.POINTER(B._MatrixTensor), C.c_int64]
    L.muon.argtypes = [C.POINTER(B._MuonConfig)]
    L.muon_tensors.argtypes = [C.POINTER(B._MuonTensor), C.c_int64]
    L.work.argtypes = [C.c_void_p, C.c_int64]
    L.groups.argtypes, L.groups.restype = [C.POINTER(B._MatrixTensor), C.c_int64, C.POINTER(C.c_int64), C.c_int64], C.c_int64
    return L


P = 0x1000          # any aligned address: the checks read none
NAN, INF = math.nan, math.inf
ABC = B.NEWTON_COEFFICIENTS


def _newton(abc=ABC, eps=1e-7, steps=5):
    return _lib().newton(C.byref(B._NewtonConfig(*abc, eps, steps)))


def _matrix(d_in=P, d_out=P + 64, count=2, rows=3, cols=4, in_dtype=0, out_dtype=0):
    return _lib().matrices(C.byref(B._MatrixTensor(d_in, d_out, count, rows, cols, in_dtype, out_dtype)), 1)


def _muon(newton=(*ABC, 1e-7, 5), lr=0.1, momentum=0.9, wd=0.0, d_lr=None, nesterov=1, scaling=1):
    return _lib().muon(C.byref(B._MuonConfig(B._NewtonConfig(*newton), lr, momentum, wd, d_lr, nesterov, scaling)))


def _tensor(p=P, w=None, g=P, m=P, count=2, rows=3, cols=4, pt=0, gt=0):
    return _lib().muon_tensors(C.byref(B._MuonTensor(p, w, g, m, count, rows, cols, pt, gt)), 1)


@pytest.mark.parametrize("f, change", [
    (_newton, dict()), (_newton, dict(steps=64)), (_newton, dict(eps=0.0)), (_newton, dict(abc=(1.875, -1.25, 0.375), steps=30)), (_newton, dict(abc=(1.5, -0.5, 0.0), steps=30)),
    (_newton, dict(abc=(1.0, 0.0, 0.0))), (_newton, dict(abc=(0.0, 0.0, 0.0))), (_matrix, dict()), (_matrix, dict(d_out=P)), (_matrix, dict(in_dtype=1, d_in=P + 2)),
    (_matrix, dict(count=0, d_in=None, d_out=None)), (_matrix, dict(rows=0, d_in=None, d_out=None)), (_matrix, dict(rows=65536, cols=65536)),
    (_muon, dict()), (_muon, dict(lr=NAN, d_lr=P)), (_muon, dict(momentum=0.0, scaling=2)), (_tensor, dict()), (_tensor, dict(pt=1, w=P)), (_tensor, dict(gt=1, g=P + 2)),
    (_tensor, dict(p=None, g=None, m=None, count=0))])
def test_accepts(f, change):
    assert f(**change) is None


@pytest.mark.parametrize("f, change, message", [
    (_newton, dict(steps=0), "steps"), (_newton, dict(steps=65), "steps"), (_newton, dict(eps=-1.0), "eps"), (_newton, dict(eps=INF), "eps"), (_newton, dict(eps=NAN), "eps"),
    (_newton, dict(abc=(2.0, 0.0, 0.0)), "bounds"), (_newton, dict(abc=(1.2, 0.0, 0.0), steps=5), "bounds"), (_newton, dict(abc=(NAN, 0.0, 0.0)), "bounds"), (_newton, dict(abc=(INF, 0.0, 0.0)), "bounds"),
    (_newton, dict(abc=(16.0, -16.0, 1.0)), "bounds"), (_newton, dict(abc=(5.0, -5.0, 1.0)), "bounds"),
    (_matrix, dict(rows=-1), "rows"), (_matrix, dict(cols=65537), "cols"), (_matrix, dict(count=-1), "number"), (_matrix, dict(count=2 ** 31, rows=65536), "number"),
    (_matrix, dict(d_in=None), "NULL"), (_matrix, dict(d_out=None), "NULL"), (_matrix, dict(d_in=P + 2), "misaligned"), (_matrix, dict(d_out=P + 1, out_dtype=1), "misaligned"),
    (_matrix, dict(in_dtype=2), "dtype"), (_matrix, dict(out_dtype=-1), "dtype"), (_matrix, dict(d_out=P, out_dtype=1), "in place"),
    (_muon, dict(newton=(*ABC, 1e-7, 0)), "steps"), (_muon, dict(momentum=1.0), "momentum"), (_muon, dict(momentum=-0.1), "momentum"), (_muon, dict(momentum=NAN), "momentum"),
    (_muon, dict(lr=-1.0), "lr"), (_muon, dict(lr=NAN), "lr"), (_muon, dict(wd=-1.0), "weight_decay"), (_muon, dict(scaling=3), "scaling"), (_muon, dict(scaling=-1), "scaling"), (_muon, dict(d_lr=P + 2), "misaligned"),
    (_tensor, dict(w=P), "no d_master"), (_tensor, dict(pt=1), "NULL"), (_tensor, dict(p=None), "NULL"), (_tensor, dict(g=None), "NULL"), (_tensor, dict(m=None), "NULL"),
    (_tensor, dict(m=P + 2), "misaligned"), (_tensor, dict(pt=2), "dtype"), (_tensor, dict(rows=65537), "rows")])
def test_refuses(f, change, message):
    got = f(**change)
    assert got is not None and message in got.decode()


def test_lists_work_and_contexts():
    lib = B.load_library()
    assert _lib().matrices(None, 0) is None and b"list" in _lib().matrices(None, 1) and b"list" in _lib().muon_tensors(None, -1)
    assert b"config" in _lib().newton(None) and b"config" in _lib().muon(None)
    assert _lib().work(None, 0) is None and b"NULL" in _lib().work(None, 16) and b"misaligned" in _lib().work(P + 8, 16)
    assert lib.gsplit_orthogonalize(None, None, None, 0, None, None) == -1 and lib.gsplit_muon_step(None, None, None, 0, None, None) == -1
    assert lib.gsplit_orthogonalize_work(None, 0) == 0 and lib.gsplit_orthogonalize_work(None, 1) == -1 and lib.gsplit_muon_work(None, -1) == -1


def test_coefficients_are_held_to_what_halves_carry():
    """The bounds the check goes by are those of the polynomial on a fine grid."""
    rng = random.Random(2)
    seen = {True: 0, False: 0}
    for _ in range(400):
        a, b, c = rng.uniform(-1, 5), rng.uniform(-8, 3), rng.uniform(-3, 5) if rng.random() < 0.8 else 0.0
        steps, top, ok, near = rng.randint(1, 6), 1.0, True, False
        for _ in range(steps):
            s = np.linspace(0.0, top, 20001)
            nxt, most = np.abs(s * (a + b * s ** 2 + c * s ** 4)).max(), np.abs(a + b * s ** 2 + c * s ** 4).max()
            near |= abs(nxt - 1.99) < 1e-3 or abs(most - 15.0) < 1e-3
            ok, top = ok and nxt <= 1.99 and most <= 15.0, min(nxt, 10.0)
        if not near:
            assert (_newton(abc=(a, b, c), steps=steps) is None) == ok, (a, b, c, steps)
            seen[ok] += 1
    assert min(seen.values()) > 20


def test_every_matrix_is_in_one_launch():
    rng = random.Random(3)
    out = (C.c_int64 * (8 * 4096))()
    tiles = set()
    for k in range(200):
        big = rng.random() < 0.4
        shapes = [(rng.choice([0, 1, 2, 7, 40]), rng.choice([0, 1, 5, 64, 65, 300, 1000 if big else 90]), rng.choice([0, 1, 9, 128, 700, 4000 if big else 33]))
                  for _ in range(rng.choice([0, 1, 3, 24, 25, 60]))]
        if k % 20 == 0:
            shapes.append((3, 9000, 8000))
        t = (B._MatrixTensor * max(1, len(shapes)))(*[B._MatrixTensor(P, P + 64, c, r, q, 0, 0) for c, r, q in shapes])
        n = _lib().groups(t, len(shapes), out, 4096)
        assert n <= 4096
        rows = np.array(out[:8 * n]).reshape(n, 8)
        covered = {i: [] for i in range(len(shapes))}
        for launch, tile, i, first, count, mp, np_, words in rows.tolist():
            c, r, q = shapes[i]
            tiles.add(tile)
            m, w = min(r, q), max(r, q)
            pad = 64 if tile == 1 else tile
            assert count >= 1 and mp % pad == 0 and np_ % pad == 0 and m <= mp < m + pad and w <= np_ < w + pad
            assert (words == 0 and m <= 64 and w <= 384) if tile == 1 else words >= count * (mp * np_ // 2 + mp * mp // 2 + -(-r * q // max(4096, -(-(r * q // 1024) // 4096) * 4096)) // 2)
            covered[i] += range(first, first + count)
        for i, (c, r, q) in enumerate(shapes):
            assert covered[i] == (list(range(c)) if r and q else [])
        for launch in range(int(rows[-1, 0]) + 1 if n else 0):
            own = rows[rows[:, 0] == launch]
            assert 1 <= len(own) <= 24 and len(set(own[:, 1])) == 1
            assert (own[:, 4] * own[:, 5] * own[:, 6]).sum() <= 1 << 27 or (len(own) == 1 and own[0, 4] == 1)
        assert B.load_library().gsplit_orthogonalize_work(t, len(shapes)) == 16 * max([0] + [int(rows[rows[:, 0] == l, 7].sum()) for l in set(rows[:, 0])])
    assert tiles == {1, 64, 128}


def test_a_matrix_above_a_launch_s_limit_is_one_by_itself():
    """A matrix of more padded elements than a launch takes, in front of, between and behind smaller ones: those keep the limit."""
    rng = random.Random(6)
    out = (C.c_int64 * (8 * 4096))()
    limit = 1 << 27
    for k in range(60):
        shapes = [(rng.choice([1, 5, 48]), rng.choice([100, 4096, 8192]), rng.choice([300, 4096, 8192])) for _ in range(rng.choice([1, 4, 30]))]
        above = rng.choice([(1, 32000, 8192), (1, 16384, 16384), (1, 50304, 4096), (2, 65536, 65536)])
        for at in {0: [0], 1: [len(shapes)]}.get(k % 3, [rng.randint(0, len(shapes)), 0]):
            shapes.insert(at, above)
        t = (B._MatrixTensor * len(shapes))(*[B._MatrixTensor(P, P + 64, c, r, q, 0, 0) for c, r, q in shapes])
        n = _lib().groups(t, len(shapes), out, 4096)
        assert n <= 4096
        rows = np.array(out[:8 * n]).reshape(n, 8)
        taken = {i: [] for i in range(len(shapes))}
        for row in rows.tolist():
            taken[row[2]] += range(row[3], row[3] + row[4])
        assert all(taken[i] == list(range(c)) for i, (c, _, _) in enumerate(shapes))
        words = []
        for launch in range(int(rows[-1, 0]) + 1):
            own = rows[rows[:, 0] == launch]
            assert (own[:, 4] * own[:, 5] * own[:, 6]).sum() <= limit or (len(own) == 1 and own[0, 4] == 1), shapes
            words.append(int(own[:, 7].sum()))
        # no more working memory than the largest launch within the limit (A and B no larger than X; the sums a 256th) or the matrix above it needs
        most = max([limit] + [row[5] * row[6] for row in rows.tolist()])
        work = B.load_library().gsplit_orthogonalize_work(t, len(shapes))
        assert work == 16 * max(words) and work <= 16 * (most + most // 256)


def test_bounds_of_coefficients_with_a_last_one_near_zero():
    """The largest value lies where the derivative is 0, also where the last coefficient all but drops out of its equation."""
    rng = random.Random(7)
    seen = {True: 0, False: 0}
    for _ in range(600):
        a, c = rng.uniform(0, 12), rng.choice([-1, 1]) * 10.0 ** rng.uniform(-320, -6)
        b = -a * rng.uniform(0.5, 2.0)
        s = np.linspace(0.0, 1.0, 20001)
        nxt, most = np.abs(s * (a + b * s ** 2 + c * s ** 4)).max(), np.abs(a + b * s ** 2 + c * s ** 4).max()
        if abs(nxt - 1.99) > 1e-3 and abs(most - 15.0) > 1e-3:
            ok = bool(nxt <= 1.99 and most <= 15.0)
            assert (_newton(abc=(a, b, c), steps=1) is None) == ok, (a, b, c, nxt, most)
            seen[ok] += 1
    assert min(seen.values()) > 50
    for c in (1e-320, 1e-300, 1e-20, 1e-17, 1e-14, 1e-9):
        for sign in (1, -1):
            assert b"bounds" in _newton(abc=(8.0, -8.0, sign * c), steps=5) and _newton(abc=(1.5, -0.5, sign * c), steps=5) is None
