"""What the losses over rows and the update refuse (csrc/op_checks.h, compiled for the host): every kind of bad argument, and
that the calls themselves answer a NULL context."""
import ctypes as C
import functools
import math
import os
import subprocess
import tempfile

import pytest

from conftest import ROOT
from paper_2303_13775_amd import binding as B

CSRC = os.path.join(ROOT, "paper_2303_13775_amd", "csrc")
_SOURCE = r"""
#include <initializer_list>
#include "op_checks.h"
typedef const void *V;
typedef const float *F;
typedef const int64_t *I;
extern "C" const char *policy(const gsplit_policy_config *c, V z, int64_t n, int32_t C, int64_t ld, I a, F old, F ref, F adv, F w, V g,
                              int64_t gld, F loss, F logp, F kl) { return op_check_policy(c, z, n, C, ld, a, old, ref, adv, w, g, gld, loss, logp, kl); }
extern "C" const char *preference(const gsplit_preference_config *c, V z, int64_t n, int32_t C, int64_t ld, I a, I ptr, int64_t pairs, F ref,
                                  F w, V g, int64_t gld, F logp, F loss, F margin, F work) { return op_check_preference(c, z, n, C, ld, a, ptr, pairs, ref, w, g, gld, logp, loss, margin, work); }
extern "C" const char *grads(const gsplit_grad_tensor *t, int64_t n, double max_norm, int clip) { return op_check_grads(t, n, max_norm, clip != 0); }
extern "C" const char *adamw(const gsplit_adamw_config *c, const gsplit_adamw_tensor *t, int64_t n) { return op_check_adamw(c, t, n); }
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
    for f in (L.policy, L.preference, L.grads, L.adamw):
        f.restype = C.c_char_p
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    L.policy.argtypes = [C.POINTER(B._PolicyConfig), vp, i64, i32, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp]
    L.preference.argtypes = [C.POINTER(B._PreferenceConfig), vp, i64, i32, i64, vp, vp, i64, vp, vp, vp, i64, vp, vp, vp, vp]
    L.grads.argtypes = [C.POINTER(B._GradTensor), i64, C.c_double, C.c_int]
    L.adamw.argtypes = [C.POINTER(B._AdamwConfig), C.POINTER(B._AdamwTensor), i64]
    return L


P = 0x1000          # any aligned address: the checks read none
NAN, INF = math.nan, math.inf


def _policy(cfg=(0, 0.2, 0.2, 0.1), z=P, n=4, classes=8, ld=8, a=P, old=P, ref=P, adv=P, w=P, g=P + 64, gld=8, loss=P, logp=P, kl=P):
    return _lib().policy(B._PolicyConfig(*cfg), z, n, classes, ld, a, old, ref, adv, w, g, gld, loss, logp, kl)


@pytest.mark.parametrize("change", [
    dict(n=0, z=None, a=None, old=None, adv=None), dict(g=None, gld=0), dict(cfg=(0, 0.2, 0.2, 0.0), ref=None), dict(w=None, loss=None),
    dict(g=P), dict(cfg=(1, 0.0, 0.0, 0.0), z=P + 2, g=P + 6), dict(ld=9, gld=11), dict(cfg=(0, 1.0, 5.0, 0.0)), dict(logp=None, kl=None)])
def test_policy_takes(change):
    assert _policy(**change) is None


@pytest.mark.parametrize("change", [
    dict(cfg=(2, 0.2, 0.2, 0.1)), dict(cfg=(-1, 0.2, 0.2, 0.1)), dict(n=-1), dict(classes=0), dict(classes=(1 << 30) + 1, ld=1 << 31, gld=1 << 31), dict(ld=7), dict(gld=7), dict(z=None), dict(a=None),
    dict(old=None), dict(adv=None), dict(ref=None), dict(z=P + 2), dict(a=P + 4), dict(g=P + 2), dict(cfg=(1, 0.2, 0.2, 0.1), z=P + 1),
    dict(old=P + 2), dict(kl=P + 1), dict(g=P, gld=9), dict(n=1 << 41), dict(ld=1 << 41)]
    + [dict(cfg=(0, x, 0.2, 0.1)) for x in (-0.1, 1.1, NAN, INF)] + [dict(cfg=(0, 0.2, x, 0.1)) for x in (-0.1, NAN, INF)]
    + [dict(cfg=(0, 0.2, 0.2, x)) for x in (-0.1, NAN, INF)])
def test_policy_refuses(change):
    assert _policy(**change)


def _preference(cfg=(0, 0.1, 0.0), z=P, n=4, classes=8, ld=8, a=P, ptr=P, pairs=2, ref=P, w=P, g=P + 64, gld=8, logp=P, loss=P, margin=P, work=P):
    return _lib().preference(B._PreferenceConfig(*cfg), z, n, classes, ld, a, ptr, pairs, ref, w, g, gld, logp, loss, margin, work)


@pytest.mark.parametrize("change", [
    dict(), dict(pairs=0, ptr=None, work=None), dict(n=0, z=None, a=None, work=None), dict(g=None), dict(ref=None, w=None),
    dict(logp=None, loss=None, margin=None), dict(cfg=(1, -1.0, 1.0))])
def test_preference_takes(change):
    assert _preference(**change) is None


@pytest.mark.parametrize("change", [
    dict(pairs=-1), dict(ptr=None), dict(work=None), dict(work=P + 8), dict(ptr=P + 4), dict(ref=P + 2), dict(z=None), dict(ld=7),
    dict(cfg=(3, 0.1, 0.0)), dict(pairs=1 << 41)]
    + [dict(cfg=(0, x, 0.0)) for x in (NAN, INF)] + [dict(cfg=(0, 0.1, x)) for x in (-0.1, 1.5, NAN)])
def test_preference_refuses(change):
    assert _preference(**change)


def _grads(ts, max_norm=1.0, clip=1):
    return _lib().grads((B._GradTensor * max(1, len(ts)))(*[B._GradTensor(*t) for t in ts]), len(ts), max_norm, clip)


def test_gradient_tensors():
    for ts in ([], [(P, None, 5, 0)], [(P, P, 5, 1)], [(None, None, 0, 0)], [(P + 2, P + 4, 5, 1), (P + 4, None, 3, 0)]):
        assert _grads(ts) is None, ts
    assert _grads([(P, None, 1, 0)], INF) is None and _grads([(P, None, 1, 0)], NAN, 0) is None
    for ts in ([(None, P, 5, 0)], [(P, P, -1, 0)], [(P, P, 1, 2)], [(P + 2, P, 1, 0)], [(P, P + 2, 1, 0)], [(P, P, 1 << 47, 0)],
               [(P, P, 1, 0), (P + 1, P, 1, 1)]):
        assert _grads(ts), ts
    for x in (0.0, -1.0, NAN):
        assert _grads([(P, P, 1, 0)], x)
    assert _lib().grads(None, 1, 1.0, 1) and _lib().grads(None, -1, 1.0, 1) and _lib().grads(None, 0, 1.0, 1) is None


def _adamw(t=(P, None, P, P, P, 4, 0, 0), lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, max_norm=0.0, step=1, d_step=None, d_lr=None):
    cfg = B._AdamwConfig(lr, b1, b2, eps, wd, max_norm, step, d_step, d_lr)
    return _lib().adamw(cfg, (B._AdamwTensor * 1)(B._AdamwTensor(*t)), 1)


@pytest.mark.parametrize("change", [
    dict(), dict(t=(P + 2, P, P + 2, P, P, 4, 1, 1)), dict(t=(None, None, None, None, None, 0, 0, 0)), dict(step=0, d_step=P),
    dict(lr=NAN, d_lr=P), dict(b1=0.0, b2=0.0, eps=0.0), dict(max_norm=INF), dict(t=(P, None, P + 2, P, P, 4, 0, 1))])
def test_adamw_takes(change):
    assert _adamw(**change) is None


@pytest.mark.parametrize("change", [
    dict(t=(P, P, P, P, P, 4, 0, 0)), dict(t=(P, None, P, P, P, 4, 1, 0)), dict(t=(None, None, P, P, P, 4, 0, 0)),
    dict(t=(P, None, None, P, P, 4, 0, 0)), dict(t=(P, None, P, None, P, 4, 0, 0)), dict(t=(P, None, P, P, None, 4, 0, 0)),
    dict(t=(P, None, P, P, P, -4, 0, 0)), dict(t=(P, None, P, P, P, 4, 5, 0)), dict(t=(P, None, P, P, P, 4, 0, 5)),
    dict(t=(P + 2, None, P, P, P, 4, 0, 0)), dict(t=(P, None, P, P + 2, P, 4, 0, 0)), dict(t=(P, P + 2, P, P, P, 4, 1, 0)),
    dict(step=0), dict(d_step=P + 4), dict(d_lr=P + 2), dict(b1=1.0), dict(b2=1.0), dict(b1=-0.1), dict(b2=NAN), dict(lr=-1.0), dict(lr=NAN),
    dict(eps=-1.0), dict(eps=INF), dict(wd=-1.0), dict(wd=NAN), dict(max_norm=-1.0), dict(max_norm=NAN)])
def test_adamw_refuses(change):
    assert _adamw(**change)


def test_calls_refuse_a_null_context():
    lib = B.load_library()
    assert lib.gsplit_policy_loss(None, None, None, 0, 1, 1, None, None, None, None, None, None, 1, None, None, None, None) == -1
    assert lib.gsplit_preference_loss(None, None, None, 0, 1, 1, None, None, 0, None, None, None, 1, None, None, None, None, None) == -1
    assert lib.gsplit_grad_norm(None, None, 0, None, None) == -1
    assert lib.gsplit_clip_grads(None, None, 0, 1.0, None, None) == -1
    assert lib.gsplit_adamw_step(None, None, None, 0, None, None) == -1
