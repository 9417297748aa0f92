"""The rules of the norm and the update (csrc/update_rules.h), compiled for the host, and the tables a launch takes (not a test module
itself)."""
import ctypes as C
import functools
import os
import re
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2303_13775_amd", "csrc")
N_CU = 256

_SOURCE = r"""
#include "update_rules.h"
typedef long long I;
extern "C" int chunk(I total, int most, int n_cu) { return update_chunk(total, most, n_cu); }
extern "C" int chunk_norm(I total, int n_cu) { return norm_chunk(total, n_cu); }
extern "C" int clip_small(I total, I tensors) { return update_clip_small(total, tensors); }
extern "C" int norm_here(I total) { return update_norm_here(total); }
extern "C" int large(I total) { return update_large(total); }
extern "C" int one_slot(I workgroups, int n_cu) { return norm_in_one_slot(workgroups, n_cu); }
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        L = C.CDLL(out)
    i, q = C.c_int, C.c_longlong
    for name, args in dict(chunk=[q, i, i], chunk_norm=[q, i], clip_small=[q, q], norm_here=[q], large=[q], one_slot=[q, i]).items():
        getattr(L, name).argtypes = args
    return L


@functools.lru_cache(maxsize=None)
def tensors_of_a_launch():
    """(norm, clip, update) tensors that the arguments of a launch hold."""
    text = open(os.path.join(CSRC, "update.hip")).read()
    return tuple(int(re.search(rf"\b{k}_TENSORS = (\d+)", text).group(1)) for k in ("NORM", "CLIP", "ADAMW"))


def clip_form(sizes):
    """How gsplit_clip_grads takes tensors of these sizes, as gsplit_clip_grads in csrc/update.hip has it."""
    L, (norm, clip, _) = _lib(), tensors_of_a_launch()
    full, total = [n for n in sizes if n], sum(sizes)
    chunk = L.chunk(total, 4096, N_CU)
    if L.clip_small(total, len(full)):
        return ("one workgroup",)
    return ("launches", L.chunk_norm(total, N_CU), chunk, "one slot" if L.one_slot(total // chunk, N_CU) else "slots", _parts(full, norm), _parts(full, clip))


def adamw_form(sizes, clipped):
    L, (norm, _, adamw) = _lib(), tensors_of_a_launch()
    full, total = [n for n in sizes if n], sum(sizes)
    chunk = L.chunk(total, 2048, N_CU)
    size = "large" if L.large(total) else "small"
    if not clipped:
        return (size, chunk, "no norm", _parts(full, adamw))
    if len(full) <= adamw and L.norm_here(total):
        return (size, chunk, "norm here")
    return (size, chunk, "one slot" if L.one_slot(total // chunk, N_CU) else "slots", _parts(full, norm), _parts(full, adamw))


def _parts(full, room):
    return "one" if len(full) <= room else "several"
