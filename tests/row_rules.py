"""The rules of the losses over rows and of the update (csrc/row_rules.h, csrc/update_rules.h), compiled for the host (not a test
module itself)."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2303_13775_amd", "csrc")
N_CU = 256
FORMS = ["16x8", "16x16", "16x32", "64x16", "64x32", "256x8", "256x32", "256x64", "512x64", "1024x64", "1024x96", "512x128_RAW", "1024x128_RAW", "STREAMED"]

_SOURCE = r"""
#include "row_rules.h"
#include "update_rules.h"
typedef long long I;
extern "C" int form(I rows, int C, int piece, int n_cu) { return row_form(rows, C, piece, n_cu); }
extern "C" int part(int C) { return row_part(C); }
extern "C" int whole(I rows, I pairs, int C, int n_cu) { return preference_whole(rows, pairs, C, n_cu); }
extern "C" int chunks(I rows, int C, int n_cu) { return row_chunks(rows, C, n_cu); }
extern "C" int policy_parts(I rows, int C, int piece, int n_cu) { return policy_in_parts(rows, C, piece, n_cu); }
extern "C" int preference_parts(I rows, int C, int n_cu) { return preference_in_parts(rows, C, n_cu); }
extern "C" int parts_held() { return GS_ROW_PARTS; }
extern "C" int chunk(I total, int most, int n_cu) { return update_chunk(total, most, n_cu); }
extern "C" int chunk_norm(I total, int n_cu) { return norm_chunk(total, n_cu); }
extern "C" int clip_small(I total) { return update_clip_small(total); }
extern "C" int norm_here(I total) { return update_norm_here(total); }
"""


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        L = C.CDLL(out)
    i, q = C.c_int, C.c_longlong
    for name, args in dict(form=[q, i, i, i], part=[i], whole=[q, q, i, i], chunks=[q, i, i], policy_parts=[q, i, i, i],
                           preference_parts=[q, i, i], parts_held=[], chunk=[q, i, i], chunk_norm=[q, i], clip_small=[q], norm_here=[q]).items():
        getattr(L, name).argtypes = args
    return L


def form(rows, C, piece):
    return FORMS[lib().form(rows, C, piece, N_CU)]
