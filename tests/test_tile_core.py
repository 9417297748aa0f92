"""Fetches into LDS (csrc/tile_core.h) and the register that holds their place, from the assembly of a kernel compiled here."""
import re
import shutil
import subprocess

import pytest

from paper_2303_13775_amd import build

_SOURCE = r"""
#include <hip/hip_runtime.h>
#include <cstdint>
#include "tile_core.h"
__global__ void k(const void *from, uint32_t x) {
    __shared__ core_u32x4 lds[64];
    uint32_t v;
    asm volatile("s_mov_b32 %0, %1 ; set here" : "={m0}"(v) : "s"(x));
    core_fetch(from, lds);
    asm volatile("; used here: %0" ::"{m0}"(v));
}
"""


def test_a_value_in_m0_outlives_a_fetch(tmp_path):
    hipcc = build._hipcc()
    if not shutil.which(hipcc):
        pytest.skip("needs hipcc")
    src, out = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(_SOURCE)
    subprocess.run([hipcc, *build.HIPCC_FLAGS, "-S", "--cuda-device-only", str(src), "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    own, fetch, use = (text.index(s) for s in ("set here", "global_load_lds_dwordx4", "used here"))
    assert own < fetch < use
    saved = re.search(r"s_mov_b32 (s\d+), m0\b", text[own:fetch])
    assert saved and re.search(rf"s_mov_b32 m0, {saved.group(1)}\b", text[fetch:use])
    place = text[own:fetch].rfind(" m0,")       # the fetch's own place, and a wait state behind it
    assert place > saved.start() and "s_nop 0" in text[own + place:fetch]
