"""The plan of an attention over prompts or pages, as csrc/paged_plan.hpp makes it, built by the host compiler."""
from __future__ import annotations

import ctypes
import os
import subprocess
import tempfile
from functools import lru_cache

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_11661_amd", "csrc")
FIELDS = ("kg", "joins", "max_items", "max_slots", "tile_rows", "bytes")
SOURCE = """#include "paged_plan.hpp"
extern "C" void plan(int dtype, int d, int hq, int hkv, int n_seq, int n_rows, int max_new, int max_len, int paged, long long* o) {
  const samkv::PagedAttnPlan p = samkv::paged_attn_plan(dtype, d, hq, hkv, n_seq, n_rows, max_new, max_len, paged != 0);
  const long long x[] = {p.kg, p.joins, p.max_items, p.max_slots, p.tile_rows, (long long)p.bytes};
  for (int i = 0; i < 6; ++i) o[i] = x[i];
}
"""


@lru_cache(maxsize=1)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "plan.cpp"), os.path.join(tmp, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
        return ctypes.CDLL(so)


def plan(dtype, d, hq, hkv, n_seq, n_rows, max_new, max_len, paged):
    o = (ctypes.c_longlong * len(FIELDS))()
    _lib().plan(int(dtype == "bf16"), d, hq, hkv, n_seq, n_rows, min(max_new, n_rows), max_len, int(paged), o)
    return dict(zip(FIELDS, o))


def of_prompts(dtype, d, hq, hkv, lens, extra=0):
    most = min(max(lens), sum(lens) + extra)
    return plan(dtype, d, hq, hkv, len(lens), sum(lens) + extra, most, most, False)


def of_pages(dtype, d, hq, hkv, lens, new, extra=0, max_len=None):
    return plan(dtype, d, hq, hkv, len(lens), sum(new) + extra, max(new), max(lens) if max_len is None else max_len, True)
