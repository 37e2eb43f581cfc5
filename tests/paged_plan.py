"""The plan of an attention over prompts or pages, as csrc/paged_plan.hpp makes it, built by the host compiler."""
from __future__ import annotations

import ctypes
import os
import subprocess
import tempfile
from functools import lru_cache

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_11661_amd", "csrc")
FIELDS = ("kg", "joins", "max_items", "max_slots", "tile_rows", "bytes", "target_log2", "ragged_log2", "min_chunk")
SOURCE = """#include "paged_plan.hpp"
extern "C" void plan(int dtype, int d, int hq, int hkv, int n_seq, int n_rows, int max_new, int max_len, int paged, long long* o) {
  const samkv::PagedAttnPlan p = samkv::paged_attn_plan(dtype, d, hq, hkv, n_seq, n_rows, max_new, max_len, paged != 0);
  const long long x[] = {p.kg, p.joins, p.max_items, p.max_slots, p.tile_rows, (long long)p.bytes, p.target_log2, p.ragged_log2,
                         p.min_chunk};
  for (int i = 0; i < 9; ++i) o[i] = x[i];
}

template <int KG>
static void count(int hq, int hkv, int n_seq, const int* lens, const int* rows, int log2, int ragged_log2, int min_chunk, int cut, long long* o) {
  const long long group = hq / hkv, few = samkv::kFewRows;
  auto wide = [&](int s) { return KG > 0 && rows[s] * group > few; };
  auto tiles = [&](int s) -> long long { const int tile = wide(s) ? samkv::wide_rows<KG>() : 32; return (rows[s] * group + tile - 1) / tile; };
  unsigned long long total = 0;
  long long n = 0, longest = 0;
  for (int s = 0; s < n_seq; ++s) {
    total += (unsigned long long)tiles(s) * lens[s] * (wide(s) ? samkv::wide_cost<KG>() : 1);
    n += tiles(s);
    longest = lens[s] > longest ? lens[s] : longest;
  }
  const bool uneven = ragged_log2 > log2 && (float)longest * (float)n > 1.25f * (float)total;
  const samkv::ChunkKeys c = samkv::chunk_keys<KG>(total, hkv, uneven ? ragged_log2 : log2, min_chunk);
  for (int s = 0; s < n_seq; ++s) {
    const long long chunks = cut ? samkv::chunks_of(wide(s), lens[s], c) : 1;
    o[0] += tiles(s) * chunks;
    if (chunks > 1) o[1] += tiles(s) * chunks * (wide(s) ? samkv::wide_rows<KG>() / 32 : 1);
  }
}
extern "C" void items(int kg, int hq, int hkv, int n_seq, const int* lens, const int* rows, int log2, int ragged_log2, int min_chunk, int cut,
                      long long* o) {
  o[0] = o[1] = 0;
  (kg == 2 ? count<2> : kg == 1 ? count<1> : count<0>)(hq, hkv, n_seq, lens, rows, log2, ragged_log2, min_chunk, cut, o);
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


def items(kg, p, hq, hkv, lens, new):
    """Work items of a batch and slots of its partial results, as the device counts them (Items in csrc/paged_attn.hpp)."""
    ints = lambda x: (ctypes.c_int * len(x))(*x)
    o = (ctypes.c_longlong * 2)()
    _lib().items(kg, hq, hkv, len(lens), ints(lens), ints(new), p["target_log2"], p["ragged_log2"], p["min_chunk"], p["joins"], o)
    return o[0], o[1]
