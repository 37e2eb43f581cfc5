// Pieces of the kernels that attend over packed prompts and pages (paged_attn.hip: bf16, paged_attn_f32.hip: float32).
#pragma once
#include "attn_common.hpp"
#include "paged.hpp"

namespace samkv {

// Read-only arrays whose address is the same for all lanes: loads from here become scalar loads, also between the tile
// requests, which the compiler has to take for writes to memory.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int scan64(int x, int lane) {  // inclusive prefix sum over the lanes
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const int y = __shfl_up(x, w);
    if (lane >= w) x += y;
  }
  return x;
}

struct Item {
  int s;                     // sequence; < 0: no item
  int tile, chunk, n_chunks, tiles;
  int c;                     // keys of a chunk
  int first_part;            // items ahead of the sequence's
  SeqSpan q;
};

// Item number `index`, or, with BY_TILE, the sequence and tile of row tile number `index` (chunk 0).  Called by whole waves; the
// result is the same in every lane.  Within a sequence items run chunk by chunk, the last tile (with the most keys) first.
template <int TILE_ROWS, bool BY_TILE>
__device__ __forceinline__ Item find_item(const PagedAttnLaunch& a, int group, int index, int lane) {
  const BatchArg& b = a.b;
  auto span = [&](int s) {
    SeqSpan q = seq_span(b, min(s, b.n_seq - 1));
    if (s >= b.n_seq) q.n = q.len = 0;
    return q;
  };
  auto n_tiles = [&](const SeqSpan& q) { return (int)(((long long)q.n * group + TILE_ROWS - 1) / TILE_ROWS); };
  SeqSpan q = span(lane);
  int tiles = n_tiles(q);
  // keys of a chunk: those of all tiles and heads over the number of workgroups
  unsigned long long total = 0;
  for (int s = lane; s < b.n_seq; s += 64) {
    const SeqSpan x = s == lane ? q : span(s);
    total += (unsigned long long)(s == lane ? tiles : n_tiles(x)) * x.len;
  }
#pragma unroll
  for (int w = 1; w < 64; w *= 2) total += __shfl_xor(total, w);
  const unsigned long long share = (total * a.hkv + a.target - 1) / a.target;
  Item it;
  it.c = uniform((int)min((share + 63) / 64 * 64, 0x40000000ull));
  it.c = max(it.c, a.min_chunk);
  it.s = -1;
  int tiles_before = 0, items_before = 0;
  for (int s0 = 0; s0 < b.n_seq; s0 += 64) {
    if (s0 > 0) {
      q = span(s0 + lane);
      tiles = n_tiles(q);
    }
    const int chunks = max((q.len + it.c - 1) / it.c, 1), items = tiles * chunks;
    const int tiles_to = scan64(tiles, lane) + tiles_before, items_to = scan64(items, lane) + items_before;
    const int upto = BY_TILE ? tiles_to : items_to;
    const unsigned long long past = __ballot(upto > index);
    if (past != 0) {
      const int at = __ffsll(past) - 1;
      auto of = [&](int x) { return uniform(__shfl(x, at)); };
      it.s = s0 + at;
      it.tiles = of(tiles);
      it.n_chunks = of(chunks);
      it.first_part = of(items_to - items);
      it.q.first = of(q.first);
      it.q.n = of(q.n);
      it.q.len = of(q.len);
      const int local = index - (BY_TILE ? of(tiles_to - tiles) : it.first_part);
      it.chunk = BY_TILE ? 0 : local / it.tiles;
      it.tile = it.tiles - 1 - (BY_TILE ? local : local % it.tiles);
      return it;
    }
    tiles_before = uniform(__shfl(tiles_to, 63));
    items_before = uniform(__shfl(items_to, 63));
  }
  return it;
}

// Number of a (tile, chunk)'s partial result.
__device__ __forceinline__ int part_of(const Item& it, int chunk) { return it.first_part + chunk * it.tiles + it.tiles - 1 - it.tile; }

// Where the keys and values of a sequence's KV head lie.
template <bool PAGED>
struct KvSource {
  const PagedAttnLaunch& a;
  int s, kvh, first, last;  // sequence, KV head, its first row (prompts), its last key

  // byte offset of key `key` <= last in k or v (uniform); `page` of it comes from page_of
  __device__ __forceinline__ long long at(const RowsArg& r, int key, int page) const {
    if constexpr (PAGED) return ((long long)page * a.hkv + kvh) * r.hs + (long long)(key & ((1 << a.b.page_log2) - 1)) * r.rs;
    else return (long long)kvh * r.hs + (long long)(first + key) * r.rs;
  }
  __device__ __forceinline__ int page_of(int key) const {
    if constexpr (!PAGED) return 0;
    const int p = ((ScalarInts)a.b.table)[(long long)s * a.b.max_pages + (min(key, last) >> a.b.page_log2)];
    return min(max(p, 0), a.b.n_pages - 1);
  }
};

// One row of a sequence against the keys of its item's chunk by a wave, key by key: what a workgroup falls back on that has met
// an infinity or a NaN among its values.  The matrix products multiply the values of keys that a row does not see by zero, and
// two-term weights have terms of zero and of either sign; here a value meets the weight of a row that sees it, and nothing else.
template <bool BF16, int D, bool PAGED>
__device__ __forceinline__ void attend_row(const PagedAttnLaunch& a, const Item& it, const KvSource<PAGED>& src, int r, int begin, int row) {
  constexpr int CPL = D / 64;
  const int lane = threadIdx.x & 63, group = a.hq / a.hkv;
  const int t = r / group, head = src.kvh * group + r % group, tok = it.q.first + t;
  const int end = min(min(it.q.len - it.q.n + t + 1, it.q.len), begin + it.c);
  auto element = [](const char* p, int c) {
    if constexpr (BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[c] << 16);
    else return reinterpret_cast<const float*>(p)[c];
  };
  auto page_of = [&](int key) { return PAGED ? min(max(a.b.table[(long long)it.s * a.b.max_pages + (key >> a.b.page_log2)], 0), a.b.n_pages - 1) : 0; };
  const char* qr = a.q.p + head * a.q.hs + tok * a.q.rs;
  float m = -INFINITY, l = 0.f, o[CPL] = {};
  for (int k0 = begin; k0 < end; k0 += 64) {
    float x = -INFINITY;
    if (k0 + lane < end) {
      const char* kr = a.k.p + src.at(a.k, k0 + lane, page_of(k0 + lane));
      float dot = 0.f;
#pragma unroll 4
      for (int c = 0; c < D; ++c) dot = fmaf(element(qr, c), element(kr, c), dot);
      x = dot * a.scale;
    }
    float mx = x;
    for (int w = 1; w < 64; w *= 2) mx = fmaxf(mx, __shfl_xor(mx, w));
    const float m_new = fmaxf(m, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float p = expf(x - m_use), alpha = expf(m - m_use);
    float sum = p;
    for (int w = 1; w < 64; w *= 2) sum += __shfl_xor(sum, w);
    l = l * alpha + sum;
    m = m_new;
    for (int e = 0; e < CPL; ++e) o[e] *= alpha;
#pragma unroll 1
    for (int j = 0; j < min(64, end - k0); ++j) {
      const float w = __shfl(p, j);
      const char* vr = a.v.p + src.at(a.v, k0 + j, page_of(k0 + j));
      for (int e = 0; e < CPL; ++e) o[e] = fmaf(w, element(vr, lane + 64 * e), o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int e = 0; e < CPL; ++e) o[e] *= inv;
  const float lse = m + logf(l);
  if (it.n_chunks > 1) {
    const long long at = ((long long)part_of(it, it.chunk) * a.hkv + src.kvh) * a.tile_rows + row;
    for (int e = 0; e < CPL; ++e) a.part_o[at * D + lane + 64 * e] = o[e];
    if (lane == 0) a.part_lse[at] = lse * kLog2e;
    return;
  }
  char* out = a.out.p + head * a.out.hs + tok * a.out.rs;
  for (int e = 0; e < CPL; ++e) {
    if constexpr (BF16) reinterpret_cast<__bf16*>(out)[lane + 64 * e] = (__bf16)o[e];
    else reinterpret_cast<float*>(out)[lane + 64 * e] = o[e];
  }
  if (a.lse != nullptr && lane == 0) a.lse[(long long)head * a.b.n_rows + tok] = lse;
}

}  // namespace samkv
