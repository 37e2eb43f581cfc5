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

// Sequences of at most kFewRows rows per KV head are cut into tiles of 32 rows, the others, where there is a kernel for that
// (WIDE), into tiles of kWideRows.
constexpr int kFewRows = 128, kWideRows = 256;
constexpr int kWideCost = 5;  // time of a wide tile over a number of keys, in tiles of 32 rows

struct Item {
  int s;                     // sequence; < 0: no item
  bool wide;
  int tile, chunk, n_chunks, tiles;
  int c;                     // keys of a chunk
  int first_slot;            // slots of partial results ahead of the sequence's
  SeqSpan q;
  __device__ __forceinline__ int slots() const { return wide ? kWideRows / 32 : 1; }  // of a (tile, chunk) that is a part
};

// Item number `index`.  JOIN: group of 32 rows number `index` among the tiles whose keys are cut; *rows32 is the group's number in
// its tile, and the chunk is the first.  Called by whole waves; the result is the same in every lane.  Within a sequence items
// run chunk by chunk, the last tile (with the most keys) first.
template <bool WIDE, bool JOIN>
__device__ __forceinline__ Item find_item(const PagedAttnLaunch& a, int group, int index, int lane, int* rows32 = nullptr) {
  const BatchArg& b = a.b;
  auto span = [&](int s) {
    SeqSpan q = seq_span(b, min(s, b.n_seq - 1));
    if (s >= b.n_seq) q.n = q.len = 0;
    return q;
  };
  auto is_wide = [&](const SeqSpan& q) { return WIDE && (long long)q.n * group > kFewRows; };
  auto n_tiles = [&](const SeqSpan& q) {
    const int rows = is_wide(q) ? kWideRows : 32;
    return (int)(((long long)q.n * group + rows - 1) / rows);
  };
  SeqSpan q = span(lane);
  int tiles = n_tiles(q);
  Item it;
  it.c = 0x40000000;
  if (a.max_chunks > 1) {
    // keys of a chunk of 32 rows: the cost of all tiles and heads over the number of workgroups; a wide tile's are fewer by
    // what it costs more.  A tile of new tokens sees on average half of them, and at least half of len.
    unsigned long long total = 0;
    for (int s = lane; s < b.n_seq; s += 64) {
      const SeqSpan x = s == lane ? q : span(s);
      const long long keys = max(x.len - x.n / 2, (x.len + 1) / 2);
      total += (unsigned long long)(s == lane ? tiles : n_tiles(x)) * keys * (is_wide(x) ? kWideCost : 1);
    }
#pragma unroll
    for (int w = 1; w < 64; w *= 2) total += __shfl_xor(total, w);
    const unsigned long long share = (total * a.hkv + a.target - 1) / a.target;
    it.c = uniform((int)min(share, 0x40000000ull));
  }
  const int c_few = max((it.c + 63) / 64 * 64, a.min_chunk), c_wide = max((it.c / kWideCost + 64) / 64 * 64, 2 * a.min_chunk);
  it.s = -1;
  int before = 0, slots_before = 0;
  for (int s0 = 0; s0 < b.n_seq; s0 += 64) {
    if (s0 > 0) {
      q = span(s0 + lane);
      tiles = n_tiles(q);
    }
    const int c = is_wide(q) ? c_wide : c_few, per = is_wide(q) ? kWideRows / 32 : 1;
    const int chunks = max((q.len + c - 1) / c, 1), items = tiles * chunks, slots = chunks > 1 ? items * per : 0;
    const int count = JOIN ? (chunks > 1 ? tiles * per : 0) : items;
    const int upto = scan64(count, lane) + before, slots_to = scan64(slots, lane) + slots_before;
    const unsigned long long past = __ballot(upto > index);
    if (past != 0) {
      const int at = __ffsll(past) - 1;
      auto of = [&](int x) { return uniform(__shfl(x, at)); };
      it.s = s0 + at;
      it.tiles = of(tiles);
      it.n_chunks = of(chunks);
      it.first_slot = of(slots_to - slots);
      it.q.first = of(q.first);
      it.q.n = of(q.n);
      it.q.len = of(q.len);
      it.wide = is_wide(it.q);
      it.c = it.wide ? c_wide : c_few;
      const int local = index - of(upto - count);
      if constexpr (JOIN) {
        it.chunk = 0;
        it.tile = local / it.slots();
        *rows32 = local % it.slots();
      } else {
        it.chunk = local / it.tiles;
        it.tile = it.tiles - 1 - local % it.tiles;
      }
      return it;
    }
    before = uniform(__shfl(upto, 63));
    slots_before = uniform(__shfl(slots_to, 63));
  }
  return it;
}

// First slot of a (tile, chunk)'s partial result (one of every KV head stands there), and the row of part_lse and part_o that
// one head's begins at.
__device__ __forceinline__ int part_slot(const Item& it, int chunk) {
  return it.first_slot + (chunk * it.tiles + it.tiles - 1 - it.tile) * it.slots();
}
__device__ __forceinline__ long long part_row(const PagedAttnLaunch& a, const Item& it, int chunk, int kvh) {
  return ((long long)part_slot(it, chunk) * a.hkv + (long long)kvh * it.slots()) * a.tile_rows;
}
// Prefix sums that go backwards can ask for more room than the batch's rows do; what has none is left out.
__device__ __forceinline__ bool has_room(const PagedAttnLaunch& a, const Item& it) {
  return it.n_chunks == 1 || part_slot(it, it.n_chunks - 1) + it.slots() <= a.max_slots;
}

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
    const long long at = part_row(a, it, it.chunk, src.kvh) + row;
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
