// Pieces of the kernels that attend over packed prompts and pages (paged_attn.hip: bf16, paged_attn_f32.hip: float32).
#pragma once
#include "attn_common.hpp"
#include "paged.hpp"

namespace samkv {

// Read-only arrays whose address is the same for all lanes: loads from here become scalar loads, also between the tile
// requests, which the compiler has to take for writes to memory.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int scan64(int x) {  // inclusive prefix sum over the lanes, on the vector ALU
#define SAMKV_STEP(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, false)
  SAMKV_STEP(0x111, 0xF);  // one, two, four and eight lanes up within a row of 16
  SAMKV_STEP(0x112, 0xF);
  SAMKV_STEP(0x114, 0xF);
  SAMKV_STEP(0x118, 0xF);
  SAMKV_STEP(0x142, 0xA);  // the last lane of a row to the next row, of the first half to the second
  SAMKV_STEP(0x143, 0xC);
#undef SAMKV_STEP
  return x;
}
__device__ __forceinline__ int last_of(int x) { return __builtin_amdgcn_readlane(x, 63); }

struct Item {
  int s;                     // sequence; < 0: no item
  bool wide;
  int slots;                 // of a (tile, chunk) whose result is a part: one per 32 rows
  int tile, chunk, n_chunks, tiles;
  int c;                     // keys of a chunk
  int first_slot;            // slots of partial results ahead of the sequence's
  SeqSpan q;
};

// Finds work items: JOIN = false, number `index` of them; JOIN = true, group of 32 rows number `index` among the tiles whose keys
// are cut (the chunk is the first).  All calls are by whole waves, and the results are the same in every lane.  A lane holds one of
// 64 sequences; batches of up to that many are read once, and over a cache wide tiles are taken in order of falling length, so that
// a long sequence's are not the last to start (24 sequences with 1 to 1024 new tokens, those with many in front: 532 -> 525 us, at
// the end: 587 -> 483; prompts gain less than the order costs, 2 %).  Within a sequence items run chunk by chunk, the last tile
// (with the most keys) first.
template <int KG, bool JOIN>
struct Items {
  const PagedAttnLaunch& a;
  const int lane, group;
  ChunkKeys c;                    // keys of a chunk
  int seq, tiles, chunks, slots;  // of this lane's sequence: number, tiles, chunks and partial results
  SeqSpan q;
  int upto, slots_to;             // items (or groups of rows) and partial results up to it in its block of 64

  __device__ __forceinline__ bool is_wide(const SeqSpan& x) const { return KG > 0 && (long long)x.n * group > kFewRows; }
  __device__ __forceinline__ int n_tiles(const SeqSpan& x) const {
    const int rows = is_wide(x) ? wide_rows<KG>() : 32;
    return (int)(((long long)x.n * group + rows - 1) / rows);
  }
  __device__ __forceinline__ void read(int s0) {
    seq = s0 + lane;
    q = seq_span(a.b, min(seq, a.b.n_seq - 1));
    if (seq >= a.b.n_seq) q.n = q.len = 0;
    tiles = n_tiles(q);
  }
  __device__ __forceinline__ void count() {
    const int per = is_wide(q) ? wide_rows<KG>() / 32 : 1;
    chunks = a.max_chunks > 1 ? chunks_of(is_wide(q), q.len, c) : 1;
    slots = chunks > 1 ? tiles * chunks * per : 0;
    upto = scan64(JOIN ? (chunks > 1 ? tiles * per : 0) : tiles * chunks);
    slots_to = a.max_chunks > 1 ? scan64(slots) : 0;
  }

  __device__ __forceinline__ Items(const PagedAttnLaunch& a_) : a(a_), lane(threadIdx.x & 63), group(a_.hq / a_.hkv) {
    read(0);
    c = {};
    if (a.max_chunks > 1) {
      // keys of a chunk of 32 rows: the cost of all tiles and heads over the number of workgroups (2^target_log2); a wide tile's
      // are fewer by what it costs more
      unsigned long long total = 0;
      int n = 0, longest = 0;
      for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
        if (s0 > 0) read(s0);
        total += (unsigned long long)tiles * q.len * (is_wide(q) ? wide_cost<KG>() : 1);
        n += tiles;
        longest = max(longest, q.len);
      }
      if (a.b.n_seq > 64) read(0);
      // lane by lane in two halves: sums of 64 numbers below 2^24 and of their upper parts
      const unsigned long long high = (unsigned)last_of(scan64((int)(total >> 24)));
      total = (high << 24) + (unsigned)last_of(scan64((int)(total & 0xFFFFFF)));
      // sequences of one length make chunks of one length, and as many workgroups as are resident end together; others do not,
      // and half as long ones leave less at the end (64 sequences, 1024 to 8192 keys, 8 heads: 222 -> 204 us; all of 4096: 168 and 175)
      const bool uneven = a.ragged_log2 > a.target_log2 && __any((float)longest * (float)last_of(scan64(n)) > 1.25f * (float)total);
      c = chunk_keys<KG>(total, a.hkv, uneven ? a.ragged_log2 : a.target_log2, a.min_chunk);
    }
    if (KG > 0 && a.paged && a.b.n_seq > 1 && a.b.n_seq <= 64) {
      int rank = 0;
      for (int j = 0; j < a.b.n_seq; ++j) {
        const int other = __builtin_amdgcn_readlane(q.len, j);
        rank += other > q.len || (other == q.len && j < lane) ? 1 : 0;
      }
      auto move = [&](int x) { return __builtin_amdgcn_ds_permute(rank * 4, x); };
      if (lane >= a.b.n_seq) rank = lane;
      seq = move(seq);
      q.first = move(q.first);
      q.n = move(q.n);
      q.len = move(q.len);
      tiles = move(tiles);
    }
    count();
  }

  // Groups of rows in all (JOIN).
  __device__ __forceinline__ int total() {
    int n = last_of(upto);
    for (int s0 = 64; s0 < a.b.n_seq; s0 += 64) {
      read(s0);
      count();
      n += last_of(upto);
    }
    return n;
  }

  __device__ __forceinline__ Item find(int index, int* rows32 = nullptr) {
    Item it;
    it.s = -1;
    int before = 0, slots_before = 0;
    for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
      if (a.b.n_seq > 64) {
        read(s0);
        count();
      }
      const unsigned long long past = __ballot(upto + before > index);
      if (past != 0) {
        const int at = __ffsll(past) - 1;
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
        it.s = of(seq);
        it.tiles = of(tiles);
        it.n_chunks = of(chunks);
        it.q.first = of(q.first);
        it.q.n = of(q.n);
        it.q.len = of(q.len);
        it.wide = is_wide(it.q);
        // even chunks, rounded up to 128 keys: the last ones may be short (700 keys in six: five of 128 and one of 60) or empty
        it.c = a.max_chunks > 1 ? ((it.q.len + it.n_chunks - 1) / it.n_chunks + 127) / 128 * 128 : 0x40000000;
        it.slots = it.wide ? wide_rows<KG>() / 32 : 1;
        it.first_slot = slots_before + of(slots_to - slots);
        const int mine = JOIN ? it.tiles * it.slots : it.tiles * it.n_chunks, local = index - (before + of(upto) - mine);
        if constexpr (JOIN) {
          it.chunk = 0;
          it.tile = local / it.slots;
          *rows32 = local % it.slots;
        } else {
          it.chunk = local / it.tiles;
          it.tile = it.tiles - 1 - local % it.tiles;
        }
        // counts that have overflowed, and prefix sums that go backwards and so ask for more room than the batch's rows do
        if (local < 0 || it.chunk >= it.n_chunks || it.tile >= it.tiles) it.s = -1;
        if (it.n_chunks > 1 && (it.first_slot < 0 || (long long)it.first_slot + (long long)it.tiles * it.n_chunks * it.slots > a.max_slots))
          it.s = -1;
        return it;
      }
      before += last_of(upto);
      slots_before += last_of(slots_to);
    }
    return it;
  }
};

// First slot of a (tile, chunk)'s partial result (one of every KV head stands there), and the row of part_lse and part_o that
// one head's begins at.
__device__ __forceinline__ int part_slot(const Item& it, int chunk) {
  return it.first_slot + (chunk * it.tiles + it.tiles - 1 - it.tile) * it.slots;
}
__device__ __forceinline__ long long part_row(const PagedAttnLaunch& a, const Item& it, int chunk, int kvh) {
  return ((long long)part_slot(it, chunk) * a.hkv + (long long)kvh * it.slots) * a.tile_rows;
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

// One row of a sequence against the keys of its item's chunk by a wave, so that a value meets the weight of a row that sees it and
// nothing else.  The matrix products multiply the values of keys that a row does not see by zero, and two-term weights have terms
// of zero and of either sign: infinities and NaN among the values make NaN of the outputs of any row.  Rows whose outputs are not
// all finite are therefore computed once more like this, unless their sum is NaN: a score that they see is, and so is every output.
// A lane takes a key for the scores, channels for the outputs.
template <bool BF16, int D, bool PAGED>
__device__ __forceinline__ void attend_row(const PagedAttnLaunch& a, const Item& it, const KvSource<PAGED>& src, int r, int begin, int row) {
  constexpr int CPL = D / 64, PIECES = D * (BF16 ? 2 : 4) / 16, U = 8;
  const int lane = threadIdx.x & 63, group = a.hq / a.hkv;
  const int t = r / group, head = src.kvh * group + r % group, tok = it.q.first + t;
  const int end = min(min(it.q.len - it.q.n + t + 1, it.q.len), begin + it.c);
  auto element = [](const char* p, int c) {
    if constexpr (BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[c] << 16);
    else return reinterpret_cast<const float*>(p)[c];
  };
  const char* qr = a.q.p + head * a.q.hs + tok * a.q.rs;
  float m = -INFINITY, l = 0.f, o[CPL] = {};
#pragma unroll 1
  for (int k0 = begin; k0 < end; k0 += 64) {
    const int n = min(64, end - k0), key = k0 + min(lane, n - 1);
    int page = 0;
    if constexpr (PAGED) page = min(max(a.b.table[(long long)it.s * a.b.max_pages + (key >> a.b.page_log2)], 0), a.b.n_pages - 1);
    const char* kr = a.k.p + src.at(a.k, key, page);
    float dot = 0.f;
#pragma unroll 4
    for (int c = 0; c < PIECES; ++c) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(qr + c * 16), y = *reinterpret_cast<const u32x4*>(kr + c * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF16) dot = fmaf(bf16_hi(x[e]), bf16_hi(y[e]), fmaf(bf16_lo(x[e]), bf16_lo(y[e]), dot));
        else dot = fmaf(__uint_as_float(x[e]), __uint_as_float(y[e]), dot);
      }
    }
    const float x = lane < n ? dot * a.scale : -INFINITY;
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
    for (int j = 0; j < n; j += U) {
      float y[U][CPL];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = min(j + u, n - 1);
        const char* vr = a.v.p + src.at(a.v, k0 + at, __builtin_amdgcn_readlane(page, at));
#pragma unroll
        for (int e = 0; e < CPL; ++e) y[u][e] = element(vr, lane + 64 * e);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u < n) {
          const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), min(j + u, 63)));
#pragma unroll
          for (int e = 0; e < CPL; ++e) o[e] = fmaf(w, y[u][e], o[e]);
        }
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

// Joins the partial results of NW waves over one tile of 32 rows and writes them (as the item's, or as a part of them): maxima
// and sums first, then the rows, each wave's scaled to the common maximum, through LDS.
constexpr int join_area(int d) { return 32 * (d * 4 + 16); }  // LDS bytes of a wave's rows (pad: 16 rows hit 64 distinct banks)
constexpr int join_lds(int nw, int area) { return nw * area + nw * 32 * 8; }
template <int D, int NW, bool BF16, bool PAGED, int AREA>
__device__ __forceinline__ void join_waves(const PagedAttnLaunch& a, const Item& it, const KvSource<PAGED>& src, f32x16 (&o)[D / 32],
                                           float m_run, float l_run, int begin) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int NV = D / 32, OROW = D * 4 + 16;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), rw = lane & 31, h = lane >> 5;
  const int group = a.hq / a.hkv, kvh = src.kvh, n_rows = it.q.n * group, r0 = it.tile * 32;
  float* s_m = reinterpret_cast<float*>(smem + NW * AREA);
  float* s_l = s_m + NW * 32;
  const float l_row = sum_across_halves(l_run);
  if (h == 0) {
    s_m[wave * 32 + rw] = m_run;
    s_l[wave * 32 + rw] = l_row;
  }
  __syncthreads();
  const int n_valid = min(32, n_rows - r0);
  auto joined = [&](int row, float* m_out) {
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, s_m[w * 32 + row]);
    const float m_use = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < NW; ++w) l = fmaf(s_l[w * 32 + row], __builtin_amdgcn_exp2f(s_m[w * 32 + row] - m_use), l);
    *m_out = m;
    return l;
  };
  {
    float m;
    joined(rw, &m);
    const float f = __builtin_amdgcn_exp2f(m_run - (m == -INFINITY ? 0.f : m));
    char* mine = smem + wave * AREA + rw * OROW + h * 16;
    if (rw < n_valid) {
#pragma unroll
      for (int dvb = 0; dvb < NV; ++dvb)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[dvb][4 * j4 + e] * f;
          *reinterpret_cast<f32x4*>(mine + (dvb * 32 + 8 * j4) * 4) = x;
        }
    }
  }
  __syncthreads();
  constexpr int LPR = D / 4, RPW = 64 / LPR;  // lanes per row, rows of a wave at a time
  for (int row0 = wave * RPW; row0 < n_valid; row0 += NW * RPW) {
    const int row = min(row0 + lane / LPR, n_valid - 1), c4 = lane % LPR;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(smem + w * AREA + row * OROW + c4 * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    float m;
    const float l = joined(row, &m), inv = l == 0.f ? 0.f : 1.f / l;
    const unsigned long long odd = __ballot(l == l && !(fabsf(x[0]) + fabsf(x[1]) + fabsf(x[2]) + fabsf(x[3]) < INFINITY));
    if (odd != 0) {
#pragma unroll 1
      for (int i = 0; i < RPW && row0 + i < n_valid; ++i)
        if ((odd >> (i * LPR) & ((1ull << LPR) - 1)) != 0)
          attend_row<BF16, D, PAGED>(a, it, src, r0 + row0 + i, begin, row0 + i);
      if (row0 + lane / LPR >= n_valid || (odd >> (lane / LPR * LPR) & ((1ull << LPR) - 1)) != 0) continue;
    }
    if (row0 + lane / LPR >= n_valid) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    const float lse2 = m + __log2f(l);
    if (it.n_chunks > 1) {
      const long long at = part_row(a, it, it.chunk, kvh) + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + c4 * 4) = x;
      if (c4 == 0) a.part_lse[at] = lse2;
    } else {
      const int rr = r0 + row, tok = it.q.first + rr / group, hd = kvh * group + rr % group;
      char* out = a.out.p + hd * a.out.hs + tok * a.out.rs;
      if constexpr (BF16) {
        const bf16x4 y = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *reinterpret_cast<bf16x4*>(out + c4 * 8) = y;
      } else {
        *reinterpret_cast<f32x4*>(out + c4 * 16) = x;
      }
      if (c4 == 0 && a.lse != nullptr) a.lse[(long long)hd * a.b.n_rows + tok] = lse2 * kLn2;
    }
  }
}

// out = sum_c w_c part_o[c], w_c = 2^(lse_c - lse).  D / 4 threads take a row's channels, four each; they are a row's only group
// of threads where there are few chunks, and the workgroup's groups share a row's chunks where there are many: a group that walks
// 512 chunks spends a trip to memory on every eight.  Chunks without mass (lse = -inf)
// have outputs of zero.
template <int D, bool BF16, int KG>
__global__ __launch_bounds__(256) void k_join_chunks(PagedAttnLaunch a) {
  constexpr int LPR = D / 4, NG = 256 / LPR, U = 8;  // threads and groups of threads per row, chunks requested at once
  __shared__ f32x4 s_acc[256];
  __shared__ float s_m[256], s_den[256];
  const int group = a.hq / a.hkv, c4 = threadIdx.x % LPR, g = threadIdx.x / LPR;
  // A workgroup takes a part of the rows of a group and head: of one where there are enough of them.
  Items<KG, true> items(a);
  const int heads = min(max(items.total(), 0), a.max_slots / 2) * a.hkv;
  const int parts = heads >= (int)gridDim.x ? 1 : min((int)gridDim.x / max(heads, 1), a.tile_rows);
  for (int u = blockIdx.x; u < heads * parts; u += gridDim.x) {
    int rows32 = 0;
    const int head = u % heads, kvh = head % a.hkv;
    const Item it = items.find(head / a.hkv, &rows32);
    if (it.s < 0) continue;
    const int tile0 = it.tile * 32 * it.slots, n_rows = min(it.q.n * group - tile0, 32 * (rows32 + 1));
    const bool many = it.n_chunks > U;
    const int from = many ? g : 0, by = many ? NG : 1, step = many ? 1 : NG;
    for (int row0 = rows32 * 32 + u / heads * step; row0 < n_rows; row0 += parts * step) {
      const int row = min(many ? row0 : row0 + g, n_rows - 1);
      const long long at0 = part_row(a, it, 0, kvh) + row, apart = (long long)it.tiles * it.slots * a.hkv * a.tile_rows;
      float m = -INFINITY, den = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int c = from; c < it.n_chunks; c += by * U) {
        float l[U];
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long at = at0 + min(c + u * by, it.n_chunks - 1) * apart;
          l[u] = a.part_lse[at];
          x[u] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + c4 * 4);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (c + u * by >= it.n_chunks) l[u] = -INFINITY;
          top = fmaxf(top, l[u]);
        }
        const float use = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m - use);
        m = top;
        den *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (c + u * by >= it.n_chunks) continue;
          const float w = __builtin_amdgcn_exp2f(l[u] - use);
          den += w;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, x[u][e], acc[e]);
        }
      }
      if (many) {
        s_acc[threadIdx.x] = acc;
        s_m[threadIdx.x] = m;
        s_den[threadIdx.x] = den;
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NG; ++i) top = fmaxf(top, s_m[c4 + i * LPR]);
        const float use = top == -INFINITY ? 0.f : top;
        m = top;
        den = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = 0.f;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int from_i = c4 + i * LPR;
          const float w = __builtin_amdgcn_exp2f(s_m[from_i] - use);
          den = fmaf(w, s_den[from_i], den);
          const f32x4 x = s_acc[from_i];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, x[e], acc[e]);
        }
        __syncthreads();
      }
      if (many ? g > 0 : row0 + g >= n_rows) continue;
      const float inv = den == 0.f ? 0.f : 1.f / den;
      const int rr = tile0 + row, tok = it.q.first + rr / group, hd = kvh * group + rr % group;
      char* out = a.out.p + hd * a.out.hs + tok * a.out.rs;
      if constexpr (BF16) {
        const bf16x4 y = {(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
        *reinterpret_cast<bf16x4*>(out + c4 * 8) = y;
      } else {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = acc[e] * inv;
        *reinterpret_cast<f32x4*>(out + c4 * 16) = y;
      }
      if (c4 == 0 && a.lse != nullptr) a.lse[(long long)hd * a.b.n_rows + tok] = (m + __log2f(den)) * kLn2;
    }
  }
}

template <int D, bool BF16>
hipError_t launch_join(const PagedAttnLaunch& a, const PagedAttnPlan& p, hipStream_t s) {
  // a tile that is cut has two slots at least; no more workgroups than are resident at once
  const long long rows = (long long)(p.max_slots / 2) * a.hkv * p.tile_rows;
  const dim3 grid((unsigned)(rows < 1536 ? rows : 1536));
  if constexpr (BF16) {  // float32 has no wide tiles
    if (p.kg == 2) hipLaunchKernelGGL((k_join_chunks<D, true, 2>), grid, dim3(256), 0, s, a);
    if (p.kg == 1) hipLaunchKernelGGL((k_join_chunks<D, true, 1>), grid, dim3(256), 0, s, a);
  }
  if (p.kg == 0) hipLaunchKernelGGL((k_join_chunks<D, BF16, 0>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attn_f32(const PagedAttnLaunch& a, const PagedAttnPlan& p, hipStream_t s);
hipError_t paged_attn_f32_raise_limits();

}  // namespace samkv
