// Attention of the rows of a batch of sequences over packed prompts (samkv_prefill_attn) or over pages (samkv_paged_attn):
// the row at slot p of its sequence sees slots 0..p.  bf16; float32: paged_attn_f32.hip.
//
// Products as in attn.hip: S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, a wave holding 32 rows in its lanes'
// columns, so that the softmax weights come out of the first product in the operand layout of the second and V is turned by
// the transposing LDS read.
#include <mutex>

#include "paged_attn.hpp"

namespace samkv {
namespace {

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---------------------------------------------------------------------------------------------- few rows
// A workgroup is NW waves that share one tile of 32 rows and split the keys of their chunk: wave w takes tiles of BK keys w, w
// + NW, ...  Each wave has its own K and V slot in LDS, filled by asynchronous loads (K of the next tile is requested as soon as K's
// fragments are in registers, V likewise), so there is no barrier until the waves' results are joined.  The first products of a
// pass do wait for all requests, K of the next tile among them: the compiler cannot see these, and puts its wait for the query
// fragments, which are loaded before the loop, there.  What overlaps a wave's loads are the other waves.
// Bound by HBM while each key is read once: 64 sequences x 4096 keys, 32 heads over 8, d = 128: 163 us, 6.6 TB/s (reading 2 GiB: 7.1);
// one of 131072 keys 86 + 5 us for the join, 6.0 TB/s.  Few short sequences are bound by the chain launch, lengths, page table, K, V,
// join: 4 x 1000 keys 15 us with the append before it.
template <int D, int NW>
struct FewCfg {
  static constexpr int ROWB = D * 2, CPR = ROWB / 16, RPI = 1024 / ROWB;  // bytes and chunks per row, rows per request
  static constexpr int BK = 8192 / ROWB, NI = 8;                          // keys and requests of a tile
  static constexpr int AREA = join_area(D) > 16384 ? join_area(D) : 16384;  // of a wave: K slot and V slot, then its output rows
  static constexpr int LDS_BYTES = join_lds(NW, AREA);
  static __device__ __forceinline__ int kswz(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int vswz(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }
};

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(uint32_t at) {
  return (__attribute__((address_space(3))) T*)(size_t)at;
}

// Lane L of a wave-wide request lands at lds + 16 L.  ONCE: nobody reads these bytes again, and they are not kept in L2.
template <bool ONCE = false>
__device__ __forceinline__ void request(const char* base, uint32_t off, uint32_t lds) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N requests are on their way
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

union Frag {
  struct { s16x4 lo, hi; } s;
  bf16x8 b;
  u32x4 u;
};
// ONCE: sequences are one tile, so that each K and V row is read once (64 x 4096 keys, 8 heads: 192 -> 170 us, 6.3 TB/s; where
// the sequences share all pages, 78 -> 79 us, 16 x 16384 keys 81 -> 88 us).
template <int D, bool PAGED, int NW, bool ONCE>
__device__ __forceinline__ void attend_few(const PagedAttnLaunch& a, const Item& it, int kvh) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using C = FewCfg<D, NW>;
  constexpr int ND = D / 16, NV = D / 32, NKB = C::BK / 32, NG = C::BK / 16, ROWB = C::ROWB, CPR = C::CPR, RPI = C::RPI;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int rw = lane & 31, h = lane >> 5;
  const int group = a.hq / a.hkv, n_rows = it.q.n * group, r0 = it.tile * 32;
  const int pos0 = it.q.len - it.q.n;  // slot of the first new token

  const int r = min(r0 + rw, n_rows - 1), t = r / group, head = kvh * group + r % group;
  const int t_first = r0 / group, t_last = min(r0 + 31, n_rows - 1) / group;
  const int seen_first = pos0 + t_first + 1;                       // keys that the tile's first and last row see
  const int begin = it.chunk * it.c, end = min(min(pos0 + t_last + 1, it.q.len), begin + it.c);
  const int key_end = min(pos0 + t + 1, end);                      // one past the last key that counts for this lane's row

  bf16x8 bq[ND];
  {
    const char* qp = a.q.p + head * a.q.hs + (long long)(it.q.first + t) * a.q.rs + h * 16;
#pragma unroll
    for (int dc = 0; dc < ND; ++dc) bq[dc] = *reinterpret_cast<const bf16x8*>(qp + dc * 32);
  }
  const KvSource<PAGED> src{a, it.s, kvh, it.q.first, it.q.len - 1};
  const uint32_t smem_at = (uint32_t)(size_t)(const __attribute__((address_space(3))) char*)smem;
  const uint32_t k_lds = uniform(smem_at + wave * C::AREA), v_lds = k_lds + 8192;
  const char* ks = smem + wave * C::AREA;
  const char* vs = ks + 8192;

  // Tiles are requested 16 keys at a time, which lie in one page.  Keys past the last one re-read that one: their weights are
  // zero.
  auto pages_of = [&](int k0, int (&pg)[NG]) {
#pragma unroll
    for (int g = 0; g < NG; ++g) pg[g] = src.page_of(k0 + 16 * g);
  };
  const int lrow = lane / CPR, pos = lane % CPR;
  auto request_tile = [&](int k0, const int (&pg)[NG], const RowsArg& rows, bool is_v, uint32_t lds) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const char* base = rows.p + src.at(rows, min(k0 + 16 * g, src.last), pg[g]);
      const int lim = max(src.last - k0 - 16 * g, 0);
#pragma unroll
      for (int i = 0; i < 16 / RPI; ++i) {
        const int row = i * RPI + lrow;
        const uint32_t chunk = (uint32_t)(pos ^ (is_v ? C::vswz(16 * g + row) : C::kswz(16 * g + row))) * 16;
        request<ONCE>(base, (uint32_t)min(row, lim) * (uint32_t)rows.rs + chunk, lds + (g * (16 / RPI) + i) * 1024);
      }
    }
  };

  // LDS addresses of the fragments: every further one differs from the first in bits that the swizzle leaves to an exclusive or
  uint32_t k_at = (uint32_t)(rw * ROWB + ((h ^ C::kswz(rw)) * 16)), v_at;
  {
    const int i16 = lane & 15, q2 = (lane >> 4) & 1, vrow = 4 * h + (i16 >> 2);
    v_at = (uint32_t)(vrow * ROWB + (((2 * q2 + ((i16 & 3) >> 1)) ^ C::vswz(vrow)) * 16) + 8 * (i16 & 1));
  }

  f32x16 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float c2 = a.scale * kLog2e;

  int k0 = begin + wave * C::BK;
  int pg[NG];
  if (k0 < end) {
    pages_of(k0, pg);
    request_tile(k0, pg, a.k, false, k_lds);
    request_tile(k0, pg, a.v, true, v_lds);
  }
  for (; k0 < end; k0 += NW * C::BK) {
    const int k1 = k0 + NW * C::BK;
    const bool more = k1 < end;
    if (more) pages_of(k1, pg);

    wait_loads<C::NI>();  // K has landed, V may be on its way
    bf16x8 ak[NKB][ND];
    asm volatile("" : "+v"(k_at), "+v"(v_at));  // the exclusive ors stay in the loop, not in registers
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int dc = 0; dc < ND; ++dc) ak[kb][dc] = *reinterpret_cast<const bf16x8*>(ks + (k_at ^ (dc << 5)) + kb * 32 * ROWB);
    wait_lds();
    if (more) request_tile(k1, pg, a.k, false, k_lds);
    f32x16 s[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s[kb][j] = 0.f;
#pragma unroll
      for (int dc = 0; dc < ND; ++dc) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[kb][dc], bq[dc], s[kb], 0, 0, 0);
    }
    // accumulator register j of block kb: key k0 + 32 kb + 8 (j / 4) + 4 h + j % 4
    const bool masked = k0 + C::BK > min(seen_first, end);
    const int n_ok = key_end - k0 - 4 * h;
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (kb * 32 + 8 * (j >> 2) + (j & 3) >= n_ok) s[kb][j] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[kb][j]);
    mx = max_across_halves(mx);
    const float m_new = fmaxf(m_run, mx * c2);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
    m_run = m_new;
    // Weights as the sum of two bf16 terms (16 significant bits): this kernel waits for memory, so the second product's
    // second half costs nothing, and the outputs carry their own rounding alone.
    bf16x8 bhi[NG], blo[NG];
    float psum = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[g >> 1][8 * (g & 1) + e], c2, -m_use));
        psum += p;
        bhi[g][e] = (__bf16)p;
        blo[g][e] = (__bf16)(p - (float)bhi[g][e]);
      }
    l_run = fmaf(l_run, alpha, psum);
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] *= alpha;
    }
    if (more) wait_loads<C::NI>();
    else wait_loads<0>();
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      Frag av[NV];
#pragma unroll
      for (int dvb = 0; dvb < NV; ++dvb) {
        const char* vp = vs + (v_at ^ (dvb << 6)) + g * 16 * ROWB;
        av[dvb].s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp));
        av[dvb].s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp + 8 * ROWB));
      }
      if (g == NG - 1) {
        wait_lds();
        if (more) request_tile(k1, pg, a.v, true, v_lds);
      }
#pragma unroll
      for (int dvb = 0; dvb < NV; ++dvb) {
        o[dvb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[dvb].b, bhi[g], o[dvb], 0, 0, 0);
        o[dvb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[dvb].b, blo[g], o[dvb], 0, 0, 0);
      }
    }
  }

  join_waves<D, NW, true, PAGED, C::AREA>(a, it, src, o, m_run, l_run, begin);
}

template <int D, bool PAGED, bool ONCE>
__global__ __launch_bounds__(256, 2) void k_attend_few(PagedAttnLaunch a) {
  const int index = blockIdx.x / a.hkv, kvh = blockIdx.x % a.hkv;
  const Item it = Items<0, false>(a).find(index);
  if (it.s < 0) return;
  attend_few<D, PAGED, 4, ONCE>(a, it, kvh);
}

// ---------------------------------------------------------------------------------------------- many rows
// Eight waves of 32 rows each, one workgroup per compute unit; tiles of keys that the waves share.  K and V tiles travel straight
// into a ring of LDS slots.  Inside a wave the products of the next tile's scores are issued among the weights of the current one,
// so that the matrix unit and the vector unit work at the same time:
//     step t:  S(t+1) = K(t+1) Q^T (matrix)  |  P(t) = 2^(S(t) c - m) (vector);  O^T += V(t)^T P(t)^T (matrix)
// The running maximum is raised only when a row outgrows it by 2^8, which keeps the rescaling of O off the common path: weights
// stay below 256.  A weight is the sum of two bf16 terms (16 significant bits), each multiplied by V, as in attend_few: a token's
// error is that of its output's rounding, whatever batch it comes in.  One term (half a step, 2^-8 relative) would take two matrix
// products per key instead of three, 4.3 ms instead of 5.7 for 16 prompts of 4096 tokens, 64 heads over 8, but doubles the squared
// error of the outputs (2.2e-3 of their norm instead of 1.6e-3).  The sum is that of the unrounded weights, in float32.
// KG = 1: 256 rows and 64 keys a step, tiles requested two steps ahead.  KG = 2, where 256 rows at a time would leave compute
// units idle or the longest tile's chain of steps would last: 128 rows, and 128 keys a step of which either half of the waves
// takes 64; the halves meet through LDS at the end.
// Bound by the power limit.  One prompt of 24000 tokens, 32 heads over 8: d = 128 824 TFLOP/s of the operator, 1240 of the matrix
// unit; d = 64 664; 10 of 1024 tokens 520: a workgroup's start and end (lengths, first K tile, queries, output rows) take as long as
// three steps of a mean of 8.5.  Measured with one-term weights: two workgroups of 128 rows and four waves per compute unit, whose starts
// and ends overlap, read K and V twice as often: 16 x 1024 217 -> 203 us, but 23 of 580 to 2999 tokens 813 -> 817, 1 x 8000 498 -> 514,
// chunks over pages up to 8 % slower.
template <int D, int KG>
struct WideCfg {
  static constexpr int NW = 8, RG = NW / KG, BK = 64, BKT = BK * KG;    // waves, row groups, keys per wave and per step
  static constexpr int NSLOT = KG == 2 && D == 128 ? 2 : 3;             // K is requested NSLOT tiles ahead, V one less
  static constexpr int ROWB = D * 2, CPR = ROWB / 16, RPI = 1024 / ROWB;
  static constexpr int TILE = BKT * ROWB, NI = TILE / 1024 / NW;        // a wave requests 8 KG rows of a tile, which lie in one page
  static constexpr int MERGE = 64 * (D / 2 + 2) * 4;                    // one wave's outputs, maxima and sums
  static constexpr int LDS_BYTES = 2 * NSLOT * TILE;
  static constexpr int AHEAD = NSLOT == 3 ? 2 * NI : 0;                 // requests that may be on their way at a step's end
  static_assert(NI * RPI == 8 * KG, "rows of a wave");
};

template <bool M>
struct Masked {
  static constexpr bool value = M;
};

template <int D, bool PAGED, int KG>
__device__ __forceinline__ void attend_wide(const PagedAttnLaunch& a, const Item& it, int kvh) {
  using C = WideCfg<D, KG>;
  using F = FewCfg<D, 8>;  // the swizzles
  constexpr int ND = D / 16, NV = D / 32, ROWB = C::ROWB, CPR = C::CPR, NI = C::NI, TILE = C::TILE, NSLOT = C::NSLOT;
  constexpr int BK = C::BK, BKT = C::BKT, ROWS = wide_rows<KG>();
  constexpr float TAU = 8.f;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  // K(j) in slot j % NSLOT at smem + slot * TILE, V(j) at smem + (NSLOT + slot) * TILE
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int rw = lane & 31, h = lane >> 5, rg = wave % C::RG, key_g = wave / C::RG * BK;
  const int group = a.hq / a.hkv, n_rows = it.q.n * group, r0 = it.tile * ROWS + rg * 32;
  const int pos0 = it.q.len - it.q.n;
  auto slots_seen = [&](int r) { return min(pos0 + min(r, n_rows - 1) / group + 1, it.q.len); };  // keys that row r sees

  const int begin = it.chunk * it.c;
  const int end = min(slots_seen(it.tile * ROWS + ROWS - 1), begin + it.c);
  const int n_tiles = max((end - begin + BKT - 1) / BKT, 0);
  const bool has_rows = r0 < n_rows;
  // tiles whose keys of this wave the first row sees all, and tiles of which the last row sees any
  const int seen_first = has_rows ? min(slots_seen(r0), end) - begin - key_g : 0;
  const int seen_last = has_rows ? min(slots_seen(r0 + 31), end) - begin - key_g : 0;
  const int n_full = max(seen_first + BKT - BK, 0) / BKT, n_any = max(seen_last + BKT - 1, 0) / BKT;

  bf16x8 bq[ND];
  int key_end;  // one past the last key that counts for this lane's row, in the wave's keys

  // ---- requests: rows 8 KG wave .. 8 KG wave + 8 KG - 1 of every tile.  The pages of 64 tiles are looked up at once, one per
  // lane.
  const KvSource<PAGED> src{a, it.s, kvh, it.q.first, it.q.len - 1};
  const uint32_t smem_at = (uint32_t)(size_t)(const __attribute__((address_space(3))) char*)smem;
  const uint32_t wave_rows = uniform(smem_at + NI * wave * 1024);
  const int lrow = lane / CPR, key0 = begin + 8 * KG * wave;
  // chunks of a request's rows in their swizzled places: of K's request i, other by an exclusive or; of V the same in all
  const uint32_t k_chunk = (uint32_t)((lane % CPR) ^ F::kswz(8 * KG * wave + lrow)) * 16;
  const uint32_t v_chunk = (uint32_t)((lane % CPR) ^ F::vswz(lrow)) * 16;
  int pages = 0;
  auto look_up = [&](int j) {
    if constexpr (PAGED) {
      const int key = min(key0 + (j + lane) * BKT, src.last);
      pages = min(max(a.b.table[(long long)it.s * a.b.max_pages + (key >> a.b.page_log2)], 0), a.b.n_pages - 1);
    }
  };
  auto page_of = [&](int j) { return PAGED ? __builtin_amdgcn_readlane(pages, j & 63) : 0; };
  auto request_rows = [&](const RowsArg& rows, bool is_v, int j, int page, uint32_t slot) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = key0 + j * BKT + i * C::RPI, lim = max(src.last - key, 0);
      const uint32_t chunk = is_v ? v_chunk : k_chunk ^ (uint32_t)(F::kswz(i * C::RPI) * 16);
      request(rows.p + src.at(rows, min(key, src.last), page), (uint32_t)min(lrow, lim) * ((uint32_t)rows.rs & 0xFFFFFFu) + chunk,
              wave_rows + slot + i * 1024);
    }
  };
  // Past the last tile that one is requested again, into a slot that nobody reads any more: unmasked steps request without a
  // branch, and have the same number on their way.
  auto request_k = [&](int j, int page, uint32_t slot) { request_rows(a.k, false, min(j, n_tiles - 1), page, slot); };
  auto request_v = [&](int j, int page, uint32_t slot) { request_rows(a.v, true, min(j, n_tiles - 1), page, NSLOT * TILE + slot); };

  // ---- fragments: LDS addresses of the first one in slot 0; the others differ in bits that an exclusive or turns (slots, and the
  // ring, start at multiples of 1 KB).  Made where they are used: kept, they would cost registers that the two sets of scores need.
  const uint32_t k_at = smem_at + key_g * ROWB + (uint32_t)(rw * ROWB + ((h ^ F::kswz(rw)) * 16));
  uint32_t v_at;
  {
    const int i16 = lane & 15, q2 = (lane >> 4) & 1, vrow = 4 * h + (i16 >> 2);
    v_at = smem_at + key_g * ROWB + NSLOT * TILE + (uint32_t)(vrow * ROWB + (((2 * q2 + ((i16 & 3) >> 1)) ^ F::vswz(vrow)) * 16) + 8 * (i16 & 1));
  }
  auto kfrags = [&](uint32_t slot, int kb, bf16x8 (&ak)[ND]) {
    uint32_t at = k_at + slot;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int dc = 0; dc < ND; ++dc) ak[dc] = *lds_at<bf16x8>((at ^ (dc << 5)) + kb * 32 * ROWB);
  };

  f32x16 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;
  const float c2 = a.scale * kLog2e;

  auto lift = [&](float mx) {
    if (__any(mx > m_ref + TAU)) {
      const float m_new = fmaxf(m_ref, mx);
      const float al = __builtin_amdgcn_exp2f(m_ref - (m_new == -INFINITY ? 0.f : m_new));
      if (__any(m_ref != -INFINITY)) {  // not the first tile
        l_run *= al;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] *= al;
      }
      m_ref = m_new;
    }
  };
  auto row_max = [&](const f32x16 (&s)[2]) {
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[kb][j]);
    return max_across_halves(mx) * c2;
  };
  auto mask = [&](int tile, f32x16 (&s)[2]) {
    int n_ok = key_end - tile * BKT - 4 * h;  // keys of the tile that count, less the lane's first: made here
    asm volatile("" : "+v"(n_ok));
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (kb * 32 + 8 * (j >> 2) + (j & 3) >= n_ok) s[kb][j] = -INFINITY;
  };
  auto scores = [&](uint32_t ks, f32x16 (&s)[2]) {
    bf16x8 ak0[ND], ak1[ND];
    kfrags(ks, 0, ak0);
    kfrags(ks, 1, ak1);
#pragma unroll
    for (int j = 0; j < 16; ++j) { s[0][j] = 0.f; s[1][j] = 0.f; }
#pragma unroll
    for (int dc = 0; dc < ND; ++dc) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak0[dc], bq[dc], s[0], 0, 0, 0);
#pragma unroll
    for (int dc = 0; dc < ND; ++dc) s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak1[dc], bq[dc], s[1], 0, 0, 0);
  };

  // K(0) and the query rows together, the other tiles when they are here: the wait for the rows, which are loaded into
  // registers, would be one for every request ahead of their use.
  int page_k = 0, page_v = 0;
  if (n_tiles > 0) {
    look_up(0);
    page_k = page_of(0);
    request_k(0, page_k, 0);
  }
  const int r = min(r0 + rw, n_rows - 1);
  key_end = min(slots_seen(r), end) - begin - key_g;
  {
    const char* qp = a.q.p + (kvh * group + r % group) * a.q.hs + (long long)(it.q.first + r / group) * a.q.rs + h * 16;
#pragma unroll
    for (int dc = 0; dc < ND; ++dc) bq[dc] = *reinterpret_cast<const bf16x8*>(qp + dc * 32);
  }

#pragma unroll
  for (int dc = 0; dc < ND; ++dc) asm volatile("" : "+v"(bq[dc]));

  if (n_tiles > 0) {
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    request_v(0, page_k, 0);
    if (n_tiles > 1) {
      page_k = page_of(1);
      request_k(1, page_k, TILE);
    }
    if (NSLOT == 3 && n_tiles > 1) request_v(1, page_k, TILE);
    if (NSLOT == 3 && n_tiles > 2) {
      page_k = page_of(2);
      request_k(2, page_k, 2 * TILE);
    }
    f32x16 sA[2], sB[2];
    scores(0, sA);
    // V(0) and K(1) for step 0; K(0) has been read by every wave before step 0 requests its slot's next tile
    if (NSLOT == 3 && n_tiles > 2) wait_loads<2 * NI>();
    else if (NSLOT == 3 && n_tiles > 1) wait_loads<NI>();
    else wait_loads<0>();
    wait_lds();
    __builtin_amdgcn_s_barrier();

    // Every wave walks all tiles: it requests its rows and meets the barriers, whatever it computes.  Step t requests K(t + NSLOT)
    // into the slot of K(t), which step t - 1 has read, and V(t + NSLOT - 1) into that of V(t - 1).
    int tile = 0;
    uint32_t s0 = 0, s1 = TILE, s2 = 2 * TILE;  // slots of tiles t, t + 1 and, of three, t + 2
    auto ahead_k = [&]() {
      const int j = tile + NSLOT;
      page_v = page_k;
      if (PAGED && (j & 63) == 0 && j < n_tiles) look_up(j);
      page_k = page_of(min(j, n_tiles - 1));
      request_k(j, page_k, s0);
    };
    auto ahead_v = [&]() { request_v(tile + NSLOT - 1, page_v, NSLOT == 3 ? s2 : s1); };
    auto next = [&]() {  // all that the next step reads has landed: of three slots it was requested one step ago
      wait_lds();
      __builtin_amdgcn_s_barrier();
      const uint32_t s = s0;
      s0 = s1;
      if constexpr (NSLOT == 3) {
        s1 = s2;
        s2 = s;
      } else {
        s1 = s;
      }
      ++tile;
    };
    // S(tile) is in sc, its row maximum in mx; S(tile + 1) and its maximum take their places.  The order of the instructions is
    // fixed (a wave issues in order, and the two waves of a SIMD are in step after every barrier): a product every 32 cycles,
    // between them the weights (a pair takes the vector unit for two products), the fragment reads eight products ahead of their
    // use, and the maximum of the new scores under the last products.
    float mx = 0.f;
    auto step = [&](f32x16 (&sc)[2], f32x16 (&sn)[2], auto kind) {
      constexpr bool masked = kind.value;
      constexpr int NS = 2 * ND, NP = 8 * NV, RV = 4;  // products of S and of O, fragments of V that are here
      constexpr int FIRST = 2, UNDER_S = 6, LATE = 16 - FIRST - UNDER_S;  // pairs of weights made ahead of the products, under S, under O
      static_assert(FIRST + UNDER_S >= 8, "the weights of two groups of 16 keys are here before O's first product, the others in time");
      uint32_t ks = k_at + s1, vs = v_at + s0;
      asm volatile("" : "+v"(ks), "+v"(vs));
      bf16x8 ak[ND];
      Frag hi[4], lo[4];
      Frag va[RV];
      float psum = 0.f;
      auto k_read = [&](int i) {
        ak[i % ND] = *lds_at<bf16x8>((ks ^ ((i % ND) << 5)) + (i / ND) * 32 * ROWB);
      };
      auto v_read = [&](int j) {
        const uint32_t vp = (vs ^ ((j % NV) << 6)) + (j / NV) * 16 * ROWB;
        va[j % RV].s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(vp));
        va[j % RV].s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(vp + 8 * ROWB));
      };
#pragma unroll
      for (int i = 0; i < ND; ++i) k_read(i);
      lift(mx);
      const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
      auto pair = [&](int k) {  // weights 2 k and 2 k + 1 of the lane
        const int g = k / 4, e = 2 * (k % 4);
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[g >> 1][8 * (g & 1) + e], c2, -m_use));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[g >> 1][8 * (g & 1) + e + 1], c2, -m_use));
        const bf16x2 first = {(__bf16)p0, (__bf16)p1};
        uint32_t both = __builtin_bit_cast(uint32_t, first);
        asm("" : "+v"(both));  // taken apart as they lie: the compiler would convert them again, one by one
        const bf16x2 second = {(__bf16)(p0 - bf16_lo(both)), (__bf16)(p1 - bf16_hi(both))};
        hi[g].u[e / 2] = both;
        lo[g].u[e / 2] = __builtin_bit_cast(uint32_t, second);
        psum += p0 + p1;
        asm volatile("" : : "v"(psum));  // here, not where the sum is used
      };
#pragma unroll
      for (int k = 0; k < FIRST; ++k) pair(k);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        if (i % ND == 0) {
#pragma unroll
          for (int j = 0; j < 16; ++j) sn[i / ND][j] = 0.f;
        }
        sn[i / ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[i % ND], bq[i % ND], sn[i / ND], 0, 0, 0);
        if (i < ND) k_read(i + ND);
        else if (i - (NS - RV) >= 0) v_read(i - (NS - RV));
        if ((i + 1) * UNDER_S / NS > i * UNDER_S / NS) pair(FIRST + i * UNDER_S / NS);
        if (i == NS / 4 && !masked) ahead_k();
        if (i == NS / 2 && !masked) ahead_v();
        __builtin_amdgcn_sched_barrier(0);
      }
      float top = -INFINITY;  // of the new scores
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        const int f = j / 2, g = f / NV;  // fragment of V, its 16 keys
        o[f % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[f % RV].b, j % 2 == 0 ? hi[g].b : lo[g].b, o[f % NV], 0, 0, 0);
        if (j % 2 != 0 && f + RV < 4 * NV) v_read(f + RV);
        constexpr int EARLY = NP / 2, MAXES = (32 / (NP - EARLY) + 2) / 2 * 2;  // maxima: one instruction takes two
        if (j < EARLY) {
          if ((j + 1) * LATE / EARLY > j * LATE / EARLY) pair(FIRST + UNDER_S + j * LATE / EARLY);
        } else if constexpr (!masked) {
#pragma unroll
          for (int k = 0; k < MAXES; ++k) {
            const int v = (j - EARLY) * MAXES + k;
            if (v < 32) top = fmaxf(top, sn[v / 16][v % 16]);
          }
          asm volatile("" : : "v"(top));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += psum;
      if constexpr (!masked) {
        mx = max_across_halves(top) * c2;
        wait_loads<C::AHEAD>();
        next();
      }
    };
    if (n_full > 1) mx = row_max(sA);
    while (tile + 1 < n_full) {
      step(sA, sB, Masked<false>{});
      step(sB, sA, Masked<false>{});
    }
    // the masked ones behind them, and an odd unmasked one; then the other waves' tiles
    while (tile < n_tiles) {
      const bool more_k = tile + NSLOT < n_tiles, more_v = tile + NSLOT - 1 < n_tiles;
      if (more_k) ahead_k();
      else page_v = page_k;
      if (more_v) ahead_v();
      if (tile < n_any) {
        mask(tile, sA);
        mx = row_max(sA);
        step(sA, sB, Masked<true>{});
        sA[0] = sB[0];
        sA[1] = sB[1];
      }
      if (NSLOT == 3 && more_k) wait_loads<2 * NI>();
      else if (NSLOT == 3 && more_v) wait_loads<NI>();
      else wait_loads<0>();
      next();
    }
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();  // the ring is free for the output rows once nobody's requests are on their way
  }

  if constexpr (KG == 2) {
    // the second key group hands its running maximum, row sum and outputs to the first (element e of lane l at word e * 64 + l),
    // which takes both to the common maximum
    float* mg = reinterpret_cast<float*>(smem + rg * C::MERGE) + lane;
    if (key_g > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) mg[(i * 16 + j) * 64] = o[i][j];
      mg[NV * 16 * 64] = m_ref;
      mg[(NV * 16 + 1) * 64] = l_run;
    }
    __syncthreads();
    if (key_g > 0) return;
    const float m1 = mg[NV * 16 * 64], l1 = mg[(NV * 16 + 1) * 64];
    const float m_new = fmaxf(m_ref, m1), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float a0 = __builtin_amdgcn_exp2f(m_ref - m_use), a1 = __builtin_amdgcn_exp2f(m1 - m_use);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = o[i][j] * a0 + mg[(i * 16 + j) * 64] * a1;
    l_run = l_run * a0 + l1 * a1;
    m_ref = m_new;
  }
  if (!has_rows) return;
  int rw_end = lane & 31;
  asm volatile("" : "+v"(rw_end));  // the row again: kept, it would cost registers
  const int n_valid = min(32, n_rows - r0);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum += fabsf(o[i][j]);
  const float l_tot = sum_across_halves(l_run), inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const unsigned long long odd2 = __ballot(l_tot == l_tot && !(sum < INFINITY));
  uint32_t odd = (uint32_t)odd2 | (uint32_t)(odd2 >> 32);  // rows to be computed again
  odd &= n_valid < 32 ? (1u << n_valid) - 1 : ~0u;
  const float lse2 = m_ref + __log2f(l_tot);
  auto again = [&]() {  // behind the wave's own stores
    for (; odd != 0; odd &= odd - 1) {
      const int row = __ffs(odd) - 1;
      attend_row<true, D, PAGED>(a, it, src, r0 + row, begin, rg * 32 + row);
    }
  };
  constexpr int TURN = KG == 2 ? C::MERGE : C::LDS_BYTES / 8;
  char* turn = smem + rg * TURN;  // of this wave alone: the ring is free since the last barrier
  if (it.n_chunks > 1) {
    const long long at = part_row(a, it, it.chunk, kvh) + rg * 32;
    store_rows_via_lds<D, 2>(o, inv, a.part_o + at * D, n_valid, turn, lane);
    if (h == 0 && rw_end < n_valid) a.part_lse[at + rw_end] = lse2;
    again();
    return;
  }
  constexpr int RS = ROWB + 16;
  static_assert(32 * RS <= TURN && 16 * (D * 4 + 16) <= TURN, "rows are turned in the ring");
#pragma unroll
  for (int dvb = 0; dvb < NV; ++dvb)
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4) {
      const bf16x4 y = {(__bf16)(o[dvb][4 * j4] * inv), (__bf16)(o[dvb][4 * j4 + 1] * inv), (__bf16)(o[dvb][4 * j4 + 2] * inv),
                        (__bf16)(o[dvb][4 * j4 + 3] * inv)};
      *reinterpret_cast<bf16x4*>(turn + rw_end * RS + (dvb * 32 + 8 * j4 + 4 * h) * 2) = y;
    }
  const int r_end = min(r0 + rw_end, n_rows - 1);
  const int head = kvh * group + r_end % group, tok = it.q.first + r_end / group, pos = lane % CPR;
  const long long to = head * a.out.hs + tok * a.out.rs;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 32 / C::RPI; ++i) {
    const int row = i * C::RPI + lrow;
    const u32x4 y = *reinterpret_cast<const u32x4*>(turn + row * RS + pos * 16);
    const uint32_t lo = __shfl((uint32_t)to, row), hi = __shfl((uint32_t)((unsigned long long)to >> 32), row);
    if (row < n_valid) *reinterpret_cast<u32x4*>(a.out.p + (long long)((unsigned long long)hi << 32 | lo) + pos * 16) = y;
  }
  if (h == 0 && rw_end < n_valid && a.lse != nullptr) a.lse[(long long)head * a.b.n_rows + tok] = lse2 * kLn2;
  again();
}

// Batches in which some sequences have many rows: wide tiles for those, 32 rows shared by the eight waves for the others.
template <int D, bool PAGED, int KG>
__global__ __launch_bounds__(512, 2) void k_attend_mixed(PagedAttnLaunch a) {
  const int index = blockIdx.x / a.hkv, kvh = blockIdx.x % a.hkv;
  const Item it = Items<KG, false>(a).find(index);
  if (it.s < 0) return;
  if (it.wide) attend_wide<D, PAGED, KG>(a, it, kvh);
  else attend_few<D, PAGED, 8, true>(a, it, kvh);
}

// ---------------------------------------------------------------------------------------------- launches
template <int D, int KG>
constexpr int mixed_lds() {
  return WideCfg<D, KG>::LDS_BYTES > FewCfg<D, 8>::LDS_BYTES ? WideCfg<D, KG>::LDS_BYTES : FewCfg<D, 8>::LDS_BYTES;
}

template <int D, bool PAGED>
hipError_t run_bf16(const PagedAttnLaunch& a, const PagedAttnPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)(p.max_items * a.hkv));
  if (p.kg == 2) hipLaunchKernelGGL((k_attend_mixed<D, PAGED, 2>), grid, dim3(512), (mixed_lds<D, 2>()), s, a);
  else if (p.kg == 1) hipLaunchKernelGGL((k_attend_mixed<D, PAGED, 1>), grid, dim3(512), (mixed_lds<D, 1>()), s, a);
  else if (p.once) hipLaunchKernelGGL((k_attend_few<D, PAGED, true>), grid, dim3(256), (FewCfg<D, 4>::LDS_BYTES), s, a);
  else hipLaunchKernelGGL((k_attend_few<D, PAGED, false>), grid, dim3(256), (FewCfg<D, 4>::LDS_BYTES), s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.joins) return e;
  return launch_join<D, true>(a, p, s);
}

template <int D, bool PAGED>
hipError_t raise_limit() {
  auto raise = [](const void* f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
  hipError_t e = raise(reinterpret_cast<const void*>(&k_attend_few<D, PAGED, false>), FewCfg<D, 4>::LDS_BYTES);
  if (e == hipSuccess) e = raise(reinterpret_cast<const void*>(&k_attend_few<D, PAGED, true>), FewCfg<D, 4>::LDS_BYTES);
  if (e == hipSuccess) e = raise(reinterpret_cast<const void*>(&k_attend_mixed<D, PAGED, 1>), mixed_lds<D, 1>());
  return e != hipSuccess ? e : raise(reinterpret_cast<const void*>(&k_attend_mixed<D, PAGED, 2>), mixed_lds<D, 2>());
}

}  // namespace

hipError_t paged_attn_raise_limits() {
  const hipError_t all[] = {raise_limit<128, true>(), raise_limit<128, false>(), raise_limit<64, true>(), raise_limit<64, false>(),
                            paged_attn_f32_raise_limits()};
  for (hipError_t e : all)
    if (e != hipSuccess) return e;
  return hipSuccess;
}

hipError_t launch_paged_attn(const PagedAttnLaunch& a, hipStream_t s) {
  const hipError_t e = attn_prepare_device();
  if (e != hipSuccess) return e;
  const PagedAttnPlan p = paged_attn_plan(a.dtype, a.d, a.hq, a.hkv, a.b.n_seq, a.b.n_rows, a.b.max_new, a.b.max_len, a.paged != 0);
  if (a.dtype != SAMKV_BF16) return launch_paged_attn_f32(a, p, s);
  if (a.paged) return a.d == 128 ? run_bf16<128, true>(a, p, s) : run_bf16<64, true>(a, p, s);
  return a.d == 128 ? run_bf16<128, false>(a, p, s) : run_bf16<64, false>(a, p, s);
}

}  // namespace samkv
