// Attention over packed prompts and pages (paged_attn.hip: definitions), float32.
//
// A workgroup is four waves that share a tile of 32 rows; wave w takes the key tiles w, w + 4, ... of 32 keys of its chunk.
// Products are v_mfma_f32_32x32x2_f32, S^T = K Q^T and O^T += V^T P^T as in attn_f32.hip: 64 cycles of the matrix unit for an
// operand register of each side, so that K and V come straight from memory into registers, K in 16-byte pieces of a row, V a
// value per lane (128 bytes of two rows per request), requested 8 pieces and 32 values ahead.
// Many rows: bound by the float32 matrix rate (a large library product: 154 TFLOP/s), 93 to 120 TFLOP/s.  Single tokens: bound
// by HBM, 5.3 TB/s for 64 sequences x 4096 keys; small batches by latency (4 x 64 to 256 tokens, 8 heads over 2, d = 64: 10 us).
#include "paged_attn.hpp"

namespace samkv {
namespace {

constexpr int NW = 4;

template <int D, bool PAGED>
__device__ __forceinline__ void attend_f32(const PagedAttnLaunch& a, const Item& it, int kvh) {
  constexpr int NV = D / 32, NI = D / 8, NKX = 8, NVX = 32;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int rw = lane & 31, h = lane >> 5;
  const int group = a.hq / a.hkv, n_rows = it.q.n * group, r0 = it.tile * 32;
  const int pos0 = it.q.len - it.q.n;
  const int r = min(r0 + rw, n_rows - 1), t = r / group;
  const int seen_first = pos0 + r0 / group + 1, t_last = min(r0 + 31, n_rows - 1) / group;
  const int begin = it.chunk * it.c, end = min(min(pos0 + t_last + 1, it.q.len), begin + it.c);
  const int key_end = min(pos0 + t + 1, end);
  const KvSource<PAGED> src{a, it.s, kvh, it.q.first, it.q.len - 1};

  f32x4 bq[NI], kx[NKX];
  float vx[NVX];
  {
    const char* qp = a.q.p + (kvh * group + r % group) * a.q.hs + (long long)(it.q.first + t) * a.q.rs + h * 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) bq[i] = *reinterpret_cast<const f32x4*>(qp + i * 32);
  }
  // A tile's keys lie in two groups of 16, each in one page.  Keys past the last one are read as that one (weights of zero).
  struct Tile { int k0, page[2]; };
  auto tile_at = [&](int k0) { return Tile{k0, {src.page_of(k0), src.page_of(k0 + 16)}}; };
  auto base = [&](const RowsArg& rows, const Tile& x, int g) { return rows.p + src.at(rows, min(x.k0 + 16 * g, src.last), x.page[g]); };
  auto limit = [&](const Tile& x, int g) { return max(src.last - x.k0 - 16 * g, 0); };
  auto k_row = [&](const Tile& x) {  // this lane's key
    const char* b0 = base(a.k, x, 0);
    const char* b1 = base(a.k, x, 1);
    return (rw < 16 ? b0 : b1) + (long long)min(rw & 15, rw < 16 ? limit(x, 0) : limit(x, 1)) * a.k.rs + h * 16;
  };
  auto k_piece = [&](const char* row, int i) { return *reinterpret_cast<const f32x4*>(row + i * 32); };
  // V value (j, b): key 8 (j / 4) + 4 h + j % 4, channel 32 b + rw
  auto v_value = [&](const Tile& x, int j, int b) {
    const int g = j >> 3, row = min(8 * (j >> 2 & 1) + 4 * h + (j & 3), limit(x, g));
    return *reinterpret_cast<const float*>(base(a.v, x, g) + ((uint32_t)row * (uint32_t)a.v.rs + rw * 4) + b * 128);
  };

  f32x16 o[NV];
#pragma unroll
  for (int b = 0; b < NV; ++b)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[b][j] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float c2 = (float)((double)a.scale * 1.4426950408889634074);

  int k0 = begin + wave * 32;
  Tile x{}, next{};
  if (k0 < end) {
    x = tile_at(k0);
    const char* kr = k_row(x);
#pragma unroll
    for (int i = 0; i < NKX; ++i) kx[i] = k_piece(kr, i);
  }
  const char* kr = nullptr;
  for (; k0 < end; k0 += 32 * NW) {
    kr = k_row(x);
    next = tile_at(min(k0 + 32 * NW, src.last));  // its first pieces are requested whether or not there is one
    const char* kr_next = k_row(next);
    f32x16 s;
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[i % NKX][e], bq[i][e], s, 0, 0, 0);
      constexpr int F = NI - NKX;
      if (i < F && i % 4 == 3) {
#pragma unroll
        for (int u = 0; u < 4; ++u) kx[(i - 3 + u) % NKX] = k_piece(kr, i - 3 + u + NKX);
      }
      if (i >= F) {  // the last eight pieces: four V values with each, the first NVX of the tile
#pragma unroll
        for (int u = 0; u < 4; ++u) vx[(i - F) * 4 + u] = v_value(x, ((i - F) * 4 + u) / NV, ((i - F) * 4 + u) % NV);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (k0 + 32 > min(seen_first, end)) {
      const int n_ok = key_end - k0 - 4 * h;
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (8 * (j >> 2) + (j & 3) >= n_ok) s[j] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
    mx = max_across_halves(mx);
    const float m_new = fmaxf(m_run, mx * c2);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
    m_run = m_new;
    float psum = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], c2, -m_use));
      psum += s[j];
    }
    l_run = fmaf(l_run, alpha, psum);
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int b = 0; b < NV; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[b][j] *= alpha;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
#pragma unroll
      for (int b = 0; b < NV; ++b) {
        o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(vx[(j * NV + b) % NVX], s[j], o[b], 0, 0, 0);
      }
      if ((j + 1) * NV + NVX <= 16 * NV) {
#pragma unroll
        for (int b = 0; b < NV; ++b) vx[(j * NV + b) % NVX] = v_value(x, (j * NV + b + NVX) / NV, b);
      }
      if (j == 9 || j == 13) {
#pragma unroll
        for (int u = 0; u < 4; ++u) kx[j - 9 + u] = k_piece(kr_next, j - 9 + u);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    x = next;
  }
  join_waves<D, NW, false, PAGED, join_area(D)>(a, it, src, o, m_run, l_run, begin);
}

template <int D, bool PAGED>
__global__ __launch_bounds__(64 * NW, 2) void k_attend_f32(PagedAttnLaunch a) {
  const int index = blockIdx.x / a.hkv, kvh = blockIdx.x % a.hkv;
  const Item it = Items<0, false>(a).find(index);
  if (it.s < 0) return;
  attend_f32<D, PAGED>(a, it, kvh);
}

template <int D, bool PAGED>
hipError_t run_f32(const PagedAttnLaunch& a, const PagedAttnPlan& p, hipStream_t s) {
  hipLaunchKernelGGL((k_attend_f32<D, PAGED>), dim3((unsigned)(p.max_items * a.hkv)), dim3(64 * NW), join_lds(NW, join_area(D)), s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !p.joins ? e : launch_join<D, false>(a, p, s);
}

template <int D, bool PAGED>
hipError_t raise_limit() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_attend_f32<D, PAGED>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             join_lds(NW, join_area(D)));
}

}  // namespace

hipError_t paged_attn_f32_raise_limits() {
  const hipError_t all[] = {raise_limit<128, true>(), raise_limit<128, false>(), raise_limit<64, true>(), raise_limit<64, false>()};
  for (hipError_t e : all)
    if (e != hipSuccess) return e;
  return hipSuccess;
}

hipError_t launch_paged_attn_f32(const PagedAttnLaunch& a, const PagedAttnPlan& p, hipStream_t s) {
  if (a.paged) return a.d == 128 ? run_f32<128, true>(a, p, s) : run_f32<64, true>(a, p, s);
  return a.d == 128 ? run_f32<128, false>(a, p, s) : run_f32<64, false>(a, p, s);
}

}  // namespace samkv
