// Attention of the rows of a batch of sequences over packed prompts (samkv_prefill_attn) or over pages (samkv_paged_attn):
// the row at slot p of its sequence sees slots 0..p.
// One wave per (row, query head): a lane scores one key of 64, the wave's maximum and sum run along, and every lane then
// adds the weighted values of its own channels.
#include "attn_common.hpp"
#include "paged.hpp"

namespace samkv {
namespace {

template <bool BF16>
__device__ __forceinline__ float element(const char* row, int c) {
  if constexpr (BF16) return (float)reinterpret_cast<const __bf16*>(row)[c];
  else return reinterpret_cast<const float*>(row)[c];
}

template <bool BF16, int D, bool PAGED>
__global__ __launch_bounds__(256) void k_paged_attn(PagedAttnLaunch a) {
  constexpr int CPL = D / 64;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y;
  if (row >= a.b.n_rows) return;
  const int s = seq_of_row(a.b, row, lane);
  if (s >= a.b.n_seq) return;
  const SeqSpan q = seq_span(a.b, s);
  const int t = row - q.first;
  if (t < 0 || t >= q.n) return;
  const int n_keys = q.len - q.n + t + 1, kvh = head / (a.hq / a.hkv);
  auto at = [&](const RowsArg& r, int key) {
    if constexpr (PAGED) {
      const int page = min(max(a.b.table[(long long)s * a.b.max_pages + (key >> a.b.page_log2)], 0), a.b.n_pages - 1);
      return r.p + ((long long)page * a.hkv + kvh) * r.hs + (key & ((1 << a.b.page_log2) - 1)) * r.rs;
    } else {
      return r.p + kvh * r.hs + (q.first + key) * r.rs;
    }
  };
  const char* qr = a.q.p + head * a.q.hs + row * a.q.rs;
  float m = -INFINITY, l = 0.f, o[CPL] = {};
  for (int k0 = 0; k0 < n_keys; k0 += 64) {
    float x = -INFINITY;
    if (k0 + lane < n_keys) {
      const char* kr = at(a.k, k0 + lane);
      float dot = 0.f;
      for (int c = 0; c < D; ++c) dot = fmaf(element<BF16>(qr, c), element<BF16>(kr, c), dot);
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
    for (int j = 0; j < min(64, n_keys - k0); ++j) {
      const float w = __shfl(p, j);
      const char* vr = at(a.v, k0 + j);
      for (int e = 0; e < CPL; ++e) o[e] = fmaf(w, element<BF16>(vr, lane + 64 * e), o[e]);
    }
  }
  char* out = a.out.p + head * a.out.hs + row * a.out.rs;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int e = 0; e < CPL; ++e) {
    if constexpr (BF16) reinterpret_cast<__bf16*>(out)[lane + 64 * e] = (__bf16)(o[e] * inv);
    else reinterpret_cast<float*>(out)[lane + 64 * e] = o[e] * inv;
  }
  if (a.lse != nullptr && lane == 0) a.lse[(long long)head * a.b.n_rows + row] = m + logf(l);
}

template <bool BF16, int D>
hipError_t run(const PagedAttnLaunch& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.b.n_rows + 3) / 4), (unsigned)a.hq);
  if (a.paged) hipLaunchKernelGGL((k_paged_attn<BF16, D, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_paged_attn<BF16, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

size_t paged_attn_ws_bytes(int, int, int, int, int, int, int, int) { return 0; }

hipError_t launch_paged_attn(const PagedAttnLaunch& a, hipStream_t s) {
  if (a.dtype == SAMKV_BF16) return a.d == 128 ? run<true, 128>(a, s) : run<true, 64>(a, s);
  return a.d == 128 ? run<false, 128>(a, s) : run<false, 64>(a, s);
}

}  // namespace samkv
