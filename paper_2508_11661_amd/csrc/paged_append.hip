// samkv_paged_append: rows of new tokens into the pages of their sequences, K and Q turned by the rotary position embedding
// on the way: (x, y) <- (x cos t - y sin t, y cos t + x sin t), t = pos * inv_freq.  A row is LPR 16-byte chunks, one per lane, so
// a row lies within a wave and a chunk gets its partner (the other half of its pairs) from another lane: every value is read once
// and written once, and q_out may be q.
//
// Many tokens: bound by HBM, 2 d e (2 Hkv + Hq) bytes per token read and written.  32 heads over 8, d = 128, bf16: 65536 tokens
// 305 us, 5.28 TB/s, 4096 tokens 21 us (a copy of 2 GiB: 5.8 TB/s; float32, 32768 tokens: 318 us, 5.06).  A workgroup takes four
// tokens of 4 KB / (d e) heads, or walks all their heads (run()).
// Rows as (token, head) pairs in one list, so that few heads keep all lanes busy, lose what they gain: 306 us, 8 heads over 2 of
// 64 channels 107 -> 125 us.  Non-temporal stores take 287 us, but the attention that reads the pages next pays more than that (8
// sequences of 1024 tokens, both: 164 -> 167 us; 64: 1193 -> 1217).
// Few tokens: bound by the launch and the chain of loads prefix sums -> length -> page table (5 us); the rows are requested
// ahead of that chain, and the prefix sums at once.
#include "paged.hpp"

namespace samkv {
namespace {

constexpr int TPB = 4;  // tokens of a workgroup: one per wave while slots and angles are found

template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_paged_append(AppendLaunch a) {
  constexpr int EPL = BF16 ? 8 : 4, LPR = D / EPL, ROWB = D * (BF16 ? 2 : 4);
  constexpr int RPB = 256 / LPR;  // heads that the workgroup takes at a time
  __shared__ float s_cos[TPB][D / 2], s_sin[TPB][D / 2];
  __shared__ long long s_at[TPB];  // byte offset of the token's row for head 0, in K and V pages alike; -1: no slot
  __shared__ int s_row[TPB];       // the token belongs to a sequence
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = threadIdx.x % LPR, rg = threadIdx.x / LPR;
  const int heads = a.hq + 2 * a.hkv, tok0 = blockIdx.x * TPB;
  const int half = a.rot / 2;

  u32x4 x[TPB];
  auto load = [&](int hh) {
    const RowsArg& r = hh < a.hq ? a.q : hh < a.hq + a.hkv ? a.k_new : a.v_new;
    const int head = hh < a.hq ? hh : hh < a.hq + a.hkv ? hh - a.hq : hh - a.hq - a.hkv;
#pragma unroll
    for (int t = 0; t < TPB; ++t) {
      const int tok = min(tok0 + t, a.b.n_rows - 1);
      x[t] = *reinterpret_cast<const u32x4*>(r.p + head * r.hs + tok * r.rs + c * 16);
    }
  };
  int hh = blockIdx.y * RPB + rg;
  load(min(hh, heads - 1));

  {
    const int tok = tok0 + wave;
    const int s = tok < a.b.n_rows ? seq_of_row(a.b, tok, lane) : a.b.n_seq;
    bool in = s < a.b.n_seq;
    int slot = -1;
    long long at = -1;
    if (in) {
      const SeqSpan q = seq_span(a.b, s);
      const int t = tok - q.first;
      in = t >= 0 && t < q.n;
      slot = q.len - q.n + t;
      if (in && slot >= 0) {
        const int page = a.b.table[(long long)s * a.b.max_pages + (slot >> a.b.page_log2)];
        if (page >= 0 && page < a.b.n_pages)
          at = (((long long)page * a.hkv << a.b.page_log2) + (slot & ((1 << a.b.page_log2) - 1))) * ROWB;
      }
    }
    if (lane == 0) {
      s_at[wave] = at;
      s_row[wave] = in;
    }
    if (lane < half && in) {
      // turns = pos * inv_freq / (2 pi), less whole ones, in float64: the angle of position 10^6 is as exact as that of 1
      const int pos = a.positions != nullptr ? a.positions[tok] : max(slot, 0);
      double turns = (double)pos * (double)a.inv_freq[lane] * 0.15915494309189535;
      turns -= rint(turns);
      float sn, cs;
      sincospif((float)(2.0 * turns), &sn, &cs);
      s_cos[wave][lane] = cs;
      s_sin[wave][lane] = sn;
    }
  }
  __syncthreads();

  for (; hh < heads; hh += gridDim.y * RPB) {
    const int kind = hh < a.hq ? 0 : hh < a.hq + a.hkv ? 1 : 2;  // query, key, value
    const int head = kind == 0 ? hh : kind == 1 ? hh - a.hq : hh - a.hq - a.hkv;
#pragma unroll
    for (int t = 0; t < TPB; ++t) {
      u32x4 y = x[t];
      // the chunk that holds the other halves of this one's pairs (half / EPL chunks away; rot is a multiple of 16)
      const int n_half = half / EPL, shift = c < n_half ? n_half : c < 2 * n_half ? -n_half : 0;
      u32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = __shfl(y[e], lane + (a.interleaved ? 0 : shift));
      if (kind < 2 && c * EPL < a.rot) {
        float f[EPL], g[EPL], r[EPL];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (BF16) {
            f[2 * e] = bf16_lo(y[e]); f[2 * e + 1] = bf16_hi(y[e]);
            g[2 * e] = bf16_lo(p[e]); g[2 * e + 1] = bf16_hi(p[e]);
          } else {
            f[e] = __uint_as_float(y[e]);
            g[e] = __uint_as_float(p[e]);
          }
        }
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            const float cs = s_cos[t][(c * EPL + e) / 2], sn = s_sin[t][(c * EPL + e) / 2];
            r[e] = f[e] * cs - f[e + 1] * sn;
            r[e + 1] = f[e + 1] * cs + f[e] * sn;
          }
        } else {
          const int i0 = (c < n_half ? c : c - n_half) * EPL;
          const float sign = c < n_half ? -1.f : 1.f;
#pragma unroll
          for (int e = 0; e < EPL; ++e) r[e] = f[e] * s_cos[t][i0 + e] + sign * (g[e] * s_sin[t][i0 + e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (BF16) {
            const bf16x2 w = {(__bf16)r[2 * e], (__bf16)r[2 * e + 1]};
            y[e] = __builtin_bit_cast(uint32_t, w);
          } else {
            y[e] = __float_as_uint(r[e]);
          }
        }
      }
      char* to;
      if (kind == 0) to = s_row[t] ? a.q_out.p + head * a.q_out.hs + (tok0 + t) * a.q_out.rs : nullptr;
      else to = s_at[t] >= 0 ? (kind == 1 ? a.k : a.v) + s_at[t] + ((long long)head << a.b.page_log2) * ROWB : nullptr;
      if (to != nullptr) *reinterpret_cast<u32x4*>(to + c * 16) = y;
    }
    if (hh + (int)gridDim.y * RPB < heads) load(hh + gridDim.y * RPB);
  }
}

template <bool BF16, int D>
hipError_t run(const AppendLaunch& a, hipStream_t s) {
  constexpr int RPB = 256 / (D / (BF16 ? 8 : 4));
  const int heads = a.hq + 2 * a.hkv, per = (heads + RPB - 1) / RPB;
  const unsigned n = (unsigned)((a.b.n_rows + TPB - 1) / TPB);
  // A workgroup per RPB heads, except where a quarter of its lanes or more would have no head and there are tokens enough: then one
  // walks all heads of its tokens.  Spread / walked, us: 16384 tokens of 32 heads over 8, bf16, d = 128: 78.6 / 84.0, 2048: 10.8 / 12.7;
  // 14 heads over 2 (18 rows for workgroups of 16), float32, d = 64: 16384 tokens 28.1 / 25.7, 6144 13.3 / 12.6, 2048 7.3 / 7.8.
  const bool spread = n < 1024 || 4 * heads >= 3 * per * RPB;
  hipLaunchKernelGGL((k_paged_append<BF16, D>), dim3(n, spread ? per : 1), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const AppendLaunch& a, hipStream_t s) {
  if (a.dtype == SAMKV_BF16) return a.d == 128 ? run<true, 128>(a, s) : run<true, 64>(a, s);
  return a.d == 128 ? run<false, 128>(a, s) : run<false, 64>(a, s);
}

}  // namespace samkv
