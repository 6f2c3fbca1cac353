// Cross attention of few query rows a head on CUDA cores: single new tokens against
// an encoder's states, of which a sample has some number valid.
//
//   s_ij = scale <q_i, k_j> for j < len; LSE_i = ln sum_j exp(s_ij);
//   P = exp(s - LSE), O = P V; len = 0: O = 0, LSE = -inf
//
// L lanes hold one key's d channels, 8 each, so that a warp works on 32 / L keys at
// once; a dot product is 8 FMAs and log2(L) shuffles.
#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool there, float (&v)[8]) {
  const uint4 a = there ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(w[k] << 16);
    v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
  }
}

// <a, b> over the channels of L lanes, in each of them.
template <int L>
__device__ __forceinline__ float dot(const float (&a)[8], const float (&b)[8]) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) s = fmaf(a[k], b[k], s);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

__device__ __forceinline__ int valid_keys(const XattnParams& p, int bh) {
  if (!p.kv_len) return p.S;
  const int n = p.kv_len[bh / p.heads];
  return n < 0 ? 0 : n > p.S ? p.S : n;
}

// R rows of one head a block; its warps take the keys in turn.
template <int L, int R>
__global__ void __launch_bounds__(kWarps * 32) xattn_fwd_kernel(const XattnParams p) {
  constexpr int G = 32 / L;  // keys of a warp at once
  __shared__ float sm[kWarps][R], sl[kWarps][R], so[kWarps][R][L * 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane % L, c = 8 * sub;
  const bool in = c < p.d;
  const int blocks = (p.M + R - 1) / R;
  const int bh = blockIdx.x / blocks, m0 = blockIdx.x % blocks * R;
  const int len = valid_keys(p, bh);
  float q[R][8], acc[R][8], m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    load8(p.q + (static_cast<size_t>(bh) * p.M + m0 + r) * p.d + c, in && m0 + r < p.M, q[r]);
#pragma unroll
    for (int k = 0; k < 8; ++k) q[r][k] *= p.scale_log2, acc[r][k] = 0.f;
    m[r] = -INFINITY;
    l[r] = 0.f;
  }
  for (int j0 = warp * G; j0 < len; j0 += kWarps * G) {
    const int j = j0 + lane / L;
    const size_t at = (static_cast<size_t>(bh) * p.S + j) * p.d + c;
    float k8[8], v8[8];
    load8(p.k + at, in && j < len, k8);
    load8(p.v + at, in && j < len, v8);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float s = dot<L>(q[r], k8);
      if (j >= len) continue;
      const float top = fmaxf(m[r], s);
      const float keep = ex2_approx(m[r] - top), w = ex2_approx(s - top);
      m[r] = top;
      l[r] = fmaf(l[r], keep, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[r][k] = fmaf(acc[r][k], keep, w * v8[k]);
    }
  }
  // join the warp's keys, then the warps
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[r], o), lo = __shfl_xor_sync(0xffffffffu, l[r], o);
      const float top = fmaxf(m[r], mo);
      const float a = m[r] == -INFINITY ? 0.f : ex2_approx(m[r] - top);
      const float b = mo == -INFINITY ? 0.f : ex2_approx(mo - top);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        acc[r][k] = acc[r][k] * a + __shfl_xor_sync(0xffffffffu, acc[r][k], o) * b;
      l[r] = l[r] * a + lo * b;
      m[r] = top;
    }
    if (lane < L) {
#pragma unroll
      for (int k = 0; k < 8; ++k) so[warp][r][c + k] = acc[r][k];
      if (sub == 0) sm[warp][r] = m[r], sl[warp][r] = l[r];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * p.d; i += kWarps * 32) {
    const int r = i / p.d, ch = i % p.d;
    if (m0 + r >= p.M) continue;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w][r]);
    for (int w = 0; w < kWarps; ++w) {
      const float a = sm[w][r] == -INFINITY ? 0.f : ex2_approx(sm[w][r] - top);
      sum = fmaf(sl[w][r], a, sum);
      o = fmaf(so[w][r][ch], a, o);
    }
    const size_t row = static_cast<size_t>(bh) * p.M + m0 + r;
    p.o[row * p.d + ch] = __float2bfloat16(sum > 0.f ? o / sum : 0.f);
    if (p.lse && ch == 0)
      p.lse[row] = sum > 0.f ? (top + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
  }
}

template <int L, int R>
cudaError_t fwd(const XattnParams& p, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>(p.BH) * ((p.M + R - 1) / R);
  xattn_fwd_kernel<L, R><<<grid, kWarps * 32, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_xattn_fwd(const XattnParams& p, cudaStream_t s) {
  if (p.M == 1) return p.d == 64 ? fwd<8, 1>(p, s) : fwd<16, 1>(p, s);
  return p.d == 64 ? fwd<8, 4>(p, s) : fwd<16, 4>(p, s);
}

}  // namespace mw
