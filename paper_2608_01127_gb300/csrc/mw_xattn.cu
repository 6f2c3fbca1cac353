// Cross attention of few query rows a head on CUDA cores: single new tokens against
// an encoder's states, of which a sample has some number valid.
//
//   s_ij = scale <q_i, k_j> for j < len; LSE_i = ln sum_j exp(s_ij);
//   P = exp(s - LSE), O = P V; len = 0: O = 0, LSE = -inf
//
// Bound by reading K and V once.  L lanes hold one key's d channels, 8 each, so that
// a warp has 32 / L keys at once and U times as many in flight; a dot product is 4
// packed FMAs and log2(L) shuffles.  The keys of a head are shared by the warps of
// up to 16 CTAs, one thread-block cluster, which join their running maxima, sums and
// outputs through distributed shared memory: one launch, no workspace.
#include <cooperative_groups.h>

#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 8;

struct Piece {
  float2 v[4];  // 8 channels
};

__device__ __forceinline__ Piece widen(uint4 a) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  Piece p;
#pragma unroll
  for (int k = 0; k < 4; ++k) p.v[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
  return p;
}

// 16 bytes that are read once
__device__ __forceinline__ uint4 load_once(const __nv_bfloat16* p, bool there) {
  uint4 a = make_uint4(0u, 0u, 0u, 0u);
  if (there)
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w)
                 : "l"(p));
  return a;
}

// The weight of a part whose maximum is m once the whole's is top (-inf: no keys).
__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : ex2_approx(m - top); }

// What a CTA leaves for the cluster: per row its maximum, sum and output.
template <int L, int R>
struct Part {
  float m[R], l[R], o[R][L * 8];
};

// Cluster: a head's R (or fewer) rows; CTA: a share of its keys.
template <int L, int R>
__global__ void __launch_bounds__(kWarps * 32) xattn_few_kernel(const XattnParams p) {
  constexpr int G = 32 / L;            // keys of a warp at once
  constexpr int U = R <= 4 ? 4 : 2;    // and in flight
  __shared__ Part<L, R> of_warp[kWarps];
  __shared__ Part<L, R> whole;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = 8 * (lane % L);
  const bool in = c < p.d;
  const int bh = blockIdx.x / ranks;
  pdl_wait();
  pdl_trigger();
  int len = p.S;
  if (p.kv_len) len = min(max(p.kv_len[bh / p.heads], 0), p.S);
  const int share = (len + ranks - 1) / ranks;
  const int j_end = min(len, (rank + 1) * share);
  float2 q[R][4], acc[R][4];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint4 raw = in && r < p.M ? *reinterpret_cast<const uint4*>(p.q + (static_cast<size_t>(bh) * p.M + r) * p.d + c)
                                    : make_uint4(0u, 0u, 0u, 0u);
    const Piece x = widen(raw);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      q[r][k] = make_float2(x.v[k].x * p.scale_log2, x.v[k].y * p.scale_log2);
      acc[r][k] = make_float2(0.f, 0.f);
    }
    m[r] = -INFINITY;
    l[r] = 0.f;
  }
  for (int j0 = rank * share + warp * G * U; j0 < j_end; j0 += kWarps * G * U) {
    uint4 k16[U], v16[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * G + lane / L;
      const size_t at = (static_cast<size_t>(bh) * p.S + j) * p.d + c;
      k16[u] = load_once(p.k + at, in && j < j_end);
      v16[u] = load_once(p.v + at, in && j < j_end);
    }
    float s[U][R];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const Piece k8 = widen(k16[u]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float2 x = mul2(q[r][0], k8.v[0]);
#pragma unroll
        for (int k = 1; k < 4; ++k) x = fma2(q[r][k], k8.v[k], x);
        s[u][r] = x.x + x.y;
      }
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < R; ++r) s[u][r] += __shfl_xor_sync(0xffffffffu, s[u][r], o);
    // (a lane's keys run up: the first is valid where any is)
    const int there = (j_end - j0 - lane / L + G - 1) / G;  // of its U
    if (there > 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = fmaxf(m[r], s[0][r]);
#pragma unroll
        for (int u = 1; u < U; ++u)
          if (u < there) top = fmaxf(top, s[u][r]);
        const float keep = ex2_approx(m[r] - top);
        m[r] = top;
        l[r] *= keep;
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[r][k] = mul2(acc[r][k], make_float2(keep, keep));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          s[u][r] = u < there ? ex2_approx(s[u][r] - top) : 0.f;
          l[r] += s[u][r];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const Piece v8 = widen(v16[u]);  // (zeros where there is no key)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[r][k] = fma2(make_float2(s[u][r], s[u][r]), v8.v[k], acc[r][k]);
      }
    }
  }
  // join the warp's keys, the CTA's warps, the cluster's CTAs
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[r], o), lo = __shfl_xor_sync(0xffffffffu, l[r], o);
      const float top = fmaxf(m[r], mo);
      const float a = weight(m[r], top), b = weight(mo, top);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = __shfl_xor_sync(0xffffffffu, acc[r][k].x, o), y = __shfl_xor_sync(0xffffffffu, acc[r][k].y, o);
        acc[r][k] = make_float2(acc[r][k].x * a + x * b, acc[r][k].y * a + y * b);
      }
      l[r] = l[r] * a + lo * b;
      m[r] = top;
    }
    if (lane < L) {
#pragma unroll
      for (int k = 0; k < 4; ++k) *reinterpret_cast<float2*>(&of_warp[warp].o[r][c + 2 * k]) = acc[r][k];
      if (lane == 0) of_warp[warp].m[r] = m[r], of_warp[warp].l[r] = l[r];
    }
  }
  __syncthreads();
  const int n = min(R, p.M) * p.d;
  for (int i = threadIdx.x; i < n; i += kWarps * 32) {
    const int r = i / p.d, ch = i - r * p.d;
    float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, of_warp[w].m[r]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float a = weight(of_warp[w].m[r], top);
      sum = fmaf(of_warp[w].l[r], a, sum);
      o = fmaf(of_warp[w].o[r][ch], a, o);
    }
    whole.o[r][ch] = o;
    if (ch == 0) whole.m[r] = top, whole.l[r] = sum;
  }
  cluster.sync();
  for (int i = rank * kWarps * 32 + threadIdx.x; i < n; i += ranks * kWarps * 32) {
    const int r = i / p.d, ch = i - r * p.d;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int k = 0; k < ranks; ++k) top = fmaxf(top, cluster.map_shared_rank(&whole, k)->m[r]);
    for (int k = 0; k < ranks; ++k) {
      const Part<L, R>* other = cluster.map_shared_rank(&whole, k);
      const float a = weight(other->m[r], top);
      sum = fmaf(other->l[r], a, sum);
      o = fmaf(other->o[r][ch], a, o);
    }
    const size_t row = static_cast<size_t>(bh) * p.M + r;
    p.o[row * p.d + ch] = __float2bfloat16(sum > 0.f ? o / sum : 0.f);
    if (p.lse && ch == 0)
      p.lse[row] = sum > 0.f ? (top + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
  }
  cluster.sync();  // shared memory stays until all have read it
}

template <int L, int R>
cudaError_t launch(const XattnParams& p, int dev, cudaStream_t s) {
  // CTAs a head: about two an SM, each with a turn of keys for all its warps at least
  constexpr int kTurn = kWarps * (32 / L) * (R <= 4 ? 4 : 2);
  int ranks = 1;
  while (ranks < 16 && p.BH * ranks * 2 <= 2 * p.sms && p.S > ranks * kTurn) ranks *= 2;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(dev, [] {
    return cudaFuncSetAttribute(xattn_few_kernel<L, R>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(p.BH) * ranks);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl_enabled ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, xattn_few_kernel<L, R>, p);
}

template <int L>
cudaError_t by_rows(const XattnParams& p, int dev, cudaStream_t s) {
  switch (p.M) {
    case 1: return launch<L, 1>(p, dev, s);
    case 2: return launch<L, 2>(p, dev, s);
    case 3: return launch<L, 3>(p, dev, s);
    case 4: return launch<L, 4>(p, dev, s);
    case 5: return launch<L, 5>(p, dev, s);
    case 6: return launch<L, 6>(p, dev, s);
    default: return launch<L, 8>(p, dev, s);
  }
}

}  // namespace

cudaError_t launch_xattn_few(const XattnParams& p, int dev, cudaStream_t s) {
  return p.d == 64 ? by_rows<8>(p, dev, s) : by_rows<16>(p, dev, s);
}

}  // namespace mw
