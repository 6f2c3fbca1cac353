// Cross attention of few query rows a head: single new tokens against an encoder's
// states, of which a sample has some number valid.
//
//   s_ij = scale <q_i, k_j> for j < len; LSE_i = ln sum_j exp(s_ij);
//   P = exp(s - LSE), O = P V; len = 0: O = 0, LSE = -inf
//
// Bound by reading K and V once.  TMA copies of 64 keys run three stages ahead of four
// warps, which take 16 keys of a stage each: up to 16 rows fit one side of the
// m16n8k16 product of a warp, so that a key costs a few instructions however many rows
// share it (on CUDA cores 8 x 4 heads of 128, 8192 keys took 35 us with one row and 133
// with eight; tcgen05 with its 128 rows 40 us, one warp's softmax a key tile).  The
// keys of a head are shared by up to 16 CTAs, one thread-block cluster, which join
// their maxima, sums and outputs through distributed shared memory: one launch, no
// workspace.  Measured: 8 x 20 rows on 8 x 4 heads of 128, 8192 keys each (134 MB) 25 us
// (5.4 TB/s, of which some 6 us are the start, the first loads and the join).
#include <cooperative_groups.h>

#include <cfloat>

#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 4;                // that compute; one more copies
constexpr int kKeys = kXattnFewKeys;     // of a stage
constexpr int kStages = 3;
static_assert(kKeys == 16 * kWarps, "a warp takes 16 keys of a stage");

// D: channels of the tiles (64, or 128 with zeros past the caller's); R: rows (8, 16)
template <int D, int R>
struct Layout {
  static constexpr int REG = D / 64;
  static constexpr int REGION_BYTES = kKeys * 128;  // 64 channels of a stage's keys, 128-byte swizzle
  static constexpr int TILE_BYTES = REG * REGION_BYTES;
  static constexpr int OFF_K = 0;
  static constexpr int OFF_V = OFF_K + kStages * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_V + kStages * TILE_BYTES;
  static constexpr int OFF_MISC = OFF_BAR + 2 * kStages * 8;
  // the parts to join, over the stages once those are read: per warp, and the CTA's
  struct Part {
    float m[R], l[R], e[R], o[R][D];
  };
  static constexpr int OFF_PARTS = 0;
  static_assert((kWarps + 1) * sizeof(Part) <= OFF_BAR, "the parts fit the stages");
  static constexpr int BYTES = OFF_MISC + 16;
  static constexpr int THREADS = (kWarps + 1) * 32;
};

// four 8 x 8 matrices of 16-bit values; row addresses from lanes 0-7, 8-15, 16-23, 24-31
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// d (16 x 8) += a (16 x 16) b (16 x 8), bf16 in, fp32 out
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The weight of a part whose maximum is m once the whole's is top (-inf: no keys).
__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : ex2_approx(m - top); }

// Cluster: a head's rows; CTA: a share of its stages of keys.  HOOK: with the test option, in
// a kernel of its own (a look at it in the copying warp cost 0.1 of 3.5 us).
template <int D, int R, bool HOOK>
__global__ void __launch_bounds__(Layout<D, R>::THREADS)
    xattn_few_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const XattnFewParams p) {
  using L = Layout<D, R>;
  using Part = typename L::Part;
  constexpr int H = R / 8;  // halves of the product's 16 rows in use
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* empty = full + kStages;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC);
  Part* parts = reinterpret_cast<Part*>(smem + L::OFF_PARTS);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int bh = blockIdx.x / ranks;
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // (the same in every CTA)
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], kWarps);
    }
    *abort_flag = aligned ? 0 : 1;
    fence_mbar_init();
    if (!aligned) atomicOr(p.status, kDevMisaligned);
  }
  if (warp == kWarps && lane == 0) {
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
  }
  __syncthreads();
  const WaitCtl ctl{abort_flag, p.status, p.budget_ns};
  pdl_wait();
  pdl_trigger();
  int len = p.S;
  if (p.kv_len) len = min(max(p.kv_len[bh / p.heads], 0), p.S);
  // stages [i0, i1) of the head's are this CTA's
  const int all = (len + kKeys - 1) / kKeys, base = all / ranks, rest = all - base * ranks;
  const int i0 = rank * base + min(rank, rest), n = aligned ? base + (rank < rest) : 0;

  float o[D / 8][4];  // channels 8 k + 2 (lane % 4) and + 1 of rows lane / 4 and + 8
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, e[2] = {0.f, 0.f};
  bool ok = true;
  if (warp == kWarps) {
    // ------------------------------------------------------------ copies
    if (lane == 0) {
      int issued = 0;
      const int copies = HOOK && skips_loads(p.debug_skip_q) ? 0 : n;
      for (; issued < copies; ++issued) {
        const int st = issued % kStages;
        if (!mbar_wait(&empty[st], ((issued / kStages) & 1) ^ 1, ctl)) break;
        mbar_arrive_expect_tx(&full[st], 2 * L::TILE_BYTES);
        for (int r = 0; r < L::REG; ++r) {
          tma_load_3d(smem + L::OFF_K + st * L::TILE_BYTES + r * L::REGION_BYTES, &tm_k, &full[st], 64 * r,
                      (i0 + issued) * kKeys, bh);
          tma_load_3d(smem + L::OFF_V + st * L::TILE_BYTES + r * L::REGION_BYTES, &tm_v, &full[st], 64 * r,
                      (i0 + issued) * kKeys, bh);
        }
      }
      // every copy has landed before the stages take the parts or go away
      for (int i = max(0, issued - kStages); i < issued; ++i)
        drain_wait(&full[i % kStages], (i / kStages) & 1, p.budget_ns);
    }
  } else {
    // ------------------------------------------------------------ attention (whole warps)
    const int row = lane >> 2, pair = 2 * (lane & 3);
    uint32_t q[D / 16][4];  // rows as the product's left side; those past the head's are zeros
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int ch = 16 * k + 8 * c + pair;
          q[k][2 * c + h] = h < H && row + 8 * h < p.M && ch < p.d
                                ? *reinterpret_cast<const uint32_t*>(
                                      p.q + (static_cast<size_t>(bh) * p.M + row + 8 * h) * p.d + ch)
                                : 0u;
        }
#pragma unroll
    for (int k = 0; k < D / 8; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[k][e] = 0.f;
    // lane -> row address of its 8 x 8 matrix: K, matrices are keys 0-7 of four
    // 8-channel chunks; V (transposed), keys 0-7 and 8-15 of two chunks
    const int kr = lane & 7, kc = lane >> 3;
    const int vr = (lane & 7) + 8 * ((lane >> 3) & 1), vc = lane >> 4;
    for (int i = 0; i < n; ++i) {
      const int st = i % kStages;
      if (!(ok = warp_wait(&full[st], (i / kStages) & 1, ctl))) break;
      uint8_t* sk = smem + L::OFF_K + st * L::TILE_BYTES + 16 * warp * 128;
      uint8_t* sv = smem + L::OFF_V + st * L::TILE_BYTES + 16 * warp * 128;
      const int there = len - (i0 + i) * kKeys - 16 * warp;  // valid keys of this warp's 16
      if (there < 16) {
        // what V holds past them does not count, but may be NaN
        if ((lane >> 1) >= there)
          for (int c = lane & 1; c < D / 8; c += 2)
            *reinterpret_cast<uint4*>(sv + (c >> 3) * L::REGION_BYTES + (lane >> 1) * 128 +
                                      (((c & 7) ^ ((lane >> 1) & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
      }
      float s[2][4];  // keys 8 b + pair and + 1 of rows `row` and + 8
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[b][e] = 0.f;
        const int r = 8 * b + kr;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {  // 32 channels a turn
          uint32_t f[4];
          const int ch = 4 * c + kc;
          ldmatrix4(smem_u32(sk + (ch >> 3) * L::REGION_BYTES + r * 128 + (((ch & 7) ^ (r & 7)) << 4)), f);
          mma(s[b], q[2 * c], f[0], f[1]);
          mma(s[b], q[2 * c + 1], f[2], f[3]);
        }
      }
      uint32_t w[4] = {0u, 0u, 0u, 0u};  // the weights as the next product's left side
#pragma unroll
      for (int h = 0; h < H; ++h) {
        float x[2][2], top = m[h];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[b][e] = 8 * b + pair + e < there ? s[b][2 * h + e] * p.scale_log2 : -INFINITY;
            top = fmaxf(top, x[b][e]);
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float from = top == -INFINITY ? 0.f : top;
        if (__any_sync(0xffffffffu, top > m[h])) {
          const float keep = ex2_approx(m[h] - from);
          l[h] *= keep;
          e[h] *= keep;
#pragma unroll
          for (int k = 0; k < D / 8; ++k) o[k][2 * h] *= keep, o[k][2 * h + 1] *= keep;
          m[h] = top;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float w0 = ex2_approx(x[b][0] - from), w1 = ex2_approx(x[b][1] - from);
          w[2 * b + h] = pack_bf16x2(w0, w1);
          e[h] += w0 + w1;  // for the LSE, and the sum of the weights that the product uses
          l[h] += __uint_as_float(w[2 * b + h] << 16) + __uint_as_float(w[2 * b + h] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {  // 16 channels a turn
        uint32_t f[4];
        const int ch = 2 * c + vc;
        ldmatrix4_trans(smem_u32(sv + (ch >> 3) * L::REGION_BYTES + vr * 128 + (((ch & 7) ^ (vr & 7)) << 4)), f);
        mma(o[2 * c], w, f[0], f[1]);
        mma(o[2 * c + 1], w, f[2], f[3]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[st]);
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      e[h] += __shfl_xor_sync(0xffffffffu, e[h], 1);
      e[h] += __shfl_xor_sync(0xffffffffu, e[h], 2);
    }
  }
  // join the warps, then the cluster's CTAs
  __syncthreads();  // the stages are read, and no copy is on its way
  if (warp < kWarps) {
    Part& mine = parts[warp];
    const int row = lane >> 2, pair = 2 * (lane & 3);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int r = row + 8 * h;
#pragma unroll
      for (int k = 0; k < D / 8; ++k)
        *reinterpret_cast<float2*>(&mine.o[r][8 * k + pair]) = make_float2(o[k][2 * h], o[k][2 * h + 1]);
      if (pair == 0) {
        // a warp whose wait ran out: a part that outweighs all others and makes the sum -inf
        mine.m[r] = ok ? m[h] : FLT_MAX;
        mine.l[r] = ok ? l[h] : -INFINITY;
        mine.e[r] = e[h];
      }
    }
  }
  __syncthreads();
  const int rows = min(R, p.M), total = rows * p.d;
  Part& whole = parts[kWarps];
  for (int i = threadIdx.x; i < total; i += L::THREADS) {
    const int r = i / p.d, ch = i - r * p.d;
    float top = -INFINITY, sum = 0.f, exact = 0.f, acc = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) top = fmaxf(top, parts[k].m[r]);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float a = weight(parts[k].m[r], top);
      sum = fmaf(parts[k].l[r], a, sum);
      exact = fmaf(parts[k].e[r], a, exact);
      acc = fmaf(parts[k].o[r][ch], a, acc);
    }
    whole.o[r][ch] = acc;
    if (ch == 0) whole.m[r] = top, whole.l[r] = sum, whole.e[r] = exact;
  }
  cluster.sync();
  for (int i = rank * L::THREADS + threadIdx.x; i < total; i += ranks * L::THREADS) {
    const int r = i / p.d, ch = i - r * p.d;
    float top = -INFINITY, sum = 0.f, exact = 0.f, acc = 0.f;
    for (int k = 0; k < ranks; ++k) top = fmaxf(top, cluster.map_shared_rank(&whole, k)->m[r]);
    for (int k = 0; k < ranks; ++k) {
      const Part* other = cluster.map_shared_rank(&whole, k);
      const float a = weight(other->m[r], top);
      sum = fmaf(other->l[r], a, sum);
      exact = fmaf(other->e[r], a, exact);
      acc = fmaf(other->o[r][ch], a, acc);
    }
    const size_t at = static_cast<size_t>(bh) * p.M + r;
    // 0: no states; -inf: a wait ran out, and what the others read is no result either (a NaN is)
    p.o[at * p.d + ch] = __float2bfloat16(sum <= 0.f ? 0.f : acc / sum);
    if (p.lse && ch == 0)
      p.lse[at] = sum <= 0.f ? -INFINITY : (top + __log2f(exact)) * 0.69314718055994530942f;
  }
  cluster.sync();  // shared memory stays until all have read it
}

template <int D, int R, bool HOOK = false>
cudaError_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const XattnFewParams& p, int dev, cudaStream_t s) {
  using L = Layout<D, R>;
  // CTAs a head: as many as the SMs hold at once (their shared memory: two, or four of
  // 64 channels), each with some stages.  (Two stages and more CTAs: 160 heads of 128,
  // 4096 keys 66 -> 80 us.  160 heads of 64 with two CTAs an SM 44 us, four 37.)
  int ranks = 1;
  while (ranks < 16 && p.BH * ranks * 2 <= (D == 64 ? 4 : 2) * p.sms && p.S > 2 * ranks * kKeys) ranks *= 2;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(dev, [] {
    const cudaError_t e0 =
        cudaFuncSetAttribute(xattn_few_kernel<D, R, HOOK>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (e0 != cudaSuccess) return e0;
    return cudaFuncSetAttribute(xattn_few_kernel<D, R, HOOK>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
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
  cfg.blockDim = dim3(L::THREADS);
  cfg.dynamicSmemBytes = L::BYTES;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl_enabled ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, xattn_few_kernel<D, R, HOOK>, tk, tv, p);
}

}  // namespace

cudaError_t launch_xattn_few(int d, const CUtensorMap& tk, const CUtensorMap& tv, const XattnFewParams& p, int dev,
                             cudaStream_t s) {
  if (p.debug_skip_q) return d == 64 ? launch<64, 16, true>(tk, tv, p, dev, s) : launch<128, 16, true>(tk, tv, p, dev, s);
  if (d == 64) return p.M <= 8 ? launch<64, 8>(tk, tv, p, dev, s) : launch<64, 16>(tk, tv, p, dev, s);
  return p.M <= 8 ? launch<128, 8>(tk, tv, p, dev, s) : launch<128, 16>(tk, tv, p, dev, s);
}

}  // namespace mw
