// Product of two matrices in 8 bits with a power-of-two scale for every 128 of the
// contraction:
//
//   C[p, q] = sum over blocks kb of 2^(ea[p, kb] + eb[q, kb]) sum over k in kb of a[p, k] b[q, k]
//
// a, b e4m3; the scales e8m0, one for a row (or for 128 rows) and block.  The tensor cores
// take them as they are: kind::mxf8f6f4 multiplies every 32 of the contraction by a scale of
// A and of B from tensor memory, so a block's scale serves four instructions, sums stay in
// fp32 in tensor memory, and nothing passes over the accumulators between blocks.  (Scales
// of any value would need that: a load from tensor memory and an FMA an element for every
// 128 of the contraction.)
//
// One warp copies tiles of 128 x 128 bytes (TMA, 128-byte swizzle) of operands that run along
// the contraction (rows of A and B) or across it (columns: the transposed forms, which the
// MMA reads as they lie), one gathers scale words, one issues MMAs, four write the tile.
// Scale words: a word holds four blocks' scales of a row; words of rows l, l + 32, l + 64,
// l + 96 lie together in shared memory and go to the lane l of four columns of tensor memory.
#include <cooperative_groups.h>

#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace cg = cooperative_groups;

namespace mw {
namespace {

constexpr int kBlock = 128;          // of the contraction: a stage, and what a scale covers
constexpr int kA = 128 * kBlock;     // bytes of A's tile
constexpr int kThreads = 256;
constexpr int kEpiWarps = 4;
constexpr int kGroup = 4;            // blocks of a scale word

// BN: rows of B of a tile.  JOIN: the CTAs of a cluster share a tile's contraction and add
// their parts up in shared memory; else a CTA takes tiles in turn.
template <int BN, bool JOIN>
struct Layout {
  static constexpr int B = BN * kBlock;  // (columns of B: 128 at a time, so BN >= 128 there)
  static constexpr int STAGE = kA + B;
  static constexpr int ATOMS = 1 + (BN + 127) / 128;  // of scale words, 512 bytes each
  static constexpr int SETS = BN == 256 ? 2 : 4;      // groups of scales in shared and tensor memory
  static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 5 : 4;
  static constexpr int STORES = JOIN ? 0 : BN == 256 ? 1 : 2;  // boxes of 32 rows x 128 bytes a warp
  static constexpr int OFF_STORE = STAGES * STAGE;
  static constexpr int OFF_SCALE = OFF_STORE + kEpiWarps * STORES * 4096;
  static constexpr int OFF_BAR = OFF_SCALE + SETS * ATOMS * 512;
  static constexpr int N_BAR = 2 * STAGES + 2 * SETS + 5;
  static constexpr int OFF_MISC = OFF_BAR + N_BAR * 8;
  static constexpr int SMEM = OFF_MISC + 16;
  static_assert(SMEM <= 232448, "shared memory of a CTA");
  // Tensor memory: two accumulators; of 256 columns they overlap in 32, which are read first
  static constexpr int OVERLAP = BN == 256 ? 32 : 0;
  static constexpr int ACCS = JOIN ? 1 : 2;
  static constexpr int SCALES = ACCS * BN - (JOIN ? 0 : OVERLAP);
  static constexpr int WORDS = 4 * ATOMS;  // columns of a set
  static constexpr int USED = SCALES + SETS * WORDS;
  static constexpr int COLS = USED <= 64 ? 64 : USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
  static_assert(USED <= 512, "tensor memory");
  // the parts that a cluster adds up: rows of a padded pitch
  static constexpr int PART = JOIN ? (BN + 4) * 128 > 132 * BN ? (BN + 4) * 128 * 4 : 132 * BN * 4 : 0;
  static_assert(PART <= STAGES * STAGE, "the parts take the stages' place");
};

// The scale words of blocks kb ... kb + 3 (of n) and of one row.
__device__ __forceinline__ uint32_t scale_word(const Fp8Scales& s, int row, int rows, int kb, int n) {
  row = min(row, rows - 1);
  const uint8_t* p = s.p + static_cast<long long>(s.tile ? row >> 7 : row) * s.row + kb * s.block;
  if (s.words && (kb & 3) == 0 && kb + 3 < n) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (kb + i < n) w |= static_cast<uint32_t>(p[i * s.block]) << (8 * i);
  return w;
}

// Tile t of the persistent order: bands of 16 tiles of A's rows, in which B's rows go on
// slowly, so that both operands' tiles in work stay in L2.
__device__ __forceinline__ void tile_at(const Fp8MmParams& p, int t, int* tp, int* tq) {
  const int band = 16 * p.tiles_q, first = t / band * 16, n = min(16, p.tiles_p - first);
  const int i = t % band;
  *tp = first + i % n;
  *tq = i / n;
}

__device__ __forceinline__ void store_one(const Fp8MmParams& p, long long at, float v) {
  if (p.out_f32)
    static_cast<float*>(p.out)[at] = v;
  else
    static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16(v);
}

// Four results in a row of the output, of which n count.
__device__ __forceinline__ void store_four(const Fp8MmParams& p, long long at, float4 v, int n) {
  if (n >= 4 && p.out_quads) {
    if (p.out_f32)
      *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = v;
    else
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) =
          make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    return;
  }
  const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) store_one(p, at + i, e[i]);
}

template <int BN, bool JOIN>
__global__ void __launch_bounds__(kThreads, JOIN && BN <= 64 ? 2 : 1)
    fp8_mm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                  const __grid_constant__ CUtensorMap tm_c, const Fp8MmParams p) {
  using L = Layout<BN, JOIN>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* empty = full + L::STAGES;
  uint64_t* sc_full = empty + L::STAGES;
  uint64_t* sc_empty = sc_full + L::SETS;
  uint64_t* acc_full = sc_empty + L::SETS;  // [2]
  uint64_t* acc_free = acc_full + 2;        // [2]
  uint64_t* done = acc_free + 2;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC);
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::STAGES; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1);
    for (int s = 0; s < L::SETS; ++s) mbar_init(&sc_full[s], 1), mbar_init(&sc_empty[s], 1);
    for (int s = 0; s < 2; ++s) mbar_init(&acc_full[s], 1), mbar_init(&acc_free[s], kEpiWarps);
    mbar_init(done, 1);
    *abort_flag = aligned ? 0 : 1;
    fence_mbar_init();
    if (!aligned) atomicOr(p.status, kDevMisaligned);
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_b);
    if (!JOIN && p.tma_out) prefetch_tmap(&tm_c);
  }
  if (warp == 1) {
    tmem_alloc(tmem_at, L::COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  const WaitCtl ctl{abort_flag, p.status, p.budget_ns};
  pdl_wait();
  pdl_trigger();

  // JOIN: tile blockIdx.x / ranks, a share of its blocks
  int rank = 0, ranks = 1, tile0 = blockIdx.x, tile_step = gridDim.x;
  if constexpr (JOIN) {
    cg::cluster_group cluster = cg::this_cluster();
    rank = static_cast<int>(cluster.block_rank());
    ranks = static_cast<int>(cluster.num_blocks());
    tile0 = blockIdx.x / ranks;
    tile_step = p.tiles_p * p.tiles_q;
  }
  const int n_tiles = p.tiles_p * p.tiles_q;
  const int kb0 = p.blocks * rank / ranks, kb1 = p.blocks * (rank + 1) / ranks;

  if (warp == 0) {
    // ------------------------------------------------------------ tiles of A and B
    if (lane == 0 && aligned) {
      const bool skip = skips_loads(p.debug_skip_q);
      int i = 0, issued = 0;
      bool ok = true;
      for (int t = tile0; t < n_tiles && ok; t += tile_step) {
        int tp, tq;
        tile_at(p, t, &tp, &tq);
        for (int kb = kb0; kb < kb1; ++kb, ++i) {
          const int st = i % L::STAGES;
          if (!mbar_wait(&empty[st], ((i / L::STAGES) & 1) ^ 1, ctl)) {
            ok = false;
            break;
          }
          if (skip) continue;
          uint8_t* a = smem + st * L::STAGE;
          uint8_t* b = a + kA;
          mbar_arrive_expect_tx(&full[st], L::STAGE);
          if (p.a_columns)
            tma_load_2d(a, &tm_a, &full[st], tp * 128, kb * kBlock);
          else
            tma_load_2d(a, &tm_a, &full[st], kb * kBlock, tp * 128);
          if (p.b_columns) {
            if constexpr (BN >= 128) {
#pragma unroll
              for (int r = 0; r < BN / 128; ++r)
                tma_load_2d(b + r * 128 * kBlock, &tm_b, &full[st], tq * BN + r * 128, kb * kBlock);
            }
          } else {
            tma_load_2d(b, &tm_b, &full[st], kb * kBlock, tq * BN);
          }
          issued = i + 1;
        }
      }
      // every copy has landed before the CTA goes
      for (int k = max(0, issued - L::STAGES); k < issued; ++k)
        drain_wait(&full[k % L::STAGES], (k / L::STAGES) & 1, p.budget_ns);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    const uint32_t idesc = idesc_mxf8(128, BN, p.a_columns, p.b_columns);
    // along the contraction: 32 bytes of a row an instruction; across it: 32 rows of 128 bytes
    const uint32_t a_step = p.a_columns ? 256u : 2u, b_step = p.b_columns ? 256u : 2u;
    const uint32_t a0 = sdesc_sw128(smem_u32(smem), 128 * kBlock);
    const uint32_t sc0 = smem_u32(smem + L::OFF_SCALE);
    bool ok = aligned;
    int i = 0, g = 0, j = 0;  // stages, scale groups, tiles
    for (int t = tile0; t < n_tiles && ok; t += tile_step, ++j) {
      uint32_t acc = tmem;
      if constexpr (!JOIN) {
        acc += (j & 1) * (BN - L::OVERLAP);
        // this accumulator's columns have been read: of the tile before (their overlap) or
        // of the one before that
        const int wait = L::OVERLAP ? j - 1 : j - 2;
        if (wait >= 0) ok = warp_wait(&acc_free[wait & 1], (wait >> 1) & 1, ctl);
        tc_fence_after();
      }
      for (int kb = kb0; kb < kb1 && ok; ++kb, ++i) {
        const int in = (kb - kb0) % kGroup, set = g % L::SETS;
        const uint32_t words = tmem + L::SCALES + set * L::WORDS;
        if (in == 0) {
          ok = warp_wait(&sc_full[set], (g / L::SETS) & 1, ctl);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int a = 0; a < L::ATOMS; ++a)
            tmem_copy_scales(words + 4 * a, sc0 + (set * L::ATOMS + a) * 512);
        }
        const int st = i % L::STAGES;
        ok = warp_wait(&full[st], (i / L::STAGES) & 1, ctl);
        if (!ok) break;
        tc_fence_after();
        const uint32_t a = a0 + st * (L::STAGE >> 4);
        umma_mx4(acc, a, a + (kA >> 4), a_step, b_step, idesc | idesc_scale_byte(in), words, words + 4,
                 kb > kb0);
        umma_commit(&empty[st]);
        if (in == kGroup - 1 || kb + 1 == kb1) {
          umma_commit(&sc_empty[set]);
          ++g;
        }
      }
      if (ok) umma_commit(&acc_full[j & 1]);
    }
    if (!ok) {  // what was issued ends before the CTA goes
      umma_commit(done);
      drain_wait(done, 0, p.budget_ns);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------ scale words
    uint4* to = reinterpret_cast<uint4*>(smem + L::OFF_SCALE);
    bool ok = aligned;
    int g = 0;
    for (int t = tile0; t < n_tiles && ok; t += tile_step) {
      int tp, tq;
      tile_at(p, t, &tp, &tq);
      for (int kb = kb0; kb < kb1; kb += kGroup, ++g) {
        const int set = g % L::SETS;
        uint32_t w[L::ATOMS][4];
#pragma unroll
        for (int a = 0; a < L::ATOMS; ++a) {
          const Fp8Scales& s = a == 0 ? p.a_scales : p.b_scales;
          const int rows = a == 0 ? p.rows_a : p.rows_b;
          const int row = a == 0 ? tp * 128 : tq * BN + (a - 1) * 128;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            w[a][r] = s.tile && r > 0 ? w[a][0] : scale_word(s, row + (s.tile ? 0 : r * 32 + lane), rows, kb, kb1);
        }
        ok = warp_wait(&sc_empty[set], ((g / L::SETS) & 1) ^ 1, ctl);
        if (!ok) break;
#pragma unroll
        for (int a = 0; a < L::ATOMS; ++a)
          to[(set * L::ATOMS + a) * 32 + lane] = make_uint4(w[a][0], w[a][1], w[a][2], w[a][3]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sc_full[set]);
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ results
    const int quarter = warp - 4;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    [[maybe_unused]] uint8_t* stores = smem + L::OFF_STORE + quarter * L::STORES * 4096;
    bool ok = aligned;
    int j = 0;
    [[maybe_unused]] int sent = 0;
    for (int t = tile0; t < n_tiles; t += tile_step, ++j) {
      int tp, tq;
      tile_at(p, t, &tp, &tq);
      ok = ok && warp_wait(&acc_full[j & 1], (j >> 1) & 1, ctl);
      tc_fence_after();
      const uint32_t acc = tmem + lanes + (JOIN ? 0 : (j & 1) * (BN - L::OVERLAP));
      if constexpr (JOIN) {
        float* part = reinterpret_cast<float*>(smem);
        const int row = quarter * 32 + lane;
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
          uint32_t v[16];
          if (ok) {
            tmem_ld16(acc + c, v);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = 0u;
          }
          if (p.swap) {
#pragma unroll
            for (int k = 0; k < 16; ++k) part[(c + k) * 132 + row] = __uint_as_float(v[k]);
          } else {
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              *reinterpret_cast<uint4*>(part + row * (BN + 4) + c + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
          }
        }
      } else {
        const int per = p.out_f32 ? 32 : 64;  // columns of a box
        const int n_boxes = BN / per;
        const int row0 = tp * 128 + quarter * 32;
        // accumulator 0 ends in the overlap, 1 begins with it
        const bool backwards = L::OVERLAP && (j & 1) == 0;
#pragma unroll 1
        for (int k = 0; k < n_boxes; ++k) {
          const int box = backwards ? n_boxes - 1 - k : k;
          const int c0 = box * per;
          uint8_t* to = stores + (sent % (L::STORES ? L::STORES : 1)) * 4096;
          uint32_t w[32];
          if (ok) {
            tmem_ld32(acc + c0, w);
            if (p.out_f32) {
              tmem_wait_ld();
            } else {
              uint32_t v[32];
              tmem_ld32(acc + c0 + 32, v);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
#pragma unroll
              for (int e = 0; e < 16; ++e)
                w[16 + e] = pack_bf16x2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] = 0u;
          }
          if (L::OVERLAP ? k == 0 : k == n_boxes - 1) {  // (every box covers the overlap's 32 columns)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_free[j & 1]);
          }
          const int col0 = tq * BN + c0;
          if (col0 >= p.rows_b || row0 >= p.rows_a) continue;
          if (lane == 0) bulk_wait_read<L::STORES ? L::STORES - 1 : 0>();
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(to + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
          if (p.tma_out) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_2d(&tm_c, to, col0, row0);
              bulk_commit_group();
            }
            ++sent;
          } else {  // rows that do not start at 16 bytes: single elements, a row a turn
            __syncwarp();
            for (int r = 0; r < 32 && row0 + r < p.rows_a; ++r)
              for (int c = lane; c < per && col0 + c < p.rows_b; c += 32) {
                const int at = p.out_f32 ? c * 4 : c * 2;
                const uint8_t* from = to + r * 128 + (((at >> 4) ^ (r & 7)) << 4) + (at & 15);
                const long long dst = static_cast<long long>(row0 + r) * p.ld + col0 + c;
                if (p.out_f32)
                  static_cast<float*>(p.out)[dst] = *reinterpret_cast<const float*>(from);
                else
                  static_cast<__nv_bfloat16*>(p.out)[dst] = *reinterpret_cast<const __nv_bfloat16*>(from);
              }
            __syncwarp();
          }
        }
      }
    }
    if (!JOIN && lane == 0) bulk_wait_all();
  }

  if constexpr (JOIN) {
    // every CTA adds up a share of the tile, the parts in their order
    __syncwarp();
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    int tp, tq;
    tile_at(p, tile0, &tp, &tq);
    // swapped: a row of the output is a row of B, and runs over A's rows
    const int inner = p.swap ? 128 : BN, pitch = inner + 4;
    const int o0 = p.swap ? tq * BN : tp * 128, i0 = p.swap ? tp * 128 : tq * BN;
    const int outer = min(p.swap ? BN : 128, (p.swap ? p.rows_b : p.rows_a) - o0);
    const int in_n = (p.swap ? p.rows_a : p.rows_b) - i0;
    const int quads = outer * (inner / 4);
    const int q0 = quads * rank / ranks, q1 = quads * (rank + 1) / ranks;
    float* part = reinterpret_cast<float*>(smem);
    for (int e = q0 + threadIdx.x; e < q1; e += kThreads) {
      const int o = e / (inner / 4), i = e % (inner / 4) * 4;
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int r = 0; r < ranks; ++r) {
        const float4 v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(part, r) + o * pitch + i);
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
      }
      if (i < in_n) store_four(p, static_cast<long long>(o0 + o) * p.ld + i0 + i, s, in_n - i);
    }
    cluster.sync();  // shared memory stays until all have read it
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, L::COLS);
  }
}

template <int BN, bool JOIN>
cudaError_t run(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const Fp8MmParams& p, int dev,
                cudaStream_t s) {
  using L = Layout<BN, JOIN>;
  auto kernel = fp8_mm_kernel<BN, JOIN>;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(dev, [&] {
    const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
    if (f != cudaSuccess || !JOIN) return f;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  const int tiles = p.tiles_p * p.tiles_q;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[2];
  pdl_config(cfg, attr[0], dim3(JOIN ? tiles * p.splits : tiles < p.ctas ? tiles : p.ctas), dim3(kThreads), L::SMEM,
             s);
  if (JOIN) {
    cudaLaunchAttribute& c = attr[cfg.numAttrs++];
    c.id = cudaLaunchAttributeClusterDimension;
    c.val.clusterDim.x = p.splits;
    c.val.clusterDim.y = c.val.clusterDim.z = 1;
    cfg.attrs = attr;
  }
  return cudaLaunchKernelEx(&cfg, kernel, ta, tb, tc, p);
}

}  // namespace

cudaError_t launch_fp8_mm(int bn, bool join, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc,
                          const Fp8MmParams& p, int dev, cudaStream_t s) {
  if (join) {
    if (bn == 16) return run<16, true>(ta, tb, tc, p, dev, s);
    if (bn == 32) return run<32, true>(ta, tb, tc, p, dev, s);
    if (bn == 64) return run<64, true>(ta, tb, tc, p, dev, s);
    return run<128, true>(ta, tb, tc, p, dev, s);
  }
  if (bn == 128) return run<128, false>(ta, tb, tc, p, dev, s);
  return run<256, false>(ta, tb, tc, p, dev, s);
}

}  // namespace mw
