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
// Warps of a CTA: one copies tiles of 128 x 128 bytes (TMA, 128-byte swizzle) of operands that
// run along the contraction (rows of A and B) or across it (columns: the transposed forms,
// which the MMA reads as they lie, at the same rate), one gathers scale words, one issues
// MMAs, the others write the tile.  Scale words: a word holds four blocks' scales of a row; words of
// rows l, l + 32, l + 64, l + 96 lie together in shared memory and go to the lane l of four
// columns of tensor memory.
//
// Two kernels: pairs of CTAs that share tiles of 256 x BN, for many rows of both operands,
// and clusters that share the contraction of a tile, for few.
#include <cooperative_groups.h>

#include <atomic>

#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace cg = cooperative_groups;

namespace mw {
namespace {

constexpr int kBlock = 128;       // of the contraction: a stage, and what a scale covers
constexpr int kA = 128 * kBlock;  // bytes of A's tile
constexpr int kThreads = 256;
constexpr int kGroup = 4;         // blocks of a scale word

// ------------------------------------------------------------------ scale words

// The scales of blocks kb ... kb + 3 (of n) of 128 rows from `row` on (of `rows`), as they are
// read: lane l has rows l, l + 32, ... (kQuads: 4 l ... 4 l + 3).  The way is known at compile
// time: chosen at each load, the ways' results came together in registers, which waited
// for each operand's loads before the next one's (weight's gradient of 10240 x 2560 over 14080:
// 318 us).
template <Fp8Read WAY>
struct RawScales {
  uint32_t v[WAY == Fp8Read::kBytes ? 16 : 4];
  __device__ __forceinline__ void load(const Fp8Scales& s, int row, int rows, int kb, int n) {
    const int lane = threadIdx.x & 31;
    const uint8_t* p = s.p + kb * s.block;
    if constexpr (WAY == Fp8Read::kTile) {
      p += static_cast<long long>(min(row, rows - 1) >> 7) * s.row;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = p[min(i, n - 1 - kb) * s.block];
    } else if constexpr (WAY == Fp8Read::kQuads) {
      p += min(row + 4 * lane, rows - 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t*>(p + min(i, n - 1 - kb) * s.block);
    } else if constexpr (WAY == Fp8Read::kWords) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = *reinterpret_cast<const uint32_t*>(p + min(row + 32 * r + lane, rows - 1) * s.row);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[4 * r + i] = p[min(row + 32 * r + lane, rows - 1) * s.row + min(i, n - 1 - kb) * s.block];
    }
  }
  // Into an atom of 512 bytes: the word of row r of the 128 at 16 (r % 32) + 4 (r / 32).
  __device__ __forceinline__ void store(uint8_t* atom) const {
    const int lane = threadIdx.x & 31;
    uint4* mine = reinterpret_cast<uint4*>(atom) + lane;
    if constexpr (WAY == Fp8Read::kTile) {
      const uint32_t w = v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24;
      *mine = make_uint4(w, w, w, w);
    } else if constexpr (WAY == Fp8Read::kQuads) {
      // four blocks of four rows, turned: byte i of word b to byte b of word i
      const uint32_t lo01 = __byte_perm(v[0], v[1], 0x5140), hi01 = __byte_perm(v[0], v[1], 0x7362);
      const uint32_t lo23 = __byte_perm(v[2], v[3], 0x5140), hi23 = __byte_perm(v[2], v[3], 0x7362);
      const uint32_t t[4] = {__byte_perm(lo01, lo23, 0x5410), __byte_perm(lo01, lo23, 0x7632),
                             __byte_perm(hi01, hi23, 0x5410), __byte_perm(hi01, hi23, 0x7632)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * lane + i;
        *reinterpret_cast<uint32_t*>(atom + 16 * (r & 31) + 4 * (r >> 5)) = t[i];
      }
    } else if constexpr (WAY == Fp8Read::kWords) {
      *mine = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
      uint32_t t[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) t[r] = v[4 * r] | v[4 * r + 1] << 8 | v[4 * r + 2] << 16 | v[4 * r + 3] << 24;
      *mine = make_uint4(t[0], t[1], t[2], t[3]);
    }
  }
};

// f with the ways of A's and of B's scales as types.
template <Fp8Read WAY>
struct Way {
  static constexpr Fp8Read value = WAY;
};
template <class F>
__device__ __forceinline__ void with_way(Fp8Read way, F&& f) {
  if (way == Fp8Read::kTile)
    f(Way<Fp8Read::kTile>{});
  else if (way == Fp8Read::kWords)
    f(Way<Fp8Read::kWords>{});
  else if (way == Fp8Read::kQuads)
    f(Way<Fp8Read::kQuads>{});
  else
    f(Way<Fp8Read::kBytes>{});
}

// Tile t: bands of 16 tiles of A's rows, in which B's rows go on slowly, so that both
// operands' tiles in work stay in L2.
__device__ __forceinline__ void tile_at(const Fp8MmParams& p, int t, int* tp, int* tq) {
  const int band = 16 * p.tiles_q, first = t / band * 16, n = min(16, p.tiles_p - first);
  const int i = t % band;
  *tp = first + i % n;
  *tq = i / n;
}

// ------------------------------------------------------------------ parts

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
  for (int i = 0; i < 4; ++i) {
    if (i >= n) continue;
    if (p.out_f32)
      static_cast<float*>(p.out)[at + i] = e[i];
    else
      static_cast<__nv_bfloat16*>(p.out)[at + i] = __float2bfloat16(e[i]);
  }
}

// The sum of the parts that `ranks` CTAs have in shared memory at `part`, [outer][inner] at a
// pitch of inner + 4 floats, in the order of the ranks: this one, `rank`, does its share of
// them.  CTA r of these is cta(r) of the cluster.  To row o0 and column i0 of the output, of which in_n
// columns are left.
template <class Cta>
__device__ __forceinline__ void join_parts(const Fp8MmParams& p, float* part, int outer, int inner, long long o0,
                                           int i0, int in_n, int rank, int ranks, int threads, Cta cta) {
  cg::cluster_group cluster = cg::this_cluster();
  const int quads = outer * (inner / 4), pitch = inner + 4;
  const int q0 = quads * rank / ranks, q1 = quads * (rank + 1) / ranks;
  for (int e = q0 + threadIdx.x; e < q1; e += threads) {
    const int o = e / (inner / 4), i = e % (inner / 4) * 4;
    if (i >= in_n) continue;
    // (all on their way at once: one after another, eight of them took 5 us)
    float4 v[kFp8Splits];
#pragma unroll
    for (int r = 0; r < kFp8Splits; ++r)
      if (r < ranks) v[r] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(part, cta(r)) + o * pitch + i);
    float4 s = v[0];
#pragma unroll
    for (int r = 1; r < kFp8Splits; ++r)
      if (r < ranks) s.x += v[r].x, s.y += v[r].y, s.z += v[r].z, s.w += v[r].w;
    store_four(p, (o0 + o) * p.ld + i0 + i, s, in_n - i);
  }
}

// ------------------------------------------------------------------ pairs of CTAs
//
// Two CTAs (of one pair of SMs) take a tile of 256 x BN: each copies 128 rows of A and half of
// B's, and the MMAs of the first one read both halves of B, so that an SM takes 32 KB from
// L2 for 128 x 256 x 128 products, not 48 (a CTA alone with 128 x 256: 14080 x 10240 x 2560 in
// 322 us, held by L2 at 13 TB/s).  Both have the scales of all of B's rows.
//
// fp32 sums of more than `chunk` blocks leave tensor memory in parts, which the output adds up:
// the tensor cores cut, not round, what falls below a sum's last place, and 440 such additions
// (14080 tokens) came to 1e-6 of the result, of positive terms to 2^-23.6 for each addition.  (bf16
// results of more are left to clusters of CTAs, below, which add up in tensor memory.)
//
// JOIN: few tiles and a long contraction, as a weight's gradient has: a cluster of up to four
// pairs shares the blocks of a tile, and each CTA adds up a share of its rows' parts, which takes
// 4 us and saves half of the blocks or more (gradient of 2304 x 768 over 14080: 35.6 to
// 24.9 us, by 27 x 2 pairs of 76).

constexpr int kPairThreads = 384;
constexpr int kPairEpiWarps = 8;  // two for a quarter of the rows, half of the columns each
constexpr int kBoxBytes = 32 * 64;

template <int BN>
struct PairLayout {
  static constexpr int B = 128 * kBlock;       // a CTA's half of B (BN = 128: 64 rows, or 64 of the
                                               // 128 columns of a box)
  static constexpr int STAGE = kA + B;
  static constexpr int ATOMS = 1 + BN / 128;   // of scale words, 512 bytes each
  static constexpr int SETS = BN == 256 ? 2 : 4;  // groups of scales in shared and tensor memory
  static constexpr int STAGES = 6;                  // (5: 2% more time)
  static constexpr int OFF_STORE = STAGES * STAGE;  // a box of 32 rows x 64 bytes a warp
  static constexpr int OFF_SCALE = OFF_STORE + kPairEpiWarps * kBoxBytes;
  static constexpr int OFF_BAR = OFF_SCALE + SETS * ATOMS * 512;
  static constexpr int N_BAR = 2 * STAGES + 2 * SETS + 5;
  static constexpr int OFF_MISC = OFF_BAR + N_BAR * 8;
  static constexpr int SMEM = OFF_MISC + 16;
  static_assert(SMEM <= 232448, "shared memory of a CTA");
  static_assert((BN + 4) * 128 * 4 <= OFF_STORE, "a part fits");
  // Tensor memory: two accumulators; of 256 columns they overlap in 32, which are read first
  static constexpr int OVERLAP = BN == 256 ? 32 : 0;
  static constexpr int SCALES = 2 * BN - OVERLAP;
  static constexpr int WORDS = 4 * ATOMS;      // columns of a set
  static_assert(SCALES + SETS * WORDS <= 512, "tensor memory");
};

template <int BN, bool JOIN>
__global__ void __launch_bounds__(kPairThreads, 1)
    fp8_mm_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                       const __grid_constant__ CUtensorMap tm_c, const Fp8MmParams p) {
  using L = PairLayout<BN>;
  extern __shared__ __align__(1024) uint8_t smem[];
  // (of the first CTA: full, sc_full, acc_free; both: empty, sc_empty, acc_full)
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
  cg::cluster_group cluster = cg::this_cluster();
  // of the pair, whose first CTA is `leader` of the cluster
  const uint32_t rank = cluster.block_rank() & 1u, leader = cluster.block_rank() & ~1u;
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // (the same in all)
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::STAGES; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1);
    for (int s = 0; s < L::SETS; ++s) mbar_init(&sc_full[s], 2), mbar_init(&sc_empty[s], 1);
    for (int s = 0; s < 2; ++s) mbar_init(&acc_full[s], 1), mbar_init(&acc_free[s], 2 * kPairEpiWarps);
    mbar_init(done, 1);
    *abort_flag = aligned ? 0 : 1;
    fence_mbar_init();
    if (!aligned) atomicOr(p.status, kDevMisaligned);
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_b);
    if (p.tma_out) prefetch_tmap(&tm_c);
  }
  if (warp == 1) tmem_alloc_pair(tmem_at, 512);
  tc_fence_before();
  __syncthreads();
  cluster.sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  const WaitCtl ctl{abort_flag, p.status, p.budget_ns};
  pdl_wait();
  pdl_trigger();

  const int n_tiles = p.tiles_p * p.tiles_q;
  const int pairs = JOIN ? p.splits : 1;  // of a tile
  const int tile0 = blockIdx.x / (2 * pairs), tile_step = gridDim.x / (2 * pairs);
  // this pair's blocks (JOIN: a chunk of them, and one tile a cluster)
  const int k0 = JOIN ? static_cast<int>(leader / 2) * p.chunk : 0, k1 = JOIN ? min(k0 + p.chunk, p.blocks) : p.blocks;

  if (warp == 0) {
    // ------------------------------------------------------------ tiles of A and B
    if (lane == 0 && aligned) {
      const bool skip = p.debug_skip_q != 0;
      const uint32_t bytes = kA + (BN == 256 || p.b_columns ? L::B : L::B / 2);  // of a CTA
      int i = 0, issued = 0;
      bool ok = true;
      for (int t = tile0; t < n_tiles && ok; t += tile_step) {
        int tp, tq;
        tile_at(p, t, &tp, &tq);
        const int row_a = tp * 256 + rank * 128, row_b = tq * BN + rank * (BN / 2);
        for (int kb = k0; kb < k1; ++kb, ++i) {
          const int st = i % L::STAGES;
          if (!mbar_wait(&empty[st], ((i / L::STAGES) & 1) ^ 1, ctl)) {
            ok = false;
            break;
          }
          if (skip) continue;
          uint8_t* a = smem + st * L::STAGE;
          const uint32_t bar = cluster_address(smem_u32(&full[st]), leader);
          if (rank == 0) mbar_arrive_expect_tx(&full[st], 2 * bytes);
          if (p.a_columns)
            tma_load_2d_pair(a, &tm_a, bar, row_a, kb * kBlock);
          else
            tma_load_2d_pair(a, &tm_a, bar, kb * kBlock, row_a);
          if (p.b_columns)
            tma_load_2d_pair(a + kA, &tm_b, bar, row_b, kb * kBlock);
          else
            tma_load_2d_pair(a + kA, &tm_b, bar, kb * kBlock, row_b);
          issued = i + 1;
        }
      }
      // every copy has landed before the CTAs go (the other one's are counted here too)
      if (rank == 0)
        for (int k = max(0, issued - L::STAGES); k < issued; ++k)
          drain_wait(&full[k % L::STAGES], (k / L::STAGES) & 1, p.budget_ns);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs, by the first CTA
    if (rank == 0) {
      const uint32_t idesc = idesc_mxf8(256, BN, p.a_columns, p.b_columns);
      // along the contraction: 32 bytes of a row an instruction; across it: 32 rows of 128 bytes
      const uint32_t a_step = p.a_columns ? 256u : 2u, b_step = p.b_columns ? 256u : 2u;
      const uint32_t a0 = sdesc_sw128(smem_u32(smem), 128 * kBlock);
      const uint32_t sc0 = smem_u32(smem + L::OFF_SCALE);
      bool ok = aligned;
      int i = 0, g = 0, j = 0;  // stages, scale groups, chunks
      for (int t = tile0; t < n_tiles && ok; t += tile_step) {
        for (int first = k0; first < k1 && ok; first += p.chunk, ++j) {
          const uint32_t acc = tmem + (j & 1) * (BN - L::OVERLAP);
          // this accumulator's columns have been read: of the chunk before (their overlap, and
          // by then all of the one before that) or of the one before that
          const int wait = L::OVERLAP ? j - 1 : j - 2;
          if (wait >= 0) ok = warp_wait(&acc_free[wait & 1], (wait >> 1) & 1, ctl);
          tc_fence_after();
          const int end = min(first + p.chunk, k1);
          for (int kb = first; kb < end && ok; ++kb, ++i) {
            const int in = (kb - first) % kGroup, set = g % L::SETS;
            const uint32_t words = tmem + L::SCALES + set * L::WORDS;
            if (in == 0) {
              ok = warp_wait(&sc_full[set], (g / L::SETS) & 1, ctl);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int a = 0; a < L::ATOMS; ++a)
                tmem_copy_scales<true>(words + 4 * a, sc0 + (set * L::ATOMS + a) * 512);
            }
            const int st = i % L::STAGES;
            ok = warp_wait(&full[st], (i / L::STAGES) & 1, ctl);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = a0 + st * (L::STAGE >> 4);
            umma_mx4<true>(acc, a, a + (kA >> 4), a_step, b_step, idesc | idesc_scale_byte(in), words, words + 4,
                           kb > first);
            umma_commit_pair(&empty[st], leader);
            if (in == kGroup - 1 || kb + 1 == end) {
              umma_commit_pair(&sc_empty[set], leader);
              ++g;
            }
          }
          if (ok) umma_commit_pair(&acc_full[j & 1], leader);
        }
      }
      if (!ok) {  // what was issued ends before the CTAs go
        umma_commit_pair(done, leader);
        drain_wait(done, 0, p.budget_ns);
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------ scale words
    with_way(p.a_scales.read, [&](auto wa) {
      with_way(p.b_scales.read, [&](auto wb) {
        // a group's loads are on their way while the one before is stored
        struct Raw {
          RawScales<decltype(wa)::value> a;
          RawScales<decltype(wb)::value> b[L::ATOMS - 1];
        } raw, next;
        // the group after (t, first, kb)
        auto advance = [&](int* t, int* first, int* kb) {
          *kb += kGroup;
          if (*kb < min(*first + p.chunk, k1)) return;
          *first += p.chunk;
          if (*first >= k1) *first = k0, *t += tile_step;
          *kb = *first;
        };
        auto load = [&](Raw* to, int t, int first, int kb) {
          if (t >= n_tiles) return;
          int tp, tq;
          tile_at(p, t, &tp, &tq);
          const int end = min(first + p.chunk, k1);
          to->a.load(p.a_scales, tp * 256 + rank * 128, p.rows_a, kb, end);
#pragma unroll
          for (int a = 0; a < L::ATOMS - 1; ++a) to->b[a].load(p.b_scales, tq * BN + a * 128, p.rows_b, kb, end);
        };
        int t = aligned ? tile0 : n_tiles, first = k0, kb = k0;
        load(&raw, t, first, kb);
        for (int g = 0; t < n_tiles; ++g) {
          const int set = g % L::SETS;
          advance(&t, &first, &kb);
          load(&next, t, first, kb);
          if (!warp_wait(&sc_empty[set], ((g / L::SETS) & 1) ^ 1, ctl)) break;
          uint8_t* to = smem + L::OFF_SCALE + set * L::ATOMS * 512;
          raw.a.store(to);
#pragma unroll
          for (int a = 0; a < L::ATOMS - 1; ++a) raw.b[a].store(to + (a + 1) * 512);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(cluster_address(smem_u32(&sc_full[set]), leader));
          raw = next;
        }
      });
    });
    __syncwarp();
  } else if (JOIN && warp >= 4) {
    // ------------------------------------------------------------ this CTA's part, in the stages' place
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    const bool ok = aligned && warp_wait(acc_full, 0, ctl);
    tc_fence_after();
    const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    float* part = reinterpret_cast<float*>(smem) + (quarter * 32 + lane) * (BN + 4);
#pragma unroll 1
    for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += 16) {
      uint32_t v[16];
      if (ok) {
        tmem_ld16(acc + c, v);
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = 0u;
      }
#pragma unroll
      for (int k = 0; k < 16; k += 4)
        *reinterpret_cast<uint4*>(part + c + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    }
    __syncwarp();
  } else if (!JOIN && warp >= 4) {
    // ------------------------------------------------------------ results
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    uint8_t* to = smem + L::OFF_STORE + (warp - 4) * kBoxBytes;
    const uint32_t freed = cluster_address(smem_u32(&acc_free[0]), leader);
    const int per = p.out_f32 ? 16 : 32;  // columns of a box
    const int n_boxes = BN / 2 / per;     // of a warp
    bool ok = aligned;
    int j = 0;
    for (int t = tile0; t < n_tiles; t += tile_step) {
      int tp, tq;
      tile_at(p, t, &tp, &tq);
      const int row0 = tp * 256 + rank * 128 + quarter * 32;
      for (int first = 0; first < p.blocks; first += p.chunk, ++j) {
        ok = ok && warp_wait(&acc_full[j & 1], (j >> 1) & 1, ctl);
        tc_fence_after();
        const uint32_t acc = tmem + lanes + (j & 1) * (BN - L::OVERLAP);
        const bool add = first > 0;
        if (add && lane == 0) bulk_wait_all();  // the part before is in the output
        __syncwarp();
        // accumulator 0 ends in the overlap, 1 begins with it: its 32 columns are read first, and
        // then the next tile's MMAs go on, into what the chunk before left.  The warps without a
        // part in the overlap say that they are through with that one: they may be far behind the
        // others, where the half of a tile at the edge left these nothing to write.
        const bool backwards = L::OVERLAP && (j & 1) == 0;
        const int frees = !L::OVERLAP ? n_boxes - 1 : (half == 1) == backwards ? L::OVERLAP / per - 1 : -1;
        if (frees < 0) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(freed + 8 * (j & 1));
        }
#pragma unroll 1
        for (int k = 0; k < n_boxes; ++k) {
          const int c0 = half * (BN / 2) + (backwards ? n_boxes - 1 - k : k) * per;
          uint32_t w[16];
          if (!ok) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 0u;
          } else if (p.out_f32) {
            tmem_ld16(acc + c0, w);
            tmem_wait_ld();
          } else {
            uint32_t v[32];
            tmem_ld32(acc + c0, v);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e)
              w[e] = pack_bf16x2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
          }
          if (k == frees) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(freed + 8 * (j & 1));
          }
          const int col0 = tq * BN + c0;
          if (col0 >= p.rows_b || row0 >= p.rows_a) continue;
          if (lane == 0) bulk_wait_read<0>();
          __syncwarp();
          // (the 64-byte swizzle: 16-byte piece e of row r at e ^ (r / 2 % 4))
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(to + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
                make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
          if (p.tma_out) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (add)
                tma_reduce_add_2d(&tm_c, to, col0, row0);
              else
                tma_store_2d(&tm_c, to, col0, row0);
              bulk_commit_group();
            }
          } else {  // rows that do not start at 16 bytes: single elements, a row a turn
            __syncwarp();
            for (int r = 0; r < 32 && row0 + r < p.rows_a; ++r)
              if (lane < per && col0 + lane < p.rows_b) {
                const int at = p.out_f32 ? lane * 4 : lane * 2;
                const uint8_t* from = to + r * 64 + (((at >> 4) ^ ((r >> 1) & 3)) << 4) + (at & 15);
                const long long dst = static_cast<long long>(row0 + r) * p.ld + col0 + lane;
                if (p.out_f32) {
                  float* o = static_cast<float*>(p.out) + dst;
                  const float v = *reinterpret_cast<const float*>(from);
                  *o = add ? *o + v : v;
                } else {
                  static_cast<__nv_bfloat16*>(p.out)[dst] = *reinterpret_cast<const __nv_bfloat16*>(from);
                }
              }
            __syncwarp();
          }
        }
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (JOIN) {
    cluster.sync();  // all parts are there
    int tp, tq;
    tile_at(p, tile0, &tp, &tq);
    const int row0 = tp * 256 + rank * 128;
    join_parts(p, reinterpret_cast<float*>(smem), max(0, min(128, p.rows_a - row0)), BN, row0, tq * BN,
               p.rows_b - tq * BN, leader / 2, pairs, kPairThreads,
               [&](int r) { return 2 * r + static_cast<int>(rank); });
  }
  cluster.sync();  // nobody's shared memory is in use any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// ------------------------------------------------------------------ clusters that share a contraction
//
// Few rows of one operand (16, 32 or 64 of them are the B of 128 of the other's: a token's
// product reads weights), or few tiles and a long contraction: the CTAs of a cluster take
// each a share of the blocks, and each adds up a share of the tile in the order of the ranks.
// Up to 16 rows (SEND) a CTA owns a share of the tile's rows, and all send it their parts of
// these.  More than that is left where it was made and read from there, 16 bytes at a time,
// which takes two more trips through the cluster but moves parts faster (us, sent / read: one
// token x 2304 x 768 3.1 / 3.5; 64 x 7680 x 2560 16.3 / 13.8).
//
// LONG: a CTA's share of more than `chunk` blocks is summed in parts here too.  Two accumulators
// take turns, and while the MMAs go on with one, the warps that read results add the other to a
// sum in tensor memory beside them, which takes no time of its own (16 x 19456 x 16384 in fp32, 128
// blocks: 56.5 us in two parts and in one).  A kernel of its own, for what the code costs where
// there is one part (one token x 2304 x 768 3.2 us, with it 3.5).

template <int BN, bool LONG>
struct JoinLayout {
  static constexpr bool SEND = BN == 16;
  static constexpr int B = BN * kBlock;  // (columns of B: 128 at a time, so BN = 128 there)
  static constexpr int STAGE = kA + B;
  static constexpr int ATOMS = 2;
  static constexpr int SETS = 4;
  static constexpr int STAGES = BN == 128 ? 6 : SEND ? 5 : 4;
  // SEND: parts of the CTA's rows, [ranks][BN][rows] at an odd pitch: 128 to 138 floats a
  // column; else the CTA's part, in the stages' place
  static constexpr int PARTS = SEND ? BN * 138 * 4 : 0;
  static constexpr int OFF_PARTS = SEND ? STAGES * STAGE : 0;
  static constexpr int OFF_SCALE = STAGES * STAGE + (PARTS + 511) / 512 * 512;
  static constexpr int OFF_BAR = OFF_SCALE + SETS * ATOMS * 512;
  static constexpr int ACCS = LONG ? 2 : 1;
  static constexpr int N_BAR = 2 * STAGES + 2 * SETS + 2 * ACCS + 1;
  static constexpr int OFF_MISC = OFF_BAR + N_BAR * 8;
  static constexpr int SMEM = OFF_MISC + 16;
  static_assert(SMEM <= (BN <= 64 ? 233472 / 2 - 1024 : 232448), "shared memory (up to 64: of two CTAs an SM)");
  // columns of tensor memory: the accumulators, the scale words, the sum
  static constexpr int SCALES = ACCS * BN;
  static constexpr int WORDS = 4 * ATOMS;
  static constexpr int SUM = SCALES + SETS * WORDS;
  static constexpr int USED = SUM + (LONG ? BN : 0);
  static constexpr int COLS = USED <= 64 ? 64 : USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
  static_assert(COLS * (BN <= 64 ? 2 : 1) <= 512, "tensor memory (up to 64: of two CTAs an SM)");
  static_assert(((BN + 4) * 128 > 132 * BN ? (BN + 4) * 128 : 132 * BN) * 4 <= STAGES * STAGE, "a part fits");
};

// The rows [r0, r1) of 128 that a rank owns, and their pitch.
struct OwnRows {
  int r0, r1;
  __device__ __forceinline__ OwnRows(int rank, int ranks) : r0(128 * rank / ranks), r1(128 * (rank + 1) / ranks) {}
  __device__ __forceinline__ int pitch() const { return (r1 - r0) | 1; }
};

template <int BN, bool LONG>
__global__ void __launch_bounds__(kThreads, BN <= 64 ? 2 : 1)
    fp8_mm_join_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                       const Fp8MmParams p) {
  using L = JoinLayout<BN, LONG>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* empty = full + L::STAGES;
  uint64_t* sc_full = empty + L::STAGES;
  uint64_t* sc_empty = sc_full + L::SETS;
  uint64_t* acc_full = sc_empty + L::SETS;  // [ACCS]
  uint64_t* acc_free = acc_full + L::ACCS;  // [ACCS]
  uint64_t* done = acc_free + L::ACCS;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC);
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::STAGES; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1);
    for (int s = 0; s < L::SETS; ++s) mbar_init(&sc_full[s], 1), mbar_init(&sc_empty[s], 1);
    for (int s = 0; s < L::ACCS; ++s) mbar_init(&acc_full[s], 1);
    if constexpr (LONG)
      for (int s = 0; s < L::ACCS; ++s) mbar_init(&acc_free[s], 4);
    mbar_init(done, 1);
    *abort_flag = aligned ? 0 : 1;
    fence_mbar_init();
    if (!aligned) atomicOr(p.status, kDevMisaligned);
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_b);
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
  cluster_arrive();  // (this CTA is there)
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
  int tp, tq;
  tile_at(p, blockIdx.x / ranks, &tp, &tq);
  const int kb0 = p.blocks * rank / ranks, kb1 = p.blocks * (rank + 1) / ranks;
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    // ------------------------------------------------------------ tiles of A and B
    if (lane == 0 && aligned) {
      const int n = skips_loads(p.debug_skip_q) ? 0 : kb1 - kb0;
      int i = 0;
      for (; i < n; ++i) {
        const int st = i % L::STAGES, k = (kb0 + i) * kBlock;
        if (!mbar_wait(&empty[st], ((i / L::STAGES) & 1) ^ 1, ctl)) break;
        uint8_t* a = smem + st * L::STAGE;
        mbar_arrive_expect_tx(&full[st], L::STAGE);
        if (p.a_columns)
          tma_load_2d(a, &tm_a, &full[st], tp * 128, k);
        else
          tma_load_2d(a, &tm_a, &full[st], k, tp * 128);
        if (p.b_columns)
          tma_load_2d(a + kA, &tm_b, &full[st], tq * BN, k);
        else
          tma_load_2d(a + kA, &tm_b, &full[st], k, tq * BN);
      }
      // every copy has landed before the CTA goes
      for (int k = max(0, i - L::STAGES); k < i; ++k)
        drain_wait(&full[k % L::STAGES], (k / L::STAGES) & 1, p.budget_ns);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    const uint32_t idesc = idesc_mxf8(128, BN, p.a_columns, p.b_columns);
    const uint32_t a_step = p.a_columns ? 256u : 2u, b_step = p.b_columns ? 256u : 2u;
    const uint32_t a0 = sdesc_sw128(smem_u32(smem), 128 * kBlock);
    const uint32_t sc0 = smem_u32(smem + L::OFF_SCALE);
    bool ok = aligned;
    int part = 0, first = 0;  // and the block that it begins with
    for (int i = 0; i < kb1 - kb0; ++i) {
      if constexpr (LONG) {
        if (i - first == p.chunk) {
          umma_commit(&acc_full[part & 1]);
          ++part;
          first = i;
          // this accumulator's part of two before has been read
          if (part > 1) ok = warp_wait(&acc_free[part & 1], ((part >> 1) - 1) & 1, ctl);
          if (!ok) break;
          tc_fence_after();
        }
      }
      const int in = i % kGroup, g = i / kGroup, set = g % L::SETS;
      const uint32_t words = tmem + L::SCALES + set * L::WORDS;
      if (in == 0) {
        ok = ok && warp_wait(&sc_full[set], (g / L::SETS) & 1, ctl);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int a = 0; a < L::ATOMS; ++a) tmem_copy_scales(words + 4 * a, sc0 + (set * L::ATOMS + a) * 512);
      }
      const int st = i % L::STAGES;
      ok = ok && warp_wait(&full[st], (i / L::STAGES) & 1, ctl);
      if (!ok) break;
      tc_fence_after();
      const uint32_t a = a0 + st * (L::STAGE >> 4);
      umma_mx4(tmem + (part & 1) * BN, a, a + (kA >> 4), a_step, b_step, idesc | idesc_scale_byte(in), words, words + 4,
               i > first);
      umma_commit(&empty[st]);
      if (in == kGroup - 1) umma_commit(&sc_empty[set]);
    }
    umma_commit(ok ? &acc_full[part & 1] : done);
    if (!ok) drain_wait(done, 0, p.budget_ns);  // what was issued ends before the CTA goes
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------ scale words
    // (a word of four blocks starts at a multiple of four)
    auto way = [&](const Fp8Scales& z) { return z.read == Fp8Read::kWords && kb0 % 4 ? Fp8Read::kBytes : z.read; };
    with_way(way(p.a_scales), [&](auto wa) {
      with_way(way(p.b_scales), [&](auto wb) {
        for (int kb = kb0, g = 0; kb < kb1 && aligned; kb += kGroup, ++g) {
          const int set = g % L::SETS;
          RawScales<decltype(wa)::value> a;
          RawScales<decltype(wb)::value> b;
          a.load(p.a_scales, tp * 128, p.rows_a, kb, kb1);
          b.load(p.b_scales, tq * BN, p.rows_b, kb, kb1);
          if (!warp_wait(&sc_empty[set], ((g / L::SETS) & 1) ^ 1, ctl)) break;
          uint8_t* to = smem + L::OFF_SCALE + set * L::ATOMS * 512;
          a.store(to);
          b.store(to + 512);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_full[set]);
        }
      });
    });
    __syncwarp();
  } else if (warp >= 4) {
    // ------------------------------------------------------------ this CTA's part
    const int row = (warp - 4) * 32 + lane;
    int owner = row * ranks / 128;
    if (OwnRows(owner, ranks).r1 <= row) ++owner;
    const OwnRows own(owner, ranks);
    [[maybe_unused]] const uint32_t to = cluster_address(smem_u32(smem + L::OFF_PARTS), owner) +
                                         4 * (rank * BN * own.pitch() + row - own.r0);
    [[maybe_unused]] float* part = reinterpret_cast<float*>(smem);
    const int n = min(BN, p.rows_b - tq * BN);
    const uint32_t acc = tmem + (static_cast<uint32_t>((warp - 4) * 32) << 16);
    const int last = LONG ? (kb1 - kb0 - 1) / p.chunk : 0;
    // 16 columns of part k, with the sum of those before it
    auto read = [&](int k, int c, uint32_t (&v)[16]) {
      tmem_ld16(acc + (k & 1) * BN + c, v);
      if (!LONG || k == 0) {
        tmem_wait_ld();
        return;
      }
      uint32_t s[16];
      tmem_ld16(acc + L::SUM + c, s);
      tmem_wait_ld();
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(s[e]) + __uint_as_float(v[e]));
    };
    bool ok = aligned;
    for (int k = 0; k < last && ok; ++k) {
      ok = warp_wait(&acc_full[k & 1], (k >> 1) & 1, ctl);
      if (!ok) break;
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < n; c += 16) {
        uint32_t v[16];
        read(k, c, v);
        tmem_st16(acc + L::SUM + c, v);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_free[k & 1]);
    }
    ok = ok && warp_wait(&acc_full[last & 1], (last >> 1) & 1, ctl);
    tc_fence_after();
    cluster_wait();  // all CTAs are there
#pragma unroll 1
    for (int c = 0; c < n; c += 16) {
      uint32_t v[16];
      if (ok) {
        read(last, c, v);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = 0u;
      }
      if constexpr (L::SEND) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (c + k < n) store_cluster(to + 4 * (c + k) * own.pitch(), v[k]);
      } else if (p.swap) {
#pragma unroll
        for (int k = 0; k < 16; ++k) part[(c + k) * 132 + row] = __uint_as_float(v[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 16; k += 4)
          *reinterpret_cast<uint4*>(part + row * (BN + 4) + c + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
      }
    }
    __syncwarp();
  }
  if (warp < 4) cluster_wait();

  // ------------------------------------------------------------ the sums of this CTA's share
  tc_fence_before();
  cluster_arrive();
  cluster_wait();
  if constexpr (L::SEND) {
    const OwnRows own(rank, ranks);
    const int pitch = own.pitch(), rows = min(own.r1, p.rows_a - tp * 128) - own.r0, n = min(BN, p.rows_b - tq * BN);
    const float* parts = reinterpret_cast<const float*>(smem + L::OFF_PARTS);
    // swapped: a row of the output is a row of B, and runs over A's rows
    const int inner = p.swap ? rows : n, outer = p.swap ? n : rows;
    const long long o0 = p.swap ? tq * BN : tp * 128 + own.r0, i0 = p.swap ? tp * 128 + own.r0 : tq * BN;
    const int wide = inner > 32 ? 64 : 32;  // threads to a row of the output
    for (int o = threadIdx.x / wide; o < outer; o += kThreads / wide)
      for (int i = threadIdx.x % wide; i < inner; i += wide) {
        const float* at = parts + (p.swap ? o : i) * pitch + (p.swap ? i : o);
        float s = at[0];
        for (int r = 1; r < ranks; ++r) s += at[r * BN * pitch];
        const long long dst = (o0 + o) * p.ld + i0 + i;
        if (p.out_f32)
          static_cast<float*>(p.out)[dst] = s;
        else
          static_cast<__nv_bfloat16*>(p.out)[dst] = __float2bfloat16(s);
      }
  } else {
    const int inner = p.swap ? 128 : BN;
    const int o0 = p.swap ? tq * BN : tp * 128, i0 = p.swap ? tp * 128 : tq * BN;
    const int outer = min(p.swap ? BN : 128, (p.swap ? p.rows_b : p.rows_a) - o0);
    const int in_n = (p.swap ? p.rows_a : p.rows_b) - i0;
    join_parts(p, reinterpret_cast<float*>(smem), outer, inner, o0, i0, in_n, rank, ranks, kThreads,
               [](int r) { return r; });
    cluster_arrive();  // shared memory stays until all have read it
    cluster_wait();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, L::COLS);
  }
}

// ------------------------------------------------------------------ launches

// The attributes of a launch in clusters of `ranks` CTAs.
struct ClusterConfig {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[2];
  ClusterConfig(int blocks, int threads, int ranks, int smem, cudaStream_t s) {
    pdl_config(cfg, attr[0], dim3(blocks), dim3(threads), smem, s);
    cudaLaunchAttribute& c = attr[cfg.numAttrs++];
    c.id = cudaLaunchAttributeClusterDimension;
    c.val.clusterDim.x = ranks;
    c.val.clusterDim.y = c.val.clusterDim.z = 1;
  }
  ClusterConfig(const ClusterConfig&) = delete;  // (cfg points into it)
};

// ranks: CTAs of a cluster
template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, OncePerDevice& prepared, int dev, int blocks, int threads, int ranks, int smem,
                   cudaStream_t s, const Args&... args) {
  const cudaError_t e = prepared(
      dev, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  if (e != cudaSuccess) return e;
  const ClusterConfig c(blocks, threads, ranks, smem, s);
  return cudaLaunchKernelEx(&c.cfg, kernel, args...);
}

template <int BN, bool JOIN>
cudaError_t run_pair(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const Fp8MmParams& p, int dev,
                     cudaStream_t s) {
  static OncePerDevice prepared;
  const int tiles = p.tiles_p * p.tiles_q, most = p.ctas / 2, pairs = JOIN ? p.splits : 1;
  return launch(fp8_mm_pair_kernel<BN, JOIN>, prepared, dev, 2 * (JOIN ? tiles * pairs : tiles < most ? tiles : most),
                kPairThreads, 2 * pairs, PairLayout<BN>::SMEM, s, ta, tb, tc, p);
}

template <int BN, bool LONG>
cudaError_t run_join(const CUtensorMap& ta, const CUtensorMap& tb, const Fp8MmParams& p, int dev, cudaStream_t s) {
  static OncePerDevice prepared;
  return launch(fp8_mm_join_kernel<BN, LONG>, prepared, dev, p.tiles_p * p.tiles_q * p.splits, kThreads, p.splits,
                JoinLayout<BN, LONG>::SMEM, s, ta, tb, p);
}

}  // namespace

cudaError_t fp8_clusters(int r, int dev, int* n) {
  static std::atomic<int> known[kMaxDevices][kFp8Splits + 1];  // one more than there are
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::atomic<int>& here = known[dev][r];
  *n = here.load(std::memory_order_relaxed) - 1;
  if (*n >= 0) return cudaSuccess;
  const auto kernel = fp8_mm_join_kernel<128, false>;
  constexpr int smem = JoinLayout<128, false>::SMEM;
  const ClusterConfig c(r, kThreads, r, smem, nullptr);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(n, kernel, &c.cfg);
  if (e == cudaSuccess)
    here.store(*n + 1, std::memory_order_relaxed);
  else
    cudaGetLastError();
  return e;
}

cudaError_t launch_fp8_mm(int bn, bool join, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc,
                          const Fp8MmParams& p, int dev, cudaStream_t s) {
  if (join) {
    const bool parts = (p.blocks + p.splits - 1) / p.splits > p.chunk;
    if (bn == 16) return parts ? run_join<16, true>(ta, tb, p, dev, s) : run_join<16, false>(ta, tb, p, dev, s);
    if (bn == 32) return parts ? run_join<32, true>(ta, tb, p, dev, s) : run_join<32, false>(ta, tb, p, dev, s);
    if (bn == 64) return parts ? run_join<64, true>(ta, tb, p, dev, s) : run_join<64, false>(ta, tb, p, dev, s);
    return parts ? run_join<128, true>(ta, tb, p, dev, s) : run_join<128, false>(ta, tb, p, dev, s);
  }
  if (bn == 128) return run_pair<128, false>(ta, tb, tc, p, dev, s);
  if (p.splits > 1) return run_pair<256, true>(ta, tb, tc, p, dev, s);
  return run_pair<256, false>(ta, tb, tc, p, dev, s);
}

}  // namespace mw
