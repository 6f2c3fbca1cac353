// Cross attention forward on sm_103a: blocks of 2 x 128 query rows against an
// encoder's states, all of which (up to the sample's valid number) every row sees.
//
//   S = Q K^T, P = exp2(scale log2e S - m), O = sum over key tiles of P V / l,
//   LSE = (m + log2 l) ln 2
//
// There is no order among the rows, so the query heads that share a head of K
// and V are one sequence of rows.  An encoder's states are few next to a video's
// tokens (a prompt is one to four key tiles), so a block is short and what
// surrounds its key tiles counts: the CTAs are persistent, one an SM, and every
// role runs through the blocks without a stop.  The next block's Q and K/V tiles
// are loaded, and its first S is computed, while the softmax warps finish the
// last one; they take O into registers, hand its tensor memory back, and store
// rows while the next block's MMAs run.  What bounds a step is the chain from S through
// softmax and P to the next S (d = 64: 2300 cycles, of which S to registers 350, P 1600),
// not the exponentials (1024 cycles at 32 a clock) or the MMAs (1024; d = 128 2048 of
// 3070).  Steps of 64 keys with two S in flight were slower (d = 64 1.16 -> 1.59 us, 128
// 1.65 -> 1.88): half of the softmax is latency that does not shrink with the step.
// Measured, 24 query and 40 key tiles a head: d = 64 1.17, 72 1.24, 128 1.58 us a step of
// 256 rows x 128 keys (128: 1.6 PFLOP/s over the SMs); two key tiles 2.02, 2.62, 2.69.
//
// Roles (384 threads):
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (one thread per row = TMEM lane)
//   warp 8           TMA producer
//   warps 9, 10      tcgen05 issuers: of query tile 0 and of tile 1 (d > 80: 9 of both)
//   warp 11          V tiles that end inside the valid states: rows past them are
//                    zeroed (their weights are 0, but what they hold may be NaN)
// TMEM: S_t at column 128 t, O_t at 256 + DM t; P_t, bf16, over S_t, its second half in
// columns of its own where there is room.  The row sums are of the weights before their
// rounding to bf16 (the block-causal forward takes those after it), in 32 bits: LSE is as
// exact as S, and the backward's P with it.  O is divided by the same sum, so that the mean
// rounding of a row's weights, 2^-9 at most and less over many states, scales what its values
// have in common: within O's own rounding to bf16.  (The form for few rows keeps both sums:
// a second one here would lengthen the chain that bounds a step.)
#include <type_traits>

#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

// D: width of the shared-memory tiles; DM <= D: the columns the MMAs cover
template <int D, int DM>
struct Layout {
  static constexpr int QT = kFwdQTiles;
  static constexpr int REG = D / 64;  // 64-column swizzle regions per row
  static constexpr int REGION_BYTES = kTileRows * 128;
  static constexpr int TILE_BYTES = REG * REGION_BYTES;
  static constexpr int STAGES = (D == 64) ? 3 : 2;
  static constexpr int QBUFS = (D == 64) ? 2 : 1;  // blocks of Q in shared memory
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + QBUFS * QT * TILE_BYTES;
  static constexpr int OFF_V = OFF_K + STAGES * TILE_BYTES;
  static constexpr int OFF_BOX = OFF_V + STAGES * TILE_BYTES;
  static constexpr int BOX_BYTES = 32 * 128;  // O leaves through TMA stores, 32 x 64 a warp
  static constexpr int OFF_BAR = OFF_BOX + 8 * BOX_BYTES;
  // P's second half has columns of its own (d <= 80): S of the next tile is computed once
  // P's first half is used.  (Both halves in columns of their own, d = 64, and S once this
  // one is in registers: 1.21 -> 1.30 us a step.)
  static constexpr bool SPLIT_P = 256 + DM * QT + 32 * QT <= 512;
  // A warp a query tile issues MMAs, or one both: 24 x 40 tiles, two / one: d = 72 1.31 /
  // 1.46 us a step, 128 (where the tensor core has more to do) 2.03 / 1.60
  static constexpr int ISSUERS = DM < 128 ? QT : 1;
  // A block's O leaves after the first softmax of the next block, while that one's MMAs
  // run.  Where P overwrites all of S, S of the tile after that would wait for it: there
  // O leaves at the end of its own block (us a step of 2 x 128 rows, blocks of two key
  // tiles: d = 64 2.31 -> 2.18, 72 2.98 -> 2.75; 128 2.81, 2.95 if deferred)
  static constexpr bool DEFER = SPLIT_P;
  static constexpr int SLOTS = 4;  // blocks announced ahead
  static constexpr int NBAR = 2 * QBUFS + 5 * STAGES + 5 * QT + 2 * SLOTS;
  static constexpr int OFF_SLOTS = (OFF_BAR + NBAR * 8 + 15) / 16 * 16;
  static constexpr int OFF_MISC = OFF_SLOTS + SLOTS * 32;
  static constexpr int BYTES = OFF_MISC + 16;
  static_assert(BYTES <= 232448, "shared memory");
  static constexpr uint32_t S_COL(int t) { return 128u * t; }
  static constexpr uint32_t O_COL(int t) { return 256u + DM * t; }
  static constexpr uint32_t P_COL(int t, int half) {
    return half == 0 ? S_COL(t) : SPLIT_P ? 256u + DM * QT + 32u * t : S_COL(t) + 32u;
  }
  static constexpr int THREADS = 384;
  // registers per thread after the re-split: 2 * 128 * S + 128 * C is exactly the
  // launch's 384 * 168
  static constexpr int REGS_LAUNCH = 168;
  static constexpr int REGS_SOFTMAX = (D == 64) ? 224 : 208;
  static constexpr int REGS_CONTROL = (D == 64) ? 56 : 88;
  static_assert(2 * 128 * REGS_SOFTMAX + 128 * REGS_CONTROL == THREADS * REGS_LAUNCH,
                "register re-split must hand out exactly the launch's registers");
};

// A block of a CTA, as the producer announces it to the other roles.
struct Block {
  int bh;        // head; below 0: no more blocks
  int r0;        // first row
  int split;     // range of key tiles
  int row0, n;   // its first key row, its key tiles
  int len;       // valid states
  __device__ __forceinline__ bool present(int t, int M) const { return r0 + kTileRows * t < M; }
  // V tile i of the block passes through a helper warp: it has rows that count as
  // nothing but may hold anything (past S are zeros)
  __device__ __forceinline__ bool helped(int i, int S) const {
    return row0 + (i + 1) * kTileRows > len && len < S;
  }
};

// Block x of the launch.
__device__ __forceinline__ Block block_of(const XattnTcParams& p, int x) {
  Block b;
  b.split = 0;
  if (p.num_splits > 1) {
    const int y = x / p.num_splits;
    b.split = x - y * p.num_splits;
    x = y;
  }
  b.bh = x / p.n_qblocks;
  b.r0 = (x - b.bh * p.n_qblocks) * kFwdBlockRows;
  b.len = p.kv_len ? min(max(p.kv_len[b.bh / p.heads], 0), p.S) : p.S;
  b.n = (b.len + kTileRows - 1) / kTileRows;
  b.row0 = 0;
  if (p.num_splits > 1) {  // ranges that differ by a tile at most
    const int base = b.n / p.num_splits, rest = b.n - base * p.num_splits;
    b.row0 = (b.split * base + min(b.split, rest)) * kTileRows;
    b.n = base + (b.split < rest);
  }
  return b;
}

template <int D, int DM>
__global__ void __launch_bounds__(Layout<D, DM>::THREADS, 1)
    xattn_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
                     const __grid_constant__ XattnTcParams p) {
  using L = Layout<D, DM>;
  constexpr int QT = L::QT, NS = L::STAGES, NQ = L::QBUFS;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;

  // Row `row` of head bh gets its value: bf16 O and LSE, or a split's partials.
  auto store_lse = [&](const Block& w, int row, float lse) {
    const size_t at = static_cast<size_t>(w.bh) * p.M + row;
    if (p.num_splits > 1)
      p.lse_part[static_cast<size_t>(w.split) * p.BH * p.M + at] = lse;
    else if (p.lse)
      p.lse[at] = lse;
  };
  auto store_nothing = [&](const Block& w, int row, float lse) {
    if (p.num_splits == 1) {  // (the combine does not read O of a split that saw nothing)
      uint4* dst = reinterpret_cast<uint4*>(p.o + (static_cast<size_t>(w.bh) * p.M + row) * p.d);
      for (int c = 0; c < p.d / 8; ++c) dst[c] = make_uint4(0u, 0u, 0u, 0u);
    }
    store_lse(w, row, lse);
  };

  // in all blocks of this CTA; a range of a row's keys takes the others along (+inf)
  auto leave_nothing = [&]() {
#pragma unroll 1
    for (int x = blockIdx.x; x < p.items; x += gridDim.x) {
      const Block w = block_of(p, x);
      const int row = w.r0 + static_cast<int>(threadIdx.x);
      if (threadIdx.x < kFwdBlockRows && row < p.M) store_nothing(w, row, p.num_splits > 1 ? INFINITY : -INFINITY);
    }
  };

  if ((smem_u32(smem) & 1023u) != 0u) {
    // nothing runs without aligned shared memory: report it, and give this CTA's
    // rows a defined result
    if (threadIdx.x == 0) atomicOr(p.status, kDevMisaligned);
    leave_nothing();
    return;  // uniform across the CTA, before any barrier or TMEM use
  }
  uint64_t* q_full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* q_empty = q_full + NQ;
  uint64_t* k_full = q_empty + NQ;
  uint64_t* k_empty = k_full + NS;
  uint64_t* v_full = k_empty + NS;
  uint64_t* v_empty = v_full + NS;
  uint64_t* v_raw = v_empty + NS;   // V tile that a helper warp makes ready, then v_full
  uint64_t* s_full = v_raw + NS;
  uint64_t* p_half = s_full + QT;   // first 64 keys of P in TMEM
  uint64_t* p_full = p_half + QT;
  uint64_t* pv_done = p_full + QT;  // PV of a key tile (SPLIT_P), of a block's last one (else)
  uint64_t* o_free = pv_done + QT;  // O of a block is in registers
  uint64_t* b_full = o_free + QT;   // a block is announced, and
  uint64_t* b_empty = b_full + L::SLOTS;  // read by all roles
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC + 4);

  if (threadIdx.x == 0) {
    for (int b = 0; b < NQ; ++b) {
      mbar_init(&q_full[b], 1);
      mbar_init(&q_empty[b], L::ISSUERS);
    }
    for (int s = 0; s < NS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], L::ISSUERS);
      mbar_init(&v_full[s], 1);
      mbar_init(&v_empty[s], L::ISSUERS);
      mbar_init(&v_raw[s], 1);
    }
    for (int t = 0; t < QT; ++t) {
      mbar_init(&s_full[t], 1);
      mbar_init(&p_half[t], 4);
      mbar_init(&p_full[t], 4);
      mbar_init(&pv_done[t], 1);
      mbar_init(&o_free[t], 4);
    }
    for (int b = 0; b < L::SLOTS; ++b) {
      mbar_init(&b_full[b], 1);
      mbar_init(&b_empty[b], 11);  // the other warps
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 8 && lane == 0) {
    prefetch_tmap(&tm_q);
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
    prefetch_tmap(&tm_o);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  constexpr uint32_t tmem = 0;  // the allocation of all 512 columns can only start at 0
  const WaitCtl ctl{abort_flag, p.status, p.budget_ns};
  pdl_wait();  // global memory only from here on

  uint8_t* sQ = smem + L::OFF_Q;
  uint8_t* sK = smem + L::OFF_K;
  uint8_t* sV = smem + L::OFF_V;
  int4* slots = reinterpret_cast<int4*>(smem + L::OFF_SLOTS);
  // The next block, for a whole warp (its fields agree over the lanes: the shuffles
  // tell the compiler, which then works in uniform registers).
  int turn = 0;
  Block w;
  auto read_block = [&]() {  // (announced)
    const int slot = turn % L::SLOTS;
    ++turn;
    const int4 a = slots[2 * slot], b = slots[2 * slot + 1];
    w.bh = __shfl_sync(0xffffffffu, a.x, 0);
    w.r0 = __shfl_sync(0xffffffffu, a.y, 0);
    w.split = __shfl_sync(0xffffffffu, a.z, 0);
    w.row0 = __shfl_sync(0xffffffffu, a.w, 0);
    w.n = __shfl_sync(0xffffffffu, b.x, 0);
    w.len = __shfl_sync(0xffffffffu, b.y, 0);
    if (lane == 0) mbar_arrive(&b_empty[slot]);
    return w.bh >= 0;
  };
  auto next_block = [&]() {
    return warp_wait(&b_full[turn % L::SLOTS], (turn / L::SLOTS) & 1, ctl) && read_block();
  };
  // the next one that has keys
  auto next_keys = [&]() {
    do {
      if (!next_block()) return false;
    } while (w.n == 0);
    return true;
  };

  if (warp >= 8) {
  regs_dec<L::REGS_CONTROL>();
  if (warp == 8) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int nq = 0, nk = 0, nv = 0;  // blocks, K and V tiles so far
      uint32_t raw = 0, raws = 0;  // per stage: its last V tile went to a helper; parity of those
      bool ok = true;
      Block next = block_of(p, blockIdx.x);
      for (int x = blockIdx.x; ok; x += gridDim.x, ++turn) {
        const int slot = turn % L::SLOTS;
        if (!(ok = mbar_wait(&b_empty[slot], ((turn / L::SLOTS) & 1) ^ 1, ctl))) break;
        w = next;
        if (x >= p.items) w.bh = -1;
        slots[2 * slot] = make_int4(w.bh, w.r0, w.split, w.row0);
        slots[2 * slot + 1] = make_int4(w.n, w.len, 0, 0);
        mbar_arrive(&b_full[slot]);  // (releases the stores above)
        if (w.bh < 0) break;
        // the block after it, its Q on the way into L2 (a block of one key tile is over
        // in less than HBM's latency)
        if (x + static_cast<int>(gridDim.x) < p.items) {
          next = block_of(p, x + gridDim.x);
          if (next.n > 0)
            for (int t = 0; t < QT; ++t)
              if (next.present(t, p.M))
                for (int r = 0; r < L::REG; ++r) tma_prefetch_3d(&tm_q, 64 * r, next.r0 + kTileRows * t, next.bh);
        }
        if (w.n == 0) continue;
        const int qb = nq % NQ;
        if (!(ok = mbar_wait(&q_empty[qb], ((nq / NQ) & 1) ^ 1, ctl))) break;
        if (!skips_loads(p.debug_skip_q)) {
          const int tiles = w.present(1, p.M) ? QT : 1;
          mbar_arrive_expect_tx(&q_full[qb], tiles * L::TILE_BYTES);
          for (int t = 0; t < tiles; ++t)
            for (int r = 0; r < L::REG; ++r)
              tma_load_3d(sQ + (qb * QT + t) * L::TILE_BYTES + r * L::REGION_BYTES, &tm_q, &q_full[qb],
                          64 * r, w.r0 + kTileRows * t, w.bh);
          ++nq;
        }
        for (int i = 0; i < w.n; ++i) {
          const int st = nk % NS;
          const uint32_t ph = ((nk / NS) & 1) ^ 1;
          const int row0 = w.row0 + i * kTileRows;
          if (!(ok = mbar_wait(&k_empty[st], ph, ctl))) break;
          mbar_arrive_expect_tx(&k_full[st], L::TILE_BYTES);
          for (int r = 0; r < L::REG; ++r)
            tma_load_3d(sK + st * L::TILE_BYTES + r * L::REGION_BYTES, &tm_k, &k_full[st], 64 * r, row0, w.bh);
          ++nk;
          if (!(ok = mbar_wait(&v_empty[st], ph, ctl))) break;
          const bool help = w.helped(i, p.S);
          uint64_t* bar = help ? &v_raw[st] : &v_full[st];
          mbar_arrive_expect_tx(bar, L::TILE_BYTES);
          for (int r = 0; r < L::REG; ++r)
            tma_load_3d(sV + st * L::TILE_BYTES + r * L::REGION_BYTES, &tm_v, bar, 64 * r, row0, w.bh);
          raw = (raw & ~(1u << st)) | (help ? 1u << st : 0u);
          raws ^= help ? 1u << st : 0u;
          ++nv;
        }
      }
      if (*abort_flag || !ok) {
        // let every copy this CTA started land before shared memory goes away
        for (int i = max(0, nq - NQ); i < nq; ++i) drain_wait(&q_full[i % NQ], (i / NQ) & 1, p.budget_ns);
        for (int i = max(0, nk - NS); i < nk; ++i) drain_wait(&k_full[i % NS], (i / NS) & 1, p.budget_ns);
        for (int i = max(0, nv - NS); i < nv; ++i) {
          const int st = i % NS;
          if ((raw >> st) & 1)
            drain_wait(&v_raw[st], ((raws >> st) & 1) ^ 1, p.budget_ns);
          else
            drain_wait(&v_full[st], (i / NS) & 1, p.budget_ns);
        }
      }
    }
  } else if (warp == 9 || (L::ISSUERS > 1 && warp == 10)) {
    // ------------------------------------------------------------ MMA issuers (whole warps)
    constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, false, false);
    constexpr uint32_t idesc_pv = idesc_bf16_f32(128, DM, false, true);
    const uint32_t q_desc = sdesc_sw128(smem_u32(sQ), 16);
    const uint32_t k_desc = sdesc_sw128(smem_u32(sK), 16);
    const uint32_t v_addr = smem_u32(sV);
    auto issue_qk = [&](int t, int qb, int st) {
      const uint32_t qa = sdesc_add(q_desc, (qb * QT + t) * L::TILE_BYTES);
      const uint32_t kb = sdesc_add(k_desc, st * L::TILE_BYTES);
#pragma unroll
      for (int r = 0; r < DM / 64; ++r)
        umma_ss4<2, 2>(tmem + L::S_COL(t), sdesc_add(qa, r * L::REGION_BYTES), sdesc_add(kb, r * L::REGION_BYTES),
                       idesc_qk, r > 0 ? 1u : 0u);
      if constexpr (DM % 64 != 0) {
        static_assert(DM % 64 == 0 || DM == 80, "one more slice");
        umma_ss(tmem + L::S_COL(t), sdesc_add(qa, L::REGION_BYTES), sdesc_add(kb, L::REGION_BYTES), idesc_qk, 1u);
      }
    };
    auto issue_pv = [&](int t, int st, bool acc, int half) {
      const uint32_t vb = sdesc_sw128(v_addr + st * L::TILE_BYTES, L::REGION_BYTES);
      umma_ts4<8, 128>(tmem + L::O_COL(t), tmem + L::P_COL(t, half), sdesc_add(vb, half * 8192), idesc_pv,
                       (acc || half > 0) ? 1u : 0u);
    };
    int nq = 0, nk = 0;       // blocks and key tiles whose S is issued
    // of this warp's query tiles (all; d = 64: one, tile t0)
    constexpr int NT = QT / L::ISSUERS;
    const int t0 = L::ISSUERS == 1 ? 0 : warp - 9;
    int done[NT] = {};    // key tiles whose PV is issued
    int blocks[NT] = {};  // blocks begun
    int i = -1;               // tile of the block in work (none yet)
    bool have[NT] = {};
    w.n = 0;
    bool ok = true, more = true;
    // In turn: S of the next tile, and PV of this one, of which S is there.  Where P
    // leaves S free in time, the next S goes between the halves of the PV.  A block that
    // is not announced yet is waited for only after this PV (a turn without one): blocks
    // without keys may lie in between, which the softmax warps pass only once they have
    // the O that this PV makes.
    while (ok && more) {
      const int st = (nk + NS - 1) % NS;
      const uint32_t ph = ((nk - 1) / NS) & 1;
      const bool any = i >= 0, first_tile = i == 0, last_tile = i + 1 == w.n;
      bool known = true;
      if (!last_tile) {
        ++i;
      } else if (!any) {
        more = next_keys();
        i = 0;
      } else {
        w.n = 0;
        while (more && w.n == 0 && known) {
          known = __all_sync(0xffffffffu, mbar_try_wait(&b_full[turn % L::SLOTS], (turn / L::SLOTS) & 1));
          if (known) more = read_block();
        }
        i = known ? 0 : -1;
      }
      const int st1 = nk % NS;
      const int qb1 = (i == 0 ? nq : nq - 1) % NQ;
      bool waited = false;
      auto next_s = [&](int t) {
        if (!waited) {  // Q (of a new block) and K of the next tile
          waited = true;
          if (i == 0 && !warp_wait(&q_full[qb1], (nq / NQ) & 1, ctl)) return false;
          if (!warp_wait(&k_full[st1], (nk / NS) & 1, ctl)) return false;
          tc_fence_after();
        }
        if (w.present(t, p.M)) {
          issue_qk(t, qb1, st1);
          umma_commit(&s_full[t]);
        }
        return true;
      };
      if (any && !(ok = warp_wait(&v_full[st], ph, ctl))) break;
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const int t = t0 + u;
        if (have[u]) {
          if (!(ok = warp_wait(&p_half[t], done[u] & 1, ctl))) break;
          if (first_tile) {
            // the last block's O is in the softmax warps' registers
            if (blocks[u] > 0 && !(ok = warp_wait(&o_free[t], (blocks[u] - 1) & 1, ctl))) break;
            ++blocks[u];
          }
          tc_fence_after();
          issue_pv(t, st, !first_tile, 0);
        }
        if (L::SPLIT_P && more && known && !(ok = next_s(t))) break;
        if (have[u]) {
          if (!(ok = warp_wait(&p_full[t], done[u] & 1, ctl))) break;
          tc_fence_after();
          issue_pv(t, st, true, 1);
          ++done[u];
          if (L::SPLIT_P || last_tile) umma_commit(&pv_done[t]);
        }
        if (!L::SPLIT_P && more && known && !(ok = next_s(t))) break;
      }
      if (!ok) break;
      if (any) umma_commit(&v_empty[st]);
#pragma unroll
      for (int u = 0; u < NT; ++u) have[u] = more && known && w.present(t0 + u, p.M);
      if (more && known) {
        umma_commit(&k_empty[st1]);
        if (i + 1 == w.n) umma_commit(&q_empty[qb1]);
        nq += i == 0;
        ++nk;
      }
    }
  } else {
    // ------------------------------------------------------------ V tiles made ready
    // Only ragged ones pass through here (warp 11).  A stage's v_raw cannot complete again
    // before the helper has looked: the stage is free for another tile only once the MMAs,
    // which wait for the helper, have read this one.
    int nv = 0;
    uint32_t raws = 0;  // parity of each stage's uses
    bool ok = true;
    while (ok && next_keys()) {
      for (int i = 0; i < w.n; ++i, ++nv) {
        if (warp != 11 || !w.helped(i, p.S)) continue;
        const int st = nv % NS;
        if (!(ok = warp_wait(&v_raw[st], (raws >> st) & 1, ctl))) break;
        raws ^= 1u << st;
        uint8_t* tile = sV + st * L::TILE_BYTES;
        const int limit = w.len - w.row0 - i * kTileRows;
#pragma unroll
        for (int k = 0; k < kTileRows / 32; ++k) {
          const int r = 32 * k + lane;
          if (r >= limit) {
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int c = 0; c < DM / 8; ++c)
              *reinterpret_cast<uint4*>(tile + (c >> 3) * L::REGION_BYTES + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = zero;
          }
        }
        fence_proxy_async_smem();  // the tensor core reads the tile next
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_full[st]);
      }
    }
  }
  } else {
    regs_inc<L::REGS_SOFTMAX>();
    // ------------------------------------------------------------ softmax
    const int t = warp >> 2;
    const int wq = warp & 3;
    const int row_local = t * kTileRows + wq * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(wq * 32) << 16);
    const uint32_t s_addr = lane_base + L::S_COL(t);
    const uint32_t o_addr = lane_base + L::O_COL(t);
    const float sl2 = p.scale_log2;
    int begun = 0;   // blocks of this query tile whose O is out
    int done = 0;    // key tiles of this query tile
    // the block whose O has to leave, and its statistics
    bool pending = false;
    Block pw;
    float pm = 0.f, pl = 0.f;
    while (true) {
      bool ok = true;
      const bool more = next_block();  // (at the end one more turn, for the last block's O)
      if (!more && (*abort_flag || !pending)) break;
      const int row = w.r0 + row_local;
      if (more && w.n == 0) {  // no keys
        if (row < p.M) store_nothing(w, row, -INFINITY);
        __syncwarp();
        continue;
      }
      if (more && !w.present(t, p.M)) continue;
      if (!more) w.n = 1;
      float m_used = -INFINITY;
      float l = 0.f;
      const bool idle = !more || w.r0 + t * kTileRows + wq * 32 >= p.M;  // a warp without rows only keeps step
#pragma unroll 1
      for (int i = 0; i < w.n; ++i, ++done) {
        if (more && !(ok = warp_wait(&s_full[t], done & 1, ctl))) break;
        if (!idle) {
          tc_fence_after();
          float s[128];
          {
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, r[c]);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 128; ++c) s[c] = __uint_as_float(r[c >> 5][c & 31]);
          }
          const int limit = w.len - w.row0 - i * kTileRows;
          if (limit < kTileRows) {
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c >= limit) s[c] = -INFINITY;
          }
          float mq[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) mq[k] = fmaxf(s[k], s[k + 4]);
#pragma unroll
          for (int c = 8; c < 128; c += 8) {
            mq[0] = max3(mq[0], s[c], s[c + 1]);
            mq[1] = max3(mq[1], s[c + 2], s[c + 3]);
            mq[2] = max3(mq[2], s[c + 4], s[c + 5]);
            mq[3] = max3(mq[3], s[c + 6], s[c + 7]);
          }
          const float m_tile = max3(fmaxf(mq[0], mq[1]), mq[2], mq[3]) * sl2;  // scale > 0
          const float m_cand = fmaxf(m_used, m_tile);
          // rescale only when the running maximum grew by more than 2^8: P stays
          // below 256 in between, and the final O / l is exact either way
          const bool need = m_cand > m_used + 8.0f;
          if (__any_sync(0xffffffffu, need)) {
            float alpha = 1.f;
            if (need) {
              alpha = ex2_approx(m_used - m_cand);
              m_used = m_cand;
            }
            l *= alpha;
            if (i > 0) {
              if constexpr (L::SPLIT_P) {  // (else S of this tile implies it)
                if (!(ok = warp_wait(&pv_done[t], (done - 1) & 1, ctl))) break;
                tc_fence_after();
              }
              // exactly the tile's O columns
#pragma unroll 1
              for (int c = 0; c < DM; c += 16) {
                uint32_t r[16];
                tmem_ld16(o_addr + c, r);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * alpha);
                tmem_st16(o_addr + c, r);
              }
              tmem_wait_st();
            }
          }
          const float m_eff = m_used == -INFINITY ? 0.f : m_used;
          const float2 sl2x2 = make_float2(sl2, sl2), negm = make_float2(-m_eff, -m_eff);
          float2 acc = make_float2(0.f, 0.f);
          // P in halves of 64 keys, each stored as a whole; the first is announced while the
          // second is computed
          uint32_t held[16];
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            uint32_t packed[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float2 x = fma2(make_float2(s[32 * g4 + 2 * k], s[32 * g4 + 2 * k + 1]), sl2x2, negm);
              const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
              packed[k] = pack_bf16x2(e.x, e.y);
              acc = add2(acc, e);  // of the weights before their rounding: the LSE is exact
            }
            if (g4 == 2) {
              tmem_wait_st();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&p_half[t]);
              // the previous tile's PV has read the columns of the second half
              if (L::SPLIT_P && done > 0) {
                if (!(ok = warp_wait(&pv_done[t], (done - 1) & 1, ctl))) break;
                tc_fence_after();
              }
            }
            if (g4 & 1) {
              uint32_t half[32];
#pragma unroll
              for (int k = 0; k < 16; ++k) half[k] = held[k], half[16 + k] = packed[k];
              tmem_st32(lane_base + L::P_COL(t, g4 >> 1), half);
            } else {
#pragma unroll
              for (int k = 0; k < 16; ++k) held[k] = packed[k];
            }
          }
          if (!ok) break;
          l += acc.x + acc.y;
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full[t]);
        } else if (more && lane == 0) {
          mbar_arrive(&p_half[t]);
          mbar_arrive(&p_full[t]);
        }
        if constexpr (!L::DEFER) {
          pw = w;
          pm = m_used;
          pl = l;
        }
        if (L::DEFER ? i == 0 && pending : i + 1 == w.n) {
          // ---- a block's O, 64 columns a turn.  It runs once a block, and what runs once
          // waits for its instructions: unrolled it took longer, and with turns of 32
          // columns too (blocks of two key tiles, us a step: d = 64 2.23 -> 2.07, 72 2.83 ->
          // 2.70, 128 2.87 -> 2.74).
          if (!(ok = warp_wait(&pv_done[t], (L::DEFER ? done - 1 : begun) & 1, ctl))) break;
          ++begun;
          tc_fence_after();
          const int prow = pw.r0 + row_local;
          const bool pidle = prow - lane >= p.M;
          const bool nonzero = !(pl == 0.f);  // (a NaN is a result, not a row without states)
          const float inv_l = nonzero ? 1.f / pl : 0.f;
          const size_t at = static_cast<size_t>(pw.bh) * p.M + prow;
          constexpr int kChunks = (DM + 63) / 64;
          const bool all_nonzero = __all_sync(0xffffffffu, nonzero);
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            uint32_t r[2][32];  // (the last chunk's columns past the caller's are not stored)
            tmem_ld32(o_addr + 64 * c, r[0]);
            tmem_ld32(o_addr + 64 * c + 32, r[1]);
            tmem_wait_ld();
            if (c == kChunks - 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&o_free[t]);
            }
            if (pidle || 64 * c >= p.d) continue;
            float2 v[32];
#pragma unroll
            for (int k = 0; k < 32; ++k)
              v[k] = mul2(make_float2(__uint_as_float(r[k >> 4][2 * k & 31]), __uint_as_float(r[k >> 4][(2 * k & 31) + 1])),
                          make_float2(inv_l, inv_l));
            if (!all_nonzero && !nonzero) {
#pragma unroll
              for (int k = 0; k < 32; ++k) v[k] = make_float2(0.f, 0.f);
            }
            if (p.num_splits == 1) {
              // 32 rows of 128 bytes with the 128-byte swizzle: 16-byte chunk k of row i at
              // k ^ (i & 7).  The map clips rows and columns past the caller's.
              uint8_t* stg = smem + L::OFF_BOX + warp * L::BOX_BYTES;
              if (lane == 0) bulk_wait_read<0>();  // the TMA unit has read the box
              __syncwarp();
#pragma unroll
              for (int k = 0; k < 8; ++k)
                *reinterpret_cast<uint4*>(stg + lane * 128 + ((k ^ (lane & 7)) << 4)) =
                    make_uint4(pack_bf16x2(v[4 * k].x, v[4 * k].y), pack_bf16x2(v[4 * k + 1].x, v[4 * k + 1].y),
                               pack_bf16x2(v[4 * k + 2].x, v[4 * k + 2].y), pack_bf16x2(v[4 * k + 3].x, v[4 * k + 3].y));
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&tm_o, stg, 64 * c, prow - lane, pw.bh);
                bulk_commit_group();
              }
            } else if (prow < p.M) {
              float4* dst = reinterpret_cast<float4*>(
                  p.o_part + (static_cast<size_t>(pw.split) * p.BH * p.M + at) * D + 64 * c);
#pragma unroll
              for (int k = 0; k < 16; ++k)
                dst[k] = make_float4(v[2 * k].x, v[2 * k].y, v[2 * k + 1].x, v[2 * k + 1].y);
            }
            __syncwarp();
          }
          if (prow < p.M) {
            const float m_eff = pm == -INFINITY ? 0.f : pm;
            store_lse(pw, prow, nonzero ? (m_eff + __log2f(pl)) * 0.69314718055994530942f : -INFINITY);
          }
          __syncwarp();
          pending = false;
        }
        // (a warp without rows not a tile ahead of the others: their arrivals for this
        // one count first)
        if (L::SPLIT_P && idle && more && !(ok = warp_wait(&pv_done[t], done & 1, ctl))) break;
      }
      if (!ok || !more) break;
      if constexpr (L::DEFER) {
        pending = true;
        pw = w;
        pm = m_used;
        pl = l;
      }
    }
    if (lane == 0) {
      if (*abort_flag) bulk_wait_all();  // (these rows are written once more below)
      bulk_wait_read<0>();               // the boxes are read before shared memory goes
    }
    __syncwarp();
    pdl_trigger();  // the next kernel (the split combine) may be scheduled now
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (*abort_flag) leave_nothing();  // a wait gave up: the rows get a defined result
}

template <int D, int DM>
cudaError_t launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                   const CUtensorMap& to, const XattnTcParams& p, int dev, int sms, cudaStream_t s) {
  using L = Layout<D, DM>;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(dev, [] {
    // the in-kernel register re-split assumes the launch register count; with any
    // other its setmaxnreg.inc could never be satisfied, so refuse
    cudaFuncAttributes fa;
    const cudaError_t e0 = cudaFuncGetAttributes(&fa, xattn_fwd_kernel<D, DM>);
    if (e0 != cudaSuccess) return e0;
    if (fa.numRegs != L::REGS_LAUNCH) return cudaErrorInvalidKernelImage;
    return cudaFuncSetAttribute(xattn_fwd_kernel<D, DM>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(p.items < sms ? p.items : sms), dim3(L::THREADS), L::BYTES, s);
  return cudaLaunchKernelEx(&cfg, xattn_fwd_kernel<D, DM>, tq, tk, tv, to, p);
}

}  // namespace

cudaError_t launch_xattn_tc(int d, int dm, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                            const CUtensorMap& to, const XattnTcParams& p, int dev, int sms, cudaStream_t s) {
  if (d == 64) return launch<64, 64>(tq, tk, tv, to, p, dev, sms, s);
  if (dm == 80) return launch<128, 80>(tq, tk, tv, to, p, dev, sms, s);
  return launch<128, 128>(tq, tk, tv, to, p, dev, sms, s);
}

}  // namespace mw
