// Cross attention backward on sm_103a: the gradients of queries against an
// encoder's states.
//
// A sweep takes one key tile through a range of query tiles, with dK and dV of the
// tile in tensor memory; dQ of every step goes out.  Two orders:
//   query-major  a piece of work is a run of query tiles, taken through all key tiles of
//                its head, and every CTA takes an equal share of all steps; dK and dV are
//                added to accumulators at the end of a sweep.  With one key tile dQ is
//                written as it is; else (d = 64 only) the first key tile's is stored, the
//                others' added while the run is still in L2, the last one's read back
//                and written in bf16: no pass over accumulators in HBM.
//   key-major    a piece is one key tile, taken through all query tiles (or a few
//                ranges of them).  The key tiles of a head run side by side, so that dQ,
//                zeroed before, is added up in L2 and becomes bf16 afterwards; dK and dV
//                are written as they are (one range) or added to accumulators.
// Per step (128 keys x 128 queries), as in the block-causal backward, whose arrangement
// of tensor memory and roles this kernel shares:
//   S^T = K Q^T, dP^T = V dO^T              (tcgen05 -> TMEM)
//   P^T = exp2(scale log2e S^T - LSE2), dS^T = P^T (dP^T - D)   (registers)
//   dV += P^T dO, dK += dS^T Q, dQ = dS K   (tcgen05)
//   dQacc += dQ                             (TMA reduce-add of fp32 boxes)
// d = 64: LSE and D enter S^T and dP^T through a tf32 MMA each.  P and dS are rounded to
// bf16 for their products, D comes from O in bf16; all sums are fp32.
//
// Bound by the chain S -> P -> dS -> dK, dQ of a step, and at d = 64 by instructions that
// have to be fetched (3.0 stalls an issue), at 128 by the tensor core's share of 49%
// besides.  Measured, us a step and an SM, 24 query x 40 key tiles a head (key-major):
// d = 64 1.35, 72 2.03, 128 2.21, where the products alone take 0.84, 1.05 and 1.68 at the
// measured tensor rate; 40 x 2 tiles 1.94 (query-major), 2.16, 2.67.
//
// Roles (512 threads): warps 0-7 P/dS (two warpgroups, one half of the query
// columns each, one key row per thread), warps 8-11 drain (dQ after every step, dK
// and dV after a sweep, while the next one starts), warp 12 TMA producer, warps 13
// and 14 MMA issuers (13: S^T, dV, dP^T; 14: dK, dQ), warp 15 K and V tiles that end
// inside the valid states (what the rows past them hold, NaN included, becomes 0).
#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

// D: width of the shared-memory tiles; DM <= D: the columns the MMAs cover
template <int D, int DM>
struct Layout {
  static constexpr int QN = bwd_q_rows(D);           // query rows per step
  static constexpr bool DQT = (D == 128);            // dQ produced transposed
  static constexpr int CW = QN / 2;                  // query columns per P/dS warpgroup
  static constexpr int REG = D / 64;                 // 64-column swizzle regions per row
  static constexpr int KREGION = kTileRows * 128;
  static constexpr int QREGION = QN * 128;
  static constexpr int KTILE = REG * KREGION;
  static constexpr int QTILE = REG * QREGION;
  static constexpr int QSTAGES = (D == 64) ? 3 : 2;
  static constexpr int DOSTAGES = (D == 64) ? 3 : 1;
  static constexpr int DS_BYTES = (QN / 64) * KREGION;  // dS^T: 128 key rows x QN columns
  static constexpr int BOX_BYTES = 32 * 32 * 4;
  // staging boxes per drain warp: two for sums, d = 64 a third that dQ in bf16 leaves from
  static constexpr int BOXES = 2;
  static constexpr int OUT_BYTES = (D == 64) ? 4 * BOX_BYTES : 0;
  static constexpr bool FOLD = (D == 64);            // LSE and D through tf32 MMAs
  static constexpr int BIAS_BYTES = FOLD ? QN * 32 : 0;
  static constexpr int QSTRIDE = QTILE + BIAS_BYTES;
  static constexpr int VEC_BYTES = FOLD ? 0 : QN * 4;
  static constexpr int ONES_BYTES = FOLD ? 512 : 0;
  static constexpr int OFF_K = 0;
  static constexpr int OFF_V = OFF_K + KTILE;
  static constexpr int OFF_Q = OFF_V + KTILE;
  static constexpr int OFF_DO = OFF_Q + QSTAGES * QSTRIDE;
  static constexpr int OFF_DS = OFF_DO + DOSTAGES * QTILE;
  static constexpr int OFF_STG = OFF_DS + DS_BYTES;
  static constexpr int OFF_OUT = OFF_STG + BOXES * 4 * BOX_BYTES;
  static constexpr int OFF_LSE = OFF_OUT + OUT_BYTES;
  static constexpr int OFF_DELTA = OFF_LSE + QSTAGES * VEC_BYTES;
  static constexpr int OFF_ONES = OFF_DELTA + 2 * VEC_BYTES;
  static constexpr int OFF_BAR = OFF_ONES + ONES_BYTES;
  static constexpr int SLOTS = 4;  // sweeps announced ahead
  static constexpr int NBAR = 6 + 2 * (QSTAGES + DOSTAGES) + 11 + 2 * SLOTS + 4;
  static constexpr int OFF_SLOTS = (OFF_BAR + NBAR * 8 + 15) / 16 * 16;
  static constexpr int OFF_MISC = OFF_SLOTS + SLOTS * 32;
  static constexpr int BYTES = OFF_MISC + 16;
  // d = 128 has no room for S^T, dP^T, P^T and dQ^T in columns of their own: P^T
  // overwrites S^T and dQ^T overwrites dP^T (each is in registers by then)
  static constexpr bool PAIRED = (D == 128);
  static constexpr uint32_t DV_COL = 0;
  static constexpr uint32_t DK_COL = D;
  static constexpr uint32_t S_COL = 2 * D;
  static constexpr uint32_t DP_COL = 2 * D + QN;
  static constexpr uint32_t P_COL = PAIRED ? S_COL : 384u;
  static constexpr uint32_t DQ_COL = PAIRED ? DP_COL : 448u;
  static constexpr int THREADS = 512;
  // registers after the re-split between the P/dS warpgroups, the drain and the
  // control warpgroup: exactly the launch's 512 x 128
  static constexpr int REGS_LAUNCH = 128;
  static constexpr int REGS_PDS = (D == 64) ? 168 : 144;
  static constexpr int REGS_DRAIN = (D == 64) ? 88 : 144;
  static constexpr int REGS_CONTROL = (D == 64) ? 88 : 80;
  static_assert(256 * REGS_PDS + 128 * REGS_DRAIN + 128 * REGS_CONTROL == THREADS * REGS_LAUNCH,
                "register re-split must hand out exactly the launch's registers");
  static_assert(BYTES <= 232448, "shared memory");
};

// A sweep as the producer announces it to the other roles: a key tile against a run of
// query tiles.
struct Sweep {
  int bh;           // head; below 0: no more
  int q0, n_q;      // first query tile, query tiles
  int kt, n_kt;     // key tile; key tiles of the head's sample
  int len;          // its valid states
  // first row of the j-th query tile: key-major, each key tile starts at its own
  // offset, so that those of one head side by side reduce into different dQ tiles
  // instead of contending for the same L2 lines
  __device__ __forceinline__ int query_row(int j, bool key_major) const {
    const int rot = key_major ? kt % n_q : 0;
    int t = j + rot;
    if (t >= n_q) t -= n_q;
    return (q0 + t) * kTileRows;
  }
  // the key tile has rows that count as nothing but may hold anything
  __device__ __forceinline__ bool ragged(int S) const { return (kt + 1) * kTileRows > len && len < S; }
};

__device__ __forceinline__ int valid_states(const XattnBwdParams& p, int sample) {
  return p.kv_len ? min(max(p.kv_len[sample], 0), p.S) : p.S;
}

__device__ __forceinline__ int key_tiles(const XattnBwdParams& p, int sample) {
  return (valid_states(p, sample) + kTileRows - 1) / kTileRows;
}

// The sweeps of this CTA in turn (one thread).
struct Plan {
  const XattnBwdParams& p;
  Sweep w;
  int k_end = 0;     // of the piece in work
  // query-major: the CTA's share of all units (query tiles of a sample's heads) goes
  // from unit `unit` of sample `sample` up to unit `last` of sample `last_sample`
  int sample = 0, unit = 0, last_sample = 0, last = 0;
  int next;          // key-major: index of the next (head, range, key tile), and those
  int before = 0;    // of the samples before `sample`
  int ranges;        // of a head's query tiles
  __device__ explicit Plan(const XattnBwdParams& p_) : p(p_), next(blockIdx.x) {
    w.kt = 0;
    ranges = p.shares[0].x;
    if (p.key_major) return;
    const int2 a = p.shares[blockIdx.x], b = p.shares[blockIdx.x + 1];
    sample = a.x, unit = a.y, last_sample = b.x, last = b.y;
  }
  __device__ __forceinline__ bool query_piece() {
    for (;; ++sample, unit = 0) {
      if (sample > last_sample || (sample == last_sample && unit >= last)) return false;
      const int end = sample == last_sample ? last : p.heads * p.q_tiles;
      w.n_kt = key_tiles(p, sample);
      if (w.n_kt == 0 || unit >= end) continue;
      const int h = unit / p.q_tiles;
      w.bh = sample * p.heads + h;
      w.q0 = unit - h * p.q_tiles;
      w.len = valid_states(p, sample);
      // what is left of the head, in equal runs that stay in L2
      const int left = min(p.q_tiles - w.q0, end - unit);
      const int runs = w.n_kt == 1 ? 1 : (left + p.run - 1) / p.run;
      w.n_q = (left + runs - 1) / runs;
      unit += w.n_q;
      w.kt = 0;
      k_end = w.n_kt;
      return true;
    }
  }
  // (pieces of key tiles that a sample does not have are not counted, so that the CTAs'
  // numbers of pieces differ by one at most: 8 x 12 heads of 3520 rows of 64, 256 to 1024
  // states, 285 -> 230 us for all kernels)
  __device__ __forceinline__ bool key_piece() {
    int x = next;
    next += gridDim.x;
    for (; sample < p.samples; ++sample) {
      w.n_kt = key_tiles(p, sample);
      const int count = p.heads * ranges * w.n_kt;
      if (x - before < count) break;
      before += count;
    }
    if (sample == p.samples) return false;
    x -= before;
    const int h = x / w.n_kt;
    w.kt = x - h * w.n_kt;
    w.bh = h / ranges;
    const int r = h - w.bh * ranges;
    w.bh += sample * p.heads;
    const int tiles = p.q_tiles / ranges, rest = p.q_tiles - tiles * ranges;
    w.q0 = r * tiles + min(r, rest);  // (the first ones have one more)
    w.n_q = tiles + (r < rest);
    w.len = valid_states(p, sample);
    k_end = w.kt + 1;
    return true;
  }
  __device__ __forceinline__ bool step() { return ++w.kt < k_end || (p.key_major ? key_piece() : query_piece()); }
};

// After a wait gave up: zeros for gradients that are written whole.  Other CTAs' rows as
// well, which the call's status makes no worse: each CTA's own from its plan took 8 KB of
// code next to this path's 1.
__device__ __forceinline__ void leave_zeros(const XattnBwdParams& p, unsigned thread, unsigned threads) {
#pragma unroll 1
  for (int a = 0; a < 3; ++a) {
    const unsigned n = static_cast<unsigned>(p.BH) * (a == 0 ? p.M : p.S);
    uint4* out = reinterpret_cast<uint4*>(a == 0 ? p.dq : a == 1 ? p.dk : p.dv);
#pragma unroll 1
    for (size_t i = thread; i < static_cast<size_t>(n) * (p.d / 8); i += threads) out[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

template <int D, int DM>
__global__ void __launch_bounds__(Layout<D, DM>::THREADS, 1)
    xattn_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                     const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                     const __grid_constant__ CUtensorMap tm_dv, const __grid_constant__ CUtensorMap tm_bias,
                     const __grid_constant__ CUtensorMap tm_dqo,
                     const __grid_constant__ XattnBwdParams p) {
  using L = Layout<D, DM>;
  constexpr int NQ = L::QSTAGES;
  constexpr int ND = L::DOSTAGES;
  constexpr int QN = L::QN;
  constexpr int CW = L::CW;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0u) {
    // nothing runs without aligned shared memory: report it, and leave zeros (the
    // accumulators start with them)
    if (threadIdx.x == 0) atomicOr(p.status, kDevMisaligned);
    if (blockIdx.x == 0) leave_zeros(p, threadIdx.x, L::THREADS);
    return;  // uniform across the CTA, before any barrier or TMEM use
  }
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* k_raw = k_full + 1;    // a K tile that warp 15 makes ready, then k_full
  uint64_t* k_empty = k_raw + 1;
  uint64_t* v_full = k_empty + 1;
  uint64_t* v_raw = v_full + 1;
  uint64_t* v_empty = v_raw + 1;
  uint64_t* q_full = v_empty + 1;
  uint64_t* q_empty = q_full + NQ;
  uint64_t* do_full = q_empty + NQ;
  uint64_t* do_empty = do_full + ND;
  uint64_t* s_full = do_empty + ND;
  uint64_t* s_free = s_full + 1;
  uint64_t* dp_full = s_free + 1;
  uint64_t* dp_free = dp_full + 1;
  uint64_t* pt_ready = dp_free + 1;
  uint64_t* dq_full = pt_ready + 1;
  uint64_t* dq_free = dq_full + 1;
  uint64_t* dkv_full = dq_free + 1;
  uint64_t* dkv_free = dkv_full + 1;
  uint64_t* p_ready = dkv_free + 1;
  uint64_t* ds_free = p_ready + 1;
  uint64_t* w_full = ds_free + 1;          // a sweep is announced, and
  uint64_t* w_empty = w_full + L::SLOTS;   // read by all roles
  uint64_t* acc_full = w_empty + L::SLOTS;  // dQ so far, for a drain warp each
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC + 4);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  if constexpr (L::FOLD) {
    // A rows of the bias MMAs: [1 1 0 0 | 1 1 0 0] picks the LSE pair of a bias
    // row, [0 0 1 1 | 0 0 1 1] its D pair; both 16-byte halves alike, so the
    // 32-byte swizzle leaves them unchanged (8 rows of each)
    if (threadIdx.x < 128) {
      const int a = threadIdx.x >> 6, c = threadIdx.x & 7;
      reinterpret_cast<float*>(smem + L::OFF_ONES)[threadIdx.x] = (((c & 3) < 2) == (a == 0)) ? 1.f : 0.f;
      fence_proxy_async_smem();
    }
  }
  if (threadIdx.x == 0) {
    mbar_init(k_full, 1);
    mbar_init(k_raw, 1);
    mbar_init(k_empty, 2);
    for (int b = 0; b < L::SLOTS; ++b) {
      mbar_init(&w_full[b], 1);
      mbar_init(&w_empty[b], 15);  // the other warps
    }
    for (int b = 0; b < 4; ++b) mbar_init(&acc_full[b], 1);
    mbar_init(v_full, 1);
    mbar_init(v_raw, 1);
    mbar_init(v_empty, 1);
    for (int s = 0; s < NQ; ++s) {
      mbar_init(&q_full[s], 1);
      mbar_init(&q_empty[s], 1);
    }
    for (int s = 0; s < ND; ++s) {
      mbar_init(&do_full[s], 1);
      mbar_init(&do_empty[s], 1);
    }
    mbar_init(s_full, 1);
    mbar_init(s_free, 8);
    mbar_init(dp_full, 1);
    mbar_init(dp_free, 8);
    mbar_init(pt_ready, 8);
    mbar_init(dq_full, 1);
    mbar_init(dq_free, 4);
    mbar_init(dkv_full, 2);
    mbar_init(dkv_free, 4);
    mbar_init(p_ready, 8);
    mbar_init(ds_free, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 13) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const WaitCtl ctl{abort_flag, p.status, p.budget_ns};

  uint8_t* sK = smem + L::OFF_K;
  uint8_t* sV = smem + L::OFF_V;
  uint8_t* sQ = smem + L::OFF_Q;
  uint8_t* sDO = smem + L::OFF_DO;
  uint8_t* sDS = smem + L::OFF_DS;
  float* sLSE = reinterpret_cast<float*>(smem + L::OFF_LSE);
  float* sDelta = reinterpret_cast<float*>(smem + L::OFF_DELTA);
  int4* slots = reinterpret_cast<int4*>(smem + L::OFF_SLOTS);
  // The next sweep, for a whole warp (its fields agree over the lanes: the shuffles tell
  // the compiler, which then works in uniform registers).
  int turn = 0;
  Sweep w;
  auto next_sweep = [&]() {
    const int slot = turn % L::SLOTS;
    if (!warp_wait(&w_full[slot], (turn / L::SLOTS) & 1, ctl)) return false;
    ++turn;
    const int4 a = slots[2 * slot], b = slots[2 * slot + 1];
    w.bh = __shfl_sync(0xffffffffu, a.x, 0);
    w.q0 = __shfl_sync(0xffffffffu, a.y, 0);
    w.n_q = __shfl_sync(0xffffffffu, a.z, 0);
    w.kt = __shfl_sync(0xffffffffu, a.w, 0);
    w.n_kt = __shfl_sync(0xffffffffu, b.x, 0);
    w.len = __shfl_sync(0xffffffffu, b.y, 0);
    if (lane == 0) mbar_arrive(&w_empty[slot]);
    return w.bh >= 0;
  };

  if (warp >= 12) {
  regs_dec<L::REGS_CONTROL>();
  if (warp == 12) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      prefetch_tmap(&tm_q);
      prefetch_tmap(&tm_do);
      int sw = 0, raws = 0, n_q = 0, n_do = 0;  // K tiles, V tiles through warp 15, Q and dO tiles so far
      int n_v = 0;                              // V tiles (one a sweep, loaded ahead of K)
      int k_raws = 0;                           // K tiles through warp 15
      bool ok = true, raw = false, k_was_raw = false;
      Plan plan(p);
      auto load_q = [&](int q) {
        const int st = n_q % NQ;
        if (!mbar_wait(&q_empty[st], ((n_q / NQ) & 1) ^ 1, ctl)) return false;
        if (p.debug_skip_q) return true;
        mbar_arrive_expect_tx(&q_full[st], L::QTILE + L::BIAS_BYTES + L::VEC_BYTES);
        for (int r = 0; r < L::REG; ++r)
          tma_load_3d(sQ + st * L::QSTRIDE + r * L::QREGION, &tm_q, &q_full[st], 64 * r, q, w.bh);
        if constexpr (L::FOLD)
          tma_load_3d(sQ + st * L::QSTRIDE + L::QTILE, &tm_bias, &q_full[st], 0, q, w.bh);
        else
          bulk_load(sLSE + st * QN, p.lse2 + static_cast<size_t>(w.bh) * p.M_pad + q, L::VEC_BYTES, &q_full[st]);
        ++n_q;
        return true;
      };
      auto load_do = [&](int q) {
        const int sd = n_do % ND;
        if (!mbar_wait(&do_empty[sd], ((n_do / ND) & 1) ^ 1, ctl)) return false;
        mbar_arrive_expect_tx(&do_full[sd], L::QTILE + L::VEC_BYTES);
        for (int r = 0; r < L::REG; ++r)
          tma_load_3d(sDO + sd * L::QTILE + r * L::QREGION, &tm_do, &do_full[sd], 64 * r, q, w.bh);
        if constexpr (!L::FOLD)
          bulk_load(sDelta + (n_do & 1) * QN, p.delta + static_cast<size_t>(w.bh) * p.M_pad + q, L::VEC_BYTES,
                    &do_full[sd]);
        ++n_do;
        return true;
      };
      for (;; ++turn) {
        const int slot = turn % L::SLOTS;
        if (!(ok = mbar_wait(&w_empty[slot], ((turn / L::SLOTS) & 1) ^ 1, ctl))) break;
        const bool more = plan.step();
        if (!more) plan.w.bh = -1;
        w = plan.w;
        slots[2 * slot] = make_int4(w.bh, w.q0, w.n_q, w.kt);
        slots[2 * slot + 1] = make_int4(w.n_kt, w.len, 0, 0);
        mbar_arrive(&w_full[slot]);  // (releases the stores above)
        if (!more) break;
        raw = w.ragged(p.S);
        // Q, dO and V of the sweep's first step; K waits for the last dQ of the sweep before
        if (!(ok = load_q(w.query_row(0, p.key_major)))) break;
        auto load_tile = [&](uint8_t* dst, const CUtensorMap* map, uint64_t* bar) {
          mbar_arrive_expect_tx(bar, L::KTILE);
          for (int r = 0; r < L::REG; ++r)
            tma_load_3d(dst + r * L::KREGION, map, bar, 64 * r, w.kt * kTileRows, w.bh);
        };
        if (!(ok = mbar_wait(v_empty, (n_v & 1) ^ 1, ctl))) break;
        load_tile(sV, &tm_v, raw ? v_raw : v_full);
        ++n_v;
        raws += raw;
        if (!(ok = load_do(w.query_row(0, p.key_major)))) break;
        if (!(ok = mbar_wait(k_empty, (sw & 1) ^ 1, ctl))) break;
        load_tile(sK, &tm_k, raw ? k_raw : k_full);
        k_raws += raw;
        k_was_raw = raw;
        ++sw;
        for (int j = 1; ok && j < w.n_q; ++j)
          ok = load_q(w.query_row(j, p.key_major)) && load_do(w.query_row(j, p.key_major));
        if (!ok) break;
      }
      if (*abort_flag || !ok) {
        // let every copy this CTA started land before shared memory goes away
        if (sw > 0) drain_wait(k_was_raw ? k_raw : k_full, ((k_was_raw ? k_raws : sw) - 1) & 1, p.budget_ns);
        if (n_v > 0) drain_wait(raw ? v_raw : v_full, ((raw ? raws : n_v) - 1) & 1, p.budget_ns);
        for (int j = max(0, n_q - NQ); j < n_q; ++j) drain_wait(&q_full[j % NQ], (j / NQ) & 1, p.budget_ns);
        for (int j = max(0, n_do - ND); j < n_do; ++j) drain_wait(&do_full[j % ND], (j / ND) & 1, p.budget_ns);
      }
    }
  } else if (warp == 13 || warp == 14) {
    // ------------------------------------------------------------ MMA issuers (whole warps)
    const bool role_a = warp == 13;  // S^T, dV, dP^T
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, QN, false, false);    // S^T, dP^T
    constexpr uint32_t idesc_tn = idesc_bf16_f32(128, DM, false, true);    // dV, dK
    // d = 64: dQ = dS K (M = query rows); d = 128: dQ^T = K^T dS^T (M = head dim)
    constexpr uint32_t idesc_dq = L::DQT ? idesc_bf16_f32(128, QN, true, true)
                                         : idesc_bf16_f32(128, D, true, true);
    const uint32_t k_kmaj = sdesc_sw128(smem_u32(sK), 16);
    const uint32_t v_kmaj = sdesc_sw128(smem_u32(sV), 16);
    const uint32_t k_mn = sdesc_sw128(smem_u32(sK), L::KREGION);
    const uint32_t q_kmaj0 = sdesc_sw128(smem_u32(sQ), 16);
    const uint32_t do_kmaj0 = sdesc_sw128(smem_u32(sDO), 16);
    const uint32_t q_mn0 = sdesc_sw128(smem_u32(sQ), L::QREGION);
    const uint32_t do_mn0 = sdesc_sw128(smem_u32(sDO), L::QREGION);
    const uint32_t ds_mn = sdesc_sw128(smem_u32(sDS), L::KREGION);
    const uint32_t ds_kmaj = sdesc_sw128(smem_u32(sDS), 16);
    const uint64_t ones_l = sdesc_sw32(smem_u32(smem + L::OFF_ONES), 0);
    const uint64_t ones_d = sdesc_sw32(smem_u32(smem + L::OFF_ONES + 256), 0);
    const uint64_t bias0 = sdesc_sw32(smem_u32(sQ + L::QTILE), 256);
    auto add_bias = [&](uint32_t d_col, uint64_t ones, int stage) {
      if constexpr (L::FOLD)
        umma_ss_tf32(tmem + d_col, ones, sdesc_add(bias0, stage * L::QSTRIDE), idesc_tf32_f32(128, QN), 1u);
    };
    // X = A B^T, both K-major over d
    auto issue_kmajor = [&](uint32_t d_col, uint32_t a, uint32_t b) {
#pragma unroll
      for (int r = 0; r < DM / 64; ++r)
        umma_ss4<2, 2>(tmem + d_col, sdesc_add(a, r * L::KREGION), sdesc_add(b, r * L::QREGION), idesc_s, r > 0 ? 1u : 0u);
      if constexpr (DM % 64 != 0) {
        static_assert(DM % 64 == 0 || DM == 80, "one more slice");
        umma_ss(tmem + d_col, sdesc_add(a, L::KREGION), sdesc_add(b, L::QREGION), idesc_s, 1u);
      }
    };
    auto issue_s = [&](int g) {
      issue_kmajor(L::S_COL, k_kmaj, sdesc_add(q_kmaj0, (g % NQ) * L::QSTRIDE));
      add_bias(L::S_COL, ones_l, g % NQ);
      umma_commit(s_full);
    };
    auto issue_dp = [&](int g) {
      issue_kmajor(L::DP_COL, v_kmaj, sdesc_add(do_kmaj0, (g % ND) * L::QTILE));
      add_bias(L::DP_COL, ones_d, g % NQ);
      umma_commit(dp_full);
    };
    // TMEM column of 64 queries of P^T (d = 128: each warpgroup's half in its own 64
    // columns of S^T)
    auto pt_col = [](int r) -> uint32_t { return L::P_COL + r * (L::PAIRED ? 64 : 32); };
    auto issue_dv = [&](int g, bool acc) {  // dV += P^T dO
      const uint32_t do_mn = sdesc_add(do_mn0, (g % ND) * L::QTILE);
#pragma unroll
      for (int r = 0; r < QN / 64; ++r)
        umma_ts4<8, 128>(tmem + L::DV_COL, tmem + pt_col(r), sdesc_add(do_mn, r * 8192), idesc_tn,
                         (acc || r > 0) ? 1u : 0u);
    };
    auto issue_dk = [&](int g, bool acc) {  // dK += dS^T Q
      const uint32_t q_mn = sdesc_add(q_mn0, (g % NQ) * L::QSTRIDE);
#pragma unroll
      for (int r = 0; r < QN / 64; ++r)
        umma_ss4<2, 128>(tmem + L::DK_COL, sdesc_add(ds_kmaj, r * L::KREGION), sdesc_add(q_mn, r * 8192), idesc_tn,
                         (acc || r > 0) ? 1u : 0u);
    };
    auto issue_dq = [&]() {
#pragma unroll
      for (int r = 0; r < kTileRows / 64; ++r)
        umma_ss4<128, 128>(tmem + L::DQ_COL, sdesc_add(L::DQT ? k_mn : ds_mn, r * 8192),
                           sdesc_add(L::DQT ? ds_mn : k_mn, r * 8192), idesc_dq, r > 0 ? 1u : 0u);
    };
    bool ok = true;
    int g = 0, sw = 0;  // steps and sweeps so far
    while (ok && next_sweep()) {
      if (!(ok = warp_wait(k_full, sw & 1, ctl))) break;
      // the last sweep's dK and dV are out of tensor memory
      auto wait_dkv = [&]() { return sw == 0 || warp_wait(dkv_free, (sw - 1) & 1, ctl); };
      if (role_a) {
        // j = -1: the sweep's first S (and dP); g counts the steps whose S is issued
        for (int j = -1; j < w.n_q; ++j) {
          const bool more = j + 1 < w.n_q;
          auto next_dp = [&](int x) {  // dP^T of step x, the (j + 1)-th of the sweep (PAIRED: the j-th)
            if (!warp_wait(&do_full[x % ND], (x / ND) & 1, ctl)) return false;
            // d = 64: the P/dS warps hold the last dP^T; else the drain holds the last
            // dQ, whose columns this takes
            if (x > 0 && !warp_wait(L::PAIRED ? dq_free : dp_free, (x - 1) & 1, ctl)) return false;
            tc_fence_after();
            issue_dp(x);
            return true;
          };
          if constexpr (L::PAIRED) {
            // dP, dV, the next S: MMAs of one issuer run in order, so the next S may
            // land on P once dV is issued
            if (j >= 0) {
              if (j == 0 && !(ok = warp_wait(v_full, sw & 1, ctl))) break;
              if (!(ok = next_dp(g - 1))) break;
              if (!more) umma_commit(v_empty);
            }
          } else if (more) {
            // S^T of the next step as soon as the P/dS warps hold the last one
            if (!(ok = warp_wait(&q_full[g % NQ], (g / NQ) & 1, ctl))) break;
            if (g > 0 && !(ok = warp_wait(s_free, (g - 1) & 1, ctl))) break;
            tc_fence_after();
            issue_s(g++);
          }
          if (j >= 0) {
            const int x = L::PAIRED || !more ? g - 1 : g - 2;  // the step in work
            if (!(ok = warp_wait(pt_ready, x & 1, ctl))) break;
            if (j == 0 && !(ok = wait_dkv())) break;
            tc_fence_after();
            issue_dv(x, j > 0);
            umma_commit(&do_empty[x % ND]);
          }
          if (!more) continue;
          if constexpr (L::PAIRED) {
            if (!(ok = warp_wait(&q_full[g % NQ], (g / NQ) & 1, ctl))) break;
            tc_fence_after();
            issue_s(g++);
          } else {
            if (j < 0 && !(ok = warp_wait(v_full, sw & 1, ctl))) break;
            if (!(ok = next_dp(g - 1))) break;
            if (j + 2 == w.n_q) umma_commit(v_empty);
          }
        }
      } else {
        for (int j = 0; j < w.n_q; ++j, ++g) {
          // dS is in shared memory (and so dP in registers)
          if (!(ok = warp_wait(p_ready, g & 1, ctl))) break;
          // dQ first, so the drain starts while dK runs
          if constexpr (!L::PAIRED)
            if (g > 0 && !(ok = warp_wait(dq_free, (g - 1) & 1, ctl))) break;
          tc_fence_after();
          issue_dq();
          umma_commit(dq_full);
          if (j == 0) {
            if (!(ok = wait_dkv())) break;
            tc_fence_after();
          }
          issue_dk(g, j > 0);
          umma_commit(&q_empty[g % NQ]);
          umma_commit(ds_free);
        }
      }
      if (!ok) break;
      umma_commit(dkv_full);  // one arrival per issuing warp
      umma_commit(k_empty);
      ++sw;
    }
  } else {
    // ------------------------------------------------------------ ragged K and V tiles
    int raws = 0;
    bool ok = true;
    while (ok && next_sweep()) {
      if (!w.ragged(p.S)) continue;
      const int limit = w.len - w.kt * kTileRows;
      for (int m = 0; ok && m < 2; ++m) {  // in the order of the loads
        if (!(ok = warp_wait(m == 0 ? v_raw : k_raw, raws & 1, ctl))) break;
        uint8_t* tile = m == 0 ? sV : sK;
        for (int i = limit * 8 + lane; i < kTileRows * 8; i += 32)
          for (int r = 0; r < L::REG; ++r)
            *reinterpret_cast<uint4*>(tile + r * L::KREGION + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();  // the tensor core reads the tile next
        __syncwarp();
        if (lane == 0) mbar_arrive(m == 0 ? v_full : k_full);
      }
      ++raws;
    }
  }
  } else if (warp < 8) {
    regs_inc<L::REGS_PDS>();
    // ------------------------------------------------------------ P / dS (thread = key row)
    const int wg = warp >> 2;            // query columns [CW wg, CW wg + CW)
    const int wq = warp & 3;             // TMEM lane quadrant
    const int j_local = wq * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(wq * 32) << 16);
    const uint32_t s_addr = lane_base + L::S_COL + CW * wg;
    const uint32_t dp_addr = lane_base + L::DP_COL + CW * wg;
    const uint32_t p_addr = lane_base + L::P_COL + (L::PAIRED ? 64 : 32) * wg;
    const float sl2 = p.scale_log2;
    const int c0 = CW * wg;
    const int ds_off = (c0 >> 6) * L::KREGION + j_local * 128;
    const int chunk0 = (c0 & 63) >> 3;
    const int sw = j_local & 7;
    bool ok = true;
    int g = 0;
    while (ok && next_sweep()) {
    const bool k_valid = w.kt * kTileRows + j_local < w.len;
    const bool some_invalid = !__all_sync(0xffffffffu, k_valid);
    for (int j = 0; j < w.n_q; ++j, ++g) {
      const float* lse2 = sLSE + (g % NQ) * QN + c0;
      const float* delta = sDelta + (g & 1) * QN + c0;
      if (!(ok = warp_wait(s_full, g & 1, ctl))) break;
      tc_fence_after();
      float2 nl[CW / 2];
      auto load_lse = [&]() {
#pragma unroll
        for (int c = 0; c < CW / 4; ++c) {
          const float4 v = reinterpret_cast<const float4*>(lse2)[c];
          nl[2 * c] = make_float2(-v.x, -v.y);
          nl[2 * c + 1] = make_float2(-v.z, -v.w);
        }
      };
      float pr[CW];
      {
        uint32_t r[CW / 32][32];
#pragma unroll
        for (int h = 0; h < CW / 32; ++h) tmem_ld32(s_addr + 32 * h, r[h]);
        tmem_wait_ld();
#pragma unroll
        for (int h = 0; h < CW / 32; ++h)
#pragma unroll
          for (int k = 0; k < 32; ++k) pr[32 * h + k] = __uint_as_float(r[h][k]);
      }
      if constexpr (!L::PAIRED) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_free);
      }
      if constexpr (!L::FOLD) load_lse();
      const float2 sl2x2 = make_float2(sl2, sl2);
#pragma unroll
      for (int c = 0; c < CW / 2; ++c) {
        // d = 64: the MMA already subtracted LSE/scale
        const float2 x = L::FOLD ? mul2(make_float2(pr[2 * c], pr[2 * c + 1]), sl2x2)
                                 : fma2(make_float2(pr[2 * c], pr[2 * c + 1]), sl2x2, nl[c]);
        pr[2 * c] = ex2_approx(x.x);
        pr[2 * c + 1] = ex2_approx(x.y);
      }
      if (some_invalid) {
#pragma unroll
        for (int c = 0; c < CW; ++c)
          if (!k_valid) pr[c] = 0.f;
      }
      // P^T (bf16 pairs) -> TMEM right away, so that dV starts while dS is computed
      uint32_t r[CW / 32][32];  // dP^T
      if constexpr (!L::PAIRED) {
        // dP^T is issued after the last dV: once it is there, that has read P^T.
        // Its first half loads while P^T is stored.
        if (!(ok = warp_wait(dp_full, g & 1, ctl))) break;
        tc_fence_after();
        tmem_ld32(dp_addr, r[0]);
      }
      {
        uint32_t pe[CW / 2];
#pragma unroll
        for (int c = 0; c < CW / 2; ++c) pe[c] = pack_bf16x2(pr[2 * c], pr[2 * c + 1]);
        tmem_st32(p_addr, pe);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pt_ready);
      }
      if constexpr (L::PAIRED) {
        if (!(ok = warp_wait(dp_full, g & 1, ctl))) break;
        tc_fence_after();
        tmem_ld32(dp_addr, r[0]);
      }
#pragma unroll
      for (int h = 1; h < CW / 32; ++h) tmem_ld32(dp_addr + 32 * h, r[h]);
      // the wait for the dS^T buffer passes while dP^T loads
      if (g > 0 && !(ok = warp_wait(ds_free, (g - 1) & 1, ctl))) break;
      tmem_wait_ld();
      if constexpr (!L::PAIRED) {
        // dP^T is in registers: its columns can take the next step's
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(dp_free);
      }
      uint32_t dk[CW / 2];
#pragma unroll
      for (int h = 0; h < CW / 32; ++h) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          // d = 64: the MMA already subtracted D
          const float4 dv = L::FOLD ? make_float4(0.f, 0.f, 0.f, 0.f)
                                    : reinterpret_cast<const float4*>(delta)[8 * h + k];
          const int c = 32 * h + 4 * k;
          const float2 dp0 = make_float2(__uint_as_float(r[h][4 * k]), __uint_as_float(r[h][4 * k + 1]));
          const float2 dp1 = make_float2(__uint_as_float(r[h][4 * k + 2]), __uint_as_float(r[h][4 * k + 3]));
          const float2 t0 = L::FOLD ? dp0 : add2(dp0, make_float2(-dv.x, -dv.y));
          const float2 t1 = L::FOLD ? dp1 : add2(dp1, make_float2(-dv.z, -dv.w));
          const float2 s0 = mul2(make_float2(pr[c], pr[c + 1]), t0);
          const float2 s1 = mul2(make_float2(pr[c + 2], pr[c + 3]), t1);
          dk[16 * h + 2 * k] = pack_bf16x2(s0.x, s0.y);
          dk[16 * h + 2 * k + 1] = pack_bf16x2(s1.x, s1.y);
        }
      }
      // dS^T row segment -> shared memory (swizzled like a TMA 128-byte tile)
      uint8_t* ds_row = sDS + ds_off;
#pragma unroll
      for (int q = 0; q < CW / 8; ++q)
        *reinterpret_cast<uint4*>(ds_row + (((chunk0 + q) ^ sw) << 4)) =
            make_uint4(dk[4 * q], dk[4 * q + 1], dk[4 * q + 2], dk[4 * q + 3]);
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_ready);
    }
    }
  } else {
    if constexpr (L::REGS_DRAIN > L::REGS_LAUNCH)
      regs_inc<L::REGS_DRAIN>();
    else
      regs_dec<L::REGS_DRAIN>();
    // ------------------------------------------------------------ drain
    const int wq = warp & 3;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(wq * 32) << 16);
    int box = 0;    // the staging box whose turn it is
    int loads = 0;  // of dQ so far
    // 32 lanes x 32 columns as a box of 32 rows (128 bytes, 16-byte chunk c of row r
    // at c ^ (r mod 8)) that the TMA unit adds to `map` at column c0, row `row`, or
    // stores there
    auto put_rows = [&](const CUtensorMap* map, const uint32_t (&r)[32], int c0, int row, bool add) {
      uint8_t* stg = smem + L::OFF_STG + (L::BOXES * wq + box) * L::BOX_BYTES;
      if (lane == 0) bulk_wait_read<L::BOXES - 1>();  // the TMA unit has read this box
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint4*>(stg + lane * 128 + ((i ^ (lane & 7)) << 4)) =
            make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (add)
          tma_reduce_add_3d(map, stg, c0, row, w.bh);
        else
          tma_store_3d(map, stg, c0, row, w.bh);
        bulk_commit_group();
      }
      box ^= L::BOXES - 1;
    };
    bool ok = true;
    int g = 0, sw = 0;
    while (ok && next_sweep()) {
      // dQ of a step: whole, where the sample has one key tile; key-major all are added to
      // zeros; query-major (d = 64) the first key tile's is stored, the others' added and
      // the last one's finished, each once the copies before are complete
      const bool whole = w.n_kt == 1;
      const bool add = L::DQT || p.key_major || w.kt > 0;
      const bool finish = !L::DQT && !p.key_major && !whole && w.kt == w.n_kt - 1;
      if (finish || (!L::DQT && !p.key_major && w.kt == 1)) {
        if (lane == 0) bulk_wait_all();
        __syncwarp();
      }
      // dQ of the sweeps before, back into the staging boxes (which nothing else uses
      // then) while the step's MMAs run
      [[maybe_unused]] auto load_acc = [&](int j) {
        if (lane == 0) {
          uint8_t* stg = smem + L::OFF_STG + L::BOXES * wq * L::BOX_BYTES;
          mbar_arrive_expect_tx(&acc_full[wq], 2 * L::BOX_BYTES);
          for (int c = 0; c < 2; ++c)
            tma_load_3d(stg + c * L::BOX_BYTES, &tm_dq, &acc_full[wq], 32 * c, (w.q0 + j) * QN + 32 * wq, w.bh);
        }
        ++loads;
      };
      if (finish) load_acc(0);
      for (int j = 0; j < w.n_q; ++j, ++g) {
        const int q0 = w.query_row(j, p.key_major);
        if (!(ok = warp_wait(dq_full, g & 1, ctl))) break;
        tc_fence_after();
        if constexpr (L::DQT) {
          // lanes = head-dim columns, TMEM columns = the QN query rows: boxes of 32
          // queries.  The maps clip columns past the caller's; warps with none skip.
          auto hand_over = [&]() {  // dQ is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(dq_free);
          };
          auto next_box = [&]() {
            uint8_t* stg = smem + L::OFF_STG + (2 * wq + box) * L::BOX_BYTES;
            if (lane == 0) bulk_wait_read<1>();  // the TMA unit has read this box
            __syncwarp();
            box ^= 1;
            return stg;
          };
          if (whole) {
#pragma unroll 1
            for (int c = 0; c < QN / 32; ++c) {
              uint32_t r[32];
              tmem_ld32(lane_base + L::DQ_COL + 32 * c, r);
              tmem_wait_ld();
              if (c == QN / 32 - 1) hand_over();
              if (32 * wq >= p.d) continue;
              uint8_t* stg = next_box();
              // bf16 rows of 64 bytes: of two queries, even lanes take the first and odd
              // ones the second, a pair of columns each
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                const float a = __uint_as_float(r[k]) * p.scale, b = __uint_as_float(r[k + 1]) * p.scale;
                const float other = __shfl_xor_sync(0xffffffffu, lane & 1 ? a : b, 1);
                const uint32_t pair = lane & 1 ? pack_bf16x2(other, b) : pack_bf16x2(a, other);
                *reinterpret_cast<uint32_t*>(stg + (k + (lane & 1)) * 64 + (lane >> 1) * 4) = pair;
              }
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&tm_dqo, stg, 32 * wq, q0 + 32 * c, w.bh);
                bulk_commit_group();
              }
            }
          } else {
            uint32_t r[QN / 32][32];
#pragma unroll
            for (int c = 0; c < QN / 32; ++c) tmem_ld32(lane_base + L::DQ_COL + 32 * c, r[c]);
            tmem_wait_ld();
            hand_over();
            if (32 * wq < p.d) {
#pragma unroll
              for (int c = 0; c < QN / 32; ++c) {
                uint8_t* stg = next_box();
#pragma unroll
                for (int k = 0; k < 32; ++k)  // each instruction one row, 16-byte chunks swizzled
                  *reinterpret_cast<uint32_t*>(stg + k * 128 + (((lane >> 2) ^ (k & 7)) << 4) + (lane & 3) * 4) =
                      r[c][k];
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                  tma_reduce_add_3d(&tm_dq, stg, 32 * wq, q0 + 32 * c, w.bh);
                  bulk_commit_group();
                }
              }
            }
          }
        } else {
          // lanes = query rows
          static_assert(D == 64 || L::DQT, "the drain below covers two 32-column boxes");
          const int row = q0 + wq * 32;
          // bf16 rows of 128 bytes, 16-byte chunk k of row i at k ^ (i & 7); the map clips
          // rows past the caller's
          auto store_rows = [&](const uint32_t (&r)[2][32]) {
            uint8_t* stg = smem + L::OFF_OUT + wq * L::BOX_BYTES;
            if (lane == 0) bulk_wait_read<0>();  // the TMA unit has read the box
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              uint32_t v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                v[i] = pack_bf16x2(__uint_as_float(r[k >> 2][8 * (k & 3) + 2 * i]) * p.scale,
                                   __uint_as_float(r[k >> 2][8 * (k & 3) + 2 * i + 1]) * p.scale);
              *reinterpret_cast<uint4*>(stg + lane * 128 + ((k ^ (lane & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_3d(&tm_dqo, stg, 0, row, w.bh);
              bulk_commit_group();
            }
          };
          uint32_t r[2][32];
          tmem_ld32(lane_base + L::DQ_COL, r[0]);
          tmem_ld32(lane_base + L::DQ_COL + 32, r[1]);
          tmem_wait_ld();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(dq_free);  // dQ is in registers
          if (finish) {
            if (!(ok = warp_wait(&acc_full[wq], (loads - 1) & 1, ctl))) break;
            const uint8_t* stg = smem + L::OFF_STG + L::BOXES * wq * L::BOX_BYTES + lane * 128;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 x =
                    *reinterpret_cast<const float4*>(stg + c * L::BOX_BYTES + ((i ^ (lane & 7)) << 4));
                r[c][4 * i] = __float_as_uint(__uint_as_float(r[c][4 * i]) + x.x);
                r[c][4 * i + 1] = __float_as_uint(__uint_as_float(r[c][4 * i + 1]) + x.y);
                r[c][4 * i + 2] = __float_as_uint(__uint_as_float(r[c][4 * i + 2]) + x.z);
                r[c][4 * i + 3] = __float_as_uint(__uint_as_float(r[c][4 * i + 3]) + x.w);
              }
            fence_proxy_async_smem();  // the boxes are read before the next copy into them
            __syncwarp();
            if (j + 1 < w.n_q) load_acc(j + 1);
          }
          if (finish || whole) {
            store_rows(r);
          } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) put_rows(&tm_dq, r[c], 32 * c, row, add);
          }
          __syncwarp();
        }
      }
      // the sweep's dK and dV (lanes = key rows)
      if (!ok || !(ok = warp_wait(dkv_full, sw & 1, ctl))) break;
      tc_fence_after();
      const int row = w.kt * kTileRows + wq * 32;
      constexpr int kChunks = (DM + 31) / 32;
#pragma unroll 1
      for (int i = 0; i < 2 * kChunks; ++i) {
        const bool is_dk = i >= kChunks;
        const int c = is_dk ? i - kChunks : i;
        uint32_t r[32];
        tmem_ld32(lane_base + (is_dk ? L::DK_COL : L::DV_COL) + 32 * c, r);
        tmem_wait_ld();
        if (i == 2 * kChunks - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(dkv_free);
        }
        if (32 * c >= p.d) continue;
        // past the valid states: weights of 0, but a NaN or an infinity of dO or D times them is NaN
        if (row + 32 > w.len) {
          const uint32_t keep = row + lane < w.len ? 0xffffffffu : 0u;
#pragma unroll
          for (int k = 0; k < 32; ++k) r[k] &= keep;
        }
        if (!p.dkv_whole) {
          put_rows(is_dk ? &tm_dk : &tm_dv, r, 32 * c, row, true);
        } else if (row + lane < p.S) {
          const float mul = is_dk ? p.scale : 1.f;
          float v[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(r[k]) * mul;
          store_row32((is_dk ? p.dk : p.dv) + (static_cast<size_t>(w.bh) * p.S + row + lane) * p.d + 32 * c, v,
                      min(4, (p.d - 32 * c) / 8), p.wide_dkv);
        }
        __syncwarp();
      }
      ++sw;
    }
    // every copy has completed before the CTA's shared memory goes away
    if (lane == 0 && !ok && loads > 0) drain_wait(&acc_full[wq], (loads - 1) & 1, p.budget_ns);
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 13) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (*abort_flag) leave_zeros(p, threadIdx.x, L::THREADS);
}

// D_i = <dO_i, O_i> and LSE_i log2(e) (padding rows 0 and +inf, so that their P is
// exactly 0); d = 64: both again as bias rows, -LSE/scale and -D as tf32 high and
// low parts.  D / 8 lanes a row, 16 bytes each, kPreRows rows a group of lanes.
// Also zeroes what is only added to, and the gradients that no sweep writes: dQ of
// samples without states here; in the blocks after the rows' the accumulators of dK
// and dV or, where each key tile's one sweep writes them whole, their rows past a
// sample's key tiles.  The last block divides the work.
// Of few states D is summed from P and dP again instead: P is near 0 or 1 there, dP - D a
// small difference, and what O lost in bf16 was up to 1e-2 of dQ and dK (two states, q and k
// twice the usual size; of 11700 calls of 2 and more states 6% were off by over 5e-3, all but
// one with fewer than 16; with this one in 7500).  Five blocks an SM: 48 x 14080 rows of 64
// 44 -> 41 us.
constexpr int kPreRows = 4;
constexpr int kFewStates = 8;
template <int D>
__global__ void __launch_bounds__(256, 5) xattn_pre_kernel(const XattnBwdParams p, long long row_blocks, int ctas) {
  constexpr int G = D / 8;
  constexpr int kGroups = 256 / G;
  const int d_io = (D == 64) ? D : p.d;
  if (blockIdx.x == gridDim.x - 1) {
    if (p.key_major) {
      // the ranges that take the least rounds of the CTAs through the samples' key tiles
      // (2 x 4 heads of 22000 rows of 128, 1500 and 600 states: those for 1500 each 300 us
      // for all kernels, these 239)
      __shared__ float us[kXattnMaxRanges];
      const int r = threadIdx.x + 1;
      if (r <= kXattnMaxRanges) {
        long long pieces = 0;
        for (int b = 0; b < p.samples; ++b) pieces += static_cast<long long>(p.heads) * r * key_tiles(p, b);
        us[r - 1] = static_cast<float>((pieces + ctas - 1) / ctas) *
                    (static_cast<float>((p.q_tiles + r - 1) / r) * xattn_step_us(D) + xattn_sweep_us(D));
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        int best = 1;
        if (!p.dkv_whole)
          for (int k = 2; k <= min(p.q_tiles, kXattnMaxRanges); ++k)
            if (us[k - 1] < us[best - 1]) best = k;
        p.shares[0] = make_int2(best, 0);
      }
      return;
    }
    // share c begins where c / ctas of all steps are done: units of a sample count as its
    // key tiles
    long long total = 0;
    for (int b = 0; b < p.samples; ++b) total += static_cast<long long>(p.heads) * p.q_tiles * key_tiles(p, b);
    for (int c = threadIdx.x; c <= ctas; c += 256) {
      const long long at = total * c / ctas;
      long long before = 0;
      int b = 0, unit = 0;
      for (; b < p.samples; ++b) {
        const int n = key_tiles(p, b);
        const long long all = static_cast<long long>(p.heads) * p.q_tiles * n;
        if (before + all > at) {
          unit = static_cast<int>((at - before) / n);
          break;
        }
        before += all;
      }
      p.shares[c] = make_int2(b, unit);
    }
    return;
  }
  if (blockIdx.x >= row_blocks) {
    const long long x = blockIdx.x - row_blocks;
    if (!p.dkv_whole) {
      float4* acc = reinterpret_cast<float4*>(p.dkv_acc);
      const long long i = x * 1024 + threadIdx.x;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + 256 * k < p.dkv_float4s) acc[i + 256 * k] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {  // a head a block
      const int first = key_tiles(p, static_cast<int>(x / p.heads)) * kTileRows;
      const long long at = (x * p.S + first) * (d_io / 8);
      const int n = max(0, p.S - first) * (d_io / 8);
      for (int i = threadIdx.x; i < n; i += 256) {
        reinterpret_cast<uint4*>(p.dk)[at + i] = make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4*>(p.dv)[at + i] = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    return;
  }
  const long long rows = static_cast<long long>(p.BH) * p.M_pad;
  const int sub = threadIdx.x % G;
  const long long row0 = (blockIdx.x * static_cast<long long>(kGroups) + threadIdx.x / G) * kPreRows;
  // (M_pad is a multiple of kPreRows: the rows are of one head)
  const int bh = static_cast<int>(min(row0, rows - 1) / p.M_pad);
  const int i0 = static_cast<int>(row0 - static_cast<long long>(bh) * p.M_pad);
  const bool valid = row0 < rows;
  const int keys = valid_states(p, bh / p.heads);
  auto dot = [](const uint4& x, const uint4& y) {  // over the row's lanes
    const uint32_t xv[4] = {x.x, x.y, x.z, x.w}, yv[4] = {y.x, y.y, y.z, y.w};
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sum = fmaf(__uint_as_float(xv[k] << 16), __uint_as_float(yv[k] << 16), sum);
      sum = fmaf(__uint_as_float(xv[k] & 0xffff0000u), __uint_as_float(yv[k] & 0xffff0000u), sum);
    }
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    return sum;
  };
  auto piece = [&](const __nv_bfloat16* base, size_t row) {
    return 8 * sub < d_io ? *reinterpret_cast<const uint4*>(base + row * d_io + 8 * sub) : make_uint4(0u, 0u, 0u, 0u);
  };
  auto finish = [&](int r, float sum) {
    const long long gr = row0 + r;
    if (valid && p.zero_dq) {
      float4* acc = reinterpret_cast<float4*>(p.dq_acc + gr * D);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (4 * (sub + k * G) < d_io) acc[sub + k * G] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (valid && sub == 0) {
      const float lse = i0 + r < p.M ? p.lse[static_cast<size_t>(bh) * p.M + i0 + r] : INFINITY;
      if constexpr (D == 64) {
        const float lb = i0 + r < p.M ? -lse / p.scale : -1e30f;
        const float lh = __uint_as_float(__float_as_uint(lb) & 0xffffe000u);
        const float dh = __uint_as_float(__float_as_uint(-sum) & 0xffffe000u);
        float4* row = reinterpret_cast<float4*>(p.bias + gr * 8);
        row[0] = make_float4(lh, lb - lh, dh, -sum - dh);
        row[1] = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        p.delta[gr] = sum;
        p.lse2[gr] = lse * 1.4426950408889634f;
      }
    }
  };
  if (keys > 1 && keys <= kFewStates) {  // (of one state O is exact, V itself)
#pragma unroll 1
    for (int r = 0; r < kPreRows; ++r) {  // (a warp's lanes see the same sample)
      const bool there = valid && i0 + r < p.M;
      const size_t row = static_cast<size_t>(bh) * p.M + (there ? i0 + r : 0);
      const uint4 q = piece(p.q, row), g = piece(p.dout, row);
      const float lse2 = p.lse[row] * 1.4426950408889634f;
      float sum = 0.f;
#pragma unroll 1
      for (int j = 0; j < keys; ++j) {
        const size_t state = static_cast<size_t>(bh) * p.S + j;
        sum = fmaf(ex2_approx(fmaf(dot(q, piece(p.k, state)), p.scale_log2, -lse2)), dot(g, piece(p.v, state)), sum);
      }
      finish(r, there ? sum : 0.f);
    }
    return;
  }
  uint4 a[kPreRows], b[kPreRows];
#pragma unroll
  for (int r = 0; r < kPreRows; ++r) {
    a[r] = b[r] = make_uint4(0u, 0u, 0u, 0u);
    if (valid && i0 + r < p.M && 8 * sub < d_io) {
      const size_t off = (static_cast<size_t>(bh) * p.M + i0 + r) * d_io + 8 * sub;
      if (keys == 0) {
        *reinterpret_cast<uint4*>(p.dq + off) = a[r];
      } else {
        a[r] = *reinterpret_cast<const uint4*>(p.o + off);
        b[r] = *reinterpret_cast<const uint4*>(p.dout + off);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kPreRows; ++r) finish(r, dot(a[r], b[r]));
}

// bf16 rows from the accumulators: dQ of samples with several key tiles (the others'
// is written already), dK and dV where several sweeps add to them.  D / 8 lanes a row,
// 8 columns each, kPostRows rows in flight a thread; blockIdx.y 0: dQ, 1: dK, 2: dV.
constexpr int kPostRows = 4;
template <int D>
__global__ void __launch_bounds__(256) xattn_post_kernel(const XattnBwdParams p, int first) {
  constexpr int G = D / 8;
  constexpr int kGroups = 256 / G;
  const int which = blockIdx.y + first;
  const int d_io = (D == 64) ? D : p.d;
  const int rows = which == 0 ? p.M : p.S;
  const int padded = which == 0 ? p.M_pad : p.S_pad;
  // (padded is a multiple of the block's rows, which are of one head)
  const int blocks = padded / (kGroups * kPostRows);
  const int bh = blockIdx.x / blocks;
  if (bh >= p.BH) return;
  if (which == 0 && p.kv_len && p.kv_len[bh / p.heads] <= kTileRows) return;
  const int r0 = (blockIdx.x - bh * blocks) * (kGroups * kPostRows) + threadIdx.x / G;
  const int c = 8 * (threadIdx.x % G);
  if (c >= d_io) return;
  const float* acc = which == 0 ? p.dq_acc : which == 1 ? p.dkv_acc : p.dkv_acc + static_cast<size_t>(p.BH) * p.S_pad * D;
  __nv_bfloat16* out = which == 0 ? p.dq : which == 1 ? p.dk : p.dv;
  const float mul = which == 2 ? 1.f : p.scale;
  const float* src = acc + (static_cast<size_t>(bh) * padded + r0) * D + c;
  float4 a[kPostRows], b[kPostRows];
#pragma unroll
  for (int k = 0; k < kPostRows; ++k) {  // (rows past `rows` are padding of the accumulators)
    a[k] = *reinterpret_cast<const float4*>(src + k * kGroups * D);
    b[k] = *reinterpret_cast<const float4*>(src + k * kGroups * D + 4);
  }
#pragma unroll
  for (int k = 0; k < kPostRows; ++k) {
    const int r = r0 + k * kGroups;
    if (r < rows)
      *reinterpret_cast<uint4*>(out + (static_cast<size_t>(bh) * rows + r) * d_io + c) =
          make_uint4(pack_bf16x2(a[k].x * mul, a[k].y * mul), pack_bf16x2(a[k].z * mul, a[k].w * mul),
                     pack_bf16x2(b[k].x * mul, b[k].y * mul), pack_bf16x2(b[k].z * mul, b[k].w * mul));
  }
}

template <int D, int DM>
cudaError_t launch(const XattnBwdMaps& m, const XattnBwdParams& p, int dev, int sms, cudaStream_t s) {
  using L = Layout<D, DM>;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(dev, [] {
    // the in-kernel register re-split assumes the launch register count; with any
    // other its setmaxnreg.inc could never be satisfied, so refuse
    cudaFuncAttributes fa;
    const cudaError_t e0 = cudaFuncGetAttributes(&fa, xattn_bwd_kernel<D, DM>);
    if (e0 != cudaSuccess) return e0;
    if (fa.numRegs != L::REGS_LAUNCH) return cudaErrorInvalidKernelImage;
    return cudaFuncSetAttribute(xattn_bwd_kernel<D, DM>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
  });
  if (e != cudaSuccess) return e;
  const long long work = !p.key_major  ? static_cast<long long>(p.BH) * p.q_tiles
                         : p.dkv_whole ? static_cast<long long>(p.BH) * p.k_tiles
                                       : sms;
  const unsigned grid = static_cast<unsigned>(work < sms ? work : sms);
  constexpr int kBlockRows = kPreRows * 256 / (D / 8);
  const long long row_blocks = (static_cast<long long>(p.BH) * p.M_pad + kBlockRows - 1) / kBlockRows;
  const long long zero_blocks = p.dkv_whole ? p.BH : (p.dkv_float4s + 1023) / 1024;
  xattn_pre_kernel<D><<<static_cast<unsigned>(row_blocks + zero_blocks + 1), 256, 0, s>>>(p, row_blocks, grid);
  xattn_bwd_kernel<D, DM><<<grid, L::THREADS, L::BYTES, s>>>(m.q, m.k, m.v, m.dout, m.dq, m.dk, m.dv, m.bias,
                                                             m.dq_out, p);
  // what several sweeps add to becomes bf16
  const int first = p.key_major ? 0 : 1, last = p.dkv_whole ? 1 : 3;
  if (first < last) {
    const int most = first == 0 && (p.M_pad > p.S_pad || last == 1) ? p.M_pad : p.S_pad;
    const unsigned blocks = static_cast<unsigned>(p.BH) * (most / (kPostRows * 256 / (D / 8)));
    xattn_post_kernel<D><<<dim3(blocks, last - first), 256, 0, s>>>(p, first);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_xattn_bwd(int d, int dm, const XattnBwdMaps& m, const XattnBwdParams& p, int dev, int sms,
                                  cudaStream_t s) {
  if (d == 64) return launch<64, 64>(m, p, dev, sms, s);
  if (dm == 80) return launch<128, 80>(m, p, dev, sms, s);
  return launch<128, 128>(m, p, dev, sms, s);
}

}  // namespace mw
