// Internal interfaces between the C-ABI layer and the CUDA kernels.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace mw {

// Rows of one query tile / key tile (the tcgen05 M and N of S = Q K^T).
constexpr int kTileRows = 128;
// Query tiles that share one key/value stream inside a forward CTA.
constexpr int kFwdQTiles = 2;
constexpr int kFwdBlockRows = kTileRows * kFwdQTiles;
constexpr int kMaxSplits = 16;

// Query rows per step of the backward key-tile kernel.
__host__ __device__ constexpr int bwd_q_rows(int) { return 128; }

// Forward over one (b,h) query block against up to three key segments:
//   A: ring rows [head, head + lenA)        (committed history, all visible)
//   B: ring rows [0, lenB)                  (the part after the wrap)
//   C: the queries' own rows [0, rows_q)    (chunk-causal: key < (chunk(i)+1) T)
// Training uses C only (ring_len = 0).
// RoPE frequencies omega_i = base^(-2i / rope_dims), i < rope_dims / 2,
// computed in fp64 on the host and handed over as two floats (hi + lo), so
// that frame * omega keeps its low bits for frames up to 2^24.
constexpr int kMaxRopePairs = 64;  // head dims up to 128
struct RopeFreq {
  float hi[kMaxRopePairs];
  float lo[kMaxRopePairs];
};

struct FwdParams {
  int BH;
  int rows_q;       // query rows (= rows of segment C) per (b,h)
  int d_io;         // head dim of the caller's tensors (<= the kernel's D; the
                    // TMA maps zero-fill the columns in between)
  int T;            // chunk length in tokens
  int n_qblocks;    // ceil(rows_q / kFwdBlockRows)
  int head_groups;  // the heads are scheduled in this many groups (1..BH)
  int ring_cap;
  int ring_head;
  int ring_len;
  int sink_len;     // tokens of the sink anchor, visited before the ring
  // RoPE re-shift (0 rope_dims: off): the sink anchor's keys turn forward by
  // rope_shift frames as they are read (the frequencies are a kernel
  // parameter of their own)
  int rope_dims;
  int rope_shift;
  int num_splits;   // 1: write bf16 O + LSE; >1: fp32 partials for the combine
  float scale_log2; // softmax scale * log2(e)
  __nv_bfloat16* o;
  bool wide_out;    // every row of o starts at a multiple of 32 bytes
  float* lse;       // nullable
  float* o_part;    // [splits, BH, rows_q, d]
  float* lse_part;  // [splits, BH, rows_q]
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;  // test hook: never load Q, so the MMA warp's wait expires
};

struct BwdParams {
  int BH;
  int head_groups;  // CTA order: groups of heads one after another
  int N;            // tokens per (b,h)
  int N_pad;        // N rounded up to kTileRows
  int d_io;         // head dim of the caller's tensors (<= the kernel's D)
  int T;
  float scale_log2;
  float scale;
  const float* lse2;   // [BH, N_pad]  LSE * log2(e); +inf on padding rows
  const float* delta;  // [BH, N_pad]  rowsum(dO * O); 0 on padding rows
  float* dq_acc;       // [BH, N_pad, d] fp32
  __nv_bfloat16* dk;
  __nv_bfloat16* dv;
  bool wide_out;       // every row of both starts at a multiple of 32 bytes
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;  // test hook: never load Q, so the first S^T wait expires
};

// A ring commit (Sec. 3.5): rows [0, rows) of each head of k_src / v_src
// ([B,H,src_rows,d], src_rows >= rows) go to ring rows (slot + r) mod cap of
// k_cache / v_cache ([B,H,cap,d]).  rows == 0: nothing to do.
struct CommitJob {
  __nv_bfloat16* kc = nullptr;
  __nv_bfloat16* vc = nullptr;
  const __nv_bfloat16* ks = nullptr;
  const __nv_bfloat16* vs = nullptr;
  int cap = 1, slot = 0, rows = 0, src_rows = 0, d = 0, BH = 0;
};

// One 16-byte piece of a commit: piece `idx` of head bh (row idx / (d/8),
// 16-byte column chunk idx % (d/8)) of K and of V.
__device__ __forceinline__ void commit_piece(const CommitJob& j, int bh, int idx) {
  const int pieces = j.d / 8;
  const int piece = idx % pieces;
  const int r = idx / pieces;
  int dst = j.slot + r;
  if (dst >= j.cap) dst -= j.cap;  // slot < cap and rows <= cap
  const size_t so = (static_cast<size_t>(bh) * j.src_rows + r) * j.d + piece * 8;
  const size_t dso = (static_cast<size_t>(bh) * j.cap + dst) * j.d + piece * 8;
  *reinterpret_cast<uint4*>(j.kc + dso) = *reinterpret_cast<const uint4*>(j.ks + so);
  *reinterpret_cast<uint4*>(j.vc + dso) = *reinterpret_cast<const uint4*>(j.vs + so);
}

// Programmatic dependent launch of the forward, the split combine and the
// commit (option "pdl", on by default): each may start while the previous
// kernel in the stream finishes and waits in-kernel before touching global
// memory.  pdl_config fills `cfg` (and its one attribute `attr`).
extern int g_pdl_enabled;
inline void pdl_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute& attr, dim3 grid, dim3 block,
                       size_t smem, cudaStream_t s) {
  cfg = cudaLaunchConfig_t{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = g_pdl_enabled ? 1 : 0;
}

constexpr int kMaxDevices = 64;

// Runs a kernel's setup once on each device: a function's attributes (its
// dynamic shared memory) hold on the device that is current when they are set.
// Threads may run it side by side; a setup that fails is tried again.
class OncePerDevice {
 public:
  // dev: the current device
  template <class F>
  cudaError_t operator()(int dev, F&& setup) {
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (done_[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t e = setup();
    if (e == cudaSuccess) done_[dev].store(true, std::memory_order_release);
    return e;
  }

 private:
  std::atomic<bool> done_[kMaxDevices] = {};
};

// Launchers (return cudaGetLastError() of the launch; dev: the current device).
// tkr/tvr: ring buffer maps; tks/tvs: sink anchor maps (any valid map when
// the segment is empty)
// d: tile width (64 or 128); dm: MMA width (d, or 80 on the 128-wide tiles
// for head dims up to 80)
// top: the fp32 split partials p.o_part as [splits * BH][rows_q][d] with
// 32-column boxes (any valid map when p.num_splits == 1)
cudaError_t launch_fwd(int d, int dm, const CUtensorMap& tq, const CUtensorMap& tk,
                       const CUtensorMap& tv, const CUtensorMap& tkr, const CUtensorMap& tvr, const CUtensorMap& tks,
                       const CUtensorMap& tvs, const CUtensorMap& top, const FwdParams& p,
                       const RopeFreq& rope_om, int dev, cudaStream_t s);
// d: the kernels' head dim (64 or 128); d_io: the caller's (a multiple of 8, <= d)
// The combine's launch also carries the ring commit `cj` (if cj.rows > 0)
// in blocks of its own: both only run once the forward has finished, and
// they touch disjoint memory.
cudaError_t launch_combine(int d, int d_io, const float* o_part, const float* lse_part,
                           __nv_bfloat16* o, float* lse, int splits, int BH, int rows,
                           const CommitJob& cj, cudaStream_t s);
// bias (d = 64, else null): per padded row 8 floats (hi, lo of -LSE/scale;
// hi, lo of -D; 4 zeros), the B operand of the tf32 MMAs that add those
// per-query terms to S^T and dP^T
cudaError_t launch_bwd_pre(int d, int d_io, const __nv_bfloat16* o, const __nv_bfloat16* dout,
                           const float* lse, float* lse2, float* delta, float* dq_acc,
                           float* bias, float inv_scale, int BH, int N, int N_pad, cudaStream_t s);
// tdq: f32 map over dQacc [BH, N_pad, d] with 32 x 32 boxes (128-byte
// swizzle), the target of the TMA reduce-adds
// dm: MMA width as for launch_fwd
// tbias (d = 64): f32 map over the bias rows [BH, N_pad, 8], 8 x 128 boxes,
// 32-byte swizzle (d = 128: any map, unused)
cudaError_t launch_bwd_main(int d, int dm, const CUtensorMap& tq, const CUtensorMap& tk,
                            const CUtensorMap& tv, const CUtensorMap& tdo, const CUtensorMap& tdq,
                            const CUtensorMap& tbias, const BwdParams& p, int dev, cudaStream_t s);
cudaError_t launch_bwd_post(int d, int d_io, const float* dq_acc, __nv_bfloat16* dq, float scale,
                            int BH, int N, int N_pad, cudaStream_t s);
// d: any multiple of 8 (rows are copied in 16-byte pieces)
cudaError_t launch_commit(const CommitJob& j, cudaStream_t s);
// QKV split + temporal RoPE: qkv [B, N, 3, H, d] -> q, k, v [B, H, N, d]
// (d a multiple of 8; rope_dims = 0 is a plain split)
cudaError_t launch_qkv_rope(const __nv_bfloat16* qkv, __nv_bfloat16* q, __nv_bfloat16* k,
                            __nv_bfloat16* v, int B, int N, int H, int d, int rope_dims,
                            const RopeFreq& omega, int per_frame, int first_frame,
                            cudaStream_t s);


// Layer norm (mw_norm.cu).
constexpr int kNormMaxC = 8192;
// The SMs that the backward's parts are planned for (a GB300's, so that the plan
// needs no device).
constexpr int kNormSms = 152;
struct NormParams {
  const void* x;       // [rows, C], bf16 or fp32
  const void* weight;  // [groups, C] or null (all 1)
  const void* bias;    // [groups, C] or null (all 0)
  void* y;             // forward: [rows, C], bf16 or fp32
  float* mean;         // [rows]; forward: nullable
  float* rstd;
  const void* dy;      // backward: y's type
  void* dx;            // x's type
  void* dweight;       // the parameters' type, nullable
  void* dbias;
  float* partial;      // [groups * parts, 2, C] where parts > 1
  long long rows, rows_per_group;
  int C, groups;
  int parts;           // backward: blocks that share a group's rows
  int W;               // warps that share a row (set by the launcher)
  float eps;
  bool x_f32, y_f32, param_f32;
};
// Blocks a group of the backward.
int norm_parts(long long rows_per_group, int C, int groups);
// vec: C is a multiple of 8 and every pointer 16-byte aligned
cudaError_t launch_norm_fwd(NormParams p, bool vec, int sms, cudaStream_t s);
cudaError_t launch_norm_bwd(NormParams p, bool vec, int dev, cudaStream_t s);

// RMS norm (mw_rms.cu).
enum { kRmsBf16 = 0, kRmsF32 = 1, kRmsCodes = 2 };  // y
struct RmsParams {
  const void* x;         // [rows, C], bf16 or fp32
  const void* residual;  // x's type, nullable
  const void* weight;    // [groups, C] or null (all 1)
  void* y;               // forward: [rows, C]
  uint8_t* y_scale;      // [rows, ceil(C / 128)] with codes
  void* h;               // x's type: the sum (forward: with a residual), the backward's rows
  float* rstd;           // [rows]; forward: nullable
  const void* dy;        // backward: y's type
  const void* dh;        // x's type, nullable
  void* dx;
  void* dweight;         // the weight's type, nullable
  float* partial;        // [groups * parts, C] where parts > 1
  long long rows, rows_per_group;
  int C, groups;
  int parts;             // blocks that share a group's rows (forward: set by the launcher)
  int W;                 // warps that share a row (set by the launcher)
  float eps;
  int y_type;
  bool x_f32, param_f32;
};
int rms_parts(long long rows_per_group, int C, int groups);
// vec: C is a multiple of 8 and every pointer 16-byte aligned
cudaError_t launch_rms_fwd(RmsParams p, bool vec, int dev, int sms, cudaStream_t s);
cudaError_t launch_rms_bwd(RmsParams p, bool vec, int dev, cudaStream_t s);

// Cross attention: BH heads of K and V [BH, S, d], each with M rows of Q (those of all
// the query heads that share it, which lie one after another); head bh belongs to
// sample bh / heads, whose first kv_len[...] keys count (null: all S).
// Forward on tensor cores (mw_xattn_fwd.cu): blocks of kFwdBlockRows rows of one
// head against one of num_splits ranges of its key tiles.
struct XattnTcParams {
  const int* kv_len;
  __nv_bfloat16* o;
  float* lse;          // nullable
  float* o_part;       // [num_splits, BH * M, D] where num_splits > 1
  float* lse_part;     // [num_splits, BH * M]; +inf: its range was given up
  int BH, heads, M, S, d;
  int n_qblocks, num_splits;
  int items;           // BH * n_qblocks * num_splits
  float scale_log2;
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;    // test hook: never load Q, so the issuers' wait expires
};
// d, dm: tile and MMA width as for launch_fwd; to: o in 32 x 64 boxes with the 128-byte
// swizzle; sms: CTAs at most
cudaError_t launch_xattn_tc(int d, int dm, const CUtensorMap& tq, const CUtensorMap& tk,
                            const CUtensorMap& tv, const CUtensorMap& to, const XattnTcParams& p, int dev, int sms,
                            cudaStream_t s);
// Forward of at most kXattnFewRows rows a head (mw_xattn_few.cu).
constexpr int kXattnFewRows = 16;
constexpr int kXattnFewKeys = 64;  // of a copy: the rows of tk's and tv's boxes
struct XattnFewParams {
  const __nv_bfloat16* q;
  const int* kv_len;
  __nv_bfloat16* o;
  float* lse;          // nullable
  int BH, heads, M, S, d;
  int sms;
  float scale_log2;
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;    // test hook: never load K and V
};
// d: tile width (64 or 128); without states any maps
cudaError_t launch_xattn_few(int d, const CUtensorMap& tk, const CUtensorMap& tv, const XattnFewParams& p, int dev,
                             cudaStream_t s);

// Backward on tensor cores (mw_xattn_bwd.cu).
constexpr int kXattnMaxCtas = 1023;
constexpr int kXattnMaxRanges = 64;
// Key-major, us: a step, and what a sweep's start and end add (24 x 40, 12 x 8 tiles).
constexpr float xattn_step_us(int D) { return D == 64 ? 1.55f : 2.25f; }
constexpr float xattn_sweep_us(int D) { return D == 64 ? 1.f : 2.f; }
struct XattnBwdParams {
  const int* kv_len;
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  const __nv_bfloat16* o;
  const __nv_bfloat16* dout;
  const float* lse;
  __nv_bfloat16* dq;
  __nv_bfloat16* dk;
  __nv_bfloat16* dv;
  int BH, heads, M, M_pad, S, S_pad, d;  // _pad: rounded up to kTileRows
  int samples;         // BH / heads (without kv_len one of BH heads, which is the same)
  int q_tiles, k_tiles;  // of a head's rows; of S states
  bool key_major;      // a piece of work is one key tile, else a run of query tiles
  int run;             // query-major: query tiles of a run at most
  bool dkv_whole;      // key-major: one sweep makes all of a key tile's dK and dV
  bool zero_dq;        // dq_acc is only added to
  bool wide_dkv;  // every row of dK and dV starts at a multiple of 32 bytes
  float scale, scale_log2;
  float* lse2;         // [BH, M_pad] (d = 64: unused, as delta)
  float* delta;        // [BH, M_pad]
  float* bias;         // [BH, M_pad, 8] (d = 64)
  int2* shares;        // query-major: where each CTA's share begins, and the end (sample, unit);
                       // key-major: [0].x ranges of a head's query tiles
  float* dq_acc;       // [BH, M_pad, D]
  float* dkv_acc;      // [2, BH, S_pad, D] unless dkv_whole: dK, then dV
  long long dkv_float4s;  // its size
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;
};
// dq [BH, M_pad, D], dk, dv [BH, S_pad, D]: f32 accumulators, 32 x 32 boxes; bias as
// for launch_bwd_main; dq_out: the caller's dQ, 32 x 32 boxes without swizzle
struct XattnBwdMaps {
  CUtensorMap q, k, v, dout, dq, dk, dv, bias, dq_out;
};
cudaError_t launch_xattn_bwd(int d, int dm, const XattnBwdMaps& m, const XattnBwdParams& p, int dev, int sms,
                             cudaStream_t s);

// Matrices in 8 bits (e4m3) with a scale (e8m0) for every block of 128: of a row's
// elements (rows), of a column's (columns), or of both (tiles).
constexpr int kFp8Block = 128;
constexpr int kFp8Splits = 8;  // CTAs that share a contraction at most
// Blocks that a result sums in tensor memory in a row at most, four additions each, which cut: of
// positive terms 2e-5 is lost of an fp32 result, and 6.5e-4 of one in bf16, a third of its rounding.
constexpr int kFp8Chunk = 64, kFp8ChunkBf16 = 2048;
struct Fp8FormParams {
  const void* x;         // [rows, C], bf16 or fp32
  uint8_t* q;            // rows or tiles: [rows, C]
  uint8_t* scale;        // [rows, ceil(C / 128)], tiles [ceil(rows / 128), ceil(C / 128)]
  uint8_t* q_columns;    // columns: [rows, C]
  uint8_t* scale_columns;  // [ceil(rows / 128), C]
  long long rows;
  int C;
  bool x_f32;
};
enum class Fp8Form { kRows, kColumns, kTiles, kBoth };
cudaError_t launch_fp8_form(const Fp8FormParams& p, Fp8Form form, cudaStream_t s);

// Product of two of them (mw_fp8_mm.cu): rows_a x rows_b results over `blocks` of the contraction.
// How the scales of a row's blocks are read: one for 128 rows; four blocks of a row as a word;
// a block of four rows as a word; a byte each.
enum class Fp8Read { kTile, kWords, kQuads, kBytes };
struct Fp8Scales {
  const uint8_t* p;
  long long row, block;  // bytes from a row (kTile: from 128 rows), and from a block, to the next
  Fp8Read read;
};
struct Fp8MmParams {
  Fp8Scales a_scales, b_scales;
  void* out;             // bf16 or fp32, rows of ld
  long long ld;
  int rows_a, rows_b, blocks;
  int tiles_p, tiles_q;  // of 128 rows of A (pairs: 256), of bn rows of B
  int splits;            // join: CTAs of a tile; pairs: pairs of a tile
  int ctas;              // pairs: CTAs at most
  int chunk;             // blocks (whole words of scales) that are summed in tensor memory at once, before the
                         // output takes them (pairs) or a sum beside them (join); or a pair's share of a tile's
  bool a_columns, b_columns;  // rows of the operand lie across the contraction
  bool swap;             // join: a row of the output is one of B
  bool out_f32;
  bool out_quads;        // groups of four elements from any multiple of four on are aligned
  bool tma_out;          // tc is a map of the output
  unsigned* status;
  unsigned long long budget_ns;
  int debug_skip_q;      // test hook: never load A and B
};
// Clusters of r CTAs (1 to kFp8Splits), a CTA an SM, that device dev, the current one, runs at once.
// Its groups of SMs are not alike (152 SMs: 76 clusters of 2, 46 of 3, 36 of 4, 23 of 6, 15 of 8).
// Asked of the device once.
cudaError_t fp8_clusters(int r, int dev, int* n);
// bn: rows of B of a tile (join: 16, 32, 64 or 128; pairs: 128 or 256); ta, tb: boxes of 128
// bytes x 128 rows (join's tb, and pairs' of 128 rows: x bn and 64 rows where B runs along the
// contraction); tc: 32 rows x 64 bytes
cudaError_t launch_fp8_mm(int bn, bool join, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc,
                          const Fp8MmParams& p, int dev, cudaStream_t s);

}  // namespace mw
