// C ABI of the conditioning path (declared in include/mw_bca.h): cross attention
// to an encoder's states and layer norm.  As in mw_abi.cu, arguments are checked
// on the host before any CUDA call.
#include <algorithm>
#include <climits>
#include <cmath>

#include "mw_bca.h"
#include "mw_host.h"
#include "mw_internal.h"

using namespace mw;

namespace {

// Sizes of a cross attention call, with the query heads that share a head of K
// and V as one sequence of rows (they lie one after another in [B, H, M, d]).
struct XattnSizes {
  int BH = 0, rows = 0;  // heads of K and V over the batch; query rows of each
};

mw_status xattn_sizes(XattnSizes* out, int B, int H, int Hkv, int M, int S, int d) {
  MW_TRY(check_dims(B, H, d));
  if (Hkv < 1 || H % Hkv != 0)
    return fail(MW_ERR_INVALID_ARG, "H=%d is not a multiple of Hkv=%d", H, Hkv);
  if (M < 0 || S < 0 || S > (1 << 24))
    return fail(MW_ERR_INVALID_ARG, "M=%d and S=%d must be >= 0 and S <= 2^24", M, S);
  const long long rows = static_cast<long long>(H / Hkv) * M;
  if (rows > (1 << 24))
    return fail(MW_ERR_INVALID_ARG, "H/Hkv*M=%lld exceeds 2^24", rows);
  MW_TRY(check_tokens(static_cast<long long>(B) * Hkv, rows));
  MW_TRY(check_tokens(static_cast<long long>(B) * Hkv, S));
  out->BH = B * Hkv;
  out->rows = static_cast<int>(rows);
  return MW_OK;
}

// Key ranges of the forward on tensor cores: enough that the blocks fill the SMs,
// against the cost of a range (about three key tiles' time).
int xattn_splits(int BH, int rows, int S) {
  const long long blocks = static_cast<long long>(BH) * ceil_div(rows, kFwdBlockRows);
  const int tiles = ceil_div(S, kTileRows);
  int best = 1;
  long long best_cost = LLONG_MAX;
  for (int s = 1; s <= kMaxSplits && s <= tiles; ++s) {
    const long long waves = ceil_div(blocks * s, kNormSms);
    const long long cost = waves * (ceil_div(tiles, s) + (s > 1 ? 3 : 0)) + (s > 1 ? 6 : 0);
    if (cost < best_cost) {
      best_cost = cost;
      best = s;
    }
  }
  return best;
}

size_t xattn_ws(const XattnSizes& z, int S, int d) {
  if (z.rows <= kXattnFewRows) return 0;
  const int splits = xattn_splits(z.BH, z.rows, S);
  if (splits == 1) return 0;
  const size_t rows = static_cast<size_t>(splits) * z.BH * z.rows;
  return align256(rows * kernel_d(d) * sizeof(float)) + align256(rows * sizeof(float));
}

// The order of the backward's work, from a model of the time (us): steps of t and a
// sweep's start and end; key-major also two passes and a quarter over dQ in HBM (zeroed,
// read, bf16 written; written once in bf16 query-major).  Query-major a run ends after
// few tiles, and its dQ is read back: a step costs more, and the first ones 6 us.  Heads x
// query tiles x key tiles at d = 64, us of all kernels, query-/key-major: 48 x 110 x 2 181 /
// 223, 152 x 40 x 2 204 / 231, 100 x 24 x 5 195 / 183, 16 x 110 x 9 220 / 177, 64 x 3 x 2 28 /
// 21.  d = 128, where dQ cannot leave with the last sweep (no shared memory for it), was
// slower query-major (152 x 40 x 2 522 / 424, 16 x 110 x 9 395 / 305, 48 x 110 x 2 420 each):
// key-major from two key tiles on.
struct XattnBwdPlan {
  bool key_major = false;
  int ranges = 1;  // key-major: of a head's query tiles (more than one: the number is worked
                   // out again on the device, for the states that the samples have)
  int run = 1;     // query-major: query tiles of a run, so that the dQ of all runs in work stays in L2
};

XattnBwdPlan xattn_bwd_plan(int BH, int q_tiles, int k_tiles, int D) {
  XattnBwdPlan best;
  best.run = 16;  // 48 x 110 x 2: runs of 4 227, of 8 201, of 16 186, of 20 182 us
  if (k_tiles == 1) return best;
  const double acc = 4e-6 * BH * static_cast<double>(q_tiles) * kTileRows * D / 6.5;  // us a pass
  double best_cost = D == 64 ? ceil_div(static_cast<long long>(BH) * q_tiles, kNormSms) * k_tiles * 2.05 + 6 : INFINITY;
  const double acc_kv = 8e-6 * BH * static_cast<double>(k_tiles) * kTileRows * D / 6.5;  // of dK's and dV's
  auto cost = [&](int r) {
    return ceil_div(static_cast<long long>(BH) * r * k_tiles, kNormSms) *
               (ceil_div(q_tiles, r) * xattn_step_us(D) + xattn_sweep_us(D)) +
           2.25 * (acc + (r > 1 ? acc_kv : 0));
  };
  const int most = q_tiles < kXattnMaxRanges ? q_tiles : kXattnMaxRanges;
  for (int r = 1; r <= most; ++r)
    if (cost(r) < best_cost) {
      best_cost = cost(r);
      best.key_major = true;
      best.ranges = r;
    }
  return best;
}

// The backward's workspace: byte offsets of its fp32 arrays.
struct XattnBwdWs {
  int M_pad = 0, S_pad = 0;
  bool dkv_whole = false;  // no accumulators of dK and dV
  XattnBwdPlan plan;
  size_t shares = 0, dq = 0, dkv = 0, dkv_bytes = 0, lse2 = 0, delta = 0, bias = 0, total = 0;
};

XattnBwdWs xattn_bwd_ws(const XattnSizes& z, int S, int d) {
  XattnBwdWs w;
  const int D = kernel_d(d);
  w.M_pad = ceil_div(z.rows, kTileRows) * kTileRows;
  w.S_pad = ceil_div(S, kTileRows) * kTileRows;
  w.plan = xattn_bwd_plan(z.BH, w.M_pad / kTileRows, w.S_pad / kTileRows, D);
  const size_t rows = static_cast<size_t>(z.BH) * w.M_pad, keys = static_cast<size_t>(z.BH) * w.S_pad;
  w.dq = align256((kXattnMaxCtas + 1) * sizeof(int2));
  const bool dq_acc = w.S_pad > kTileRows;
  w.dkv = w.dq + (dq_acc ? align256(rows * D * 4) : 0);
  w.dkv_whole = w.plan.key_major && w.plan.ranges == 1;
  w.dkv_bytes = w.dkv_whole ? 0 : 2 * keys * D * 4;
  w.lse2 = w.dkv + align256(w.dkv_bytes);
  w.delta = w.lse2 + (D == 64 ? 0 : align256(rows * 4));
  w.bias = w.delta + (D == 64 ? 0 : align256(rows * 4));
  w.total = w.bias + (D == 64 ? align256(rows * 32) : 0);
  return w;
}

mw_status check_scale(float scale) {
  if (!(scale > 0.f) || !std::isfinite(scale))
    return fail(MW_ERR_INVALID_ARG, "scale must be > 0 and finite");
  return MW_OK;
}

}  // namespace

extern "C" {

size_t mw_xattn_workspace_size(int B, int H, int Hkv, int M, int S, int d) {
  XattnSizes z;
  if (xattn_sizes(&z, B, H, Hkv, M, S, d) != MW_OK) return 0;
  return xattn_ws(z, S, d);
}

mw_status mw_xattn_fwd(const void* q, const void* k, const void* v, const int* kv_len, void* o,
                       float* lse, void* workspace, size_t ws_bytes, int B, int H, int Hkv, int M,
                       int S, int d, float scale, void* stream) {
  XattnSizes z;
  MW_TRY(xattn_sizes(&z, B, H, Hkv, M, S, d));
  MW_TRY(check_scale(scale));
  if (M == 0) return ok();
  MW_TRY(check_ptr(q, "q"));
  MW_TRY(check_ptr(o, "o"));
  if (S > 0) {
    MW_TRY(check_ptr(k, "k"));
    MW_TRY(check_ptr(v, "v"));
  }
  MW_TRY(check_f32(kv_len, "kv_len"));
  MW_TRY(check_f32(lse, "lse"));
  const size_t need = xattn_ws(z, S, d);
  if (need > 0) {
    if (workspace == nullptr || ws_bytes < need)
      return fail(MW_ERR_WORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u)
      return fail(MW_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  if (z.rows > kXattnFewRows) {
    const int D = kernel_d(d);
    XattnTcParams p{};
    MW_TRY(status_ptr(scope.device(), &p.status));
    CUtensorMap tq, tk, tv, to;
    MW_TRY(make_map(&tq, q, z.rows, z.BH, d, "q"));
    tk = tv = tq;  // (no states: never read)
    if (S > 0) {
      MW_TRY(make_map(&tk, k, S, z.BH, d, "k"));
      MW_TRY(make_map(&tv, v, S, z.BH, d, "v"));
    }
    MW_TRY(encode_rows_map(&to, o, z.rows, z.BH, d, true));
    p.kv_len = kv_len;
    p.o = static_cast<__nv_bfloat16*>(o);
    p.lse = lse;
    p.BH = z.BH;
    p.heads = Hkv;
    p.M = z.rows;
    p.S = S;
    p.d = d;
    p.n_qblocks = ceil_div(z.rows, kFwdBlockRows);
    p.num_splits = need > 0 ? xattn_splits(z.BH, z.rows, S) : 1;
    p.items = z.BH * p.n_qblocks * p.num_splits;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.budget_ns = budget_ns();
    p.debug_skip_q = debug_skip_q();
    if (p.num_splits > 1) {
      p.o_part = static_cast<float*>(workspace);
      p.lse_part = reinterpret_cast<float*>(
          static_cast<char*>(workspace) +
          align256(static_cast<size_t>(p.num_splits) * z.BH * z.rows * D * sizeof(float)));
    }
    MW_TRY(launch_status(launch_xattn_tc(D, mma_d(d), tq, tk, tv, to, p, scope.device(), sm_count(), s),
                         "cross attention forward launch"));
    if (p.num_splits > 1)
      MW_TRY(launch_status(launch_combine(D, d, p.o_part, p.lse_part, p.o, lse, p.num_splits, z.BH,
                                          z.rows, CommitJob{}, s),
                           "combine kernel launch"));
    return ok();
  }
  XattnFewParams p{};
  MW_TRY(status_ptr(scope.device(), &p.status));
  CUtensorMap tk, tv;
  if (S > 0) {
    MW_TRY(make_map(&tk, k, S, z.BH, d, "k", kXattnFewKeys));
    MW_TRY(make_map(&tv, v, S, z.BH, d, "v", kXattnFewKeys));
  } else {  // never read
    MW_TRY(make_map(&tk, q, z.rows, z.BH, d, "q"));
    tv = tk;
  }
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.kv_len = kv_len;
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  p.BH = z.BH;
  p.heads = Hkv;
  p.M = z.rows;
  p.S = S;
  p.d = d;
  p.sms = sm_count();
  p.scale_log2 = scale * 1.4426950408889634f;
  p.budget_ns = budget_ns();
  p.debug_skip_q = debug_skip_q();
  return launch_status(launch_xattn_few(kernel_d(d), tk, tv, p, scope.device(), s),
                       "cross attention forward launch");
}

size_t mw_xattn_bwd_workspace_size(int B, int H, int Hkv, int M, int S, int d) {
  XattnSizes z;
  if (xattn_sizes(&z, B, H, Hkv, M, S, d) != MW_OK || M == 0 || S == 0) return 0;
  return xattn_bwd_ws(z, S, d).total;
}

mw_status mw_xattn_bwd(const void* q, const void* k, const void* v, const int* kv_len, const void* o,
                       const float* lse, const void* dout, void* dq, void* dk, void* dv,
                       void* workspace, size_t ws_bytes, int B, int H, int Hkv, int M, int S, int d,
                       float scale, void* stream) {
  XattnSizes z;
  MW_TRY(xattn_sizes(&z, B, H, Hkv, M, S, d));
  MW_TRY(check_scale(scale));
  if (M > 0) {
    MW_TRY(check_ptr(q, "q"));
    MW_TRY(check_ptr(o, "o"));
    MW_TRY(check_ptr(dout, "dout"));
    MW_TRY(check_ptr(dq, "dq"));
    if (lse == nullptr) return fail(MW_ERR_INVALID_ARG, "lse is NULL");
    MW_TRY(check_f32(lse, "lse"));
  }
  if (S > 0) {
    MW_TRY(check_ptr(k, "k"));
    MW_TRY(check_ptr(v, "v"));
    MW_TRY(check_ptr(dk, "dk"));
    MW_TRY(check_ptr(dv, "dv"));
  }
  MW_TRY(check_f32(kv_len, "kv_len"));
  const bool empty = M == 0 || S == 0;
  const XattnBwdWs ws = empty ? XattnBwdWs{} : xattn_bwd_ws(z, S, d);
  if (!empty) {
    if (workspace == nullptr || ws_bytes < ws.total)
      return fail(MW_ERR_WORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, ws.total);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u)
      return fail(MW_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  if (empty) {  // no pairs: zero gradients
    const size_t row = static_cast<size_t>(d) * 2;
    if (M > 0) MW_TRY(launch_status(cudaMemsetAsync(dq, 0, z.BH * row * z.rows, s), "clearing dq"));
    if (S > 0) {
      MW_TRY(launch_status(cudaMemsetAsync(dk, 0, z.BH * row * S, s), "clearing dk"));
      MW_TRY(launch_status(cudaMemsetAsync(dv, 0, z.BH * row * S, s), "clearing dv"));
    }
    return ok();
  }
  const int D = kernel_d(d);
  char* base = static_cast<char*>(workspace);
  auto at = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
  XattnBwdParams p{};
  MW_TRY(status_ptr(scope.device(), &p.status));
  p.kv_len = kv_len;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.o = static_cast<const __nv_bfloat16*>(o);
  p.dout = static_cast<const __nv_bfloat16*>(dout);
  p.lse = lse;
  p.dq = static_cast<__nv_bfloat16*>(dq);
  p.dk = static_cast<__nv_bfloat16*>(dk);
  p.dv = static_cast<__nv_bfloat16*>(dv);
  p.BH = z.BH;
  p.heads = Hkv;
  p.M = z.rows;
  p.M_pad = ws.M_pad;
  p.S = S;
  p.S_pad = ws.S_pad;
  p.d = d;
  if (kv_len == nullptr) p.heads = z.BH;  // one sample of all heads
  p.samples = z.BH / p.heads;
  p.q_tiles = ws.M_pad / kTileRows;
  p.k_tiles = ws.S_pad / kTileRows;
  p.key_major = ws.plan.key_major;
  p.run = ws.plan.run;
  p.dkv_whole = ws.dkv_whole;
  p.zero_dq = p.key_major;
  p.wide_dkv = wide_rows(dk, d) && wide_rows(dv, d);
  p.scale = scale;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.lse2 = at(ws.lse2);
  p.delta = at(ws.delta);
  p.bias = at(ws.bias);
  p.shares = reinterpret_cast<int2*>(base + ws.shares);
  p.dq_acc = at(ws.dq);
  p.dkv_acc = at(ws.dkv);
  p.dkv_float4s = static_cast<long long>(ws.dkv_bytes / 16);
  p.budget_ns = budget_ns();
  p.debug_skip_q = debug_skip_q();
  XattnBwdMaps m;
  MW_TRY(make_map(&m.q, q, z.rows, z.BH, d, "q"));
  MW_TRY(make_map(&m.k, k, S, z.BH, d, "k"));
  MW_TRY(make_map(&m.v, v, S, z.BH, d, "v"));
  MW_TRY(make_map(&m.dout, dout, z.rows, z.BH, d, "dout"));
  // (maps that no launch of these sizes uses stand in for one another)
  m.dq = m.dk = m.dv = m.bias = m.dq_out = m.q;
  if (ws.dkv > ws.dq) MW_TRY(make_map(&m.dq, p.dq_acc, ws.M_pad, z.BH, D, "dq_acc", 32, true, d));
  if (ws.dkv_bytes > 0) {
    MW_TRY(make_map(&m.dk, p.dkv_acc, ws.S_pad, z.BH, D, "dk_acc", 32, true, d));
    MW_TRY(make_map(&m.dv, p.dkv_acc + static_cast<size_t>(z.BH) * ws.S_pad * D, ws.S_pad, z.BH, D, "dv_acc", 32,
                    true, d));
  }
  if (D == 64) MW_TRY(encode_bias_map(&m.bias, p.bias, ws.M_pad, z.BH, kTileRows));
  MW_TRY(encode_rows_map(&m.dq_out, dq, z.rows, z.BH, d, D == 64));
  return launch_status(launch_xattn_bwd(D, mma_d(d), m, p, scope.device(), std::min(sm_count(), kXattnMaxCtas), s),
                       "cross attention backward launch");
}

mw_status mw_layernorm_fwd(const void* x, const void* weight, const void* bias, void* y, float* mean,
                           float* rstd, long long rows, int C, int groups, float eps, int x_dtype,
                           int y_dtype, int param_dtype, void* stream) {
  MW_TRY(norm_sizes(rows, C, groups, eps));
  if (!dtype_ok(x_dtype) || !dtype_ok(y_dtype) || !dtype_ok(param_dtype))
    return fail(MW_ERR_INVALID_ARG, "types must be MW_BF16 or MW_F32");
  if (x_dtype == MW_BF16 && y_dtype == MW_F32)
    return fail(MW_ERR_UNSUPPORTED, "y in fp32 needs x in fp32");
  if (rows == 0) return ok();
  MW_TRY(check_elems(x, x_dtype, "x"));
  MW_TRY(check_elems(y, y_dtype, "y"));
  if (weight) MW_TRY(check_elems(weight, param_dtype, "weight"));
  if (bias) MW_TRY(check_elems(bias, param_dtype, "bias"));
  MW_TRY(check_f32(mean, "mean"));
  MW_TRY(check_f32(rstd, "rstd"));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  NormParams p{};
  p.x = x;
  p.weight = weight;
  p.bias = bias;
  p.y = y;
  p.mean = mean;
  p.rstd = rstd;
  p.rows = rows;
  p.rows_per_group = rows / groups;
  p.C = C;
  p.groups = groups;
  p.eps = eps;
  p.x_f32 = x_dtype == MW_F32;
  p.y_f32 = y_dtype == MW_F32;
  p.param_f32 = param_dtype == MW_F32;
  return launch_status(launch_norm_fwd(p, vector_rows(C, x, weight, bias, y), sm_count(), s),
                       "layer norm forward launch");
}

size_t mw_layernorm_bwd_workspace_size(long long rows, int C, int groups) {
  if (norm_sizes(rows, C, groups, 0.f) != MW_OK || rows == 0) return 0;
  const int parts = norm_parts(rows / groups, C, groups);
  return parts > 1 ? align256(static_cast<size_t>(groups) * parts * 2 * C * sizeof(float)) : 0;
}

mw_status mw_layernorm_bwd(const void* dy, const void* x, const float* mean, const float* rstd,
                           const void* weight, void* dx, void* dweight, void* dbias, void* workspace,
                           size_t ws_bytes, long long rows, int C, int groups, int x_dtype,
                           int y_dtype, int param_dtype, void* stream) {
  MW_TRY(norm_sizes(rows, C, groups, 0.f));
  if (!dtype_ok(x_dtype) || !dtype_ok(y_dtype) || !dtype_ok(param_dtype))
    return fail(MW_ERR_INVALID_ARG, "types must be MW_BF16 or MW_F32");
  if (x_dtype == MW_BF16 && y_dtype == MW_F32)
    return fail(MW_ERR_UNSUPPORTED, "y in fp32 needs x in fp32");
  if (weight) MW_TRY(check_elems(weight, param_dtype, "weight"));
  if (dweight) MW_TRY(check_elems(dweight, param_dtype, "dweight"));
  if (dbias) MW_TRY(check_elems(dbias, param_dtype, "dbias"));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    DeviceScope scope(s);
    MW_TRY(scope.status());
    const size_t bytes = static_cast<size_t>(groups) * C * (param_dtype == MW_F32 ? 4 : 2);
    for (void* g : {dweight, dbias})
      if (g) MW_TRY(launch_status(cudaMemsetAsync(g, 0, bytes, s), "clearing a gradient"));
    return ok();
  }
  MW_TRY(check_elems(dy, y_dtype, "dy"));
  MW_TRY(check_elems(x, x_dtype, "x"));
  MW_TRY(check_elems(dx, x_dtype, "dx"));
  MW_TRY(check_elems(mean, MW_F32, "mean"));
  MW_TRY(check_elems(rstd, MW_F32, "rstd"));
  const size_t need = dweight || dbias ? mw_layernorm_bwd_workspace_size(rows, C, groups) : 0;
  if (need > 0) {
    if (workspace == nullptr || ws_bytes < need)
      return fail(MW_ERR_WORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u)
      return fail(MW_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  }
  DeviceScope scope(s);
  MW_TRY(scope.status());
  NormParams p{};
  p.dy = dy;
  p.x = x;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.weight = weight;
  p.dx = dx;
  p.dweight = dweight;
  p.dbias = dbias;
  p.partial = static_cast<float*>(workspace);
  p.rows = rows;
  p.rows_per_group = rows / groups;
  p.C = C;
  p.groups = groups;
  p.parts = norm_parts(rows / groups, C, groups);
  p.x_f32 = x_dtype == MW_F32;
  p.y_f32 = y_dtype == MW_F32;
  p.param_f32 = param_dtype == MW_F32;
  return launch_status(launch_norm_bwd(p, vector_rows(C, dy, x, weight, dx), scope.device(), s),
                       "layer norm backward launch");
}

}  // extern "C"
