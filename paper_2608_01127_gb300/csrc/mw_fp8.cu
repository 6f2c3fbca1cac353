// C ABI of the 8-bit projections (declared in include/mw_bca.h): RMS norm, the 8-bit form
// of a matrix and the product of two.  As in mw_abi.cu, arguments are checked on the host before
// any CUDA call.
#include <algorithm>
#include <climits>
#include <cmath>

#include "mw_bca.h"
#include "mw_host.h"
#include "mw_internal.h"

using namespace mw;

namespace {

mw_status check_type(int t, const char* name) {
  if (!dtype_ok(t)) return fail(MW_ERR_INVALID_ARG, "%s must be MW_BF16 or MW_F32", name);
  return MW_OK;
}

// Rows of codes start at multiples of 16 bytes, for the copies of the product.
mw_status check_width(long long n, const char* name) {
  if (n % 16 != 0) return fail(MW_ERR_UNSUPPORTED, "%s=%lld: rows of 8-bit codes must be multiples of 16", name, n);
  return MW_OK;
}

mw_status check_size(long long n, const char* name) {
  if (n < 0 || n > (1 << 24)) return fail(MW_ERR_INVALID_ARG, "%s=%lld out of range [0, 2^24]", name, n);
  return MW_OK;
}

// How a product is cut: tiles of 256 x bn by pairs of CTAs, of which `splits` share a tile's
// contraction (bn = 256), or of 128 x bn by clusters of `splits` CTAs (join) that do.
struct MmPlan {
  int bn = 128, splits = 1;
  bool join = false, swap = false;
};

// Blocks of each of r pairs that share a contraction: whole words of scales.
int pair_share(int blocks, int r) { return ceil_div(ceil_div(blocks, r), 4) * 4; }

// A device that does not tell how many clusters it runs is an error: with a guess in its place a
// call's sums would be made in another order than the next one's.
mw_status mm_plan(int M, int N, int blocks, bool a_columns, bool b_columns, bool f32, int sms, int dev, MmPlan* plan) {
  MmPlan& best = *plan;
  const int most = std::min(kFp8Splits, blocks);
  int clusters[kFp8Splits + 1] = {};
  for (int r = 1; r <= most; ++r)
    MW_TRY(launch_status(fp8_clusters(r, dev, &clusters[r]), "asking for the clusters of a device"));
  if (clusters[1] < 1) return fail(MW_ERR_CUDA, "the device has no SM with the shared memory of a product");
  double best_cost = INFINITY;
  const bool few_m = M <= 64 && !a_columns, few_n = N <= 64 && !b_columns;
  if (few_m || few_n) {
    const int few = few_m ? M : N, tiles = ceil_div(few_m ? N : M, 128);
    best.swap = few_m;
    best.join = true;
    best.bn = few <= 16 ? 16 : few <= 32 ? 32 : 64;
    // blocks that a CTA goes through; clusters past those that run at once share SMs, which
    // costs more than their number (us for 1 to 8 CTAs: 8 x 2560 x 10240 21.2 12.7 10.2 8.6 8.0
    // 7.9 8.3 8.3; 16 x 7680 x 2560 8.8 7.4 7.6 7.2 11.2 11.5 12.1 12.4)
    for (int r = 1; r <= most; ++r) {
      if (clusters[r] == 0) continue;
      const double load = std::max(1.0, static_cast<double>(tiles) / clusters[r]);
      const double cost = ceil_div(blocks, r) * load * load;
      if (cost < best_cost) best_cost = cost, best.splits = r;
    }
    return MW_OK;
  }
  // us, fitted to 22 sizes: what a launch takes, a block of the contraction, a tile
  auto take = [&](int bn, bool join, int splits, double cost) {
    if (cost < best_cost) best_cost = cost, best.bn = bn, best.join = join, best.splits = splits;
  };
  auto tiles = [&](int rows, int bn) { return static_cast<long long>(ceil_div(M, rows)) * ceil_div(N, bn); };
  // (parts of a pair's sum are added up in the output, which bf16 cannot take; clusters keep them
  // in tensor memory: 2048 x 2048 x 524288 in 2.1 ms, by pairs in one part 1.1 ms)
  const int limit = f32 ? kFp8Chunk : kFp8ChunkBf16;
  if (f32 || blocks <= limit) {
    take(256, false, 1, 4.8 + ceil_div(tiles(256, 256), sms / 2) * (0.265 * blocks + 1.0));
    take(128, false, 1, 4.0 + ceil_div(tiles(256, 128), sms / 2) * (0.26 * blocks + 0.5));
  }
  for (int r = 1; r <= most; ++r) {
    const int share = ceil_div(blocks, r);
    if ((f32 && share > kFp8Chunk) || clusters[r] == 0) continue;
    const double load = static_cast<double>(tiles(128, 128)) / clusters[r];
    take(128, true, r, std::ceil(load) * (7.1 + 0.225 * share));
  }
  // (one round of clusters: a second one starts from nothing)
  for (int r = 2; 2 * r <= kFp8Splits && tiles(256, 256) * 2 * r <= sms; ++r) {
    const int share = pair_share(blocks, r);
    if (share > limit || share * (r - 1) >= blocks) continue;
    const double cost = 9.5 + 0.272 * share;
    if (cost < best_cost && tiles(256, 256) <= clusters[2 * r]) take(256, false, r, cost);
  }
  return MW_OK;
}

}  // namespace

extern "C" {

mw_status mw_rmsnorm_fwd(const void* x, const void* residual, const void* weight, void* y, void* y_scale, void* h,
                         float* rstd, long long rows, int C, int groups, float eps, int x_dtype, int y_dtype,
                         int param_dtype, void* stream) {
  MW_TRY(norm_sizes(rows, C, groups, eps));
  if (!dtype_ok(x_dtype) || !(dtype_ok(y_dtype) || y_dtype == MW_E4M3) || !dtype_ok(param_dtype))
    return fail(MW_ERR_INVALID_ARG, "types must be MW_BF16 or MW_F32, y's or MW_E4M3");
  if (x_dtype == MW_BF16 && y_dtype == MW_F32)
    return fail(MW_ERR_UNSUPPORTED, "y in fp32 needs x in fp32");
  const bool codes = y_dtype == MW_E4M3;
  if (codes) MW_TRY(check_width(C, "C"));
  if (rows == 0) return ok();
  MW_TRY(check_elems(x, x_dtype, "x"));
  if (residual) {
    MW_TRY(check_elems(residual, x_dtype, "residual"));
    MW_TRY(check_elems(h, x_dtype, "h"));
  }
  if (weight) MW_TRY(check_elems(weight, param_dtype, "weight"));
  if (codes) {
    for (const void* p : {x, residual, weight, const_cast<const void*>(y), const_cast<const void*>(h)})
      if (!aligned16(p))
        return fail(MW_ERR_INVALID_ARG, "y in 8 bits needs x, residual, weight, y and h 16-byte aligned");
    if (y == nullptr || y_scale == nullptr) return fail(MW_ERR_INVALID_ARG, "y or y_scale is NULL");
  } else {
    MW_TRY(check_elems(y, y_dtype, "y"));
  }
  MW_TRY(check_f32(rstd, "rstd"));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  RmsParams p{};
  p.x = x;
  p.residual = residual;
  p.weight = weight;
  p.y = y;
  p.y_scale = static_cast<uint8_t*>(y_scale);
  p.h = residual ? h : nullptr;
  p.rstd = rstd;
  p.rows = rows;
  p.rows_per_group = rows / groups;
  p.C = C;
  p.groups = groups;
  p.eps = eps;
  p.x_f32 = x_dtype == MW_F32;
  p.y_type = codes ? kRmsCodes : y_dtype == MW_F32 ? kRmsF32 : kRmsBf16;
  p.param_f32 = param_dtype == MW_F32;
  return launch_status(launch_rms_fwd(p, vector_rows(C, x, residual, weight, y, p.h), scope.device(), sm_count(), s),
                       "RMS norm forward launch");
}

size_t mw_rmsnorm_bwd_workspace_size(long long rows, int C, int groups) {
  if (norm_sizes(rows, C, groups, 0.f) != MW_OK || rows == 0) return 0;
  const int parts = rms_parts(rows / groups, C, groups);
  return parts > 1 ? align256(static_cast<size_t>(groups) * parts * C * sizeof(float)) : 0;
}

mw_status mw_rmsnorm_bwd(const void* dy, const void* h, const float* rstd, const void* weight, const void* dh,
                         void* dx, void* dweight, void* workspace, size_t ws_bytes, long long rows, int C, int groups,
                         int x_dtype, int y_dtype, int param_dtype, void* stream) {
  MW_TRY(norm_sizes(rows, C, groups, 0.f));
  if (!dtype_ok(x_dtype) || !dtype_ok(y_dtype) || !dtype_ok(param_dtype))
    return fail(MW_ERR_INVALID_ARG, "types must be MW_BF16 or MW_F32");
  if (x_dtype == MW_BF16 && y_dtype == MW_F32)
    return fail(MW_ERR_UNSUPPORTED, "y in fp32 needs x in fp32");
  if (weight) MW_TRY(check_elems(weight, param_dtype, "weight"));
  if (dweight) MW_TRY(check_elems(dweight, param_dtype, "dweight"));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    DeviceScope scope(s);
    MW_TRY(scope.status());
    const size_t bytes = static_cast<size_t>(groups) * C * (param_dtype == MW_F32 ? 4 : 2);
    if (dweight) MW_TRY(launch_status(cudaMemsetAsync(dweight, 0, bytes, s), "clearing a gradient"));
    return ok();
  }
  MW_TRY(check_elems(dy, y_dtype, "dy"));
  MW_TRY(check_elems(h, x_dtype, "h"));
  MW_TRY(check_elems(dx, x_dtype, "dx"));
  MW_TRY(check_elems(rstd, MW_F32, "rstd"));
  if (dh) MW_TRY(check_elems(dh, x_dtype, "dh"));
  const size_t need = dweight ? mw_rmsnorm_bwd_workspace_size(rows, C, groups) : 0;
  if (need > 0) {
    if (workspace == nullptr || ws_bytes < need)
      return fail(MW_ERR_WORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u)
      return fail(MW_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  }
  DeviceScope scope(s);
  MW_TRY(scope.status());
  RmsParams p{};
  p.dy = dy;
  p.h = const_cast<void*>(h);
  p.rstd = const_cast<float*>(rstd);
  p.weight = weight;
  p.dh = dh;
  p.dx = dx;
  p.dweight = dweight;
  p.partial = static_cast<float*>(workspace);
  p.rows = rows;
  p.rows_per_group = rows / groups;
  p.C = C;
  p.groups = groups;
  p.parts = rms_parts(rows / groups, C, groups);
  p.x_f32 = x_dtype == MW_F32;
  p.y_type = y_dtype == MW_F32 ? kRmsF32 : kRmsBf16;
  p.param_f32 = param_dtype == MW_F32;
  return launch_status(launch_rms_bwd(p, vector_rows(C, dy, h, weight, dh, dx), scope.device(), s),
                       "RMS norm backward launch");
}

mw_status mw_quantize(const void* x, void* q, void* scale, void* q_columns, void* scale_columns, long long rows,
                      int C, int form, int x_dtype, void* stream) {
  if (form < MW_FP8_ROWS || form > MW_FP8_ROWS_AND_COLUMNS)
    return fail(MW_ERR_INVALID_ARG, "form=%d is none of MW_FP8_ROWS ... MW_FP8_ROWS_AND_COLUMNS", form);
  MW_TRY(check_type(x_dtype, "x_dtype"));
  if (rows < 0 || rows > INT_MAX) return fail(MW_ERR_INVALID_ARG, "rows=%lld out of range [0, 2^31)", rows);
  MW_TRY(check_size(C, "C"));
  MW_TRY(check_width(C, "C"));
  const long long blocks = (rows + 127) / 128 * ceil_div(C, 128);
  if (blocks > INT_MAX) return fail(MW_ERR_INVALID_ARG, "rows=%lld x C=%d exceeds 2^31 blocks", rows, C);
  if (blocks == 0) return ok();
  MW_TRY(check_ptr(x, "x"));
  const bool columns = form == MW_FP8_COLUMNS || form == MW_FP8_ROWS_AND_COLUMNS;
  if (form != MW_FP8_COLUMNS) {
    MW_TRY(check_ptr(q, "q"));
    if (scale == nullptr) return fail(MW_ERR_INVALID_ARG, "scale is NULL");
  }
  if (columns) {
    MW_TRY(check_ptr(q_columns, "q_columns"));
    MW_TRY(check_ptr(scale_columns, "scale_columns"));
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  Fp8FormParams p{};
  p.x = x;
  p.q = static_cast<uint8_t*>(q);
  p.scale = static_cast<uint8_t*>(scale);
  p.q_columns = static_cast<uint8_t*>(q_columns);
  p.scale_columns = static_cast<uint8_t*>(scale_columns);
  p.rows = rows;
  p.C = C;
  p.x_f32 = x_dtype == MW_F32;
  return launch_status(launch_fp8_form(p, static_cast<Fp8Form>(form), s), "8-bit form launch");
}

mw_status mw_scaled_matmul(const void* a, const void* a_scale, int a_tiles, int a_transposed, const void* b,
                           const void* b_scale, int b_tiles, int b_transposed, void* c, int M, int N, int K,
                           int c_dtype, void* stream) {
  MW_TRY(check_size(M, "M"));
  MW_TRY(check_size(N, "N"));
  MW_TRY(check_size(K, "K"));
  MW_TRY(check_type(c_dtype, "c_dtype"));
  MW_TRY(check_width(a_transposed ? M : K, a_transposed ? "M" : "K"));
  MW_TRY(check_width(b_transposed ? N : K, b_transposed ? "N" : "K"));
  const long long tiles = static_cast<long long>(ceil_div(M, 128)) * ceil_div(N, 128);
  if (tiles > (1 << 27)) return fail(MW_ERR_INVALID_ARG, "M=%d x N=%d exceeds 2^27 tiles of 128 x 128", M, N);
  if (M == 0 || N == 0) return ok();
  const bool f32 = c_dtype == MW_F32;
  if (c == nullptr) return fail(MW_ERR_INVALID_ARG, "c is NULL");
  if (reinterpret_cast<uintptr_t>(c) & (f32 ? 3u : 1u))
    return fail(MW_ERR_INVALID_ARG, "c is not aligned to its elements");
  if (K > 0) {
    MW_TRY(check_ptr(a, "a"));
    MW_TRY(check_ptr(b, "b"));
    if (a_scale == nullptr || b_scale == nullptr) return fail(MW_ERR_INVALID_ARG, "a_scale or b_scale is NULL");
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  MW_TRY(scope.status());
  const size_t elem = f32 ? 4 : 2;
  if (K == 0)
    return launch_status(cudaMemsetAsync(c, 0, static_cast<size_t>(M) * N * elem, s), "clearing c");
  Fp8MmParams p{};
  MW_TRY(status_ptr(scope.device(), &p.status));
  p.blocks = ceil_div(K, kFp8Block);
  MmPlan plan;
  MW_TRY(mm_plan(M, N, p.blocks, a_transposed, b_transposed, f32, sm_count(), scope.device(), &plan));
  auto scales = [&](const void* at, int rows, bool transposed, bool tile) {
    Fp8Scales z{};
    z.p = static_cast<const uint8_t*>(at);
    const long long n = tile ? ceil_div(rows, 128) : rows;
    z.row = transposed ? 1 : p.blocks;
    z.block = transposed ? n : 1;
    const bool words = (reinterpret_cast<uintptr_t>(at) & 3u) == 0;
    z.read = tile                                             ? Fp8Read::kTile
             : transposed && words                            ? Fp8Read::kQuads  // (rows: a multiple of 16)
             : !transposed && words && p.blocks % 4 == 0      ? Fp8Read::kWords
                                                              : Fp8Read::kBytes;
    return z;
  };
  Fp8Scales sa = scales(a_scale, M, a_transposed, a_tiles), sb = scales(b_scale, N, b_transposed, b_tiles);
  int rows_a = M, rows_b = N;
  bool ta_cols = a_transposed, tb_cols = b_transposed;
  p.ld = N;
  if (plan.swap) {
    std::swap(a, b);
    std::swap(sa, sb);
    std::swap(rows_a, rows_b);
    std::swap(ta_cols, tb_cols);
  }
  p.a_scales = sa;
  p.b_scales = sb;
  p.rows_a = rows_a;
  p.rows_b = rows_b;
  p.a_columns = ta_cols;
  p.b_columns = tb_cols;
  p.swap = plan.swap;
  p.splits = plan.splits;
  p.tiles_p = ceil_div(rows_a, plan.join ? 128 : 256);
  p.tiles_q = ceil_div(rows_b, plan.bn);
  p.ctas = sm_count();
  // (whole words of scales)
  const int limit = f32 ? kFp8Chunk : kFp8ChunkBf16;
  p.chunk = plan.join         ? limit
            : plan.splits > 1 ? pair_share(p.blocks, plan.splits)
                              : pair_share(p.blocks, ceil_div(p.blocks, limit));
  p.out = c;
  p.out_f32 = f32;
  p.out_quads = N % 4 == 0 && (reinterpret_cast<uintptr_t>(c) & (4 * elem - 1)) == 0;
  p.tma_out = !plan.join && plan.splits == 1 && aligned16(c) && N * elem % 16 == 0;
  p.budget_ns = budget_ns();
  p.debug_skip_q = debug_skip_q();
  CUtensorMap ma, mb, mc;
  auto operand = [&](CUtensorMap* m, const void* at, int rows, bool columns, int box, const char* name) {
    return columns ? make_map_2d(m, at, K, rows, 1, kFp8Block, name) : make_map_2d(m, at, rows, K, 1, box, name);
  };
  MW_TRY(operand(&ma, a, rows_a, p.a_columns, 128, "a"));
  MW_TRY(operand(&mb, b, rows_b, p.b_columns, plan.join ? plan.bn : plan.bn / 2, "b"));
  mc = ma;
  if (p.tma_out) MW_TRY(make_map_2d(&mc, c, M, N, static_cast<int>(elem), 32, "c", 64));
  return launch_status(launch_fp8_mm(plan.bn, plan.join, ma, mb, mc, p, scope.device(), s), "8-bit product launch");
}

}  // extern "C"
