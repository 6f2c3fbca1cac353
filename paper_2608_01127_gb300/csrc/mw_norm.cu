// Layer norm over the channels of a row, forward and backward, with one weight
// and bias for every group of rows (one group: the usual layer norm; a group a
// sample or a frame: the adaptive modulation of Sec. 4.1's blocks).
//
//   mean = sum x / C, rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),
//   xh = (x - mean) rstd, y = xh w_g + b_g
//   g = dy w_g, dx = rstd (g - sum g / C - xh sum(g xh) / C),
//   dw_g = sum of dy xh over the group's rows, db_g = sum of dy
//
// Bound by HBM: a row is read once (the variance is the second pass over registers, in
// fp32 as all sums).  W warps share a row.  VEC = 8 where rows start at multiples of 16
// bytes, else 1 (any width, any alignment).  Forward: a thread holds at most V accesses of
// VEC elements of a row, or of two, in registers.  Backward: a block takes a range of
// one group's rows, its threads keep the sums of their columns in registers over all of
// them, and leave one partial [2, C] a block; a second kernel adds the blocks' partials of
// a group in their order, so that results do not depend on timing.
// Measured from HBM, forward / backward with the parameter sums, us (GB/s): 14080 x 2560
// bf16 38 (3800) / 44 (4960), 28160 x 768 19 (4580) / 30 (4300), 40000 x 1024 34 (4820) /
// 45 (5440), 8000 x 8192 67 (3890) / 68 (5770); 14080 x 1152 fp32 22 (4420) / 44 (3660),
// 5003 x 1155 fp32 20 / 31 (single elements).
#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

using bf16 = __nv_bfloat16;

// VEC elements as they lie in memory, so that a row on its way takes few registers.
template <class T, int VEC>
struct Raw;
template <>
struct Raw<float, 8> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};
template <>
struct Raw<bf16, 8> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
};
template <class T>
struct Raw<T, 1> {
  T a;
  __device__ __forceinline__ void load(const T* p) { a = *p; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = static_cast<float>(a); }
};

template <int VEC>
__device__ __forceinline__ void store(float* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *p = v[0];
  }
}
template <int VEC>
__device__ __forceinline__ void store(bf16* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  else
    *p = __float2bfloat16(v[0]);
}
// a weight, bias or a gradient of one: fp32 or bf16
template <int VEC>
__device__ __forceinline__ void load_param(const void* base, bool f32, size_t i, float (&v)[VEC]) {
  if (f32) {
    Raw<float, VEC> r;
    r.load(static_cast<const float*>(base) + i);
    r.get(v);
  } else {
    Raw<bf16, VEC> r;
    r.load(static_cast<const bf16*>(base) + i);
    r.get(v);
  }
}
__device__ __forceinline__ void store_param(void* base, bool f32, size_t i, float v) {
  if (f32)
    static_cast<float*>(base)[i] = v;
  else
    static_cast<bf16*>(base)[i] = __float2bfloat16(v);
}

// Sums that a team makes at once.
template <int N>
struct Sums {
  float v[N];
};

// A block's threads: teams of W warps, a row each.
struct Team {
  int W, index, count, t, warp;  // t: thread of the team
  __device__ explicit Team(int W_) : W(W_) {
    const int w = threadIdx.x >> 5;
    index = w / W;
    count = (blockDim.x >> 5) / W;
    warp = w % W;
    t = warp * 32 + (threadIdx.x & 31);
  }
  // Sums over the team in a fixed order; red: a value a warp of the block.  (A barrier
  // a call is enough where calls alternate between two buffers.)
  template <int N>
  __device__ __forceinline__ Sums<N> sum(Sums<N> v, Sums<N>* red) const {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v = plus(v, shuffled(v, s));
    if (W == 1) return v;
    if ((threadIdx.x & 31) == 0) red[index * W + warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(W * 32) : "memory");
    Sums<N> s = red[index * W];
    for (int w = 1; w < W; ++w) s = plus(s, red[index * W + w]);
    return s;
  }

 private:
  template <int N>
  static __device__ __forceinline__ Sums<N> plus(Sums<N> a, const Sums<N>& b) {
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] += b.v[i];
    return a;
  }
  template <int N>
  static __device__ __forceinline__ Sums<N> shuffled(Sums<N> a, int s) {
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = __shfl_xor_sync(0xffffffffu, a.v[i], s);
    return a;
  }
};

// Threads of a block at most, and the blocks of 256 threads that an SM holds for the
// registers that a thread's columns take (x: bytes of an element of x).
constexpr int max_threads(int VEC, int V) { return VEC == 1 && V > 8 ? 512 : 256; }
constexpr int fwd_blocks(int VEC, int V, int x) {
  return VEC == 1 ? (V <= 4 ? 5 : V <= 8 ? 3 : 1) : V <= 2 ? 4 : V <= 4 ? 3 : V <= 6 && x == 2 ? 3 : 2;
}
constexpr int bwd_blocks(int V) { return V <= 4 ? 3 : V <= 8 ? 2 : 1; }

// Rows that a team of the forward works on at once: their loads, sums and barriers
// overlap, and they share what a group's weight and bias cost (read from L1 for every
// turn: in registers they would take the room of rows).  14080 rows of 2560 bf16: one
// row with the next on its way, five warps a row 59 us; one warp, one row 43; two 39.
template <class TX, int VEC, int V>
constexpr int kRows = VEC == 8 && V >= 3 && sizeof(TX) == 2 ? 2 : 1;

// Each team takes a run of rows.  A warp alone holds rows of up to 2560 elements: no
// barrier, and many rows on their way at once.
template <class TX, class TY, int VEC, int V>
__global__ void __launch_bounds__(max_threads(VEC, V), fwd_blocks(VEC, V, sizeof(TX)))
    norm_fwd_kernel(const NormParams p) {
  constexpr int R = kRows<TX, VEC, V>;
  __shared__ Sums<R> red[2][16];
  const Team team(p.W);
  const TX* x = static_cast<const TX*>(p.x);
  TY* y = static_cast<TY*>(p.y);
  const float inv_c = 1.f / static_cast<float>(p.C);
  const long long teams = static_cast<long long>(gridDim.x) * team.count;
  const long long mine = static_cast<long long>(blockIdx.x) * team.count + team.index;
  const long long r0 = p.rows * mine / teams, r1 = p.rows * (mine + 1) / teams;
  auto column = [&](int k) { return (k * team.W * 32 + team.t) * VEC; };
  long long left = 0;  // rows of the group from this one on
  size_t params = 0;   // where the group's weight and bias start
  if (p.groups > 1 && r0 < r1) {
    const long long group = r0 / p.rows_per_group;
    left = (group + 1) * p.rows_per_group - r0;
    params = static_cast<size_t>(group) * p.C;
  }
  pdl_wait();
  pdl_trigger();
  auto fetch = [&](long long row, int n, Raw<TX, VEC> (&to)[R][V]) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (r < n && column(k) < p.C) to[r][k].load(x + (row + r) * p.C + column(k));
  };
  auto load_params = [&](int k, float (&w)[VEC], float (&b)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = 1.f, b[e] = 0.f;
    if (column(k) >= p.C) return;
    if (p.weight) load_param<VEC>(p.weight, p.param_f32, params + column(k), w);
    if (p.bias) load_param<VEC>(p.bias, p.param_f32, params + column(k), b);
  };
  // (single elements: 5003 rows of 1155 fp32 33 us with weights read for every row)
  constexpr int kHeld = VEC == 1 ? V : 1;
  [[maybe_unused]] float hw[kHeld][VEC], hb[kHeld][VEC];
  auto hold_params = [&]() {
    if constexpr (VEC == 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) load_params(k, hw[k], hb[k]);
    }
  };
  hold_params();
  Raw<TX, VEC> raw[R][V];
  [[maybe_unused]] Raw<TX, VEC> next[R][V];  // a row at a time: the next one on its way
  if (R == 1 && r0 < r1) fetch(r0, 1, raw);
  for (long long row = r0; row < r1;) {
    // rows of one group
    int n = static_cast<int>(min(static_cast<long long>(R), r1 - row));
    if (p.groups > 1) n = static_cast<int>(min(static_cast<long long>(n), left));
    if constexpr (R == 1) {
      if (row + 1 < r1) fetch(row + 1, 1, next);
    } else {
      fetch(row, n, raw);
    }
    Sums<R> mean, rstd;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean.v[r] = 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (r >= n || column(k) >= p.C) continue;
        float v[VEC];
        raw[r][k].get(v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) mean.v[r] += v[e];
      }
    }
    mean = team.sum(mean, red[0]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean.v[r] *= inv_c;
      rstd.v[r] = 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (r >= n || column(k) >= p.C) continue;
        float v[VEC];
        raw[r][k].get(v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) rstd.v[r] = fmaf(v[e] - mean.v[r], v[e] - mean.v[r], rstd.v[r]);
      }
    }
    rstd = team.sum(rstd, red[1]);
#pragma unroll
    for (int r = 0; r < R; ++r) rstd.v[r] = rsqrtf(rstd.v[r] * inv_c + p.eps);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (column(k) >= p.C) continue;
      float w[VEC], b[VEC];
      if constexpr (VEC == 1)
        w[0] = hw[k][0], b[0] = hb[k][0];
      else
        load_params(k, w, b);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= n) continue;
        float v[VEC];
        raw[r][k].get(v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - mean.v[r]) * rstd.v[r], w[e], b[e]);
        store<VEC>(y + (row + r) * p.C + column(k), v);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < n && team.t == 0) {
        if (p.mean) p.mean[row + r] = mean.v[r];
        if (p.rstd) p.rstd[row + r] = rstd.v[r];
      }
    if constexpr (R == 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) raw[0][k] = next[0][k];
    }
    row += n;
    left -= n;
    if (p.groups > 1 && left == 0) {
      left = p.rows_per_group;
      params += p.C;
      if (row < r1) hold_params();
    }
  }
}

// A block's sums of dw and db over its rows: its partial, or the result.
__device__ __forceinline__ void write_params(const NormParams& p, size_t g, const float* sums) {
  for (int c = threadIdx.x; c < 2 * p.C; c += blockDim.x) {
    if (p.parts > 1)
      p.partial[static_cast<size_t>(blockIdx.x) * 2 * p.C + c] = sums[c];
    else if (c < p.C ? p.dweight != nullptr : p.dbias != nullptr)
      store_param(c < p.C ? p.dweight : p.dbias, p.param_f32, g + (c < p.C ? c : c - p.C), sums[c]);
  }
}

// Block (part, group): rows [part n / parts, (part + 1) n / parts) of the group.
template <class TX, class TY, int V>
__global__ void __launch_bounds__(max_threads(1, V), bwd_blocks(V)) norm_bwd_kernel(const NormParams p) {
  constexpr int VEC = 1;
  __shared__ Sums<2> red[2][16];
  extern __shared__ float sums[];  // [2][C]
  const Team team(p.W);
  const TX* x = static_cast<const TX*>(p.x);
  const TY* dy = static_cast<const TY*>(p.dy);
  TX* dx = static_cast<TX*>(p.dx);
  const float inv_c = 1.f / static_cast<float>(p.C);
  const int part = blockIdx.x % p.parts;
  const long long group = blockIdx.x / p.parts;
  const long long n = p.rows_per_group;
  const long long r0 = group * n + part * n / p.parts, r1 = group * n + (part + 1) * n / p.parts;
  const size_t g = static_cast<size_t>(group) * p.C;
  auto column = [&](int k) { return (k * team.W * 32 + team.t) * VEC; };
  pdl_wait();
  pdl_trigger();
  Raw<TX, VEC> rx[V];
  Raw<TY, VEC> rg[V];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](long long row) {
    mean = p.mean[row];
    rstd = p.rstd[row];
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (column(k) < p.C) {
        rx[k].load(x + row * p.C + column(k));
        rg[k].load(dy + row * p.C + column(k));
      }
  };
  if (r0 + team.index < r1) fetch(r0 + team.index);
  float w[V][VEC], aw[V][VEC], ab[V][VEC];
#pragma unroll
  for (int k = 0; k < V; ++k) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) aw[k][e] = ab[k][e] = 0.f, w[k][e] = 1.f;
    if (p.weight && column(k) < p.C) load_param<VEC>(p.weight, p.param_f32, g + column(k), w[k]);
  }
  int turn = 0;
  for (long long row = r0 + team.index; row < r1; row += team.count, turn ^= 1) {
    float xh[V][VEC], gr[V][VEC];
    Sums<2> s = {{0.f, 0.f}};
    const float rs = rstd;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (column(k) >= p.C) continue;
      rx[k].get(xh[k]);
      rg[k].get(gr[k]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xh[k][e] = (xh[k][e] - mean) * rs;
        aw[k][e] = fmaf(gr[k][e], xh[k][e], aw[k][e]);
        ab[k][e] += gr[k][e];
        gr[k][e] *= w[k][e];
        s.v[0] += gr[k][e];
        s.v[1] = fmaf(gr[k][e], xh[k][e], s.v[1]);
      }
    }
    if (row + team.count < r1) fetch(row + team.count);
    s = team.sum(s, red[turn]);
    const float m1 = s.v[0] * inv_c, m2 = s.v[1] * inv_c;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (column(k) >= p.C) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) gr[k][e] = rs * (gr[k][e] - m1 - xh[k][e] * m2);
      store<VEC>(dx + row * p.C + column(k), gr[k]);
    }
  }
  if (!p.dweight && !p.dbias) return;
  for (int t = 0; t < team.count; ++t) {
    if (team.index == t) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = column(k);
        if (c >= p.C) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sums[c + e] = t == 0 ? aw[k][e] : sums[c + e] + aw[k][e];
          sums[p.C + c + e] = t == 0 ? ab[k][e] : sums[p.C + c + e] + ab[k][e];
        }
      }
    }
    __syncthreads();
  }
  write_params(p, g, sums);
}

// N sums over a warp at once, N = 2, 4 or 8: halves of the values change sides until one is
// left, so 9 shuffles do for 8; lane l ends with value l / (32 / N).
template <int N>
__device__ __forceinline__ float warp_sums(float (&v)[N]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = N / 2, m = 16; m > 0; h /= 2, m /= 2) {
    if (h > 0) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i >= h) continue;
        const bool up = lane & m;
        const float mine = up ? v[i + h] : v[i], other = up ? v[i] : v[i + h];
        v[i] = mine + __shfl_xor_sync(0xffffffffu, other, m);
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
    }
  }
  return v[0];
}

// The same with rows in 16-byte pieces.  A team takes kBatch rows at a time, and every
// thread copies its own columns of the next ones to shared memory meanwhile (no barrier:
// nobody else reads them): the copies keep HBM busy while a batch waits for its sums, of
// which there is one barrier a batch, and the registers hold sums alone.
constexpr int kBatch = 4;
template <class TX, class TY>
constexpr int kPieces = (sizeof(TX) + sizeof(TY)) / 2;  // of x and dy, a thread's 8 columns
template <class TX, class TY, int V>
constexpr int kRowsOf = kBatch / V / (kPieces<TX, TY> > 2 ? 2 : 1);

template <class TX, class TY, int V>
__global__ void __maxnreg__(V == 1 ? 80 : 128) norm_bwd_rows_kernel(const NormParams p) {
  constexpr int R = kRowsOf<TX, TY, V>, N = 2 * R;
  constexpr int PX = sizeof(TX) / 2, PY = sizeof(TY) / 2;  // pieces of x and dy
  __shared__ float red[2][16][N];
  extern __shared__ __align__(16) uint8_t ring[];  // [2][R][V][PX + PY][threads] pieces; then [2][C] sums
  const Team team(p.W);
  const TX* x = static_cast<const TX*>(p.x);
  const TY* dy = static_cast<const TY*>(p.dy);
  TX* dx = static_cast<TX*>(p.dx);
  const int lane = threadIdx.x & 31;
  const float inv_c = 1.f / static_cast<float>(p.C);
  const int part = blockIdx.x % p.parts;
  const long long group = blockIdx.x / p.parts;
  const long long n = p.rows_per_group;
  const long long r0 = group * n + part * n / p.parts, r1 = group * n + (part + 1) * n / p.parts;
  const size_t g = static_cast<size_t>(group) * p.C;
  auto column = [&](int k) { return (k * team.W * 32 + team.t) * 8; };
  const uint32_t mine = smem_u32(ring) + 16 * threadIdx.x;
  const uint32_t piece = 16 * blockDim.x;
  auto at = [&](int stage, int r, int k, int i) {
    return mine + piece * (((stage * R + r) * V + k) * (PX + PY) + i);
  };
  pdl_wait();
  pdl_trigger();
  float mean[R], rstd[R], next_mean[R], next_rstd[R];
  auto fetch = [&](long long row, int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= r1) continue;
      next_mean[r] = p.mean[row + r];
      next_rstd[r] = p.rstd[row + r];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        const size_t from = static_cast<size_t>(row + r) * p.C + column(k);
#pragma unroll
        for (int i = 0; i < PX; ++i) copy_16b(at(stage, r, k, i), reinterpret_cast<const uint4*>(x + from) + i);
#pragma unroll
        for (int i = 0; i < PY; ++i) copy_16b(at(stage, r, k, PX + i), reinterpret_cast<const uint4*>(dy + from) + i);
      }
    }
  };
  long long row = r0 + static_cast<long long>(team.index) * R;
  const long long step = static_cast<long long>(team.count) * R;
#pragma unroll
  for (int r = 0; r < R; ++r) next_mean[r] = next_rstd[r] = 0.f;
  fetch(row, 0);
  copy_commit();
  // (pairs of columns: an instruction does two)
  float2 w[V][4], aw[V][4], ab[V][4];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float one[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (p.weight && column(k) < p.C) load_param<8>(p.weight, p.param_f32, g + column(k), one);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      aw[k][e] = ab[k][e] = make_float2(0.f, 0.f);
      w[k][e] = make_float2(one[2 * e], one[2 * e + 1]);
    }
  }
  // x and dy of a row's columns, as fp32
  auto read = [&](int stage, int r, int k, float2 (&vx)[4], float2 (&vy)[4]) {
    Raw<TX, 8> rx;
    Raw<TY, 8> ry;
#pragma unroll
    for (int i = 0; i < PX; ++i) reinterpret_cast<uint4*>(&rx)[i] = shared_16b(at(stage, r, k, i));
#pragma unroll
    for (int i = 0; i < PY; ++i) reinterpret_cast<uint4*>(&ry)[i] = shared_16b(at(stage, r, k, PX + i));
    float fx[8], fy[8];
    rx.get(fx);
    ry.get(fy);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      vx[e] = make_float2(fx[2 * e], fx[2 * e + 1]);
      vy[e] = make_float2(fy[2 * e], fy[2 * e + 1]);
    }
  };
  auto both = [](float v) { return make_float2(v, v); };
  for (int turn = 0; row < r1; row += step, turn ^= 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = next_mean[r], rstd[r] = next_rstd[r];
    fetch(row + step, turn ^ 1);
    copy_commit();
    copy_wait<1>();
    float s[N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[2 * r] = s[2 * r + 1] = 0.f;
      if (row + r >= r1) continue;
      float2 s1 = make_float2(0.f, 0.f), s2 = s1;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        float2 xh[4], gr[4];
        read(turn, r, k, xh, gr);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xh[e] = mul2(add2(xh[e], both(-mean[r])), both(rstd[r]));
          aw[k][e] = fma2(gr[e], xh[e], aw[k][e]);
          ab[k][e] = add2(ab[k][e], gr[e]);
          gr[e] = mul2(gr[e], w[k][e]);
          s1 = add2(s1, gr[e]);
          s2 = fma2(gr[e], xh[e], s2);
        }
      }
      s[2 * r] = s1.x + s1.y;
      s[2 * r + 1] = s2.x + s2.y;
    }
    float sum = warp_sums<N>(s);
    constexpr int kShare = 32 / N;  // lanes of a value
    int from = kShare;
    if (p.W > 1) {
      if (lane % kShare == 0) red[turn][team.index * p.W + team.warp][lane / kShare] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(team.index + 1), "r"(p.W * 32) : "memory");
      sum = 0.f;
      for (int i = lane / N; i < p.W; i += kShare) sum += red[turn][team.index * p.W + i][lane % N];
#pragma unroll
      for (int m = N; m < 32; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
      from = 1;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = __shfl_sync(0xffffffffu, sum, i * from) * inv_c;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= r1) continue;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        float2 xh[4], gr[4];
        read(turn, r, k, xh, gr);
        const float2 slope = both(-rstd[r] * s[2 * r + 1]);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = fma2(add2(xh[e], both(-mean[r])), slope, fma2(gr[e], w[k][e], both(-s[2 * r])));
          const float2 u = mul2(t, both(rstd[r]));
          v[2 * e] = u.x;
          v[2 * e + 1] = u.y;
        }
        store<8>(dx + static_cast<size_t>(row + r) * p.C + column(k), v);
      }
    }
  }
  if (!p.dweight && !p.dbias) return;
  copy_wait<0>();
  __syncthreads();  // the ring is read
  float* sums = reinterpret_cast<float*>(ring);
  for (int t = 0; t < team.count; ++t) {
    if (team.index == t) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = column(k);
        if (c >= p.C) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float2* to = reinterpret_cast<float2*>(sums + c) + e;
          *to = t == 0 ? aw[k][e] : add2(*to, aw[k][e]);
          to = reinterpret_cast<float2*>(sums + p.C + c) + e;
          *to = t == 0 ? ab[k][e] : add2(*to, ab[k][e]);
        }
      }
    }
    __syncthreads();
  }
  write_params(p, g, sums);
}

// dw and db of a group from its blocks' partials: `split` threads a column, each an
// equal share of the parts in their order.
__global__ void __launch_bounds__(256) norm_params_kernel(const NormParams p, int split) {
  __shared__ float sums[256];
  const int columns = 256 / split;
  const int lane = threadIdx.x / columns, at = threadIdx.x % columns;
  const int c = blockIdx.x * columns + at;
  pdl_wait();
  pdl_trigger();
  for (int g = blockIdx.y; g < p.groups; g += gridDim.y) {
    float s = 0.f;
    if (c < 2 * p.C) {
      const float* in = p.partial + static_cast<size_t>(g) * p.parts * 2 * p.C + c;
      const int i1 = p.parts * (lane + 1) / split;
#pragma unroll 8
      for (int i = p.parts * lane / split; i < i1; ++i) s += in[static_cast<size_t>(i) * 2 * p.C];
    }
    if (split > 1) {
      sums[threadIdx.x] = s;
      __syncthreads();
      for (int k = 1; lane == 0 && k < split; ++k) s += sums[k * columns + at];
    }
    if (lane == 0 && c < 2 * p.C) {
      void* out = c < p.C ? p.dweight : p.dbias;
      if (out) store_param(out, p.param_f32, static_cast<size_t>(g) * p.C + (c < p.C ? c : c - p.C), s);
    }
    __syncthreads();
  }
}

// The row kernel's shape: 8 or 16 columns a thread, W warps a row, teams up to 256 threads;
// blocks of an SM up to 768 threads (their registers, and 256 bytes of the ring each).
struct RowsShape {
  int W, V, threads, blocks;
};
RowsShape rows_shape(int C) {
  RowsShape s{};
  s.V = C <= 4096 ? 1 : 2;
  s.W = (C + 256 * s.V - 1) / (256 * s.V);
  s.threads = 32 * s.W * (s.W < 8 ? 8 / s.W : 1);
  s.blocks = 768 / (s.threads * s.V) < 1 ? 1 : 768 / (s.threads * s.V);
  return s;
}

// Warps a row and accesses a thread of the other kernels.  VEC = 8 (forward): the fewest
// warps that hold the row in ten accesses.  VEC = 1: the fewest slots with 8 accesses, 16
// of the widest rows.
struct Shape {
  int W, V, threads;
};
int form(int V, bool vec) {  // the least V that is compiled
  if (!vec) return V <= 2 ? 2 : V <= 4 ? 4 : V <= 8 ? 8 : V <= 16 ? 16 : 99;
  return V <= 4 ? V : V <= 6 ? 6 : V <= 10 ? 10 : 99;
}
// Few rows (forward): all SMs' warps for them, a thread's part of a row as short as can be.
Shape shape_of(int C, bool vec, bool few) {
  const int elems = vec ? 256 : 32;
  const int max_v = vec ? (!few ? 10 : C <= 4096 ? 2 : 4) : (C <= 2048 ? 8 : 16);
  const int max_w = vec || C <= 2048 ? 8 : 16;
  Shape best{0, 0, 0};
  for (int W = 1; W <= max_w; ++W) {
    const int V = form((C + elems * W - 1) / (elems * W), vec);
    if (V > max_v || 32 * W > max_threads(vec ? 8 : 1, V)) continue;
    if (best.W == 0 || (W * V < best.W * best.V && (few || !vec))) best = {W, V, 0};
  }
  best.threads = 32 * best.W * (best.W < 8 ? 8 / best.W : 1);
  return best;
}

template <class X, class Y, int VEC, int V>
struct Kernels {
  static constexpr auto fwd() { return norm_fwd_kernel<X, Y, VEC, V>; }
  static constexpr int blocks = fwd_blocks(VEC, V, sizeof(X));
};

// f of the kernels for these types and accesses a thread.
template <class F>
cudaError_t by_shape(const NormParams& p, bool vec, int V, F&& f) {
  auto types = [&](auto tx, auto ty) {
    using X = decltype(tx);
    using Y = decltype(ty);
    if (vec) {
      if (V == 1) return f(Kernels<X, Y, 8, 1>{});
      if (V == 2) return f(Kernels<X, Y, 8, 2>{});
      if (V == 3) return f(Kernels<X, Y, 8, 3>{});
      if (V == 6) return f(Kernels<X, Y, 8, 6>{});
      if (V == 10) return f(Kernels<X, Y, 8, 10>{});
      return f(Kernels<X, Y, 8, 4>{});
    }
    if (V == 2) return f(Kernels<X, Y, 1, 2>{});
    if (V == 4) return f(Kernels<X, Y, 1, 4>{});
    if (V == 8) return f(Kernels<X, Y, 1, 8>{});
    return f(Kernels<X, Y, 1, 16>{});
  };
  if (!p.x_f32) return types(bf16{}, bf16{});
  if (!p.y_f32) return types(float{}, bf16{});
  return types(float{}, float{});
}

// The backward's shared memory: the rows' ring, or the sums of the widest row.
constexpr int kNormMaxSmem = 512 * 256;
static_assert(kNormMaxSmem >= 2 * kNormMaxC * static_cast<int>(sizeof(float)), "the sums fit");

template <auto kKernel>
cudaError_t run_bwd(const NormParams& p, unsigned blocks, int threads, size_t smem, int dev, cudaStream_t s) {
  static OncePerDevice prepared;
  const cudaError_t e = prepared(
      dev, [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormMaxSmem); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(blocks), dim3(threads), smem, s);
  return cudaLaunchKernelEx(&cfg, kKernel, p);
}

}  // namespace

int norm_parts(long long rows_per_group, int C, int groups) {
  // as many blocks as the SMs hold, by the form that aligned rows take
  long long parts;
  if (C % 8 == 0) {
    parts = static_cast<long long>(kNormSms) * rows_shape(C).blocks / groups;
  } else {
    const Shape sh = shape_of(C, false, false);
    parts = static_cast<long long>(kNormSms) * bwd_blocks(sh.V) * max_threads(1, sh.V) / sh.threads / groups;
  }
  if (parts > rows_per_group) parts = rows_per_group;
  return parts < 1 ? 1 : static_cast<int>(parts);
}

cudaError_t launch_norm_fwd(NormParams p, bool vec, int sms, cudaStream_t s) {
  const Shape sh = shape_of(p.C, vec, p.rows <= 8ll * sms);
  p.W = sh.W;
  const int teams = sh.threads / 32 / sh.W;
  const long long blocks = (p.rows + teams - 1) / teams;
  return by_shape(p, vec, sh.V, [&](auto k) {
    // as many blocks as the SMs hold (of fewer threads, more)
    const long long most = static_cast<long long>(sms) * decltype(k)::blocks * 256 / sh.threads;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr;
    pdl_config(cfg, attr, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), dim3(sh.threads), 0, s);
    return cudaLaunchKernelEx(&cfg, decltype(k)::fwd(), p);
  });
}

cudaError_t launch_norm_bwd(NormParams p, bool vec, int dev, cudaStream_t s) {
  const size_t sums = static_cast<size_t>(2) * p.C * sizeof(float);
  const unsigned blocks = static_cast<unsigned>(p.groups) * p.parts;
  cudaError_t e;
  auto types = [&](auto f) {
    if (!p.x_f32) return f(bf16{}, bf16{});
    if (!p.y_f32) return f(float{}, bf16{});
    return f(float{}, float{});
  };
  if (vec) {
    const RowsShape sh = rows_shape(p.C);
    p.W = sh.W;
    e = types([&](auto tx, auto ty) {
      using X = decltype(tx);
      using Y = decltype(ty);
      auto smem = [&](int rows) {
        const size_t ring = static_cast<size_t>(2) * rows * sh.V * kPieces<X, Y> * 16 * sh.threads;
        return ring > sums ? ring : sums;
      };
      return sh.V == 1
                 ? run_bwd<norm_bwd_rows_kernel<X, Y, 1>>(p, blocks, sh.threads, smem(kRowsOf<X, Y, 1>), dev, s)
                 : run_bwd<norm_bwd_rows_kernel<X, Y, 2>>(p, blocks, sh.threads, smem(kRowsOf<X, Y, 2>), dev, s);
    });
  } else {
    const Shape sh = shape_of(p.C, false, false);
    p.W = sh.W;
    e = types([&](auto tx, auto ty) {
      using X = decltype(tx);
      using Y = decltype(ty);
      if (sh.V == 2) return run_bwd<norm_bwd_kernel<X, Y, 2>>(p, blocks, sh.threads, sums, dev, s);
      if (sh.V == 4) return run_bwd<norm_bwd_kernel<X, Y, 4>>(p, blocks, sh.threads, sums, dev, s);
      if (sh.V == 8) return run_bwd<norm_bwd_kernel<X, Y, 8>>(p, blocks, sh.threads, sums, dev, s);
      return run_bwd<norm_bwd_kernel<X, Y, 16>>(p, blocks, sh.threads, sums, dev, s);
    });
  }
  if (e != cudaSuccess || p.parts == 1 || (!p.dweight && !p.dbias)) return e;
  int split = 1;
  while (split < 32 && p.parts >= 16 * split) split *= 2;
  const int columns = 256 / split;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3((2 * p.C + columns - 1) / columns, p.groups < 65535 ? p.groups : 65535), dim3(256), 0, s);
  return cudaLaunchKernelEx(&cfg, norm_params_kernel, p, split);
}

}  // namespace mw
