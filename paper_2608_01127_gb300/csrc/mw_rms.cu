// Root-mean-square norm over the channels of a row, with the residual's addition in front
// and an output in 8 bits for the product behind; its gradients.
//
//   h = x + r (rounded to x's type),  rstd = 1 / sqrt(sum h^2 / C + eps),  xh = h rstd,
//   y = xh w_g, in bf16 or fp32, or codes and a scale for every 128 of a row (mw_fp8.cuh)
//   g = dy w_g,  d = rstd (g - xh sum(g xh) / C) + dh,  dw_g = sum of dy xh over the group's rows
// d is the gradient of x and of r alike; dh comes down the residual stream.
//
// Bound by HBM: every array is read or written once, sums are fp32.  The kernels' shapes are
// the layer norm's (mw_norm.cu): W warps to a row, 16-byte accesses where rows allow them.
// 128 columns of a row lie in 16 lanes, whose maximum gives the scale without leaving the
// registers.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "mw_fp8.cuh"
#include "mw_internal.h"
#include "mw_ptx.cuh"
#include "mw_rows.cuh"

namespace mw {
namespace {

struct E4m3 {};  // codes, as a type of y

template <class TY, int VEC>
__device__ __forceinline__ void store_y(void* base, size_t at, const float (&v)[VEC]) {
  store<VEC>(static_cast<TY*>(base) + at, v);
}

// An element as it is stored.
__device__ __forceinline__ float rounded(float v, const float*) { return v; }
__device__ __forceinline__ float rounded(float v, const bf16*) { return __bfloat162float(__float2bfloat16(v)); }

constexpr int fwd_blocks(int VEC, int V, int x) {
  return VEC == 1 ? (V <= 4 ? 5 : V <= 8 ? 3 : 1) : V <= 2 ? 4 : x == 2 ? 3 : 2;
}

// Each team takes a run of rows, R at once where they are short in registers.
template <class TX, class TY, int VEC, int V, bool RES>
__global__ void __launch_bounds__(max_threads(VEC, V), fwd_blocks(VEC, V, sizeof(TX)))
    rms_fwd_kernel(const RmsParams p) {
  constexpr bool CODES = std::is_same_v<TY, E4m3>;
  constexpr int R = VEC == 8 && V >= 3 && sizeof(TX) == 2 && !RES && !CODES ? 2 : 1;
  __shared__ Sums<R> red[2][16];
  const Team team(p.W);
  const TX* x = static_cast<const TX*>(p.x);
  [[maybe_unused]] const TX* res = static_cast<const TX*>(p.residual);
  [[maybe_unused]] TX* hs = static_cast<TX*>(p.h);
  const float inv_c = 1.f / static_cast<float>(p.C);
  const long long teams = static_cast<long long>(gridDim.x) * team.count;
  const long long mine = static_cast<long long>(blockIdx.x) * team.count + team.index;
  const long long r0 = p.rows * mine / teams, r1 = p.rows * (mine + 1) / teams;
  auto column = [&](int k) { return (k * team.W * 32 + team.t) * VEC; };
  long long left = 0;  // rows of the group from this one on
  size_t params = 0;   // where the group's weight starts
  if (p.groups > 1 && r0 < r1) {
    const long long group = r0 / p.rows_per_group;
    left = (group + 1) * p.rows_per_group - r0;
    params = static_cast<size_t>(group) * p.C;
  }
  pdl_wait();
  pdl_trigger();
  int turn = 0;
  for (long long row = r0; row < r1; turn ^= 1) {
    // rows of one group
    int n = static_cast<int>(min(static_cast<long long>(R), r1 - row));
    if (p.groups > 1) n = static_cast<int>(min(static_cast<long long>(n), left));
    Raw<TX, VEC> raw[R][V];
    [[maybe_unused]] Raw<TX, VEC> add[RES ? V : 1];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (r < n && column(k) < p.C) {
          raw[r][k].load(x + (row + r) * p.C + column(k));
          if constexpr (RES) add[k].load(res + row * p.C + column(k));
        }
    Sums<R> rstd;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rstd.v[r] = 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (r >= n || column(k) >= p.C) continue;
        float v[VEC];
        raw[r][k].get(v);
        if constexpr (RES) {
          float a[VEC];
          add[k].get(a);
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[e] = rounded(v[e] + a[e], static_cast<const TX*>(nullptr));
          raw[r][k].put(v);
          store<VEC>(hs + row * p.C + column(k), v);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) rstd.v[r] = fmaf(v[e], v[e], rstd.v[r]);
      }
    }
    rstd = team.sum(rstd, red[turn]);
#pragma unroll
    for (int r = 0; r < R; ++r) rstd.v[r] = rsqrtf(rstd.v[r] * inv_c + p.eps);
    if constexpr (CODES) {
      // scale bytes of four of a thread's blocks to a word: 16 lanes hold a block, and the
      // largest of them is found for four at once (lanes past the row's end hold zeros)
      float v[V][VEC];
      uint32_t bytes[(V + 3) / 4];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        uint32_t top = 0u;
        if (column(k) < p.C) {
          float w[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) w[e] = 1.f;
          if (p.weight) load_param<VEC>(p.weight, p.param_f32, params + column(k), w);
          raw[0][k].get(v[k]);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            v[k][e] = v[k][e] * rstd.v[0] * w[e];
            top = max(top, fp8_magnitude(v[k][e]));
          }
        }
        const uint32_t byte = static_cast<uint32_t>(fp8_scale(top)) << (8 * (k % 4));
        bytes[k / 4] = k % 4 == 0 ? byte : bytes[k / 4] | byte;
      }
#pragma unroll
      for (int s = 8; s > 0; s >>= 1)
#pragma unroll
        for (int i = 0; i < (V + 3) / 4; ++i)
          bytes[i] = __vmaxu4(bytes[i], __shfl_xor_sync(0xffffffffu, bytes[i], s));
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        const uint8_t scale = static_cast<uint8_t>(bytes[k / 4] >> (8 * (k % 4)));
        const float inv = fp8_inverse(scale);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[k][e] *= inv;
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + row * p.C + column(k)) = fp8_codes(v[k]);
        if ((team.t & 15) == 0) p.y_scale[row * ((p.C + 127) / 128) + (column(k) >> 7)] = scale;
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        float w[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = 1.f;
        if (p.weight) load_param<VEC>(p.weight, p.param_f32, params + column(k), w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r >= n) continue;
          float v[VEC];
          raw[r][k].get(v);
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[e] = v[e] * rstd.v[r] * w[e];
          store_y<TY, VEC>(p.y, static_cast<size_t>(row + r) * p.C + column(k), v);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < n && team.t == 0 && p.rstd) p.rstd[row + r] = rstd.v[r];
    row += n;
    left -= n;
    if (p.groups > 1 && left == 0) {
      left = p.rows_per_group;
      params += p.C;
    }
  }
}

// A thread's ring in shared memory, of the rows kernels: [2][R][V] slots of `pieces` 16-byte
// pieces for each thread of the block.  The 32 lanes of a warp copy the 8 columns of each of
// them together, 512 bytes at a time (in fp32 a lane's own 32 bytes would make every copy
// fetch half of each sector), so a warp waits for all of its lanes before it reads or copies.
struct Ring {
  uint32_t base;     // of the block
  uint32_t threads, warp, lane;
  int columns;       // of a row
  int slots_k, pieces, rows;
  template <class T>
  __device__ __forceinline__ void copy(int stage, int r, int k, int from_piece, const T* row, int at_column) const {
    constexpr int P = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = at_column + (i * 32 + lane) * (16 / static_cast<int>(sizeof(T)));
      if (c < columns) copy_16b(at<T>(stage, r, k, from_piece) + (i * 32 + lane) * 16, row + c);
    }
  }
  template <class T>
  __device__ __forceinline__ Raw<T, 8> read(int stage, int r, int k, int from_piece) const {
    constexpr int P = sizeof(T) / 2;
    Raw<T, 8> raw;
#pragma unroll
    for (int i = 0; i < P; ++i)
      reinterpret_cast<uint4*>(&raw)[i] = shared_16b(at<T>(stage, r, k, from_piece) + (lane * P + i) * 16);
    return raw;
  }

 private:
  template <class T>
  __device__ __forceinline__ uint32_t at(int stage, int r, int k, int from_piece) const {
    constexpr int P = sizeof(T) / 2;
    return base + 16 * threads * (((stage * rows + r) * slots_k + k) * pieces + from_piece) + warp * 512 * P;
  }
};

// Many rows in 16-byte pieces, as the backward below: a team takes R rows at a time, every
// thread copies its columns of the next ones to shared memory meanwhile, one barrier a
// batch.  Block (part, group): rows [part n / parts, (part + 1) n / parts) of the group, whose
// weight stays in registers.  Pieces of a thread's 8 columns: of x and the residual.
template <class TX, bool RES>
constexpr int kFwdPieces = sizeof(TX) / 2 * (RES ? 2 : 1);
template <class TX, int V, bool RES>
constexpr int kFwdRows = 4 / V / (kFwdPieces<TX, RES> > 2 ? 2 : 1);

template <class TX, class TY, int V, bool RES>
__global__ void __maxnreg__(V == 1 ? 80 : 128) rms_fwd_rows_kernel(const RmsParams p) {
  constexpr bool CODES = std::is_same_v<TY, E4m3>;
  constexpr int R = kFwdRows<TX, V, RES>, PX = sizeof(TX) / 2, PIECES = kFwdPieces<TX, RES>;
  __shared__ float red[2][16][R];
  extern __shared__ __align__(16) uint8_t ring[];  // [2][R][V][PIECES][threads] pieces
  const Team team(p.W);
  const TX* x = static_cast<const TX*>(p.x);
  [[maybe_unused]] const TX* res = static_cast<const TX*>(p.residual);
  [[maybe_unused]] TX* hs = static_cast<TX*>(p.h);
  const int lane = threadIdx.x & 31;
  const float inv_c = 1.f / static_cast<float>(p.C);
  const int part = blockIdx.x % p.parts;
  const long long group = blockIdx.x / p.parts;
  const long long n = p.rows_per_group;
  const long long r0 = group * n + part * n / p.parts, r1 = group * n + (part + 1) * n / p.parts;
  const size_t g = static_cast<size_t>(group) * p.C;
  auto column = [&](int k) { return (k * team.W * 32 + team.t) * 8; };
  const Ring slots{smem_u32(ring), blockDim.x, threadIdx.x >> 5, threadIdx.x & 31, p.C, V, PIECES, R};
  auto warp_column = [&](int k) { return (k * team.W + team.warp) * 256; };
  pdl_wait();
  pdl_trigger();
  auto fetch = [&](long long row, int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= r1) continue;
      const size_t from = static_cast<size_t>(row + r) * p.C;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        slots.copy(stage, r, k, 0, x + from, warp_column(k));
        if constexpr (RES) slots.copy(stage, r, k, PX, res + from, warp_column(k));
      }
    }
  };
  long long row = r0 + static_cast<long long>(team.index) * R;
  const long long step = static_cast<long long>(team.count) * R;
  fetch(row, 0);
  copy_commit();
  float2 w[V][4];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float one[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (p.weight && column(k) < p.C) load_param<8>(p.weight, p.param_f32, g + column(k), one);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[k][e] = make_float2(one[2 * e], one[2 * e + 1]);
  }
  for (int turn = 0; row < r1; row += step, turn ^= 1) {
    __syncwarp();
    fetch(row + step, turn ^ 1);
    copy_commit();
    copy_wait<1>();
    __syncwarp();
    Raw<TX, 8> held[R][V];
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = 0.f;
      if (row + r >= r1) continue;
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        held[r][k] = slots.read<TX>(turn, r, k, 0);
        float v[8];
        held[r][k].get(v);
        if constexpr (RES) {
          float a[8];
          slots.read<TX>(turn, r, k, PX).get(a);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += a[e];
          held[r][k].put(v);
          held[r][k].get(v);
          store<8>(hs + static_cast<size_t>(row + r) * p.C + column(k), v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = make_float2(v[2 * e], v[2 * e + 1]);
          s2 = fma2(u, u, s2);
        }
      }
      s[r] = s2.x + s2.y;
    }
    float sum = warp_sums<R>(s);
    constexpr int kShare = 32 / R;  // lanes of a value
    int from = kShare;
    if (p.W > 1) {
      if (lane % kShare == 0) red[turn][team.index * p.W + team.warp][lane / kShare] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(team.index + 1), "r"(p.W * 32) : "memory");
      sum = 0.f;
      for (int i = lane / R; i < p.W; i += kShare) sum += red[turn][team.index * p.W + i][lane % R];
#pragma unroll
      for (int m = R; m < 32; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
      from = 1;
    }
    sum = rsqrtf(sum * inv_c + p.eps);
    float rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) rstd[r] = __shfl_sync(0xffffffffu, sum, r * from);
    if (team.t == 0 && p.rstd) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (row + r < r1) p.rstd[row + r] = rstd[r];
    }
    // y of a row's columns
    auto result = [&](int r, int k, float2 (&y)[4]) {
      float v[8];
      held[r][k].get(v);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = mul2(mul2(make_float2(v[2 * e], v[2 * e + 1]), make_float2(rstd[r], rstd[r])), w[k][e]);
    };
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const bool in = column(k) < p.C;
      if constexpr (CODES) {
        // scale bytes of the rows: 16 lanes hold a block, and the largest is found for all rows
        // at once (lanes past the row's end hold zeros)
        // (y is worked out twice: held for all rows it spilled, 14080 x 2560 bf16 43 -> 55 us)
        uint32_t bytes = 0u;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (!in || row + r >= r1) continue;
          float2 y[4];
          result(r, k, y);
          float top = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fp8_largest(top, y[e].x, y[e].y);
          bytes |= static_cast<uint32_t>(fp8_scale(__float_as_uint(top))) << (8 * r);
        }
#pragma unroll
        for (int i = 8; i > 0; i >>= 1) bytes = __vmaxu4(bytes, __shfl_xor_sync(0xffffffffu, bytes, i));
        if (!in) continue;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (row + r >= r1) continue;
          float2 y[4];
          result(r, k, y);
          const uint8_t scale = static_cast<uint8_t>(bytes >> (8 * r));
          const float inv = fp8_inverse(scale);
          const float2 by = make_float2(inv, inv);
          *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (row + r) * p.C + column(k)) =
              make_uint2(fp8_four(mul2(y[0], by), mul2(y[1], by)), fp8_four(mul2(y[2], by), mul2(y[3], by)));
          if ((team.t & 15) == 0) p.y_scale[(row + r) * ((p.C + 127) / 128) + (column(k) >> 7)] = scale;
        }
      } else {
        if (!in) continue;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (row + r >= r1) continue;
          float2 y[4];
          result(r, k, y);
          const float v[8] = {y[0].x, y[0].y, y[1].x, y[1].y, y[2].x, y[2].y, y[3].x, y[3].y};
          store_y<TY, 8>(p.y, static_cast<size_t>(row + r) * p.C + column(k), v);
        }
      }
    }
  }
}

// A block's sums of dw over its rows: its partial, or the result.
__device__ __forceinline__ void write_weight(const RmsParams& p, size_t g, const float* sums) {
  for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
    if (p.parts > 1)
      p.partial[static_cast<size_t>(blockIdx.x) * p.C + c] = sums[c];
    else
      store_param(p.dweight, p.param_f32, g + c, sums[c]);
  }
}

// Single elements.  Block (part, group): rows [part n / parts, (part + 1) n / parts) of the group.
template <class TX, class TY, int V>
__global__ void __launch_bounds__(max_threads(1, V), V <= 4 ? 3 : V <= 8 ? 2 : 1) rms_bwd_kernel(const RmsParams p) {
  __shared__ Sums<1> red[2][16];
  extern __shared__ float sums[];  // [C]
  const Team team(p.W);
  const TX* h = static_cast<const TX*>(p.h);
  const TX* dh = static_cast<const TX*>(p.dh);
  const TY* dy = static_cast<const TY*>(p.dy);
  TX* dx = static_cast<TX*>(p.dx);
  const float inv_c = 1.f / static_cast<float>(p.C);
  const int part = blockIdx.x % p.parts;
  const long long group = blockIdx.x / p.parts;
  const long long n = p.rows_per_group;
  const long long r0 = group * n + part * n / p.parts, r1 = group * n + (part + 1) * n / p.parts;
  const size_t g = static_cast<size_t>(group) * p.C;
  auto column = [&](int k) { return k * team.W * 32 + team.t; };
  pdl_wait();
  pdl_trigger();
  Raw<TX, 1> rh[V], rd[V];
  Raw<TY, 1> rg[V];
  float rstd = 0.f;
  auto fetch = [&](long long row) {
    rstd = p.rstd[row];
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (column(k) < p.C) {
        rh[k].load(h + row * p.C + column(k));
        rg[k].load(dy + row * p.C + column(k));
        if (dh) rd[k].load(dh + row * p.C + column(k));
      }
  };
  if (r0 + team.index < r1) fetch(r0 + team.index);
  float w[V], aw[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float one[1] = {1.f};
    if (p.weight && column(k) < p.C) load_param<1>(p.weight, p.param_f32, g + column(k), one);
    w[k] = one[0];
    aw[k] = 0.f;
  }
  int turn = 0;
  for (long long row = r0 + team.index; row < r1; row += team.count, turn ^= 1) {
    float xh[V], gr[V], add[V];
    Sums<1> s = {{0.f}};
    const float rs = rstd;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (column(k) >= p.C) continue;
      float v[1];
      rh[k].get(v);
      xh[k] = v[0] * rs;
      rg[k].get(v);
      aw[k] = fmaf(v[0], xh[k], aw[k]);
      gr[k] = v[0] * w[k];
      s.v[0] = fmaf(gr[k], xh[k], s.v[0]);
      v[0] = 0.f;
      if (dh) rd[k].get(v);
      add[k] = v[0];
    }
    if (row + team.count < r1) fetch(row + team.count);
    s = team.sum(s, red[turn]);
    const float m = s.v[0] * inv_c;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (column(k) >= p.C) continue;
      float v[1] = {fmaf(rs, gr[k] - xh[k] * m, add[k])};
      store<1>(dx + row * p.C + column(k), v);
    }
  }
  if (!p.dweight) return;
  for (int t = 0; t < team.count; ++t) {
    if (team.index == t) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = column(k);
        if (c < p.C) sums[c] = t == 0 ? aw[k] : sums[c] + aw[k];
      }
    }
    __syncthreads();
  }
  write_weight(p, g, sums);
}

// The same with rows in 16-byte pieces, the layer norm's way: a team takes R rows at a
// time, every thread copies its columns of the next ones to shared memory meanwhile.
// Pieces of a thread's 8 columns: of h, dy and dh.
template <class TX, class TY, bool DH>
constexpr int kPieces = (sizeof(TX) * (DH ? 2 : 1) + sizeof(TY)) / 2;
template <class TX, class TY, int V, bool DH>
constexpr int kRowsOf = kPieces<TX, TY, DH> <= 2 ? 4 / V : kPieces<TX, TY, DH> <= 4 ? 2 / V : 1;

template <class TX, class TY, int V, bool DH>
__global__ void __maxnreg__(V == 1 ? 80 : 128) rms_bwd_rows_kernel(const RmsParams p) {
  constexpr int R = kRowsOf<TX, TY, V, DH>;
  constexpr int PX = sizeof(TX) / 2, PY = sizeof(TY) / 2;  // pieces of h (and dh), of dy
  constexpr int PIECES = kPieces<TX, TY, DH>;
  __shared__ float red[2][16][R];
  extern __shared__ __align__(16) uint8_t ring[];  // [2][R][V][PIECES][threads] pieces; then [C] sums
  const Team team(p.W);
  const TX* h = static_cast<const TX*>(p.h);
  [[maybe_unused]] const TX* dh = static_cast<const TX*>(p.dh);
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
  const Ring slots{smem_u32(ring), blockDim.x, threadIdx.x >> 5, threadIdx.x & 31, p.C, V, PIECES, R};
  auto warp_column = [&](int k) { return (k * team.W + team.warp) * 256; };
  pdl_wait();
  pdl_trigger();
  float rstd[R], next_rstd[R];
  auto fetch = [&](long long row, int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= r1) continue;
      next_rstd[r] = p.rstd[row + r];
      const size_t from = static_cast<size_t>(row + r) * p.C;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        slots.copy(stage, r, k, 0, h + from, warp_column(k));
        slots.copy(stage, r, k, PX, dy + from, warp_column(k));
        if constexpr (DH) slots.copy(stage, r, k, PX + PY, dh + from, warp_column(k));
      }
    }
  };
  long long row = r0 + static_cast<long long>(team.index) * R;
  const long long step = static_cast<long long>(team.count) * R;
#pragma unroll
  for (int r = 0; r < R; ++r) next_rstd[r] = 0.f;
  fetch(row, 0);
  copy_commit();
  // (pairs of columns: an instruction does two)
  float2 w[V][4], aw[V][4];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float one[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (p.weight && column(k) < p.C) load_param<8>(p.weight, p.param_f32, g + column(k), one);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      aw[k][e] = make_float2(0.f, 0.f);
      w[k][e] = make_float2(one[2 * e], one[2 * e + 1]);
    }
  }
  // 8 columns of a row as fp32, from piece `first` on
  auto read = [&](auto like, int stage, int r, int k, int first, float2 (&v)[4]) {
    float f[8];
    slots.read<decltype(like)>(stage, r, k, first).get(f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = make_float2(f[2 * e], f[2 * e + 1]);
  };
  auto both = [](float v) { return make_float2(v, v); };
  for (int turn = 0; row < r1; row += step, turn ^= 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) rstd[r] = next_rstd[r];
    __syncwarp();
    fetch(row + step, turn ^ 1);
    copy_commit();
    copy_wait<1>();
    __syncwarp();
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = 0.f;
      if (row + r >= r1) continue;
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        float2 xh[4], gr[4];
        read(TX(), turn, r, k, 0, xh);
        read(TY(), turn, r, k, PX, gr);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = mul2(gr[e], mul2(xh[e], both(rstd[r])));  // dy xh
          aw[k][e] = add2(aw[k][e], t);
          s2 = fma2(t, w[k][e], s2);
        }
      }
      s[r] = s2.x + s2.y;
    }
    float sum = warp_sums<R>(s);
    constexpr int kShare = 32 / R;  // lanes of a value
    int from = kShare;
    if (p.W > 1) {
      if (lane % kShare == 0) red[turn][team.index * p.W + team.warp][lane / kShare] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(team.index + 1), "r"(p.W * 32) : "memory");
      sum = 0.f;
      for (int i = lane / R; i < p.W; i += kShare) sum += red[turn][team.index * p.W + i][lane % R];
#pragma unroll
      for (int m = R; m < 32; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
      from = 1;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = __shfl_sync(0xffffffffu, sum, r * from) * inv_c;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= r1) continue;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (column(k) >= p.C) continue;
        float2 xh[4], gr[4], add[4];
        read(TX(), turn, r, k, 0, xh);
        read(TY(), turn, r, k, PX, gr);
        if constexpr (DH) read(TX(), turn, r, k, PX + PY, add);
        const float2 slope = both(-rstd[r] * s[r]);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = fma2(xh[e], slope, mul2(gr[e], w[k][e]));
          const float2 u = DH ? fma2(t, both(rstd[r]), add[e]) : mul2(t, both(rstd[r]));
          v[2 * e] = u.x;
          v[2 * e + 1] = u.y;
        }
        store<8>(dx + static_cast<size_t>(row + r) * p.C + column(k), v);
      }
    }
  }
  if (!p.dweight) return;
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
        }
      }
    }
    __syncthreads();
  }
  write_weight(p, g, sums);
}

// dw of a group from its blocks' partials: `split` threads a column, each an equal share
// of the parts in their order.
__global__ void __launch_bounds__(256) rms_weight_kernel(const RmsParams p, int split) {
  __shared__ float sums[256];
  const int columns = 256 / split;
  const int lane = threadIdx.x / columns, at = threadIdx.x % columns;
  const int c = blockIdx.x * columns + at;
  pdl_wait();
  pdl_trigger();
  for (int g = blockIdx.y; g < p.groups; g += gridDim.y) {
    float s = 0.f;
    if (c < p.C) {
      const float* in = p.partial + static_cast<size_t>(g) * p.parts * p.C + c;
      const int i1 = p.parts * (lane + 1) / split;
#pragma unroll 8
      for (int i = p.parts * lane / split; i < i1; ++i) s += in[static_cast<size_t>(i) * p.C];
    }
    if (split > 1) {
      sums[threadIdx.x] = s;
      __syncthreads();
      for (int k = 1; lane == 0 && k < split; ++k) s += sums[k * columns + at];
    }
    if (lane == 0 && c < p.C) store_param(p.dweight, p.param_f32, static_cast<size_t>(g) * p.C + c, s);
    __syncthreads();
  }
}

// The rows kernels' shared memory: the rows' ring (of 512 threads in fp32 with dh: two stages of
// two times six pieces), or the sums of the widest row.
constexpr int kRmsMaxSmem = 2 * 2 * 6 * 16 * 512;
static_assert(kRmsMaxSmem >= kNormMaxC * static_cast<int>(sizeof(float)), "the sums fit");

template <class X, class Y, int VEC, int V, bool RES>
cudaError_t run_fwd(const RmsParams& p, const Shape& sh, int sms, cudaStream_t s) {
  const int teams = sh.threads / 32 / sh.W;
  const long long blocks = (p.rows + teams - 1) / teams;
  // as many blocks as the SMs hold (of fewer threads, more)
  const long long most = static_cast<long long>(sms) * fwd_blocks(VEC, V, sizeof(X)) * 256 / sh.threads;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), dim3(sh.threads), 0, s);
  return cudaLaunchKernelEx(&cfg, rms_fwd_kernel<X, Y, VEC, V, RES>, p);
}

template <class X, class Y, int V, bool RES>
cudaError_t run_fwd_rows(RmsParams p, const RowsShape& sh, int dev, int sms, cudaStream_t s) {
  constexpr auto kKernel = rms_fwd_rows_kernel<X, Y, V, RES>;
  const size_t ring = static_cast<size_t>(2) * kFwdRows<X, V, RES> * V * kFwdPieces<X, RES> * 16 * sh.threads;
  static OncePerDevice prepared;
  const cudaError_t e = prepared(
      dev, [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRmsMaxSmem); });
  if (e != cudaSuccess) return e;
  // A group's rows are in parts for as many blocks as the backward has, or, where instructions
  // and not HBM bound the time, as many as the SMs hold.  The two differ at 14080 x 5120, one block of 320
  // threads and two (us): bf16 58 and 46, with the residual 89 and 95; to 8 bits 87 and 60, with the
  // residual 103 and 84; fp32 98 and 98, with the residual 175 and 197, to 8 bits 83 and 83, but with the
  // residual, where the rule is wrong, 153 and 163.  At 768, 1536, 2560, 4096 and 8192 channels, all types,
  // they are within 1%.
  p.parts = rms_parts(p.rows_per_group, p.C, p.groups);
  if constexpr (std::is_same_v<Y, E4m3> || !RES) {
    static std::atomic<int> held[kMaxDevices][kNormMaxC / 256 + 1];
    std::atomic<int>& here = held[dev][sh.W];  // (dev is one that `prepared` has taken)
    int blocks = here.load(std::memory_order_relaxed);
    if (blocks == 0) {
      const cudaError_t o = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kKernel, sh.threads, ring);
      if (o != cudaSuccess) return o;
      here.store(blocks, std::memory_order_relaxed);
    }
    const long long parts = std::min(static_cast<long long>(sms) * blocks / p.groups, p.rows_per_group);
    p.parts = static_cast<int>(std::max(parts, 1ll));
  }
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(static_cast<unsigned>(p.groups) * p.parts), dim3(sh.threads), ring, s);
  return cudaLaunchKernelEx(&cfg, kKernel, p);
}

template <class X, class Y, bool RES>
cudaError_t run_fwd_shape(const RmsParams& p, bool vec, const Shape& sh, int sms, cudaStream_t s) {
  if (vec) {
    if (sh.V == 1) return run_fwd<X, Y, 8, 1, RES>(p, sh, sms, s);
    if (sh.V == 2) return run_fwd<X, Y, 8, 2, RES>(p, sh, sms, s);
    if (sh.V == 3) return run_fwd<X, Y, 8, 3, RES>(p, sh, sms, s);
    return run_fwd<X, Y, 8, 4, RES>(p, sh, sms, s);
  }
  if constexpr (!std::is_same_v<Y, E4m3>) {
    if (sh.V == 2) return run_fwd<X, Y, 1, 2, RES>(p, sh, sms, s);
    if (sh.V == 4) return run_fwd<X, Y, 1, 4, RES>(p, sh, sms, s);
    if (sh.V == 8) return run_fwd<X, Y, 1, 8, RES>(p, sh, sms, s);
    return run_fwd<X, Y, 1, 16, RES>(p, sh, sms, s);
  }
  return cudaErrorInvalidValue;  // (codes are written in pieces of eight)
}

template <auto kKernel>
cudaError_t run_bwd(const RmsParams& p, unsigned blocks, int threads, size_t smem, int dev, cudaStream_t s) {
  static OncePerDevice prepared;
  const cudaError_t e = prepared(
      dev, [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRmsMaxSmem); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(blocks), dim3(threads), smem, s);
  return cudaLaunchKernelEx(&cfg, kKernel, p);
}

template <class X, class Y, int V, bool DH>
cudaError_t run_bwd_rows(const RmsParams& p, unsigned blocks, const RowsShape& sh, int dev, cudaStream_t s) {
  const size_t ring = static_cast<size_t>(2) * kRowsOf<X, Y, V, DH> * V * kPieces<X, Y, DH> * 16 * sh.threads;
  const size_t sums = static_cast<size_t>(p.C) * sizeof(float);
  return run_bwd<rms_bwd_rows_kernel<X, Y, V, DH>>(p, blocks, sh.threads, ring > sums ? ring : sums, dev, s);
}

}  // namespace

int rms_parts(long long rows_per_group, int C, int groups) {
  // as many blocks as the SMs hold, by the form that aligned rows take
  long long parts;
  if (C % 8 == 0) {
    parts = static_cast<long long>(kNormSms) * rows_shape(C).blocks / groups;
  } else {
    const Shape sh = shape_of(C, false, false);
    parts = static_cast<long long>(kNormSms) * (sh.V <= 4 ? 3 : sh.V <= 8 ? 2 : 1) * max_threads(1, sh.V) /
            sh.threads / groups;
  }
  if (parts > rows_per_group) parts = rows_per_group;
  return parts < 1 ? 1 : static_cast<int>(parts);
}

cudaError_t launch_rms_fwd(RmsParams p, bool vec, int dev, int sms, cudaStream_t s) {
  auto types = [&](auto f) {
    if (p.y_type == kRmsCodes) return p.x_f32 ? f(float{}, E4m3{}) : f(bf16{}, E4m3{});
    if (!p.x_f32) return f(bf16{}, bf16{});
    return p.y_type == kRmsF32 ? f(float{}, float{}) : f(float{}, bf16{});
  };
  // Rows that a warp or few hold are started sooner than copied ahead.  us of rms_fwd_kernel and of this
  // one, cold, bf16: 1216 x 768 2.2 and 2.6, 1824 x 768 4.9 and 3.1 (fp32 with the residual 4.3 and 4.3, 7.3 and
  // 5.3).  Of wide rows fewer would do: 608 x 2560 3.1 and 3.1, but 1216 x 2560 7.1 and 4.4.
  if (vec && p.rows > 8ll * sms) {
    const RowsShape sh = rows_shape(p.C);
    p.W = sh.W;
    return types([&](auto tx, auto ty) {
      using X = decltype(tx);
      using Y = decltype(ty);
      if (sh.V == 1)
        return p.residual ? run_fwd_rows<X, Y, 1, true>(p, sh, dev, sms, s)
                          : run_fwd_rows<X, Y, 1, false>(p, sh, dev, sms, s);
      return p.residual ? run_fwd_rows<X, Y, 2, true>(p, sh, dev, sms, s)
                        : run_fwd_rows<X, Y, 2, false>(p, sh, dev, sms, s);
    });
  }
  const Shape sh = shape_of(p.C, vec, true);
  p.W = sh.W;
  return types([&](auto tx, auto ty) {
    using X = decltype(tx);
    using Y = decltype(ty);
    return p.residual ? run_fwd_shape<X, Y, true>(p, vec, sh, sms, s) : run_fwd_shape<X, Y, false>(p, vec, sh, sms, s);
  });
}

cudaError_t launch_rms_bwd(RmsParams p, bool vec, int dev, cudaStream_t s) {
  const unsigned blocks = static_cast<unsigned>(p.groups) * p.parts;
  cudaError_t e;
  auto types = [&](auto f) {
    if (!p.x_f32) return f(bf16{}, bf16{});
    if (p.y_type == kRmsF32) return f(float{}, float{});
    return f(float{}, bf16{});
  };
  if (vec) {
    const RowsShape sh = rows_shape(p.C);
    p.W = sh.W;
    e = types([&](auto tx, auto ty) {
      using X = decltype(tx);
      using Y = decltype(ty);
      if (sh.V == 1)
        return p.dh ? run_bwd_rows<X, Y, 1, true>(p, blocks, sh, dev, s)
                    : run_bwd_rows<X, Y, 1, false>(p, blocks, sh, dev, s);
      return p.dh ? run_bwd_rows<X, Y, 2, true>(p, blocks, sh, dev, s)
                  : run_bwd_rows<X, Y, 2, false>(p, blocks, sh, dev, s);
    });
  } else {
    const Shape sh = shape_of(p.C, false, false);
    p.W = sh.W;
    const size_t sums = static_cast<size_t>(p.C) * sizeof(float);
    e = types([&](auto tx, auto ty) {
      using X = decltype(tx);
      using Y = decltype(ty);
      if (sh.V == 2) return run_bwd<rms_bwd_kernel<X, Y, 2>>(p, blocks, sh.threads, sums, dev, s);
      if (sh.V == 4) return run_bwd<rms_bwd_kernel<X, Y, 4>>(p, blocks, sh.threads, sums, dev, s);
      if (sh.V == 8) return run_bwd<rms_bwd_kernel<X, Y, 8>>(p, blocks, sh.threads, sums, dev, s);
      return run_bwd<rms_bwd_kernel<X, Y, 16>>(p, blocks, sh.threads, sums, dev, s);
    });
  }
  if (e != cudaSuccess || p.parts == 1 || !p.dweight) return e;
  int split = 1;
  while (split < 32 && p.parts >= 16 * split) split *= 2;
  const int columns = 256 / split;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3((p.C + columns - 1) / columns, p.groups < 65535 ? p.groups : 65535), dim3(256), 0, s);
  return cudaLaunchKernelEx(&cfg, rms_weight_kernel, p, split);
}

}  // namespace mw
