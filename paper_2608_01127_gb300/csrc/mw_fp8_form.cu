// Matrices put into 8 bits: e4m3 codes with a power-of-two scale for every block of 128
// elements of a row, of a column, or of 128 x 128.
//
//   s = 2^ceil(log2(max |x| / 448)) (at least 2^-127),   q = e4m3(x / s), to nearest even
//
// A power of two divides without rounding, so a code is off by e4m3's rounding alone, and
// the tensor cores take it as it is (mw_fp8_mm.cu).  A block with a NaN or an infinity has
// the scale NaN and the codes NaN: what it stands for is NaN, wherever it is read.
//
// Bound by HBM: an element is read once for all the forms asked for.  A block of 256
// threads holds 128 x 128 elements in registers, a thread 8 columns of 8 rows.  The scale
// grows with the maximum, so that what lanes and warps put together are scale bytes, four to
// a word: four shuffles for a thread's eight rows.  (With maxima in 32 bits, 32 shuffles and
// a scale for every row in every lane: rows and columns of 14080 x 2560 bf16 46 us.)
#include "mw_fp8.cuh"
#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

// 8 columns of 8 rows of a thread as they lie in memory.
template <class T>
struct Held;
template <>
struct Held<__nv_bfloat16> {
  uint4 a[8];
  __device__ __forceinline__ void load(int i, const __nv_bfloat16* p) { a[i] = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero(int i) { a[i] = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(int i, float2 (&v)[4]) const {
    const uint32_t w[4] = {a[i].x, a[i].y, a[i].z, a[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
  }
  // Scale bytes of the rows (byte i % 4 of word i / 4) and of the columns.
  __device__ __forceinline__ void scales(uint32_t (&rows)[2], uint32_t (&columns)[2]) const {
    uint32_t c[4] = {0u, 0u, 0u, 0u}, r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w[4] = {a[i].x & 0x7fff7fffu, a[i].y & 0x7fff7fffu, a[i].z & 0x7fff7fffu, a[i].w & 0x7fff7fffu};
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] = __vmaxu2(c[k], w[k]);
      r[i] = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      columns[h] = __byte_perm(fp8_scale2(c[2 * h]), fp8_scale2(c[2 * h + 1]), 0x6420);
      uint32_t pair[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t x = r[4 * h + 2 * k], y = r[4 * h + 2 * k + 1];
        pair[k] = fp8_scale2(__vmaxu2(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632)));
      }
      rows[h] = __byte_perm(pair[0], pair[1], 0x6420);
    }
  }
};
template <>
struct Held<float> {
  float4 a[8], b[8];
  __device__ __forceinline__ void load(int i, const float* p) {
    a[i] = reinterpret_cast<const float4*>(p)[0];
    b[i] = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero(int i) { a[i] = b[i] = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(int i, float2 (&v)[4]) const {
    v[0] = make_float2(a[i].x, a[i].y), v[1] = make_float2(a[i].z, a[i].w);
    v[2] = make_float2(b[i].x, b[i].y), v[3] = make_float2(b[i].z, b[i].w);
  }
  __device__ __forceinline__ void scales(uint32_t (&rows)[2], uint32_t (&columns)[2]) const {
    uint32_t c[8] = {};
    rows[0] = rows[1] = columns[0] = columns[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float2 v[4];
      get(i, v);
      uint32_t r = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = fp8_magnitude(v[k].x), y = fp8_magnitude(v[k].y);
        c[2 * k] = max(c[2 * k], x);
        c[2 * k + 1] = max(c[2 * k + 1], y);
        r = max(r, max(x, y));
      }
      rows[i / 4] |= static_cast<uint32_t>(fp8_scale(r)) << (8 * (i % 4));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) columns[k / 4] |= static_cast<uint32_t>(fp8_scale(c[k])) << (8 * (k % 4));
  }
};

__device__ __forceinline__ uint8_t byte_of(const uint32_t (&w)[2], int i) {
  return static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
}

template <class T, Fp8Form FORM>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) fp8_form_kernel(const Fp8FormParams p, int tiles_c) {
  constexpr bool ROWS = FORM == Fp8Form::kRows || FORM == Fp8Form::kBoth;
  constexpr bool COLUMNS = FORM == Fp8Form::kColumns || FORM == Fp8Form::kBoth;
  constexpr bool TILES = FORM == Fp8Form::kTiles;
  __shared__ uint2 tops[COLUMNS ? 8 * 16 : 1];
  __shared__ uint32_t whole[8];
  const int tile_c = blockIdx.x % tiles_c;
  const long long tile_r = blockIdx.x / tiles_c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int c = tile_c * 128 + part * 8;
  const long long r0 = tile_r * 128 + ry;
  // rows r0, r0 + 16, ... that there are, and of this thread's columns
  const int all = static_cast<int>(min(8ll, max(0ll, (p.rows - r0 + 15) / 16))), n = c < p.C ? all : 0;
  const T* x = static_cast<const T*>(p.x) + r0 * p.C + c;
  const size_t pitch = static_cast<size_t>(16) * p.C;
  pdl_wait();
  pdl_trigger();
  Held<T> e;
  if (n == 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) e.load(i, x + i * pitch);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < n)
        e.load(i, x + i * pitch);
      else
        e.zero(i);
    }
  }
  uint32_t rows[2], columns[2];
  e.scales(rows, columns);
  if constexpr (ROWS) {
    // the largest over 16 lanes: halves of the rows change sides, then four bytes go on
    const uint32_t other = __shfl_xor_sync(0xffffffffu, lane & 8 ? rows[0] : rows[1], 8);
    uint32_t r = __vmaxu4(lane & 8 ? rows[1] : rows[0], other);
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) r = __vmaxu4(r, __shfl_xor_sync(0xffffffffu, r, s));
    rows[0] = __shfl_sync(0xffffffffu, r, lane & 16);
    rows[1] = __shfl_sync(0xffffffffu, r, (lane & 16) + 8);
    if (part < all) p.scale[(r0 + 16 * part) * tiles_c + tile_c] = byte_of(rows, part);
  }
  if constexpr (COLUMNS) {
#pragma unroll
    for (int h = 0; h < 2; ++h) columns[h] = __vmaxu4(columns[h], __shfl_xor_sync(0xffffffffu, columns[h], 16));
    if (lane < 16) tops[warp * 16 + part] = make_uint2(columns[0], columns[1]);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const uint2 o = tops[w * 16 + part];
      columns[0] = __vmaxu4(columns[0], o.x);
      columns[1] = __vmaxu4(columns[1], o.y);
    }
    if (ry == 0 && c < p.C)
      *reinterpret_cast<uint2*>(p.scale_columns + tile_r * p.C + c) = make_uint2(columns[0], columns[1]);
  }
  uint8_t tile = 0;
  if constexpr (TILES) {
    uint32_t t = __vmaxu4(rows[0], rows[1]);
    t = __vmaxu4(t, t >> 16);
    t = max(t & 0xffu, t >> 8 & 0xffu);
    t = __reduce_max_sync(0xffffffffu, t);
    if (lane == 0) whole[warp] = t;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) t = max(t, whole[w]);
    tile = static_cast<uint8_t>(t);
    if (threadIdx.x == 0) p.scale[tile_r * tiles_c + tile_c] = tile;
  }
  [[maybe_unused]] float2 inv[4];  // of the columns
  if constexpr (COLUMNS) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      inv[k] = make_float2(fp8_inverse(byte_of(columns, 2 * k)), fp8_inverse(byte_of(columns, 2 * k + 1)));
  }
  const size_t out = static_cast<size_t>(r0) * p.C + c;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= n) continue;
    float2 v[4];
    e.get(i, v);
    if constexpr (ROWS || TILES) {
      const float s = fp8_inverse(ROWS ? byte_of(rows, i) : tile);
      const float2 by = make_float2(s, s);
      *reinterpret_cast<uint2*>(p.q + out + i * pitch) =
          make_uint2(fp8_four(mul2(v[0], by), mul2(v[1], by)), fp8_four(mul2(v[2], by), mul2(v[3], by)));
    }
    if constexpr (COLUMNS)
      *reinterpret_cast<uint2*>(p.q_columns + out + i * pitch) = make_uint2(
          fp8_four(mul2(v[0], inv[0]), mul2(v[1], inv[1])), fp8_four(mul2(v[2], inv[2]), mul2(v[3], inv[3])));
  }
}

template <class T>
cudaError_t run(const Fp8FormParams& p, Fp8Form form, cudaStream_t s) {
  const int tiles_c = (p.C + 127) / 128;
  const long long blocks = (p.rows + 127) / 128 * tiles_c;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr;
  pdl_config(cfg, attr, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s);
  switch (form) {
    case Fp8Form::kRows: return cudaLaunchKernelEx(&cfg, fp8_form_kernel<T, Fp8Form::kRows>, p, tiles_c);
    case Fp8Form::kColumns: return cudaLaunchKernelEx(&cfg, fp8_form_kernel<T, Fp8Form::kColumns>, p, tiles_c);
    case Fp8Form::kTiles: return cudaLaunchKernelEx(&cfg, fp8_form_kernel<T, Fp8Form::kTiles>, p, tiles_c);
    default: return cudaLaunchKernelEx(&cfg, fp8_form_kernel<T, Fp8Form::kBoth>, p, tiles_c);
  }
}

}  // namespace

cudaError_t launch_fp8_form(const Fp8FormParams& p, Fp8Form form, cudaStream_t s) {
  return p.x_f32 ? run<float>(p, form, s) : run<__nv_bfloat16>(p, form, s);
}

}  // namespace mw
