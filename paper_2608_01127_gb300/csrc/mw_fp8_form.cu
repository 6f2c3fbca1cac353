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
// threads holds 128 x 128 elements in registers, a thread 8 columns of 8 rows; a row's
// maximum is one over 16 lanes, a column's over the 16 groups of lanes.
#include "mw_fp8.cuh"
#include "mw_internal.h"
#include "mw_ptx.cuh"

namespace mw {
namespace {

template <class T>
struct Eight;  // elements of a row as they lie in memory
template <>
struct Eight<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ float get(int k) const {
    const uint32_t w = k < 2 ? a.x : k < 4 ? a.y : k < 6 ? a.z : a.w;
    return __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ float get(int k) const {
    return k == 0 ? a.x : k == 1 ? a.y : k == 2 ? a.z : k == 3 ? a.w : k == 4 ? b.x : k == 5 ? b.y : k == 6 ? b.z : b.w;
  }
};

template <class T, Fp8Form FORM>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) fp8_form_kernel(const Fp8FormParams p, int tiles_c) {
  constexpr bool ROWS = FORM == Fp8Form::kRows || FORM == Fp8Form::kBoth;
  constexpr bool COLUMNS = FORM == Fp8Form::kColumns || FORM == Fp8Form::kBoth;
  constexpr bool TILES = FORM == Fp8Form::kTiles;
  __shared__ uint32_t tops[COLUMNS ? 8 * 128 : 8];
  const int tile_c = blockIdx.x % tiles_c;
  const long long tile_r = blockIdx.x / tiles_c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int c = tile_c * 128 + part * 8;
  const long long r0 = tile_r * 128 + ry;
  const T* x = static_cast<const T*>(p.x) + r0 * p.C + c;
  pdl_wait();
  pdl_trigger();
  Eight<T> e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (c < p.C && r0 + 16 * i < p.rows)
      e[i].load(x + static_cast<long long>(16 * i) * p.C);
    else
      e[i].zero();
  }
  uint32_t column[8];  // largest magnitudes of the thread's columns
#pragma unroll
  for (int k = 0; k < 8; ++k) column[k] = 0u;
  uint32_t tile = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t top = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t m = fp8_magnitude(e[i].get(k));
      if (COLUMNS) column[k] = max(column[k], m);
      top = max(top, m);
    }
    if constexpr (ROWS) {
#pragma unroll
      for (int s = 8; s > 0; s >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
      const uint8_t scale = fp8_scale(top);
      const long long row = r0 + 16 * i;
      if (row < p.rows && c < p.C) {
        const float inv = fp8_inverse(scale);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = e[i].get(k) * inv;
        *reinterpret_cast<uint2*>(p.q + row * p.C + c) = fp8_codes(v, scale);
        if (part == 0) p.scale[row * tiles_c + tile_c] = scale;
      }
    }
    tile = max(tile, top);
  }
  if constexpr (COLUMNS) {
#pragma unroll
    for (int k = 0; k < 8; ++k) column[k] = max(column[k], __shfl_xor_sync(0xffffffffu, column[k], 16));
    if (lane < 16) {
      uint4* to = reinterpret_cast<uint4*>(tops + warp * 128 + part * 8);
      to[0] = make_uint4(column[0], column[1], column[2], column[3]);
      to[1] = make_uint4(column[4], column[5], column[6], column[7]);
    }
    __syncthreads();
    uint32_t bytes[2] = {0u, 0u};
    float inv[8];
    bool bad[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const uint4 o = reinterpret_cast<const uint4*>(tops + w * 128 + part * 8)[h];
        m.x = max(m.x, o.x), m.y = max(m.y, o.y), m.z = max(m.z, o.z), m.w = max(m.w, o.w);
      }
      const uint32_t top[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint8_t scale = fp8_scale(top[k]);
        bytes[h] |= static_cast<uint32_t>(scale) << (8 * k);
        inv[4 * h + k] = fp8_inverse(scale);
        bad[4 * h + k] = scale == kFp8NanScale;
      }
    }
    if (c < p.C) {
      if (ry == 0) *reinterpret_cast<uint2*>(p.scale_columns + tile_r * p.C + c) = make_uint2(bytes[0], bytes[1]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const long long row = r0 + 16 * i;
        if (row >= p.rows) continue;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = bad[k] ? __uint_as_float(0x7fffffffu) : e[i].get(k) * inv[k];
        *reinterpret_cast<uint2*>(p.q_columns + row * p.C + c) = fp8_codes(v, 0);
      }
    }
  }
  if constexpr (TILES) {
    tile = __reduce_max_sync(0xffffffffu, tile);
    if (lane == 0) tops[warp] = tile;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) tile = max(tile, tops[w]);
    const uint8_t scale = fp8_scale(tile);
    const float inv = fp8_inverse(scale);
    if (threadIdx.x == 0) p.scale[tile_r * tiles_c + tile_c] = scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long long row = r0 + 16 * i;
      if (row >= p.rows || c >= p.C) continue;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = e[i].get(k) * inv;
      *reinterpret_cast<uint2*>(p.q + row * p.C + c) = fp8_codes(v, scale);
    }
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
