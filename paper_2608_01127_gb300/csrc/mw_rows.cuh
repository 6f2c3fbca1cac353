// What the kernels over the rows of a matrix share: accesses of single elements or 16 bytes
// of bf16 and fp32, sums over the warps of a row.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

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
  __device__ __forceinline__ void put(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
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
  __device__ __forceinline__ void put(const float (&v)[8]) {
    a = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
};
template <class T>
struct Raw<T, 1> {
  T a;
  __device__ __forceinline__ void load(const T* p) { a = *p; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = static_cast<float>(a); }
  __device__ __forceinline__ void put(const float (&v)[1]) { a = static_cast<T>(v[0]); }
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

// Threads of a block at most.
constexpr int max_threads(int VEC, int V) { return VEC == 1 && V > 8 ? 512 : 256; }

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

}  // namespace
}  // namespace mw
