// Keys and values into the 8-bit cache and back.
//
// A row of d elements is d / 8 lanes of 8 elements: one wave holds 8 rows (d = 64) or 4 (d = 128), and
// a row's largest magnitude is a maximum over neighbouring lanes.  A workgroup takes consecutive rows
// of one batch row and head, keys and values together.  A value is scaled in fp32 (one
// rounding at 2^-24) and rounded to the code (store) or to the tensors' type (load).
//
// Bound by HBM where there are many rows, else by a launch and two dependent loads.  Measured, bf16, H32 d128,
// 6 d + 8 bytes per row: store of 64 positions 3.0 us, 1024 6.8 us (3.7 TB/s), 8 x 2048 74 us (5.5 TB/s; a large
// copy reaches 5.1); load 2.7, 6.2 (4.1 TB/s), 71 us (5.8 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cover_e4m3.h"
#include "cover_internal.h"

namespace cover {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
  *(bf16x8*)p = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// this thread's row: batch row, head, row of the call, its position; first element of the lane
template <int D>
struct Place {
  int b, h, n, p, e;
  __device__ explicit Place(const CacheArgs& a) {
    constexpr int kLanes = D / 8, kRows = kThreads / kLanes;
    const int per = (a.N + kRows - 1) / kRows;
    const int64_t bh = blockIdx.x / per;
    b = (int)(bh / a.H);
    h = (int)(bh % a.H);
    n = (int)(blockIdx.x % per) * kRows + threadIdx.x / kLanes;
    e = 8 * (threadIdx.x % kLanes);
    p = -1;
    if (n < a.N) p = a.pos ? a.pos[(int64_t)b * a.N + n] : a.first + n;
  }
};

template <class T, int D>
__global__ __launch_bounds__(kThreads) void cover_cache_store_kernel(const CacheArgs a) {
  const Place<D> at(a);
  const bool there = (unsigned)at.p < (unsigned)a.L;
  float k[8] = {}, v[8] = {};
  if (there) {
    load8((const T*)a.k + at.b * a.k_sb + at.h * a.k_sh + at.n * a.k_sl + at.e, k);
    load8((const T*)a.v + at.b * a.v_sb + at.h * a.v_sh + at.n * a.v_sl + at.e, v);
  }
  uint32_t kt = 0u, vt = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    kt = max(kt, magnitude(k[e]));
    vt = max(vt, magnitude(v[e]));
  }
#pragma unroll
  for (int m = D / 16; m >= 1; m >>= 1) {
    kt = max(kt, (uint32_t)__shfl_xor((int)kt, m));
    vt = max(vt, (uint32_t)__shfl_xor((int)vt, m));
  }
  if (!there) return;
  const float ks = e4m3_scale(__uint_as_float(kt)), vs = e4m3_scale(__uint_as_float(vt));
  const float ki = 1.0f / ks, vi = 1.0f / vs;
  const int64_t c = at.b * a.c_sb + at.h * a.c_sh + at.p * a.c_sl + at.e;
  *(u32x2*)((uint8_t*)a.kc + c) = u32x2{e4m3_pack(k[0], k[1], k[2], k[3], ki), e4m3_pack(k[4], k[5], k[6], k[7], ki)};
  *(u32x2*)((uint8_t*)a.vc + c) = u32x2{e4m3_pack(v[0], v[1], v[2], v[3], vi), e4m3_pack(v[4], v[5], v[6], v[7], vi)};
  if (at.e == 0) {
    const int64_t s = at.b * a.s_sb + at.h * a.s_sh + at.p;
    a.ks[s] = ks;
    a.vs[s] = vs;
  }
}

__device__ __forceinline__ void decode8(u32x2 c, float s, float (&x)[8]) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
    x[4 * w] = lo[0] * s;
    x[4 * w + 1] = lo[1] * s;
    x[4 * w + 2] = hi[0] * s;
    x[4 * w + 3] = hi[1] * s;
  }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void cover_cache_load_kernel(const CacheArgs a) {
  const Place<D> at(a);
  if (at.n >= a.N) return;
  float k[8] = {}, v[8] = {};
  if ((unsigned)at.p < (unsigned)a.L) {
    const int64_t c = at.b * a.c_sb + at.h * a.c_sh + at.p * a.c_sl + at.e;
    const int64_t s = at.b * a.s_sb + at.h * a.s_sh + at.p;
    decode8(*(const u32x2*)((const uint8_t*)a.kc + c), a.ks[s], k);
    decode8(*(const u32x2*)((const uint8_t*)a.vc + c), a.vs[s], v);
  }
  store8((T*)a.k + at.b * a.k_sb + at.h * a.k_sh + at.n * a.k_sl + at.e, k);
  store8((T*)a.v + at.b * a.v_sb + at.h * a.v_sh + at.n * a.v_sl + at.e, v);
}

dim3 grid(const CacheArgs& a) {
  const int rows = kThreads / (a.d / 8);
  return dim3((unsigned)((int64_t)a.B * a.H * ((a.N + rows - 1) / rows)));
}

}  // namespace

hipError_t launch_cache_store(const CacheArgs& a, hipStream_t stream) {
  const dim3 g = grid(a), block(kThreads);
  if (a.bf16) {
    if (a.d == 128) hipLaunchKernelGGL((cover_cache_store_kernel<__bf16, 128>), g, block, 0, stream, a);
    else hipLaunchKernelGGL((cover_cache_store_kernel<__bf16, 64>), g, block, 0, stream, a);
  } else {
    if (a.d == 128) hipLaunchKernelGGL((cover_cache_store_kernel<float, 128>), g, block, 0, stream, a);
    else hipLaunchKernelGGL((cover_cache_store_kernel<float, 64>), g, block, 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_load(const CacheArgs& a, hipStream_t stream) {
  const dim3 g = grid(a), block(kThreads);
  if (a.bf16) {
    if (a.d == 128) hipLaunchKernelGGL((cover_cache_load_kernel<__bf16, 128>), g, block, 0, stream, a);
    else hipLaunchKernelGGL((cover_cache_load_kernel<__bf16, 64>), g, block, 0, stream, a);
  } else {
    if (a.d == 128) hipLaunchKernelGGL((cover_cache_load_kernel<float, 128>), g, block, 0, stream, a);
    else hipLaunchKernelGGL((cover_cache_load_kernel<float, 64>), g, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace cover
