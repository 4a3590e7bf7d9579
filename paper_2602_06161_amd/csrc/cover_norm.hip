// Residual addition and root-mean-square norm, optionally into e4m3 with a scale per row.
//
// A row is read once and kept in registers: h = x + residual, then one reduction of sum h^2 and (for
// e4m3) max |h w|, then y = h * rs * w.  The row's largest |y| is rs * max |h w| up to two roundings,
// so both statistics take a single pass across the workgroup (a second one where h w leaves fp32's normal
// range, as y need not).  Everything is fp32 (so the sum of squares,
// and an |h| of up to 1.8e19); what is rounded to fewer bits is only what is stored, h and y or its codes.
//
// Bound by HBM from about 1000 rows on, below that by one launch and one row's latency.  Measured, bf16 with
// a residual, 8 D bytes of traffic per row: 64 x 4096 3.2 us, 1024 x 4096 7.8 us (4.3 TB/s), 4096 x 4096
// 21.3 us (6.3 TB/s, part of it in the last-level cache), 16384 x 4096 93 us (5.75 TB/s; a large copy reaches
// 5.1); with e4m3 codes 64 x 4096 3.6 us, 2048 x 8192 19.0 us; fp32 2048 x 4096 23.0 us (5.8 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cover.h"
#include "cover_e4m3.h"
#include "cover_internal.h"

namespace cover {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Chunk;  // 16 bytes of a row
template <> struct Chunk<__bf16> { typedef bf16x8 V; static constexpr int E = 8; };
template <> struct Chunk<float> { typedef f32x4 V; static constexpr int E = 4; };

// One workgroup per row; thread t holds chunks t, t + threads, ... (CH of them).
template <class T, int CH, bool E4M3>
__global__ __launch_bounds__(1024) void cover_rms_norm_kernel(const NormArgs p) {
  typedef typename Chunk<T>::V V;
  constexpr int E = Chunk<T>::E;
  __shared__ float s_sum[16];
  __shared__ uint32_t s_top[16];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int64_t row = blockIdx.x;
  const T* x = (const T*)p.x + row * p.x_stride;
  const T* res = p.residual ? (const T*)p.residual + row * p.res_stride : nullptr;
  const T* w = (const T*)p.weight;
  const int whole = p.D / E, tail = p.D % E;  // elements of the last chunk, if it is not whole

  float h[CH][E], g[CH][E];
  float sum = 0.0f;
  uint32_t top = 0u;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = tid + j * nt, e0 = c * E;
    V a = {}, b = {}, f;
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = (T)1.0f;
    if (c < whole) {
      a = *(const V*)(x + e0);
      if (res) b = *(const V*)(res + e0);
      if (w) f = *(const V*)(w + e0);
    } else if (c == whole) {
#pragma unroll
      for (int e = 0; e < E - 1; ++e)
        if (e < tail) {
          a[e] = x[e0 + e];
          if (res) b[e] = res[e0 + e];
          if (w) f[e] = w[e0 + e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      h[j][e] = (float)a[e] + (float)b[e];
      g[j][e] = (float)f[e];
      sum = __builtin_fmaf(h[j][e], h[j][e], sum);
      if constexpr (E4M3) top = max(top, magnitude(h[j][e] * g[j][e]));
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    sum += __shfl_xor(sum, m);
    if constexpr (E4M3) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  }
  if ((tid & 63) == 0) {
    s_sum[tid >> 6] = sum;
    if constexpr (E4M3) s_top[tid >> 6] = top;
  }
  __syncthreads();
  sum = s_sum[0];
  if constexpr (E4M3) top = s_top[0];
  for (int i = 1; i < nt >> 6; ++i) {
    sum += s_sum[i];
    if constexpr (E4M3) top = max(top, s_top[i]);
  }
  const float rs = 1.0f / sqrtf(sum / (float)p.D + p.eps);
  float inv = 1.0f;
  if constexpr (E4M3) {
    float largest = __uint_as_float(top) * rs;
    if (top >= 0x7f800000u || top < 0x00800000u) {  // (the same in every thread)
      top = 0u;
#pragma unroll
      for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) top = max(top, magnitude(h[j][e] * rs * g[j][e]));
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
      __syncthreads();
      if ((tid & 63) == 0) s_top[tid >> 6] = top;
      __syncthreads();
      top = s_top[0];
      for (int i = 1; i < nt >> 6; ++i) top = max(top, s_top[i]);
      largest = __uint_as_float(top);
    }
    const float s = e4m3_scale(largest);
    inv = 1.0f / s;
    if (tid == 0) p.scale[row] = s;
  }

  T* ro = p.residual_out ? (T*)p.residual_out + row * p.res_out_stride : nullptr;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = tid + j * nt, e0 = c * E;
    if (c > whole || (c == whole && tail == 0)) continue;
    float y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = h[j][e] * rs * g[j][e];
    V hv, yv;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      hv[e] = (T)h[j][e];
      yv[e] = (T)y[e];
    }
    uint32_t code[E / 4];
    if constexpr (E4M3) {
#pragma unroll
      for (int e = 0; e < E; e += 4) code[e / 4] = e4m3_pack(y[e], y[e + 1], y[e + 2], y[e + 3], inv);
    }
    uint8_t* o8 = (uint8_t*)p.out + row * p.out_stride;
    T* o = (T*)p.out + row * p.out_stride;
    if (c < whole) {
      if (ro) *(V*)(ro + e0) = hv;
      if constexpr (E4M3) {
#pragma unroll
        for (int e = 0; e < E / 4; ++e) ((uint32_t*)(o8 + e0))[e] = code[e];
      } else {
        *(V*)(o + e0) = yv;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E - 1; ++e)
        if (e < tail) {
          if (ro) ro[e0 + e] = hv[e];
          if constexpr (E4M3) o8[e0 + e] = (uint8_t)(code[e / 4] >> (8 * (e % 4)));
          else o[e0 + e] = yv[e];
        }
    }
  }
}

// Two chunks per thread in a power-of-two workgroup: half the row per thread means half the waves to join.
// Measured (us) with 1, 2, 4 per thread in bf16: 1 x 4096 3.1, 3.1, 3.5; 64 x 4096 3.2, 3.2, 3.6; 4096 x 4096
// 21.5, 21.3, 22.8; 2048 x 8192 in e4m3 21.9, 19.0, 19.2.  One chunk only up to a single wave, more than two
// where 1024 threads do not hold the row (fp32 has twice the chunks).
int threads_for(int chunks) {
  int nt = 64;
  while (nt < 1024 && nt * 2 < chunks) nt *= 2;
  return nt;
}

template <class T, bool E4M3>
void launch(const NormArgs& a, hipStream_t stream) {
  constexpr int E = Chunk<T>::E;
  static_assert(COVER_NORM_MAX_D <= 1024 * 32, "the widest row fits 1024 threads");
  const int chunks = (a.D + E - 1) / E, nt = threads_for(chunks);
  const dim3 grid((unsigned)a.R);
  if (chunks <= nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 1, E4M3>), grid, dim3(nt), 0, stream, a);
  else if (chunks <= 2 * nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 2, E4M3>), grid, dim3(nt), 0, stream, a);
  else if (E == 8 || chunks <= 4 * nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 4, E4M3>), grid, dim3(nt), 0, stream, a);
  else hipLaunchKernelGGL((cover_rms_norm_kernel<T, 32 / E, E4M3>), grid, dim3(nt), 0, stream, a);
}

}  // namespace

bool rms_norm_fits(const NormArgs& a) {  // a launch has at most 2^32 work-items
  const int per = a.bf16 ? Chunk<__bf16>::E : Chunk<float>::E;
  return (int64_t)a.R * threads_for((a.D + per - 1) / per) < (int64_t(1) << 32);
}

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream) {
  if (a.bf16) {
    if (a.scale) launch<__bf16, true>(a, stream);
    else launch<__bf16, false>(a, stream);
  } else {
    if (a.scale) launch<float, true>(a, stream);
    else launch<float, false>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace cover
