// Residual addition and root-mean-square norm, optionally into e4m3 with a scale per row.
//
// A row is read once and kept in registers: h = x + residual, then one reduction of sum h^2 and (for
// e4m3) max |h w|, then y = h * rs * w.  The row's largest |y| is rs * max |h w| up to two roundings,
// so both statistics take a single pass across the workgroup.
#include <hip/hip_runtime.h>
#include <stdint.h>

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
    const float s = e4m3_scale(__uint_as_float(top) * rs);
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

template <class T, bool E4M3>
void launch(const NormArgs& a, hipStream_t stream) {
  const int chunks = (a.D + Chunk<T>::E - 1) / Chunk<T>::E;
  const dim3 grid((unsigned)a.R);
  int nt = 64;
  while (nt < 1024 && nt * 2 < chunks) nt *= 2;
  if (chunks <= nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 1, E4M3>), grid, dim3(nt), 0, stream, a);
  else if (chunks <= 2 * nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 2, E4M3>), grid, dim3(nt), 0, stream, a);
  else if (chunks <= 4 * nt) hipLaunchKernelGGL((cover_rms_norm_kernel<T, 4, E4M3>), grid, dim3(nt), 0, stream, a);
  else hipLaunchKernelGGL((cover_rms_norm_kernel<T, 8, E4M3>), grid, dim3(nt), 0, stream, a);
}

}  // namespace

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
