// Rotary positions of queries and keys.
//
// A workgroup takes `rows` positions of one batch row.  Its threads first fill an LDS table of cosines
// and sines, one pair of a position each: the angle in turns pos * freq is reduced in fp64 (its
// fraction of a turn is exact to 2^-53 of the turns), the rest is fp32.  Then `tr` threads per
// position walk the heads: a thread owns the same 2 V elements of every head it visits (V pairs of the
// half layout as two pieces rot / 2 apart, V interleaved pairs as one run, or elements past rot, which
// are copied), so it reads its cosines and sines from the table once, and rotating in place is safe.
// The rotation is fp32; only the result is rounded, to the tensors' type.
//
// Bound by HBM where there are many positions, by a launch, the table (rot / 2 angles per position, 256 at a
// time) and one element's latency where there are few.  Measured, bf16, in place or not, H 32 and 32, d 128:
// 64 positions 3.6 us, 1024 8.1 us (4.1 TB/s of reads and writes), 8 x 2048 95 us (5.7 TB/s; a large copy
// reaches 5.1); B4 Hq40/Hkv8 L256 6.9 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cover_internal.h"

namespace cover {
namespace {

constexpr int kThreads = 256;

template <class T, int V>
struct Vec {
  typedef T type __attribute__((ext_vector_type(V)));
};
template <class T>
struct Vec<T, 1> {
  struct type {
    T x;
    __device__ T& operator[](int) { return x; }
    __device__ const T& operator[](int) const { return x; }
  };
};

struct RopeParams {
  RopeArgs a;
  int tr, rows;         // threads per position, positions per workgroup
  int heads, hsplit;    // heads of q and k together, parts they are cut into
};

template <class T, int V, int D, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void cover_rope_kernel(const RopeParams p) {
  typedef typename Vec<T, V>::type VT;
  constexpr int U = D / (2 * V);  // threads per head
  extern __shared__ float2 table[];  // [rows][rot / 2]
  const RopeArgs& a = p.a;
  const int tid = threadIdx.x, half = a.rot / 2;
  const int hs = blockIdx.x % p.hsplit;
  const int64_t tile = blockIdx.x / p.hsplit;
  const int tiles = (a.L + p.rows - 1) / p.rows;
  const int b = (int)(tile / tiles), l0 = (int)(tile % tiles) * p.rows;
  const int n = min(p.rows, a.L - l0);

  for (int e = tid; e < n * half; e += kThreads) {
    const int l = e / half, i = e % half;
    const double turns = (double)a.pos[b * a.pos_sb + l0 + l] * a.freq[i];
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    table[e] = make_float2(c * a.factor, s * a.factor);
  }
  __syncthreads();

  const int l = tid / p.tr, t = tid % p.tr;
  if (l >= n) return;
  const int u = t % U;
  const bool turn = u * V < half;
  // the two pieces of this thread's elements
  const int e0 = INTERLEAVED ? 2 * V * u : (turn ? V * u : a.rot + 2 * V * (u - half / V));
  const int e1 = INTERLEAVED || !turn ? e0 + V : e0 + half;
  float c[V], s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float2 cs = turn ? table[l * half + V * u + v] : make_float2(1.0f, 0.0f);
    c[v] = cs.x;
    s[v] = cs.y;
  }
  const int step = p.tr / U;
  const int h0 = (int)((int64_t)p.heads * hs / p.hsplit), h1 = (int)((int64_t)p.heads * (hs + 1) / p.hsplit);
  for (int h = h0 + t / U; h < h1; h += step) {
    const bool isq = h < a.Hq;
    const int hh = isq ? h : h - a.Hq;
    const T* src = isq ? (const T*)a.q + b * a.q_sb + hh * a.q_sh + (l0 + l) * a.q_sl
                       : (const T*)a.k + b * a.k_sb + hh * a.k_sh + (l0 + l) * a.k_sl;
    T* dst = isq ? (T*)a.q_out + b * a.qo_sb + hh * a.qo_sh + (l0 + l) * a.qo_sl
                 : (T*)a.k_out + b * a.ko_sb + hh * a.ko_sh + (l0 + l) * a.ko_sl;
    VT x = *(const VT*)(src + e0), y = *(const VT*)(src + e1);
    if (turn) {
      float z[2 * V];  // x and y as one run
#pragma unroll
      for (int v = 0; v < V; ++v) {
        z[v] = (float)x[v];
        z[V + v] = (float)y[v];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        constexpr int kStep = INTERLEAVED ? 2 : 1, kPartner = INTERLEAVED ? 1 : V;
        const float p0 = z[kStep * v], p1 = z[kStep * v + kPartner];
        z[kStep * v] = p0 * c[v] - p1 * s[v];
        z[kStep * v + kPartner] = p1 * c[v] + p0 * s[v];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        x[v] = (T)z[v];
        y[v] = (T)z[V + v];
      }
    }
    *(VT*)(dst + e0) = x;
    *(VT*)(dst + e1) = y;
  }
}

// elements of a thread's pieces: the widest of 16 bytes or less that divides the half
int width(const RopeArgs& a) {
  int v = a.bf16 ? 8 : 4;
  while ((a.rot / 2) % v != 0) v /= 2;
  return v;
}

RopeParams plan(const RopeArgs& a, int64_t* groups) {
  RopeParams p;
  p.a = a;
  p.heads = a.Hq + a.Hkv;
  const int64_t units = (int64_t)p.heads * (a.d / (2 * width(a)));  // threads' worth of work per position
  p.tr = a.d / (2 * width(a));
  while (p.tr < kThreads && p.tr < units) p.tr *= 2;
  p.rows = kThreads / p.tr;
  const int64_t tiles = (int64_t)a.B * ((a.L + p.rows - 1) / p.rows);
  // fewer workgroups than CUs: the heads are cut, down to one per thread, and each part has its own table.
  // Measured (us) cut and whole at H 32 and 32, d 128: 1 position 3.3, 3.5; 64 3.6, 3.8; 256 4.7, 4.3; B4
  // Hq40/Hkv8 L256 7.5, 6.9.
  p.hsplit = tiles < 256 ? (int)((units + p.tr - 1) / p.tr) : 1;
  *groups = tiles * p.hsplit;
  return p;
}

template <class T, int V>
void launch(const RopeParams& p, unsigned groups, hipStream_t stream) {
  const size_t lds = sizeof(float2) * p.rows * (p.a.rot / 2);
  const dim3 grid(groups), block(kThreads);
  if (p.a.d == 128) {
    if (p.a.interleaved) hipLaunchKernelGGL((cover_rope_kernel<T, V, 128, true>), grid, block, lds, stream, p);
    else hipLaunchKernelGGL((cover_rope_kernel<T, V, 128, false>), grid, block, lds, stream, p);
  } else {
    if (p.a.interleaved) hipLaunchKernelGGL((cover_rope_kernel<T, V, 64, true>), grid, block, lds, stream, p);
    else hipLaunchKernelGGL((cover_rope_kernel<T, V, 64, false>), grid, block, lds, stream, p);
  }
}

}  // namespace

bool rope_fits(const RopeArgs& a) {
  int64_t groups;
  plan(a, &groups);
  return groups < (int64_t(1) << 32) / kThreads;
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  int64_t groups;
  const RopeParams p = plan(a, &groups);
  const int v = width(a);
  if (a.bf16) {
    if (v == 8) launch<__bf16, 8>(p, (unsigned)groups, stream);
    else if (v == 4) launch<__bf16, 4>(p, (unsigned)groups, stream);
    else if (v == 2) launch<__bf16, 2>(p, (unsigned)groups, stream);
    else launch<__bf16, 1>(p, (unsigned)groups, stream);
  } else {
    if (v == 4) launch<float, 4>(p, (unsigned)groups, stream);
    else if (v == 2) launch<float, 2>(p, (unsigned)groups, stream);
    else launch<float, 1>(p, (unsigned)groups, stream);
  }
  return hipGetLastError();
}

}  // namespace cover
