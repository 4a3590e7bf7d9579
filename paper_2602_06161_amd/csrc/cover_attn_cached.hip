// COVER attention for a block of query rows against an 8-bit cache and the block's own live rows
// (prefix-cache decoding, Sec. 6.6), bf16 queries and live rows, head size 64 or 128, on gfx950.
//
// The keys of a batch row with len positions and a block of nv existing rows from o on are three
// lists, in stages of 32 keys:
//   cache   positions [0, o) and [o + nv, len): scale * code
//   seeds   the block's seed positions, gathered: scale * code; a seed row does not see its own
//   live    the block's rows that are no seeds
// and a seed row's own live key and value are one more term of its softmax, added where the partial
// results meet (the leave-one-out view of App. B.4).  Nothing else of the block's cache is read, so a
// stage's source does not change from row to row and only the two short lists need masks.
//
// One workgroup of 8 waves per 32 query rows of a key/value head (rows of all its query heads, head
// after head, so that few rows per head still fill a tile); the waves split the stages, and their
// (max, sum, O) meet in LDS.  n_split > 1: a workgroup takes one of n_split ranges of the stages and
// leaves its (O, max, sum) in fp32 in the workspace; a second kernel joins them.
//
// S^T = K Q^T and O^T += V^T P^T with 32x32x16 bf16 MFMAs, a query row in a lane pair.  A code is
// exact in bf16; its row's scale multiplies the score (K) or the weight (V) in fp32, before the
// weight is rounded to bf16 (2^-9 relative, as the weights of a bf16 attention are).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cover.h"
#include "cover_internal.h"

namespace cover {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_t;

constexpr int kTW = 8;                  // waves per workgroup
constexpr int kTQ = 32;                 // query rows per workgroup
constexpr int kStage = 32;              // keys per stage
constexpr float kInit = -1.0e30f;       // finite "nothing seen yet" max
constexpr float kLazyT = 8.0f;
constexpr float kLn2 = 0.693147180559945309f;

struct CachedParams {
  CachedArgs a;
  int group, n_qt, n_split;
  int n_wg, xcd_slots;  // workgroups of the launch, and of them per XCD
  float c2;             // scale * log2(e)
};

// LDS layouts as in the block kernel on bf16 keys: K rows with the 16-byte chunk index XOR-ed by
// row % 16 (head size 64: row / 2 % 8), V rows by 4 (row % 4) (2 (row % 4)).
template <int D>
__device__ __forceinline__ int k_swz(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int D>
__device__ __forceinline__ int v_swz(int row) { return (row & 3) << (D == 128 ? 2 : 1); }
template <int D>
__device__ __forceinline__ uint32_t k_off(int row, int c) { return row * (2 * D) + ((c ^ k_swz<D>(row)) << 4); }
template <int D>
__device__ __forceinline__ uint32_t v_off(int row, int c) { return row * (2 * D) + ((c ^ v_swz<D>(row)) << 4); }

__device__ __forceinline__ float pair_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ i16x4 v_tr(const lds_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
}

// 8 codes as bf16 (exact)
__device__ __forceinline__ bf16x8 decode(uint32_t lo, uint32_t hi) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, true);
  return bf16x8{(__bf16)a[0], (__bf16)a[1], (__bf16)b[0], (__bf16)b[1],
                (__bf16)c[0], (__bf16)c[1], (__bf16)d[0], (__bf16)d[1]};
}

// a batch row's keys, the start of its block and the block's rows that exist
struct Extent {
  int len, o, nv;
  __device__ Extent(const CachedArgs& a, int b) {
    len = a.kv_len ? min(max(a.kv_len[b], 0), a.L) : a.L;
    o = min(max(a.off ? a.off[b] : a.q_off, 0), len);
    nv = min(a.Lq, len - o);
  }
};

template <int D, bool SPLIT>
__global__ __launch_bounds__(64 * kTW, 1) void cover_attn_cached_kernel(const CachedParams p) {
  constexpr int kRow = 2 * D;         // bytes per row in LDS
  constexpr int kSB = kStage * kRow;  // bytes of one stage of K (or V)
  // per wave: a K slot and a V slot (at the end: its partial O, 32 rows of D fp32)
  __shared__ __attribute__((aligned(1024))) char sKV[kTW][2][kSB];
  __shared__ __attribute__((aligned(16))) float sScale[kTW][2][kStage];
  __shared__ uint32_t sBits[COVER_CACHED_MAX_LQ / 32];  // the block's seed rows
  __shared__ uint16_t sList[COVER_CACHED_MAX_LQ];       // and their list, ascending
  __shared__ int sCount;
  __shared__ float sM[kTW][kTQ], sL[kTW][kTQ];
  static_assert(COVER_CACHED_MAX_LQ / 32 == 64, "one word of the seed bitmap per lane");

  const CachedArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hl = lane >> 5;

  // workgroup -> (b, g, split, tile), tile fastest; consecutive ones (of one KV head) share an XCD
  const int li = (blockIdx.x & 7) * p.xcd_slots + (blockIdx.x >> 3);
  if (li >= p.n_wg) return;
  const int qt = li % p.n_qt;
  int rest = li / p.n_qt;
  const int split = SPLIT ? rest % p.n_split : 0;
  if (SPLIT) rest /= p.n_split;
  const int g = rest % a.Hkv, b = rest / a.Hkv;
  const Extent x(a, b);
  // this lane's query row: head f / Lq of the group, row f % Lq of the block
  const int n_rows = p.group * a.Lq;
  const int f = min(qt * kTQ + l32, n_rows - 1);
  const int qr = f % a.Lq;
  if (__builtin_amdgcn_ballot_w64(qt * kTQ + l32 < n_rows && qr < x.nv) == 0) return;  // no row exists

  // ---- the block's seeds: bitmap, then list ------------------------------------------------
  if (tid < 64) sBits[tid] = 0u;
  __syncthreads();
  if (a.max_seeds > 0) {
    const int ns = min(max(a.n_seed[b], 0), a.max_seeds);
    for (int t = tid; t < ns; t += 64 * kTW) {
      const int r = a.seed_idx[(int64_t)b * a.max_seeds + t] - x.o;
      if ((unsigned)r < (unsigned)x.nv) atomicOr(&sBits[r >> 5], 1u << (r & 31));
    }
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t word = sBits[lane];
    int at = __popc(word);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int v = __shfl_up(at, m);
      if (lane >= m) at += v;
    }
    if (lane == 63) sCount = at;
    at -= __popc(word);
    while (word) {
      sList[at++] = (uint16_t)(32 * lane + __ffs(word) - 1);
      word &= word - 1;
    }
  }
  __syncthreads();
  const int n_seeds = sCount;
  auto is_seed = [&](int r) -> bool { return (sBits[r >> 5] >> (r & 31)) & 1u; };

  // ---- stages ------------------------------------------------------------------------------
  const int nA1 = (x.o + kStage - 1) / kStage, nA2 = (x.len - x.o - x.nv + kStage - 1) / kStage;
  const int nB = (n_seeds + kStage - 1) / kStage, nC = (x.nv + kStage - 1) / kStage;
  const int total = nA1 + nA2 + nB + nC;
  const int per = SPLIT ? (total + p.n_split - 1) / p.n_split : total;
  const int sb = split * per, nst = max(min(total - sb, per), 0);
  const int s0 = sb + nst * wave / kTW, s1 = sb + nst * (wave + 1) / kTW;

  const int h = g * p.group + f / a.Lq;
  bf16x8 qreg[D / 16];
  {
    const __bf16* qp = (const __bf16*)a.q + b * a.q_sb + h * a.q_sh + qr * a.q_sl + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qreg[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  uint32_t vaddr[D / 32];
  {
    const int G = lane >> 4, ii = lane & 15;
    const int row = 4 * (G >> 1) + (ii >> 2);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const int col = db * 32 + 16 * (G & 1) + 4 * (ii & 3);
      vaddr[db] = v_off<D>(row, col >> 3) + ((col & 7) << 1);
    }
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
  float m = kInit, l = 0.0f;
  lds_t* const kb = (lds_t*)sKV[wave][0];
  lds_t* const vb = (lds_t*)sKV[wave][1];
  typedef __attribute__((address_space(3))) bf16x8 lds8;

  for (int st = s0; st < s1; ++st) {
    // the stage's list: 0 cache, 1 seeds, 2 live; first index and end
    int kind = 0, base = st * kStage, end = x.o;
    if (st >= nA1) {
      base = x.o + x.nv + (st - nA1) * kStage;
      end = x.len;
    }
    if (st >= nA1 + nA2) {
      kind = 1;
      base = (st - nA1 - nA2) * kStage;
      end = n_seeds;
    }
    if (st >= nA1 + nA2 + nB) {
      kind = 2;
      base = (st - nA1 - nA2 - nB) * kStage;
      end = x.nv;
    }
    // stage -> LDS: rows past the end repeat the last one
    if (kind < 2) {
      constexpr int kCh = D / 16, kRPL = 64 / kCh;  // 16-byte chunks of codes per row, rows per load
      const int c = lane % kCh;
#pragma unroll
      for (int j = 0; j < kStage / kRPL; ++j) {
        const int row = kRPL * j + lane / kCh;
        int pos = min(base + row, end - 1);
        if (kind == 1) pos = x.o + sList[pos];
        const int64_t src = b * a.c_sb + g * a.c_sh + pos * a.c_sl + 16 * c;
        const u32x4 k = *(const u32x4*)((const char*)a.kc + src);
        u32x4 v = *(const u32x4*)((const char*)a.vc + src);
        const int64_t ss = b * a.s_sb + g * a.s_sh + pos;
        const float ks = a.ks[ss], vs = a.vs[ss];
        // a value row that stands for NaN gives NaN through its scale; its codes would reach
        // the one row that does not see it
        if (!__builtin_isfinite(vs)) v = u32x4{0u, 0u, 0u, 0u};
        if (c == 0) {
          sScale[wave][0][row] = ks;
          sScale[wave][1][row] = vs;
        }
        *(lds8*)(kb + k_off<D>(row, 2 * c)) = decode(k[0], k[1]);
        *(lds8*)(kb + k_off<D>(row, 2 * c + 1)) = decode(k[2], k[3]);
        *(lds8*)(vb + v_off<D>(row, 2 * c)) = decode(v[0], v[1]);
        *(lds8*)(vb + v_off<D>(row, 2 * c + 1)) = decode(v[2], v[3]);
      }
    } else {
      constexpr int kCh = D / 8, kRPL = 64 / kCh;
      const int c = lane % kCh;
#pragma unroll
      for (int j = 0; j < kStage / kRPL; ++j) {
        const int row = kRPL * j + lane / kCh;
        const int r = min(base + row, end - 1);
        u32x4 k = *(const u32x4*)((const __bf16*)a.k_live + b * a.k_sb + g * a.k_sh + r * a.k_sl + 8 * c);
        u32x4 v = *(const u32x4*)((const __bf16*)a.v_live + b * a.v_sb + g * a.v_sh + r * a.v_sl + 8 * c);
        // a seed's live row is for that row alone, which adds it at the end
        if (is_seed(r)) v = u32x4{0u, 0u, 0u, 0u};
        if (c == 0) {
          sScale[wave][0][row] = 1.0f;
          sScale[wave][1][row] = 1.0f;
        }
        *(__attribute__((address_space(3))) u32x4*)(kb + k_off<D>(row, c)) = k;
        *(__attribute__((address_space(3))) u32x4*)(vb + v_off<D>(row, c)) = v;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const lds8*)(kb + k_off<D>(l32, 2 * ks + hl)), qreg[ks], sc, 0, 0, 0);
    // register r holds key base + 8 (r / 4) + 4 hl + r % 4 of the lane's query row
    float mx = kInit;
    uint32_t hidden = 0u;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = 8 * (r >> 2) + 4 * hl + (r & 3);
      const int e = base + key;
      float t = sc[r] * (sScale[wave][0][key] * p.c2);
      bool hide = e >= end;
      if (!hide && kind == 1) hide = sList[e] == qr;
      if (!hide && kind == 2) hide = is_seed(e);
      if (hide) {
        t = -INFINITY;
        hidden |= 1u << r;
      }
      sc[r] = t;
      mx = __builtin_fmaxf(mx, t);
    }
    mx = pair_max(mx);
    if (__builtin_amdgcn_ballot_w64(mx > m + kLazyT)) {
      const float mn = __builtin_fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[db] *= alpha;
      m = mn;
    }
    bf16x8 pk[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = 8 * kk + e;
        const float pr = __builtin_amdgcn_exp2f(sc[r] - m);
        l += pr;
        const float pv = pr * sScale[wave][1][8 * (r >> 2) + 4 * hl + (r & 3)];
        pk[kk][e] = (__bf16)((hidden >> r) & 1u ? 0.0f : pv);
      }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const lds_t* vp = vb + vaddr[db] + kk * 16 * kRow;
        const bf16x8 va = __builtin_bit_cast(
            bf16x8, __builtin_shufflevector(v_tr(vp), v_tr(vp + 8 * kRow), 0, 1, 2, 3, 4, 5, 6, 7));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pk[kk], o[db], 0, 0, 0);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // ---- merge: every wave's (max, sum, O) through LDS ---------------------------------------
  // row l32, 16-byte chunk c (dims 4 c .. 4 c + 3) at byte 4 D l32 + 16 (c ^ l32 % (D / 4))
  constexpr int kOM = D / 4 - 1;
  const float lt = pair_sum(l);
  if (hl == 0) {
    sM[wave][l32] = m;
    sL[wave][l32] = lt;
  }
  {
    lds_t* const ob = (lds_t*)sKV[wave][0] + 4 * D * l32;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const int c = 8 * db + 2 * gq + hl;
        *(__attribute__((address_space(3))) f32x4*)(ob + ((c ^ (l32 & kOM)) << 4)) =
            f32x4{o[db][4 * gq], o[db][4 * gq + 1], o[db][4 * gq + 2], o[db][4 * gq + 3]};
      }
  }
  __syncthreads();
  // wave w finishes rows kFin w + fq (lane group fq of 16), lane dims kE fj .. kE fj + kE - 1
  constexpr int kFin = kTQ / kTW, kE = D / 16;
  typedef __bf16 out_t __attribute__((ext_vector_type(kE)));
  const int fq = lane >> 4, fj = lane & 15;
  const int row = kFin * wave + fq, ff = qt * kTQ + row;
  const int fr = ff % a.Lq, fh = g * p.group + ff / a.Lq;
  const bool ok = ff < n_rows && fr < x.nv;
  const bool seed = ok && split == 0 && is_seed(fr);
  float acc[kE], den = 0.0f, M = kInit, t = -INFINITY;
#pragma unroll
  for (int e = 0; e < kE; ++e) acc[e] = 0.0f;
  out_t vd = {};
  if (seed) {  // (uniform over a row's 16 lanes)
    const out_t qv = *(const out_t*)((const __bf16*)a.q + b * a.q_sb + fh * a.q_sh + fr * a.q_sl + kE * fj);
    const out_t kd = *(const out_t*)((const __bf16*)a.k_live + b * a.k_sb + g * a.k_sh + fr * a.k_sl + kE * fj);
    vd = *(const out_t*)((const __bf16*)a.v_live + b * a.v_sb + g * a.v_sh + fr * a.v_sl + kE * fj);
    float dot = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) dot = __builtin_fmaf((float)qv[e], (float)kd[e], dot);
#pragma unroll
    for (int s = 8; s >= 1; s >>= 1) dot += __shfl_xor(dot, s);
    t = dot * p.c2;
    M = __builtin_fmaxf(M, t);
  }
#pragma unroll
  for (int w = 0; w < kTW; ++w) M = __builtin_fmaxf(M, sM[w][row]);
#pragma unroll
  for (int w = 0; w < kTW; ++w) {
    const float s = __builtin_amdgcn_exp2f(sM[w][row] - M);
    den = __builtin_fmaf(sL[w][row], s, den);
    const lds_t* rb = (const lds_t*)sKV[w][0] + 4 * D * row;
#pragma unroll
    for (int e = 0; e < kE; e += 4) {
      const f32x4 v = *(const __attribute__((address_space(3))) f32x4*)(rb + ((((kE * fj + e) / 4) ^ (row & kOM)) << 4));
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[e + u] = __builtin_fmaf(s, v[u], acc[e + u]);
    }
  }
  if (seed) {
    const float s = __builtin_amdgcn_exp2f(t - M);
    den += s;
#pragma unroll
    for (int e = 0; e < kE; ++e) acc[e] = __builtin_fmaf(s, (float)vd[e], acc[e]);
  }
  if (!ok) return;
  const int64_t bh = (int64_t)b * a.Hq + fh;
  if constexpr (SPLIT) {
    float* rec = a.workspace + ((bh * p.n_split + split) * a.Lq + fr) * (D + 4);
#pragma unroll
    for (int e = 0; e < kE; e += 4) *(f32x4*)(rec + kE * fj + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
    if (fj == 0) {
      rec[D] = M;
      rec[D + 1] = den;
    }
  } else {
    const float inv = 1.0f / den;
    out_t ob;
#pragma unroll
    for (int e = 0; e < kE; ++e) ob[e] = (__bf16)(acc[e] * inv);
    *(out_t*)((__bf16*)a.out + b * a.o_sb + fh * a.o_sh + fr * a.o_sl + kE * fj) = ob;
    if (a.lse && fj == 0) a.lse[bh * a.Lq + fr] = (M + __builtin_amdgcn_logf(den)) * kLn2;
  }
}

// One wave per query row: the ranges' (O, max, sum) joined, in their order.
template <int D>
__global__ __launch_bounds__(256) void cover_attn_cached_join_kernel(const CachedParams p) {
  const CachedArgs& a = p.a;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);  // over B * Hq * Lq
  if (row >= (int64_t)a.B * a.Hq * a.Lq) return;
  const int64_t bh = row / a.Lq;
  const int r = (int)(row % a.Lq), b = (int)(bh / a.Hq), h = (int)(bh % a.Hq);
  const Extent x(a, b);
  if (r >= x.nv) return;
  const float* rec = a.workspace + (bh * p.n_split * a.Lq + r) * (D + 4);
  const int64_t step = (int64_t)a.Lq * (D + 4);
  constexpr int kE = D / 64, kChunk = 8;  // ranges in chunks whose loads are all issued first
  float M = kInit, den = 0.0f, acc[kE] = {};
  for (int s0 = 0; s0 < p.n_split; s0 += kChunk) {
    float ms[kChunk], ls[kChunk], v[kChunk][kE];
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      ms[u] = kInit;
      ls[u] = 0.0f;
#pragma unroll
      for (int e = 0; e < kE; ++e) v[u][e] = 0.0f;
      if (s0 + u < p.n_split) {
        const float* q = rec + (s0 + u) * step;
        ms[u] = q[D];
        ls[u] = q[D + 1];
#pragma unroll
        for (int e = 0; e < kE; ++e) v[u][e] = q[kE * lane + e];
      }
    }
    float Mn = M;
#pragma unroll
    for (int u = 0; u < kChunk; ++u) Mn = __builtin_fmaxf(Mn, ms[u]);
    const float al = __builtin_amdgcn_exp2f(M - Mn);
    den *= al;
#pragma unroll
    for (int e = 0; e < kE; ++e) acc[e] *= al;
    M = Mn;
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      const float w = __builtin_amdgcn_exp2f(ms[u] - M);
      den = __builtin_fmaf(ls[u], w, den);
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[e] = __builtin_fmaf(v[u][e], w, acc[e]);
    }
  }
  const float inv = 1.0f / den;
  __bf16* op = (__bf16*)a.out + b * a.o_sb + h * a.o_sh + r * a.o_sl + kE * lane;
#pragma unroll
  for (int e = 0; e < kE; ++e) op[e] = (__bf16)(acc[e] * inv);
  if (a.lse && lane == 0) a.lse[row] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

int64_t tiles_of(const CachedArgs& a) {
  return (int64_t)a.B * a.Hkv * (((int64_t)(a.Hq / a.Hkv) * a.Lq + kTQ - 1) / kTQ);
}

}  // namespace

// About 256 workgroups of at least 512 keys each (64 per wave).
int attn_cached_splits(int B, int Hq, int Hkv, int L, int Lq) {
  CachedArgs a = {};
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lq = Lq;
  const int64_t n = std::min<int64_t>(256 / std::max<int64_t>(tiles_of(a), 1), L / 512);
  return (int)std::max<int64_t>(1, std::min<int64_t>(n, 256));
}

bool attn_cached_fits(const CachedArgs& a) {
  return tiles_of(a) * a.n_split <= (int64_t(1) << 23) - 8 &&
         (int64_t)a.B * a.Hq * a.Lq <= (int64_t(1) << 26) - 4;
}

hipError_t launch_attn_cached(const CachedArgs& a, hipStream_t stream) {
  CachedParams p;
  p.a = a;
  p.group = a.Hq / a.Hkv;
  p.n_qt = (p.group * a.Lq + kTQ - 1) / kTQ;
  p.n_split = a.n_split;
  p.c2 = a.scale * 1.44269504088896341f;
  p.n_wg = (int)(tiles_of(a) * p.n_split);
  p.xcd_slots = (p.n_wg + 7) / 8;
  const dim3 grid(8u * p.xcd_slots), block(64 * kTW);
  if (p.n_split == 1) {
    if (a.d == 128) hipLaunchKernelGGL((cover_attn_cached_kernel<128, false>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((cover_attn_cached_kernel<64, false>), grid, block, 0, stream, p);
    return hipGetLastError();
  }
  if (a.d == 128) hipLaunchKernelGGL((cover_attn_cached_kernel<128, true>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((cover_attn_cached_kernel<64, true>), grid, block, 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 rows((unsigned)(((int64_t)a.B * a.Hq * a.Lq + 3) / 4));
  if (a.d == 128) hipLaunchKernelGGL((cover_attn_cached_join_kernel<128>), rows, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((cover_attn_cached_join_kernel<64>), rows, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace cover
