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
// A workgroup of 8 waves takes 32 or 64 query rows of a key/value head (rows of all its query heads, head
// after head, so that few rows per head still fill a tile); the waves split the stages, and their
// (max, sum, O) meet in LDS.  n_split > 1: a workgroup takes one of n_split ranges of the stages and
// leaves its (O, max, sum) in fp32 in the workspace; a second kernel joins them.  Where 128 rows per
// workgroup fill the chip, each of 4 waves has 32 rows of its own and all keys instead.
//
// S^T = K Q^T and O^T += V^T P^T with 32x32x16 MFMAs, a query row in a lane pair.  A code is exact in
// bf16 and in fp16; its row's scale multiplies the score (K) or the weight (V) in fp32.  The weights are
// then rounded to fp16 (2^-11 relative, against 2^-8 of bf16, whose rounding alone would add as much noise
// as the output's own: 0.0024 instead of 0.0017 of the output's norm).  Its range suffices since V's scales
// are taken in units of a power of two near them, and weights below 2^-28 of a row's largest do not count.
// Live rows are bf16, so their weights go in two bf16 parts.  Sums, maxima and partial results are fp32.
//
// Bounds and measured times (launches back to back): with one row per sequence or few, the chain of one
// launch (lengths, loads from HBM, 1 to 14 stages per wave, merge) and the join: B1 Hq32/Hkv8 L8192, 1 row
// 12.0 us (17 MB, 1.45 TB/s), B1 H32 L1024, 64 rows 12.7 us; with many sequences of few rows HBM: B8 H32
// L4096, 32 rows 57 us (4.95 TB/s); with many rows the issue of two waves per SIMD, which decode K and V for
// every 32 rows and weigh beside the matrix cores (busy 0.29 of the time, the vector ALUs 0.51): B8 H32 L2048,
// 256 rows 95.5 us (720 TFLOP/s), B1 Hq28/Hkv4 L32768, 32 rows 30.6 us (490).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cover.h"
#include "cover_internal.h"

namespace cover {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_t;
typedef __attribute__((address_space(1))) const char gmem_t;
typedef __attribute__((address_space(3))) float ldsf;
typedef __attribute__((address_space(3))) f32x4 ldsf4;
typedef __attribute__((address_space(3))) bf16x8 lds8;
typedef __attribute__((address_space(3))) u32x4 lds16;

constexpr int kTW = 8;                  // waves per workgroup
constexpr int kRW = 4;                  // the same where each has query rows of its own
constexpr int kStage = 32;              // keys per stage
constexpr float kInit = -3.402823466e38f;  // "nothing seen yet": the lowest number, which no score is below
constexpr float kStart = 3.0f, kMost = 9.0f;  // log2 of a row's largest weight, where its maximum is set and at most
constexpr float kLeast = 0x1p-30f;             // least power of two that V's scales are taken relative to
constexpr float kLn2 = 0.693147180559945309f;

// n / d for 0 <= n < 2^24, 1 <= d <= 2^24: m = floor(2^s / d) + 1 with 2^(s - 24) >= d, so that
// n (m d - 2^s) < 2^s (an integer division is 20 to 40 instructions, and the prologue needs several)
struct Divisor {
  uint32_t d, m, s;
};
__device__ __forceinline__ int div(int n, const Divisor& v) { return (int)(((uint64_t)(uint32_t)n * v.m) >> v.s); }

struct CachedParams {
  CachedArgs a;
  int group, n_split;
  Divisor n_qt, splits, heads, lq;  // tiles per head, n_split, Hkv, Lq
  int n_wg, xcd_slots;              // workgroups of the launch, and of them per XCD
  int spread;                       // heads (and ranges) in turn over the XCDs
  int wide;                         // code rows too far apart for 32-bit offsets in a stage
  float c2;                         // scale * log2(e)
};

// LDS layouts.  Codes: rows of D bytes whose 16-byte chunk index is XOR-ed so that the 32 rows of one
// K operand read, and the 16 rows x 32 bytes of one transposing V read, cover all banks evenly.  Live
// rows in bf16: as in the block kernel, K by row % 16 (head size 64: row / 2 % 8), V by 4 (row % 4)
// (2 (row % 4)).
template <int D>
__device__ __forceinline__ int kc_swz(int row) { return D == 128 ? ((row >> 1) & 7) : ((row >> 2) & 3); }
template <int D>
__device__ __forceinline__ int vc_swz(int row) { return D == 128 ? ((row >> 1) & 3) << 1 : ((row >> 2) & 1) << 1; }
template <int D>
__device__ __forceinline__ int k_swz(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int D>
__device__ __forceinline__ int v_swz(int row) { return (row & 3) << (D == 128 ? 2 : 1); }
template <int D>
__device__ __forceinline__ uint32_t k_off(int row, int c) { return row * (2 * D) + ((c ^ k_swz<D>(row)) << 4); }

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

__device__ __forceinline__ i32x2 v_tr8(const lds_t* p) {
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p);
}

// 8 codes as bf16 (exact)
__device__ __forceinline__ bf16x8 decode(uint32_t lo, uint32_t hi) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ f16x8 decode16(uint32_t lo, uint32_t hi) {  // in fp16, exact too
  const uint32_t x[4] = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true))};
  return __builtin_bit_cast(f16x8, x);
}
// Global -> LDS loads: lane l's 16 bytes (4 for the dword form) land at LDS byte lds + 16 l (+ 4 l);
// lds is wave-uniform.  The compiler does not track them: every read of their data follows an
// explicit vmcnt wait of the issuing wave.  A wave's loads land in issue order.  The nop is the wait
// state that a load to LDS needs behind a write of M0.
__device__ __forceinline__ void dma16(uint32_t lds, gmem_t* addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(lds), "v"((uint64_t)addr) : "memory", "m0");
}
__device__ __forceinline__ void dma16s(uint32_t lds, gmem_t* base, uint32_t voff) {  // uniform base
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void dma4(uint32_t lds, gmem_t* addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :: "s"(lds), "v"((uint64_t)addr) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N of this wave's loads are in flight
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
// x, whose later tests the compiler keeps behind the branch that they are in
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t lds_addr(const lds_t* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p);
}

// The power of two at or below a scale (not negative), and at or below the largest finite one of the lanes' scales,
// for units of V's scales: the scales in them are below kOver, so that a weight (at most 2^kMost) times one is in
// fp16's range.
constexpr float kOver = 64.0f;
__device__ __forceinline__ float power_at(uint32_t bits) {
  const uint32_t e = bits & 0x7f800000u, least = __float_as_uint(kLeast), most = __float_as_uint(0x1p126f);
  return __uint_as_float(e == 0x7f800000u ? least : min(max(e, least), most));  // (its reciprocal is normal)
}
__device__ __forceinline__ float power_of(float scale) {
  uint32_t top = __builtin_isfinite(scale) ? __float_as_uint(scale) : 0u;
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x121, 0xf, 0xf, false));  // within 16 lanes:
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x122, 0xf, 0xf, false));  // rotated by 1, 2,
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x124, 0xf, 0xf, false));  // 4
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x128, 0xf, 0xf, false));  // and 8
  top = max(max((uint32_t)__builtin_amdgcn_readlane((int)top, 0), (uint32_t)__builtin_amdgcn_readlane((int)top, 16)),
            max((uint32_t)__builtin_amdgcn_readlane((int)top, 32), (uint32_t)__builtin_amdgcn_readlane((int)top, 48)));
  return power_at(top);
}
// the reciprocal of a power of two
__device__ __forceinline__ float over_of(float power) { return __uint_as_float(0x7f000000u - __float_as_uint(power)); }

// half kk of the weights of live rows in two bf16 parts, what the first leaves in the second
__device__ __forceinline__ void two_parts(const f32x16& w, int kk, float mul, bf16x8& hi, bf16x8& lo) {
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const float x = w[8 * kk + r] * mul;
    hi[r] = (__bf16)x;
    lo[r] = (__bf16)(x - (float)hi[r]);
  }
}

// The kernel's parameters, read where they are used: what only the start or the end needs would otherwise hold
// scalar registers (or be spilled) all the way.
__device__ __forceinline__ const CachedParams& late() {
  auto k = (const __attribute__((address_space(4))) CachedParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(k));
  return *(const CachedParams*)k;
}

// A stage's scores (register r holds key 8 (r / 4) + 4 hl + r % 4 of the lane's query row) to weights in
// place: times the keys' scales ks (c2 included), `hidden` ones (where masked) to zero, against a maximum that
// is set kStart below the first stage's and follows where a weight passes 2^kMost; l sums them.
// S stages at a time: sc[t * S + s] are the scores of row tile t and stage s.  ratio: O's old units in its new.
template <int D, int R, int S>
__device__ __forceinline__ void weigh(f32x16 (&sc)[R * S], const f32x4 (&ks)[S][4], bool masked,
                                      const uint32_t (&hidden)[R * S], float ratio, float (&m)[R], float (&l)[R],
                                      f32x16 (&o)[R][D / 32]) {
#pragma unroll
  for (int t = 0; t < R; ++t)
    if (__builtin_amdgcn_ballot_w64(m[t] == kInit)) {  // a row that has seen nothing
      float top = kInit;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const uint32_t h = opaque(masked ? hidden[t * S + s] : 0u);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          top = __builtin_fmaxf(top, (h >> r) & 1u ? kInit : sc[t * S + s][r] * ks[s][r >> 2][r & 3]);
      }
      // (a score's product is unrounded in the difference below, so the maximum starts below it by more than its rounding)
      top = pair_max(top);
      top = __builtin_fmaxf(top - __builtin_fmaxf(kStart, __builtin_fabsf(top) * 0x1p-22f), kInit);
      m[t] = m[t] == kInit ? top : m[t];
    }
#pragma unroll
  for (int t = 0; t < R * S; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[t][r] = __builtin_fmaf(sc[t][r], ks[t % S][r >> 2][r & 3], -m[t / S]);
  if (masked) {
#pragma unroll
    for (int t = 0; t < R * S; ++t) {
      const uint32_t h = opaque(hidden[t]);
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[t][r] = (h >> r) & 1u ? -INFINITY : sc[t][r];
    }
  }
  float mx[R], most = kInit;
#pragma unroll
  for (int t = 0; t < R; ++t) {
    mx[t] = kInit;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx[t] = __builtin_fmaxf(mx[t], sc[t * S + s][r]);
    most = __builtin_fmaxf(most, mx[t]);
  }
  if (__builtin_amdgcn_ballot_w64(most > kMost || ratio != 1.0f)) {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const float up = pair_max(mx[t]) > kMost ? pair_max(mx[t]) - kStart : 0.0f, alpha = __builtin_amdgcn_exp2f(-up);
      l[t] *= alpha;
      const float both = alpha * ratio;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[t][db] *= both;
      m[t] += up;
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[t * S + s][r] -= up;
    }
  }
#pragma unroll
  for (int t = 0; t < R * S; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[t][r] = __builtin_amdgcn_exp2f(sc[t][r]);
      l[t / S] += sc[t][r];
    }
}

// a lane's registers of the keys in a stage's mask, and the keys at or past n
__device__ __forceinline__ uint32_t registers_of(uint32_t keys, int hl) {
  const uint32_t k = keys >> (4 * hl);
  return (k & 0xfu) | ((k >> 4) & 0xf0u) | ((k >> 8) & 0xf00u) | ((k >> 12) & 0xf000u);
}
__device__ __forceinline__ uint32_t past(int n) { return n >= kStage ? 0u : ~0u << max(n, 0); }

// This workgroup's place in (b, g, range, tile), tile fastest.  The tiles of a head (and range) read the same
// keys and share an XCD, so its L2.  Heads take XCDs in turn where that gives each as many, since rows of a
// batch differ in length (B8 H32 L1024..2048 Lq256: 96 us with a batch row per XCD, 87 so), else by the slot.
__device__ __forceinline__ int place_of(const CachedParams& p) {
  const int j = blockIdx.x >> 3, xcd = blockIdx.x & 7;
  if (!p.spread) return xcd * p.xcd_slots + j;
  const int unit = uniform(div(j, p.n_qt));
  return j + (7 * unit + xcd) * (int)p.n_qt.d;
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

template <int D, int R, bool SPLIT>
__global__ __launch_bounds__(64 * kTW, R * D == 64 ? 4 : 2) void cover_attn_cached_kernel(const CachedParams p) {
  constexpr int kTQ = 32 * R;                // query rows per workgroup
  constexpr int kSB = kStage * D;            // bytes of one stage of K (or V) codes
  constexpr int kCh = D / 16, kRPL = 64 / kCh;  // 16-byte chunks of codes per row, rows per load
  constexpr int kNK = kStage / kRPL, kNL = 2 * kNK + 1;  // loads of K (or V) of a stage, all its loads
  constexpr int kLC = D / 8, kLR = 64 / kLC, kNV = kStage / kLR;  // the same of live rows in bf16
  constexpr bool kQReg = R * D <= 128;       // Q's operands stay in registers
  // per wave: two slots of K and V codes, or one of live rows (at the end: a partial O, 32 rows of D
  // fp32); the two slots' scales
  __shared__ __attribute__((aligned(1024))) char sKV[kTW][4 * kSB];
  __shared__ __attribute__((aligned(1024))) char sQ[kTQ * 2 * D];
  __shared__ __attribute__((aligned(16))) float sScale[kTW][2][2][kStage];
  __shared__ uint32_t sBits[COVER_CACHED_MAX_LQ / 32];  // the block's seed rows
  __shared__ uint16_t sList[COVER_CACHED_MAX_LQ];       // and their list, ascending
  // the call's list of seeds, and at the end the maxima and sums
  __shared__ __attribute__((aligned(16))) char sShared[64 * kTW * 4 * R];
  int32_t* const sSeeds = (int32_t*)sShared;
  float (*const sM)[kTQ] = (float (*)[kTQ])sShared;
  float (*const sL)[kTQ] = sM + kTW;
  __shared__ float sPower[kTW];
  static_assert(COVER_CACHED_MAX_LQ / 32 == 64 && 2 * kTW * kTQ * 4 <= (int)sizeof(sShared), "what shares LDS fits");

  const CachedArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hl = lane >> 5;

  const int li = place_of(p);
  if (li >= p.n_wg) return;
  int rest = uniform(div(li, p.n_qt));
  const int qt = li - rest * (int)p.n_qt.d;
  int split = 0;
  if constexpr (SPLIT) {
    const int next = uniform(div(rest, p.splits));
    split = rest - next * p.n_split;
    rest = next;
  }
  const int b = uniform(div(rest, p.heads)), g = rest - b * a.Hkv;
  Extent x(a, b);
  x.len = uniform(x.len);
  x.o = uniform(x.o);
  x.nv = uniform(x.nv);
  // this lane's query rows: head f / Lq of the group, row f % Lq of the block
  const int n_rows = p.group * a.Lq;
  int qr[R];
  bool any = false;
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const int ft = qt * kTQ + 32 * t + l32, f = min(ft, n_rows - 1);
    qr[t] = f - div(f, p.lq) * a.Lq;
    any |= ft < n_rows && qr[t] < x.nv;
  }
  if (__builtin_amdgcn_ballot_w64(any) == 0) return;  // no row exists

  // ---- stages: this workgroup's range of them, its cache stages and short ones -----------------------
  // (as many stages of seeds as the list's length asks for: those that its distinct seeds in the block leave empty are
  // skipped once the seeds are known)
  const int ns = a.max_seeds > 0 ? uniform(min(max(a.n_seed[b], 0), a.max_seeds)) : 0;
  const int nA1 = (x.o + kStage - 1) / kStage, nA2 = (x.len - x.o - x.nv + kStage - 1) / kStage;
  const int nA = nA1 + nA2, nC = (x.nv + kStage - 1) / kStage, nB = min((ns + kStage - 1) / kStage, nC);
  const int total = nA + nB + nC;
  const int per = SPLIT ? uniform(div(total + p.n_split - 1, p.splits)) : total;
  const int w0 = min(split * per, total), w1 = min(w0 + per, total);
  const int e0 = max(w0 - nA, 0), e1 = max(w1 - nA, 0);
  // cache stages in eight runs, the longer ones first; short stages dealt out from the first shorter one on
  const int first_cache = min(w0, nA), n_cache = min(w1, nA) - first_cache, longer = n_cache % kTW;
  const int a0 = first_cache + n_cache / kTW * wave + min(wave, longer);
  const int nW = n_cache / kTW + (wave < longer ? 1 : 0);
  const int seeds0 = e0 + ((wave - longer) & (kTW - 1));
  auto stages_from = [&](int first, int end) { return first < end ? (end - first + kTW - 1) / kTW : 0; };
  const int nS = stages_from(seeds0, min(e1, nB));
  const int live0 = seeds0 + nS * kTW;  // this wave's first stage of live rows, if below e1

  const char* const kcb = (const char*)a.kc + b * a.c_sb + g * a.c_sh;
  const char* const vcb = (const char*)a.vc + b * a.c_sb + g * a.c_sh;
  const float* const scb = (hl ? a.vs : a.ks) + (b * a.s_sb + g * a.s_sh);  // lanes 0-31: K's scales, 32-63: V's
  lds_t* const slots = (lds_t*)sKV[wave];
  ldsf* const scales = (ldsf*)sScale[wave][0][0];
  const uint32_t slot0 = lds_addr(slots), scale0 = lds_addr((lds_t*)scales);
  // load j of a stage covers stage rows kRPL j + lane / kCh at physical chunk lane % kCh; the source
  // chunk is the one that the swizzle puts there, the same for loads j and j + 2
  uint32_t offK[2], offV[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = kRPL * j + lane / kCh, pc = lane % kCh;
    offK[j] = (uint32_t)(row * (uint32_t)a.c_sl) + ((pc ^ kc_swz<D>(row)) << 4);
    offV[j] = (uint32_t)(row * (uint32_t)a.c_sl) + ((pc ^ vc_swz<D>(row)) << 4);
  }
  // (what only the rarer loads need is computed from opaque(lane) there, or it would be kept in registers)
  const int past_block = x.o + x.nv - nA1 * kStage;  // from a stage's place in the list to its first key
  // cache stage st into slot s; rows past the end repeat the last one
  auto issue_cache = [&](int st, int s) __attribute__((always_inline)) {
    const int first = st * kStage + (st < nA1 ? 0 : past_block);
    const int end = st < nA1 ? x.o : x.len;
    const uint32_t kd = slot0 + 2 * kSB * s, vd = kd + kSB;
    if (first + kStage <= end && !p.wide) {
      const int64_t at = (int64_t)((uint64_t)(uint32_t)first * (uint32_t)a.c_sl);
      gmem_t* const kp = (gmem_t*)(kcb + at);
      gmem_t* const vp = (gmem_t*)(vcb + at);
#pragma unroll
      for (int j = 0; j < kNK; ++j) dma16s(kd + 1024 * j, kp + (j >> 1) * 2 * kRPL * a.c_sl, offK[j & 1]);
#pragma unroll
      for (int j = 0; j < kNK; ++j) dma16s(vd + 1024 * j, vp + (j >> 1) * 2 * kRPL * a.c_sl, offV[j & 1]);
      dma4(scale0 + 256 * s, (gmem_t*)(scb + (first + l32)));
    } else {
      const int ln = opaque(lane);
#pragma unroll
      for (int j = 0; j < kNK; ++j) {
        const int row = kRPL * j + ln / kCh, pc = ln % kCh;
        const int64_t at = min(first + row, end - 1) * a.c_sl;
        dma16(kd + 1024 * j, (gmem_t*)(kcb + at + ((pc ^ kc_swz<D>(row)) << 4)));
        dma16(vd + 1024 * j, (gmem_t*)(vcb + at + ((pc ^ vc_swz<D>(row)) << 4)));
      }
      dma4(scale0 + 256 * s, (gmem_t*)(scb + min(first + (ln & 31), end - 1)));
    }
  };

  // ---- the first loads: the call's seeds, Q, this wave's first two stages of the cache ---------------
  if (ns > 0 && tid < a.max_seeds)
    dma4(lds_addr((lds_t*)(sSeeds + 64 * wave)), (gmem_t*)(a.seed_idx + (int64_t)b * a.max_seeds + tid));
#pragma unroll
  for (int t = 0; t < R; ++t)  // load w of a tile covers its rows kLR w + lane / kLC
    if (32 / kLR == kTW || wave < 32 / kLR) {
      const int row = 32 * t + kLR * wave + lane / kLC, pc = lane % kLC;
      const int f = min(qt * kTQ + row, n_rows - 1), fh = div(f, p.lq);
      const __bf16* src = (const __bf16*)a.q + b * a.q_sb + (g * p.group + fh) * a.q_sh + (f - fh * a.Lq) * a.q_sl;
      dma16(lds_addr((lds_t*)sQ) + 2 * D * (32 * t + kLR * wave), (gmem_t*)((const char*)src + ((pc ^ k_swz<D>(row)) << 4)));
    }
  if (nW > 0) issue_cache(a0, 0);
  if (tid < 64) sBits[tid] = 0u;
  f32x16 o[R][D / 32];
  float m[R], l[R];
#pragma unroll
  for (int t = 0; t < R; ++t) {
    m[t] = kInit;
    l[t] = 0.0f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][db][r] = 0.0f;
      asm volatile("" : "+v"(o[t][db]));  // here, while the loads are under way
    }
  }
  if (nW > 0) wait_loads<kNL>();  // the seeds and Q have landed
  else wait_loads<0>();
  __syncthreads();
  if (nW > 1) issue_cache(a0 + 1, 1);

  // ---- the block's seeds: bitmap, their list, and this lane's rows' places in it ---------------------
  int n_seeds = 0, my_seed[R];
#pragma unroll
  for (int t = 0; t < R; ++t) my_seed[t] = -1;
  if (ns > 0) {
    for (int t = tid; t < ns; t += 64 * kTW) {
      const int r = (t < 64 * kTW ? sSeeds[t] : a.seed_idx[(int64_t)b * a.max_seeds + t]) - x.o;
      if ((unsigned)r < (unsigned)x.nv) atomicOr(&sBits[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int w = 0; w < nC; ++w) n_seeds += __popc(sBits[w]);
    n_seeds = __builtin_amdgcn_readfirstlane(n_seeds);
    if (nS > 0) {  // only waves that gather seeds need the list: each of them writes all of it, the same
      int before = 0;
      for (int w = 0; w < nC; ++w) {
        const uint32_t word = sBits[w];
        const int r = 32 * w + l32, at = before + __popc(word & ((1u << l32) - 1u));
        if (hl == 0 && ((word >> l32) & 1u)) sList[at] = (uint16_t)r;
#pragma unroll
        for (int t = 0; t < R; ++t)
          if (qr[t] >> 5 == w && ((word >> (qr[t] & 31)) & 1u))
            my_seed[t] = before + __popc(word & ((1u << (qr[t] & 31)) - 1u));
        before += __popc(word);
      }
      wait_lds();
    }
  }
  const int n8 = nW + stages_from(seeds0, min(e1, (n_seeds + kStage - 1) / kStage));  // this wave's stages of codes
  auto is_seed = [&](int r) -> bool { return n_seeds > 0 && ((sBits[r >> 5] >> (r & 31)) & 1u); };
  // stage e of the seeds, gathered, into slot s
  auto issue_seeds = [&](int e, int s) __attribute__((always_inline)) {
    const int ln = opaque(lane);
    auto pos_of = [&](int i) { return x.o + (int)sList[min(e * kStage + i, n_seeds - 1)]; };
#pragma unroll
    for (int j = 0; j < kNK; ++j) {
      const int row = kRPL * j + ln / kCh, pc = ln % kCh;
      const int64_t at = pos_of(row) * a.c_sl;
      dma16(slot0 + 2 * kSB * s + 1024 * j, (gmem_t*)(kcb + at + ((pc ^ kc_swz<D>(row)) << 4)));
      dma16(slot0 + 2 * kSB * s + kSB + 1024 * j, (gmem_t*)(vcb + at + ((pc ^ vc_swz<D>(row)) << 4)));
    }
    dma4(scale0 + 256 * s, (gmem_t*)(scb + pos_of(ln & 31)));
  };
  // K (or V) of live stage e into a slot: bf16 rows, as the block kernel lays them out
  auto issue_live = [&](int e, int s, bool v) __attribute__((always_inline)) {
    const CachedArgs& z = late().a;
    const char* const src = v ? (const char*)((const __bf16*)z.v_live + b * z.v_sb + g * z.v_sh)
                              : (const char*)((const __bf16*)z.k_live + b * z.k_sb + g * z.k_sh);
    const int64_t step = 2 * (v ? z.v_sl : z.k_sl);
    const int ln = opaque(lane);
#pragma unroll
    for (int j = 0; j < kNV; ++j) {
      const int row = kLR * j + ln / kLC, pc = ln % kLC;
      const int c = pc ^ (v ? v_swz<D>(row) : k_swz<D>(row));
      dma16(slot0 + 2 * kSB * s + 1024 * j,
            (gmem_t*)(src + min((e - nB) * kStage + row, x.nv - 1) * step + 16 * c));
    }
  };
  // what follows in slot i & 1: code stage i, or K or V of the first live stage
  const int kslot = n8 & 1;
  auto issue = [&](int i) __attribute__((always_inline)) {
    if (i < nW) issue_cache(a0 + i, i & 1);
    else if (i < n8) issue_seeds(seeds0 + (i - nW) * kTW, i & 1);
    else if (i < n8 + 2 && live0 < e1) issue_live(live0, i & 1, i > n8);
  };
  for (int i = nW; i < 2; ++i) issue(i);

  // Q (B operand): element order of step 2 u + t is dims 16 (2 u + hl) + 8 t .. + 7, so that a lane's
  // 16-byte chunk of K codes feeds two steps.  (It came through LDS: a load into registers would make the
  // compiler wait for every load in flight at its first use, inside the loop.)
  const uint32_t qa = lds_addr((lds_t*)sQ) + l32 * (2 * D) + (((2 * hl) ^ k_swz<D>(l32)) << 4);
  auto q_of = [&](uint32_t base, int t, int step) __attribute__((always_inline)) -> bf16x8 {
    return *(const lds8*)((base ^ ((4 * (step >> 1) + (step & 1)) << 4)) + t * (64 * D));
  };
  bf16x8 qreg[R][D / 16];
  if constexpr (kQReg) {
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int k = 0; k < D / 16; ++k) qreg[t][k] = q_of(qa, t, k);
  }
  auto q_at = [&](uint32_t base, int t, int step) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (kQReg) return qreg[t][step];
    else return q_of(base, t, step);
  };
  // Operand addresses of codes.  The XOR-ed chunk index makes those of a row's chunks differ by an XOR, which
  // costs less than the registers that hold them (hence opaque() where they are used).  V^T: a transposing
  // read gives lane (G = lane / 16, i = lane % 16) of 8 rows x 16 columns the 8 rows of column i, here
  // keys {0 .. 3, 8 .. 11} + 4 hl, the order of the S^T registers.
  const uint32_t ka = slot0 + l32 * D + ((hl ^ kc_swz<D>(l32)) << 4);
  uint32_t va;
  {
    const int r8 = (lane & 15) >> 1, row = (r8 & 3) + 8 * (r8 >> 2) + 4 * hl;
    va = slot0 + kSB + row * D + ((((lane >> 4) & 1) ^ vc_swz<D>(row)) << 4) + 8 * (lane & 1);
  }
  // V's scales are taken in units of a power of two, two_f, the first one's until one exceeds it kOver times; O is
  // kept in these units, and the weights stay where fp16 is fine (lanes 32-63; lanes 0-31 have K's scales)
  float two_f = 1.0f, over_f = 1.0f;
  // ---- stages of codes, two in flight: the wave's cache stages, then its stages of seeds ---------------
  for (int i = 0; i < n8; ++i) {
    const int s = i & 1;
    if (i + 1 < n8) wait_loads<kNL>();
    else if (live0 < e1) wait_loads<kNV>();
    else wait_loads<0>();
    ldsf* const sb = scales + 64 * s;
    bool masked = false;
    uint32_t hidden[R] = {};
    if (i < nW) {
      const int st = a0 + i;
      const int left = (st < nA1 ? x.o : x.len - past_block) - st * kStage;
      if (left < kStage) {
        masked = true;
#pragma unroll
        for (int t = 0; t < R; ++t) hidden[t] = registers_of(past(left), hl);
      }
    } else {
      const int first = (seeds0 + (i - nW) * kTW) * kStage;
      masked = true;
#pragma unroll
      for (int t = 0; t < R; ++t) {
        uint32_t keys = past(n_seeds - first);
        if ((unsigned)(my_seed[t] - first) < (unsigned)kStage) keys |= 1u << (my_seed[t] - first);
        hidden[t] = registers_of(keys, hl);
      }
      // a value row that stands for NaN gives NaN through its scale; its codes would also reach the
      // one row that does not see it
      const uint64_t odd = __builtin_amdgcn_ballot_w64(!__builtin_isfinite(sb[lane])) >> 32;
      for (uint32_t rows = (uint32_t)odd; rows; rows &= rows - 1u)
        if (lane < kCh)
          *(lds16*)(slots + 2 * kSB * s + kSB + (__ffs(rows) - 1) * D + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
    }
    const float mine = sb[lane];
    float ratio = 1.0f;  // of O's old units to its new ones
    u32x4 kr[D / 32];
    const uint32_t ks0 = opaque(ka + 2 * kSB * s), qs0 = kQReg ? 0u : opaque(qa);
#pragma unroll
    for (int u = 0; u < D / 32; ++u) kr[u] = *(const lds16*)(ks0 ^ (u << 5));
    if (i == 0) two_f = power_at((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(mine), 32));
    if (i == 0) over_f = over_of(two_f);
    if (__builtin_amdgcn_ballot_w64(hl && mine >= kOver * two_f && mine < INFINITY)) {
      const float e = power_of(hl ? mine : 0.0f);
      ratio = two_f * over_of(e);
      two_f = e;
      over_f = over_of(e);
    }
    sb[lane] = mine * (hl ? over_f : p.c2);
    f32x16 sc[R];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[t][r] = 0.0f;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      const bf16x8 k0 = decode(kr[u][0], kr[u][1]), k1 = decode(kr[u][2], kr[u][3]);
#pragma unroll
      for (int t = 0; t < R; ++t) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, q_at(qs0, t, 2 * u), sc[t], 0, 0, 0);
#pragma unroll
      for (int t = 0; t < R; ++t) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, q_at(qs0, t, 2 * u + 1), sc[t], 0, 0, 0);
    }
    f32x4 ks[1][4];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) ks[0][g4] = *(const ldsf4*)(sb + 4 * hl + 8 * g4);
    weigh<D, R, 1>(sc, ks, masked, hidden, ratio, m, l, o);
    i32x2 vr[2][D / 32];
    const uint32_t vs0 = opaque(va + 2 * kSB * s);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) vr[kk][db] = v_tr8((const lds_t*)((vs0 ^ (db << 5)) + kk * 16 * D));
    f16x8 pk[R][2];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      const f32x4 vs = *(const ldsf4*)(sb + 32 + 4 * hl + 8 * g4);
#pragma unroll
      for (int t = 0; t < R; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) pk[t][g4 >> 1][4 * (g4 & 1) + e] = (_Float16)(sc[t][4 * g4 + e] * vs[e]);
    }
    if (masked) {  // (a hidden key's scale may be anything)
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const uint32_t h = opaque(hidden[t]);
#pragma unroll
        for (int r = 0; r < 16; ++r) pk[t][r >> 3][r & 7] = (h >> r) & 1u ? (_Float16)0.0f : pk[t][r >> 3][r & 7];
      }
    }
    wait_lds();  // the slot has been read: refill it
    issue(i + 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const f16x8 va = decode16(vr[kk][db][0], vr[kk][db][1]);
#pragma unroll
        for (int t = 0; t < R; ++t) o[t][db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va, pk[t][kk], o[t][db], 0, 0, 0);
      }
  }

  // ---- stages of live rows: K in slot kslot, V in the other -------------------------------------------
  for (int e = live0; e < e1; e += kTW) {
    const int first = (e - nB) * kStage;
    const lds_t* const kb = slots + 2 * kSB * kslot;
    lds_t* const vb = slots + 2 * kSB * (1 - kslot);
    if (e != live0) {
      issue_live(e, kslot, false);
      issue_live(e, 1 - kslot, true);
    }
    // a seed's live row is for that row alone, which adds it at the end
    const uint32_t seeds = n_seeds > 0 ? __builtin_amdgcn_readfirstlane(sBits[first >> 5]) : 0u;
    const uint32_t keys = past(x.nv - first) | seeds;
    uint32_t hidden[R];
#pragma unroll
    for (int t = 0; t < R; ++t) hidden[t] = registers_of(keys, hl);
    wait_loads<kNV>();
    f32x16 sc[R];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[t][r] = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const bf16x8 kr = *(const lds8*)(kb + k_off<D>(l32, 2 * ((k & ~1) + hl) + (k & 1)));
#pragma unroll
      for (int t = 0; t < R; ++t) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr, q_at(qa, t, k), sc[t], 0, 0, 0);
    }
    const f32x4 cc = {p.c2, p.c2, p.c2, p.c2};
    const f32x4 ks[1][4] = {{cc, cc, cc, cc}};
    weigh<D, R, 1>(sc, ks, keys != 0u, hidden, 1.0f, m, l, o);
    wait_loads<0>();
    for (uint32_t rows = seeds; rows; rows &= rows - 1u)
      if (lane < kLC) *(lds16*)(vb + (__ffs(rows) - 1) * (2 * D) + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
    // a transposing read of bf16: 4 rows x 16 columns per 16 lanes
    const int G = lane >> 4, ii = lane & 15, lrow = 4 * hl + (ii >> 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 pk[R], pl[R];
#pragma unroll
      for (int t = 0; t < R; ++t) two_parts(sc[t], kk, over_f, pk[t], pl[t]);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int col = db * 32 + 16 * (G & 1) + 4 * (ii & 3);
        const lds_t* vp = vb + lrow * (2 * D) + (((col >> 3) ^ v_swz<D>(lrow)) << 4) + ((col & 7) << 1) + kk * 32 * D;
        const bf16x8 va = __builtin_bit_cast(
            bf16x8, __builtin_shufflevector(v_tr(vp), v_tr(vp + 16 * D), 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int t = 0; t < R; ++t) {
          o[t][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pk[t], o[t][db], 0, 0, 0);
          o[t][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pl[t], o[t][db], 0, 0, 0);
        }
      }
    }
    wait_lds();
  }

  // ---- merge: every wave's (max, sum, O) through LDS, 32 rows at a time ------------------------------
  const CachedParams& lp = late();
  const CachedArgs& z = lp.a;
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const float lt = pair_sum(l[t]);
    if (hl == 0) {
      sM[wave][32 * t + l32] = m[t];
      sL[wave][32 * t + l32] = lt;
    }
  }
  if (lane == 0) sPower[wave] = two_f;
  // row l32, 16-byte chunk c (dims 4 c .. 4 c + 3) at byte 4 D l32 + 16 (c ^ l32 % (D / 4))
  constexpr int kOM = D / 4 - 1;
  // wave w finishes rows kFin w + fq (lane group fq of 16) of each 32, lane dims kE fj .. kE fj + kE - 1
  constexpr int kFin = 32 / kTW, kE = D / 16;
  typedef __bf16 out_t __attribute__((ext_vector_type(kE)));
  const int fq = lane >> 4, fj = lane & 15;
#pragma unroll
  for (int tile = 0; tile < R; ++tile) {
    if (tile > 0) __syncthreads();
    lds_t* const ob = slots + 4 * D * l32;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const int c = 8 * db + 2 * gq + hl;
        *(ldsf4*)(ob + ((c ^ (l32 & kOM)) << 4)) = f32x4{o[tile][db][4 * gq], o[tile][db][4 * gq + 1],
                                                         o[tile][db][4 * gq + 2], o[tile][db][4 * gq + 3]};
      }
    __syncthreads();
    const int row = kFin * wave + fq, ff = qt * kTQ + 32 * tile + row, fc = min(ff, n_rows - 1);
    const int hg = div(fc, lp.lq), fr = fc - hg * z.Lq, fh = g * lp.group + hg;
    const bool ok = ff < n_rows && fr < x.nv;
    const bool seed = ok && split == 0 && is_seed(fr);
    float acc[kE], den = 0.0f, M = kInit, ts = -INFINITY;
#pragma unroll
    for (int e = 0; e < kE; ++e) acc[e] = 0.0f;
    out_t vd = {};
    if (seed) {  // (uniform over a row's 16 lanes)
      const out_t qv = *(const out_t*)((const __bf16*)z.q + b * z.q_sb + fh * z.q_sh + fr * z.q_sl + kE * fj);
      const out_t kd = *(const out_t*)((const __bf16*)z.k_live + b * z.k_sb + g * z.k_sh + fr * z.k_sl + kE * fj);
      vd = *(const out_t*)((const __bf16*)z.v_live + b * z.v_sb + g * z.v_sh + fr * z.v_sl + kE * fj);
      float dot = 0.0f;
#pragma unroll
      for (int e = 0; e < kE; ++e) dot = __builtin_fmaf((float)qv[e], (float)kd[e], dot);
#pragma unroll
      for (int s = 8; s >= 1; s >>= 1) dot += __shfl_xor(dot, s);
      ts = dot * lp.c2;
      M = __builtin_fmaxf(M, ts);
    }
    float mw[kTW], lw[kTW];
#pragma unroll
    for (int w = 0; w < kTW; ++w) {
      mw[w] = sM[w][32 * tile + row];
      lw[w] = sL[w][32 * tile + row];
      M = __builtin_fmaxf(M, mw[w]);
    }
#pragma unroll
    for (int w = 0; w < kTW; ++w) {
      float s = __builtin_amdgcn_exp2f(mw[w] - M);
      den = __builtin_fmaf(lw[w], s, den);
      s *= sPower[w];
      const lds_t* rb = (const lds_t*)sKV[w] + 4 * D * row;
#pragma unroll
      for (int e = 0; e < kE; e += 4) {
        const f32x4 v = *(const ldsf4*)(rb + ((((kE * fj + e) / 4) ^ (row & kOM)) << 4));
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[e + u] = __builtin_fmaf(s, v[u], acc[e + u]);
      }
    }
    if (seed) {
      const float s = __builtin_amdgcn_exp2f(ts - M);
      den += s;
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[e] = __builtin_fmaf(s, (float)vd[e], acc[e]);
    }
    if (!ok) continue;
    const int64_t bh = (int64_t)b * z.Hq + fh;
    if constexpr (SPLIT) {
      float* rec = z.workspace + ((bh * lp.n_split + split) * z.Lq + fr) * (D + 4);
#pragma unroll
      for (int e = 0; e < kE; e += 4) *(f32x4*)(rec + kE * fj + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
      if (fj == 0) *(f32x4*)(rec + D) = f32x4{M, den, 0.0f, 0.0f};
    } else {
      const float inv = 1.0f / den;
      out_t out;
#pragma unroll
      for (int e = 0; e < kE; ++e) out[e] = (__bf16)(acc[e] * inv);
      *(out_t*)((__bf16*)z.out + b * z.o_sb + fh * z.o_sh + fr * z.o_sl + kE * fj) = out;
      if (z.lse && fj == 0) z.lse[bh * z.Lq + fr] = (M + __builtin_amdgcn_logf(den)) * kLn2;
    }
  }
}

// Many query rows: one workgroup of 4 waves per 128 rows of a key/value head, each wave with 32 rows of its own
// over all of the keys, so that nothing is merged and K and V are loaded once for the 128 rows.  Steps of
// 64 keys (32 of the live rows) go through three slots that all waves read: at the top of a step a wave waits
// for the step's loads of its own, the barrier makes that all of them and says that the step before has been
// read, and the loads two steps on go out into its slot.
__global__ __launch_bounds__(64 * kRW, 2) void cover_attn_cached_rows_kernel(const CachedParams p) {
  constexpr int D = 128, kTQ = 32 * kRW, kStep = 2 * kStage;
  constexpr int kHalf = kStep * D;             // bytes of K (or V) of a step: codes, or 32 live rows in bf16
  constexpr int kCh = D / 16, kRPL = 64 / kCh;  // 16-byte chunks of codes per row, rows per load
  constexpr int kLC = D / 8, kLR = 64 / kLC;    // the same of live rows
  constexpr int kOwn = 4;                       // a wave's loads of a step, but for the scales
  __shared__ __attribute__((aligned(1024))) char sKV[3][2 * kHalf];
  __shared__ __attribute__((aligned(16))) float sScale[3][2][kStep];
  __shared__ float sPower[3];
  __shared__ uint32_t sBits[COVER_CACHED_MAX_LQ / 32];
  __shared__ uint16_t sList[COVER_CACHED_MAX_LQ];

  const CachedArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hl = lane >> 5;
  const int li = place_of(p);
  if (li >= p.n_wg) return;
  const int rest = uniform(div(li, p.n_qt));
  const int qt = li - rest * (int)p.n_qt.d;
  const int b = uniform(div(rest, p.heads)), g = rest - b * a.Hkv;
  Extent x(a, b);
  x.len = uniform(x.len);
  x.o = uniform(x.o);
  x.nv = uniform(x.nv);
  const int n_rows = p.group * a.Lq;
  const int ft = qt * kTQ + 32 * wave + l32, f = min(ft, n_rows - 1);
  const int hg = div(f, p.lq), qr = f - hg * a.Lq;
  const bool there = ft < n_rows && qr < x.nv;
  {  // no row exists: the first is past the end, and no head begins in the tile
    const int f0 = qt * kTQ, r0 = f0 - uniform(div(f0, p.lq)) * a.Lq;
    if (x.nv <= 0 || (r0 >= x.nv && f0 + a.Lq - r0 >= min(f0 + kTQ, n_rows))) return;
  }

  const int ns = a.max_seeds > 0 ? uniform(min(max(a.n_seed[b], 0), a.max_seeds)) : 0;
  const int past_block = x.len - x.o - x.nv;
  const int nA1 = (x.o + kStep - 1) / kStep, nA = nA1 + (past_block + kStep - 1) / kStep;
  const int nC = (x.nv + kStage - 1) / kStage;
  int nB = 0, total = nA + nC;  // steps of seeds, and all, once the seeds are known

  const char* const kcb = (const char*)a.kc + b * a.c_sb + g * a.c_sh;
  const char* const vcb = (const char*)a.vc + b * a.c_sb + g * a.c_sh;
  const uint32_t slot0 = lds_addr((lds_t*)sKV[0]), scale0 = lds_addr((lds_t*)sScale[0][0]);
  int n_seeds = 0;  // distinct, once the bitmap is there
  // this wave's share of step i's loads: of K and V each 1024 bytes twice, and the scales of K (wave 0) or V (wave 1)
  const int my_row = kRPL * wave + lane / kCh;  // and the one kStage further, whose chunks are in the same places
  const uint32_t off = (uint32_t)my_row * (uint32_t)a.c_sl;
  const uint32_t offK = off + (((lane % kCh) ^ kc_swz<D>(my_row)) << 4), offV = off + (((lane % kCh) ^ vc_swz<D>(my_row)) << 4);
  const float* const sc_b = (wave ? a.vs : a.ks) + (b * a.s_sb + g * a.s_sh);
  auto issue = [&](int i) __attribute__((always_inline)) {
    if (i >= total) return;
    const int slot = i % 3;
    const uint32_t kd = uniform(slot0 + 2 * kHalf * slot + 1024 * wave), vd = kd + kHalf;
    const uint32_t sd = uniform(scale0 + 4 * kStep * (2 * slot + wave));
    const int first = i < nA1 ? i * kStep : (i < nA ? x.o + x.nv + (i - nA1) * kStep : (i - nA) * kStep);
    const int end = i < nA1 ? x.o : x.len;
    if (i < nA && first + kStep <= end && !p.wide) {
      const int64_t at = (int64_t)((uint64_t)(uint32_t)first * (uint32_t)a.c_sl), more = kStage * a.c_sl;
      gmem_t* const kp = (gmem_t*)(kcb + at);
      gmem_t* const vp = (gmem_t*)(vcb + at);
      dma16s(kd, kp, offK);
      dma16s(vd, vp, offV);
      dma16s(kd + 1024 * kRW, kp + more, offK);
      dma16s(vd + 1024 * kRW, vp + more, offV);
      if (wave < 2) dma4(sd, (gmem_t*)(sc_b + first + lane));
    } else if (i < nA + nB) {
      const int ln = opaque(lane);
      auto key_of = [&](int row) {
        if (i < nA) return min(first + row, end - 1);
        return x.o + (int)sList[min(first + row, n_seeds - 1)];
      };
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = kRPL * (wave + kRW * j) + ln / kCh, pc = ln % kCh;
        const int64_t at = key_of(row) * a.c_sl;
        dma16(kd + 1024 * kRW * j, (gmem_t*)(kcb + at + ((pc ^ kc_swz<D>(row)) << 4)));
        dma16(vd + 1024 * kRW * j, (gmem_t*)(vcb + at + ((pc ^ vc_swz<D>(row)) << 4)));
      }
      if (wave < 2) dma4(sd, (gmem_t*)(sc_b + key_of(ln)));
    } else {
      const CachedArgs& z = late().a;
      const int ln = opaque(lane);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = kLR * (wave + kRW * j) + ln / kLC, pc = ln % kLC;
        const int64_t key = min((i - nA - nB) * kStage + row, x.nv - 1);
        const char* const kl = (const char*)((const __bf16*)z.k_live + b * z.k_sb + g * z.k_sh + key * z.k_sl);
        const char* const vl = (const char*)((const __bf16*)z.v_live + b * z.v_sb + g * z.v_sh + key * z.v_sl);
        dma16(kd + 1024 * kRW * j, (gmem_t*)(kl + ((pc ^ k_swz<D>(row)) << 4)));
        dma16(vd + 1024 * kRW * j, (gmem_t*)(vl + ((pc ^ v_swz<D>(row)) << 4)));
      }
    }
  };
  // ---- Q of the wave's rows, and the first two steps where they are the cache's ------------------------
  {
    const __bf16* const qb = (const __bf16*)a.q + b * a.q_sb + g * p.group * a.q_sh;
#pragma unroll
    for (int j = 0; j < 32 / kLR; ++j) {
      const int row = kLR * j + lane / kLC, pc = lane % kLC, fq = min(qt * kTQ + 32 * wave + row, n_rows - 1);
      const int fh = div(fq, p.lq);
      dma16(lds_addr((lds_t*)sKV[1]) + 2 * D * 32 * wave + 1024 * j,
            (gmem_t*)((const char*)(qb + fh * a.q_sh + (fq - fh * a.Lq) * a.q_sl) + ((pc ^ k_swz<D>(row)) << 4)));
    }
  }
  if (nA > 0) issue(0);
  if (tid < 64) sBits[tid] = 0u;
  __syncthreads();
  // ---- the block's seeds ---------------------------------------------------------------------------------
  int my_seed = -1;
  if (ns > 0) {
    for (int t = tid; t < ns; t += 64 * kRW) {
      const int r = a.seed_idx[(int64_t)b * a.max_seeds + t] - x.o;
      if ((unsigned)r < (unsigned)x.nv) atomicOr(&sBits[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int w = 0; w < nC; ++w) {  // (every wave writes the same list)
      const uint32_t word = sBits[w];
      if (hl == 0 && ((word >> l32) & 1u)) sList[n_seeds + __popc(word & ((1u << l32) - 1u))] = (uint16_t)(32 * w + l32);
      if (qr >> 5 == w && ((word >> (qr & 31)) & 1u)) my_seed = n_seeds + __popc(word & ((1u << (qr & 31)) - 1u));
      n_seeds += uniform(__popc(word));
    }
    wait_lds();
    nB = (n_seeds + kStep - 1) / kStep;
    total += nB;
  }
  if (nA == 0) issue(0);

  f32x16 o[1][D / 32];
  float m[1] = {kInit}, l[1] = {0.0f};
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][db][r] = 0.0f;
  wait_loads<0>();  // Q has landed (this wave's own, which no other reads)
  bf16x8 qreg[D / 16];
  lds_t* const qs = (lds_t*)sKV[1] + 2 * D * 32 * wave;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) qreg[k] = *(const lds8*)(qs + k_off<D>(l32, 2 * ((k & ~1) + hl) + (k & 1)));
  wait_lds();
  __syncthreads();
  issue(1);
  const uint32_t ka = slot0 + l32 * D + ((hl ^ kc_swz<D>(l32)) << 4);
  uint32_t va;
  {
    const int r8 = (lane & 15) >> 1, row = (r8 & 3) + 8 * (r8 >> 2) + 4 * hl;
    va = slot0 + kHalf + row * D + ((((lane >> 4) & 1) ^ vc_swz<D>(row)) << 4) + 8 * (lane & 1);
  }

  // K's scales times c2 (wave 0); V's in units of a power of two (wave 1), as in the other kernel
  float power = 1.0f, two_f = 1.0f;
  auto prepare = [&](int slot, float mine) {
    if (wave == 1 && __builtin_amdgcn_ballot_w64(mine >= kOver * power && mine < INFINITY)) power = power_of(mine);
    sScale[slot][wave][lane] = mine * (wave == 0 ? p.c2 : over_of(power));
    if (wave == 1 && lane == 0) sPower[slot] = power;
  };
  int s = 0;
  for (int i = 0; i < nA + nB; ++i, s = s == 2 ? 0 : s + 1) {
    if (i + 1 < nA + nB && wave < 2) wait_loads<kOwn + 1>();
    else wait_loads<kOwn>();  // (live rows follow the last step of codes)
    ldsf* const sb = (ldsf*)sScale[s][0];
    if (wave < 2 && i == 0) {
      const float mine = sScale[0][wave][lane];
      power = power_at((uint32_t)uniform((int)__float_as_uint(mine)));
      prepare(0, mine);
    }
    __syncthreads();
    issue(i + 2);
    const int first = i < nA1 ? i * kStep : (i < nA ? (i - nA1) * kStep : (i - nA) * kStep);
    const int left = (i < nA1 ? x.o : (i < nA ? past_block : n_seeds)) - first;
    if (i >= nA) {
      // a value row that stands for NaN gives NaN through its scale; its codes would also reach the one
      // row that does not see it
      if (wave == 0) {
        for (uint64_t rows = __builtin_amdgcn_ballot_w64(!__builtin_isfinite(sb[kStep + lane])); rows; rows &= rows - 1u)
          if (lane < kCh)
            *(lds16*)((lds_t*)sKV[s] + kHalf + __builtin_ctzll(rows) * D + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
        wait_lds();
      }
      __syncthreads();
    }
    const bool masked = left < kStep || i >= nA;
    uint32_t hidden[2] = {0u, 0u};
    if (masked) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        uint32_t keys = past(left - 32 * sub);
        const int mine = my_seed - first - 32 * sub;
        if (i >= nA && (unsigned)mine < (unsigned)kStage) keys |= 1u << mine;
        hidden[sub] = registers_of(keys, hl);
      }
    }
    const float power_s = __uint_as_float((uint32_t)uniform((int)__float_as_uint(sPower[s])));
    const uint32_t k0 = opaque(ka + 2 * kHalf * s), v0 = opaque(va + 2 * kHalf * s);
    ldsf* const sc4 = sb + 4 * hl;
    f32x16 sc[2];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[sub][r] = 0.0f;
#pragma unroll
    for (int u = 0; u < D / 32; ++u)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const u32x4 kr = *(const lds16*)((k0 ^ (u << 5)) + kStage * D * sub);
        sc[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(kr[0], kr[1]), qreg[2 * u], sc[sub], 0, 0, 0);
        sc[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(kr[2], kr[3]), qreg[2 * u + 1], sc[sub], 0, 0, 0);
      }
    f32x4 ks[2][4];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) ks[sub][g4] = *(const ldsf4*)(sc4 + 32 * sub + 8 * g4);
    const float ratio = i == 0 ? 1.0f : two_f * over_of(power_s);
    two_f = power_s;
    weigh<D, 1, 2>(sc, ks, masked, hidden, ratio, m, l, o);
    const int next = s == 2 ? 0 : s + 1;
    float mine = 0.0f;  // the next step's scales, prepared behind this one's products
    if (wave < 2 && i + 1 < nA + nB) {
      if (i + 2 < nA + nB) wait_loads<kOwn + 1>();
      else wait_loads<kOwn>();
      mine = sScale[next][wave][lane];
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      f16x8 pk[2];
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4 vs = *(const ldsf4*)(sc4 + kStep + 32 * sub + 8 * g4);
#pragma unroll
        for (int e = 0; e < 4; ++e) pk[g4 >> 1][4 * (g4 & 1) + e] = (_Float16)(sc[sub][4 * g4 + e] * vs[e]);
      }
      if (masked) {  // (a hidden key's scale may be anything)
        const uint32_t h = opaque(hidden[sub]);
#pragma unroll
        for (int r = 0; r < 16; ++r) pk[r >> 3][r & 7] = (h >> r) & 1u ? (_Float16)0.0f : pk[r >> 3][r & 7];
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const i32x2 vr = v_tr8((const lds_t*)((v0 ^ (db << 5)) + kStage * D * sub + kk * 16 * D));
          o[0][db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(decode16(vr[0], vr[1]), pk[kk], o[0][db], 0, 0, 0);
        }
    }
    if (wave < 2 && i + 1 < nA + nB) prepare(next, mine);
  }
  const float over_f = over_of(two_f);
  for (int i = nA + nB; i < total; ++i, s = s == 2 ? 0 : s + 1) {
    if (i + 1 < total) wait_loads<kOwn>();
    else wait_loads<0>();
    __syncthreads();
    issue(i + 2);
    const int first = (i - nA - nB) * kStage;
    // a seed's live row is for that row alone, which adds it at the end
    const uint32_t seeds = n_seeds > 0 ? (uint32_t)uniform((int)sBits[first >> 5]) : 0u;
    lds_t* const kb = (lds_t*)sKV[s];
    lds_t* const vb = kb + kHalf;
    if (seeds) {
      if (wave == 0) {
        for (uint32_t rows = seeds; rows; rows &= rows - 1u)
          if (lane < kLC) *(lds16*)(vb + (__ffs(rows) - 1) * (2 * D) + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
        wait_lds();
      }
      __syncthreads();
    }
    const uint32_t keys = past(x.nv - first) | seeds;
    const uint32_t hidden[1] = {registers_of(keys, hl)};
    f32x16 sc[1];
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[0][r] = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const lds8*)(kb + k_off<D>(l32, 2 * ((k & ~1) + hl) + (k & 1))),
                                                      qreg[k], sc[0], 0, 0, 0);
    const f32x4 cc = {p.c2, p.c2, p.c2, p.c2};
    const f32x4 ks[1][4] = {{cc, cc, cc, cc}};
    weigh<D, 1, 1>(sc, ks, keys != 0u, hidden, 1.0f, m, l, o);
    const int G = lane >> 4, ii = lane & 15, lrow = 4 * hl + (ii >> 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 pk, pl;
      two_parts(sc[0], kk, over_f, pk, pl);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int col = db * 32 + 16 * (G & 1) + 4 * (ii & 3);
        const lds_t* vp = vb + lrow * (2 * D) + (((col >> 3) ^ v_swz<D>(lrow)) << 4) + ((col & 7) << 1) + kk * 32 * D;
        const bf16x8 vt = __builtin_bit_cast(
            bf16x8, __builtin_shufflevector(v_tr(vp), v_tr(vp + 16 * D), 0, 1, 2, 3, 4, 5, 6, 7));
        o[0][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt, pk, o[0][db], 0, 0, 0);
        o[0][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt, pl, o[0][db], 0, 0, 0);
      }
    }
  }

  __syncthreads();  // (the slots take the output)
  const CachedParams& lp = late();
  const CachedArgs& z = lp.a;
  // ---- a seed row's own live key and value, the division, the output through LDS ------------------------
  float lt = pair_sum(l[0]);
  const bool seed = there && my_seed >= 0;
  if (__builtin_amdgcn_ballot_w64(seed)) {
    float alpha = 1.0f, pd = 0.0f;
    const __bf16* const kl = (const __bf16*)z.k_live + b * z.k_sb + g * z.k_sh + qr * z.k_sl;
    const __bf16* const vl = (const __bf16*)z.v_live + b * z.v_sb + g * z.v_sh + qr * z.v_sl;
    float dot = 0.0f;
    if (seed) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const bf16x8 kd = *(const bf16x8*)(kl + 16 * ((k & ~1) + hl) + 8 * (k & 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = __builtin_fmaf((float)qreg[k][e], (float)kd[e], dot);
      }
    }
    const float t = pair_sum(dot) * lp.c2;
    if (seed) {
      const float M = __builtin_fmaxf(m[0], t);
      alpha = __builtin_amdgcn_exp2f(m[0] - M);
      pd = __builtin_amdgcn_exp2f(t - M);
      m[0] = M;
      lt = __builtin_fmaf(lt, alpha, pd);
      pd *= over_f;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
          const bf16x4 vd = *(const bf16x4*)(vl + 32 * db + 8 * q4 + 4 * hl);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[0][db][4 * q4 + e] = __builtin_fmaf(pd, (float)vd[e], o[0][db][4 * q4 + e] * alpha);
        }
    }
  }
  const int64_t bh = (int64_t)b * z.Hq + g * lp.group;
  if (z.lse && there && hl == 0) z.lse[(bh + hg) * z.Lq + qr] = (m[0] + __builtin_amdgcn_logf(lt)) * kLn2;
  const float inv = two_f / lt;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      const bf16x4 v = {(__bf16)(o[0][db][4 * q4] * inv), (__bf16)(o[0][db][4 * q4 + 1] * inv),
                        (__bf16)(o[0][db][4 * q4 + 2] * inv), (__bf16)(o[0][db][4 * q4 + 3] * inv)};
      *(__attribute__((address_space(3))) bf16x4*)(qs + k_off<D>(l32, 4 * db + q4) + 8 * hl) = v;
    }
  wait_lds();
#pragma unroll
  for (int j = 0; j < 32 / kLR; ++j) {
    const int row = kLR * j + lane / kLC, c = lane % kLC, fo = qt * kTQ + 32 * wave + row;
    const u32x4 v = *(const lds16*)(qs + k_off<D>(row, c));
    if (fo >= n_rows) continue;
    const int fh = div(fo, lp.lq), r = fo - fh * z.Lq;
    if (r < x.nv)
      *(u32x4*)((__bf16*)z.out + b * z.o_sb + (g * lp.group + fh) * z.o_sh + r * z.o_sl + 8 * c) = v;
  }
}

// The ranges' (O, max, sum) of a query row joined by W waves: lane group e of D / 4 lanes (4 elements
// each) takes every (64 W / (D / 4))th range, four loads in flight, and the groups meet in a fixed order.
template <int D, int W>
__global__ __launch_bounds__(256) void cover_attn_cached_join_kernel(const CachedParams p) {
  constexpr int kLanes = D / 4, kGroups = 64 * W / kLanes, kRows = 4 / W;  // rows per workgroup
  __shared__ float sM[kRows][kGroups], sL[kRows][kGroups];
  __shared__ __attribute__((aligned(16))) float sO[kRows][kGroups][D];
  const CachedArgs& a = p.a;
  const int tid = threadIdx.x, slot = tid / (64 * W), group = tid % (64 * W) / kLanes, e4 = tid % kLanes;
  const int64_t row = (int64_t)blockIdx.x * kRows + slot;  // over B * Hq * Lq
  const bool in = row < (int64_t)a.B * a.Hq * a.Lq;
  const int64_t bh = in ? row / a.Lq : 0;
  const int r = in ? (int)(row - bh * a.Lq) : 0, b = (int)(bh / a.Hq), h = (int)(bh - (int64_t)b * a.Hq);
  const Extent x(a, b);
  const bool there = in && r < x.nv;
  const float* rec = a.workspace + (bh * p.n_split * a.Lq + r) * (D + 4);
  const int64_t step = (int64_t)a.Lq * (D + 4);
  float M = kInit, den = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kChunk = 4;
  for (int s0 = group; there && s0 < p.n_split; s0 += kChunk * kGroups) {
    f32x4 v[kChunk], ml[kChunk];
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      const int s = s0 + u * kGroups;
      v[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      ml[u] = f32x4{kInit, 0.0f, 0.0f, 0.0f};
      if (s < p.n_split) {
        v[u] = *(const f32x4*)(rec + s * step + 4 * e4);
        ml[u] = *(const f32x4*)(rec + s * step + D);
      }
    }
    float Mn = M;
#pragma unroll
    for (int u = 0; u < kChunk; ++u) Mn = __builtin_fmaxf(Mn, ml[u][0]);
    const float al = __builtin_amdgcn_exp2f(M - Mn);
    den *= al;
    acc *= al;
    M = Mn;
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      const float w = __builtin_amdgcn_exp2f(ml[u][0] - M);
      den = __builtin_fmaf(ml[u][1], w, den);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(v[u][e], w, acc[e]);
    }
  }
  *(f32x4*)&sO[slot][group][4 * e4] = acc;
  if (e4 == 0) {
    sM[slot][group] = M;
    sL[slot][group] = den;
  }
  __syncthreads();
  if (group != 0 || !there) return;
#pragma unroll
  for (int u = 1; u < kGroups; ++u) M = __builtin_fmaxf(M, sM[slot][u]);
  acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  den = 0.0f;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const float w = __builtin_amdgcn_exp2f(sM[slot][u] - M);
    den = __builtin_fmaf(sL[slot][u], w, den);
    const f32x4 v = *(const f32x4*)&sO[slot][u][4 * e4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(v[e], w, acc[e]);
  }
  const float inv = 1.0f / den;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *(bf16x4*)((__bf16*)a.out + b * a.o_sb + h * a.o_sh + r * a.o_sl + 4 * e4) =
      bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
  if (a.lse && e4 == 0) a.lse[row] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

template <int D>
void launch_join(const CachedParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.a.B * p.a.Hq * p.a.Lq;
  // One wave holds 8 (16 at head size 64) ranges in flight.  Measured (us, the whole call) with one and four waves
  // per row: 3 ranges of 2560 rows 19.3, 20.6 (d64 14.0, 16.0); 8 of 1024 22.3, 22.4; 9 of 896 31.2, 30.7; 17 of
  // 32 14.1, 12.6 (d64 10.2, 9.7); 26 of 32 22.0, 19.4.
  if (p.n_split <= 1024 / D) {
    hipLaunchKernelGGL((cover_attn_cached_join_kernel<D, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, p);
  } else {
    hipLaunchKernelGGL((cover_attn_cached_join_kernel<D, 4>), dim3((unsigned)rows), dim3(256), 0, stream, p);
  }
}

Divisor divisor(uint32_t d) {
  Divisor v;
  v.d = d;
  v.s = 24;
  while ((1u << (v.s - 24)) < d) ++v.s;
  v.m = (uint32_t)((uint64_t(1) << v.s) / d + 1);
  return v;
}

int64_t tiles_of(const CachedArgs& a, int rows) {
  return (int64_t)a.B * a.Hkv * (((int64_t)(a.Hq / a.Hkv) * a.Lq + rows - 1) / rows);
}

template <int D, int R>
void launch(const CachedParams& p, hipStream_t stream) {
  const dim3 grid(8u * p.xcd_slots), block(64 * kTW);
  if (p.n_split == 1) hipLaunchKernelGGL((cover_attn_cached_kernel<D, R, false>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((cover_attn_cached_kernel<D, R, true>), grid, block, 0, stream, p);
}

}  // namespace

// The number of key ranges, at most `most`, that finishes soonest.  In units of what a SIMD's two waves take for
// two stages (about 0.9 us): a workgroup's start and merge take 7, its stages are shared by 4 SIMDs, rounds of
// 256 workgroups follow each other; the join takes 4 and its records 1 for every 128 tiles.  Measured (us)
// with 1, 2, 4, 8 ranges at B1 H32 L1024, 64 rows: 12.7, 13.9, 13.9, 18.8; with 8, 16, 17, 22, 24, 32, 64 at
// B1 Hq32/Hkv8 L8192, one row: 14.2, 12.4, 12.5, 12.0, 12.0, 12.4, 17.9; with 4, 9, 16 at B1 Hq28/Hkv4 L32768,
// 32 rows: 49, 30.6, 32.5.
static int ranges(int64_t tiles, int L, int most) {
  const int64_t stages = L / kStage + 2;
  int best = 1;
  int64_t least = INT64_MAX;
  auto offer = [&](int64_t n) {
    if (n < 1 || n > most) return;
    const int64_t rounds = (tiles * n + 255) / 256, halves = ((stages + n - 1) / n + 3) / 4;
    const int64_t cost = 64 * (rounds * (14 + halves) + (n > 1 ? 8 : 0)) + (n > 1 ? tiles * n : 0);
    if (cost < least) {
      best = (int)n;
      least = cost;
    }
  };
  offer(1);
  for (int r = 1; r <= 4; ++r) offer(256 * r / tiles);
  for (int halves = 1; halves <= 16; ++halves) offer((stages + 4 * halves - 1) / (4 * halves));
  offer(most);
  return best;
}

bool attn_cached_fits(const CachedArgs& a) {  // (the heads first: the other products could pass 64 bits)
  constexpr int64_t kRows = (int64_t(1) << 24) - 4;
  return (int64_t)a.B * a.Hq <= kRows && (int64_t)a.B * a.Hq * a.Lq <= kRows &&
         tiles_of(a, 32) * a.n_split <= (int64_t(1) << 23) - 8;
}

int attn_cached_splits(int B, int Hq, int Hkv, int L, int Lq) {
  CachedArgs a = {};
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lq = Lq; a.n_split = 1;
  return attn_cached_fits(a) ? ranges(tiles_of(a, 32), L, 256) : 1;
}

// Query rows per workgroup.  A round of 256 workgroups takes 1 and 1.7 for 32 and 64 rows, 512 workgroups of 128
// rows (two to a CU) take 5.7 and the last 256 of them 3.8; the rest is how full the rounds are.  Measured (us) at
// H32 L2048 d128 with 32, 64, 128 rows: B8 Lq32 31.6, 36.5, 61.5; B6 Lq64 35.6, 30.0, 60.6; B10 Lq64 53.8, 57.4,
// 80.1; B8 Lq128 69.2, 58.9, 63.8; B8 Lq256 134, 112, 95.5; B8 Lq384 201, 172, 149; B8 Hq64/Hkv8 Lq200 197, 175,
// 166.  At head size 64 half the shared data per row leaves 128 rows little to win (B8 Lq256: 72.0 with 32 rows,
// 69.8 with 64, and 128 rows were within 1 % of that): they are not built.
static int rows_per_workgroup(const CachedArgs& a, int n_split) {
  auto rounds = [&](int rows) { return (tiles_of(a, rows) * n_split + 255) / 256; };
  int64_t least = 10 * rounds(32);
  int rows = 32;
  if (17 * rounds(64) < least) {
    least = 17 * rounds(64);
    rows = 64;
  }
  const bool may = a.d == 128 && n_split == 1;
  return may && 57 * (rounds(128) / 2) + 38 * (rounds(128) % 2) < least ? 128 : rows;
}

void attn_cached_plan(const CachedArgs& a, int* n_ranges, int* rows) {
  *n_ranges = ranges(tiles_of(a, 32), a.L, a.n_split);
  *rows = rows_per_workgroup(a, *n_ranges);
}

hipError_t launch_attn_cached(const CachedArgs& a, hipStream_t stream) {
  CachedParams p;
  p.a = a;
  p.group = a.Hq / a.Hkv;
  int rows;
  attn_cached_plan(a, &p.n_split, &rows);
  p.n_qt = divisor((uint32_t)((p.group * a.Lq + rows - 1) / rows));
  p.splits = divisor((uint32_t)p.n_split);
  p.heads = divisor((uint32_t)a.Hkv);
  p.lq = divisor((uint32_t)a.Lq);
  p.wide = a.c_sl >= (int64_t(1) << 26);
  p.c2 = a.scale * 1.44269504088896341f;
  p.n_wg = (int)(tiles_of(a, rows) * p.n_split);
  p.xcd_slots = (p.n_wg + 7) / 8;
  p.spread = (int64_t)a.B * a.Hkv * p.n_split % 8 == 0;
  if (rows == 32 * kRW) {
    hipLaunchKernelGGL(cover_attn_cached_rows_kernel, dim3(8u * p.xcd_slots), dim3(64 * kRW), 0, stream, p);
  } else if (a.d == 128) {
    if (rows == 64) launch<128, 2>(p, stream);
    else launch<128, 1>(p, stream);
  } else {
    if (rows == 64) launch<64, 2>(p, stream);
    else launch<64, 1>(p, stream);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  if (a.d == 128) launch_join<128>(p, stream);
  else launch_join<64>(p, stream);
  return hipGetLastError();
}

}  // namespace cover
