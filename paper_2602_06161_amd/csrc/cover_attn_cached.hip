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
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_t;
typedef __attribute__((address_space(1))) const char gmem_t;

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
  int wide;             // code rows too far apart for 32-bit offsets in a stage
  float c2;             // scale * log2(e)
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
__device__ __forceinline__ uint32_t k_off(int row, int c) {
  return row * (2 * D) + ((c ^ (D == 128 ? (row & 15) : ((row >> 1) & 7))) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t v_off(int row, int c) {
  return row * (2 * D) + ((c ^ ((row & 3) << (D == 128 ? 2 : 1))) << 4);
}

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

// Global -> LDS loads: lane l's 16 bytes (4 for the dword form) land at LDS byte lds + 16 l (+ 4 l);
// lds is wave-uniform.  The compiler does not track them: every read of their data follows an
// explicit vmcnt wait of the issuing wave.  A wave's loads land in issue order.
__device__ __forceinline__ void dma16(uint32_t lds, gmem_t* addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(lds), "v"((uint64_t)addr) : "memory", "m0");
}
__device__ __forceinline__ void dma16s(uint32_t lds, gmem_t* base, uint32_t voff) {  // uniform base
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void dma4(uint32_t lds, gmem_t* addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off"
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
__device__ __forceinline__ gmem_t* uniform_ptr(const void* ptr) {
  const uint64_t v = (uint64_t)ptr;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (gmem_t*)(((uint64_t)hi << 32) | lo);
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
  constexpr int kSB = kStage * D;            // bytes of one stage of K (or V) codes
  constexpr int kCh = D / 16, kRPL = 64 / kCh;  // 16-byte chunks of codes per row, rows per load
  constexpr int kNK = kStage / kRPL, kNL = 2 * kNK + 1;  // loads of K (or V) of a stage, all its loads
  // per wave: two slots of K and V codes, or one of live rows (at the end: its partial O, 32 rows of D
  // fp32); the two slots' scales
  __shared__ __attribute__((aligned(1024))) char sKV[kTW][4 * kSB];
  __shared__ __attribute__((aligned(16))) float sScale[kTW][2][2][kStage];
  __shared__ __attribute__((aligned(1024))) char sQ[kTQ * 2 * D];
  __shared__ uint32_t sBits[COVER_CACHED_MAX_LQ / 32];  // the block's seed rows
  __shared__ uint16_t sList[COVER_CACHED_MAX_LQ];       // and their list, ascending
  __shared__ float sM[kTW][kTQ], sL[kTW][kTQ];
  static_assert(COVER_CACHED_MAX_LQ / 32 == 64, "the words of the seed bitmap that are cleared");

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

  // ---- stages: this workgroup's range of them, its cache stages [a0, a1) and short ones [e0, e1) -----
  // (as many stages of seeds as the list's length asks for; fewer distinct ones leave some empty)
  const int ns = a.max_seeds > 0 ? min(max(a.n_seed[b], 0), a.max_seeds) : 0;
  const int nA1 = (x.o + kStage - 1) / kStage, nA2 = (x.len - x.o - x.nv + kStage - 1) / kStage;
  const int nA = nA1 + nA2, nC = (x.nv + kStage - 1) / kStage, nB = min((ns + kStage - 1) / kStage, nC);
  const int total = nA + nB + nC;
  const int per = SPLIT ? (total + p.n_split - 1) / p.n_split : total;
  const int w0 = min(split * per, total), w1 = min(w0 + per, total);
  const int e0 = max(w0 - nA, 0), e1 = max(w1 - nA, 0);
  // short stage e0 + i goes to wave i % 8; the waves' cache stages even that out
  int a0 = min(w0, nA), a1 = a0;
  {
    const int n = w1 - w0, end = min(w1, nA);
    for (int w = 0; w <= wave; ++w) {
      a0 = a1;
      const int quota = n * (w + 1) / kTW - n * w / kTW, own = (e1 - e0 + kTW - 1 - w) / kTW;
      a1 = w == kTW - 1 ? end : min(a0 + max(quota - own, 0), end);
    }
  }
  const int nW = a1 - a0;
  const int seeds0 = e0 + wave, nS = seeds0 < min(e1, nB) ? (min(e1, nB) - seeds0 + kTW - 1) / kTW : 0;
  const int n8 = nW + nS;             // this wave's stages of codes
  const int live0 = seeds0 + nS * kTW;  // its first stage of live rows, if below e1

  const char* const kcb = (const char*)a.kc + b * a.c_sb + g * a.c_sh;
  const char* const vcb = (const char*)a.vc + b * a.c_sb + g * a.c_sh;
  const int64_t s_off = b * a.s_sb + g * a.s_sh;
  const float* const scb = (hl ? a.vs : a.ks) + s_off;  // lanes 0-31: K's scales, 32-63: V's
  lds_t* const slots = (lds_t*)sKV[wave];
  typedef __attribute__((address_space(3))) float ldsf;
  ldsf* const scales = (ldsf*)sScale[wave][0][0];
  const uint32_t slot0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)slots);
  const uint32_t scale0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)scales);
  // load j of a stage covers stage rows kRPL j + lane / kCh at physical chunk lane % kCh; the source
  // chunk is the one that the swizzle puts there
  uint32_t offK[kNK], offV[kNK];
#pragma unroll
  for (int j = 0; j < kNK; ++j) {
    const int row = kRPL * j + lane / kCh, pc = lane % kCh;
    offK[j] = (uint32_t)(row * a.c_sl) + ((pc ^ kc_swz<D>(row)) << 4);
    offV[j] = (uint32_t)(row * a.c_sl) + ((pc ^ vc_swz<D>(row)) << 4);
  }
  // cache stage st into slot s; rows past the end repeat the last one
  auto issue_cache = [&](int st, int s) __attribute__((always_inline)) {
    const int first = st < nA1 ? st * kStage : x.o + x.nv + (st - nA1) * kStage;
    const int end = st < nA1 ? x.o : x.len;
    const uint32_t kd = slot0 + 2 * kSB * s, vd = kd + kSB;
    if (first + kStage <= end && !p.wide) {
      gmem_t* const kp = uniform_ptr(kcb + first * a.c_sl);
      gmem_t* const vp = uniform_ptr(vcb + first * a.c_sl);
#pragma unroll
      for (int j = 0; j < kNK; ++j) dma16s(kd + 1024 * j, kp, offK[j]);
#pragma unroll
      for (int j = 0; j < kNK; ++j) dma16s(vd + 1024 * j, vp, offV[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kNK; ++j) {
        const int row = kRPL * j + lane / kCh, pc = lane % kCh;
        const int64_t at = min(first + row, end - 1) * a.c_sl;
        dma16(kd + 1024 * j, (gmem_t*)(kcb + at + ((pc ^ kc_swz<D>(row)) << 4)));
        dma16(vd + 1024 * j, (gmem_t*)(vcb + at + ((pc ^ vc_swz<D>(row)) << 4)));
      }
    }
    dma4(scale0 + 256 * s, (gmem_t*)(scb + min(first + l32, end - 1)));
  };
  // Q: load w covers rows kQR w + lane / kQC of the tile
  constexpr int kQC = D / 8, kQR = 64 / kQC;
  if (kTQ / kQR == kTW || wave < kTQ / kQR) {
    const int row = kQR * wave + lane / kQC, pc = lane % kQC;
    const int fq = min(qt * kTQ + row, n_rows - 1);
    const __bf16* src = (const __bf16*)a.q + b * a.q_sb + (g * p.group + fq / a.Lq) * a.q_sh + (fq % a.Lq) * a.q_sl;
    dma16(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_t*)sQ) + 1024 * wave,
          (gmem_t*)((const char*)src + ((pc ^ (D == 128 ? (row & 15) : ((row >> 1) & 7))) << 4)));
  }
  if (nW > 0) issue_cache(a0, 0);
  if (nW > 1) issue_cache(a0 + 1, 1);

  // ---- the block's seeds: bitmap, their list, and this lane's row's place in it ---------------------
  int n_seeds = 0, my_seed = -1;
  if (ns > 0) {
    if (tid < 64) sBits[tid] = 0u;
    __syncthreads();
    for (int t = tid; t < ns; t += 64 * kTW) {
      const int r = a.seed_idx[(int64_t)b * a.max_seeds + t] - x.o;
      if ((unsigned)r < (unsigned)x.nv) atomicOr(&sBits[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    int mine = 0;
    for (int w = 0; w < nC; ++w) {
      const int c = __popc(sBits[w]);
      n_seeds += c;
      mine += w < qr >> 5 ? c : 0;
    }
    n_seeds = __builtin_amdgcn_readfirstlane(n_seeds);
    const uint32_t word = sBits[qr >> 5];
    if ((word >> (qr & 31)) & 1u) my_seed = mine + __popc(word & ((1u << (qr & 31)) - 1u));
    for (int r = tid; r < x.nv; r += 64 * kTW) {
      const uint32_t wr = sBits[r >> 5];
      if (!((wr >> (r & 31)) & 1u)) continue;
      int at = __popc(wr & ((1u << (r & 31)) - 1u));
      for (int w = 0; w < r >> 5; ++w) at += __popc(sBits[w]);
      sList[at] = (uint16_t)r;
    }
    __syncthreads();
  }
  auto is_seed = [&](int r) -> bool { return n_seeds > 0 && ((sBits[r >> 5] >> (r & 31)) & 1u); };
  // stage e of the seeds, gathered, into slot s
  auto issue_seeds = [&](int e, int s) __attribute__((always_inline)) {
    auto pos_of = [&](int i) { return x.o + (n_seeds > 0 ? (int)sList[min(e * kStage + i, n_seeds - 1)] : 0); };
#pragma unroll
    for (int j = 0; j < kNK; ++j) {
      const int row = kRPL * j + lane / kCh, pc = lane % kCh;
      const int64_t at = pos_of(row) * a.c_sl;
      dma16(slot0 + 2 * kSB * s + 1024 * j, (gmem_t*)(kcb + at + ((pc ^ kc_swz<D>(row)) << 4)));
      dma16(slot0 + 2 * kSB * s + kSB + 1024 * j, (gmem_t*)(vcb + at + ((pc ^ vc_swz<D>(row)) << 4)));
    }
    dma4(scale0 + 256 * s, (gmem_t*)(scb + pos_of(l32)));
  };
  // K (or V) of live stage e into a slot: bf16 rows, as the block kernel lays them out
  constexpr int kLC = D / 8, kLR = 64 / kLC, kNV = kStage / kLR;  // chunks per row, rows per load, loads
  auto issue_live = [&](int e, int s, bool v) __attribute__((always_inline)) {
    const char* const src = v ? (const char*)((const __bf16*)a.v_live + b * a.v_sb + g * a.v_sh)
                              : (const char*)((const __bf16*)a.k_live + b * a.k_sb + g * a.k_sh);
    const int64_t step = 2 * (v ? a.v_sl : a.k_sl);
#pragma unroll
    for (int j = 0; j < kNV; ++j) {
      const int row = kLR * j + lane / kLC, pc = lane % kLC;
      const int c = v ? pc ^ ((row & 3) << (D == 128 ? 2 : 1)) : pc ^ (D == 128 ? (row & 15) : ((row >> 1) & 7));
      dma16(slot0 + 2 * kSB * s + 1024 * j,
            (gmem_t*)(src + min((e - nB) * kStage + row, x.nv - 1) * step + 16 * c));
    }
  };
  // the stage that follows in a slot: code stage i, or K or V of the first live stage
  const int kslot = n8 & 1;
  auto issue = [&](int i) __attribute__((always_inline)) {
    if (i < nW) issue_cache(a0 + i, i & 1);
    else if (i < n8) issue_seeds(seeds0 + (i - nW) * kTW, i & 1);
    else if (i < n8 + 2 && live0 < e1) issue_live(live0, i & 1, i > n8);
  };
  for (int i = nW; i < 2; ++i) issue(i);

  // Q (B operand): element order of step 2 u + t is dims 16 (2 u + hl) + 8 t .. + 7, so that a lane's
  // 16-byte chunk of K codes feeds two steps.  It comes through LDS: a load into registers would make
  // the compiler wait for every load in flight at its first use, inside the loop.
  if (n8 > 1) wait_loads<2 * kNL>();  // (no more than the loads that follow Q's)
  else if (n8 == 1) wait_loads<kNL>();
  else wait_loads<0>();
  __syncthreads();
  typedef __attribute__((address_space(3))) bf16x8 lds8;
  typedef __attribute__((address_space(3))) u32x4 lds16;
  typedef __attribute__((address_space(3))) f32x4 ldsf4;
  bf16x8 qreg[D / 16];
#pragma unroll
  for (int u = 0; u < D / 32; ++u)
#pragma unroll
    for (int t = 0; t < 2; ++t) qreg[2 * u + t] = *(const lds8*)((const lds_t*)sQ + k_off<D>(l32, 2 * (2 * u + hl) + t));
  // V^T operand addresses.  A transposing read gives lane (G = lane / 16, i = lane % 16) of 8 rows x 16
  // columns of codes the 8 rows of column i: keys {0 .. 3, 8 .. 11} + 4 hl, the S^T registers' order
  uint32_t vaddr[D / 32], laddr[D / 32];
  {
    const int G = lane >> 4, ii = lane & 15;
    const int r8 = ii >> 1, row = (r8 & 3) + 8 * (r8 >> 2) + 4 * hl;
    const int lrow = 4 * hl + (ii >> 2);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      vaddr[db] = row * D + (((2 * db + (G & 1)) ^ vc_swz<D>(row)) << 4) + 8 * (ii & 1);
      const int col = db * 32 + 16 * (G & 1) + 4 * (ii & 3);
      laddr[db] = v_off<D>(lrow, col >> 3) + ((col & 7) << 1);
    }
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
  float m = kInit, l = 0.0f;

  // Scores (register r holds key 8 (r / 4) + 4 hl + r % 4 of the lane's query row) to weights in place:
  // times the keys' scales ks (c2 included), `hidden` ones (where masked) to zero, against a maximum that
  // follows where a score passes it by 2^8; l sums them.
  auto weights = [&](f32x16& sc, const f32x4 (&ks)[4], bool masked, uint32_t hidden) __attribute__((always_inline)) {
    float u[16], mx = kInit;
#pragma unroll
    for (int r = 0; r < 16; ++r) u[r] = __builtin_fmaf(sc[r], ks[r >> 2][r & 3], -m);
    if (masked) {
      const uint32_t h = opaque(hidden);
#pragma unroll
      for (int r = 0; r < 16; ++r) u[r] = (h >> r) & 1u ? -INFINITY : u[r];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = __builtin_fmaxf(mx, u[r]);
    mx = pair_max(mx);
    if (__builtin_amdgcn_ballot_w64(mx > kLazyT)) {
      const uint32_t h = opaque(masked ? hidden : 0u);
      float top = m;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        top = __builtin_fmaxf(top, (h >> r) & 1u ? kInit : sc[r] * ks[r >> 2][r & 3]);
      top = pair_max(top);
      const float alpha = __builtin_amdgcn_exp2f(m - top);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[db] *= alpha;
      m = top;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        u[r] = __builtin_fmaf(sc[r], ks[r >> 2][r & 3], -m);
        u[r] = (h >> r) & 1u ? -INFINITY : u[r];
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(u[r]);
      l += sc[r];
    }
  };
  // a lane's registers of the keys in a stage's mask
  auto registers_of = [&](uint32_t keys) -> uint32_t {
    const uint32_t k = keys >> (4 * hl);
    return (k & 0xfu) | ((k >> 4) & 0xf0u) | ((k >> 8) & 0xf00u) | ((k >> 12) & 0xf000u);
  };
  auto past = [](int n) -> uint32_t { return n >= kStage ? 0u : ~0u << max(n, 0); };  // keys at or past n

  // ---- stages of codes, two in flight: the wave's cache stages, then its stages of seeds ---------------
  for (int i = 0; i < n8; ++i) {
    const int s = i & 1;
    if (i + 1 < n8) wait_loads<kNL>();
    else if (live0 < e1) wait_loads<kNV>();
    else wait_loads<0>();
    bool masked = false;
    uint32_t hidden = 0u;
    if (i < nW) {
      const int st = a0 + i;
      const int left = st < nA1 ? x.o - st * kStage : x.len - x.o - x.nv - (st - nA1) * kStage;
      if (left < kStage) {
        masked = true;
        hidden = registers_of(past(left));
      }
    } else {
      const int first = (seeds0 + (i - nW) * kTW) * kStage;
      masked = true;
      uint32_t keys = past(n_seeds - first);
      if ((unsigned)(my_seed - first) < (unsigned)kStage) keys |= 1u << (my_seed - first);
      hidden = registers_of(keys);
      // a value row that stands for NaN gives NaN through its scale; its codes would also reach the
      // one row that does not see it
      const uint64_t odd = __builtin_amdgcn_ballot_w64(!__builtin_isfinite(scales[64 * s + lane])) >> 32;
      for (uint32_t rows = (uint32_t)odd; rows; rows &= rows - 1u)
        if (lane < kCh) *(lds16*)(slots + 2 * kSB * s + kSB + (__ffs(rows) - 1) * D + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
    }
    const lds_t* const kb = slots + 2 * kSB * s;
    const lds_t* const vb = kb + kSB;
    const ldsf* const sb = scales + 64 * s + 4 * hl;
    u32x4 kreg[D / 32];
#pragma unroll
    for (int u = 0; u < D / 32; ++u) kreg[u] = *(const lds16*)(kb + l32 * D + (((2 * u + hl) ^ kc_swz<D>(l32)) << 4));
    if (hl == 0) scales[64 * s + l32] *= p.c2;
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.0f;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      const u32x4 kr = kreg[u];
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(kr[0], kr[1]), qreg[2 * u], sc, 0, 0, 0);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(kr[2], kr[3]), qreg[2 * u + 1], sc, 0, 0, 0);
    }
    f32x4 ks[4];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) ks[g4] = *(const ldsf4*)(sb + 8 * g4);
    weights(sc, ks, masked, hidden);
    i32x2 vr[2][D / 32];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) vr[kk][db] = v_tr8(vb + vaddr[db] + kk * 16 * D);
    bf16x8 pk[2];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      const f32x4 vs = *(const ldsf4*)(sb + 32 + 8 * g4);
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[g4 >> 1][4 * (g4 & 1) + e] = (__bf16)(sc[4 * g4 + e] * vs[e]);
    }
    if (masked) {  // (a hidden key's scale may be anything)
      const uint32_t h = opaque(hidden);
#pragma unroll
      for (int r = 0; r < 16; ++r) pk[r >> 3][r & 7] = (h >> r) & 1u ? (__bf16)0.0f : pk[r >> 3][r & 7];
    }
    wait_lds();  // the slot has been read: refill it
    issue(i + 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(vr[kk][db][0], vr[kk][db][1]), pk[kk], o[db], 0, 0, 0);
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
    const uint32_t hidden = registers_of(past(x.nv - first) | seeds);
    wait_loads<kNV>();
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.0f;
#pragma unroll
    for (int u = 0; u < D / 32; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const lds8*)(kb + k_off<D>(l32, 2 * (2 * u + hl) + t)),
                                                     qreg[2 * u + t], sc, 0, 0, 0);
    const f32x4 cc = {p.c2, p.c2, p.c2, p.c2};
    const f32x4 ks[4] = {cc, cc, cc, cc};
    weights(sc, ks, true, hidden);
    bf16x8 pk[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) pk[r >> 3][r & 7] = (__bf16)sc[r];
    wait_loads<0>();
    for (uint32_t rows = seeds; rows; rows &= rows - 1u)
      if (lane < kLC) *(lds16*)(vb + (__ffs(rows) - 1) * (2 * D) + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const lds_t* vp = vb + laddr[db] + kk * 32 * D;
        const bf16x8 va = __builtin_bit_cast(
            bf16x8, __builtin_shufflevector(v_tr(vp), v_tr(vp + 16 * D), 0, 1, 2, 3, 4, 5, 6, 7));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pk[kk], o[db], 0, 0, 0);
      }
    wait_lds();
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
    lds_t* const ob = slots + 4 * D * l32;
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
    const lds_t* rb = (const lds_t*)sKV[w] + 4 * D * row;
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
  p.wide = a.c_sl >= (int64_t(1) << 26);
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
