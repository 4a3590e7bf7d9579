// C ABI of the layer's operators around the attention (norm, rotary positions, the 8-bit cache and
// the attention over it): host-side validation, then the launch.  Every check here runs before
// anything is enqueued, so a rejected call writes nothing.
#include <math.h>
#include <stdint.h>

#include "cover.h"
#include "cover_internal.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

cover_status hip_status(hipError_t e) { return e == hipSuccess ? COVER_OK : COVER_ERR_HIP; }

bool known(cover_dtype t) { return t == COVER_F32 || t == COVER_BF16; }

// non-negative strides, each a multiple of `vec` elements
template <class... S>
bool strides_ok(int64_t vec, S... s) {
  return ((s >= 0 && s % vec == 0) && ...);
}

// The rows (of `row` elements) of a tensor that is written lie apart: with its dimensions of more than one
// entry in the order of their strides, each stride is at least the one before times that one's entries.
bool apart(int64_t row, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2 = 1, int64_t s2 = 0) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (n[j] <= 1 ? n[i] > 1 : n[i] > 1 && s[j] < s[i]) {
        const int64_t tn = n[i], ts = s[i];
        n[i] = n[j]; s[i] = s[j];
        n[j] = tn; s[j] = ts;
      }
  int64_t least = row;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < least) return false;
    if (s[i] > INT64_MAX / n[i]) return false;
    least = s[i] * n[i];
  }
  return true;
}

// a launch has at most 2^32 work-items: n0 n1 groups, none of which is negative, of 256 of them
bool grid_ok(int64_t n0, int64_t n1) { return n1 == 0 || n0 <= ((int64_t(1) << 24) - 1) / n1; }

}  // namespace

extern "C" {

cover_status cover_rms_norm(const void* x, const void* residual, const void* weight,
                            void* residual_out, void* out, float* scale,
                            const cover_norm_desc* desc, hipStream_t stream) {
  if (!desc) return COVER_ERR_INVALID;
  const cover_norm_desc& D = *desc;
  if (D.R < 0 || D.D < 1 || !known(D.dtype)) return COVER_ERR_INVALID;
  if (!(D.eps >= 0.0f) || isinf(D.eps)) return COVER_ERR_INVALID;  // rejects NaN too
  if (D.D > COVER_NORM_MAX_D) return COVER_ERR_UNSUPPORTED;
  const int64_t esz = D.dtype == COVER_BF16 ? 2 : 4, osz = scale ? 1 : esz;
  if (D.R > 1) {  // a single row has no stride
    if (D.x_stride < D.D || !strides_ok(16 / esz, D.x_stride)) return COVER_ERR_INVALID;
    if (residual && (D.res_stride < D.D || !strides_ok(16 / esz, D.res_stride))) return COVER_ERR_INVALID;
    if (residual_out && (D.res_out_stride < D.D || !strides_ok(16 / esz, D.res_out_stride))) return COVER_ERR_INVALID;
    if (D.out_stride < D.D || !strides_ok(16 / osz, D.out_stride)) return COVER_ERR_INVALID;
  }
  if (D.R == 0) return COVER_OK;
  if (!x || !out || !aligned(x, 16) || !aligned(out, 16)) return COVER_ERR_INVALID;
  if (!aligned(residual, 16) || !aligned(residual_out, 16) || !aligned(weight, 16) || !aligned(scale, 4))
    return COVER_ERR_INVALID;
  // in place only where a row is read and written at the same addresses
  if (D.R > 1 && residual_out && ((residual_out == x && D.res_out_stride != D.x_stride) ||
                                  (residual_out == residual && D.res_out_stride != D.res_stride)))
    return COVER_ERR_INVALID;
  if (out == x && (scale || (D.R > 1 && D.out_stride != D.x_stride))) return COVER_ERR_INVALID;
  if (out == residual || out == residual_out) return COVER_ERR_INVALID;
  cover::NormArgs a;
  a.x = x; a.residual = residual; a.weight = weight; a.residual_out = residual_out; a.out = out; a.scale = scale;
  a.R = D.R; a.D = D.D; a.bf16 = D.dtype == COVER_BF16; a.eps = D.eps;
  a.x_stride = D.x_stride; a.res_stride = D.res_stride; a.res_out_stride = D.res_out_stride;
  a.out_stride = D.out_stride;
  if (!cover::rms_norm_fits(a)) return COVER_ERR_UNSUPPORTED;
  return hip_status(cover::launch_rms_norm(a, stream));
}

cover_status cover_rope_freq(double* freq, int32_t rot, double base, cover_rope_scaling scaling,
                             double factor, double original_length, double low, double high) {
  if (!freq || rot < 2 || rot % 2 != 0) return COVER_ERR_INVALID;
  if (!(base > 1.0) || isinf(base)) return COVER_ERR_INVALID;
  if (scaling < COVER_ROPE_PLAIN || scaling > COVER_ROPE_PARTS) return COVER_ERR_INVALID;
  if (scaling != COVER_ROPE_PLAIN && (!(factor >= 1.0) || isinf(factor))) return COVER_ERR_INVALID;
  if (scaling == COVER_ROPE_BASE && rot < 4) return COVER_ERR_INVALID;
  if (scaling == COVER_ROPE_PARTS && (!(original_length >= 1.0) || isinf(original_length) || !(low < high) ||
                                      isinf(low) || isinf(high)))
    return COVER_ERR_INVALID;
  if (scaling == COVER_ROPE_BASE) base *= pow(factor, (double)rot / (rot - 2));
  if (isinf(base)) return COVER_ERR_INVALID;
  for (int32_t i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot) / 6.283185307179586476925;
    if (scaling == COVER_ROPE_LINEAR) f /= factor;
    if (scaling == COVER_ROPE_PARTS) {
      const double t = (original_length * f - low) / (high - low);
      const double g = t < 0.0 ? 0.0 : (t > 1.0 ? 1.0 : t);
      f *= g + (1.0 - g) / factor;
    }
    freq[i] = f;
  }
  return COVER_OK;
}

cover_status cover_rope(const void* q, const void* k, const int32_t* pos, const double* freq,
                        void* q_out, void* k_out, const cover_rope_desc* desc, hipStream_t stream) {
  if (!desc) return COVER_ERR_INVALID;
  const cover_rope_desc& D = *desc;
  if (D.B < 0 || D.L < 0 || D.Hq < 0 || D.Hkv < 0 || D.d < 1 || !known(D.dtype)) return COVER_ERR_INVALID;
  if (D.rot < 2 || D.rot % 2 != 0 || D.rot > D.d || (D.interleaved != 0 && D.interleaved != 1))
    return COVER_ERR_INVALID;
  if (!isfinite(D.attention_factor) || D.pos_sb < 0) return COVER_ERR_INVALID;
  if (D.d != 64 && D.d != 128) return COVER_ERR_UNSUPPORTED;
  const int64_t vec = D.dtype == COVER_BF16 ? 8 : 4;
  if (D.Hq > 0 && !strides_ok(vec, D.q_sb, D.q_sh, D.q_sl, D.qo_sb, D.qo_sh, D.qo_sl)) return COVER_ERR_INVALID;
  if (D.Hkv > 0 && !strides_ok(vec, D.k_sb, D.k_sh, D.k_sl, D.ko_sb, D.ko_sh, D.ko_sl)) return COVER_ERR_INVALID;
  if (D.B == 0 || D.L == 0 || D.Hq + (int64_t)D.Hkv == 0) return COVER_OK;
  if (D.Hq + (int64_t)D.Hkv > 65536) return COVER_ERR_UNSUPPORTED;
  if (!pos || !aligned(pos, 4) || !freq || !aligned(freq, 8)) return COVER_ERR_INVALID;
  if (D.Hq > 0 && (!q || !q_out || !aligned(q, 16) || !aligned(q_out, 16))) return COVER_ERR_INVALID;
  if (D.Hkv > 0 && (!k || !k_out || !aligned(k, 16) || !aligned(k_out, 16))) return COVER_ERR_INVALID;
  // in place only at the same addresses
  if (D.Hq > 0 && q == q_out && (D.q_sb != D.qo_sb || D.q_sh != D.qo_sh || D.q_sl != D.qo_sl))
    return COVER_ERR_INVALID;
  if (D.Hkv > 0 && k == k_out && (D.k_sb != D.ko_sb || D.k_sh != D.ko_sh || D.k_sl != D.ko_sl))
    return COVER_ERR_INVALID;
  if (D.Hq > 0 && D.Hkv > 0 && (q_out == k_out || q_out == k || k_out == q)) return COVER_ERR_INVALID;
  cover::RopeArgs a;
  a.q = q; a.k = k; a.pos = pos; a.freq = freq; a.q_out = q_out; a.k_out = k_out;
  a.B = D.B; a.L = D.L; a.Hq = D.Hq; a.Hkv = D.Hkv; a.d = D.d; a.rot = D.rot;
  a.interleaved = D.interleaved; a.bf16 = D.dtype == COVER_BF16; a.factor = D.attention_factor;
  a.pos_sb = D.pos_sb;
  a.q_sb = D.q_sb; a.q_sh = D.q_sh; a.q_sl = D.q_sl; a.qo_sb = D.qo_sb; a.qo_sh = D.qo_sh; a.qo_sl = D.qo_sl;
  a.k_sb = D.k_sb; a.k_sh = D.k_sh; a.k_sl = D.k_sl; a.ko_sb = D.ko_sb; a.ko_sh = D.ko_sh; a.ko_sl = D.ko_sl;
  if (!cover::rope_fits(a)) return COVER_ERR_UNSUPPORTED;
  if ((D.Hq > 0 && !apart(D.d, D.L, D.qo_sl, D.Hq, D.qo_sh, D.B, D.qo_sb)) ||
      (D.Hkv > 0 && !apart(D.d, D.L, D.ko_sl, D.Hkv, D.ko_sh, D.B, D.ko_sb)))
    return COVER_ERR_INVALID;
  return hip_status(cover::launch_rope(a, stream));
}

}  // extern "C"

namespace {

// checks shared by cover_cache_store and cover_cache_load; *empty: a valid call with nothing to do
cover_status prepare_cache(const void* k, const void* v, const int32_t* pos, const void* kc, const void* vc,
                           const float* ks, const float* vs, const cover_cache_desc* desc, cover::CacheArgs& a,
                           bool* empty) {
  *empty = false;
  if (!desc) return COVER_ERR_INVALID;
  const cover_cache_desc& D = *desc;
  if (D.B < 0 || D.H < 0 || D.N < 0 || D.L < 1 || D.d < 1 || !known(D.dtype)) return COVER_ERR_INVALID;
  if (D.d != 64 && D.d != 128) return COVER_ERR_UNSUPPORTED;
  if (!pos && (D.first < 0 || (int64_t)D.first + D.N > D.L)) return COVER_ERR_INVALID;
  const int64_t vec = D.dtype == COVER_BF16 ? 8 : 4;
  if (!strides_ok(vec, D.k_sb, D.k_sh, D.k_sl, D.v_sb, D.v_sh, D.v_sl)) return COVER_ERR_INVALID;
  if (!strides_ok(16, D.c_sb, D.c_sh, D.c_sl) || !strides_ok(1, D.s_sb, D.s_sh)) return COVER_ERR_INVALID;
  if (D.L > 1 && D.c_sl < D.d) return COVER_ERR_INVALID;
  if (D.B == 0 || D.H == 0 || D.N == 0) {
    *empty = true;
    return COVER_OK;
  }
  for (const void* t : {k, v, kc, vc})
    if (!t || !aligned(t, 16)) return COVER_ERR_INVALID;
  for (const float* t : {ks, vs})
    if (!t || !aligned(t, 4)) return COVER_ERR_INVALID;
  if (pos && !aligned(pos, 4)) return COVER_ERR_INVALID;
  if (!grid_ok((int64_t)D.B * D.H, ((int64_t)D.N + 15) / 16)) return COVER_ERR_UNSUPPORTED;
  a.k = (void*)k; a.v = (void*)v; a.pos = pos;
  a.kc = (void*)kc; a.vc = (void*)vc; a.ks = (float*)ks; a.vs = (float*)vs;
  a.B = D.B; a.H = D.H; a.N = D.N; a.L = D.L; a.d = D.d; a.first = D.first; a.bf16 = D.dtype == COVER_BF16;
  a.k_sb = D.k_sb; a.k_sh = D.k_sh; a.k_sl = D.k_sl; a.v_sb = D.v_sb; a.v_sh = D.v_sh; a.v_sl = D.v_sl;
  a.c_sb = D.c_sb; a.c_sh = D.c_sh; a.c_sl = D.c_sl; a.s_sb = D.s_sb; a.s_sh = D.s_sh;
  return COVER_OK;
}

}  // namespace

extern "C" {

cover_status cover_cache_store(const void* k, const void* v, const int32_t* pos,
                               void* k_codes, void* v_codes, float* k_scale, float* v_scale,
                               const cover_cache_desc* desc, hipStream_t stream) {
  cover::CacheArgs a;
  bool empty;
  const cover_status st = prepare_cache(k, v, pos, k_codes, v_codes, k_scale, v_scale, desc, a, &empty);
  if (st != COVER_OK || empty) return st;
  if (!apart(a.d, a.L, a.c_sl, a.H, a.c_sh, a.B, a.c_sb) || !apart(a.L, a.H, a.s_sh, a.B, a.s_sb) ||
      k_codes == v_codes || k_scale == v_scale)
    return COVER_ERR_INVALID;
  if (pos && cover::debug_enabled()) {
    const hipError_t e = cover::launch_check_positions(pos, a.B, a.N, a.L, stream);
    if (e != hipSuccess) return COVER_ERR_HIP;
  }
  return hip_status(cover::launch_cache_store(a, stream));
}

cover_status cover_cache_load(void* k, void* v, const int32_t* pos, const void* k_codes,
                              const void* v_codes, const float* k_scale, const float* v_scale,
                              const cover_cache_desc* desc, hipStream_t stream) {
  cover::CacheArgs a;
  bool empty;
  const cover_status st = prepare_cache(k, v, pos, k_codes, v_codes, k_scale, v_scale, desc, a, &empty);
  if (st != COVER_OK || empty) return st;
  if (!apart(a.d, a.N, a.k_sl, a.H, a.k_sh, a.B, a.k_sb) || !apart(a.d, a.N, a.v_sl, a.H, a.v_sh, a.B, a.v_sb) || k == v)
    return COVER_ERR_INVALID;
  return hip_status(cover::launch_cache_load(a, stream));
}

int32_t cover_attn_cached_splits(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t Lq) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || L < 1 || L > COVER_MAX_L || Lq < 1 || Lq > COVER_CACHED_MAX_LQ)
    return 1;
  return cover::attn_cached_splits(B, Hq, Hkv, L, Lq);
}

cover_status cover_attn_cached_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t Lq, int32_t d,
                                    int32_t n_split, int32_t* ranges, int32_t* rows) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || L < 1 || Lq < 1 || d < 1 || n_split < 1 || n_split > 256 ||
      !ranges || !rows)
    return COVER_ERR_INVALID;
  if ((d != 64 && d != 128) || L > COVER_MAX_L || Lq > COVER_CACHED_MAX_LQ) return COVER_ERR_UNSUPPORTED;
  cover::CachedArgs a = {};
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.L = L; a.Lq = Lq; a.d = d; a.n_split = n_split;
  if (!cover::attn_cached_fits(a)) return COVER_ERR_UNSUPPORTED;
  cover::attn_cached_plan(a, ranges, rows);
  return COVER_OK;
}

cover_status cover_attn_cached(const void* q, const void* k_live, const void* v_live,
                               const void* k_codes, const void* v_codes,
                               const float* k_scale, const float* v_scale,
                               const int32_t* off, const int32_t* kv_len,
                               const int32_t* seed_idx, const int32_t* n_seed,
                               void* out, float* lse, float* workspace,
                               const cover_cached_desc* desc, hipStream_t stream) {
  if (!desc) return COVER_ERR_INVALID;
  const cover_cached_desc& D = *desc;
  if (D.B < 0 || D.Hq < 1 || D.Hkv < 1 || D.L < 0 || D.Lq < 0 || D.d < 1 || D.max_seeds < 0)
    return COVER_ERR_INVALID;
  if (D.Hq % D.Hkv != 0) return COVER_ERR_INVALID;
  if (!(D.scale >= 0.0f) || isinf(D.scale)) return COVER_ERR_INVALID;  // rejects NaN too
  if (D.n_split < 1 || D.n_split > 256) return COVER_ERR_INVALID;
  if (!off && (D.q_off < 0 || (int64_t)D.q_off + D.Lq > D.L)) return COVER_ERR_INVALID;
  if (D.d != 64 && D.d != 128) return COVER_ERR_UNSUPPORTED;
  if (D.L > COVER_MAX_L || D.Lq > COVER_CACHED_MAX_LQ) return COVER_ERR_UNSUPPORTED;
  if (D.B == 0 || D.Lq == 0 || D.L == 0) return COVER_OK;
  for (const void* t : {q, k_live, v_live, k_codes, v_codes, (const void*)out})
    if (!t || !aligned(t, 16)) return COVER_ERR_INVALID;
  for (const float* t : {k_scale, v_scale})
    if (!t || !aligned(t, 4)) return COVER_ERR_INVALID;
  if (!aligned(off, 4) || !aligned(kv_len, 4) || !aligned(lse, 4)) return COVER_ERR_INVALID;
  if (!strides_ok(8, D.q_sb, D.q_sh, D.q_sl, D.o_sb, D.o_sh, D.o_sl, D.k_sb, D.k_sh, D.k_sl, D.v_sb, D.v_sh, D.v_sl) ||
      !strides_ok(16, D.c_sb, D.c_sh, D.c_sl) || !strides_ok(1, D.s_sb, D.s_sh))
    return COVER_ERR_INVALID;
  if ((D.Lq > 1 && (D.q_sl < D.d || D.k_sl < D.d || D.v_sl < D.d)) || (D.L > 1 && D.c_sl < D.d))
    return COVER_ERR_INVALID;
  if (D.max_seeds > 0 && (!seed_idx || !n_seed || !aligned(seed_idx, 4) || !aligned(n_seed, 4)))
    return COVER_ERR_INVALID;
  if (D.n_split > 1 && (!workspace || !aligned(workspace, 16))) return COVER_ERR_INVALID;
  cover::CachedArgs a;
  a.q = q; a.k_live = k_live; a.v_live = v_live; a.kc = k_codes; a.vc = v_codes; a.ks = k_scale; a.vs = v_scale;
  a.off = off; a.kv_len = kv_len;
  a.seed_idx = D.max_seeds > 0 ? seed_idx : nullptr;
  a.n_seed = D.max_seeds > 0 ? n_seed : nullptr;
  a.out = out; a.lse = lse; a.workspace = D.n_split > 1 ? workspace : nullptr;
  a.B = D.B; a.Hq = D.Hq; a.Hkv = D.Hkv; a.L = D.L; a.Lq = D.Lq; a.d = D.d; a.max_seeds = D.max_seeds;
  a.q_off = D.q_off; a.n_split = D.n_split;
  a.scale = D.scale > 0.0f ? D.scale : 1.0f / sqrtf((float)D.d);
  a.q_sb = D.q_sb; a.q_sh = D.q_sh; a.q_sl = D.q_sl; a.o_sb = D.o_sb; a.o_sh = D.o_sh; a.o_sl = D.o_sl;
  a.k_sb = D.k_sb; a.k_sh = D.k_sh; a.k_sl = D.k_sl; a.v_sb = D.v_sb; a.v_sh = D.v_sh; a.v_sl = D.v_sl;
  a.c_sb = D.c_sb; a.c_sh = D.c_sh; a.c_sl = D.c_sl; a.s_sb = D.s_sb; a.s_sh = D.s_sh;
  if (!cover::attn_cached_fits(a)) return COVER_ERR_UNSUPPORTED;
  if (!apart(D.d, D.Lq, D.o_sl, D.Hq, D.o_sh, D.B, D.o_sb)) return COVER_ERR_INVALID;
  if (out == q || out == k_live || out == v_live) return COVER_ERR_INVALID;
  if (cover::debug_enabled()) {
    const hipError_t e = cover::launch_check_seeds(a.seed_idx, a.n_seed, D.B, D.max_seeds, D.L, stream);
    if (e != hipSuccess) return COVER_ERR_HIP;
  }
  return hip_status(cover::launch_attn_cached(a, stream));
}

}  // extern "C"
