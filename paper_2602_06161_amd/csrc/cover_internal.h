// Internal launch interface between the C ABI (api.cpp) and the HIP kernels.
// Host-validated arguments only: every entry here assumes the descriptor checks passed.
#pragma once
#include <stdint.h>
#include <hip/hip_runtime_api.h>

namespace cover {

struct AttnArgs {
  const void* q;
  const void* k_live;
  const void* v_live;
  const void* k_cache;
  const void* v_cache;
  const int32_t* seed_idx;  // may be null when max_seeds == 0
  const int32_t* n_seed;    // may be null when max_seeds == 0
  void* out;
  float* lse;               // may be null
  int32_t B, Hq, Hkv, L, d, max_seeds;
  float scale;              // > 0
  int64_t q_sb, q_sh, q_sl, kv_sb, kv_sh, kv_sl;
};

struct SelectArgs {
  const float* logp;
  const float* d_in;
  const float* d_out;
  const uint8_t* flags;
  int32_t* seed_idx;
  int32_t* n_seed;
  double* score;  // may be null
  int32_t B, Lr, max_seeds, pos_offset;
};

struct TokenArgs {
  const void* logits;
  const int32_t* tokens;  // may be null when logp is null
  float* logp;            // may be null
  float* conf;            // may be null
  int32_t* argmax;        // may be null
  int32_t R, V;
  int bf16;               // element type of logits: bf16 (1) or fp32 (0)
  int64_t row_stride;     // elements
};

struct SampleArgs {
  const void* logits;
  int32_t* token;
  float* prob;  // may be null
  int32_t R, V;
  int bf16;
  int64_t row_stride;  // elements
  float temperature;   // > 0
  uint64_t seed;
  uint32_t step;
};

struct StatsArgs {
  const void* q;
  const void* k_live;
  const void* k_cache;
  const int32_t* seed_idx;  // may be null when max_seeds == 0
  const int32_t* n_seed;    // may be null when max_seeds == 0
  const float* lse;
  const uint8_t* masked;
  const uint8_t* drafted;
  float* d_in;
  float* d_out;
  float* workspace;
  int32_t B, Hq, Hkv, L, d, max_seeds, r0, Lr;
  float scale;  // > 0
  int64_t q_sb, q_sh, q_sl, kv_sb, kv_sh, kv_sl;
};

struct RectArgs {
  const void* q;
  const void* k_live;
  const void* v_live;
  const void* k_cache;
  const void* v_cache;
  const int32_t* seed_idx;  // may be null when max_seeds == 0
  const int32_t* n_seed;    // may be null when max_seeds == 0
  void* out;
  float* lse;  // may be null
  float* workspace;
  int32_t B, Hq, Hkv, L, d, max_seeds, q_off, Lq, n_split;
  float scale;  // > 0
  int64_t q_sb, q_sh, q_sl, kv_sb, kv_sh, kv_sl;
};

struct UpdateArgs {
  int32_t* tokens;
  const int32_t* argmax;
  const float* conf;
  const int32_t* seed_idx;  // may be null when max_seeds == 0
  const int32_t* n_seed;    // may be null when max_seeds == 0
  int32_t* remask_count;
  uint8_t* flags;    // may be null
  uint8_t* drafted;  // may be null
  int32_t* counts;   // may be null
  int32_t* last_unmask;  // may be null
  int32_t* flipflops;    // may be null (always null when last_unmask is)
  int32_t B, Lr, max_seeds, pos_offset, mask_id, draft_cap, remask_budget;
  float tau;
  int32_t min_draft;
};

struct NormArgs {
  const void* x;
  const void* residual;  // may be null
  const void* weight;    // may be null
  void* residual_out;    // may be null
  void* out;             // e4m3 codes where scale is given
  float* scale;          // may be null
  int32_t R, D;
  int bf16;  // element type of the tensors: bf16 (1) or fp32 (0)
  float eps;
  int64_t x_stride, res_stride, res_out_stride, out_stride;  // elements
};

struct RopeArgs {
  const void* q;
  const void* k;
  const int32_t* pos;
  const double* freq;
  void* q_out;
  void* k_out;
  int32_t B, L, Hq, Hkv, d, rot, interleaved;
  int bf16;
  float factor;
  int64_t pos_sb;
  int64_t q_sb, q_sh, q_sl, qo_sb, qo_sh, qo_sl, k_sb, k_sh, k_sl, ko_sb, ko_sh, ko_sl;
};

struct CacheArgs {
  void* k;  // read by the store, written by the load
  void* v;
  const int32_t* pos;  // may be null: rows first, first + 1, ...
  void* kc;
  void* vc;
  float* ks;
  float* vs;
  int32_t B, H, N, L, d, first;
  int bf16;
  int64_t k_sb, k_sh, k_sl, v_sb, v_sh, v_sl, c_sb, c_sh, c_sl, s_sb, s_sh;
};

struct CachedArgs {
  const void* q;
  const void* k_live;
  const void* v_live;
  const void* kc;
  const void* vc;
  const float* ks;
  const float* vs;
  const int32_t* off;       // may be null: q_off
  const int32_t* kv_len;    // may be null: L
  const int32_t* seed_idx;  // may be null when max_seeds == 0
  const int32_t* n_seed;    // may be null when max_seeds == 0
  void* out;
  float* lse;        // may be null
  float* workspace;  // null when n_split == 1
  int32_t B, Hq, Hkv, L, Lq, d, max_seeds, q_off, n_split;
  float scale;  // > 0
  int64_t q_sb, q_sh, q_sl, o_sb, o_sh, o_sl;
  int64_t k_sb, k_sh, k_sl, v_sb, v_sh, v_sl, c_sb, c_sh, c_sl, s_sb, s_sh;
};

hipError_t launch_attn_bf16(const AttnArgs& a, hipStream_t stream);  // bf16, d = 64 or 128
hipError_t launch_attn_f32(const AttnArgs& a, hipStream_t stream);
hipError_t launch_select(const SelectArgs& a, hipStream_t stream);
hipError_t launch_token_stats(const TokenArgs& a, hipStream_t stream);
hipError_t launch_token_sample(const SampleArgs& a, hipStream_t stream);
hipError_t launch_attn_stats(const StatsArgs& a, hipStream_t stream);
// workgroups per head of the attention-mass launch (32-position tiles per workgroup, workgroups),
// and the workspace floats a caller of that launch provides: 1 + workgroups rows per head, of which
// the launch uses two, d_in and d_out (the size callers have been told to provide is kept)
void stats_key_groups(int B, int Hq, int Lr, int* tpg, int* kg);
int64_t stats_workspace_floats(int B, int Hq, int Lr);
// device address of the attention-mass kernels' own static scratch array on the current GPU
// (COVER_STATS_SCRATCH_FLOATS floats), looked up once per device
hipError_t stats_scratch(float** ptr);
hipError_t launch_decode_update(const UpdateArgs& a, hipStream_t stream);
hipError_t launch_attn_rect(const RectArgs& a, hipStream_t stream);  // bf16, d = 128 (n_split 1: or 64)
bool attn_small(const AttnArgs& a);  // a square call better served by launch_attn_rect (bf16)
bool rms_norm_fits(const NormArgs& a);  // in one launch
hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream);
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);
bool rope_fits(const RopeArgs& a);  // its grid is within a launch's limit
hipError_t launch_cache_store(const CacheArgs& a, hipStream_t stream);
hipError_t launch_cache_load(const CacheArgs& a, hipStream_t stream);
hipError_t launch_attn_cached(const CachedArgs& a, hipStream_t stream);
bool attn_cached_fits(const CachedArgs& a);  // its grids are within a launch's limit
int attn_cached_splits(int B, int Hq, int Hkv, int L, int Lq);  // the n_split that suits a call
void attn_cached_plan(const CachedArgs& a, int* n_ranges, int* rows);  // key ranges, query rows per workgroup

// contract checks (COVER_DEBUG=1)
bool debug_enabled();
hipError_t launch_check_seeds(const int32_t* seed_idx, const int32_t* n_seed, int B, int max_seeds,
                              int L, hipStream_t stream);
hipError_t launch_check_select(const float* logp, const float* d_in, const float* d_out,
                               const uint8_t* flags, int64_t n, hipStream_t stream);
hipError_t launch_check_positions(const int32_t* pos, int B, int N, int L, hipStream_t stream);
hipError_t debug_status(int32_t* status, bool clear, hipStream_t stream);

}  // namespace cover
