// What the operators on the caller's own tensors hand to their kernels: rotary positions and the append to a paged cache, attention
// over it, verification from given probabilities.
#pragma once

#include "common.h"

namespace ssd {

constexpr int kMaxPairs = 64;   // pairs of a head: head_dim is at most 128

// Turns (angle / 2 pi) a pair makes per position.
struct RopeTurns {
  double turns[kMaxPairs];
};

// Row r of q is at q + r q_ld, its heads one behind the other; k, v and q_out likewise.  Position and slot of row r: positions and
// slots [r row_step].  Row r belongs to sequence r / rows_per_seq.
struct RopeArgs {
  const void *q, *k, *v;
  int64_t q_ld, k_ld, v_ld;
  void* q_out;
  int64_t q_out_ld;
  const int32_t *positions, *slots;
  int row_step, rows, rows_per_seq;
  int n_q, n_kv, head_dim, rot, interleaved;
  float magnitude;
  // the cache; table null: page r belongs to row r alone
  void *pool_k, *pool_v;
  const int32_t* table;
  int64_t page_stride;
  int n_pages, page_size, table_stride;
  int head_groups;   // set by the launcher
};
// The settings as the kernels take them; EINVAL (and a message that starts with `who`) where they make no rotation.
int rope_scaling(const char* who, const ssd_rope_config* r, int head_dim, RopeScaling* out);
void rope_turns(float theta, int rot, const RopeScaling& scaling, RopeTurns* out);
int launch_rope(int dtype, int cache_dtype, const RopeArgs& a, const RopeTurns& f, hipStream_t s);

// Rows b T .. b T + T - 1 are sequence b's; row r sees positions 0 .. visible[r vis_step] - 1 of its pages, at most max_visible, and
// the first tail_len of its tail's tail_cap positions.
struct PagedAttnArgs {
  const void* q;
  int64_t q_ld;
  const void *k, *v;         // pools
  const int32_t* table;
  int64_t page_stride;
  int n_pages, page_shift, table_stride;
  const int32_t* visible;
  int vis_step;
  int B, T, n_q, n_kv, head_dim, max_visible;
  float scale_log2;          // scores are taken in powers of two
  const void *tail_k, *tail_v;
  int tail_cap, tail_len;
  void* out;
  int64_t out_ld, out_plane; // out_plane > 0: two bf16 planes that far apart (head and remainder) instead of the queries' type
  float* lse;
  void* workspace;
};
int launch_paged_attention(int dtype, int cache_dtype, const PagedAttnArgs& a, hipStream_t s);
size_t paged_attention_workspace(int B, int T, int n_q, int n_kv, int head_dim, int max_visible);
// enough for any max_visible up to this one, which may change from call to call
size_t paged_attention_workspace_bound(int B, int T, int n_q, int n_kv, int head_dim, int max_visible);

struct VerifyProbsArgs {
  const float *target, *draft;   // [B][K + 1][V] and [B][K][V], rows target_ld and draft_ld apart; draft null: the tokens were certain
  int64_t target_ld, draft_ld;
  const int32_t *spec, *drafted; // [B][K]; [B] or null
  const float *u_accept, *u_bonus;
  int B, K, V;
  int32_t *accept_len, *bonus;
  void* workspace;
};
int launch_verify_probs(const VerifyProbsArgs& a, hipStream_t s);
size_t verify_probs_workspace(int B, int V);

}  // namespace ssd
