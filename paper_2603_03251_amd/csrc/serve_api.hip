// C entry points of the operators on the caller's own tensors: argument checks, then one launcher each.
#include <math.h>

#include "serve.h"

using namespace ssd;

namespace ssd {

constexpr double kTwoPi = 6.283185307179586476925;

int rope_scaling(const char* who, const ssd_rope_config* r, int head_dim, RopeScaling* out) {
  SSD_CHECK_ARG(head_dim == 64 || head_dim == 128, "%s: head_dim %d not supported (64 or 128)", who, head_dim);
  SSD_CHECK_ARG(r->rot_dim >= 2 && r->rot_dim <= head_dim && r->rot_dim % 2 == 0, "%s: rot_dim %d must be even, in 2..head_dim", who, r->rot_dim);
  SSD_CHECK_ARG(r->layout == SSD_ROPE_HALF || r->layout == SSD_ROPE_INTERLEAVED, "%s: layout %d unknown", who, r->layout);
  SSD_CHECK_ARG(r->scaling >= SSD_ROPE_PLAIN && r->scaling <= SSD_ROPE_RAMP, "%s: scaling %d unknown", who, r->scaling);
  SSD_CHECK_ARG(r->theta > 1.f && isfinite(r->theta), "%s: theta must be greater than 1", who);
  SSD_CHECK_ARG(r->magnitude > 0.f && isfinite(r->magnitude), "%s: magnitude must be positive", who);
  if (r->scaling != SSD_ROPE_PLAIN) SSD_CHECK_ARG(r->factor > 0.f && isfinite(r->factor), "%s: factor must be positive", who);
  if (r->scaling >= SSD_ROPE_BANDS)
    SSD_CHECK_ARG(r->original > 0.f && isfinite(r->original) && r->low > 0.f && r->high > r->low && isfinite(r->high),
                  "%s: original > 0 and 0 < low < high required", who);
  *out = {r->scaling, r->factor, r->low, r->high, r->original, r->magnitude, 0.f, 0.f};
  if (r->scaling == SSD_ROPE_RAMP) {
    const double per_log = r->rot_dim / (2.0 * log((double)r->theta));
    out->i0 = (float)fmax(floor(per_log * log((double)r->original / (kTwoPi * r->high))), 0.0);
    out->i1 = (float)fmin(ceil(per_log * log((double)r->original / (kTwoPi * r->low))), r->rot_dim - 1.0);
  }
  return SSD_OK;
}

// Turns per position of every pair, in fp64.
void rope_turns(float theta, int rot, const RopeScaling& scaling, RopeTurns* out) {
  const double log2_theta = log2((double)theta);
  for (int i = 0; i < kMaxPairs; ++i) {
    const double t = i < rot / 2 ? exp2(-2.0 * i / rot * log2_theta) / kTwoPi : 0.0;
    out->turns[i] = t * rope_share(scaling, t, i);
  }
}

}  // namespace ssd

namespace {

int check_paged_kv(const char* who, const ssd_paged_kv* kv) {
  SSD_CHECK_ARG(kv->d_k && kv->d_v && kv->d_table, "%s: null pointer in the cache", who);
  SSD_CHECK_ARG(kv->dtype == SSD_F32 || kv->dtype == SSD_BF16, "%s: cache dtype %d unknown", who, kv->dtype);
  SSD_CHECK_ARG(kv->head_dim == 64 || kv->head_dim == 128, "%s: head_dim %d not supported (64 or 128)", who, kv->head_dim);
  SSD_CHECK_ARG(kv->n_kv_heads >= 1 && kv->n_kv_heads <= 1024, "%s: n_kv_heads must be in 1..1024", who);
  SSD_CHECK_ARG(kv->page_size >= 8 && kv->page_size <= 1024 && (kv->page_size & (kv->page_size - 1)) == 0,
                "%s: page_size %d must be a power of two in 8..1024", who, kv->page_size);
  SSD_CHECK_ARG(kv->n_pages >= 1 && kv->table_stride >= 1, "%s: n_pages and table_stride must be at least 1", who);
  const int per16 = kv->dtype == SSD_BF16 ? 8 : 4;
  SSD_CHECK_ARG(kv->page_stride >= (int64_t)kv->page_size * kv->n_kv_heads * kv->head_dim && kv->page_stride % per16 == 0 &&
                    kv->page_stride <= (1 << 29),
                "%s: page_stride must hold a page, be a multiple of 16 bytes and at most 2^29", who);
  SSD_CHECK_ARG((((uintptr_t)kv->d_k | (uintptr_t)kv->d_v) & 15) == 0, "%s: the cache must start on 16 bytes", who);
  return SSD_OK;
}

bool dtype_ok(int32_t d) { return d == SSD_F32 || d == SSD_BF16; }
size_t elem_bytes(int32_t d) { return d == SSD_BF16 ? 2 : 4; }

}  // namespace

extern "C" {

int ssd_rope(const ssd_rope_config* rope, const void* d_x, int64_t x_ld, int32_t dtype, const int32_t* d_positions, int32_t rows,
             int32_t n_heads, int32_t head_dim, void* d_out, int64_t out_ld, void* stream) {
  SSD_CHECK_ARG(rope && (rows == 0 || (d_x && d_positions && d_out)), "ssd_rope: null argument");
  RopeScaling scaling;
  SSD_TRY(rope_scaling("ssd_rope", rope, head_dim, &scaling));
  SSD_CHECK_ARG(dtype_ok(dtype), "ssd_rope: dtype %d unknown", dtype);
  SSD_CHECK_ARG(rows >= 0 && rows <= (1 << 24) && n_heads >= 1 && n_heads <= 1024 && (int64_t)rows * n_heads <= (1 << 28),
                "ssd_rope: rows in 0..2^24, n_heads in 1..1024 and at most 2^28 of both together required");
  SSD_CHECK_ARG(x_ld >= (int64_t)n_heads * head_dim && out_ld >= (int64_t)n_heads * head_dim, "ssd_rope: a row must hold its heads");
  RopeTurns turns;
  rope_turns(rope->theta, rope->rot_dim, scaling, &turns);
  RopeArgs a = {};
  a.q = d_x; a.q_ld = x_ld; a.q_out = d_out; a.q_out_ld = out_ld;
  a.positions = d_positions; a.row_step = 1; a.rows = rows; a.rows_per_seq = 1;
  a.n_q = n_heads; a.head_dim = head_dim; a.rot = rope->rot_dim; a.interleaved = rope->layout == SSD_ROPE_INTERLEAVED;
  a.magnitude = rope->magnitude;
  return launch_rope(dtype, dtype, a, turns, (hipStream_t)stream);
}

int ssd_rope_append(const ssd_rope_config* rope, const ssd_paged_kv* kv, const void* d_q, int64_t q_ld, const void* d_k, int64_t k_ld,
                    const void* d_v, int64_t v_ld, int32_t dtype, const int32_t* d_positions, const int32_t* d_slots, int32_t B, int32_t T,
                    int32_t n_q_heads, void* d_q_out, int64_t q_out_ld, void* stream) {
  SSD_CHECK_ARG(rope && kv && (B == 0 || (d_q && d_k && d_v && d_positions && d_q_out)), "ssd_rope_append: null argument");
  SSD_TRY(check_paged_kv("ssd_rope_append", kv));
  RopeScaling scaling;
  SSD_TRY(rope_scaling("ssd_rope_append", rope, kv->head_dim, &scaling));
  SSD_CHECK_ARG(dtype_ok(dtype), "ssd_rope_append: dtype %d unknown", dtype);
  SSD_CHECK_ARG(B >= 0 && T >= 1 && (int64_t)B * T <= (1 << 24), "ssd_rope_append: B >= 0, T >= 1 and at most 2^24 rows required");
  SSD_CHECK_ARG(n_q_heads >= 1 && n_q_heads <= 1024 && (int64_t)B * T * (n_q_heads + 2 * kv->n_kv_heads) <= (1 << 28),
                "ssd_rope_append: n_q_heads in 1..1024 and at most 2^28 rows x heads required");
  const int64_t qd = (int64_t)n_q_heads * kv->head_dim, kvd = (int64_t)kv->n_kv_heads * kv->head_dim;
  SSD_CHECK_ARG(q_ld >= qd && q_out_ld >= qd && k_ld >= kvd && v_ld >= kvd, "ssd_rope_append: a row must hold its heads");
  RopeTurns turns;
  rope_turns(rope->theta, rope->rot_dim, scaling, &turns);
  RopeArgs a = {};
  a.q = d_q; a.q_ld = q_ld; a.k = d_k; a.k_ld = k_ld; a.v = d_v; a.v_ld = v_ld; a.q_out = d_q_out; a.q_out_ld = q_out_ld;
  a.positions = d_positions; a.slots = d_slots ? d_slots : d_positions; a.row_step = 1; a.rows = B * T; a.rows_per_seq = T;
  a.n_q = n_q_heads; a.n_kv = kv->n_kv_heads; a.head_dim = kv->head_dim; a.rot = rope->rot_dim;
  a.interleaved = rope->layout == SSD_ROPE_INTERLEAVED; a.magnitude = rope->magnitude;
  a.pool_k = kv->d_k; a.pool_v = kv->d_v; a.table = kv->d_table; a.page_stride = kv->page_stride;
  a.n_pages = kv->n_pages; a.page_size = kv->page_size; a.table_stride = kv->table_stride;
  return launch_rope(dtype, kv->dtype, a, turns, (hipStream_t)stream);
}

size_t ssd_paged_attention_workspace_bytes(const ssd_paged_kv* kv, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_visible) {
  if (!kv || B < 1 || T < 1 || n_q_heads < 1 || kv->n_kv_heads < 1 || n_q_heads % kv->n_kv_heads != 0 || max_visible < 0 ||
      (int64_t)B * T > (1 << 24))
    return 0;
  return paged_attention_workspace(B, T, n_q_heads, kv->n_kv_heads, kv->head_dim, max_visible);
}

int ssd_paged_attention(const ssd_paged_kv* kv, const void* d_q, int64_t q_ld, int32_t dtype, const int32_t* d_visible, int32_t B, int32_t T,
                        int32_t n_q_heads, int32_t max_visible, float scale, const ssd_tail_kv* tail, void* d_out, int64_t out_ld,
                        float* d_lse, void* d_workspace, void* stream) {
  SSD_CHECK_ARG(kv && (B == 0 || (d_q && d_visible && d_out && d_workspace)), "ssd_paged_attention: null argument");
  SSD_TRY(check_paged_kv("ssd_paged_attention", kv));
  SSD_CHECK_ARG(dtype_ok(dtype), "ssd_paged_attention: dtype %d unknown", dtype);
  SSD_CHECK_ARG(n_q_heads >= 1 && n_q_heads <= 1024 && n_q_heads % kv->n_kv_heads == 0,
                "ssd_paged_attention: n_q_heads must be a multiple of n_kv_heads, at most 1024");
  SSD_CHECK_ARG(B >= 0 && B <= 65535 && T >= 1 && T <= 65535 && (int64_t)B * T * n_q_heads <= (1 << 23) &&
                    (int64_t)T * (n_q_heads / kv->n_kv_heads) <= 16 * 65535,
                "ssd_paged_attention: B in 0..65535, T in 1..65535, at most 2^23 rows x heads and 16 x 65535 rows x heads of a KV head and sequence required");
  SSD_CHECK_ARG(max_visible >= 0 && max_visible <= (1 << 30) && max_visible <= (int64_t)kv->table_stride * kv->page_size,
                "ssd_paged_attention: max_visible %d exceeds the block table", max_visible);
  SSD_CHECK_ARG(isfinite(scale), "ssd_paged_attention: scale must be finite");
  const int64_t qd = (int64_t)n_q_heads * kv->head_dim, row16 = 16 / (int64_t)elem_bytes(dtype);
  SSD_CHECK_ARG(q_ld >= qd && out_ld >= qd, "ssd_paged_attention: a row must hold its heads");
  SSD_CHECK_ARG((((uintptr_t)d_q | (uintptr_t)d_out | (uintptr_t)d_workspace) & 15) == 0 && q_ld % row16 == 0 && out_ld % row16 == 0,
                "ssd_paged_attention: queries, output, their rows and the workspace must start on 16 bytes");
  PagedAttnArgs a = {};
  if (tail) {
    SSD_CHECK_ARG(tail->d_k && tail->d_v, "ssd_paged_attention: null pointer in the tail");
    SSD_CHECK_ARG(tail->capacity >= 1 && tail->capacity <= 256 && tail->length >= 0 && tail->length <= tail->capacity,
                  "ssd_paged_attention: a tail holds 1..256 positions, of which 0..capacity are seen");
    a.tail_k = tail->d_k; a.tail_v = tail->d_v; a.tail_cap = tail->capacity; a.tail_len = tail->length;
  }
  if (B == 0) return SSD_OK;
  a.q = d_q; a.q_ld = q_ld; a.k = kv->d_k; a.v = kv->d_v; a.table = kv->d_table; a.page_stride = kv->page_stride;
  a.n_pages = kv->n_pages; a.page_shift = __builtin_ctz((unsigned)kv->page_size); a.table_stride = kv->table_stride;
  a.visible = d_visible; a.vis_step = 1; a.B = B; a.T = T; a.n_q = n_q_heads; a.n_kv = kv->n_kv_heads; a.head_dim = kv->head_dim;
  a.max_visible = max_visible; a.scale_log2 = scale * 1.44269504088896341f;
  a.out = d_out; a.out_ld = out_ld; a.lse = d_lse; a.workspace = d_workspace;
  return launch_paged_attention(dtype, kv->dtype, a, (hipStream_t)stream);
}

size_t ssd_verify_probs_workspace_bytes(int32_t B, int32_t V) { return B >= 1 && V >= 1 ? verify_probs_workspace(B, V) : 0; }

int ssd_verify_probs(const float* d_target_probs, int64_t target_ld, const float* d_draft_probs, int64_t draft_ld, const int32_t* d_spec_tokens,
                     const int32_t* d_drafted, const float* d_u_accept, const float* d_u_bonus, int32_t B, int32_t K, int32_t V,
                     int32_t* d_accept_len, int32_t* d_bonus, void* d_workspace, void* stream) {
  SSD_CHECK_ARG(B == 0 || (d_target_probs && d_spec_tokens && d_u_accept && d_u_bonus && d_accept_len && d_bonus && d_workspace),
                "ssd_verify_probs: null argument");
  SSD_CHECK_ARG(B >= 0 && B <= 65535 && K >= 1 && K <= SSD_MAX_K && V >= 2 && V <= (1 << 30),
                "ssd_verify_probs: 0 <= B <= 65535, 1 <= K <= %d, 2 <= V <= 2^30 required", SSD_MAX_K);
  SSD_CHECK_ARG(target_ld >= V && (!d_draft_probs || draft_ld >= V), "ssd_verify_probs: a row must hold V probabilities");
  SSD_CHECK_ARG(((uintptr_t)d_workspace & 15) == 0, "ssd_verify_probs: the workspace must start on 16 bytes");
  if (B == 0) return SSD_OK;
  VerifyProbsArgs a = {};
  a.target = d_target_probs; a.target_ld = target_ld; a.draft = d_draft_probs; a.draft_ld = draft_ld; a.spec = d_spec_tokens;
  a.drafted = d_drafted; a.u_accept = d_u_accept; a.u_bonus = d_u_bonus; a.B = B; a.K = K; a.V = V;
  a.accept_len = d_accept_len; a.bonus = d_bonus; a.workspace = d_workspace;
  return launch_verify_probs(a, (hipStream_t)stream);
}

}  // extern "C"
