// C entry points of the operators around the blocks (include/merak_stage.h):
// embedding, query/key norm with rotation, 8-bit activation checkpoints, residual norm,
// distillation loss.
// Arguments are checked here, before anything is enqueued.
#include <cmath>
#include <initializer_list>

#include "abi.h"
#include "kernels.h"

using namespace merak;

namespace {

int check_dtype(int dtype) { return dtype == MERAK_BF16 || dtype == MERAK_FP32 ? MERAK_OK : MERAK_ERR_INVALID_ARG; }
int check_flag(int f) { return f == 0 || f == 1 ? MERAK_OK : MERAK_ERR_INVALID_ARG; }

// A call that needs more workgroups than a launch can have is refused by its launcher, before
// anything is enqueued.
#define LAUNCH_TRY(expr)                                                  \
  do {                                                                    \
    const hipError_t e_ = (expr);                                         \
    if (e_ == hipErrorInvalidConfiguration) return MERAK_ERR_SHAPE;       \
    if (e_ != hipSuccess) return MERAK_ERR_HIP;                           \
  } while (0)

// A call's arrays: what it writes must not overlap anything else it uses.
struct Span {
  const void* p;
  size_t bytes;
};

int check_apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  auto meet = [](const Span& a, const Span& b) {
    const uintptr_t p = (uintptr_t)a.p, q = (uintptr_t)b.p;
    return p && q && a.bytes && b.bytes && p < q + b.bytes && q < p + a.bytes;
  };
  for (const Span* a = written.begin(); a != written.end(); ++a) {
    for (const Span* b = written.begin(); b != a; ++b)
      if (meet(*a, *b)) return MERAK_ERR_INVALID_ARG;
    for (const Span& b : read)
      if (meet(*a, b)) return MERAK_ERR_INVALID_ARG;
  }
  return MERAK_OK;
}

size_t elem(int dtype) { return dtype == MERAK_BF16 ? 2 : 4; }

// Tokens of one embedding gradient: sorting compares every pair of 2048-token blocks.
constexpr int kMaxSorted = 1 << 22;
constexpr int kMaxRows = 1 << 30;  // tokens and table rows: the kernels count them in 32 bits

size_t id_bytes(int id_type) { return id_type == MERAK_I32 ? 4 : 8; }

int check_embedding(int dtype, int id_type, int tokens, int hidden, int rows, int64_t first, float scale) {
  TRY(check_dtype(dtype));
  if (id_type != MERAK_I32 && id_type != MERAK_I64) return MERAK_ERR_INVALID_ARG;
  if (tokens <= 0 || hidden <= 0 || rows <= 0 || hidden % 8) return MERAK_ERR_SHAPE;
  if (tokens > kMaxRows || rows > kMaxRows || hidden > (1 << 20)) return MERAK_ERR_SHAPE;
  // the last row's id is an int64 too: the kernels form id - first in 64 bits
  if (first < 0 || first > INT64_MAX - (rows - 1) || !std::isfinite(scale)) return MERAK_ERR_INVALID_ARG;
  return MERAK_OK;
}

int check_qk(int dtype, int tokens, int q_heads, int kv_heads, int head_dim, int rope_dim, int interleaved, float eps,
             const float* table, int table_rows, const int32_t* positions, int seq_len) {
  TRY(check_dtype(dtype));
  TRY(check_flag(interleaved));
  if (tokens <= 0 || tokens > kMaxRows || q_heads <= 0 || kv_heads <= 0 || q_heads > 4096 || kv_heads > 4096 ||
      head_dim <= 0)
    return MERAK_ERR_SHAPE;
  if (head_dim % 8 || rope_dim < 0 || rope_dim > head_dim || rope_dim % 16) return MERAK_ERR_SHAPE;
  if (head_dim > 256) return MERAK_ERR_UNSUPPORTED;
  if (!(eps > 0.0f) || !std::isfinite(eps)) return MERAK_ERR_SHAPE;
  if (rope_dim > 0) {
    TRY(check_ptr(table));
    if (table_rows <= 0) return MERAK_ERR_SHAPE;
    if (positions) TRY(check_ptr(positions));
    else if (seq_len <= 0 || seq_len > table_rows) return MERAK_ERR_SHAPE;
  }
  return MERAK_OK;
}

size_t qk_row_bytes(const QkShape& q, int dtype) {
  return (size_t)q.tokens * (q.q_heads + 2 * q.kv_heads) * q.head_dim * elem(dtype);
}

// What the calls of a shape read besides the rows.
Span table_span(const QkShape& q) { return {q.table, q.rope_dim > 0 ? (size_t)q.table_rows * q.rope_dim * 4 : 0}; }
Span position_span(const QkShape& q) { return {q.positions, q.rope_dim > 0 ? (size_t)q.tokens * 4 : 0}; }

int check_act8(int dtype, int rows, int cols, const uint8_t* q, const uint8_t* scales) {
  TRY(check_dtype(dtype));
  if (rows <= 0 || cols <= 0 || cols % 32) return MERAK_ERR_SHAPE;
  if ((int64_t)rows * cols > (int64_t)1 << 40) return MERAK_ERR_SHAPE;
  TRY(check_ptr(q));
  return check_ptr(scales);
}

int check_norm(int dtype, int rows, int cols, float eps) {
  TRY(check_dtype(dtype));
  if (rows <= 0 || rows > kMaxRows || cols <= 0 || cols % 8) return MERAK_ERR_SHAPE;
  if (cols > kMaxNormCols) return MERAK_ERR_UNSUPPORTED;
  return eps > 0.0f && std::isfinite(eps) ? MERAK_OK : MERAK_ERR_SHAPE;
}

int check_mix(float alpha, float tau) {
  // (the kernels' exponentials are made for these temperatures)
  if (!(alpha >= 0.0f && alpha <= 1.0f) || !(tau >= 0x1p-10f && tau <= 0x1p10f)) return MERAK_ERR_INVALID_ARG;
  return MERAK_OK;
}

int check_id_type(int t) { return t == MERAK_I32 || t == MERAK_I64 ? MERAK_OK : MERAK_ERR_INVALID_ARG; }

// The loss's terms that have a weight; the arrays of another one are not looked at.
bool has_teacher(const DistillShape& q) { return q.top > 0 && q.alpha > 0.0f; }
bool has_labels(const DistillShape& q) { return q.labels && q.alpha < 1.0f; }

int check_distill(int dtype, const DistillShape& q, const void* logits) {
  TRY(check_dtype(dtype));
  TRY(check_mix(q.alpha, q.tau));
  if (q.tokens <= 0 || q.tokens > kMaxRows || q.vocab <= 0 || q.ld < q.vocab || q.ld % 8 || q.ld > (1 << 28) ||
      q.top < 0 || q.top > kMaxTop)
    return MERAK_ERR_SHAPE;
  if (q.first < 0 || q.total < q.vocab || q.first > q.total - q.vocab) return MERAK_ERR_INVALID_ARG;
  TRY(check_ptr(logits));
  if (has_teacher(q)) {
    TRY(check_id_type(q.id_type));
    TRY(check_dtype(q.teacher_type));
    TRY(check_ptr(q.ids)); TRY(check_ptr(q.teacher));
  }
  if (has_labels(q)) {
    TRY(check_id_type(q.label_type));
    TRY(check_ptr(q.labels));
  }
  return has_teacher(q) || has_labels(q) ? MERAK_OK : MERAK_ERR_INVALID_ARG;  // else nothing to learn from
}

size_t logits_bytes(int dtype, const DistillShape& q) { return (size_t)q.tokens * q.ld * elem(dtype); }
size_t stats_bytes(int tokens) { return (size_t)tokens * kDistillStats * sizeof(float); }
Span ids_span(const DistillShape& q) {
  return {q.ids, has_teacher(q) ? (size_t)q.tokens * q.top * id_bytes(q.id_type) : 0};
}
Span teacher_span(const DistillShape& q) {
  return {q.teacher, has_teacher(q) ? (size_t)q.tokens * q.top * elem(q.teacher_type) : 0};
}
Span labels_span(const DistillShape& q) {
  return {q.labels, has_labels(q) ? (size_t)q.tokens * id_bytes(q.label_type) : 0};
}

}  // namespace

extern "C" {

int merak_embedding_fwd(int dtype, int id_type, int tokens, int hidden, int table_rows, int64_t first_id, float scale,
                        const void* ids, const void* table, void* y, void* stream) {
  TRY(check_embedding(dtype, id_type, tokens, hidden, table_rows, first_id, scale));
  TRY(check_ptr(ids)); TRY(check_ptr(table)); TRY(check_ptr(y));
  const size_t row = hidden * elem(dtype);
  TRY(check_apart({{y, tokens * row}}, {{ids, tokens * id_bytes(id_type)}, {table, table_rows * row}}));
  LAUNCH_TRY(launch_embedding_fwd(dtype, id_type, tokens, hidden, table_rows, first_id, scale, ids, table, y,
                                  (hipStream_t)stream));
  return MERAK_OK;
}

size_t merak_embedding_scratch_bytes(int tokens, int hidden) {
  if (tokens <= 0 || hidden <= 0) return 0;
  return embedding_scratch_bytes(tokens, hidden);
}

int merak_embedding_bwd(int dtype, int id_type, int tokens, int hidden, int table_rows, int64_t first_id, float scale,
                        const void* ids, const void* dy, float* dtable, int accumulate, void* scratch, void* stream) {
  TRY(check_embedding(dtype, id_type, tokens, hidden, table_rows, first_id, scale));
  if (tokens > kMaxSorted) return MERAK_ERR_SHAPE;
  TRY(check_flag(accumulate));
  TRY(check_ptr(ids)); TRY(check_ptr(dy)); TRY(check_ptr(dtable));
  const size_t sb = merak_embedding_scratch_bytes(tokens, hidden);
  if (sb > 0) TRY(check_ptr(scratch));
  TRY(check_apart({{dtable, (size_t)table_rows * hidden * 4}, {scratch, sb}},
                  {{ids, tokens * id_bytes(id_type)}, {dy, (size_t)tokens * hidden * elem(dtype)}}));
  LAUNCH_TRY(launch_embedding_bwd(dtype, id_type, tokens, hidden, table_rows, first_id, scale, ids, dy, dtable,
                                  accumulate, scratch, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_rope_table(int positions, int rope_dim, double theta, float* table, void* stream) {
  if (positions <= 0 || rope_dim <= 0 || rope_dim % 16 || rope_dim > 256) return MERAK_ERR_SHAPE;
  if (!(theta > 0.0) || !std::isfinite(theta)) return MERAK_ERR_INVALID_ARG;
  TRY(check_ptr(table));
  LAUNCH_TRY(launch_rope_table(positions, rope_dim, theta, table, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_qk_norm_rope_fwd(int dtype, int tokens, int q_heads, int kv_heads, int head_dim, int rope_dim,
                           int interleaved, float eps, const void* qkv, const void* q_gamma, const void* k_gamma,
                           const float* table, int table_rows, const int32_t* positions, int seq_len, void* out,
                           void* stream) {
  TRY(check_qk(dtype, tokens, q_heads, kv_heads, head_dim, rope_dim, interleaved, eps, table, table_rows, positions,
               seq_len));
  TRY(check_ptr(qkv)); TRY(check_ptr(q_gamma)); TRY(check_ptr(k_gamma)); TRY(check_ptr(out));
  const QkShape shape{tokens, q_heads, kv_heads, head_dim, rope_dim, interleaved, eps, table, table_rows, positions,
                      seq_len};
  const size_t row = qk_row_bytes(shape, dtype), gain = head_dim * elem(dtype);
  TRY(check_apart({{out, row}}, {{out == qkv ? nullptr : qkv, row}, {q_gamma, gain}, {k_gamma, gain}, table_span(shape),
                                 position_span(shape)}));
  LAUNCH_TRY(launch_qk_norm_rope_fwd(dtype, shape, qkv, q_gamma, k_gamma, out, (hipStream_t)stream));
  return MERAK_OK;
}

size_t merak_qk_norm_rope_scratch_elems(int tokens, int q_heads, int kv_heads, int head_dim) {
  if (tokens <= 0 || q_heads <= 0 || kv_heads <= 0 || head_dim <= 0) return 0;
  return qk_norm_rope_scratch_elems(tokens, q_heads, kv_heads, head_dim);
}

int merak_qk_norm_rope_bwd(int dtype, int tokens, int q_heads, int kv_heads, int head_dim, int rope_dim,
                           int interleaved, float eps, const void* dout, const void* qkv, const void* q_gamma,
                           const void* k_gamma, const float* table, int table_rows, const int32_t* positions,
                           int seq_len, void* dqkv, float* dq_gamma, float* dk_gamma, int accumulate, float* scratch,
                           void* stream) {
  TRY(check_qk(dtype, tokens, q_heads, kv_heads, head_dim, rope_dim, interleaved, eps, table, table_rows, positions,
               seq_len));
  TRY(check_flag(accumulate));
  TRY(check_ptr(dout)); TRY(check_ptr(qkv)); TRY(check_ptr(q_gamma)); TRY(check_ptr(k_gamma)); TRY(check_ptr(dqkv));
  TRY(check_ptr(dq_gamma)); TRY(check_ptr(dk_gamma)); TRY(check_ptr(scratch));
  const QkShape shape{tokens, q_heads, kv_heads, head_dim, rope_dim, interleaved, eps, table, table_rows, positions,
                      seq_len};
  const size_t row = qk_row_bytes(shape, dtype), gain = head_dim * elem(dtype), dg = head_dim * sizeof(float);
  const Span sums{scratch, sizeof(float) * qk_norm_rope_scratch_elems(tokens, q_heads, kv_heads, head_dim)};
  TRY(check_apart({{dqkv, row}, {dq_gamma, dg}, {dk_gamma, dg}, sums},
                  {{qkv, row}, {q_gamma, gain}, {k_gamma, gain}, table_span(shape), position_span(shape),
                   {dqkv == dout ? nullptr : dout, row}}));
  LAUNCH_TRY(launch_qk_norm_rope_bwd(dtype, shape, dout, qkv, q_gamma, k_gamma, dqkv, dq_gamma, dk_gamma, accumulate,
                                     scratch, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_act8_save(int dtype, int rows, int cols, const void* x, uint8_t* q, uint8_t* scales, void* stream) {
  TRY(check_act8(dtype, rows, cols, q, scales));
  TRY(check_ptr(x));
  const size_t n = (size_t)rows * cols;
  TRY(check_apart({{q, n}, {scales, n / 32}}, {{x, n * elem(dtype)}}));
  LAUNCH_TRY(launch_act8_save(dtype, rows, cols, x, q, scales, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_act8_restore(int dtype, int rows, int cols, const uint8_t* q, const uint8_t* scales, void* x, void* stream) {
  TRY(check_act8(dtype, rows, cols, q, scales));
  TRY(check_ptr(x));
  const size_t n = (size_t)rows * cols;
  TRY(check_apart({{x, n * elem(dtype)}}, {{q, n}, {scales, n / 32}}));
  LAUNCH_TRY(launch_act8_restore(dtype, rows, cols, q, scales, x, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_act8_gelu_bwd(int dtype, int rows, int cols, const void* dg, const uint8_t* q, const uint8_t* scales,
                        void* du, void* g, void* stream) {
  TRY(check_act8(dtype, rows, cols, q, scales));
  TRY(check_ptr(dg)); TRY(check_ptr(du));
  if (g) TRY(check_ptr(g));
  const size_t n = (size_t)rows * cols, nb = n * elem(dtype);
  TRY(check_apart({{du, nb}, {g, nb}}, {{q, n}, {scales, n / 32}, {du == dg ? nullptr : dg, nb}}));
  LAUNCH_TRY(launch_act8_gelu_bwd(dtype, rows, cols, dg, q, scales, du, g, (hipStream_t)stream));
  return MERAK_OK;
}

size_t merak_act8_gemm_dw_scratch_bytes(int dtype, int tokens, int n_out, int n_in) {
  if (check_dtype(dtype) != MERAK_OK || tokens <= 0 || n_out <= 0 || n_in <= 0) return 0;
  return act8_gemm_dw_scratch_bytes(dtype, tokens, n_out, n_in);
}

int merak_act8_gemm_dw(int dtype, int tokens, int n_out, int n_in, const void* dy, const uint8_t* q,
                       const uint8_t* scales, float* dw, int accumulate, void* scratch, void* stream) {
  TRY(check_act8(dtype, tokens, n_in, q, scales));
  if (n_out <= 0 || n_out % 8 || tokens > kMaxRows || n_out > (1 << 20) || n_in > (1 << 20)) return MERAK_ERR_SHAPE;
  TRY(check_flag(accumulate));
  TRY(check_ptr(dy)); TRY(check_ptr(dw));
  const size_t sb = act8_gemm_dw_scratch_bytes(dtype, tokens, n_out, n_in), n = (size_t)tokens * n_in;
  if (sb > 0) TRY(check_ptr(scratch));
  TRY(check_apart({{dw, (size_t)n_out * n_in * 4}, {scratch, sb}},
                  {{dy, (size_t)tokens * n_out * elem(dtype)}, {q, n}, {scales, n / 32}}));
  LAUNCH_TRY(launch_act8_gemm_dw(dtype, tokens, n_out, n_in, dy, q, scales, dw, accumulate, scratch,
                                 (hipStream_t)stream));
  return MERAK_OK;
}

int merak_add_rms_norm_fwd(int dtype, int rows, int cols, float eps, const void* x, const void* resid,
                           const void* gamma, void* sum, void* y, uint8_t* q, uint8_t* scales, void* stream) {
  TRY(check_norm(dtype, rows, cols, eps));
  TRY(check_ptr(x)); TRY(check_ptr(gamma));
  if (resid) TRY(check_ptr(resid));
  if (!resid && sum) return MERAK_ERR_INVALID_ARG;
  if (sum) TRY(check_ptr(sum));
  if ((!y && !q) || !q != !scales) return MERAK_ERR_INVALID_ARG;
  if (y) TRY(check_ptr(y));
  const size_t n = (size_t)rows * cols, nb = n * elem(dtype);
  if (q) TRY(check_act8(dtype, rows, cols, q, scales));
  TRY(check_apart({{sum, nb}, {y, nb}, {q, n}, {scales, n / 32}},
                  {{sum == x ? nullptr : x, nb}, {sum == resid ? nullptr : resid, nb}, {gamma, cols * elem(dtype)}}));
  LAUNCH_TRY(launch_add_rms_norm_fwd(dtype, rows, cols, eps, x, resid, gamma, sum, y, q, scales, (hipStream_t)stream));
  return MERAK_OK;
}

size_t merak_add_rms_norm_scratch_elems(int rows, int cols) {
  if (rows <= 0 || cols <= 0) return 0;
  return add_rms_norm_scratch_elems(rows, cols);
}

int merak_add_rms_norm_bwd(int dtype, int rows, int cols, float eps, const void* dy, const void* dsum, const void* sum,
                           const void* gamma, void* dx, float* dgamma, int accumulate, float* scratch, void* stream) {
  TRY(check_norm(dtype, rows, cols, eps));
  TRY(check_flag(accumulate));
  TRY(check_ptr(dy)); TRY(check_ptr(sum)); TRY(check_ptr(gamma)); TRY(check_ptr(dx)); TRY(check_ptr(dgamma));
  if (dsum) TRY(check_ptr(dsum));
  const size_t se = add_rms_norm_scratch_elems(rows, cols);
  if (se > 0) TRY(check_ptr(scratch));
  const size_t nb = (size_t)rows * cols * elem(dtype);
  TRY(check_apart({{dx, nb}, {dgamma, cols * sizeof(float)}, {scratch, se * sizeof(float)}},
                  {{dx == dy ? nullptr : dy, nb}, {dx == dsum ? nullptr : dsum, nb}, {sum, nb},
                   {gamma, cols * elem(dtype)}}));
  LAUNCH_TRY(launch_add_rms_norm_bwd(dtype, rows, cols, eps, dy, dsum, sum, gamma, dx, dgamma, accumulate, scratch,
                                     (hipStream_t)stream));
  return MERAK_OK;
}

int merak_distill_loss_fwd(int dtype, int tokens, int vocab, int ld, int64_t first_id, int64_t vocab_total, int top,
                           int id_type, int teacher_dtype, int label_type, float alpha, float temperature,
                           const void* logits, const void* teacher_ids, const void* teacher_logits, const void* labels,
                           float* stats, float* loss, void* stream) {
  const DistillShape q{tokens, vocab, ld, top, first_id, vocab_total, id_type, teacher_dtype, label_type, alpha,
                       temperature, teacher_ids, teacher_logits, labels};
  TRY(check_distill(dtype, q, logits));
  if (!stats && !loss) return MERAK_ERR_INVALID_ARG;
  if (loss && vocab != vocab_total) return MERAK_ERR_INVALID_ARG;  // a share has no loss of its own
  if (stats) TRY(check_ptr(stats));
  if (loss) TRY(check_ptr(loss));
  TRY(check_apart({{stats, stats_bytes(tokens)}, {loss, tokens * sizeof(float)}},
                  {{logits, logits_bytes(dtype, q)}, ids_span(q), teacher_span(q), labels_span(q)}));
  LAUNCH_TRY(launch_distill(dtype, q, logits, stats, loss, nullptr, nullptr, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_distill_loss_join(int tokens, int ranks, float alpha, float temperature, const float* parts, float* stats,
                            float* loss, void* stream) {
  TRY(check_mix(alpha, temperature));
  if (tokens <= 0 || tokens > kMaxRows || ranks <= 0 || ranks > (1 << 16)) return MERAK_ERR_SHAPE;
  TRY(check_ptr(parts)); TRY(check_ptr(stats)); TRY(check_ptr(loss));
  TRY(check_apart({{stats, stats_bytes(tokens)}, {loss, tokens * sizeof(float)}}, {{parts, ranks * stats_bytes(tokens)}}));
  LAUNCH_TRY(launch_distill_join(tokens, ranks, alpha, temperature, parts, stats, loss, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_distill_loss_bwd(int dtype, int tokens, int vocab, int ld, int64_t first_id, int64_t vocab_total, int top,
                           int id_type, int teacher_dtype, int label_type, float alpha, float temperature,
                           const void* logits, const void* teacher_ids, const void* teacher_logits, const void* labels,
                           const float* stats, const float* dloss, void* dlogits, void* stream) {
  const DistillShape q{tokens, vocab, ld, top, first_id, vocab_total, id_type, teacher_dtype, label_type, alpha,
                       temperature, teacher_ids, teacher_logits, labels};
  TRY(check_distill(dtype, q, logits));
  TRY(check_ptr(stats)); TRY(check_ptr(dloss)); TRY(check_ptr(dlogits));
  const size_t nb = logits_bytes(dtype, q);
  TRY(check_apart({{dlogits, nb}}, {{dlogits == logits ? nullptr : logits, nb}, ids_span(q), teacher_span(q),
                                    labels_span(q), {stats, stats_bytes(tokens)}, {dloss, tokens * sizeof(float)}}));
  LAUNCH_TRY(launch_distill_bwd(dtype, q, logits, stats, dloss, dlogits, (hipStream_t)stream));
  return MERAK_OK;
}

int merak_distill_loss_fwd_bwd(int dtype, int tokens, int vocab, int ld, int top, int id_type, int teacher_dtype,
                               int label_type, float alpha, float temperature, const void* logits,
                               const void* teacher_ids, const void* teacher_logits, const void* labels,
                               const float* dloss, float* loss, void* dlogits, void* stream) {
  const DistillShape q{tokens, vocab, ld, top, 0, vocab, id_type, teacher_dtype, label_type, alpha, temperature,
                       teacher_ids, teacher_logits, labels};
  TRY(check_distill(dtype, q, logits));
  TRY(check_ptr(dloss)); TRY(check_ptr(loss)); TRY(check_ptr(dlogits));
  const size_t nb = logits_bytes(dtype, q);
  TRY(check_apart({{dlogits, nb}, {loss, tokens * sizeof(float)}},
                  {{dlogits == logits ? nullptr : logits, nb}, ids_span(q), teacher_span(q), labels_span(q),
                   {dloss, tokens * sizeof(float)}}));
  LAUNCH_TRY(launch_distill(dtype, q, logits, nullptr, loss, dloss, dlogits, (hipStream_t)stream));
  return MERAK_OK;
}

}  // extern "C"
