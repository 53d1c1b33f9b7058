// The C entries of the decoding operators: they check their arguments and enqueue; nothing is allocated, copied to the host or
// waited for, so that every one of them can be captured into a graph.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "../../include/cytonmt_hip.h"
#include "lowbit.h"

using namespace cmt;

namespace {

thread_local char t_error[256] = "";

int refuse(const char* format, ...) {
  va_list args;
  va_start(args, format);
  vsnprintf(t_error, sizeof t_error, format, args);
  va_end(args);
  return CMT_EINVAL;
}
int done(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return CMT_OK;
  snprintf(t_error, sizeof t_error, "%s: %s", what, hipGetErrorString(e));
  return CMT_EHIP;
}
bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
size_t type_size(int32_t t) { return t == CMT_BF16 ? 2 : 4; }
bool type_ok(int32_t t) { return t == CMT_FP32 || t == CMT_BF16; }

// Rows of so many bytes, a pitch apart.  Columns of one matrix (equal pitches) may lie side by side; of different
// pitches the whole extents have to be apart.
struct Rows { uint64_t at, pitch, bytes, count; };
bool overlap(const Rows& a, const Rows& b) {
  if (a.count == 0 || b.count == 0) return false;
  if (a.at >= b.at + (b.count - 1) * b.pitch + b.bytes || b.at >= a.at + (a.count - 1) * a.pitch + a.bytes) return false;
  if (a.pitch != b.pitch || a.count == 1 || b.count == 1) return true;
  const uint64_t ahead = b.at >= a.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;   // where b's rows begin within a's pitch
  return ahead < a.bytes || ahead + b.bytes > a.pitch;
}

bool quant_shape(int32_t outputs, int32_t inputs, int32_t group, QuantShape* q) {
  if (outputs < 1 || outputs > 1 << 24 || inputs < 1 || inputs > 1 << 16) { refuse("outputs must be in [1, 2^24], inputs in [1, 2^16]"); return false; }
  if ((int64_t)outputs * inputs > (int64_t)1 << 34) { refuse("outputs * inputs must be at most 2^34"); return false; }   // (a grid has less than 2^32 threads)
  if (group != 32 && group != 64 && group != 128) { refuse("group must be 32, 64 or 128"); return false; }
  *q = QuantShape{outputs, inputs, group};
  return true;
}
bool cache_shape(const cmt_cache_config* c, CacheShape* s) {
  if (!c) { refuse("null pointer"); return false; }
  if (c->sequences < 1 || c->heads < 1 || (int64_t)c->sequences * c->heads > 65535) { refuse("sequences and heads must be positive, their product at most 65535"); return false; }
  if (c->head_dim < 1 || c->head_dim > 1024) { refuse("head_dim must be in [1, 1024]"); return false; }
  if (c->max_tokens < 1 || c->max_tokens > 1 << 24) { refuse("max_tokens must be in [1, 2^24]"); return false; }
  *s = CacheShape{c->sequences, c->heads, c->head_dim, c->max_tokens};
  return true;
}
// queries per sequence and key head, as an int that the kernels can index with
bool attend_shape(const CacheShape& s, int32_t rows_per_sequence, int32_t query_heads, int32_t tokens) {
  if (rows_per_sequence < 1 || query_heads < 1 || query_heads % s.heads) { refuse("rows_per_sequence must be positive, query_heads a positive multiple of heads"); return false; }
  if (tokens < 1 || tokens > s.tokens) { refuse("tokens must be in [1, max_tokens]"); return false; }
  if ((int64_t)s.seqs * rows_per_sequence * query_heads > 1 << 24 || (int64_t)rows_per_sequence * (query_heads / s.heads) > 1 << 19) {
    refuse("more than 2^24 queries, or 2^19 of one sequence and head");
    return false;
  }
  return true;
}

}  // namespace

extern "C" {

const char* cmt_operator_error(void) { return t_error; }

int cmt_quant_weight_bytes(int32_t outputs, int32_t inputs, int32_t group, size_t* bytes) {
  QuantShape q;
  if (!bytes) return refuse("null pointer");
  if (!quant_shape(outputs, inputs, group, &q)) return CMT_EINVAL;
  *bytes = q.bytes();
  return CMT_OK;
}
int cmt_quant_weight_pack(const void* weight_dev, int32_t type, int64_t pitch, int32_t outputs, int32_t inputs, int32_t group, void* packed_dev,
                          void* hip_stream) {
  QuantShape q;
  if (!quant_shape(outputs, inputs, group, &q)) return CMT_EINVAL;
  if (!weight_dev || !packed_dev) return refuse("null pointer");
  if (!type_ok(type)) return refuse("type must be CMT_FP32 or CMT_BF16");
  if (pitch < inputs) return refuse("pitch is less than inputs");
  if (misaligned(packed_dev, 256) || misaligned(weight_dev, type_size(type))) return refuse("packed weights are 256-byte aligned, others as their elements");
  launch_quant_pack(type, weight_dev, (size_t)pitch, q, false, packed_dev, (hipStream_t)hip_stream);
  return done("cmt_quant_weight_pack");
}
int cmt_quant_weight_encode(const uint8_t* codes_dev, const uint16_t* scales_dev, int32_t outputs, int32_t inputs, int32_t group, void* packed_dev,
                            void* hip_stream) {
  QuantShape q;
  if (!quant_shape(outputs, inputs, group, &q)) return CMT_EINVAL;
  if (!codes_dev || !scales_dev || !packed_dev) return refuse("null pointer");
  if (misaligned(packed_dev, 256) || misaligned(scales_dev, 2)) return refuse("packed weights are 256-byte aligned, scales 2-byte");
  launch_quant_encode(codes_dev, scales_dev, q, packed_dev, (hipStream_t)hip_stream);
  return done("cmt_quant_weight_encode");
}
int cmt_quant_weight_values(const void* packed_dev, int32_t outputs, int32_t inputs, int32_t group, float* weight_dev, void* hip_stream) {
  QuantShape q;
  if (!quant_shape(outputs, inputs, group, &q)) return CMT_EINVAL;
  if (!packed_dev || !weight_dev) return refuse("null pointer");
  if (misaligned(packed_dev, 256) || misaligned(weight_dev, 4)) return refuse("packed weights are 256-byte aligned, others as their elements");
  launch_quant_values(packed_dev, q, weight_dev, (hipStream_t)hip_stream);
  return done("cmt_quant_weight_values");
}
int cmt_quant_product(const void* x_dev, int32_t type, int64_t x_pitch, int32_t rows, const void* packed_dev, int32_t outputs, int32_t inputs,
                      int32_t group, const float* bias_dev, int32_t tanh_of, void* y_dev, int32_t y_type, int64_t y_pitch, void* hip_stream) {
  QuantShape q;
  if (!quant_shape(outputs, inputs, group, &q)) return CMT_EINVAL;
  if (!type_ok(type) || !type_ok(y_type)) return refuse("types must be CMT_FP32 or CMT_BF16");
  if (rows < 0 || rows > 65535 || (int64_t)q.row_blocks() * ((rows + 15) / 16) > 1 << 28) return refuse("rows must be in [0, 65535], outputs * rows at most 2^36");
  if (rows == 0) return CMT_OK;
  if (!x_dev || !packed_dev || !y_dev) return refuse("null pointer");
  if (x_pitch < inputs || y_pitch < outputs) return refuse("a pitch is less than its row");
  if (misaligned(packed_dev, 256) || misaligned(x_dev, type_size(type)) || misaligned(y_dev, type_size(y_type)) || misaligned(bias_dev, 4))
    return refuse("packed weights are 256-byte aligned, others as their elements");
  launch_quant_product(type, x_dev, (size_t)x_pitch, QuantWeightRef{q, (const char*)packed_dev}, rows, bias_dev, tanh_of != 0, y_type, y_dev,
                       (size_t)y_pitch, (hipStream_t)hip_stream);
  return done("cmt_quant_product");
}

int cmt_cache_bytes(const cmt_cache_config* cache, size_t* bytes) {
  CacheShape s;
  if (!bytes) return refuse("null pointer");
  if (!cache_shape(cache, &s)) return CMT_EINVAL;
  *bytes = s.bytes();
  return CMT_OK;
}
int cmt_cache_fill(const cmt_cache_config* cache, void* cache_dev, const cmt_cache_rows* keys, const cmt_cache_rows* values, int32_t type,
                   const int32_t* lengths_dev, int32_t tokens, void* hip_stream) {
  CacheShape s;
  if (!cache_shape(cache, &s)) return CMT_EINVAL;
  if (!cache_dev || !keys || !values || !keys->data_dev || !values->data_dev || !lengths_dev) return refuse("null pointer");
  if (!type_ok(type)) return refuse("type must be CMT_FP32 or CMT_BF16");
  if (tokens < 1 || tokens > s.tokens) return refuse("tokens must be in [1, max_tokens]");
  for (const cmt_cache_rows* r : {keys, values})
    if (r->sequence_stride < 0 || r->token_stride < 0 || r->head_stride < 0) return refuse("strides must not be negative");
  if (misaligned(cache_dev, 256) || misaligned(keys->data_dev, type_size(type)) || misaligned(values->data_dev, type_size(type)) || misaligned(lengths_dev, 4))
    return refuse("the cache is 256-byte aligned, others as their elements");
  const CacheSource src{keys->data_dev, values->data_dev, (size_t)keys->sequence_stride, (size_t)keys->token_stride, (size_t)keys->head_stride,
                        (size_t)values->sequence_stride, (size_t)values->token_stride, (size_t)values->head_stride};
  launch_cache_fill(type, src, lengths_dev, tokens, s, cache_dev, (hipStream_t)hip_stream);
  return done("cmt_cache_fill");
}
int cmt_cache_read(const cmt_cache_config* cache, const void* cache_dev, int32_t tokens, float* keys_dev, float* values_dev, void* hip_stream) {
  CacheShape s;
  if (!cache_shape(cache, &s)) return CMT_EINVAL;
  if (!cache_dev || !keys_dev || !values_dev) return refuse("null pointer");
  if (tokens < 1 || tokens > s.tokens) return refuse("tokens must be in [1, max_tokens]");
  if ((double)s.seqs * tokens * s.heads * s.dim > 1e11) return refuse("more than 10^11 values");
  if (misaligned(cache_dev, 256) || misaligned(keys_dev, 4) || misaligned(values_dev, 4)) return refuse("the cache is 256-byte aligned, others as their elements");
  launch_cache_read(s, cache_dev, tokens, keys_dev, values_dev, (hipStream_t)hip_stream);
  return done("cmt_cache_read");
}
int cmt_cache_attend_workspace(const cmt_cache_config* cache, int32_t rows_per_sequence, int32_t query_heads, int32_t tokens, size_t* bytes) {
  CacheShape s;
  if (!bytes) return refuse("null pointer");
  if (!cache_shape(cache, &s) || !attend_shape(s, rows_per_sequence, query_heads, tokens)) return CMT_EINVAL;
  *bytes = cache_attend_workspace(s, rows_per_sequence, query_heads, tokens);
  return CMT_OK;
}
int cmt_cache_attend(const cmt_cache_config* cache, const void* cache_dev, const void* query_dev, int32_t type, int64_t query_pitch,
                     int32_t rows_per_sequence, int32_t query_heads, int32_t tokens, float scale, void* out_dev, int64_t out_pitch, void* workspace_dev,
                     size_t workspace_bytes, void* hip_stream) {
  CacheShape s;
  if (!cache_shape(cache, &s) || !attend_shape(s, rows_per_sequence, query_heads, tokens)) return CMT_EINVAL;
  if (!cache_dev || !query_dev || !out_dev) return refuse("null pointer");
  if (!type_ok(type)) return refuse("type must be CMT_FP32 or CMT_BF16");
  if (!isfinite(scale)) return refuse("scale is not finite");
  if (query_pitch < (int64_t)query_heads * s.dim || out_pitch < (int64_t)query_heads * s.dim) return refuse("a pitch is less than its row");
  if (misaligned(cache_dev, 256) || misaligned(query_dev, type_size(type)) || misaligned(out_dev, type_size(type)) || misaligned(workspace_dev, 256))
    return refuse("the cache and the workspace are 256-byte aligned, others as their elements");
  const size_t need = cache_attend_workspace(s, rows_per_sequence, query_heads, tokens);
  if (need && (!workspace_dev || workspace_bytes < need)) return refuse("the workspace has %zu bytes, %zu are needed", workspace_dev ? workspace_bytes : (size_t)0, need);
  launch_cache_attend(type, s, cache_dev, query_dev, (size_t)query_pitch, rows_per_sequence, query_heads, tokens, scale, out_dev, (size_t)out_pitch,
                      workspace_dev, (hipStream_t)hip_stream);
  return done("cmt_cache_attend");
}

static bool select_shape(int32_t sentences, int32_t beam, int32_t vocab, int32_t n) {
  if (sentences < 1 || sentences > 1 << 20) { refuse("sentences must be in [1, 2^20]"); return false; }
  if (beam < 1 || beam > SEARCH_MAX || n < 1 || n > SEARCH_MAX) { refuse("beam and n must be in [1, %d]", SEARCH_MAX); return false; }
  if (vocab < 1 || vocab > SEARCH_MAX_VOCAB) { refuse("vocab must be in [1, %d]", SEARCH_MAX_VOCAB); return false; }
  if ((double)sentences * beam * ((vocab + SEARCH_GROUP - 1) / SEARCH_GROUP) > 1 << 25) { refuse("more than 2^25 groups of %d logits", SEARCH_GROUP); return false; }
  return true;
}
int cmt_beam_select_workspace(int32_t sentences, int32_t beam, int32_t vocab, size_t* bytes) {
  if (!bytes) return refuse("null pointer");
  if (!select_shape(sentences, beam, vocab, 1)) return CMT_EINVAL;
  *bytes = search_workspace(sentences, beam, vocab);
  return CMT_OK;
}
int cmt_beam_select(const void* logits_dev, int32_t type, int64_t pitch, const float* scores_dev, int32_t sentences, int32_t beam, int32_t vocab,
                    int32_t n, float* out_scores_dev, int32_t* out_rows_dev, int32_t* out_tokens_dev, void* workspace_dev, size_t workspace_bytes,
                    void* hip_stream) {
  if (!select_shape(sentences, beam, vocab, n)) return CMT_EINVAL;
  if (!logits_dev || !scores_dev || !out_scores_dev || !out_rows_dev || !out_tokens_dev || !workspace_dev) return refuse("null pointer");
  if (!type_ok(type)) return refuse("type must be CMT_FP32 or CMT_BF16");
  if (pitch < vocab) return refuse("pitch is less than vocab");
  if (misaligned(logits_dev, type_size(type)) || misaligned(scores_dev, 4) || misaligned(out_scores_dev, 4) || misaligned(out_rows_dev, 4) ||
      misaligned(out_tokens_dev, 4) || misaligned(workspace_dev, 256))
    return refuse("the workspace is 256-byte aligned, others as their elements");
  const size_t need = search_workspace(sentences, beam, vocab);
  if (workspace_bytes < need) return refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need);
  launch_search_select(type, logits_dev, (size_t)pitch, scores_dev, sentences, beam, vocab, n, out_scores_dev, out_rows_dev, out_tokens_dev, nullptr,
                       workspace_dev, (hipStream_t)hip_stream);
  return done("cmt_beam_select");
}
int cmt_beam_reorder(const int32_t* rows_dev, int32_t count, int32_t source_rows, const cmt_reorder_tensor* tensors, int32_t n, void* hip_stream) {
  if (n < 0 || n > 256 || count < 0 || count > 1 << 24 || source_rows < 0) return refuse("counts must not be negative, tensors at most 256, rows at most 2^24");
  if (n == 0 || count == 0) return CMT_OK;
  if (!rows_dev || !tensors) return refuse("null pointer");
  if (misaligned(rows_dev, 4)) return refuse("rows are 4-byte aligned");
  for (int i = 0; i < n; ++i) {
    const cmt_reorder_tensor& a = tensors[i];
    if (!a.source_dev || !a.target_dev) return refuse("tensor %d: null pointer", i);
    if (a.row_bytes < 1 || a.row_bytes > 1 << 30) return refuse("tensor %d: row_bytes must be in [1, 2^30]", i);
    if (a.source_pitch < a.row_bytes || a.target_pitch < a.row_bytes) return refuse("tensor %d: a pitch is less than its row", i);
  }
  for (int i = 0; i < n; ++i)                                // (rows are written in any order: what is read must stay)
    for (int k = 0; k < n; ++k) {
      const cmt_reorder_tensor &a = tensors[i], &b = tensors[k];
      const Rows target{(uintptr_t)a.target_dev, (uint64_t)a.target_pitch, (uint64_t)a.row_bytes, (uint64_t)count};
      if (overlap(target, Rows{(uintptr_t)b.source_dev, (uint64_t)b.source_pitch, (uint64_t)b.row_bytes, (uint64_t)source_rows}))
        return refuse("the target of tensor %d overlaps the source of tensor %d", i, k);
      if (k < i && overlap(target, Rows{(uintptr_t)b.target_dev, (uint64_t)b.target_pitch, (uint64_t)b.row_bytes, (uint64_t)count}))
        return refuse("the targets of tensors %d and %d overlap", k, i);
      if (k == i && overlap(target, Rows{(uintptr_t)rows_dev, (uint64_t)count * 4, (uint64_t)count * 4, 1})) return refuse("the target of tensor %d overlaps the rows' numbers", i);
    }
  for (int i0 = 0; i0 < n; i0 += REORDER_MAX) {
    ReorderJobs jobs{};
    const int m = n - i0 < REORDER_MAX ? n - i0 : REORDER_MAX;
    for (int i = 0; i < m; ++i) {
      const cmt_reorder_tensor& a = tensors[i0 + i];
      const uint64_t bits = (uintptr_t)a.source_dev | (uintptr_t)a.target_dev | (uint64_t)a.source_pitch | (uint64_t)a.target_pitch | (uint64_t)a.row_bytes;
      jobs.job[i] = ReorderJob{(const char*)a.source_dev, (char*)a.target_dev, (size_t)a.source_pitch, (size_t)a.target_pitch, rows_dev, source_rows, (int)a.row_bytes,
                               bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : bits % 2 == 0 ? 2 : 1};
    }
    launch_search_reorder(jobs, m, count, (hipStream_t)hip_stream);
  }
  return done("cmt_beam_reorder");
}

}  // extern "C"
