// Launchers of the kernels for decoding in small numbers (quant.hip, cache.hip, search.hip) and what they share.  As in kernels.h: they
// only enqueue work on `st`; none allocates or synchronises.  `prec`: 0 = float, 1 = bf16 (raw uint16).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace cmt {

// ---- quant.hip: products with 4-bit weights ---------------------------------------------------------
// A weight [N, K] is held as e2m1 codes (the format that the hardware turns into bf16, two to an instruction) in tiles of 16 rows x 128 k:
// 1 KB, lane l's 16 bytes being row l % 16, of which dword s holds k = 32 s + 8 (l / 16) + 0..7 (low nibble first) - the register
// operand of the 16x16x32 matrix instruction.  Tiles of a row block follow each other in k; rows and k beyond the matrix are 0.
// Behind the codes: bf16 scales [row block][k / group][16 rows], 0 beyond the matrix.
constexpr int QUANT_TILE_K = 128;
struct QuantShape {
  int N, K, group;
  __host__ __device__ int row_blocks() const { return (N + 15) / 16; }
  __host__ __device__ int k_tiles() const { return (K + QUANT_TILE_K - 1) / QUANT_TILE_K; }
  size_t code_bytes() const { return (size_t)row_blocks() * k_tiles() * 1024; }
  size_t scale_bytes() const { return (size_t)row_blocks() * k_tiles() * (QUANT_TILE_K / group) * 32; }
  size_t bytes() const { return (code_bytes() + scale_bytes() + 255) & ~(size_t)255; }
};
struct QuantWeightRef { QuantShape shape; const char* packed; };
// gates: an LSTM layer's weight (blocks of N / 4 rows i, f, g, o), packed with a unit's four rows side by side.
void launch_quant_pack(int prec, const void* w, size_t ldw, const QuantShape& q, bool gates, void* packed, hipStream_t st);
void launch_quant_encode(const uint8_t* codes, const bf16_t* scales, const QuantShape& q, void* packed, hipStream_t st);
void launch_quant_values(const void* packed, const QuantShape& q, float* out, hipStream_t st);
// y [M, N] = f(x [M, K] W^T + bias), f = tanh or nothing; x of type prec, y of type y_prec; bias fp32 or null.
void launch_quant_product(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, bool tanh, int y_prec, void* y,
                          size_t ldy, hipStream_t st);
// An LSTM layer's position: the gates x W^T + bias (W packed as gates; bias in blocks i, f, g, o of H) and their cells, c_prev [M, H] -> c [M, H]
// fp32 and the state in type prec to two places (pitches in elements).
void launch_quant_lstm(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, const float* c_prev, float* c, void* h,
                       size_t ldh, void* h2, size_t ldh2, hipStream_t st);

// ---- cache.hip: source rows in 8 bits -------------------------------------------------------------
// Per (sequence, head, block of 32 tokens) one fp32 scale for the keys and one for the values; codes are whole numbers -127..127.
// Keys: tiles of 32 tokens x 32 d, 1 KB, lane l's bytes 8 h + j (h = 0, 1) being token 16 h + l % 16, d = 8 (l / 16) + j: two operands of 16 tokens.
// Values: tiles of 32 tokens x 32 d, 1 KB, lane l's bytes 8 h + j (h = 0, 1) being d = 16 h + l % 16 and token 4 (l / 16) + j (j < 4)
// or 12 + 4 (l / 16) + j: the order in which the scores' accumulators hold the tokens, so that weights go from one
// product into the other without leaving their lanes.
constexpr int CACHE_BLOCK = 32;
struct CacheShape {
  int seqs, heads, dim, tokens;                            // tokens: the capacity
  __host__ __device__ int blocks() const { return (tokens + CACHE_BLOCK - 1) / CACHE_BLOCK; }
  __host__ __device__ int chunks() const { return (dim + 31) / 32; }           // of 32 d
  size_t part() const { return (size_t)seqs * heads * blocks(); }
  size_t lengths_bytes() const { return ((size_t)seqs * 4 + 255) & ~(size_t)255; }
  size_t scales_bytes() const { return (part() * 4 + 255) & ~(size_t)255; }
  size_t codes_bytes() const { return part() * chunks() * 1024; }
  size_t bytes() const { return lengths_bytes() + 2 * scales_bytes() + 2 * codes_bytes(); }
};
struct CacheView {
  int32_t* lengths; float *kscale, *vscale; char *k, *v;
  CacheView(const CacheShape& s, void* base) {
    char* p = (char*)base;
    lengths = (int32_t*)p; p += s.lengths_bytes();
    kscale = (float*)p; p += s.scales_bytes();
    vscale = (float*)p; p += s.scales_bytes();
    k = p; p += s.codes_bytes();
    v = p;
  }
};
struct CacheSource { const void *k, *v; size_t k_seq, k_tok, k_head, v_seq, v_tok, v_head; };   // strides in elements; d contiguous
void launch_cache_fill(int prec, const CacheSource& src, const int32_t* lengths, int tokens, const CacheShape& s, void* cache, hipStream_t st);
void launch_cache_read(const CacheShape& s, const void* cache, int tokens, float* k, float* v, hipStream_t st);
// Attention of rows x q_heads queries; row r belongs to sequence r / per.  q, out: [rows, q_heads, dim] with row pitches, heads side by side.
size_t cache_attend_workspace(const CacheShape& s, int per, int q_heads, int tokens);
void launch_cache_attend(int prec, const CacheShape& s, const void* cache, const void* q, size_t ldq, int per, int q_heads, int tokens, float scale,
                         void* out, size_t ldo, void* workspace, hipStream_t st);

// ---- search.hip: a beam search's choice --------------------------------------------------------------
constexpr int SEARCH_MAX = 32, SEARCH_GROUP = 512;
constexpr int SEARCH_MAX_VOCAB = 1 << 26;
// What a search that is kept on the device does with the best extensions (the rules of cmt_beam_decode): those that end leave the
// beam, the others fill its places, best first.  Rows beyond R and lists as in BeamState.
struct SearchAdvance {
  int32_t *hist_tok, *hist_par, *fin_step, *fin_par, *fin_tok; float* fin_score;
  int hist_ld, j, max_len, eos; float alpha;
};
size_t search_workspace(int B, int K, int V);
void launch_search_select(int prec, const void* logits, size_t ld, const float* scores, int B, int K, int V, int n, float* out_scores,
                          int32_t* out_rows, int32_t* out_tokens, const SearchAdvance* adv, void* workspace, hipStream_t st);
constexpr int REORDER_MAX = 32;
struct ReorderJob { const char* src; char* dst; size_t src_pitch, dst_pitch; const int32_t* rows; int src_rows, bytes, step; };   // step: 16, 4, 2 or 1 bytes at a time
struct ReorderJobs { ReorderJob job[REORDER_MAX]; };
void launch_search_reorder(const ReorderJobs& jobs, int n, int count, hipStream_t st);

// ---- shared ------------------------------------------------------------------------------------------
// Over the 16 lanes of a row, in every lane, by DPP moves (a shuffle through LDS is ten times as long).
#define CMT_ROW16(v, op)                                                                                                        \
  do {                                                                                                                          \
    v = op(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true)));  /* quad_perm 1 0 3 2 */ \
    v = op(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true)));  /* quad_perm 2 3 0 1 */ \
    v = op(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true))); /* row_half_mirror */   \
    v = op(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true))); /* row_mirror */        \
  } while (0)
__device__ __forceinline__ float add_of(float a, float b) { return a + b; }
__device__ __forceinline__ float row16_max(float v) { CMT_ROW16(v, fmaxf); return v; }
__device__ __forceinline__ float row16_sum(float v) { CMT_ROW16(v, add_of); return v; }
#undef CMT_ROW16
__device__ __forceinline__ float half_max(float v) { v = row16_max(v); return fmaxf(v, __shfl_xor(v, 16, 64)); }   // over 32 lanes
__device__ __forceinline__ float half_sum(float v) { v = row16_sum(v); return v + __shfl_xor(v, 16, 64); }
__device__ __forceinline__ float lanes_max(float v) { v = half_max(v); return fmaxf(v, __shfl_xor(v, 32, 64)); }   // over all 64
__device__ __forceinline__ float lanes_sum(float v) { v = half_sum(v); return v + __shfl_xor(v, 32, 64); }

// An fp32 number as three bf16 that add up to it, cut off rather than rounded (8 + 8 + 8 bits; none can overflow).  Infinities and NaN
// stand in the first part alone.
struct Parts3 { uint32_t h, m, l; };                       // bits as of an fp32, lower half 0
__device__ __forceinline__ Parts3 parts3(float x) {
  const uint32_t u = __float_as_uint(x);
  const bool none = (u & 0x7f800000u) == 0x7f800000u;
  Parts3 p;
  p.h = u & 0xffff0000u;
  const float r = x - __uint_as_float(p.h);
  p.m = __float_as_uint(r) & 0xffff0000u;
  p.l = none ? 0u : __float_as_uint(r - __uint_as_float(p.m)) & 0xffff0000u;
  p.m = none ? 0u : p.m;
  p.h = none && (u & 0x007fffffu) ? 0x7fc00000u : p.h;
  return p;
}
__device__ __forceinline__ uint32_t pack_hi(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }   // upper halves of both

// Operand parts of 8 consecutive elements: 1 of bf16, 3 of fp32.
template <typename T> constexpr int OPERAND_PARTS = sizeof(T) == 2 ? 1 : 3;
// four elements that lie anywhere, stored as one
typedef float any_v4f __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t any_v4h __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store_four(float* p, float a, float b, float c, float d) { *reinterpret_cast<any_v4f*>(p) = any_v4f{a, b, c, d}; }
__device__ __forceinline__ void store_four(bf16_t* p, float a, float b, float c, float d) { *reinterpret_cast<any_v4h*>(p) = any_v4h{f2bf(a), f2bf(b), f2bf(c), f2bf(d)}; }
// the first n (or all 8) elements at p, wherever p is, 0 behind them
__device__ __forceinline__ void load_elements(const bf16_t* p, int n, Frag<bf16_t>& f) {
  if (n >= 8) { __builtin_memcpy(&f.v, p, 16); return; }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
  f.v = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void load_elements(const float* p, int n, Frag<float>& f) {
  if (n >= 8) { __builtin_memcpy(&f.lo, p, 16); __builtin_memcpy(&f.hi, p + 4, 16); return; }
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = i < n ? p[i] : 0.f;
  f.lo = make_float4(x[0], x[1], x[2], x[3]);
  f.hi = make_float4(x[4], x[5], x[6], x[7]);
}
// The same in two steps, so that many loads go out one behind the other, of a row of 8 elements or more: those from `at` on, near the row's end its last 8,
// and their move to where they belong, 0 behind them.
template <typename T>
__device__ __forceinline__ void load_near(const T* row, int at, int size, Frag<T>& f) { load_elements(row + min(at, size - 8), 8, f); }
__device__ __forceinline__ void move_near(int at, int size, Frag<bf16_t>& f) {
  const int by = at - (size - 8);
  if (by <= 0) return;
  uint4 v = f.v;
  if (by & 1) v = make_uint4(v.x >> 16 | v.y << 16, v.y >> 16 | v.z << 16, v.z >> 16 | v.w << 16, v.w >> 16);
  if (by & 2) v = make_uint4(v.y, v.z, v.w, 0);
  if (by & 4) v = make_uint4(v.z, v.w, 0, 0);
  f.v = by < 8 ? v : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void move_near(int at, int size, Frag<float>& f) {
  const int by = at - (size - 8);
  if (by <= 0) return;
  float4 a = f.lo, b = f.hi;
  if (by & 1) { a = make_float4(a.y, a.z, a.w, b.x); b = make_float4(b.y, b.z, b.w, 0.f); }
  if (by & 2) { a = make_float4(a.z, a.w, b.x, b.y); b = make_float4(b.z, b.w, 0.f, 0.f); }
  if (by & 4) { a = b; b = make_float4(0.f, 0.f, 0.f, 0.f); }
  f.lo = by < 8 ? a : make_float4(0.f, 0.f, 0.f, 0.f);
  f.hi = by < 8 ? b : make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ void operand_of(const Frag<bf16_t>& x, bool in, Frag<bf16_t> (&f)[1]) {   // in = false: zeros
  f[0].v = make_uint4(in ? x.v.x : 0u, in ? x.v.y : 0u, in ? x.v.z : 0u, in ? x.v.w : 0u);
}
__device__ __forceinline__ void operand_of(const Frag<float>& x, bool in, Frag<bf16_t> (&f)[3]) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Parts3 a = parts3(in ? x.get(2 * i) : 0.f), b = parts3(in ? x.get(2 * i + 1) : 0.f);
    h[i] = pack_hi(a.h, b.h); m[i] = pack_hi(a.m, b.m); l[i] = pack_hi(a.l, b.l);
  }
  f[0].v = make_uint4(h[0], h[1], h[2], h[3]);
  f[1].v = make_uint4(m[0], m[1], m[2], m[3]);
  f[2].v = make_uint4(l[0], l[1], l[2], l[3]);
}

}  // namespace cmt
