// Source rows in 8 bits and the attention that reads them: keys and values of every block of 32 tokens and head as whole numbers of
// -127..127 times one fp32 scale each.
//
// o = sum_i a_i v_i, a = softmax over the tokens i below the sequence's length of scale q.k_i.  The codes are exact in bf16, so
// both products run on the bf16 matrix instructions: the queries as they are (fp32 ones as three bf16 parts), the weights
// a_i (times the values' scale) as two (three) bf16 parts; sums, maxima and scales are fp32.
// Every query of a sequence and key head shares its tokens' bytes: 2 D bytes a token for 4 D flop a query.  The read bounds it.
#include <algorithm>
#include <type_traits>

#include "lowbit.h"

namespace cmt {

// Nearest whole number to x / s, the even one of two, as if the quotient were exact.  inv ~ 1 / s.
__device__ __forceinline__ float cache_code(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), r2 = 2.f * fabsf(r);       // (exact: |r| < 2 s and a multiple of half an ulp of s)
  if (r2 > s || (r2 == s && ((int)q & 1))) q += copysignf(1.f, r);
  return fminf(fmaxf(q, -127.f), 127.f);
}

// ---- writing ---------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void fill_load(const T* p, int n, bool wide, Frag<T> (&x)[2]) {   // the first n of 16 elements, then 0
  if (n >= 16 && wide) { x[0].load(p); x[1].load(p + 8); }
  else { load_elements(p, n, x[0]); load_elements(p + 8, n - 8, x[1]); }
}
// One workgroup per block of 32 tokens, sequence and head; blockIdx.z: keys, values.  The block is read once: a thread keeps its NS
// slots of 16 d of a token until the scale is known.
template <typename T, int NS>
__global__ __launch_bounds__(512) void cache_fill_kernel(CacheSource src, const int32_t* __restrict__ lengths, int tokens, CacheShape s, CacheView c, int wide) {
  __shared__ uint4 code[512 * NS];                           // values: in the cache's order
  __shared__ float s_most[8];
  __shared__ int s_bad[8];
  const int b = blockIdx.y / s.heads, head = blockIdx.y % s.heads, blk = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
  const bool is_v = blockIdx.z;
  const int len = min(max(lengths[b], 0), tokens);
  if (t == 0 && head == 0 && blk == 0 && !is_v) c.lengths[b] = len;
  const int n = min(len - blk * CACHE_BLOCK, CACHE_BLOCK);   // valid tokens of the block
  if (n <= 0) return;                                        // (nothing reads it)
  const size_t tok = is_v ? src.v_tok : src.k_tok;
  const T* p = (const T*)(is_v ? src.v : src.k) + (size_t)b * (is_v ? src.v_seq : src.k_seq) + (size_t)head * (is_v ? src.v_head : src.k_head) +
               (size_t)blk * CACHE_BLOCK * tok;
  const int chunks = s.chunks(), slots = chunks * 128;       // at most 512 NS
  const bool wd = wide >> is_v & 1;
  Frag<T> x[NS][2];                                          // as they come: 16-bit ones take half the registers
  float most = 0.f;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int i = k * 512 + t, r = (i & 15) + 16 * (i >> 6 & 1), d = 64 * (i >> 7) + 16 * (i >> 4 & 3);
    fill_load(p + (size_t)r * tok + d, i < slots && r < n ? s.dim - d : 0, wd, x[k]);
  }
#pragma unroll
  for (int k = 0; k < NS; ++k)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float a = fabsf(x[k][e >> 3].get(e & 7));
      most = fmaxf(most, a);
      bad |= !(a <= 3.4028235e38f);
    }
  most = lanes_max(most);
  const bool any = __ballot(bad) != 0;
  if (lane == 0) { s_most[w] = most; s_bad[w] = any; }
  __syncthreads();
  bool finite = true;
#pragma unroll
  for (int k = 0; k < 8; ++k) { most = fmaxf(most, s_most[k]); finite &= !s_bad[k]; }
  const float scale = finite ? most / 127.0f : __uint_as_float(0x7fc00000u);   // (a block with a number that is none: no result hides it)
  const size_t at = ((size_t)b * s.heads + head) * s.blocks() + blk;
  if (t == 0) (is_v ? c.vscale : c.kscale)[at] = scale;
  const bool some = scale > 0.f, tiny = scale < 1e-36f;
  const float inv = 1.0f / scale;
  char* const out = (is_v ? c.v : c.k) + at * chunks * 2048;
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int i = k * 512 + t;
    uint32_t o[4] = {0, 0, 0, 0};
    if (tiny && some) {                                      // (uniform; 1 / scale may be infinite)
#pragma unroll 1
      for (int e = 0; e < 16; ++e) {
        float y = 0.f;
#pragma unroll
        for (int f = 0; f < 16; ++f) y = f == e ? x[k][f >> 3].get(f & 7) : y;
        const uint32_t q = (uint32_t)((int)fmin(fmax(rint((double)y / (double)scale), -127.0), 127.0) & 255) << (8 * (e & 3));
#pragma unroll
        for (int f = 0; f < 4; ++f) o[f] |= f == e >> 2 ? q : 0u;
      }
    } else if (some) {
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e >> 2] |= (uint32_t)((int)cache_code(x[k][e >> 3].get(e & 7), scale, inv) & 255) << (8 * (e & 3));
    }
    if (!is_v) {                                             // a slot is a lane's 16 bytes: [16-token tile][chunk][lane]
      if (i < slots) *reinterpret_cast<uint4*>(out + ((size_t)((i >> 6 & 1) * chunks + (i >> 7)) * 64 + (i & 63)) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
      continue;
    }
    // Four neighbouring lanes hold 16 d of four tokens.  Each takes four of the d from all of them (their dwords first, one lane after the
    // other), and then turns the 4 x 4 bytes over: a dword is four tokens of one d.
    auto give = [&](int j) {                                 // what lane ^ j takes
      const int want = (lane ^ j) & 3;
      return (int)(want == 0 ? o[0] : want == 1 ? o[1] : want == 2 ? o[2] : o[3]);
    };
    const uint32_t g[4] = {(uint32_t)give(0), (uint32_t)__builtin_amdgcn_update_dpp(0, give(1), 0xb1, 0xf, 0xf, true),
                           (uint32_t)__builtin_amdgcn_update_dpp(0, give(2), 0x4e, 0xf, 0xf, true),
                           (uint32_t)__builtin_amdgcn_update_dpp(0, give(3), 0x1b, 0xf, 0xf, true)};
    uint32_t a[4];                                           // by token: g[j] came from lane ^ j
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = (lane ^ r) & 3;
      a[r] = j == 0 ? g[0] : j == 1 ? g[1] : j == 2 ? g[2] : g[3];
    }
    const uint32_t p01 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400), q01 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602);   // d 0 1 and 2 3 of tokens 0, 1
    const uint32_t p23 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400), q23 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602);
    const uint32_t by[4] = {__builtin_amdgcn_perm(p23, p01, 0x05040100), __builtin_amdgcn_perm(p23, p01, 0x07060302),
                            __builtin_amdgcn_perm(q23, q01, 0x05040100), __builtin_amdgcn_perm(q23, q01, 0x07060302)};
    if (i < slots) {
      const int d = 64 * (i >> 7) + 16 * (i >> 4 & 3) + 4 * (lane & 3);
      uint32_t* const to = reinterpret_cast<uint32_t*>(code) + ((d >> 5) * 64 + 16 * (i >> 2 & 3) + (d & 15)) * 4 + 2 * (d >> 4 & 1) + (i >> 6 & 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) to[4 * e] = by[e];
    }
  }
  if (!is_v) return;
  __syncthreads();
  for (int i = t; i < slots; i += 512) reinterpret_cast<uint4*>(out)[i] = code[i];
}
void launch_cache_fill(int prec, const CacheSource& src, const int32_t* lengths, int tokens, const CacheShape& s, void* cache, hipStream_t st) {
  const size_t es = prec ? 2 : 4;
  auto wide = [&](const void* p, size_t a, size_t b, size_t c) { return (((uintptr_t)p | a * es | b * es | c * es) & 15) == 0; };
  const int flags = (wide(src.k, src.k_seq, src.k_tok, src.k_head) ? 1 : 0) | (wide(src.v, src.v_seq, src.v_tok, src.v_head) ? 2 : 0);
  const dim3 grid((unsigned)((tokens + CACHE_BLOCK - 1) / CACHE_BLOCK), (unsigned)(s.seqs * s.heads), 2);
  auto go = [&](auto type, auto ns) {
    hipLaunchKernelGGL((cache_fill_kernel<decltype(type), decltype(ns)::value>), grid, dim3(512), 0, st, src, lengths, tokens, s, CacheView(s, cache), flags);
  };
  auto by_width = [&](auto type) {
    if (s.chunks() <= 4) go(type, std::integral_constant<int, 1>());
    else if (s.chunks() <= 8) go(type, std::integral_constant<int, 2>());
    else go(type, std::integral_constant<int, 4>());
  };
  if (prec) by_width(bf16_t{}); else by_width(float{});
}

// ---- reading back: [seqs, tokens, heads, dim], 0 behind a sequence's end -------------------------------------
// One workgroup per block, sequence and head; blockIdx.z: keys, values.  The block's codes pass through LDS as they are.
__global__ __launch_bounds__(256) void cache_read_kernel(CacheShape s, CacheView c, int tokens, int wide, float* __restrict__ k, float* __restrict__ v) {
  __shared__ uint4 code[2048];
  const int b = blockIdx.y / s.heads, head = blockIdx.y % s.heads, blk = blockIdx.x, t = threadIdx.x;
  const bool is_v = blockIdx.z;
  const int chunks = s.chunks(), t0 = blk * CACHE_BLOCK;
  const int n = min(tokens - t0, CACHE_BLOCK), valid = min(c.lengths[b] - t0, n);
  const size_t at = ((size_t)b * s.heads + head) * s.blocks() + blk;
  float scale = 0.f;
  if (valid > 0) {
    const uint4* p = reinterpret_cast<const uint4*>((is_v ? c.v : c.k) + at * chunks * 2048);
    for (int i = t; i < chunks * 128; i += 256) code[i] = p[i];
    scale = (is_v ? c.vscale : c.kscale)[at];
  }
  __syncthreads();
  const int8_t* q = reinterpret_cast<const int8_t*>(code);
  float* const out = (is_v ? v : k) + (((size_t)b * tokens + t0) * s.heads + head) * s.dim;
  const size_t row = (size_t)s.heads * s.dim;
  const int quads = (s.dim + 3) / 4;
  for (int i = t; i < n * quads; i += 256) {
    const int r = i / quads, d = (i - r * quads) * 4, lo = r & 15, hi = r >> 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < valid) {
      const int8_t* o = q + (is_v ? (d >> 5) * 1024 + ((lo >> 2) * 16 + (d & 15)) * 16 + 8 * (d >> 4 & 1) + 4 * hi + (lo & 3)
                                  : (hi * chunks + (d >> 6)) * 1024 + ((d >> 4 & 3) * 16 + lo) * 16 + (d & 15));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (float)o[is_v ? 16 * e : e] * scale;
    }
    float* const to = out + r * row + d;
    if (wide) *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
    else
      for (int e = 0; e < 4; ++e) if (d + e < s.dim) to[e] = x[e];
  }
}
void launch_cache_read(const CacheShape& s, const void* cache, int tokens, float* k, float* v, hipStream_t st) {
  const dim3 grid((unsigned)((tokens + CACHE_BLOCK - 1) / CACHE_BLOCK), (unsigned)(s.seqs * s.heads), 2);
  const int wide = s.dim % 4 == 0 && (((uintptr_t)k | (uintptr_t)v) & 15) == 0;
  hipLaunchKernelGGL(cache_read_kernel, grid, dim3(256), 0, st, s, CacheView(s, const_cast<void*>(cache)), tokens, wide, k, v);
}

// ---- the attention -------------------------------------------------------------------------------------------
// 8 codes -> operand of 8 bf16 (exact)
__device__ __forceinline__ void cache_operand(uint32_t a, uint32_t b, Frag<bf16_t>& f) {
  auto two = [](uint32_t w, int sh) {
    const float x = (float)(int8_t)(w >> sh), y = (float)(int8_t)(w >> (sh + 8));
    return pack_hi(__float_as_uint(x), __float_as_uint(y));
  };
  f.v = make_uint4(two(a, 0), two(a, 16), two(b, 0), two(b, 16));
}

constexpr int ATTEND_WAVES = 8, ATTEND_CHUNK = 128, ATTEND_LD = ATTEND_CHUNK + 4, ATTEND_SPLITS = 512;
struct AttendPlan { int g_tiles, splits; };                 // tiles of 16 queries; ranges of the tokens
static AttendPlan attend_plan(const CacheShape& s, int per, int q_heads, int tokens) {
  AttendPlan p;
  p.g_tiles = (per * (q_heads / s.heads) + 15) / 16;
  const long units = (long)s.seqs * s.heads * p.g_tiles;
  const int chunks = std::max(1, (tokens + ATTEND_CHUNK - 1) / ATTEND_CHUNK);
  p.splits = (int)std::min<long>(std::min(chunks, ATTEND_SPLITS), std::max<long>(1, 512 / units));
  return p;
}
size_t cache_attend_workspace(const CacheShape& s, int per, int q_heads, int tokens) {
  const AttendPlan p = attend_plan(s, per, q_heads, tokens);
  if (p.splits == 1) return 0;
  return (size_t)s.seqs * s.heads * p.g_tiles * p.splits * 16 * (2 + (size_t)s.chunks() * 64) * 4;
}

struct AttendArgs {
  const void* q; size_t ldq; void* out; size_t ldo;
  int per, share, splits, tokens, wide_q, wide_o;           // queries in aligned pieces of 8; results of 4
  float scale;
  float* ml; float* part;                                    // of splits: (maximum, sum) [unit][split][16], products [unit][split][16][64 chunks]
};
// A workgroup takes one tile of 16 queries of a sequence and key head through a range of its tokens, 128 at a time: its wavefronts
// make the scores of 16 tokens each, then the weights together, then each the products of 32 EPW (of few d: of some of the tokens)
// columns of the values.
template <typename T, int EPW>
__global__ __launch_bounds__(64 * ATTEND_WAVES) void cache_attend_kernel(AttendArgs a, CacheShape s, CacheView c) {
  constexpr int QP = OPERAND_PARTS<T>, PP = QP + (QP == 1);
  constexpr bool FAST = sizeof(T) == 2;
  __shared__ uint4 s_q[8 * EPW * QP * 64];
  __shared__ __align__(16) float s_s[16 * ATTEND_LD];
  __shared__ __align__(16) uint4 s_p[4 * PP * 64];
  __shared__ float s_f[16], s_l[16], s_m[16];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int split = blockIdx.x, G = a.per * a.share, g0 = blockIdx.y * 16, unit = blockIdx.z * gridDim.y + blockIdx.y;
  const int b = s.heads == 1 ? blockIdx.z : blockIdx.z / s.heads, head = blockIdx.z - b * s.heads;
  const int len = min(c.lengths[b], a.tokens);
  const int chunks = s.chunks(), E = chunks * 2;
  const int span = ((len + ATTEND_CHUNK - 1) / ATTEND_CHUNK + a.splits - 1) / a.splits * ATTEND_CHUNK;   // of this sequence: equal shares
  const int first = split * span, last = min(len, first + span);
  const size_t at = ((size_t)b * s.heads + head) * s.blocks();
  const char* const kc = c.k + at * chunks * 2048;
  const char* const vc = c.v + at * chunks * 2048;
  const int q4 = lane >> 4, g = lane & 15;
  // row and column of the lane's query: number g of the tile
  const int qr = a.share == 1 ? g0 + g : (g0 + g) / a.share;
  const size_t row = (size_t)b * a.per + qr, column = (size_t)(head * a.share + (g0 + g - qr * a.share)) * s.dim;
  const int ts = E >= 6 ? 1 : 8 / E, mine = E >= 6 ? w * EPW : w % E, my_ts = E >= 6 ? 0 : w / E;   // columns 32 mine.., tokens' share
  v4f acc[EPW][2];
#pragma unroll
  for (int e = 0; e < EPW; ++e) acc[e][0] = acc[e][1] = v4f{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                              // of query t / 32, in its 32 threads
  // keys are asked for a chunk ahead, values before the chunk's scores are made: both are on their way in every phase.  Without ranges the
  // first of them do not wait for the sequence's length: what lies behind it is there, and not used.
  // Few tokens leave wavefronts without a tile: `parts` of them then share one, each some of its d.
  const int bound = a.splits == 1 ? a.tokens : last;
  const int parts = a.splits > 1 || a.tokens > 64 ? 1 : a.tokens > 32 ? 2 : a.tokens > 16 ? 4 : 8, tiles = 8 / parts;
  const int share = (chunks + parts - 1) / parts, ch0 = w / tiles * share, nch = min(share, chunks - ch0), my_tile = 16 * (w % tiles);
  uint4 kr[4 * EPW], vr[4][EPW];
  float ks = 0.f;
  auto fetch_keys = [&](int t0) {
    const int tile = t0 + my_tile;
    if (tile >= bound) return;
    const uint4* kp = reinterpret_cast<const uint4*>(kc + ((size_t)(tile >> 4) * chunks + ch0) * 1024) + lane;
#pragma unroll
    for (int ch = 0; ch < 4 * EPW; ++ch) if (ch < nch) kr[ch] = kp[ch * 64];
    ks = c.kscale[at + (tile >> 5)];
  };
  fetch_keys(first);
  if (first < bound) {                                       // the queries as operands: [chunk][half][part][lane]
    Frag<T> raw[EPW];
    const T* const qp = (const T*)a.q + (g0 + g < G ? row * a.ldq + column : 0);
#pragma unroll
    for (int u = 0; u < EPW; ++u) {                          // a thread's (lane, chunk, half) are those of its loads
      const int i = u * 8 + w, d = 64 * (i >> 1) + 16 * q4 + 8 * (i & 1);
      if (a.wide_q) raw[u].load(qp + (d < s.dim ? d : 0));
      else load_elements(qp + d, g0 + g < G ? s.dim - d : 0, raw[u]);
    }
#pragma unroll
    for (int u = 0; u < EPW; ++u) {
      const int i = u * 8 + w, d = 64 * (i >> 1) + 16 * q4 + 8 * (i & 1);
      Frag<bf16_t> f[QP];
      operand_of(raw[u], d < s.dim && g0 + g < G, f);
      if (i < 2 * chunks)
#pragma unroll
        for (int p = 0; p < QP; ++p) s_q[(i * QP + p) * 64 + lane] = f[p].v;
    }
  }
  __syncthreads();
  for (int t0 = first; t0 < last; t0 += ATTEND_CHUNK) {
    const int tok = t0 + 4 * (t & 31);
    const float vs = tok < bound ? c.vscale[at + (tok >> 5)] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int blk = my_ts + i * ts;
      if (blk >= ATTEND_CHUNK / CACHE_BLOCK || t0 + blk * CACHE_BLOCK >= bound) break;
      const uint4* vp = reinterpret_cast<const uint4*>(vc + (size_t)((t0 >> 5) + blk) * chunks * 2048) + lane;
#pragma unroll
      for (int e = 0; e < EPW; ++e) if (mine + e < E) vr[i][e] = vp[(mine + e) * 64];
    }
    if (t0 + my_tile < last) {
      v4f z[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int ch = 0; ch < 4 * EPW; ++ch)
        if (ch < nch) {
          Frag<bf16_t> k0, k1, qf;
          const uint4* const qp = s_q + (size_t)(ch0 + ch) * 2 * QP * 64 + lane;
          cache_operand(kr[ch].x, kr[ch].y, k0);
          cache_operand(kr[ch].z, kr[ch].w, k1);
#pragma unroll
          for (int p = QP - 1; p >= 0; --p) {
            qf.v = qp[p * 64]; mma16(z[0], k0, qf);
            qf.v = qp[(QP + p) * 64]; mma16(z[1], k1, qf);
          }
        }
      const float sc = ks * a.scale;
      *reinterpret_cast<float4*>(s_s + g * ATTEND_LD + 16 * w + 4 * q4) =
          make_float4((z[0][0] + z[1][0]) * sc, (z[0][1] + z[1][1]) * sc, (z[0][2] + z[1][2]) * sc, (z[0][3] + z[1][3]) * sc);
    }
    fetch_keys(t0 + ATTEND_CHUNK);
    __syncthreads();
    {
      const int i = t >> 5, j = t & 31;
      float x[4] = {0.f, 0.f, 0.f, 0.f}, mx = -INFINITY;
      if (j < 4 * tiles)
        for (int p = 0; p < parts; ++p) {
          const float4 x4 = *reinterpret_cast<const float4*>(s_s + i * ATTEND_LD + 16 * tiles * p + 4 * j);
          x[0] += x4.x; x[1] += x4.y; x[2] += x4.z; x[3] += x4.w;
        }
#pragma unroll
      for (int e = 0; e < 4; ++e) if (tok + e < last) mx = fmaxf(mx, x[e]);
      mx = half_max(mx);
      const float mn = fmaxf(m, mx), ms = mn > -INFINITY ? mn : 0.f;
      const float f = m > -INFINITY ? (FAST ? __expf(m - ms) : expf(m - ms)) : 0.f;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = tok + e < last ? (FAST ? __expf(x[e] - ms) : expf(x[e] - ms)) : 0.f;
        sum += x[e];
        x[e] = tok + e < last ? x[e] * vs : 0.f;
      }
      sum = half_sum(sum);
      l = l * f + sum;
      m = mn;
      if (j == 0) s_f[i] = f;
      // as an operand: token 4 c + e of the block's first half in slots 0..3 of quarter c, of its second half in slots 4..7
      uint2* const to = reinterpret_cast<uint2*>(s_p) + ((j >> 3) * PP * 64 + (j & 3) * 16 + i) * 2 + (j >> 2 & 1);
      if (PP == 2) {
        const uint32_t h0 = f2bf(x[0]), h1 = f2bf(x[1]), h2 = f2bf(x[2]), h3 = f2bf(x[3]);
        to[0] = make_uint2(h0 | h1 << 16, h2 | h3 << 16);
        const uint32_t l0 = f2bf(x[0] - bf2f((bf16_t)h0)), l1 = f2bf(x[1] - bf2f((bf16_t)h1)), l2 = f2bf(x[2] - bf2f((bf16_t)h2)),
                       l3 = f2bf(x[3] - bf2f((bf16_t)h3));
        to[128] = make_uint2(l0 | l1 << 16, l2 | l3 << 16);
      } else {
        const Parts3 a0 = parts3(x[0]), a1 = parts3(x[1]), a2 = parts3(x[2]), a3 = parts3(x[3]);
        to[0] = make_uint2(pack_hi(a0.h, a1.h), pack_hi(a2.h, a3.h));
        to[128] = make_uint2(pack_hi(a0.m, a1.m), pack_hi(a2.m, a3.m));
        to[256] = make_uint2(pack_hi(a0.l, a1.l), pack_hi(a2.l, a3.l));
      }
    }
    __syncthreads();
    const float f = s_f[g];
#pragma unroll
    for (int e = 0; e < EPW; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[e][h][i] *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int blk = my_ts + i * ts;
      if (blk >= ATTEND_CHUNK / CACHE_BLOCK || t0 + blk * CACHE_BLOCK >= last) break;
      Frag<bf16_t> pf[PP];
#pragma unroll
      for (int p = 0; p < PP; ++p) pf[p].v = s_p[(blk * PP + p) * 64 + lane];
#pragma unroll
      for (int e = 0; e < EPW; ++e)
        if (mine + e < E) {
          Frag<bf16_t> v0, v1;
          cache_operand(vr[i][e].x, vr[i][e].y, v0);
          cache_operand(vr[i][e].z, vr[i][e].w, v1);
#pragma unroll
          for (int p = PP - 1; p >= 0; --p) { mma16(acc[e][0], v0, pf[p]); mma16(acc[e][1], v1, pf[p]); }
        }
    }
  }
  if ((t & 31) == 0) { s_m[t >> 5] = m; s_l[t >> 5] = l; }
  if (ts > 1) {                                              // the tokens' shares of the same columns (E is 2 or 4: EPW is 1)
    __syncthreads();                                         // (also: the last weights have been read)
    float4* const red = reinterpret_cast<float4*>(s_q);      // 8 KB x QP: [wavefront][half][lane] is 16 KB where ts is 4 or 2
    // wavefronts of the upper shares hand over in turn, so that two halves of one wavefront's 2 KB fit
    for (int k = 1; k < ts; ++k) {
      if (my_ts == k) { red[(mine * 2) * 64 + lane] = make_float4(acc[0][0][0], acc[0][0][1], acc[0][0][2], acc[0][0][3]);
                        red[(mine * 2 + 1) * 64 + lane] = make_float4(acc[0][1][0], acc[0][1][1], acc[0][1][2], acc[0][1][3]); }
      __syncthreads();
      if (my_ts == 0)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 x = red[(mine * 2 + h) * 64 + lane];
          acc[0][h][0] += x.x; acc[0][h][1] += x.y; acc[0][h][2] += x.z; acc[0][h][3] += x.w;
        }
      __syncthreads();
    }
    if (my_ts) return;
  } else
    __syncthreads();
  if (a.splits > 1) {
    const size_t slot = (size_t)unit * a.splits + split;
    if (t < 16) { a.ml[(slot * 16 + t) * 2] = s_m[t]; a.ml[(slot * 16 + t) * 2 + 1] = s_l[t]; }
    if (first >= last || g0 + g >= G) return;
    float* part = a.part + (slot * 16 + g) * chunks * 64;
#pragma unroll
    for (int e = 0; e < EPW; ++e)
      if (mine + e < E)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float4*>(part + 32 * (mine + e) + 16 * h + 4 * q4) = make_float4(acc[e][h][0], acc[e][h][1], acc[e][h][2], acc[e][h][3]);
    return;
  }
  if (g0 + g >= G) return;
  const float sum = s_l[g], inv = sum == 0.f ? 0.f : 1.0f / sum;
  T* const out = (T*)a.out + row * a.ldo + column;
  struct alignas(4 * sizeof(T)) Four { T v[4]; };
#pragma unroll
  for (int e = 0; e < EPW; ++e)
    if (mine + e < E)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int d = 32 * (mine + e) + 16 * h + 4 * q4;
        const Four o{{from_f<T>(acc[e][h][0] * inv), from_f<T>(acc[e][h][1] * inv), from_f<T>(acc[e][h][2] * inv), from_f<T>(acc[e][h][3] * inv)}};
        if (a.wide_o) { if (d < s.dim) *reinterpret_cast<Four*>(out + d) = o; }
        else
#pragma unroll
          for (int i = 0; i < 4; ++i) if (d + i < s.dim) out[d + i] = o.v[i];
      }
}
// joins the ranges of a query: one workgroup each, its threads a column of four and a share of the ranges
template <typename T>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendArgs a, CacheShape s) {
  __shared__ float s_w[ATTEND_SPLITS];
  __shared__ float s_r[8];
  __shared__ float4 s_o[256];
  const int G = a.per * a.share, g_tiles = (G + 15) / 16, t = threadIdx.x, lane = t & 63, w = t >> 6;
  int u = blockIdx.x;
  const int g = u % G; u /= G;
  const int head = u % s.heads, b = u / s.heads;
  const size_t slot = ((size_t)(b * s.heads + head) * g_tiles + g / 16) * a.splits;
  const float2* ml = reinterpret_cast<const float2*>(a.ml) + slot * 16 + g % 16;
  const float none = -INFINITY;
  const float2 x0 = t < a.splits ? ml[t * 16] : make_float2(none, 0.f), x1 = t + 256 < a.splits ? ml[(t + 256) * 16] : make_float2(none, 0.f);
  float most = wave_max(fmaxf(x0.x, x1.x));
  if (lane == 0) s_r[w] = most;
  __syncthreads();
  most = fmaxf(fmaxf(s_r[0], s_r[1]), fmaxf(s_r[2], s_r[3]));
  const float ms = most > none ? most : 0.f;
  const float w0 = x0.y != 0.f ? expf(x0.x - ms) : 0.f, w1 = x1.y != 0.f ? expf(x1.x - ms) : 0.f;   // (a range without tokens: its products were not written)
  if (t < a.splits) s_w[t] = w0;
  if (t + 256 < a.splits) s_w[t + 256] = w1;
  const float sum = wave_sum(x0.y * w0 + x1.y * w1);
  if (lane == 0) s_r[4 + w] = sum;
  __syncthreads();
  const float all = s_r[4] + s_r[5] + s_r[6] + s_r[7], inv = all == 0.f ? 0.f : 1.0f / all;
  const int cols = s.chunks() * 16, shares = 256 / cols, col = t % cols, share = t / cols;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (share < shares) {
    const float4* p = reinterpret_cast<const float4*>(a.part) + (slot * 16 + g % 16) * cols + col;
#pragma unroll 4
    for (int k = share; k < a.splits; k += shares) {
      const float f = s_w[k];
      if (f == 0.f) continue;
      const float4 x = p[(size_t)k * 16 * cols];
      o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
    }
  }
  s_o[t] = o;
  __syncthreads();
  if (share) return;
  for (int k = 1; k < shares; ++k) { const float4 x = s_o[k * cols + col]; o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w; }
  T* const out = (T*)a.out + ((size_t)b * a.per + g / a.share) * a.ldo + (size_t)(head * a.share + g % a.share) * s.dim + 4 * col;
  const float r[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
#pragma unroll
  for (int e = 0; e < 4; ++e) if (4 * col + e < s.dim) out[e] = from_f<T>(r[e]);
}
void launch_cache_attend(int prec, const CacheShape& s, const void* cache, const void* q, size_t ldq, int per, int q_heads, int tokens, float scale,
                         void* out, size_t ldo, void* workspace, hipStream_t st) {
  const AttendPlan p = attend_plan(s, per, q_heads, tokens);
  const size_t es = prec ? 2 : 4;
  const long units = (long)s.seqs * s.heads * p.g_tiles;
  AttendArgs a{};
  a.q = q; a.ldq = ldq; a.out = out; a.ldo = ldo; a.per = per; a.share = q_heads / s.heads; a.splits = p.splits;
  a.tokens = tokens; a.scale = scale;
  a.wide_q = (((uintptr_t)q | ldq * es) & 15) == 0 && s.dim % 8 == 0;
  a.wide_o = (((uintptr_t)out | ldo * es | s.dim * es) & (4 * es - 1)) == 0;
  a.ml = (float*)workspace; a.part = a.ml + (size_t)units * p.splits * 32;
  auto go = [&](auto type, auto epw) {
    using T = decltype(type);
    hipLaunchKernelGGL((cache_attend_kernel<T, decltype(epw)::value>), dim3(p.splits, p.g_tiles, s.seqs * s.heads), dim3(64 * ATTEND_WAVES), 0, st, a, s,
                       CacheView(s, const_cast<void*>(cache)));
    if (p.splits > 1) hipLaunchKernelGGL(cache_join_kernel<T>, dim3((unsigned)((long)s.seqs * s.heads * per * a.share)), dim3(256), 0, st, a, s);
  };
  auto by_width = [&](auto type) {
    const int chunks = s.chunks();
    if (chunks <= 4) go(type, std::integral_constant<int, 1>());
    else if (chunks <= 8) go(type, std::integral_constant<int, 2>());
    else go(type, std::integral_constant<int, 4>());
  };
  if (prec) by_width(bf16_t{}); else by_width(float{});
}

}  // namespace cmt
