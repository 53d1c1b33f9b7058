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

// The whole numbers nearest to 16 quotients x / s, the even one of two, as if the quotients were exact; packed.  x inv + 1.5 2^23 has the code in its
// lowest bits, and is right wherever the remainder stays below half a step.  A slot with one that does not (a tie, or inv's rounding next to one) is
// corrected by the remainders, which are exact (below 2 s and multiples of half an ulp of s); so is one of a scale so small that inv or a remainder
// would leave fp32's range or precision, raised by a power of two (a scale rounded as a subnormal number: quotients up to 190).  (A division for
// every number: three times the instructions, which bound the fill: 128 x 55 x 1024 31 us.)
template <typename T>
__device__ __forceinline__ void cache_codes(const Frag<T> (&x)[2], float s, float inv, uint32_t (&o)[4]) {
  const float big = 12582912.f;
  float worst = 0.f;
  uint32_t c[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float v = x[e >> 3].get(e & 7), y = fmaf(v, inv, big);
    worst = fmaxf(worst, fabsf(fmaf(-(y - big), s, v)));
    c[e] = __float_as_uint(y);
  }
  if (s < 1e-36f || !(2.f * worst < s)) {
    const float up = s < 1e-36f ? 0x1p64f : 1.f, step = s * up, per = 1.f / step;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float v = x[e >> 3].get(e & 7) * up;
      float q = fmaf(v, per, big) - big;
      const float r = fmaf(-q, step, v), r2 = 2.f * fabsf(r);
      if (r2 > step || (r2 == step && ((int)q & 1))) q += copysignf(1.f, r);
      c[e] = (uint32_t)(int)fminf(fmaxf(q, -127.f), 127.f);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = __builtin_amdgcn_perm(c[4 * k + 1], c[4 * k], 0x0c0c0400), hi = __builtin_amdgcn_perm(c[4 * k + 3], c[4 * k + 2], 0x04000c0c);
    o[k] = lo | hi;
  }
}

// ---- writing ---------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void fill_load(const T* p, int n, Frag<T> (&x)[2]) {   // the first n of 16 elements, then 0
  if (n >= 16) { load_elements(p, 8, x[0]); load_elements(p + 8, 8, x[1]); }
  else { load_elements(p, n, x[0]); load_elements(p + 8, n - 8, x[1]); }
}
// One workgroup per block of 32 tokens, sequence and head (of few d: as many blocks as have a wavefront for every 32 d); blockIdx.z:
// keys, values.  A block is read once: a thread keeps its NS slots of 16 d of a token until the scale is known; 16-bit rows
// take the registers of three workgroups to a CU (96 d, 3 x 22432 tokens 22 -> 16 us).  Bound by the phases of a block, read, code, write, of which a
// CU holds three at a time: 128 x 55 x 1024 in 16 bits, 43 MB, 20 us.  (16 d, 4 heads x 7604 tokens, a workgroup per block: 29 us.)
__host__ __device__ inline int fill_blocks(int chunks) { return chunks > 4 ? 1 : 8 / chunks; }
template <typename T, int NS>
__global__ __launch_bounds__(512, sizeof(T) == 2 ? 6 : 4) void cache_fill_kernel(CacheSource src, const int32_t* __restrict__ lengths, int tokens, CacheShape s, CacheView c) {
  __shared__ uint4 code[512 * NS];                           // in the cache's order
  __shared__ uint32_t s_most[8];
  const int b = s.heads == 1 ? blockIdx.y : blockIdx.y / s.heads, head = blockIdx.y - b * s.heads, t = threadIdx.x, lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const bool is_v = blockIdx.z;
  const int len = min(max(lengths[b], 0), tokens);
  if (t == 0 && head == 0 && blockIdx.x == 0 && !is_v) c.lengths[b] = len;
  const int chunks = s.chunks(), slots = chunks * 64;        // at most 512 NS
  const int together = fill_blocks(chunks), mine = together == 1 ? 0 : w / chunks, w0 = mine * chunks, wn = together == 1 ? 8 : chunks;   // the block's wavefronts
  const int blk = blockIdx.x * together + mine, i0 = together == 1 ? t : t - 64 * w0;
  // Slot k 512 + i0: 16 d of a token, the thread's next one 256 d on.  Four lanes side by side are four tokens (their bytes are turned over below), the
  // next bits d: a load takes 128 bytes of 16 tokens (where the chunks are odd 64 of 32).
  const bool pairs = !(chunks & 1);
  const int r = (i0 & 3) | (pairs ? i0 >> 2 & 28 : i0 >> 1 & 28), d16_0 = pairs ? (i0 >> 2 & 3) | i0 >> 7 << 2 : (i0 >> 2 & 1) | i0 >> 6 << 1;
  const int n = mine < together ? min(len - blk * CACHE_BLOCK, CACHE_BLOCK) : 0;   // valid tokens of the block (none: nothing reads it)
  if (blockIdx.x * together * CACHE_BLOCK >= len) return;
  const size_t tok = is_v ? src.v_tok : src.k_tok;
  const T* p = (const T*)(is_v ? src.v : src.k) + (size_t)b * (is_v ? src.v_seq : src.k_seq) + (size_t)head * (is_v ? src.v_head : src.k_head) +
               ((size_t)blk * CACHE_BLOCK + r) * tok + 16 * d16_0;
  Frag<T> x[NS][2];                                          // as they come: 16-bit ones take half the registers
  uint32_t bits = 0;                                         // the largest without its sign: as numbers, infinities and NaN above all
#pragma unroll
  for (int k = 0; k < NS; ++k) fill_load(p + 256 * k, k * 512 + i0 < slots && r < n ? s.dim - 16 * d16_0 - 256 * k : 0, x[k]);
#pragma unroll
  for (int k = 0; k < NS; ++k)
#pragma unroll
    for (int e = 0; e < 16; ++e) bits = max(bits, __float_as_uint(x[k][e >> 3].get(e & 7)) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, o, 64));
  if (lane == 0) s_most[w] = bits;
  __syncthreads();
  for (int k = w0; k < min(w0 + wn, 8); ++k) bits = max(bits, s_most[k]);
  const bool finite = bits < 0x7f800000u;
  const float most = __uint_as_float(bits);
  const float scale = finite ? most / 127.0f : __uint_as_float(0x7fc00000u);   // (a block with a number that is none: no result hides it)
  const size_t at = ((size_t)b * s.heads + head) * s.blocks() + blk;
  if (i0 == 0 && n > 0) (is_v ? c.vscale : c.kscale)[at] = scale;
  const bool some = scale > 0.f;
  const float inv = 1.0f / scale;
  char* const out = (is_v ? c.v : c.k) + at * chunks * 1024;
  uint4* const block = code + 64 * w0;
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int i = k * 512 + i0, d16 = d16_0 + 16 * k;
    uint32_t o[4] = {0, 0, 0, 0};
    if (some) cache_codes(x[k], scale, inv, o);
    if (!is_v) {
      if (i < slots) {                                       // two lanes' pieces of 8 d
        uint2* const to = reinterpret_cast<uint2*>(block) + ((d16 >> 1) * 64 + 32 * (d16 & 1) + (r & 15)) * 2 + (r >> 4);
        to[0] = make_uint2(o[0], o[1]);
        to[32] = make_uint2(o[2], o[3]);
      }
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
    for (int u = 0; u < 4; ++u) {
      const int j = (lane ^ u) & 3;
      a[u] = j == 0 ? g[0] : j == 1 ? g[1] : j == 2 ? g[2] : g[3];
    }
    const uint32_t p01 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400), q01 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602);   // d 0 1 and 2 3 of tokens 0, 1
    const uint32_t p23 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400), q23 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602);
    const uint32_t by[4] = {__builtin_amdgcn_perm(p23, p01, 0x05040100), __builtin_amdgcn_perm(p23, p01, 0x07060302),
                            __builtin_amdgcn_perm(q23, q01, 0x05040100), __builtin_amdgcn_perm(q23, q01, 0x07060302)};
    if (i < slots) {
      uint32_t* const to = reinterpret_cast<uint32_t*>(block) + ((d16 >> 1) * 64 + 16 * (r >> 2 & 3) + 4 * (lane & 3)) * 4 + 2 * (d16 & 1) + (r >> 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) to[4 * e] = by[e];
    }
  }
  __syncthreads();
  if (n > 0)
    for (int i = i0; i < slots; i += 512) reinterpret_cast<uint4*>(out)[i] = block[i];
}
void launch_cache_fill(int prec, const CacheSource& src, const int32_t* lengths, int tokens, const CacheShape& s, void* cache, hipStream_t st) {
  const int blocks = (tokens + CACHE_BLOCK - 1) / CACHE_BLOCK, together = fill_blocks(s.chunks());
  const dim3 grid((unsigned)((blocks + together - 1) / together), (unsigned)(s.seqs * s.heads), 2);
  auto go = [&](auto type, auto ns) {
    hipLaunchKernelGGL((cache_fill_kernel<decltype(type), decltype(ns)::value>), grid, dim3(512), 0, st, src, lengths, tokens, s, CacheView(s, cache));
  };
  auto by_width = [&](auto type) {
    if (s.chunks() <= 8) go(type, std::integral_constant<int, 1>());
    else if (s.chunks() <= 16) go(type, std::integral_constant<int, 2>());
    else go(type, std::integral_constant<int, 4>());
  };
  if (prec) by_width(bf16_t{}); else by_width(float{});
}

// ---- reading back: [seqs, tokens, heads, dim], 0 behind a sequence's end -------------------------------------
// One workgroup per block, sequence and head; blockIdx.z: keys, values.  The block's codes pass through LDS as they are.
// Bound by the fp32 rows that it writes (128 x 80 x 1024 twice, 84 MB: 19.6 us).
__global__ __launch_bounds__(256) void cache_read_kernel(CacheShape s, CacheView c, int tokens, float* __restrict__ k, float* __restrict__ v) {
  __shared__ uint4 code[2048];
  const int b = blockIdx.y / s.heads, head = blockIdx.y % s.heads, blk = blockIdx.x, t = threadIdx.x;
  const bool is_v = blockIdx.z;
  const int chunks = s.chunks(), t0 = blk * CACHE_BLOCK;
  const int n = min(tokens - t0, CACHE_BLOCK), valid = min(c.lengths[b] - t0, n);
  const size_t at = ((size_t)b * s.heads + head) * s.blocks() + blk;
  float scale = 0.f;
  if (valid > 0) {
    const uint4* p = reinterpret_cast<const uint4*>((is_v ? c.v : c.k) + at * chunks * 1024);
    for (int i = t; i < chunks * 64; i += 256) code[(i & ~15) | ((i + (i >> 4)) & 15)] = p[i];   // (turned by its 16: else lanes read one bank)
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
      const int row = (d >> 5) * 4 + (is_v ? lo >> 2 : d >> 3 & 3), cell = is_v ? d & 15 : lo;
      const int8_t* o = q + row * 256 + (is_v ? 8 * (d >> 4 & 1) + 4 * hi + (lo & 3) : 8 * hi + (d & 7));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (float)o[((cell + (is_v ? e : 0) + row) & 15) * 16 + (is_v ? 0 : e)] * scale;
    }
    float* const to = out + r * row + d;
    if (s.dim % 4 == 0 || d + 4 <= s.dim) store_four(to, x[0], x[1], x[2], x[3]);
    else
      for (int e = 0; e < 4; ++e) if (d + e < s.dim) to[e] = x[e];
  }
}
void launch_cache_read(const CacheShape& s, const void* cache, int tokens, float* k, float* v, hipStream_t st) {
  const dim3 grid((unsigned)((tokens + CACHE_BLOCK - 1) / CACHE_BLOCK), (unsigned)(s.seqs * s.heads), 2);
  hipLaunchKernelGGL(cache_read_kernel, grid, dim3(256), 0, st, s, CacheView(s, const_cast<void*>(cache)), tokens, k, v);
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

constexpr int ATTEND_WAVES = 8, ATTEND_LD = 260, ATTEND_SPLITS = 512;
// tokens at a time: few columns leave a chunk short of work for its barriers (64 wide: 42 us with 256, 47 with 128; 128 wide: 53, 50)
static int attend_chunk(const CacheShape& s) { return s.chunks() <= 2 ? 256 : 128; }
// Tiles of 16 or 32 queries (32 share one turning of the codes into operands; of wide heads they would leave a CU one workgroup), and ranges
// of the tokens: as many as give two workgroups to a CU (8 documents of up to 32768 tokens, 4 heads: 512 workgroups 50 us, 1024 52, 2048 59).
struct AttendPlan { int tile, g_tiles, splits; };
static AttendPlan attend_plan(const CacheShape& s, int per, int q_heads, int tokens) {
  AttendPlan p;
  const int G = per * (q_heads / s.heads);
  p.tile = G > 16 && s.chunks() <= 8 ? 32 : 16;
  p.g_tiles = (G + p.tile - 1) / p.tile;
  const long units = (long)s.seqs * s.heads * p.g_tiles;
  const int chunks = (tokens + attend_chunk(s) - 1) / attend_chunk(s);
  p.splits = (int)std::min<long>(std::min(chunks, ATTEND_SPLITS), std::max<long>(1, 512 / units));
  return p;
}
size_t cache_attend_workspace(const CacheShape& s, int per, int q_heads, int tokens) {
  const AttendPlan p = attend_plan(s, per, q_heads, tokens);
  if (p.splits == 1) return 0;
  return (size_t)s.seqs * s.heads * p.g_tiles * p.splits * p.tile * (2 + (size_t)s.chunks() * 32) * 4;
}

struct AttendArgs {
  const void* q; size_t ldq; void* out; size_t ldo;
  int per, share, splits, tokens;
  float scale;
  float* ml; float* part;                                    // of ranges: (maximum, sum) [unit][range][tile], products [unit][range][tile][32 chunks]
};
// A workgroup takes one tile of 16 GT queries of a sequence and key head through a range of its tokens, 128 at a time: its wavefronts
// make the scores of 32 tokens each over a share of the d, then the weights together, then each the products of 32 EPW (of few
// d: of some of the tokens) columns of the values.  A few tokens are a chain of those phases (64 x 10 queries of 1024, 35 tokens: 10 us), many are
// bound by the read (8 documents of 20384 tokens, 4 heads of 128: 167 MB in 41 us, 4.1 TB/s).
template <typename T, int EPW, int GT, int BLK>
__global__ __launch_bounds__(64 * ATTEND_WAVES) void cache_attend_kernel(AttendArgs a, CacheShape s, CacheView c) {
  constexpr int QP = OPERAND_PARTS<T>, PP = QP + (QP == 1), CHUNK = 32 * BLK, QUADS = BLK / 4;
  constexpr bool FAST = sizeof(T) == 2;
  __shared__ uint4 s_q[GT][BLK == 8 ? 2 : 8 * EPW][QP][64];
  __shared__ __align__(16) float s_s[GT * 16 * ATTEND_LD];
  __shared__ __align__(16) uint4 s_p[GT][BLK][PP][64];
  __shared__ float s_f[GT * 16], s_l[GT * 16], s_m[GT * 16];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int split = blockIdx.x, G = a.per * a.share, g0 = blockIdx.y * 16 * GT, unit = blockIdx.z * gridDim.y + blockIdx.y;
  const int b = s.heads == 1 ? blockIdx.z : blockIdx.z / s.heads, head = blockIdx.z - b * s.heads;
  const int len = min(c.lengths[b], a.tokens);
  const int E = s.chunks();                                  // chunks of 32 d
  const int span = ((len + CHUNK - 1) / CHUNK + a.splits - 1) / a.splits * CHUNK;   // of this sequence: equal shares
  const int first = split * span, last = min(len, first + span);
  const size_t at = ((size_t)b * s.heads + head) * s.blocks();
  const char* const kc = c.k + at * E * 1024;
  const char* const vc = c.v + at * E * 1024;
  const int q4 = lane >> 4, g = lane & 15;
  // row and column of the lane's query in tile x: number 16 x + g
  auto row_of = [&](int x, size_t& column) {
    const int i = g0 + 16 * x + g, r = a.share == 1 ? i : i / a.share;
    column = (size_t)(head * a.share + (i - r * a.share)) * s.dim;
    return (size_t)b * a.per + r;
  };
  // columns 32 mine.., and of few columns a share of the tokens
  const int across = E >= 5 ? 8 : E >= 3 ? 4 : 2, ts = 8 / across, mine = E >= 5 ? w * EPW : w % across, my_ts = E >= 5 ? 0 : w / across;
  v4f acc[GT][EPW][2];
#pragma unroll
  for (int x = 0; x < GT; ++x)
#pragma unroll
    for (int e = 0; e < EPW; ++e) acc[x][e][0] = acc[x][e][1] = v4f{0.f, 0.f, 0.f, 0.f};
  float m[GT], l[GT];                                        // of query 16 x + t / 32, in its 32 threads
#pragma unroll
  for (int x = 0; x < GT; ++x) { m[x] = -INFINITY; l[x] = 0.f; }
  // Keys are asked for a chunk ahead, values before the chunk's scores are made: both are on their way in every phase.  Without ranges the
  // first of them do not wait for the sequence's length: what lies behind it is there, and not used.
  // `blocks` of 32 tokens at a time go to the wavefronts, `parts` of which share one: each takes some of its d.
  const int bound = a.splits == 1 ? a.tokens : last;
  const int blocks = a.splits > 1 || bound > CHUNK / 2 ? BLK : bound > 64 ? 4 : bound > 32 ? 2 : 1, parts = 8 / blocks, cols = 32 * blocks;
  const int share = (E + parts - 1) / parts, part = w / blocks, ch0 = part * share, nch = min(share, E - ch0), my_block = 32 * (w % blocks);
  uint4 kr[4 * EPW], vr[4][EPW];
  float ks = 0.f;
  auto fetch_keys = [&](int t0) {
    const int tok = t0 + my_block;
    if (tok >= bound) return;
    const uint4* kp = reinterpret_cast<const uint4*>(kc + ((size_t)(tok >> 5) * E + ch0) * 1024) + lane;
#pragma unroll
    for (int ch = 0; ch < 4 * EPW; ++ch) if (ch < nch) kr[ch] = kp[ch * 64];
    ks = c.kscale[at + (tok >> 5)];
  };
  fetch_keys(first);
  if (first < bound) {                                       // the queries as operands: [tile][chunk][part][lane]
    Frag<T> raw[GT][EPW];
    auto each = [&](auto f) {                                // f(the query's row, whether there is one, d, the fragment)
#pragma unroll
      for (int x = 0; x < GT; ++x) {
        size_t column;
        const size_t row = row_of(x, column);
        const bool in = g0 + 16 * x + g < G;
        const T* const qp = (const T*)a.q + (in ? row * a.ldq + column : 0);
#pragma unroll
        for (int u = 0; u < EPW; ++u) f(qp, in, 32 * (u * 8 + w) + 8 * q4, raw[x][u]);
      }
    };
    if (s.dim >= 8) {
      each([&](const T* qp, bool, int d, Frag<T>& f) { load_near(qp, d, s.dim, f); });
      if (s.dim % 8) each([&](const T*, bool, int d, Frag<T>& f) { move_near(d, s.dim, f); });
    } else {
      each([&](const T* qp, bool in, int d, Frag<T>& f) { load_elements(qp + d, in ? s.dim - d : 0, f); });
    }
#pragma unroll
    for (int x = 0; x < GT; ++x)
#pragma unroll
      for (int u = 0; u < EPW; ++u) {
        Frag<bf16_t> f[QP];
        operand_of(raw[x][u], 32 * (u * 8 + w) + 8 * q4 < s.dim && g0 + 16 * x + g < G, f);
        if (u * 8 + w < E)
#pragma unroll
          for (int p = 0; p < QP; ++p) s_q[x][u * 8 + w][p][lane] = f[p].v;
      }
  }
  __syncthreads();
  for (int t0 = first; t0 < last; t0 += CHUNK) {
    const int j = t & 31, col = 4 * QUADS * j, tok = t0 + col;   // the thread's tokens: 4 or 8, of one block
    const float vs = tok < bound ? c.vscale[at + (tok >> 5)] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int blk = my_ts + i * ts;
      if (blk >= BLK || t0 + blk * CACHE_BLOCK >= bound) break;
      const uint4* vp = reinterpret_cast<const uint4*>(vc + (size_t)((t0 >> 5) + blk) * E * 1024) + lane;
#pragma unroll
      for (int e = 0; e < EPW; ++e) if (mine + e < E) vr[i][e] = vp[(mine + e) * 64];
    }
    if (t0 + my_block < last) {
      v4f z[GT][2];
#pragma unroll
      for (int x = 0; x < GT; ++x) z[x][0] = z[x][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < 4 * EPW; ++ch)
        if (ch < nch) {
          Frag<bf16_t> k0, k1, qf;
          cache_operand(kr[ch].x, kr[ch].y, k0);
          cache_operand(kr[ch].z, kr[ch].w, k1);
#pragma unroll
          for (int p = QP - 1; p >= 0; --p)
#pragma unroll
            for (int x = 0; x < GT; ++x) { qf.v = s_q[x][ch0 + ch][p][lane]; mma16(z[x][0], k0, qf); mma16(z[x][1], k1, qf); }
        }
      const float sc = ks * a.scale;
#pragma unroll
      for (int x = 0; x < GT; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float4*>(s_s + (16 * x + g) * ATTEND_LD + part * cols + my_block + 16 * h + 4 * q4) =
              make_float4(z[x][h][0] * sc, z[x][h][1] * sc, z[x][h][2] * sc, z[x][h][3] * sc);
    }
    fetch_keys(t0 + CHUNK);
    __syncthreads();
#pragma unroll
    for (int gx = 0; gx < GT; ++gx) {
      const int i = 16 * gx + (t >> 5);
      float x[4 * QUADS], mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4 * QUADS; ++e) x[e] = 0.f;
      if (col < cols)
        for (int p = 0; p < parts; ++p) {
          if (p * share >= E) break;                         // (fewer chunks than shares)
#pragma unroll
          for (int u = 0; u < QUADS; ++u) {
            const float4 x4 = *reinterpret_cast<const float4*>(s_s + i * ATTEND_LD + p * cols + col + 4 * u);
            x[4 * u] += x4.x; x[4 * u + 1] += x4.y; x[4 * u + 2] += x4.z; x[4 * u + 3] += x4.w;
          }
        }
#pragma unroll
      for (int e = 0; e < 4 * QUADS; ++e) if (tok + e < last) mx = fmaxf(mx, x[e]);
      mx = half_max(mx);
      const float mn = fmaxf(m[gx], mx), ms = mn > -INFINITY ? mn : 0.f;
      const float f = m[gx] > -INFINITY ? (FAST ? __expf(m[gx] - ms) : expf(m[gx] - ms)) : 0.f;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4 * QUADS; ++e) {
        x[e] = tok + e < last ? (FAST ? __expf(x[e] - ms) : expf(x[e] - ms)) : 0.f;
        sum += x[e];
        x[e] = tok + e < last ? x[e] * vs : 0.f;
      }
      sum = half_sum(sum);
      l[gx] = l[gx] * f + sum;
      m[gx] = mn;
      if (j == 0) s_f[i] = f;
      // as an operand: token 4 c + e of the block's first half in slots 0..3 of quarter c, of its second half in slots 4..7
#pragma unroll
      for (int u = 0; u < QUADS; ++u) {
        const int fours = QUADS * j + u;
        uint2* const to = reinterpret_cast<uint2*>(&s_p[gx][fours >> 3][0][(fours & 3) * 16 + (t >> 5)]) + (fours >> 2 & 1);
        const float* y = x + 4 * u;
        if (PP == 2) {
          const uint32_t h0 = f2bf(y[0]), h1 = f2bf(y[1]), h2 = f2bf(y[2]), h3 = f2bf(y[3]);
          to[0] = make_uint2(h0 | h1 << 16, h2 | h3 << 16);
          const uint32_t l0 = f2bf(y[0] - bf2f((bf16_t)h0)), l1 = f2bf(y[1] - bf2f((bf16_t)h1)), l2 = f2bf(y[2] - bf2f((bf16_t)h2)),
                         l3 = f2bf(y[3] - bf2f((bf16_t)h3));
          to[128] = make_uint2(l0 | l1 << 16, l2 | l3 << 16);
        } else {
          const Parts3 a0 = parts3(y[0]), a1 = parts3(y[1]), a2 = parts3(y[2]), a3 = parts3(y[3]);
          to[0] = make_uint2(pack_hi(a0.h, a1.h), pack_hi(a2.h, a3.h));
          to[128] = make_uint2(pack_hi(a0.m, a1.m), pack_hi(a2.m, a3.m));
          to[256] = make_uint2(pack_hi(a0.l, a1.l), pack_hi(a2.l, a3.l));
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < GT; ++x) {
      const float f = s_f[16 * x + g];
#pragma unroll
      for (int e = 0; e < EPW; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[x][e][h][i] *= f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int blk = my_ts + i * ts;
      if (blk >= BLK || t0 + blk * CACHE_BLOCK >= last) break;
      Frag<bf16_t> pf[GT][PP];
#pragma unroll
      for (int x = 0; x < GT; ++x)
#pragma unroll
        for (int p = 0; p < PP; ++p) pf[x][p].v = s_p[x][blk][p][lane];
#pragma unroll
      for (int e = 0; e < EPW; ++e)
        if (mine + e < E) {
          Frag<bf16_t> v0, v1;
          cache_operand(vr[i][e].x, vr[i][e].y, v0);
          cache_operand(vr[i][e].z, vr[i][e].w, v1);
#pragma unroll
          for (int x = 0; x < GT; ++x)
#pragma unroll
            for (int p = PP - 1; p >= 0; --p) { mma16(acc[x][e][0], v0, pf[x][p]); mma16(acc[x][e][1], v1, pf[x][p]); }
        }
    }
  }
  if ((t & 31) == 0)
#pragma unroll
    for (int x = 0; x < GT; ++x) { s_m[16 * x + (t >> 5)] = m[x]; s_l[16 * x + (t >> 5)] = l[x]; }
  __syncthreads();                                           // (also: the last scores have been read)
  if (ts > 1) {                                              // the tokens' shares of the same columns (at most 4 of them: EPW is 1)
    float4* const red = reinterpret_cast<float4*>(s_s);      // [column of 32][half][lane], 8 KB, tile by tile and share by share
#pragma unroll
    for (int x = 0; x < GT; ++x)
      for (int k = 1; k < ts; ++k) {
        if (my_ts == k)
#pragma unroll
          for (int h = 0; h < 2; ++h) red[(mine * 2 + h) * 64 + lane] = make_float4(acc[x][0][h][0], acc[x][0][h][1], acc[x][0][h][2], acc[x][0][h][3]);
        __syncthreads();
        if (my_ts == 0)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float4 r = red[(mine * 2 + h) * 64 + lane];
            acc[x][0][h][0] += r.x; acc[x][0][h][1] += r.y; acc[x][0][h][2] += r.z; acc[x][0][h][3] += r.w;
          }
        __syncthreads();
      }
    if (my_ts) return;
  }
  if (a.splits > 1) {
    const size_t slot = ((size_t)unit * a.splits + split) * 16 * GT;
    if (t < 16 * GT) { a.ml[(slot + t) * 2] = s_m[t]; a.ml[(slot + t) * 2 + 1] = s_l[t]; }
    if (first >= last) return;
#pragma unroll
    for (int x = 0; x < GT; ++x) {
      if (g0 + 16 * x + g >= G) continue;
      float* const to = a.part + (slot + 16 * x + g) * E * 32;
#pragma unroll
      for (int e = 0; e < EPW; ++e)
        if (mine + e < E)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *reinterpret_cast<float4*>(to + 32 * (mine + e) + 16 * h + 4 * q4) = make_float4(acc[x][e][h][0], acc[x][e][h][1], acc[x][e][h][2], acc[x][e][h][3]);
    }
    return;
  }
#pragma unroll
  for (int x = 0; x < GT; ++x) {
    if (g0 + 16 * x + g >= G) continue;
    const float sum = s_l[16 * x + g], inv = sum == 0.f ? 0.f : 1.0f / sum;
    size_t column;
    const size_t row = row_of(x, column);
    T* const out = (T*)a.out + row * a.ldo + column;
#pragma unroll
    for (int e = 0; e < EPW; ++e)
      if (mine + e < E)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int d = 32 * (mine + e) + 16 * h + 4 * q4;
          const v4f& y = acc[x][e][h];
          if (s.dim % 4 == 0) {
            if (d < s.dim) store_four(out + d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
          } else if (d + 4 <= s.dim) store_four(out + d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
          else
#pragma unroll
            for (int i = 0; i < 4; ++i) if (d + i < s.dim) out[d + i] = from_f<T>(y[i] * inv);
        }
  }
}
// joins the ranges of a query: a workgroup for 64 columns of four, its threads a column and a share of the ranges
template <typename T>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendArgs a, CacheShape s, int tile) {
  __shared__ float s_w[ATTEND_SPLITS];
  __shared__ float s_r[8];
  __shared__ float4 s_o[256];
  const int G = a.per * a.share, g_tiles = (G + tile - 1) / tile, t = threadIdx.x, lane = t & 63, w = t >> 6;
  int u = blockIdx.x;
  const int g = u % G; u /= G;
  const int head = u % s.heads, b = u / s.heads;
  const size_t slot = ((size_t)(b * s.heads + head) * g_tiles + g / tile) * a.splits * tile + g % tile;
  const float2* ml = reinterpret_cast<const float2*>(a.ml) + slot;
  const float none = -INFINITY;
  const float2 x0 = t < a.splits ? ml[t * tile] : make_float2(none, 0.f), x1 = t + 256 < a.splits ? ml[(t + 256) * tile] : make_float2(none, 0.f);
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
  const int all_cols = s.chunks() * 8, cols = min(64, all_cols), shares = 256 / cols, share = t / cols, col = blockIdx.y * 64 + t - share * cols;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (share < shares && col < all_cols) {
    const float4* p = reinterpret_cast<const float4*>(a.part) + slot * all_cols + col;
#pragma unroll 4
    for (int k = share; k < a.splits; k += shares) {
      const float f = s_w[k];
      if (f == 0.f) continue;
      const float4 x = p[(size_t)k * tile * all_cols];
      o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
    }
  }
  s_o[t] = o;
  __syncthreads();
  if (share || col >= all_cols) return;
  for (int k = 1; k < shares; ++k) { const float4 x = s_o[k * cols + t]; o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w; }
  T* const out = (T*)a.out + ((size_t)b * a.per + g / a.share) * a.ldo + (size_t)(head * a.share + g % a.share) * s.dim + 4 * col;
  const float r[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
#pragma unroll
  for (int e = 0; e < 4; ++e) if (4 * col + e < s.dim) out[e] = from_f<T>(r[e]);
}
void launch_cache_attend(int prec, const CacheShape& s, const void* cache, const void* q, size_t ldq, int per, int q_heads, int tokens, float scale,
                         void* out, size_t ldo, void* workspace, hipStream_t st) {
  const AttendPlan p = attend_plan(s, per, q_heads, tokens);
  const long units = (long)s.seqs * s.heads * p.g_tiles;
  AttendArgs a{};
  a.q = q; a.ldq = ldq; a.out = out; a.ldo = ldo; a.per = per; a.share = q_heads / s.heads; a.splits = p.splits;
  a.tokens = tokens; a.scale = scale;
  a.ml = (float*)workspace; a.part = a.ml + (size_t)units * p.splits * p.tile * 2;
  auto go = [&](auto type, auto epw, auto gt, auto blk) {
    using T = decltype(type);
    hipLaunchKernelGGL((cache_attend_kernel<T, decltype(epw)::value, decltype(gt)::value, decltype(blk)::value>), dim3(p.splits, p.g_tiles, s.seqs * s.heads), dim3(64 * ATTEND_WAVES),
                       0, st, a, s, CacheView(s, const_cast<void*>(cache)));
    if (p.splits > 1) hipLaunchKernelGGL(cache_join_kernel<T>, dim3((unsigned)((long)s.seqs * s.heads * per * a.share), (s.chunks() + 7) / 8), dim3(256), 0, st, a, s, p.tile);
  };
  auto by_width = [&](auto type) {
    using std::integral_constant;
    const int chunks = s.chunks();
    const integral_constant<int, 1> one; const integral_constant<int, 2> two; const integral_constant<int, 4> four; const integral_constant<int, 8> eight;
    if (attend_chunk(s) == 256) { if (p.tile == 32) go(type, one, two, eight); else go(type, one, one, eight); }
    else if (chunks <= 8) { if (p.tile == 32) go(type, one, two, four); else go(type, one, one, four); }
    else if (chunks <= 16) go(type, two, one, four);
    else go(type, four, one, four);
  };
  if (prec) by_width(bf16_t{}); else by_width(float{});
}

}  // namespace cmt
