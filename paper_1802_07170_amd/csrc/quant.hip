// Products with 4-bit weights: y = f(x W^T + b), W[n, k] = e2m1(code) * scale[n, k / group], for the few rows that a decoder has.
//
// A code is one of 0, .5, 1, 1.5, 2, 3, 4, 6 and a sign: all exact in bf16, so the products with bf16 operands (or with the three bf16
// parts of an fp32 one) are exact and their sums fp32; a group's sum is scaled in fp32 behind its matrix instructions.
// One row needs N K / 2 bytes of weights and does 2 flop a weight: the read bounds it until some hundred rows share it.
#include "lowbit.h"

namespace cmt {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// dword of 8 codes -> operand of 8 bf16, exact: one instruction for two codes
__device__ __forceinline__ void quant_operand(uint32_t w, Frag<bf16_t>& f) {
  f.v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
  f.v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
  f.v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
  f.v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
}

// ---- laying out -----------------------------------------------------------------------------------------
__device__ __forceinline__ size_t quant_dword(int n, int k, int k_tiles) {   // where the 8 codes from k (a multiple of 8) on are
  return ((size_t)(n >> 4) * k_tiles + (k >> 7)) * 256 + (((k >> 3) & 3) * 16 + (n & 15)) * 4 + ((k >> 5) & 3);
}
// One thread per 8 weights; the threads of a group are neighbours.  scale = bf16(max|w| / 6), code = the nearest one (the even one of two);
// a group with a weight that is no finite number has the scale NaN, so that no product hides it.
template <typename T>
__global__ __launch_bounds__(256) void quant_pack_kernel(const T* __restrict__ w, size_t ldw, QuantShape q, int gates, int k_tiles, int row_blocks,
                                                         uint32_t* __restrict__ codes, bf16_t* __restrict__ scales) {
  const int per_row = k_tiles * (QUANT_TILE_K / 8), share = q.group / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t n = i / per_row;                              // (per_row is a multiple of 16: a group's threads are in one row)
  const int k = (int)(i - n * per_row) * 8;
  if (n >= (size_t)row_blocks * 16) return;
  const size_t from = gates ? (n & 3) * (q.N >> 2) + (n >> 2) : n;
  float x[8], most = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = n < (size_t)q.N && k + e < q.K ? to_f(w[from * ldw + k + e]) : 0.f;
    bad |= !(fabsf(x[e]) <= 3.4028235e38f);
    most = fmaxf(most, fabsf(x[e]));
  }
  if (bad) most = INFINITY;
  for (int o = 1; o < share; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
  const bf16_t sb = most < INFINITY ? f2bf(most / 6.0f) : (bf16_t)0x7fc0;
  const float s = bf2f(sb);
  uint32_t word = 0;
  if (s > 0.f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = fabsf(x[e]) / s;
      const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
      word |= (c | (x[e] < 0.f ? 8u : 0u)) << (4 * e);
    }
  }
  codes[quant_dword((int)n, k, k_tiles)] = word;
  if (k % q.group == 0) scales[((n >> 4) * (size_t)k_tiles * (QUANT_TILE_K / q.group) + k / q.group) * 16 + (n & 15)] = sb;
}
void launch_quant_pack(int prec, const void* w, size_t ldw, const QuantShape& q, bool gates, void* packed, hipStream_t st) {
  const size_t threads = (size_t)q.row_blocks() * 16 * q.k_tiles() * (QUANT_TILE_K / 8);
  const dim3 grid((unsigned)((threads + 255) / 256));
  bf16_t* scales = (bf16_t*)((char*)packed + q.code_bytes());
  if (prec)
    hipLaunchKernelGGL(quant_pack_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)w, ldw, q, gates, q.k_tiles(), q.row_blocks(), (uint32_t*)packed, scales);
  else
    hipLaunchKernelGGL(quant_pack_kernel<float>, grid, dim3(256), 0, st, (const float*)w, ldw, q, gates, q.k_tiles(), q.row_blocks(), (uint32_t*)packed, scales);
}
// codes [N, K] one to a byte (the lower four bits count), scales [N, ceil(K / group)]
__global__ __launch_bounds__(256) void quant_encode_kernel(const uint8_t* __restrict__ src, const bf16_t* __restrict__ src_scales, QuantShape q,
                                                           int k_tiles, int row_blocks, uint32_t* __restrict__ codes, bf16_t* __restrict__ scales) {
  const int per_row = k_tiles * (QUANT_TILE_K / 8);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t n = i / per_row;
  const int k = (int)(i - n * per_row) * 8;
  if (n >= (size_t)row_blocks * 16) return;
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (n < (size_t)q.N && k + e < q.K) word |= (uint32_t)(src[n * q.K + k + e] & 15) << (4 * e);
  codes[quant_dword((int)n, k, k_tiles)] = word;
  const int groups = (q.K + q.group - 1) / q.group;
  if (k % q.group == 0)
    scales[((n >> 4) * (size_t)k_tiles * (QUANT_TILE_K / q.group) + k / q.group) * 16 + (n & 15)] =
        n < (size_t)q.N && k / q.group < groups ? src_scales[n * groups + k / q.group] : (bf16_t)0;
}
void launch_quant_encode(const uint8_t* codes, const bf16_t* scales, const QuantShape& q, void* packed, hipStream_t st) {
  const size_t threads = (size_t)q.row_blocks() * 16 * q.k_tiles() * (QUANT_TILE_K / 8);
  hipLaunchKernelGGL(quant_encode_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, codes, scales, q, q.k_tiles(), q.row_blocks(),
                     (uint32_t*)packed, (bf16_t*)((char*)packed + q.code_bytes()));
}
__global__ __launch_bounds__(128) void quant_values_kernel(const uint32_t* __restrict__ codes, const bf16_t* __restrict__ scales, QuantShape q,
                                                           int k_tiles, float* __restrict__ out) {
  const size_t n = blockIdx.x;
  const int k = blockIdx.y * 128 + threadIdx.x;
  if (k >= q.K) return;
  const uint32_t c = codes[quant_dword((int)n, k & ~7, k_tiles)] >> (4 * (k & 7)) & 15;
  const uint32_t e = c & 7;                                  // two exponent bits, one of the mantissa
  const float size = e < 2 ? 0.5f * e : (1.0f + 0.5f * (e & 1)) * (float)(1 << ((e >> 1) - 1));
  const float s = bf2f(scales[((n >> 4) * (size_t)k_tiles * (QUANT_TILE_K / q.group) + k / q.group) * 16 + (n & 15)]);
  out[n * q.K + k] = (c & 8 ? -size : size) * s;
}
void launch_quant_values(const void* packed, const QuantShape& q, float* out, hipStream_t st) {
  hipLaunchKernelGGL(quant_values_kernel, dim3(q.N, q.k_tiles()), dim3(128), 0, st, (const uint32_t*)packed,
                     (const bf16_t*)((const char*)packed + q.code_bytes()), q, q.k_tiles(), out);
}

// Four neighbouring outputs of row m; flags: 1 tanh, 2 y in bf16, 16 they are the gates of an LSTM's unit.
// An LSTM layer's weight is packed with a unit's four gates side by side, so that the lane that ends up with them makes the unit's cell: no
// gates in memory and no launch for the cells (10 rows, width 1024: 5.0 us a layer against 4.4 + 2.6; 640 rows 38 against 37 + 5).
struct QuantCell { const float* c_prev; float* c; void *h, *h2; size_t ldh, ldh2; };
template <typename T>
__device__ __forceinline__ void quant_store(float a, float b, float c, float d, int m, int n, int N, const float* __restrict__ bias, int flags,
                                            void* __restrict__ y, size_t ldy, const QuantCell& cell) {
  if (flags & 16) {
    constexpr bool FAST = sizeof(T) == 2;
    const int H = N >> 2, u = n >> 2;
    const float in = sigm_of<FAST>(a + bias[u]), forget = sigm_of<FAST>(b + bias[H + u]), out = sigm_of<FAST>(d + bias[3 * H + u]);
    const float x = forget * cell.c_prev[(size_t)m * H + u] + in * tanh_of<FAST>(c + bias[2 * H + u]);
    const T h = from_f<T>(out * tanh_of<FAST>(x));
    cell.c[(size_t)m * H + u] = x;
    ((T*)cell.h)[m * cell.ldh + u] = h;
    ((T*)cell.h2)[m * cell.ldh2 + u] = h;
    return;
  }
  float r[4] = {a, b, c, d};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (bias && n + e < N) r[e] += bias[n + e];
    if (flags & 1) r[e] = tanhf(r[e]);
  }
  if (flags & 2) {
    bf16_t* o = (bf16_t*)y + (size_t)m * ldy + n;
    if (n + 4 <= N) store_four(o, r[0], r[1], r[2], r[3]);
    else
      for (int e = 0; e < 4; ++e) if (n + e < N) o[e] = f2bf(r[e]);
  } else {
    float* o = (float*)y + (size_t)m * ldy + n;
    if (n + 4 <= N) store_four(o, r[0], r[1], r[2], r[3]);
    else
      for (int e = 0; e < 4; ++e) if (n + e < N) o[e] = r[e];
  }
}

// ---- the product -------------------------------------------------------------------------------------------
// A workgroup makes NT row blocks of the weight for CT tiles of 16 rows of x; its wavefronts split k, tile by tile, and add
// up through LDS.  The weight is the instruction's first operand: a lane then holds 4 neighbouring outputs of one row of x.
// (bf16, groups of 64: 1 x 4096 x 2048 4.0 us, one trip to HBM and the sum; 10 x 32000 x 1024 7.8 us, 2.3 TB/s of codes: they are read before
// all workgroups have started.)
constexpr int QUANT_WAVES = 8;
template <typename T, int GROUP, int NT, int CT, bool WHOLE>
__global__ __launch_bounds__(64 * QUANT_WAVES) void quant_product_kernel(const T* __restrict__ x, size_t ldx, const uint4* __restrict__ codes,
                                                                         const bf16_t* __restrict__ scales, int M, int N, int K, int k_tiles,
                                                                         int row_blocks, int m_blocks, const float* __restrict__ bias, int flags,
                                                                         void* __restrict__ y, size_t ldy, QuantCell cell) {
  constexpr int PARTS = OPERAND_PARTS<T>, PER = QUANT_TILE_K / GROUP, STEPS = GROUP / 32;
  __shared__ float4 red[QUANT_WAVES][NT * CT][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroups that share weights are neighbours on one XCD (workgroups go to the 8 XCDs in turn)
  const int id = blockIdx.x, seq = id >> 3, mb = seq % m_blocks, nb = ((seq / m_blocks) * 8 + (id & 7)) * NT;
  if (nb >= row_blocks) return;
  const int m0 = mb * 16 * CT, q = lane >> 4, c = lane & 15;
  v4f acc[NT][CT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  for (int kt = w; kt < k_tiles; kt += QUANT_WAVES) {
    uint4 code[NT];
    uint2 sc[NT][PER];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const size_t tile = (size_t)min(nb + i, row_blocks - 1) * k_tiles + kt;
      code[i] = codes[tile * 64 + lane];
#pragma unroll
      for (int g = 0; g < PER; ++g) sc[i][g] = *reinterpret_cast<const uint2*>(scales + (tile * PER + g) * 16 + 4 * q);
    }
    Frag<bf16_t> xf[CT][4][PARTS];
    Frag<T> xr[CT][4];
    auto each = [&](auto f) {                                // f(row of x, k, the fragment)
#pragma unroll
      for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) f(x + (size_t)min(m0 + 16 * j + c, M - 1) * ldx, kt * QUANT_TILE_K + 32 * s + 8 * q, xr[j][s]);   // (rows beyond M: not stored)
    };
    if constexpr (WHOLE) {
      each([&](const T* row, int k, Frag<T>& f) { f.load(row + (k < K ? k : 0)); });
    } else if (K >= 8) {
      each([&](const T* row, int k, Frag<T>& f) { load_near(row, k, K, f); });
      if (kt == k_tiles - 1) each([&](const T*, int k, Frag<T>& f) { move_near(k, K, f); });
    } else {
      each([&](const T* row, int k, Frag<T>& f) { load_elements(row + k, K - k, f); });
    }
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int s = 0; s < 4; ++s) operand_of(xr[j][s], !WHOLE || kt * QUANT_TILE_K + 32 * s + 8 * q < K, xf[j][s]);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int g = 0; g < PER; ++g) {
        v4f part[CT];
#pragma unroll
        for (int j = 0; j < CT; ++j) part[j] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
          const int s = g * STEPS + t;
          Frag<bf16_t> wf;
          quant_operand((&code[i].x)[s], wf);
#pragma unroll
          for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) mma16(part[j], wf, xf[j][s][p]);
        }
        const float s0 = __uint_as_float(sc[i][g].x << 16), s1 = __uint_as_float(sc[i][g].x & 0xffff0000u);
        const float s2 = __uint_as_float(sc[i][g].y << 16), s3 = __uint_as_float(sc[i][g].y & 0xffff0000u);
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          acc[i][j][0] = fmaf(part[j][0], s0, acc[i][j][0]);
          acc[i][j][1] = fmaf(part[j][1], s1, acc[i][j][1]);
          acc[i][j][2] = fmaf(part[j][2], s2, acc[i][j][2]);
          acc[i][j][3] = fmaf(part[j][3], s3, acc[i][j][3]);
        }
      }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) red[w][i * CT + j][lane] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
  __syncthreads();
  const int used = min(QUANT_WAVES, k_tiles);
  for (int o = threadIdx.x; o < NT * CT * 64; o += 64 * QUANT_WAVES) {
    const int t = o >> 6, l = o & 63;
    float4 v = red[0][t][l];
    for (int k = 1; k < used; ++k) {
      const float4 u = red[k][t][l];
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    const int m = m0 + 16 * (t % CT) + (l & 15), n = (nb + t / CT) * 16 + 4 * (l >> 4);
    if (m >= M || n >= N) continue;
    quant_store<T>(v.x, v.y, v.z, v.w, m, n, N, bias, flags, y, ldy, cell);
  }
}

// ---- many rows -----------------------------------------------------------------------------------------------
// From some dozens of rows on the matrix instructions and the trips of x to the CUs bound the product, not the weights' read.  A workgroup
// of 4 x 2 wavefronts makes 256 outputs for 32 MT rows: x comes through LDS, 128 k at a time and a tile ahead, in operand order; a
// wavefront turns its 64 x 128 codes into operands once per tile (they stay in registers) and passes its MT tiles of rows by them.
// 640 x 32000 x 1024, groups of 128: 61 us, 0.69 PFLOP/s.  Per tile 1.2 us of matrix instructions, 0.5 of codes and scales that they do not hide, 0.6 of
// loads; then 82 MB are written.
constexpr int QUANT_WIDE = 512;
template <typename T, int GROUP, int MT, bool WHOLE>
__global__ __launch_bounds__(QUANT_WIDE) void quant_product_wide_kernel(const T* __restrict__ x, size_t ldx, const uint4* __restrict__ codes,
                                                                 const bf16_t* __restrict__ scales, int M, int N, int K, int k_tiles, int row_blocks,
                                                                 int m_blocks, const float* __restrict__ bias, int flags, void* __restrict__ y,
                                                                 size_t ldy, QuantCell cell) {
  constexpr int PARTS = OPERAND_PARTS<T>, PER = QUANT_TILE_K / GROUP, STEPS = GROUP / 32, WN = 4, NT = 4;
  constexpr bool DIRECT = WHOLE && sizeof(T) == 2;
  constexpr int THREADS = QUANT_WIDE, SLOTS = 2 * MT * 4 * 64, MINE = SLOTS / THREADS;
  // Slots of 8 k of x: row slot / 16, and in it chunk (slot ^ row) % 16 - a load takes whole lines of four rows, and the 16 rows of an operand lie
  // in 16 different banks' worth of LDS.  (16 rows x 64 bytes to a load, in operand order: 5 of 67 us more.)
  __shared__ uint4 xs[2][PARTS][SLOTS];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = w >> 1, wm = w & 1;
  const int id = blockIdx.x, seq = id >> 3, mb = seq % m_blocks, nb = ((seq / m_blocks) * 8 + (id & 7)) * NT * WN + wn * NT;
  if (nb - wn * NT >= row_blocks) return;
  const int m0 = mb * 32 * MT, q = lane >> 4, c = lane & 15;
  v4f acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  const uint4* cp[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) cp[i] = codes + (size_t)min(nb + i, row_blocks - 1) * k_tiles * 64 + lane;
  Frag<T> xn[MINE];                                          // as they come: nothing waits for them before they go to LDS
  uint4 code[NT];
  uint2 sn[NT][PER];
  const bf16_t* const sp = scales + 4 * q;
  // 16-bit rows of whole pieces go from memory to LDS without passing registers (the instruction is written out because the compiler would
  // wait for it before the next read of LDS); the last tile's pieces behind K are zeros.
  auto chunk_of = [](int slot) { return (slot ^ slot >> 4) & 15; };
  unsigned off[MINE];
  const char* const xb = (const char*)(x + (size_t)m0 * ldx);
  if constexpr (DIRECT) {
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
      const int slot = u * THREADS + threadIdx.x, m = min(m0 + (slot >> 4), M - 1) - m0;
      off[u] = ((unsigned)m * (unsigned)ldx + 8 * chunk_of(slot)) * 2;
    }
  }
  auto request = [&](int kt, uint4* to) {
    const char* const src = xb + (size_t)kt * QUANT_TILE_K * 2;
    if ((kt + 1) * QUANT_TILE_K <= K) {
#pragma unroll
      for (int u = 0; u < MINE; ++u) {
        const unsigned dst = (unsigned)(size_t)(__attribute__((address_space(3))) const char*)(to + u * THREADS + w * 64);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off[u]), "s"(src) : "memory");
      }
    } else {
#pragma unroll
      for (int u = 0; u < MINE; ++u) {
        const int slot = u * THREADS + threadIdx.x;
        const bool in = kt * QUANT_TILE_K + 8 * chunk_of(slot) < K;
        to[slot] = in ? *reinterpret_cast<const uint4*>(src + off[u]) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  auto fetch = [&](int kt) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      code[i] = cp[i][(size_t)kt * 64];
#pragma unroll
      for (int g = 0; g < PER; ++g)
        sn[i][g] = *reinterpret_cast<const uint2*>(sp + (((size_t)min(nb + i, row_blocks - 1) * k_tiles + kt) * PER + g) * 16);
    }
    if constexpr (DIRECT) return;
    auto each = [&](auto f) {                                // f(row of x, k, the fragment)
#pragma unroll
      for (int u = 0; u < MINE; ++u) {
        const int slot = u * THREADS + threadIdx.x;
        f(x + (size_t)min(m0 + (slot >> 4), M - 1) * ldx, kt * QUANT_TILE_K + 8 * chunk_of(slot), xn[u]);   // (rows beyond M: not stored)
      }
    };
    if constexpr (WHOLE) each([&](const T* row, int k, Frag<T>& f) { f.load(row + (k < K ? k : 0)); });
    else if (K >= 8) each([&](const T* row, int k, Frag<T>& f) { load_near(row, k, K, f); });
    else each([&](const T* row, int k, Frag<T>& f) { load_elements(row + k, K - k, f); });
  };
  if constexpr (DIRECT) request(0, xs[0][0]);
  fetch(0);
  for (int kt = 0; kt < k_tiles; ++kt) {
    uint4 (&buf)[PARTS][SLOTS] = xs[kt & 1];
    if constexpr (!DIRECT)
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
      const int slot = u * THREADS + threadIdx.x;
      Frag<bf16_t> f[PARTS];
      if constexpr (!WHOLE)
        if (kt == k_tiles - 1 && K >= 8) move_near(kt * QUANT_TILE_K + 8 * chunk_of(slot), K, xn[u]);
      operand_of(xn[u], !WHOLE || kt * QUANT_TILE_K + 8 * chunk_of(slot) < K, f);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) buf[p][slot] = f[p].v;
    }
    Frag<bf16_t> wf[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int s = 0; s < 4; ++s) quant_operand((&code[i].x)[s], wf[i][s]);
    uint2 sc[NT][PER];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int g = 0; g < PER; ++g)
        sc[i][g] = sn[i][g];
    if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < k_tiles) {
      if constexpr (DIRECT) request(kt + 1, xs[(kt + 1) & 1][0]);
      fetch(kt + 1);
    }
    // the next step's x is asked of LDS before a step's products begin
    constexpr int SEQ = MT * 4;
    Frag<bf16_t> xf[2][PARTS];
    auto read = [&](int i, Frag<bf16_t> (&f)[PARTS]) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p) f[p].v = buf[p][(wm * MT + (i >> 2)) * 256 + c * 16 + ((4 * (i & 3) + q) ^ c)];
    };
    read(0, xf[0]);
    // a group's sums are scaled while the next group's products are being made
    v4f part[2][NT];
    auto scale = [&](int group) {
      const int j = group / PER, g = group % PER;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const v4f& y = part[group & 1][n];
        acc[n][j][0] = fmaf(y[0], __uint_as_float(sc[n][g].x << 16), acc[n][j][0]);
        acc[n][j][1] = fmaf(y[1], __uint_as_float(sc[n][g].x & 0xffff0000u), acc[n][j][1]);
        acc[n][j][2] = fmaf(y[2], __uint_as_float(sc[n][g].y << 16), acc[n][j][2]);
        acc[n][j][3] = fmaf(y[3], __uint_as_float(sc[n][g].y & 0xffff0000u), acc[n][j][3]);
      }
    };
#pragma unroll
    for (int i = 0; i < SEQ; ++i) {
      const int s = i & 3, group = i / STEPS;
      if (i + 1 < SEQ) read(i + 1, xf[(i + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
      if (i % STEPS == 0)
#pragma unroll
        for (int n = 0; n < NT; ++n) part[group & 1][n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16(part[group & 1][n], wf[n][s], xf[i & 1][p]);
      if (i % STEPS == 0 && group > 0) scale(group - 1);
    }
    scale(SEQ / STEPS - 1);
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int n = (nb + i) * 16 + 4 * q;
    if (n >= N) continue;
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m0 + 16 * (wm * MT + j) + c;
      if (m < M) quant_store<T>(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], m, n, N, bias, flags, y, ldy, cell);
    }
  }
}

template <typename T, int GROUP, int NT, int CT>
static void quant_product_go(const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy, const QuantCell& cell,
                             hipStream_t st) {
  const QuantShape& q = w.shape;
  const int m_blocks = (M + 16 * CT - 1) / (16 * CT);
  const int n_blocks = ((q.row_blocks() + NT - 1) / NT + 7) / 8 * 8;
  auto* kernel = flags & 4 ? quant_product_kernel<T, GROUP, NT, CT, true> : quant_product_kernel<T, GROUP, NT, CT, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)n_blocks * m_blocks), dim3(64 * QUANT_WAVES), 0, st, (const T*)x, ldx, (const uint4*)w.packed,
                     (const bf16_t*)(w.packed + q.code_bytes()), M, q.N, q.K, q.k_tiles(), q.row_blocks(), m_blocks, bias, flags, y, ldy, cell);
}
template <typename T, int GROUP, int MT>
static void quant_product_wide_go(const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy,
                                  const QuantCell& cell, hipStream_t st) {
  const QuantShape& q = w.shape;
  const int m_blocks = (M + 32 * MT - 1) / (32 * MT), n_blocks = ((q.row_blocks() + 15) / 16 + 7) / 8 * 8;
  auto* kernel = flags & 4 ? quant_product_wide_kernel<T, GROUP, MT, true> : quant_product_wide_kernel<T, GROUP, MT, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)n_blocks * m_blocks), dim3(QUANT_WIDE), 0, st, (const T*)x, ldx, (const uint4*)w.packed,
                     (const bf16_t*)(w.packed + q.code_bytes()), M, q.N, q.K, q.k_tiles(), q.row_blocks(), m_blocks, bias, flags, y, ldy, cell);
}
// Which kernel and tile, by sizes alone; times are of whole calls, us, 11 of them the host's (bf16 unless said).
//   Many rows: k is not split there, so it takes workgroups of 64 rows for most of the chip.  32000 x 1024, groups of 128 | 32: 64 rows
//   15 | 23 with k split against 17 | 26, 96 rows 21 | 32 against 19 | 27, 640 rows 108 | 187 against 78 | 116; 4096 x 2048, 640 rows (160
//   workgroups) 27 | 42 against 30 | 44.  More rows to a workgroup (as many as a wavefront's registers hold the sums of beside the
//   scales of its groups: 160 rows with groups of 128, 128 of 64) where rounds of workgroups times their rows are fewer: 640 rows 62 against 78, 128 rows 28 against 18.
//   Else two tiles of rows to a workgroup where there are two (640 rows 108 against 129; fp32, whose parts are three times the registers, 285
//   against 226: one), and four row blocks of the weight, which share x, where one each would be 512 workgroups or more (4096 x 2048, 128 rows
//   11 against 18; 512 x 4096 in fp32, 128 rows 17 against 12).  Few rows of many inputs have little to share (without the host's share: 10000 x 4096, 1 | 4 | 8
//   rows 13 against 8.3 | 9.6 | 11.6; 16000 x 2048, 1 | 4 | 8 rows 8.4 against 6.6 | 7.4 | 8.7; 30000 x 1024, 1 | 2 | 4 rows 6.9 against 6.6 | 6.6 | 7.5): one
//   row block from 512 inputs a row on (in fp32 the parts cost more than that: 16.7 against 20.7).
template <typename T, int GROUP>
static void quant_product_tiles(const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy,
                                const QuantCell& cell, hipStream_t st) {
  constexpr int MOST = sizeof(T) == 4 || GROUP == 32 ? 2 : GROUP == 64 ? 4 : 5, CT = sizeof(T) == 4 ? 1 : 2;
  const long rb = w.shape.row_blocks();
  auto wgs = [&](int mt) { return (rb + 15) / 16 * ((M + 32 * mt - 1) / (32 * mt)); };
  if (M > 64 && wgs(2) >= 200) {
    if constexpr (MOST > 2)
      if ((wgs(MOST) + 255) / 256 * (MOST + 1) <= (wgs(2) + 255) / 256 * 3) { quant_product_wide_go<T, GROUP, MOST>(x, ldx, w, M, bias, flags, y, ldy, cell, st); return; }
    quant_product_wide_go<T, GROUP, 2>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
    return;
  }
  if constexpr (CT > 1)
    if (M > 16) {
      if (rb * ((M + 31) / 32) < 512) quant_product_go<T, GROUP, 1, CT>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
      else quant_product_go<T, GROUP, 4, CT>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
      return;
    }
  if (rb * ((M + 15) / 16) < 512 || (sizeof(T) == 2 && 512l * M <= w.shape.K)) quant_product_go<T, GROUP, 1, 1>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
  else quant_product_go<T, GROUP, 4, 1>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
}
static void quant_product_any(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy,
                              const QuantCell& cell, hipStream_t st) {
  if (((uintptr_t)x | ldx * (prec ? 2 : 4)) % 16 == 0 && w.shape.K % 8 == 0 && ldx <= 1 << 20) flags |= 4;
  auto go = [&](auto type) {
    using T = decltype(type);
    if (w.shape.group == 32) quant_product_tiles<T, 32>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
    else if (w.shape.group == 64) quant_product_tiles<T, 64>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
    else quant_product_tiles<T, 128>(x, ldx, w, M, bias, flags, y, ldy, cell, st);
  };
  if (prec) go(bf16_t{}); else go(float{});
}
void launch_quant_product(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, bool tanh, int y_prec, void* y,
                          size_t ldy, hipStream_t st) {
  quant_product_any(prec, x, ldx, w, M, bias, (tanh ? 1 : 0) | (y_prec ? 2 : 0), y, ldy, QuantCell{}, st);
}
void launch_quant_lstm(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, const float* c_prev, float* c, void* h,
                       size_t ldh, void* h2, size_t ldh2, hipStream_t st) {
  quant_product_any(prec, x, ldx, w, M, bias, 16, nullptr, 0, QuantCell{c_prev, c, h, h2, ldh, ldh2}, st);
}

}  // namespace cmt
