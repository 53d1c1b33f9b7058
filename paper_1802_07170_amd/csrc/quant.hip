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
__global__ __launch_bounds__(256) void quant_pack_kernel(const T* __restrict__ w, size_t ldw, QuantShape q, int k_tiles, int row_blocks,
                                                         uint32_t* __restrict__ codes, bf16_t* __restrict__ scales) {
  const int per_row = k_tiles * (QUANT_TILE_K / 8), share = q.group / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t n = i / per_row;                              // (per_row is a multiple of 16: a group's threads are in one row)
  const int k = (int)(i - n * per_row) * 8;
  if (n >= (size_t)row_blocks * 16) return;
  float x[8], most = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = n < (size_t)q.N && k + e < q.K ? to_f(w[n * ldw + k + e]) : 0.f;
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
void launch_quant_pack(int prec, const void* w, size_t ldw, const QuantShape& q, void* packed, hipStream_t st) {
  const size_t threads = (size_t)q.row_blocks() * 16 * q.k_tiles() * (QUANT_TILE_K / 8);
  const dim3 grid((unsigned)((threads + 255) / 256));
  bf16_t* scales = (bf16_t*)((char*)packed + q.code_bytes());
  if (prec)
    hipLaunchKernelGGL(quant_pack_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)w, ldw, q, q.k_tiles(), q.row_blocks(), (uint32_t*)packed, scales);
  else
    hipLaunchKernelGGL(quant_pack_kernel<float>, grid, dim3(256), 0, st, (const float*)w, ldw, q, q.k_tiles(), q.row_blocks(), (uint32_t*)packed, scales);
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
__global__ __launch_bounds__(256) void quant_values_kernel(const uint32_t* __restrict__ codes, const bf16_t* __restrict__ scales, QuantShape q,
                                                           int k_tiles, float* __restrict__ out) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)q.N * q.K) return;
  const size_t n = i / q.K;
  const int k = (int)(i - n * q.K);
  const uint32_t c = codes[quant_dword((int)n, k & ~7, k_tiles)] >> (4 * (k & 7)) & 15;
  const uint32_t e = c & 7;                                  // two exponent bits, one of the mantissa
  const float size = e < 2 ? 0.5f * e : (1.0f + 0.5f * (e & 1)) * (float)(1 << ((e >> 1) - 1));
  const float s = bf2f(scales[((n >> 4) * (size_t)k_tiles * (QUANT_TILE_K / q.group) + k / q.group) * 16 + (n & 15)]);
  out[i] = (c & 8 ? -size : size) * s;
}
void launch_quant_values(const void* packed, const QuantShape& q, float* out, hipStream_t st) {
  const size_t n = (size_t)q.N * q.K;
  hipLaunchKernelGGL(quant_values_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const uint32_t*)packed,
                     (const bf16_t*)((const char*)packed + q.code_bytes()), q, q.k_tiles(), out);
}

// ---- the product -------------------------------------------------------------------------------------------
// A workgroup makes NT row blocks of the weight for CT tiles of 16 rows of x; its wavefronts split k, tile by tile, and add
// up through LDS.  The weight is the instruction's first operand: a lane then holds 4 neighbouring outputs of one row of x.
constexpr int QUANT_WAVES = 8;
template <typename T, int GROUP, int NT, int CT>
__global__ __launch_bounds__(64 * QUANT_WAVES) void quant_product_kernel(const T* __restrict__ x, size_t ldx, const uint4* __restrict__ codes,
                                                                         const bf16_t* __restrict__ scales, int M, int N, int K, int k_tiles,
                                                                         int row_blocks, int m_blocks, const float* __restrict__ bias, int flags,
                                                                         void* __restrict__ y, size_t ldy) {
  constexpr int PARTS = OPERAND_PARTS<T>, PER = QUANT_TILE_K / GROUP, STEPS = GROUP / 32;
  __shared__ float4 red[QUANT_WAVES][NT * CT][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroups that share weights are neighbours on one XCD (workgroups go to the 8 XCDs in turn)
  const int id = blockIdx.x, seq = id >> 3, mb = seq % m_blocks, nb = ((seq / m_blocks) * 8 + (id & 7)) * NT;
  if (nb >= row_blocks) return;
  const int m0 = mb * 16 * CT, q = lane >> 4, c = lane & 15;
  const bool wide = flags & 4;
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
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const int m = m0 + 16 * j + c;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = kt * QUANT_TILE_K + 32 * s + 8 * q;
        load_operand(x + (m < M ? (size_t)m * ldx + k : 0), m < M ? K - k : 0, wide, xf[j][s]);
      }
    }
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
    float r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (bias && n + e < N) r[e] += bias[n + e];
      if (flags & 1) r[e] = tanhf(r[e]);
    }
    if (flags & 2) {
      bf16_t* d = (bf16_t*)y + (size_t)m * ldy + n;
      if ((flags & 8) && n + 4 <= N) *reinterpret_cast<uint2*>(d) = make_uint2(f2bf(r[0]) | (uint32_t)f2bf(r[1]) << 16, f2bf(r[2]) | (uint32_t)f2bf(r[3]) << 16);
      else
        for (int e = 0; e < 4; ++e) if (n + e < N) d[e] = f2bf(r[e]);
    } else {
      float* d = (float*)y + (size_t)m * ldy + n;
      if ((flags & 8) && n + 4 <= N) *reinterpret_cast<float4*>(d) = make_float4(r[0], r[1], r[2], r[3]);
      else
        for (int e = 0; e < 4; ++e) if (n + e < N) d[e] = r[e];
    }
  }
}
template <typename T, int GROUP, int NT, int CT>
static void quant_product_go(const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy, hipStream_t st) {
  const QuantShape& q = w.shape;
  const int m_blocks = (M + 16 * CT - 1) / (16 * CT);
  const int n_blocks = ((q.row_blocks() + NT - 1) / NT + 7) / 8 * 8;
  hipLaunchKernelGGL((quant_product_kernel<T, GROUP, NT, CT>), dim3((unsigned)n_blocks * m_blocks), dim3(64 * QUANT_WAVES), 0, st, (const T*)x, ldx,
                     (const uint4*)w.packed, (const bf16_t*)(w.packed + q.code_bytes()), M, q.N, q.K, q.k_tiles(), q.row_blocks(), m_blocks, bias, flags,
                     y, ldy);
}
template <typename T, int GROUP>
static void quant_product_tiles(const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, int flags, void* y, size_t ldy,
                                hipStream_t st) {
  const int rb = w.shape.row_blocks();
  if (M <= 16) {
    if (rb <= 512) quant_product_go<T, GROUP, 1, 1>(x, ldx, w, M, bias, flags, y, ldy, st);
    else quant_product_go<T, GROUP, 4, 1>(x, ldx, w, M, bias, flags, y, ldy, st);
  } else {
    if (rb <= 512) quant_product_go<T, GROUP, 1, 2>(x, ldx, w, M, bias, flags, y, ldy, st);
    else quant_product_go<T, GROUP, 4, 2>(x, ldx, w, M, bias, flags, y, ldy, st);
  }
}
void launch_quant_product(int prec, const void* x, size_t ldx, const QuantWeightRef& w, int M, const float* bias, bool tanh, int y_prec, void* y,
                          size_t ldy, hipStream_t st) {
  const size_t xs = prec ? 2 : 4, ys = y_prec ? 2 : 4;
  const int flags = (tanh ? 1 : 0) | (y_prec ? 2 : 0) | (((uintptr_t)x | ldx * xs) % 16 == 0 ? 4 : 0) | (((uintptr_t)y | ldy * ys) % (4 * ys) == 0 ? 8 : 0);
  auto go = [&](auto type) {
    using T = decltype(type);
    if (w.shape.group == 32) quant_product_tiles<T, 32>(x, ldx, w, M, bias, flags, y, ldy, st);
    else if (w.shape.group == 64) quant_product_tiles<T, 64>(x, ldx, w, M, bias, flags, y, ldy, st);
    else quant_product_tiles<T, 128>(x, ldx, w, M, bias, flags, y, ldy, st);
  };
  if (prec) go(bf16_t{}); else go(float{});
}

}  // namespace cmt
