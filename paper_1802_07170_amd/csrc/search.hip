// A beam search's choice on logits that the caller has, and the rows that follow it.
//
// Extension v of hypothesis s scores c_s + z_sv - lse_s.  The logits are read once: a wavefront leaves the maximum and the sum of
// exponentials of every 512 of them.  One workgroup per sentence then has each row's lse from those, finds the n groups whose best
// extensions are best - they hold the n best extensions - and reads their entries again, n x 512.  Extensions are compared in 64
// bits, equal ones by (slot, token): the first is better.  The first pass is bound by its read (640 x 32000 in fp32 15 us, 5.4 TB/s), the second by
// its chain of steps (10 hypotheses a sentence: 6.6 us for one sentence, 7.0 for 64).
#include <algorithm>

#include "lowbit.h"

namespace cmt {

__device__ __forceinline__ unsigned search_sortable(float v) {   // larger numbers as larger unsigned ones
  const unsigned u = __float_as_uint(v + 0.f);
  return u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}
// ---- statistics of the groups ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void search_groups_kernel(const T* __restrict__ logits, size_t ld, const float* __restrict__ scores, int rows, int V,
                                                            int groups, float2* __restrict__ stat) {
  const int lane = threadIdx.x & 63;
  const int id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = id / groups, g = id - row * groups;
  if (row >= rows || !(scores[row] > -INFINITY)) return;     // (nothing reads a dead row's)
  const T* p = logits + (size_t)row * ld;
  const int v0 = g * SEARCH_GROUP;
  float x[8];
  if (v0 + SEARCH_GROUP <= V) {                              // (wherever the row begins)
    if (sizeof(T) == 2) {
      Frag<T> f;
      load_elements(p + v0 + 8 * lane, 8, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = f.get(i);
    } else {
      __builtin_memcpy(x, p + v0 + 4 * lane, 16);
      __builtin_memcpy(x + 4, p + v0 + 256 + 4 * lane, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v0 + 64 * i + lane < V ? to_f(p[v0 + 64 * i + lane]) : -INFINITY;
  }
  float mx = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);          // (a NaN is never the largest, but is in the sum)
  mx = lanes_max(mx);
  const float ms = mx > -INFINITY ? mx : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += expf(x[i] - ms);
  sum = lanes_sum(sum);
  if (lane == 0) stat[id] = make_float2(mx, sum);
}

// ---- the choice --------------------------------------------------------------------------------------------
// One workgroup per sentence, a wavefront to a hypothesis (two where there are more than 16).  With 16 wavefronts every instruction takes 16 clocks of
// the CU: what bounds this kernel is how many there are, so rows and groups go by wavefronts and lanes and by shifts, without divisions.
constexpr int SELECT_WAVES = 16, SELECT_CAP = 1024, SELECT_BATCH = 8;
constexpr int GROUP_BITS = 17, TOKEN_BITS = 26;              // (slot, group) and (slot, token) as ordered numbers
static_assert(SEARCH_MAX_VOCAB == 1 << TOKEN_BITS && SEARCH_MAX_VOCAB / SEARCH_GROUP == 1 << GROUP_BITS && SEARCH_MAX == 32, "31 bits");
__device__ __forceinline__ bool better(double a, unsigned ia, double b, unsigned ib) { return a > b || (a == b && ia < ib); }

struct SelectShared {
  double base[SEARCH_MAX];
  double lv[SELECT_CAP]; unsigned li[SELECT_CAP];            // a list of candidates
  double wv[SEARCH_MAX]; unsigned wi[SEARCH_MAX];            // the best of them, in order
  float reach[SELECT_WAVES];
  double rv[SELECT_WAVES]; unsigned ri[SELECT_WAVES];
  int count;
};
// appends the candidates of the lanes with `take`: one atomic per wavefront
__device__ __forceinline__ void select_append(SelectShared& sh, bool take, double v, unsigned index) {
  const unsigned long long mask = __ballot(take);
  if (!mask) return;
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (lane == 0) at = atomicAdd(&sh.count, __popcll(mask));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(mask & ((1ull << lane) - 1));
  if (take && at < SELECT_CAP) { sh.lv[at] = v; sh.li[at] = index; }
}
// The n best candidates into sh.wv / sh.wi (returns how many there are): a wavefront counts, 64 at a time, how many are better than one (a thread that
// goes through the list for each: 2.3 us for 22 candidates, against 0.6).  A list that has overflowed - equal values in great
// number - is answered by n rounds of a maximum over all items: scan(f) passes a thread's items to f(value, index).
template <typename F>
__device__ __forceinline__ int select_best(SelectShared& sh, int n, F scan) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, threads = blockDim.x;
  __syncthreads();
  const int count = sh.count;
  if (count <= SELECT_CAP) {
    const double v0 = sh.lv[lane];                           // (behind the list's end: anything)
    const unsigned i0 = sh.li[lane];
    for (int i = __builtin_amdgcn_readfirstlane(w); i < count; i += threads >> 6) {
      const double v = sh.lv[i];
      const unsigned ix = sh.li[i];
      int place = __popcll(__ballot(lane < count && better(v0, i0, v, ix)));
      for (int k0 = 64; k0 < count; k0 += 64) {
        const int k = min(k0 + lane, SELECT_CAP - 1);
        place += __popcll(__ballot(k0 + lane < count && better(sh.lv[k], sh.li[k], v, ix)));
      }
      if (lane == 0 && place < n) { sh.wv[place] = v; sh.wi[place] = ix; }
    }
    __syncthreads();
    return min(count, n);
  }
  double last = INFINITY;
  unsigned last_index = 0;
#pragma unroll 1
  for (int round = 0; round < n; ++round) {                  // (more than SELECT_CAP take part: there is a best one in each round)
    double bv = -INFINITY;
    unsigned bi = 0xffffffffu;
    scan([&](double v, unsigned index) {
      if (v > -INFINITY && (round == 0 || better(last, last_index, v, index)) && better(v, index, bv, bi)) { bv = v; bi = index; }
    });
#pragma unroll 1
    for (int o = 32; o > 0; o >>= 1) {
      const double ov = __shfl_xor(bv, o, 64);
      const unsigned oi = __shfl_xor(bi, o, 64);
      if (better(ov, oi, bv, bi)) { bv = ov; bi = oi; }
    }
    if (lane == 0) { sh.rv[w] = bv; sh.ri[w] = bi; }
    __syncthreads();
    bv = sh.rv[0]; bi = sh.ri[0];
#pragma unroll 1
    for (int k = 1; k < threads >> 6; ++k)
      if (better(sh.rv[k], sh.ri[k], bv, bi)) { bv = sh.rv[k]; bi = sh.ri[k]; }
    if (t == 0) { sh.wv[round] = bv; sh.wi[round] = bi; }
    last = bv; last_index = bi;
    __syncthreads();
  }
  return n;
}
template <typename T, bool ADVANCE>
__global__ __launch_bounds__(64 * SELECT_WAVES) void search_select_kernel(const T* __restrict__ logits, size_t ld, const float* __restrict__ scores,
                                                                          const float2* __restrict__ stat, int K, int V, int groups, int n,
                                                                          float* __restrict__ out_scores, int32_t* __restrict__ out_rows,
                                                                          int32_t* __restrict__ out_tokens, SearchAdvance adv) {
  __shared__ SelectShared sh;
  __shared__ unsigned s_top[SEARCH_MAX];
  const int b = blockIdx.x, t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), waves = blockDim.x >> 6, row0 = b * K;
  if (t == 0) sh.count = 0;
  // a row's score less its lse (-inf: it takes no part), and a bound: the n-th best of the lanes' best groups is one that n groups reach
  unsigned bound = 0;
  float x_first = -INFINITY;                                 // the lane's first group of the wavefront's first row
  double base_first = -INFINITY;
  for (int s = w; s < K; s += waves) {
    const float c = scores[row0 + s];
    const float2* p = stat + (size_t)(row0 + s) * groups;
    float2 x0 = p[min(lane, groups - 1)];                    // (asked for with the score; a dead row's: anything)
    if (lane >= groups) x0 = make_float2(-INFINITY, 0.f);
    double base = -INFINITY;
    float mine = x0.x;
    if (c > -INFINITY) {
      for (int g = lane + 64; g < groups; g += 64) mine = fmaxf(mine, p[g].x);
      const float mx = lanes_max(mine), ms = mx > -INFINITY ? mx : 0.f;
      float sum = x0.x > -INFINITY ? x0.y * expf(x0.x - ms) : x0.y;
      for (int g = lane + 64; g < groups; g += 64) { const float2 x = p[g]; sum += x.x > -INFINITY ? x.y * expf(x.x - ms) : x.y; }
      sum = lanes_sum(sum);
      // (no finite logit, an infinite one or one that is no number: no extension of this row)
      if (c < INFINITY && mx > -INFINITY && mx < INFINITY && sum < INFINITY) base = (double)c - (double)mx - (double)logf(sum);
    }
    if (lane == 0) sh.base[s] = base;
    if (s == w) { x_first = x0.x; base_first = base; }
    if (base > -INFINITY) {                                  // (uniform over the wavefront)
      const unsigned key = mine > -INFINITY ? search_sortable((float)(base + (double)mine)) : 0u;
      unsigned least = 0;                                    // (its lower bits do not pay for themselves)
#pragma unroll
      for (int bit = 31; bit >= 12; --bit)
        if (__popcll(__ballot(key >= (least | 1u << bit))) >= n) least |= 1u << bit;
      bound = max(bound, least);
    }
  }
  if (lane == 0) sh.reach[w] = bound < 0x00800000u ? -INFINITY : __uint_as_float((int)bound < 0 ? bound ^ 0x80000000u : ~bound);
  __syncthreads();
  const float reach = lanes_max(sh.reach[min(lane, waves - 1)]);
  auto group_value = [&](double base, float x) { return base > -INFINITY ? base + (double)x : -(double)INFINITY; };
  for (int s = w; s < K; s += waves) {
    const double base = s == w ? base_first : sh.base[s];
    if (!(base > -INFINITY)) continue;
    for (int g = lane, g0 = 0; g0 < groups; g += 64, g0 += 64) {
      const float x = g0 == 0 && s == w ? x_first : g < groups ? stat[(size_t)(row0 + s) * groups + g].x : -INFINITY;
      const double v = group_value(base, x);
      select_append(sh, v > -INFINITY && (float)v >= reach, v, (unsigned)s << GROUP_BITS | (unsigned)g);
    }
  }
  const int tops = select_best(sh, n, [&](auto f) {
#pragma unroll 1
    for (int s = w; s < K; s += waves)
#pragma unroll 1
      for (int g = lane; g < groups; g += 64) f(group_value(sh.base[s], stat[(size_t)(row0 + s) * groups + g].x), (unsigned)s << GROUP_BITS | (unsigned)g);
  });
  const double least = tops == n ? sh.wv[n - 1] : -(double)INFINITY;
  if (t < tops) s_top[t] = sh.wi[t];
  if (t == 0) sh.count = 0;
  __syncthreads();
  // the entries of the best groups that reach the n-th group's best
  const int entries = tops * SEARCH_GROUP, threads = blockDim.x;
  auto entry = [&](int i, unsigned& index) {                 // its logit (-inf: there is none)
    const unsigned id = s_top[i / SEARCH_GROUP], s = id >> GROUP_BITS, v = (id & ((1u << GROUP_BITS) - 1)) * SEARCH_GROUP + i % SEARCH_GROUP;
    index = s << TOKEN_BITS | v;
    return v < (unsigned)V ? to_f(logits[(size_t)(row0 + s) * ld + v]) : -INFINITY;
  };
  for (int i0 = 0; i0 < entries; i0 += SELECT_BATCH * threads) {
    float z[SELECT_BATCH];
    unsigned index[SELECT_BATCH];
#pragma unroll
    for (int u = 0; u < SELECT_BATCH; ++u) {                 // (all on their way before the first is looked at)
      z[u] = -INFINITY; index[u] = 0;
      const int i = i0 + u * threads + t;
      if (i0 + u * threads < entries && i < entries) z[u] = entry(i, index[u]);
    }
#pragma unroll
    for (int u = 0; u < SELECT_BATCH; ++u) {
      if (i0 + u * threads >= entries) break;
      const double v = sh.base[index[u] >> TOKEN_BITS] + (double)z[u];
      select_append(sh, z[u] > -INFINITY && v >= least, v, index[u]);   // (a logit of NaN makes its row's lse one: not here)
    }
  }
  const int found = select_best(sh, n, [&](auto f) {
#pragma unroll 1
    for (int i = t; i < entries; i += threads) {
      unsigned index;
      const float z = entry(i, index);
      f(z > -INFINITY ? sh.base[index >> TOKEN_BITS] + (double)z : -(double)INFINITY, index);
    }
  });
  if (!ADVANCE) {
    if (t < n) {
      const bool in = t < found;
      const unsigned ix = in ? sh.wi[t] : 0, s = ix >> TOKEN_BITS;
      out_scores[(size_t)b * n + t] = in ? (float)sh.wv[t] : -INFINITY;
      out_rows[(size_t)b * n + t] = in ? row0 + (int)s : -1;
      out_tokens[(size_t)b * n + t] = in ? (int)(ix & ((1u << TOKEN_BITS) - 1)) : -1;
    }
    return;
  }
  // ---- a search kept on the device: n = K, the winners split into finished and live hypotheses ------------------
  if (t >= 64) return;
  const bool won = t < found;
  const double v = won ? sh.wv[t] : -INFINITY;
  const unsigned ix = won ? sh.wi[t] : 0;
  const int s = ix >> TOKEN_BITS, tk = ix & ((1u << TOKEN_BITS) - 1);
  const bool fin = won && (tk == adv.eos || adv.j == adv.max_len - 1), live = won && !fin;
  const unsigned long long m_fin = __ballot(fin), m_live = __ballot(live);
  const int n_new = __popcll(m_live);
  if (live) {
    const int r = row0 + __popcll(m_live & ((1ull << t) - 1));
    out_scores[r] = (float)v;
    out_rows[r] = row0 + s;
    out_tokens[r] = tk;
    adv.hist_tok[(size_t)adv.j * adv.hist_ld + r] = tk;
    adv.hist_par[(size_t)adv.j * adv.hist_ld + r] = s;
  }
  if (t >= n_new && t < K) { out_scores[row0 + t] = -INFINITY; out_rows[row0 + t] = -1; out_tokens[row0 + t] = -1; }
  if (m_fin) {
    const float norm = (float)v / powf((5.f + (float)(adv.j + 1)) / 6.f, adv.alpha);
    float best = adv.fin_score[b];
    int at = -1;
    for (unsigned long long m = m_fin; m; m &= m - 1) {
      const int q = __ffsll(m) - 1;
      const float x = __shfl(norm, q, 64);
      if (x > best) { best = x; at = q; }                    // strict: the hypothesis finished first keeps a tie
    }
    if (t == at) { adv.fin_score[b] = best; adv.fin_step[b] = adv.j; adv.fin_par[b] = s; adv.fin_tok[b] = tk; }
  }
}
static int search_groups(int V) { return (V + SEARCH_GROUP - 1) / SEARCH_GROUP; }
size_t search_workspace(int B, int K, int V) { return (size_t)B * K * search_groups(V) * sizeof(float2); }
void launch_search_select(int prec, const void* logits, size_t ld, const float* scores, int B, int K, int V, int n, float* out_scores,
                          int32_t* out_rows, int32_t* out_tokens, const SearchAdvance* adv, void* workspace, hipStream_t st) {
  const int groups = search_groups(V);
  float2* stat = (float2*)workspace;
  const dim3 grid((unsigned)(((long)B * K * groups + 3) / 4)), threads(64 * std::min(SELECT_WAVES, std::max(4, K)));
  auto go = [&](auto type) {
    using T = decltype(type);
    hipLaunchKernelGGL(search_groups_kernel<T>, grid, dim3(256), 0, st, (const T*)logits, ld, scores, B * K, V, groups, stat);
    if (adv)
      hipLaunchKernelGGL((search_select_kernel<T, true>), dim3(B), threads, 0, st, (const T*)logits, ld, scores, stat, K, V, groups, n, out_scores,
                         out_rows, out_tokens, *adv);
    else
      hipLaunchKernelGGL((search_select_kernel<T, false>), dim3(B), threads, 0, st, (const T*)logits, ld, scores, stat, K, V, groups, n, out_scores,
                         out_rows, out_tokens, SearchAdvance{});
  };
  if (prec) go(bf16_t{}); else go(float{});
}

// ---- rows that follow ----------------------------------------------------------------------------------------
// dst[r] = src[rows[r]] of several tensors, a workgroup per row and tensor; rows whose number is outside the source stay as they were.  Bound by its
// traffic: 640 rows of nine tensors, 34 MB moved, 9.8 us; 10 rows 2.6 us, the launch.
template <typename V>
__device__ __forceinline__ void reorder_row(const char* s, char* d, int bytes) {
  for (int i = threadIdx.x; i < bytes / (int)sizeof(V); i += 128) reinterpret_cast<V*>(d)[i] = reinterpret_cast<const V*>(s)[i];
}
__global__ __launch_bounds__(128) void search_reorder_kernel(ReorderJobs jobs) {
  const ReorderJob& j = jobs.job[blockIdx.y];
  const int r = blockIdx.x, from = j.rows[r];
  if ((unsigned)from >= (unsigned)j.src_rows) return;
  const char* s = j.src + (size_t)from * j.src_pitch;
  char* d = j.dst + (size_t)r * j.dst_pitch;
  if (j.step == 16) reorder_row<uint4>(s, d, j.bytes);
  else if (j.step == 4) reorder_row<uint32_t>(s, d, j.bytes);
  else if (j.step == 2) reorder_row<uint16_t>(s, d, j.bytes);
  else reorder_row<uint8_t>(s, d, j.bytes);
}
void launch_search_reorder(const ReorderJobs& jobs, int n, int count, hipStream_t st) {
  hipLaunchKernelGGL(search_reorder_kernel, dim3(count, n), dim3(128), 0, st, jobs);
}

}  // namespace cmt
