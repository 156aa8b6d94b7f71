// gfx950 kernels of sampling: from a query's scores (k_fuse_scores) to its token.
//
// The tokens of finite or infinite score, in falling order (equal scores: the lower token first), have weights
// w = exp((s - s_max) / T). Every filter keeps a prefix of that order, so that three numbers say what is
// kept, and the token is where the running sum of the kept weights passes u times their total. No sort: the
// order is first known by bins (k_sample_bins), which place each cut and the token within one bin or a few;
// only those bins' tokens are listed and put in order (k_sample_list).
// Weights are whole numbers, rint(w 2^shift) with shift + log2 V <= 62: their sums are exact, so they are the
// same whatever the order of the atomics, and every comparison is made with the same numbers. A weight below
// 2^-shift-1 (2^-45 at 150000 tokens) counts as 0. w comes from fp64: an error of 2^-24 in each of 10^5 weights
// would move cuts of flat distributions, whose steps are 10^-6 of the sum.
#include "pced_device.h"

#include <algorithm>

namespace pced {
namespace {

constexpr int kSampleList = 1024;  // tokens that one block puts in order by comparing all pairs

constexpr float kMaxT = 3.402823466e38f;  // an infinite temperature counts as this (inf times min_p's ln 1 is no number)

typedef unsigned long long u64;

// A query's softmax: how scores become bins and weights (SampleBins holds it for the later launches)
struct Softmax {
  float top, inv;
  double rate;
};
// (grows with the distance from the highest score: a product of it with one number)
__device__ __forceinline__ int bin_of(const Softmax& s, float x) {
  const float d = x == s.top ? 0.f : s.top - x;
  return (int)fminf(d * s.inv, (float)(kSampleBins - 1));
}
__device__ __forceinline__ u64 weight_of(const Softmax& s, float x, int shift) {
  if (x == s.top) return (u64)1 << shift;
  const double e = shift - ((double)s.top - (double)x) * s.rate;
  return e >= -1.0 ? (u64)rint(exp2(e)) : 0ull;  // (inf - x: 0)
}
// A score and its token as a number: fp32 order as unsigned order, and of equal scores the lower token higher
__device__ __forceinline__ u64 order_of(float x, int v) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 counts as 0)
  return (u64)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~v;
}
__device__ __forceinline__ float score_in(u64 key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int token_in(u64 key) { return (int)~(uint32_t)key; }

// The tokens of a block's part of a query's row, N per thread at a time, the first of them
// loaded before anything else: the settings, the slices' ranges and the bins come from other dies'
// launches, 1 us away, and so do the scores.
constexpr int kBinThreads = 512, kListThreads = 1024;
template <int NT, int N>
struct Part {
  static constexpr int kStep = NT * N;
  const float* x;
  int v0, v1;
  float y[N];
  __device__ __forceinline__ Part(const SampleArgs& a, int b) {
    x = a.scores + (size_t)b * a.V;
    const int per = ((a.V + (int)gridDim.y - 1) / (int)gridDim.y + 3) & ~3;
    v0 = blockIdx.y * per;
    v1 = min(a.V, v0 + per);
    load(v0);
  }
  __device__ __forceinline__ int token(int v, int i) const { return v + i * NT + (int)threadIdx.x; }
  __device__ __forceinline__ void load(int v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int t = token(v, i);
      y[i] = t < v1 ? x[t] : kNegInf;
    }
  }
};

// A block's part of a query's tokens into the bins: counted in LDS, then added to the query's. Bound: the way of
// the settings and scores, the atomics' turns in LDS, the flush (one query of 32000 tokens 5.0 us, of 128256 6.5; 16 of
// 151936 14.4: see launch_sample).
__global__ __launch_bounds__(kBinThreads) void k_sample_bins(SampleArgs a) {
  constexpr int NW = kBinThreads / 64, N = 10;
  __shared__ u64 mass[kSampleBins];
  __shared__ uint32_t count[kSampleBins];
  __shared__ float red[2][NW];
  __shared__ u64 fm;
  __shared__ uint32_t fc;
  const int b = blockIdx.x, tid = threadIdx.x;
  Part<kBinThreads, N> part(a, b);
  const float given = a.temperature[b], mp = a.min_p ? a.min_p[b] : 0.f;
  const float T = given > kMaxT ? kMaxT : given;  // (NaN stays)
  float hi = kNegInf, lo = -kNegInf;
  for (int i = tid; i < a.nblk; i += kBinThreads) {
    const float2 x = *(const float2*)(a.part + 2 * ((size_t)b * a.nblk + i));
    hi = fmaxf(hi, x.x);
    lo = fminf(lo, x.y);
  }
  for (int i = tid; i < kSampleBins; i += kBinThreads) { mass[i] = 0; count[i] = 0; }
  if (tid == 0) { fm = 0; fc = 0; }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) { hi = fmaxf(hi, __shfl_xor(hi, o)); lo = fminf(lo, __shfl_xor(lo, o)); }
  if ((tid & 63) == 0) { red[0][tid >> 6] = hi; red[1][tid >> 6] = lo; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) { hi = fmaxf(hi, red[0][w]); lo = fminf(lo, red[1][w]); }
  const bool greedy = !(T > 0.f), has_floor = mp > 0.f && !greedy;
  Softmax s;
  s.top = hi;
  s.rate = greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)T;
  // beyond shift + 1 octaves the weights are 0: no need to tell those tokens apart
  const float span = (float)fmin((double)hi - (double)lo, fmin((a.shift + 1) / s.rate, 3.0e38));
  s.inv = span > 0.f ? (float)kSampleBins / span : 0.f;  // (NaN where the highest is infinite: 0)
  const double floor = has_floor ? (double)hi + (double)T * log((double)mp) : 0.0;
  SampleBins* q = a.bins + b;
  if (blockIdx.y == 0 && tid == 0) {
    q->rate = s.rate;
    q->top = s.top;
    q->inv = s.inv;
  }
  u64 my_mass = 0;
  uint32_t my_count = 0;
  for (int v = part.v0;;) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = part.y[i];
      if (!(y > kNegInf)) continue;
      const u64 w = weight_of(s, y, a.shift);
      const int bin = bin_of(s, y);
      atomicAdd(&count[bin], 1u);
      if (w) atomicAdd(&mass[bin], w);
      if (has_floor && (double)y >= floor) { my_mass += w; ++my_count; }
    }
    v += part.kStep;
    if (v >= part.v1) break;
    part.load(v);
  }
  if (has_floor) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      my_mass += __shfl_xor(my_mass, o);
      my_count += (uint32_t)__shfl_xor((int)my_count, o);
    }
    if ((tid & 63) == 0 && my_count) { atomicAdd(&fm, my_mass); atomicAdd(&fc, my_count); }
  }
  __syncthreads();
  for (int i = tid; i < kSampleBins; i += kBinThreads) {
    if (!count[i]) continue;
    atomicAdd(&q->count[i], count[i]);
    if (mass[i]) atomicAdd(&q->mass[i], mass[i]);
  }
  if (tid == 0 && fc) { atomicAdd(&q->floor_mass, fm); atomicAdd(&q->floor_count, fc); }
}

// A query's bins summed from the highest on, in LDS, and where its cuts and its token can be.
struct Sums {
  u64 mass[kSampleBins + 1];       // before each bin, and of all
  uint32_t count[kSampleBins + 1];
};
struct Cuts {
  uint32_t n_k, floor_count;       // tokens that top_k (or the temperature) and min_p keep
  u64 floor_mass;
  u64 mass_k;                      // of the first n_k, where k_open is false
  bool none, k_open, has_p, has_floor;
  float p, u;
  int bk;                          // bin of the last of n_k
  int p0, p1, t0, t1;              // bins that top_p's cut and the token can be in (p0 > p1: no cut)
};
__device__ __forceinline__ bool wanted(const Cuts& c, int bin) {
  return (c.k_open && bin == c.bk) || (bin >= c.p0 && bin <= c.p1) || (bin >= c.t0 && bin <= c.t1);
}
// the first bin whose sum reaches (or passes) t, for t up to the sum of all
template <bool PASS>
__device__ __forceinline__ int bin_at(const Sums& s, double t) {
  int lo = 0, hi = kSampleBins - 1;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    const double x = (double)s.mass[m + 1];
    if (PASS ? x > t : x >= t) hi = m;
    else lo = m + 1;
  }
  return lo;
}
// By all of the block's threads: each has PER neighbouring bins, and the one whose bin a cut falls into says so.
template <int NT>
struct Scan {
  static constexpr int PER = kSampleBins / NT;
  static_assert(PER * NT == kSampleBins, "");
  u64 m[PER];
  uint32_t n[PER];
  Softmax s;
  float T, p, mp, u;
  int k;
  u64 floor_mass;
  uint32_t floor_count;
  // the loads, ahead of everything else
  __device__ __forceinline__ Scan(const SampleArgs& a, int b) {
    const SampleBins* q = a.bins + b;
#pragma unroll
    for (int i = 0; i < PER; ++i) { m[i] = q->mass[PER * threadIdx.x + i]; n[i] = q->count[PER * threadIdx.x + i]; }
    s = Softmax{q->top, q->inv, q->rate};
    floor_mass = q->floor_mass;
    floor_count = q->floor_count;
    T = a.temperature[b];
    k = a.top_k ? a.top_k[b] : 0;
    p = a.top_p ? a.top_p[b] : 1.f;
    mp = a.min_p ? a.min_p[b] : 0.f;
    u = a.uniform[b];
  }
  __device__ __forceinline__ Cuts cuts(const SampleArgs& a, Sums& sums) {
    __shared__ u64 wm[NT / 64];
    __shared__ uint32_t wc[NT / 64];
    __shared__ int s_bk, s_p0, s_p1, s_t0, s_t1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 ms = 0;
    uint32_t ns = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { ms += m[i]; ns += n[i]; }
    u64 rm = ms;
    uint32_t rn = ns;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const u64 x = __shfl_up(rm, o);
      const uint32_t y = (uint32_t)__shfl_up((int)rn, o);
      if (lane >= o) { rm += x; rn += y; }
    }
    if (lane == 63) { wm[wave] = rm; wc[wave] = rn; }
    __syncthreads();
    u64 M = 0;
    uint32_t N = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) { rm += wm[w]; rn += wc[w]; }
      M += wm[w];
      N += wc[w];
    }
    u64 at_m[PER + 1];
    uint32_t at_n[PER + 1];
    at_m[0] = rm - ms;
    at_n[0] = rn - ns;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      at_m[i + 1] = at_m[i] + m[i];
      at_n[i + 1] = at_n[i] + n[i];
      sums.mass[PER * tid + i] = at_m[i];
      sums.count[PER * tid + i] = at_n[i];
    }
    if (tid == 0) { sums.mass[kSampleBins] = M; sums.count[kSampleBins] = N; }
    const bool greedy = !(T > 0.f);
    Cuts c;
    c.none = N == 0;
    c.n_k = greedy ? 1u : k > 0 ? min((uint32_t)k, N) : N;
    c.has_p = p < 1.f && !greedy;
    c.p = fmaxf(p, 0.f);
    c.u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
    c.has_floor = mp > 0.f && !greedy;
    c.floor_count = max(floor_count, 1u);              // the highest stays whatever min_p says
    c.floor_mass = max(floor_mass, (u64)1 << a.shift);
    c.bk = c.t0 = c.t1 = 0;
    c.p0 = 1;
    c.p1 = 0;
    c.k_open = false;
    c.mass_k = 0;
    if (c.none) {  // uniform
      __syncthreads();
      return c;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)                      // the bin of rank n_k - 1
      if (at_n[i] < c.n_k && c.n_k <= at_n[i + 1]) s_bk = PER * tid + i;
    __syncthreads();
    c.bk = s_bk;
    const u64 b0 = sums.mass[c.bk], b1 = sums.mass[c.bk + 1];
    const bool whole = sums.count[c.bk + 1] == c.n_k;
    // all of the bin, or a bin without weight: its sum is known
    c.k_open = !whole && b0 != b1;
    c.mass_k = whole ? b1 : b0;
    const u64 k0 = c.k_open ? b0 : c.mass_k, k1 = c.k_open ? b1 : c.mass_k;
    u64 m0 = k0, m1 = k1;                              // what is kept weighs between these
    if (c.has_p) {
      const double t0 = (double)c.p * (double)k0, t1 = (double)c.p * (double)k1;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const double x = (double)at_m[i], y = (double)at_m[i + 1];
        const bool first = i == 0 && tid == 0;
        if (y >= t0 && (x < t0 || first)) s_p0 = PER * tid + i;
        if (y >= t1 && (x < t1 || first)) s_p1 = PER * tid + i;
      }
      __syncthreads();
      c.p0 = s_p0;
      c.p1 = s_p1;
      m0 = min(m0, sums.mass[c.p0]);
      m1 = min(m1, sums.mass[c.p1 + 1]);
    }
    if (c.has_floor) { m0 = min(m0, c.floor_mass); m1 = min(m1, c.floor_mass); }
    const double t0 = (double)c.u * (double)m0, t1 = (double)c.u * (double)m1;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const double x = (double)at_m[i], y = (double)at_m[i + 1];
      if (x <= t0 && t0 < y) s_t0 = PER * tid + i;
      if (x <= t1 && t1 < y) s_t1 = PER * tid + i;
    }
    __syncthreads();
    c.t0 = s_t0;
    c.t1 = s_t1;
    return c;
  }
};

struct Found {
  u64 key;        // of the token at the cut
  u64 mass;       // of the tokens before it, in all
  uint32_t rank;  // how many they are
};
// Long lists: the token of bin `bin` at which the count reaches r (1 on; MODE 0), or the sum reaches (1) or
// passes (2) t, by its key's digits from the highest on, those that all of the bin's keys share left out.
template <int MODE>
__device__ __forceinline__ Found search(const SampleArgs& a, const u64* list, const Softmax& s, const Sums& sums, int n,
                                        int bin, uint32_t r, double t) {
  __shared__ u64 hm[256], s_key[2];
  __shared__ uint32_t hc[256];
  __shared__ int s_digit;
  const int tid = threadIdx.x;
  if (tid == 0) { s_key[0] = ~(u64)0; s_key[1] = 0; }
  __syncthreads();
  u64 all = ~(u64)0, any = 0;
  for (int i = tid; i < n; i += kListThreads) {
    const u64 k = list[i];
    if (bin_of(s, score_in(k)) != bin) continue;
    all &= k;
    any |= k;
  }
  atomicAnd(&s_key[0], all);
  atomicOr(&s_key[1], any);
  __syncthreads();
  const u64 differ = s_key[0] ^ s_key[1];
  Found f{s_key[0], sums.mass[bin], sums.count[bin]};
  for (int sh = 56; sh >= 0; sh -= 8) {
    if (!(differ >> sh & 255)) continue;  // (the digit is in f.key already)
    for (int i = tid; i < 256; i += kListThreads) { hm[i] = 0; hc[i] = 0; }
    __syncthreads();
    for (int i = tid; i < n; i += kListThreads) {
      const u64 k = list[i];
      const float y = score_in(k);
      if (bin_of(s, y) != bin) continue;
      if (sh < 56 && (k >> (sh + 8)) != (f.key >> (sh + 8))) continue;
      atomicAdd(&hc[k >> sh & 255], 1u);
      atomicAdd(&hm[k >> sh & 255], weight_of(s, y, a.shift));
    }
    __syncthreads();
    if (tid == 0) {
      u64 m = f.mass;
      uint32_t c = f.rank;
      int d = 255, last = 255;
      for (; d >= 0; --d) {
        if (!hc[d]) continue;
        last = d;
        if (MODE == 0 ? c + hc[d] >= r : MODE == 1 ? (double)(m + hm[d]) >= t : (double)(m + hm[d]) > t) break;
        m += hm[d];
        c += hc[d];
      }
      if (d < 0) {  // (not reached: the sums of a bin are those of its tokens)
        m -= hm[last];
        c -= hc[last];
      }
      s_digit = last;
      s_key[0] = m;
      s_key[1] = c;
    }
    __syncthreads();
    f.mass = s_key[0];
    f.rank = (uint32_t)s_key[1];
    f.key = (f.key & ~((u64)255 << sh)) | (u64)s_digit << sh;
    __syncthreads();
  }
  __syncthreads();
  return f;
}

// The exact cuts, and the token, by one block, from the bins' sums, the cuts and the whole list.
__device__ __forceinline__ void sample_token(const SampleArgs& a, int b, const Softmax& s, const Cuts& c, const Sums& sums) {
  __shared__ u64 key[kSampleList], weight[kSampleList];
  __shared__ uint16_t bins[kSampleList];
  __shared__ u64 s_mass_k, s_p_mass;
  __shared__ uint32_t s_p_count;
  const int tid = threadIdx.x;
  const u64* list = a.list + (size_t)b * a.V;
  const int n = (int)__hip_atomic_load(&a.bins[b].listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const u64 entry = tid < a.V ? __hip_atomic_load(&list[tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;  // (as far as it is one)
  if (a.beta_used) {
    const int e1 = a.query_exp0[b + 1];
    for (int e = a.query_exp0[b] + tid; e < e1; e += kListThreads) a.beta_used[e] = a.beta[e];
  }
  const bool few = n <= kSampleList;
  const float y = score_in(entry);
  int bin = -1;
  u64 w = 0;
  if (few && tid < n) {
    bin = bin_of(s, y);
    w = weight_of(s, y, a.shift);
    key[tid] = entry;
    weight[tid] = w;
    bins[tid] = (uint16_t)bin;
  }
  __syncthreads();
  auto write = [&](int v, float x, uint32_t kept, u64 mass) {  // one thread
    a.tokens_out[b] = v;
    a.prev_tok[b] = v;
    if (a.winner) a.winner[b] = v >= 0 ? a.who[(size_t)b * a.V + v] : 0;
    if (a.score) a.score[b] = x;
    if (a.kept) a.kept[b] = (int32_t)kept;
    if (a.logprob) {
      // ln of the weight over the sum: the weight's exponent as it is, not as rounded to 2^-shift
      const double z = x == s.top ? 0.0 : ((double)x - (double)s.top) * s.rate;
      a.logprob[b] = v >= 0 ? (float)((z - (log2((double)mass) - a.shift)) * 0.6931471805599453) : kNegInf;
    }
  };
  if (c.none) {  // uniform
    if (tid == 0) write(-1, kNegInf, 0, 0);
    return;
  }
  // what all three filters keep, once top_k's sum and top_p's cut are known
  auto keep = [&](u64 mass_k, uint32_t p_count, u64 p_mass, uint32_t* count, u64* mass) {
    *count = c.n_k;
    *mass = mass_k;
    if (c.has_p && p_count < *count) { *count = p_count; *mass = p_mass; }
    if (c.has_floor && c.floor_count < *count) { *count = c.floor_count; *mass = c.floor_mass; }
  };
  uint32_t count;
  u64 mass;
  if (!few) {
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");  // the list by plain loads from here on
    u64 mass_k = c.mass_k;
    if (c.k_open) {
      const Found f = search<0>(a, list, s, sums, n, c.bk, c.n_k, 0.0);
      mass_k = f.mass + weight_of(s, score_in(f.key), a.shift);
    }
    uint32_t p_count = 0;
    u64 p_mass = 0;
    if (c.has_p) {
      const double t = (double)c.p * (double)mass_k;
      const Found f = search<1>(a, list, s, sums, n, bin_at<false>(sums, t), 0, t);
      p_count = f.rank + 1;
      p_mass = f.mass + weight_of(s, score_in(f.key), a.shift);
    }
    keep(mass_k, p_count, p_mass, &count, &mass);
    const double t = (double)c.u * (double)mass;
    const Found f = search<2>(a, list, s, sums, n, bin_at<true>(sums, t), 0, t);
    if (tid == 0) write(token_in(f.key), score_in(f.key), count, mass);
    return;
  }
  // The tokens before each: those of the bins before, and those of its bin with a higher key. 2^lg
  // neighbouring threads take a token together.
  int lg = 0;
  while (lg < 6 && (n << (lg + 1)) <= kListThreads) ++lg;
  const int i = tid >> lg, step = 1 << lg;
  u64 before = 0, mine = 0;
  uint32_t rank = 0;
  if (i < n) {
    mine = key[i];
    bin = bins[i];
    for (int j = tid & (step - 1); j < n; j += step)
      if (bins[j] == bin && key[j] > mine) { before += weight[j]; ++rank; }
  }
  for (int o = 1; o < step; o <<= 1) {
    before += __shfl_xor(before, o);
    rank += (uint32_t)__shfl_xor((int)rank, o);
  }
  const bool one = i < n && (tid & (step - 1)) == 0;
  if (one) {
    w = weight[i];
    before += sums.mass[bin];
    rank += sums.count[bin];
    if (c.k_open && rank + 1 == c.n_k) s_mass_k = before + w;
  }
  __syncthreads();
  const u64 mass_k = c.k_open ? s_mass_k : c.mass_k;
  if (c.has_p) {  // uniform
    const double t = (double)c.p * (double)mass_k;
    if (one && (double)(before + w) >= t && ((double)before < t || rank == 0)) { s_p_count = rank + 1; s_p_mass = before + w; }
    __syncthreads();
  }
  keep(mass_k, s_p_count, s_p_mass, &count, &mass);
  const double t = (double)c.u * (double)mass;
  if (one && (double)before <= t && t < (double)(before + w)) write(token_in(mine), score_in(mine), count, mass);
}

// The tokens of the bins that hold a cut or the token into the query's list, in any order; the block that
// is the last to do so finds the token. Bound: one wait after the other (bins and scores, a place in the list, the blocks'
// turns, the list; one query of 32000 tokens 10.2 us, 16 of 151936 14.5).
__global__ __launch_bounds__(kListThreads) void k_sample_list(SampleArgs a) {
  __shared__ Sums sums;
  __shared__ uint32_t s_n, s_base, s_done;
  constexpr int N = 5;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  Part<kListThreads, N> part(a, b);
  Scan<kListThreads> scan(a, b);
  const Softmax s = scan.s;
  const Cuts c = scan.cuts(a, sums);
  for (int v = part.v0; v < part.v1 && !c.none; v += part.kStep) {
    if (v > part.v0) part.load(v);
    if (tid == 0) s_n = 0;
    __syncthreads();
    // a place in the list per wave and block: one global atomic, 1 us and more away
    u64 m[N];
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = part.y[i];
      m[i] = __ballot(y > kNegInf && wanted(c, bin_of(s, y)));
      mine += (uint32_t)__popcll(m[i]);
    }
    uint32_t at = 0;
    if (lane == 0 && mine) at = atomicAdd(&s_n, mine);
    __syncthreads();
    if (tid == 0 && s_n) s_base = atomicAdd(&a.bins[b].listed, s_n);
    __syncthreads();
    if (mine) {
      at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + s_base;
      u64* list = a.list + (size_t)b * a.V;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (m[i] >> lane & 1) 
          __hip_atomic_store(&list[at + __popcll(m[i] & (((u64)1 << lane) - 1))], order_of(part.y[i], part.token(v, i)), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
        at += (uint32_t)__popcll(m[i]);
      }
    }
  }
  // The entries are stored and loaded at agent scope, past the dies' own L2s: each wave waits until its own have arrived,
  // the barrier puts that before the count, and no cache is written back or emptied (by one thread's release and acquire
  // 1.2 us more for one query, 2.7 for 16 of 151936; by every thread's 20). As a launch of its own the rest took another 2 us.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s_done = __hip_atomic_fetch_add(&a.bins[b].done[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_done != gridDim.y - 1) return;
  sample_token(a, b, s, c, sums);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int n_queries, int num_cus, hipStream_t st, const Timing* tm) {
  // a work-group per compute unit, none below 1024 tokens, and at most 32 per query, since each adds its bins to
  // the query's (k_sample_bins, 512 threads, 16 queries of 151936 tokens, us at 8 / 16 / 32 / 64 / 128 per query: 17.5 /
  // 14.2 / 15.6 / 21.6 / 34.2; one of 128256: 13.9 / 8.8 / 6.2 / 6.1 / 6.9)
  const long parts = std::min({(long)num_cus / n_queries, (a.V + 1023L) / 1024, 32L});
  const dim3 grid(n_queries, (unsigned)std::max(1L, parts));
  hipError_t e = go(k_sample_bins, grid, dim3(kBinThreads), 0, st, t0(tm), nullptr, a);
  if (e != hipSuccess) return e;
  return go(k_sample_list, grid, dim3(kListThreads), 0, st, nullptr, t1(tm), a);
}

}  // namespace pced
