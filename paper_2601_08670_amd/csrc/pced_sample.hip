// gfx950 kernels of sampling: from a query's scores (k_fuse_scores) to its token.
//
// The tokens of finite or infinite score, in falling order (equal scores: the lower token first), have weights
// w = exp((s - s_max) / T). Every filter keeps a prefix of that order, so that three numbers say what is
// kept, and the token is where the running sum of the kept weights passes u times their total. No sort: the
// order is first known by bins (k_sample_bins), which place each cut and the token within one bin or a few;
// only those bins' tokens are listed (k_sample_list) and put in order (k_sample_token).
// Weights are whole numbers, rint(w 2^shift) with shift + log2 V <= 62: their sums are exact, so they are the
// same whatever the order of the atomics, and every comparison is made with the same numbers. A weight below
// 2^-shift-1 (2^-45 at 150000 tokens) counts as 0. w comes from fp64: an error of 2^-24 in each of 10^5 weights
// would move cuts of flat distributions, whose steps are 10^-6 of the sum.
#include "pced_device.h"

#include <algorithm>

namespace pced {
namespace {

constexpr int kSampleList = 1024;  // tokens that one block puts in order by comparing all pairs

typedef unsigned long long u64;

// What a query's settings and the range of its scores say
struct Softmax {
  float top;       // the highest score; -inf: no candidate
  float inv;       // bins per unit of score
  double rate;     // log2(e) / T
  double floor;    // the lowest score that min_p keeps
  bool greedy, has_floor;
};
// by all of the block's threads; ends with a barrier
template <int NT>
__device__ __forceinline__ Softmax softmax_of(const SampleArgs& a, int b) {
  __shared__ float red[2][NT / 64];
  float hi = kNegInf, lo = -kNegInf;
  for (int i = threadIdx.x; i < a.nblk; i += NT) {
    const float2 x = *(const float2*)(a.part + 2 * ((size_t)b * a.nblk + i));
    hi = fmaxf(hi, x.x);
    lo = fminf(lo, x.y);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) { hi = fmaxf(hi, __shfl_xor(hi, o)); lo = fminf(lo, __shfl_xor(lo, o)); }
  if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = hi; red[1][threadIdx.x >> 6] = lo; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { hi = fmaxf(hi, red[0][w]); lo = fminf(lo, red[1][w]); }
  Softmax s;
  s.top = hi;
  const float T = a.temperature[b];
  s.greedy = !(T > 0.f);
  s.rate = s.greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)T;
  // beyond shift + 1 octaves the weights are 0: no need to tell those tokens apart
  const double reach = (a.shift + 1) / s.rate;
  const float span = (float)fmin((double)hi - (double)lo, fmin(reach, 3.0e38));
  s.inv = span > 0.f ? (float)kSampleBins / span : 0.f;  // (NaN where the highest is infinite: 0)
  const float mp = a.min_p ? a.min_p[b] : 0.f;
  s.has_floor = mp > 0.f && !s.greedy;
  s.floor = s.has_floor ? (double)hi + (double)T * log((double)mp) : 0.0;
  return s;
}
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

// A block's part of a query's tokens into the bins: counted in LDS, then added to the query's.
constexpr int kBinThreads = 512;
__global__ __launch_bounds__(kBinThreads) void k_sample_bins(SampleArgs a) {
  __shared__ u64 mass[kSampleBins];
  __shared__ uint32_t count[kSampleBins];
  __shared__ u64 fm;
  __shared__ uint32_t fc;
  const int b = blockIdx.y, tid = threadIdx.x;
  const int per = ((a.V + (int)gridDim.x - 1) / (int)gridDim.x + 3) & ~3;
  const int v0 = blockIdx.x * per, v1 = min(a.V, v0 + per);
  for (int i = tid; i < kSampleBins; i += kBinThreads) { mass[i] = 0; count[i] = 0; }
  if (tid == 0) { fm = 0; fc = 0; }
  const Softmax s = softmax_of<kBinThreads>(a, b);  // (ends with a barrier)
  const float* x = a.scores + (size_t)b * a.V;
  u64 my_mass = 0;
  uint32_t my_count = 0;
  for (int v = v0 + tid; v < v1; v += kBinThreads) {
    const float y = x[v];
    if (!(y > kNegInf)) continue;
    const u64 w = weight_of(s, y, a.shift);
    const int bin = bin_of(s, y);
    atomicAdd(&count[bin], 1u);
    if (w) atomicAdd(&mass[bin], w);
    if (s.has_floor && (double)y >= s.floor) { my_mass += w; ++my_count; }
  }
  if (s.has_floor) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      my_mass += __shfl_xor(my_mass, o);
      my_count += (uint32_t)__shfl_xor((int)my_count, o);
    }
    if ((tid & 63) == 0 && my_count) { atomicAdd(&fm, my_mass); atomicAdd(&fc, my_count); }
  }
  __syncthreads();
  SampleBins* q = a.bins + b;
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
// by all of the block's threads
template <int NT>
__device__ __forceinline__ Cuts cuts_of(const SampleArgs& a, int b, Sums& s) {
  constexpr int PER = kSampleBins / NT;
  static_assert(PER * NT == kSampleBins, "");
  __shared__ u64 wm[NT / 64];
  __shared__ uint32_t wc[NT / 64];
  __shared__ Cuts cuts;
  const SampleBins* q = a.bins + b;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 m[PER], ms = 0;
  uint32_t n[PER], ns = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) { m[i] = q->mass[PER * tid + i]; n[i] = q->count[PER * tid + i]; }
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
#pragma unroll
  for (int w = 0; w < NT / 64; ++w)
    if (w < wave) { rm += wm[w]; rn += wc[w]; }
  rm -= ms;
  rn -= ns;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    s.mass[PER * tid + i] = rm;
    s.count[PER * tid + i] = rn;
    rm += m[i];
    rn += n[i];
  }
  if (tid == NT - 1) { s.mass[kSampleBins] = rm; s.count[kSampleBins] = rn; }
  __syncthreads();
  if (tid == 0) {
    Cuts c;
    const uint32_t N = s.count[kSampleBins];
    const float T = a.temperature[b];
    const bool greedy = !(T > 0.f);
    const int k = a.top_k ? a.top_k[b] : 0;
    const float mp = a.min_p ? a.min_p[b] : 0.f;
    c.none = N == 0;
    c.n_k = greedy ? 1u : k > 0 ? min((uint32_t)k, N) : N;
    c.p = a.top_p ? a.top_p[b] : 1.f;
    c.has_p = c.p < 1.f && !greedy;
    c.p = fmaxf(c.p, 0.f);
    const float u = a.uniform[b];
    c.u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
    c.has_floor = mp > 0.f && !greedy;
    c.floor_count = max(q->floor_count, 1u);          // the highest stays whatever min_p says
    c.floor_mass = max(q->floor_mass, (u64)1 << a.shift);
    int lo = 0, hi = kSampleBins - 1;                  // the bin of rank n_k - 1
    while (lo < hi) {
      const int x = (lo + hi) >> 1;
      if (s.count[x + 1] >= c.n_k) hi = x;
      else lo = x + 1;
    }
    c.bk = lo;
    // all of the bin, or a bin without weight: its sum is known
    c.k_open = s.count[lo + 1] != c.n_k && s.mass[lo] != s.mass[lo + 1];
    c.mass_k = s.count[lo + 1] == c.n_k ? s.mass[lo + 1] : s.mass[lo];
    const u64 k0 = c.k_open ? s.mass[lo] : c.mass_k, k1 = c.k_open ? s.mass[lo + 1] : c.mass_k;
    u64 m0 = k0, m1 = k1;                              // what is kept weighs between these
    c.p0 = 1;
    c.p1 = 0;
    if (c.has_p) {
      c.p0 = bin_at<false>(s, (double)c.p * (double)k0);
      c.p1 = bin_at<false>(s, (double)c.p * (double)k1);
      m0 = min(m0, s.mass[c.p0]);
      m1 = min(m1, s.mass[c.p1 + 1]);
    }
    if (c.has_floor) { m0 = min(m0, c.floor_mass); m1 = min(m1, c.floor_mass); }
    c.t0 = bin_at<true>(s, (double)c.u * (double)m0);
    c.t1 = bin_at<true>(s, (double)c.u * (double)m1);
    cuts = c;
  }
  __syncthreads();
  return cuts;
}

// The tokens of the bins that hold a cut or the token, in any order.
__global__ __launch_bounds__(kBinThreads) void k_sample_list(SampleArgs a) {
  __shared__ Sums sums;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int per = ((a.V + (int)gridDim.x - 1) / (int)gridDim.x + 3) & ~3;
  const int v0 = blockIdx.x * per, v1 = min(a.V, v0 + per);
  if (v0 >= v1) return;
  const Softmax s = softmax_of<kBinThreads>(a, b);
  const Cuts c = cuts_of<kBinThreads>(a, b, sums);
  if (c.none) return;
  const float* x = a.scores + (size_t)b * a.V;
  for (int v = v0 + tid; v - tid < v1; v += kBinThreads) {
    const float y = v < v1 ? x[v] : kNegInf;
    const bool mine = y > kNegInf && wanted(c, bin_of(s, y));
    const u64 m = __ballot(mine);
    if (!m) continue;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(&a.bins[b].listed, (uint32_t)__popcll(m));
    at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    if (mine) a.list[(size_t)b * a.V + at + __popcll(m & (((u64)1 << lane) - 1))] = v;
  }
}

// fp32 order as unsigned order, and of equal scores the lower token higher
__device__ __forceinline__ u64 order_of(float x, int v) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 counts as 0)
  return (u64)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~v;
}

constexpr int kTokenThreads = 1024;
struct Found {
  u64 key;        // of the token at the cut
  u64 mass;       // of the tokens before it, in all
  uint32_t rank;  // how many they are
};
// Long lists: the token of bin `bin` at which the count reaches r (1 on; MODE 0), or the sum reaches (1) or
// passes (2) t, by its key's digits from the highest on, those that all of the bin's keys share left out.
template <int MODE>
__device__ __forceinline__ Found search(const SampleArgs& a, int b, const Softmax& s, const Sums& sums, int n, int bin,
                                        uint32_t r, double t) {
  __shared__ u64 hm[256], s_key[2];
  __shared__ uint32_t hc[256];
  __shared__ int s_digit;
  const int tid = threadIdx.x;
  const float* x = a.scores + (size_t)b * a.V;
  const int32_t* list = a.list + (size_t)b * a.V;
  if (tid == 0) { s_key[0] = ~(u64)0; s_key[1] = 0; }
  __syncthreads();
  u64 all = ~(u64)0, any = 0;
  for (int i = tid; i < n; i += kTokenThreads) {
    const int v = list[i];
    const float y = x[v];
    if (bin_of(s, y) != bin) continue;
    const u64 k = order_of(y, v);
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
    for (int i = tid; i < 256; i += kTokenThreads) { hm[i] = 0; hc[i] = 0; }
    __syncthreads();
    for (int i = tid; i < n; i += kTokenThreads) {
      const int v = list[i];
      const float y = x[v];
      if (bin_of(s, y) != bin) continue;
      const u64 k = order_of(y, v);
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

// One block per query: the exact cuts, and the token.
__global__ __launch_bounds__(kTokenThreads) void k_sample_token(SampleArgs a) {
  __shared__ Sums sums;
  __shared__ u64 key[kSampleList], weight[kSampleList];
  __shared__ uint16_t bins[kSampleList];
  __shared__ u64 s_mass_k, s_p_mass, s_mass;
  __shared__ uint32_t s_p_count, s_count;
  const int b = blockIdx.x, tid = threadIdx.x;
  if (a.beta_used) {
    const int e1 = a.query_exp0[b + 1];
    for (int e = a.query_exp0[b] + tid; e < e1; e += kTokenThreads) a.beta_used[e] = a.beta[e];
  }
  const Softmax s = softmax_of<kTokenThreads>(a, b);
  const Cuts c = cuts_of<kTokenThreads>(a, b, sums);
  const float* x = a.scores + (size_t)b * a.V;
  auto write = [&](int v, uint32_t kept, u64 mass) {  // one thread
    const float y = v >= 0 ? x[v] : kNegInf;
    a.tokens_out[b] = v;
    a.prev_tok[b] = v;
    if (a.winner) a.winner[b] = v >= 0 ? a.who[(size_t)b * a.V + v] : 0;
    if (a.score) a.score[b] = y;
    if (a.kept) a.kept[b] = (int32_t)kept;
    if (a.logprob) {
      // ln of the weight over the sum: the weight's exponent as it is, not as rounded to 2^-shift
      const double z = y == s.top ? 0.0 : ((double)y - (double)s.top) * s.rate;
      a.logprob[b] = v >= 0 ? (float)((z - (log2((double)mass) - a.shift)) * 0.6931471805599453) : kNegInf;
    }
  };
  if (c.none) {
    if (tid == 0) write(-1, 0, 0);
    return;
  }
  const int n = (int)a.bins[b].listed;
  // what all three filters keep, once top_k's sum and top_p's cut are known
  auto keep = [&](u64 mass_k, uint32_t p_count, u64 p_mass, uint32_t* count, u64* mass) {
    *count = c.n_k;
    *mass = mass_k;
    if (c.has_p && p_count < *count) { *count = p_count; *mass = p_mass; }
    if (c.has_floor && c.floor_count < *count) { *count = c.floor_count; *mass = c.floor_mass; }
  };
  if (n > kSampleList) {
    u64 mass_k = c.mass_k;
    if (c.k_open) {
      const Found f = search<0>(a, b, s, sums, n, c.bk, c.n_k, 0.0);
      mass_k = f.mass + weight_of(s, x[(int)~(uint32_t)f.key], a.shift);
    }
    uint32_t p_count = 0, count;
    u64 p_mass = 0, mass;
    if (c.has_p) {
      const double t = (double)c.p * (double)mass_k;
      const Found f = search<1>(a, b, s, sums, n, bin_at<false>(sums, t), 0, t);
      p_count = f.rank + 1;
      p_mass = f.mass + weight_of(s, x[(int)~(uint32_t)f.key], a.shift);
    }
    keep(mass_k, p_count, p_mass, &count, &mass);
    const double t = (double)c.u * (double)mass;
    const Found f = search<2>(a, b, s, sums, n, bin_at<true>(sums, t), 0, t);
    if (tid == 0) write((int)~(uint32_t)f.key, count, mass);
    return;
  }
  int v = -1, bin = -1;
  u64 mine = 0, w = 0;
  if (tid < n) {
    v = a.list[(size_t)b * a.V + tid];
    const float y = x[v];
    bin = bin_of(s, y);
    key[tid] = mine = order_of(y, v);
    weight[tid] = w = weight_of(s, y, a.shift);
    bins[tid] = (uint16_t)bin;
  }
  __syncthreads();
  // the tokens before each: those of the bins before, and those of its bin with a higher key
  u64 before = 0;
  uint32_t rank = 0;
  if (tid < n) {
    before = sums.mass[bin];
    rank = sums.count[bin];
    for (int j = 0; j < n; ++j)
      if (bins[j] == bin && key[j] > mine) { before += weight[j]; ++rank; }
    if (c.k_open && rank + 1 == c.n_k) s_mass_k = before + w;
  }
  __syncthreads();
  const u64 mass_k = c.k_open ? s_mass_k : c.mass_k;
  if (tid < n && c.has_p) {
    const double t = (double)c.p * (double)mass_k;
    if ((double)(before + w) >= t && ((double)before < t || rank == 0)) { s_p_count = rank + 1; s_p_mass = before + w; }
  }
  __syncthreads();
  if (tid == 0) {
    uint32_t count;
    u64 mass;
    keep(mass_k, s_p_count, s_p_mass, &count, &mass);
    s_count = count;
    s_mass = mass;
  }
  __syncthreads();
  const double t = (double)c.u * (double)s_mass;
  if (tid < n && (double)before <= t && t < (double)(before + w)) write(v, s_count, s_mass);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int n_queries, int num_cus, hipStream_t st, const Timing* tm) {
  const long want = std::max(1L, 2L * num_cus / n_queries), most = std::max(1, a.V / 2048);
  const dim3 grid((unsigned)std::min({want, most, 64L}), n_queries);
  hipError_t e = go(k_sample_bins, grid, dim3(kBinThreads), 0, st, t0(tm), nullptr, a);
  if (e != hipSuccess) return e;
  e = go(k_sample_list, grid, dim3(kBinThreads), 0, st, nullptr, nullptr, a);
  if (e != hipSuccess) return e;
  return go(k_sample_token, dim3(n_queries), dim3(kTokenThreads), 0, st, nullptr, t1(tm), a);
}

}  // namespace pced
