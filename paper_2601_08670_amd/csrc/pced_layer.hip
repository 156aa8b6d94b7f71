// gfx950 kernels of the layer-wise calls: append of new rows with rotation, 8-bit
// page summaries, the choice of pages from them, and attention over the chosen
// pages. Tile layouts: see pced_kernels.hip.
#include "pced_device.h"

namespace pced {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row as fp32 values, and back (rounded to nearest even)
template <bool BF16>
struct Unit {
  static constexpr int N = BF16 ? 8 : 4;  // elements
  float x[N];
  __device__ __forceinline__ void set(const u32x4& v) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = BF16 ? bf2f(el16(v, e)) : __uint_as_float(v[e & 3]);
  }
  __device__ __forceinline__ u32x4 get() const {
    u32x4 v;
    if constexpr (BF16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x2 p = {(__bf16)x[2 * e], (__bf16)x[2 * e + 1]};
        v[e] = __builtin_bit_cast(uint32_t, p);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
    }
    return v;
  }
};

// Offset of the 16-byte unit at (token, dim) in a K tile, in elements
template <bool BF16>
__device__ __forceinline__ int kunit(int t, int d, int D) {
  return BF16 ? kswz(t, d) : t * D + d;
}

// ------------------------------------------------------------ page summaries

// Summary of one full page and kv-head by one wave: per key dimension the largest
// and the smallest of the page's 16 values, as int8 codes with one scale 2^e,
//   max codes = ceil(max 2^-e), min codes = floor(min 2^-e),
// e the smallest exponent (within +-kSumExp) that keeps every code within 127. So
// the codes bound the keys from outside, and, e being a power of two, neither
// scaling nor rounding depends on how the page came to be. NaN keys are left out;
// keys beyond 127 * 2^kSumExp saturate.
// Lane = (token group, unit): tokens per group in registers, groups by shuffles.
template <bool BF16>
__device__ __forceinline__ void summarize_page(const void* tile, int D, int row, int8_t* codes, float* scale) {
  constexpr int N = Unit<BF16>::N;
  constexpr int W = BF16 ? 16 : 32;  // lanes per token group; D / N <= W of them hold a unit
  constexpr int TPG = kPage / (64 / W);
  const int lane = threadIdx.x & 63, u = lane % W, d = min(u * N, D - N);
  float hi[N], lo[N];
#pragma unroll
  for (int e = 0; e < N; ++e) { hi[e] = kNegInf; lo[e] = -kNegInf; }
  u32x4 v[TPG];
#pragma unroll
  for (int i = 0; i < TPG; ++i) {
    const int o = kunit<BF16>(lane / W * TPG + i, d, D);
    v[i] = BF16 ? *(const u32x4*)((const uint16_t*)tile + o) : *(const u32x4*)((const float*)tile + o);
  }
#pragma unroll
  for (int i = 0; i < TPG; ++i) {
    Unit<BF16> x;
    x.set(v[i]);
#pragma unroll
    for (int e = 0; e < N; ++e) { hi[e] = fmaxf(hi[e], x.x[e]); lo[e] = fminf(lo[e], x.x[e]); }
  }
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
#pragma unroll
    for (int o = W; o < 64; o <<= 1) { hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o)); lo[e] = fminf(lo[e], __shfl_xor(lo[e], o)); }
    // (a dimension whose keys are all NaN has hi < lo: nothing to bound)
    if (lo[e] > hi[e]) hi[e] = lo[e] = 0.f;
    top = fmaxf(top, fmaxf(fabsf(hi[e]), fabsf(lo[e])));
  }
#pragma unroll
  for (int o = W / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  int ex = -kSumExp;
  if (top > 0.f) {
    ex = ilogbf(fminf(top, 3.0e38f)) - 6;
    if (ceil(ldexp((double)top, -ex)) > 127.0) ++ex;
    ex = min(max(ex, -kSumExp), kSumExp);
  }
  if (lane < W && u * N < D) {
    uint32_t ch[N / 4] = {}, cl[N / 4] = {};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int a = (int)fmin(fmax(ceil(ldexp((double)hi[e], -ex)), -127.0), 127.0);
      const int b = (int)fmin(fmax(floor(ldexp((double)lo[e], -ex)), -127.0), 127.0);
      ch[e >> 2] |= (uint32_t)(a & 0xFF) << (8 * (e & 3));
      cl[e >> 2] |= (uint32_t)(b & 0xFF) << (8 * (e & 3));
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      *(uint32_t*)(codes + u * N + 4 * i) = ch[i];
      *(uint32_t*)(codes + D + u * N + 4 * i) = cl[i];
    }
  }
  for (int i = 2 * D + 4 * lane; i < row; i += 256) *(uint32_t*)(codes + i) = 0u;  // the padding counts for nothing
  if (lane == 0) *scale = ldexpf(1.f, ex);
}

// One wave per (page, layer, kv-head): the complete pages of every sequence from
// token len - behind on.
template <bool BF16>
__global__ __launch_bounds__(256) void k_summarize(SummaryArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long task = (long)blockIdx.x * 4 + wave;
  const int h = (int)(task % a.n_kv_heads);
  long rest = task / a.n_kv_heads;
  const int i = (int)(rest % a.span);
  rest /= a.span;
  const int s = (int)(rest % a.n_seqs), l = (int)(rest / a.n_seqs);
  if (l >= a.n_layers) return;
  const int len = a.len0[s] + a.t;
  const int p = max(len - a.behind, 0) / kPage + i;
  if (p >= len / kPage) return;
  const int phys = a.page_table[(size_t)s * a.maxpps + p];
  const size_t tile = (size_t)kPage * a.head_dim * (BF16 ? 2 : 4);
  const size_t at = ((size_t)l * a.n_kv_heads + h) * a.max_pages + phys;
  summarize_page<BF16>((const char*)a.kpool + (((size_t)l * a.max_pages + phys) * a.n_kv_heads + h) * tile,
                       a.head_dim, a.sum_row, a.codes + at * a.sum_row, a.scale + at);
}

// ------------------------------------------------------ append with rotation

// The units of a row of D dims whose first `rot` dims are rotated, as slots of a
// thread's work: with pairs (j, j + rot/2) a slot is the unit of the first member
// and the unit of the second, else one unit.
template <bool BF16>
struct Slot {
  int d, d2;  // dims of the unit and of its partner (d2 < 0: none)
  static __device__ __forceinline__ int count(int D, int rot, bool halves) {
    return (D - (halves ? rot / 2 : 0)) / Unit<BF16>::N;
  }
  __device__ __forceinline__ Slot(int u, int rot, bool halves) {
    d = u * Unit<BF16>::N;
    d2 = -1;
    if (halves) {
      if (d < rot / 2) d2 = d + rot / 2;
      else d += rot / 2;
    }
  }
};

// A slot's unit(s) of a row, rotated: (a, b) -> (a cos - b sin, a sin + b cos) in fp32
template <bool BF16>
__device__ __forceinline__ void turned(const char* row, const Slot<BF16>& sl, const float2* cs, int rot, bool turn,
                                       u32x4& o1, u32x4& o2) {
  constexpr int N = Unit<BF16>::N, es = BF16 ? 2 : 4;
  o1 = *(const u32x4*)(row + (size_t)sl.d * es);
  if (sl.d2 >= 0) o2 = *(const u32x4*)(row + (size_t)sl.d2 * es);
  if (!turn || sl.d >= rot) return;
  Unit<BF16> x;
  x.set(o1);
  if (sl.d2 >= 0) {
    Unit<BF16> y;
    y.set(o2);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float2 c = cs[sl.d + e];
      const float p = x.x[e], q = y.x[e];
      x.x[e] = p * c.x - q * c.y;
      y.x[e] = p * c.y + q * c.x;
    }
    o2 = y.get();
  } else {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      if (sl.d + e >= rot) break;
      const float2 c = cs[(sl.d + e) / 2];
      const float p = x.x[e], q = x.x[e + 1];
      x.x[e] = p * c.x - q * c.y;
      x.x[e + 1] = p * c.y + q * c.x;
    }
  }
  o1 = x.get();
}

// One block per (sequence, page that the sequence's new tokens touch, layer). The
// page's K units are written by token pairs and its V runs by token quads, so that
// only whole 32-byte sectors are stored (see k_append): tokens of the sector that
// are not new keep what they hold. The angles' cos and sin, in fp64 and rounded
// once, are made by the block for its at most 16 positions and shared by its
// heads. A page that becomes full is summarised by the block that filled it.
template <bool BF16>
__global__ __launch_bounds__(256) void k_append_rows(AppendRowsArgs a) {
  constexpr int N = Unit<BF16>::N, es = BF16 ? 2 : 4;
  __shared__ float2 cs[kPage][64];
  const int tid = threadIdx.x;
  const int l = blockIdx.x / (a.n_seqs * a.slots), rest = blockIdx.x - l * a.n_seqs * a.slots;
  const int s = rest / a.slots;
  const int len = a.len0[s] + a.t, p = len / kPage + rest % a.slots;
  const int t0 = max(len - kPage * p, 0), t1 = min(len + a.n_tokens - kPage * p, kPage);  // new tokens of the page
  if (t0 >= t1) return;
  const int phys = a.page_table[(size_t)s * a.maxpps + p];
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, D = a.head_dim, rot = a.rot_dim;
  const bool halves = a.halves != 0;
  const size_t row0 = (size_t)s * a.n_tokens + (kPage * p - len);  // row of the page's token 0 (as a difference)
  const int half = rot / 2, n = t1 - t0;
  for (int e = tid; e < n * half; e += 256) {
    const int t = t0 + e / half, i = e % half;
    double sn, co;
    sincos((double)(kPage * p + t) * exp2(-(2.0 * i / rot) * a.log2_theta), &sn, &co);
    cs[t][i] = make_float2((float)co, (float)sn);
  }
  __syncthreads();
  const size_t tile = (size_t)kPage * D;
  const size_t tile0 = ((size_t)(a.layer0 + l) * a.max_pages + phys) * Hkv;
  const int nslot = Slot<BF16>::count(D, rot, halves);
  auto row_of = [&](const void* base, int64_t stride, int t, int heads, int h) {
    return (const char*)base + ((size_t)(row0 + t) * stride + ((size_t)l * heads + h) * D) * es;
  };

  // q rows
  if (a.q) {
    for (int e = tid; e < n * Hq * nslot; e += 256) {
      const int t = t0 + e / (Hq * nslot), h = e / nslot % Hq;
      const Slot<BF16> sl(e % nslot, rot, halves);
      u32x4 o1, o2;
      turned<BF16>(row_of(a.q, a.q_row, t, Hq, h), sl, cs[t], rot, true, o1, o2);
      char* out = (char*)a.q_out + (((row0 + t) * a.n_layers + l) * Hq + h) * D * es;
      *(u32x4*)(out + sl.d * es) = o1;
      if (sl.d2 >= 0) *(u32x4*)(out + sl.d2 * es) = o2;
    }
  }
  if constexpr (BF16) {
    // K: token pairs, a sector each
    const int j0 = t0 >> 1, np = ((t1 - 1) >> 1) - j0 + 1;
    for (int e = tid; e < np * nslot * Hkv; e += 256) {
      const int j = j0 + e % np, h = e / (np * nslot);
      const Slot<BF16> sl(e / np % nslot, rot, halves);
      const bool na = 2 * j >= t0, nb = 2 * j + 1 < t1;  // (one of the two is new)
      u32x4 a1{}, a2{}, b1{}, b2{};
      if (na) turned<BF16>(row_of(a.k, a.k_row, 2 * j, Hkv, h), sl, cs[2 * j], rot, true, a1, a2);
      if (nb) turned<BF16>(row_of(a.k, a.k_row, 2 * j + 1, Hkv, h), sl, cs[2 * j + 1], rot, true, b1, b2);
      auto put = [&](int d, u32x4 x, u32x4 y) {
        u32x4* sec = (u32x4*)((uint16_t*)a.kpool + (tile0 + h) * tile + kswz(2 * j, d));
        if (!na) x = sec[0];
        if (!nb) y = sec[1];
        __builtin_nontemporal_store(x, sec);
        __builtin_nontemporal_store(y, sec + 1);
      };
      put(sl.d, a1, b1);
      if (sl.d2 >= 0) put(sl.d2, a2, b2);
    }
    // V: runs of 128 bytes, four tokens of dims d0 .. d0 + 7 and d0 + 16 .. d0 + 23
    const int q0 = t0 >> 2, nq = ((t1 - 1) >> 2) - q0 + 1, runs = D / 16;
    for (int e = tid; e < nq * Hkv * runs; e += 256) {
      const int r = e % runs, h = e / runs % Hkv, q = q0 + e / (runs * Hkv);
      const int d0 = 32 * (r >> 1) + 8 * (r & 1);
      u32x4* run = (u32x4*)((uint16_t*)a.vpool + (tile0 + h) * tile + vswz(4 * q, d0));
      u32x4 v[4][2] = {}, cur[8] = {};
      const bool all = 4 * q >= t0 && 4 * q + 4 <= t1;
      if (!all) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cur[i] = run[i];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (4 * q + t < t0 || 4 * q + t >= t1) continue;
        const char* row = row_of(a.v, a.v_row, 4 * q + t, Hkv, h) + d0 * 2;
        v[t][0] = *(const u32x4*)row;
        v[t][1] = *(const u32x4*)(row + 32);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (4 * q + t < t0 || 4 * q + t >= t1) continue;
        const uint32_t sh = 16 * (t & 1), keep = ~(0xFFFFu << sh);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          cur[i][t >> 1] = (cur[i][t >> 1] & keep) | (el16(v[t][0], i) << sh);
          cur[i][2 + (t >> 1)] = (cur[i][2 + (t >> 1)] & keep) | (el16(v[t][1], i) << sh);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) __builtin_nontemporal_store(cur[i], run + i);
    }
  } else {
    // row-major fp32 tiles: a token's row is whole lines
    for (int e = tid; e < n * Hkv * nslot; e += 256) {
      const int t = t0 + e / (Hkv * nslot), h = e / nslot % Hkv;
      const Slot<BF16> sl(e % nslot, rot, halves);
      u32x4 o1, o2;
      turned<BF16>(row_of(a.k, a.k_row, t, Hkv, h), sl, cs[t], rot, true, o1, o2);
      float* out = (float*)a.kpool + (tile0 + h) * tile + (size_t)t * D;
      *(u32x4*)(out + sl.d) = o1;
      if (sl.d2 >= 0) *(u32x4*)(out + sl.d2) = o2;
    }
    for (int e = tid; e < n * Hkv * (D / N); e += 256) {
      const int t = t0 + e / (Hkv * (D / N)), h = e / (D / N) % Hkv, d = e % (D / N) * N;
      *(u32x4*)((float*)a.vpool + (tile0 + h) * tile + (size_t)t * D + d) =
          *(const u32x4*)(row_of(a.v, a.v_row, t, Hkv, h) + d * es);
    }
  }
  if (a.codes && t1 == kPage) {
    __syncthreads();  // the block's own stores of the page's keys are read back
    for (int h = tid >> 6; h < Hkv; h += 4) {
      const size_t at = ((size_t)(a.layer0 + l) * Hkv + h) * a.max_pages + phys;
      summarize_page<BF16>((const char*)a.kpool + (tile0 + h) * tile * es, D, a.sum_row, a.codes + at * a.sum_row,
                           a.scale + at);
    }
  }
}

// ------------------------------------------------------------- page selection

// A launch's items: (token group, token of the group, layer, kv-head), the groups
// being gt consecutive new tokens of one sequence.
struct AttendItem {
  int s, tok, l, h, pos, pages;  // pos: the token's position; pages: how many it sees (0: no such token)
  size_t row;                    // (sequence, token) row of q, x and the page lists
};
__device__ __forceinline__ AttendItem attend_item(const AttendArgs& a, size_t item) {
  AttendItem r;
  r.h = (int)(item % a.n_kv_heads);
  item /= a.n_kv_heads;
  r.l = (int)(item % a.launch_layers);
  item /= a.launch_layers;
  const int j = (int)(item % a.gt), g = a.group0 + (int)(item / a.gt);
  r.s = g / a.seq_groups;
  r.tok = g % a.seq_groups * a.gt + j;
  r.pos = a.len0[r.s] + a.t + r.tok;
  r.pages = r.tok < a.n_tokens ? r.pos / kPage + 1 : 0;
  r.row = (size_t)r.s * a.n_tokens + r.tok;
  return r;
}
__device__ __forceinline__ const int32_t* page_list(const AttendArgs& a, const AttendItem& it, size_t item) {
  return a.pages_out ? a.pages_out + ((it.row * a.n_layers + a.layer - a.layer0 + it.l) * a.n_kv_heads + it.h) * a.n_pages
                     : a.list + item * a.n_pages;
}

// Bounds on the scores of every page that a token may select. With the q-heads
// of a kv-head taken together,
//   sum_g q_g . k  <=  sum_d (w+_d max_d + w-_d min_d),
//   w+ = sum_g max(q_g, 0),  w- = sum_g min(q_g, 0),
// for every key k of the page. The weights go to int8 with one power of two as
// scale (to nearest; the same for all pages, so it is left out), max and min are
// the page's codes: a product of 2 D int8 pairs on the matrix cores, exact in
// int32, times the page's power of two, exact in fp32 (2 * 128 * 127^2 < 2^24). So a
// page's bound has one value however the work is split. One block per (token
// group, layer, kv-head, kScorePages pages): 16 pages x up to 16 tokens per product,
// pages in rows, tokens in columns. Bound: HBM, the summaries are read once.
__global__ __launch_bounds__(256) void k_page_score(AttendArgs a) {
  __shared__ __align__(16) int8_t w[16][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int chunk = blockIdx.x % a.chunks;
  size_t item = blockIdx.x / a.chunks;  // (group, layer, kv-head)
  const int h = (int)(item % a.n_kv_heads);
  item /= a.n_kv_heads;
  const int l = (int)(item % a.launch_layers), gl = (int)(item / a.launch_layers), g = a.group0 + gl;
  const int s = g / a.seq_groups, tok0 = g % a.seq_groups * a.gt, nt = min(a.gt, a.n_tokens - tok0);
  const int len = a.len0[s] + a.t;
  const int pages = (len + tok0 + nt - 1) / kPage + 1;   // that the group's last token sees
  const int p0 = chunk * kScorePages, p1 = min(pages - a.last, p0 + kScorePages);
  if (pages <= a.n_pages || p0 >= p1) return;
  const int G = a.group, D = a.head_dim, row = a.sum_row;
  for (int i = tid; i < 16 * 256 / 4; i += 256) ((uint32_t*)w)[i] = 0u;
  __syncthreads();
  for (int j = wave; j < nt; j += 4) {
    const size_t qr = (((size_t)s * a.n_tokens + tok0 + j) * a.n_layers + a.layer - a.layer0 + l) * a.n_q_heads + (size_t)h * G;
    double up[2] = {0., 0.}, dn[2] = {0., 0.};
    for (int q = 0; q < G; ++q)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int d = lane + 64 * c;
        if (d >= D) continue;
        const size_t o = (qr + q) * D + d;
        const float x = a.bf16 ? bf2f(((const uint16_t*)a.q)[o]) : ((const float*)a.q)[o];
        up[c] += (double)fmaxf(x, 0.f);
        dn[c] += (double)fminf(x, 0.f);
      }
    double top = fmax(fmax(up[0], -dn[0]), fmax(up[1], -dn[1]));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmax(top, __shfl_xor(top, o));
    int ex = -kSumExp;
    if (top > 0.) {
      ex = ilogb(fmin(top, 1e300)) - 6;
      if (rint(ldexp(top, -ex)) > 127.) ++ex;
      ex = min(max(ex, -kSumExp), kSumExp);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int d = lane + 64 * c;
      if (d >= D) continue;
      w[j][d] = (int8_t)(int)fmin(rint(ldexp(up[c], -ex)), 127.);
      w[j][D + d] = (int8_t)(int)fmax(rint(ldexp(dn[c], -ex)), -127.);
    }
  }
  __syncthreads();
  const int col = lane & 15, quad = lane >> 4;
  i32x4 b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = *(const i32x4*)&w[col][64 * k + 16 * quad];
  const size_t base = ((size_t)(a.layer + l) * a.n_kv_heads + h) * a.max_pages;
  const int32_t* pt = a.page_table + (size_t)s * a.maxpps;
  const size_t out0 = ((size_t)gl * a.gt + col) * a.launch_layers + l;
  float* out = a.scores + (out0 * a.n_kv_heads + h) * a.score_row;
  for (int q = p0 + 16 * wave; q < p1; q += 64) {
    const int phys = pt[min(q + col, p1 - 1)];  // (pages past the range repeat its last one)
    const int8_t* code = a.codes + (base + phys) * row + 16 * quad;
    const float sc = a.scale[base + phys];
    i32x4 c = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (64 * k < row) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i32x4*)(code + 64 * k), b[k], c, 0, 0, 0);
    float4 o;
    o.x = (float)c[0] * __shfl(sc, 4 * quad);
    o.y = (float)c[1] * __shfl(sc, 4 * quad + 1);
    o.z = (float)c[2] * __shfl(sc, 4 * quad + 2);
    o.w = (float)c[3] * __shfl(sc, 4 * quad + 3);
    if (col < nt) *(float4*)(out + q + 4 * quad) = o;  // (rows hold whole groups of 16 pages)
  }
}

// fp32 order as unsigned order
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);  // (-0 counts as 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The chosen pages of one item, ascending: the first and the last ones and, of
// those between, the `want` highest bounds (the lower page of equal ones). The
// want-th highest key is found by radix, 8 bits a pass; then the pages are written
// in order, their places from prefix sums.
__global__ __launch_bounds__(256) void k_page_select(AttendArgs a) {
  __shared__ int hist[256];
  __shared__ uint32_t s_key;
  __shared__ int s_want, s_base;
  __shared__ int wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t item = blockIdx.x;
  const AttendItem it = attend_item(a, item);
  if (it.pages == 0) return;
  int32_t* list = const_cast<int32_t*>(page_list(a, it, item));
  if (it.pages <= a.n_pages) {
    for (int i = tid; i < a.n_pages; i += 256) list[i] = i < it.pages ? i : -1;
    return;
  }
  const int lo = a.first, hi = it.pages - a.last;
  int want = a.n_pages - a.first - a.last;
  for (int i = tid; i < a.first; i += 256) list[i] = i;
  for (int i = tid; i < a.last; i += 256) list[a.n_pages - a.last + i] = hi + i;
  if (want == 0) return;
  const float* sc = a.scores + item * a.score_row;
  uint32_t key = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int p = lo + tid; p < hi; p += 256) {
      const uint32_t k = order_key(sc[p]);
      if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {
      // lane i: bins 255 - 4i .. 252 - 4i, from the highest down
      int c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) { c[j] = hist[255 - 4 * lane - j]; sum += c[j]; }
      int before = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) { const int t = __shfl_up(before, o); if (lane >= o) before += t; }
      before -= sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < want && want <= before + c[j]) {
          s_key = key | ((uint32_t)(255 - 4 * lane - j) << shift);
          s_want = want - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    key = s_key;
    want = s_want;  // of the pages with this prefix
  }
  // want pages equal to the key are taken, the lowest first
  int base = a.first, ties = 0;
  for (int p0 = lo; p0 < hi; p0 += 256) {
    const int p = p0 + tid;
    const uint32_t k = p < hi ? order_key(sc[p]) : 0u;
    const bool gt = p < hi && k > key, eq = p < hi && k == key;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    if (lane == 0) wsum[wave] = (__popcll(mg) << 16) | __popcll(me);
    __syncthreads();
    int pre = 0, all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { if (i < wave) pre += wsum[i]; all += wsum[i]; }
    const int g = (pre >> 16) + __popcll(mg & below), e = ties + (pre & 0xFFFF) + __popcll(me & below);
    if (gt || (eq && e < want)) list[base + g + min(e, want) - min(ties, want)] = p;
    base += (all >> 16) + min(ties + (all & 0xFFFF), want) - min(ties, want);
    ties += all & 0xFFFF;
    __syncthreads();
  }
}

// ------------------------------------------------ attention over chosen pages

// Four output dims of a q-head in the storage type
template <bool BF16>
__device__ __forceinline__ void store_x4(const AttendArgs& a, const AttendItem& it, int g, int d, int D, f32x4 o) {
  const size_t at = ((it.row * a.n_layers + a.layer - a.layer0 + it.l) * a.n_q_heads + (size_t)it.h * a.group + g) * D + d;
  if constexpr (BF16) {
    const bf16x2 x = {(__bf16)o[0], (__bf16)o[1]}, y = {(__bf16)o[2], (__bf16)o[3]};
    *(uint2*)((uint16_t*)a.x_out + at) = make_uint2(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y));
  } else {
    *(f32x4*)((float*)a.x_out + at) = o;
  }
}

// One block of 4 waves per (item, part of its pages): the waves take batches of
// pages in turn, each with an online softmax of its own, and are merged in LDS.
// As in k_attn_bf16 the G q-heads of the kv-head are the columns of both products:
//   S^T[16 tok x 16 heads] = K[16 x D] Q^T,   O^T[D x 16 heads] += V^T[D x 16 tok] P^T.
// bf16: P goes into the second product as the sum of two bf16 values (what the
// first leaves over goes into the second, a relative error of 2^-18): the products
// are idle anyway while the pages come in. fp32: fp32 matrix cores throughout.
// Tokens behind the row's own position get score -inf, and their V counts as 0
// (those rows may hold anything).
template <bool BF16, int NU>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 4))) void k_attend(AttendArgs a) {
  constexpr int NJ = BF16 ? 2 * NU : NU;  // 16-dim output blocks
  constexpr int NB = 2;                   // pages per batch
  constexpr int DP = 16 * NJ + 4;
  __shared__ __align__(16) float sacc[4][kMaxGroup][DP];
  __shared__ float sm[4][kMaxGroup], sl[4][kMaxGroup];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int part = blockIdx.x % a.parts;
  const size_t item = blockIdx.x / a.parts;
  const AttendItem it = attend_item(a, item);
  const int total = min(it.pages, a.n_pages), c0 = part * a.part_pages, cnt = min(total - c0, a.part_pages);
  if (cnt <= 0) return;
  const int G = a.group, D = BF16 ? 32 * NU : a.head_dim;
  const bool chosen = it.pages > a.n_pages;
  const int32_t* list = chosen ? page_list(a, it, item) : nullptr;
  const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
  const int call_l = a.layer - a.layer0 + it.l;
  const size_t qrow = ((it.row * a.n_layers + call_l) * a.n_q_heads + (size_t)it.h * G + min(col, G - 1)) * D;
  u32x4 q[NU];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    if constexpr (BF16) q[i] = *(const u32x4*)((const uint16_t*)a.q + qrow + 32 * i + 8 * quad);
    else {
      const int d = 16 * i + 4 * quad;
      q[i] = *(const u32x4*)((const float*)a.q + qrow + min(d, D - 4));
      if (d >= D) q[i] = u32x4{0u, 0u, 0u, 0u};
    }
  }
  const size_t lay = (size_t)(a.layer + it.l) * a.max_pages;
  const size_t tile = (size_t)kPage * D;
  f32x4 acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNegInf, lsum = 0.f;
  for (int k0 = NB * wave; k0 < cnt; k0 += 4 * NB) {
    u32x4 kb[NB][NU], vb[NB][BF16 ? NU : 4];
    float vf[NB][BF16 ? 1 : NU][4];
    int lim[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int i = c0 + min(k0 + b, cnt - 1);
      const int page = __builtin_amdgcn_readfirstlane(chosen ? list[i] : i);
      const int phys = __builtin_amdgcn_readfirstlane(pt[page]);
      // tokens of the page that count (a batch's slots past the part's pages: none)
      lim[b] = k0 + b < cnt ? min(it.pos + 1 - kPage * page, kPage) : 0;
      const size_t t = ((lay + phys) * a.n_kv_heads + it.h) * tile;
      if constexpr (BF16) {
        const u32x4* kp = (const u32x4*)((const uint16_t*)a.kpool + t) + lane;
        const u32x4* vp = (const u32x4*)((const uint16_t*)a.vpool + t) + lane;
#pragma unroll
        for (int i2 = 0; i2 < NU; ++i2) { kb[b][i2] = kp[64 * i2]; vb[b][i2] = vp[64 * i2]; }
      } else {
        const float* kp = (const float*)a.kpool + t + (size_t)col * D;
        const float* vp = (const float*)a.vpool + t;
#pragma unroll
        for (int i2 = 0; i2 < NU; ++i2) {
          kb[b][i2] = *(const u32x4*)(kp + min(16 * i2 + 4 * quad, D - 4));
#pragma unroll
          for (int r = 0; r < 4; ++r) vf[b][i2][r] = vp[(size_t)(4 * quad + r) * D + min(16 * i2 + col, D - 1)];
        }
      }
    }
    f32x4 c[NB];
    float top = kNegInf;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        if constexpr (BF16) {
          c[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kb[b][i]),
                                                         __builtin_bit_cast(bf16x8, q[i]), c[b], 0, 0, 0);
        } else {
          const bool in = 16 * i + 4 * quad < D;  // (dims past D: 0 x 0)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            c[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? __uint_as_float(kb[b][i][e]) : 0.f,
                                                        __uint_as_float(q[i][e]), c[b], 0, 0, 0);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        c[b][r] = 4 * quad + r < lim[b] ? c[b][r] * a.scale_log2 : kNegInf;
        top = fmaxf(top, c[b][r]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float mn = fmaxf(m, top), alpha = m == mn ? 1.f : exp2f(m - mn);
    m = mn;
    lsum *= alpha;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float pr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        pr[r] = 4 * quad + r < lim[b] ? exp2f(c[b][r] - m) : 0.f;
        lsum += pr[r];
      }
      if (lim[b] < kPage) {  // uniform
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * quad + r >= lim[b]) {
            if constexpr (BF16) {
              const uint32_t keep = ~(0xFFFFu << (16 * (r & 1)));
#pragma unroll
              for (int i = 0; i < NU; ++i) { vb[b][i][r >> 1] &= keep; vb[b][i][2 + (r >> 1)] &= keep; }
            } else {
#pragma unroll
              for (int i = 0; i < NU; ++i) vf[b][i][r] = 0.f;
            }
          }
      }
      if constexpr (BF16) {
        s16x4 ph, pl;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const __bf16 x = (__bf16)pr[r];
          ph[r] = __builtin_bit_cast(short, x);
          pl[r] = __builtin_bit_cast(short, (__bf16)(pr[r] - (float)x));
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          const s16x4 v0 = __builtin_bit_cast(s16x4, uint2{vb[b][i][0], vb[b][i][1]});
          const s16x4 v1 = __builtin_bit_cast(s16x4, uint2{vb[b][i][2], vb[b][i][3]});
          acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v0, ph, acc[2 * i], 0, 0, 0);
          acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v1, ph, acc[2 * i + 1], 0, 0, 0);
          acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v0, pl, acc[2 * i], 0, 0, 0);
          acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v1, pl, acc[2 * i + 1], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < NU; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[b][i][r], pr[r], acc[i], 0, 0, 0);
      }
    }
  }
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (col < G) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) *(f32x4*)&sacc[wave][col][16 * j + 4 * quad] = acc[j];
    if (quad == 0) { sm[wave][col] = m; sl[wave][col] = lsum; }
  }
  __syncthreads();
  for (int e = tid; e < G * (D / 4); e += 256) {
    const int g = e / (D / 4), d = e % (D / 4) * 4;
    float mm = sm[0][g];
#pragma unroll
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, sm[w][g]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // (a wave without pages has l = 0 and m = -inf)
      const float f = sl[w][g] == 0.f ? 0.f : exp2f(sm[w][g] - mm);
      den += f * sl[w][g];
      o += f * *(const f32x4*)&sacc[w][g][d];
    }
    if (a.parts == 1) {
      store_x4<BF16>(a, it, g, d, D, o * (1.f / den));
    } else {
      const size_t w = (item * a.parts + part) * G + g;
      *(f32x4*)(a.part_acc + w * D + d) = o;
      if (d == 0) *(float2*)(a.part_ml + 2 * w) = make_float2(mm, den);
    }
  }
}

// The merge of an item's parts: o = sum_j acc_j 2^(m_j - m*) / sum_j l_j 2^(m_j - m*).
template <bool BF16>
__global__ __launch_bounds__(256) void k_attend_merge(AttendArgs a) {
  const size_t item = blockIdx.x;
  const AttendItem it = attend_item(a, item);
  if (it.pages == 0) return;
  const int G = a.group, D = a.head_dim;
  const int n = (min(it.pages, a.n_pages) + a.part_pages - 1) / a.part_pages;
  for (int e = threadIdx.x; e < G * (D / 4); e += 256) {
    const int g = e / (D / 4), d = e % (D / 4) * 4;
    const size_t w0 = item * a.parts * G + g;
    float mm = kNegInf;
    for (int j = 0; j < n; ++j) mm = fmaxf(mm, a.part_ml[2 * (w0 + (size_t)j * G)]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
    for (int j = 0; j < n; ++j) {
      const size_t w = w0 + (size_t)j * G;
      const float2 ml = *(const float2*)(a.part_ml + 2 * w);
      const float f = exp2f(ml.x - mm);
      den += f * ml.y;
      o += f * *(const f32x4*)(a.part_acc + w * D + d);
    }
    store_x4<BF16>(a, it, g, d, D, o * (1.f / den));
  }
}

}  // namespace

// ------------------------------------------------------------------ launchers

hipError_t launch_append_rows(const AppendRowsArgs& a, bool bf16, hipStream_t st, const Timing* tm) {
  const size_t blocks = (size_t)a.n_seqs * a.slots * a.n_layers;
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (bf16) return go(k_append_rows<true>, grid, dim3(256), 0, st, t0(tm), t1(tm), a);
  return go(k_append_rows<false>, grid, dim3(256), 0, st, t0(tm), t1(tm), a);
}

hipError_t launch_summarize(const SummaryArgs& a, bool bf16, hipStream_t st) {
  const size_t waves = (size_t)a.span * a.n_seqs * a.n_layers * a.n_kv_heads;
  if (waves == 0) return hipSuccess;
  if ((waves + 3) / 4 > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (bf16) return go(k_summarize<true>, grid, dim3(256), 0, st, nullptr, nullptr, a);
  return go(k_summarize<false>, grid, dim3(256), 0, st, nullptr, nullptr, a);
}

hipError_t launch_page_select(const AttendArgs& a, bool score, hipStream_t st, const Timing* tm) {
  const size_t items = (size_t)a.n_groups * a.gt * a.launch_layers * a.n_kv_heads;
  if (score) {
    const size_t blocks = items / a.gt * a.chunks;
    if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
    const hipError_t e = go(k_page_score, dim3((unsigned)blocks), dim3(256), 0, st, t0(tm), nullptr, a);
    if (e != hipSuccess) return e;
  }
  return go(k_page_select, dim3((unsigned)items), dim3(256), 0, st, score ? nullptr : t0(tm), t1(tm), a);
}

hipError_t launch_attend(const AttendArgs& a, hipStream_t st, const Timing* tm, const Timing* tm_merge) {
  const size_t items = (size_t)a.n_groups * a.gt * a.launch_layers * a.n_kv_heads;
  if (items * a.parts > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(items * a.parts));
  hipError_t e = hipErrorInvalidValue;
  auto run = [&](auto kernel) { e = go(kernel, grid, dim3(256), 0, st, t0(tm), t1(tm), a); };
  if (a.bf16) {
    if (a.head_dim == 128) run(k_attend<true, 4>);
    else if (a.head_dim == 64) run(k_attend<true, 2>);
  } else {
    switch ((a.head_dim + 15) / 16) {  // (head_dim <= 128)
      case 1: run(k_attend<false, 1>); break;
      case 2: run(k_attend<false, 2>); break;
      case 3: run(k_attend<false, 3>); break;
      case 4: run(k_attend<false, 4>); break;
      case 5: run(k_attend<false, 5>); break;
      case 6: run(k_attend<false, 6>); break;
      case 7: run(k_attend<false, 7>); break;
      case 8: run(k_attend<false, 8>); break;
    }
  }
  if (e != hipSuccess || a.parts == 1) return e;
  if (a.bf16) return go(k_attend_merge<true>, dim3((unsigned)items), dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a);
  return go(k_attend_merge<false>, dim3((unsigned)items), dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a);
}

}  // namespace pced
