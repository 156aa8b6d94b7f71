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

// Bounds on the scores of the pages that a token may select. With the q-heads of a
// kv-head taken together,
//   sum_g q_g . k  <=  sum_d (w+_d max_d + w-_d min_d),
//   w+ = sum_g max(q_g, 0),  w- = sum_g min(q_g, 0),
// for every key k of the page. The weights go to int8 with one power of two as
// scale (to nearest; the same for all pages, so it is left out), max and min are
// the page's codes: a product of 2 D int8 pairs on the matrix cores, exact in
// int32, times the page's power of two, exact in fp32 (2 * 128 * 127^2 < 2^24). So a
// page's bound has one value however the work is split, and the choice of pages
// is one and the same for every launch shape.

// The smallest exponent whose scale keeps v, rounded, within 127 (it grows with v,
// so the largest over a row's values is the row's). Sums are exact in fp64.
__device__ __forceinline__ int weight_exp(double v) {
  if (!(v > 0.)) return -kSumExp;
  int ex = ilogb(fmin(v, 1e300)) - 6;
  if (rint(ldexp(v, -ex)) > 127.) ++ex;
  return min(max(ex, -kSumExp), kSumExp);
}

// The weights of one row's kv-head (q at its first head) by one wave, lane i holding
// dims 2i and 2i + 1, to row[0 .. 2D).
__device__ __forceinline__ void query_weights(const AttendArgs& a, const void* q, int lane, int8_t* row) {
  const int G = a.group, D = a.head_dim, d = min(2 * lane, D - 2);
  double up[2] = {0., 0.}, dn[2] = {0., 0.};
  for (int g0 = 0; g0 < G; g0 += 4) {
    float x[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t o = (size_t)min(g0 + i, G - 1) * D + d;
      if (a.bf16) {
        const uint32_t u = *(const uint32_t*)((const uint16_t*)q + o);
        x[i][0] = bf2f(u & 0xFFFFu);
        x[i][1] = bf2f(u >> 16);
      } else {
        const f32x2 u = *(const f32x2*)((const float*)q + o);
        x[i][0] = u[0];
        x[i][1] = u[1];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (g0 + i < G)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          up[c] += (double)fmaxf(x[i][c], 0.f);
          dn[c] += (double)fminf(x[i][c], 0.f);
        }
  }
  int ex = max(max(weight_exp(up[0]), weight_exp(up[1])), max(weight_exp(-dn[0]), weight_exp(-dn[1])));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) ex = max(ex, __shfl_xor(ex, o));
  int8_t w[4];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    w[c] = (int8_t)(int)fmin(rint(ldexp(up[c], -ex)), 127.);
    w[2 + c] = (int8_t)(int)fmax(rint(ldexp(dn[c], -ex)), -127.);
  }
  if (2 * lane < D) {
    *(uint16_t*)(row + d) = (uint16_t)((uint8_t)w[0] | (uint8_t)w[1] << 8);
    *(uint16_t*)(row + D + d) = (uint16_t)((uint8_t)w[2] | (uint8_t)w[3] << 8);
  }
}

// 16 pages' codes as the rows of a product (lane: page lane % 16, bytes 16 (lane / 16)
// of each 64), and the pages' scales.
struct CodeTile {
  i32x4 c[4];
  float scale;
};
__device__ __forceinline__ void load_codes(const AttendArgs& a, size_t base, int phys, int quad, CodeTile& t) {
  const int8_t* code = a.codes + (base + phys) * a.sum_row + 16 * quad;
#pragma unroll
  for (int k = 0; k < 4; ++k) t.c[k] = *(const i32x4*)(code + min(64 * k, a.sum_row - 64));
  t.scale = a.scale[base + phys];
}
// bounds of pages 4 (lane / 16) .. + 3 of the tile for the token of column lane % 16
__device__ __forceinline__ float4 tile_bounds(const AttendArgs& a, const CodeTile& t, const i32x4 (&w)[4], int quad) {
  i32x4 c = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (64 * k < a.sum_row) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.c[k], w[k], c, 0, 0, 0);
  return make_float4((float)c[0] * __shfl(t.scale, 4 * quad), (float)c[1] * __shfl(t.scale, 4 * quad + 1),
                     (float)c[2] * __shfl(t.scale, 4 * quad + 2), (float)c[3] * __shfl(t.scale, 4 * quad + 3));
}

// fp32 order as unsigned order; 0 is below every number's key
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);  // (-0 counts as 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A token group's (group, layer, kv-head) of a launch
struct GroupItem {
  int s, l, h, gl, tok0, nt, len, pages;  // nt tokens from tok0 on; pages: that the last of them sees
};
__device__ __forceinline__ GroupItem group_item(const AttendArgs& a, size_t item) {
  GroupItem r;
  r.h = (int)(item % a.n_kv_heads);
  item /= a.n_kv_heads;
  r.l = (int)(item % a.launch_layers);
  r.gl = (int)(item / a.launch_layers);
  const int g = a.group0 + r.gl;
  r.s = g / a.seq_groups;
  r.tok0 = g % a.seq_groups * a.gt;
  r.nt = min(a.gt, a.n_tokens - r.tok0);
  r.len = a.len0[r.s] + a.t;
  r.pages = (r.len + r.tok0 + r.nt - 1) / kPage + 1;
  return r;
}
__device__ __forceinline__ const void* group_q(const AttendArgs& a, const GroupItem& it, int j) {
  const size_t row = ((size_t)it.s * a.n_tokens + it.tok0 + j) * a.n_layers + a.layer - a.layer0 + it.l;
  return (const char*)a.q + (row * a.n_q_heads + (size_t)it.h * a.group) * a.head_dim * (a.bf16 ? 2 : 4);
}
__device__ __forceinline__ size_t group_slot(const AttendArgs& a, const GroupItem& it, int j) {
  return (((size_t)it.gl * a.gt + j) * a.launch_layers + it.l) * a.n_kv_heads + it.h;
}

// The pages of one token from the keys of its candidates, page lo + 64 i + lane at
// key[i] (0: no candidate), by one wave: the want-th highest key bit by bit, from
// counts over the wave, then the pages in order, each at its place. want >= 1, and
// there are at least as many candidates. Returns nothing but the list.
template <int R>
__device__ __forceinline__ void pick_pages(const uint32_t (&key)[R], int lo, int want, int32_t* list, int lane) {
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | (1u << b);
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] >= c));
    if (n >= want) t = c;
  }
  int above = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) above += __popcll(__ballot(key[i] > t));
  const int ties = want - above;  // pages equal to the key that are taken, the lowest first
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int base = 0, eq = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t mg = __ballot(key[i] > t), me = __ballot(key[i] == t);
    const int e = eq + __popcll(me & below);
    if (key[i] > t || (key[i] == t && e < ties))
      list[base + __popcll(mg & below) + min(e, ties) - min(eq, ties)] = lo + 64 * i + lane;
    const int eq1 = eq + __popcll(me);
    base += __popcll(mg) + min(eq1, ties) - min(eq, ties);
    eq = eq1;
  }
}

// The pages that need no choice: all of them, or the first and the last ones.
// Returns how many are to be chosen between.
__device__ __forceinline__ int fixed_pages(const AttendArgs& a, int pages, int32_t* list, int i0, int step) {
  if (pages <= a.n_pages) {
    for (int i = i0; i < a.n_pages; i += step) list[i] = i < pages ? i : -1;
    return 0;
  }
  for (int i = i0; i < a.first; i += step) list[i] = i;
  for (int i = i0; i < a.last; i += step) list[a.n_pages - a.last + i] = pages - a.last + i;
  return a.n_pages - a.first - a.last;
}

// Bounds and choice in one launch, for at most 64 R pages: one block of 8 waves per
// (token group, layer, kv-head), R/2 tiles of 16 pages per wave. The codes are on
// their way while the weights are made; the bounds meet in LDS, from where each
// wave chooses the pages of a token.
template <int R>
__global__ __launch_bounds__(512) void k_page_pick(AttendArgs a) {
  constexpr int NT = R / 2;
  __shared__ __align__(16) int8_t w[16][256];
  __shared__ __align__(16) float bound[16][64 * R + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const GroupItem it = group_item(a, blockIdx.x);
  if (it.pages > a.n_pages) {
    const int p1 = it.pages - a.last;  // pages [first, p1) are chosen between
    const size_t base = ((size_t)(a.layer + it.l) * a.n_kv_heads + it.h) * a.max_pages;
    const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
    CodeTile t[NT];
    int phys[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) phys[i] = pt[min(16 * (wave + 8 * i) + col, p1 - 1)];
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (16 * (wave + 8 * i) < p1) load_codes(a, base, phys[i], quad, t[i]);
    for (int j = wave; j < it.nt; j += 8) query_weights(a, group_q(a, it, j), lane, w[j]);
    __syncthreads();
    i32x4 b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = *(const i32x4*)&w[col][64 * k + 16 * quad];
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (16 * (wave + 8 * i) < p1) {
        const float4 o = tile_bounds(a, t[i], b, quad);
        if (col < it.nt) *(float4*)&bound[col][16 * (wave + 8 * i) + 4 * quad] = o;
      }
    __syncthreads();
  }
  for (int j = wave; j < it.nt; j += 8) {
    const size_t slot = group_slot(a, it, j);
    const AttendItem row = attend_item(a, slot);
    int32_t* list = const_cast<int32_t*>(page_list(a, row, slot));
    if (row.pages <= a.n_pages && !a.pages_out) continue;  // (all pages: nobody reads the list)
    const int want = fixed_pages(a, row.pages, list, lane, 64);
    if (want == 0) continue;
    uint32_t key[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int p = 64 * i + lane;
      key[i] = p >= a.first && p < row.pages - a.last ? order_key(bound[j][p]) : 0u;
    }
    pick_pages<R>(key, 0, want, list + a.first, lane);
  }
}

// The same in two launches for long sequences, whose summaries one work-group would
// take long to read. Bounds: a block per (token group, layer, kv-head, kScorePages
// pages), four tiles of 16 pages per wave. Bound: HBM, the summaries are read once.
__global__ __launch_bounds__(256) void k_page_score(AttendArgs a) {
  constexpr int NT = kScorePages / 64;
  __shared__ __align__(16) int8_t w[16][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const GroupItem it = group_item(a, blockIdx.x / a.chunks);
  const int p0 = blockIdx.x % a.chunks * kScorePages, p1 = min(it.pages - a.last, p0 + kScorePages);
  if (it.pages <= a.n_pages || p0 >= p1) return;
  const size_t base = ((size_t)(a.layer + it.l) * a.n_kv_heads + it.h) * a.max_pages;
  const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
  CodeTile t[NT];
  int phys[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) phys[i] = pt[min(p0 + 16 * (wave + 4 * i) + col, p1 - 1)];
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (p0 + 16 * (wave + 4 * i) < p1) load_codes(a, base, phys[i], quad, t[i]);
  for (int j = wave; j < it.nt; j += 4) query_weights(a, group_q(a, it, j), lane, w[j]);
  __syncthreads();
  i32x4 b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = *(const i32x4*)&w[col][64 * k + 16 * quad];
  float* out = a.scores + group_slot(a, it, col) * a.score_row + p0 + 4 * quad;
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (p0 + 16 * (wave + 4 * i) < p1) {
      const float4 o = tile_bounds(a, t[i], b, quad);
      if (col < it.nt) *(float4*)(out + 16 * (wave + 4 * i)) = o;  // (rows hold whole tiles)
    }
}

// The choice from those bounds: a block of 16 waves per item, wave v's keys being the
// v-th run of 64 R candidates. As pick_pages, with the counts of the waves added up
// in LDS, one barrier per bit. A row of more than 1024 R candidates (MANY) goes in
// rounds, whose keys are read again for every bit.
template <int R, bool MANY>
__global__ __launch_bounds__(1024) void k_page_select(AttendArgs a) {
  __shared__ int count[33];
  __shared__ int wsum[2][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t item = blockIdx.x;
  const AttendItem it = attend_item(a, item);
  if (it.pages == 0 || (it.pages <= a.n_pages && !a.pages_out)) return;
  int32_t* list = const_cast<int32_t*>(page_list(a, it, item));
  const int want = fixed_pages(a, it.pages, list, tid, 1024);
  if (want == 0) return;
  list += a.first;
  const int lo = a.first, hi = it.pages - a.last;
  const int rounds = MANY ? (hi - lo + 1024 * R - 1) / (1024 * R) : 1;
  const float* sc = a.scores + item * a.score_row;
  uint32_t key[R];
  auto load = [&](int round) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int p = lo + (round * 16 + wave) * 64 * R + 64 * i + lane;
      key[i] = p < hi ? order_key(sc[min(p, hi - 1)]) : 0u;
    }
  };
  if (tid < 33) count[tid] = 0;
  load(0);
  __syncthreads();
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | (1u << b);
    int n = 0;
    for (int r = 0; r < rounds; ++r) {
      if (MANY) load(r);
#pragma unroll
      for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] >= c));
    }
    if (lane == 0 && n) atomicAdd(&count[b], n);
    __syncthreads();
    if (count[b] >= want) t = c;
  }
  int n = 0;
  for (int r = 0; r < rounds; ++r) {
    if (MANY) load(r);
#pragma unroll
    for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] > t));
  }
  if (lane == 0 && n) atomicAdd(&count[32], n);
  __syncthreads();
  const int ties = want - count[32];
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int base = 0, eq = 0;  // places taken and equal keys met before the round
  for (int r = 0; r < rounds; ++r) {
    if (MANY) load(r);
    int g = 0, e = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) { g += __popcll(__ballot(key[i] > t)); e += __popcll(__ballot(key[i] == t)); }
    if (lane == 0) { wsum[0][wave] = g; wsum[1][wave] = e; }
    __syncthreads();
    int gb = 0, eb = 0, ga = 0, ea = 0;  // before this wave, and of all
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if (v < wave) { gb += wsum[0][v]; eb += wsum[1][v]; }
      ga += wsum[0][v];
      ea += wsum[1][v];
    }
    int at = base + gb + min(eq + eb, ties) - min(eq, ties), seen = eq + eb;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint64_t mg = __ballot(key[i] > t), me = __ballot(key[i] == t);
      const int k = seen + __popcll(me & below);
      if (key[i] > t || (key[i] == t && k < ties))
        list[at + __popcll(mg & below) + min(k, ties) - min(seen, ties)] = lo + (r * 16 + wave) * 64 * R + 64 * i + lane;
      const int seen1 = seen + __popcll(me);
      at += __popcll(mg) + min(seen1, ties) - min(seen, ties);
      seen = seen1;
    }
    base += ga + min(eq + ea, ties) - min(eq, ties);
    eq += ea;
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
//   S^T[16 tok x 16 heads] = K[16 x D] Q^T,   O^T[D x 16 heads] += V^T[D x 32 tok] P^T,
// and the softmax's reference moves only when a score exceeds it by 8 (weights stay
// within 2^8), so that the common page needs no rescaling.
// bf16: a batch is two pages, which the second product takes at once: its inner
// dimension holds four tokens of the one and four of the other per lane, which is
// where the scores' registers and V's 16-byte units have them. P goes in as the sum
// of two bf16 values (what the first leaves over goes into the second, a relative
// error of 2^-17): the matrix cores are idle anyway while the pages come in. fp32:
// one page, fp32 matrix cores throughout.
// A wave holds the physical ids of its pages (64 at a time) one per lane, so that no
// batch waits for a chain of list and page table, and loads a batch while it works
// on the one before.
// Tokens behind the row's own position get weight 0, and their V counts as 0 (those
// rows may hold anything).
template <bool BF16, int NU>
struct PageRegs {
  static constexpr int NB = BF16 ? 2 : 1;
  u32x4 k[NB][NU];
  u32x4 v[BF16 ? NB : 1][BF16 ? NU : 1];
  float vf[BF16 ? 1 : NU][4];
};

template <bool BF16, int NU>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(!BF16 && NU > 6 ? 1 : 2, 4))) void k_attend(AttendArgs a) {
  using Regs = PageRegs<BF16, NU>;
  constexpr int NJ = BF16 ? 2 * NU : NU;  // 16-dim output blocks
  constexpr int NB = Regs::NB;            // pages per batch
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
  // the wave's u-th page is page (u / NB) 4 NB + NB wave + u % NB of the part
  auto nth = [&](int u) { return u / NB * 4 * NB + NB * wave + u % NB; };
  int my_page = 0, my_phys = 0;
  auto ids = [&](int u0) {  // lane i: the wave's page u0 + i (past the part's end its last one)
    const int i = c0 + min(nth(u0 + lane), cnt - 1);
    my_page = chosen ? list[i] : i;
    my_phys = pt[my_page];
  };
  ids(0);
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
  auto load = [&](int u, Regs& r) __attribute__((always_inline)) {  // pages u .. u + NB - 1 of those in the lanes
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const size_t t = ((lay + __builtin_amdgcn_readlane(my_phys, u + b)) * a.n_kv_heads + it.h) * tile;
      if constexpr (BF16) {
        const u32x4* kp = (const u32x4*)((const uint16_t*)a.kpool + t) + lane;
        const u32x4* vp = (const u32x4*)((const uint16_t*)a.vpool + t) + lane;
#pragma unroll
        for (int i = 0; i < NU; ++i) r.k[b][i] = kp[64 * i];
#pragma unroll
        for (int i = 0; i < NU; ++i) r.v[b][i] = vp[64 * i];
      } else {
        const float* kp = (const float*)a.kpool + t + (size_t)col * D;
        const float* vp = (const float*)a.vpool + t;
#pragma unroll
        for (int i = 0; i < NU; ++i) r.k[b][i] = *(const u32x4*)(kp + min(16 * i + 4 * quad, D - 4));
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) r.vf[i][e] = vp[(size_t)(4 * quad + e) * D + min(16 * i + col, D - 1)];
      }
    }
  };
  f32x4 acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNegInf, lsum = 0.f;
  auto work = [&](int u, int k0, Regs& r) __attribute__((always_inline)) {
    f32x4 c[NB];
    int lim[NB];  // tokens of the page that count (a batch's slots past the part's end: none)
    float top = kNegInf;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int page = __builtin_amdgcn_readlane(my_page, u + b);
      lim[b] = k0 + b < cnt ? min(it.pos + 1 - kPage * page, kPage) : 0;
      c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        if constexpr (BF16) {
          c[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[b][i]),
                                                         __builtin_bit_cast(bf16x8, q[i]), c[b], 0, 0, 0);
        } else {
          const bool in = 16 * i + 4 * quad < D;  // (dims past D: 0 x 0)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            c[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? __uint_as_float(r.k[b][i][e]) : 0.f,
                                                        __uint_as_float(q[i][e]), c[b], 0, 0, 0);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) c[b][e] *= a.scale_log2;
      if (lim[b] < kPage) {  // uniform
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (4 * quad + e < lim[b]) continue;
          c[b][e] = kNegInf;
          if constexpr (BF16) {
            const uint32_t keep = ~(0xFFFFu << (16 * (e & 1)));
#pragma unroll
            for (int i = 0; i < NU; ++i) { r.v[b][i][e >> 1] &= keep; r.v[b][i][2 + (e >> 1)] &= keep; }
          } else {
#pragma unroll
            for (int i = 0; i < NU; ++i) r.vf[i][e] = 0.f;
          }
        }
      }
      top = fmaxf(top, fmaxf(fmaxf(c[b][0], c[b][1]), fmaxf(c[b][2], c[b][3])));
    }
    if (__any(top > m + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top), alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      lsum *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
    }
    // a column whose scores so far are all -inf keeps the reference -inf: its weights, 2^(-inf + inf), are NaN,
    // as the softmax of nothing but -inf is; slots and tokens that do not count weigh 0 all the same
    float p[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[b][e] = __builtin_amdgcn_exp2f(c[b][e] - m);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (lim[b] < kPage)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[b][e] = 4 * quad + e < lim[b] ? p[b][e] : 0.f;
      lsum += (p[b][0] + p[b][1]) + (p[b][2] + p[b][3]);
    }
    if constexpr (BF16) {
      bf16x8 hi, lo;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          hi[4 * b + e] = (__bf16)p[b][e];
          lo[4 * b + e] = (__bf16)(p[b][e] - (float)hi[4 * b + e]);
        }
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const bf16x8 v0 = __builtin_bit_cast(bf16x8, u32x4{r.v[0][i][0], r.v[0][i][1], r.v[1][i][0], r.v[1][i][1]});
        const bf16x8 v1 = __builtin_bit_cast(bf16x8, u32x4{r.v[0][i][2], r.v[0][i][3], r.v[1][i][2], r.v[1][i][3]});
        acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, hi, acc[2 * i], 0, 0, 0);
        acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, hi, acc[2 * i + 1], 0, 0, 0);
        acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, lo, acc[2 * i], 0, 0, 0);
        acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, lo, acc[2 * i + 1], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < NU; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(r.vf[i][e], p[0][e], acc[i], 0, 0, 0);
    }
  };
  // two batches of registers in turn; ids are read again every 64 pages of the wave, when
  // the next batch is the first of the new ones (64 / NB batches: an even number)
  Regs ra, rb;
  if (NB * wave < cnt) load(0, ra);
  for (int v0 = 0, k0 = NB * wave; k0 < cnt; v0 += 64) {
    for (int u = 0; u < 64 && k0 < cnt; u += 2 * NB) {
      const int page_k1 = k0 + 4 * NB, page_k2 = k0 + 8 * NB;
      if (page_k1 < cnt) load(u + NB, rb);
      work(u, k0, ra);
      const bool turn = u + 2 * NB == 64;
      if (page_k2 < cnt && !turn) load(u + 2 * NB, ra);
      if (page_k1 < cnt) work(u + NB, page_k1, rb);
      if (page_k2 < cnt && turn) {
        ids(v0 + 64);
        load(0, ra);
      }
      k0 = page_k2;
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
  const size_t items = (size_t)a.n_groups * a.gt * a.launch_layers * a.n_kv_heads, groups = items / a.gt;
  if (items > 0x7FFFFFFFu || groups * a.chunks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const int pages = a.score_row;
  if (!score || pages <= kPickPages) {
    const dim3 grid((unsigned)groups);
    if (!score || pages <= 128) return go(k_page_pick<2>, grid, dim3(512), 0, st, t0(tm), t1(tm), a);
    if (pages <= 256) return go(k_page_pick<4>, grid, dim3(512), 0, st, t0(tm), t1(tm), a);
    return go(k_page_pick<8>, grid, dim3(512), 0, st, t0(tm), t1(tm), a);
  }
  const hipError_t e = go(k_page_score, dim3((unsigned)(groups * a.chunks)), dim3(256), 0, st, t0(tm), nullptr, a);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)items);
  if (pages <= 2048) return go(k_page_select<2, false>, grid, dim3(1024), 0, st, nullptr, t1(tm), a);
  if (pages <= 8192) return go(k_page_select<8, false>, grid, dim3(1024), 0, st, nullptr, t1(tm), a);
  if (pages <= 16384) return go(k_page_select<16, false>, grid, dim3(1024), 0, st, nullptr, t1(tm), a);
  return go(k_page_select<16, true>, grid, dim3(1024), 0, st, nullptr, t1(tm), a);
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
