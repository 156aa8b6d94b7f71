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

// A slot's unit(s) of a row
template <bool BF16>
__device__ __forceinline__ void load_slot(const char* row, const Slot<BF16>& sl, u32x4& o1, u32x4& o2) {
  constexpr int es = BF16 ? 2 : 4;
  o1 = *(const u32x4*)(row + (size_t)sl.d * es);
  o2 = *(const u32x4*)(row + (size_t)(sl.d2 >= 0 ? sl.d2 : sl.d) * es);
}
// Rotated: (a, b) -> (a cos - b sin, a sin + b cos) in fp32, rounded once
template <bool BF16>
__device__ __forceinline__ void turn_slot(const Slot<BF16>& sl, const float2* cs, int rot, u32x4& o1, u32x4& o2) {
  constexpr int N = Unit<BF16>::N;
  if (sl.d >= rot) return;
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

// For every (sequence, page that the sequence's new tokens touch, layer) one block for
// K, one for V, and blocks of kAppendTasks slots for the q rows. A page that is new from
// end to end is written in contiguous 1 KiB wave stores, V through LDS (as in k_load);
// of other pages the K units are written by token pairs and the V runs by token quads,
// so that only whole 32-byte sectors are stored (see k_append): tokens of the sector
// that are not new keep what they hold. The
// angles' cos and sin, in fp64 and rounded once, are made by the block for its at most
// 16 positions and shared by its heads, while the rows' first loads are under way
// (several slots of a thread at once: a store may not pass a later slot's load). A page
// that becomes full is summarised by the block that filled it. Bound: HBM for many
// tokens (64 of 33 sequences, 32/8 heads of 128: 15.8 us for 52 MB, 3.3 TB/s; reads and
// writes in turn reach 5.1), the chain of length, rows and stores for one (eight layers
// of 33 sequences 6.8 us, one of five 3.6).
constexpr int kAppendTasks = 1024;
template <bool BF16>
__global__ __launch_bounds__(256) void k_append_rows(AppendRowsArgs a) {
  constexpr int N = Unit<BF16>::N, es = BF16 ? 2 : 4;
  __shared__ union {
    struct {
      float2 cs[kPage][64];
      double turn_of[64];
    } t;
    uint4 v[BF16 ? 4 : 1][BF16 ? 512 : 1];
  } lds;
  auto& cs = lds.t.cs;
  auto& turn_of = lds.t.turn_of;
  const int tid = threadIdx.x;
  const uint32_t per = 2 + a.q_blocks;
  uint32_t x = blockIdx.x / per;
  const int z = blockIdx.x - x * per;  // 0: K, 1: V, from 2 on: q
  const uint32_t x1 = x / (uint32_t)a.slots;
  const int slot = x - x1 * a.slots;
  int s = x1, l = 0;
  if (a.n_layers > 1) {
    l = x1 / (uint32_t)a.n_seqs;
    s = x1 - l * a.n_seqs;
  }
  const int len = a.len0[s] + a.t, p = len / kPage + slot;
  const int t0 = max(len - kPage * p, 0), t1 = min(len + a.n_tokens - kPage * p, kPage);  // new tokens of the page
  if (t0 >= t1) return;
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, D = a.head_dim, rot = a.rot_dim;
  const bool halves = a.halves != 0;
  const size_t row0 = (size_t)s * a.n_tokens + (kPage * p - len);  // row of the page's token 0 (as a difference)
  const int half = rot / 2, n = t1 - t0;
  const int nslot = Slot<BF16>::count(D, rot, halves);
  if (z > 1 && (z - 2) * kAppendTasks >= n * Hq * nslot) return;
  auto row_of = [&](const void* base, int64_t stride, int t, int heads, int h) {
    return (const char*)base + ((size_t)(row0 + t) * stride + ((size_t)l * heads + h) * D) * es;
  };
  // cos and sin of the block's positions; ends with a barrier
  auto trig = [&] {
    if (rot == 0) return;
    if (tid < half) turn_of[tid] = exp2(-(2.0 * tid / rot) * a.log2_theta) * 0.31830988618379067154;  // over pi
    __syncthreads();
    for (int e = tid; e < n * half; e += 256) {
      const int t = e / half, i = e - t * half;
      double sn, co;
      sincospi((double)(kPage * p + t0 + t) * turn_of[i], &sn, &co);
      cs[t0 + t][i] = make_float2((float)co, (float)sn);
    }
    __syncthreads();
  };

  if (z > 1) {
    constexpr int U = kAppendTasks / 256;
    const int total = n * Hq * nslot;
    u32x4 o1[U], o2[U];
    int tok[U], head[U], un[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = min((z - 2) * kAppendTasks + 256 * i + tid, total - 1);
      const int r = e / nslot;
      un[i] = e - r * nslot;
      tok[i] = r / Hq;
      head[i] = r - tok[i] * Hq;
      load_slot<BF16>(row_of(a.q, a.q_row, t0 + tok[i], Hq, head[i]), Slot<BF16>(un[i], rot, halves), o1[i], o2[i]);
    }
    trig();
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if ((z - 2) * kAppendTasks + 256 * i + tid >= total) break;
      const Slot<BF16> sl(un[i], rot, halves);
      turn_slot<BF16>(sl, cs[t0 + tok[i]], rot, o1[i], o2[i]);
      char* out = (char*)a.q_out + (((row0 + t0 + tok[i]) * a.n_layers + l) * Hq + head[i]) * D * es;
      *(u32x4*)(out + sl.d * es) = o1[i];
      if (sl.d2 >= 0) *(u32x4*)(out + sl.d2 * es) = o2[i];
    }
    return;
  }

  const int phys = a.page_table[(size_t)s * a.maxpps + p];
  const size_t tile = (size_t)kPage * D;
  const size_t tile0 = ((size_t)(a.layer0 + l) * a.max_pages + phys) * Hkv;
  if constexpr (BF16) {
    if (z == 1) {
      const int runs = D / 16;  // of a kv-head's token quad
      if (n == kPage) {
        // a wave takes 64 runs: 4 x 2 pieces of a run's rows, transposed in registers, to the wave's 8 KiB of LDS
        // (units XOR-swizzled against bank conflicts) and out as contiguous units
        uint4* mine = lds.v[tid >> 6];
        const int lane = tid & 63, all = 4 * Hkv * runs;
        for (int b = tid >> 6; 64 * b < all; b += 4) {
          const RunPos rp = run_pos(min(64 * b + lane, all - 1), D);
          u32x4 v[4][2];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const char* row = row_of(a.v, a.v_row, 4 * rp.q + t, Hkv, rp.g) + rp.d0 * 2;
            v[t][0] = *(const u32x4*)row;
            v[t][1] = *(const u32x4*)(row + 32);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            mine[lane * 8 + (i ^ (lane & 7))] =
                make_uint4(el16(v[0][0], i) | (el16(v[1][0], i) << 16), el16(v[2][0], i) | (el16(v[3][0], i) << 16),
                           el16(v[0][1], i) | (el16(v[1][1], i) << 16), el16(v[2][1], i) | (el16(v[3][1], i) << 16));
          wave_lds_sync();
          u32x4* out = (u32x4*)((uint16_t*)a.vpool + tile0 * tile) + 512 * b + lane;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int m = 64 * i + lane;
            const uint4 w = mine[(m >> 3) * 8 + ((m & 7) ^ ((m >> 3) & 7))];
            if (512 * b + m < 8 * all) __builtin_nontemporal_store(u32x4{w.x, w.y, w.z, w.w}, out + 64 * i);
          }
          wave_lds_sync();
        }
        return;
      }
      // runs of 128 bytes, four tokens of dims d0 .. d0 + 7 and d0 + 16 .. d0 + 23
      const int q0 = t0 >> 2, nq = ((t1 - 1) >> 2) - q0 + 1;
      for (int e = tid; e < nq * Hkv * runs; e += 256) {
        const int r = e % runs, h = e / runs % Hkv, q = q0 + e / (runs * Hkv);
        const int d0 = 32 * (r >> 1) + 8 * (r & 1);
        u32x4* run = (u32x4*)((uint16_t*)a.vpool + (tile0 + h) * tile + vswz(4 * q, d0));
        u32x4 v[4][2], cur[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) cur[i] = run[i];
#pragma unroll
        for (int t = 0; t < 4; ++t) {  // (tokens that are not new: a new one's row again)
          const char* row = row_of(a.v, a.v_row, min(max(4 * q + t, t0), t1 - 1), Hkv, h) + d0 * 2;
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
      return;
    }
    if (n == kPage) {
      // K: a lane per token, 16 tokens of a unit next to each other
      constexpr int U = 4;
      const int total = kPage * nslot * Hkv, t = tid & 15;
      u32x4 v1[U], v2[U];
      auto load = [&](int e0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int r = min(e0 + 256 * i + tid, total - 1) >> 4, h = r / nslot;
          load_slot<BF16>(row_of(a.k, a.k_row, t, Hkv, h), Slot<BF16>(r - h * nslot, rot, halves), v1[i], v2[i]);
        }
      };
      load(0);
      trig();
      for (int e0 = 0;;) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int e = e0 + 256 * i + tid, r = e >> 4, h = r / nslot;
          if (e >= total) break;
          const Slot<BF16> sl(r - h * nslot, rot, halves);
          turn_slot<BF16>(sl, cs[t], rot, v1[i], v2[i]);
          uint16_t* out = (uint16_t*)a.kpool + (tile0 + h) * tile;
          __builtin_nontemporal_store(v1[i], (u32x4*)(out + kswz(t, sl.d)));
          if (sl.d2 >= 0) __builtin_nontemporal_store(v2[i], (u32x4*)(out + kswz(t, sl.d2)));
        }
        e0 += 256 * U;
        if (e0 >= total) break;
        load(e0);
      }
    } else {
      // K: token pairs, a sector each
      constexpr int U = 2;
      const int j0 = t0 >> 1, np = ((t1 - 1) >> 1) - j0 + 1, total = np * nslot * Hkv;
      u32x4 v1[U][2], v2[U][2];
      int pair[U], head[U], un[U];
      auto load = [&](int e0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int e = min(e0 + 256 * i + tid, total - 1), r = e / np;
          pair[i] = j0 + e - r * np;
          head[i] = r / nslot;
          un[i] = r - head[i] * nslot;
          const Slot<BF16> sl(un[i], rot, halves);
#pragma unroll
          for (int c = 0; c < 2; ++c)  // (a token of the sector that is not new: its neighbour's row again)
            load_slot<BF16>(row_of(a.k, a.k_row, min(max(2 * pair[i] + c, t0), t1 - 1), Hkv, head[i]), sl, v1[i][c],
                            v2[i][c]);
        }
      };
      load(0);
      trig();
      for (int e0 = 0;;) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (e0 + 256 * i + tid >= total) break;
          const Slot<BF16> sl(un[i], rot, halves);
          const int ta = 2 * pair[i];
          const bool na = ta >= t0, nb = ta + 1 < t1;  // (one of the two is new)
          if (na) turn_slot<BF16>(sl, cs[ta], rot, v1[i][0], v2[i][0]);
          if (nb) turn_slot<BF16>(sl, cs[ta + 1], rot, v1[i][1], v2[i][1]);
          auto put = [&](int d, u32x4 x, u32x4 y) {
            u32x4* sec = (u32x4*)((uint16_t*)a.kpool + (tile0 + head[i]) * tile + kswz(ta, d));
            if (!na) x = sec[0];
            if (!nb) y = sec[1];
            __builtin_nontemporal_store(x, sec);
            __builtin_nontemporal_store(y, sec + 1);
          };
          put(sl.d, v1[i][0], v1[i][1]);
          if (sl.d2 >= 0) put(sl.d2, v2[i][0], v2[i][1]);
        }
        e0 += 256 * U;
        if (e0 >= total) break;
        load(e0);
      }
    }
  } else if (z == 1) {
    // row-major fp32 tiles: a token's row is whole lines
    for (int e = tid; e < n * Hkv * (D / N); e += 256) {
      const int t = t0 + e / (Hkv * (D / N)), h = e / (D / N) % Hkv, d = e % (D / N) * N;
      *(u32x4*)((float*)a.vpool + (tile0 + h) * tile + (size_t)t * D + d) =
          *(const u32x4*)(row_of(a.v, a.v_row, t, Hkv, h) + d * es);
    }
    return;
  } else {
    trig();
    for (int e = tid; e < n * Hkv * nslot; e += 256) {
      const int t = t0 + e / (Hkv * nslot), h = e / nslot % Hkv;
      const Slot<BF16> sl(e % nslot, rot, halves);
      u32x4 o1, o2;
      load_slot<BF16>(row_of(a.k, a.k_row, t, Hkv, h), sl, o1, o2);
      turn_slot<BF16>(sl, cs[t], rot, o1, o2);
      float* out = (float*)a.kpool + (tile0 + h) * tile + (size_t)t * D;
      *(u32x4*)(out + sl.d) = o1;
      if (sl.d2 >= 0) *(u32x4*)(out + sl.d2) = o2;
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
// being gt consecutive new tokens of one sequence. (Fewer than 2^31 of them.)
struct AttendItem {
  int s, tok, l, h, pos, pages;  // pos: the token's position; pages: how many it sees (0: no such token)
  size_t row;                    // (sequence, token) row of q, x and the page lists
};
__device__ __forceinline__ AttendItem attend_item(const AttendArgs& a, uint32_t item) {
  AttendItem r;
  r.h = item % (uint32_t)a.n_kv_heads;
  item /= (uint32_t)a.n_kv_heads;
  r.l = 0;
  if (a.launch_layers > 1) {
    r.l = item % (uint32_t)a.launch_layers;
    item /= (uint32_t)a.launch_layers;
  }
  uint32_t j = 0, g = item;
  if (a.gt > 1) {
    j = item % (uint32_t)a.gt;
    g = item / (uint32_t)a.gt;
  }
  g += a.group0;
  r.s = g;
  r.tok = j;
  if (a.seq_groups > 1) {
    r.s = g / (uint32_t)a.seq_groups;
    r.tok = (g - r.s * a.seq_groups) * a.gt + j;
  }
  r.pos = a.len0[r.s] + a.t + r.tok;
  r.pages = r.tok < a.n_tokens ? r.pos / kPage + 1 : 0;
  r.row = (size_t)r.s * a.n_tokens + r.tok;
  return r;
}
__device__ __forceinline__ const int32_t* page_list(const AttendArgs& a, const AttendItem& it, uint32_t item) {
  return a.pages_out ? a.pages_out + ((it.row * a.n_layers + a.layer - a.layer0 + it.l) * a.n_kv_heads + it.h) * a.n_pages
                     : a.list + (size_t)item * a.n_pages;
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

// The smallest exponent whose scale keeps v >= 0, rounded to nearest, within 127 (it
// grows with v, so the largest over a row's values is the row's): v's own exponent less
// 6, and one more where v 2^-e would be 127.5 or more, which is where the fraction's
// first 7 bits are all ones. Sums are exact in fp64.
__device__ __forceinline__ int weight_exp(double v) {
  return min(max((__double2hiint(v) + (1 << 13) >> 20) - 1023 - 6, -kSumExp), kSumExp);
}

// The largest of the lanes' values, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto step = [&](uint32_t y) { x = max(x, y); };
  // (row shifts by 1, 2, 4, 8, then the rows' last lanes to the rows behind; lanes without a source keep their own)
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x111, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x112, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x114, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x118, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x142, 0xA, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x143, 0xC, 0xF, false));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
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
  const int mine = max(max(weight_exp(up[0]), weight_exp(up[1])), max(weight_exp(-dn[0]), weight_exp(-dn[1])));
  const int ex = (int)wave_max((uint32_t)(mine + kSumExp)) - kSumExp;
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
template <int K>
struct CodeTile {
  i32x4 c[K];
  float scale;
};
template <int K>
__device__ __forceinline__ void load_codes(const AttendArgs& a, size_t base, int phys, int quad, CodeTile<K>& t) {
  const int8_t* code = a.codes + (base + phys) * a.sum_row + 16 * quad;
#pragma unroll
  for (int k = 0; k < K; ++k) t.c[k] = *(const i32x4*)(code + min(64 * k, a.sum_row - 64));
  t.scale = a.scale[base + phys];
}
// the sums of pages 4 (lane / 16) .. + 3 of the tile for the token of column lane % 16
template <int K>
__device__ __forceinline__ float4 tile_sums(const AttendArgs& a, const CodeTile<K>& t, const i32x4 (&w)[K]) {
  i32x4 c = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (64 * k < a.sum_row) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.c[k], w[k], c, 0, 0, 0);
  return make_float4((float)c[0], (float)c[1], (float)c[2], (float)c[3]);
}
// the pages' bounds: sums times scales
template <int K>
__device__ __forceinline__ float4 tile_bounds(const AttendArgs& a, const CodeTile<K>& t, const i32x4 (&w)[K], int quad) {
  const float4 c = tile_sums<K>(a, t, w);
  return make_float4(c.x * __shfl(t.scale, 4 * quad), c.y * __shfl(t.scale, 4 * quad + 1), c.z * __shfl(t.scale, 4 * quad + 2),
                     c.w * __shfl(t.scale, 4 * quad + 3));
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
__device__ __forceinline__ GroupItem group_item(const AttendArgs& a, uint32_t item) {
  GroupItem r;
  r.h = item % (uint32_t)a.n_kv_heads;
  item /= (uint32_t)a.n_kv_heads;
  r.l = 0;
  r.gl = item;
  if (a.launch_layers > 1) {
    r.l = item % (uint32_t)a.launch_layers;
    r.gl = item / (uint32_t)a.launch_layers;
  }
  const uint32_t g = a.group0 + r.gl;
  r.s = g;
  r.tok0 = 0;
  if (a.seq_groups > 1) {
    r.s = g / (uint32_t)a.seq_groups;
    r.tok0 = (g - r.s * a.seq_groups) * a.gt;
  }
  r.nt = min(a.gt, a.n_tokens - r.tok0);
  r.len = a.len0[r.s] + a.t;
  r.pages = (r.len + r.tok0 + r.nt - 1) / kPage + 1;
  return r;
}
__device__ __forceinline__ const void* group_q(const AttendArgs& a, const GroupItem& it, int j) {
  const size_t row = ((size_t)it.s * a.n_tokens + it.tok0 + j) * a.n_layers + a.layer - a.layer0 + it.l;
  return (const char*)a.q + (row * a.n_q_heads + (size_t)it.h * a.group) * a.head_dim * (a.bf16 ? 2 : 4);
}
__device__ __forceinline__ uint32_t group_slot(const AttendArgs& a, const GroupItem& it, int j) {
  return (((uint32_t)it.gl * a.gt + j) * a.launch_layers + it.l) * a.n_kv_heads + it.h;
}
// the token's item
__device__ __forceinline__ AttendItem group_row(const AttendArgs& a, const GroupItem& it, int j) {
  AttendItem r;
  r.s = it.s;
  r.tok = it.tok0 + j;
  r.l = it.l;
  r.h = it.h;
  r.pos = it.len + r.tok;
  r.pages = r.pos / kPage + 1;
  r.row = (size_t)it.s * a.n_tokens + r.tok;
  return r;
}

// The pages of one token from the keys of its candidates, page lo + 64 i + lane at
// key[i] (0: no candidate), by one wave: the want-th highest key bit by bit below the
// bits that all keys share, from counts over the wave (done as soon as a bound has just
// `want` keys above it, which takes about as many bits as tell neighbours apart), then
// the pages in order, each at its place. want >= 1, and there are at least as many
// candidates.
template <int R>
__device__ __forceinline__ void pick_pages(const uint32_t (&key)[R], int lo, int want, int32_t* list, int lane) {
  uint32_t kmax = 0, kmin = 0;  // (kmin: of the complements)
#pragma unroll
  for (int i = 0; i < R; ++i) {
    kmax = max(kmax, key[i]);
    kmin = max(kmin, key[i] ? ~key[i] : 0u);
  }
  kmax = wave_max(kmax);
  kmin = ~wave_max(kmin);
  int b = kmax == kmin ? -1 : 31 - __clz(kmax ^ kmin);
  uint32_t t = b < 0 ? kmin : kmax >> b >> 1 << b << 1;
  for (; b >= 0; --b) {
    const uint32_t c = t | (1u << b);
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] >= c));
    if (n >= want) t = c;
    if (n == want) {
      t = c - 1;  // exactly the keys above this
      break;
    }
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

// Keys of pages [lo, hi), page 64 i + lane at key[i], from their sums and scales in LDS (which hold 64 R)
template <int R>
__device__ __forceinline__ void page_keys(const float* sums, const float* scale, int lo, int hi, int lane,
                                          uint32_t (&key)[R]) {
  float x[R], y[R];
#pragma unroll
  for (int i = 0; i < R; ++i) { x[i] = sums[64 * i + lane]; y[i] = scale[64 * i + lane]; }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int p = 64 * i + lane;
    const uint32_t k = order_key(x[i] * y[i]);
    key[i] = p >= lo && p < hi ? k : 0u;
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

// Bounds and choice in one launch, for at most 64 R pages (of up to 64 K bytes of codes):
// one block of 8 waves per (token group, layer, kv-head), R / 2 tiles of 16 pages per
// wave. The codes are on their way while the weights are made; the bounds meet in LDS, from where each
// wave chooses the pages of a token. Bound: latency (lengths, ids, codes, weights and
// the choice one after the other): 24 new tokens of 17 sequences of up to 8192
// tokens, 4 kv-heads, 204 blocks, 15.2 us.
template <int R, int K>
__global__ __launch_bounds__(512) void k_page_pick(AttendArgs a) {
  constexpr int W = 8, NT = 4 * R / W, T = kAttendTokens;
  __shared__ __align__(16) int8_t w[16][256];  // (columns past the tokens' count for nothing)
  __shared__ __align__(16) float bound[T][64 * R + 4];  // (sums, to be scaled)
  __shared__ float scale[64 * R];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const GroupItem it = group_item(a, blockIdx.x);
  if (it.pages > a.n_pages) {
    const int p1 = it.pages - a.last;  // pages [first, p1) are chosen between
    const size_t base = ((size_t)(a.layer + it.l) * a.n_kv_heads + it.h) * a.max_pages;
    const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
    CodeTile<K> t[NT];
    int phys[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) phys[i] = pt[min(16 * (wave + W * i) + col, p1 - 1)];
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (16 * (wave + W * i) < p1) load_codes(a, base, phys[i], quad, t[i]);
    for (int j = wave; j < it.nt; j += W) query_weights(a, group_q(a, it, j), lane, w[j]);
    __syncthreads();
    i32x4 b[K];
#pragma unroll
    for (int k = 0; k < K; ++k) b[k] = *(const i32x4*)&w[col][64 * k + 16 * quad];
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (16 * (wave + W * i) < p1) {
        const float4 o = tile_sums<K>(a, t[i], b);
        if (col < it.nt) *(float4*)&bound[col][16 * (wave + W * i) + 4 * quad] = o;
        if (quad == 0) scale[16 * (wave + W * i) + col] = t[i].scale;
      }
    __syncthreads();
  }
  for (int j = wave; j < it.nt; j += W) {
    const uint32_t slot = group_slot(a, it, j);
    const AttendItem row = group_row(a, it, j);
    int32_t* list = const_cast<int32_t*>(page_list(a, row, slot));
    if (row.pages <= a.n_pages && !a.pages_out) continue;  // (all pages: nobody reads the list)
    const int want = fixed_pages(a, row.pages, list, lane, 64);
    if (want == 0) continue;
    uint32_t key[R];
    page_keys<R>(bound[j], scale, a.first, row.pages - a.last, lane, key);
    pick_pages<R>(key, 0, want, list + a.first, lane);
  }
}

// The same in two launches for long sequences, whose summaries one work-group would
// take long to read. Bounds: a block per (token group, layer, kv-head, chunk_pages
// pages), each wave 32 of every 128 pages at a time; their ids are two rounds ahead and
// their codes one. Bound: HBM, the summaries are read once, in pieces of 256 bytes: 9
// sequences of up to 8192 pages, 8 kv-heads, 101 MB in 28 us (3.6 TB/s) where the pages
// lie scattered, 20 us (5.0) in order. (Blocks of all kv-heads, a page's codes of all of
// them next to each other: 31 and 26 us.)
template <int K>
__global__ __launch_bounds__(256) void k_page_score(AttendArgs a) {
  __shared__ __align__(16) int8_t w[16][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const GroupItem it = group_item(a, blockIdx.x / (uint32_t)a.chunks);
  const int p0 = blockIdx.x % (uint32_t)a.chunks * a.chunk_pages, p1 = min(it.pages - a.last, p0 + a.chunk_pages);
  if (it.pages <= a.n_pages || p0 >= p1) return;
  const size_t base = ((size_t)(a.layer + it.l) * a.n_kv_heads + it.h) * a.max_pages;
  const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
  struct Ids {
    int a, b;
  };
  struct Tiles {
    CodeTile<K> a, b;
  };
  const int q0 = p0 + 32 * wave;  // the wave's first pages
  // (past the range its last page)
  auto ids = [&](int q) { return Ids{pt[min(q + col, p1 - 1)], pt[min(q + 16 + col, p1 - 1)]}; };
  auto load = [&](const Ids& p, Tiles& t) __attribute__((always_inline)) {
    load_codes(a, base, p.a, quad, t.a);
    load_codes(a, base, p.b, quad, t.b);
  };
  Ids ia = ids(q0), ib = ids(q0 + 128);
  Tiles ta, tb;
  load(ia, ta);
  for (int j = wave; j < it.nt; j += 4) query_weights(a, group_q(a, it, j), lane, w[j]);
  __syncthreads();
  i32x4 b[K];
#pragma unroll
  for (int k = 0; k < K; ++k) b[k] = *(const i32x4*)&w[col][64 * k + 16 * quad];
  float* out = a.scores + (size_t)group_slot(a, it, min(col, it.nt - 1)) * a.score_row + 4 * quad;
  auto put = [&](int q, const Tiles& t) __attribute__((always_inline)) {
    const float4 x = tile_bounds<K>(a, t.a, b, quad), y = tile_bounds<K>(a, t.b, b, quad);
    if (col < it.nt && q < p1) *(float4*)(out + q) = x;  // (rows hold whole tiles)
    if (col < it.nt && q + 16 < p1) *(float4*)(out + q + 16) = y;
  };
  for (int q = q0; q < p1; q += 256) {
    ia = ids(q + 256);
    load(ib, tb);
    put(q, ta);
    ib = ids(q + 384);
    load(ia, ta);
    put(q + 128, tb);
  }
}

// The choice from those bounds: a block of W waves per item, wave v's keys being the
// v-th run of 64 R candidates. The candidates are counted in kBins equal steps of
// their range (which spreads them, so that the LDS atomics rarely meet), the step that
// holds the want-th highest bound is found from the counts, and its candidates, a few,
// are ranked one by one. Where they are more than kNear (bounds far from the rest
// squeeze it into few steps), the bound is searched bit by bit as in pick_pages, with the
// counts of the waves added up in LDS and two bits per barrier. A row of more than
// 64 W R candidates (MANY) goes in rounds, whose keys are read again for every pass.
// Bound: latency for few rows (some ten passes between barriers), for many the passes'
// instructions, most of which are a wave's and not a key's. us with 16 / 8 / 4 waves:
// rows of up to 8192 pages, 72 of them 11.2 / 14.2 / 22, 576 20.3 / 16.2; of up to 3750,
// 72 7.5 / 8.6 / 12.8, 216 7.8 / 8.8 / 13.0, 576 13.8 / 10.0 / 14.0, 3264 74 / 37 / 33;
// of up to 2000, 72 6.1 / 6.1 / 7.8, 576 9.6 / 7.8 / 9.1. More candidates per thread
// than the pages need: 72 rows of 8192 15.4 at R = 16 (W = 16).
constexpr int kBins = 2048, kNear = 512;
__device__ __forceinline__ float order_value(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
template <int W, int R, bool MANY>
__global__ __launch_bounds__(64 * W) void k_page_select(AttendArgs a) {
  constexpr int NT = 64 * W, C = kBins / NT;
  __shared__ int count[52], hist[kBins], near_page[kNear];
  __shared__ uint32_t near_key[kNear], wmin[W], wmax[W], s_key;
  __shared__ int wsum[2][W], s_bin, s_need, s_near, s_page;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t item = blockIdx.x;
  const AttendItem it = attend_item(a, item);
  if (it.pages == 0 || (it.pages <= a.n_pages && !a.pages_out)) return;
  int32_t* list = const_cast<int32_t*>(page_list(a, it, item));
  const int want = fixed_pages(a, it.pages, list, tid, NT);
  if (want == 0) return;
  list += a.first;
  const int lo = a.first, hi = it.pages - a.last;
  const int rounds = MANY ? (hi - lo + NT * R - 1) / (NT * R) : 1;
  const float* sc = a.scores + (size_t)item * a.score_row;
  uint32_t key[R];
  auto load = [&](int round) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int p = lo + (round * W + wave) * 64 * R + 64 * i + lane;
      key[i] = p < hi ? order_key(sc[min(p, hi - 1)]) : 0u;
    }
  };
  for (int i = tid; i < kBins; i += NT) hist[i] = 0;
  if (tid < 52) count[tid] = 0;
  load(0);
  // the range of the bounds
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
  for (int r = 0; r < rounds; ++r) {
    if (MANY) load(r);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      kmin = min(kmin, key[i] ? key[i] : 0xFFFFFFFFu);
      kmax = max(kmax, key[i]);
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor((int)kmin, o));
    kmax = max(kmax, (uint32_t)__shfl_xor((int)kmax, o));
  }
  if (lane == 0) { wmin[wave] = kmin; wmax[wave] = kmax; }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < W; ++v) { kmin = min(kmin, wmin[v]); kmax = max(kmax, wmax[v]); }
  const float low = order_value(kmin), span = order_value(kmax) - low;
  const float inv = span > 0.f ? (float)(kBins - 1) / span : 0.f;
  auto bin_of = [&](uint32_t k) { return min((int)((order_value(k) - low) * inv), kBins - 1); };  // (grows with k)
  for (int r = 0; r < rounds; ++r) {
    if (MANY) load(r);
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (key[i]) atomicAdd(&hist[bin_of(key[i])], 1);
  }
  __syncthreads();
  {  // thread i: C bins from kBins - 1 - C i down
    int h[C], sum = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) sum += h[c] = hist[kBins - 1 - C * tid - c];
    int run = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(run, o); if (lane >= o) run += x; }
    if (lane == 63) wsum[0][wave] = run;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < W; ++v) if (v < wave) run += wsum[0][v];
    int above = run - sum;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (above < want && want <= above + h[c]) {
        s_bin = kBins - 1 - C * tid - c;
        s_need = want - above;
        s_near = h[c];
      }
      above += h[c];
    }
  }
  __syncthreads();
  const int bin = s_bin, need = s_need;  // the best `need` of this bin's, and all above it
  uint32_t t = 0;
  int ties = 0x7FFFFFFF, last_tie = 0x7FFFFFFF;  // equal keys that are taken: so many, and up to this page
  if (s_near <= kNear) {
    for (int r = 0; r < rounds; ++r) {
      if (MANY) load(r);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (key[i] && bin_of(key[i]) == bin) {
          const int at = atomicAdd(&count[0], 1);
          near_key[at] = key[i];
          near_page[at] = lo + (r * W + wave) * 64 * R + 64 * i + lane;
        }
    }
    __syncthreads();
    const int n = s_near;
    for (int i = tid; i < n; i += NT) {
      const uint32_t k = near_key[i];
      const int p = near_page[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += near_key[j] > k || (near_key[j] == k && near_page[j] < p);
      if (rank == need - 1) { s_key = k; s_page = p; }
    }
    __syncthreads();
    t = s_key;
    last_tie = s_page;
  } else {
    bool exact = false;
    for (int b = 30; b >= 0 && !exact; b -= 2) {  // two bits: keys from t + 2^b, 2 * 2^b and 3 * 2^b on
      const uint32_t c = 1u << b;
      int n[3] = {0, 0, 0};
      for (int r = 0; r < rounds; ++r) {
        if (MANY) load(r);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int j = 0; j < 3; ++j) n[j] += __popcll(__ballot(key[i] >= t + (j + 1) * c));
      }
      int* at = count + 3 * (b >> 1);
      if (lane < 3) {
        const int mine = lane == 0 ? n[0] : lane == 1 ? n[1] : n[2];
        if (mine) atomicAdd(&at[lane], mine);
      }
      __syncthreads();
      const int n1 = at[0], n2 = at[1], n3 = at[2];
      const int k = n3 >= want ? 3 : n2 >= want ? 2 : n1 >= want ? 1 : 0;
      exact = (k == 3 ? n3 : k == 2 ? n2 : k == 1 ? n1 : 0) == want;
      t += k * c - (exact ? 1u : 0u);  // (exactly the keys above it)
    }
    // the pages equal to the key: as many as there is room for, from the first on
    int n = 0;
    for (int r = 0; r < rounds; ++r) {
      if (MANY) load(r);
#pragma unroll
      for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] > t));
    }
    if (lane == 0 && n) atomicAdd(&count[51], n);
    __syncthreads();
    ties = want - count[51];
  }
  auto page_at = [&](int r, int i) { return lo + (r * W + wave) * 64 * R + 64 * i + lane; };
  auto tie = [&](int r, int i) { return key[i] == t && page_at(r, i) <= last_tie; };
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int base = 0, eq = 0;  // places taken and equal keys met before the round
  for (int r = 0; r < rounds; ++r) {
    if (MANY) load(r);
    int g = 0, e = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) { g += __popcll(__ballot(key[i] > t)); e += __popcll(__ballot(tie(r, i))); }
    if (lane == 0) { wsum[0][wave] = g; wsum[1][wave] = e; }
    __syncthreads();
    int gb = 0, eb = 0, ga = 0, ea = 0;  // before this wave, and of all
#pragma unroll
    for (int v = 0; v < W; ++v) {
      if (v < wave) { gb += wsum[0][v]; eb += wsum[1][v]; }
      ga += wsum[0][v];
      ea += wsum[1][v];
    }
    int at = base + gb + min(eq + eb, ties) - min(eq, ties), seen = eq + eb;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint64_t mg = __ballot(key[i] > t), me = __ballot(tie(r, i));
      const int k = seen + __popcll(me & below);
      if (key[i] > t || (tie(r, i) && k < ties))
        list[at + __popcll(mg & below) + min(k, ties) - min(seen, ties)] = page_at(r, i);
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

// The softmax's first reference: the lowest finite number, so that scores of -inf weigh
// 2^(-inf - m) = 0 wherever they come first (a reference of -inf would make that NaN), and
// every higher score still moves it. A row of nothing but -inf ends as 0 / 0, NaN.
constexpr float kLowest = -3.402823466e38f;

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
// and the softmax's reference moves only when a score exceeds it by `lead` (weights stay
// within 2^8), so that the common page needs no rescaling. Scores and references are the
// products q . k as summed; log2(e) / sqrt(D) scales their differences, so that a weight's
// error grows with its distance from the reference and not with the scores' own size.
// bf16: a batch is two pages, which the second product takes at once: its inner
// dimension holds four tokens of the one and four of the other per lane, which is
// where the scores' registers and V's 16-byte units have them. P goes in as the sum
// of two bf16 values (what the first leaves over goes into the second, a relative
// error of 2^-17): the matrix cores are idle anyway while the pages come in. fp32:
// one page, fp32 matrix cores throughout, a score summed in NA chains that are then added:
// rounding errors of a chain add up like its length (heads of 128 dims, rms error of wide
// rows' outputs 1.35e-6 with one chain, 3.7e-7 with four; of 64, 4.9e-7 and 3.9e-7 with
// two). Four need registers that only one wave per SIMD has.
// A wave holds the ids of its pages (a part has at most 64 per wave) one per lane, so
// that no batch waits for a chain of list and page table, and loads a batch while it
// works on the one before (no load is conditional: the wait for a batch must leave
// the next one in flight on every path).
// Tokens behind the row's own position get weight 0, and their V counts as 0 (those
// rows may hold anything).
// Bound: HBM where items abound (16 layers of 33 sequences, 32 of up to 128 pages, 8
// kv-heads, PICK: 1.18 GB in 209 us, 5.6 TB/s); start and drain of short streams at one
// layer (18 us for 74 MB; 256 pages of 9 sequences in 504 work-groups, 29 us for 134 MB);
// with many tokens the way from the L2, which has most of their pages (24 tokens of 17
// sequences, 64 pages each, 53 us for 0.8 GB of which HBM gives a sixth).
template <bool BF16, int NU>
struct PageRegs {
  static constexpr int NB = BF16 ? 2 : 1;
  u32x4 k[NB][NU];
  u32x4 v[BF16 ? NB : 1][BF16 ? NU : 1];
  float vf[BF16 ? 1 : NU][4];
};

// PICK: the block chooses its item's pages itself, as k_page_pick does: one new token,
// at most kPickPages pages, one part. The launch that this saves, and the list's way
// through memory, cost more than the pages that wait behind the choice: see run_attend.
template <bool BF16, int NU, bool PICK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(!BF16 && NU > 6 ? 1 : 2, 4))) void k_attend(AttendArgs a) {
  using Regs = PageRegs<BF16, NU>;
  constexpr int NJ = BF16 ? 2 * NU : NU;  // 16-dim output blocks
  constexpr int NB = Regs::NB;            // pages per batch
  constexpr int NA = BF16 ? 1 : NU > 6 ? 4 : 2;  // chains of a score's sum
  // fp32: row r of output block 4 g + c is dim 64 g + 4 r + c, so that a lane's V of four blocks is one 16-byte load
  // (the blocks past the last four: dim 16 j + r)
  constexpr int NV = BF16 ? 0 : NJ / 4 * 4;
  constexpr int DP = 16 * NJ + 4;
  __shared__ __align__(16) float sacc[4][kMaxGroup][DP];
  __shared__ float sm[4][kMaxGroup], sl[4][kMaxGroup];
  __shared__ __align__(16) int8_t s_w[PICK ? 256 : 16];
  __shared__ __align__(16) float s_bound[PICK ? kPickPages : 4];  // (sums, to be scaled)
  __shared__ float s_scale[PICK ? kPickPages : 1];
  __shared__ int32_t s_list[PICK ? kAttendPart : 1], s_phys[PICK ? kPickPages : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  // Work-groups go to the eight dies in turn. With several new tokens, all those of one
  // (sequence, layer, kv-head) go to one die and follow each other there, so that pages
  // which several of them chose are in its L2.
  uint32_t item, part;
  if (a.n_tokens == 1) {
    item = blockIdx.x / (uint32_t)a.parts;
    part = blockIdx.x - item * a.parts;
  } else {
    const uint32_t s0 = (uint32_t)a.group0 / a.seq_groups, tok = (uint32_t)a.seq_groups * a.gt, per = tok * a.parts;
    const uint32_t r = blockIdx.x >> 3, k = r / per, rest = r - k * per;
    const uint32_t pair = (blockIdx.x & 7) + 8 * k;  // (layer, kv-head, sequence)
    const uint32_t heads = (uint32_t)a.launch_layers * a.n_kv_heads;
    const uint32_t lh = pair / a.launch_seqs, s = pair - lh * a.launch_seqs;
    const uint32_t i = rest / a.parts, g = (s0 + s) * a.seq_groups + i / a.gt - a.group0;  // the token's group
    if (lh >= heads || g >= (uint32_t)a.n_groups) return;
    part = rest - i * a.parts;
    item = (g * a.gt + i % a.gt) * heads + lh;
  }
  const AttendItem it = attend_item(a, item);
  const int total = min(it.pages, a.n_pages), c0 = part * a.part_pages, cnt = min(total - c0, a.part_pages);
  if (cnt <= 0) return;
  const int G = a.group, D = BF16 ? 32 * NU : a.head_dim;
  const bool chosen = it.pages > a.n_pages;
  const int32_t* list = chosen && !PICK ? page_list(a, it, item) : nullptr;
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
  if constexpr (PICK) {
    // (the page ids do not wait for the length: pages that the sequence does not have get some id)
    constexpr int R = kPickPages / 64, KC = BF16 ? NU : (NU + 1) / 2;  // (sum_row / 64)
    int phys[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      phys[i] = 0;
      if (16 * (wave + 4 * i) < a.score_row) phys[i] = max(pt[min(16 * (wave + 4 * i) + col, a.maxpps - 1)], 0);
    }
    int32_t* out = a.pages_out ? const_cast<int32_t*>(page_list(a, it, item)) : nullptr;
    if (!chosen) {
      if (out) fixed_pages(a, it.pages, out, tid, 256);
    } else {
      const int p1 = it.pages - a.last;
      const size_t base = ((size_t)(a.layer + it.l) * a.n_kv_heads + it.h) * a.max_pages;
      CodeTile<KC> t[R];
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (16 * (wave + 4 * i) < p1) load_codes(a, base, phys[i], quad, t[i]);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (quad == 0) s_phys[16 * (wave + 4 * i) + col] = phys[i];
      if (wave == 0)
        query_weights(a, (const char*)a.q + (qrow - (size_t)min(col, G - 1) * D) * (BF16 ? 2 : 4), lane, s_w);
      __syncthreads();
      i32x4 w[KC];
#pragma unroll
      for (int k = 0; k < KC; ++k) w[k] = *(const i32x4*)&s_w[64 * k + 16 * quad];  // (every column the token's)
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (16 * (wave + 4 * i) < p1) {
          const float4 o = tile_sums<KC>(a, t[i], w);
          if (col == 0) *(float4*)&s_bound[16 * (wave + 4 * i) + 4 * quad] = o;
          if (quad == 0) s_scale[16 * (wave + 4 * i) + col] = t[i].scale;
        }
      __syncthreads();
      if (wave == 0) {
        const int want = fixed_pages(a, it.pages, s_list, lane, 64);
        if (want > 0) {
          uint32_t key[R];
          page_keys<R>(s_bound, s_scale, a.first, p1, lane, key);
          pick_pages<R>(key, 0, want, s_list + a.first, lane);
        }
      }
      __syncthreads();
      if (out && tid < a.n_pages) out[tid] = s_list[tid];  // (n_pages <= kAttendPart)
    }
  }
  // the wave's u-th page is page (u / NB) 4 NB + NB wave + u % NB of the part
  auto nth = [&](int u) { return u / NB * 4 * NB + NB * wave + u % NB; };
  const int mine = c0 + min(nth(lane), cnt - 1);  // (past the part's end its last page)
  const int my_page = !chosen ? mine : PICK ? s_list[mine] : list[mine];
  const int my_phys = PICK && chosen ? s_phys[my_page] : pt[my_page];
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
        for (int e = 0; e < 4; ++e) {
          const float* row = vp + (4 * quad + e) * D;
#pragma unroll
          for (int i = 0; i < NV; i += 4) {
            const f32x4 x = *(const f32x4*)(row + min(16 * i + 4 * col, D - 4));
#pragma unroll
            for (int c = 0; c < 4; ++c) r.vf[i + c][e] = x[c];
          }
#pragma unroll
          for (int i = NV; i < NU; ++i) r.vf[i][e] = row[min(16 * i + col, D - 1)];
        }
      }
    }
  };
  f32x4 acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kLowest, lsum = 0.f;
  auto work = [&](int u, int k0, Regs& r) __attribute__((always_inline)) {
    f32x4 c[NB];
    float top = kNegInf;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int page = __builtin_amdgcn_readlane(my_page, u + b);
      // tokens of the page that count (a batch's slots past the part's end: none)
      const int lim = k0 + b < cnt ? min(it.pos + 1 - kPage * page, kPage) : 0;
      c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      f32x4 ch[NA];
#pragma unroll
      for (int e = 0; e < NA; ++e) ch[e] = c[b];
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        if constexpr (BF16) {
          c[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[b][i]),
                                                         __builtin_bit_cast(bf16x8, q[i]), c[b], 0, 0, 0);
        } else {
          const bool in = 16 * i + 4 * quad < D;  // (dims past D: 0 x 0)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            ch[e % NA] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? __uint_as_float(r.k[b][i][e]) : 0.f,
                                                              __uint_as_float(q[i][e]), ch[e % NA], 0, 0, 0);
        }
      }
      if constexpr (!BF16) c[b] = NA == 4 ? (ch[0] + ch[1]) + (ch[2] + ch[NA - 1]) : ch[0] + ch[NA - 1];
      if (lim < kPage) {  // uniform
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (4 * quad + e < lim) continue;
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
    if (__any(top > m + a.lead)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top), alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.scale_log2);
      m = mn;
      lsum *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
    }
    float p[NB][4];  // (of slots and tokens that do not count 2^(-inf - m) = 0)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[b][e] = __builtin_amdgcn_exp2f((c[b][e] - m) * a.scale_log2);
#pragma unroll
    for (int b = 0; b < NB; ++b) lsum += (p[b][0] + p[b][1]) + (p[b][2] + p[b][3]);
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
  const int nb = (cnt - NB * wave + 4 * NB - 1) / (4 * NB);  // the wave's batches
  auto step = [&](int i, Regs& r) __attribute__((always_inline)) { work(NB * i, NB * wave + 4 * NB * i, r); };
  if (cnt > NB * wave) {
    Regs ra, rb;
    load(0, ra);
    int i = 0;
    for (; i + 2 < nb; i += 2) {
      load(NB * (i + 1), rb);
      step(i, ra);
      load(NB * (i + 2), ra);
      step(i + 1, rb);
    }
    if (nb - i == 2) {
      load(NB * (i + 1), rb);
      step(i, ra);
      step(i + 1, rb);
    } else {
      step(i, ra);
    }
  }
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (col < G) {
#pragma unroll
    for (int j = 0; j < NV; j += 4)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *(f32x4*)&sacc[wave][col][16 * (j + quad) + 4 * e] = f32x4{acc[j][e], acc[j + 1][e], acc[j + 2][e], acc[j + 3][e]};
#pragma unroll
    for (int j = NV; j < NJ; ++j) *(f32x4*)&sacc[wave][col][16 * j + 4 * quad] = acc[j];
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
      const float f = exp2f((sm[w][g] - mm) * a.scale_log2);  // (a wave without pages: l = 0 and m = kLowest)
      den += f * sl[w][g];
      o += f * *(const f32x4*)&sacc[w][g][d];
    }
    if (a.parts == 1) {
      store_x4<BF16>(a, it, g, d, D, o / den);
    } else {
      const size_t w = ((size_t)item * a.parts + part) * G + g;
      *(f32x4*)(a.part_acc + w * D + d) = o;
      if (d == 0) *(float2*)(a.part_ml + 2 * w) = make_float2(mm, den);
    }
  }
}

// The merge of an item's parts: o = sum_j acc_j 2^(c (m_j - m*)) / sum_j l_j 2^(c (m_j - m*)), c = scale_log2.
template <bool BF16>
__global__ __launch_bounds__(256) void k_attend_merge(AttendArgs a) {
  const uint32_t item = blockIdx.x;
  const AttendItem it = attend_item(a, item);
  if (it.pages == 0) return;
  const int G = a.group, D = a.head_dim;
  const int n = (min(it.pages, a.n_pages) + a.part_pages - 1) / a.part_pages;
  for (int e = threadIdx.x; e < G * (D / 4); e += 256) {
    const int g = e / (D / 4), d = e % (D / 4) * 4;
    const size_t w0 = (size_t)item * a.parts * G + g;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float mm = kLowest, den = 0.f;
    for (int j0 = 0; j0 < n; j0 += 8) {  // (slots past the last part read it again and weigh nothing)
      f32x4 v[8];
      float2 ml[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const size_t w = w0 + (size_t)min(j0 + j, n - 1) * G;
        v[j] = *(const f32x4*)(a.part_acc + w * D + d);
        ml[j] = *(const float2*)(a.part_ml + 2 * w);
      }
      float top = mm;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
      const float r = mm == top ? 1.f : exp2f((mm - top) * a.scale_log2);
      mm = top;
      den *= r;
      o *= r;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float f = j0 + j < n ? exp2f((ml[j].x - mm) * a.scale_log2) : 0.f;
        if (j0 + j < n) {
          den += f * ml[j].y;
          o += f * v[j];
        }
      }
    }
    store_x4<BF16>(a, it, g, d, D, o / den);
  }
}

}  // namespace

// ------------------------------------------------------------------ launchers

hipError_t launch_append_rows(const AppendRowsArgs& a0, bool bf16, hipStream_t st, const Timing* tm) {
  AppendRowsArgs a = a0;
  const int unit = bf16 ? 8 : 4, nslot = (a.head_dim - (a.halves ? a.rot_dim / 2 : 0)) / unit;
  const int tasks = (a.n_tokens < kPage ? a.n_tokens : kPage) * a.n_q_heads * nslot;  // of a page, at most
  a.q_blocks = a.q ? (tasks + kAppendTasks - 1) / kAppendTasks : 0;
  const size_t blocks = (size_t)a.n_seqs * a.slots * a.n_layers * (2 + a.q_blocks);
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
    auto run = [&](auto two, auto four) {  // (by the 64-byte pieces of a page's codes)
      return go(a.sum_row <= 128 ? two : four, dim3((unsigned)groups), dim3(512), 0, st, t0(tm), t1(tm), a);
    };
    if (!score || pages <= 128) return run(k_page_pick<2, 2>, k_page_pick<2, 4>);
    if (pages <= 256) return run(k_page_pick<4, 2>, k_page_pick<4, 4>);
    return run(k_page_pick<8, 2>, k_page_pick<8, 4>);
  }
  const dim3 sgrid((unsigned)(groups * a.chunks));
  const hipError_t e = a.sum_row <= 128 ? go(k_page_score<2>, sgrid, dim3(256), 0, st, t0(tm), nullptr, a)
                                        : go(k_page_score<4>, sgrid, dim3(256), 0, st, t0(tm), nullptr, a);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)items);
  auto run = [&](auto kernel, int waves) { return go(kernel, grid, dim3(64 * waves), 0, st, nullptr, t1(tm), a); };
  // Few rows: 16 waves each, the sooner done; more than one per compute unit: 8, whose
  // passes cost half as much (see k_page_select).
  if (items > (size_t)a.num_cus && pages <= 8192) {
    if (pages <= 2048) return run(k_page_select<8, 4, false>, 8);
    if (pages <= 4096) return run(k_page_select<8, 8, false>, 8);
    return run(k_page_select<8, 16, false>, 8);
  }
  if (pages <= 2048) return run(k_page_select<16, 2, false>, 16);
  if (pages <= 4096) return run(k_page_select<16, 4, false>, 16);
  if (pages <= 8192) return run(k_page_select<16, 8, false>, 16);
  if (pages <= 16384) return run(k_page_select<16, 16, false>, 16);
  return run(k_page_select<16, 16, true>, 16);
}

hipError_t launch_attend(const AttendArgs& a0, bool pick, hipStream_t st, const Timing* tm, const Timing* tm_merge) {
  const size_t items = (size_t)a0.n_groups * a0.gt * a0.launch_layers * a0.n_kv_heads;
  AttendArgs a = a0;
  a.launch_seqs = (a.group0 + a.n_groups - 1) / a.seq_groups - a.group0 / a.seq_groups + 1;
  const size_t pairs = (size_t)a.launch_seqs * a.launch_layers * a.n_kv_heads;
  const size_t blocks = (a.n_tokens == 1 ? items : (pairs + 7) / 8 * 8 * a.seq_groups * a.gt) * a.parts;
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  hipError_t e = hipErrorInvalidValue;
  auto run = [&](auto kernel) { e = go(kernel, grid, dim3(256), 0, st, t0(tm), t1(tm), a); };
  auto pick_or_not = [&](auto yes, auto no) { pick ? run(yes) : run(no); };
  if (a.bf16) {
    if (a.head_dim == 128) pick_or_not(k_attend<true, 4, true>, k_attend<true, 4, false>);
    else if (a.head_dim == 64) pick_or_not(k_attend<true, 2, true>, k_attend<true, 2, false>);
  } else {
    switch ((a.head_dim + 15) / 16) {  // (head_dim <= 128)
      case 1: pick_or_not(k_attend<false, 1, true>, k_attend<false, 1, false>); break;
      case 2: pick_or_not(k_attend<false, 2, true>, k_attend<false, 2, false>); break;
      case 3: pick_or_not(k_attend<false, 3, true>, k_attend<false, 3, false>); break;
      case 4: pick_or_not(k_attend<false, 4, true>, k_attend<false, 4, false>); break;
      case 5: pick_or_not(k_attend<false, 5, true>, k_attend<false, 5, false>); break;
      case 6: pick_or_not(k_attend<false, 6, true>, k_attend<false, 6, false>); break;
      case 7: pick_or_not(k_attend<false, 7, true>, k_attend<false, 7, false>); break;
      case 8: pick_or_not(k_attend<false, 8, true>, k_attend<false, 8, false>); break;
    }
  }
  if (e != hipSuccess || a.parts == 1) return e;
  if (a.bf16) return go(k_attend_merge<true>, dim3((unsigned)items), dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a);
  return go(k_attend_merge<false>, dim3((unsigned)items), dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a);
}

}  // namespace pced
