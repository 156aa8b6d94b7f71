// gfx950 kernels of caches held in 8 bits: loading, attention, reading back. Codes: see
// pced_code8.h; appending: k_append8 in pced_layer.hip.
#include "pced_code8.h"
#include "pced_device.h"

namespace pced {
namespace {

typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));  // at any bf16's address

// ------------------------------------------------------------------- loading

struct TileUnit {
  int g, t, d;
};
// the kv-head, token and first dim of K unit n of a bf16 page
__device__ __forceinline__ TileUnit tile_unit(int n, int D) {
  const int u = n % (2 * D);
  return TileUnit{n / (2 * D), u & 15, 32 * (u >> 6) + 8 * ((u >> 4) & 3)};
}

// k_load's movement into a cache in 8 bits: one wave per (item, layer, 8 KiB of K and of V, which
// are the tiles of whole kv-heads). A wave that holds the units of a complete page's tiles
// encodes them; the units of a page behind the last complete one go to its place as they are, slots past
// the length zero-filled. Bound: HBM, 2 bytes read and 1 written per value.
template <int CODE, int D>
__global__ __launch_bounds__(256) void k_load8(LoadArgs a, Cache8Args c) {
  constexpr int NU = D / 32, HPW = 8 / NU;  // a tile's units per lane, kv-heads per wave
  __shared__ uint4 lds[4][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.n_kv_heads, units = Hkv * D * 2, nb = (units + 511) / 512;
  const int task = blockIdx.x * 4 + wave;
  const int item = task / nb, batch = task - item * nb, l = blockIdx.y;
  if (item >= a.n_items) return;
  const int s = a.items ? a.items[2 * item] : a.one_s, p = a.items ? a.items[2 * item + 1] : a.page0 + item;
  const int len = a.len0[s];
  const int phys = a.page_table[(size_t)s * a.maxpps + p];
  const char* sk = a.items ? (const char*)a.src_k[s] : (const char*)a.one_k;
  const char* sv = a.items ? (const char*)a.src_v[s] : (const char*)a.one_v;
  const int ld = a.items ? len : a.one_len, row0 = kPage * (a.items ? p : item);
  const int last = min(len - kPage * p, kPage) - 1;  // last token of the page
  const size_t src0 = ((size_t)l * ld + row0) * Hkv * D;
  const uint16_t* k16 = (const uint16_t*)sk + src0;
  const uint16_t* v16 = (const uint16_t*)sv + src0;
  const u32x4 zero = {0u, 0u, 0u, 0u};
  const int run = batch * 64 + lane;
  const RunPos rp = run_pos(min(run, units / 8 - 1), D);
  u32x4 ku[8], vv[4][2];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint16_t* row = v16 + ((size_t)min(4 * rp.q + t, last) * Hkv + rp.g) * D + rp.d0;
    vv[t][0] = *(const u32x4_a2*)row;
    vv[t][1] = *(const u32x4_a2*)(row + 16);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const TileUnit u = tile_unit(min(batch * 512 + 64 * i + lane, units - 1), D);
    ku[i] = *(const u32x4_a2*)(k16 + ((size_t)min(u.t, last) * Hkv + u.g) * D + u.d);
    if (u.t > last) ku[i] = zero;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (4 * rp.q + t > last) vv[t][0] = vv[t][1] = zero;
  uint4* mine = lds[wave];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    mine[lane * 8 + (i ^ (lane & 7))] =
        make_uint4(el16(vv[0][0], i) | (el16(vv[1][0], i) << 16), el16(vv[2][0], i) | (el16(vv[3][0], i) << 16),
                   el16(vv[0][1], i) | (el16(vv[1][1], i) << 16), el16(vv[2][1], i) | (el16(vv[3][1], i) << 16));
  wave_lds_sync();
  u32x4 vu[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int n = 64 * i + lane;
    vu[i] = __builtin_bit_cast(u32x4, mine[(n >> 3) * 8 + ((n & 7) ^ ((n >> 3) & 7))]);
  }
  const int layer = a.layer0 + l;
  if (last < kPage - 1) {
    const size_t at = ((size_t)layer * c.open_pages + s * c.ring + p % c.ring) * units + batch * 512 + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (batch * 512 + 64 * i + lane < units) {
        ((u32x4*)c.k_open)[at + 64 * i] = ku[i];
        ((u32x4*)c.v_open)[at + 64 * i] = vu[i];
      }
    return;
  }
#pragma unroll
  for (int hh = 0; hh < HPW; ++hh) {
    const int h = batch * HPW + hh;
    if (h >= Hkv) break;
    const size_t at = (((size_t)layer * c.max_pages + phys) * Hkv + h) * (NU / 2) * 64 + lane;
    u32x4 t[NU], w[NU / 2];
    uint32_t sk8, sv8;
#pragma unroll
    for (int i = 0; i < NU; ++i) t[i] = ku[hh * NU + i];
    encode_tile<CODE, NU>(t, w, &sk8);
#pragma unroll
    for (int i = 0; i < NU / 2; ++i) ((u32x4*)c.k_codes)[at + 64 * i] = w[i];
#pragma unroll
    for (int i = 0; i < NU; ++i) t[i] = vu[hh * NU + i];
    encode_tile<CODE, NU>(t, w, &sv8);
#pragma unroll
    for (int i = 0; i < NU / 2; ++i) ((u32x4*)c.v_codes)[at + 64 * i] = w[i];
    if (lane == 0) c.scales[((size_t)layer * Hkv + h) * c.max_pages + phys] = sk8 | sv8 << 16;
  }
}

// ----------------------------------------------------------------- attention

constexpr float kLowest8 = -3.402823466e38f;  // the softmax's first reference (see k_attend)

struct Item8 {
  int s, h, l, tok0, nt, len;  // nt new tokens from tok0 on; len: tokens before the call's
};
__device__ __forceinline__ Item8 item8(const Attend8Args& a, uint32_t item) {
  Item8 r;
  r.h = item % (uint32_t)a.n_kv_heads;
  item /= (uint32_t)a.n_kv_heads;
  r.l = 0;
  if (a.launch_layers > 1) {
    r.l = item % (uint32_t)a.launch_layers;
    item /= (uint32_t)a.launch_layers;
  }
  const uint32_t g = item + a.group0;
  r.s = g;
  r.tok0 = 0;
  if (a.seq_groups > 1) {
    r.s = g / (uint32_t)a.seq_groups;
    r.tok0 = (g - r.s * a.seq_groups) * a.gt;
  }
  r.nt = min(a.gt, a.n_tokens - r.tok0);
  r.len = a.len0[r.s] + a.t;
  return r;
}
// pages that an item's tokens see
__device__ __forceinline__ int pages8(const Item8& it) { return (it.len + it.tok0 + it.nt - 1) / kPage + 1; }

// Where query row (token i of the group, q-head g) begins in q and x, in elements
__device__ __forceinline__ size_t qrow8(const Attend8Args& a, const Item8& it, int i, int g, int D) {
  const size_t row = (size_t)it.s * a.n_tokens + it.tok0 + i;
  return ((row * a.n_layers + a.layer - a.layer0 + it.l) * a.n_q_heads + (size_t)it.h * a.group + g) * D;
}
__device__ __forceinline__ void store_x4_bf16(void* x, size_t at, f32x4 o) {
  const bf16x2 p = {(__bf16)o[0], (__bf16)o[1]}, q = {(__bf16)o[2], (__bf16)o[3]};
  *(uint2*)((uint16_t*)x + at) = make_uint2(__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q));
}

__device__ __forceinline__ bf16x8 join8(uint2 a, uint2 b) { return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y}); }

// One block of 4 waves per (item, part of its pages): as k_attend, but the columns of both
// products are the q-heads of a kv-head for up to 16 NC / G new tokens, so that those share
// a page's way into registers, and the pages come as codes: a page's K product is summed over
// codes and then scaled, its softmax weights are scaled by V's scale before they meet V's codes. Codes
// are exact in bf16, so nothing is rounded on the way that k_attend does not round.
// The pages that were complete before the call lie before every new token: no mask. The pages
// behind them are 16-bit tiles, one at a time, masked by each column's own position. There, V of tokens behind
// the group's last counts as 0 (unwritten rows hold anything); V of the group's own later
// tokens is written, but may be inf or NaN, whose product with a weight of 0 is not 0: if it is,
// the page is taken token by token.
template <int CODE, int D, int NC>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NC == 1 ? 2 : 1, 4))) void k_attend8(Attend8Args a) {
  constexpr int NU = D / 32, NW = D / 64, NJ = D / 16;  // 16-bit units, code units, 16-dim output blocks
  constexpr int DP = D + 4;
  __shared__ __align__(16) float sacc[4][16 * NC][DP];
  __shared__ float sm[4][16 * NC], sl[4][16 * NC];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  // Work-groups go to the eight dies in turn. The token groups of one (sequence, layer, kv-head) go to
  // one die and follow each other there: its L2 then has the pages.
  uint32_t item, part;
  if (a.seq_groups == 1) {
    item = blockIdx.x / (uint32_t)a.parts;
    part = blockIdx.x - item * a.parts;
  } else {
    const uint32_t s0 = (uint32_t)a.group0 / a.seq_groups, per = (uint32_t)a.seq_groups * a.parts;
    const uint32_t r = blockIdx.x >> 3, k = r / per, rest = r - k * per;
    const uint32_t pair = (blockIdx.x & 7) + 8 * k;  // (layer, kv-head, sequence)
    const uint32_t heads = (uint32_t)a.launch_layers * a.n_kv_heads;
    const uint32_t lh = pair / a.launch_seqs, s = pair - lh * a.launch_seqs;
    part = rest / a.seq_groups;
    const uint32_t i = rest - part * a.seq_groups, g = (s0 + s) * a.seq_groups + i - a.group0;
    if (lh >= heads || g >= (uint32_t)a.n_groups) return;
    item = g * heads + lh;
  }
  const Item8 it = item8(a, item);
  const int total = pages8(it), full = it.len / kPage;
  const int c0 = part * a.part_pages, c1 = min(total, c0 + a.part_pages);
  if (c0 >= c1) return;
  const int G = a.group, cols = it.nt * G;
  const int layer = a.layer + it.l;
  const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
  const int cnt = min(c1, full) - c0;  // pages of codes (<= 0: none)
  // the wave's u-th page of codes is page u / 2 * 8 + 2 wave + u % 2 of the part; ids and scales one per lane
  const int my_page = c0 + min(lane / 2 * 8 + 2 * wave + lane % 2, max(cnt, 1) - 1);
  const int my_phys = max(pt[my_page], 0);
  const uint32_t my_scale = cnt > 0 ? a.c.scales[((size_t)layer * a.n_kv_heads + it.h) * a.c.max_pages + my_phys] : 0u;
  u32x4 q[NC][NU];
  int lim[NC];  // the column's own position
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int cc = min(16 * n + col, cols - 1), i = cc / G;
    const uint16_t* row = (const uint16_t*)a.q + qrow8(a, it, i, cc - i * G, D) + 8 * quad;
    lim[n] = it.len + it.tok0 + i;
#pragma unroll
    for (int u = 0; u < NU; ++u) q[n][u] = *(const u32x4*)(row + 32 * u);
  }
  f32x4 acc[NC][NJ];
  float m[NC], lsum[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = kLowest8;
    lsum[n] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // moves column tile n's reference where a score exceeds it by `lead`
  auto refer = [&](int n, float top) __attribute__((always_inline)) {
    if (__any(top > m[n] + a.lead)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m[n], top), alpha = m[n] == mn ? 1.f : __builtin_amdgcn_exp2f((m[n] - mn) * a.scale_log2);
      m[n] = mn;
      lsum[n] *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[n][j] *= alpha;
    }
  };

  // ------------------------------------------------ pages of codes, two at a time
  struct Regs {
    u32x4 k[2][NW], v[2][NW];
  };
  const size_t tile = (size_t)kPage * D;
  auto load = [&](int u, Regs& r) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const size_t at = (((size_t)layer * a.c.max_pages + __builtin_amdgcn_readlane(my_phys, u + b)) * a.n_kv_heads + it.h) * tile;
      const u32x4* kp = (const u32x4*)(a.c.k_codes + at) + lane;
      const u32x4* vp = (const u32x4*)(a.c.v_codes + at) + lane;
#pragma unroll
      for (int j = 0; j < NW; ++j) r.k[b][j] = kp[64 * j];
#pragma unroll
      for (int j = 0; j < NW; ++j) r.v[b][j] = vp[64 * j];
    }
  };
  auto work = [&](int i, Regs& r) __attribute__((always_inline)) {
    const int u = 2 * i, k0 = 2 * wave + 8 * i;  // first page in lanes, and in the part
    f32x4 sc[2][NC];
    float vs[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t s2 = (uint32_t)__builtin_amdgcn_readlane((int)my_scale, u + b);
      const float ks = bf2f(s2 & 0xFFFFu);
      vs[b] = bf2f(s2 >> 16);
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NU; ++x) {
        const u32x4& w = r.k[b][x >> 1];
        const bf16x8 kk = join8(decode4<CODE>(w[2 * (x & 1)]), decode4<CODE>(w[2 * (x & 1) + 1]));
#pragma unroll
        for (int n = 0; n < NC; ++n)
          sc[b][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, __builtin_bit_cast(bf16x8, q[n][x]), sc[b][n], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[b][n] *= ks;
    }
    if (k0 + 1 >= cnt) {  // uniform: the batch's second slot is past the part's pages
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[1][n] = f32x4{kNegInf, kNegInf, kNegInf, kNegInf};
    }
    bf16x8 hi[NC], lo[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float top = kNegInf;
#pragma unroll
      for (int b = 0; b < 2; ++b) top = fmaxf(top, fmaxf(fmaxf(sc[b][n][0], sc[b][n][1]), fmaxf(sc[b][n][2], sc[b][n][3])));
      refer(n, top);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f((sc[b][n][e] - m[n]) * a.scale_log2);
        lsum[n] += (p[0] + p[1]) + (p[2] + p[3]);
        // a weight goes in as the sum of two bf16 (relative error 2^-17; the matrix cores are idle anyway)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = p[e] * vs[b];
          hi[n][4 * b + e] = (__bf16)x;
          lo[n][4 * b + e] = (__bf16)(x - (float)hi[n][4 * b + e]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const bf16x8 vv = join8(decode4<CODE>(r.v[0][j >> 2][j & 3]), decode4<CODE>(r.v[1][j >> 2][j & 3]));
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, hi[n], acc[n][j], 0, 0, 0);
        acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, lo[n], acc[n][j], 0, 0, 0);
      }
    }
  };
  if (cnt > 2 * wave) {
    const int nb = (cnt - 2 * wave + 7) / 8;
    Regs ra, rb;
    load(0, ra);
    int i = 0;
    for (; i + 2 < nb; i += 2) {
      load(2 * (i + 1), rb);
      work(i, ra);
      load(2 * (i + 2), ra);
      work(i + 1, rb);
    }
    if (nb - i == 2) {
      load(2 * (i + 1), rb);
      work(i, ra);
      work(i + 1, rb);
    } else {
      work(i, ra);
    }
  }

  // --------------------------------- the pages behind, one at a time, in 16 bits
  for (int p = max(c0, full) + wave; p < c1; p += 4) {
    const size_t at = (((size_t)layer * a.c.open_pages + it.s * a.c.ring + p % a.c.ring) * a.n_kv_heads + it.h) * tile;
    const u32x4* kp = (const u32x4*)(a.c.k_open + at) + lane;
    const u32x4* vp = (const u32x4*)(a.c.v_open + at) + lane;
    u32x4 k[NU], v[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) { k[u] = kp[64 * u]; v[u] = vp[64 * u]; }
    const int t0 = kPage * p + 4 * quad;  // the lane's first token
    // keeps V's tokens up to position `end`
    auto keep = [&](u32x4 (&w)[NU], int end) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t mask = t0 + e <= end ? 0xFFFFFFFFu : ~(0xFFFFu << (16 * (e & 1)));
#pragma unroll
        for (int u = 0; u < NU; ++u) { w[u][e >> 1] &= mask; w[u][2 + (e >> 1)] &= mask; }
      }
    };
    const int first = it.len + it.tok0, end = first + it.nt - 1;
    keep(v, end);
    bool odd = false;  // some inf or NaN that not all of the group's tokens see
    if (kPage * p + kPage - 1 > first) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) odd |= t0 + (e & 3) > first && (el16(v[u], e) & 0x7F80u) == 0x7F80u;
      odd = __any(odd);
    }
    s16x4 hi[NC], lo[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < NU; ++u)
        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[u]), __builtin_bit_cast(bf16x8, q[n][u]), sc, 0, 0, 0);
      float top = kNegInf;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (t0 + e > lim[n]) sc[e] = kNegInf;
        top = fmaxf(top, sc[e]);
      }
      refer(n, top);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f((sc[e] - m[n]) * a.scale_log2);
        lsum[n] += x;
        const __bf16 h = (__bf16)x;
        hi[n][e] = __builtin_bit_cast(short, h);
        lo[n][e] = __builtin_bit_cast(short, (__bf16)(x - (float)h));
      }
    }
    auto tokens4 = [](const u32x4& w, int half) { return __builtin_bit_cast(s16x4, half ? make_uint2(w[2], w[3]) : make_uint2(w[0], w[1])); };
    if (!odd) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const s16x4 vv = tokens4(v[j >> 1], j & 1);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, hi[n], acc[n][j], 0, 0, 0);
          acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, lo[n], acc[n][j], 0, 0, 0);
        }
      }
    } else {
      for (int i = 0; i < it.nt; ++i) {  // each token's columns see V up to it
        u32x4 w[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u) w[u] = v[u];
        keep(w, first + i);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const s16x4 vv = tokens4(w[j >> 1], j & 1);
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            f32x4 o = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, hi[n], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, lo[n], o, 0, 0, 0);
            if (lim[n] == first + i) acc[n][j] += o;
          }
        }
      }
    }
  }

  // -------------------------------------------------------- the waves' states
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    lsum[n] += __shfl_xor(lsum[n], 16);
    lsum[n] += __shfl_xor(lsum[n], 32);
    const int cc = 16 * n + col;
    if (cc < cols) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)&sacc[wave][cc][16 * j + 4 * quad] = acc[n][j];
      if (quad == 0) { sm[wave][cc] = m[n]; sl[wave][cc] = lsum[n]; }
    }
  }
  __syncthreads();
  for (int e = tid; e < cols * (D / 4); e += 256) {
    const int cc = e / (D / 4), d = e % (D / 4) * 4;
    float mm = sm[0][cc];
#pragma unroll
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, sm[w][cc]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2f((sm[w][cc] - mm) * a.scale_log2);  // (a wave without pages: l = 0 and m = kLowest8)
      den += f * sl[w][cc];
      o += f * *(const f32x4*)&sacc[w][cc][d];
    }
    if (a.parts == 1) {
      const int i = cc / G;
      store_x4_bf16(a.x_out, qrow8(a, it, i, cc - i * G, D) + d, o / den);
    } else {
      const size_t w = ((size_t)item * a.parts + part) * (a.gt * G) + cc;
      *(f32x4*)(a.part_acc + w * D + d) = o;
      if (d == 0) *(float2*)(a.part_ml + 2 * w) = make_float2(mm, den);
    }
  }
}

// The merge of an item's parts (see k_attend_merge), a block per item and 1024 of its outputs
__global__ __launch_bounds__(256) void k_attend8_merge(Attend8Args a) {
  const uint32_t item = blockIdx.x;
  const Item8 it = item8(a, item);
  const int G = a.group, D = a.head_dim, stride = a.gt * G;
  const int n = (pages8(it) + a.part_pages - 1) / a.part_pages;
  const int e = blockIdx.y * 256 + threadIdx.x;
  const int cc = e / (D / 4), d = e % (D / 4) * 4;
  if (cc >= it.nt * G) return;
  const size_t w0 = (size_t)item * a.parts * stride + cc;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float mm = kLowest8, den = 0.f;
  for (int j0 = 0; j0 < n; j0 += 8) {  // (slots past the last part read it again and weigh nothing)
    f32x4 v[8];
    float2 ml[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const size_t w = w0 + (size_t)min(j0 + j, n - 1) * stride;
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
    for (int j = 0; j < 8; ++j)
      if (j0 + j < n) {
        const float f = exp2f((ml[j].x - mm) * a.scale_log2);
        den += f * ml[j].y;
        o += f * v[j];
      }
  }
  const int i = cc / G;
  store_x4_bf16(a.x_out, qrow8(a, it, i, cc - i * G, D) + d, o / den);
}

// ------------------------------------------------------------- reading back

// Tokens [start, start + count) of a sequence and layer as bf16 rows [count][Hkv][D]: codes times their
// scale, rounded once; the tokens behind the complete pages as they are. A thread per 8 dims of a
// token's K or V row: the units of a tile that hold them are 8 bytes (K) or 8 dims' single bytes (V).
__global__ __launch_bounds__(256) void k_read8(ReadCacheArgs a, Cache8Args c, int len) {
  const int Hkv = a.n_kv_heads, D = a.head_dim, oct = D / 8;
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x, per = (size_t)Hkv * oct;
  if (e >= 2 * per * a.count) return;
  const bool is_v = e >= per * a.count;
  const size_t x = is_v ? e - per * a.count : e;
  const int i = (int)(x / per), r = (int)(x - (size_t)i * per), h = r / oct, d = r % oct * 8;
  const int tok = a.start + i, p = tok / kPage, t = tok % kPage;
  uint32_t o[4];
  if (p >= len / kPage) {
    const size_t at = (((size_t)a.layer * c.open_pages + a.seq * c.ring + p % c.ring) * Hkv + h) * kPage * D;
    const uint16_t* tile = (is_v ? c.v_open : c.k_open) + at;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      o[w] = is_v ? tile[vswz(t, d + 2 * w)] | (uint32_t)tile[vswz(t, d + 2 * w + 1)] << 16
                  : *(const uint32_t*)(tile + kswz(t, d) + 2 * w);
  } else {
    const int phys = a.page_table[(size_t)a.seq * a.maxpps + p];
    const size_t at = (((size_t)a.layer * c.max_pages + phys) * Hkv + h) * kPage * D;
    const uint32_t s2 = c.scales[((size_t)a.layer * Hkv + h) * c.max_pages + phys];
    const float s = bf2f(is_v ? s2 >> 16 : s2 & 0xFFFFu);
    const uint8_t* tile = (is_v ? c.v_codes : c.k_codes) + at;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t two = 0;  // two codes
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int dd = d + 2 * w + b;
        const int place = is_v ? ((dd >> 6) * 64 + (dd & 15) + 16 * (t >> 2)) * 16 + ((dd & 63) >> 4) * 4 + (t & 3)
                               : ((dd >> 6) * 64 + t + 16 * ((dd & 31) >> 3)) * 16 + ((dd & 63) >> 5) * 8 + (dd & 7);
        two |= (uint32_t)tile[place] << (8 * b);
      }
      const uint32_t y = c.code == kE4m3 ? decode4<kE4m3>(two).x : decode4<kInt8>(two).x;
      const bf16x2 z = {(__bf16)(bf2f(y & 0xFFFFu) * s), (__bf16)(bf2f(y >> 16) * s)};
      o[w] = __builtin_bit_cast(uint32_t, z);
    }
  }
  uint16_t* out = (uint16_t*)(is_v ? a.v_out : a.k_out) + ((size_t)i * Hkv + h) * D + d;
  *(u32x4_a2*)out = u32x4{o[0], o[1], o[2], o[3]};
}

}  // namespace

// ------------------------------------------------------------------ launchers

hipError_t launch_load8(const LoadArgs& a0, const Cache8Args& c, int n_items, hipStream_t st) {
  LoadArgs a = a0;
  a.n_items = n_items;
  const long tasks = (long)n_items * ((a.n_kv_heads * a.head_dim * 2 + 511) / 512);
  if ((tasks + 3) / 4 > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 g((unsigned)((tasks + 3) / 4), a.n_layers);
  auto run = [&](auto kernel) { return go(kernel, g, dim3(256), 0, st, nullptr, nullptr, a, c); };
  if (a.head_dim == 128) return c.code == kE4m3 ? run(k_load8<kE4m3, 128>) : run(k_load8<kInt8, 128>);
  return c.code == kE4m3 ? run(k_load8<kE4m3, 64>) : run(k_load8<kInt8, 64>);
}

hipError_t launch_attend8(const Attend8Args& a0, hipStream_t st, const Timing* tm, const Timing* tm_merge) {
  Attend8Args a = a0;
  const size_t items = (size_t)a.n_groups * a.launch_layers * a.n_kv_heads;
  a.launch_seqs = (a.group0 + a.n_groups - 1) / a.seq_groups - a.group0 / a.seq_groups + 1;
  const size_t pairs = (size_t)a.launch_seqs * a.launch_layers * a.n_kv_heads;
  const size_t blocks = (a.seq_groups == 1 ? items : (pairs + 7) / 8 * 8 * a.seq_groups) * a.parts;
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  auto run = [&](auto kernel) { return go(kernel, dim3((unsigned)blocks), dim3(256), 0, st, t0(tm), t1(tm), a); };
  auto tiles = [&](auto one, auto two) { return a.tiles == 1 ? run(one) : run(two); };
  hipError_t e;
  if (a.head_dim == 128) {
    e = a.c.code == kE4m3 ? tiles(k_attend8<kE4m3, 128, 1>, k_attend8<kE4m3, 128, 2>)
                          : tiles(k_attend8<kInt8, 128, 1>, k_attend8<kInt8, 128, 2>);
  } else {
    e = a.c.code == kE4m3 ? tiles(k_attend8<kE4m3, 64, 1>, k_attend8<kE4m3, 64, 2>)
                          : tiles(k_attend8<kInt8, 64, 1>, k_attend8<kInt8, 64, 2>);
  }
  if (e != hipSuccess || a.parts == 1) return e;
  const dim3 grid((unsigned)items, (a.gt * a.group * (a.head_dim / 4) + 255) / 256);
  return go(k_attend8_merge, grid, dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a);
}

hipError_t launch_read8(const ReadCacheArgs& a, const Cache8Args& c, int len, hipStream_t st) {
  const size_t tasks = (size_t)a.count * a.n_kv_heads * (a.head_dim / 8) * 2;
  if ((tasks + 255) / 256 > 0x7FFFFFFFu) return hipErrorInvalidValue;
  return go(k_read8, dim3((unsigned)((tasks + 255) / 256)), dim3(256), 0, st, nullptr, nullptr, a, c, len);
}

}  // namespace pced
