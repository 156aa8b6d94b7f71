// gfx950 kernels of caches held in 8 bits: loading, attention, reading back. Codes: see
// pced_code8.h; appending: k_append8 in pced_layer.hip.
#include "pced_code8.h"
#include "pced_device.h"

#include <type_traits>

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
// the length zero-filled. Bound: HBM, 2 bytes read and 1 written per value (16 layers of 33 sequences, 8 heads of 128:
// 750 us for 4.0 GB, 5.4 TB/s; a copy reaches 4.9).
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
// group i of sequence s, and the (layer, kv-head) number lh of the launch
__device__ __forceinline__ Item8 item8(const Attend8Args& a, int s, int i, uint32_t lh) {
  Item8 r;
  r.s = s;
  r.l = 0;
  r.h = lh;
  if (a.launch_layers > 1) {
    r.l = lh / (uint32_t)a.n_kv_heads;
    r.h = lh - r.l * a.n_kv_heads;
  }
  r.tok0 = i * a.gt;
  r.nt = min(a.gt, a.n_tokens - r.tok0);
  r.len = a.len0[s] + a.t;
  return r;
}
// pages that an item's tokens see
__device__ __forceinline__ int pages8(const Item8& it) { return (it.len + it.tok0 + it.nt - 1) / kPage + 1; }
// pages of a part of sequence s: as few parts as a.part_pages allows, of equal length
__device__ __forceinline__ int part8(const Attend8Args& a, int s) {
  const int pages = (a.len0[s] + a.t + a.n_tokens - 1) / kPage + 1, n = (pages + a.part_pages - 1) / a.part_pages;
  return (pages + n - 1) / n;
}

// The item and part of a block. Only parts that some token sees have blocks: the sequences' lengths are far
// apart, and blocks without work would take turns with the others and leave the eight dies uneven shares. A wave
// counts the sequences' parts, 64 sequences at a time, up to the block's. Work-groups go to the dies in turn; the
// token groups of one (sequence, part, layer, kv-head) go to one die and follow each other there, so that its L2 has
// their pages.
__device__ __forceinline__ bool block8(const Attend8Args& a, Item8& it, uint32_t& item, int& part) {
  const int lane = threadIdx.x & 63;
  const uint32_t heads = (uint32_t)a.launch_layers * a.n_kv_heads;
  uint32_t u = blockIdx.x, i = 0;
  if (a.n_groups > 1) {
    const uint32_t r = u >> 3, k = r / (uint32_t)a.n_groups;
    i = r - k * a.n_groups;
    u = (u & 7) + 8 * k;
  }
  const uint32_t sp = u / heads, lh = u - sp * heads;
  if (sp >= (uint32_t)a.seq_parts) return false;
  int s = sp, before = 0;
  part = 0;
  for (int base = 0; a.seq_parts > a.launch_seqs; base += 64) {  // (sp is below the sum of all)
    int n = 0;
    if (base + lane < a.launch_seqs) {
      const int pages = (a.len0[a.seq0 + base + lane] + a.t + a.n_tokens - 1) / kPage + 1;
      n = (pages + a.part_pages - 1) / a.part_pages;
    }
    int run = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(run, o); if (lane >= o) run += x; }
    const uint64_t past = __ballot((int)sp < before + run);
    if (past) {
      const int at = __builtin_ctzll(past);
      s = base + at;
      part = (int)sp - before - __builtin_amdgcn_readlane(run, at) + __builtin_amdgcn_readlane(n, at);
      break;
    }
    before += __builtin_amdgcn_readlane(run, 63);
  }
  item = ((uint32_t)s * a.n_groups + i) * heads + lh;
  it = item8(a, a.seq0 + s, a.group0 + i, lh);
  return true;
}

// Where query row (token i of the group, q-head g) begins in q and x, in elements
__device__ __forceinline__ size_t qrow8(const Attend8Args& a, const Item8& it, int i, int g, int D) {
  const size_t row = (size_t)it.s * a.n_tokens + it.tok0 + i;
  return ((row * a.n_layers + a.layer - a.layer0 + it.l) * a.n_q_heads + (size_t)it.h * a.group + g) * D;
}
__device__ __forceinline__ void store_x4_bf16(void* x, size_t at, f32x4 o) {
  const bf16x2 p = {(__bf16)o[0], (__bf16)o[1]}, q = {(__bf16)o[2], (__bf16)o[3]};
  *(uint2*)((uint16_t*)x + at) = make_uint2(__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q));
}

__device__ __forceinline__ float lane_f(float x, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

__device__ __forceinline__ bf16x8 join8(uint2 a, uint2 b) { return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y}); }

// Two pages' weights as the sum of two bf16 each: relative 2^-17, with fp32's exponent
struct Weights8 {
  bf16x8 hi, lo;
};

// A wave's part of an item: NC tiles of 16 columns (a column is a q-head of one of the group's new tokens), each
// with an online softmax. As in k_attend the products are
//   S^T[16 tok x 16 cols] = K[16 x D] Q^T,   O^T[D x 16 cols] += V^T[D x tok] P^T,
// and the softmax's reference (in log2 units) moves only when a score exceeds it by 8, so that weights stay within
// 2^8. Codes are exact in bf16: a page's K product is summed over codes and scaled behind; its softmax weights are
// scaled by V's scale and meet V's codes as the sum of two bf16, which hold any weight and scale of fp32 to 2^-17, however
// far apart the pages' scales lie. (In fp16, which holds neither, with half the products of V: a question of 24 tokens
// 85 us instead of 98, a token over 33 sequences 18.1 instead of 19.1, and no difference over longer caches.)
template <int D, int NC>
struct Columns {
  static constexpr int NU = D / 32, NJ = D / 16;  // 16-byte units of a bf16 tile per lane, 16-dim output blocks
  u32x4 q[NC][NU];
  f32x4 acc[NC][NJ];
  float m[NC], lsum[NC];
  int lim[NC];  // the column's own position
  __device__ __forceinline__ void begin(const Attend8Args& a, const Item8& it) {
    const int col = threadIdx.x & 15, quad = (threadIdx.x & 63) >> 4, G = a.group;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int cc = min(16 * n + col, it.nt * G - 1), i = cc / G;
      const uint16_t* row = (const uint16_t*)a.q + qrow8(a, it, i, cc - i * G, D) + 8 * quad;
      lim[n] = it.len + it.tok0 + i;
#pragma unroll
      for (int u = 0; u < NU; ++u) q[n][u] = *(const u32x4*)(row + 32 * u);
      m[n] = kLowest8;
      lsum[n] = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void refer(int n, float top) {
    if (__any(top > m[n] + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m[n], top), alpha = m[n] == mn ? 1.f : __builtin_amdgcn_exp2f(m[n] - mn);
      m[n] = mn;
      lsum[n] *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[n][j] *= alpha;
    }
  }
  // tile n's weights for two pages' scores (sums over codes), times V's scales
  __device__ __forceinline__ Weights8 weights(int n, const f32x4 (&sc)[2], const float (&kc)[2], const float (&vs)[2]) {
    float top = kNegInf;
#pragma unroll
    for (int b = 0; b < 2; ++b) top = fmaxf(top, kc[b] * fmaxf(fmaxf(sc[b][0], sc[b][1]), fmaxf(sc[b][2], sc[b][3])));
    refer(n, top);
    Weights8 w;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][e], kc[b], -m[n]));
      lsum[n] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = p[e] * vs[b];
        w.hi[4 * b + e] = (__bf16)x;
        w.lo[4 * b + e] = (__bf16)(x - (float)w.hi[4 * b + e]);
      }
    }
    return w;
  }
  __device__ __forceinline__ void unscale(float f) {
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[n][j] *= f;
  }
  // A page behind the complete ones: a 16-bit tile, masked by each column's own position. V of tokens behind the
  // group's last counts as 0 (unwritten rows hold anything). V that is inf or NaN is kept out of the products, where
  // columns that do not see it would get 0 times it, and those that do its products with two bf16, one of which may be 0 or
  // negative: the columns that see it get it one by one, times the whole weight.
  __device__ __forceinline__ void open_page(const Attend8Args& a, const Item8& it, int p) {
    const int lane = threadIdx.x & 63, quad = lane >> 4;
    const size_t at = (((size_t)(a.layer + it.l) * a.c.open_pages + it.s * a.c.ring + p % a.c.ring) * a.n_kv_heads + it.h) *
                      (size_t)(kPage * D);
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
    const int end = it.len + it.tok0 + it.nt - 1;
    keep(v, end);
    // inf and NaN: out, and in again where they are seen
    bool odd = false;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool bad = (el16(v[u], e) & 0x7F80u) == 0x7F80u;
        odd |= bad;
        if (bad) v[u][e >> 1] &= ~(0xFFFFu << (16 * (e & 1)));
      }
    odd = __any(odd);
    float x[NC][4];
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
        sc[e] = t0 + e > lim[n] ? kNegInf : sc[e] * a.scale_log2;
        top = fmaxf(top, sc[e]);
      }
      refer(n, top);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[n][e] = __builtin_amdgcn_exp2f(sc[e] - m[n]);
        lsum[n] += x[n][e];
        const __bf16 h = (__bf16)x[n][e];
        hi[n][e] = __builtin_bit_cast(short, h);
        lo[n][e] = __builtin_bit_cast(short, (__bf16)(x[n][e] - (float)h));
      }
    }
    auto tokens4 = [](const u32x4& w, int half) { return __builtin_bit_cast(s16x4, half ? make_uint2(w[2], w[3]) : make_uint2(w[0], w[1])); };
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const s16x4 vv = tokens4(v[j >> 1], j & 1);
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, hi[n], acc[n][j], 0, 0, 0);
        acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, lo[n], acc[n][j], 0, 0, 0);
      }
    }
    if (!odd) return;
    const uint16_t* tile = (const uint16_t*)a.c.v_open + at;
#pragma unroll 1
    for (int t = 0; t < kPage && kPage * p + t <= end; ++t) {
      const int from = (lane & 15) + 16 * (t >> 2);  // where the token's weights are
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const float mine = (t & 3) == 0 ? x[n][0] : (t & 3) == 1 ? x[n][1] : (t & 3) == 2 ? x[n][2] : x[n][3];
        const float w = __shfl(mine, from);
        const bool sees = kPage * p + t <= lim[n];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = tile[vswz(t, 16 * j + 4 * quad + e)];
            acc[n][j][e] += sees && (y & 0x7F80u) == 0x7F80u ? w * bf2f(y) : 0.f;
          }
      }
    }
  }
  __device__ __forceinline__ void sum(int n) {
    lsum[n] += __shfl_xor(lsum[n], 16);
    lsum[n] += __shfl_xor(lsum[n], 32);
  }
};

// One block of W waves per (item, part of its pages), whose waves take pairs of pages in turn, all columns each, and
// are merged in LDS. The pages that were complete before the call lie before every new token: no mask. A wave holds
// the ids and scales of its pages one per lane and loads a pair of pages while it works on the one before.
// Bound: HBM for a token (33 sequences, 16 layers of 8 heads: 233 us, 5.9 TB/s, as much as a plain read of memory
// reaches; a layer of it, int8, 19.1 us, half of which is the launch, a first page and the merge of the waves; 8 books of
// up to 131 072 tokens and their query: 215 us); for a question of 24 tokens (17 sequences of 5000, int8, 7 heads
// each: 98 us) the instructions of decoding, softmax and products, which a SIMD issues one after another.
template <int CODE, int D, int NC, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2, 4))) void k_attend8(Attend8Args a) {
  constexpr int NU = D / 32, NW = D / 64, NJ = D / 16;  // 16-bit units, code units, 16-dim output blocks
  constexpr int DP = D + 4;
  __shared__ __align__(16) float sacc[W][16 * NC][DP];
  __shared__ float sm[W][16 * NC], sl[W][16 * NC];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  uint32_t item;
  int part;
  Item8 it;
  if (!block8(a, it, item, part)) return;
  const int total = pages8(it), full = it.len / kPage;
  const int size = part8(a, it.s), c0 = part * size, c1 = min(total, c0 + size);
  if (c0 >= c1) return;
  const int G = a.group, cols = it.nt * G;
  const int layer = a.layer + it.l;
  const int32_t* pt = a.page_table + (size_t)it.s * a.maxpps;
  const int cnt = min(c1, full) - c0;  // pages of codes (<= 0: none)
  // the wave's u-th page of codes is page u / 2 * 2 W + 2 wave + u % 2 of the part; ids and scales one per lane
  const int my_page = c0 + min(lane / 2 * (2 * W) + 2 * wave + lane % 2, max(cnt, 1) - 1);
  const int my_phys = max(pt[my_page], 0);
  const uint32_t my_scale = cnt > 0 ? a.c.scales[((size_t)layer * a.n_kv_heads + it.h) * a.c.max_pages + my_phys] : 0u;
  Columns<D, NC> C;
  C.begin(a, it);
  struct Regs {
    u32x4 k[2][NW], v[2][NW];
  };
  // A wave's 1024 tokens with weights up to 2^8 and codes up to 448 reach 2^27 times the largest V scale: from 2^100 on
  // all are held 2^18 smaller, so that the sums stay finite until the end.
  const bool vast = __any((my_scale >> 16) >= 0x7180u);
  const float my_kc = bf2f(my_scale & 0xFFFFu) * a.scale_log2, my_vs = bf2f(my_scale >> 16) * (vast ? 0x1p-18f : 1.f);
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
    const int u = 2 * i, k0 = 2 * wave + 2 * W * i;  // first page in lanes, and in the part
    f32x4 sc[NC][2];
    float kc[2], vs[2];  // a page's scales: K's with log2(e) / sqrt(D), V's
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      kc[b] = lane_f(my_kc, u + b);
      vs[b] = lane_f(my_vs, u + b);
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NU; ++x) {
        const u32x4& w = r.k[b][x >> 1];
        const bf16x8 kk = join8(decode4<CODE>(w[2 * (x & 1)]), decode4<CODE>(w[2 * (x & 1) + 1]));
#pragma unroll
        for (int n = 0; n < NC; ++n)
          sc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, __builtin_bit_cast(bf16x8, C.q[n][x]), sc[n][b], 0, 0, 0);
      }
    }
    if (k0 + 1 >= cnt) {  // uniform: the pair's second slot is past the part's pages
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[n][1] = f32x4{kNegInf, kNegInf, kNegInf, kNegInf};
    }
    Weights8 wt[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) wt[n] = C.weights(n, sc[n], kc, vs);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const bf16x8 vv = join8(decode4<CODE>(r.v[0][j >> 2][j & 3]), decode4<CODE>(r.v[1][j >> 2][j & 3]));
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        C.acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, wt[n].hi, C.acc[n][j], 0, 0, 0);
        C.acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, wt[n].lo, C.acc[n][j], 0, 0, 0);
      }
    }
  };
  if (cnt > 2 * wave) {
    const int nb = (cnt - 2 * wave + 2 * W - 1) / (2 * W);
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
    if (vast) C.unscale(0x1p18f);
  }
#pragma unroll 1
  for (int p = max(c0, full) + wave; p < c1; p += W) C.open_page(a, it, p);
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    C.sum(n);
    const int cc = 16 * n + col;
    if (cc < cols) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)&sacc[wave][cc][16 * j + 4 * quad] = C.acc[n][j];
      if (quad == 0) { sm[wave][cc] = C.m[n]; sl[wave][cc] = C.lsum[n]; }
    }
  }
  __syncthreads();
  for (int e = tid; e < cols * (D / 4); e += 64 * W) {
    const int cc = e / (D / 4), d = e % (D / 4) * 4;
    float mm = sm[0][cc];
#pragma unroll
    for (int w = 1; w < W; ++w) mm = fmaxf(mm, sm[w][cc]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2f(sm[w][cc] - mm);  // (a wave without pages: l = 0 and m = kLowest8)
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

// The merge of an item's parts (see k_attend_merge): a block per item and 8 of its columns, of each of which a
// wave takes half, or (SPREAD: many parts, few columns) a block per column, whose 256 / (D / 4) groups of threads take the
// parts in turn and meet in LDS. Bound: the launch and one way to the states (288 columns of up to 32 parts 5.3 us; 11424 of
// two, 10 MB, 6.8).
template <bool SPREAD>
__global__ __launch_bounds__(256) void k_attend8_merge(Attend8Args a) {
  __shared__ f32x4 so[SPREAD ? 256 : 1];
  __shared__ float2 sml[SPREAD ? 256 : 1];
  const uint32_t item = blockIdx.x, heads = (uint32_t)a.launch_layers * a.n_kv_heads;
  const uint32_t g = item / heads, s = g / (uint32_t)a.n_groups;
  const Item8 it = item8(a, a.seq0 + s, a.group0 + g - s * a.n_groups, item - g * heads);
  const int G = a.group, D = a.head_dim, stride = a.gt * G, lanes = D / 4, groups = 256 / lanes;
  const int size = part8(a, it.s), n = (pages8(it) + size - 1) / size;
  const int grp = threadIdx.x / lanes, d = threadIdx.x % lanes * 4;
  const int cc = SPREAD ? blockIdx.y : blockIdx.y * groups + grp;
  if (cc >= it.nt * G) return;  // (SPREAD: the whole block)
  const size_t w0 = (size_t)item * a.parts * stride + cc;
  const int step = SPREAD ? groups : 1;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float mm = kLowest8, den = 0.f;
  for (int j0 = SPREAD ? grp : 0; j0 < n; j0 += 8 * step) {  // (slots past the last part read it again and weigh nothing)
    f32x4 v[8];
    float2 ml[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const size_t w = w0 + (size_t)min(j0 + j * step, n - 1) * stride;
      v[j] = *(const f32x4*)(a.part_acc + w * D + d);
      ml[j] = *(const float2*)(a.part_ml + 2 * w);
    }
    float top = mm;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
    const float r = mm == top ? 1.f : exp2f(mm - top);
    mm = top;
    den *= r;
    o *= r;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j0 + j * step < n) {
        const float f = exp2f(ml[j].x - mm);
        den += f * ml[j].y;
        o += f * v[j];
      }
  }
  if constexpr (SPREAD) {
    so[threadIdx.x] = o;
    sml[threadIdx.x] = make_float2(mm, den);
    __syncthreads();
    if (grp > 0) return;
    for (int x = 1; x < groups && x < n; ++x) {
      const float2 ml = sml[x * lanes + threadIdx.x];
      const float top = fmaxf(mm, ml.x), f0 = exp2f(mm - top), f1 = exp2f(ml.x - top);
      mm = top;
      den = f0 * den + f1 * ml.y;
      o = f0 * o + f1 * so[x * lanes + threadIdx.x];
    }
  }
  const int i = cc / G;
  store_x4_bf16(a.x_out, qrow8(a, it, i, cc - i * G, D) + d, o / den);
}

// ------------------------------------------------------------- reading back

// Tokens [start, start + count) of a sequence and layer as bf16 rows [count][Hkv][D]: codes times their
// scale, rounded once; the tokens behind the complete pages as they are. A thread per 8 dims of a
// token's K or V row: the units of a tile that hold them are 8 bytes (K) or 8 dims' single bytes (V).
// Bound: V's single-byte loads (131072 tokens, 8 heads of 128: 399 us for 0.8 GB, 2.0 TB/s).
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

hipError_t launch_attend8(const Attend8Args& a, hipStream_t st, const Timing* tm, const Timing* tm_merge) {
  const size_t heads = (size_t)a.launch_layers * a.n_kv_heads, units = a.seq_parts * heads;
  const size_t items = (size_t)a.launch_seqs * a.n_groups * heads;
  const size_t blocks = a.n_groups == 1 ? units : (units + 7) / 8 * 8 * a.n_groups;
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  auto run = [&](auto kernel) { return go(kernel, dim3((unsigned)blocks), dim3(64 * a.waves), 0, st, t0(tm), t1(tm), a); };
  auto pick = [&](auto code, auto dim) {
    constexpr int CODE = decltype(code)::value, D = decltype(dim)::value;
    if (a.tiles == 1) return a.waves == 8 ? run(k_attend8<CODE, D, 1, 8>) : run(k_attend8<CODE, D, 1, 4>);
    return run(k_attend8<CODE, D, 2, 4>);
  };
  using E = std::integral_constant<int, kE4m3>;
  using I = std::integral_constant<int, kInt8>;
  auto dims = [&](auto code) {
    return a.head_dim == 128 ? pick(code, std::integral_constant<int, 128>{}) : pick(code, std::integral_constant<int, 64>{});
  };
  const hipError_t e = a.c.code == kE4m3 ? dims(E{}) : dims(I{});
  if (e != hipSuccess || a.parts == 1) return e;
  const int cols = a.gt * a.group, per = 1024 / a.head_dim;  // columns of a block
  auto merge = [&](auto kernel, int y) { return go(kernel, dim3((unsigned)items, y), dim3(256), 0, st, t0(tm_merge), t1(tm_merge), a); };
  return a.parts > 8 && items * cols < 4096 ? merge(k_attend8_merge<true>, cols) : merge(k_attend8_merge<false>, (cols + per - 1) / per);
}

hipError_t launch_read8(const ReadCacheArgs& a, const Cache8Args& c, int len, hipStream_t st) {
  const size_t tasks = (size_t)a.count * a.n_kv_heads * (a.head_dim / 8) * 2;
  if ((tasks + 255) / 256 > 0x7FFFFFFFu) return hipErrorInvalidValue;
  return go(k_read8, dim3((unsigned)((tasks + 255) / 256)), dim3(256), 0, st, nullptr, nullptr, a, c, len);
}

}  // namespace pced
