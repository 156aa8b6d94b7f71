// Host side of caches held in 8 bits: loading, append, attention, reading back. See
// include/pced.h.
#include "pced_host.h"

#include <algorithm>
#include <cmath>

using namespace pced;

namespace {

// Pages that n new tokens touch, at most: one open place each
int ring_of(int n) { return (int)(((long)n + kPage - 2) / kPage) + 1; }

size_t code_bytes(const pced_config& c) {
  return (size_t)c.n_layers * c.max_pages * c.n_kv_heads * kPage * c.head_dim;
}

pced_status check_cache8(const pced_ctx* c, const pced_cache8* m) {
  const pced_config& cfg = c->cfg;
  if (!m) return fail(PCED_ERR_INVALID_ARG, "cache is NULL");
  if (!c->bf16) return fail(PCED_ERR_UNSUPPORTED, "caches in 8 bits need a bf16 context");
  if (m->code != PCED_CODE_E4M3 && m->code != PCED_CODE_INT8) return fail(PCED_ERR_INVALID_ARG, "unknown code %d", m->code);
  if (m->max_new < 1 || m->max_new > 1 << 20) return fail(PCED_ERR_INVALID_ARG, "max_new %d: 1 .. 2^20", m->max_new);
  if ((long)cfg.max_seqs * ring_of(m->max_new) > 0x7FFFFFFF)  // (places of open pages are 32-bit)
    return fail(PCED_ERR_INVALID_ARG, "max_new %d for %d sequences: too many open pages", m->max_new, cfg.max_seqs);
  const void* at[5] = {m->k_codes, m->v_codes, m->scales, m->k_open, m->v_open};
  const size_t n[5] = {pced_codes_bytes(&cfg), pced_codes_bytes(&cfg), pced_scales_bytes(&cfg),
                       pced_open_bytes(&cfg, m->max_new), pced_open_bytes(&cfg, m->max_new)};
  for (int i = 0; i < 5; ++i) {
    if (!at[i]) return fail(PCED_ERR_INVALID_ARG, "NULL buffer in cache");
    if ((uintptr_t)at[i] % kAlign) return fail(PCED_ERR_INVALID_ARG, "cache's buffers must be 256-byte aligned");
    for (int j = 0; j < i; ++j)
      if (ranges_meet(at[i], n[i], at[j], n[j])) return fail(PCED_ERR_INVALID_ARG, "cache's buffers overlap");
  }
  return PCED_OK;
}

pced_status check_loaded8(const pced_ctx* c) {
  const pced_status r = check_ctx(c, true);
  if (r == PCED_OK && !c->c8.code) return fail(PCED_ERR_STATE, "the batch's caches are not in 8 bits (call pced_load_codes)");
  return r;
}

pced_status check_new(const pced_ctx* c, int n_tokens) {
  if (n_tokens > c->max_new) return fail(PCED_ERR_CAPACITY, "%d tokens > max_new %d", n_tokens, c->max_new);
  return PCED_OK;
}

// How pced_attend_codes divides its work: sequences, groups per sequence and layers per launch, pages per part, and
// the workspace that the parts' states take.
struct Plan8 {
  int seqs, groups, layers, part_pages;
  int parts;         // of the longest sequence
  size_t ml, bytes;  // (offset of the second array)
};
void size_plan(Plan8* p, const Attend8Args& a, int max_pages) {
  const size_t cols = (size_t)a.gt * a.group;
  p->parts = ceil_div(max_pages, p->part_pages);
  const size_t states = (size_t)p->seqs * p->groups * p->layers * a.n_kv_heads * p->parts * cols;
  p->ml = p->parts > 1 ? align_up(states * a.head_dim * 4) : 0;
  p->bytes = p->parts > 1 ? p->ml + align_up(states * 8) : 0;
}
// The pages that n new tokens of sequence s end in, and all before
int pages_of(const pced_ctx* c, int s, int n) { return (c->len[s] + n - 1) / kPage + 1; }

// The waves of a work-group hold kWavePages page numbers each.
//
// Parts. Splitting a sequence costs a second launch and the states' way through memory (about 2 us), so sequences of
// up to 96 pages stay whole (4 x 63 pages and a query's own, 8 heads: 8.2 us, split 10.1), and so do longer ones
// where they keep every CU busy as they are (33 x 188 pages on average: 40 us, in parts of 64 pages 44). Otherwise
// parts are as short as one work-group per CU allows (5 x up to 250 pages, us in parts of 32 / 48 / 96 / 256 pages: 11.7 /
// 12.2 / 14.8 / 18.8), 32 pages at least.
bool plan8(const pced_ctx* c, const Attend8Args& a, int groups, Plan8* out) {
  const int most = 4 * kWavePages, S = c->S;
  int max_pages = 0;
  long sum = 0;
  for (int s = 0; s < S; ++s) {
    const int x = pages_of(c, s, a.n_tokens);
    max_pages = std::max(max_pages, x);
    sum += x;
  }
  const double per = (double)groups * a.n_layers * a.n_kv_heads;  // work-groups for a part of a sequence
  int part = most;
  if (max_pages > 96 && S * per <= c->num_cus) {
    for (part = (int)std::min<double>(most, std::max(32., std::ceil(sum * per / c->num_cus / 8) * 8)); part < most; part += 8) {
      long n = 0;
      for (int s = 0; s < S; ++s) n += ceil_div(pages_of(c, s, a.n_tokens), part);
      if (n * per <= c->num_cus) break;
    }
  }
  Plan8 p{S, groups, a.n_layers, part, 0, 0, 0};
  size_plan(&p, a, max_pages);
  while (p.bytes > c->lay.part_acc_bytes) {
    if (p.layers > 1) p.layers = (p.layers + 1) / 2;
    else if (p.seqs > 1) p.seqs = (p.seqs + 1) / 2;
    else if (p.groups > 1) p.groups = (p.groups + 1) / 2;
    else if (p.part_pages < most) p.part_pages = std::min(2 * p.part_pages, most);
    else return false;
    size_plan(&p, a, max_pages);
  }
  *out = p;
  return true;
}

}  // namespace

extern "C" {

size_t pced_codes_bytes(const pced_config* cfg) {
  if (!cfg_valid(cfg, nullptr) || cfg->dtype != PCED_BF16) return 0;
  return code_bytes(*cfg);
}

size_t pced_scales_bytes(const pced_config* cfg) {
  if (!cfg_valid(cfg, nullptr) || cfg->dtype != PCED_BF16) return 0;
  return (size_t)cfg->n_layers * cfg->n_kv_heads * cfg->max_pages * 4;
}

size_t pced_open_bytes(const pced_config* cfg, int32_t max_new) {
  if (!cfg_valid(cfg, nullptr) || cfg->dtype != PCED_BF16 || max_new < 1) return 0;
  return (size_t)cfg->n_layers * cfg->max_seqs * ring_of(max_new) * cfg->n_kv_heads * kPage * cfg->head_dim * 2;
}

pced_status pced_load_codes(pced_ctx* c, int32_t n_queries, const int32_t* n_experts, const int32_t* cache_len,
                            const void* const* src_k, const void* const* src_v, const pced_cache8* cache,
                            const int32_t* page_table, int32_t reserve_tokens, const float* relevance, float gamma,
                            const float* beta, hipStream_t st) {
  pced_status r = check_ctx(c, false);
  if (r == PCED_OK) r = check_cache8(c, cache);
  if (r != PCED_OK) return r;
  LoadTarget to{cache->k_codes, cache->v_codes, {}, cache->max_new,
                [](const LoadArgs& a, const LoadTarget& t, int n_items, bool, hipStream_t s) {
                  return launch_load8(a, t.c8, n_items, s);
                }};
  to.c8.k_codes = (uint8_t*)cache->k_codes;
  to.c8.v_codes = (uint8_t*)cache->v_codes;
  to.c8.scales = (uint32_t*)cache->scales;
  to.c8.k_open = (uint16_t*)cache->k_open;
  to.c8.v_open = (uint16_t*)cache->v_open;
  to.c8.code = cache->code;
  to.c8.ring = ring_of(cache->max_new);
  to.c8.open_pages = c->cfg.max_seqs * to.c8.ring;
  to.c8.max_pages = c->cfg.max_pages;
  return load_batch(c, n_queries, n_experts, cache_len, src_k, src_v, to, page_table, reserve_tokens, relevance, gamma,
                    beta, st);
}

pced_status pced_append_codes(pced_ctx* c, int32_t layer, int32_t n_layers, int32_t n_tokens, const pced_rows* rows,
                              const pced_rope* rope, void* q_out, hipStream_t st) {
  pced_status r = check_loaded8(c);
  if (r != PCED_OK) return r;
  AppendRowsArgs a{};
  r = append_args(c, layer, n_layers, n_tokens, rows, rope, q_out, &a);
  if (r == PCED_OK) r = check_new(c, n_tokens);
  if (r != PCED_OK) return r;
  const pced_config& cfg = c->cfg;
  a.kpool = c->c8.k_open;
  a.vpool = c->c8.v_open;
  a.max_pages = c->c8.open_pages;
  {
    const double heads = (rows->q ? cfg.n_q_heads : 0) + 2.0 * cfg.n_kv_heads;
    ProfScope ps(c, PCED_PROF_APPEND, 4.0 * c->S * n_tokens * n_layers * heads * cfg.head_dim, 0);
    HIP_OK(launch_append8(a, c->c8, st, ps.timing()));
  }
  for (int l = layer; l < layer + n_layers; ++l) {
    c->appended[l] = n_tokens;
    c->ahead[l] = 0;
  }
  return PCED_OK;
}

pced_status pced_attend_codes(pced_ctx* c, int32_t layer, int32_t n_layers, int32_t n_tokens, const void* q, void* x_out,
                              hipStream_t st) {
  pced_status r = check_loaded8(c);
  if (r == PCED_OK) r = check_layers(c, layer, n_layers, n_tokens);
  if (r == PCED_OK) r = check_new(c, n_tokens);
  if (r != PCED_OK) return r;
  const pced_config& cfg = c->cfg;
  if (!q || !x_out) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)q | (uintptr_t)x_out) % 16) return fail(PCED_ERR_INVALID_ARG, "q and x_out must be 16-byte aligned");
  const size_t bytes = (size_t)c->S * n_tokens * n_layers * cfg.hidden * 2;
  if (ranges_meet(q, bytes, x_out, bytes)) return fail(PCED_ERR_INVALID_ARG, "q and x_out overlap");
  for (int l = layer; l < layer + n_layers; ++l)
    if (c->appended[l] < n_tokens)
      return fail(PCED_ERR_STATE, "layer %d has %d appended tokens, not %d", l, c->appended[l], n_tokens);
  Attend8Args a{};
  a.c = c->c8;
  a.q = q;
  a.x_out = x_out;
  a.len0 = c->at<int32_t>(c->lay.len0);
  a.page_table = c->at<int32_t>(c->lay.page_table);
  a.t = c->t;
  a.n_tokens = n_tokens;
  a.layer0 = layer;
  a.n_layers = n_layers;
  a.n_q_heads = cfg.n_q_heads;
  a.n_kv_heads = cfg.n_kv_heads;
  a.group = c->G;
  a.head_dim = cfg.head_dim;
  a.maxpps = cfg.max_pages_per_seq;
  // Two tiles share a page's loads and decoding, one leaves room for more waves. 33 sequences of 82 pages on average,
  // 8 heads of 128, e4m3: 8 columns 18.6 us (two tiles 21.3), 32 columns 22.0 (24.3), 64 columns 33.3 (35.0), 128 columns
  // 56.4 (53.8), 256 columns 104 (95); int8, 64 columns 40.5 (40.3), 256 columns 132 (112). 64 columns of 5 x up to 250
  // pages: e4m3 18.3 (17.2), int8 21.7 (18.8).
  a.tiles = n_tokens * c->G <= 32 ? 1 : 2;
  const int groups = ceil_div(n_tokens, 16 * a.tiles / c->G);  // per sequence
  a.gt = ceil_div(n_tokens, groups);
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)cfg.head_dim));
  Plan8 p{};
  if (!plan8(c, a, groups, &p))
    return fail(PCED_ERR_CAPACITY, "a token group's partial states exceed the workspace");
  // Eight waves for a whole sequence where four would leave a CU's SIMDs with two each or less (e4m3, 8 heads of 128:
  // 5 sequences of up to 63 pages 8.3 us, four waves 8.8; 33 of up to 128 pages 18.1 and 18.4, 64 of them 33.5 and 36.3;
  // not where more work-groups than CUs have short sequences: 33 of up to 44 pages 11.2 and 9.3);
  // four where work-groups abound or parts are short.
  a.waves = a.tiles == 1 && p.parts == 1 && (double)c->S * groups * n_layers * cfg.n_kv_heads <= 2. * c->num_cus ? 8 : 4;
  char* ws = c->at<char>(c->lay.part_acc);
  a.part_acc = (float*)ws;
  a.part_ml = (float*)(ws + p.ml);
  a.parts = p.parts;
  a.part_pages = p.part_pages;
  for (int l = 0; l < n_layers; l += p.layers) {
    a.layer = layer + l;
    a.launch_layers = std::min(p.layers, n_layers - l);
    for (a.seq0 = 0; a.seq0 < c->S; a.seq0 += p.seqs) {
      a.launch_seqs = std::min(p.seqs, c->S - a.seq0);
      a.seq_parts = 0;
      double tokens = 0;  // seen, per layer and kv-head
      for (int s = a.seq0; s < a.seq0 + a.launch_seqs; ++s) {
        a.seq_parts += ceil_div(pages_of(c, s, n_tokens), p.part_pages);
        tokens += c->len[s] + n_tokens;
      }
      for (a.group0 = 0; a.group0 < groups; a.group0 += p.groups) {
        a.n_groups = std::min(p.groups, groups - a.group0);
        const double part = tokens * a.n_groups / groups * a.launch_layers * cfg.n_kv_heads * cfg.head_dim;
        ProfScope ps(c, PCED_PROF_ATTN, part * 2, part * 4 * c->G * n_tokens);
        ProfScope pm(c, PCED_PROF_COMBINE, 0, 0);
        if (p.parts == 1) pm.drop();
        HIP_OK(launch_attend8(a, st, ps.timing(), pm.timing()));
      }
    }
  }
  return PCED_OK;
}

pced_status pced_read_codes(pced_ctx* c, int32_t seq, int32_t layer, int32_t start, int32_t count, void* k_out, void* v_out,
                            hipStream_t st) {
  pced_status r = check_loaded8(c);
  if (r != PCED_OK) return r;
  if (seq < 0 || seq >= c->S) return fail(PCED_ERR_INVALID_ARG, "seq %d not in [0, %d)", seq, c->S);
  if (layer < 0 || layer >= c->cfg.n_layers)
    return fail(PCED_ERR_INVALID_ARG, "layer %d not in [0, %d)", layer, c->cfg.n_layers);
  if (start < 0 || count < 0 || (long)start + count > c->len[seq])
    return fail(PCED_ERR_INVALID_ARG, "tokens [%d, %ld) beyond the %d of sequence %d", start, (long)start + count,
                c->len[seq], seq);
  if (count == 0) return PCED_OK;
  if (!k_out || !v_out) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  ReadCacheArgs a{};
  a.page_table = c->at<int32_t>(c->lay.page_table);
  a.k_out = k_out;
  a.v_out = v_out;
  a.seq = seq;
  a.layer = layer;
  a.start = start;
  a.count = count;
  a.n_kv_heads = c->cfg.n_kv_heads;
  a.head_dim = c->cfg.head_dim;
  a.max_pages = c->cfg.max_pages;
  a.maxpps = c->cfg.max_pages_per_seq;
  a.bf16 = 1;
  HIP_OK(launch_read8(a, c->c8, c->len[seq], st));
  return PCED_OK;
}

}  // extern "C"
