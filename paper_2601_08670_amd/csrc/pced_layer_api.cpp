// Host side of the layer-wise calls (append with rotation, page summaries, attention
// over chosen pages) and of the adjusted logits. See include/pced.h.
#include "pced_host.h"

#include <algorithm>
#include <cmath>

using namespace pced;

namespace pced {

bool ranges_meet(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

pced_status check_layers(const pced_ctx* c, int layer, int n_layers, int n_tokens) {
  pced_status r = check_ctx(c, true);
  if (r != PCED_OK) return r;
  if (layer < 0 || n_layers < 1 || (long)layer + n_layers > c->cfg.n_layers)
    return fail(PCED_ERR_INVALID_ARG, "layers [%d, %ld) not in [0, %d)", layer, (long)layer + n_layers, c->cfg.n_layers);
  if (n_tokens < 1) return fail(PCED_ERR_INVALID_ARG, "n_tokens %d < 1", n_tokens);
  if ((long)n_tokens > (long)c->cfg.max_pages_per_seq * kPage)
    return fail(PCED_ERR_CAPACITY, "%d tokens > max_pages_per_seq", n_tokens);
  return check_room(c, n_tokens);
}

pced_status append_args(const pced_ctx* c, int layer, int n_layers, int n_tokens, const pced_rows* rows,
                        const pced_rope* rope, void* q_out, AppendRowsArgs* out) {
  pced_status r = check_layers(c, layer, n_layers, n_tokens);
  if (r != PCED_OK) return r;
  const pced_config& cfg = c->cfg;
  if (!rows || !rows->k || !rows->v) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  if (!rows->q != !q_out) return fail(PCED_ERR_INVALID_ARG, "q rows without q_out, or q_out without q rows");
  const size_t es = esize_of(cfg), D = cfg.head_dim, R = (size_t)c->S * n_tokens;
  const int64_t qd = (int64_t)n_layers * cfg.n_q_heads * D, kd = (int64_t)n_layers * cfg.n_kv_heads * D;
  AppendRowsArgs a{};
  a.q = rows->q;
  a.k = rows->k;
  a.v = rows->v;
  a.q_out = q_out;
  a.q_row = rows->q && rows->q_row ? rows->q_row : qd;
  a.k_row = rows->k_row ? rows->k_row : kd;
  a.v_row = rows->v_row ? rows->v_row : kd;
  if (a.q_row < qd || a.k_row < kd || a.v_row < kd)
    return fail(PCED_ERR_INVALID_ARG, "rows overlap: distances %lld, %lld, %lld", (long long)a.q_row, (long long)a.k_row,
                (long long)a.v_row);
  // the kernel moves rows in 16-byte units
  if (((uintptr_t)rows->q | (uintptr_t)rows->k | (uintptr_t)rows->v | (uintptr_t)q_out) % 16 ||
      (size_t)a.q_row * es % 16 || (size_t)a.k_row * es % 16 || (size_t)a.v_row * es % 16)
    return fail(PCED_ERR_INVALID_ARG, "rows and q_out must be 16-byte aligned, and the rows' distances too");
  if (q_out) {
    const size_t nq = ((R - 1) * a.q_row + qd) * es, nk = ((R - 1) * a.k_row + kd) * es, nv = ((R - 1) * a.v_row + kd) * es;
    const bool in_place = q_out == rows->q && a.q_row == qd;
    if ((!in_place && ranges_meet(q_out, R * qd * es, rows->q, nq)) || ranges_meet(q_out, R * qd * es, rows->k, nk) ||
        ranges_meet(q_out, R * qd * es, rows->v, nv))
      return fail(PCED_ERR_INVALID_ARG, "q_out overlaps the rows");
  }
  if (rope) {
    const int unit = c->bf16 ? 16 : 8;
    if (!(rope->theta > 1.0) || !std::isfinite(rope->theta)) return fail(PCED_ERR_INVALID_ARG, "rope theta must be > 1");
    if (rope->rot_dim < 0 || rope->rot_dim > cfg.head_dim || rope->rot_dim % 2)
      return fail(PCED_ERR_INVALID_ARG, "rot_dim %d: even, 0 .. %d", rope->rot_dim, cfg.head_dim);
    if (rope->halves != 0 && rope->halves != 1) return fail(PCED_ERR_INVALID_ARG, "halves must be 0 or 1");
    if (rope->halves && rope->rot_dim % unit)
      return fail(PCED_ERR_INVALID_ARG, "rot_dim %d: a multiple of %d with halves", rope->rot_dim, unit);
    a.rot_dim = rope->rot_dim;
    a.halves = rope->halves;
    a.log2_theta = std::log2(rope->theta);
  }
  a.len0 = (const int32_t*)(c->ws + c->lay.len0);
  a.page_table = (const int32_t*)(c->ws + c->lay.page_table);
  a.n_seqs = c->S;
  a.n_tokens = n_tokens;
  a.layer0 = layer;
  a.n_layers = n_layers;
  a.n_q_heads = cfg.n_q_heads;
  a.n_kv_heads = cfg.n_kv_heads;
  a.head_dim = cfg.head_dim;
  a.max_pages = cfg.max_pages;
  a.maxpps = cfg.max_pages_per_seq;
  a.t = c->t;
  a.sum_row = summary_row(cfg.head_dim);
  for (int s = 0; s < c->S; ++s)
    a.slots = std::max(a.slots, (c->len[s] + n_tokens - 1) / kPage - c->len[s] / kPage + 1);
  *out = a;
  return PCED_OK;
}
}  // namespace pced
namespace {

size_t summary_codes(const pced_config& c) {
  return align_up((size_t)c.n_layers * c.n_kv_heads * c.max_pages * summary_row(c.head_dim));
}

// How a launch of pced_attend divides its work: groups x layers, parts of the
// items' pages, and the workspace that takes (in the attention's partial states,
// of which none outlives its launches).
struct AttendPlan {
  int groups, layers, parts, part_pages;
  size_t scores, list, acc, ml, bytes;  // offsets
};

AttendPlan attend_plan(const pced_ctx* c, const AttendArgs& a, int max_pages, bool select, int groups, int layers,
                       int min_part) {
  AttendPlan p{};
  p.groups = groups;
  p.layers = layers;
  const size_t items = (size_t)groups * a.gt * layers * a.n_kv_heads;
  const int cnt = std::min(max_pages, a.n_pages);
  // two work-groups per compute unit, as far as a part keeps a batch of pages per wave (9 sequences, 256 pages each,
  // 8 kv-heads, attention and merge in us at 1 / 2 / 4 / 8 per unit: 33 / 34 / 34 / 35; 3 sequences, 128 pages: 9.9 /
  // 10.6 / 10.7 / 11; rounded down, one per unit would leave half of them idle at some counts)
  const size_t want = std::max<size_t>(1, 2 * (size_t)c->num_cus / items);
  p.part_pages = std::min(std::max<int>({min_part, ceil_div(ceil_div(cnt, (long)want), 8) * 8, 8}), kAttendPart);
  p.parts = ceil_div(cnt, p.part_pages);
  size_t o = 0;
  auto take = [&](size_t n) { const size_t at = o; o = align_up(o + n); return at; };
  p.scores = take(select ? items * a.score_row * 4 : 0);
  p.list = take(select && !a.pages_out ? items * a.n_pages * 4 : 0);
  p.acc = take(p.parts > 1 ? items * p.parts * a.group * a.head_dim * 4 : 0);
  p.ml = take(p.parts > 1 ? items * p.parts * a.group * 8 : 0);
  p.bytes = o;
  return p;
}

pced_status run_attend(pced_ctx* c, AttendArgs a, bool select, hipStream_t st) {
  const pced_config& cfg = c->cfg;
  const size_t room = c->lay.part_acc_bytes;
  int max_pages = 0;
  for (int s = 0; s < c->S; ++s) max_pages = std::max(max_pages, (c->len[s] + a.n_tokens - 1) / kPage + 1);
  a.score_row = ceil_div(max_pages, 16) * 16;
  const int all = c->S * a.seq_groups;
  // as many layers and groups per launch as the workspace takes
  int groups = all, layers = a.n_layers;
  // One new token and few pages: one launch chooses them and attends to them, each item in one part. bf16, 5
  // sequences of 4000 to 6000 tokens, us in one launch / in three (choice, parts, merge): 16 pages 14 / 20, 64 pages
  // 19 / 22, 128 pages 24 / 25; 2 sequences: 64 pages 17 / 20, 128 pages 22 / 20.
  const bool pick = select && a.n_tokens == 1 && max_pages <= kPickPages;
  int min_part = pick && a.n_pages <= 64 ? kAttendPart : 8;
  AttendPlan p = attend_plan(c, a, max_pages, select, groups, layers, min_part);
  while (p.bytes > room) {
    if (layers > 1) layers = (layers + 1) / 2;
    else if (groups > 1) groups = (groups + 1) / 2;
    else if (p.parts > 1 && p.part_pages < kAttendPart) min_part = 2 * p.part_pages;
    else return fail(PCED_ERR_CAPACITY, "a row's page lists exceed the workspace");
    p = attend_plan(c, a, max_pages, select, groups, layers, min_part);
  }
  const bool fused = pick && p.parts == 1;
  char* ws = c->at<char>(c->lay.part_acc);
  a.scores = (float*)(ws + p.scores);
  a.list = (int32_t*)(ws + p.list);
  a.part_acc = (float*)(ws + p.acc);
  a.part_ml = (float*)(ws + p.ml);
  a.parts = p.parts;
  a.part_pages = p.part_pages;
  const double es = (double)esize_of(cfg);
  double sums = 0, kv = 0;  // pages scored and attended to, per layer and kv-head
  for (int s = 0; c->prof && s < c->S; ++s)
    for (int i = 0; i < a.n_tokens; ++i) {
      const int n = (c->len[s] + i) / kPage + 1;
      if (n > a.n_pages) sums += n;
      kv += std::min(n, a.n_pages);
    }
  const double share = 1.0 / ((double)all * a.n_layers);
  for (int l = 0; l < a.n_layers; l += layers) {
    a.layer = a.layer0 + l;
    a.launch_layers = std::min(layers, a.n_layers - l);
    for (int g = 0; g < all; g += groups) {
      a.group0 = g;
      a.n_groups = std::min(groups, all - g);
      const double part = share * a.n_groups * a.launch_layers * a.n_layers * cfg.n_kv_heads;
      if (!fused && (select || a.pages_out)) {
        // the bounds of long sequences: six work-groups per compute unit, each at least 128 pages (9 books
        // of up to 131072 tokens, us at 4 / 6 / 12 / 24: scattered pages 33 / 29 / 28 / 33, in order 23 / 20 / 20 / 25)
        const long blocks = std::max<long>(1, 6L * c->num_cus / ((long)a.n_groups * a.launch_layers * a.n_kv_heads));
        a.chunk_pages = ceil_div(ceil_div(max_pages, blocks), 128) * 128;
        a.chunks = ceil_div(max_pages, a.chunk_pages);
        ProfScope ps(c, PCED_PROF_ATTN, select ? part * sums * (2.0 * cfg.head_dim + 4) : 0,
                     select ? part * sums * 4.0 * cfg.head_dim : 0);
        HIP_OK(launch_page_select(a, select, st, ps.timing()));
      }
      ProfScope ps(c, PCED_PROF_ATTN, part * kv * 2 * kPage * cfg.head_dim * es, part * kv * 4 * kPage * cfg.head_dim * c->G);
      ProfScope pm(c, PCED_PROF_COMBINE, 0, 0);
      if (p.parts == 1) pm.drop();
      HIP_OK(launch_attend(a, fused, st, ps.timing(), pm.timing()));
    }
  }
  return PCED_OK;
}

}  // namespace
namespace pced {
pced_status adjust_args(const pced_ctx* c, const pced_adjust* d, AdjustArgs* out) {
  if (!d) return fail(PCED_ERR_INVALID_ARG, "adjust is NULL");
  constexpr int kMaxList = 1 << 30;  // (the kernels' places in a list are 32-bit)
  if (d->n_history < 0 || d->n_history > kMaxList || d->n_bias < 0 || d->n_bias > kMaxList)
    return fail(PCED_ERR_INVALID_ARG, "n_history %d, n_bias %d: 0 .. 2^30", d->n_history, d->n_bias);
  if (d->history && !d->history_off) return fail(PCED_ERR_INVALID_ARG, "history without history_off");
  if (d->bias_token && (!d->bias_value || !d->bias_off))
    return fail(PCED_ERR_INVALID_ARG, "bias_token without bias_value or bias_off");
  const int64_t words = ceil_div(c->cfg.vocab, 32);
  if (d->mask && d->mask_row != 0 && d->mask_row < words)
    return fail(PCED_ERR_INVALID_ARG, "mask_row %lld < %lld words", (long long)d->mask_row, (long long)words);
  AdjustArgs a{};
  a.history = d->history;
  a.history_off = d->history_off;
  a.repetition = d->repetition;
  a.presence = d->presence;
  a.frequency = d->frequency;
  a.bias_token = d->bias_token;
  a.bias_value = d->bias_value;
  a.bias_off = d->bias_off;
  a.mask = d->mask;
  a.mask_row = d->mask_row ? d->mask_row : words;
  a.n_history = d->n_history;
  a.n_bias = d->n_bias;
  a.V = c->cfg.vocab;
  *out = a;
  return PCED_OK;
}
}  // namespace pced

extern "C" {

pced_status pced_append(pced_ctx* c, int32_t layer, int32_t n_layers, int32_t n_tokens, const pced_rows* rows,
                        const pced_rope* rope, void* q_out, hipStream_t st) {
  pced_status r = check_pools(c);
  if (r != PCED_OK) return r;
  AppendRowsArgs a{};
  r = append_args(c, layer, n_layers, n_tokens, rows, rope, q_out, &a);
  if (r != PCED_OK) return r;
  const pced_config& cfg = c->cfg;
  a.kpool = c->kpool;
  a.vpool = c->vpool;
  bool covered = c->summary != nullptr;  // (of several layers all or none: a launch has one answer)
  for (int l = layer; l < layer + n_layers; ++l) covered = covered && c->behind[l] == 0;
  if (covered) {
    a.codes = (int8_t*)c->summary;
    a.scale = (float*)(c->summary + summary_codes(cfg));
  }
  {
    const double heads = (rows->q ? cfg.n_q_heads : 0) + 2.0 * cfg.n_kv_heads;
    ProfScope ps(c, PCED_PROF_APPEND, 2.0 * c->S * n_tokens * n_layers * heads * cfg.head_dim * esize_of(cfg), 0);
    HIP_OK(launch_append_rows(a, c->bf16, st, ps.timing()));
  }
  for (int l = layer; l < layer + n_layers; ++l) {
    c->appended[l] = n_tokens;
    c->ahead[l] = covered ? n_tokens : 0;
  }
  return PCED_OK;
}

pced_status pced_advance(pced_ctx* c, int32_t n_tokens) {
  pced_status r = check_ctx(c, true);
  if (r != PCED_OK) return r;
  if (n_tokens < 1) return fail(PCED_ERR_INVALID_ARG, "n_tokens %d < 1", n_tokens);
  for (int l = 0; l < c->cfg.n_layers; ++l)
    if (c->appended[l] < n_tokens)
      return fail(PCED_ERR_STATE, "layer %d has %d appended tokens, not %d", l, c->appended[l], n_tokens);
  advance(c, n_tokens, true);
  return PCED_OK;
}

size_t pced_summary_bytes(const pced_config* cfg) {
  if (!cfg_valid(cfg, nullptr)) return 0;
  return summary_codes(*cfg) + align_up((size_t)cfg->n_layers * cfg->n_kv_heads * cfg->max_pages * 4);
}

pced_status pced_bind_summary(pced_ctx* c, void* summary) {
  pced_status r = check_ctx(c, false);
  if (r != PCED_OK) return r;
  if ((uintptr_t)summary % kAlign) return fail(PCED_ERR_INVALID_ARG, "summary must be 256-byte aligned");
  c->summary = (char*)summary;
  std::fill(c->ahead.begin(), c->ahead.end(), 0);
  std::fill(c->behind.begin(), c->behind.end(), kNotCovered);
  return PCED_OK;
}

pced_status pced_summarize(pced_ctx* c, hipStream_t st) {
  pced_status r = check_pools(c);
  if (r != PCED_OK) return r;
  if (!c->summary) return fail(PCED_ERR_STATE, "no summary buffer bound (call pced_bind_summary first)");
  const pced_config& cfg = c->cfg;
  SummaryArgs a{};
  a.kpool = c->kpool;
  a.len0 = c->at<int32_t>(c->lay.len0);
  a.page_table = c->at<int32_t>(c->lay.page_table);
  a.codes = (int8_t*)c->summary;
  a.scale = (float*)(c->summary + summary_codes(cfg));
  a.n_seqs = c->S;
  a.n_layers = cfg.n_layers;
  a.n_kv_heads = cfg.n_kv_heads;
  a.head_dim = cfg.head_dim;
  a.max_pages = cfg.max_pages;
  a.maxpps = cfg.max_pages_per_seq;
  a.t = c->t;
  a.sum_row = summary_row(cfg.head_dim);
  // one span for all layers: the pages from the oldest token that some layer lacks
  a.behind = *std::max_element(c->behind.begin(), c->behind.end());
  for (int s = 0; s < c->S; ++s)
    a.span = std::max(a.span, c->len[s] / kPage - std::max(c->len[s] - a.behind, 0) / kPage);
  HIP_OK(launch_summarize(a, c->bf16, st));
  // (rows behind the lengths that pced_append has summarised stay so: their layers were up to date)
  std::fill(c->behind.begin(), c->behind.end(), 0);
  return PCED_OK;
}

pced_status pced_attend(pced_ctx* c, int32_t layer, int32_t n_layers, int32_t n_tokens, const void* q,
                        const pced_select* sel, void* x_out, int32_t* pages_out, hipStream_t st) {
  pced_status r = check_pools(c);
  if (r == PCED_OK) r = check_layers(c, layer, n_layers, n_tokens);
  if (r != PCED_OK) return r;
  const pced_config& cfg = c->cfg;
  if (!q || !x_out) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)q | (uintptr_t)x_out) % 16) return fail(PCED_ERR_INVALID_ARG, "q and x_out must be 16-byte aligned");
  if (pages_out && !sel) return fail(PCED_ERR_INVALID_ARG, "pages_out without sel");
  if (sel && (sel->n_first < 0 || sel->n_last < 1 || (long)sel->n_first + sel->n_last > sel->n_pages))
    return fail(PCED_ERR_INVALID_ARG, "n_first %d >= 0, n_last %d >= 1, their sum at most n_pages %d", sel->n_first,
                sel->n_last, sel->n_pages);
  if (sel && sel->n_pages > 1 << 30)  // (places in a list are 32-bit)
    return fail(PCED_ERR_INVALID_ARG, "n_pages %d > 2^30", sel->n_pages);
  const size_t bytes = (size_t)c->S * n_tokens * n_layers * cfg.hidden * esize_of(cfg);
  if (ranges_meet(q, bytes, x_out, bytes)) return fail(PCED_ERR_INVALID_ARG, "q and x_out overlap");
  for (int l = layer; l < layer + n_layers; ++l)
    if (c->appended[l] < n_tokens)
      return fail(PCED_ERR_STATE, "layer %d has %d appended tokens, not %d", l, c->appended[l], n_tokens);
  int max_pages = 0;
  for (int s = 0; s < c->S; ++s) max_pages = std::max(max_pages, (c->len[s] + n_tokens - 1) / kPage + 1);
  const bool select = sel && sel->n_pages < max_pages;
  if (select) {
    if (!c->summary) return fail(PCED_ERR_STATE, "no summary buffer bound (call pced_bind_summary first)");
    for (int l = layer; l < layer + n_layers; ++l)
      if (c->behind[l] != 0 || c->ahead[l] < n_tokens)
        return fail(PCED_ERR_STATE, "layer %d: the page summaries are not up to date (call pced_summarize before pced_append)",
                    l);
  }
  AttendArgs a{};
  a.q = q;
  a.kpool = c->kpool;
  a.vpool = c->vpool;
  a.codes = (const int8_t*)c->summary;
  a.scale = c->summary ? (const float*)(c->summary + summary_codes(cfg)) : nullptr;
  a.len0 = c->at<int32_t>(c->lay.len0);
  a.page_table = c->at<int32_t>(c->lay.page_table);
  a.pages_out = pages_out;
  a.x_out = x_out;
  a.t = c->t;
  a.n_tokens = n_tokens;
  a.seq_groups = ceil_div(n_tokens, kAttendTokens);
  a.gt = ceil_div(n_tokens, a.seq_groups);
  a.layer0 = layer;
  a.n_layers = n_layers;
  a.n_q_heads = cfg.n_q_heads;
  a.n_kv_heads = cfg.n_kv_heads;
  a.group = c->G;
  a.head_dim = cfg.head_dim;
  a.max_pages = cfg.max_pages;
  a.maxpps = cfg.max_pages_per_seq;
  a.sum_row = summary_row(cfg.head_dim);
  a.bf16 = c->bf16;
  a.num_cus = c->num_cus;
  a.n_pages = sel ? sel->n_pages : max_pages;
  a.first = sel ? sel->n_first : 0;
  a.last = sel ? sel->n_last : 1;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)cfg.head_dim));
  a.lead = 8.f / a.scale_log2;
  return run_attend(c, a, select, st);
}

pced_status pced_adjust_logits(pced_ctx* c, const float* logits, const pced_adjust* adjust, float* out,
                               hipStream_t st) {
  pced_status r = check_ctx(c, true);
  if (r != PCED_OK) return r;
  if (!logits || !out) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  const size_t bytes = (size_t)c->S * c->cfg.vocab * 4;
  if (out != logits && ranges_meet(logits, bytes, out, bytes))
    return fail(PCED_ERR_INVALID_ARG, "out overlaps logits");
  AdjustArgs a{};
  r = adjust_args(c, adjust, &a);
  if (r != PCED_OK) return r;
  a.logits = logits;
  a.out = out;
  a.query_seq0 = c->at<int32_t>(c->lay.query_seq0);
  const int rows = *std::max_element(c->n_experts.begin(), c->n_experts.end()) + 1;
  HIP_OK(launch_adjust(a, c->B, rows, c->num_cus, st));
  return PCED_OK;
}

pced_status pced_fuse_adjusted(pced_ctx* c, const float* logits, int32_t refresh_beta, const pced_adjust* adjust,
                               int32_t* tokens_out, const pced_step_out* extra, hipStream_t st) {
  pced_status r = check_ctx(c, true);
  if (r != PCED_OK) return r;
  if (!logits || !tokens_out) return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  if (c->cfg.aggregation != PCED_AGG_MAX)
    return fail(PCED_ERR_UNSUPPORTED, "adjusted logits are fused by PCED_AGG_MAX only");
  if (c->dynamic_beta && !refresh_beta && !c->beta_frozen)
    return fail(PCED_ERR_STATE, "dynamic beta has not been computed yet (pass refresh_beta)");
  AdjustArgs d{};
  r = adjust_args(c, adjust, &d);
  if (r != PCED_OK) return r;
  if (c->dynamic_beta && refresh_beta) {
    r = run_beta(c, logits, st);
    if (r != PCED_OK) return r;
  }
  FuseArgs f = fuse_args(c, logits, tokens_out, 1, extra,
                         ceil_div(c->cfg.vocab, adjusted_slice(c->cfg.vocab, c->B, c->num_cus)));
  f.none_token = 1;
  ProfScope ps(c, PCED_PROF_FUSE, (double)c->S * c->cfg.vocab * 4, 0);
  ProfScope pm(c, PCED_PROF_FUSE_MERGE, (double)c->B * f.nblk * 5 * 4, 0);
  HIP_OK(launch_fuse_adjusted(f, d, c->B, st, ps.timing(), pm.timing()));
  return PCED_OK;
}

}  // extern "C"
