// Host side of sampling. See include/pced.h.
#include "pced_host.h"

using namespace pced;

namespace {

// Weights of V tokens, multiples of 2^-shift up to 1, add up to at most 2^62
int weight_shift(int V) {
  int bits = 0;
  while (((long)1 << bits) < V) ++bits;
  return 62 - bits;
}

}  // namespace

extern "C" {

pced_status pced_sample(pced_ctx* c, const float* logits, int32_t refresh_beta, const pced_adjust* adjust,
                        const pced_sampling* sampling, const float* uniform, int32_t* tokens_out,
                        const pced_sample_out* extra, hipStream_t st) {
  pced_status r = check_ctx(c, true);
  if (r != PCED_OK) return r;
  if (!logits || !sampling || !sampling->temperature || !uniform || !tokens_out)
    return fail(PCED_ERR_INVALID_ARG, "NULL argument");
  if (c->cfg.aggregation != PCED_AGG_MAX)
    return fail(PCED_ERR_UNSUPPORTED, "tokens are sampled from the scores of PCED_AGG_MAX only");
  if (c->dynamic_beta && !refresh_beta && !c->beta_frozen)
    return fail(PCED_ERR_STATE, "dynamic beta has not been computed yet (pass refresh_beta)");
  AdjustArgs d{};
  const pced_adjust none{};
  r = adjust_args(c, adjust ? adjust : &none, &d);
  if (r != PCED_OK) return r;
  if (c->dynamic_beta && refresh_beta) {
    r = run_beta(c, logits, st);
    if (r != PCED_OK) return r;
  }
  const int V = c->cfg.vocab;
  FuseArgs f = fuse_args(c, logits, tokens_out, 1, nullptr, ceil_div(V, adjusted_slice(V, c->B, c->num_cus)));
  SampleArgs a{};
  a.scores = c->at<float>(c->lay.logits);
  a.who = (int32_t*)(a.scores + (size_t)c->B * V);
  a.part = f.part;
  a.bins = c->at<SampleBins>(c->lay.smp_bins);
  a.list = c->at<unsigned long long>(c->lay.smp_list);
  a.temperature = sampling->temperature;
  a.top_k = sampling->top_k;
  a.top_p = sampling->top_p;
  a.min_p = sampling->min_p;
  a.uniform = uniform;
  a.tokens_out = tokens_out;
  a.prev_tok = f.prev_tok;
  if (extra) {
    a.winner = extra->winner;
    a.score = extra->score;
    a.logprob = extra->logprob;
    a.kept = extra->kept;
    a.beta_used = extra->beta_used;
  }
  a.beta = f.beta;
  a.query_exp0 = f.query_exp0;
  a.V = V;
  a.nblk = f.nblk;
  a.shift = weight_shift(V);
  {
    ProfScope ps(c, PCED_PROF_FUSE, (double)c->S * V * 4, 0);
    HIP_OK(launch_fuse_scores(f, d, a, c->B, st, ps.timing()));
  }
  ProfScope pm(c, PCED_PROF_FUSE_MERGE, (double)c->B * V * 8, 0);
  HIP_OK(launch_sample(a, c->B, c->num_cus, st, pm.timing()));
  return PCED_OK;
}

}  // extern "C"
