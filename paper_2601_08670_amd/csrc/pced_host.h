// The library's host state and the helpers that its entry points share.
#pragma once
#include "pced.h"

#include <hip/hip_runtime.h>
#include <rocblas/rocblas.h>

#include <string>
#include <vector>

#include "pced_internal.h"

namespace pced {

// Sets the thread's error text and returns st.
pced_status fail(pced_status st, const char* fmt, ...);

#define HIP_OK(expr)                                                               \
  do {                                                                             \
    hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess) return fail(PCED_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline size_t esize_of(const pced_config& c) { return c.dtype == PCED_BF16 ? 2 : 4; }
inline int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

struct Layout {
  size_t len0, page_table, seq_query, query_seq0, query_exp0, exp_seq, exp_query, prior, logw, beta_fixed,
      load_items, src_k, src_v, meta_end;
  size_t chunk_info, seg, nparts, work_pages, prev_tok, beta, part_acc, part_ml, x, logits,
      rho, x_packed, fuse_part, lse_part, jsd_part, syn_q, syn_k, syn_v, dec_h, dec_a, dec_act, dec_ss, dec_rho, dec_part,
      rope, pf_len0, pf_pt, pf_tok, pf_glen0, pf_gpt, pf_nparts, pf_rho, pf_h, pf_a, pf_act, pf_ss, pf_q, pf_x, pf_part_acc, pf_part_ml, pf_proj,
      smp_bins, smp_list, stage_bytes, total;
  int packed_rows;      // rows x_packed holds
  int pf_rows;          // rows of one prefill chunk (sequences x suffix tokens)
  size_t pf_proj_cols;  // slices x columns per row of the prefill projection partials
  size_t pf_proj_elems; // floats of that buffer
  int rows_pad, nchunk, max_work;
  size_t seg_slots;     // segment descriptors of the attention plan
  size_t part_slots;
  size_t part_acc_bytes;  // of the attention's partial outputs
  size_t part_cols;  // slices x columns one row of the projection partial buffer holds
};

struct ProfRec {
  int cls;
  hipEvent_t a, b;
  double bytes, flops;
};

constexpr int kNotCovered = 0x7FFFFFFF;  // page summaries: of no token yet

}  // namespace pced

struct pced_ctx {
  pced_config cfg;
  pced::Layout lay;
  char* ws;
  bool bf16;
  int G;
  // host mirror of the loaded batch
  bool loaded = false;
  int B = 0, S = 0, NE = 0;
  std::vector<int32_t> n_experts, seq_off, exp_off, len, page_table;
  bool dynamic_beta = false, beta_frozen = false;
  pced::LmWidePlan head_groups;  // the fused LM head's row groups for more than 288 rows
  int t = 0;
  // layer-wise calls: rows appended behind the lengths, per layer; page summaries
  // and, per layer, the tokens before the lengths (behind) that they do not cover
  // yet (kNotCovered: all) or the appended ones behind the lengths (ahead) that they do
  std::vector<int> appended, ahead, behind;
  char* summary = nullptr;
  void* kpool = nullptr;
  void* vpool = nullptr;
  // a batch loaded by pced_load_codes (code 0: by pced_load_caches)
  pced::Cache8Args c8{};
  int max_new = 0;
  std::vector<char> staging;
  int num_cus = 0;
  int attn_waves_per_cu = 8;
  // profiling
  bool prof = false;
  std::vector<pced::ProfRec> recs;
  std::vector<hipEvent_t> ev_free;
  rocblas_handle blas = nullptr;  // created at the first many-row projection
  pced_profile totals{};

  template <class T> T* at(size_t off) { return reinterpret_cast<T*>(ws + off); }
};

namespace pced {

// Start/stop events of one kernel class launch when profiling is on. They are
// handed to the launcher, which attaches them to the dispatch itself
// (hipExtLaunchKernelGGL), so they time the kernels and not the queue.
struct ProfScope {
  pced_ctx* c;
  ProfRec rec;
  Timing tm;
  bool on;
  ProfScope(pced_ctx* ctx, int cls, double bytes, double flops) : c(ctx), on(ctx->prof) {
    if (!on) return;
    rec.cls = cls;
    rec.bytes = bytes;
    rec.flops = flops;
    rec.a = take();
    rec.b = take();
    if (!rec.a || !rec.b) {  // no events to be had: this launch goes untimed
      if (rec.a) c->ev_free.push_back(rec.a);
      if (rec.b) c->ev_free.push_back(rec.b);
      on = false;
      return;
    }
    tm.start = rec.a;
    tm.stop = rec.b;
  }
  const Timing* timing() const { return on ? &tm : nullptr; }
  void drop() {  // nothing was launched
    if (!on) return;
    c->ev_free.push_back(rec.a);
    c->ev_free.push_back(rec.b);
    on = false;
  }
  hipEvent_t take() {
    if (!c->ev_free.empty()) { hipEvent_t e = c->ev_free.back(); c->ev_free.pop_back(); return e; }
    hipEvent_t e = nullptr;
    if (hipEventCreateWithFlags(&e, hipEventDisableSystemFence) != hipSuccess) {
      (void)hipGetLastError();
      return nullptr;
    }
    return e;
  }
  ~ProfScope() {
    if (on) c->recs.push_back(rec);
  }
};

// Checks that entry points share: cfg's fields (why: what is wrong), a context and
// its loaded batch, room for n_tokens more tokens in every sequence.
bool cfg_valid(const pced_config* c, std::string* why);
pced_status check_ctx(const pced_ctx* c, bool need_loaded);
pced_status check_room(const pced_ctx* c, int n_tokens);
// A loaded batch whose caches are in the pools, for the calls that read or write them there.
pced_status check_pools(const pced_ctx* c);
// The layers and tokens of a layer-wise call.
pced_status check_layers(const pced_ctx* c, int layer, int n_layers, int n_tokens);
bool ranges_meet(const void* a, size_t na, const void* b, size_t nb);
// pced_append's checks of its arguments, and the kernel's arguments but for the pages.
pced_status append_args(const pced_ctx* c, int layer, int n_layers, int n_tokens, const pced_rows* rows,
                        const pced_rope* rope, void* q_out, AppendRowsArgs* out);

// Where a load puts the caches: the pools, or (c8.code != 0) a cache in 8 bits; `launch` moves pages there.
struct LoadTarget {
  void* k_pool;
  void* v_pool;
  Cache8Args c8;
  int max_new;
  hipError_t (*launch)(const LoadArgs& a, const LoadTarget& to, int n_items, bool bf16, hipStream_t st);
};
pced_status load_batch(pced_ctx* c, int32_t n_queries, const int32_t* n_experts, const int32_t* cache_len,
                       const void* const* src_k, const void* const* src_v, const LoadTarget& to,
                       const int32_t* page_table, int32_t reserve_tokens, const float* relevance, float gamma,
                       const float* beta, hipStream_t st);

// The lengths grow by n tokens. by_rows: tokens that pced_append wrote (the
// summaries cover what they covered of them); otherwise other calls wrote them.
void advance(pced_ctx* c, int n, bool by_rows);

FuseArgs fuse_args(pced_ctx* c, const float* logits, int32_t* tokens_out, int tok_stride, const pced_step_out* extra,
                   int nblk);
// The device form of a caller's adjustments.
pced_status adjust_args(const pced_ctx* c, const pced_adjust* d, AdjustArgs* out);
// Dynamic beta from `logits`, summed, ready for a later launch.
pced_status run_beta(pced_ctx* c, const float* logits, hipStream_t st);

}  // namespace pced
