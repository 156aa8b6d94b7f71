// The host code of sampling (csrc/pced_sample_api.cpp) over the recording stand-ins of
// layer_path.cpp and these. Compiled by tests/test_sample_path.py.
#include "layer_path.cpp"

#include "pced_host.h"

namespace {
const pced_ctx* g_ctx;  // whose workspace the launches are held against
// the region [p, p + bytes) within the workspace's [from, to)
long inside(const void* p, size_t bytes, size_t from, size_t to) {
  const char *a = (const char*)p, *b = g_ctx->ws;
  return a >= b + from && a + bytes <= b + to;
}
}  // namespace

extern "C" void watch(const pced_ctx* c) { g_ctx = c; }

namespace pced {
hipError_t launch_fuse_scores(const FuseArgs& a, const AdjustArgs& d, const SampleArgs& p, int B, hipStream_t, const Timing*) {
  const Layout& l = g_ctx->lay;
  const size_t n = (size_t)B * p.V * 4;
  return note("fuse_scores", a.nblk, d.mask != nullptr, inside(p.scores, n, l.logits, l.rho), inside(p.who, n, l.logits, l.rho),
              (char*)p.scores + n <= (char*)p.who, inside(p.bins, B * sizeof(SampleBins), l.smp_bins, l.smp_list),
              inside(p.list, 2 * n, l.smp_list, l.total), inside(p.part, (size_t)B * a.nblk * 8, l.fuse_part, l.lse_part));
}
hipError_t launch_sample(const SampleArgs& p, int B, int, hipStream_t, const Timing*) {
  return note("sample", B, p.shift, p.nblk, p.top_k != nullptr, p.kept != nullptr);
}
}  // namespace pced
