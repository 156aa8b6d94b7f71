// The host code of the layer-wise calls over stand-ins that record where every launch of
// pced_attend reads and writes in the workspace. Compiled by tests/test_layer_room.py.
#include "host_path.cpp"

#include "pced_host.h"

namespace {
// What a launch uses of its scores, page lists and partial states, as their kernels index them: an item is a
// (token, layer, kv-head), row `items - 1` the last.
void use(const char* name, const void* p, size_t bytes) {
  if (bytes) note(name, (long)(uintptr_t)p, (long)((uintptr_t)p + bytes));
}
size_t items_of(const pced::AttendArgs& a) { return (size_t)a.n_groups * a.gt * a.launch_layers * a.n_kv_heads; }
}  // namespace

extern "C" {
// first and past-the-last address of the region that the calls may use
long room_begin(const pced_ctx* c) { return (long)(uintptr_t)(c->ws + c->lay.part_acc); }
long room_end(const pced_ctx* c) { return (long)(uintptr_t)(c->ws + c->lay.part_acc + c->lay.part_acc_bytes); }
long next_region(const pced_ctx* c) { return (long)(uintptr_t)(c->ws + c->lay.part_ml); }
}

namespace pced {
hipError_t launch_append_rows(const AppendRowsArgs& a, bool, hipStream_t, const Timing*) { return note("append_rows", a.layer0); }
hipError_t launch_summarize(const SummaryArgs& a, bool, hipStream_t) { return note("summarize", a.span); }
hipError_t launch_page_select(const AttendArgs& a, bool score, hipStream_t, const Timing*) {
  note("choice", a.layer, a.launch_layers, a.group0, a.n_groups, score, a.score_row);
  if (score && a.score_row > kPickPages) use("scores", a.scores, items_of(a) * a.score_row * 4);
  if (!a.pages_out) use("list", a.list, items_of(a) * a.n_pages * 4);
  return hipSuccess;
}
hipError_t launch_attend(const AttendArgs& a, bool pick, hipStream_t, const Timing*, const Timing*) {
  note("attend", a.layer, a.launch_layers, a.group0, a.n_groups, a.parts, a.part_pages, pick, a.gt);
  if (a.parts > 1) {
    use("acc", a.part_acc, items_of(a) * a.parts * a.group * a.head_dim * 4);
    use("ml", a.part_ml, items_of(a) * a.parts * a.group * 8);
  }
  return hipSuccess;
}
hipError_t launch_adjust(const AdjustArgs&, int, int, int, hipStream_t) { return note("adjust"); }
int adjusted_slice(int, int, int) { return 256; }
hipError_t launch_fuse_adjusted(const FuseArgs&, const AdjustArgs&, int, hipStream_t, const Timing*, const Timing*) {
  return note("fuse_adjusted");
}
}  // namespace pced
