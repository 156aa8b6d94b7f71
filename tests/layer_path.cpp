// The host code of the layer-wise calls (csrc/pced_layer_api.cpp) over the recording
// stand-ins of host_path.cpp and these. Compiled by tests/test_layer_path.py.
#include "host_path.cpp"

namespace pced {
hipError_t launch_append_rows(const AppendRowsArgs& a, bool, hipStream_t, const Timing*) {
  return note("append_rows", a.layer0, a.n_layers, a.n_tokens, a.slots, a.codes != nullptr, a.t, (long)a.q_row);
}
hipError_t launch_summarize(const SummaryArgs& a, bool, hipStream_t) { return note("summarize", a.span, a.behind, a.t); }
hipError_t launch_page_select(const AttendArgs& a, bool score, hipStream_t, const Timing*) {
  return note("select", a.layer, a.launch_layers, a.group0, a.n_groups, score, a.gt);
}
hipError_t launch_attend(const AttendArgs& a, bool pick, hipStream_t, const Timing*, const Timing*) {
  if (pick) note("select", a.layer, a.launch_layers, a.group0, a.n_groups, 1, a.gt);
  const size_t items = (size_t)a.n_groups * a.gt * a.launch_layers * a.n_kv_heads;
  const size_t end = a.parts > 1 ? (uintptr_t)(a.part_ml + items * a.parts * a.group * 2) : (uintptr_t)(a.list + 1);
  return note("attend", a.layer, a.launch_layers, a.group0, a.n_groups, a.parts, a.part_pages, (long)end, (long)(uintptr_t)a.scores);
}
hipError_t launch_adjust(const AdjustArgs& a, int, int max_rows, int, hipStream_t) { return note("adjust", max_rows, (long)a.mask_row); }
int adjusted_slice(int, int, int) { return 256; }
hipError_t launch_fuse_adjusted(const FuseArgs& a, const AdjustArgs&, int, hipStream_t, const Timing*, const Timing*) {
  return note("fuse_adjusted", a.none_token);
}
}  // namespace pced
