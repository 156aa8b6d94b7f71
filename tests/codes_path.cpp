// The host code of caches in 8 bits (csrc/pced_cache8_api.cpp) over the recording stand-ins of
// layer_path.cpp and these. Compiled by tests/test_codes_path.py.
#include "layer_path.cpp"

#include "pced_host.h"

extern "C" {
// first and past-the-last address of the region that the attention may use
long room_begin(const pced_ctx* c) { return (long)(uintptr_t)(c->ws + c->lay.part_acc); }
long room_end(const pced_ctx* c) { return (long)(uintptr_t)(c->ws + c->lay.part_acc + c->lay.part_acc_bytes); }
}

namespace pced {
hipError_t launch_load8(const LoadArgs& a, const Cache8Args& c, int n_items, hipStream_t) {
  return note("load_codes", n_items, a.items != nullptr, a.layer0, a.n_layers, a.page0, a.one_len, c.code, c.ring);
}
hipError_t launch_append8(const AppendRowsArgs& a, const Cache8Args& c, hipStream_t, const Timing*) {
  return note("append_codes", a.layer0, a.n_layers, a.n_tokens, a.slots, c.ring, a.t, a.max_pages, a.kpool == c.k_open);
}
hipError_t launch_attend8(const Attend8Args& a, hipStream_t, const Timing*, const Timing*) {
  if (a.parts > 1) {
    // what the launch's items use, as the kernels index it
    const size_t states = (size_t)a.launch_seqs * a.n_groups * a.launch_layers * a.n_kv_heads * a.parts * a.gt * a.group;
    note("acc", (long)(uintptr_t)a.part_acc, (long)((uintptr_t)a.part_acc + states * a.head_dim * 4));
    note("ml", (long)(uintptr_t)a.part_ml, (long)((uintptr_t)a.part_ml + states * 8));
  }
  note("attend_split", a.parts, a.part_pages, a.gt, a.tiles, a.seq_parts);
  return note("attend_codes", a.layer, a.launch_layers, a.seq0, a.launch_seqs, a.group0, a.n_groups);
}
hipError_t launch_read8(const ReadCacheArgs& a, const Cache8Args&, int len, hipStream_t) {
  return note("read_codes", a.seq, a.layer, a.start, a.count, len);
}
}  // namespace pced
