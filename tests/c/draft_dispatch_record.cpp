// Launchers that write down what they are asked to launch, in place of the kernels of the
// operators over drafted tokens: linked with dv_attn.cpp and dv_draft.cpp they make a
// library whose calls run without a GPU (tests/test_draft_dispatch_cpu.py).  One line per
// launch, and one for each of its sequences where its table is of interest.
#include <stdio.h>

#include <string>

#include "../../paper_2403_01876_amd/csrc/dv_draft_internal.h"

namespace {

std::string g_log, g_out;

template <typename... T>
void note(const char* format, T... values) {
  char line[256];
  snprintf(line, sizeof line, format, values...);
  g_log += line;
}
template <typename... T>
hipError_t record(const char* format, T... values) {
  note(format, values...);
  return hipSuccess;
}

}  // namespace

namespace dv {

hipError_t launch_quant(const QuantArgs&, uint32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_evict_select(const EvictArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_evict_move(const EvictArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attend_weigh(const AttendArgs& a, int, hipStream_t) { return record("weigh b0=%d\n", a.b0); }
hipError_t launch_attend_join(const AttendArgs& a, int rows, hipStream_t) {
  return record("join items=%d rows=%d\n", a.items, rows);
}
static hipError_t attend(const char* what, const AttendArgs& a, bool direct) {
  note("%s b0=%d nseq=%d items=%d chunk=%d direct=%d row0=%d parent=%lld\n", what, a.b0, a.nseq,
         a.items, a.chunk, (int)direct, a.row0, (long long)(intptr_t)a.parent);
  for (int i = 0; i < a.nseq; ++i)
    note("tree b=%d nq=%d tok=%d len=%d item=%d\n", a.soff[i] >> 8, a.soff[i] & 255, a.tok[i],
           a.len[i], a.item[i]);
  return hipSuccess;
}
hipError_t launch_attend_split(const AttendArgs& a, int, bool direct, hipStream_t) {
  return attend("split", a, direct);
}
hipError_t launch_attend_tile(const AttendArgs& a, bool direct, hipStream_t) {
  return attend("tile", a, direct);
}
hipError_t launch_verify_sums(const VerifyArgs& a, hipStream_t) {
  return record("sums b0=%d nseq=%d row0=%d rows=%d pieces=%d parts=%d\n", a.b0, a.nseq, a.row0,
                a.tok[kQSeqs], a.pieces, a.parts);
}
hipError_t launch_verify_walk(const VerifyArgs& a, hipStream_t) {
  note("walk b0=%d nseq=%d row0=%d rows=%d pieces=%d parts=%d\n", a.b0, a.nseq, a.row0,
         a.tok[kQSeqs], a.pieces, a.parts);
  for (int i = 0; i < a.nseq; ++i)
    note("rows tok=%d n=%d zero=%d\n", a.tok[i], a.tok[i + 1] - a.tok[i], (int)(a.scale2[i] == 0.));
  return hipSuccess;
}
hipError_t launch_keep(const KeepArgs& a, uint32_t layers, hipStream_t) {
  note("keep b0=%d nseq=%d l0=%d layers=%u heads=%d path=%lld count=%lld\n", a.b0, a.nseq, a.l0,
         layers, a.q.heads, (long long)(intptr_t)a.path, (long long)(intptr_t)a.count);
  for (int i = 0; i < a.nseq; ++i)
    note("kept base=%d tok=%d n=%d\n", a.base[i], a.tok[i], a.tok[i + 1] - a.tok[i]);
  return hipSuccess;
}
hipError_t launch_quant_out(const QuantArgs& a, uint32_t nslabs, hipStream_t) {
  return record("out b0=%d nseq=%d items=%d lanes=%d slab0=%d rows=%u wire=%lld\n", a.b0, a.nseq,
                a.items, 1 << a.lanes_log2, a.slab0, nslabs, (long long)(intptr_t)a.wire);
}

}  // namespace dv

// The launches since the last call of this, a line each.
extern "C" __attribute__((visibility("default"))) const char* dispatch_record_take() {
  g_out.swap(g_log);
  g_log.clear();
  return g_out.c_str();
}
