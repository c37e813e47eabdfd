// Launchers that write down what they are asked to launch, in place of dv_quant.hip,
// dv_attend.hip and dv_evict.hip: linked with dv_attn.cpp they make a library whose
// calls run without a GPU (tests/test_attn_dispatch_cpu.py).  One line per launch.
#include <stdio.h>

#include <string>

#include "../../paper_2403_01876_amd/csrc/dv_attn_internal.h"

namespace {

std::string g_log, g_out;

template <typename... T>
hipError_t record(const char* format, T... values) {
  char line[256];
  snprintf(line, sizeof line, format, values...);
  g_log += line;
  return hipSuccess;
}

}  // namespace

namespace dv {

hipError_t launch_quant(const QuantArgs& a, uint32_t nslabs, hipStream_t) {
  return record("quant b0=%d nseq=%d items=%d lanes=%d rows=%u\n", a.b0, a.nseq, a.items,
                1 << a.lanes_log2, nslabs);
}
hipError_t launch_attend_split(const AttendArgs& a, int rt, bool direct, hipStream_t) {
  return record("split b0=%d nseq=%d items=%d rt=%d chunk=%d direct=%d\n", a.b0, a.nseq, a.items,
                rt, a.chunk, (int)direct);
}
hipError_t launch_attend_join(const AttendArgs& a, int rows, hipStream_t) {
  return record("join b0=%d nseq=%d items=%d rows=%d\n", a.b0, a.nseq, a.items, rows);
}
hipError_t launch_attend_tile(const AttendArgs& a, bool direct, hipStream_t) {
  return record("tile b0=%d nseq=%d items=%d chunk=%d direct=%d\n", a.b0, a.nseq, a.items, a.chunk,
                (int)direct);
}
hipError_t launch_attend_weigh(const AttendArgs& a, int shares, hipStream_t) {
  return record("weigh b0=%d nseq=%d items=%d shares=%d\n", a.b0, a.nseq, a.items, shares);
}
hipError_t launch_evict_select(const EvictArgs& a, hipStream_t) {
  return record("select b0=%d nseq=%d heads=%d rows=%d most=%d\n", a.b0, a.nseq, a.s.heads, a.nl,
                a.most);
}
hipError_t launch_evict_move(const EvictArgs& a, hipStream_t) {
  return record("move b0=%d nseq=%d items=%d rows=%d group=%d\n", a.b0, a.nseq, a.items, a.nl,
                a.group);
}

}  // namespace dv

// The launches since the last call of this, a line each.
extern "C" __attribute__((visibility("default"))) const char* dispatch_record_take() {
  g_out.swap(g_log);
  g_log.clear();
  return g_out.c_str();
}
