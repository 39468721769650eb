// Tensor-core path of gated linear attention, host side: workspace, segments, launches.
#include "tc.cuh"

namespace ha_la {
namespace gla {

// Segments that a sequence is cut into where there are few (sequence, V-head) pairs: their sums are taken at the same time, chained, and then
// all segments are walked at the same time.  `units`: CTAs without.  us as measured: a step of the sums 0.9, of the walk 2.8, of the states for the
// backward pass 2.0; the two further launches 16 and 14.  16 heads, whole and in segments: 512 tokens 19 and 24 us, 1024 30 and 26, 4096 98 and 40;
// backward 1024 tokens 43 and 45 us, 1536 63 and 59, 4096 145 and 109; four rows of 2048 (two segments at most) 55 and 63.
int segments(const Problem& p, bool back) {
  const long long units = (long long)p.N * p.HV * (back ? 2 : 1);
  const int steps = p.max_seq_chunks, most = units > 0 ? (int)(sm_count() / units) : 0;
  const double sum = 0.9, walk = back ? 2.0 : 2.8, launches = back ? 14 : 16;
  double best = walk * steps;
  int s = 1;
  for (int i = 2; i <= most && i <= steps; ++i) {
    const double us = (sum + walk) * ((steps + i - 1) / i) + launches;
    if (us < best) { best = us; s = i; }
  }
  return s;
}

size_t tc_bytes(const Problem& p, bool back, TcWork* tw, Work* w, void* base) {
  char* b = reinterpret_cast<char*>(base);
  size_t at = 0;
  auto take = [&](auto** ptr, size_t bytes) {
    if (ptr) *ptr = reinterpret_cast<std::remove_reference_t<decltype(**ptr)>*>(b + at);
    at = align_up(at + bytes, 1024);
  };
  const size_t units = (size_t)p.max_chunks * p.HV;
  const int nseg = segments(p, back);
  const size_t parts = nseg > 1 ? (size_t)p.N * p.HV * nseg : 0;
  take(tw ? &tw->part : nullptr, parts * 65536);
  take(tw ? &tw->total : nullptr, parts * 4);
  if (back) {
    take(tw ? &tw->image : nullptr, units * kTileBytes * 2);
    const int per = heads_per_run(p);
    const size_t parts_of = p.HV / per != p.HK ? (size_t)p.T_total * (p.HV / per) * 128 * 4 : 0;
    take(tw ? &tw->image_back : nullptr, units * kTileBytes * 2);
    take(tw ? &tw->part_back : nullptr, parts * 65536);
    take(tw ? &tw->total_back : nullptr, parts * 4);
    take(tw ? &tw->sums : nullptr, local_back_bytes());
    take(tw ? &tw->shared : nullptr, per > 1 ? (size_t)sm_count() * 2 * 65536 : 0);
    take(w ? &w->dq : nullptr, parts_of);
    take(w ? &w->dk : nullptr, parts_of);
  }
  return at;
}

namespace {

cudaError_t make(TcCall* t, const Call& c, PlanView plan, const TcWork& w) {
  t->c = &c;
  t->w = w;
  t->nseg = segments(c.p, c.back);
  t->seqs = {plan.seq_tok0, plan.seq_len, plan.seq_chunk0, plan.seq_order, c.p.T_row, c.p.max_seq_chunks};
  if (!make_map_tile(&t->q, c.a.q, c.p.T_total, c.p.HK) || !make_map_tile(&t->k, c.a.k, c.p.T_total, c.p.HK) ||
      !make_map_tile(&t->v, c.a.v, c.p.T_total, c.p.HV) || !make_map_tile(&t->d_o, c.back ? c.a.do_ : c.a.v, c.p.T_total, c.p.HV) ||
      !make_map_tile(&t->o, c.back ? c.a.v : c.a.o, c.p.T_total, c.p.HV))
    return cudaErrorInvalidValue;
  return cudaSuccess;
}

cudaError_t sums(const TcCall& t, cudaStream_t stream) {   // the segments' start states
  const Call& c = *t.c;
  cudaError_t e = launch_tc_states(t, true, stream);
  if (e == cudaSuccess) e = launch_chain(t.w.total, t.w.part, c.a.h0, t.nseg, c.p.N, c.p.HV, 16384, false, stream);
  if (e == cudaSuccess && c.back) e = launch_chain(t.w.total_back, t.w.part_back, c.a.dhT, t.nseg, c.p.N, c.p.HV, 16384, true, stream);
  return e;
}

}  // namespace

cudaError_t launch_tc_forward(const Call& c, PlanView plan, const TcWork& w, cudaStream_t stream) {
  if (c.p.T_total == 0) return launch_combine(c, false, stream);   // (no token, no tensor map: hT = h0)
  TcCall t;
  cudaError_t e = make(&t, c, plan, w);
  if (e == cudaSuccess && t.nseg > 1) e = sums(t, stream);
  return e == cudaSuccess ? launch_tc_walk(t, stream) : e;
}

cudaError_t launch_tc_backward(const Call& c, PlanView plan, const TcWork& w, cudaStream_t stream) {
  if (c.p.T_total == 0) return launch_combine(c, true, stream);
  TcCall t;
  cudaError_t e = make(&t, c, plan, w);
  if (e == cudaSuccess && t.nseg > 1) e = sums(t, stream);
  if (e == cudaSuccess) e = launch_tc_states(t, false, stream);
  if (e == cudaSuccess) e = launch_tc_local_back(t, stream);
  return e == cudaSuccess ? launch_head_sums(c, c.p.HV / heads_per_run(c.p), stream) : e;
}

}  // namespace gla
}  // namespace ha_la
