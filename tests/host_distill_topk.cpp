// The teacher's side of csrc/distill_geometry.hpp for the host: which form a call takes and what it needs.
#include "../paper_2105_07829_amd/csrc/distill_geometry.hpp"
using namespace bpc;
extern "C" {
void dt_plan(uint64_t rows, uint32_t vocab, uint32_t k, int dtype, uint64_t stride, uint64_t *out) {
  const TopkPlan p = topk_plan(rows, vocab, k, dtype, stride);
  const uint64_t v[10] = {(uint64_t)p.form, p.threads, p.lds, p.lanes, p.n_groups, p.cap, p.region, p.few, p.ws,
                          row_vecs(vocab, dtype, stride)};
  for (int i = 0; i < 10; ++i) out[i] = v[i];
}
}
