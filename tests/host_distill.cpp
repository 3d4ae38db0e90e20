// csrc/distill_geometry.hpp for the host: that no call's layout exceeds what the sizing call answers.
#include "../paper_2105_07829_amd/csrc/distill_geometry.hpp"
using namespace bpc;
extern "C" {
uint64_t dg_needed(uint64_t rows, uint32_t vocab, int dtype, uint64_t stride, int step) {
  return distill_ws(rows, cut_rows(rows, vocab, dtype, stride, step != 0)).total;
}
void dg_cut(uint64_t rows, uint32_t vocab, int dtype, uint64_t stride, int step, uint32_t *chunks, uint32_t *vecs, uint32_t *nv) {
  const Cut c = cut_rows(rows, vocab, dtype, stride, step != 0);
  *chunks = c.chunks;
  *vecs = c.vecs;
  *nv = row_vecs(vocab, dtype, stride);
}
}
