// Host+device description of distillation calls: records of rows of logits, how rows are cut into
// chunks, workspace.
#pragma once
#include "geometry.hpp"

namespace bpc {

constexpr uint32_t kMaxVocab = 1u << 24;       // logits a row
constexpr uint32_t kMaxLogitsK = 1024;         // entries of a row's record
constexpr uint64_t kMaxRows = (1u << 22) - 1;  // (times 1024 threads a row: below 2^32, what a launch can count)
constexpr uint64_t kMaxRowStride = 1ull << 40; // elements
constexpr uint32_t kChunkVecs = 16384;         // most 16-byte vectors of a row that one workgroup handles

inline size_t logits_stride(const bpc_distill_t *d) {
  const uint64_t words = d->kind == BPC_TOPK ? ru4(d->k) : ru4(cdiv(d->k, 2));
  return (size_t)(kHeaderBytes + 4 * ru4(d->k) + 4 * words);
}
inline bool distill_valid(const bpc_distill_t *d) {
  if (!d) return false;
  if (d->kind != BPC_TOPK && d->kind != BPC_TOPK16) return false;
  if (d->tail != BPC_TAIL_DROP && d->tail != BPC_TAIL_REST) return false;
  if (d->vocab == 0 || d->k == 0) return false;
  // (1 / temperature and its product with log2 e are formed in f32)
  if (!(d->temperature >= 1e-30f && d->temperature <= 1e30f)) return false;
  return isfinite(d->soft_weight) && isfinite(d->hard_weight);
}
inline bool distill_built(const bpc_distill_t *d, uint64_t rows) {
  return d->vocab <= kMaxVocab && d->k <= kMaxLogitsK && rows <= kMaxRows;
}

inline uint32_t elem_bytes(int dtype) { return dtype == BPC_F32 ? 4 : 2; }
// Vectors of the row that spans most of them: rows may start anywhere in a 16-byte block unless their stride is a
// multiple of one.
inline uint32_t row_vecs(uint32_t vocab, int dtype, uint64_t row_stride) {
  const uint32_t e = 16 / elem_bytes(dtype);
  return (uint32_t)cdiv(vocab + (row_stride % e ? e - 1 : 0), e);
}

constexpr uint32_t kGradVecs = 16384;   // vectors of a row whose gradient one workgroup writes

// Rows are cut into chunks, a workgroup each, where one workgroup may not have them whole.
struct Cut {
  uint32_t chunks;   // a row
  uint32_t vecs;     // of a chunk
};
inline Cut cut_rows(uint64_t rows, uint32_t vocab, int dtype, uint64_t row_stride) {
  (void)rows;
  Cut c;
  c.chunks = (uint32_t)cdiv(row_vecs(vocab, dtype, row_stride), kChunkVecs);
  c.vecs = (uint32_t)cdiv(row_vecs(vocab, dtype, row_stride), c.chunks);
  return c;
}

constexpr uint32_t kPartialFloats = 4;   // what a chunk hands on: largest logit, sums at both temperatures
constexpr uint32_t kStatsFloats = BPC_DISTILL_STATS_BYTES / 4;

// Workspace of the student's calls: partial sums of the chunks, statistics of the rows.
struct DistillWs {
  size_t partial, stats, total;
};
inline DistillWs distill_ws(uint64_t rows, const Cut &cut) {
  DistillWs w{};
  size_t at = 0;
  w.partial = at;
  if (cut.chunks > 1) at += (size_t)rows * cut.chunks * kPartialFloats * 4;
  at = (at + 255) / 256 * 256;
  w.stats = at;
  if (cut.chunks > 1) at += (size_t)rows * BPC_DISTILL_STATS_BYTES;
  w.total = (at + 255) / 256 * 256;
  return w;
}

// Of every call of `rows` rows (or fewer) whatever the type: what bpc_distill_workspace_bytes answers.
inline size_t distill_workspace(const bpc_distill_t *d, uint64_t rows) {
  size_t most = 256;
  for (int dtype = BPC_F32; dtype <= BPC_BF16; ++dtype) {
    for (uint64_t stride = 0; stride < 2; ++stride) {   // aligned rows and others
      const size_t s = distill_ws(rows, cut_rows(rows, d->vocab, dtype, stride)).total;
      if (s > most) most = s;
    }
  }
  return most;
}

}  // namespace bpc
