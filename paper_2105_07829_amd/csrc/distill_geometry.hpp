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

constexpr uint32_t kFewRows = 32;       // most rows of a call that are cut though a workgroup could have each whole,
constexpr uint32_t kLongVecs = 4096;    // ... from this length on, in vectors,
constexpr uint32_t kLeastVecs = 512;    // ... into chunks of at least this,
constexpr uint32_t kFillChunks = 256;   // ... until every compute unit has one (512 or 1024: the same within 2 %)
constexpr uint32_t kGradVecs = 16384;   // vectors of a row whose gradient one workgroup writes

// How the sums over a row are formed: by one workgroup, which keeps a bit a logit in LDS, or by one for each of its
// chunks and a launch that joins them.
struct Cut {
  uint32_t chunks;   // a row
  uint32_t vecs;     // of a chunk, at most kChunkVecs where there are several
};
constexpr uint32_t kMarkWords = 1u << 18;   // logits that have a bit in LDS
inline Cut cut_rows(uint64_t rows, uint32_t vocab, int dtype, uint64_t row_stride, bool step) {
  const uint32_t nv = row_vecs(vocab, dtype, row_stride), e = 16 / elem_bytes(dtype);
  const bool whole = (uint64_t)nv * e <= kMarkWords;
  // Few long rows are cut, too.  Loss: 8 x 151,936 bf16 9.4 us cut and 16.1 whole, 1 x 50,257 9.0 and 10.4; 64 x 50,257
  // 11.5 and 11.0.  Loss and gradient, in three launches: 10 x 262,144 f32 24.5 and 29.2, so only very long ones.
  if (whole && (rows > kFewRows || nv < (step ? kChunkVecs + 1 : kLongVecs))) return {1, nv};
  uint64_t chunks = cdiv(kFillChunks, rows);   // for every compute unit
  const uint64_t most = cdiv(nv, kLeastVecs), least = cdiv(nv, kChunkVecs);
  chunks = chunks < most ? chunks : most;
  chunks = chunks > least ? chunks : least;
  return {(uint32_t)chunks, (uint32_t)cdiv(nv, chunks)};
}

// Rows of which the teacher's call keeps the largest logits and sums of groups: at most 4096 groups of at most 16
// vectors, and a bit a logit in the 32 KB that these take.
constexpr uint32_t kMostGroups = 4096, kGroupVecs = 16 * kMostGroups, kGroupWords = 64 * kMostGroups;

// The teacher's call: which form it takes, a workgroup a row, and what that needs.
enum class TopkForm {
  any,     // radix select
  dense,   // the whole row in LDS
  groups   // by largest logits and sums of groups
};
struct TopkPlan {
  TopkForm form;
  uint32_t threads;    // of a row's workgroup
  uint32_t lds;        // dynamic LDS of it, bytes
  uint32_t lanes;      // groups: neighbouring vectors of a group,
  uint32_t n_groups;   // ... groups of a row (of whole loads: four vectors a thread),
  uint32_t cap;        // ... candidates there is room for,
  uint32_t region;     // ... bytes of LDS for the groups' keys and sums, later the indices level with the k-th, then a bit a
                       // logit (in whole quads of words a thread)
  bool few;            // groups: by workgroups for every compute unit, in a launch of their own,
  size_t ws;           // ... through this much workspace
};
constexpr uint32_t kTopThreads = 256;     // of dense rows, of rows by the radix select, of the launch for few rows' groups
constexpr uint32_t kDenseVocab = 15360;   // most logits of a row in LDS (60 KB)
inline TopkPlan topk_plan(uint64_t rows, uint32_t vocab, uint32_t k, int dtype, uint64_t row_stride) {
  const uint32_t nv = row_vecs(vocab, dtype, row_stride), e = 16 / elem_bytes(dtype);
  TopkPlan p{};
  p.threads = kTopThreads;
  if (nv > kGroupVecs || nv * e > kGroupWords) {
    p.form = TopkForm::any;
    return p;
  }
  if (nv < 2 * k && vocab <= kDenseVocab) {
    p.form = TopkForm::dense;
    p.lds = 4 * nv * e;
    return p;
  }
  p.form = TopkForm::groups;
  // What follows the pass over a row costs every wave about the same, so short rows of few entries take one wave, where
  // there are rows enough (64 / 256 threads: 16000 x 9000 bf16, k = 20, 90 / 149 us; 4096 x 30522 f16 65 / 74; f32 128 /
  // 98; k = 300 191 / 120).  Others take 256 threads where they fill the device (512: 119 us for 98 of 4096 x 50257
  // bf16), and 1024 where they do not (one row of 50,257 f32 20 us with 256; a compute unit has room for one such
  // workgroup: 256 / 257 / 511 / 512 rows of 50,257 bf16 19.2 / 30.2 / 36.0 / 25.1 us).
  p.threads = nv <= 512 || (rows >= 512 && nv + 8 * k <= 4096) ? 64 : rows >= 512 ? 256 : 1024;
  // The largest groups of which there are still two or more for each entry (then some 1.4 candidates an entry pass);
  // never more than kMostGroups.
  p.lanes = nv > 8 * kMostGroups ? 16 : nv >= 16 * k ? 8 : nv >= 8 * k ? 4 : nv >= 4 * k ? 2 : 1;
  p.n_groups = (uint32_t)cdiv(nv, 4 * p.threads) * 4 * p.threads / p.lanes;
  p.cap = 2 * (uint32_t)ru4(k) + 256;
  const uint32_t words = (uint32_t)cdiv((uint64_t)nv * e, 128 * p.threads) * 4 * p.threads;
  p.region = 8 * p.n_groups > 4 * words ? 8 * p.n_groups : 4 * words;
  if (p.region < 4 * p.cap) p.region = 4 * p.cap;
  p.lds = p.region + 8 * p.cap + 2 * p.n_groups;
  p.few = rows <= kFewRows && nv >= kLongVecs;
  p.ws = p.few ? (size_t)rows * p.n_groups * 8 : 0;
  return p;
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

// Enough for every call of `rows` rows or fewer, whatever the type and the stride: what bpc_distill_workspace_bytes
// answers.  (cut_rows makes at most rows * (chunks that a row needs) chunks, or kFillChunks + rows.)
inline size_t distill_workspace(const bpc_distill_t *d, uint64_t rows) {
  const uint64_t nv = row_vecs(d->vocab, BPC_F32, 1);   // (the type with most vectors, unaligned)
  if (nv < kLongVecs && nv <= kChunkVecs) return 256;
  const uint64_t whole = rows * cdiv(nv, kChunkVecs), fill = kFillChunks + rows;
  const size_t partial = (size_t)(whole > fill ? whole : fill) * kPartialFloats * 4;
  const size_t student = (partial + 255) / 256 * 256 + ((size_t)rows * BPC_DISTILL_STATS_BYTES + 255) / 256 * 256;
  const size_t teacher = (size_t)(rows < kFewRows ? rows : kFewRows) * kMostGroups * 8;
  return student > teacher ? student : teacher;
}

}  // namespace bpc
