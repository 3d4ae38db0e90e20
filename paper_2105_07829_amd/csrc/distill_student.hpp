// Student side of the distillation from top logits: loss of a row against the teacher's record and
// its gradient.
//
// With c = 1 / temperature and S the listed words, everything a row needs of its unlisted words is
// their largest logit m_R, R = sum exp((s_j - m_R) c) and H_R = sum exp(s_j - m_R): one pass that keeps
// a running maximum and rescales its sums when that grows.  The listed words (at most 1024) are
// gathered apart, so that the mass of the rest is never formed as a difference 1 - sum p_i, which
// would lose all of it where the listed words hold nearly everything.  For that the pass has to
// leave the listed words out: a bit a word in LDS says which (with TAIL_DROP the rest is not needed,
// and the pass takes the whole row).  The gradient of an unlisted word is
//   w exp((s_j - m_R) c) a c [exp((m_R - m) c) / Z - q_R / R] + w b exp(s_j - m_R) exp(m_R - m) / H,
// two coefficients a row; the listed words and the label are written apart, after the others.
//
// What bounds it: the loss reads 2 or 4 bytes a logit for 7 to 9 vector instructions, so 4096 x 50257
// bf16 with hard labels (68 us, 353 MB) is bound by vector issue (88 % busy) and smaller calls by the
// chain record -> listed logits -> sums -> logarithms of a row; the gradient (136 us, 765 MB, 5.6 TB/s) by
// the memory.  Both in one call: rows of which a compute unit holds two or more stay in registers (2048 x
// 30522 f16 54 us for 225 MB), longer ones are read twice, the second time from the last-level cache (8192 x
// 131072 bf16 953 us for 4.3 GB).  Not kept, measured on that last case: workgroups that take row after
// row and load the next row while they write a gradient (1140 us: all of them read and write at the same
// time); listed logits and gradients passed through a table in LDS instead of a gather and a scatter (1178).
#pragma once
#include "distill.hpp"
#include "distill_call.hpp"

namespace bpc {

// Statistics of a row, as bpc_distill_loss hands them to bpc_distill_grad.
struct Stats {
  float m, inv_z, inv_h;   // of the whole row: largest logit, 1 / sum at the temperature, at temperature 1
  float m_r, c_soft, c_hard;  // the unlisted words: reference and coefficients above (without weights)
  float inv_q;             // 1 / Q of the teacher; 0: no soft term
  float pad;
};
static_assert(sizeof(Stats) == BPC_DISTILL_STATS_BYTES, "");

struct Args {
  DistillCall a;
  float c, c2;        // 1 / temperature, times log2 e
  uint32_t chunks, vecs;
};

// Largest of a set of logits and the sums of their exponentials relative to it.
struct Part {
  float m = kNegInf, s = 0.0f, h = 0.0f;
};

// A bit a word of a stretch of a row: listed.  `bits` starts at vector v0.
template <int DT>
struct Marks {
  static constexpr int E = Num<DT>::E;
  const uint8_t *bits;   // NULL: nothing is marked
  uint32_t v0;
  __device__ uint32_t of(uint32_t v) const {
    const uint32_t i = v - v0;
    return E == 8 ? bits[i] : (bits[i >> 1] >> (4 * (i & 1))) & 15u;
  }
  // Marked words count as masked.  N vectors, `apart` apart, from v on.
  template <int N>
  __device__ void apply(uint32_t v, uint32_t apart, u32x4 *w) const {
    if (!bits) return;
    uint32_t b[N], any = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) any |= b[u] = of(v + u * apart);
    if (any) {
#pragma unroll
      for (int u = 0; u < N; ++u) w[u] = Num<DT>::mask(w[u], b[u]);
    }
  }
  __device__ void apply_to(uint32_t v, float *x) const {
    if (!bits) return;
    const uint32_t b = of(v);
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = (b >> k) & 1 ? kNegInf : x[k];
  }
};

// ---- sums over a stretch of a row, each thread its own

// The hard term of a call, which is at temperature 1: none; at the soft one's temperature; at its own; or at its own
// where that of the soft one is 2 or 4, so that its exponentials are the second and fourth powers of the soft one's
// (a product or two instead of a multiply-add and an exponential).  Powers / own, us: loss and gradient in one call of
// 2048 x 30522 f16 at temperature 2 55.3 / 61.0, at 4 57.7 / 61.0; of 4096 x 50257 bf16 178 / 183, without the rest 175 /
// 173; of 1024 x 32000 f32 48.6 / 49.8.  The loss of 4096 x 50257 bf16 81 / 89, without the rest 84 to 88 / 82; the
// gradient of 2048 x 30522 f16 48.6 / 60.2.
enum Hard { kNoHard, kSameHard, kOwnHard, kSquareHard, kFourthHard };
constexpr bool two_sums(int hard) { return hard >= kOwnHard; }
// 2^(x log2e - ref1) from e = 2^(x c2 - ref2) (ref1 = 2 ref2 or 4 ref2 where that is what it takes).
template <int HARD>
__device__ inline float hard_exp(float x, float e, float ref1) {
  if (HARD == kSquareHard) return e * e;
  if (HARD == kFourthHard) return (e * e) * (e * e);
  return base2_exp(x, kLog2e, ref1);
}

// With references of base 2 (see base2_ref).
struct FastSum : Part {
  template <int HARD, int N>
  __device__ void add(const float *x, float c2) {
    constexpr bool TWO = two_sums(HARD);
    float nm = m;
#pragma unroll
    for (int i = 0; i < N; ++i) nm = fmaxf(nm, x[i]);
    const float ref = base2_ref(nm, c2), ref1 = base2_ref(nm, kLog2e);
    s *= exp2_hw(base2_ref(m, c2) - ref);
    if (TWO) h *= exp2_hw(base2_ref(m, kLog2e) - ref1);
    m = nm;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = base2_exp(x[i], c2, ref);
      s += e;
      if (TWO) h += hard_exp<HARD>(x[i], e, ref1);
    }
  }
  // relative to the largest of all threads' instead
  template <bool TWO>
  __device__ void move_to(float all, float c2) {
    s *= exp2_hw(base2_ref(m, c2) - base2_ref(all, c2));
    if (TWO) h *= exp2_hw(base2_ref(m, kLog2e) - base2_ref(all, kLog2e));
    m = all;
  }
  // ... and to that logit itself, not its rounded multiple
  template <bool TWO>
  __device__ void settle(float c2) {
    if (m == kNegInf) return;
    s *= exp2_hw(-__builtin_fmaf(m, c2, -base2_ref(m, c2)));
    if (TWO) h *= exp2_hw(-__builtin_fmaf(m, kLog2e, -base2_ref(m, kLog2e)));
  }
};
// With differences formed first: for rows whose largest logit is far from 0 (a type's lowest value among them).
struct PlainSum : Part {
  template <bool TWO>
  __device__ void move_to(float nm, float c2) {
    const float d = m - ref_of(nm);
    s *= exp2_hw(d * c2);
    if (TWO) h *= exp2_hw(d * kLog2e);
    m = nm;
  }
  template <int HARD, int N>
  __device__ void add(const float *x, float c2) {
    constexpr bool TWO = two_sums(HARD);
    float nm = m;
#pragma unroll
    for (int i = 0; i < N; ++i) nm = fmaxf(nm, x[i]);
    move_to<TWO>(nm, c2);
    const float ref = ref_of(nm);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - ref;
      s += exp2_hw(d * c2);
      if (TWO) h += exp2_hw(d * kLog2e);
    }
  }
};

// The vectors beside a stretch's body.
template <int DT, int HARD, class Sum>
__device__ void add_edges(const Row<DT> &row, const Stretch &st, const Marks<DT> &marks, float c2, Sum *p) {
  uint32_t v;
  if (st.edge(&v)) {
    float x[Num<DT>::E];
    row.load_any(v, x);
    marks.apply_to(v, x);
    p->template add<HARD, Num<DT>::E>(x, c2);
  }
}

// Four vectors of a body a thread, T apart, from v on; what is past its end reads as masked.
template <int DT, int T, bool ONCE = true>
struct Four {
  u32x4 w[4];
  __device__ static u32x4 get(const Row<DT> &row, uint32_t v) { return ONCE ? row.load_once(v, threadIdx.x) : row.load(v, threadIdx.x); }
  __device__ void load(const Row<DT> &row, const Stretch &st, uint32_t v) {
    if (v + 4 * T <= st.b1) {
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = get(row, v + u * T);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        w[u] = Num<DT>::masked();
        if (v + u * T + threadIdx.x < st.b1) w[u] = get(row, v + u * T);
      }
    }
  }
};

// A thread's share of a stretch; `now`: the first four vectors, loaded by the caller before whatever else a row needs.
template <int DT, int HARD, int T, bool ONCE>
__device__ FastSum scan(const Row<DT> &row, const Stretch &st, Four<DT, T, ONCE> now, const Marks<DT> &marks, float c2) {
  constexpr int E = Num<DT>::E;
  FastSum p;
  uint32_t v = st.b0;
  while (v + 4 * T <= st.b1) {
    float x[4 * E];
    marks.template apply<4>(v + threadIdx.x, T, now.w);
#pragma unroll
    for (int u = 0; u < 4; ++u) Num<DT>::widen(now.w[u], x + u * E);
    v += 4 * T;
    if (v < st.b1) now.load(row, st, v);   // (the next four are on their way)
    p.add<HARD, 4 * E>(x, c2);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (v + u * T + threadIdx.x < st.b1) {
      float x[E];
      marks.template apply<1>(v + u * T + threadIdx.x, 0, &now.w[u]);
      Num<DT>::widen(now.w[u], x);
      p.add<HARD, E>(x, c2);
    }
  }
  add_edges<DT, HARD>(row, st, marks, c2, &p);
  return p;
}
template <int DT, int HARD, int T>
__device__ PlainSum scan_plain(const Row<DT> &row, const Stretch &st, const Marks<DT> &marks, float c2) {
  constexpr int E = Num<DT>::E;
  PlainSum p;
  for (uint32_t v = st.b0 + threadIdx.x; v < st.b1; v += T) {
    float x[E];
    Num<DT>::widen(row.load(0, v), x);
    marks.apply_to(v, x);
    p.add<HARD, E>(x, c2);
  }
  add_edges<DT, HARD>(row, st, marks, c2, &p);
  return p;
}

// ---- exchanges between the waves of a workgroup: sums of N values and maxima of M, in every thread

template <int T, int N, int M>
struct Exchange {
  float v[T / 64][N + M];
  __device__ void all(float *sums, float *most) {   // (one barrier; each Exchange is used once)
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i] = wave_all(sums[i], Plus());
#pragma unroll
    for (int i = 0; i < M; ++i) most[i] = wave_all(most[i], Larger());
    if (T == 64) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[threadIdx.x >> 6][i] = sums[i];
#pragma unroll
      for (int i = 0; i < M; ++i) v[threadIdx.x >> 6][N + i] = most[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i] = waves_all<T / 64>(&v[0][i], N + M, Plus());
#pragma unroll
    for (int i = 0; i < M; ++i) most[i] = waves_all<T / 64>(&v[0][N + i], N + M, Larger());
  }
};

// ---- what the teacher listed for a row, an entry or a few a thread

__device__ inline float weight_of(const Args &g, uint64_t r) { return g.a.weight ? uniform_load(g.a.weight + r) : 1.0f; }

constexpr uint32_t kOneWaveK = 256;   // most entries of rows that one wave handles (three registers an entry)

template <int DT, int T>
struct Listed {
  static constexpr int PER = T == 64 ? (int)kOneWaveK / 64 : (int)kMaxLogitsK / T;   // entries a thread, at most
  static constexpr uint32_t kNone = 0xffffffffu;
  uint32_t n;            // entries of the record
  uint32_t idx[PER];     // kNone: no entry, or one of no word
  float val[PER], s[PER];  // the teacher's value, the student's logit
  uint32_t label;        // kNone: no hard term
  float s_label;
  float rest;

  // The record and the label ...
  template <bool HARD>
  __device__ void request(const Args &g, uint64_t r) {
    const Record rec(g.a.messages, r, g.a.message_stride, g.a.k, g.a.half);
    n = rec.count(g.a.k);
    rest = g.a.rest_too ? rec.rest() : 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t e = threadIdx.x + i * T;
      if (e < g.a.k) {   // (the record has room for k entries: read before n is known)
        idx[i] = rec.idx(e);
        val[i] = rec.val(e);
      }
    }
    label = kNone;
    if (HARD) {
      const int64_t l = g.a.labels[r];
      if (l >= 0 && l < (int64_t)g.a.vocab) label = (uint32_t)l;
    }
  }
  // ... and the student's logits of the words [lo, hi) among them (all words for the sums over a row, those of a stretch
  // for its gradient: another stretch's gradient may just be written over the others).
  __device__ void gather(const Row<DT> &row, uint32_t lo, uint32_t hi) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (!(threadIdx.x + i * T < n && idx[i] >= lo && idx[i] < hi)) idx[i] = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (idx[i] != kNone) s[i] = Num<DT>::get(row.p + idx[i]);
    s_label = label != kNone && label >= lo && label < hi ? Num<DT>::get(row.p + label) : 0.0f;
  }
  template <bool HARD>
  __device__ void read(const Args &g, const Row<DT> &row, uint64_t r, uint32_t lo, uint32_t hi) {
    request<HARD>(g, r);
    gather(row, lo, hi);
  }
  // Marks the words of the vectors [v0, v1); barriers inside.
  __device__ void mark(const Row<DT> &row, uint32_t v0, uint32_t v1, uint32_t *bits) const {
    constexpr int E = Num<DT>::E;
    for (uint32_t w = threadIdx.x; w < ((v1 - v0) * E + 31) / 32; w += T) bits[w] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t at = idx[i] + row.off - v0 * E;   // (from the first word of vector v0)
      if (idx[i] != kNone && idx[i] + row.off >= v0 * E && at < (v1 - v0) * E) atomicOr(&bits[at >> 5], 1u << (at & 31));
    }
    __syncthreads();
  }
};

template <int T>
struct FinishLds {
  Exchange<T, 0, 2> most;
  Exchange<T, 5, 0> sums;
  Exchange<T, 1, 0> kl;
};

__device__ inline bool far(float m, float c2, bool two) {
  return m != kNegInf && !(fabsf(m) * fmaxf(c2, two ? kLog2e : 0.0f) < kFarRef);
}

// A thread's sums over a stretch relative to the largest logit m of all threads.
template <int DT, int HARD, int T>
__device__ Part settled(FastSum f, float m, const Row<DT> &row, const Stretch &st, const Marks<DT> &marks, float c2) {
  constexpr bool TWO = two_sums(HARD);
  if (far(m, c2, TWO)) {
    PlainSum q = scan_plain<DT, HARD, T>(row, st, marks, c2);
    q.template move_to<TWO>(m, c2);
    return q;
  }
  f.template move_to<TWO>(m, c2);
  f.template settle<TWO>(c2);
  return f;
}

// The row's loss and statistics from the sums of its unlisted words (TAIL_DROP: of all words), each thread's own.
// settle(m): a thread's sums relative
// to m, the largest unlisted logit of all (0 where that is -inf).
template <int DT, int HARD, int T, class Settle>
__device__ Stats finish(const Args &g, const Listed<DT, T> &list, float largest, const Settle &settle, float weight, float *loss,
                        FinishLds<T> &lds) {
  constexpr int PER = Listed<DT, T>::PER;
  constexpr bool TWO = two_sums(HARD);
  const bool rest_too = g.a.rest_too;
  float most[2] = {largest, kNegInf};
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (list.idx[i] != list.kNone) most[1] = fmaxf(most[1], list.s[i]);
  lds.most.all(nullptr, most);
  const Part p = settle(most[0]);
  // (TAIL_DROP: the listed words are in the sums already)
  const float m = rest_too ? fmaxf(most[0], most[1]) : most[0], ref = ref_of(m);
  float sums[5] = {p.s, TWO ? p.h : 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (list.idx[i] == list.kNone) continue;
    sums[2] += exp2_hw(list.val[i] * g.c2);
    if (rest_too) {
      const float d = list.s[i] - ref;
      sums[3] += exp2_hw(d * g.c2);
      if (TWO) sums[4] += exp2_hw(d * kLog2e);
    }
  }
  lds.sums.all(sums, nullptr);
  const float q = list.n == 0 || g.a.soft == 0.0f ? 0.0f : sums[2] + list.rest;   // 0: no soft term
  const float down = ref_of(most[0]) - ref;   // from the reference of the unlisted words to that of the row
  const float scale = most[0] == kNegInf ? 0.0f : exp2_hw(down * g.c2), scale1 = most[0] == kNegInf ? 0.0f : exp2_hw(down * kLog2e);
  // (nothing unlisted: the sums are 0 whatever the scale)
  const float z = (rest_too ? sums[0] * scale : sums[0]) + sums[3];
  const float h = TWO ? (rest_too ? sums[1] * scale1 : sums[1]) + sums[4] : z;
  const float log_z = logf(z);
  float kl[1] = {0.0f};
  if (q != 0.0f) {
    const float log_q = logf(q);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (list.idx[i] == list.kNone) continue;
      const float w = exp2_hw(list.val[i] * g.c2) / q;
      // log(q_i / p_i); a word that the teacher gives nothing counts nothing, whatever the student gives it
      if (w != 0.0f) kl[0] += w * ((list.val[i] - (list.s[i] - ref)) * g.c + (log_z - log_q));
    }
  }
  lds.kl.all(kl, nullptr);
  Stats st;
  st.m = m;
  st.m_r = most[0];
  st.inv_z = 1.0f / z;
  st.inv_h = 1.0f / h;
  st.inv_q = q != 0.0f ? 1.0f / q : 0.0f;
  st.c_soft = scale * st.inv_z;
  const float q_r = q != 0.0f ? list.rest / q : 0.0f;
  if (q_r != 0.0f && sums[0] != 0.0f) st.c_soft -= q_r / sums[0];
  st.c_hard = HARD == kNoHard ? 0.0f : scale1 * st.inv_h;
  st.pad = 0.0f;
  if (loss && threadIdx.x == 0) {
    if (q_r != 0.0f) kl[0] += q_r * (logf(q_r) - ((most[0] - ref) * g.c + logf(sums[0]) - log_z));
    float l = g.a.soft * kl[0];
    if (HARD && list.label != list.kNone) l += g.a.hard * (logf(h) - (list.s_label - ref));
    *loss = weight * l;
  }
  return st;
}

// ---- gradient of a stretch of a row

// What makes a gradient of an unlisted word's logit.
struct Slope {
  float c2, soft, hard, ref2, ref1;   // fast: soft * 2^(x c2 - ref2) + hard * 2^(x log2e - ref1)
  float m;                            // plain: soft * 2^((x - m) c2) + ...
  bool far_;
  template <int HARD, int E>
  __device__ void fast(float *x) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float e = base2_exp(x[i], c2, ref2);
      float y = soft * e;
      if (two_sums(HARD)) y = __builtin_fmaf(hard, hard_exp<HARD>(x[i], e, ref1), y);
      x[i] = y;
    }
  }
  template <int HARD, int E>
  __device__ void plain(float *x) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = x[i] - m;
      float y = soft * exp2_hw(d * c2);
      if (two_sums(HARD)) y = __builtin_fmaf(hard, exp2_hw(d * kLog2e), y);
      x[i] = y;
    }
  }
};

template <int DT, int HARD, int T>
struct Gradient {
  using raw = typename Num<DT>::raw;
  static constexpr int E = Num<DT>::E, PER = Listed<DT, T>::PER;
  const Row<DT> &row;
  raw *out;
  Stretch st;
  Slope k;
  bool none;   // the row has neither term (set by prepare, the same in every thread): its gradient is 0, whatever its logits
  __device__ Gradient(const Args &g, const Row<DT> &row_, uint64_t r, uint32_t v0_, uint32_t v1_)
      : row(row_), out(reinterpret_cast<raw *>(g.a.grad) + uniform_off(r * g.a.grad_stride)), st(row_, v0_, v1_) {}
  // (the gradient may be aligned otherwise than the logits)
  __device__ void put(int v, u32x4 y) const {   // vector v + threadIdx.x, v the same in every lane
    uint8_t *at = reinterpret_cast<uint8_t *>(out) + ((int64_t)v * 16 - (int64_t)(row.off * sizeof(raw)));
    // (past the caches: nothing here reads it again; loss and gradient of 4096 rows of 50,257 bf16 270 us without, 223 so)
    __builtin_nontemporal_store(y, reinterpret_cast<u32x4_any *>(at + threadIdx.x * 16u));
  }
  __device__ void put_any(uint32_t v, const float *x) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = (int)(v * E) - (int)row.off + i;
      if (j >= 0 && j < (int)row.vocab) Num<DT>::put(out + j, x[i]);
    }
  }
  __device__ void zero() const {
    const u32x4 none = {0, 0, 0, 0};
    for (uint32_t v = st.b0; v < st.b1; v += T)
      if (v + threadIdx.x < st.b1) put(v, none);
    const float x[E] = {};
    uint32_t v;
    if (st.edge(&v)) put_any(v, x);
  }
  // The slope; listed words' gradients take the place of their logits, the label's that of its own.
  __device__ void prepare(const Args &g, float weight, const Stats &stats, Listed<DT, T> &list) {
    // (a term that is not there counts nothing: its coefficient is no number in a row without a softmax)
    const bool soft_term = stats.inv_q != 0.0f && g.a.soft != 0.0f, hard_term = HARD && list.label != list.kNone;
    none = !soft_term && !hard_term;
    const float soft = soft_term ? weight * g.a.soft * g.c : 0.0f;
    const float hard = hard_term ? weight * g.a.hard : 0.0f;
    const float ref = ref_of(stats.m);
    k.c2 = g.c2;
    k.m = ref_of(stats.m_r);
    k.far_ = far(stats.m_r, g.c2, two_sums(HARD));
    k.soft = soft_term ? soft * stats.c_soft : 0.0f;
    k.hard = hard_term ? hard * stats.c_hard : 0.0f;
    if (list.label != list.kNone) {
      const float d = list.s_label - k.m;
      list.s_label = k.soft * exp2_hw(d * g.c2) + (HARD ? k.hard * exp2_hw(d * kLog2e) : 0.0f) - hard;
    }
    if (HARD == kSameHard) k.soft += k.hard;
    k.ref2 = base2_ref(stats.m_r, g.c2);
    k.ref1 = base2_ref(stats.m_r, kLog2e);
    if (!k.far_ && stats.m_r != kNegInf) {
      // (nothing else has to change: a coefficient takes up the rounding of the reference)
      if (k.soft != 0.0f) k.soft *= exp2_hw(-__builtin_fmaf(stats.m_r, g.c2, -k.ref2));
      if (k.hard != 0.0f) k.hard *= exp2_hw(-__builtin_fmaf(stats.m_r, kLog2e, -k.ref1));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (list.idx[i] == list.kNone) continue;
      const float d = list.s[i] - ref;
      // (without a soft term what a record says counts nothing, also where its values are no numbers)
      float x = soft_term ? soft * (exp2_hw(d * g.c2) * stats.inv_z - exp2_hw(list.val[i] * g.c2) * stats.inv_q) : 0.0f;
      if (HARD && hard != 0.0f) x += hard * (exp2_hw(d * kLog2e) * stats.inv_h - (list.idx[i] == list.label ? 1.0f : 0.0f));
      list.s[i] = x;
    }
  }
  __device__ void one(float *x) const {
    if (k.far_) k.template plain<HARD, E>(x);
    else k.template fast<HARD, E>(x);
  }
  __device__ void edges() const {
    uint32_t v;
    if (st.edge(&v)) {
      float x[E];
      row.load_any(v, x);
      one(x);
      put_any(v, x);
    }
  }
  // The body; `now`: its first four vectors.
  __device__ void stream(Four<DT, T> now) const {
    if (k.far_) {
      for (uint32_t v = st.b0; v < st.b1; v += T) {
        if (v + threadIdx.x < st.b1) {
          float x[E];
          Num<DT>::widen(row.load(v, threadIdx.x), x);
          k.template plain<HARD, E>(x);
          put(v, Num<DT>::narrow(x));
        }
      }
      return;
    }
    for (uint32_t v = st.b0; v < st.b1; v += 4 * T) {
      Four<DT, T> next;
      if (v + 4 * T < st.b1) next.load(row, st, v + 4 * T);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (v + u * T + threadIdx.x < st.b1) {
          float x[E];
          Num<DT>::widen(now.w[u], x);
          k.template fast<HARD, E>(x);
          put(v + u * T, Num<DT>::narrow(x));
        }
      }
      now = next;
    }
  }
  // The listed words and the label, after the others: those were written by other threads, too.
  __device__ void listed(const Args &g, const Listed<DT, T> &list) const {
    bool label_listed = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) label_listed = label_listed || (list.idx[i] != list.kNone && list.idx[i] == list.label);
    label_listed = __syncthreads_or(label_listed);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (list.idx[i] != list.kNone) Num<DT>::put(out + list.idx[i], list.s[i]);
    const uint32_t lo = st.v0 * E > row.off ? st.v0 * E - row.off : 0, hi = st.v1 * E - row.off < row.vocab ? st.v1 * E - row.off : row.vocab;
    if (HARD && list.label >= lo && list.label < hi && !label_listed && threadIdx.x == 0) Num<DT>::put(out + list.label, list.s_label);
  }
};

// ---- kernels

__device__ inline void put_stats(const Args &g, uint64_t r, const Stats &st) {
  if (g.a.stats && threadIdx.x == 0) reinterpret_cast<Stats *>(g.a.stats)[r] = st;
}

// Whole rows, a workgroup each: the loss.
template <int DT, int HARD, int T>
__global__ __launch_bounds__(T) void distill_loss_kernel(Args g) {
  extern __shared__ uint32_t bits[];   // (TAIL_REST)
  __shared__ FinishLds<T> lds;
  const uint64_t r = blockIdx.x;
  const float weight = weight_of(g, r);
  if (weight == 0.0f) {
    if (threadIdx.x == 0) g.a.loss[r] = 0.0f;
    put_stats(g, r, Stats{});
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const Stretch whole(row, 0, row.nv);
  Four<DT, T> first;
  first.load(row, whole, whole.b0);
  Listed<DT, T> list;
  list.template read<HARD != kNoHard>(g, row, r, 0, row.vocab);
  if (g.a.rest_too) list.mark(row, 0, row.nv, bits);
  const Marks<DT> marks{g.a.rest_too ? (const uint8_t *)bits : nullptr, 0};
  const FastSum f = scan<DT, HARD, T>(row, whole, first, marks, g.c2);
  const auto settle = [&](float m) { return settled<DT, HARD, T>(f, m, row, whole, marks, g.c2); };
  const Stats st = finish<DT, HARD, T>(g, list, f.m, settle, weight, g.a.loss + r, lds);
  put_stats(g, r, st);
}

// Whole rows, a workgroup each, loss and gradient in two passes: the second finds the row in the last-level cache.
template <int DT, int HARD, int T, int WAVES>
__global__ __launch_bounds__(T, WAVES) void distill_twice_kernel(Args g) {
  extern __shared__ uint32_t bits[];   // (TAIL_REST)
  __shared__ FinishLds<T> lds;
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const float weight = weight_of(g, r);
  Gradient<DT, HARD, T> grad(g, row, r, 0, row.nv);
  if (weight == 0.0f) {
    if (threadIdx.x == 0) g.a.loss[r] = 0.0f;
    grad.zero();
    return;
  }
  Four<DT, T, false> first;
  first.load(row, grad.st, grad.st.b0);
  Listed<DT, T> list;
  list.template read<HARD != kNoHard>(g, row, r, 0, row.vocab);
  if (g.a.rest_too) list.mark(row, 0, row.nv, bits);
  const Marks<DT> marks{g.a.rest_too ? (const uint8_t *)bits : nullptr, 0};
  const FastSum f = scan<DT, HARD, T>(row, grad.st, first, marks, g.c2);
  const auto settle = [&](float m) { return settled<DT, HARD, T>(f, m, row, grad.st, marks, g.c2); };
  const Stats st = finish<DT, HARD, T>(g, list, f.m, settle, weight, g.a.loss + r, lds);
  Four<DT, T> again;
  again.load(row, grad.st, grad.st.b0);
  grad.prepare(g, weight, st, list);
  if (grad.none) {
    grad.zero();
    return;
  }
  __syncthreads();   // (every listed logit has been read)
  grad.stream(again);
  grad.edges();
  grad.listed(g, list);
}

// Whole rows, a workgroup each, loss and gradient: the row stays in registers, HOLD vectors a thread, all of them
// requested before anything else.
template <int DT, int HARD, int T, int HOLD, int WAVES>
__global__ __launch_bounds__(T, WAVES) void distill_held_kernel(Args g) {
  constexpr int E = Num<DT>::E;
  constexpr bool TWO = two_sums(HARD);
  __shared__ uint32_t bits[(T * HOLD + 2) * E / 32 + 1];   // (whole vectors and two partial ones)
  __shared__ FinishLds<T> lds;
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const float weight = weight_of(g, r);
  Gradient<DT, HARD, T> grad(g, row, r, 0, row.nv);
  if (weight == 0.0f) {
    if (threadIdx.x == 0) g.a.loss[r] = 0.0f;
    grad.zero();
    return;
  }
  const uint32_t b0 = grad.st.b0, b1 = grad.st.b1;
  u32x4 w[HOLD];
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const uint32_t v = b0 + i * T;
    if (v + T <= b1) {   // (uniform)
      w[i] = row.load_once(v, threadIdx.x);
    } else {
      w[i] = Num<DT>::masked();
      if (v + threadIdx.x < b1) w[i] = row.load_once(v, threadIdx.x);
    }
  }
  Listed<DT, T> list;
  list.template read<HARD != kNoHard>(g, row, r, 0, row.vocab);
  float ends[E];
  uint32_t end_v;
  const bool has_end = grad.st.edge(&end_v);
  if (has_end) row.load_any(end_v, ends);
  if (g.a.rest_too) list.mark(row, 0, row.nv, bits);
  const Marks<DT> marks{g.a.rest_too ? (const uint8_t *)bits : nullptr, 0};
  // largest unlisted logit; from here on the listed ones are -inf here (their gradients are written apart)
  float largest = kNegInf;
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const uint32_t v = b0 + i * T;
    if (v < b1) {
      if (v + threadIdx.x < b1) marks.template apply<1>(v + threadIdx.x, 0, &w[i]);
      float x[E];
      Num<DT>::widen(w[i], x);
#pragma unroll
      for (int e = 0; e < E; ++e) largest = fmaxf(largest, x[e]);
    }
  }
  if (has_end) {
    marks.apply_to(end_v, ends);
#pragma unroll
    for (int e = 0; e < E; ++e) largest = fmaxf(largest, ends[e]);
  }
  const auto settle = [&](float m) -> Part {
    if (far(m, g.c2, TWO)) {
      PlainSum q = scan_plain<DT, HARD, T>(row, grad.st, marks, g.c2);
      q.template move_to<TWO>(m, g.c2);
      return q;
    }
    FastSum f;
    f.m = m;
    const float ref = base2_ref(m, g.c2), ref1 = base2_ref(m, kLog2e);
    const auto add = [&](const float *x) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float y = base2_exp(x[e], g.c2, ref);
        f.s += y;
        if (TWO) f.h += hard_exp<HARD>(x[e], y, ref1);
      }
    };
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      if (b0 + i * T < b1) {
        float x[E];
        Num<DT>::widen(w[i], x);
        add(x);
      }
    }
    if (has_end) add(ends);
    f.template settle<TWO>(g.c2);
    return f;
  };
  const Stats st = finish<DT, HARD, T>(g, list, largest, settle, weight, g.a.loss + r, lds);
  grad.prepare(g, weight, st, list);
  if (grad.none) {
    grad.zero();
    return;
  }
  if (grad.k.far_) {
    grad.stream(Four<DT, T>{});
  } else {
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      const uint32_t v = b0 + i * T;
      if (v + threadIdx.x < b1) {
        float x[E];
        Num<DT>::widen(w[i], x);
        grad.k.template fast<HARD, E>(x);
        grad.put(v, Num<DT>::narrow(x));
      }
    }
  }
  if (has_end) {
    grad.one(ends);
    grad.put_any(end_v, ends);
  }
  grad.listed(g, list);
}

// Rows that one workgroup cannot hold: sums of chunks, loss and statistics from those, gradients of chunks.  (Gradients
// wait for a launch of their own, because they may be written over listed logits that other chunks' losses need.)
constexpr int kChunkThreads = 256;

template <int DT, int HARD>
__global__ __launch_bounds__(kChunkThreads) void distill_scan_kernel(Args g, float *partial) {
  constexpr int T = kChunkThreads;
  constexpr bool TWO = two_sums(HARD);
  __shared__ uint32_t bits[kChunkVecs * Num<DT>::E / 32];
  __shared__ Exchange<T, 0, 1> most;
  __shared__ Exchange<T, 2, 0> sums;
  const uint64_t r = blockIdx.x;
  if (weight_of(g, r) == 0.0f) return;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const uint32_t v0 = blockIdx.y * g.vecs < row.nv ? blockIdx.y * g.vecs : row.nv;
  const uint32_t v1 = v0 + g.vecs < row.nv ? v0 + g.vecs : row.nv;
  const Stretch chunk(row, v0, v1);
  Four<DT, T> first;
  first.load(row, chunk, chunk.b0);
  if (g.a.rest_too) {
    Listed<DT, T> list;
    list.template read<false>(g, row, r, 0, row.vocab);
    list.mark(row, v0, v1, bits);
  }
  const Marks<DT> marks{g.a.rest_too ? (const uint8_t *)bits : nullptr, v0};
  const FastSum f = scan<DT, HARD, T>(row, chunk, first, marks, g.c2);
  float m[1] = {f.m};
  most.all(nullptr, m);
  const Part p = settled<DT, HARD, T>(f, m[0], row, chunk, marks, g.c2);
  float s[2] = {p.s, TWO ? p.h : 0.0f};
  sums.all(s, nullptr);
  if (threadIdx.x == 0) {
    float *o = partial + (r * g.chunks + blockIdx.y) * kPartialFloats;
    o[0] = m[0];
    o[1] = s[0];
    o[2] = s[1];
  }
}

// Loss and statistics of a row from its chunks' sums.
template <int DT, int HARD>
__global__ __launch_bounds__(kChunkThreads) void distill_join_kernel(Args g, const float *partial) {
  constexpr int T = kChunkThreads;
  constexpr bool TWO = two_sums(HARD);
  __shared__ FinishLds<T> lds;
  const uint64_t r = blockIdx.x;
  const float weight = weight_of(g, r);
  if (weight == 0.0f) {
    if (threadIdx.x == 0) g.a.loss[r] = 0.0f;
    put_stats(g, r, Stats{});
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  Listed<DT, T> list;
  list.template read<HARD != kNoHard>(g, row, r, 0, row.vocab);
  PlainSum p;
  for (uint32_t i = threadIdx.x; i < g.chunks; i += T) {
    const float *o = partial + (r * g.chunks + i) * kPartialFloats;
    PlainSum x;
    x.m = o[0];
    x.s = o[1];
    x.h = o[2];
    const float nm = fmaxf(p.m, x.m);
    p.template move_to<TWO>(nm, g.c2);
    x.template move_to<TWO>(nm, g.c2);
    p.s += x.s;
    p.h += x.h;
  }
  const auto settle = [&](float m) {
    PlainSum q = p;
    q.template move_to<TWO>(m, g.c2);
    return q;
  };
  put_stats(g, r, finish<DT, HARD, T>(g, list, p.m, settle, weight, g.a.loss + r, lds));
}

// The gradient from statistics, a workgroup a row (or a stretch of kGradVecs vectors of it).
template <int DT, int HARD, int T>
__global__ __launch_bounds__(T) void distill_grad_kernel(Args g) {
  constexpr int E = Num<DT>::E;
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const uint32_t v0 = blockIdx.y * g.vecs, v1 = v0 + g.vecs < row.nv ? v0 + g.vecs : row.nv;
  if (v0 >= v1) return;
  const float weight = weight_of(g, r);
  Gradient<DT, HARD, T> grad(g, row, r, v0, v1);
  if (weight == 0.0f) {
    grad.zero();
    return;
  }
  Four<DT, T> first;
  first.load(row, grad.st, grad.st.b0);
  Listed<DT, T> list;
  const uint32_t lo = v0 * E > row.off ? v0 * E - row.off : 0, hi = v1 * E - row.off < row.vocab ? v1 * E - row.off : row.vocab;
  list.template read<HARD != kNoHard>(g, row, r, lo, hi);
  grad.prepare(g, weight, reinterpret_cast<const Stats *>(g.a.stats)[r], list);
  if (grad.none) {
    grad.zero();
    return;
  }
  // every thread has read the listed logits of its entries before any is written over
  __syncthreads();
  grad.stream(first);
  grad.edges();
  grad.listed(g, list);
}

template <int DT, int HARD, int T, int HOLD, int WAVES>
static hipError_t held_rows(const Args &g, hipStream_t stream) {
  distill_held_kernel<DT, HARD, T, HOLD, WAVES><<<(uint32_t)g.a.rows, T, 0, stream>>>(g);
  return hipGetLastError();
}

template <int DT, int HARD>
static hipError_t run_typed(Args g, DistillRole role, uint8_t *ws, hipStream_t stream) {
  const uint32_t rows = (uint32_t)g.a.rows, nv = row_vecs(g.a.vocab, DT, g.a.row_stride);
  const Cut cut = cut_rows(g.a.rows, g.a.vocab, DT, g.a.row_stride, role == DistillRole::step);
  const uint32_t marks_lds = g.a.rest_too ? (uint32_t)cdiv((uint64_t)nv * Num<DT>::E, 32) * 4 : 0;
  if (role == DistillRole::loss && cut.chunks == 1) {
    // (4096 x 50257 bf16 with 256 / 512 / 1024 threads: 68 / 77 / 153 us, what a row costs beside its logits is the same
    // for each.  Fewer rows take 1024; a compute unit has room for one such workgroup, so that more than 256 rows go in two
    // rounds: 256 / 257 / 511 / 512 rows of 50257 bf16 9.3 / 15.8 / 17.9 / 15.6 us)
    if (nv <= 1024 && g.a.k <= kOneWaveK) distill_loss_kernel<DT, HARD, 64><<<rows, 64, marks_lds, stream>>>(g);
    else if (rows >= 512) distill_loss_kernel<DT, HARD, 256><<<rows, 256, marks_lds, stream>>>(g);
    else distill_loss_kernel<DT, HARD, 1024><<<rows, 1024, marks_lds, stream>>>(g);
    return hipGetLastError();
  }
  if (role == DistillRole::step && cut.chunks == 1) {
    // Held where two rows or more fit the registers of a compute unit and there are rows enough: 4096 x 50257 bf16 176 us
    // held and 199 in two passes, 2048 x 30522 f16 56 and 80, 2000 x 32000 f32 97 and 119.  One row at a time leaves
    // the memory idle while its sums are joined: 8192 x 131072 bf16 1023 held, 951 in two passes (three rows at a
    // time).  Few rows: 100 x 30000 bf16 12.9 and 11.0, 61 x 128000 23.2 and 20.5; 256 / 257 / 511 / 512 rows of 50257 bf16
    // 14.7 / 22.8 / 30.1 / 23.3 (two rounds of 1024 threads, then held).  The bound of 512 x 6 holds two passes to 80
    // registers, chosen on bf16, which spills none (own temperature: one); f16 spills 7 to 31: 1024 x 131072 bf16 128 us,
    // f16 135; with hard labels at temperature 2 131 and 150.
    if (nv <= 512 && g.a.k <= kOneWaveK) return held_rows<DT, HARD, 64, 8, 4>(g, stream);
    if (nv <= 2048) return held_rows<DT, HARD, 256, 8, 5>(g, stream);
    if (nv <= 4096 && rows >= 512) return held_rows<DT, HARD, 256, 16, 4>(g, stream);
    if (nv <= 8192 && rows >= 512) return held_rows<DT, HARD, 512, 16, 4>(g, stream);
    if (rows >= 512) distill_twice_kernel<DT, HARD, 512, 6><<<rows, 512, marks_lds, stream>>>(g);
    else distill_twice_kernel<DT, HARD, 1024, 4><<<rows, 1024, marks_lds, stream>>>(g);
    return hipGetLastError();
  }
  if (role != DistillRole::grad) {
    const DistillWs lay = distill_ws(g.a.rows, cut);
    float *partial = reinterpret_cast<float *>(ws + lay.partial);
    if (!g.a.stats) g.a.stats = ws + lay.stats;
    g.chunks = cut.chunks;
    g.vecs = cut.vecs;
    distill_scan_kernel<DT, HARD><<<dim3(rows, cut.chunks), kChunkThreads, 0, stream>>>(g, partial);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    distill_join_kernel<DT, HARD><<<rows, kChunkThreads, 0, stream>>>(g, partial);
    e = hipGetLastError();
    if (e != hipSuccess || role == DistillRole::loss) return e;
  }
  // As many threads as a row keeps busy: the fewer rows are on their way at a time, the better the memory takes the
  // writes (4096 x 50,257 bf16, whose loss takes 68 us, 229 / 218 / 209 us for both with 256 / 512 / 1024 threads).
  // Short rows where there are many of them take fewer, for what a row costs beside its logits (loss and gradient of
  // 16000 x 1000 bf16 46 us with 64 threads and 65 with 256, of 4000 x 10000 56 with 256 and 64 with 1024).
  g.vecs = kGradVecs;
  const dim3 grid(rows, (uint32_t)cdiv(nv, kGradVecs));
  if (nv <= 512 && g.a.k <= kOneWaveK) distill_grad_kernel<DT, HARD, 64><<<grid, 64, 0, stream>>>(g);
  else if (nv <= 512 || (nv <= 2048 && rows >= 512)) distill_grad_kernel<DT, HARD, 256><<<grid, 256, 0, stream>>>(g);
  else distill_grad_kernel<DT, HARD, 1024><<<grid, 1024, 0, stream>>>(g);
  return hipGetLastError();
}

template <int DT>
static hipError_t run_hard(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream) {
  Args g{};
  g.a = call;
  g.c = 1.0f / call.temperature;
  g.c2 = (float)(1.44269504088896340736 / (double)call.temperature);
  if (!call.labels || call.hard == 0.0f) return run_typed<DT, kNoHard>(g, role, ws, stream);
  if (call.temperature == 1.0f) return run_typed<DT, kSameHard>(g, role, ws, stream);
  if (call.temperature == 2.0f) return run_typed<DT, kSquareHard>(g, role, ws, stream);
  if (call.temperature == 4.0f) return run_typed<DT, kFourthHard>(g, role, ws, stream);
  return run_typed<DT, kOwnHard>(g, role, ws, stream);
}

}  // namespace bpc
