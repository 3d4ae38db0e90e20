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
#include "distill.hpp"
#include "kernels.hpp"

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

// Sums of a set of words relative to the largest of them.
struct Part {
  float m = kNegInf, s = 0.0f, h = 0.0f;
  template <bool TWO>
  __device__ void rescale(float nm, float c2) {
    const float d = m - ref_of(nm);
    s *= exp2_hw(d * c2);
    if (TWO) h *= exp2_hw(d * kLog2e);
    m = nm;
  }
  template <bool TWO, int N>
  __device__ void add(const float *x, float c2) {
    float nm = m;
#pragma unroll
    for (int i = 0; i < N; ++i) nm = fmaxf(nm, x[i]);
    rescale<TWO>(nm, c2);
    const float ref = ref_of(nm);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - ref;
      s += exp2_hw(d * c2);
      if (TWO) h += exp2_hw(d * kLog2e);
    }
  }
};

template <int DT>
struct Marks {   // a bit a word of a chunk: listed
  static constexpr int E = Num<DT>::E;
  const uint8_t *bits;
  uint32_t v0;
  __device__ uint32_t of(uint32_t v) const {
    const uint32_t i = v - v0;
    return E == 8 ? bits[i] : (bits[i >> 1] >> (4 * (i & 1))) & 15u;
  }
};

// Sums over the vectors [v0, v1) of a row, without the marked words, in every thread.
template <int DT, bool TWO, int THREADS>
__device__ Part scan(const Row<DT> &row, uint32_t v0, uint32_t v1, bool marked, const Marks<DT> &marks, float c2, float *lds) {
  constexpr int E = Num<DT>::E;
  Part p;
  uint32_t b0, b1;
  row.body(v0, v1, &b0, &b1);
  const auto one = [&](uint32_t v, float *x) {
    if (marked) {
      const uint32_t bits = marks.of(v);
      if (bits) {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = (bits >> i) & 1 ? kNegInf : x[i];
      }
    }
  };
  for (uint32_t v = b0 + threadIdx.x; v < b1; v += THREADS) {
    float x[E];
    Num<DT>::widen(row.load(v), x);
    one(v, x);
    p.add<TWO, E>(x, c2);
  }
  const bool first = b0 > v0, last = b1 < v1;
  if ((threadIdx.x == 0 && first) || (threadIdx.x == 1 && last)) {
    const uint32_t v = threadIdx.x == 0 ? v0 : v1 - 1;
    float x[E];
    row.load_any(v, x);
    one(v, x);
    p.add<TWO, E>(x, c2);
  }
  p.rescale<TWO>(all_max<THREADS>(p.m, lds), c2);
  p.s = all_sum<THREADS>(p.s, lds);
  if (TWO) p.h = all_sum<THREADS>(p.h, lds);
  return p;
}

// Marks the listed words of the vectors [v0, v1).
template <int DT, int THREADS>
__device__ void mark(const Args &g, const Row<DT> &row, uint64_t r, uint32_t v0, uint32_t v1, uint32_t *bits) {
  constexpr int E = Num<DT>::E;
  const Record rec(g.a.messages, r, g.a.message_stride, g.a.k, g.a.half);
  const uint32_t n = rec.count(g.a.k), words = ((v1 - v0) * E + 31) / 32;
  for (uint32_t w = threadIdx.x; w < words; w += THREADS) bits[w] = 0;
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < n; e += THREADS) {
    const uint32_t j = rec.idx(e);
    const uint32_t at = j + row.off - v0 * E;   // (from the first word of vector v0)
    if (j < g.a.vocab && j + row.off >= v0 * E && at < (v1 - v0) * E) atomicOr(&bits[at >> 5], 1u << (at & 31));
  }
  __syncthreads();
}

__device__ inline bool hard_label(const Args &g, uint64_t r, uint32_t *label) {
  if (!g.a.labels || g.a.hard == 0.0f) return false;
  const int64_t l = g.a.labels[r];
  if (l < 0 || l >= (int64_t)g.a.vocab) return false;
  *label = (uint32_t)l;
  return true;
}

// The row's loss and statistics from the sums of its unlisted words (TAIL_DROP: of all words).
// HARD: 0 no hard term, 1 at the same temperature as the soft one, 2 at its own.
template <int DT, int HARD, int THREADS>
__device__ Stats finish(const Args &g, const Row<DT> &row, uint64_t r, Part p, float weight, float *loss, float *lds) {
  const bool rest_too = g.a.rest_too;
  const Record rec(g.a.messages, r, g.a.message_stride, g.a.k, g.a.half);
  const uint32_t n = rec.count(g.a.k);
  float m = kNegInf, q = 0.0f;
  for (uint32_t e = threadIdx.x; e < n; e += THREADS) {
    const uint32_t j = rec.idx(e);
    if (j >= g.a.vocab) continue;
    m = fmaxf(m, Num<DT>::get(row.p + j));
    q += exp2_hw(rec.val(e) * g.c2);
  }
  m = all_max<THREADS>(m, lds);
  q = all_sum<THREADS>(q, lds);
  Stats st;
  const float rest = rest_too ? rec.rest() : 0.0f;
  q += rest;
  if (n == 0) q = 0.0f;
  st.m_r = p.m;
  float z = p.s, h = HARD == 1 ? p.s : p.h;
  if (rest_too) {
    st.m = fmaxf(m, p.m);
    const float ref = ref_of(st.m);
    float zs = 0.0f, hs = 0.0f;
    for (uint32_t e = threadIdx.x; e < n; e += THREADS) {
      const uint32_t j = rec.idx(e);
      if (j >= g.a.vocab) continue;
      const float d = Num<DT>::get(row.p + j) - ref;
      zs += exp2_hw(d * g.c2);
      if (HARD == 2) hs += exp2_hw(d * kLog2e);
    }
    zs = all_sum<THREADS>(zs, lds);
    z = p.s * exp2_hw((p.m - ref) * g.c2) + zs;
    h = z;
    if (HARD == 2) h = p.h * exp2_hw((p.m - ref) * kLog2e) + all_sum<THREADS>(hs, lds);
  } else {
    st.m = p.m;
  }
  const float ref = ref_of(st.m), log_z = logf(z);
  float kl = 0.0f;
  if (q != 0.0f) {
    const float log_q = logf(q);
    for (uint32_t e = threadIdx.x; e < n; e += THREADS) {
      const uint32_t j = rec.idx(e);
      if (j >= g.a.vocab) continue;
      const float val = rec.val(e), w = exp2_hw(val * g.c2) / q;
      // log(q_i / p_i); a word that the teacher gives nothing counts nothing, whatever the student gives it
      if (w != 0.0f) kl += w * ((val - (Num<DT>::get(row.p + j) - ref)) * g.c + (log_z - log_q));
    }
    kl = all_sum<THREADS>(kl, lds);
    const float qr = rest / q;
    if (rest_too && qr != 0.0f) kl += qr * (logf(qr) - ((p.m - ref) * g.c + logf(p.s) - log_z));
  }
  st.inv_z = 1.0f / z;
  st.inv_h = 1.0f / h;
  st.inv_q = q != 0.0f ? 1.0f / q : 0.0f;
  const float down = (ref_of(p.m) - ref) * 1.0f;
  st.c_soft = exp2_hw(down * g.c2) * st.inv_z;
  if (rest_too && rest != 0.0f && p.s != 0.0f) st.c_soft -= rest * st.inv_q / p.s;
  st.c_hard = HARD == 0 ? 0.0f : exp2_hw(down * kLog2e) * st.inv_h;
  st.pad = 0.0f;
  if (loss && threadIdx.x == 0) {
    float l = g.a.soft * kl;
    uint32_t label;
    if (HARD && hard_label(g, r, &label)) l += g.a.hard * (logf(h) - (Num<DT>::get(row.p + label) - ref));
    *loss = weight == 0.0f ? 0.0f : weight * l;
  }
  return st;
}

// Gradient of the vectors [v0, v1) of a row.
template <int DT, int HARD, int THREADS>
__device__ void gradient(const Args &g, const Row<DT> &row, uint64_t r, uint32_t v0, uint32_t v1, float weight, const Stats &st) {
  constexpr int E = Num<DT>::E;
  using raw = typename Num<DT>::raw;
  raw *out = reinterpret_cast<raw *>(g.a.grad) + uniform_off(r * g.a.grad_stride);
  uint32_t b0, b1, label = 0xffffffffu;
  row.body(v0, v1, &b0, &b1);
  const bool hard = HARD && hard_label(g, r, &label);
  const float soft = st.inv_q != 0.0f ? weight * g.a.soft * g.c : 0.0f;
  const float ks = soft * st.c_soft, kh = hard ? weight * g.a.hard * st.c_hard : 0.0f;
  const float ref = ref_of(st.m_r);
  // the listed words of this stretch are read before anything is written (the gradient may lie over the logits)
  const Record rec(g.a.messages, r, g.a.message_stride, g.a.k, g.a.half);
  const uint32_t n = rec.count(g.a.k);
  const uint32_t lo = v0 * E > row.off ? v0 * E - row.off : 0, hi = v1 * E - row.off < g.a.vocab ? v1 * E - row.off : g.a.vocab;
  constexpr int PER = (kMaxLogitsK + THREADS - 1) / THREADS;
  float kept[PER];
  uint32_t at[PER];
  bool label_listed = false;
  const float ref_all = ref_of(st.m);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = threadIdx.x + i * THREADS;
    at[i] = 0xffffffffu;
    if (weight == 0.0f || e >= n) continue;
    const uint32_t j = rec.idx(e);
    if (j < lo || j >= hi) continue;
    at[i] = j;
    const float d = Num<DT>::get(row.p + j) - ref_all;
    float x = soft * (exp2_hw(d * g.c2) * st.inv_z - exp2_hw(rec.val(e) * g.c2) * st.inv_q);
    if (hard) x += weight * g.a.hard * (exp2_hw(d * kLog2e) * st.inv_h - (j == label ? 1.0f : 0.0f));
    if (j == label) label_listed = true;
    kept[i] = x;
  }
  float at_label = 0.0f;
  const bool mine = hard && weight != 0.0f && label >= lo && label < hi;
  if (mine) {
    const float d = Num<DT>::get(row.p + label) - ref;
    at_label = ks * exp2_hw(d * g.c2) + kh * exp2_hw(d * kLog2e) - weight * g.a.hard;
  }
  label_listed = __syncthreads_or(label_listed);
  const auto one = [&](float *x) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = x[i] - ref;
      float y = (HARD == 1 ? ks + kh : ks) * exp2_hw(d * g.c2);
      if (HARD == 2) y += kh * exp2_hw(d * kLog2e);
      x[i] = weight == 0.0f ? 0.0f : y;
    }
  };
  for (uint32_t v = b0 + threadIdx.x; v < b1; v += THREADS) {
    float x[E];
    if (weight != 0.0f) Num<DT>::widen(row.load(v), x);
    one(x);
    const u32x4 y = Num<DT>::narrow(x);
    __builtin_memcpy(out + ((int)(v * E) - (int)row.off), &y, 16);   // (grad may be aligned otherwise than the logits)
  }
  const bool first = b0 > v0, last = b1 < v1;
  if ((threadIdx.x == 0 && first) || (threadIdx.x == 1 && last)) {
    const uint32_t v = threadIdx.x == 0 ? v0 : v1 - 1;
    float x[E];
    if (weight != 0.0f) row.load_any(v, x);
    one(x);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = (int)(v * E) - (int)row.off + i;
      if (j >= 0 && j < (int)g.a.vocab) Num<DT>::put(out + j, x[i]);
    }
  }
  __syncthreads();   // the words below were written by other threads, too
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (at[i] != 0xffffffffu) Num<DT>::put(out + at[i], kept[i]);
  if (mine && !label_listed && threadIdx.x == 0) Num<DT>::put(out + label, at_label);
}

__device__ inline float weight_of(const Args &g, uint64_t r) { return g.a.weight ? uniform_load(g.a.weight + r) : 1.0f; }

// Whole rows, a workgroup each: the loss and, with STEP, the gradient.
template <int DT, int HARD, int THREADS, bool STEP>
__global__ __launch_bounds__(THREADS) void distill_rows_kernel(Args g) {
  __shared__ uint32_t bits[kChunkVecs * Num<DT>::E / 32];
  __shared__ float lds[THREADS / 64];
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const float weight = weight_of(g, r);
  Stats st{};
  if (weight != 0.0f) {
    if (g.a.rest_too) mark<DT, THREADS>(g, row, r, 0, row.nv, bits);
    const Part p = scan<DT, HARD == 2, THREADS>(row, 0, row.nv, g.a.rest_too, Marks<DT>{(const uint8_t *)bits, 0}, g.c2, lds);
    st = finish<DT, HARD, THREADS>(g, row, r, p, weight, g.a.loss + r, lds);
  } else if (threadIdx.x == 0) {
    g.a.loss[r] = 0.0f;
  }
  if (g.a.stats && threadIdx.x == 0) reinterpret_cast<Stats *>(g.a.stats)[r] = st;
  if (STEP) gradient<DT, HARD, THREADS>(g, row, r, 0, row.nv, weight, st);
}

// Sums of one chunk of a row.
template <int DT, int HARD, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_scan_kernel(Args g, float *partial) {
  __shared__ uint32_t bits[kChunkVecs * Num<DT>::E / 32];
  __shared__ float lds[THREADS / 64];
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const uint32_t v0 = blockIdx.y * g.vecs < row.nv ? blockIdx.y * g.vecs : row.nv;
  const uint32_t v1 = v0 + g.vecs < row.nv ? v0 + g.vecs : row.nv;
  Part p;
  if (weight_of(g, r) != 0.0f) {
    if (g.a.rest_too) mark<DT, THREADS>(g, row, r, v0, v1, bits);
    p = scan<DT, HARD == 2, THREADS>(row, v0, v1, g.a.rest_too, Marks<DT>{(const uint8_t *)bits, v0}, g.c2, lds);
  }
  if (threadIdx.x == 0) {
    float *o = partial + (r * g.chunks + blockIdx.y) * kPartialFloats;
    o[0] = p.m;
    o[1] = p.s;
    o[2] = p.h;
  }
}

template <int DT, int HARD, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_finish_kernel(Args g, const float *partial) {
  __shared__ float lds[THREADS / 64];
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const float weight = weight_of(g, r);
  Stats st{};
  if (weight != 0.0f) {
    Part p;
    for (uint32_t i = threadIdx.x; i < g.chunks; i += THREADS) {
      const float *o = partial + (r * g.chunks + i) * kPartialFloats;
      Part x;
      x.m = o[0]; x.s = o[1]; x.h = o[2];
      const float nm = fmaxf(p.m, x.m);
      p.rescale<HARD == 2>(nm, g.c2);
      x.rescale<HARD == 2>(nm, g.c2);
      p.s += x.s;
      p.h += x.h;
    }
    p.rescale<HARD == 2>(all_max<THREADS>(p.m, lds), g.c2);
    p.s = all_sum<THREADS>(p.s, lds);
    if (HARD == 2) p.h = all_sum<THREADS>(p.h, lds);
    st = finish<DT, HARD, THREADS>(g, row, r, p, weight, g.a.loss + r, lds);
  } else if (threadIdx.x == 0) {
    g.a.loss[r] = 0.0f;
  }
  if (g.a.stats && threadIdx.x == 0) reinterpret_cast<Stats *>(g.a.stats)[r] = st;
}

template <int DT, int HARD, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(Args g) {
  const uint64_t r = blockIdx.x;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const uint32_t v0 = blockIdx.y * g.vecs < row.nv ? blockIdx.y * g.vecs : row.nv;
  const uint32_t v1 = v0 + g.vecs < row.nv ? v0 + g.vecs : row.nv;
  if (v0 >= v1) return;
  gradient<DT, HARD, THREADS>(g, row, r, v0, v1, weight_of(g, r), reinterpret_cast<const Stats *>(g.a.stats)[r]);
}

constexpr int kRowThreads = 256;

template <int DT, int HARD>
static hipError_t run_typed(Args g, DistillRole role, uint8_t *ws, hipStream_t stream) {
  const uint32_t rows = (uint32_t)g.a.rows;
  const Cut cut = cut_rows(g.a.rows, g.a.vocab, DT, g.a.row_stride);
  g.chunks = cut.chunks;
  g.vecs = cut.vecs;
  const DistillWs lay = distill_ws(g.a.rows, cut);
  const dim3 grid(rows, cut.chunks);
  if (role == DistillRole::grad) {
    distill_grad_kernel<DT, HARD, kRowThreads><<<grid, kRowThreads, 0, stream>>>(g);
    return hipGetLastError();
  }
  if (cut.chunks == 1) {
    if (role == DistillRole::loss) distill_rows_kernel<DT, HARD, kRowThreads, false><<<rows, kRowThreads, 0, stream>>>(g);
    else distill_rows_kernel<DT, HARD, kRowThreads, true><<<rows, kRowThreads, 0, stream>>>(g);
    return hipGetLastError();
  }
  float *partial = reinterpret_cast<float *>(ws + lay.partial);
  if (!g.a.stats) g.a.stats = ws + lay.stats;
  distill_scan_kernel<DT, HARD, kRowThreads><<<grid, kRowThreads, 0, stream>>>(g, partial);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  distill_finish_kernel<DT, HARD, kRowThreads><<<rows, kRowThreads, 0, stream>>>(g, partial);
  e = hipGetLastError();
  if (e != hipSuccess || role == DistillRole::loss) return e;
  distill_grad_kernel<DT, HARD, kRowThreads><<<grid, kRowThreads, 0, stream>>>(g);
  return hipGetLastError();
}

template <int DT>
static hipError_t run_hard(const Args &g, DistillRole role, uint8_t *ws, hipStream_t stream) {
  if (!g.a.labels || g.a.hard == 0.0f) return run_typed<DT, 0>(g, role, ws, stream);
  if (g.c == 1.0f) return run_typed<DT, 1>(g, role, ws, stream);
  return run_typed<DT, 2>(g, role, ws, stream);
}

hipError_t distill_run(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream) {
  Args g{};
  g.a = call;
  g.c = 1.0f / call.temperature;
  g.c2 = (float)(1.44269504088896340736 / (double)call.temperature);
  switch (call.dtype) {
    case BPC_F32: return run_hard<BPC_F32>(g, role, ws, stream);
    case BPC_F16: return run_hard<BPC_F16>(g, role, ws, stream);
    default: return run_hard<BPC_BF16>(g, role, ws, stream);
  }
}

}  // namespace bpc
