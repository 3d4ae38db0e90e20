// Teacher side of the distillation from top logits: the k largest logits of every row, in index
// order, and the mass of all others (record format in include/bpc.h).
//
// Logits are ordered by integer keys.  The usual form passes over a row once, in groups of a line of 128 bytes: the
// k-th largest of the groups' largest logits bounds the row's k-th largest from below, and only groups that reach that
// bound are looked through for candidates, of which a bisection finds the k-th.  Short rows of which a good part is
// listed stay in LDS as keys; rows of NaN, infinities, numbers far from 0 or more candidates than there is room for go
// through a radix select, which is right for every row.  Of the logits level with the k-th the first ones are listed.
// The mass of the rest is summed over the unlisted logits, never formed as a difference.
//
// The radix select also takes every row past 2^18 logits, for which the bits of the index order and the groups' keys have no
// room: 4096 x 262080 bf16, k = 64, 462 us and 4096 x 262208 3614; one such row 15 and 681.  4096 x 50257 bf16 with all
// logits equal, or with fewer than k that are not the type's lowest value, take 3055 and 2919 us for 112.
//
// What bounds it: vector issue.  A logit takes 6 to 7 instructions in the pass and about as much again for what follows
// it (bisections, second look, index order): 8192 x 131072 bf16, k = 256, 447 us (95 % busy; the pass alone 346 us, 6.2
// TB/s), 4096 x 50257, k = 64, 97 us (83 %; the pass 63).
#include "distill.hpp"
#include "distill_call.hpp"

namespace bpc {

struct TeacherArgs {
  DistillCall a;
  float c2;         // log2 e / temperature
  uint8_t *out;
};

// Keys that order logits as numbers (-0 as +0, a NaN above all); 0 for -inf, which is never listed.
__device__ inline uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  const uint32_t k = (int32_t)u < 0 ? ~u : u | 0x80000000u;
  return x != x ? 0xffffffffu : x == kNegInf ? 0u : k;
}

constexpr uint32_t kLowestKey = 0x00800000u;   // of the lowest finite number

// Writes the entries of a record from n on (idx -1, val -inf) and its header.
template <int THREADS>
__device__ void close_record(const TeacherArgs &g, uint8_t *rec, uint32_t n, float rest, float top) {
  uint32_t *idx = reinterpret_cast<uint32_t *>(rec + kHeaderBytes);
  uint8_t *val = rec + kHeaderBytes + 4 * ru4(g.a.k);
  for (uint32_t e = n + threadIdx.x; e < g.a.k; e += THREADS) {
    idx[e] = 0xffffffffu;
    if (g.a.half) reinterpret_cast<uint16_t *>(val)[e] = 0xfc00u;
    else reinterpret_cast<float *>(val)[e] = kNegInf;
  }
  if (threadIdx.x == 0) {
    uint32_t *h = reinterpret_cast<uint32_t *>(rec);
    h[0] = n;
    h[1] = __float_as_uint(rest);
    h[2] = __float_as_uint(top);
    h[3] = 0;
  }
}
__device__ inline void put_entry(const TeacherArgs &g, uint8_t *rec, uint32_t e, uint32_t j, float val) {
  reinterpret_cast<uint32_t *>(rec + kHeaderBytes)[e] = j;
  uint8_t *v = rec + kHeaderBytes + 4 * ru4(g.a.k);
  if (g.a.half) reinterpret_cast<_Float16 *>(v)[e] = (_Float16)val;
  else reinterpret_cast<float *>(v)[e] = val;
}

// A whole row by a radix select: four passes for the key, one to write.  Right for every row.  (8192 x 131072 bf16 3486
// us: 256 counters in LDS take turns for logits of a few exponents.)
template <int DT, int THREADS>
__device__ void select_any(const TeacherArgs &g, const Row<DT> &row, uint8_t *rec) {
  constexpr int E = Num<DT>::E;
  __shared__ uint32_t hist[256];
  __shared__ uint32_t scan_lds[THREADS / 64];
  __shared__ float lds[THREADS / 64];
  __shared__ uint32_t pick[2];
  uint32_t prefix = 0, want = g.a.k;
  float top = kNegInf;
  bool nan = false;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (uint32_t i = threadIdx.x; i < 256; i += THREADS) hist[i] = 0;
    __syncthreads();
    for (uint32_t v = threadIdx.x; v < row.nv; v += THREADS) {
      float x[E];
      row.load_any(v, x);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint32_t key = order_key(x[i]);
        if (shift == 24) {
          top = fmaxf(top, x[i]);
          nan = nan || x[i] != x[i];
        }
        if (key != 0 && (shift == 24 || (key >> (shift + 8)) == prefix)) atomicAdd(&hist[(key >> shift) & 255], 1u);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t above = 0;
      int b = 255;
      for (; b > 0 && above + hist[b] < want; --b) above += hist[b];
      pick[0] = (uint32_t)b;
      pick[1] = above;
    }
    __syncthreads();
    // (fewer than k candidates: bin 0 is taken and every candidate is at or above the key)
    prefix = (prefix << 8) | pick[0];
    want -= pick[1];
  }
  top = all_max<THREADS>(top, lds);
  if (__syncthreads_or(nan)) top = __builtin_nanf("");
  const uint32_t kth = prefix;
  const float ref = ref_of(top);
  float rest = 0.0f;
  uint32_t listed = 0, level = 0;   // so far: entries written, logits level with the k-th
  for (uint32_t v0 = 0; v0 < row.nv; v0 += THREADS) {
    const uint32_t v = v0 + threadIdx.x;
    float x[E];
    uint32_t above = 0, same = 0;
    if (v < row.nv) {
      row.load_any(v, x);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint32_t key = order_key(x[i]);
        above += key != 0 && key > kth;
        same += key != 0 && key == kth;
      }
    }
    uint32_t all_same, all_taken;
    const uint32_t same_before = level + block_exclusive_scan<THREADS>(same, scan_lds, &all_same);
    const uint32_t open = same_before < want ? want - same_before : 0;
    uint32_t left = same < open ? same : open;
    uint32_t at = listed + block_exclusive_scan<THREADS>(above + left, scan_lds, &all_taken);
    if (v < row.nv) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint32_t key = order_key(x[i]);
        bool take = key != 0 && key > kth;
        if (key != 0 && key == kth && left > 0) {
          take = true;
          --left;
        }
        if (take) put_entry(g, rec, at++, v * E - row.off + i, x[i] - ref);
        else if (x[i] != kNegInf) rest += exp2_hw((x[i] - ref) * g.c2);   // (also what lies outside the row)
      }
    }
    level += all_same;
    listed += all_taken;
  }
  rest = all_sum<THREADS>(rest, lds);
  close_record<THREADS>(g, rec, listed, rest, top);
}

// ---- rows whose k-th largest logit can be bounded from below by largest logits of groups

// Keys without the low bits that logits of a type leave 0 as f32 (13 of f16, 16 of bf16): fewer steps for a bisection.
template <int DT>
struct Key {
  static constexpr int S = DT == BPC_F32 ? 0 : DT == BPC_F16 ? 13 : 16;
  static constexpr uint32_t kLowest = kLowestKey >> S;
  static __device__ uint32_t of(float x) { return order_key(x) >> S; }
  static __device__ float value(uint32_t key) {   // of a key that is neither 0 nor a NaN's
    const uint32_t k = key << S | ((1u << S) - 1);
    return __uint_as_float(k & 0x80000000u ? key << S & 0x7fffffffu : ~k);
  }
};

// How many of a wave's keys reach `least`: a comparison each, the counting is the scalar unit's.
__device__ inline uint32_t wave_count(uint32_t key, uint32_t least) { return (uint32_t)__popcll(__ballot(key >= least)); }

// The k-th largest of n keys (1 <= k): the largest key that at least k of them reach, or 0 if fewer than k
// reach `lo`.  No key is above `hi`.  Stops as soon as a key is found that no more than k + slack reach (slack 0:
// the keys that reach it are those that reach the k-th largest all the same).  *reach: how many reach the answer.
// count(least): how many keys reach `least`, the same in every thread.
template <class Count>
__device__ uint32_t kth_key(const Count &count, uint32_t k, uint32_t lo, uint32_t hi, uint32_t slack, uint32_t *reach) {
  uint32_t at = count(lo);
  if (at < k) {
    *reach = at;
    return 0;
  }
  while (lo < hi && at > k + slack) {
    const uint32_t mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);
    const uint32_t c = count(mid);
    if (c >= k) {
      lo = mid;
      at = c;
    } else {
      hi = mid - 1;
    }
  }
  *reach = at;
  return lo;
}

// The same, beginning in steps down from the largest logit: a few are enough for logits of ordinary spread.
template <class K, class Count>
__device__ uint32_t kth_key_from_top(const Count &count, uint32_t k, float top, uint32_t slack, uint32_t *reach) {
  uint32_t lo = K::kLowest, hi = K::of(top);
  for (float x = 2.0f; x < 1e5f; x *= 2.0f) {
    const uint32_t key = K::of(top - x);
    if (key <= K::kLowest) break;
    if (count(key) >= k) {
      lo = key;
      break;
    }
    hi = key - 1;
  }
  return kth_key(count, k, lo, hi, slack, reach);
}

// Adds up the waves' counts with one barrier a count: three counters take turns, each is cleared behind the barrier
// after the one that it was read behind.  (All threads, a barrier before the first add and before the next Tally.)
struct Tally {
  uint32_t *counters, turn = 0;
  __device__ explicit Tally(uint32_t *lds) : counters(lds) {
    if (threadIdx.x < 3) counters[threadIdx.x] = 0;
    __syncthreads();
  }
  __device__ uint32_t add(uint32_t wave_total) {
    if ((threadIdx.x & 63) == 0 && wave_total) atomicAdd(&counters[turn], wave_total);
    __syncthreads();
    const uint32_t all = counters[turn];
    turn = turn == 2 ? 0 : turn + 1;
    if (threadIdx.x == 0) counters[turn == 2 ? 0 : turn + 1] = 0;
    return all;
  }
};

// Largest logits and sums of exponentials of the groups of four vectors a thread, from vector v of the row on.
template <int DT, int LANES, int T>
__device__ void group_sums(const Row<DT> &row, const Stretch &all, uint32_t v, float c2, float (&m)[4], float (&s)[4]) {
  constexpr int E = Num<DT>::E;
  u32x4 w[4];
  if (v + 4 * T <= all.b1) {
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = row.load_once(v + u * T, threadIdx.x);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      w[u] = Num<DT>::masked();
      if (v + u * T + threadIdx.x < all.b1) w[u] = row.load_once(v + u * T, threadIdx.x);
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float x[E];
    Num<DT>::widen(w[u], x);
    m[u] = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) m[u] = fmaxf(m[u], x[i]);
    m[u] = lanes_all<LANES>(m[u], Larger());
    const float ref2 = base2_ref(m[u], c2);
    s[u] = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) s[u] += base2_exp(x[i], c2, ref2);
    s[u] = lanes_all<LANES>(s[u], Plus());
  }
}

// The groups of a row by many workgroups, a load of four vectors a thread each: largest logits and sums of row r at
// `groups` + 2 * n_groups * r.
template <int DT, int LANES>
__global__ __launch_bounds__(kTopThreads) void logits_groups_kernel(TeacherArgs g, uint32_t n_groups, float *groups) {
  constexpr int T = kTopThreads;
  const uint64_t r = blockIdx.y;
  if (g.a.weight && uniform_load(g.a.weight + r) == 0.0f) return;
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  const Stretch all(row, 0, row.nv);
  const uint32_t v = blockIdx.x * 4 * T;
  float m[4], s[4];
  group_sums<DT, LANES, T>(row, all, all.b0 + v, g.c2, m, s);
  float *at = groups + 2ull * n_groups * r;
  if (threadIdx.x % LANES == 0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t id = (v + u * T + threadIdx.x) / LANES;
      at[id] = m[u];
      at[n_groups + id] = s[u];
    }
  }
}

// Rows by groups.  One pass finds every group's largest logit and its sum of exponentials (relative to that logit); at
// least k logits reach the k-th largest of the groups' largest (or a little less), so only the few groups that reach
// it are looked through again for candidates.  A group is LANES neighbouring vectors, a line of 128 bytes or a part of one
// (two lines in long rows), so that looking through it again moves no more than it holds.  (8192 x 131072 bf16, k = 256:
// with groups of vectors 4 KB apart the second look moved a whole row, 560 us against 531 at that time; with half lines
// 535 us against 447, more groups to search and fewer workgroups a compute unit.)
template <int DT, int LANES, int T>
__global__ __launch_bounds__(T) void logits_topk_groups_kernel(TeacherArgs g, uint32_t n_groups, uint32_t cap, uint32_t region,
                                                             const float *groups) {
  using K = Key<DT>;
  constexpr int E = Num<DT>::E;
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ float lds[T / 64];
  __shared__ uint32_t counters[3], scan_lds[T / 64], before[T];
  __shared__ uint32_t n_cand, n_level, pick[2];
  __shared__ unsigned long long left_sum;
  const uint64_t r = blockIdx.x;
  uint8_t *rec = g.out + uniform_off(r * g.a.message_stride);
  if (g.a.weight && uniform_load(g.a.weight + r) == 0.0f) {
    close_record<T>(g, rec, 0, 0.0f, kNegInf);
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  uint32_t *gkey = reinterpret_cast<uint32_t *>(dyn);
  float *gsum = reinterpret_cast<float *>(gkey + n_groups);
  uint32_t *ckey = reinterpret_cast<uint32_t *>(dyn + region);
  uint32_t *cidx = ckey + cap;
  uint16_t *glist = reinterpret_cast<uint16_t *>(cidx + cap);
  const Stretch all(row, 0, row.nv);
  const uint32_t b0 = all.b0, b1 = all.b1;
  const float c2 = g.c2;
  float top = kNegInf;
  if (groups) {   // (by logits_groups_kernel)
    const float *at = groups + 2ull * n_groups * r;
    for (uint32_t i = threadIdx.x; i < n_groups; i += T) {
      const float m = at[i];
      top = fmaxf(top, m);
      gkey[i] = __float_as_uint(m);
      gsum[i] = at[n_groups + i];
    }
  } else {
    for (uint32_t v = 0; v < n_groups * LANES; v += 4 * T) {
      float m[4], s[4];
      group_sums<DT, LANES, T>(row, all, b0 + v, c2, m, s);
#pragma unroll
      for (int u = 0; u < 4; ++u) top = fmaxf(top, m[u]);
      if (threadIdx.x % LANES == 0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t id = (v + u * T + threadIdx.x) / LANES;
          gkey[id] = __float_as_uint(m[u]);
          gsum[id] = s[u];
        }
      }
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n_groups; i += T) gkey[i] = K::of(__uint_as_float(gkey[i]));
  // the vectors beside the body are nobody's group: they are looked through in any case
  float edge[E];
  uint32_t edge_v;
  const bool has_edge = all.edge(&edge_v);
  bool odd = false;
  if (has_edge) {
    row.load_any(edge_v, edge);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      top = fmaxf(top, edge[i]);
      odd = odd || edge[i] != edge[i];
    }
  }
  if (threadIdx.x == 0) {
    n_cand = 0;
    n_level = 0;
    left_sum = 0;
  }
  top = all_max<T>(top, lds);
  const float top2 = base2_ref(top, c2);
  uint32_t low = 0, reach;
  {
    // a lower bound of the k-th largest logit: k groups reach it
    Tally tally(counters);
    const uint4 *quad = reinterpret_cast<const uint4 *>(gkey);
    const auto count = [&](uint32_t key) {
      uint32_t c = 0;
      for (uint32_t i = threadIdx.x; i < n_groups / 4; i += T) {
        const uint4 q = quad[i];
        c += wave_count(q.x, key) + wave_count(q.y, key) + wave_count(q.z, key) + wave_count(q.w, key);
      }
      return tally.add(c);
    };
    low = kth_key_from_top<K>(count, g.a.k, top, g.a.k / 8 + 4, &reach);
    if (low == 0) low = K::kLowest;
  }
  float rest = 0.0f;   // relative to 2^top2
  uint32_t mine = 0, n_listed;
  for (uint32_t i = threadIdx.x; i < n_groups; i += T) {
    const uint32_t key = gkey[i];
    const float sum = gsum[i];
    odd = odd || sum != sum;
    if (key >= low) ++mine;
    else if (key != 0) rest += sum * exp2_hw(base2_ref(K::value(key), c2) - top2);
  }
  // (listed by a prefix sum, so that the sum over what these groups hold beside the candidates is always formed in
  // the same order)
  uint32_t at = block_exclusive_scan<T>(mine, scan_lds, &n_listed);
  for (uint32_t i = threadIdx.x; mine && i < n_groups; i += T)
    if (gkey[i] >= low) glist[at++] = (uint16_t)i;
  if (__syncthreads_or(odd || !(fabsf(top * c2) < kFarRef))) {   // a NaN, an infinity, numbers far from 0, nothing at all
    select_any<DT, T>(g, row, rec);
    return;
  }
  const float low_value = K::value(low);
  const auto look = [&](const float *x, uint32_t j0) {
    float most = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) most = fmaxf(most, x[i]);
#pragma unroll
    for (int i = 0; i < E; ++i) rest += x[i] >= low_value ? 0.0f : base2_exp(x[i], c2, top2);
    if (most >= low_value) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (x[i] >= low_value) {
          const uint32_t to = atomicAdd(&n_cand, 1u);
          if (to < cap) {
            ckey[to] = K::of(x[i]);
            cidx[to] = j0 + i;
          }
        }
      }
    }
  };
  const uint32_t pairs = n_listed * LANES;
  for (uint32_t p0 = 0; p0 < pairs; p0 += 4 * T) {   // (four loads on their way at a time)
    uint32_t v[4];
    u32x4 w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t p = p0 + u * T + threadIdx.x;
      v[u] = p < pairs ? b0 + glist[p / LANES] * LANES + p % LANES : b1;
      if (v[u] < b1) w[u] = row.load(0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (v[u] < b1) {
        float x[E];
        Num<DT>::widen(w[u], x);
        look(x, v[u] * E - row.off);
      }
    }
  }
  if (has_edge) look(edge, edge_v * E - row.off);
  __syncthreads();
  const uint32_t cand = n_cand;
  if (cand > cap) {   // more logits level with the bound than there is room for
    __syncthreads();
    select_any<DT, T>(g, row, rec);
    return;
  }
  const uint32_t take = cand < g.a.k ? cand : g.a.k;
  // candidates to list: those above `kth`, and of those level with it the ones up to index `last`
  uint32_t kth = low, last = 0xffffffffu;
  if (take < cand) {
    constexpr uint32_t kOneWave = 512;
    const uint32_t high = K::of(top);
    if (cand <= kOneWave) {   // (uniform) by one wave, out of its registers
      if (threadIdx.x < 64) {
        uint32_t key[kOneWave / 64];
#pragma unroll
        for (uint32_t i = 0; i < kOneWave / 64; ++i) {
          const uint32_t e = threadIdx.x + i * 64;
          key[i] = e < cand ? ckey[e] : 0u;
        }
        const auto count = [&](uint32_t least) {
          uint32_t c = 0;
#pragma unroll
          for (uint32_t i = 0; i < kOneWave / 64; ++i)
            if (i * 64 < cand) c += wave_count(key[i], least);
          return c;
        };
        const uint32_t found = kth_key(count, take, low, high, 0, &reach);
        const uint32_t above = reach > take ? count(found + 1) : 0;
        if (threadIdx.x == 0) {
          pick[0] = found;
          pick[1] = reach > take ? take - above : 0xffffffffu;
        }
      }
    } else {
      Tally tally(counters);
      const uint32_t rounds = (cand + T - 1) / T;
      const auto count = [&](uint32_t least) {
        uint32_t c = 0;
        for (uint32_t i = 0; i < rounds; ++i) {
          const uint32_t e = threadIdx.x + i * T;
          c += wave_count(e < cand ? ckey[e] : 0u, least);
        }
        return tally.add(c);
      };
      const uint32_t found = kth_key(count, take, low, high, 0, &reach);
      const uint32_t above = reach > take ? count(found + 1) : 0;
      if (threadIdx.x == 0) {
        pick[0] = found;
        pick[1] = reach > take ? take - above : 0xffffffffu;
      }
    }
    __syncthreads();
    kth = pick[0];
    const uint32_t open = pick[1];   // how many of those level with the k-th are listed (all of them: 2^32 - 1)
    if (open != 0xffffffffu) {
      // those with the lowest indices: their indices side by side, the one with open - 1 smaller ones is the last
      uint32_t *level = gkey;
      for (uint32_t i = threadIdx.x; i < cand; i += T)
        if (ckey[i] == kth) level[atomicAdd(&n_level, 1u)] = cidx[i];
      __syncthreads();
      const uint32_t n = n_level;
      for (uint32_t i = threadIdx.x; i < n; i += T) {
        uint32_t smaller = 0;
        for (uint32_t o = 0; o < n; ++o) smaller += level[o] < level[i] ? 1u : 0u;
        if (smaller == open - 1) pick[1] = level[i];
      }
      __syncthreads();
      last = pick[1];
    }
  }
  // index order: a bit a logit for what is listed (in place of the groups), a prefix sum over stretches of words
  uint32_t *bits = gkey;
  const uint32_t span = (row.nv * E + 128 * T - 1) / (128 * T) * 4;   // words of a thread's stretch, whole quads
  for (uint32_t i = threadIdx.x; i < span / 4 * T; i += T) reinterpret_cast<uint4 *>(bits)[i] = uint4{0, 0, 0, 0};
  __syncthreads();
  const auto listed = [&](uint32_t i) { return ckey[i] > kth || (ckey[i] == kth && cidx[i] <= last); };
  float over = kNegInf;   // the largest candidate that is not listed
  for (uint32_t i = threadIdx.x; i < cand; i += T) {
    if (listed(i)) atomicOr(&bits[cidx[i] >> 5], 1u << (cidx[i] & 31));
    else over = fmaxf(over, K::value(ckey[i]));
  }
  __syncthreads();
  {
    uint32_t n = 0, all;
    for (uint32_t i = 0; i < span / 4; ++i) {
      const uint4 q = reinterpret_cast<const uint4 *>(bits)[threadIdx.x * (span / 4) + i];
      n += __popc(q.x) + __popc(q.y) + __popc(q.z) + __popc(q.w);
    }
    before[threadIdx.x] = block_exclusive_scan<T>(n, scan_lds, &all);
  }
  if (take < cand) {
    // the candidates lie in any order: the sum of those not listed is formed in whole numbers, 2^-40 of the largest
    over = base2_ref(all_max<T>(over, lds), c2);
    unsigned long long sum = 0;
    for (uint32_t i = threadIdx.x; i < cand; i += T)
      if (!listed(i)) sum += (unsigned long long)(base2_exp(K::value(ckey[i]), c2, over) * 0x1p40f);
    if (sum) atomicAdd(&left_sum, sum);
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < cand; i += T) {
    if (!listed(i)) continue;
    const uint32_t j = cidx[i], word = j >> 5, stretch = word / span;
    uint32_t place = before[stretch];
    for (uint32_t q = stretch * span; q < word; ++q) place += __popc(bits[q]);
    place += __popc(bits[word] & ((1u << (j & 31)) - 1));
    if (place < g.a.k) put_entry(g, rec, place, j, K::value(ckey[i]) - top);
  }
  rest = all_sum<T>(rest, lds);
  if (take < cand) rest += (float)left_sum * 0x1p-40f * exp2_hw(over - top2);
  // (from the rounded reference to the largest logit itself)
  close_record<T>(g, rec, take, rest * exp2_hw(-__builtin_fmaf(top, c2, -top2)), top);
}

// ---- short rows of which many logits are listed: the whole row in LDS

template <int DT>
__global__ __launch_bounds__(kTopThreads) void logits_topk_dense_kernel(TeacherArgs g) {
  using K = Key<DT>;
  constexpr int E = Num<DT>::E, T = kTopThreads, WAVES = T / 64;
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ float lds[WAVES];
  __shared__ uint32_t counters[3], above_of[WAVES], level_of[WAVES];
  const uint64_t r = blockIdx.x;
  uint8_t *rec = g.out + uniform_off(r * g.a.message_stride);
  if (g.a.weight && uniform_load(g.a.weight + r) == 0.0f) {
    close_record<T>(g, rec, 0, 0.0f, kNegInf);
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  // (keys as the vectors lie: logit j is number j + row.off, what is outside the row has key 0)
  uint32_t *key = reinterpret_cast<uint32_t *>(dyn);
  const uint32_t n = row.nv * E, quads = n / 4;
  float top = kNegInf;
  bool odd = false;
  for (uint32_t v = threadIdx.x; v < row.nv; v += T) {
    float y[E];
    row.load_any(v, y);
    uint4 *to = reinterpret_cast<uint4 *>(key + v * E);
#pragma unroll
    for (int i = 0; i < E; i += 4) to[i / 4] = uint4{K::of(y[i]), K::of(y[i + 1]), K::of(y[i + 2]), K::of(y[i + 3])};
#pragma unroll
    for (int i = 0; i < E; ++i) {
      top = fmaxf(top, y[i]);
      odd = odd || y[i] != y[i];
    }
  }
  top = all_max<T>(top, lds);
  if (__syncthreads_or(odd || !(fabsf(top * g.c2) < kFarRef))) {   // a NaN, an infinity, numbers far from 0, nothing at all
    select_any<DT, T>(g, row, rec);
    return;
  }
  uint32_t reach, kth;
  {
    Tally tally(counters);
    const auto count = [&](uint32_t least) {
      uint32_t c = 0;
      for (uint32_t i = threadIdx.x; i < quads; i += T) {
        const uint4 q = reinterpret_cast<const uint4 *>(key)[i];
        c += wave_count(q.x, least) + wave_count(q.y, least) + wave_count(q.z, least) + wave_count(q.w, least);
      }
      return tally.add(c);
    };
    kth = kth_key_from_top<K>(count, g.a.k, top, 0, &reach);
    if (kth == 0) kth = K::kLowest;   // (fewer than k: all of them)
  }
  // each wave a stretch of the row, 64 logits at a time: how many are above the k-th and level with it ...
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, stretch = (n + T - 1) / T * 64;
  const uint32_t lo = wave * stretch < n ? wave * stretch : n, hi = lo + stretch < n ? lo + stretch : n;
  uint32_t above = 0, level = 0;
  for (uint32_t j = lo; j < hi; j += 64) {
    const uint32_t x = j + lane < hi ? key[j + lane] : 0u;
    above += (uint32_t)__popcll(__ballot(x > kth));
    level += (uint32_t)__popcll(__ballot(x == kth));
  }
  if (lane == 0) {
    above_of[wave] = above;
    level_of[wave] = level;
  }
  __syncthreads();
  uint32_t all_above = 0, all_level = 0, level_at = 0;
  above = 0;
#pragma unroll
  for (uint32_t w = 0; w < WAVES; ++w) {
    above += w < wave ? above_of[w] : 0u;
    level_at += w < wave ? level_of[w] : 0u;
    all_above += above_of[w];
    all_level += level_of[w];
  }
  // ... of which the first `open` are listed; then where each goes
  const uint32_t open = g.a.k - all_above;
  uint32_t at = above + (level_at < open ? level_at : open);
  const float top2 = base2_ref(top, g.c2);
  float rest = 0.0f;
  for (uint32_t j = lo; j < hi; j += 64) {
    const uint32_t x = j + lane < hi ? key[j + lane] : 0u;
    const uint64_t before = (1ull << lane) - 1, same = __ballot(x == kth);
    const bool take = x > kth || (x == kth && level_at + (uint32_t)__popcll(same & before) < open);
    const uint64_t taken = __ballot(take);
    if (take) put_entry(g, rec, at + (uint32_t)__popcll(taken & before), j + lane - row.off, K::value(x) - top);
    else if (x != 0) rest += base2_exp(K::value(x), g.c2, top2);
    level_at += (uint32_t)__popcll(same);
    at += (uint32_t)__popcll(taken);
  }
  rest = all_sum<T>(rest, lds);
  close_record<T>(g, rec, all_above + (all_level < open ? all_level : open), rest * exp2_hw(-__builtin_fmaf(top, g.c2, -top2)), top);
}

// Rows of any length by the radix select alone.
template <int DT>
__global__ __launch_bounds__(kTopThreads) void logits_topk_any_kernel(TeacherArgs g) {
  const uint64_t r = blockIdx.x;
  uint8_t *rec = g.out + uniform_off(r * g.a.message_stride);
  if (g.a.weight && uniform_load(g.a.weight + r) == 0.0f) {
    close_record<kTopThreads>(g, rec, 0, 0.0f, kNegInf);
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  select_any<DT, kTopThreads>(g, row, rec);
}

template <int DT, int LANES, int T>
static hipError_t run_groups(const TeacherArgs &g, const TopkPlan &p, uint8_t *ws, hipStream_t stream) {
  float *groups = nullptr;
  if constexpr (T == 1024 && LANES > 1) {   // (few rows are long: 1024 threads, four vectors or more for each entry)
    if (p.few) {
      groups = reinterpret_cast<float *>(ws);
      const uint32_t per = 4 * kTopThreads;
      logits_groups_kernel<DT, LANES><<<dim3(p.n_groups * LANES / per, (uint32_t)g.a.rows), kTopThreads, 0, stream>>>(g, p.n_groups, groups);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  logits_topk_groups_kernel<DT, LANES, T><<<(uint32_t)g.a.rows, T, p.lds, stream>>>(g, p.n_groups, p.cap, p.region, groups);
  return hipGetLastError();
}

template <int DT, int T>
static hipError_t run_lanes(const TeacherArgs &g, const TopkPlan &p, uint8_t *ws, hipStream_t stream) {
  if constexpr (T != 64)   // (one wave takes short rows only)
    if (p.lanes == 16) return run_groups<DT, 16, T>(g, p, ws, stream);
  if (p.lanes == 8) return run_groups<DT, 8, T>(g, p, ws, stream);
  if (p.lanes == 4) return run_groups<DT, 4, T>(g, p, ws, stream);
  if (p.lanes == 2) return run_groups<DT, 2, T>(g, p, ws, stream);
  return run_groups<DT, 1, T>(g, p, ws, stream);
}

template <int DT>
static hipError_t run_typed(const TeacherArgs &g, uint8_t *ws, hipStream_t stream) {
  const TopkPlan p = topk_plan(g.a.rows, g.a.vocab, g.a.k, DT, g.a.row_stride);
  if (p.form == TopkForm::any) {
    logits_topk_any_kernel<DT><<<(uint32_t)g.a.rows, kTopThreads, 0, stream>>>(g);
    return hipGetLastError();
  }
  if (p.form == TopkForm::dense) {
    logits_topk_dense_kernel<DT><<<(uint32_t)g.a.rows, kTopThreads, p.lds, stream>>>(g);
    return hipGetLastError();
  }
  return p.threads == 64 ? run_lanes<DT, 64>(g, p, ws, stream)
         : p.threads == 256 ? run_lanes<DT, 256>(g, p, ws, stream)
                            : run_lanes<DT, 1024>(g, p, ws, stream);
}

hipError_t logits_topk(const DistillCall &call, uint8_t *out, uint8_t *ws, hipStream_t stream) {
  TeacherArgs g{};
  g.a = call;
  g.c2 = (float)(1.44269504088896340736 / (double)call.temperature);
  g.out = out;
  switch (call.dtype) {
    case BPC_F32: return run_typed<BPC_F32>(g, ws, stream);
    case BPC_F16: return run_typed<BPC_F16>(g, ws, stream);
    default: return run_typed<BPC_BF16>(g, ws, stream);
  }
}

}  // namespace bpc
