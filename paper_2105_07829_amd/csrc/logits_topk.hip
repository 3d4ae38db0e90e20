// Teacher side of the distillation from top logits: the k largest logits of every row, in index
// order, and the mass of all others (record format in include/bpc.h).
//
// Logits are ordered by 32-bit keys (order_key): the k-th largest key comes from a radix select,
// whatever the row looks like; of the logits level with it the first ones are listed, by a prefix
// sum over the row in index order.  The mass of the rest is summed over the unlisted logits, never
// formed as a difference.
#include "distill.hpp"
#include "kernels.hpp"

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

// A whole row by a radix select: four passes for the key, one to write.  Right for every row.
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

template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void logits_topk_kernel(TeacherArgs g) {
  const uint64_t r = blockIdx.x;
  uint8_t *rec = g.out + uniform_off(r * g.a.message_stride);
  if (g.a.weight && uniform_load(g.a.weight + r) == 0.0f) {
    close_record<THREADS>(g, rec, 0, 0.0f, kNegInf);
    return;
  }
  const Row<DT> row(g.a.logits, r, g.a.row_stride, g.a.vocab);
  select_any<DT, THREADS>(g, row, rec);
}

template <int DT>
static hipError_t run_typed(const TeacherArgs &g, hipStream_t stream) {
  logits_topk_kernel<DT, 256><<<(uint32_t)g.a.rows, 256, 0, stream>>>(g);
  return hipGetLastError();
}

hipError_t logits_topk(const DistillCall &call, uint8_t *out, uint8_t *ws, hipStream_t stream) {
  (void)ws;
  TeacherArgs g{};
  g.a = call;
  g.c2 = (float)(1.44269504088896340736 / (double)call.temperature);
  g.out = out;
  switch (call.dtype) {
    case BPC_F32: return run_typed<BPC_F32>(g, stream);
    case BPC_F16: return run_typed<BPC_F16>(g, stream);
    default: return run_typed<BPC_BF16>(g, stream);
  }
}

}  // namespace bpc
