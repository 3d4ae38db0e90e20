// Rows of logits: how a row is cut into 16-byte vectors and chunks, number types, workgroup
// reductions.  Shared by the teacher's top-k messages (logits_topk.hip) and the student's loss and
// gradient (distill_student.hpp).
#pragma once
#include "device_utils.hpp"
#include "distill_geometry.hpp"
#include <type_traits>

namespace bpc {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_huge_valf();

// 16 bytes at any element's address (the hardware takes such accesses; 2 % slower than aligned ones in a copy of
// 1 GiB of 2-byte elements, reads 8 %: reads are aligned here).
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// Eight 16-bit elements of which those whose bit is set become -inf.
__device__ inline u32x4 mask_halves(u32x4 v, uint32_t bits, uint32_t minus_inf) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * i, 1), hi = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * i + 1, 1);
    const uint32_t m = __builtin_amdgcn_perm(hi, lo, 0x07060100u);
    v[i] = (v[i] & ~m) | (minus_inf & m);
  }
  return v;
}

// One type of logits: E of them fill a 16-byte vector.
template <int DT> struct Num;
template <> struct Num<BPC_F32> {
  using raw = float;
  static constexpr int E = 4;
  static __device__ void widen(u32x4 v, float *x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ u32x4 narrow(const float *x) { return as_u32x4(x[0], x[1], x[2], x[3]); }
  static __device__ u32x4 masked() { return u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }   // -inf
  // The elements whose bit is set become -inf.
  static __device__ u32x4 mask(u32x4 v, uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)bits, i, 1);
      v[i] = (v[i] & ~m) | (0xff800000u & m);
    }
    return v;
  }
  static __device__ float get(const raw *p) { return *p; }
  static __device__ void put(raw *p, float x) { *p = x; }
};
template <> struct Num<BPC_F16> {
  using raw = _Float16;
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static constexpr int E = 8;
  static __device__ void widen(u32x4 v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = v[i];   // (a vector's component has no address)
      const x2 h = __builtin_bit_cast(x2, w);
      x[2 * i] = (float)h.x;
      x[2 * i + 1] = (float)h.y;
    }
  }
  static __device__ u32x4 narrow(const float *x) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x2 h;
      h.x = (_Float16)x[2 * i];
      h.y = (_Float16)x[2 * i + 1];
      v[i] = __builtin_bit_cast(uint32_t, h);
    }
    return v;
  }
  static __device__ u32x4 masked() { return u32x4{0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u}; }   // -inf
  static __device__ u32x4 mask(u32x4 v, uint32_t bits) { return mask_halves(v, bits, 0xfc00fc00u); }
  static __device__ float get(const raw *p) { return (float)*p; }
  static __device__ void put(raw *p, float x) { *p = (_Float16)x; }
};
template <> struct Num<BPC_BF16> {
  using raw = __bf16;
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  static constexpr int E = 8;
  static __device__ void widen(u32x4 v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ u32x4 narrow(const float *x) {   // (rounds to nearest even)
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x2 h;
      h.x = (__bf16)x[2 * i];
      h.y = (__bf16)x[2 * i + 1];
      v[i] = __builtin_bit_cast(uint32_t, h);
    }
    return v;
  }
  static __device__ u32x4 masked() { return u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }   // -inf
  static __device__ u32x4 mask(u32x4 v, uint32_t bits) { return mask_halves(v, bits, 0xff80ff80u); }
  static __device__ float get(const raw *p) { return (float)*p; }
  static __device__ void put(raw *p, float x) { *p = (__bf16)x; }
};

// 2^x with the hardware's instruction (1 ulp; results below 2^-126 become 0, 2^-inf = 0).
__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// What exponents are taken relative to: m, or 0 where everything is masked (-inf - -inf is no number).
__device__ inline float ref_of(float m) { return m == kNegInf ? 0.0f : m; }

// What exponents of base 2 are taken relative to: the largest logit times c2, as f32 rounds it.  Any reference will
// do as long as all parties to a sum know it, so the rounding costs nothing, and x * c2 - reference is one
// instruction, with one rounding.  Below -2^20 (masked by -inf or by a type's lowest value) it stays there: 2^x is 0
// next to any row that is handled so.
constexpr float kLowRef = -0x1p20f;
__device__ inline float base2_ref(float m, float c2) { return fmaxf(m * c2, kLowRef); }
__device__ inline float base2_exp(float x, float c2, float ref2) { return exp2_hw(__builtin_fmaf(x, c2, -ref2)); }
// Rows whose largest logit is further from 0 than this (or NaN, or infinite) go the other way: the rounding of the
// reference would be felt.
constexpr float kFarRef = 0x1p16f;

// A row whose elements start `off` elements into its first 16-byte block: vector v holds elements
// v * E - off and on.  The first and the last vector may be partial, the others are read whole.
template <int DT>
struct Row {
  using N = Num<DT>;
  static constexpr int E = N::E;
  const typename N::raw *p;
  uint32_t vocab, off, nv;
  __device__ Row(const void *base, uint64_t row, uint64_t stride, uint32_t vocab_)
      : p(reinterpret_cast<const typename N::raw *>(base) + uniform_off(row * stride)), vocab(vocab_) {
    off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15) / sizeof(typename N::raw);
    nv = (off + vocab + E - 1) / E;
  }
  __device__ bool whole(uint32_t v) const { return v * E >= off && v * E - off + E <= vocab; }
  // Whole vectors: vector v + lane, v the same in every lane and lane < 2^28 (one scalar base and a 32-bit lane offset:
  // no vector instruction for the address).  once: read once only, so not kept in the caches (a read of 2 GiB 7.1 TB/s
  // against 6.4).
  __device__ const u32x4 *at(int v, uint32_t lane) const {
    return reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint8_t *>(p) + ((int64_t)v * 16 - (int64_t)(off * sizeof(*p))) + lane * 16u);
  }
  __device__ u32x4 load(int v, uint32_t lane) const { return *at(v, lane); }
  __device__ u32x4 load_once(int v, uint32_t lane) const { return __builtin_nontemporal_load(at(v, lane)); }
  // Any vector; what lies outside the row reads as -inf and is not touched.
  __device__ void load_any(uint32_t v, float *x) const {
    if (whole(v)) {
      N::widen(load(0, v), x);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int j = (int)(v * E) - (int)off + i;
        x[i] = j >= 0 && j < (int)vocab ? N::get(p + j) : kNegInf;
      }
    }
  }
};

// A stretch [v0, v1) of a row's vectors: a body [b0, b1) of whole vectors from the start of a 128-byte line on, so that
// what a wave reads and writes at a time is whole lines (gradients of rows of 100,514 bytes: 238 us without, 223 with
// it), and up to nine vectors around it, a thread each.
struct Stretch {
  uint32_t v0, v1, b0, b1;
  template <int DT>
  __device__ Stretch(const Row<DT> &row, uint32_t v0_, uint32_t v1_) : v0(v0_), v1(v1_) {
    const uint32_t w0 = v0 < v1 && !row.whole(v0) ? v0 + 1 : v0;
    b0 = w0 + ((8 - ((uint32_t)(reinterpret_cast<uintptr_t>(row.at((int)w0, 0)) >> 4) & 7)) & 7);
    b1 = v0 < v1 && !row.whole(v1 - 1) ? v1 - 1 : v1;
    b0 = b0 < b1 ? b0 : b1;
  }
  // This thread's vector beside the body.
  __device__ bool edge(uint32_t *v) const {
    const uint32_t n = b0 - v0;
    *v = threadIdx.x < n ? v0 + threadIdx.x : b1 + (threadIdx.x - n);
    return *v < (threadIdx.x < n ? b0 : v1);
  }
};

// Over 2, 4, 8 or 16 neighbouring lanes, in all of them: moves inside a row of lanes cost no LDS access.
template <int LANES, class Op>
__device__ inline float lanes_all(float x, const Op &op) {
  const auto from = [](float y, auto ctrl) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (LANES >= 2) x = op(x, from(x, std::integral_constant<int, 0xB1>{}));    // quad_perm: the other of a pair
  if (LANES >= 4) x = op(x, from(x, std::integral_constant<int, 0x4E>{}));    // the other pair of a quad
  if (LANES >= 8) x = op(x, from(x, std::integral_constant<int, 0x141>{}));   // row_half_mirror: the other quad
  if (LANES >= 16) x = op(x, from(x, std::integral_constant<int, 0x140>{}));  // row_mirror: the other eight
  return x;
}

struct Plus {
  __device__ float operator()(float x, float y) const { return x + y; }
};
struct Larger {
  __device__ float operator()(float x, float y) const { return fmaxf(x, y); }
};
template <class Op>
__device__ inline float wave_all(float x, const Op &op) {
  x = lanes_all<16>(x, op);
  x = op(x, __shfl_xor(x, 16, 64));
  return op(x, __shfl_xor(x, 32, 64));
}
// Over the values that the waves of a workgroup left in LDS, `apart` floats apart, in every thread.
template <int WAVES, class Op>
__device__ inline float waves_all(const float *v, int apart, const Op &op) {
  static_assert(WAVES == 1 || WAVES == 4 || WAVES == 8 || WAVES == 16, "");
  return lanes_all<WAVES>(v[(threadIdx.x % WAVES) * apart], op);
}

// Sum and maximum over a workgroup in a fixed order, in every thread.  `lds`: one float a wave.
template <int THREADS, class Op>
__device__ inline float all_of(float x, float *lds, const Op &op) {
  x = wave_all(x, op);
  if (THREADS == 64) return x;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return waves_all<THREADS / 64>(lds, 1, op);
}
template <int THREADS>
__device__ inline float all_sum(float x, float *lds) { return all_of<THREADS>(x, lds, Plus()); }
template <int THREADS>
__device__ inline float all_max(float x, float *lds) { return all_of<THREADS>(x, lds, Larger()); }

// The fields of a row's record (the record of TOPK / TOPK16 with the mass of the rest and the row's
// largest logit in the header).
struct Record {
  const uint8_t *p;
  uint32_t val_off;
  bool half;
  __device__ Record(const uint8_t *messages, uint64_t row, uint64_t stride, uint32_t k, bool half_)
      : p(messages + uniform_off(row * stride)), val_off(kHeaderBytes + 4 * (uint32_t)ru4(k)), half(half_) {}
  __device__ uint32_t count(uint32_t k) const {   // (never more than there is room for, whatever it says)
    const uint32_t n = *reinterpret_cast<const uint32_t *>(p);
    return n < k ? n : k;
  }
  __device__ float rest() const { return reinterpret_cast<const float *>(p)[1]; }
  __device__ uint32_t idx(uint32_t e) const { return reinterpret_cast<const uint32_t *>(p + kHeaderBytes)[e]; }
  __device__ float val(uint32_t e) const {
    return half ? (float)reinterpret_cast<const _Float16 *>(p + val_off)[e] : reinterpret_cast<const float *>(p + val_off)[e];
  }
};

}  // namespace bpc
