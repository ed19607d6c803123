// Shared by the sequence operators' kernels (seq_*.hip): element types, eight
// consecutive steps as one load or store, and the elementwise functions.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "seq_ops.h"

namespace seqops {

struct bf16 {
  uint16_t v;
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16 x) { return __uint_as_float(uint32_t(x.v) << 16); }

// (nearest even, one instruction for two)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ bf16 from_f<bf16>(float x) {
  return bf16{uint16_t(pack_bf16(x, 0.f))};
}

// Eight consecutive elements as they lie in memory.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
};

// The first `valid` of eight elements at p (more than eight: all), zeros behind
// them; nothing behind them is read.  p needs element alignment only: global
// memory takes 16-byte accesses at any address.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int valid) {
  Raw8<T> r;
  if (valid >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
  }
#pragma unroll
  for (int i = 0; i < int(2 * sizeof(T)); ++i) r.w[i] = 0;
  if (valid > 0) {
#pragma unroll
    for (int j = 0; j < 7; ++j) {
      if (j < valid) {
        if constexpr (sizeof(T) == 4)
          r.w[j] = __float_as_uint(p[j]);
        else
          r.w[j / 2] |= uint32_t(p[j].v) << (16 * (j % 2));
      }
    }
  }
  return r;
}

// The same bits, which the compiler has to unpack again instead of holding what
// it unpacked before: registers.
template <typename T>
__device__ __forceinline__ Raw8<T> again(Raw8<T> r) {
#pragma unroll
  for (int i = 0; i < int(2 * sizeof(T)); ++i) asm volatile("" : "+v"(r.w[i]));
  return r;
}

template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float* v) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 4)
      v[j] = __uint_as_float(r.w[j]);
    else
      v[j] = __uint_as_float(j % 2 ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  }
}

template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float* v) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j] = __float_as_uint(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r.w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
  }
  return r;
}

// Stores the first `valid` of eight elements.  STREAM: past the caches, where
// whole cache lines are written that nothing reads soon (the convolution's
// training step 80 -> 77 us); lines that several stores fill have to meet in the
// L2 (norms: twice as long without).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
template <bool STREAM = false, typename T>
__device__ __forceinline__ void store8(T* p, int valid, const float* v) {
  const Raw8<T> r = pack8<T>(v);
  if (valid >= 8) {
    if constexpr (STREAM) {
#pragma unroll
      for (int i = 0; i < int(sizeof(T)) / 2; ++i)
        __builtin_nontemporal_store(u32x4{r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]},
                                    reinterpret_cast<u32x4*>(p) + i);
    } else {
      __builtin_memcpy(p, &r, sizeof(r));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 7; ++j) {
    if (j < valid) {
      if constexpr (sizeof(T) == 4)
        p[j] = __uint_as_float(r.w[j]);
      else
        p[j].v = uint16_t(r.w[j / 2] >> (16 * (j % 2)));
    }
  }
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// v 2^x, also where 2^x is past fp32's range: zero stays zero, and what the product
// has in range is right.  (Beyond 2^504 and 2^-504 no v but zero has.)
__device__ __forceinline__ float times_exp2(float v, float x) {
  x = x > 504.f ? 504.f : x < -504.f ? -504.f : x;  // (NaN: kept)
  const float f = exp2_fast(0.25f * x);
  return v * f * f * f * f;
}

// 1 / (1 + exp(-x)): one exp2 and one reciprocal, each good to an ulp; exp(-x)
// overflows to infinity, its reciprocal to 0.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp2_fast(-kLog2e * x)); }

// log(1 + exp(x)) = max(x, 0) + log1p(e), e = exp(-|x|) in (0, 1], and
// log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3: steps of 1e-3 keep their
// digits.  2 artanh(s) / s is a polynomial in q = s^2, interpolated at the
// Chebyshev nodes of [0, 1/9] (with these fp32 coefficients within 1.6e-8 of it, a
// relative 7.7e-9).
__device__ __forceinline__ float softplus(float x) {
  const float e = exp2_fast(-kLog2e * __builtin_fabsf(x));
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 0.2815778f;
  p = __builtin_fmaf(p, q, 0.27965158f);
  p = __builtin_fmaf(p, q, 0.40024596f);
  p = __builtin_fmaf(p, q, 0.6666632f);
  p = __builtin_fmaf(p, q, 2.f);
  // (the median of x, 0 and infinity: the larger of x and 0 as one instruction;
  // a NaN comes through s)
  return __builtin_fmaf(s, p, __builtin_amdgcn_fmed3f(x, 0.f, __builtin_inff()));
}

// Keeps what follows in a branch of its own.
__device__ __forceinline__ void branch() { asm volatile(""); }

// Before lanes read what other lanes of their wave have put into LDS.  (The LDS
// serves a wave in order: this holds the compiler to it and is no instruction.)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// DPP moves within a row of 16 lanes or the wave.  `old` is what lanes without
// a source keep.
enum { kRowShl = 0x100, kRowShr = 0x110, kWaveShl1 = 0x130 };
template <int CTRL>
__device__ __forceinline__ float dpp(float old, float src) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(src), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ float dpp0(float src) {  // (zero without a source)
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(src), CTRL, 0xf, 0xf, true));
}

// A seq length of [N], clamped; L without lengths.
__device__ __forceinline__ int seq_len(const int32_t* lengths, int n, int L) {
  if (!lengths) return L;
  const int v = lengths[n];
  return v < 0 ? 0 : v > L ? L : v;
}

}  // namespace seqops
