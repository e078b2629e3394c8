// What the kernels that write the cache's blocks share: the lookups of a
// sequence's part of a call, and the block quantiser.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mds_cache_internal.h"

namespace mds {
namespace cache {

namespace {

constexpr unsigned kFull = 0xffffffffu;

__device__ __forceinline__ int sequence(const State& s, const int32_t* seqs, int b) {
  const int q = seqs[b];
  if (q >= s.max_seqs) atomicOr(s.status, MDS_ST_BADSEQ);
  return q >= s.max_seqs ? -1 : q;
}

__device__ __forceinline__ int live_count(const int32_t* counts, int b, int n) {
  return counts ? min(max(counts[b], 0), n) : n;
}

__device__ __forceinline__ int64_t tile_of(const State& s, int layer, int page, int kv, int h) {
  return (((int64_t)layer * s.pages + page) * 2 + kv) * s.kv_heads + h;
}

// ------------------------------------------------------------ the quantiser

// A warp holds one block of one head: U = head_dim / 16 lanes a row, 16
// values a lane, 32 / U rows at once, U / 2 times.  The kernels wait for
// memory, not for arithmetic, so what a lane holds decides how many warps hide
// that: bfloat16 inputs, and the values of stored bytes (exact in bfloat16),
// stay packed.
constexpr unsigned kInf = 0x7f800000u;   // magnitudes of floats order as their bits do

template <typename T>
struct Lane16;

template <>
struct Lane16<__nv_bfloat16> {
  uint4 w[2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    w[0] = __ldg(reinterpret_cast<const uint4*>(p));
    w[1] = __ldg(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ void zero() { w[0] = w[1] = uint4{0, 0, 0, 0}; }
  __device__ __forceinline__ unsigned get(int i) const {
    const uint4& x = w[i >> 2];
    return (i & 3) == 0 ? x.x : (i & 3) == 1 ? x.y : (i & 3) == 2 ? x.z : x.w;
  }
  __device__ __forceinline__ void set(int i, unsigned v) {
    uint4& x = w[i >> 2];
    ((i & 3) == 0 ? x.x : (i & 3) == 1 ? x.y : (i & 3) == 2 ? x.z : x.w) = v;
  }
  __device__ __forceinline__ void values(const float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __nv_bfloat162 x = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      set(i, *reinterpret_cast<const unsigned*>(&x));
    }
  }
  // NaN becomes 0; the largest magnitude of the finite values, or kInf and
  // more where any is not (then once more with `clean`)
  template <bool clean>
  __device__ __forceinline__ unsigned largest() {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned lo = get(i) << 16 & 0x7fff0000u, hi = get(i) & 0x7fff0000u;
      if (clean) {
        set(i, (lo > kInf ? 0u : get(i) & 0xffffu) | (hi > kInf ? 0u : get(i) & 0xffff0000u));
        lo = lo >= kInf ? 0u : lo;
        hi = hi >= kInf ? 0u : hi;
      }
      m = max(m, max(lo, hi));
    }
    return m;
  }
  __device__ __forceinline__ float at(int i) const {
    return __uint_as_float(i & 1 ? get(i >> 1) & 0xffff0000u : get(i >> 1) << 16);
  }
};

template <>
struct Lane16<float> {
  float v[16];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = __ldg(reinterpret_cast<const float4*>(p) + i);
      v[4 * i] = x.x, v[4 * i + 1] = x.y, v[4 * i + 2] = x.z, v[4 * i + 3] = x.w;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ void values(const float* x) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = x[i];
  }
  template <bool clean>
  __device__ __forceinline__ unsigned largest() {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      unsigned x = __float_as_uint(v[i]) & 0x7fffffffu;
      if (clean) {
        if (x > kInf) v[i] = 0.f;
        x = x >= kInf ? 0u : x;
      }
      m = max(m, x);
    }
    return m;
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
};

// The scale: the least e in [-117, 119] with max <= 448 * 2^e, from the
// maximum's exponent x and mantissa m: 448 = 1.75 * 2^8, so e = x - 8 if
// m <= 1.75, else x - 7.  Returns 2^e and sets inv to 2^-e.
__device__ __forceinline__ float block_scale(unsigned bits, float* inv) {
  int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = bits == 0 ? 0 : min(max(e, -117), 119);
  *inv = __uint_as_float((unsigned)(127 - e) << 23);
  return __uint_as_float((unsigned)(127 + e) << 23);
}

template <typename T, int U>
struct Block {
  static constexpr int kPasses = U / 2;
  static constexpr int kRows = 32 / U;
  Lane16<T> v[kPasses];

  // The block's scale; lane-uniform.
  __device__ __forceinline__ float scale(float* inv, bool* odd) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) m = max(m, v[i].template largest<false>());
    unsigned bits = __reduce_max_sync(kFull, m);
    *odd = bits >= kInf;
    if (*odd) {
      m = 0;
#pragma unroll
      for (int i = 0; i < kPasses; ++i) m = max(m, v[i].template largest<true>());
      bits = __reduce_max_sync(kFull, m);
    }
    return block_scale(bits, inv);
  }
};

__device__ __forceinline__ void decode4(unsigned w, float scale, float* v) {
  unsigned lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  v[0] = a.x * scale, v[1] = a.y * scale, v[2] = b.x * scale, v[3] = b.y * scale;
}
__device__ __forceinline__ void decode16(const uint4& x, float scale, float* v) {
  decode4(x.x, scale, v);
  decode4(x.y, scale, v + 4);
  decode4(x.z, scale, v + 8);
  decode4(x.w, scale, v + 12);
}

__device__ __forceinline__ unsigned encode4(float a, float b, float c, float d) {
  unsigned w;
  asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(w)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return w;
}
template <typename T>
__device__ __forceinline__ uint4 encode16(const Lane16<T>& v, float inv) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = encode4(v.at(4 * i) * inv, v.at(4 * i + 1) * inv, v.at(4 * i + 2) * inv, v.at(4 * i + 3) * inv);
  return uint4{w[0], w[1], w[2], w[3]};
}

}  // namespace

}  // namespace cache
}  // namespace mds
