// Rotary positions of tree nodes: queries (or any heads) rotated, and keys
// rotated on their way into the cache's 8-bit blocks.
//
//   (a, b) -> m (a cos t - b sin t, a sin t + b cos t),   t = position * f
//
// for the pairs of a head's first `dim` dimensions.
//
// Angles.  f / 2 pi is held as a fraction of a turn in 64 bits, and an integer
// product modulo 2^64 with the position is the angle's fraction of a turn,
// off by at most 2^-64 of a turn a position: nothing to reduce, and as exact
// at position 2^20 as at 1.  Sine and cosine are Taylor sums on an eighth of a turn either way,
// in pairs of floats for the terms that matter (2^-40 absolute).
//
// Rounding.  Queries take the leading floats and are rounded to their type
// once.  A key is rounded to 8 bits behind the rotation, where an error of
// 2^-24 would turn one number in half a million into its neighbour, a
// sixteenth away: its products and sum are kept in two floats, and their sum
// goes to one float by rounding to odd (of the two floats around it the one
// whose last bit is set), which a second rounding cannot tell from the sum
// itself.  What is stored is the quantiser's answer on the exact rotation.
#include <cfloat>

#include "mds_cache_quant.cuh"

namespace mds {
namespace cache {

namespace {

constexpr int kThreads = 256;

struct Turns {
  uint64_t turn[64];   // of a pair, a position
  float2 magnitude;    // in two parts
  int dim, interleaved;
};

template <typename T>
struct Call {
  State s;
  Turns t;
  const int32_t* seqs;
  const int32_t* counts;
  const T* k;
  const T* v;
  const T* q;
  T* out;
  longlong3 ks, vs, qs;
  int layer, n, L, chunks;     // chunks of 16 nodes a sequence
  int q_heads, q_each, q_parts;   // heads a block turns; blocks for them
};

// ------------------------------------------------------- pairs of floats

__device__ __forceinline__ float2 quick_sum(float a, float b) {   // |a| >= |b|
  const float s = __fadd_rn(a, b);
  return float2{s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ float2 sum(float a, float b) {
  const float s = __fadd_rn(a, b), v = __fsub_rn(s, a);
  return float2{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, v)), __fsub_rn(b, v))};
}
__device__ __forceinline__ float2 product(float2 a, float2 b) {
  const float h = __fmul_rn(a.x, b.x);
  return float2{h, __fadd_rn(__fmaf_rn(a.x, b.x, -h), __fmaf_rn(a.x, b.y, __fmul_rn(a.y, b.x)))};
}
// c + z u where the term is smaller than c
__device__ __forceinline__ float2 term(double c, float2 z, float2 u) {
  const float high = (float)c, low = (float)(c - (double)high);
  const float2 p = product(z, u), s = quick_sum(high, p.x);
  return float2{s.x, __fadd_rn(s.y, __fadd_rn(p.y, low))};
}
__device__ __forceinline__ float2 term(double c, float z, float u) {
  const float high = (float)c, low = (float)(c - (double)high);
  const float2 s = quick_sum(high, __fmul_rn(z, u));
  return float2{s.x, __fadd_rn(s.y, low)};
}

// cos and sin of a fraction of a turn (in units of 2^-64): the nearest quarter
// and at most an eighth either way, whose Taylor sums are cut behind a^13 and
// a^14 (the next terms are below 2^-45 and 2^-44).
__device__ __forceinline__ void turn_cos_sin(uint64_t f, float2& c, float2& s) {
  const unsigned quarter = (unsigned)((f + (1ull << 61)) >> 62) & 3u;
  const int64_t r = (int64_t)(f - ((uint64_t)quarter << 62));
  const float rh = __ll2float_rn(r), rl = __ll2float_rn(r - __float2ll_rn(rh));
  constexpr double kTurn = 6.283185307179586476925286766559 / 18446744073709551616.0;
  const float2 p = product(float2{rh, rl}, float2{(float)kTurn, (float)(kTurn - (double)(float)kTurn)});
  const float2 a = quick_sum(p.x, p.y), z = product(a, a);
  float t = __fmaf_rn(z.x, __fmaf_rn(z.x, 1.f / 6227020800.f, -1.f / 39916800.f), 1.f / 362880.f);
  float2 u = term(-1. / 6, z, term(1. / 120, z, term(-1. / 5040, z.x, t)));
  const float2 w = product(a, product(z, u)), y = quick_sum(a.x, w.x);
  const float2 sine{y.x, __fadd_rn(y.y, __fadd_rn(w.y, a.y))};
  t = __fmaf_rn(z.x, __fmaf_rn(z.x, __fmaf_rn(z.x, -1.f / 87178291200.f, 1.f / 479001600.f), -1.f / 3628800.f), 1.f / 40320.f);
  u = term(-0.5, z, term(1. / 24, z, term(-1. / 720, z.x, t)));
  const float2 cosine = term(1., z, u);
  c = quarter & 1u ? sine : cosine;
  s = quarter & 1u ? cosine : sine;
  if (quarter == 1u || quarter == 2u) c = float2{-c.x, -c.y};
  if (quarter & 2u) s = float2{-s.x, -s.y};
}

// x c + y s to one float, rounded to odd.  A sum that is not finite stays as it
// is: what rounding left of it is not a number.
__device__ __forceinline__ float odd_sum(float x, float ch, float cl, float y, float sh, float sl) {
  const float p = __fmul_rn(x, ch), q = __fmul_rn(y, sh);
  const float2 t = sum(p, q);
  if (!(fabsf(t.x) <= FLT_MAX)) return t.x;
  const float rest = __fadd_rn(__fadd_rn(__fmaf_rn(x, ch, -p), __fmaf_rn(y, sh, -q)), __fmaf_rn(x, cl, __fmul_rn(y, sl)));
  const float2 r = sum(t.x, __fadd_rn(t.y, rest));
  const unsigned bits = __float_as_uint(r.x);
  if (!(fabsf(r.y) > 0.f) || (bits & 1u)) return r.x;
  return __uint_as_float((bits ^ __float_as_uint(r.y)) >> 31 ? bits - 1u : bits + 1u);
}

// ----------------------------------------------------------- the lanes' part

// U = head_dim / 16 lanes a row, two chunks of 8 dimensions a lane, chosen so
// that a lane holds both parts of its pairs, 8 unit .. 8 unit + 7.
template <int U>
struct Lane {
  int first, second;   // chunks
  bool turns;
  __device__ __forceinline__ Lane(const Turns& t, int unit) {
    const int half = t.dim >> 4;
    turns = unit < half;
    first = !t.interleaved && turns ? unit : 2 * unit;
    second = !t.interleaved && turns ? unit + half : 2 * unit + 1;
  }
};

__device__ __forceinline__ void load8(float* x, const __nv_bfloat16* p) {
  const uint4 y = *reinterpret_cast<const uint4*>(p);
  const unsigned w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(float* x, const float* p) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 y = reinterpret_cast<const float4*>(p)[i];
    x[4 * i] = y.x, x[4 * i + 1] = y.y, x[4 * i + 2] = y.z, x[4 * i + 3] = y.w;
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const unsigned*>(&y);
  }
  *reinterpret_cast<uint4*>(p) = uint4{w[0], w[1], w[2], w[3]};
}
__device__ __forceinline__ void store8(float* p, const float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) reinterpret_cast<float4*>(p)[i] = float4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}

// Where pair p of a row stands in a table's row of `pairs`: what the lanes of
// a row read together, four pairs each, is contiguous.
__device__ __forceinline__ int place(int p, int pairs) { return ((p >> 2) & 1) * (pairs >> 1) + (p >> 3) * 4 + (p & 3); }

// A lane's eight pairs of one table.
__device__ __forceinline__ void pairs8(float* x, const float* row, int unit, int pairs) {
  const float4 a = *reinterpret_cast<const float4*>(row + unit * 4), b = *reinterpret_cast<const float4*>(row + (pairs >> 1) + unit * 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// Element indices of pair i's two parts in a lane's 16 values.
template <bool kInterleaved>
__device__ __forceinline__ constexpr int part_a(int i) { return kInterleaved ? 2 * i : i; }
template <bool kInterleaved>
__device__ __forceinline__ constexpr int part_b(int i) { return kInterleaved ? 2 * i + 1 : i + 8; }

template <bool kInterleaved>
__device__ __forceinline__ void turn_query(float* x, const float* c, const float* s) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float &a = x[part_a<kInterleaved>(i)], &b = x[part_b<kInterleaved>(i)];
    const float y = fmaf(a, c[i], -(b * s[i]));
    b = fmaf(a, s[i], b * c[i]);
    a = y;
  }
}
template <bool kInterleaved>
__device__ __forceinline__ void turn_key(float* x, const float* c, const float* cl, const float* s, const float* sl) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float &a = x[part_a<kInterleaved>(i)], &b = x[part_b<kInterleaved>(i)];
    const float y = odd_sum(a, c[i], cl[i], -b, s[i], sl[i]);
    b = odd_sum(a, s[i], sl[i], b, c[i], cl[i]);
    a = y;
  }
}

// One block of threads takes 16 nodes of one sequence (kStore: the 16 slots of
// a block of the cache), and some of its heads: it fills a table of their cosines and
// sines once, and turns the heads by it.  With kStore the blocks behind those
// of the queries take a key's or a value's head a warp, like append's.
template <typename T, int D, bool kStore>
__global__ void __launch_bounds__(kThreads, 2) rotary_kernel(const __grid_constant__ Call<T> p) {
  constexpr int U = D / 16, P = D / 2;
  __shared__ __align__(16) float table[kStore ? 4 : 2][16 * P];
  const State& s = p.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = (int)(blockIdx.x / p.chunks), j = (int)(blockIdx.x % p.chunks), part = blockIdx.y;
  const bool stores = kStore && part >= p.q_parts;
  int id = p.seqs[b];
  if (id >= s.max_seqs) {
    if (tid == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    id = -1;
  }
  const int len = id >= 0 ? s.lens[id] : 0, asked = id >= 0 ? live_count(p.counts, b, p.n) : 0;
  const int t0 = kStore ? (len / kBlock + j) * kBlock : len + j * kBlock;   // the chunk's first slot
  if (t0 >= len + (stores ? asked : p.n)) return;
  const int from = max(len - t0, 0), to = min(len + asked - t0, kBlock);    // its rows that turn
  const int units0 = (part - p.q_parts) * (kThreads / 32);                  // keys' heads, then values'
  const int pairs = p.t.dim >> 1;
  if (!stores || units0 < s.kv_heads) {
    for (int x = from * pairs + tid; x < to * pairs; x += kThreads) {
      const int r = x / pairs, i = x - r * pairs, node = t0 + r - len;
      const int depth = node > 0 ? (node - 1) % p.L + 1 : 0;
      float2 c, sn;
      turn_cos_sin(p.t.turn[i] * (uint64_t)(len + depth), c, sn);
      c = product(c, p.t.magnitude);
      sn = product(sn, p.t.magnitude);
      const int at = r * P + place(i, pairs);
      if constexpr (kStore) {
        if (stores) {
          c = quick_sum(c.x, c.y);
          sn = quick_sum(sn.x, sn.y);
          table[2][at] = c.y;
          table[3][at] = sn.y;
        }
      }
      table[0][at] = c.x;
      table[1][at] = sn.x;
    }
    __syncthreads();
  }

  if (!stores) {
    // ---- queries: rows that are not live become zeros
    const int h0 = part * p.q_each, heads = min(p.q_each, p.q_heads - h0);
    const int end = min(len + p.n - t0, kBlock), unit = tid % U;
    const Lane<U> at(p.t, unit);
    const T* src = p.q + b * p.qs.x + h0 * p.qs.z;
    T* dst = p.out + (((int64_t)b * p.n) * p.q_heads + h0) * D;
#pragma unroll 2
    for (int x = from * heads + tid / U; x < end * heads; x += kThreads / U) {
      const int r = x / heads, h = x - r * heads;
      const int64_t node = t0 + r - len;
      float v[16];
      if (r < to) {
        const T* y = src + node * p.qs.y + h * p.qs.z;
        load8(v, y + at.first * 8);
        load8(v + 8, y + at.second * 8);
        if (at.turns) {
          float c[8], sn[8];
          pairs8(c, table[0] + r * P, unit, pairs);
          pairs8(sn, table[1] + r * P, unit, pairs);
          if (p.t.interleaved) turn_query<true>(v, c, sn);
          else turn_query<false>(v, c, sn);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0.f;
      }
      T* o = dst + (node * p.q_heads + h) * D;
      store8(o + at.first * 8, v);
      store8(o + at.second * 8, v + 8);
    }
    return;
  }

  if constexpr (kStore) {
    // ---- a head of keys or of values a warp: quantised with the tokens in front
    const int u = units0 + warp, kv = u >= s.kv_heads, h = u - kv * s.kv_heads;
    if (u >= 2 * s.kv_heads) return;
    const int c = min(asked, s.reach[id] - len);
    if (c < asked && lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    if (c == 0 || t0 >= len + c) return;
    using Blk = Block<float, U>;
    Blk blk;
    const int row = lane / U, unit = lane % U;
    const Lane<U> at(p.t, unit);
    const longlong3 st = kv ? p.vs : p.ks;
    const T* src = (kv ? p.v : p.k) + b * st.x + h * st.z;
#pragma unroll
    for (int i = 0; i < Blk::kPasses; ++i) {
      const int t = t0 + i * Blk::kRows + row;
      float* v = blk.v[i].v;
      if (t >= len && t < len + c) {
        const T* y = src + (int64_t)(t - len) * st.y;
        load8(v, y + at.first * 8);
        load8(v + 8, y + at.second * 8);
      } else {
        blk.v[i].zero();
      }
    }
    const int page = s.table[(int64_t)id * s.max_pages + (t0 >> s.page_log)];
    if (s.ref[page] > 1) {
      if (lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
      return;
    }
    const int64_t tile = tile_of(s, p.layer, page, kv, h);
    const int r0 = t0 & (s.page_tokens - 1);
    uint8_t* base = s.pool + tile * (s.page_tokens * D) + r0 * D;
    float* scale_at = s.scales + tile * (s.page_tokens / kBlock) + r0 / kBlock;
    if (!kv && at.turns) {
#pragma unroll
      for (int i = 0; i < Blk::kPasses; ++i) {
        const int r = i * Blk::kRows + row;
        if (r >= from && t0 + r < len + c) {
          float cs[8], cl[8], sn[8], sl[8];
          pairs8(cs, table[0] + r * P, unit, pairs);
          pairs8(sn, table[1] + r * P, unit, pairs);
          pairs8(cl, table[2] + r * P, unit, pairs);
          pairs8(sl, table[3] + r * P, unit, pairs);
          if (p.t.interleaved) turn_key<true>(blk.v[i].v, cs, cl, sn, sl);
          else turn_key<false>(blk.v[i].v, cs, cl, sn, sl);
        }
      }
    }
    float was = 0.f;
    if (t0 < len) {
      was = *scale_at;
#pragma unroll
      for (int i = 0; i < Blk::kPasses; ++i) {
        const int r = i * Blk::kRows + row;
        if (r < from) {
          const uint2 lo = *reinterpret_cast<const uint2*>(base + swizzled(r * D + at.first * 8));
          const uint2 hi = *reinterpret_cast<const uint2*>(base + swizzled(r * D + at.second * 8));
          decode16(uint4{lo.x, lo.y, hi.x, hi.y}, was, blk.v[i].v);
        }
      }
    }
    float inv;
    bool odd;
    const float scale = blk.scale(&inv, &odd);
    if (odd && lane == 0) atomicOr(s.status, MDS_ST_NONFINITE);
    if (lane == 0) *scale_at = scale;
#pragma unroll
    for (int i = 0; i < Blk::kPasses; ++i) {
      const int r = i * Blk::kRows + row, t = t0 + r;
      if (t < len + c && (t >= len || scale != was)) {
        const uint4 y = encode16(blk.v[i], inv);
        *reinterpret_cast<uint2*>(base + swizzled(r * D + at.first * 8)) = uint2{y.x, y.y};
        *reinterpret_cast<uint2*>(base + swizzled(r * D + at.second * 8)) = uint2{y.z, y.w};
      }
    }
  }
}

template <typename T, int D>
cudaError_t launch(const State& s, const Rotate& a, cudaStream_t st) {
  Call<T> p{};
  p.s = s;
  for (int i = 0; i < a.rotary->dim / 2; ++i) p.t.turn[i] = a.rotary->turns[i];
  const float m = (float)a.rotary->magnitude;
  p.t.magnitude = float2{m, (float)(a.rotary->magnitude - (double)m)};
  p.t.dim = a.rotary->dim;
  p.t.interleaved = a.rotary->interleaved;
  p.seqs = a.seqs;
  p.counts = a.counts;
  p.k = static_cast<const T*>(a.k);
  p.v = static_cast<const T*>(a.v);
  p.q = static_cast<const T*>(a.q);
  p.out = static_cast<T*>(a.out);
  if (a.k) {
    p.ks = longlong3{a.ks[0], a.ks[1], a.ks[2]};
    p.vs = longlong3{a.vs[0], a.vs[1], a.vs[2]};
  }
  if (a.q) p.qs = longlong3{a.qs[0], a.qs[1], a.qs[2]};
  p.layer = a.layer;
  p.n = a.n;
  p.L = a.L > 0 ? a.L : 1;
  p.chunks = a.k ? (a.n + 2 * kBlock - 2) / kBlock : (a.n + kBlock - 1) / kBlock;
  p.q_heads = a.heads;
  // about four items a thread
  const int rows = a.n < kBlock ? a.n : kBlock, each = 4 * kThreads / (D / 16) / rows;
  p.q_each = a.heads < each ? a.heads : each;
  p.q_parts = a.q ? (a.heads + p.q_each - 1) / p.q_each : 0;
  const dim3 grid(a.B * p.chunks, p.q_parts + (a.k ? (2 * s.kv_heads + 7) / 8 : 0));
  if (a.k) rotary_kernel<T, D, true><<<grid, kThreads, 0, st>>>(p);
  else rotary_kernel<T, D, false><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t rotate(const State& s, const Rotate& a, cudaStream_t st) {
  if (s.dtype == MDS_F32) return s.head_dim == 64 ? launch<float, 64>(s, a, st) : launch<float, 128>(s, a, st);
  return s.head_dim == 64 ? launch<__nv_bfloat16, 64>(s, a, st) : launch<__nv_bfloat16, 128>(s, a, st);
}

}  // namespace cache
}  // namespace mds
