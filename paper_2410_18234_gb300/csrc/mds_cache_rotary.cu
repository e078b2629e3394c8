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
// Rounding.  Queries are rotated in 32 bits and rounded to their type once.  A
// key is rounded to 8 bits behind the rotation, where an error of 2^-24 would
// turn one number in half a million into its neighbour, a sixteenth away.  So
// each is quantised as the two ends of its error's interval; where they differ
// (a lane in some thousands, and the ties of position 0), it is computed again
// with products and sum in two floats and angles to 2^-40, and the sum goes to
// one float by rounding to odd (of the two floats around it the one whose last
// bit is set), which a second rounding cannot tell from the sum itself.  What
// is stored is the quantiser's answer on the exact rotation.
//
// What binds it.  Queries: memory.  4 prompts of 4099 tokens, 32 heads of 128,
// bfloat16 (268 MB): 47 us, 5.7 TB/s, 84 % of a copy; in 32 bits 94.  Keys and
// values: the quantiser's instructions (half of the issue slots) and its
// registers.  256 trees of 33 nodes on 8 heads with 32 heads of queries (194
// MB, the begun blocks with them): 53 us, 3.7 TB/s; 4 prompts of 4099 tokens of
// the same heads (369 MB): 80 us, 4.6 TB/s, in 32 bits with 16 heads of queries
// and ragged lengths (283 MB) 74 us.  Every key in two floats would take 12 us
// more on the trees.
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
  int q_heads, q_each;         // heads that a block turns
  int kv_parts;                // blocks for the keys and values of a chunk
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

// The same in one float each, for what is rounded to its type once: an eighth
// of a turn either way as a float is off by 2^-24 of itself, a sum by about
// 1.5 * 2^-24 of its largest term.
__device__ __forceinline__ void turn_cos_sin(uint64_t f, float& c, float& s) {
  const unsigned quarter = (unsigned)((f + (1ull << 61)) >> 62) & 3u;
  const int64_t r = (int64_t)(f - ((uint64_t)quarter << 62));
  const float a = __ll2float_rn(r) * (float)(6.283185307179586476925286766559 / 18446744073709551616.0), z = a * a;
  const float sine = fmaf(a * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
  const float cosine = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  c = quarter & 1u ? sine : cosine;
  s = quarter & 1u ? cosine : sine;
  if (quarter == 1u || quarter == 2u) c = -c;
  if (quarter & 2u) s = -s;
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
// that a lane holds both parts of its eight pairs and the lanes' chunks lie
// next to one another: kI (interleaved) chunks u and u + U, pairs 4 u .. + 3
// and 4 (u + U) .. + 3; else chunks u and u + dim / 16, pairs 8 u .. + 7.  The
// pairs are taken in two quads: a quad's 8 numbers are two words of a block's
// bytes, and `turns` says of each quad whether it is turned.
template <int U, bool kI>
struct Lane {
  int unit, first, second;   // chunks
  bool turns[2];
  __device__ __forceinline__ Lane(const Turns& t, int u) : unit(u) {
    const int half = t.dim >> 4;
    if (kI) {
      first = u, second = u + U;
      turns[0] = u * 8 < t.dim, turns[1] = (u + U) * 8 < t.dim;
    } else {
      turns[0] = turns[1] = u < half;
      first = u < half ? u : 2 * u;
      second = u < half ? u + half : 2 * u + 1;
    }
  }
  __device__ __forceinline__ int pair(int i) const { return kI ? 4 * (unit + (i >> 2) * U) + (i & 3) : 8 * unit + i; }
};
// Where pair p of a row stands in a table's row: what the lanes of a row read
// together, a quad each, is contiguous.
template <bool kI>
__device__ __forceinline__ int place(int p, int pairs) {
  return kI ? p : ((p >> 2) & 1) * (pairs >> 1) + (p >> 3) * 4 + (p & 3);
}
template <int U, bool kI>
__device__ __forceinline__ float4 quad_of(const float* row, int unit, int q, int pairs) {
  return *reinterpret_cast<const float4*>(row + unit * 4 + (q ? (kI ? 4 * U : pairs >> 1) : 0));
}
// The words (of four numbers) of quad q: its two halves' places in a lane's 16.
template <bool kI>
__device__ __forceinline__ constexpr int word_of(int q, int half) { return kI ? 2 * q + half : q + 2 * half; }

// A lane's 16 numbers of a row as they are loaded.
template <typename T>
struct Raw {
  static constexpr int kWords = (int)sizeof(T) * 4;
  unsigned w[kWords];
  __device__ __forceinline__ void load(const T* first, const T* second) {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
      const uint4 y = reinterpret_cast<const uint4*>(i < kWords / 8 ? first : second)[i % (kWords / 8)];
      w[4 * i] = y.x, w[4 * i + 1] = y.y, w[4 * i + 2] = y.z, w[4 * i + 3] = y.w;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  // numbers of quad q
  template <bool kI>
  __device__ __forceinline__ void quad(int q, float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = at(word_of<kI>(q, i >> 2) * 4 + (i & 3));
  }
};

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

// The largest magnitude of three; no number where one is none.
__device__ __forceinline__ float largest3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Pair i of a quad's numbers.
template <bool kI>
__device__ __forceinline__ constexpr int part_a(int i) { return kI ? 2 * i : i; }
template <bool kI>
__device__ __forceinline__ constexpr int part_b(int i) { return kI ? 2 * i + 1 : i + 4; }

template <bool kI>
__device__ __forceinline__ void turn(float* x, const float4& cos4, const float4& sin4) {
  const float c[4] = {cos4.x, cos4.y, cos4.z, cos4.w}, s[4] = {sin4.x, sin4.y, sin4.z, sin4.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float &a = x[part_a<kI>(i)], &b = x[part_b<kI>(i)];
    const float y = fmaf(a, c[i], -(b * s[i]));
    b = fmaf(a, s[i], b * c[i]);
    a = y;
  }
}

__device__ __forceinline__ int depth_of(int node, int L) { return node <= L ? max(node, 0) : (node - 1) % L + 1; }

// ------------------------------------------------------------- exact blocks

// A head's rows of a block as the exact path takes them, from memory again.
template <typename T>
struct Rows {
  const T* src;             // row 0's numbers (of which rows [from, to) are there)
  int64_t stride;
  uint8_t* base;            // row 0's bytes
  const Turns* t;
  int from, to, position;   // position: of depth 0
  int node0, L;             // row 0's node
  bool key;
};

// The numbers of quad q of row r times 2^shift, turned to floats rounded to odd;
// 0 for what is no number.  Whether any is not finite.  A pair is turned with
// its larger number brought to [1, 2) by a power of two (the largest and the
// least floats to within 2^24 of that): no product passes the largest float
// where the rotation does not, and none leaves a rest below the least.
template <typename T, int D, bool kI>
__device__ bool exact_quad(const Rows<T>& w, const Lane<D / 16, kI>& at, int r, int q, int shift, float* x) {
  auto power = [](int e) { return __uint_as_float((unsigned)(127 + min(max(e, -126), 127)) << 23); };
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int word = word_of<kI>(q, half), d = (word < 2 ? at.first : at.second) * 8 + (word & 1) * 4;
    const T* from = w.src + r * w.stride + d;
    for (int i = 0; i < 4; ++i) x[half * 4 + i] = (float)from[i];
  }
  if (w.key && at.turns[q]) {
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      float &a = x[part_a<kI>(i)], &b = x[part_b<kI>(i)];
      float2 c, s;
      turn_cos_sin(w.t->turn[at.pair(4 * q + i)] * (uint64_t)(w.position + depth_of(w.node0 + r, w.L)), c, s);
      c = product(c, w.t->magnitude);
      s = product(s, w.t->magnitude);
      const int e = min(max((int)(__float_as_uint(fmaxf(fabsf(a), fabsf(b))) >> 23), 1), 253) - 127;
      // beyond the powers there are, a number is stored as 0 or the largest either way
      const float down = power(-e), up = power(e + shift);
      a *= down, b *= down;
      const float y = odd_sum(a, c.x, c.y, -b, s.x, s.y) * up;
      b = odd_sum(a, s.x, s.y, b, c.x, c.y) * up;
      a = y;
    }
  } else {
    for (int i = 0; i < 8; ++i) x[i] *= power(shift);
  }
  bool odd = false;
  for (int i = 0; i < 8; ++i) {
    odd = odd || !(fabsf(x[i]) <= FLT_MAX);
    x[i] = x[i] == x[i] ? x[i] : 0.f;
  }
  return odd;
}
// The bits of the largest finite magnitude of a lane's rows; the highest bit is
// set where one is not finite.
template <typename T, int D, bool kI>
__device__ __noinline__ unsigned exact_largest(const Rows<T>& w, int lane) {
  constexpr int U = D / 16;
  const Lane<U, kI> at(*w.t, lane % U);
  unsigned m = 0;
  bool odd = false;
#pragma unroll 1
  for (int r = lane / U; r < w.to; r += 32 / U)
#pragma unroll 1
    for (int q = 0; q < 2; ++q) {
      if (r < w.from) continue;
      float x[8];
      odd = exact_quad<T, D, kI>(w, at, r, q, 0, x) || odd;
      for (int i = 0; i < 8; ++i) {
        const unsigned a = __float_as_uint(x[i]) & 0x7fffffffu;
        m = max(m, a >= kInf ? 0u : a);
      }
    }
  return odd ? m | 0x80000000u : m;
}
// Store the quads of `mask` (bit 2 i + q of a lane's i-th row).
template <typename T, int D, bool kI>
__device__ __noinline__ void exact_store(const Rows<T>& w, int lane, unsigned mask, float inv) {
  constexpr int U = D / 16;
  const Lane<U, kI> at(*w.t, lane % U);
  const int shift = (int)(__float_as_uint(inv) >> 23) - 127;
#pragma unroll 1
  for (; mask; mask &= mask - 1) {
    const int bit = __ffs(mask) - 1, r = (bit >> 1) * (32 / U) + lane / U, q = bit & 1;
    if (r < w.from || r >= w.to) continue;
    float x[8];
    exact_quad<T, D, kI>(w, at, r, q, shift, x);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int word = word_of<kI>(q, half), d = (word < 2 ? at.first : at.second) * 8 + (word & 1) * 4;
      *reinterpret_cast<unsigned*>(w.base + swizzled(r * D + d)) =
          encode4(x[4 * half], x[4 * half + 1], x[4 * half + 2], x[4 * half + 3]);
    }
  }
}


// Cosines and sines of rows [from, to) of the chunk whose first row is node
// `node0`, by all the block's threads, a pair each.
template <int P, bool kI>
__device__ __forceinline__ void fill(float (*table)[16 * P], const Turns& t, int from, int to, int node0, int len, int L) {
  const int i = threadIdx.x % P, pairs = t.dim >> 1;
  if (i >= pairs) return;
  const uint64_t turn = t.turn[i];
  const int at = place<kI>(i, pairs);
  for (int r = from + threadIdx.x / P; r < to; r += kThreads / P) {
    float c, s;
    turn_cos_sin(turn * (uint64_t)(len + depth_of(node0 + r, L)), c, s);
    table[0][r * P + at] = c * t.magnitude.x, table[1][r * P + at] = s * t.magnitude.x;
  }
}

// One block of threads takes 16 nodes of one sequence and some of its heads
// (kStore: or the 16 slots of a block of the cache, a key's or a value's head a
// warp, like append's; those blocks come first, as they take longest).  It
// starts its loads, fills a table of the rows' cosines and sines while they
// are under way, and turns the heads by it.
// Blocks an SM: queries 2, 3, 4 take 49, 49, 47 us on the prompts above; 16-bit
// keys 2, 3 61 and 53 on the trees.
template <typename T, int D, bool kStore, bool kI>
__global__ void __launch_bounds__(kThreads, !kStore ? 4 : sizeof(T) * D <= 256 ? 3 : 2)
    rotary_kernel(const __grid_constant__ Call<T> p) {
  constexpr int U = D / 16, P = D / 2, kItems = sizeof(T) == 4 ? 1 : 2;
  __shared__ __align__(16) float table[2][16 * P];
  const State& s = p.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, pairs = p.t.dim >> 1;
  const int b = (int)(blockIdx.x / p.chunks), j = (int)(blockIdx.x % p.chunks);
  int id = p.seqs[b];
  if (id >= s.max_seqs) {
    if (tid == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    id = -1;
  }
  const int asked = id >= 0 ? live_count(p.counts, b, p.n) : 0;
  const Lane<U, kI> at(p.t, tid % U);

  if (!kStore || (int)blockIdx.y >= p.kv_parts) {
    // ---- queries, a row a thread: rows that are not live become zeros
    const int node0 = j * kBlock, end = min(p.n - node0, kBlock), to = min(asked - node0, end);
    if (end <= 0) return;
    const int h0 = ((int)blockIdx.y - p.kv_parts) * p.q_each, heads = min(p.q_each, p.q_heads - h0);
    const int log = 32 - __clz(end - 1);   // of the rows, rounded up to a power of two
    const int r = (tid / U) & ((1 << log) - 1), first = tid / U >> log, step = kThreads / U >> log;
    const bool live = r < to;
    const T* src = p.q + b * p.qs.x + (node0 + r) * p.qs.y + h0 * p.qs.z;
    T* dst = p.out + (((int64_t)b * p.n + node0 + r) * p.q_heads + h0) * D;
    Raw<T> raw[kItems];
    auto load = [&](int g) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int h = g + i * step;
        if (live && h < heads) raw[i].load(src + h * p.qs.z + at.first * 8, src + h * p.qs.z + at.second * 8);
        else raw[i].zero();
      }
    };
    load(first);
    if (to > 0) fill<P, kI>(table, p.t, 0, to, node0, s.lens[id], p.L);
    __syncthreads();
    if (r >= end) return;
    float4 c[2], sn[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      c[q] = float4{1.f, 1.f, 1.f, 1.f}, sn[q] = float4{0.f, 0.f, 0.f, 0.f};
      if (at.turns[q] && live) {
        c[q] = quad_of<U, kI>(table[0] + r * P, at.unit, q, pairs);
        sn[q] = quad_of<U, kI>(table[1] + r * P, at.unit, q, pairs);
      }
    }
    for (int g = first; g < heads; g += kItems * step) {
      if (g != first) load(g);
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int h = g + i * step;
        if (h >= heads) break;
        float v[2][8];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          raw[i].template quad<kI>(q, v[q]);
          if (at.turns[q]) turn<kI>(v[q], c[q], sn[q]);
        }
        float x[16];
#pragma unroll
        for (int y = 0; y < 16; ++y) x[word_of<kI>(y >> 3, (y >> 2) & 1) * 4 + (y & 3)] = v[y >> 3][y & 7];
        store8(dst + h * D + at.first * 8, x);
        store8(dst + h * D + at.second * 8, x + 8);
      }
    }
    return;
  }

  if constexpr (kStore) {
    // ---- a head of keys or of values a warp: quantised with the tokens in front
    if (asked == 0) return;
    const int len = s.lens[id], c = min(asked, s.reach[id] - len);
    const int t0 = (len / kBlock + j) * kBlock, from = max(len - t0, 0), to = min(len + c - t0, kBlock);   // new rows
    if (t0 >= len + asked) return;
    if (c < asked && tid == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    if (c == 0 || t0 >= len + c) return;
    const int units0 = blockIdx.y * (kThreads / 32), u = units0 + warp;   // keys' heads, then values'
    const bool mine = u < 2 * s.kv_heads;
    const int kv = u >= s.kv_heads, h = u - kv * s.kv_heads;
    constexpr int kPasses = U / 2, kRows = 32 / U;
    const int row = lane / U;
    const int page = s.table[(int64_t)id * s.max_pages + (t0 >> s.page_log)];
    const longlong3 st = kv ? p.vs : p.ks;
    const T* src = (kv ? p.v : p.k) + b * st.x + h * st.z + (int64_t)(t0 - len) * st.y;
    Raw<T> raw[kPasses];
    if (mine) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int r = i * kRows + row;
        if (r >= from && r < to) raw[i].load(src + r * st.y + at.first * 8, src + r * st.y + at.second * 8);
        else raw[i].zero();
      }
    }
    const bool shared = s.ref[page] > 1;
    if (units0 < s.kv_heads) {
      fill<P, kI>(table, p.t, from, to, t0 - len, len, p.L);
      __syncthreads();
    }
    if (!mine) return;
    if (shared) {
      if (lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
      return;
    }
    const int64_t tile = tile_of(s, p.layer, page, kv, h);
    const int r0 = t0 & (s.page_tokens - 1);
    uint8_t* base = s.pool + tile * (s.page_tokens * D) + r0 * D;
    float* scale_at = s.scales + tile * (s.page_tokens / kBlock) + r0 / kBlock;
    float was = 0.f;
    if (t0 < len) {
      was = *scale_at;
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int r = i * kRows + row;
        if (r < from) {   // bytes in the place of new numbers
          const uint2 lo = *reinterpret_cast<const uint2*>(base + swizzled(r * D + at.first * 8));
          const uint2 hi = *reinterpret_cast<const uint2*>(base + swizzled(r * D + at.second * 8));
          raw[i].w[0] = lo.x, raw[i].w[1] = lo.y, raw[i].w[2] = hi.x, raw[i].w[3] = hi.y;
        }
      }
    }
    const Rows<T> rows{src, st.y, base, &p.t, from, to, len, t0 - len, p.L, !kv};
    // Quad q of the lane's i-th row, from what was loaded: bytes of tokens in
    // front, new numbers, turned or not.
    auto numbers = [&](int i, int q, float* v, float* mag) {
      const int r = i * kRows + row;
      if (r < from) {
        decode4(raw[i].w[word_of<kI>(q, 0)], was, v);
        decode4(raw[i].w[word_of<kI>(q, 1)], was, v + 4);
        return false;
      }
      raw[i].template quad<kI>(q, v);
      if (kv || !at.turns[q] || r >= to) return false;
#pragma unroll
      for (int x = 0; x < 4; ++x) mag[x] = fabsf(v[part_a<kI>(x)]) + fabsf(v[part_b<kI>(x)]);
      turn<kI>(v, quad_of<U, kI>(table[0] + r * P, at.unit, q, pairs), quad_of<U, kI>(table[1] + r * P, at.unit, q, pairs));
      return true;
    };
    // The block's maximum and scale.  A turned number is off by less than
    // 2^-21 of its pair's |a| + |b| (times the magnitude), of which the larger
    // of the pair's two is at least half, so the maximum is off by less than
    // 2^-20 of itself, 16 steps of a float: where those decide the scale, or it
    // is not finite, the numbers are computed exactly.
    auto step_of = [](unsigned bits) { return (bits + 0x1fffffu) >> 23; };   // goes up behind 1.75 * 2^x
    float top[2] = {0.f, 0.f};   // of numbers that are as they are, and of turned ones
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      if (i * kRows >= to) break;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float v[8], mag[4];
        const bool turned = numbers(i, q, v, mag);
        float m = largest3(v[0], v[1], v[2]);
        m = largest3(m, v[3], v[4]);
        m = largest3(m, v[5], v[6]);
        if (turned) top[1] = largest3(top[1], m, v[7]);
        else top[0] = largest3(top[0], m, v[7]);
      }
    }
    unsigned known = __reduce_max_sync(kFull, __float_as_uint(top[0]) & 0x7fffffffu);
    const unsigned most = __reduce_max_sync(kFull, __float_as_uint(top[1]) & 0x7fffffffu);
    bool exact = false;
    if (max(known, most) >= kInf || step_of(max(known, most - min(most, 16u))) != step_of(max(known, most + 16u))) {
      exact = true;
      const unsigned m = exact_largest<T, D, kI>(rows, lane);
      if (__any_sync(kFull, m >> 31) && lane == 0) atomicOr(s.status, MDS_ST_NONFINITE);
      unsigned held = 0;   // tokens in front are finite
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        if (i * kRows + row >= from) break;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float v[8], mag[4];
          numbers(i, q, v, mag);
#pragma unroll
          for (int x = 0; x < 8; ++x) held = max(held, __float_as_uint(v[x]) & 0x7fffffffu);
        }
      }
      known = __reduce_max_sync(kFull, max(held, m & 0x7fffffffu));
    }
    float inv;
    const float scale = block_scale(exact ? known : max(known, most), &inv);
    if (lane == 0) *scale_at = scale;
    // Beside numbers that do not turn a small magnitude puts the error's factor
    // below the normal floats, where it would be rounded itself, or times a sum
    // |a| + |b| that is not finite no number at all: then all are computed exactly.
    const float off = inv * (p.t.magnitude.x * 0x1p-21f);   // in this order not infinite
    unsigned unsure = exact || off < FLT_MIN ? (1u << (2 * kPasses)) - 1u : 0u;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      if (i * kRows >= to) break;
      const int r = i * kRows + row;
      if (r < to && (r >= from || scale != was)) {
        unsigned w[4];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float v[8], mag[4];
          unsigned &lo = w[word_of<kI>(q, 0)], &hi = w[word_of<kI>(q, 1)];
          if (numbers(i, q, v, mag)) {
            // either end of each number's error: the same but where a rounding border lies between
            float x[8], y[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) {
              const float e = mag[kI ? z >> 1 : z & 3] * off;
              x[z] = fmaf(v[z], inv, -e);
              y[z] = fmaf(v[z], inv, e);
            }
            lo = encode4(x[0], x[1], x[2], x[3]);
            hi = encode4(x[4], x[5], x[6], x[7]);
            if (lo != encode4(y[0], y[1], y[2], y[3]) || hi != encode4(y[4], y[5], y[6], y[7])) unsure |= 1u << (2 * i + q);
          } else {
            lo = encode4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            hi = encode4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
          }
        }
        *reinterpret_cast<uint2*>(base + swizzled(r * D + at.first * 8)) = uint2{w[0], w[1]};
        *reinterpret_cast<uint2*>(base + swizzled(r * D + at.second * 8)) = uint2{w[2], w[3]};
      }
    }
    unsure = __reduce_or_sync(kFull, unsure);
    if (unsure) exact_store<T, D, kI>(rows, lane, unsure, inv);
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
  // heads for which a table is filled: eight times a thread's 16 numbers (2, 4
  // and 8 times: 53, 47, 47 us on the prompts above, and 105, 92, 86 on
  // the trees, an append and a read, before keys had three blocks an SM)
  const int rows = a.n < kBlock ? a.n : kBlock, each = 8 * kThreads / (D / 16) / rows;
  p.q_each = a.heads < each ? a.heads : each;
  p.kv_parts = a.k ? (2 * s.kv_heads + 7) / 8 : 0;
  const dim3 grid(a.B * p.chunks, p.kv_parts + (a.q ? (a.heads + p.q_each - 1) / p.q_each : 0));
  if (a.k && p.t.interleaved) rotary_kernel<T, D, true, true><<<grid, kThreads, 0, st>>>(p);
  else if (a.k) rotary_kernel<T, D, true, false><<<grid, kThreads, 0, st>>>(p);
  else if (p.t.interleaved) rotary_kernel<T, D, false, true><<<grid, kThreads, 0, st>>>(p);
  else rotary_kernel<T, D, false, false><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t rotate(const State& s, const Rotate& a, cudaStream_t st) {
  if (s.dtype == MDS_F32) return s.head_dim == 64 ? launch<float, 64>(s, a, st) : launch<float, 128>(s, a, st);
  return s.head_dim == 64 ? launch<__nv_bfloat16, 64>(s, a, st) : launch<__nv_bfloat16, 128>(s, a, st);
}

}  // namespace cache
}  // namespace mds
