// Pages of the key/value cache: reserve (allocation, copy on write), append
// (quantisation), commit (compaction of the accepted branch), fork, truncate,
// free and read.  Every kernel here moves bytes; none does arithmetic that
// would bound it.
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

// Where slot t's rows are: page id, or -1 where the sequence holds none.  (read:
// the other calls go by what is reserved.)
__device__ __forceinline__ int page_at(const State& s, int q, int t) {
  const int p = t >> s.page_log;
  return p < s.held[q] ? s.table[(int64_t)q * s.max_pages + p] : -1;
}

// Give back the pages of sequence q from index `keep` on (all the block's threads).
__device__ void release(const State& s, int q, int keep, int held) {
  int32_t* row = s.table + (int64_t)q * s.max_pages;
  int freed = 0;
  for (int p = keep + threadIdx.x; p < held; p += blockDim.x) {
    const int page = row[p];
    row[p] = -1;
    if (page >= 0 && atomicSub(s.ref + page, 1) == 1) {
      atomicOr(s.freemap + (page >> 5), 1u << (page & 31));
      ++freed;
    }
  }
  if (freed) atomicAdd(s.free_count, freed);
}

// ------------------------------------------------------------------ reserve

constexpr int kPlanThreads = 1024;

// Inclusive scan over the block of two counts packed in one word each.
__device__ int2 block_scan(int2 x, int2* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int d = 1; d < 32; d *= 2) {
    const int a = __shfl_up_sync(kFull, x.x, d), b = __shfl_up_sync(kFull, x.y, d);
    if (lane >= d) x.x += a, x.y += b;
  }
  __syncthreads();   // the sums of the scan before have been read
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int2 w = warp_sums[lane];
    for (int d = 1; d < 32; d *= 2) {
      const int a = __shfl_up_sync(kFull, w.x, d), b = __shfl_up_sync(kFull, w.y, d);
      if (lane >= d) w.x += a, w.y += b;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  if (warp) x.x += warp_sums[warp - 1].x, x.y += warp_sums[warp - 1].y;
  return x;
}

// A reserve that gave sequence q nothing: of the slots reserved before, those
// in shared pages, where the sequence cannot store, are not reserved any more.
__device__ void got_none(const State& s, int q, int len, int held) {
  const int32_t* row = s.table + (int64_t)q * s.max_pages;
  int p = len >> s.page_log;
  while (p < held && s.ref[row[p]] <= 1) ++p;
  s.reach[q] = min(s.reach[q], max(len, p << s.page_log));
}

// One block plans the whole call: which page indices of which sequence need a
// page (absent, or shared and about to be written behind), and which page
// each gets.  The order is that of the list and of the indices, and pages are
// taken lowest first, so the outcome depends on the state alone.  One block
// is enough: a call looks at a few indices a sequence and at one bit a page
// (131072 pages in one sweep of the block).
__global__ void __launch_bounds__(kPlanThreads) reserve_plan_kernel(const State s, const int32_t* seqs,
                                                                    const int32_t* counts, int n, int B) {
  __shared__ int2 need[MDS_CACHE_MAX_BATCH];   // pages, and copies among them; then their exclusive sums
  __shared__ int2 warp_sums[32];
  __shared__ int total, copied, freed;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int P = s.page_tokens;
  if (tid == 0) total = copied = freed = 0;
  for (int b = tid; b < B; b += kPlanThreads) {
    const int q = sequence(s, seqs, b);
    int2 c = {0, 0};
    if (q >= 0) {
      const int len = s.lens[q], held = s.held[q], k = live_count(counts, b, n);
      const int first = len >> s.page_log, end = (len + k + P - 1) >> s.page_log;
      if (k > 0 && end > s.max_pages) {
        atomicOr(s.status, MDS_ST_NOPAGES);
        c.x = -1;
        got_none(s, q, len, held);
      } else if (k > 0) {
        const int32_t* row = s.table + (int64_t)q * s.max_pages;
        for (int p = first; p < min(end, held); ++p) c.y += s.ref[row[p]] > 1;
        c.x = c.y + max(end - max(first, held), 0);
        if (c.x == 0) s.reach[q] = max(s.reach[q], len + k);
      }
    }
    need[b] = c;
  }
  __syncthreads();
  // exclusive sums; a sequence beyond the free pages gets none
  const int avail = *s.free_count;
  int2 before = {0, 0};
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const int2 own = b < B ? need[b] : int2{0, 0};
    const int mine = max(own.x, 0);
    const int2 inc = block_scan(int2{mine, own.y}, warp_sums);
    const int off = before.x + inc.x - mine, coff = before.y + inc.y - own.y;
    if (b < B) {
      const bool fits = own.x > 0 && off + mine <= avail;
      if (own.x > 0 && !fits) {
        atomicOr(s.status, MDS_ST_NOPAGES);
        got_none(s, seqs[b], s.lens[seqs[b]], s.held[seqs[b]]);
      }
      need[b] = int2{own.x == 0 ? 0 : fits ? off : -1, coff};
      if (own.x == 0) need[b].x = -2;   // nothing to hand out
      if (fits) {
        atomicMax(&total, off + mine);
        atomicMax(&copied, coff + own.y);
      }
    }
    before.x += warp_sums[31].x;
    before.y += warp_sums[31].y;
  }
  __syncthreads();
  // the lowest `total` free pages
  const int words = (s.pages + 31) >> 5;
  int found = 0;
  for (int w0 = 0; w0 < words && found < total; w0 += kPlanThreads * 4) {
    const int w = w0 + tid * 4;
    uint4 m = w < words ? *reinterpret_cast<const uint4*>(s.freemap + w) : uint4{0, 0, 0, 0};
    unsigned bits[4] = {m.x, m.y, m.z, m.w};
    const int mine = __popc(m.x) + __popc(m.y) + __popc(m.z) + __popc(m.w);
    const int2 inc = block_scan(int2{mine, 0}, warp_sums);
    int rank = found + inc.x - mine;
    found += warp_sums[31].x;
    if (mine && rank < total) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        while (bits[i] && rank < total) {
          const int page = (w + i) * 32 + __ffs(bits[i]) - 1;
          bits[i] &= bits[i] - 1;
          s.fresh[rank++] = page;
          s.ref[page] = 1;
        }
      }
      *reinterpret_cast<uint4*>(s.freemap + w) = uint4{bits[0], bits[1], bits[2], bits[3]};
    }
  }
  __syncthreads();
  // hand them out; which pages are shared is still as it was counted.  Pages
  // held, a thread a sequence: there are few from slot len on; then the new
  // ones, which may be thousands of a sequence, a warp a sequence.
  for (int b = tid; b < B; b += kPlanThreads) {
    int2 off = need[b];
    if (off.x < 0) continue;
    const int q = seqs[b];
    const int len = s.lens[q], held = s.held[q], k = live_count(counts, b, n);
    const int end = (len + k + P - 1) >> s.page_log;
    int32_t* row = s.table + (int64_t)q * s.max_pages;
    for (int p = len >> s.page_log; p < min(end, held); ++p) {
      const int old = row[p];
      if (s.ref[old] <= 1) continue;
      const int fresh = s.fresh[off.x++];
      row[p] = fresh;
      int32_t* c = s.copies + 3 * (int64_t)off.y++;
      c[0] = old;
      c[1] = fresh;
      c[2] = min(P, len + k - p * P);
    }
    // behind a copy's tokens nothing is this sequence's own
    s.reach[q] = off.y > need[b].y ? len + k : max(s.reach[q], len + k);
    need[b].x = off.x;
  }
  __syncthreads();
  for (int b = warp; b < B; b += kPlanThreads / 32) {
    const int at = need[b].x;
    if (at < 0) continue;
    const int q = seqs[b];
    const int len = s.lens[q], held = s.held[q], k = live_count(counts, b, n);
    const int from = max(len >> s.page_log, held), end = (len + k + P - 1) >> s.page_log;
    int32_t* row = s.table + (int64_t)q * s.max_pages;
    for (int p = from + lane; p < end; p += 32) row[p] = s.fresh[at + p - from];
    __syncwarp();
    if (lane == 0 && end > held) s.held[q] = end;
  }
  __syncthreads();
  for (int r = tid; r < copied; r += kPlanThreads) {
    const int old = s.copies[3 * (int64_t)r];
    if (atomicSub(s.ref + old, 1) == 1) {
      atomicOr(s.freemap + (old >> 5), 1u << (old & 31));
      atomicAdd(&freed, 1);
    }
  }
  __syncthreads();
  if (tid == 0) {
    *s.free_count = avail - total + freed;
    *s.n_copies = copied;
  }
}

// Copies of shared pages: one warp moves one tile's tokens, 16 bytes a lane.
__global__ void __launch_bounds__(256) copy_kernel(const State s) {
  const int lane = threadIdx.x & 31;
  const int tiles = s.layers * 2 * s.kv_heads;
  const int64_t units = (int64_t)*s.n_copies * tiles;
  const int tile_bytes = s.page_tokens * s.head_dim, per = s.page_tokens / kBlock;
  const int64_t warps = (int64_t)gridDim.x * 8;
  for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += warps) {
    const int32_t* c = s.copies + 3 * (u / tiles);
    const int rest = (int)(u % tiles), layer = rest / (2 * s.kv_heads), kvh = rest % (2 * s.kv_heads);
    const int blocks = (c[2] + kBlock - 1) / kBlock;
    const int64_t from = tile_of(s, layer, c[0], 0, kvh), to = tile_of(s, layer, c[1], 0, kvh);
    const uint4* src = reinterpret_cast<const uint4*>(s.pool + from * tile_bytes);
    uint4* dst = reinterpret_cast<uint4*>(s.pool + to * tile_bytes);
    const int units16 = blocks * kBlock * s.head_dim / 16;   // a multiple of 64
    float sc = 0.f;
    if (lane < blocks) sc = s.scales[from * per + lane];
    for (int i = lane; i < units16; i += 32 * 8) {
      uint4 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i + j * 32 < units16) x[j] = src[i + j * 32];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i + j * 32 < units16) dst[i + j * 32] = x[j];
    }
    if (lane < blocks) s.scales[to * per + lane] = sc;
  }
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

template <typename T, int U>
struct Block {
  static constexpr int kPasses = U / 2;
  static constexpr int kRows = 32 / U;
  Lane16<T> v[kPasses];

  // The scale: the least e in [-117, 119] with max <= 448 * 2^e, from the
  // maximum's exponent x and mantissa m: 448 = 1.75 * 2^8, so e = x - 8 if
  // m <= 1.75, else x - 7.  Lane-uniform.  Returns 2^e and sets inv to 2^-e.
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
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = bits == 0 ? 0 : min(max(e, -117), 119);
    *inv = __uint_as_float((unsigned)(127 - e) << 23);
    return __uint_as_float((unsigned)(127 + e) << 23);
  }
};

__device__ __forceinline__ void decode16(const uint4& x, float scale, float* v) {
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w[i]));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[4 * i] = a.x * scale;
    v[4 * i + 1] = a.y * scale;
    v[4 * i + 2] = b.x * scale;
    v[4 * i + 3] = b.y * scale;
  }
}

template <typename T>
__device__ __forceinline__ uint4 encode16(const Lane16<T>& v, float inv) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b};\n\t}"
        : "=r"(w[i])
        : "f"(v.at(4 * i) * inv), "f"(v.at(4 * i + 1) * inv), "f"(v.at(4 * i + 2) * inv), "f"(v.at(4 * i + 3) * inv));
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

// ------------------------------------------------------------------- append

// One warp per (sequence, block, key or value, head), heads next to one
// another: what the warps of a block of threads read is contiguous.  Bound by
// the latency of the lookups (sequence, length, page) in front of the new
// tokens' bytes, and by those.
template <typename T, int U>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) append_kernel(const State s, int layer, const int32_t* seqs,
                                                     const int32_t* counts, const T* k, longlong3 ks, const T* v,
                                                     longlong3 vs, int n, int nb, int64_t units) {
  const int lane = threadIdx.x & 31;
  const int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (u >= units) return;
  const int per = 2 * s.kv_heads;
  const int kvh = (int)(u % per), kv = kvh / s.kv_heads, h = kvh % s.kv_heads;
  const int64_t bj = u / per;
  const int b = (int)(bj / nb), j = (int)(bj % nb);
  const int q = sequence(s, seqs, b);
  if (q < 0) return;
  const int len = s.lens[q], reach = s.reach[q], asked = live_count(counts, b, n), c = min(asked, reach - len);
  const int t0 = (len / kBlock + j) * kBlock;
  if (asked == 0 || t0 >= len + asked) return;
  if (c < asked && lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
  if (c == 0 || t0 >= len + c) return;
  using Blk = Block<T, U>;
  Blk blk;
  const int row = lane / U, unit = lane % U;
  const longlong3 st = kv ? vs : ks;
  const T* src = (kv ? v : k) + b * st.x + h * st.z + unit * 16;
#pragma unroll
  for (int i = 0; i < Blk::kPasses; ++i) {
    const int t = t0 + i * Blk::kRows + row;
    if (t >= len && t < len + c) blk.v[i].load(src + (int64_t)(t - len) * st.y);
    else blk.v[i].zero();
  }
  const int page = s.table[(int64_t)q * s.max_pages + (t0 >> s.page_log)];
  if (s.ref[page] > 1) {
    if (lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    return;
  }
  const int64_t tile = tile_of(s, layer, page, kv, h);
  const int r0 = t0 & (s.page_tokens - 1);
  uint8_t* base = s.pool + tile * (s.page_tokens * s.head_dim) + r0 * s.head_dim;
  float* scale_at = s.scales + tile * (s.page_tokens / kBlock) + r0 / kBlock;
  float was = 0.f;
  if (t0 < len) {
    was = *scale_at;
#pragma unroll
    for (int i = 0; i < Blk::kPasses; ++i) {
      const int r = i * Blk::kRows + row;
      if (t0 + r < len) {
        float x[16];
        decode16(*reinterpret_cast<const uint4*>(base + swizzled(r * s.head_dim + unit * 16)), was, x);
        blk.v[i].values(x);
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
    if (t < len + c && (t >= len || scale != was))
      *reinterpret_cast<uint4*>(base + swizzled(r * s.head_dim + unit * 16)) = encode16(blk.v[i], inv);
  }
}

// ------------------------------------------------------------------- commit

// What a call keeps of sequence q (all the block's threads): the tokens behind
// the root, -1 for nothing, and how many slots they move towards the front.
__device__ int2 judge(const State& s, int q, int b, const int32_t* accept, const int32_t* drafts,
                      const int32_t* out_tokens, int K, int L) {
  __shared__ int branch_s;
  const int tid = threadIdx.x, lane = tid & 31;
  const int a = min(max(accept[b], -1), L);
  int k = 0;
  if (drafts && a > 0) {
    if (tid == 0) branch_s = K;
    __syncthreads();
    const int32_t* out = out_tokens + (int64_t)b * (L + 1);
    for (int i = tid >> 5; i < K; i += blockDim.x >> 5) {
      const int32_t* d = drafts + ((int64_t)b * K + i) * L;
      bool same = true;
      for (int x = lane; x < a; x += 32) same = same && d[x] == out[x];
      if (__all_sync(kFull, same) && lane == 0) atomicMin(&branch_s, i);
    }
    __syncthreads();
    k = branch_s;
    if (k >= K) {
      if (tid == 0) atomicOr(s.status, MDS_ST_BADTOKEN);
      k = 0;
    }
  }
  const int len = s.lens[q];
  const int64_t shift = a > 0 ? (int64_t)k * L : 0;
  bool bad = len + 1 + (int64_t)a + shift > s.reach[q];
  if (!bad && shift) {
    const int32_t* table = s.table + (int64_t)q * s.max_pages;
    for (int p = (len + 1) >> s.page_log; p <= (len + a) >> s.page_log; ++p) bad = bad || s.ref[table[p]] > 1;
  }
  if (bad && tid == 0) atomicOr(s.status, MDS_ST_BADSEQ);
  return bad ? int2{-1, 0} : int2{a, (int)shift};
}

// A kernel of its own where tokens may move: whether a page is shared is
// judged before any of the call's sequences gives one back.
__global__ void __launch_bounds__(256) judge_kernel(const State s, const int32_t* seqs, const int32_t* accept,
                                                    const int32_t* drafts, const int32_t* out_tokens, int K, int L) {
  const int b = blockIdx.x, q = sequence(s, seqs, b);
  if (q < 0) return;
  const int2 keeps = judge(s, q, b, accept, drafts, out_tokens, K, L);
  if (threadIdx.x == 0) reinterpret_cast<int2*>(s.kept)[b] = keeps;
}

// One block row per sequence.  Tokens move towards the front (branch k's
// token i from slot len + 1 + k L + i to len + 1 + i), so a block of slots may
// be rewritten once its own sources have been read: those of the blocks
// behind it lie behind it.  One warp moves one tile's blocks in that order.
// The last of a sequence's blocks of threads to finish shortens the sequence.
// Without drafts (`judged` false) nothing moves and one block judges for itself.
template <int U>
__global__ void __launch_bounds__(256, 3) commit_kernel(const State s, const int32_t* seqs, const int32_t* accept,
                                                     bool judged, int L) {
  __shared__ int last_s;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int q = seqs[b];
  if (judged ? q < 0 || q >= s.max_seqs : sequence(s, seqs, b) < 0) return;
  const int len = s.lens[q], held = s.held[q];
  const int2 keeps = judged ? reinterpret_cast<const int2*>(s.kept)[b]
                            : judge(s, q, b, accept, nullptr, nullptr, 1, L);
  const int a = keeps.x, shift = keeps.y;
  const int32_t* table = s.table + (int64_t)q * s.max_pages;
  if (shift) {
    using Blk = Block<__nv_bfloat16, U>;
    const int tiles = s.layers * 2 * s.kv_heads;
    const int row = lane / U, unit = lane % U;
    const int tile_bytes = s.page_tokens * s.head_dim, per = s.page_tokens / kBlock;
    for (int x = blockIdx.x * 8 + warp; x < tiles; x += gridDim.x * 8) {
      const int layer = x / (2 * s.kv_heads), kvh = x % (2 * s.kv_heads);
      for (int t0 = (len + 1) / kBlock * kBlock; t0 <= len + a; t0 += kBlock) {
        Blk blk;
        uint4 bytes[Blk::kPasses];
        float sc[Blk::kPasses];
#pragma unroll
        for (int i = 0; i < Blk::kPasses; ++i) {
          const int t = t0 + i * Blk::kRows + row;
          bytes[i] = uint4{0, 0, 0, 0};
          sc[i] = 0.f;
          if (t <= len + a) {
            const int from = t <= len ? t : t + shift, fr = from & (s.page_tokens - 1);
            const int64_t tile = tile_of(s, layer, table[from >> s.page_log], 0, kvh);
            sc[i] = s.scales[tile * per + fr / kBlock];
            bytes[i] = *reinterpret_cast<const uint4*>(s.pool + tile * tile_bytes + swizzled(fr * s.head_dim + unit * 16));
          }
        }
#pragma unroll
        for (int i = 0; i < Blk::kPasses; ++i) {
          float v[16];
          decode16(bytes[i], sc[i], v);
          blk.v[i].values(v);
        }
        float inv;
        bool odd;
        const float scale = blk.scale(&inv, &odd);   // every lane's sources have been read
        const int r0 = t0 & (s.page_tokens - 1);
        const int64_t tile = tile_of(s, layer, table[t0 >> s.page_log], 0, kvh);
        if (lane == 0) s.scales[tile * per + r0 / kBlock] = scale;
#pragma unroll
        for (int i = 0; i < Blk::kPasses; ++i) {
          const int r = i * Blk::kRows + row;
          if (t0 + r <= len + a && (t0 + r > len || scale != sc[i]))
            *reinterpret_cast<uint4*>(s.pool + tile * tile_bytes + swizzled((r0 + r) * s.head_dim + unit * 16)) =
                encode16(blk.v[i], inv);
        }
        __syncwarp();   // the stored block before the next block's sources
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    last_s = atomicAdd(s.arrive + q, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last_s) return;
  const int now = len + 1 + a, keep = (now + s.page_tokens - 1) >> s.page_log;
  release(s, q, keep, held);
  if (tid == 0) {
    s.arrive[q] = 0;
    s.lens[q] = now;
    s.held[q] = min(keep, held);
    s.reach[q] = min(s.reach[q], keep << s.page_log);
  }
}

// ------------------------------------------------- fork, truncate, free, read

__global__ void __launch_bounds__(128) fork_kernel(const State s, const int32_t* src, const int32_t* dst) {
  const int from = sequence(s, src, blockIdx.x), to = sequence(s, dst, blockIdx.x);
  if (from < 0 || to < 0) return;
  if (s.held[to] != 0 || s.lens[to] != 0 || from == to) {
    if (threadIdx.x == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    return;
  }
  __syncthreads();   // every thread has seen the empty sequence
  const int held = s.held[from];
  for (int p = threadIdx.x; p < held; p += blockDim.x) {
    const int page = s.table[(int64_t)from * s.max_pages + p];
    s.table[(int64_t)to * s.max_pages + p] = page;
    atomicAdd(s.ref + page, 1);
  }
  if (threadIdx.x == 0) {
    s.lens[to] = s.lens[from];
    s.held[to] = held;
    s.reach[to] = s.reach[from];
  }
}

__global__ void __launch_bounds__(128) truncate_kernel(const State s, const int32_t* seqs, const int32_t* lens) {
  const int q = sequence(s, seqs, blockIdx.x);
  if (q < 0) return;
  const int held = s.held[q], now = lens ? min(max(lens[blockIdx.x], 0), s.lens[q]) : 0;
  __syncthreads();   // every thread has read the old length
  const int keep = (now + s.page_tokens - 1) >> s.page_log;
  release(s, q, keep, held);
  if (threadIdx.x == 0) {
    s.lens[q] = now;
    s.held[q] = min(keep, held);
    s.reach[q] = now;
  }
}

// The values of sizeof(uint4) / sizeof(T) bytes, as 16 bytes.
__device__ __forceinline__ void widened(const uint8_t* at, float scale, uint4& y, float) {
  const unsigned x = *reinterpret_cast<const unsigned*>(at);
  float v[16];
  decode16(uint4{x, 0, 0, 0}, scale, v);
  y = uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}
__device__ __forceinline__ void widened(const uint8_t* at, float scale, uint4& y, __nv_bfloat16) {
  const uint2 x = *reinterpret_cast<const uint2*>(at);
  float v[16];
  decode16(uint4{x.x, x.y, 0, 0}, scale, v);
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 z = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);   // exact: 4 significant bits
    w[i] = *reinterpret_cast<const unsigned*>(&z);
  }
  y = uint4{w[0], w[1], w[2], w[3]};
}

// One block of threads turns 16 tokens of one sequence and layer; the lookups
// are done once a token.  A thread writes 16 bytes of a key and of a value at
// a time, so that a warp's stores are whole lines: the written bytes bound it.
template <typename T>
__global__ void __launch_bounds__(256) read_kernel(const State s, int layer0, const int32_t* seqs,
                                                   const int32_t* start, const int32_t* counts, T* k, T* v, int n) {
  __shared__ int page_s[16], row_s[16];
  constexpr int kEach = 16 / sizeof(T);
  const int U = s.head_dim / kEach, row = U * s.kv_heads, tid = threadIdx.x;
  const int b = blockIdx.y, layer = layer0 + blockIdx.z, i0 = blockIdx.x * 16, here = min(16, n - i0);
  if (tid < 16) {
    const int q = sequence(s, seqs, b), i = i0 + tid;
    int page = -1, r = 0;
    if (q >= 0 && i < live_count(counts, b, n)) {
      const int64_t t = (int64_t)(start ? start[b] : 0) + i;
      if (t >= 0 && t < (int64_t)s.held[q] << s.page_log) {
        page = page_at(s, q, (int)t);
        r = (int)t & (s.page_tokens - 1);
      }
    }
    page_s[tid] = page;
    row_s[tid] = r;
  }
  __syncthreads();
  const int64_t out = (((int64_t)blockIdx.z * gridDim.y + b) * n + i0) * row;   // units of 16 bytes
  const int per = s.page_tokens / kBlock;
  const int64_t kv_step = s.kv_heads;   // a head's value is that many tiles behind its key
#pragma unroll 4
  for (int x = tid; x < here * row; x += 256) {
    const int i = x / row, hu = x - i * row, h = hu / U, unit = hu - h * U, page = page_s[i], r = row_s[i];
    uint4 ky{0, 0, 0, 0}, vy{0, 0, 0, 0};
    if (page >= 0) {
      const int64_t tile = tile_of(s, layer, page, 0, h), tile_bytes = s.page_tokens * s.head_dim;
      const uint8_t* at = s.pool + tile * tile_bytes + swizzled(r * s.head_dim + unit * kEach);
      widened(at, s.scales[tile * per + r / kBlock], ky, T());
      widened(at + kv_step * tile_bytes, s.scales[(tile + kv_step) * per + r / kBlock], vy, T());
    }
    reinterpret_cast<uint4*>(k)[out + x] = ky;
    reinterpret_cast<uint4*>(v)[out + x] = vy;
  }
}

__global__ void __launch_bounds__(256) clear_kernel(const State s) {
  const int w = blockIdx.x * 256 + threadIdx.x;
  if (w < (s.pages + 31) / 32) s.freemap[w] = s.pages - w * 32 >= 32 ? kFull : (1u << (s.pages & 31)) - 1u;
  if (w == 0) *s.free_count = s.pages;
}

}  // namespace

cudaError_t clear(const State& s, cudaStream_t st) {
  clear_kernel<<<(s.pages / 32 + 256) / 256, 256, 0, st>>>(s);
  return cudaGetLastError();
}

cudaError_t reserve(const State& s, const int32_t* seqs, const int32_t* counts, int n, int B, cudaStream_t st) {
  reserve_plan_kernel<<<1, kPlanThreads, 0, st>>>(s, seqs, counts, n, B);
  copy_kernel<<<152 * 8, 256, 0, st>>>(s);
  return cudaGetLastError();
}

cudaError_t append(const State& s, int layer, const int32_t* seqs, const int32_t* counts, const void* k,
                   const int64_t* ks, const void* v, const int64_t* vs, int n, int B, cudaStream_t st) {
  const int nb = (n + 2 * kBlock - 2) / kBlock;   // blocks that n tokens touch at most
  const int64_t units = (int64_t)B * nb * 2 * s.kv_heads;
  const longlong3 a{ks[0], ks[1], ks[2]}, c{vs[0], vs[1], vs[2]};
  const unsigned grid = (unsigned)((units + 7) / 8);
  auto go = [&](auto kernel, auto* kp, auto* vp) {
    kernel<<<grid, 256, 0, st>>>(s, layer, seqs, counts, kp, a, vp, c, n, nb, units);
  };
  if (s.dtype == MDS_F32) {
    const float *kp = static_cast<const float*>(k), *vp = static_cast<const float*>(v);
    if (s.head_dim == 128) go(append_kernel<float, 8>, kp, vp);
    else go(append_kernel<float, 4>, kp, vp);
  } else {
    const auto *kp = static_cast<const __nv_bfloat16*>(k), *vp = static_cast<const __nv_bfloat16*>(v);
    if (s.head_dim == 128) go(append_kernel<__nv_bfloat16, 8>, kp, vp);
    else go(append_kernel<__nv_bfloat16, 4>, kp, vp);
  }
  return cudaGetLastError();
}

cudaError_t commit(const State& s, const int32_t* seqs, const int32_t* accept, const int32_t* drafts,
                   const int32_t* out_tokens, int K, int L, int B, cudaStream_t st) {
  // without drafts nothing moves: one block of threads a sequence; else one
  // for every 16 tiles, two a warp: a block's lookups cost more than a tile
  const int tiles = s.layers * 2 * s.kv_heads, want = drafts ? (tiles + 15) / 16 : 1;
  const dim3 grid((unsigned)min(want, 64), (unsigned)B);
  if (drafts) judge_kernel<<<B, 256, 0, st>>>(s, seqs, accept, drafts, out_tokens, K, L);
  if (s.head_dim == 128)
    commit_kernel<8><<<grid, 256, 0, st>>>(s, seqs, accept, drafts != nullptr, L);
  else
    commit_kernel<4><<<grid, 256, 0, st>>>(s, seqs, accept, drafts != nullptr, L);
  return cudaGetLastError();
}

cudaError_t fork(const State& s, const int32_t* src, const int32_t* dst, int B, cudaStream_t st) {
  fork_kernel<<<B, 128, 0, st>>>(s, src, dst);
  return cudaGetLastError();
}

cudaError_t truncate(const State& s, const int32_t* seqs, const int32_t* lens, int B, cudaStream_t st) {
  truncate_kernel<<<B, 128, 0, st>>>(s, seqs, lens);
  return cudaGetLastError();
}

cudaError_t read(const State& s, int layer, const int32_t* seqs, const int32_t* start, const int32_t* counts, void* k,
                 void* v, int n, int B, cudaStream_t st) {
  const dim3 grid((unsigned)((n + 15) / 16), (unsigned)B, (unsigned)(layer < 0 ? s.layers : 1));
  const int l0 = layer < 0 ? 0 : layer;
  if (s.dtype == MDS_F32)
    read_kernel<<<grid, 256, 0, st>>>(s, l0, seqs, start, counts, static_cast<float*>(k), static_cast<float*>(v), n);
  else
    read_kernel<<<grid, 256, 0, st>>>(s, l0, seqs, start, counts, static_cast<__nv_bfloat16*>(k),
                                      static_cast<__nv_bfloat16*>(v), n);
  return cudaGetLastError();
}

}  // namespace cache
}  // namespace mds
