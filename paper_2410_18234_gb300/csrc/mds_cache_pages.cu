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

// Where slot t's rows are: page id, or -1 where the sequence holds none.
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
  for (int b = warp; b < B; b += kPlanThreads / 32) {
    const int q = sequence(s, seqs, b);
    int2 c = {0, 0};
    if (q >= 0) {
      const int len = s.lens[q], held = s.held[q], k = live_count(counts, b, n);
      const int first = len >> s.page_log, end = (len + k + P - 1) >> s.page_log;
      if (k > 0 && end > s.max_pages) {
        if (lane == 0) atomicOr(s.status, MDS_ST_NOPAGES);
        c.x = -1;
      } else if (k > 0) {
        const int32_t* row = s.table + (int64_t)q * s.max_pages;
        for (int p0 = first; p0 < end; p0 += 32) {
          const int p = p0 + lane;
          const bool in = p < end, absent = in && p >= held;
          const bool shared = in && !absent && s.ref[row[p]] > 1;
          c.x += __popc(__ballot_sync(kFull, absent || shared));
          c.y += __popc(__ballot_sync(kFull, shared));
        }
      }
    }
    if (lane == 0) need[b] = c;
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
      if (own.x > 0 && !fits) atomicOr(s.status, MDS_ST_NOPAGES);
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
  // hand them out; which pages are shared is still as it was counted
  for (int b = warp; b < B; b += kPlanThreads / 32) {
    const int2 off = need[b];
    if (off.x < 0) continue;
    const int q = seqs[b];
    const int len = s.lens[q], held = s.held[q], k = live_count(counts, b, n);
    const int first = len >> s.page_log, end = (len + k + P - 1) >> s.page_log;
    int32_t* row = s.table + (int64_t)q * s.max_pages;
    int at = off.x, cat = off.y;
    for (int p0 = first; p0 < end; p0 += 32) {
      const int p = p0 + lane;
      const bool in = p < end, absent = in && p >= held;
      const int old = in && !absent ? row[p] : -1;
      const bool shared = old >= 0 && s.ref[old] > 1;
      const unsigned get = __ballot_sync(kFull, absent || shared), cp = __ballot_sync(kFull, shared);
      const unsigned below = (1u << lane) - 1u;
      if (absent || shared) {
        const int r = at + __popc(get & below);
        row[p] = s.fresh[r];
        if (shared) {
          int32_t* c = s.copies + 3 * (int64_t)(cat + __popc(cp & below));
          c[0] = old;
          c[1] = s.fresh[r];
          c[2] = min(P, len + k - p * P);
        }
      }
      at += __popc(get);
      cat += __popc(cp);
    }
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
// values a lane, 32 / U rows at once, U / 2 times.
template <int U>
struct Block {
  static constexpr int kPasses = U / 2;
  static constexpr int kRows = 32 / U;
  float v[kPasses][16];
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

__device__ __forceinline__ uint4 encode16(const float* v, float inv) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b};\n\t}"
        : "=r"(w[i])
        : "f"(v[4 * i] * inv), "f"(v[4 * i + 1] * inv), "f"(v[4 * i + 2] * inv), "f"(v[4 * i + 3] * inv));
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

// The block's scale: the least e in [-117, 119] with max <= 448 * 2^e, from
// the maximum's exponent x and mantissa m: 448 = 1.75 * 2^8, so e = x - 8 if
// m <= 1.75, else x - 7.  Lane-uniform.  Returns 2^e and sets inv to 2^-e.
template <int U>
__device__ __forceinline__ float block_scale(const Block<U>& blk, float* inv) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < Block<U>::kPasses; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float x = fabsf(blk.v[i][j]);
      a = fmaxf(a, x <= 3.402823466e38f ? x : 0.f);
    }
  const unsigned bits = __reduce_max_sync(kFull, __float_as_uint(a));   // non-negative floats order as integers
  int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = bits == 0 ? 0 : min(max(e, -117), 119);
  *inv = __uint_as_float((unsigned)(127 - e) << 23);
  return __uint_as_float((unsigned)(127 + e) << 23);
}

// ------------------------------------------------------------------- append

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* v);
template <>
__device__ __forceinline__ void load16<float>(const float* p, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 x = __ldg(reinterpret_cast<const float4*>(p) + i);
    v[4 * i] = x.x;
    v[4 * i + 1] = x.y;
    v[4 * i + 2] = x.z;
    v[4 * i + 3] = x.w;
  }
}
template <>
__device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16* p, float* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i);
    const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
      v[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
}

// One warp per (sequence, block, key or value, head), heads next to one
// another: what the warps of a block of threads read is contiguous.  Bound by
// the bytes of the new tokens in and the blocks out.
template <typename T, int U>
__global__ void __launch_bounds__(256) append_kernel(const State s, int layer, const int32_t* seqs,
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
  const int len = s.lens[q], c = live_count(counts, b, n);
  const int t0 = (len / kBlock + j) * kBlock;
  if (c == 0 || t0 >= len + c) return;
  const int page = page_at(s, q, t0);
  if (page < 0 || s.ref[page] > 1) {
    if (lane == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    return;
  }
  using Blk = Block<U>;
  Blk blk;
  const int row = lane / U, unit = lane % U;
  const int64_t tile = tile_of(s, layer, page, kv, h);
  const int r0 = t0 & (s.page_tokens - 1);
  uint8_t* base = s.pool + tile * (s.page_tokens * s.head_dim) + r0 * s.head_dim;
  float* scale_at = s.scales + tile * (s.page_tokens / kBlock) + r0 / kBlock;
  const longlong3 st = kv ? vs : ks;
  const T* src = (kv ? v : k) + b * st.x + h * st.z + unit * 16;
  const float was = t0 < len ? *scale_at : 0.f;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < Blk::kPasses; ++i) {
    const int r = i * Blk::kRows + row, t = t0 + r;
    if (t < len) {
      decode16(*reinterpret_cast<const uint4*>(base + swizzled(r * s.head_dim + unit * 16)), was, blk.v[i]);
    } else if (t < len + c) {
      load16(src + (int64_t)(t - len) * st.y, blk.v[i]);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        odd |= !(fabsf(blk.v[i][x]) <= 3.402823466e38f);
        if (blk.v[i][x] != blk.v[i][x]) blk.v[i][x] = 0.f;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x) blk.v[i][x] = 0.f;
    }
  }
  if (odd) atomicOr(s.status, MDS_ST_NONFINITE);
  float inv;
  const float scale = block_scale(blk, &inv);
  if (lane == 0) *scale_at = scale;
#pragma unroll
  for (int i = 0; i < Blk::kPasses; ++i) {
    const int r = i * Blk::kRows + row, t = t0 + r;
    if (t < len + c && (t >= len || scale != was))
      *reinterpret_cast<uint4*>(base + swizzled(r * s.head_dim + unit * 16)) = encode16(blk.v[i], inv);
  }
}

// ------------------------------------------------------------------- commit

// One block row per sequence.  Tokens move towards the front (branch k's
// token i from slot len + 1 + k L + i to len + 1 + i), so a block of slots may
// be rewritten once its own sources have been read: those of the blocks
// behind it lie behind it.  One warp moves one tile's blocks in that order.
// The last of a sequence's blocks of threads to finish shortens the sequence.
template <int U>
__global__ void __launch_bounds__(256) commit_kernel(const State s, const int32_t* seqs, const int32_t* accept,
                                                     const int32_t* drafts, const int32_t* out_tokens, int K, int L) {
  __shared__ int branch_s, last_s;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int q = sequence(s, seqs, b);
  if (q < 0) return;
  const int len = s.lens[q], held = s.held[q];
  int a = min(max(accept[b], -1), L);
  if (tid == 0) branch_s = drafts && a > 0 ? K : 0;
  __syncthreads();
  if (drafts && a > 0) {
    const int32_t* out = out_tokens + (int64_t)b * (L + 1);
    for (int k = warp; k < K; k += 8) {
      const int32_t* d = drafts + ((int64_t)b * K + k) * L;
      bool same = true;
      for (int i = lane; i < a; i += 32) same = same && d[i] == out[i];
      if (__all_sync(kFull, same) && lane == 0) atomicMin(&branch_s, k);
    }
    __syncthreads();
  }
  int k = branch_s;
  if (k >= K) {
    if (tid == 0) atomicOr(s.status, MDS_ST_BADTOKEN);
    k = 0;
  }
  const int32_t* table = s.table + (int64_t)q * s.max_pages;
  const int64_t shift = a > 0 ? (int64_t)k * L : 0;
  bool bad = len + 1 + (int64_t)a + shift > (int64_t)held << s.page_log;
  if (!bad && shift)
    for (int p = (len + 1) >> s.page_log; p <= (len + a) >> s.page_log; ++p) bad = bad || s.ref[table[p]] > 1;
  if (bad) {
    if (tid == 0) atomicOr(s.status, MDS_ST_BADSEQ);
    a = -1;
  }
  if (!bad && shift) {
    using Blk = Block<U>;
    const int tiles = s.layers * 2 * s.kv_heads;
    const int row = lane / U, unit = lane % U;
    const int tile_bytes = s.page_tokens * s.head_dim, per = s.page_tokens / kBlock;
    for (int x = blockIdx.x * 8 + warp; x < tiles; x += gridDim.x * 8) {
      const int layer = x / (2 * s.kv_heads), kvh = x % (2 * s.kv_heads);
      for (int t0 = (len + 1) / kBlock * kBlock; t0 <= len + a; t0 += kBlock) {
        Blk blk;
#pragma unroll
        for (int i = 0; i < Blk::kPasses; ++i) {
          const int t = t0 + i * Blk::kRows + row;
          if (t <= len + a) {
            const int from = t <= len ? t : t + (int)shift, fr = from & (s.page_tokens - 1);
            const int64_t tile = tile_of(s, layer, table[from >> s.page_log], 0, kvh);
            const float sc = s.scales[tile * per + fr / kBlock];
            decode16(*reinterpret_cast<const uint4*>(s.pool + tile * tile_bytes + swizzled(fr * s.head_dim + unit * 16)),
                     sc, blk.v[i]);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) blk.v[i][e] = 0.f;
          }
        }
        float inv;
        const float scale = block_scale(blk, &inv);   // every lane's sources have been read
        const int r0 = t0 & (s.page_tokens - 1);
        const int64_t tile = tile_of(s, layer, table[t0 >> s.page_log], 0, kvh);
        if (lane == 0) s.scales[tile * per + r0 / kBlock] = scale;
#pragma unroll
        for (int i = 0; i < Blk::kPasses; ++i) {
          const int r = i * Blk::kRows + row;
          if (t0 + r <= len + a)
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
  }
}

__device__ __forceinline__ void store16(float* p, const float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float* v) {
  unsigned w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);   // exact: 4 significant bits
    w[i] = *reinterpret_cast<const unsigned*>(&x);
  }
  reinterpret_cast<uint4*>(p)[0] = uint4{w[0], w[1], w[2], w[3]};
  reinterpret_cast<uint4*>(p)[1] = uint4{w[4], w[5], w[6], w[7]};
}

// One thread turns 16 bytes of one token's key and of its value.
template <typename T>
__global__ void __launch_bounds__(256) read_kernel(const State s, int layer0, const int32_t* seqs,
                                                   const int32_t* start, const int32_t* counts, T* k, T* v, int n,
                                                   int B, int64_t units) {
  const int U = s.head_dim / 16, row = U * s.kv_heads;
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (u >= units) return;
  const int hu = (int)(u % row), h = hu / U, unit = hu % U;
  const int64_t token = u / row;
  const int i = (int)(token % n);
  const int64_t lb = token / n;
  const int b = (int)(lb % B), layer = layer0 + (int)(lb / B);
  const int q = sequence(s, seqs, b);
  float x[2][16] = {};
  if (q >= 0 && i < live_count(counts, b, n)) {
    const int64_t t = (int64_t)(start ? start[b] : 0) + i;
    if (t >= 0 && t < (int64_t)s.held[q] << s.page_log) {
      const int page = page_at(s, q, (int)t), r = (int)t & (s.page_tokens - 1);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const int64_t tile = tile_of(s, layer, page, kv, h);
        decode16(*reinterpret_cast<const uint4*>(s.pool + tile * (s.page_tokens * s.head_dim) +
                                                 swizzled(r * s.head_dim + unit * 16)),
                 s.scales[tile * (s.page_tokens / kBlock) + r / kBlock], x[kv]);
      }
    }
  }
  store16(k + u * 16, x[0]);
  store16(v + u * 16, x[1]);
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
  // without drafts nothing moves: one block a sequence
  const int tiles = s.layers * 2 * s.kv_heads, want = drafts ? (tiles + 7) / 8 : 1;
  const dim3 grid((unsigned)min(want, 64), (unsigned)B);
  if (s.head_dim == 128)
    commit_kernel<8><<<grid, 256, 0, st>>>(s, seqs, accept, drafts, out_tokens, K, L);
  else
    commit_kernel<4><<<grid, 256, 0, st>>>(s, seqs, accept, drafts, out_tokens, K, L);
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
  const int64_t units = (int64_t)(layer < 0 ? s.layers : 1) * B * n * s.kv_heads * (s.head_dim / 16);
  const unsigned grid = (unsigned)((units + 255) / 256);
  const int l0 = layer < 0 ? 0 : layer;
  if (s.dtype == MDS_F32)
    read_kernel<<<grid, 256, 0, st>>>(s, l0, seqs, start, counts, static_cast<float*>(k), static_cast<float*>(v), n, B,
                                      units);
  else
    read_kernel<<<grid, 256, 0, st>>>(s, l0, seqs, start, counts, static_cast<__nv_bfloat16*>(k),
                                      static_cast<__nv_bfloat16*>(v), n, B, units);
  return cudaGetLastError();
}

}  // namespace cache
}  // namespace mds
