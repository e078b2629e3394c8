// What the attention kernels over the paged cache share: the parameters, the
// line of key tiles that the blocks of a grid divide among themselves, bounded
// waits, and the join of pieces.
//
// Rows.  The g query heads that share a key/value head and the nodes of a
// tree read the same cache: row r = node * g + head of the group.  Work is cut
// into (sequence, key/value head, tile of rows) groups of key tiles of 128
// slots; all groups' tiles lie on one line that the blocks of the grid (one
// per SM) share evenly, so ragged lengths and few sequences load every SM.  A
// group cut between blocks is joined by the last of them to finish, which
// adds the pieces in their order: results do not depend on timing.
//
// Parts.  A call is one launch (kAll), or four where sequences share a prefix
// (more in several turns, mds_cache_shared.cu).  The first finds what is
// shared.  kPrefix takes every group of sequences as one of `members` times as
// many nodes over the prefix's tiles, and leaves each row's reference,
// normaliser and sums in `prior`, or in pieces that the third launch joins (a
// few groups may be cut into many pieces, which one block each would be long
// over).  kRest takes the sequences over the tiles behind it, and joins what it
// finds there like one more piece.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <climits>

#include "mds_cache_internal.h"
#include "mds_device.cuh"

namespace mds {
namespace cache {
namespace {

using dev::bulk_copy;
using dev::ex2;
using dev::mbar_arrive;
using dev::mbar_expect_tx;
using dev::mbar_init;
using dev::mbar_init_fence;
using dev::smem_u32;

constexpr unsigned kFull = 0xffffffffu;
constexpr int kTile = 128;                 // slots of a key tile
constexpr float kNone = -FLT_MAX;          // reference of a row that has seen nothing: below every score
constexpr float kSlack = 32.f;             // the reference moves when a weight passes 2^32
constexpr unsigned kWaitTries = 1u << 18;
constexpr int kRestExtra = 3;              // what a group costs beside its blocks, in blocks (mds_cache_rest.cu)

enum Part { kAll, kPrefix, kRest };

struct Params {
  State s;
  Attend a;                // kPrefix: a.B groups of a.n nodes of all members together
  int span;                // slots that one copy brings: a page, or a tile's part of it
  int g, rows, row_tiles, stages;
  int rows_per;            // rows of a row tile
  // 1, in a form that the compiler does not know: it joins a packed product
  // and a packed sum behind it into one fused operation, rounding modes or
  // not, but not a product and a fused operation by this number.
  float one = 1.f;
  int members = 1, nodes = 0;      // sequences of a group, and nodes of one
  int part = 0;                    // members that one turn takes, where several share a group (mds_cache_shared.cu)
  float* prior = nullptr;          // [B][n][heads][D + 4], like pieces
  int64_t worth = 0, each = 0;     // tokens that must be saved, in all and a live sequence, for the prefix to be attended to by itself
  const int64_t* saved = nullptr;  // what the call saves, where that is not what its plan sees
};

// The launches of attention over a shared prefix follow one another without a
// pause: each may start while the one before ends, and waits for it before it
// reads anything.  (Every block waits, so that a launch is over only when all
// before it are.  Letting the next one start earlier than that costs more than
// it gives: 45 us for 37 with 8 sequences over 4100 tokens.)
__device__ __forceinline__ void after_launch_before() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
inline cudaError_t launch_behind(void (*kernel)(Params), int grid, int threads, int smem, cudaStream_t st, const Params& p) {
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(grid);
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = st;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, p);
}

// A sequence's part of the call.
template <int kPart>
struct Seq {
  int q, len, live, end;   // id, committed, live nodes, slots reserved (a slot behind them is not read)
};
template <>
struct Seq<kRest> {
  int q, len, live, end;
  int from;                // the prefix's tokens
};
// Bytes of B of them, in whole units of 16.
template <int kPart>
__host__ __device__ constexpr int seq_bytes(int B) {
  return (B * (int)sizeof(Seq<kPart>) + 15) / 16 * 16;
}

// A group's key tiles: `sink` tiles from slot 0, then those from `first` on.
struct Group {
  int lo, sinks, hi;       // slots seen by a row of the tile: [0, sinks) and [lo, hi)
  int sink_tiles, first, tiles;
};

template <int kPart>
__device__ __forceinline__ Group group_of(const Params& p, const Seq<kPart>& q, int rt) {
  Group r;
  const int i0 = rt * p.rows_per / p.g, i1 = min((rt * p.rows_per + p.rows_per - 1) / p.g, q.live - 1);
  r.tiles = 0;
  r.hi = r.lo = r.sinks = r.sink_tiles = r.first = 0;
  if (i0 >= q.live) return r;
  r.hi = min(q.len + i1 + 1, q.end);
  if (p.a.window > 0) {
    // a chain's node is at its own position; a branch's first node at depth 1
    const int64_t pos = (int64_t)q.len + (p.a.n - 1 <= p.a.L ? i0 : min(i0, 1));
    r.lo = (int)min(max(pos - p.a.window + 1, (int64_t)0), (int64_t)q.len);
    r.sinks = min(p.a.sinks, r.lo);
  }
  if constexpr (kPart == kRest) r.lo = q.from;   // a multiple of kTile
  r.first = r.lo / kTile;
  r.sink_tiles = min((r.sinks + kTile - 1) / kTile, r.first);
  r.tiles = r.sink_tiles + max((r.hi + kTile - 1) / kTile - r.first, 0);
  return r;
}

__device__ __forceinline__ int tile_slot(const Group& r, int i) {
  return (i < r.sink_tiles ? i : r.first + i - r.sink_tiles) * kTile;
}

// Whether any row of the tile sees a slot of the block of 16 from t on; or of
// `span` slots from t on.  The pool holds finite numbers everywhere, so a copy
// may bring slots that no row sees.
__device__ __forceinline__ bool block_seen(const Group& r, int t, int span = kBlock) {
  return t < r.hi && (t + span > r.lo || t < r.sinks);
}

// A wait on a barrier gives up after kWaitTries tries, and at once after
// another wait of the block has.  A try suspends the thread for up to 20 us by
// itself; tries that return at once still make milliseconds, far beyond the
// longest wait of a block for itself.  Kept short: the waits are a good part
// of the kernels' code, which has to stay in the instruction cache.  A block
// that gave up says so at its end (report).
__device__ __forceinline__ bool try_wait(uint64_t* bar, unsigned parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(smem_u32(bar)), "r"(parity), "r"(20000u)
      : "memory");
  return done != 0;
}
// False: it gave up.
__device__ __forceinline__ bool wait(uint64_t* bar, unsigned parity, int* abort) {
  unsigned i = 0;
#pragma unroll 1
  while (!try_wait(bar, parity)) {
    if (++i > kWaitTries || *reinterpret_cast<volatile int*>(abort)) {
      *reinterpret_cast<volatile int*>(abort) = 1;
      return false;
    }
  }
  return true;
}
// Whether the block gave up, the same answer for a warp's lanes: a loader then
// starts no more copies, as their places may still be written or read.
__device__ __forceinline__ bool gave_up(const int* abort) {
  return __any_sync(kFull, *reinterpret_cast<const volatile int*>(abort));
}
// Behind a thread's last wait: says so if the block gave up, and leaves copies
// and products in flight time to end before the block, and what it holds, goes.
__device__ __forceinline__ void report(int* abort, uint32_t* status) {
  if (!*reinterpret_cast<volatile int*>(abort)) return;
  atomicOr(status, MDS_ST_TIMEOUT);
  for (int i = 0; i < 1000; ++i) __nanosleep(10000);
}

// Two e4m3 numbers as two halves.
__device__ __forceinline__ void to_f16(unsigned x, unsigned& lo, unsigned& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(x));
}
// The even and the odd bytes of a word as two bfloat16 each, times a power of
// two: e4m3's exponent and mantissa laid over bfloat16's are the number times
// 2^-120, and `factor` (two bfloat16) is 2^120 times the power.  A block's
// values are exact in bfloat16: their scale is at least 2^-117.
__device__ __forceinline__ void to_bf16(unsigned x, unsigned factor, unsigned& even, unsigned& odd) {
  const unsigned e = ((x << 4) & 0x07f007f0u) | ((x << 8) & 0x80008000u);
  const unsigned o = ((x >> 4) & 0x07f007f0u) | (x & 0x80008000u);
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(even) : "r"(e), "r"(factor));
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(odd) : "r"(o), "r"(factor));
}
// The factor of a block's scale.  2^7 is the largest that fits; `rest` is what
// is left of a larger scale (values beyond 57344), as two bfloat16, else 1.
__device__ __forceinline__ unsigned value_factor(float scale, unsigned& rest) {
  const unsigned bits = __float_as_uint(scale) >> 16, most = 0x4300u;   // 2^7
  rest = bits > most ? (bits - most + 0x3f80u) * 0x10001u : 0x3f803f80u;
  return ((bits > most ? most : bits) + (120u << 7)) * 0x10001u;
}
__device__ __forceinline__ void times_rest(unsigned& x, unsigned rest) {
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(rest));
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// What a block of threads does next on the line of key tiles.
struct Cursor {
  int b, h, rt, off;
};

// The group and tile of unit u (whole warp).
template <int kPart>
__device__ Cursor locate(const Params& p, const long long* prefix, const Seq<kPart>* seqs, long long u) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = p.a.B - 1;
  while (lo < hi) {   // the last b with prefix[b] <= u
    const int mid = (lo + hi + 1) / 2;
    if (prefix[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  Cursor c;
  c.b = lo;
  const long long per = (prefix[lo + 1] - prefix[lo]) / p.s.kv_heads;
  const long long rem = u - prefix[lo];
  c.h = (int)(rem / per);
  long long in = rem % per;
  const Seq<kPart> q = seqs[lo];
  for (int r0 = 0;; r0 += 32) {
    const int rt = r0 + lane;
    int t = rt < p.row_tiles ? group_of(p, q, rt).tiles : 0;
    const int own = t;
    for (int d = 1; d < 32; d *= 2) {
      const int x = __shfl_up_sync(kFull, t, d);
      if (lane >= d) t += x;
    }
    const unsigned past = __ballot_sync(kFull, t > in);
    if (past || r0 + 32 >= p.row_tiles) {
      const int at = past ? __ffs(past) - 1 : 31;
      c.rt = r0 + at;
      c.off = (int)in - (__shfl_sync(kFull, t, at) - __shfl_sync(kFull, own, at));
      return c;
    }
    in -= __shfl_sync(kFull, t, 31);
  }
}

// The next group that has tiles.  False past the end.
template <int kPart>
__device__ bool advance(const Params& p, const Seq<kPart>* seqs, Cursor& c, Group& grp) {
  c.off = 0;
  for (;;) {
    if (++c.rt >= p.row_tiles || c.rt * p.rows_per / p.g >= seqs[c.b].live) {
      c.rt = 0;
      if (++c.h >= p.s.kv_heads) {
        c.h = 0;
        do {
          if (++c.b >= p.a.B) return false;
        } while (seqs[c.b].live <= 0);
      }
    }
    grp = group_of(p, seqs[c.b], c.rt);
    if (grp.tiles > 0) return true;
  }
}

template <typename T>
__device__ __forceinline__ void store4(T* out, float4 x);
template <>
__device__ __forceinline__ void store4<float>(float* out, float4 x) {
  *reinterpret_cast<float4*>(out) = x;
}
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* out, float4 x) {
  *reinterpret_cast<uint2*>(out) = uint2{pack_bf16(x.x, x.y), pack_bf16(x.z, x.w)};
}

// Sequence b of the list, whose live nodes end with its reserved slots.
// True where the call asks for what is not there.
__device__ __forceinline__ bool find(const State& s, const int32_t* seqs, const int32_t* counts, int b, int n, int* q,
                                     int* len, int* live, int* end) {
  const int id = seqs[b];
  *q = -1;
  *len = *live = *end = 0;
  if (id < 0 || id >= s.max_seqs) return id >= 0;
  *q = id;
  *len = s.lens[id];
  *live = counts ? min(max(counts[b], 0), n) : n;
  *end = s.reach[id];
  const bool bad = *len + *live > *end && *live > 0;
  if (bad) *live = min(*live, max(*end - *len, 0));   // rows without a slot of their own are zeros
  return bad;
}

// Adds every thread's x to a sum in shared memory, a warp's at a time (64-bit
// additions there are loops: one a thread took some 10 us of a call with 256
// sequences).
__device__ __forceinline__ void add_up(long long* to, long long x) {
#pragma unroll
  for (int d = 16; d; d /= 2) x += __shfl_xor_sync(kFull, x, d);
  if (x && (threadIdx.x & 31) == 0) atomicAdd(reinterpret_cast<unsigned long long*>(to), (unsigned long long)x);
}

// What decides whether prefixes are attended to by themselves, in one number:
// tokens saved (at most 2^30), and live sequences above.
constexpr int kLiveShift = 40;
__device__ __forceinline__ bool worth_it(const Params& p, long long x) {
  const long long saved = x & ((1ll << kLiveShift) - 1), live = x >> kLiveShift;
  return saved >= p.worth && saved >= p.each * live;
}

// Where what the call saves is known before (several turns): whether a launch
// has nothing to do, those of the turns or the one for the whole call.
template <int kPart>
__device__ __forceinline__ bool idle(const Params& p) {
  return p.saved && worth_it(p, *p.saved) == (kPart == kAll);
}

// The plan, by all of the block's threads: seqs and the exclusive sums of
// their tiles (kFine: of blocks of 16 slots, and kRestExtra), and zeros in the rows of nodes
// that are not live.
template <typename T, int kPart, bool kFine = false>
__device__ void plan(const Params& p, long long* prefix, Seq<kPart>* seqs, int head_dim) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  // what a group's live sequences share is the least of what each shares with the first
  if constexpr (kPart == kPrefix) {
    // q: the place of the first live sequence; live: nodes up to the last one; end: live ones
    for (int g = tid; g < p.a.B; g += blockDim.x) seqs[g] = Seq<kPart>{INT_MAX, INT_MAX, 0, 0};
    if (tid == 0) prefix[0] = 0;
    __syncthreads();
    for (int b = tid; b < p.a.B * p.members; b += blockDim.x) {
      const int2 x = __ldg(p.s.share + b);
      Seq<kPart>& q = seqs[b / p.members];
      if (x.y > 0) {
        atomicMin(&q.len, x.x);
        atomicMin(&q.q, b);
        atomicMax(&q.live, (b % p.members + 1) * p.nodes);
        atomicAdd(&q.end, 1);
      }
    }
    __syncthreads();
    long long saved = 0;
    for (int g = tid; g < p.a.B; g += blockDim.x)
      if (seqs[g].end > 0) saved += (seqs[g].end - 1ll) * seqs[g].len + ((long long)seqs[g].end << kLiveShift);
    add_up(prefix, saved);
    __syncthreads();
    const bool worth = p.saved || worth_it(p, prefix[0]);
    for (int g = tid; g < p.a.B; g += blockDim.x) {
      const Seq<kPart> q = seqs[g];
      seqs[g] = worth && q.live > 0 && q.len > 0 ? Seq<kPart>{p.a.seqs[q.q], q.len, q.live, q.len} : Seq<kPart>{-1, 0, 0, 0};
    }
  } else {
    if constexpr (kPart == kRest) {
      for (int b = tid; b < p.a.B; b += blockDim.x) seqs[b].from = INT_MAX;
      if (tid == 0) prefix[0] = 0;
      __syncthreads();
    }
    for (int b = tid; b < p.a.B; b += blockDim.x) {
      Seq<kPart>& q = seqs[b];
      int2 x{0, 0};
      if constexpr (kPart == kRest) x = __ldg(p.s.share + b);
      int id, len, live, end;
      if (find(p.s, p.a.seqs, p.a.counts, b, p.a.n, &id, &len, &live, &end)) atomicOr(p.s.status, MDS_ST_BADSEQ);
      q.q = id, q.len = len, q.live = live, q.end = end;
      if constexpr (kPart == kRest)
        if (x.y > 0) atomicMin(&seqs[b / p.members * p.members].from, x.x);   // its first place has the group's
    }
    if constexpr (kPart == kRest) {
      __syncthreads();
      // saved: for each live sequence what is shared, but once for a group
      long long saved = 0;
      for (int b = tid; b < p.a.B; b += blockDim.x) {
        const int from = seqs[b / p.members * p.members].from;
        if (b % p.members) seqs[b].from = from;
        const int times = (seqs[b].live > 0) - (b % p.members == 0);
        if (from != INT_MAX) saved += (long long)times * from;
        if (seqs[b].live > 0) saved += 1ll << kLiveShift;
      }
      add_up(prefix, saved);
      __syncthreads();
      if (!p.saved && !worth_it(p, prefix[0]))
        for (int b = tid; b < p.a.B; b += blockDim.x) seqs[b].from = 0;
    }
  }
  __syncthreads();
  auto tiles_of = [&](const Seq<kPart>& q, int rt) {
    const Group grp = group_of(p, q, rt);
    return !kFine ? grp.tiles : grp.tiles ? (grp.hi - grp.lo + kBlock - 1) / kBlock + kRestExtra : 0;
  };
  // A thread a sequence where it has few row tiles, else a warp.
  if (p.row_tiles <= 4) {
    for (int b = tid; b < p.a.B; b += blockDim.x) {
      const Seq<kPart> q = seqs[b];
      long long t = 0;
      for (int rt = 0; rt < p.row_tiles; ++rt) t += tiles_of(q, rt);
      prefix[b + 1] = t * p.s.kv_heads;
    }
  } else {
    for (int b = warp; b < p.a.B; b += warps) {
      const Seq<kPart> q = seqs[b];
      long long t = 0;
      const int tiles = min(p.row_tiles, (q.live * p.g + p.rows_per - 1) / p.rows_per);
      for (int rt = lane; rt < tiles; rt += 32) t += tiles_of(q, rt);
      for (int d = 16; d; d /= 2) t += __shfl_xor_sync(kFull, t, d);
      if (lane == 0) prefix[b + 1] = t * p.s.kv_heads;
    }
  }
  __syncthreads();
  // sums within 32 sequences by a warp, then a thread adds the 32s in front of its own
  for (int b0 = warp * 32; b0 < p.a.B; b0 += warps * 32) {
    const int b = b0 + lane;
    long long x = b < p.a.B ? prefix[b + 1] : 0;
    for (int d = 1; d < 32; d *= 2) {
      const long long y = __shfl_up_sync(kFull, x, d);
      if (lane >= d) x += y;
    }
    if (b < p.a.B) prefix[b + 1] = x;
  }
  if (tid == 0) prefix[0] = 0;
  __syncthreads();
  if (p.a.B > 32) {
    constexpr int kMost = MDS_CACHE_MAX_BATCH / 256;   // sequences of a thread
    long long in_front[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int b = tid + i * (int)blockDim.x;
      in_front[i] = 0;
      if (b < p.a.B)
        for (int c = 32; c <= b; c += 32) in_front[i] += prefix[c];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int b = tid + i * (int)blockDim.x;
      if (b < p.a.B) prefix[b + 1] += in_front[i];
    }
  }
  T* out = static_cast<T*>(p.a.out);
  for (int b = blockIdx.x; b < (kPart == kPrefix ? 0 : p.a.B); b += gridDim.x) {
    const int64_t row = (int64_t)p.a.heads * head_dim;
    const int64_t from = ((int64_t)b * p.a.n + seqs[b].live) * row, to = (int64_t)(b + 1) * p.a.n * row;
    for (int64_t i = from + tid * 4; i < to; i += blockDim.x * 4) store4(out + i, float4{0.f, 0.f, 0.f, 0.f});
  }
  __syncthreads();
}

// ------------------------------------------------------- rows and pieces
//
// A piece's partial sums: per row its reference, its normaliser, two unused
// places, and D sums.  A block has two: of the group that it continues, and of
// the one that it begins and another block ends.

template <int D>
constexpr int kPieceRow = D + 4;

template <int D>
__device__ __forceinline__ float* piece_of(const Params& p, int block, bool begins) {
  return p.s.part + ((int64_t)block * 2 + (begins ? 1 : 0)) * p.rows_per * kPieceRow<D>;
}

// Where node `node` of sequence b of the list (kPrefix: of group b) has its
// queries, from the call's first, which strides below 0 put behind it; kNowhere
// for a node that is not live.
constexpr int64_t kNowhere = INT64_MIN;
template <int kPart>
__device__ __forceinline__ int64_t query_at(const Params& p, int b, int node, int live) {
  if constexpr (kPart == kPrefix) {
    if (node >= live) return kNowhere;
    const int m = b * p.members + node / p.nodes, i = node % p.nodes;
    return i < __ldg(p.s.share + m).y ? m * p.a.q_seq + i * p.a.q_tok : kNowhere;
  } else {
    return node < live ? b * p.a.q_seq + node * p.a.q_tok : kNowhere;
  }
}

// A row's place in the call, rows of heads of nodes of sequences.
__device__ __forceinline__ int64_t row_at(const Params& p, int b, int h, int row) {
  return ((int64_t)b * p.a.n + row / p.g) * p.a.heads + h * p.g + row % p.g;
}
template <int D>
__device__ __forceinline__ float* prior_of(const Params& p, int64_t row) {
  return p.prior + row * kPieceRow<D>;
}

// Where row `row` of head group h of sequence b of the list goes.
template <typename T>
__device__ __forceinline__ T* out_row(const Params& p, int b, int h, int row, int head_dim) {
  return static_cast<T*>(p.a.out) + row_at(p, b, h, row) * head_dim;
}

// ------------------------------------------------------------- the schedule
//
// One warp walks the block's part of the line and publishes its groups, kJobs
// ahead: the divisions and searches stay out of the other warps' code and
// registers.

constexpr int kJobs = 4;

// A group, or the block's piece of one, as the scheduler publishes it.
struct Job {
  int b, h, row0, off, cnt, tiles;             // cnt 0: the end
  int q, len, live;                            // of the sequence
  int first_block, last_block;                 // blocks of the grid that hold the group
  Group grp;
  __device__ __forceinline__ bool whole() const { return off == 0 && cnt == tiles; }
};

// The scheduler warp: c is the place of unit u0.
template <int D, int kPart>
__device__ __forceinline__ void schedule(const Params& p, const Seq<kPart>* seqs, Cursor c, long long per, long long u0,
                                         long long u1, Job* jobs, uint64_t* ready, uint64_t* taken, int* abort) {
  const int lane = threadIdx.x & 31;
  Group grp = group_of(p, seqs[c.b], c.rt);
  long long u = u0;
  for (int n = 0;; ++n) {
    const int slot = n & (kJobs - 1);
    wait(taken + slot, ((n / kJobs) & 1) ^ 1, abort);
    const int cnt = u < u1 ? (int)min((long long)(grp.tiles - c.off), u1 - u) : 0;
    if (lane == 0) {
      Job& j = jobs[slot];
      j.cnt = cnt;
      if (cnt) {
        const Seq<kPart> q = seqs[c.b];
        j.b = c.b, j.h = c.h, j.row0 = c.rt * p.rows_per, j.off = c.off, j.tiles = grp.tiles;
        j.q = q.q, j.len = q.len, j.live = q.live;
        j.first_block = (int)((u - c.off) / per);
        j.last_block = (int)((u - c.off + grp.tiles - 1) / per);
        j.grp = grp;
        // a cut prefix's blocks, for the launch that joins them
        if (kPart == kPrefix && c.off == 0 && cnt < grp.tiles)
          *reinterpret_cast<int2*>(prior_of<D>(p, row_at(p, c.b, c.h, j.row0)) + 2) = int2{j.first_block, j.last_block};
      }
      mbar_arrive(ready + slot);
    }
    __syncwarp();
    if (!cnt) break;
    u += cnt;
    if (u < u1) advance(p, seqs, c, grp);
  }
}

// ---------------------------------------------------------- joining pieces

// Add the pieces that blocks c0..c1 left of a row tile, in their order.  First
// the rows' references and normalisers (into `stat`, shared memory of
// rows_per), then the dimensions, four a thread, kItems such and kAhead pieces
// at a time: a join is a wait for memory at the end of a block, so loads are
// issued together (many rows have few pieces, few rows many).  kRest with
// `prior`: what is there is the last piece.
template <typename T, int D, int kItems, int kAhead, int kPart>
__device__ void join_pieces(const Params& p, int b, int h, int row0, int live, int c0, int c1, bool prior, float2* stat,
                            int tid, int threads) {
  constexpr int R = kPieceRow<D>;
  const int lane = tid & 31, blocks = c1 - c0 + 1, pieces = blocks + (kPart == kRest && prior);
  const int64_t stride = 2 * (int64_t)p.rows_per * R;
  const float* first = piece_of<D>(p, c0, true);
  const float* later = piece_of<D>(p, c0, false);   // + stride for each block further
  auto at = [&](int cc, int r) -> const float* {
    if constexpr (kPart == kRest) {
      // a row that is not live has none there, and is not stored: any piece will do
      if (cc == blocks && (row0 + r) / p.g < live) return prior_of<D>(p, row_at(p, b, h, row0 + r));
      if (cc == blocks) cc = 0;
    }
    return (cc ? later + cc * stride : first) + r * R;
  };
  if (pieces <= 8 && p.rows_per <= threads) {   // a thread a row
    if (tid < p.rows_per) {
      float2 y[8];
      float top = kNone, l = 0.f;
#pragma unroll
      for (int cc = 0; cc < 8; ++cc) y[cc] = cc < pieces ? __ldcg(reinterpret_cast<const float2*>(at(cc, tid))) : float2{kNone, 0.f};
#pragma unroll
      for (int cc = 0; cc < 8; ++cc) top = fmaxf(top, y[cc].x);
#pragma unroll
      for (int cc = 0; cc < 8; ++cc) l += y[cc].y * ex2(y[cc].x - top);
      stat[tid] = float2{top, 1.f / l};
    }
  } else {   // a warp a row, a lane a piece
    for (int r = tid >> 5; r < p.rows_per; r += threads >> 5) {
      float top = kNone, l = 0.f;
      for (int cc = lane; cc < pieces; cc += 32) top = fmaxf(top, __ldcg(at(cc, r)));
#pragma unroll
      for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
      for (int cc = lane; cc < pieces; cc += 32) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(at(cc, r)));
        l += y.y * ex2(y.x - top);
      }
#pragma unroll
      for (int d = 16; d; d /= 2) l += __shfl_xor_sync(kFull, l, d);
      if (lane == 0) stat[r] = float2{top, 1.f / l};
    }
  }
  asm volatile("bar.sync 15, %0;" ::"r"(threads) : "memory");
  const int items = p.rows_per * (D / 4);
  for (int x0 = tid; x0 < items; x0 += kItems * threads) {
    float4 o[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) o[i] = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll kAhead
    for (int cc = 0; cc < pieces; ++cc) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int x = min(x0 + i * threads, items - 1), r = x / (D / 4), d = x % (D / 4) * 4;
        const float* pr = at(cc, r);
        const float f = ex2(__ldcg(pr) - stat[r].x);
        const float4 y = __ldcg(reinterpret_cast<const float4*>(pr + 4 + d));
        o[i].x += y.x * f, o[i].y += y.y * f, o[i].z += y.z * f, o[i].w += y.w * f;
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int x = x0 + i * threads, r = x / (D / 4), d = x % (D / 4) * 4, row = row0 + r;
      if (x >= items || row / p.g >= live) continue;
      const float inv = stat[r].y;
      store4(out_row<T>(p, b, h, row, D) + d, float4{o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv});
    }
  }
}

}  // namespace
}  // namespace cache
}  // namespace mds
