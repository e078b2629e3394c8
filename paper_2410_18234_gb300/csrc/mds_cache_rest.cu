// The part behind a shared prefix where few rows read short runs of slots: one
// token of many sequences, up to 8 rows a key/value head, 16-bit queries.
//
// The kernel for few rows gives a group's tiles to all the warps of a block and
// lets their sums meet at its end, some 8 us a group: right for long caches,
// but a rest is a few tiles.  Here a warp is on its own.  The line of all
// groups' blocks of 16 slots is cut evenly among all warps of the grid; a warp
// copies its blocks into a ring of its own (8 KB), turns them into sums in
// registers, and writes a group that lies within its part out itself, the
// prefix's sums added.  A group that is cut leaves pieces: a warp has at most
// one that it continues (in shared memory of its own) and one that it begins
// (in its ring, which is empty by then).  Where the warps are done the first
// warp of each cut group adds the block's pieces, and pieces of a group that
// is cut between blocks of threads are joined like everywhere (join_pieces).
// Joins cost more than a little unevenness, so cuts go to the nearest end of a
// short group.
//
// What binds it is issue slots (46 % busy) and uneven ends (the last warp is
// done 1.4 times as late as the mean), not bytes.  Rests of 1 to 1000 tokens
// of 128 sequences, 32 heads on 8 of 128 dimensions (140 MB): 50 us, 2.8 TB/s;
// the kernel for few rows takes 102.  Behind a prefix of 32768 tokens, up to 300
// tokens of 256 sequences: 40 us, which took more than 70 off the call's 324.
#include "mds_cache_few.cuh"

namespace mds {
namespace cache {

namespace {

constexpr int kWarps = 16, kThreads = 32 * kWarps, kRows = 8;
constexpr int kRing = 8192;
// The line counts kExtra blocks more for each group: what its queries and its
// end take.  Of a warp's share there are kLeast at least.  Groups of so many
// are not cut: between warps of a block up to its share and kWarpSlack, between
// blocks of threads up to kBlockSlack (a warp's block takes about 1.2 us,
// adding a cut group's pieces 4 us, a join 9 us).
constexpr int kExtra = kRestExtra, kLeast = kExtra + 2, kWarpSlack = 3, kBlockSlack = 96;

template <int D>
struct Rest {
  static constexpr int kStage = 2 * kBlock * D, kStages = kRing / kStage;
  static constexpr int kPiece = kRows * kPieceRow<D> * 4;
  static constexpr int smem(int B) {
    return 1024 + kWarps * (kRing + kPiece + kStages * 16) + kRows * 8 + 64 + (B + 2) / 2 * 16 + seq_bytes<kRest>(B);
  }
};

// A place on the line: unit off of cnt of head h of sequence b, of which the
// first kExtra stand for no block.
struct Walk {
  int b, h, off, cnt;
  __device__ __forceinline__ int block() const { return max(off - kExtra, 0); }
};
__device__ __forceinline__ int blocks_of(const Params& p, const long long* prefix, int b) {
  return (int)(prefix[b + 1] - prefix[b]) / p.s.kv_heads;   // at most 2^26 between two sequences
}
__device__ __forceinline__ Walk walk_to(const Params& p, const long long* prefix, long long u) {
  int lo = 0, hi = p.a.B - 1;
  while (lo < hi) {   // the last b with prefix[b] <= u
    const int mid = (lo + hi + 1) / 2;
    if (prefix[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  Walk w;
  w.b = lo;
  w.cnt = blocks_of(p, prefix, lo);
  const int rest = (int)(u - prefix[lo]);
  w.h = rest / w.cnt;
  w.off = rest - w.h * w.cnt;
  return w;
}
// Where a cut at u goes: to the nearest end of its group, if that has at most
// `most` blocks.
__device__ __forceinline__ long long cut_at(const Params& p, const long long* prefix, long long u, long long total, int most) {
  if (u >= total) return total;
  const Walk w = walk_to(p, prefix, u);
  // never within the units that stand for no block
  if (w.cnt > most) return w.off > kExtra ? u : u - w.off;
  return 2 * w.off < w.cnt ? u - w.off : u - w.off + w.cnt;
}
// To the next group's first block; not past the line's end.
__device__ __forceinline__ void next_group(const Params& p, const long long* prefix, Walk& w) {
  w.off = 0;
  if (++w.h < p.s.kv_heads) return;
  w.h = 0;
  do {
    if (++w.b >= p.a.B) return;
  } while (prefix[w.b + 1] == prefix[w.b]);
  w.cnt = blocks_of(p, prefix, w.b);
}

// Add a group's `count` (at most 16) pieces of this block of threads, the
// first at `first`, the others the continued ones of the warps behind: with
// `complete` to the output, the prefix's sums too; else to `to`.  Factors
// first, four lanes a row, which go to a place of the pieces' rows that is not
// used; then the sums.
template <int D>
__device__ void add_pieces(const Params& p, int b, int h, int live, bool prior, float* first, float* others, int count,
                           bool complete, float* to) {
  constexpr int R = kPieceRow<D>, kEach = D / 32;
  const int lane = threadIdx.x & 31, row = lane >> 2, rows = min(kRows, live * p.g);
  auto piece = [&](int c, int r) { return (c ? others + (c - 1) * (kRows * R) : first) + r * R; };
  prior = prior && complete;
  float2 its{kNone, 0.f};
  if (prior && row < rows) its = __ldcg(reinterpret_cast<const float2*>(prior_of<D>(p, row_at(p, b, h, row))));
  float top = its.x, l = 0.f;
  for (int c = lane & 3; c < count; c += 4) top = fmaxf(top, piece(c, row)[0]);
  top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
  top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
  for (int c = lane & 3; c < count; c += 4) {
    float* x = piece(c, row);
    const float f = ex2(x[0] - top);
    l += x[1] * f;
    x[2] = f;
  }
  l += __shfl_xor_sync(kFull, l, 1);
  l += __shfl_xor_sync(kFull, l, 2);
  const float fp = ex2(its.x - top);
  l += its.y * fp;
  __syncwarp();
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    float o[kEach] = {};
    if (prior) {
      const float* x = prior_of<D>(p, row_at(p, b, h, r)) + 4 + lane * kEach;
#pragma unroll
      for (int i = 0; i < kEach; i += 2) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(x + i));
        o[i] = y.x, o[i + 1] = y.y;
      }
    }
    const float f0 = __shfl_sync(kFull, fp, r * 4), sum = __shfl_sync(kFull, l, r * 4), most = __shfl_sync(kFull, top, r * 4);
#pragma unroll
    for (int i = 0; i < kEach; ++i) o[i] *= f0;
    for (int c = 0; c < count; ++c) {
      const float* x = piece(c, r);
      const float f = x[2];
#pragma unroll
      for (int i = 0; i < kEach; ++i) o[i] += f * x[4 + lane * kEach + i];
    }
    if (complete) {
      const float inv = 1.f / sum;
      unsigned* out = reinterpret_cast<unsigned*>(out_row<__nv_bfloat16>(p, b, h, r, D) + lane * kEach);
#pragma unroll
      for (int i = 0; i < kEach; i += 2) out[i / 2] = pack_bf16(o[i] * inv, o[i + 1] * inv);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) __stcg(to + r * R + 4 + lane * kEach + i, o[i]);
      if (lane == 0) __stcg(reinterpret_cast<float2*>(to + r * R), float2{most, sum});
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) rest_kernel(const __grid_constant__ Params p) {
  using X = Rest<D>;
  using T = __nv_bfloat16;
  constexpr int R = kPieceRow<D>;
  extern __shared__ char raw[];
  char* at = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  char* ring = at + warp * kRing;
  at += kWarps * kRing;
  float* pieces = reinterpret_cast<float*>(at);   // of the warps, that they continue
  at += kWarps * X::kPiece;
  float* scales = reinterpret_cast<float*>(at) + warp * X::kStages * 2;
  at += kWarps * X::kStages * 8;
  uint64_t* full = reinterpret_cast<uint64_t*>(at) + warp * X::kStages;
  at += kWarps * X::kStages * 8;
  float2* stat = reinterpret_cast<float2*>(at);
  at += kRows * 8;
  int* abort = reinterpret_cast<int*>(at);
  int* cut = abort + 1;        // [2][5]: groups cut between blocks: sequence (-1: none), head, blocks, whether to join
  at += 64;
  long long* prefix = reinterpret_cast<long long*>(at);
  at += (p.a.B + 2) / 2 * 16;
  Seq<kRest>* seqs = reinterpret_cast<Seq<kRest>*>(at);

  if (lane == 0)
    for (int i = 0; i < X::kStages; ++i) mbar_init(full + i, 1 + 32);   // the byte count, and the lanes' scale copies
  if (tid == 0) *abort = 0, cut[0] = cut[5] = -1;
  mbar_init_fence();
  after_launch_before();
  if (idle<kRest>(p)) return;
  plan<T, kRest, true>(p, prefix, seqs, D);   // ends in a barrier
  const long long total = prefix[p.a.B], share = (total + gridDim.x - 1) / gridDim.x;   // of a block of threads
  const int slack = (int)max(share / 4, (long long)kBlockSlack);
  // the block's two cuts, then a warp's a lane; by every warp for itself
  long long c0 = 0, c1 = 0, cut_u = share * (blockIdx.x + lane);
  int most = slack, per = 0;
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    cut_u = cut_at(p, prefix, cut_u, total, most);
    if (i) break;
    c0 = __shfl_sync(kFull, cut_u, 0), c1 = __shfl_sync(kFull, cut_u, 1);
    if (c0 >= c1) return;
    per = max((int)(c1 - c0 + kWarps - 1) / kWarps, kLeast);
    most = per + kWarpSlack;
    cut_u = min(c0 + (long long)per * lane, c1);
  }
  // (of a block's part the ends are cuts already)
  cut_u = min(max(cut_u, c0), c1);
  if (lane == 0) cut_u = c0;
  if (lane >= kWarps) cut_u = c1;
  const long long w0 = __shfl_sync(kFull, cut_u, warp), w1 = __shfl_sync(kFull, cut_u, warp + 1);
  const State& s = p.s;
  const int gr = lane >> 2, tq = lane & 3, rows = p.rows;

  long long begun = -1;        // where the group lies that this warp begins and does not end
  Walk first{}, last{};
  if (w0 < w1) {
    const int64_t layer0 = (int64_t)p.a.layer * s.pages;
    Walk c = walk_to(p, prefix, w0), f = c;
    first = c;
    long long u = w0, uf = w0;
    if (f.off == 0) f.off = kExtra, uf += kExtra;   // a warp's part begins with a group, or behind its first block
    // the copies' part: slot and page of the next block, looked up a copy ahead;
    // lane 0 copies keys, lane 1 values
    int slot = 0, page = 0, put = 0;
    const int32_t* table = nullptr;
    auto find_group = [&] {
      const Seq<kRest> q = seqs[f.b];
      slot = q.from + f.block() * kBlock;
      table = s.table + (int64_t)q.q * s.max_pages;
      page = __ldg(table + (slot >> s.page_log));
    };
    find_group();
    bool stop = false;   // a wait gave up, of any lane: no more copies, as their places may still be written
    auto fetch = [&] {
      if (uf >= w1 || stop) return;
      if (lane == 0) mbar_expect_tx(full + put, X::kStage);
      __syncwarp();
      if (lane < 2) {
        const int64_t row = (((layer0 + page) * 2 + lane) * s.kv_heads + f.h) * s.page_tokens + (slot & (s.page_tokens - 1));
        bulk_copy(ring + put * X::kStage + lane * kBlock * D, s.pool + row * D, kBlock * D, full + put);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(scales + put * 2 + lane)), "l"(s.scales + (row >> 4))
                     : "memory");
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(full + put)) : "memory");
      if (++put == X::kStages) put = 0;
      if (++uf >= w1) return;
      if (++f.off == f.cnt) {
        next_group(p, prefix, f);
        uf += kExtra;
        f.off = kExtra;
        find_group();
      } else if (((slot += kBlock) & (s.page_tokens - 1)) == 0) {
        page = __ldg(table + (slot >> s.page_log));
      }
    };
#pragma unroll 1
    for (int i = 0; i < X::kStages; ++i) fetch();
    const Places<D> places(lane);
    int get = 0;
    unsigned parity = 0;
#pragma unroll 1
    while (u < w1) {
      const Seq<kRest> q = seqs[c.b];
      const long long end = min(w1, u + c.cnt - c.off);   // at least a block of it is in front of w1
      const long long start = u;
      const bool begins = c.off == 0, ends = u + c.cnt - c.off <= w1;
      last = c;
      // row gr's queries: lane (gr, tq) has the dimensions of units tq, tq + 4
      uint2 query[D / 16];
      float rc[1][2];
      int node[1][2], own[1][2];
      {
        const int i = gr / p.g;
        uint4 y[D / 64][2];
#pragma unroll
        for (int x = 0; x < D / 64; ++x) y[x][0] = y[x][1] = uint4{0, 0, 0, 0};
        if (gr < rows && i < q.live) {
          const T* src = static_cast<const T*>(p.a.q) + c.b * p.a.q_seq + i * p.a.q_tok + (c.h * p.g + gr % p.g) * p.a.q_head;
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
#pragma unroll
            for (int z = 0; z < 2; ++z) y[x][z] = __ldg(reinterpret_cast<const uint4*>(src + (tq + 4 * x) * 16) + z);
        }
        unsigned w[D / 64 * 8], bits = 0;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          const uint4& z = y[x >> 1][x & 1];
          w[4 * x] = z.x, w[4 * x + 1] = z.y, w[4 * x + 2] = z.z, w[4 * x + 3] = z.w;
        }
#pragma unroll
        for (int x = 0; x < D / 8; ++x) bits = max(bits, max(w[x] << 16 & 0x7fff0000u, w[x] & 0x7fff0000u));
#pragma unroll
        for (int d = 1; d < 4; d *= 2) bits = max(bits, __shfl_xor_sync(kFull, bits, d));
        // 2^-e brings the maximum into [2^14, 2^15); zero and non-finite rows stay as they are
        const int e = bits == 0 || bits >= 0x7f800000u ? 0 : max((int)(bits >> 23) - 127 - 14, -112);
        const float inv = __uint_as_float((unsigned)(127 - e) << 23);
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
          const __half2 a = __floats2half2_rn(__uint_as_float(w[2 * x] << 16) * inv, __uint_as_float(w[2 * x] & 0xffff0000u) * inv);
          const __half2 b = __floats2half2_rn(__uint_as_float(w[2 * x + 1] << 16) * inv, __uint_as_float(w[2 * x + 1] & 0xffff0000u) * inv);
          query[x] = uint2{*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b)};
        }
        const float k = p.a.scale * dev::kLog2e * __uint_as_float((unsigned)(127 + e) << 23);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          rc[0][r] = __shfl_sync(kFull, k, (tq * 2 + r) * 4);
          const int x = (tq * 2 + r) / p.g;
          node[0][r] = x;
          own[0][r] = x > 0 && p.a.L > 0 ? 1 + (x - 1) / p.a.L * p.a.L : 1;
        }
      }
      const int hi = min(q.len + q.live, q.end);
      int t0 = q.from + c.block() * kBlock;
      if (begins) u += kExtra;
      Sums<D, 1> x;
      x.clear();
#pragma unroll 1
      for (; u < end; ++u, t0 += kBlock) {
        const bool there = wait(full + get, parity, abort);
        const char* kb = ring + get * X::kStage;
        few_block<T, D, 1>(p, kb, smem_u32(kb + kBlock * D), scales[get * 2], scales[get * 2 + 1], places,
                           [&](int i) { return query[i]; }, node, own, rc, t0, q.len, hi, x);
        stop = __any_sync(kFull, !there) || stop;
        fetch();
        if (++get == X::kStages) get = 0, parity ^= 1u;
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int d = 4; d < 32; d *= 2) x.sum[0][r] += __shfl_xor_sync(kFull, x.sum[0][r], d);
      if (begins && ends) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = tq * 2 + r;
          if (row / p.g >= q.live) continue;
          const int64_t to = row_at(p, c.b, c.h, row);
          float2 y{kNone, 0.f}, z[D / 16];
#pragma unroll
          for (int i = 0; i < D / 16; ++i) z[i] = float2{0.f, 0.f};
          if (q.from > 0) {
            const float* its = prior_of<D>(p, to);
            y = __ldcg(reinterpret_cast<const float2*>(its));
#pragma unroll
            for (int i = 0; i < D / 16; ++i) z[i] = __ldcg(reinterpret_cast<const float2*>(its + 4 + i * 16 + gr * 2));
          }
          const float top = fmaxf(x.ref[0][r], y.x), mine = ex2(x.ref[0][r] - top), its = ex2(y.x - top);
          const float inv = 1.f / (x.sum[0][r] * mine + y.y * its);
          unsigned* out = reinterpret_cast<unsigned*>(static_cast<T*>(p.a.out) + to * D + gr * 2);
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            out[i * 8] = pack_bf16((x.acc[0][i][r] * mine + z[i].x * its) * inv, (x.acc[0][i][2 + r] * mine + z[i].y * its) * inv);
        }
      } else {
        // of a group that it begins the ring's place: no copy is under way behind the warp's last block
        float* piece = begins ? reinterpret_cast<float*>(ring) : pieces + warp * (kRows * R);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float* to = piece + (tq * 2 + r) * R;
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            *reinterpret_cast<float2*>(to + 4 + i * 16 + gr * 2) = float2{x.acc[0][i][r], x.acc[0][i][2 + r]};
          if (gr == 0) *reinterpret_cast<float2*>(to) = float2{x.ref[0][r], x.sum[0][r]};
        }
        if (begins) begun = start;
      }
      next_group(p, prefix, c);
    }
  }
  __syncthreads();

  // ---- cut groups, each by the first of the block's warps that has a piece of it
  if (w0 < w1) {
    auto add = [&](const Walk& w, long long start, float* piece, int slot) {
      const long long end = start + w.cnt, until = min(end, c1);
      const int count = 1 + __popc(__ballot_sync(kFull, lane > warp && lane < kWarps && cut_u < until));
      const bool complete = start >= c0 && end <= c1;
      add_pieces<D>(p, w.b, w.h, seqs[w.b].live, seqs[w.b].from > 0, piece, pieces + (warp + 1) * (kRows * R), count, complete,
                    piece_of<D>(p, blockIdx.x, start >= c0));
      if (!complete && lane == 0) {
        // cuts within a group that is cut between blocks are where they fall, but for its first kExtra units
        cut[slot + 1] = w.h, cut[slot + 2] = (int)((start + kExtra) / share), cut[slot + 3] = (int)((end - 1) / share);
        cut[slot] = w.b;
      }
    };
    if (warp == 0 && first.off > 0) add(first, w0 - first.off, pieces, 0);
    if (begun >= 0) add(last, begun, reinterpret_cast<float*>(ring), 5);
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      int* x = cut + 5 * i;
      if (x[0] < 0) continue;
      const bool join = atomicAdd(s.joins + x[2], 1u) == (unsigned)(x[3] - x[2]);
      if (join) s.joins[x[2]] = 0;
      x[4] = join;
    }
  }
  __syncthreads();
  for (int i = 0; i < 2; ++i) {
    const int* x = cut + 5 * i;
    if (x[0] < 0 || !x[4]) continue;
    __threadfence();
    join_pieces<T, D, 1, 8, kRest>(p, x[0], x[1], 0, seqs[x[0]].live, x[2], x[3], seqs[x[0]].from > 0, stat, tid, kThreads);
    __syncthreads();
  }
  if (tid == 0) report(abort, s.status);
}

template <int D>
cudaError_t launch(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  static_assert(Rest<D>::smem(MDS_CACHE_MAX_BATCH) <= 227 * 1024, "shared memory for the largest batch");
  Params p{s, a, kBlock, a.heads / s.kv_heads, 0, 1, 0, kRows};
  p.rows = a.n * p.g;
  p.members = x.members;
  p.nodes = x.nodes;
  p.prior = x.prior;
  p.worth = x.worth;
  p.each = x.each;
  p.saved = x.saved;
  return launch_behind(rest_kernel<D>, attend_grid(sms, kRows, D, kPieceFloats), kThreads, Rest<D>::smem(a.B), st, p);
}

}  // namespace

cudaError_t configure_rest() {
  const cudaError_t e = cudaFuncSetAttribute(rest_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  return e == cudaSuccess ? cudaFuncSetAttribute(rest_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) : e;
}

cudaError_t shared_rest(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  return s.head_dim == 64 ? launch<64>(s, a, x, sms, st) : launch<128>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
