// Attention of draft-tree nodes over the 8-bit paged cache, for few rows a
// key/value head and for 32-bit queries; many rows: mds_cache_many.cu.
//
//   o_i = sum_t w_it v_t / sum_t w_it,   w_it = 2^(c q_i . k_t - m_i),   c = scale * log2(e)
//
// over the slots t that node i sees, m_i a running reference.  A block of 16
// slots of one head has one scale 2^a for its keys and one 2^b for its
// values: 2^a multiplies the block's scores, 2^b its values.
//
// Products.  Every e4m3 number is exact in 16 bits, so products are taken in
// 16 bits with 32-bit sums.  Keys meet queries in half precision: a row of
// queries is first scaled by a power of two to a maximum in [2^14, 2^15),
// where a bfloat16 query has no rounding, and a 32-bit one is carried by two
// terms (22 bits and a sign).  Weights meet values in bfloat16, whose range
// holds any value: a 16-bit query's weight is rounded once (2^-8 relative, and
// the normaliser sums the rounded weights, so that a row that sees one token
// returns that token's value), a 32-bit one's is carried by three terms.
#include "mds_cache_attend.cuh"

namespace mds {
namespace cache {

namespace {

constexpr int kStageMax = 8;
constexpr int kJoinStride = 68;   // floats of a joined row's 64 dimensions: two rows are 8 banks apart

__device__ __forceinline__ void mma_f16(float* c, const unsigned* a, uint2 b) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ void mma_bf16(float* c, const unsigned* a, uint2 b) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ void ldmatrix_x4_trans(unsigned* r, unsigned addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ unsigned transposed(unsigned x) {   // an 8 x 8 matrix of 16-bit numbers
  unsigned r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// Transposed, like the kernel for many rows: a product's 16 rows are slots or
// dimensions, its 8 columns the attention's rows, so that up to 8 rows (one
// token of 8 query heads) waste nothing of the product that an instruction
// does, and hold 32 sums a lane where rows on the other side would hold 64.
//
//   S^T [16 slots][8 rows] = K Q^T,   O^T [16 dimensions][8 rows] += V^T W^T
//
// A warp takes one block of 16 slots of a tile for all the rows: its scores,
// weights and sums stay in registers, its key and value scales are two
// numbers, and the warps' sums meet once per group.  kSets sets of eight warps
// take the tiles in turn.
//
// Bound by the cache's bytes: 8 sequences of 65k to 131k tokens, 32 heads on 8:
// 251 us, 6.55 TB/s (97 % of a copy's rate).  A block of 4096 bytes takes about
// 300 instructions, half of which widen the values to bfloat16.
// NT: tiles of 8 rows.
template <typename T, int D, int NT>
struct Few {
  static constexpr int kQ = sizeof(T) == 4 ? 2 : 1;   // terms of a query
  static constexpr int kW = sizeof(T) == 4 ? 3 : 1;   // terms of a weight
  static constexpr int kSets = NT == 1 ? 2 : 1;
  static constexpr int kWarps = 8 * kSets, kThreads = 32 * kWarps;   // consumers; then a loader and a scheduler
  static constexpr int kRows = 8 * NT;
  static constexpr int kSteps = D / 16;
  static constexpr int kStageBytes = 2 * kTile * D;
  static constexpr int kQBytes = NT * kQ * kSteps * 256;
  static constexpr int kJoinBytes = 8 * 8 * kJoinStride * 4;
  // after the stages: queries, join buffer, per-warp (reference, sum), row coefficients, stage scales, barriers
  static constexpr int kFixed =
      kQBytes + kJoinBytes + kWarps * kRows * 8 + kRows * 4 + kStageMax * 16 * 4 + (2 * kStageMax + 2 * kJobs) * 8 + kJobs * (int)sizeof(Job) + 16;
  static int smem(int stages, int B) { return 1024 + stages * kStageBytes + kFixed + (B + 1) * 8 + B * 16 + 16; }
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(Few<T, D, NT>::kThreads + 64, 1) few_kernel(const __grid_constant__ Params p) {
  using F = Few<T, D, NT>;
  extern __shared__ char raw[];
  char* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  char* stage_mem = base;
  char* at = base + p.stages * F::kStageBytes;
  uint2* qf = reinterpret_cast<uint2*>(at);
  at += F::kQBytes;
  float* join = reinterpret_cast<float*>(at);
  at += F::kJoinBytes;
  float2* ml = reinterpret_cast<float2*>(at);
  at += F::kWarps * F::kRows * 8;
  float* coef = reinterpret_cast<float*>(at);
  at += F::kRows * 4;
  float* stage_scales = reinterpret_cast<float*>(at);
  at += kStageMax * 16 * 4;
  uint64_t* full = reinterpret_cast<uint64_t*>(at);
  uint64_t* empty = full + kStageMax;
  uint64_t* ready = empty + kStageMax;
  uint64_t* taken = ready + kJobs;
  at += (2 * kStageMax + 2 * kJobs) * 8;
  Job* jobs = reinterpret_cast<Job*>(at);
  at += kJobs * sizeof(Job);
  int* abort = reinterpret_cast<int*>(at);
  int* last_s = abort + 1;
  at += 16;
  long long* prefix = reinterpret_cast<long long*>(at);
  at += ((p.a.B + 1) * 8 + 15) / 16 * 16;
  Seq* seqs = reinterpret_cast<Seq*>(at);

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    *abort = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(full + i, 1 + 32);       // the loader's byte count, and its lanes' scale copies
      mbar_init(empty + i, 8);
    }
    for (int i = 0; i < kJobs; ++i) {
      mbar_init(ready + i, 1);
      mbar_init(taken + i, F::kWarps + 1);
    }
    mbar_init_fence();
  }
  plan<T>(p, prefix, seqs, D);   // ends in a barrier
  const long long total = prefix[p.a.B];
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  const long long u0 = per * blockIdx.x, u1 = min(u0 + per, total);
  if (u0 >= u1) return;

  if (warp == F::kWarps + 1) {
    schedule(p, seqs, locate(p, prefix, seqs, u0), per, u0, u1, jobs, ready, taken, abort);
    return;
  }
  auto job_at = [&](int n) -> const Job& {
    wait(ready + (n & (kJobs - 1)), (n / kJobs) & 1, abort);
    return jobs[n & (kJobs - 1)];
  };
  auto job_done = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(taken + (n & (kJobs - 1)));
  };

  if (warp == F::kWarps) {
    // ---- loader: one block of 16 slots a lane (keys: lanes 0..7, values: 8..15);
    // the first of a page's blocks copies for all of them
    const State& s = p.s;
    const int kv = (lane >> 3) & 1, blk = lane & 7;
    const int64_t layer0 = (int64_t)p.a.layer * s.pages;
    int stage = 0;
    unsigned phase = 1;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      const int off = job.off, end = off + job.cnt, h = job.h;
      if (!job.cnt) break;
      const Group grp = job.grp;
      const int32_t* table = s.table + (int64_t)job.q * s.max_pages;
      job_done(n);
      auto page_of = [&](int i) {
        const int t = (tile_slot(grp, i) + blk * kBlock) & -p.span;
        return lane < 16 && i < end && block_seen(grp, t, p.span) ? __ldg(table + (t >> s.page_log)) : -1;
      };
      int page = page_of(off);
      for (int i = off; i < end; ++i) {
        const int next = page_of(i + 1);
        const int t = tile_slot(grp, i) + blk * kBlock;
        wait(empty + stage, phase, abort);
        const bool copies = page >= 0 && (t & (p.span - 1)) == 0;   // the first block of its span
        const unsigned takes = __ballot_sync(kFull, copies);
        if (lane == 0) mbar_expect_tx(full + stage, __popc(takes) * p.span * D);
        __syncwarp();
        if (page >= 0) {
          const int64_t tile = ((layer0 + page) * 2 + kv) * s.kv_heads + h;
          const int r = t & (s.page_tokens - 1);
          const uint8_t* src = s.pool + (tile * s.page_tokens + r) * D;
          if (copies)
            bulk_copy(stage_mem + stage * F::kStageBytes + (kv * kTile + blk * kBlock) * D, src, p.span * D, full + stage);
          const float* sc = s.scales + ((tile * s.page_tokens + r) >> 4);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(stage_scales + stage * 16 + lane)),
                       "l"(sc)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(full + stage)) : "memory");
        page = next;
        if (++stage == p.stages) stage = 0, phase ^= 1u;
      }
    }
    report(abort, s.status);
    return;
  }

  // ---- consumers
  auto consumers_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(F::kThreads) : "memory"); };
  const int gr = lane >> 2, tq = lane & 3, set = warp >> 3, blk = warp & 7;
  unsigned k_at[2][D / 64], v_at[D / 32];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int x = 0; x < D / 64; ++x) k_at[j][x] = swizzled((j * 8 + gr) * D + (tq + 4 * x) * 16);
#pragma unroll
  for (int x = 0; x < D / 32; ++x) {
    const int key = (lane & 7) + ((lane >> 3) & 1) * 8, chunk = 2 * x + (lane >> 4);
    v_at[x] = swizzled(key * D + chunk * 16);
  }
  int stage = 0, turn = 0;
  unsigned phase = 0;
  for (int n = 0;; ++n) {
    const Job& job = job_at(n);
    if (!job.cnt) break;
    const int row0 = job.row0;
    // queries of the group: scaled, in the order of the products' fragments
    for (int r = warp; r < F::kRows; r += F::kWarps) {
      const int row = row0 + r, node = row / p.g, head = job.h * p.g + row - node * p.g;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (lane * 4 < D && node < job.live) {
        const T* src = static_cast<const T*>(p.a.q) + job.b * p.a.q_seq + node * p.a.q_tok + head * p.a.q_head + lane * 4;
        if constexpr (sizeof(T) == 4) {
          const float4 y = __ldg(reinterpret_cast<const float4*>(src));
          x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
        } else {
          const uint2 y = __ldg(reinterpret_cast<const uint2*>(src));
          x[0] = __uint_as_float(y.x << 16), x[1] = __uint_as_float(y.x & 0xffff0000u);
          x[2] = __uint_as_float(y.y << 16), x[3] = __uint_as_float(y.y & 0xffff0000u);
        }
      }
      const float most = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
      const unsigned bits = __reduce_max_sync(kFull, __float_as_uint(most) & 0x7fffffffu);
      // 2^-e brings the maximum into [2^14, 2^15); zero and non-finite rows stay as they are
      const int e = bits == 0 || bits >= 0x7f800000u ? 0 : max((int)(bits >> 23) - 127 - 14, -112);
      const float inv = __uint_as_float((unsigned)(127 - e) << 23);
      if (lane == 0) coef[r] = p.a.scale * dev::kLog2e * __uint_as_float((unsigned)(127 + e) << 23);
      if (lane * 4 < D) {
        const int chunk = lane >> 2, step = (chunk >> 2) * 4 + (lane & 3), to = (r & 7) * 4 + (chunk & 3);
#pragma unroll
        for (int term = 0; term < F::kQ; ++term) {
          unsigned w[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float y0 = x[2 * i] * inv, y1 = x[2 * i + 1] * inv;
            if (term) {
              y0 -= __half2float(__float2half_rn(y0));
              y1 -= __half2float(__float2half_rn(y1));
            }
            const __half2 hh = __floats2half2_rn(y0, y1);
            w[i] = *reinterpret_cast<const unsigned*>(&hh);
          }
          qf[(((r >> 3) * F::kQ + term) * F::kSteps + step) * 32 + to] = uint2{w[0], w[1]};
        }
      }
    }
    // this lane's rows, 2 tq and 2 tq + 1 of each tile of 8
    int node[NT][2], own[NT][2];   // node, and the first node of its branch
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int i = (row0 + m * 8 + tq * 2 + x) / p.g;
        node[m][x] = i;
        own[m][x] = i > 0 && p.a.L > 0 ? 1 + (i - 1) / p.a.L * p.a.L : 1;
      }
    consumers_sync();
    float rc[NT][2], ref[NT][2], sum[NT][2], acc[NT][D / 16][4];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        rc[m][x] = coef[m * 8 + tq * 2 + x];
        ref[m][x] = kNone;
        sum[m][x] = 0.f;
      }
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
#pragma unroll
        for (int z = 0; z < 4; ++z) acc[m][x][z] = 0.f;

    const Group grp = job.grp;
    const int off = job.off, end = off + job.cnt, len = job.len;
    for (int i = off; i < end; ++i) {
      const int t0 = tile_slot(grp, i) + blk * kBlock;
      if ((turn++ & (F::kSets - 1)) == set) {
        wait(full + stage, phase, abort);
        if (block_seen(grp, t0)) {
          const char* kb = stage_mem + stage * F::kStageBytes + blk * kBlock * D;
          const unsigned vb = smem_u32(kb + kTile * D);
          const float ks = stage_scales[stage * 16 + blk], vs = stage_scales[stage * 16 + 8 + blk];
          // scores: x[m][2 h + r] of slot t0 + gr + 8 h and row 2 tq + r; even and
          // odd steps into sums of their own, for shorter chains of products
          float sc[2][NT][4];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
              for (int z = 0; z < 4; ++z) sc[h][m][z] = 0.f;
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            const uint4 k0 = *reinterpret_cast<const uint4*>(kb + k_at[0][x]);
            const uint4 k1 = *reinterpret_cast<const uint4*>(kb + k_at[1][x]);
            const unsigned w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              unsigned a[4];
              to_f16(w0[y], a[0], a[2]);
              to_f16(w1[y], a[1], a[3]);
#pragma unroll
              for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int term = 0; term < F::kQ; ++term)
                  mma_f16(sc[y & 1][m], a, qf[((m * F::kQ + term) * F::kSteps + x * 4 + y) * 32 + lane]);
            }
          }
          // in log2 units, masked
          const bool plain = t0 + kBlock <= len &&
                             (p.a.window <= 0 || t0 + kBlock <= p.a.sinks || t0 > len + min(p.a.L, p.a.n - 1) - p.a.window);
          float w[NT][4];
          bool moves = false;
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int z = 0; z < 4; ++z)   // rounded: the largest, as a reference, leaves nothing of itself
              w[m][z] = __fmul_rn(sc[0][m][z] + sc[1][m][z], rc[m][z & 1] * ks);
          if (!plain) {
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const int t = t0 + (z >> 1) * 8 + gr, at_node = t - len, i_row = node[m][z & 1], b0 = own[m][z & 1];
                bool see = at_node <= i_row && (at_node <= 0 || at_node >= b0) && t < grp.hi;
                if (p.a.window > 0) {
                  const int pos = at_node <= 0 ? t : len + at_node - b0 + 1;
                  const int mine = len + (i_row > 0 ? i_row - b0 + 1 : 0);
                  see = see && (pos < p.a.sinks || pos > mine - p.a.window);
                }
                if (!see) w[m][z] = dev::kNegInf;
              }
          }
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) moves |= fmaxf(w[m][r], w[m][2 + r]) > ref[m][r] + kSlack;
          if (__any_sync(kFull, moves)) {
#pragma unroll
            for (int m = 0; m < NT; ++m) {
              float alpha[2];
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                float top = fmaxf(w[m][r], w[m][2 + r]);
#pragma unroll
                for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
                top = fmaxf(top, ref[m][r]);
                alpha[r] = ex2(ref[m][r] - top);
                ref[m][r] = top;
                sum[m][r] *= alpha[r];
              }
#pragma unroll
              for (int x = 0; x < D / 16; ++x)
#pragma unroll
                for (int z = 0; z < 4; ++z) acc[m][x][z] *= alpha[z & 1];
            }
          }
          // weights; the values' scale goes to the values
          uint2 b[NT][F::kW];
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float w0 = ex2(w[m][2 * h] - ref[m][0]), w1 = ex2(w[m][2 * h + 1] - ref[m][1]);
              if constexpr (F::kW > 1) sum[m][0] += w0, sum[m][1] += w1;
#pragma unroll
              for (int term = 0; term < F::kW; ++term) {
                const unsigned pk = pack_bf16(w0, w1);
                const float r0 = __uint_as_float(pk << 16), r1 = __uint_as_float(pk & 0xffff0000u);
                if constexpr (F::kW == 1) sum[m][0] += r0, sum[m][1] += r1;
                w0 -= r0;
                w1 -= r1;
                (h ? b[m][term].y : b[m][term].x) = transposed(pk);
              }
            }
          unsigned rest;
          const unsigned factor = value_factor(vs, rest);
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            unsigned v[4];
            ldmatrix_x4_trans(v, vb + v_at[x]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              unsigned a[4];   // even and odd dimensions of 8 slots, then of the other 8
              to_bf16(v[2 * y], factor, a[0], a[1]);
              to_bf16(v[2 * y + 1], factor, a[2], a[3]);
              if (rest != 0x3f803f80u) {
#pragma unroll
                for (int z = 0; z < 4; ++z) times_rest(a[z], rest);
              }
#pragma unroll
              for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int term = 0; term < F::kW; ++term) mma_bf16(acc[m][2 * x + y], a, b[m][term]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + stage);
      }
      if (++stage == p.stages) stage = 0, phase ^= 1u;
    }

    // ---- the warps' sums meet
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float l = sum[m][r];
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l += __shfl_xor_sync(kFull, l, d);
        if (gr == 0) ml[warp * F::kRows + m * 8 + tq * 2 + r] = float2{ref[m][r], l};
      }
    consumers_sync();
    const bool whole = job.whole();
    float* part = piece_of<D>(p, blockIdx.x, off == 0);
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      float f[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float top = kNone;
#pragma unroll
        for (int wq = 0; wq < F::kWarps; ++wq) top = fmaxf(top, ml[wq * F::kRows + m * 8 + tq * 2 + r].x);
        f[r] = ex2(ref[m][r] - top);
      }
#pragma unroll
      for (int hd = 0; hd < D / 64; ++hd) {
        // the sets after another: each adds what the one before left of its block
#pragma unroll
        for (int st = F::kSets - 1; st >= 0; --st) {
          if (set == st) {
#pragma unroll
            for (int ch = 0; ch < 4; ++ch)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const float* ac = acc[m][hd * 4 + ch];
                float2* at = reinterpret_cast<float2*>(join + (blk * 8 + tq * 2 + r) * kJoinStride + ch * 16 + gr * 2);
                float2 x{ac[r] * f[r], ac[2 + r] * f[r]};
                if (st < F::kSets - 1) x.x += at->x, x.y += at->y;
                *at = x;
              }
          }
          consumers_sync();
        }
        if (tid < 256) {
          const int r = tid >> 5, d = lane * 2, row = row0 + m * 8 + r;
          if (row / p.g < job.live) {
            float2 o{0.f, 0.f};
            float top = kNone, l = 0.f;
#pragma unroll
            for (int wq = 0; wq < 8; ++wq) {
              const float2 y = *reinterpret_cast<const float2*>(join + (wq * 8 + r) * kJoinStride + d);
              o.x += y.x, o.y += y.y;
            }
#pragma unroll
            for (int wq = 0; wq < F::kWarps; ++wq) top = fmaxf(top, ml[wq * F::kRows + m * 8 + r].x);
#pragma unroll
            for (int wq = 0; wq < F::kWarps; ++wq) {
              const float2 y = ml[wq * F::kRows + m * 8 + r];
              l += y.y * ex2(y.x - top);
            }
            if (whole) {
              const float inv = 1.f / l;
              T* to = out_row<T>(p, job.b, job.h, row, D) + hd * 64 + d;
              if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(to) = float2{o.x * inv, o.y * inv};
              else *reinterpret_cast<unsigned*>(to) = pack_bf16(o.x * inv, o.y * inv);
            } else {
              float* pr = part + (m * 8 + r) * kPieceRow<D>;
              __stcg(reinterpret_cast<float2*>(pr + 4 + hd * 64 + d), o);
              if (hd == 0 && lane == 0) __stcg(reinterpret_cast<float2*>(pr), float2{top, l});
            }
          }
        }
        consumers_sync();
      }
    }
    if (!whole) {
      // the last piece of the group to arrive adds them all, in order
      __threadfence();
      consumers_sync();
      if (tid == 0) {
        const bool last = atomicAdd(p.s.joins + job.first_block, 1u) == (unsigned)(job.last_block - job.first_block);
        if (last) p.s.joins[job.first_block] = 0;
        *last_s = last;
      }
      consumers_sync();
      if (*last_s) {
        __threadfence();
        join_pieces<T, D, 1, 8>(p, job.b, job.h, row0, job.live, job.first_block, job.last_block, ml, tid, F::kThreads);
      }
    }
    job_done(n);
  }
}

template <typename T, int D, int NT>
cudaError_t launch_few(const State& s, const Attend& a, int sms, cudaStream_t st) {
  using F = Few<T, D, NT>;
  Params p{s, a, s.page_tokens < kTile ? s.page_tokens : kTile, a.heads / s.kv_heads, 0, 0, 0, F::kRows};
  p.rows = a.n * p.g;
  p.row_tiles = (p.rows + F::kRows - 1) / F::kRows;
  const int grid = attend_grid(sms, F::kRows, D);
  p.stages = kStageMax;
  // A stage's tiles all belong to one set: a consumer waits for each of the
  // stage's phases in turn (a wait tells two phases apart, not three).
  static_assert(kStageMax % F::kSets == 0, "stages by sets");
  while (p.stages > 2 && F::smem(p.stages, a.B) > 227 * 1024) p.stages -= F::kSets;
  few_kernel<T, D, NT><<<grid, F::kThreads + 64, F::smem(p.stages, a.B), st>>>(p);
  return cudaGetLastError();
}

template <typename T, int D, int NT>
cudaError_t configure_few() {
  return cudaFuncSetAttribute(few_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
}

}  // namespace

cudaError_t configure() {
  cudaError_t e = configure_few<float, 64, 1>();
  if (e == cudaSuccess) e = configure_few<float, 64, 2>();
  if (e == cudaSuccess) e = configure_few<float, 128, 1>();
  if (e == cudaSuccess) e = configure_few<float, 128, 2>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 64, 1>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 64, 2>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 128, 1>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 128, 2>();
  if (e == cudaSuccess) e = configure_many();
  return e;
}

// Rows of 16-bit queries beyond 16 go to the kernel of mds_cache_many.cu (which
// has no second term for 32-bit queries).  Both kernels, in us: 64 sequences of
// 500 to 2000 tokens with 32 heads, and 8 of 30000 to 60000 with 8:
//    8 rows: here 222, there 228    144, 193
//   16 rows: here 287, there 232    167, 193
//   17 rows: here 509, there 234    296, 193
cudaError_t attend(const State& s, const Attend& a, int sms, cudaStream_t st) {
  const int64_t rows = (int64_t)a.n * (a.heads / s.kv_heads);
  if (s.dtype == MDS_F32) {
    if (s.head_dim == 64) return rows > 8 ? launch_few<float, 64, 2>(s, a, sms, st) : launch_few<float, 64, 1>(s, a, sms, st);
    return rows > 8 ? launch_few<float, 128, 2>(s, a, sms, st) : launch_few<float, 128, 1>(s, a, sms, st);
  }
  if (rows > 16) return attend_many(s, a, sms, st);
  if (s.head_dim == 64)
    return rows > 8 ? launch_few<__nv_bfloat16, 64, 2>(s, a, sms, st) : launch_few<__nv_bfloat16, 64, 1>(s, a, sms, st);
  return rows > 8 ? launch_few<__nv_bfloat16, 128, 2>(s, a, sms, st) : launch_few<__nv_bfloat16, 128, 1>(s, a, sms, st);
}

}  // namespace cache
}  // namespace mds
