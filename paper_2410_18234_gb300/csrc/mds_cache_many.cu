// Attention of draft-tree nodes over the 8-bit paged cache where 17 or more
// rows (nodes x query heads) share a key/value head: trees with shared heads,
// chunks of prompts.  The mathematics is that of mds_cache_few.cu; the
// products run on the tensor cores with their accumulators in tensor memory.
//
// Transposed.  A tile of 128 slots meets up to 144 rows:
//   S^T [128 slots][N rows]  = K [128][D] Q^T          (half precision)
//   O^T [D][N rows]         += V^T [D][128] W^T        (bfloat16)
// The slots and the head's dimensions fill the 128 rows that an instruction
// always has; the attention's rows are its columns (N = 48, 96 or 144): 132
// rows (33 nodes of 4 heads) cost 144 columns, where rows on the other side
// would cost 256.  Four warps widen keys from 8 bits into tensor memory, four
// widen values into shared memory, once for all rows.  Twelve warps turn
// scores into weights, four for each third of the columns.  They read
// fragments of 8 columns in which a thread holds 2 columns of 4 slots: a
// column's running sum stays in registers, sums over slots wait until the
// group ends, and a transposing store packs the weights for the second
// product.
//
// Pipeline, tile t: load K, V (bulk copies) | widen K(t + 1), V(t) | S(t + 1)
// into one of two buffers | weights(t) | O += V(t) W(t).
//
// Bound by the weighing warps, which wait for scores 13 to 20 % of the time
// (clock stamps by role), where the product warp and the widening warps wait
// for 44 to 88 %.  256 sequences of 257 to 1537 tokens, 33 nodes, 32 heads on
// 8: 300 us, 2.1 TB/s of cache and 415 TFLOP/s (626 MB and 125 GFLOP: 92 us at
// HBM's rate), of the weighing warps' time 30 % weights, 13 % votes, 21 %
// masks, references and waits for the weights' buffer, 18 % the ends of groups
// of 8 tiles.  Two prompts' chunks of 1021 tokens behind 4000 to 5000: 249 us,
// 663 TFLOP/s, 36 % weights, 9 % votes, 27 % masks and references, 8 % ends.
// Code size counts here: before waits, schedule and loops were kept short the
// instruction cache missed a third of its requests, and the same work took
// 1.4 times as long.
#include "mds_cache_attend.cuh"

namespace mds {
namespace cache {

namespace {

constexpr int kWeigh = 12;      // warps that weigh, four for each third of the columns
constexpr int kThreads = 32 * (12 + kWeigh);   // keys' loader, products, values' loader, scheduler | 4 widen keys | 4 values | 12 weigh
constexpr int kMaxN = 144;      // columns: three buffers of them and 64 of keys in 512 of tensor memory
constexpr int kRingMax = 5;
constexpr int kScaleRing = 8;   // tiles whose scales are held: kRingMax + 3
// Weights are 2^(score - reference), and sums of floats lose nothing by a
// reference that is not the maximum: it only has to keep them in range, 2^48
// from the top and, so that a weight times a small value stays a normal
// number, not far below 1 where a first reference (0) is judged.
constexpr float kMostWeight = 0x1p48f, kLeastWeight = 0x1p-20f;

enum Bar {
  kKFull = 0, kKEmpty = kKFull + kRingMax, kVFull = kKEmpty + kRingMax, kVEmpty = kVFull + kRingMax,
  kWideK = kVEmpty + kRingMax, kWideKFree, kWideV, kWideVFree = kWideV + 2, kS = kWideVFree + 2, kSFree = kS + 2, kW = kSFree + 2,
  kWFree = kW + 2, kQ = kWFree + 2, kOFree = kQ + 2, kJob, kJobFree = kJob + kJobs, kBars = kJobFree + kJobs
};

// ------------------------------------------------------------------- PTX

__device__ __forceinline__ void tmem_alloc(uint32_t* at) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(at)) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(addr));
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ bool elected() {
  unsigned r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
// Eight columns of 16 lanes: thread l has columns 2 (l % 4), + 1 of lane l / 4 (x, y) and of lane l / 4 + 8.
__device__ __forceinline__ void tmem_ld_frag(float* r, uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0, %1, %2, %3}, [%4];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_st_frag(uint32_t addr, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x1.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(r[0]), "f"(r[1]),
               "f"(r[2]), "f"(r[3])
               : "memory");
}
__device__ __forceinline__ void tmem_ld_row8(float* r, uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_st_row16(uint32_t addr, const unsigned* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// The loaded registers are read after the wait.
__device__ __forceinline__ void tmem_ld_wait(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7])::"memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void stmatrix_x4_trans(unsigned addr, const unsigned* r) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void third_sync(int third) { asm volatile("bar.sync %0, 128;" ::"r"(1 + third) : "memory"); }
__device__ __forceinline__ bool third_any(int third, bool x) {
  unsigned r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(1 + third), "r"((unsigned)x)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void weigh_sync() { asm volatile("bar.sync 4, 384;" ::: "memory"); }

// Shared-memory operands: rows of 128 bytes, their 16-byte units permuted
// (unit ^= row mod 8); `lead` is the distance of blocks of 64 elements along
// the contiguous axis where that axis is the operand's rows, 8 rows are 1024 bytes.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | 1ull << 46 |
         2ull << 61;
}
// 32-bit sums; M = 128; type 0 half, 1 bfloat16; rows_first: A's contiguous axis is its rows.
__device__ __forceinline__ uint32_t instruction(int n, uint32_t type, uint32_t rows_first) {
  return 1u << 4 | type << 7 | type << 10 | rows_first << 15 | (uint32_t)(n >> 3) << 17 | 8u << 24;
}

struct Row {
  int own, depth;   // its branch's first node; nodes of the branch that it sees: its depth
  int64_t out;      // its output's first element, -1: not one of the call's
};

// Buffers of wide values: two where they leave room for the rings.
__host__ __device__ constexpr int wide_buffers(int N) { return N <= 96 ? 2 : 1; }

// Shared memory from a 1024-byte boundary on.
struct Layout {
  int q, w, wide_v, k_ring, v_ring, small, bytes;
  int nk, nv;
};
__host__ __device__ inline Layout layout_of(int D, int N, int B) {
  Layout l;
  l.q = 0;
  l.w = l.q + N * D * 2;
  l.wide_v = l.w + 2 * N * 256;
  l.k_ring = l.wide_v + wide_buffers(N) * 128 * D * 2;
  const int small = kScaleRing * 16 * 4 + N * (2 * 16 + 8 + 2 * 8 + 8 + 24) + (kBars + 1) / 2 * 16 + kJobs * (int)sizeof(Job) + 16 + B * 16;
  const int room = 227 * 1024 - 1024 - l.k_ring - small;
  const int slots = room / (kTile * D);
  l.nk = slots / 2 < kRingMax ? slots / 2 : kRingMax;
  l.nv = slots - l.nk < kRingMax ? slots - l.nk : kRingMax;
  l.v_ring = l.k_ring + l.nk * kTile * D;
  l.small = l.v_ring + l.nv * kTile * D;
  l.bytes = 1024 + l.small + small;
  return l;
}

// kSteps: fragments of 8 columns in a third of them
template <int D, int kSteps>
__global__ void __launch_bounds__(kThreads, 1) many_kernel(const __grid_constant__ Params p) {
  constexpr int N = 24 * kSteps, NC = 8 * kSteps;   // columns, a third of them
  constexpr int kWide = wide_buffers(N);
  extern __shared__ char raw[];
  char* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const Layout lay = layout_of(D, N, p.a.B);
  char* at = base + lay.small;
  float* k_scales = reinterpret_cast<float*>(at);          // [kScaleRing][8], by tile
  at += kScaleRing * 8 * 4;
  float* v_scales = reinterpret_cast<float*>(at);          // [kRingMax][8], by the ring's slot
  at += kScaleRing * 8 * 4;
  Row* row_info = reinterpret_cast<Row*>(at);              // [2][N], by group
  at += 2 * N * 16;
  Seq* seqs = reinterpret_cast<Seq*>(at);
  at += p.a.B * 16;
  float2* stat = reinterpret_cast<float2*>(at);            // at the group's end: reference, normaliser
  at += N * 8;
  uint64_t* bar = reinterpret_cast<uint64_t*>(at);
  at += (kBars + 1) / 2 * 16;
  float4* col_info = reinterpret_cast<float4*>(at);        // [2][N / 2]: two columns' coefficients, and references negated
  at += 2 * N * 8;
  int64_t* q_at = reinterpret_cast<int64_t*>(at);          // [N]: a row's query, from the sequence's first
  at += N * 8;
  float* red = reinterpret_cast<float*>(at);               // [4][N]: a column's maximum, later sum, by each warp
  float* next = red + 4 * N;                               // [2][N]: references negated, factors of the sums
  at += 6 * N * 4;
  Job* jobs = reinterpret_cast<Job*>(at);
  at += kJobs * sizeof(Job);
  int* abort = reinterpret_cast<int*>(at);
  int* last_s = abort + 1;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(abort + 2);
  long long* prefix = reinterpret_cast<long long*>(base);  // before the queries and weights

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    *abort = 0;
    for (int i = 0; i < kRingMax; ++i) {
      mbar_init(bar + kKFull + i, 1 + 32);   // the loader's byte count, and its lanes' scale copies
      mbar_init(bar + kKEmpty + i, 4);
      mbar_init(bar + kVFull + i, 1 + 32);
      mbar_init(bar + kVEmpty + i, 4);
    }
    mbar_init(bar + kWideK, 4);
    mbar_init(bar + kWideKFree, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar + kWideV + i, 4);
      mbar_init(bar + kWideVFree + i, 1);
      mbar_init(bar + kS + i, 1);
      mbar_init(bar + kSFree + i, kWeigh);
      mbar_init(bar + kW + i, kWeigh);
      mbar_init(bar + kWFree + i, 1);
    }
    mbar_init(bar + kQ, 4);
    mbar_init(bar + kQ + 1, 4);
    mbar_init(bar + kOFree, kWeigh);
    for (int i = 0; i < kJobs; ++i) {
      mbar_init(bar + kJob + i, 1);
      mbar_init(bar + kJobFree + i, 11 + kWeigh);   // every warp but the scheduler's
    }
    mbar_init_fence();
  }
  plan<__nv_bfloat16>(p, prefix, seqs, D);   // ends in a barrier
  const long long total = prefix[p.a.B];
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  const long long u0 = per * blockIdx.x, u1 = min(u0 + per, total);
  if (u0 >= u1) return;
  Cursor c{0, 0, 0, 0};
  if (warp == 3) c = locate(p, prefix, seqs, u0);
  if (warp == 2) tmem_alloc(tmem_at);
  before_sync();
  __syncthreads();   // the plan's sums have been read
  after_sync();
  const uint32_t tmem = *tmem_at;
  const uint32_t t_s = tmem, t_o = tmem + 2 * N, t_k = tmem + 3 * N;
  auto hold = [&](int b, unsigned parity) { wait(bar + b, parity, abort); };
  // a role takes the jobs in turn
  auto job_at = [&](int n) -> const Job& {
    hold(kJob + (n & (kJobs - 1)), (n / kJobs) & 1);
    return jobs[n & (kJobs - 1)];
  };
  auto job_done = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar + kJobFree + (n & (kJobs - 1)));
  };

  if (warp == 3) {
    schedule(p, seqs, c, per, u0, u1, jobs, bar + kJob, bar + kJobFree, abort);
  } else if (warp == 0 || warp == 2) {
    // ---- loaders, of keys and of values: one block of 16 slots a lane (0..7);
    // the first of a page's blocks copies for all of them
    const State& s = p.s;
    const int kv = warp >> 1, blk = lane & 7, slots = kv ? lay.nv : lay.nk;
    char* ring = base + (kv ? lay.v_ring : lay.k_ring);
    const int full = kv ? kVFull : kKFull, empty = kv ? kVEmpty : kKEmpty;
    const int64_t layer0 = (int64_t)p.a.layer * s.pages;
    int tile = 0, slot = 0;
    unsigned parity = 1;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      const int end = job.off + job.cnt, h = job.h;
      if (!job.cnt) break;
      const Group grp = job.grp;
      const int32_t* table = s.table + (int64_t)job.q * s.max_pages;
      auto page_of = [&](int i) {
        const int t = (tile_slot(grp, i) + blk * kBlock) & -p.span;
        return lane < 8 && i < end && block_seen(grp, t, p.span) ? __ldg(table + (t >> s.page_log)) : -1;
      };
      const int off = job.off;
      int page = page_of(off);
      if (kv) {   // the queries are read by the time that the group's first tile is here
        for (int r = lane; r < p.rows_per; r += 32) {
          const int row = job.row0 + r, node = row / p.g;
          if (node < job.live) {
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.a.q) + job.b * p.a.q_seq + node * p.a.q_tok +
                                     (h * p.g + row - node * p.g) * p.a.q_head;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(q));
            if (D == 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + 64));
          }
        }
      }
      job_done(n);
      for (int i = off; i < end; ++i, ++tile) {
        const int next = page_of(i + 1);
        const int r = (tile_slot(grp, i) + blk * kBlock) & (s.page_tokens - 1);
        const bool copies = page >= 0 && ((blk * kBlock) & (p.span - 1)) == 0;   // the first block of its span
        const unsigned takes = __ballot_sync(kFull, copies);
        const int64_t row = (((layer0 + page) * 2 + kv) * s.kv_heads + h) * s.page_tokens + r;
        hold(empty + slot, parity);
        if (lane == 0) mbar_expect_tx(bar + full + slot, __popc(takes) * p.span * D);
        __syncwarp();
        if (page >= 0) {
          if (copies) bulk_copy(ring + (slot * kTile + blk * kBlock) * D, s.pool + row * D, p.span * D, bar + full + slot);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(
                           smem_u32(kv ? v_scales + slot * 8 + blk : k_scales + (tile & (kScaleRing - 1)) * 8 + blk)),
                       "l"(s.scales + (row >> 4))
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar + full + slot))
                     : "memory");
        page = next;
        if (++slot == slots) slot = 0, parity ^= 1u;
      }
    }
    report(abort, s.status);
  } else if (warp == 1) {
    // ---- products, issued by one thread: S(t + 1) before O(t)
    const uint32_t id_s = instruction(N, 0, 0), id_o = instruction(N, 1, 1);
    const uint64_t q_op = operand(smem_u32(base + lay.q), 16), v_op = operand(smem_u32(base + lay.wide_v), 16384);
    const uint64_t w_op = operand(smem_u32(base + lay.w), 16);
    int tile = 0, group = 0;
    auto out_product = [&](int t, bool first) {
      hold(kW + (t & 1), (t >> 1) & 1);
      const int wide = t & (kWide - 1);
      hold(kWideV + wide, (t / kWide) & 1);
      if (first) hold(kOFree, (group & 1) ^ 1);
      after_sync();
      if (elected()) {
        const uint64_t v = v_op + (wide * (128 * D * 2) >> 4);
        const uint64_t w = w_op + ((t & 1) * N * 256 >> 4);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)   // 16 slots: 2048 bytes of V, 32 of a row of weights
          mma_ss(t_o, v + k * (2048 >> 4), w + (((k >> 2) * N * 128 + (k & 3) * 32) >> 4), id_o, !(first && k == 0));
        commit_to(bar + kWFree + (t & 1));
        commit_to(bar + kWideVFree + wide);
      }
      __syncwarp();
    };
    for (;;) {
      const int cnt = job_at(group).cnt;
      if (!cnt) break;
      job_done(group);
      hold(kQ + (group & 1), (group >> 1) & 1);
      for (int i = 0; i < cnt; ++i, ++tile) {
        hold(kWideK, tile & 1);
        hold(kSFree + (tile & 1), ((tile >> 1) & 1) ^ 1);
        after_sync();
        if (elected()) {
          const uint32_t to = t_s + (tile & 1) * N;
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            mma_ts(to, t_k + k * 8, q_op + (((k >> 2) * N * 128 + (k & 3) * 32) >> 4), id_s, k > 0);
          commit_to(bar + kS + (tile & 1));
          commit_to(bar + kWideKFree);
        }
        __syncwarp();
        if (i > 0) out_product(tile - 1, i == 1);
      }
      out_product(tile - 1, cnt == 1);
      ++group;
    }
  } else if (warp >= 4 && warp < 8) {
    // ---- widen keys, a row a thread, into tensor memory; and the groups'
    // queries.  Rows of blocks that were not loaded hold anything: their
    // scores are masked.
    const int w4 = warp & 3, key = w4 * 32 + lane;
    int ks = 0;
    unsigned kp = 0;
    const uint32_t k_to = t_k + ((uint32_t)(w4 * 32) << 16);
    auto keys = [&](int t) {
      hold(kKFull + ks, kp);
      hold(kWideKFree, (t & 1) ^ 1);
      after_sync();
      const char* src = base + lay.k_ring + ks * kTile * D;
#pragma unroll 1
      for (int i = 0; i < D / 32; ++i) {
        unsigned x[16];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 y = *reinterpret_cast<const uint4*>(src + swizzled(key * D + (2 * i + j) * 16));
          to_f16(y.x, x[8 * j], x[8 * j + 1]);
          to_f16(y.y, x[8 * j + 2], x[8 * j + 3]);
          to_f16(y.z, x[8 * j + 4], x[8 * j + 5]);
          to_f16(y.w, x[8 * j + 6], x[8 * j + 7]);
        }
        tmem_st_row16(k_to + i * 16, x);
      }
      tmem_st_wait();
      before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar + kKEmpty + ks);
        mbar_arrive(bar + kWideK);
      }
      if (++ks == lay.nk) ks = 0, kp ^= 1u;
    };
    // a group's queries, scaled to half precision, rows of 128 bytes; and what
    // its rows are.  The products of the group before have read its queries,
    // every warp is done with what the rows of the group before that were.
    auto queries = [&](int n, const Job& job) {
      const int wt = tid - 128;
      Row* rows = row_info + (n & 1) * N;
      float4* cr = col_info + (n & 1) * (N / 2);
      const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.a.q) + job.b * p.a.q_seq;
      asm volatile("bar.sync 5, 128;" ::: "memory");
      for (int r = wt; r < N; r += 128) {
        const int row = job.row0 + r, node = row / p.g, head = job.h * p.g + row - node * p.g;
        const bool live = r < p.rows_per && node < job.live;
        const int own = node > 0 && p.a.L > 0 ? 1 + (node - 1) / p.a.L * p.a.L : 1;
        rows[r] = Row{own, node > 0 ? node - own + 1 : 0,
                      live ? (((int64_t)job.b * p.a.n + node) * p.a.heads + head) * D : -1};
        q_at[r] = live ? node * p.a.q_tok + head * p.a.q_head : -1;
      }
      asm volatile("bar.sync 5, 128;" ::: "memory");
      // each warp copies its rows (16 bytes a lane), then scales them in place
      constexpr int kUnits = D / 8, kAtOnce = 32 / kUnits;
      char* to = base + lay.q;
      for (int r0 = w4 * kAtOnce; r0 < N; r0 += 4 * kAtOnce) {
        const int r = r0 + lane / kUnits, unit = lane % kUnits;
        const int64_t from = q_at[r];
        char* dst = to + (unit >> 3) * N * 128 + r * 128 + (((unit & 7) ^ (r & 7)) << 4);
        if (from >= 0)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(q + from + unit * 8) : "memory");
        else
          *reinterpret_cast<uint4*>(dst) = uint4{0, 0, 0, 0};
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
#pragma unroll 2
      for (int r0 = w4 * kAtOnce; r0 < N; r0 += 4 * kAtOnce) {
        const int r = r0 + lane / kUnits, unit = lane % kUnits;
        uint4* at_lane = reinterpret_cast<uint4*>(to + (unit >> 3) * N * 128 + r * 128 + (((unit & 7) ^ (r & 7)) << 4));
        const uint4 y = *at_lane;
        const unsigned w[4] = {y.x, y.y, y.z, y.w};
        unsigned bits = 0;   // the largest magnitude: bfloat16 order as their bits do
#pragma unroll
        for (int i = 0; i < 4; ++i) bits = max(bits, max(w[i] << 16 & 0x7fff0000u, w[i] & 0x7fff0000u));
#pragma unroll
        for (int d = 1; d < kUnits; d *= 2) bits = max(bits, __shfl_xor_sync(kFull, bits, d));
        const int e = bits == 0 || bits >= 0x7f800000u ? 0 : max((int)(bits >> 23) - 127 - 14, -112);
        // the coefficient is not negative, so that a masked -inf stays one: the
        // scale's sign, or 0, goes to the queries
        const float inv = p.a.scale == 0.f ? 0.f : copysignf(__uint_as_float((unsigned)(127 - e) << 23), p.a.scale);
        unsigned v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __half2 a = __floats2half2_rn(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
          v[i] = *reinterpret_cast<const unsigned*>(&a);
        }
        *at_lane = uint4{v[0], v[1], v[2], v[3]};
        if (unit == 0) {
          float* at_cr = reinterpret_cast<float*>(cr + (r >> 1)) + (r & 1);
          const float k = fabsf(p.a.scale) * dev::kLog2e * __uint_as_float((unsigned)(127 + e) << 23);
          at_cr[0] = p.a.scale == 0.f ? 1.f : k;
          at_cr[2] = 0.f;
        }
      }
      dev::fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + kQ + (n & 1));
    };
    int tile = 0;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      if (!job.cnt) break;
      const int cnt = job.cnt;
      hold(kWideKFree, (tile & 1) ^ 1);
      if (n > 1) hold(kJobFree + ((n - 2) & (kJobs - 1)), ((n - 2) / kJobs) & 1);
      queries(n, job);
      job_done(n);
      for (int i = 0; i < cnt; ++i, ++tile) keys(tile);
    }
  } else if (warp >= 8 && warp < 12) {
    // ---- widen values, 16 dimensions of a slot at a time, into shared memory.
    // Rows of blocks that were not loaded become zeros.
    const int w4 = warp & 3;
    int vs = 0;
    unsigned vp = 0;
    // seen: bit i of the tile's blocks (two a warp)
    auto values = [&](int t, unsigned seen) {
      hold(kVFull + vs, vp);
      const int wide = t & (kWide - 1);
      hold(kWideVFree + wide, ((t / kWide) & 1) ^ 1);
      const float* sc = v_scales + vs * 8 + w4 * 2;
      // a block that was not loaded holds anything: times 0
      unsigned rest[2], factor[2];
      bool large = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool in = seen >> (w4 * 2 + i) & 1u;
        factor[i] = in ? value_factor(sc[i], rest[i]) : 0u;
        if (!in) rest[i] = 0x3f803f80u;
        large = large || rest[i] != 0x3f803f80u;
      }
      const char* src = base + lay.v_ring + vs * kTile * D;
      char* dst = base + lay.wide_v + wide * (128 * D * 2);
      constexpr int kChunks = D / 16;
#pragma unroll 1
      for (int i0 = 0; i0 < kChunks; i0 += 4) {
        uint4 y[4];   // read before anything is written: nothing to order between the rows
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int octet = (i0 + i) * 4 / kChunks, chunk = ((i0 + i) * 4 + (lane >> 3)) % kChunks;
          y[i] = *reinterpret_cast<const uint4*>(src + swizzled((w4 * 32 + octet * 8 + (lane & 7)) * D + chunk * 16));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // the same eight slots for all lanes, so one of the warp's two blocks
          const int octet = (i0 + i) * 4 / kChunks, chunk = ((i0 + i) * 4 + (lane >> 3)) % kChunks;
          const int k = w4 * 32 + octet * 8 + (lane & 7);
          const unsigned f = octet & 2 ? factor[1] : factor[0];
          uint4 a, b;   // of every four dimensions the order is 0, 2, 1, 3
          to_bf16(y[i].x, f, a.x, a.y);
          to_bf16(y[i].y, f, a.z, a.w);
          to_bf16(y[i].z, f, b.x, b.y);
          to_bf16(y[i].w, f, b.z, b.w);
          if (large) {
            const unsigned g = octet & 2 ? rest[1] : rest[0];
            times_rest(a.x, g), times_rest(a.y, g), times_rest(a.z, g), times_rest(a.w, g);
            times_rest(b.x, g), times_rest(b.y, g), times_rest(b.z, g), times_rest(b.w, g);
          }
          char* line = dst + (chunk >> 2) * 16384 + k * 128;
          *reinterpret_cast<uint4*>(line + ((((chunk & 3) * 2) ^ (k & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(line + ((((chunk & 3) * 2 + 1) ^ (k & 7)) << 4)) = b;
        }
      }
      dev::fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar + kVEmpty + vs);
        mbar_arrive(bar + kWideV + wide);
      }
      if (++vs == lay.nv) vs = 0, vp ^= 1u;
    };
    int tile = 0;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      if (!job.cnt) break;
      const Group grp = job.grp;
      const int off = job.off, end = off + job.cnt;
      job_done(n);
      for (int i = off; i < end; ++i, ++tile)
        values(tile, __ballot_sync(kFull, block_seen(grp, tile_slot(grp, i) + (lane & 7) * kBlock)) & 0xffu);
    }
  } else if (warp >= 12) {
    // ---- weigh: a third of the columns, a quarter of the slots a warp
    const int third = (warp - 12) >> 2, w4 = warp & 3, tq = lane & 3, gr = lane >> 2;
    const int ht = tid - 384, col0 = third * NC;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    // where this lane's rows of a transposed fragment go: slots w4 * 32 + (lane / 8) * 8 .. + 7, columns + lane % 8
    const uint32_t w_to = smem_u32(base + lay.w) + (uint32_t)((w4 >> 1) * N * 128 + (col0 + (lane & 7)) * 128 +
                                                             ((((w4 & 1) * 4 + (lane >> 3)) ^ (lane & 7)) << 4));
    int tile = 0, group = 0;
    for (;;) {
      const Job& job = job_at(group);
      if (!job.cnt) break;
      const int row0 = job.row0;
      const Row* rows = row_info + (group & 1) * N;
      float4* cr = col_info + (group & 1) * (N / 2);
      hold(kQ + (group & 1), (group >> 1) & 1);   // rows and coefficients
      float2 sum[kSteps];
      float4* my_cr = cr + col0 / 2 + tq;   // step j's are 4 j further
      unsigned unseen = (1u << (2 * kSteps)) - 1u;   // this thread's columns that have no reference yet
      bool pending = true;                          // some column of the third has none
#pragma unroll
      for (int j = 0; j < kSteps; ++j) sum[j] = float2{0.f, 0.f};
      const Group grp = job.grp;
      const int off = job.off, end = off + job.cnt, len = job.len;
      for (int i = off; i < end; ++i, ++tile) {
        const int kb = tile_slot(grp, i) + w4 * 32;
        const int b = tile & 1;
        hold(kS + b, (tile >> 1) & 1);
        after_sync();
        const float* sc = k_scales + (tile & (kScaleRing - 1)) * 8 + w4 * 2;
        const bool seen0 = block_seen(grp, kb), seen1 = block_seen(grp, kb + kBlock);
        const float ks0 = seen0 ? sc[0] : 1.f, ks1 = seen1 ? sc[1] : 1.f;
        const uint32_t s_at = t_s + b * N + col0 + lanes;
        // 8 columns: x[2 k], x[2 k + 1] of slot kb + 8 k + gr
        auto load = [&](int j, float* x) {
          tmem_ld_frag(x, s_at + j * 8);
          tmem_ld_frag(x + 4, s_at + j * 8 + (16u << 16));
        };
        // Scores in log2 units, rounded before a reference is taken from them:
        // the reference is the largest of these numbers, so that no weight
        // beside it passes 1 however large the scores are.  A fused product
        // would leave its rounding in the exponent: beyond 2^6 for scores of
        // 2^30.
        auto scores = [&](int j, float* x) {
          const float4 y4 = my_cr[4 * j];
          // never 0, so that a masked -inf stays one; what 2^-120 adds to a score is below 2^-88
          const float2 tiny{0x1p-120f, 0x1p-120f}, c0 = fma2(float2{y4.x, y4.y}, float2{ks0, ks0}, tiny),
                       c1 = fma2(float2{y4.x, y4.y}, float2{ks1, ks1}, tiny);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 y = mul2(float2{x[2 * k], x[2 * k + 1]}, k < 2 ? c0 : c1);
            x[2 * k] = y.x;
            x[2 * k + 1] = y.y;
          }
          return float2{y4.z, y4.w};   // the references, negated
        };
        if (kb + 32 > len || (p.a.window > 0 && kb + 32 > p.a.sinks && kb <= len + min(p.a.L, p.a.n - 1) - p.a.window)) {
          // some slot is masked for some row: -inf in its place.  Dead columns
          // get zeros, whatever the slots that were not loaded hold.
#pragma unroll 2
          for (int j = 0; j < kSteps; ++j) {
            float x[8];
            load(j, x);
            tmem_ld_wait(x);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const Row row = rows[col0 + j * 8 + tq * 2 + e];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int t = kb + k * 8 + gr, up = t - len - row.own;   // nodes up its branch
                bool see = t <= len || (unsigned)up < (unsigned)row.depth;
                if (p.a.window > 0) {
                  const int pos = t <= len ? t : len + up + 1;
                  see = see && (pos < p.a.sinks || pos > len + row.depth - p.a.window);
                }
                see = see && t < grp.hi;
                x[2 * k + e] = row.out < 0 ? 0.f : see ? x[2 * k + e] : dev::kNegInf;
              }
            }
            tmem_st_frag(s_at + j * 8, x);
            tmem_st_frag(s_at + j * 8 + (16u << 16), x + 4);
          }
          tmem_st_wait();
        }
        // Weights first with the references as they are (0 before the first);
        // only where that gives a weight too large, or none that a first
        // reference could be judged by, the columns' maxima over the tile's
        // slots become the references, and the tile is weighed once more: two
        // passes at most.
        float2 part[kSteps];
        bool move = false, left = false;
        for (;;) {
          if (move) {
#pragma unroll 1
            for (int j = 0; j < kSteps; ++j) {
              float x[8];
              load(j, x);
              tmem_ld_wait(x);
              scores(j, x);
              float2 m{fmaxf(fmaxf(x[0], x[2]), fmaxf(x[4], x[6])), fmaxf(fmaxf(x[1], x[3]), fmaxf(x[5], x[7]))};
#pragma unroll
              for (int d = 4; d < 32; d *= 2) {
                m.x = fmaxf(m.x, __shfl_xor_sync(kFull, m.x, d));
                m.y = fmaxf(m.y, __shfl_xor_sync(kFull, m.y, d));
              }
              if (gr == 0) *reinterpret_cast<float2*>(red + w4 * N + col0 + j * 8 + tq * 2) = m;
            }
            third_sync(third);
            const bool again = i != off;
            if (again) {   // the sums so far follow: O of the tiles before is complete
              hold(kWFree + (b ^ 1), ((tile - 1) >> 1) & 1);
              after_sync();
            }
#pragma unroll 1
            for (int j = 0; j < kSteps; ++j) {
              const int col = col0 + j * 8 + tq * 2;
              float2 m{kNone, kNone};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 y = *reinterpret_cast<const float2*>(red + k * N + col);
                m.x = fmaxf(m.x, y.x);
                m.y = fmaxf(m.y, y.y);
              }
              // a reference only moves up; a column that had none takes the maximum
              const float4 y4 = my_cr[4 * j];
              float2 now{fmaxf(m.x, -y4.z), fmaxf(m.y, -y4.w)};
              if (unseen >> (2 * j) & 1u) {
                now.x = m.x > kNone ? m.x : 0.f;
                if (m.x > kNone) unseen &= ~(1u << (2 * j));
              }
              if (unseen >> (2 * j) & 2u) {
                now.y = m.y > kNone ? m.y : 0.f;
                if (m.y > kNone) unseen &= ~(2u << (2 * j));
              }
              // a first reference below 0 finds sums of 0
              const float2 alpha{ex2(fminf(-y4.z - now.x, 0.f)), ex2(fminf(-y4.w - now.y, 0.f))};
              if (again) {
                float x[8];
                const uint32_t o_at = t_o + col0 + j * 8 + lanes;
                tmem_ld_frag(x, o_at);
                tmem_ld_frag(x + 4, o_at + (16u << 16));
                tmem_ld_wait(x);
#pragma unroll
                for (int k = 0; k < 8; k += 2) x[k] *= alpha.x, x[k + 1] *= alpha.y;
                tmem_st_frag(o_at, x);
                tmem_st_frag(o_at + (16u << 16), x + 4);
              }
              if (w4 == 0 && gr == 0) {
                *reinterpret_cast<float2*>(next + col) = float2{-now.x, -now.y};
                *reinterpret_cast<float2*>(next + N + col) = alpha;
              }
            }
            if (again) {
              tmem_st_wait();
              before_sync();
            }
            left = third_any(third, unseen != 0);   // and every thread has read the old references
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
              {
                const float2 alpha = *reinterpret_cast<const float2*>(next + N + col0 + j * 8 + tq * 2);
                sum[j].x *= alpha.x;
                sum[j].y *= alpha.y;
              }
            if ((ht & 127) < NC) {
              const int col = col0 + (ht & 127);
              reinterpret_cast<float*>(cr + (col >> 1))[2 + (col & 1)] = next[col];
            }
            third_sync(third);
          }
          hold(kWFree + b, ((tile >> 1) & 1) ^ 1);
          // two steps of fragments are weighed while the next two are loaded
          float x[2][2][8];
          load(0, x[0][0]);
          load(1, x[0][1]);
#pragma unroll
          for (int j0 = 0; j0 < kSteps; j0 += 2)
            {
              float (*now)[8] = x[(j0 >> 1) & 1], (*ahead)[8] = x[((j0 >> 1) & 1) ^ 1];
              tmem_ld_wait(now[0]);
              tmem_ld_wait(now[1]);
              if (j0 + 2 < kSteps) {
                load(j0 + 2, ahead[0]);
                load(j0 + 3, ahead[1]);
              }
#pragma unroll
              for (int j = 0; j < 2; ++j)
                {
                  float* y = now[j];
                  const float2 less = scores(j0 + j, y);
                  unsigned w[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    const float2 z = fma2(float2{y[2 * k], y[2 * k + 1]}, float2{p.one, p.one}, less);
                    w[k] = pack_bf16(ex2(z.x), ex2(z.y));
                    const float2 e{__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u)};
                    part[j0 + j] = k ? add2(part[j0 + j], e) : e;
                  }
                  stmatrix_x4_trans(w_to + b * N * 256 + (j0 + j) * 1024, w);
                }
            }
          // too large a weight for the reference, or (a first reference) too
          // small ones: this thread's four of a column together
          float top = 0.f, low = 1.f;
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
            top = max3(top, part[j].x, part[j].y);
          if (pending && !move) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
              {
                if (unseen >> (2 * j) & 1u) low = fminf(low, part[j].x);
                if (unseen >> (2 * j) & 2u) low = fminf(low, part[j].y);
              }
          }
          if (move || !third_any(third, top > kMostWeight || low < kLeastWeight)) break;
          move = true;
        }
        pending = pending && left;
        if (!pending) unseen = 0;
        before_sync();
        dev::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar + kSFree + b);
          mbar_arrive(bar + kW + b);
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
          sum[j] = add2(sum[j], part[j]);
      }

      // ---- the group's or piece's end: normalisers, then O
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
        {
          float2 s = sum[j];
#pragma unroll
          for (int d = 4; d < 32; d *= 2) {
            s.x += __shfl_xor_sync(kFull, s.x, d);
            s.y += __shfl_xor_sync(kFull, s.y, d);
          }
          if (gr == 0) {
            *reinterpret_cast<float2*>(red + w4 * N + col0 + j * 8 + tq * 2) = s;
            if (w4 == 0) {
              stat[col0 + j * 8 + tq * 2].x = unseen >> (2 * j) & 1u ? kNone : -my_cr[4 * j].z;
              stat[col0 + j * 8 + tq * 2 + 1].x = unseen >> (2 * j) & 2u ? kNone : -my_cr[4 * j].w;
            }
          }
        }
      third_sync(third);
      const int at_half = ht & 127;
      if (at_half < NC) {
        const int col = col0 + at_half;
        const float l = (red[col] + red[N + col]) + (red[2 * N + col] + red[3 * N + col]);
        stat[col].y = job.whole() ? 1.f / l : l;
      }
      third_sync(third);
      const bool whole = job.whole();
      float* piece = piece_of<D>(p, blockIdx.x, off == 0);
      hold(kWFree + ((tile - 1) & 1), ((tile - 1) >> 1) & 1);
      after_sync();
      if (whole) {
        // O to bfloat16 rows in the weights' place (transposed like them), then out
        char* stage = base + lay.w;
        if (w4 * 32 < D) {
          const uint32_t to = smem_u32(stage) + (col0 + (lane & 7)) * D * 2 +
                              (((w4 * 4 + (lane >> 3)) ^ (lane & 7)) << 4);
#pragma unroll 1
          for (int j = 0; j < kSteps; ++j) {
            float x[8];
            const uint32_t o_at = t_o + col0 + j * 8 + lanes;
            tmem_ld_frag(x, o_at);
            tmem_ld_frag(x + 4, o_at + (16u << 16));
            const float inv0 = stat[col0 + j * 8 + tq * 2].y, inv1 = stat[col0 + j * 8 + tq * 2 + 1].y;
            tmem_ld_wait(x);
            unsigned w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack_bf16(x[2 * k] * inv0, x[2 * k + 1] * inv1);
            stmatrix_x4_trans(to + j * 8 * D * 2, w);
          }
        }
        before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + kOFree);
        third_sync(third);
        constexpr int kUnits = D / 8;   // of 16 bytes a row
#pragma unroll 1
        for (int x = ht & 127; x < NC * kUnits; x += 128) {
          const int col = col0 + x / kUnits, unit = x % kUnits;
          const int64_t to = rows[col].out;
          if (to < 0) continue;
          const uint4 y = *reinterpret_cast<const uint4*>(stage + col * D * 2 + ((unit ^ (col & 7)) << 4));
          // of every four dimensions the order is 0, 2, 1, 3
          *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.a.out) + to + unit * 8) =
              uint4{__byte_perm(y.x, y.y, 0x5410), __byte_perm(y.x, y.y, 0x7632), __byte_perm(y.z, y.w, 0x5410),
                    __byte_perm(y.z, y.w, 0x7632)};
        }
      } else {
        if (w4 * 32 < D) {
          const int m = w4 * 32 + lane, dim = (m & ~3) | (m & 1) << 1 | (m >> 1 & 1);
#pragma unroll 1
          for (int j = 0; j < kSteps; ++j) {
            float x[8];
            tmem_ld_row8(x, t_o + col0 + j * 8 + lanes);
            tmem_ld_wait(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int col = col0 + j * 8 + e;
              if (rows[col].out < 0) continue;
              __stcg(piece + col * kPieceRow<D> + 4 + dim, x[e]);
              if (m == 0) __stcg(reinterpret_cast<float2*>(piece + col * kPieceRow<D>), stat[col]);
            }
          }
        }
        before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + kOFree);
      }
      if (!whole) {
        // the last piece of the group to arrive adds them all, in order
        __threadfence();
        weigh_sync();
        if (ht == 0) {
          const bool last = atomicAdd(p.s.joins + job.first_block, 1u) == (unsigned)(job.last_block - job.first_block);
          if (last) p.s.joins[job.first_block] = 0;
          *last_s = last;
        }
        weigh_sync();
        if (*last_s) {
          __threadfence();
          join_pieces<__nv_bfloat16, D, 4, 2>(p, job.b, job.h, row0, job.live, job.first_block, job.last_block, stat, ht, 32 * kWeigh);
        }
      }
      weigh_sync();   // the weights' place and stat have been read
      job_done(group);
      ++group;
    }
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == 2) tmem_free(tmem);
}

template <int D, int kSteps>
cudaError_t launch_many(const Params& p, int sms, cudaStream_t st) {
  const Layout l = layout_of(D, 24 * kSteps, p.a.B);
  const int grid = attend_grid(sms, p.rows_per, D);
  many_kernel<D, kSteps><<<grid, kThreads, l.bytes, st>>>(p);
  return cudaGetLastError();
}
template <int D, int kSteps>
cudaError_t configure_one() {
  return cudaFuncSetAttribute(many_kernel<D, kSteps>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
}

}  // namespace

cudaError_t configure_many() {
  cudaError_t e = configure_one<64, 2>();
  if (e == cudaSuccess) e = configure_one<64, 4>();
  if (e == cudaSuccess) e = configure_one<64, 6>();
  if (e == cudaSuccess) e = configure_one<128, 2>();
  if (e == cudaSuccess) e = configure_one<128, 4>();
  if (e == cudaSuccess) e = configure_one<128, 6>();
  return e;
}

cudaError_t attend_many(const State& s, const Attend& a, int sms, cudaStream_t st) {
  Params p{s, a, s.page_tokens < kTile ? s.page_tokens : kTile, a.heads / s.kv_heads, 0, 0, 0, 0};
  p.rows = a.n * p.g;
  p.row_tiles = (p.rows + kMaxN - 1) / kMaxN;
  p.rows_per = (p.rows + p.row_tiles - 1) / p.row_tiles;
  if (s.head_dim == 64)
    return p.rows_per <= 48 ? launch_many<64, 2>(p, sms, st) : p.rows_per <= 96 ? launch_many<64, 4>(p, sms, st) : launch_many<64, 6>(p, sms, st);
  return p.rows_per <= 48 ? launch_many<128, 2>(p, sms, st) : p.rows_per <= 96 ? launch_many<128, 4>(p, sms, st) : launch_many<128, 6>(p, sms, st);
}

}  // namespace cache
}  // namespace mds
