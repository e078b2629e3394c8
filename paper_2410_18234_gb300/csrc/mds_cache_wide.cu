// Attention over a shared prefix where many rows read it: the group's rows are
// the instructions' rows, two halves of up to 128 of them at a time.
//
//   S_h [128 rows][128 slots] = Q_h K^T     (half precision)
//   P_h = 2^(c S_h - m)                     (bfloat16)
//   O_h [128 rows][D]        += P_h V       (bfloat16)
//
// Nothing of a prefix is masked, so a row's weights are two threads' (64 slots
// each): its reference, its normaliser and the decision to move them need no
// others, where the transposed kernel for many rows has four warps agree on
// every tile.  The two take their row's maximum over the tile first, move the
// reference if that passes it by 2^32 (and O with it: rare), and weigh then.
// The halves alternate: one's weights are taken while the other's products
// run, and keys and values are widened once for both.  Heads of 128 dimensions
// fill tensor memory with S and O, and P takes S's place: the half's next
// scores wait until its sums have read P.  Heads of 64 leave P a place of its
// own.
//
// Four warps widen keys and four values (and all of them the groups' queries),
// eight weigh each half; one each copies keys, copies values, issues products,
// walks the line.  Values are widened into two buffers, as they are the longer
// work and would keep the products waiting from one.
//
// A tile of 256 rows takes some 4800 cycles, of which the products are issued
// for 2400; the rest are waits for weights (770), a group's keys and queries
// (620), sums that are not done (520) and values (250; clock stamps of an
// earlier build, 4 % off).  1024 rows on each of 8 heads of 128 dimensions over
// 32768 tokens (137 GFLOP): 148 us, 0.93 PFLOP/s, half of the library's plain product.  The whole call, rests with it, took 261
// us with a thread a row (too few warps to fill the exponentials' unit), 216
// with two and all widening in the same warps, and takes 200.
#include "mds_cache_tensor.cuh"

namespace mds {
namespace cache {

namespace {

constexpr int kThreads = 896, kWeigh = 512;   // all, those that weigh
constexpr int kHalf = 128, kMostRows = kWideRows;
// Groups of more than kManyRows rows come here, so that every tile of rows has two halves.
static_assert(kMostRows == 2 * kHalf && kManyRows >= kHalf, "two halves");
constexpr int kScaleRing = 8;   // tiles whose key scales are held
constexpr float kMove = 32.f;   // weights stay below 2^32

enum Bar {
  kKFull = 0, kKEmpty = kKFull + 4, kVFull = kKEmpty + 4, kVEmpty = kVFull + 4, kWideK = kVEmpty + 4, kWideKFree,
  kWideV, kWideVFree = kWideV + 2, kS = kWideVFree + 2, kP = kS + 2, kPV = kP + 2, kQ = kPV + 2, kOFree = kQ + 2, kJob = kOFree + 2,
  kJobFree = kJob + kJobs, kQFree = kJobFree + kJobs, kBars
};

// Shared memory from a 1024-byte boundary on.
template <int D>
struct Wide {
  static constexpr int kTileBytes = kTile * D;
  static constexpr int kK = 2, kV = D == 128 ? 1 : 2;     // tiles as they are stored, in rings
  static constexpr int q = 0, wide_k = q + kMostRows * D * 2, wide_v = wide_k + kTileBytes * 2,
                       k_ring = wide_v + 2 * kTileBytes * 2, v_ring = k_ring + kK * kTileBytes, small = v_ring + kV * kTileBytes;
  static constexpr int bytes(int B) {
    return 1024 + small + kScaleRing * 8 * 4 + 4 * 8 * 4 + kMostRows * (2 * 4 + 2 * 4 + 2 * 2 * 4) + (kBars + 1) / 2 * 16 +
           kJobs * (int)sizeof(Job) + 16 + seq_bytes<kPrefix>(B);
  }
};

// 16 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld16(float* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const unsigned* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// The loaded registers are read after the wait.
__device__ __forceinline__ void tmem_ld_wait16(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
                 "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15])::"memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const __grid_constant__ Params p) {
  using W = Wide<D>;
  using T = __nv_bfloat16;
  constexpr int R = kPieceRow<D>;
  extern __shared__ char raw[];
  char* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  char* at = base + W::small;
  float* k_scales = reinterpret_cast<float*>(at);          // [kScaleRing][8], by tile
  at += kScaleRing * 8 * 4;
  float* v_scales = reinterpret_cast<float*>(at);          // [W::kV][8], by the ring's slot
  at += 4 * 8 * 4;
  int* row_out = reinterpret_cast<int*>(at);               // [2][rows], by group: a row's place in the call, -1: not live
  at += 2 * kMostRows * 4;
  float* row_coef = reinterpret_cast<float*>(at);          // [2][rows]: of scores, to log2 units
  at += 2 * kMostRows * 4;
  float* shared_row = reinterpret_cast<float*>(at);        // [2][2][rows]: what a row's two threads tell one another, by tile
  at += 2 * 2 * kMostRows * 4;
  uint64_t* bar = reinterpret_cast<uint64_t*>(at);
  at += (kBars + 1) / 2 * 16;
  Job* jobs = reinterpret_cast<Job*>(at);
  at += kJobs * sizeof(Job);
  int* abort = reinterpret_cast<int*>(at);
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(abort + 1);
  // the call's status, for the end: from the parameters there it costs the whole kernel spilled registers
  uint32_t** status_at = reinterpret_cast<uint32_t**>(abort + 2);
  at += 16;
  Seq<kPrefix>* seqs = reinterpret_cast<Seq<kPrefix>*>(at);
  long long* prefix = reinterpret_cast<long long*>(base);  // before the queries

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int half0 = min(((p.rows_per + 1) / 2 + 31) & ~31, kHalf);   // rows of the first half, the second's begin
  if (tid == 0) {
    *abort = 0;
    *status_at = p.s.status;
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar + kKFull + i, 1 + 32);   // the loader's byte count, and its lanes' scale copies
      mbar_init(bar + kKEmpty + i, 4);
      mbar_init(bar + kVFull + i, 1 + 32);
      mbar_init(bar + kVEmpty + i, 4);
    }
    mbar_init(bar + kWideK, 4);
    mbar_init(bar + kWideKFree, 1);
    mbar_init(bar + kQFree, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar + kWideV + i, 4);
      mbar_init(bar + kWideVFree + i, 1);
      mbar_init(bar + kS + i, 1);
      mbar_init(bar + kP + i, 8);
      mbar_init(bar + kPV + i, 1);
      mbar_init(bar + kQ + i, 8);
      mbar_init(bar + kOFree + i, 8);
    }
    for (int i = 0; i < kJobs; ++i) {
      mbar_init(bar + kJob + i, 1);
      mbar_init(bar + kJobFree + i, 11 + kWeigh / 32);   // every warp but the scheduler's
    }
    mbar_init_fence();
  }
  after_launch_before();
  if (idle<kPrefix>(p)) return;
  plan<T, kPrefix>(p, prefix, seqs, D);
  __syncthreads();
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
  constexpr bool kApart = D == 64;
  // of half h: S 128 columns, O D, P 64, or in S's two halves
  const uint32_t t_s = tmem, t_o = tmem + 2 * kTile, t_p = kApart ? t_o + 2 * D : t_s;
  constexpr uint32_t kHalfP = kApart ? 64 : kTile, kPartP = kApart ? 32 : 64;   // from a half to the next, from 64 slots to the next
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
    schedule<D>(p, seqs, c, per, u0, u1, jobs, bar + kJob, bar + kJobFree, abort);
  } else if (warp == 0 || warp == 2) {
    // ---- loaders, of keys and of values: one block of 16 slots a lane (0..7);
    // the first of a page's blocks copies for all of them
    const State& s = p.s;
    const int kv = warp >> 1, blk = lane & 7, slots = kv ? W::kV : W::kK;
    char* ring = base + (kv ? W::v_ring : W::k_ring);
    const int full = kv ? kVFull : kKFull, empty = kv ? kVEmpty : kKEmpty;
    const int64_t layer0 = (int64_t)p.a.layer * s.pages;
    int tile = 0, slot = 0;
    unsigned parity = 1;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      const int off = job.off, end = off + job.cnt, h = job.h;
      if (!job.cnt) break;
      const int32_t* table = s.table + (int64_t)job.q * s.max_pages;
      job_done(n);
      // a prefix is whole tiles from slot 0 on
      auto page_of = [&](int i) { return lane < 8 && i < end ? __ldg(table + ((i * kTile + blk * kBlock) >> s.page_log)) : -1; };
      int page = page_of(off);
      for (int i = off; i < end; ++i, ++tile) {
        const int next = page_of(i + 1);
        const bool copies = page >= 0 && ((blk * kBlock) & (p.span - 1)) == 0;   // the first block of its span
        const int64_t row = (((layer0 + page) * 2 + kv) * s.kv_heads + h) * s.page_tokens +
                            ((i * kTile + blk * kBlock) & (s.page_tokens - 1));
        hold(empty + slot, parity);
        if (gave_up(abort)) break;
        if (lane == 0) mbar_expect_tx(bar + full + slot, W::kTileBytes);
        __syncwarp();
        if (page >= 0) {
          if (copies) bulk_copy(ring + slot * W::kTileBytes + blk * kBlock * D, s.pool + row * D, p.span * D, bar + full + slot);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(
                           smem_u32(kv ? v_scales + slot * 8 + blk : k_scales + (tile & (kScaleRing - 1)) * 8 + blk)),
                       "l"(s.scales + (row >> 4))
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar + full + slot)) : "memory");
        page = next;
        if (++slot == slots) slot = 0, parity ^= 1u;
      }
    }
  } else if (warp == 1) {
    // ---- products, issued by one thread; none once a wait for them gave up
    bool there = true;
    auto need = [&](int b, unsigned parity) { there = wait(bar + b, parity, abort) && there; };
    const uint32_t id_s = instruction(kTile, 0, 0), id_o = instruction(D, 1, 0) | 1u << 16;   // V's contiguous axis is its columns
    const uint64_t q_op = operand(smem_u32(base + W::q), 16), k_op = operand(smem_u32(base + W::wide_k), 16);
    const uint64_t v_op = operand(smem_u32(base + W::wide_v), kTile * 128);
    int tile = 0, group = 0;
    auto sums = [&](int t, int h, bool first) {
      need(kP + h, t & 1);
      if (h == 0) need(kWideV + (t & 1), (t >> 1) & 1);
      if (first) need(kOFree + h, (group & 1) ^ 1);
      after_sync();
      if (elected() && there) {
        const uint64_t v = v_op + ((t & 1) * (W::kTileBytes * 2) >> 4);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)   // 16 slots: 8 columns of weights, 2048 bytes of V
          mma_ts(t_o + h * D, t_p + h * kHalfP + (k >> 2) * kPartP + (k & 3) * 8, v + k * (2048 >> 4), id_o, !(first && k == 0));
        commit_to(bar + kPV + h);
        if (h == 1) commit_to(bar + kWideVFree + (t & 1));
      }
      __syncwarp();
    };
    auto scores = [&](int t, int h, bool last) {
      if (h == 0) need(kWideK, t & 1);
      after_sync();
      if (elected() && there) {
        const uint64_t q = q_op + (h * (kHalf * D * 2) >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t step = ((k >> 2) * kTile * 128 + (k & 3) * 32) >> 4;
          mma_ss(t_s + h * kTile, q + step, k_op + step, id_s, k > 0);
        }
        commit_to(bar + kS + h);
        if (h == 1) commit_to(bar + kWideKFree);
        if (h == 1 && last) commit_to(bar + kQFree);
      }
      __syncwarp();
    };
    for (;;) {
      const int cnt = job_at(group).cnt;
      if (!cnt) break;
      job_done(group);
      need(kQ + (group & 1), (group >> 1) & 1);
      for (int i = 0; i < cnt; ++i, ++tile) {
        for (int h = 0; h < 2; ++h) {
          if (kApart) {
            if (i > 0) need(kP + h, (tile - 1) & 1);   // the scores before have been read
            scores(tile, h, i + 1 == cnt);
            if (i > 0) sums(tile - 1, h, i == 1);
          } else {
            if (i > 0) {
              sums(tile - 1, h, i == 1);
              need(kPV + h, (tile - 1) & 1);
            }
            scores(tile, h, i + 1 == cnt);
          }
        }
      }
      for (int h = 0; h < 2; ++h) {
        sums(tile - 1, h, cnt == 1);
        // the next group's first scores may not overwrite the weights before they are read
        if (!kApart) need(kPV + h, (tile - 1) & 1);
      }
      ++group;
    }
  } else if (warp < 12) {
    // ---- widen keys, or values, and the groups' queries
    const int w4 = warp & 3;
    int ks = 0, vs = 0;
    unsigned kp = 0, vp = 0;
    auto keys = [&](int t) {
      hold(kKFull + ks, kp);
      hold(kWideKFree, (t & 1) ^ 1);
      const char* src = base + W::k_ring + ks * W::kTileBytes;
      char* dst = base + W::wide_k;
      constexpr int kUnits = D / 16;
#pragma unroll
      for (int i0 = 0; i0 < kUnits; i0 += 4) {
        uint4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // eight rows and four units at a time, a quarter of the warp a unit
          const int x = i0 + i, row = w4 * 32 + x * 4 / kUnits * 8 + (lane & 7), unit = (x * 4 + (lane >> 3)) % kUnits;
          y[i] = *reinterpret_cast<const uint4*>(src + swizzled(row * D + unit * 16));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int x = i0 + i, row = w4 * 32 + x * 4 / kUnits * 8 + (lane & 7), unit = (x * 4 + (lane >> 3)) % kUnits;
          uint4 a, b;
          to_f16(y[i].x, a.x, a.y);
          to_f16(y[i].y, a.z, a.w);
          to_f16(y[i].z, b.x, b.y);
          to_f16(y[i].w, b.z, b.w);
          char* line = dst + (unit >> 2) * (kTile * 128) + row * 128;
          *reinterpret_cast<uint4*>(line + ((((unit & 3) * 2) ^ (row & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(line + ((((unit & 3) * 2 + 1) ^ (row & 7)) << 4)) = b;
        }
      }
      dev::fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar + kKEmpty + ks);
        mbar_arrive(bar + kWideK);
      }
      if (++ks == W::kK) ks = 0, kp ^= 1u;
    };
    auto values = [&](int t) {
      hold(kVFull + vs, vp);
      hold(kWideVFree + (t & 1), ((t >> 1) & 1) ^ 1);
      const float* sc = v_scales + vs * 8 + w4 * 2;
      unsigned rest[2], factor[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) factor[i] = value_factor(sc[i], rest[i]);
      const bool large = rest[0] != 0x3f803f80u || rest[1] != 0x3f803f80u;
      const char* src = base + W::v_ring + vs * W::kTileBytes;
      char* dst = base + W::wide_v + (t & 1) * (W::kTileBytes * 2);
      constexpr int kUnits = D / 16;
#pragma unroll
      for (int i0 = 0; i0 < kUnits; i0 += 4) {
        uint4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int octet = (i0 + i) * 4 / kUnits, unit = ((i0 + i) * 4 + (lane >> 3)) % kUnits;
          y[i] = *reinterpret_cast<const uint4*>(src + swizzled((w4 * 32 + octet * 8 + (lane & 7)) * D + unit * 16));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // the same eight slots for all lanes, so one of the warp's two blocks
          const int octet = (i0 + i) * 4 / kUnits, unit = ((i0 + i) * 4 + (lane >> 3)) % kUnits;
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
          char* line = dst + (unit >> 2) * (kTile * 128) + k * 128;
          *reinterpret_cast<uint4*>(line + ((((unit & 3) * 2) ^ (k & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(line + ((((unit & 3) * 2 + 1) ^ (k & 7)) << 4)) = b;
        }
      }
      dev::fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar + kVEmpty + vs);
        mbar_arrive(bar + kWideV + (t & 1));
      }
      if (++vs == W::kV) vs = 0, vp ^= 1u;
    };
    // A group's queries, scaled to half precision, rows of 128 bytes; a warp's
    // 32 rows are its own from copy to scaling.
    auto queries = [&](int n, const Job& job) {
      constexpr int kUnits = D / 8, kAtOnce = 32 / kUnits;
      const T* q = static_cast<const T*>(p.a.q);
      int* out = row_out + (n & 1) * kMostRows;
      float* coef = row_coef + (n & 1) * kMostRows;
      const int r0 = (warp - 4) * 32;
      {   // a row a lane
        const int r = r0 + lane, h = r >> 7, in = r & (kHalf - 1);
        const int row = job.row0 + (h ? half0 + in : in), node = row / p.g, head = job.h * p.g + row - node * p.g;
        const bool mine = h ? half0 + in < p.rows_per : in < half0;
        const int64_t from = mine ? query_at<kPrefix>(p, job.b, node, job.live) : kNowhere;
        out[r] = from != kNowhere ? (int)row_at(p, job.b, job.h, row) : -1;   // `prior` has fewer than 2^18 rows
        const int64_t from_row = from != kNowhere ? from + head * p.a.q_head : kNowhere;
        // its copies: 16 bytes a lane, kAtOnce rows at a time
#pragma unroll 4
        for (int i = 0; i < 32; i += kAtOnce) {
          const int x = i + lane / kUnits, unit = lane % kUnits, rr = r0 + x;
          const int64_t src = __shfl_sync(kFull, from_row, x);
          char* dst = base + W::q + (rr >> 7) * (kHalf * D * 2) + (unit >> 3) * (kHalf * 128) + (rr & 127) * 128 +
                      (((unit & 7) ^ (rr & 7)) << 4);
          if (src != kNowhere)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(q + src + unit * 8) : "memory");
          else
            *reinterpret_cast<uint4*>(dst) = uint4{0, 0, 0, 0};
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
#pragma unroll 4
      for (int i = 0; i < 32; i += kAtOnce) {
        const int r = r0 + i + lane / kUnits, unit = lane % kUnits;
        uint4* at_lane = reinterpret_cast<uint4*>(base + W::q + (r >> 7) * (kHalf * D * 2) + (unit >> 3) * (kHalf * 128) +
                                                  (r & 127) * 128 + (((unit & 7) ^ (r & 7)) << 4));
        const uint4 y = *at_lane;
        const unsigned w[4] = {y.x, y.y, y.z, y.w};
        unsigned bits = 0;   // the largest magnitude: bfloat16 order as their bits do
#pragma unroll
        for (int z = 0; z < 4; ++z) bits = max(bits, max(w[z] << 16 & 0x7fff0000u, w[z] & 0x7fff0000u));
#pragma unroll
        for (int d = 1; d < kUnits; d *= 2) bits = max(bits, __shfl_xor_sync(kFull, bits, d));
        const int e = bits == 0 || bits >= 0x7f800000u ? 0 : max((int)(bits >> 23) - 127 - 14, -112);
        // the coefficient is positive, so that a row's largest product is its
        // largest score: the scale's sign, or 0, goes to the queries
        const float inv = p.a.scale == 0.f ? 0.f : copysignf(__uint_as_float((unsigned)(127 - e) << 23), p.a.scale);
        unsigned v[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const __half2 a = __floats2half2_rn(__uint_as_float(w[z] << 16) * inv, __uint_as_float(w[z] & 0xffff0000u) * inv);
          v[z] = *reinterpret_cast<const unsigned*>(&a);
        }
        *at_lane = uint4{v[0], v[1], v[2], v[3]};
        if (unit == 0) coef[r] = p.a.scale == 0.f ? 1.f : fabsf(p.a.scale) * dev::kLog2e * __uint_as_float((unsigned)(127 + e) << 23);
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
      // the products of the group before have read its queries, and every warp
      // is done with what the rows of the group before that were
      // (of a barrier's phases a warp waits for each in turn, and the next is not
      // over before the warp has done its part for it: a wait does not tell a
      // phase from the next but one)
      if (n) hold(kQFree, (n - 1) & 1);
      if (n > 1) hold(kJobFree + ((n - 2) & (kJobs - 1)), ((n - 2) / kJobs) & 1);
      queries(n, job);
      job_done(n);
      for (int i = 0; i < cnt; ++i, ++tile) {
        if (warp < 8) keys(tile);
        else values(tile);
      }
    }
  } else {
    // ---- weigh: 64 slots of a row of a half a thread
    const int half = (warp - 12) >> 3, part = ((warp - 12) >> 2) & 1, w4 = warp & 3, r = half * kHalf + w4 * 32 + lane;
    const int mine = half ? half0 + w4 * 32 + lane : w4 * 32 + lane;   // row of the tile of rows
    const bool used = mine - lane < (half ? p.rows_per : half0);   // the warp has rows
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    const uint32_t s_at = t_s + half * kTile + part * 64 + lanes, o_at = t_o + half * D + part * (D / 2) + lanes;
    const uint32_t p_at = t_p + half * kHalfP + part * kPartP + lanes;
    // a row's two threads: theirs and the other's places
    auto tell = [&](int t, float x) {
      float* to = shared_row + (t & 1) * (2 * kMostRows) + r;
      to[part * kMostRows] = x;
      asm volatile("bar.sync %0, 64;" ::"r"(5 + half * 4 + w4) : "memory");
      return to[(part ^ 1) * kMostRows];
    };
    int tile = 0, told = 0;
    for (int n = 0;; ++n) {
      const Job& job = job_at(n);
      if (!job.cnt) break;
      const int cnt = job.cnt;
      hold(kQ + (n & 1), (n >> 1) & 1);
      const float rc = row_coef[(n & 1) * kMostRows + r];
      const int out = row_out[(n & 1) * kMostRows + r];
      float ref = 0.f;
      float2 sum{0.f, 0.f};
      for (int i = 0; i < cnt; ++i, ++tile) {
        hold(kS + half, tile & 1);
        after_sync();
        if (used) {
          const float* sc = k_scales + (tile & (kScaleRing - 1)) * 8 + part * 4;
          float x[2][16];
          // the largest score: of a block's products the largest, times its coefficient, rounded like the scores
          float top = kNone;
          tmem_ld16(x[0], s_at);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float* y = x[j & 1];
            tmem_ld_wait16(y);
            if (j < 3) tmem_ld16(x[(j + 1) & 1], s_at + (j + 1) * 16);
            float m = max3(y[0], y[1], y[2]), m2 = max3(y[3], y[4], y[5]);
#pragma unroll
            for (int z = 6; z < 14; z += 4) m = max3(m, y[z], y[z + 1]), m2 = max3(m2, y[z + 2], y[z + 3]);
            m = fmaxf(max3(m, y[14], y[15]), m2);
            top = fmaxf(top, __fmul_rn(m, rc * sc[j]));
          }
          top = fmaxf(top, tell(told++, top));
          if (kApart && i > 0) {   // the weights before have been read
            hold(kPV + half, (tile - 1) & 1);
            after_sync();
          }
          if (i == 0) {
            ref = top;   // kNone where no score is finite: a later tile's moves it, and what it leaves weighs nothing
          } else if (__any_sync(kFull, top > ref + kMove)) {
            // the sums so far follow; O of the tiles before is complete
            const bool moves = top > ref + kMove;
            const float alpha = moves ? ex2(ref - top) : 1.f;
            if (moves) ref = top;
            sum.x *= alpha;
            sum.y *= alpha;
#pragma unroll 1
            for (int j = 0; j < D / 32; ++j) {
              tmem_ld16(x[1], o_at + j * 16);
              tmem_ld_wait16(x[1]);
              unsigned y[16];
#pragma unroll
              for (int z = 0; z < 16; ++z) y[z] = __float_as_uint(x[1][z] * alpha);
              tmem_st_row16(o_at + j * 16, y);
            }
          }
          tmem_ld16(x[0], s_at);
          const float less = -ref;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float* y = x[j & 1];
            tmem_ld_wait16(y);
            if (j < 3) tmem_ld16(x[(j + 1) & 1], s_at + (j + 1) * 16);
            const float cf = rc * sc[j];
            unsigned w[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) {
              // scores rounded, then the reference: no weight of the largest passes what it should be
              const float2 t = mul2(float2{y[2 * z], y[2 * z + 1]}, float2{cf, cf});
              const float2 e = fma2(t, float2{p.one, p.one}, float2{less, less});
              w[z] = pack_bf16(ex2(e.x), ex2(e.y));
              sum = add2(sum, float2{__uint_as_float(w[z] << 16), __uint_as_float(w[z] & 0xffff0000u)});
            }
            // in the scores' place, that has been read: block j's weights are columns 8 j .., its scores 16 j ..
            tmem_st8(p_at + j * 8, w);
          }
          tmem_st_wait();
        } else if (kApart && i > 0) {
          hold(kPV + half, (tile - 1) & 1);
        }
        before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + kP + half);
      }
      // ---- the group's or piece's end: the sums as they are
      float l = sum.x + sum.y;
      if (used) l += tell(told++, l);
      hold(kPV + half, (tile - 1) & 1);
      after_sync();
      if (used) {
        float* to = job.whole() ? prior_of<D>(p, out) : piece_of<D>(p, blockIdx.x, job.off == 0) + mine * R;
#pragma unroll 1
        for (int j = 0; j < D / 32; ++j) {
          float x[16];
          tmem_ld16(x, o_at + j * 16);
          tmem_ld_wait16(x);
          if (out >= 0) {
#pragma unroll
            for (int z = 0; z < 16; z += 4)   // of every four dimensions the order is 0, 2, 1, 3
              __stcg(reinterpret_cast<float4*>(to + 4 + part * (D / 2) + j * 16 + z), float4{x[z], x[z + 2], x[z + 1], x[z + 3]});
          }
        }
        if (out >= 0 && part == 0) __stcg(reinterpret_cast<float2*>(to), float2{ref, l});
      }
      before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + kOFree + half);
      job_done(n);
    }
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == 2) {
    report(abort, *status_at);
    __syncwarp();
    tmem_free(tmem);
  }
}

template <int D>
cudaError_t launch(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  static_assert(Wide<D>::bytes(MDS_CACHE_MAX_BATCH / 2) <= 227 * 1024, "shared memory for groups of two of the largest batch");
  Params p{s, a, s.page_tokens < kTile ? s.page_tokens : kTile, a.heads / s.kv_heads, 0, 0, 0, 0};
  p.rows = a.n * p.g;
  p.rows_per = even_rows(p.rows, kWideRows);
  p.row_tiles = (p.rows + p.rows_per - 1) / p.rows_per;
  p.members = x.members;
  p.nodes = x.nodes;
  p.prior = x.prior;
  p.worth = x.worth;
  p.each = x.each;
  p.saved = x.saved;
  return launch_behind(wide_kernel<D>, attend_grid(sms, p.rows_per, D, kPieceFloats), kThreads, Wide<D>::bytes(a.B), st, p);
}

}  // namespace

cudaError_t configure_wide() {
  const cudaError_t e = cudaFuncSetAttribute(wide_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  return e == cudaSuccess ? cudaFuncSetAttribute(wide_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) : e;
}

cudaError_t shared_wide(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  return s.head_dim == 64 ? launch<64>(s, a, x, sms, st) : launch<128>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
