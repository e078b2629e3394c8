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

constexpr int kWarps = 8;                  // consumers; one more warp loads
constexpr int kStageMax = 8;
constexpr int kJoinStride = 80;            // floats of a joined row's 64 dimensions: rows 16 banks apart

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

__device__ __forceinline__ void mma_f16(float* c, const uint4& a, unsigned b0, unsigned b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float* c, const unsigned* a, unsigned b0, unsigned b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void ldmatrix_x4_trans(unsigned* r, unsigned addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
// ------------------------------------------------------- few rows: 16 or 32
//
// Each consumer warp takes one block of 16 slots of a tile for all the rows:
// a warp's scores, weights and sums stay in its registers, its key and value
// scales are two numbers, and the eight warps' sums meet once per group.
// MT: 16-row tiles.  Q: terms of a query.  W: terms of a weight.
template <typename T, int D, int MT>
struct Few {
  static constexpr int kQ = sizeof(T) == 4 ? 2 : 1;
  static constexpr int kW = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kRows = 16 * MT;
  static constexpr int kSteps = D / 16;
  static constexpr int kStageBytes = 2 * kTile * D;
  static constexpr int kQBytes = MT * kQ * kSteps * 512;
  static constexpr int kJoinBytes = kWarps * 16 * kJoinStride * 4;
  // after the stages: queries, join buffer, per-warp (reference, sum), row coefficients, stage scales, barriers
  static constexpr int kFixed =
      kQBytes + kJoinBytes + kWarps * kRows * 8 + kRows * 4 + kStageMax * 16 * 4 + 2 * kStageMax * 8 + 16;
  static int smem(int stages, int B) { return 1024 + stages * kStageBytes + kFixed + (B + 1) * 8 + B * 16 + 16; }
};

template <typename T, int D, int MT>
__global__ void __launch_bounds__(32 * (kWarps + 1), 1) few_kernel(const __grid_constant__ Params p) {
  using F = Few<T, D, MT>;
  extern __shared__ char raw[];
  char* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  char* stage_mem = base;
  char* at = base + p.stages * F::kStageBytes;
  uint4* qf = reinterpret_cast<uint4*>(at);
  at += F::kQBytes;
  float* join = reinterpret_cast<float*>(at);
  at += F::kJoinBytes;
  float2* ml = reinterpret_cast<float2*>(at);
  at += kWarps * F::kRows * 8;
  float* coef = reinterpret_cast<float*>(at);
  at += F::kRows * 4;
  float* stage_scales = reinterpret_cast<float*>(at);
  at += kStageMax * 16 * 4;
  uint64_t* full = reinterpret_cast<uint64_t*>(at);
  uint64_t* empty = full + kStageMax;
  at += 2 * kStageMax * 8;
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
      mbar_init(empty + i, kWarps);
    }
    mbar_init_fence();
  }
  plan<T>(p, prefix, seqs, D);   // ends in a barrier
  const long long total = prefix[p.a.B];
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  const long long u0 = per * blockIdx.x, u1 = min(u0 + per, total);
  if (u0 >= u1) return;

  Cursor c = locate(p, prefix, seqs, u0);
  Group grp = group_of(p, seqs[c.b], c.rt);
  long long u = u0;

  if (warp == kWarps) {
    // ---- loader: one block of 16 slots a lane (keys: lanes 0..7, values: 8..15)
    const State& s = p.s;
    const int kv = (lane >> 3) & 1, blk = lane & 7;
    const int64_t layer0 = (int64_t)p.a.layer * s.pages;
    int stage = 0;
    unsigned phase = 1;
    while (u < u1) {
      const int cnt = (int)min((long long)(grp.tiles - c.off), u1 - u);
      const int32_t* table = s.table + (int64_t)seqs[c.b].q * s.max_pages;
      auto page_of = [&](int i) {
        const int t = tile_slot(grp, i) + blk * kBlock;
        return lane < 16 && i < c.off + cnt && block_seen(grp, t) ? __ldg(table + (t >> s.page_log)) : -1;
      };
      int page = page_of(c.off);
      for (int i = c.off; i < c.off + cnt; ++i) {
        const int next = page_of(i + 1);
        const int t = tile_slot(grp, i) + blk * kBlock;
        wait(empty + stage, phase, abort);
        const unsigned takes = __ballot_sync(kFull, page >= 0);
        if (lane == 0) mbar_expect_tx(full + stage, __popc(takes) * kBlock * D);
        __syncwarp();
        if (page >= 0) {
          const int64_t tile = ((layer0 + page) * 2 + kv) * s.kv_heads + c.h;
          const int r = t & (s.page_tokens - 1);
          const uint8_t* src = s.pool + (tile * s.page_tokens + r) * D;
          bulk_copy(stage_mem + stage * F::kStageBytes + (kv * kTile + blk * kBlock) * D, src, kBlock * D, full + stage);
          const float* sc = s.scales + ((tile * s.page_tokens + r) >> 4);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(stage_scales + stage * 16 + lane)),
                       "l"(sc)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(full + stage)) : "memory");
        page = next;
        if (++stage == p.stages) stage = 0, phase ^= 1u;
      }
      u += cnt;
      if (u < u1 && !advance(p, seqs, c, grp)) break;
    }
    report(abort, s.status);
    return;
  }

  // ---- consumers
  const int gr = lane >> 2, tq = lane & 3;
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
  int stage = 0;
  unsigned phase = 0;
  while (u < u1) {
    const Seq q = seqs[c.b];
    const int cnt = (int)min((long long)(grp.tiles - c.off), u1 - u);
    const int row0 = c.rt * F::kRows;
    // queries of the group: scaled, in the order of the products' fragments
    for (int r = warp; r < F::kRows; r += kWarps) {
      const int row = row0 + r, node = row / p.g, head = c.h * p.g + row % p.g;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (lane * 4 < D && node < q.live) {
        const T* src = static_cast<const T*>(p.a.q) + c.b * p.a.q_seq + node * p.a.q_tok + head * p.a.q_head + lane * 4;
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
        const int half = (r >> 3) & 1, mt = r >> 4;
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
          unsigned* dst = reinterpret_cast<unsigned*>(qf + ((mt * F::kQ + term) * F::kSteps + step) * 32 + to);
          dst[half] = w[0];
          dst[2 + half] = w[1];
        }
      }
    }
    // the rows' nodes
    int node[MT][2], own[MT][2];   // node, and the first node of its branch
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int i = (row0 + m * 16 + x * 8 + gr) / p.g;
        node[m][x] = i;
        own[m][x] = i > 0 && p.a.L > 0 ? 1 + (i - 1) / p.a.L * p.a.L : 1;
      }
    consumers_sync();
    float rc[MT][2], ref[MT][2], sum[MT][2], acc[MT][D / 16][2][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        rc[m][x] = coef[m * 16 + x * 8 + gr];
        ref[m][x] = kNone;
        sum[m][x] = 0.f;
      }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int z = 0; z < 4; ++z) acc[m][x][y][z] = 0.f;

    for (int i = c.off; i < c.off + cnt; ++i) {
      const int t0 = tile_slot(grp, i) + warp * kBlock;
      wait(full + stage, phase, abort);
      if (block_seen(grp, t0)) {
        const char* kb = stage_mem + stage * F::kStageBytes + warp * kBlock * D;
        const unsigned vb = smem_u32(kb + kTile * D);
        const float ks = stage_scales[stage * 16 + warp], vs = stage_scales[stage * 16 + 8 + warp];
        float sc[MT][2][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int z = 0; z < 4; ++z) sc[m][j][z] = 0.f;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          uint4 kx[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) kx[j] = *reinterpret_cast<const uint4*>(kb + k_at[j][x]);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            unsigned b[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) to_f16(y == 0 ? kx[j].x : y == 1 ? kx[j].y : y == 2 ? kx[j].z : kx[j].w, b[j][0], b[j][1]);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int term = 0; term < F::kQ; ++term) {
                const uint4 a = qf[((m * F::kQ + term) * F::kSteps + x * 4 + y) * 32 + lane];
#pragma unroll
                for (int j = 0; j < 2; ++j) mma_f16(sc[m][j], a, b[j][0], b[j][1]);
              }
          }
        }
        // scores in log2 units, masked
        const bool plain = t0 + kBlock <= q.len &&
                           (p.a.window <= 0 || t0 + kBlock <= p.a.sinks || t0 > q.len + min(p.a.L, p.a.n - 1) - p.a.window);
        bool moves = false;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float f = rc[m][x] * ks;
            float top = kNone;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                float y = sc[m][j][2 * x + z] * f;
                if (!plain) {
                  const int t = t0 + j * 8 + tq * 2 + z, at_node = t - q.len, i_row = node[m][x], b0 = own[m][x];
                  bool see = at_node <= i_row && (at_node <= 0 || at_node >= b0);
                  if (p.a.window > 0) {
                    const int pos = at_node <= 0 ? t : q.len + at_node - b0 + 1;
                    const int mine = q.len + (i_row > 0 ? i_row - b0 + 1 : 0);
                    see = see && (pos < p.a.sinks || pos > mine - p.a.window);
                  }
                  y = see && t < grp.hi ? y : dev::kNegInf;
                }
                sc[m][j][2 * x + z] = y;
                top = fmaxf(top, y);
              }
            moves |= top > ref[m][x] + kSlack;
          }
        if (__any_sync(kFull, moves)) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            float alpha[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float top = fmaxf(fmaxf(sc[m][0][2 * x], sc[m][0][2 * x + 1]), fmaxf(sc[m][1][2 * x], sc[m][1][2 * x + 1]));
              top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
              top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
              top = fmaxf(top, ref[m][x]);
              alpha[x] = ex2(ref[m][x] - top);
              ref[m][x] = top;
              sum[m][x] *= alpha[x];
            }
#pragma unroll
            for (int x = 0; x < D / 16; ++x)
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int z = 0; z < 4; ++z) acc[m][x][y][z] *= alpha[z >> 1];
          }
        }
        // weights, as the next product's rows; the values' scale goes to the values
        unsigned w[MT][F::kW][4];
        unsigned rest;
        const unsigned factor = value_factor(vs, rest);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float w0 = ex2(sc[m][j][2 * x] - ref[m][x]), w1 = ex2(sc[m][j][2 * x + 1] - ref[m][x]);
              if constexpr (F::kW > 1) sum[m][x] += w0 + w1;
#pragma unroll
              for (int term = 0; term < F::kW; ++term) {
                const unsigned pk = pack_bf16(w0, w1);
                const float r0 = __uint_as_float(pk << 16), r1 = __uint_as_float(pk & 0xffff0000u);
                if constexpr (F::kW == 1) sum[m][x] += r0 + r1;
                w0 -= r0;
                w1 -= r1;
                w[m][term][2 * j + x] = pk;
              }
            }
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          unsigned v[4];
          ldmatrix_x4_trans(v, vb + v_at[x]);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            unsigned e0, o0, e1, o1;
            to_bf16(v[2 * y], factor, e0, o0);
            to_bf16(v[2 * y + 1], factor, e1, o1);
            if (rest != 0x3f803f80u) times_rest(e0, rest), times_rest(o0, rest), times_rest(e1, rest), times_rest(o1, rest);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int term = 0; term < F::kW; ++term) {
                mma_bf16(acc[m][2 * x + y][0], w[m][term], e0, e1);
                mma_bf16(acc[m][2 * x + y][1], w[m][term], o0, o1);
              }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + stage);
      if (++stage == p.stages) stage = 0, phase ^= 1u;
    }

    // ---- the eight warps' sums meet
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float l = sum[m][x];
        l += __shfl_xor_sync(kFull, l, 1);
        l += __shfl_xor_sync(kFull, l, 2);
        if (tq == 0) ml[warp * F::kRows + m * 16 + x * 8 + gr] = float2{ref[m][x], l};
      }
    consumers_sync();
    const bool whole = c.off == 0 && cnt == grp.tiles;
    const long long g0 = u - c.off;                       // the group's first unit
    const int c0 = (int)(g0 / per), c1 = (int)((g0 + grp.tiles - 1) / per);
    float* part = piece_of(p, blockIdx.x, c.off == 0, D);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float f[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = kNone;
#pragma unroll
        for (int wq = 0; wq < kWarps; ++wq) top = fmaxf(top, ml[wq * F::kRows + m * 16 + x * 8 + gr].x);
        f[x] = ex2(ref[m][x] - top);
      }
#pragma unroll
      for (int hd = 0; hd < D / 64; ++hd) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            const float (*ac)[4] = acc[m][hd * 4 + ch];
            *reinterpret_cast<float4*>(join + (warp * 16 + x * 8 + gr) * kJoinStride + ch * 16 + tq * 4) =
                float4{ac[0][2 * x] * f[x], ac[1][2 * x] * f[x], ac[0][2 * x + 1] * f[x], ac[1][2 * x + 1] * f[x]};
          }
        consumers_sync();
        const int r = tid >> 4, d = (tid & 15) * 4, row = row0 + m * 16 + r;
        if (row / p.g < q.live) {
          float4 o{0.f, 0.f, 0.f, 0.f};
          float top = kNone, l = 0.f;
#pragma unroll
          for (int wq = 0; wq < kWarps; ++wq) {
            const float4 y = *reinterpret_cast<const float4*>(join + (wq * 16 + r) * kJoinStride + d);
            o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
            top = fmaxf(top, ml[wq * F::kRows + m * 16 + r].x);
          }
#pragma unroll
          for (int wq = 0; wq < kWarps; ++wq) {
            const float2 y = ml[wq * F::kRows + m * 16 + r];
            l += y.y * ex2(y.x - top);
          }
          if (whole) {
            const float inv = 1.f / l;
            store4(out_row<T>(p, c.b, c.h, row, D) + hd * 64 + d, float4{o.x * inv, o.y * inv, o.z * inv, o.w * inv});
          } else {
            float* pr = part + (m * 16 + r) * (D + 2);
            __stcg(reinterpret_cast<float2*>(pr + 2 + hd * 64 + d), float2{o.x, o.y});
            __stcg(reinterpret_cast<float2*>(pr + 2 + hd * 64 + d) + 1, float2{o.z, o.w});
            if (hd == 0 && (tid & 15) == 0) __stcg(reinterpret_cast<float2*>(pr), float2{top, l});
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
        const bool last = atomicAdd(p.s.joins + c0, 1u) == (unsigned)(c1 - c0);
        if (last) p.s.joins[c0] = 0;
        *last_s = last;
      }
      consumers_sync();
      if (*last_s) {
        __threadfence();
        join_pieces<T, D>(p, c.b, c.h, row0, q.live, c0, c1, tid, kWarps * 32);
      }
    }
    u += cnt;
    if (u < u1 && !advance(p, seqs, c, grp)) break;
  }
}

template <typename T, int D, int MT>
cudaError_t launch_few(const State& s, const Attend& a, int sms, cudaStream_t st) {
  using F = Few<T, D, MT>;
  Params p{s, a, a.heads / s.kv_heads, 0, 0, 0, F::kRows};
  p.rows = a.n * p.g;
  p.row_tiles = (p.rows + F::kRows - 1) / F::kRows;
  const int grid = attend_grid(sms, F::kRows, D);
  p.stages = kStageMax;
  while (p.stages > 2 && F::smem(p.stages, a.B) > 227 * 1024) --p.stages;
  few_kernel<T, D, MT><<<grid, 32 * (kWarps + 1), F::smem(p.stages, a.B), st>>>(p);
  return cudaGetLastError();
}

template <typename T, int D, int MT>
cudaError_t configure_few() {
  return cudaFuncSetAttribute(few_kernel<T, D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
}

}  // namespace

cudaError_t configure() {
  cudaError_t e = configure_few<float, 64, 1>();
  if (e == cudaSuccess) e = configure_few<float, 128, 1>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 64, 1>();
  if (e == cudaSuccess) e = configure_few<__nv_bfloat16, 128, 1>();
  if (e == cudaSuccess) e = configure_many();
  return e;
}

// Rows of 16-bit queries beyond one 16-row product go to the kernel of
// mds_cache_many.cu.
cudaError_t attend(const State& s, const Attend& a, int sms, cudaStream_t st) {
  const int64_t rows = (int64_t)a.n * (a.heads / s.kv_heads);
  if (s.dtype == MDS_F32)
    return s.head_dim == 64 ? launch_few<float, 64, 1>(s, a, sms, st) : launch_few<float, 128, 1>(s, a, sms, st);
  if (rows > 16) return attend_many(s, a, sms, st);
  return s.head_dim == 64 ? launch_few<__nv_bfloat16, 64, 1>(s, a, sms, st)
                          : launch_few<__nv_bfloat16, 128, 1>(s, a, sms, st);
}

}  // namespace cache
}  // namespace mds
