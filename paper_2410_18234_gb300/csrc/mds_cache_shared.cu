// Attention for sequences that share a prefix: what is shared is found from
// the page tables, the prefix is attended to once for all of a group's rows,
// then every sequence attends to its own tokens and joins the two.
//
// Pages that several sequences hold are the same memory at the same slots, so
// a prefix is the page indices at which the tables of all of a group's live
// sequences agree, cut to committed tokens and to whole key tiles.
#include "mds_cache_attend.cuh"

namespace mds {
namespace cache {

namespace {

// One block of threads a sequence: the tokens that it shares with the first
// live sequence of its group (none if it is the only one), and its live nodes.
__global__ void __launch_bounds__(256) share_kernel(const State s, const int32_t* seqs, const int32_t* counts, int n,
                                                    int members) {
  __shared__ int first_s, differ_s, others_s;
  const int tid = threadIdx.x, b = blockIdx.x, g0 = b / members * members;
  if (tid == 0) first_s = INT_MAX, differ_s = INT_MAX, others_s = 0;
  __syncthreads();
  int id, len, live, end, q0, len0, live0;
  for (int i = g0 + tid; i < g0 + members; i += 256) {
    find(s, seqs, counts, i, n, &q0, &len0, &live0, &end);
    if (live0 > 0) atomicMin(&first_s, i);
    if (live0 > 0 && i != b) others_s = 1;
  }
  find(s, seqs, counts, b, n, &id, &len, &live, &end);
  __syncthreads();
  if (live > 0) {
    find(s, seqs, counts, first_s, n, &q0, &len0, &live0, &end);
    const int pages = min(len, len0) >> s.page_log;
    const int32_t *row = s.table + (int64_t)id * s.max_pages, *row0 = s.table + (int64_t)q0 * s.max_pages;
    int differ = pages;
    for (int p = tid; p < pages; p += 256)
      if (row[p] != row0[p]) differ = min(differ, p);
    atomicMin(&differ_s, differ);
  }
  __syncthreads();
  if (tid == 0) s.share[b] = live <= 0 ? int2{INT_MAX, 0} : others_s ? int2{(differ_s << s.page_log) & -kTile, live} : int2{0, live};
}

}  // namespace

cudaError_t attend_shared(const State& s, const Attend& a, int members, int sms, cudaStream_t st) {
  const int g = a.heads / s.kv_heads, groups = a.B / members;
  // as many groups at a time as their rows' sums over the prefix have room for
  const int64_t row = (int64_t)a.n * a.heads * (s.head_dim + 4) * members;
  const int at_once = (int)(((int64_t)kPartFloats - kPieceFloats) / row);
  if (members < 2 || at_once == 0) return attend(s, a, sms, st);
  const int es = s.dtype == MDS_F32 ? 4 : 2;
  for (int g0 = 0; g0 < groups; g0 += at_once) {
    const int some = groups - g0 < at_once ? groups - g0 : at_once, b0 = g0 * members;
    Attend x = a;
    x.B = some * members;
    x.seqs = a.seqs + b0;
    x.counts = a.counts ? a.counts + b0 : nullptr;
    x.q = static_cast<const char*>(a.q) + b0 * a.q_seq * es;
    x.out = static_cast<char*>(a.out) + (int64_t)b0 * a.n * a.heads * s.head_dim * es;
    share_kernel<<<x.B, 256, 0, st>>>(s, x.seqs, x.counts, a.n, members);
    cudaError_t e = cudaGetLastError();
    Attend y = x;
    y.B = some;
    y.n = a.n * members;
    y.L = y.n - 1;
    Shared z{members, a.n, true, s.part + kPieceFloats};
    if (e == cudaSuccess)
      e = s.dtype != MDS_F32 && (int64_t)y.n * g > 16 ? shared_many(s, y, z, sms, st) : shared_few(s, y, z, sms, st);
    z.prefix = false;
    if (e == cudaSuccess)
      e = s.dtype == MDS_F32 ? shared_few(s, x, z, sms, st)
          : (int64_t)a.n * g <= 8 ? shared_rest(s, x, z, sms, st)
          : (int64_t)a.n * g <= 16 ? shared_few(s, x, z, sms, st) : shared_many(s, x, z, sms, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace cache
}  // namespace mds
