// Attention for sequences that share a prefix: what is shared is found from
// the page tables, the prefix is attended to once for all of a group's rows,
// its pieces are joined, then every sequence attends to its own tokens and
// joins the two.
//
// Pages that several sequences hold are the same memory at the same slots, so
// a prefix is the page indices at which the tables of all of a group's live
// sequences agree, cut to committed tokens and to whole key tiles.
#include <algorithm>

#include "mds_cache_attend.cuh"

namespace mds {
namespace cache {

namespace {

// Rows of a group up to which the prefix's launch is the transposed kernel for
// many rows, which has them as columns, so that few are empty: as many as it
// has in one tile.  The wide one has two halves of 128 rows a product, filled
// or not.  The call in us, transposed / wide, one group over 32768 tokens (a)
// and 16 over 6000 (b; from 160 rows on 12 over 8000), 4 rows a sequence:
//   rows   heads of 128: a         b     heads of 64: a        b
//    32             50 / 66   92 / 133        46 / 53   76 /  98
//    48             51 / 70   97 / 143        46 / 57   80 / 109
//    64             57 / 70  108 / 145        53 / 57   96 / 111
//    96             58 / 72  127 / 167        53 / 58  112 / 124
//   128             67 / 75  150 / 176        60 / 60  127 / 131
//   144             68 / 76  154 / 180        62 / 61  129 / 133
//   160             73 / 81  170 / 169        67 / 62  152 / 127
//   192             74 / 82  177 / 176        68 / 63  156 / 132
//   256             84 / 86  217 / 195        76 / 65  191 / 146
constexpr int kNarrow = kManyRows;
// Where the caller does not say, prefixes are attended to by themselves where
// that pays: less is over sooner without the prefix's launch.  In us, shared /
// not (this call) / mds_cache_attend, 32 heads on 8 of 128 dimensions, G
// sequences a group:
//   rows 4:    8 sequences, G 8,  4096 tokens ( 56 MB saved)  39 /  40 /  29
//              2,           G 2, 32768        ( 64 MB)        49 /  56 /  38
//              8,           G 8,  8192        (112 MB)        41 /  49 /  37
//              8,           G 8, 16384        (224 MB)        47 /  70 /  56
//             64,           G 64, 2048        (252 MB)        49 /  74 /  68
//   rows 36:   8,           G 8,  2048        ( 28 MB)        49 /  40 /  29
//              8,           G 8,  8192        (112 MB)        66 /  62 /  51
//   rows 132: 16,           G 8,  4096        (112 MB)        99 /  95 /  78
//             32,           G 32, 4096        (248 MB)       153 / 143 / 125
// The device chooses between the first two, as only it knows what is shared: a
// call that shares little is slower than mds_cache_attend either way.
// So many bytes must be saved, by the rows of a sequence (few, many).
constexpr int64_t kWorthFew = 48 << 20, kWorthMany = 192 << 20;
// Weights, not bytes, bind rows of more than 16 a sequence, and a row's sums
// over the prefix are written and read again, whatever its length: of more than
// 8 rows a sequence each takes so many tokens saved.  Shared / not (this call),
// of 64 sequences in groups of 4 (a, 3/4 of a prefix saved a sequence) and 32 in
// groups of 16 (b, 15/16), by prefix:
//   rows 20: a 4096  123 / 179, b 4096  82 / 102
//   rows 36: a 4096  146 / 183, b 4096  98 / 103, 8192 124 / 166
//   rows 72: a 4096  248 / 214, 8192 362 / 349, b 4096 134 / 124, 8192 173 / 191
//   rows 80: a 4096  253 / 216, 8192 366 / 350, b 4096 138 / 123, 8192 175 / 192
//   rows 92: a 4096  260 / 219, 8192 373 / 352, b 4096 150 / 125, 8192 193 / 193
constexpr int64_t kWorthRow = 85;
// From about 100 rows on a tile of rows is full without other sequences'.
constexpr int kFullRows = 96;
// So are tiles of 8 or 16 rows of 32-bit queries, which the prefix's launch
// takes too, from three quarters on.  Shared / mds_cache_attend, 32 sequences
// over 16384 tokens: 1 row 61 / 199, 4 rows 117 / 199, 8 rows 191 / 200, 9 rows
// 216 / 324, 12 rows 276 / 324, 16 rows 351 / 325, 36 rows 769 / 939; 64 in
// groups of 32 over 4096: 8 rows 136 / 124, 12 rows 188 / 191, 16 rows 232 / 192.
bool full_rows(int dtype, int64_t own) {
  if (dtype != MDS_F32) return own > kFullRows;
  const int64_t tiles = own <= 8 ? 8 : (own + 15) / 16 * 16;
  return 4 * own > 3 * tiles;
}
// What is shared is known to the device alone, and the call without sharing is
// still four launches: where the tables have no room for savings at which
// mds_cache_attend falls behind (few rows: 37 us for 41 at 112 MB, 56 for 47 at
// 224), the host calls that.
constexpr int64_t kAloneFew = 160 << 20;

// Whose group place b of the list is in: its first and last place and one.
__device__ __forceinline__ int2 group_at(const Params& p, int b) {
  const int first = b / p.members * p.members, end = first + p.members, part = (b - first) / p.part * p.part;
  return int2{first + part, min(first + part + p.part, end)};
}

// One block of threads a sequence: the tokens that it shares with the first
// live sequence of its group (none if it is the only one), and its live nodes.
// With `prior` a group's first block marks its tiles of rows as not cut.
template <int D>
__global__ void __launch_bounds__(256) share_kernel(const __grid_constant__ Params p) {
  const State& s = p.s;
  const int32_t *seqs = p.a.seqs, *counts = p.a.counts;
  const int n = p.nodes, g0 = group_at(p, blockIdx.x).x, g1 = group_at(p, blockIdx.x).y;
  __shared__ int first_s, differ_s, others_s;
  const int tid = threadIdx.x, b = blockIdx.x;
  if (b == g0 && p.prior)
    for (int x = tid; x < s.kv_heads * p.row_tiles; x += 256)
      *reinterpret_cast<int2*>(prior_of<D>(p, row_at(p, b / p.members, x / p.row_tiles, x % p.row_tiles * p.rows_per)) + 2) = int2{-1, -1};
  if (tid == 0) first_s = INT_MAX, differ_s = INT_MAX, others_s = 0;
  __syncthreads();
  int id, len, live, end, q0, len0, live0;
  for (int i = g0 + tid; i < g1; i += 256) {
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

// What a call in several turns saves in all its groups, a thread a place, from
// what each place shares: one number, as plans take it.
__global__ void __launch_bounds__(MDS_CACHE_MAX_BATCH) total_kernel(const __grid_constant__ Params p) {
  __shared__ int from_s[MDS_CACHE_MAX_BATCH];
  __shared__ long long saved_s;
  const int b = threadIdx.x, first = group_at(p, b).x;
  const int2 x = b < p.a.B ? p.s.share[b] : int2{INT_MAX, 0};
  from_s[b] = INT_MAX;
  if (b == 0) saved_s = 0;
  __syncthreads();
  if (x.y > 0) atomicMin(&from_s[first], x.x);
  __syncthreads();
  const int from = from_s[first];
  long long saved = x.y > 0 ? from + (1ll << kLiveShift) : 0;
  if (b == first && from != INT_MAX) saved -= from;   // once for a group
  add_up(&saved_s, saved);
  __syncthreads();
  if (b == 0) *p.s.saved = saved_s;
}

// A row a warp: the pieces of its tile of rows, where that was cut, in their order.
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Params p) {
  constexpr int R = kPieceRow<D>, kEach = D / 32;
  const int lane = threadIdx.x & 31;
  const int per = (p.rows_per + 7) / 8, r = blockIdx.x % per * 8 + (threadIdx.x >> 5);
  const int rt = blockIdx.x / per % p.row_tiles, h = blockIdx.x / per / p.row_tiles % p.s.kv_heads;
  const int b = blockIdx.x / per / p.row_tiles / p.s.kv_heads, row = rt * p.rows_per + r;
  after_launch_before();
  if (r >= p.rows_per || row >= p.rows) return;
  const int2 cut = *reinterpret_cast<const int2*>(prior_of<D>(p, row_at(p, b, h, rt * p.rows_per)) + 2);
  if (cut.x < 0 || query_at<kPrefix>(p, b, row / p.g, p.a.n) == kNowhere) return;
  const int64_t stride = 2 * (int64_t)p.rows_per * R;
  const float* first = piece_of<D>(p, cut.x, true) + r * R;
  const float* later = piece_of<D>(p, cut.x, false) + r * R;   // + stride for each block further
  const int pieces = cut.y - cut.x + 1;
  auto at = [&](int c) { return c ? later + c * stride : first; };
  float top = kNone;
  for (int c = lane; c < pieces; c += 32) top = fmaxf(top, __ldcg(at(c)));
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
  float l = 0.f, o[kEach] = {};
  for (int c0 = 0; c0 < pieces; c0 += 32) {
    float2 y{kNone, 0.f};
    if (c0 + lane < pieces) y = __ldcg(reinterpret_cast<const float2*>(at(c0 + lane)));
    const float mine = ex2(y.x - top);
    l += y.y * mine;
#pragma unroll 8
    for (int c = c0; c < min(c0 + 32, pieces); ++c) {
      const float f = __shfl_sync(kFull, mine, c - c0);
      const float* x = at(c) + 4 + lane * kEach;
#pragma unroll
      for (int i = 0; i < kEach; i += 2) {
        const float2 z = __ldcg(reinterpret_cast<const float2*>(x + i));
        o[i] += f * z.x, o[i + 1] += f * z.y;
      }
    }
  }
#pragma unroll
  for (int d = 16; d; d /= 2) l += __shfl_xor_sync(kFull, l, d);
  float* to = prior_of<D>(p, row_at(p, b, h, row));
#pragma unroll
  for (int i = 0; i < kEach; i += 2) __stcg(reinterpret_cast<float2*>(to + 4 + lane * kEach + i), float2{o[i], o[i + 1]});
  if (lane == 0) __stcg(reinterpret_cast<float2*>(to), float2{top, l});
}

}  // namespace

cudaError_t attend_shared(const State& s, const Attend& a, int members, int64_t least, int sms, cudaStream_t st) {
  const int g = a.heads / s.kv_heads, groups = a.B / members;
  // As many sequences at a time as their rows' sums over the prefix have room
  // for: several groups, one, or, of groups larger than that, as equal parts as
  // go, each shared like a group of its own (a prefix read twice or three times
  // is still not read by every sequence).
  const int64_t at_once = ((int64_t)kPartFloats - kPieceFloats) / ((int64_t)a.n * a.heads * (s.head_dim + 4));
  const int64_t own = (int64_t)a.n * g;   // rows of one sequence
  const bool few_rows = s.dtype == MDS_F32 || own <= kFewRows;
  const bool choose = least < 0;
  if (members < 2 || at_once < 2 || (choose && full_rows(s.dtype, own))) return attend(s, a, sms, st);
  if (choose) least = few_rows ? kWorthFew : kWorthMany;
  const int64_t token = 2 * (int64_t)s.kv_heads * s.head_dim;
  const int64_t worth = least / token + (least % token != 0);   // tokens
  const int64_t each = choose && own > 8 ? kWorthRow * own : 0;    // of each live sequence
  const int parts = (int)((members + at_once - 1) / at_once), part = (members + parts - 1) / parts;
  // the most that the sequences' tables have room to share, in all and in a full part
  const int64_t room = (int64_t)s.max_pages * s.page_tokens;
  if (groups * (members - parts) * room < std::max(worth, choose && few_rows ? kAloneFew / token : 0) ||
      (part - 1) * room < each * part)
    return attend(s, a, sms, st);
  const int es = s.dtype == MDS_F32 ? 4 : 2;
  // In several turns no turn's own savings decide, and what is not worth
  // sharing is left to one launch over the whole call.
  const int together = parts > 1 ? 1 : (int)std::min((int64_t)groups, at_once / members);   // groups of a turn
  const bool turns = parts > 1 || together < groups;
  if (turns) {
    Params p{s, a, 0, g, 0, 0, 0, 0};
    p.members = members;
    p.part = part;
    p.nodes = a.n;
    if (s.head_dim == 64) share_kernel<64><<<a.B, 256, 0, st>>>(p);
    else share_kernel<128><<<a.B, 256, 0, st>>>(p);
    total_kernel<<<1, MDS_CACHE_MAX_BATCH, 0, st>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  for (int b0 = 0, some, of_each; b0 < a.B; b0 += some * of_each) {
    // some groups of so many members, or a part of one
    some = std::min(together, (a.B - b0) / members);
    of_each = members;
    if (parts > 1) some = 1, of_each = std::min(part, members - b0 % members);
    Attend x = a;
    x.B = some * of_each;
    x.seqs = a.seqs + b0;
    x.counts = a.counts ? a.counts + b0 : nullptr;
    x.q = static_cast<const char*>(a.q) + b0 * a.q_seq * es;
    x.out = static_cast<char*>(a.out) + (int64_t)b0 * a.n * a.heads * s.head_dim * es;
    Attend y = x;
    y.B = some;
    y.n = a.n * of_each;
    y.L = y.n - 1;
    Shared z{of_each, a.n, true, s.part + kPieceFloats, worth, each, turns ? s.saved : nullptr};
    const int64_t rows = (int64_t)y.n * g;
    const bool few = s.dtype == MDS_F32 || rows <= kFewRows, many = !few && rows <= kNarrow;
    Params p{s, y, 0, g, (int)rows, 0, 0, 0};
    // as the launch of the prefix cuts them
    p.rows_per = few ? (rows > 8 ? 16 : 8) : even_rows(rows, many ? kManyRows : kWideRows);
    p.row_tiles = (int)((rows + p.rows_per - 1) / p.rows_per);
    p.members = p.part = of_each;
    p.nodes = a.n;
    p.prior = z.prior;
    if (s.head_dim == 64) share_kernel<64><<<x.B, 256, 0, st>>>(p);
    else share_kernel<128><<<x.B, 256, 0, st>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess)
      e = few ? shared_few(s, y, z, sms, st) : many ? shared_many(s, y, z, sms, st) : shared_wide(s, y, z, sms, st);
    if (e == cudaSuccess) {
      const int blocks = some * s.kv_heads * p.row_tiles * ((p.rows_per + 7) / 8);
      e = launch_behind(s.head_dim == 64 ? join_kernel<64> : join_kernel<128>, blocks, 256, 0, st, p);
    }
    z.prefix = false;
    if (e == cudaSuccess)
      e = s.dtype == MDS_F32 ? shared_few(s, x, z, sms, st)
          : own <= 8 ? shared_rest(s, x, z, sms, st)
          : few_rows ? shared_few(s, x, z, sms, st) : shared_many(s, x, z, sms, st);
    if (e != cudaSuccess) return e;
  }
  if (turns) return attend(s, a, sms, st, Shared{1, a.n, false, nullptr, worth, each, s.saved});
  return cudaSuccess;
}

}  // namespace cache
}  // namespace mds
