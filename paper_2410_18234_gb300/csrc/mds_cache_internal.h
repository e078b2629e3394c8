// Internal interface of the key/value cache (declared in
// include/mds_cache.h) between its entry points (mds_cache_api.cu) and its
// kernels (the other mds_cache_*.cu).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/mds_cache.h"

namespace mds {
namespace cache {

constexpr int kBlock = MDS_CACHE_BLOCK;

// The cache's memory.  A tile is one (page, key or value, head): page_tokens
// rows of head_dim bytes, its 16-byte units permuted within each 128 bytes
// (unit index ^= 128-byte line index mod 8), so that a plain copy of a tile
// into shared memory can be read by rows and by columns without bank
// conflicts, and is the 128-byte swizzle that matrix instructions take.
struct State {
  uint8_t* pool;      // [layers][pages][2][kv_heads][page_tokens][head_dim]
  float* scales;      // [layers][pages][2][kv_heads][page_tokens / 16]
  int32_t* table;     // [max_seqs][max_pages], -1 behind the held pages
  int32_t* lens;      // [max_seqs] committed tokens
  int32_t* held;      // [max_seqs] pages held
  int32_t* reach;     // [max_seqs] slots reserved: lens <= reach <= held * page_tokens
  int32_t* ref;       // [pages] sequences that hold the page
  uint32_t* freemap;  // [ceil(pages / 128) * 4] bit set: the page is free
  int32_t* free_count;
  int32_t* fresh;     // [pages] workspace of reserve: the pages it hands out
  int32_t* copies;    // [pages][3] workspace of reserve: page, its copy, tokens
  int32_t* n_copies;
  int32_t* kept;      // [MDS_CACHE_MAX_BATCH][2] workspace of commit: tokens kept behind the root, and how far they move
  uint32_t* arrive;   // [max_seqs] arrivals of commit's blocks, 0 between calls
  uint32_t* joins;    // [kJoins] arrivals of attend's pieces, 0 between calls
  int2* share;        // [MDS_CACHE_MAX_BATCH] attend over prefixes: tokens shared with the group's first, live nodes
  float* part;        // attend's partial sums; from kPieceFloats on rows' sums over a prefix
  uint32_t* status;
  int64_t* saved;     // attend over prefixes in several turns: what the whole call saves
  int layers, pages, page_tokens, page_log, kv_heads, head_dim, max_seqs, max_pages, dtype;
};

constexpr int kJoins = 1024;            // blocks of attend's grid at most
constexpr size_t kPartFloats = 16u << 20;
constexpr size_t kPieceFloats = kPartFloats / 8 * 5;   // of it, for pieces where sums over a prefix take the rest

cudaError_t reserve(const State& s, const int32_t* seqs, const int32_t* counts, int n, int B, cudaStream_t st);
cudaError_t append(const State& s, int layer, const int32_t* seqs, const int32_t* counts, const void* k,
                   const int64_t* ks, const void* v, const int64_t* vs, int n, int B, cudaStream_t st);
cudaError_t commit(const State& s, const int32_t* seqs, const int32_t* accept, const int32_t* drafts,
                   const int32_t* out_tokens, int K, int L, int B, cudaStream_t st);
cudaError_t fork(const State& s, const int32_t* src, const int32_t* dst, int B, cudaStream_t st);
// lens null: empty the sequences
cudaError_t truncate(const State& s, const int32_t* seqs, const int32_t* lens, int B, cudaStream_t st);
cudaError_t read(const State& s, int layer, const int32_t* seqs, const int32_t* start, const int32_t* counts, void* k,
                 void* v, int n, int B, cudaStream_t st);
cudaError_t clear(const State& s, cudaStream_t st);

// Heads rotated by their nodes' positions; with k, keys and values stored.
struct Rotate {
  const mds_cache_rotary* rotary;
  const int32_t* seqs;
  const int32_t* counts;
  const void* k;
  const int64_t* ks;
  const void* v;
  const int64_t* vs;
  const void* q;
  const int64_t* qs;
  void* out;
  int layer, heads, n, L, B;
};
cudaError_t rotate(const State& s, const Rotate& a, cudaStream_t st);   // mds_cache_rotary.cu

struct Attend {
  const int32_t* seqs;
  const int32_t* counts;
  const void* q;
  int64_t q_seq, q_tok, q_head;   // elements
  void* out;
  int layer, B, n, L, heads, window, sinks;
  float scale;
};
// Groups of `members` sequences of the list, over their common prefix and each
// over its rest (mds_cache_shared.cu; the launches: _shared_few.cu, _shared_many.cu).
cudaError_t attend_shared(const State& s, const Attend& a, int members, int64_t least, int sms, cudaStream_t st);
struct Shared {
  int members = 1, nodes = 0;
  bool prefix = false;     // the prefix's launch; else the rest's
  float* prior = nullptr;
  int64_t worth = 0, each = 0;     // tokens that must be saved in all, and for each live sequence
  const int64_t* saved = nullptr;  // of the call, where it has several turns
};
// x: where it has `saved`, the launch is for what is not worth sharing, and is over at once where it is.
cudaError_t attend(const State& s, const Attend& a, int sms, cudaStream_t st, const Shared& x = {});        // mds_cache_few.cu
cudaError_t attend_many(const State& s, const Attend& a, int sms, cudaStream_t st, const Shared& x = {});   // mds_cache_many.cu
// Rows of a tile of rows in the prefix's launch, by the kernel that it is.
inline int even_rows(int64_t rows, int most) {   // as even as it goes
  const int64_t tiles = (rows + most - 1) / most;
  return (int)((rows + tiles - 1) / tiles);
}
constexpr int kFewRows = 16, kManyRows = 144, kWideRows = 256;
cudaError_t shared_few(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st);
cudaError_t shared_many(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st);
cudaError_t shared_rest(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st);   // mds_cache_rest.cu
cudaError_t configure_rest();
cudaError_t shared_wide(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st);   // mds_cache_wide.cu
cudaError_t configure_wide();
cudaError_t configure_many();
cudaError_t configure_shared_few();
cudaError_t configure_shared_many();
// Blocks of an attention kernel: one per SM, as far as the partial sums reach.
inline int attend_grid(int sms, int rows, int head_dim, size_t floats = kPartFloats) {
  const size_t most = floats / (2 * (size_t)rows * (head_dim + 4));
  const int grid = sms < kJoins ? sms : kJoins;
  return (size_t)grid < most ? grid : (int)most;
}
cudaError_t configure();          // kernel attributes, on the current device

// Byte of (token row, dimension) inside a tile or a whole number of 128-byte lines of it.
__host__ __device__ __forceinline__ unsigned swizzled(unsigned byte) { return byte ^ (((byte >> 7) & 7u) << 4); }

}  // namespace cache
}  // namespace mds
