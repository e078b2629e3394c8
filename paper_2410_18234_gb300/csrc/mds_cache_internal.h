// Internal interface of the key/value cache (declared in
// include/mds_cache.h) between its entry points (mds_cache_api.cu) and its
// kernels (mds_cache_pages.cu, mds_cache_few.cu, mds_cache_many.cu).
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
  float* part;        // attend's partial sums
  uint32_t* status;
  int layers, pages, page_tokens, page_log, kv_heads, head_dim, max_seqs, max_pages, dtype;
};

constexpr int kJoins = 1024;            // blocks of attend's grid at most
constexpr size_t kPartFloats = 16u << 20;

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

struct Attend {
  const int32_t* seqs;
  const int32_t* counts;
  const void* q;
  int64_t q_seq, q_tok, q_head;   // elements
  void* out;
  int layer, B, n, L, heads, window, sinks;
  float scale;
};
cudaError_t attend(const State& s, const Attend& a, int sms, cudaStream_t st);        // mds_cache_few.cu
cudaError_t attend_many(const State& s, const Attend& a, int sms, cudaStream_t st);   // mds_cache_many.cu
cudaError_t configure_many();
// Blocks of an attention kernel: one per SM, as far as the partial sums reach.
inline int attend_grid(int sms, int rows, int head_dim) {
  const size_t most = kPartFloats / (2 * (size_t)rows * (head_dim + 4));
  const int grid = sms < kJoins ? sms : kJoins;
  return (size_t)grid < most ? grid : (int)most;
}
cudaError_t configure();          // kernel attributes, on the current device

// Byte of (token row, dimension) inside a tile or a whole number of 128-byte lines of it.
__host__ __device__ __forceinline__ unsigned swizzled(unsigned byte) { return byte ^ (((byte >> 7) & 7u) << 4); }

}  // namespace cache
}  // namespace mds
