// Attention over the cache for few rows a key/value head and for 32-bit
// queries, and the choice between the two kernels.
#include "mds_cache_few.cuh"

namespace mds {
namespace cache {

cudaError_t configure() {
  cudaError_t e = configure_few<kAll>();
  if (e == cudaSuccess) e = configure_many();
  if (e == cudaSuccess) e = configure_shared_few();
  if (e == cudaSuccess) e = configure_shared_many();
  if (e == cudaSuccess) e = configure_rest();
  if (e == cudaSuccess) e = configure_wide();
  return e;
}

// Rows of 16-bit queries beyond 16 go to the kernel of mds_cache_many.cuh (which
// has no second term for 32-bit queries).  Both kernels, in us: 64 sequences of
// 500 to 2000 tokens with 32 heads, and 8 of 30000 to 60000 with 8:
//    8 rows: here 222, there 228    144, 193
//   16 rows: here 287, there 232    167, 193
//   17 rows: here 509, there 234    296, 193
cudaError_t attend(const State& s, const Attend& a, int sms, cudaStream_t st, const Shared& x) {
  if (s.dtype != MDS_F32 && (int64_t)a.n * (a.heads / s.kv_heads) > 16) return attend_many(s, a, sms, st, x);
  return attend_few<kAll>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
