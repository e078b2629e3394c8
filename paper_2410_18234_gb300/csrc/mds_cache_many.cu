// Attention over the cache for many rows a key/value head.
#include "mds_cache_many.cuh"

namespace mds {
namespace cache {

cudaError_t configure_many() { return configure_part<kAll>(); }

cudaError_t attend_many(const State& s, const Attend& a, int sms, cudaStream_t st, const Shared& x) {
  return attend_part<kAll>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
