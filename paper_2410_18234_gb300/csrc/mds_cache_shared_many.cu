// The two launches of attention over shared prefixes, many rows a key/value head.
#include "mds_cache_many.cuh"

namespace mds {
namespace cache {

cudaError_t configure_shared_many() {
  const cudaError_t e = configure_part<kPrefix>();
  return e == cudaSuccess ? configure_part<kRest>() : e;
}

cudaError_t shared_many(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  return x.prefix ? attend_part<kPrefix>(s, a, x, sms, st) : attend_part<kRest>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
