// The two launches of attention over shared prefixes, few rows a key/value head.
#include "mds_cache_few.cuh"

namespace mds {
namespace cache {

cudaError_t configure_shared_few() {
  const cudaError_t e = configure_few<kPrefix>();
  return e == cudaSuccess ? configure_few<kRest>() : e;
}

cudaError_t shared_few(const State& s, const Attend& a, const Shared& x, int sms, cudaStream_t st) {
  return x.prefix ? attend_few<kPrefix>(s, a, x, sms, st) : attend_few<kRest>(s, a, x, sms, st);
}

}  // namespace cache
}  // namespace mds
