// Entry points of the key/value cache (include/mds_cache.h): argument checks,
// the layout of the caller's memory, and the launches.
#include <cmath>
#include <new>
#include <type_traits>

#include "mds_cache_internal.h"
#include "mds_internal.h"

struct mds_cache {
  mds_cache_config cfg;
  int device;
  int sms;
  mds::cache::State s;
};

namespace {

using mds::cache::State;

struct DeviceGuard {
  int prev = -1;
  explicit DeviceGuard(int dev) {
    cudaGetDevice(&prev);
    if (prev != dev) cudaSetDevice(dev);
  }
  ~DeviceGuard() {
    int cur = -1;
    cudaGetDevice(&cur);
    if (prev >= 0 && cur != prev) cudaSetDevice(prev);
  }
};

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

int esize_of(int dtype) { return dtype == MDS_F32 ? 4 : 2; }

bool valid(const mds_cache_config& c) {
  return c.layers >= 1 && c.layers <= 1024 && c.pages >= 1 && c.pages <= (1 << 24) &&
         (c.page_tokens == 16 || c.page_tokens == 32 || c.page_tokens == 64 || c.page_tokens == 128) &&
         c.kv_heads >= 1 && c.kv_heads <= 1024 && (c.head_dim == 64 || c.head_dim == 128) && c.max_seqs >= 1 &&
         c.max_seqs <= (1 << 20) && c.max_pages >= 1 && c.max_pages <= (1 << 16) &&
         (int64_t)c.max_pages * c.page_tokens <= MDS_CACHE_MAX_TOKENS;
}

// Lay the state out from `base` on (null: only its size).  Returns the bytes.
size_t carve(const mds_cache_config& c, char* base, State& s) {
  size_t at = 0;
  auto take = [&](auto*& ptr, size_t bytes) {
    ptr = reinterpret_cast<std::remove_reference_t<decltype(ptr)>>(base + at);
    at += (bytes + 1023) / 1024 * 1024;
  };
  const size_t tiles = (size_t)c.layers * c.pages * 2 * c.kv_heads;
  take(s.pool, tiles * c.page_tokens * c.head_dim);
  take(s.scales, tiles * (c.page_tokens / MDS_CACHE_BLOCK) * 4);
  take(s.table, (size_t)c.max_seqs * c.max_pages * 4);
  take(s.lens, (size_t)c.max_seqs * 4);
  take(s.held, (size_t)c.max_seqs * 4);
  take(s.reach, (size_t)c.max_seqs * 4);
  take(s.ref, (size_t)c.pages * 4);
  take(s.freemap, ((size_t)c.pages + 127) / 128 * 16);
  take(s.fresh, (size_t)c.pages * 4);
  take(s.copies, (size_t)c.pages * 12);
  take(s.kept, (size_t)MDS_CACHE_MAX_BATCH * 8);
  take(s.arrive, (size_t)c.max_seqs * 4);
  take(s.joins, mds::cache::kJoins * 4);
  take(s.share, (size_t)MDS_CACHE_MAX_BATCH * 8);
  take(s.free_count, 64);
  s.n_copies = s.free_count + 1;
  s.status = reinterpret_cast<uint32_t*>(s.free_count + 2);
  s.saved = reinterpret_cast<int64_t*>(s.free_count + 4);
  take(s.part, mds::cache::kPartFloats * 4);
  s.layers = c.layers;
  s.pages = c.pages;
  s.page_tokens = c.page_tokens;
  s.page_log = c.page_tokens == 16 ? 4 : c.page_tokens == 32 ? 5 : c.page_tokens == 64 ? 6 : 7;
  s.kv_heads = c.kv_heads;
  s.head_dim = c.head_dim;
  s.max_seqs = c.max_seqs;
  s.max_pages = c.max_pages;
  s.dtype = c.dtype;
  return at;
}

int done(cudaError_t e, const char* where) { return e == cudaSuccess ? MDS_OK : mds::record_cuda_error(e, where); }

// The checks that every call on a batch shares: MDS_OK, or the code to return.
int batch(const mds_cache* c, const int32_t* seqs, int B) {
  if (!c) return MDS_EINVAL;
  if (B < 0 || B > MDS_CACHE_MAX_BATCH) return MDS_ESHAPE;
  if (B > 0 && (!seqs || !aligned(seqs, 4))) return MDS_EINVAL;
  return MDS_OK;
}

// Rows that 16-byte loads can read: base and strides.
bool rows_ok(const void* p, const int64_t* strides, int es) {
  if (!p || !strides || !aligned(p, 16)) return false;
  for (int i = 0; i < 3; ++i)
    if (strides[i] * es % 16 != 0) return false;
  return true;
}

bool rotary_ok(const mds_cache_rotary* r) {
  return r && (r->interleaved == 0 || r->interleaved == 1) && r->magnitude >= 0x1p-20 && r->magnitude <= 0x1p20;
}
bool dim_ok(int dim, int head_dim) { return dim >= 16 && dim <= head_dim && dim % 16 == 0; }

cudaStream_t stream_of(void* s) { return static_cast<cudaStream_t>(s); }

}  // namespace

extern "C" {

size_t mds_cache_bytes(const mds_cache_config* cfg) {
  if (!cfg || !valid(*cfg) || (cfg->dtype != MDS_F32 && cfg->dtype != MDS_BF16)) return 0;
  State s{};
  return carve(*cfg, nullptr, s);
}

int mds_cache_create(mds_cache** out, const mds_cache_config* cfg, int device, void* memory, void* stream) {
  if (!out || !cfg) return MDS_EINVAL;
  *out = nullptr;
  if (cfg->dtype != MDS_F32 && cfg->dtype != MDS_BF16) return MDS_EINVAL;
  if (!valid(*cfg)) return MDS_ESHAPE;
  if (!memory || !aligned(memory, 1024)) return MDS_EINVAL;
  int ndev = 0;
  cudaError_t e = cudaGetDeviceCount(&ndev);
  if (e != cudaSuccess) return done(e, "cudaGetDeviceCount");
  if (device < 0 || device >= ndev) return done(cudaErrorInvalidDevice, "mds_cache_create");
  DeviceGuard g(device);
  mds_cache* c = new (std::nothrow) mds_cache{};
  if (!c) return done(cudaErrorMemoryAllocation, "mds_cache_create");
  c->cfg = *cfg;
  c->device = device;
  const size_t bytes = carve(*cfg, static_cast<char*>(memory), c->s);
  const cudaStream_t st = stream_of(stream);
  e = cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = mds::cache::configure();
  // every byte of the pool is a finite number from the start on; the partial
  // sums at the end need no clearing
  if (e == cudaSuccess) e = cudaMemsetAsync(memory, 0, bytes - mds::cache::kPartFloats * 4, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(c->s.table, 0xff, (size_t)cfg->max_seqs * cfg->max_pages * 4, st);
  if (e == cudaSuccess) e = mds::cache::clear(c->s, st);
  if (e != cudaSuccess) {
    delete c;
    return done(e, "mds_cache_create");
  }
  *out = c;
  return MDS_OK;
}

int mds_cache_state(const mds_cache* c, const int32_t** lens, const int32_t** table) {
  if (!c) return MDS_EINVAL;
  if (lens) *lens = c->s.lens;
  if (table) *table = c->s.table;
  return MDS_OK;
}

int mds_cache_reserve(mds_cache* c, const int32_t* seqs, const int32_t* counts, int n, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (n < 0 || n > MDS_CACHE_MAX_TOKENS) return MDS_ESHAPE;
  if (counts && !aligned(counts, 4)) return MDS_EINVAL;
  if (B == 0 || n == 0) return MDS_OK;
  DeviceGuard g(c->device);
  return done(mds::cache::reserve(c->s, seqs, counts, n, B, stream_of(stream)), "mds_cache_reserve");
}

int mds_cache_append(mds_cache* c, int layer, const int32_t* seqs, const int32_t* counts, const void* k,
                     const int64_t* k_strides, const void* v, const int64_t* v_strides, int n, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (layer < 0 || layer >= c->cfg.layers || n < 0 || n > MDS_CACHE_MAX_TOKENS) return MDS_ESHAPE;
  if (B == 0 || n == 0) return MDS_OK;
  // one block of threads for eight blocks of tokens and heads
  if ((int64_t)B * ((n + 30) / MDS_CACHE_BLOCK) * c->cfg.kv_heads / 4 >= INT32_MAX) return MDS_ESHAPE;
  const int es = esize_of(c->cfg.dtype);
  if (!rows_ok(k, k_strides, es) || !rows_ok(v, v_strides, es) || (counts && !aligned(counts, 4))) return MDS_EINVAL;
  DeviceGuard g(c->device);
  return done(mds::cache::append(c->s, layer, seqs, counts, k, k_strides, v, v_strides, n, B, stream_of(stream)),
              "mds_cache_append");
}

int mds_cache_rotary_init(mds_cache_rotary* rotary, const double* freqs, int dim, int interleaved, double magnitude) {
  if (!rotary || !freqs) return MDS_EINVAL;
  if (!dim_ok(dim, 128)) return MDS_ESHAPE;
  mds_cache_rotary r{dim, interleaved, magnitude, {}};
  if (!rotary_ok(&r)) return MDS_EINVAL;
  // 1 / (2 pi) in two parts: the turn is off by 2^-64, not by the 2^-53 of one product
  constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;
  for (int i = 0; i < dim / 2; ++i) {
    const double f = freqs[i];
    if (!(std::fabs(f) <= 3.14159265358979312)) return MDS_EINVAL;
    const double h = f * kHigh, l = std::fma(f, kHigh, -h) + f * kLow;
    // either part in units of 2^-64 modulo 2^64; |h| may be a half, 2^63 units
    r.turns[i] = 2 * (uint64_t)(int64_t)std::llrint(std::ldexp(h, 63)) +
                 (uint64_t)(int64_t)std::llrint(std::ldexp(h, 64) - 2 * (double)std::llrint(std::ldexp(h, 63)) + std::ldexp(l, 64));
  }
  *rotary = r;
  return MDS_OK;
}

int mds_cache_rotate(mds_cache* c, const int32_t* seqs, const int32_t* counts, const mds_cache_rotary* rotary,
                     const void* x, const int64_t* x_strides, void* out, int heads, int n, int branches, int B,
                     void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (!rotary_ok(rotary)) return MDS_EINVAL;
  if (!dim_ok(rotary->dim, c->cfg.head_dim) || n < 0 || n > MDS_CACHE_MAX_TOKENS || branches < 1 || heads < 1 ||
      heads > 65536 || (n > 0 && (n - 1) % branches))
    return MDS_ESHAPE;
  if (B == 0 || n == 0) return MDS_OK;
  const int es = esize_of(c->cfg.dtype);
  if (!rows_ok(x, x_strides, es) || !out || !aligned(out, 16) || (counts && !aligned(counts, 4))) return MDS_EINVAL;
  DeviceGuard g(c->device);
  mds::cache::Rotate a{rotary, seqs, counts, nullptr, nullptr, nullptr, nullptr, x, x_strides, out, 0, heads, n,
                       (n - 1) / branches, B};
  return done(mds::cache::rotate(c->s, a, stream_of(stream)), "mds_cache_rotate");
}

int mds_cache_append_rotated(mds_cache* c, int layer, const int32_t* seqs, const int32_t* counts,
                             const mds_cache_rotary* rotary, const void* k, const int64_t* k_strides, const void* v,
                             const int64_t* v_strides, const void* q, const int64_t* q_strides, void* q_out,
                             int q_heads, int n, int branches, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (!rotary_ok(rotary)) return MDS_EINVAL;
  if (!dim_ok(rotary->dim, c->cfg.head_dim) || layer < 0 || layer >= c->cfg.layers || n < 0 ||
      n > MDS_CACHE_MAX_TOKENS || branches < 1 || (n > 0 && (n - 1) % branches) ||
      (q && (q_heads < 1 || q_heads > 65536)))
    return MDS_ESHAPE;
  if (B == 0 || n == 0) return MDS_OK;
  const int es = esize_of(c->cfg.dtype);
  if (!rows_ok(k, k_strides, es) || !rows_ok(v, v_strides, es) || (counts && !aligned(counts, 4)) ||
      (q && (!rows_ok(q, q_strides, es) || !q_out || !aligned(q_out, 16))))
    return MDS_EINVAL;
  DeviceGuard g(c->device);
  mds::cache::Rotate a{rotary, seqs, counts, k, k_strides, v, v_strides, q, q_strides, q_out, layer, q ? q_heads : 0, n,
                       (n - 1) / branches, B};
  return done(mds::cache::rotate(c->s, a, stream_of(stream)), "mds_cache_append_rotated");
}

static int attend_call(mds_cache* c, int layer, const int32_t* seqs, const int32_t* counts, const void* q,
                       const int64_t* q_strides, void* out, int q_heads, int n, int branches, int window, int sinks,
                       float scale, int group, int64_t least, int B, void* stream, const char* name) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (layer < 0 || layer >= c->cfg.layers || n < 0 || n > MDS_CACHE_MAX_NODES || branches < 1 || q_heads < 1 ||
      q_heads % c->cfg.kv_heads || q_heads / c->cfg.kv_heads > MDS_CACHE_MAX_GROUP || group < 1 || B % group)
    return MDS_ESHAPE;
  if (n > 0 && (n - 1) % branches) return MDS_ESHAPE;
  if (window < 0 || sinks < 0 || !(scale - scale == 0.f)) return MDS_EINVAL;
  if (B == 0 || n == 0) return MDS_OK;
  if (!rows_ok(q, q_strides, esize_of(c->cfg.dtype)) || !out || !aligned(out, 16) || (counts && !aligned(counts, 4)))
    return MDS_EINVAL;
  DeviceGuard g(c->device);
  mds::cache::Attend a{seqs, counts, q, q_strides[0], q_strides[1], q_strides[2], out, layer, B, n,
                       (n - 1) / branches, q_heads, window, sinks, scale};
  return done(group > 1 ? mds::cache::attend_shared(c->s, a, group, least, c->sms, stream_of(stream))
                        : mds::cache::attend(c->s, a, c->sms, stream_of(stream)), name);
}

int mds_cache_attend(mds_cache* c, int layer, const int32_t* seqs, const int32_t* counts, const void* q,
                     const int64_t* q_strides, void* out, int q_heads, int n, int branches, int window, int sinks,
                     float scale, int B, void* stream) {
  return attend_call(c, layer, seqs, counts, q, q_strides, out, q_heads, n, branches, window, sinks, scale, 1, 0, B, stream,
                     "mds_cache_attend");
}

int mds_cache_attend_shared(mds_cache* c, int layer, const int32_t* seqs, const int32_t* counts, const void* q,
                            const int64_t* q_strides, void* out, int q_heads, int n, int branches, int group,
                            float scale, int64_t least_saved, int B, void* stream) {
  return attend_call(c, layer, seqs, counts, q, q_strides, out, q_heads, n, branches, 0, 0, scale, group, least_saved, B, stream,
                     "mds_cache_attend_shared");
}

int mds_cache_commit(mds_cache* c, const int32_t* seqs, const int32_t* accept_len, const int32_t* draft_tokens,
                     const int32_t* out_tokens, int K, int L, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (K < 1 || L < 0 || (int64_t)K * L >= MDS_CACHE_MAX_TOKENS) return MDS_ESHAPE;
  if (B == 0) return MDS_OK;
  if (L == 0) draft_tokens = out_tokens = nullptr;   // the root alone: no branch to find
  if (!accept_len || !aligned(accept_len, 4) || !draft_tokens != !out_tokens || !aligned(draft_tokens, 4) ||
      !aligned(out_tokens, 4))
    return MDS_EINVAL;
  DeviceGuard g(c->device);
  return done(mds::cache::commit(c->s, seqs, accept_len, draft_tokens, out_tokens, K, L, B, stream_of(stream)),
              "mds_cache_commit");
}

int mds_cache_fork(mds_cache* c, const int32_t* src, const int32_t* dst, int B, void* stream) {
  const int rc = batch(c, src, B);
  if (rc != MDS_OK) return rc;
  if (B == 0) return MDS_OK;
  if (!dst || !aligned(dst, 4)) return MDS_EINVAL;
  DeviceGuard g(c->device);
  return done(mds::cache::fork(c->s, src, dst, B, stream_of(stream)), "mds_cache_fork");
}

int mds_cache_truncate(mds_cache* c, const int32_t* seqs, const int32_t* lens, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (B == 0) return MDS_OK;
  if (!lens || !aligned(lens, 4)) return MDS_EINVAL;
  DeviceGuard g(c->device);
  return done(mds::cache::truncate(c->s, seqs, lens, B, stream_of(stream)), "mds_cache_truncate");
}

int mds_cache_free(mds_cache* c, const int32_t* seqs, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (B == 0) return MDS_OK;
  DeviceGuard g(c->device);
  return done(mds::cache::truncate(c->s, seqs, nullptr, B, stream_of(stream)), "mds_cache_free");
}

int mds_cache_read(mds_cache* c, int layer, const int32_t* seqs, const int32_t* start, const int32_t* counts, void* k,
                   void* v, int n, int B, void* stream) {
  const int rc = batch(c, seqs, B);
  if (rc != MDS_OK) return rc;
  if (layer < -1 || layer >= c->cfg.layers || n < 0 || n > MDS_CACHE_MAX_TOKENS) return MDS_ESHAPE;
  if (B == 0 || n == 0) return MDS_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16) || (start && !aligned(start, 4)) || (counts && !aligned(counts, 4)))
    return MDS_EINVAL;
  DeviceGuard g(c->device);
  return done(mds::cache::read(c->s, layer, seqs, start, counts, k, v, n, B, stream_of(stream)), "mds_cache_read");
}

int mds_cache_status(mds_cache* c, const char** msg) {
  if (!c) return MDS_EINVAL;
  DeviceGuard g(c->device);
  uint32_t bits = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(&bits, c->s.status, 4, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && bits) e = cudaMemset(c->s.status, 0, 4);
  if (e != cudaSuccess) return done(e, "mds_cache_status");
  if (msg)
    *msg = bits & MDS_ST_BADSEQ    ? "a sequence id out of range, a fork onto a sequence that holds pages, or tokens "
                                     "that were not reserved"
           : bits & MDS_ST_NOPAGES ? "too few free pages, or a page table too short; no pages given"
           : bits & MDS_ST_BADTOKEN ? "emitted tokens of no branch; branch 0 kept"
                                    : mds::status_message(bits);
  if (msg && bits == MDS_ST_NONFINITE) *msg = "a key or value was not finite (0, or the block's largest number, stored)";
  return (int)bits;
}

void mds_cache_destroy(mds_cache* c) { delete c; }

}  // extern "C"
