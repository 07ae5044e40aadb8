// ckv_check.hpp -- argument checks shared by the C ABI's sources.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <mutex>
#include <new>

#include "ckv.h"
#include "ckv_launch.hpp"

namespace ckv {

#define CKV_TRY_HIP(expr, what)                 \
  do {                                          \
    hipError_t e_ = (expr);                     \
    if (e_ != hipSuccess) return hip_fail(e_, what); \
  } while (0)

struct Dims {
  int B, Hq, Hkv, G, U, max_ctx;
  int64_t key_stride, kv_stride;
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_shape(const ckv_shape* s, Dims* d) {
  if (!s) return fail(CKV_EINVAL, "shape is NULL");
  if (s->reserved != 0) return fail(CKV_EINVAL, "shape.reserved must be 0");
  if (s->batch < 0 || s->num_q_heads < 1 || s->num_kv_heads < 1)
    return fail(CKV_ESHAPE, "batch=%d num_q_heads=%d num_kv_heads=%d", s->batch,
                s->num_q_heads, s->num_kv_heads);
  if (s->num_q_heads % s->num_kv_heads)
    return fail(CKV_ESHAPE, "num_q_heads %d not a multiple of num_kv_heads %d",
                s->num_q_heads, s->num_kv_heads);
  if (s->head_dim != kD)
    return fail(CKV_EUNSUPPORTED, "head_dim %d (only %d is supported)", s->head_dim, kD);
  const int G = s->num_q_heads / s->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8 && G != 16)
    return fail(CKV_EUNSUPPORTED, "group size %d not in {1,2,4,8,16}", G);
  if (s->max_ctx < 1 || s->max_ctx > (1 << 30))
    return fail(CKV_ESHAPE, "max_ctx %d outside [1, 2^30]", s->max_ctx);
  if (s->key_row_stride < kD || (s->key_row_stride & 7))
    return fail(CKV_ESHAPE, "key_row_stride %lld (>= 128, multiple of 8)",
                (long long)s->key_row_stride);
  if (s->kv_row_stride < kD || (s->kv_row_stride & 7))
    return fail(CKV_ESHAPE, "kv_row_stride %lld (>= 128, multiple of 8)",
                (long long)s->kv_row_stride);
  const int64_t units = (int64_t)s->batch * s->num_kv_heads;
  if (units > (1 << 24)) return fail(CKV_EUNSUPPORTED, "batch*num_kv_heads too large");
  d->B = s->batch;
  d->Hq = s->num_q_heads;
  d->Hkv = s->num_kv_heads;
  d->G = G;
  d->U = (int)units;
  d->max_ctx = s->max_ctx;
  d->key_stride = s->key_row_stride;
  d->kv_stride = s->kv_row_stride;
  return CKV_OK;
}

inline int check_k(int32_t k) {
  if (k < 1 || k > (1 << 20)) return fail(CKV_ESHAPE, "k %d outside [1, 2^20]", k);
  return CKV_OK;
}

inline int check_scale(float scale) {
  if (!(scale > 0.f) || scale > 3.0e38f)
    return fail(CKV_EINVAL, "scale must be a finite positive number");
  return CKV_OK;
}

#define CKV_PTR(p)                                                          \
  do {                                                                      \
    if (!(p)) return fail(CKV_EINVAL, "%s is NULL", #p);                    \
    if (!aligned16(p)) return fail(CKV_EINVAL, "%s is not 16-byte aligned", #p); \
  } while (0)

// A tag for one launch whose workgroups hand over to each other: a 32-bit value
// that is never zero in the high half and its complement in the low half.
inline uint64_t next_fused_tag() {
  static std::atomic<uint32_t> counter{0};
  uint32_t t = counter.fetch_add(1u, std::memory_order_relaxed) + 1u;
  t *= 2654435761u;  // spread consecutive calls over the 32 bits
  t |= 1u;
  return ((uint64_t)t << 32) | (uint32_t)~t;
}

// Words that are each held by one call at a time and kept until the process ends.
class FlagPool {
 public:
  struct Flag {
    unsigned long long* word;
    Flag* next;
  };
  // A free flag, or a new one whose word make(&word) gives (true: it did); NULL if
  // there is none to be had.
  template <class Make>
  Flag* take(Make make) {
    {
      std::lock_guard<std::mutex> lk(mu_);
      if (Flag* f = free_) {
        free_ = f->next;
        return f;
      }
    }
    Flag* f = new (std::nothrow) Flag{nullptr, nullptr};
    if (f && !make(&f->word)) {
      delete f;
      f = nullptr;
    }
    return f;
  }
  void give(Flag* f) {
    std::lock_guard<std::mutex> lk(mu_);
    f->next = free_;
    free_ = f;
  }

 private:
  std::mutex mu_;
  Flag* free_ = nullptr;
};

// Debug mode: runs launch(flag) on the stream, a check that leaves the smallest code
// of what it finds in *flag (all ones: nothing), and waits for it.  The flag is
// this call's own, so that calls of other threads and streams do not meet; one
// whose call failed is not used again (the device may still write it).
template <class Launch>
inline int debug_run(hipStream_t s, Launch launch, unsigned long long* got) {
  static FlagPool pools[256];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "debug check");
  if (dev < 0 || dev >= 256) return fail(CKV_EUNSUPPORTED, "device %d", dev);
  FlagPool::Flag* f = pools[dev].take([&](unsigned long long** word) {
    e = hipMalloc(word, 16);
    return e == hipSuccess;
  });
  if (!f) return hip_fail(e != hipSuccess ? e : hipErrorOutOfMemory, "debug check flag");
  if ((e = launch_fill(f->word, 16, 0xffffffffu, s)) != hipSuccess ||
      (e = launch(f->word)) != hipSuccess ||
      (e = hipMemcpyAsync(got, f->word, 8, hipMemcpyDeviceToHost, s)) != hipSuccess ||
      (e = hipStreamSynchronize(s)) != hipSuccess)
    return hip_fail(e, "debug check");
  pools[dev].give(f);
  return CKV_OK;
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace ckv
