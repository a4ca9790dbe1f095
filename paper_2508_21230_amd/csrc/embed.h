// What the kernels of ejoin_embed.h share: element types, rows read and written in pieces of eight, the context's memory.
#ifndef EJOIN_EMBED_INTERNAL_H
#define EJOIN_EMBED_INTERNAL_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "context.h"
#include "ejoin_embed.h"

namespace {

// ------------------------------------------------------------------------------------------ element types
typedef _Float16 f16;
typedef __bf16 bf16;

template <typename T>
struct Element;
template <>
struct Element<float> {
  static constexpr int type = EJOIN_F32;
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Element<f16> {
  static constexpr int type = EJOIN_F16;
  static __device__ __forceinline__ float get(f16 x) { return (float)x; }
  static __device__ __forceinline__ f16 put(float x) { return (f16)x; }
};
template <>
struct Element<bf16> {
  static constexpr int type = EJOIN_BF16;
  static __device__ __forceinline__ float get(bf16 x) { return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, x) << 16); }
  static __device__ __forceinline__ bf16 put(float x) { return (bf16)x; }
};

// Eight elements of a row, at any address: the memory pipeline takes vector accesses that are not aligned, the compiler only has to be told.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight {
  T x[8];
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  const Eight<T> e = *reinterpret_cast<const Eight<T>*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = Element<T>::get(e.x[i]);
}

// ... of which the first `have` (0 .. 8) exist; zeros in the others' place.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int have, float (&x)[8]) {
  if (have >= 8) {
    load8(p, x);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = i < have ? Element<T>::get(p[i]) : 0.f;
}

// PASSING: what no one reads soon, past the caches.
template <typename T, bool PASSING = false>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  Eight<T> e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.x[i] = Element<T>::put(x[i]);
  if constexpr (PASSING) {
    typedef uint32_t Words __attribute__((ext_vector_type(2 * sizeof(T)), aligned(sizeof(T))));
    __builtin_nontemporal_store(__builtin_bit_cast(Words, e), reinterpret_cast<Words*>(p));
  } else {
    *reinterpret_cast<Eight<T>*>(p) = e;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, int have, const float (&x)[8]) {
  if (have >= 8) {
    store8(p, x);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < have) p[i] = Element<T>::put(x[i]);
}

// ------------------------------------------------------------------------------------------ host side
inline bool bad_type(int32_t type) { return type != EJOIN_F32 && type != EJOIN_F16 && type != EJOIN_BF16; }
inline int64_t size_of(int32_t type) { return type == EJOIN_F32 ? 4 : 2; }
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// A launch has fewer than 2^32 threads: so many workgroups, of 1,024 threads at most, are one launch's.
constexpr int64_t MOST_GROUPS = 1ll << 21;
// launch(first, groups) for `groups` workgroups in as many launches as that takes.
template <typename F>
void in_launches(int64_t groups, F launch) {
  for (int64_t first = 0; first < groups; first += MOST_GROUPS) launch(first, (unsigned)(groups - first < MOST_GROUPS ? groups - first : MOST_GROUPS));
}

// f(T()) with the type that `type` names.
template <typename F>
auto with_type(int32_t type, F f) {
  switch (type) {
    case EJOIN_F16: return f(f16());
    case EJOIN_BF16: return f(bf16());
    default: return f(float());
  }
}

// The context's memory for these calls, at least `bytes` of it.  Growing frees the old, which first waits for the device to be idle; but memory that a
// captured graph may come back to is kept, and nothing is waited for then.
inline int ensure_embed(ejoin_ctx* ctx, int64_t bytes) {
  if (bytes <= ctx->embed_bytes) return EJOIN_OK;
  if (ctx->embed && ctx->embed_captured) {
    unsigned char** more = static_cast<unsigned char**>(realloc(ctx->retired, (size_t)(ctx->num_retired + 1) * sizeof(*more)));
    if (!more) return EJOIN_ENOMEM;
    ctx->retired = more;
    ctx->retired[ctx->num_retired++] = ctx->embed;
    ctx->embed_captured = false;
  } else if (ctx->embed) {
    EJ_TRY(hipDeviceSynchronize());
    EJ_TRY(hipFree(ctx->embed));
  }
  ctx->embed = nullptr;
  ctx->embed_bytes = 0;
  const hipError_t e = hipMalloc(reinterpret_cast<void**>(&ctx->embed), (size_t)bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    ctx->embed = nullptr;
    if (e == hipErrorOutOfMemory) return EJOIN_ENOMEM;
    return fail_hip(ctx, e, "hipMalloc(memory of ejoin_embed.h)");
  }
  ctx->embed_bytes = bytes;
  return EJOIN_OK;
}

// ... for a call on stream st.
inline int ensure_embed(ejoin_ctx* ctx, int64_t bytes, hipStream_t st) {
  EJ_RC(ensure_embed(ctx, bytes));
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &capture) != hipSuccess) (void)hipGetLastError();  // (the launches will say what is wrong with the stream)
  if (capture != hipStreamCaptureStatusNone) ctx->embed_captured = true;
  return EJOIN_OK;
}

}  // namespace

#endif  // EJOIN_EMBED_INTERNAL_H
