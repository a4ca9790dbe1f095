// What the translation units of the library share: the context, the error paths, the current device of a call.
#ifndef EJOIN_CONTEXT_H
#define EJOIN_CONTEXT_H

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "ejoin.h"

// Words of a status block.  0 .. 3 and 8 .. 15 are the joins' (see k_reset); of the context's own block, two more that no join kernel reads or
// clears by itself: the pair counter of a join that is returned in batches, and what was wrong with tokens (ejoin_embed_status).
constexpr int EJ_STATUS_WORDS = 64;
constexpr int EJ_BATCH_COUNTER = 32;  // 64 bits: 32 and 33
constexpr int EJ_TOKEN_STATUS = 48;
static_assert(EJ_TOKEN_STATUS >= EJ_BATCH_COUNTER + 2 && EJ_TOKEN_STATUS < EJ_STATUS_WORDS, "words of their own");

// Device memory one call works in: either the context's own (grown on demand) or a carving of the static scratch.
struct Workspace {
  uint32_t* status;  // status block, EJ_STATUS_WORDS words (see above and k_reset)
  float* s;          // norms (4 B per point)
  uint32_t* maxima;  // behind them, small problems and the dense-tile call: largest norms of the norm kernels' workgroups (at most one per NORM_POINTS points)
  uint4* Xp;         // packed copy of X plus the augmentation k-block
};

struct ejoin_ctx {
  int device;
  int num_cu;
  Workspace ws;      // owned by the context
  int64_t s_cap;     // points ws.s holds
  int64_t xp_bytes;  // bytes of ws.Xp
  bool ws_dirty;     // a call on ws did not reach its join kernel: the status block may hold leftovers
  unsigned char* once;            // device: k_join_once's state, slots and late counts, all zero between calls
  unsigned char* static_scratch;  // device address of `scratch` on this context's device
  uint32_t* last_status;          // status block of the last join or dense-tile call, and the stream it ran on
  hipStream_t last_stream;
  int profiling;
  hipEvent_t ev[4];
  int ev_valid;
  // batched result return (ejoin_selfjoin_pairs_to_host): a stream for the device-to-host copies, one event per
  // batch and the pair counter's value after each batch (pinned host memory)
  hipStream_t copy_stream;
  hipEvent_t batch_ev[EJOIN_MAX_BATCHES];
  unsigned long long* batch_count;
  // ejoin_embed.h: memory its calls work in, grown on demand, and the device word in which they leave what was wrong with tokens
  unsigned char* embed;
  int64_t embed_bytes;
  bool embed_captured;      // a call that works in it was recorded into a graph: it stays where it is until the context ends
  unsigned char** retired;  // such memory that was grown out of
  int64_t num_retired;
  uint32_t* token_status;  // word EJ_TOKEN_STATUS of the context's own status block
  uint32_t* tickets;       // device: EJ_TICKETS counters, all zero between calls
  char hip_error[256];
};

constexpr int EJ_TICKETS = 4096;

// What the kernels of f8.hip need once on a device, which is current.
__attribute__((visibility("hidden"))) hipError_t f8_prepare_kernels();

inline int fail_hip(ejoin_ctx* ctx, hipError_t e, const char* what) {
  if (ctx) snprintf(ctx->hip_error, sizeof(ctx->hip_error), "%s: %s", what, hipGetErrorString(e));
  (void)hipGetLastError();
  return EJOIN_EHIP;
}

#define EJ_TRY(call)                                     \
  do {                                                   \
    hipError_t e_ = (call);                              \
    if (e_ != hipSuccess) return fail_hip(ctx, e_, #call); \
  } while (0)
#define EJ_RC(call)                 \
  do {                              \
    const int rc_ = (call);         \
    if (rc_ != EJOIN_OK) return rc_; \
  } while (0)

struct DeviceGuard {
  int prev;
  bool ok;
  explicit DeviceGuard(int dev) : prev(-1), ok(false) {
    if (hipGetDevice(&prev) != hipSuccess) return;
    ok = (prev == dev) || (hipSetDevice(dev) == hipSuccess);
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

#endif  // EJOIN_CONTEXT_H
