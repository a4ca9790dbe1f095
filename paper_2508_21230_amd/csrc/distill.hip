// The loss that fits a row's scores to a short list of ids with logits (Kullback-Leibler divergence of the two softmaxes), and
// its gradient.
//
// A row's statistics are (top, sum): its largest score, and the sum of 2^(c (z - top)), c = log2(e) / T; q = 2^(c (z - top)) / sum.  The
// difference comes first: scores as large as FP32 holds (masks) leave no more error in it than others.
//   loss = T^2 sum_k p_k (log p_k - log q_k),  p the softmax of the list's logits / T over its entries;  dz_v = weight T (q_v - sum of the p_k with id v)
// A row without entries has no loss and a gradient of zeros.
#include <type_traits>

#include "embed.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int MOST_ENTRIES = EJOIN_DISTILL_MAX_ENTRIES;
constexpr int LONG_THREADS = 512;
constexpr int MOST_SPLITS = 256;
constexpr int MOST_TICKETS = EJ_TICKETS;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// No scores, or -infinity alone: (-infinity, 0).  A NaN or +infinity among the scores: the sum is NaN.
struct Stats {
  float top, sum;
};
__device__ __forceinline__ Stats merge(Stats a, Stats b, float c) {
  const float top = fmaxf(a.top, b.top);
  if (top == -INFINITY) return {top, a.sum + b.sum};
  return {top, a.sum * exp2_of((a.top - top) * c) + b.sum * exp2_of((b.top - top) * c)};
}
__device__ __forceinline__ Stats merge_wave(Stats s, float c) {
#pragma unroll
  for (int d = 32; d; d >>= 1) s = merge(s, Stats{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)}, c);
  return s;
}
__device__ __forceinline__ bool nothing(Stats s) { return s.top == -INFINITY && s.sum == 0.f; }
__device__ __forceinline__ float lse_of(Stats s, float inv_t) { return nothing(s) ? -INFINITY : fmaf(s.top, inv_t, logf(s.sum)); }

struct DistillArgs {
  const void* Z;
  int64_t t, v, ldz;
  int64_t first;  // row that the launch begins with (k_distill_row)
  const void* ids;
  int32_t id_type;
  const float* teacher;
  int32_t k;
  int64_t ldi;
  float inv_t, c, temperature;
  const float* weights;
  const float* lse_in;
  float* loss;
  float* lse;
  void* dZ;
  int64_t lddz;
  Stats* parts;      // long rows: t x splits
  Stats* row_stats;  // ... joined, for the gradient of the same call; may be null
  uint32_t* tickets;
  uint32_t splits;
  int64_t per_split;  // scores, a multiple of eight
  uint32_t* status;
};

// ------------------------------------------------------------------------------------------
// Lists
// ------------------------------------------------------------------------------------------
// A row's list in the LDS: ids (-1: no entry), probabilities, scores.
struct List {
  int32_t id[MOST_ENTRIES];
  float p[MOST_ENTRIES];
  float z[MOST_ENTRIES];
};

__device__ __forceinline__ float max_wave(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float sum_wave(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// Of a list's logits: the largest, -infinity where there is no entry, and log sum exp((logit - top) / T).  As with the scores the difference comes first.
struct ListStats {
  float top, log_sum;
};

// One wavefront fills the list (ids outside [from, to) too: the probabilities are those of all entries, the scores only of those inside).
template <typename T>
__device__ __forceinline__ ListStats fill_list(const DistillArgs& a, int64_t row, const T* z, int64_t from, int64_t to, List& list) {
  const int lane = threadIdx.x & 63;
  const float* teacher = a.teacher + row * a.ldi;
  float top = -INFINITY;
  for (int i = lane; i < a.k; i += 64) {
    const int64_t id = a.id_type == EJOIN_I64 ? static_cast<const int64_t*>(a.ids)[row * a.ldi + i] : static_cast<const int32_t*>(a.ids)[row * a.ldi + i];
    const float u = teacher[i];
    const bool there = id >= 0 && id < a.v && u != -INFINITY;
    if (id < -1 || id >= a.v) *a.status = EJOIN_STATUS_TOKEN;
    list.id[i] = there ? (int32_t)id : -1;
    list.p[i] = u;
    list.z[i] = there && id >= from && id < to ? Element<T>::get(z[id]) : 0.f;
    if (there) top = fmaxf(top, u != u ? INFINITY : u);  // (NaN: the exponentials below make it one)
  }
  top = max_wave(top);
  if (top == -INFINITY) return {top, 0.f};
  float sum = 0.f;
  for (int i = lane; i < a.k; i += 64)  // (a lane reads what it wrote)
    if (list.id[i] >= 0) sum += exp2_of((list.p[i] - top) * a.c);
  sum = sum_wave(sum);
  for (int i = lane; i < a.k; i += 64) list.p[i] = list.id[i] >= 0 ? exp2_of((list.p[i] - top) * a.c) / sum : 0.f;
  return {top, logf(sum)};
}

// sum_i p_i (log p_i - log q_i) of a row with entries, by the wavefront that filled the list for all of the row.
__device__ __forceinline__ float divergence(const DistillArgs& a, int64_t row, const List& list, ListStats l, Stats s) {
  const int lane = threadIdx.x & 63;
  const float* teacher = a.teacher + row * a.ldi;
  const float log_sum = logf(s.sum);
  float sum = 0.f;
  for (int i = lane; i < a.k; i += 64) {
    if (list.id[i] < 0) continue;
    const float z = list.z[i], p = list.p[i];
    const float log_q = z == -INFINITY && s.sum == s.sum ? -INFINITY : (z - s.top) * a.inv_t - log_sum;
    // (an entry whose probability is zero to 32 bits adds nothing, unless the row's loss is NaN anyway)
    sum += p == 0.f && log_q == log_q ? 0.f : p * ((teacher[i] - l.top) * a.inv_t - l.log_sum - log_q);
  }
  return sum_wave(sum);
}

// weight * q of a score: from the row's statistics, or from its lse.  An lse in 32 bits holds the sum only to 2^-24 of its own magnitude: what it
// gives is as far off as exp(|lse| 2^-24) is from one, so a call that has the statistics goes by those.
struct FromStats {
  float top, c, factor;
  static __device__ __forceinline__ Stats of_row(const DistillArgs& a, int64_t row) { return a.row_stats[row]; }
  __device__ FromStats(const DistillArgs& a, Stats s, float weight) : top(s.top == -INFINITY ? 0.f : s.top), c(a.c), factor(nothing(s) ? 0.f : weight / s.sum) {}
  __device__ __forceinline__ float operator()(float z) const { return factor * exp2_of((z - top) * c); }
};
struct FromLse {
  float lse, inv_t, factor;
  static __device__ __forceinline__ float of_row(const DistillArgs& a, int64_t row) { return a.lse_in[row]; }
  __device__ FromLse(const DistillArgs& a, float lse_, float weight) : lse(lse_ == -INFINITY ? 0.f : lse_), inv_t(a.inv_t), factor(lse_ == -INFINITY ? 0.f : weight) {}
  __device__ __forceinline__ float operator()(float z) const { return factor * exp2_of((z * inv_t - lse) * LOG2E); }
};

// The entries of [from, to) once the rest of the gradient is written: each writes the value for all entries with its id, for which it looks through the
// list.  That grows as the square of the list: 4,096 rows of 4,099 BF16 scores with lists of 1,024, loss and gradient, 605 us, where the bytes are 14; with lists
// of up to 100 or so it is lost beside the row.
template <typename T, typename Q>
__device__ __forceinline__ void put_entries(const DistillArgs& a, T* dz, int64_t from, int64_t to, const List& list, const Q& weighted_q, float weight, int threads) {
  for (int i = threadIdx.x; i < a.k; i += threads) {
    const int32_t id = list.id[i];
    if (id < from || id >= to) continue;
    float p = 0.f;
    for (int j = 0; j < a.k; ++j) p += list.id[j] == id ? list.p[j] : 0.f;
    dz[id] = Element<T>::put(weighted_q(list.z[i]) - weight * p);
  }
}

// ------------------------------------------------------------------------------------------
// Rows that fit the registers of a workgroup: read once
// ------------------------------------------------------------------------------------------
// All of a row's loads are under way together, the first wavefront sees to its list meanwhile.  One barrier for the statistics; one
// between the gradient and the entries' places in it.  Bound by the memory: loss and gradient of 4,096 rows of 50,021 BF16 scores 190 us for the 822 MB that are read
// and written once, 4.3 TB/s.  (Scores kept as FP32 take twice the registers and leave one workgroup a CU: 299 us.  Rows read a second time for the gradient: 359.)
// Threads and pieces: as few registers a thread as bring two rows or more to a CU.  13 pieces of 16-bit scores take 82 registers by themselves, two more
// than leave room for a third workgroup: held to those, loss and gradient of 4,096 rows of 41,000, 45,001 and 50,021 176, 194 and 220 us -> 153, 184 and
// 205, the two calls of one each unchanged.  Ten pieces need 68 and have three workgroups anyway; 16 need 95 (held to 80: loss of 4,096 x 60,001 146 ->
// 130 us, both 246 -> 273); a second workgroup of 1,024 threads would have to do with 64.
// Eight scores as the words they are in memory: the compiler keeps 16-bit ones two to a register only where it sees no more than that.
template <typename T>
struct Words {
  static constexpr int N = (int)sizeof(T) * 2;
  uint32_t w[N];
  __device__ __forceinline__ void load(const T* p) {
    typedef uint32_t At __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    const At x = __builtin_nontemporal_load(reinterpret_cast<const At*>(p));
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i];
  }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, x);
      else w[i] = __builtin_bit_cast(uint16_t, Element<T>::put(x)) * 0x10001u;
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
    else return Element<T>::get(__builtin_bit_cast(T, (uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
  }
  // What has been worked out of them before is of no use after, and what follows waits for `so_far`.
  __device__ __forceinline__ void as_they_are(float& so_far) {
    if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]), "+v"(so_far));
    else asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]), "+v"(w[4]), "+v"(w[5]), "+v"(w[6]), "+v"(w[7]), "+v"(so_far));
  }
};

template <typename T, int THREADS, int PIECES, bool FORWARD, bool GRAD>
__global__ __launch_bounds__(THREADS, THREADS == 512 && PIECES == 13 ? 6 : THREADS * PIECES * (int)sizeof(T) > 512 * 12 * 2 ? 4 : 2) void k_distill_row(const DistillArgs a) {
  __shared__ List list;
  __shared__ Stats wave_stats[THREADS / 64];
  __shared__ float shared_list_top;
  const int64_t row = a.first + blockIdx.x;
  const T* z = static_cast<const T*>(a.Z) + row * a.ldz;
  const uint32_t v = (uint32_t)a.v, whole = v & ~7u, mine = threadIdx.x * 8;
  Words<T> x[PIECES];
#pragma unroll
  for (int j = 0; j < PIECES; ++j) {
    const uint32_t at = j * THREADS * 8 + mine;
    if (at < whole) {
      x[j].load(z + at);
    } else {
      x[j].fill(-INFINITY);
    }
  }
  const bool odd = threadIdx.x < v - whole;  // the up to seven scores past the last eight: one a thread
  const uint32_t odd_at = whole + threadIdx.x;
  const float rest = odd ? Element<T>::get(z[odd_at]) : -INFINITY;
  ListStats l{0.f, 0.f};
  if (threadIdx.x < 64) {
    l = fill_list(a, row, z, 0, a.v, list);
    if (threadIdx.x == 0) shared_list_top = l.top;
  }
  Stats s{-INFINITY, 0.f};
  if (FORWARD) {
    s.top = rest;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s.top = fmaxf(s.top, x[j].get(i));
      x[j].as_they_are(s.top);
    }
    const float top = s.top == -INFINITY ? 0.f : s.top;
    s.sum = exp2_of((rest - top) * a.c);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = exp2_of((x[j].get(i) - top) * a.c);
      s.sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      x[j].as_they_are(s.sum);
    }
    s = merge_wave(s, a.c);
    if ((threadIdx.x & 63) == 0) wave_stats[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (FORWARD) {
    s = wave_stats[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) s = merge(s, wave_stats[w], a.c);
    if (threadIdx.x < 64) {
      const float loss = l.top == -INFINITY ? 0.f : a.temperature * a.temperature * divergence(a, row, list, l, s);
      if (threadIdx.x == 0) {
        a.loss[row] = loss;
        if (a.lse) a.lse[row] = lse_of(s, a.inv_t);
      }
    }
  }
  if constexpr (GRAD) {
    T* dz = static_cast<T*>(a.dZ) + row * a.lddz;
    if (shared_list_top == -INFINITY) {  // no entry: zeros
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (uint32_t at = mine; at < whole; at += THREADS * 8) store8<T, true>(dz + at, zero);
      if (odd) dz[odd_at] = Element<T>::put(0.f);
      return;
    }
    const float weight = a.weights[row] * a.temperature;
    auto weighted_q = [&] {
      if constexpr (FORWARD) return FromStats(a, s, weight);
      else return FromLse(a, FromLse::of_row(a, row), weight);
    }();
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const uint32_t at = j * THREADS * 8 + mine;
      if (at >= whole) break;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = weighted_q(x[j].get(i));
      store8<T, true>(dz + at, y);
      if (j + 1 < PIECES) x[j + 1].as_they_are(weighted_q.factor);  // (one piece after the other)
    }
    if (odd) dz[odd_at] = Element<T>::put(weighted_q(rest));
    __syncthreads();
    put_entries(a, dz, 0, a.v, list, weighted_q, weight, THREADS);
  }
}

// ------------------------------------------------------------------------------------------
// Longer rows, cut into pieces for a workgroup each
// ------------------------------------------------------------------------------------------
// The statistics of a piece, by eight wavefronts; a ninth sees to the list meanwhile, and if its workgroup is the last of the row to
// be done, joins the pieces' statistics and works out the loss.  5 rows of 1,000,000 FP32 scores (20 MB) 11.2 us, of which a launch and the join are some 7.
// (A list that the wavefronts see to before or after the scores: 15.7 us.)  Rows that no workgroup holds, loss and gradient, read twice: 512 of 128,256 FP32
// 193 us (76 and 114 for the launches, 788 MB: 4.1 TB/s), 2,048 of 151,936 BF16 439.
template <typename T>
__global__ __launch_bounds__(LONG_THREADS + 64) void k_distill_long(const DistillArgs a) {
  __shared__ List list;
  __shared__ Stats wave_stats[LONG_THREADS / 64];
  const int64_t row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
  const T* z = static_cast<const T*>(a.Z) + row * a.ldz;
  const int64_t from = split * a.per_split, to = from + a.per_split < a.v ? from + a.per_split : a.v;
  const int lane = threadIdx.x & 63;
  Stats s{-INFINITY, 0.f};
  if (threadIdx.x < LONG_THREADS) {
    for (int64_t at = from + threadIdx.x * 8; at < to; at += 4 * LONG_THREADS * 8) {  // four times eight scores under way at a time
      float x[4][8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t here = at + j * LONG_THREADS * 8, left = to - here;
        load8(z + here, left < 0 ? 0 : (left < 8 ? (int)left : 8), x[j]);
        if (left < 8) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i >= left) x[j][i] = -INFINITY;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, x[j][i]);
      Stats p{top, 0.f};
      if (top == -INFINITY) top = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) p.sum += exp2_of((x[j][i] - top) * a.c);
      s = merge(s, p, a.c);
    }
    s = merge_wave(s, a.c);
    if (lane == 0) wave_stats[threadIdx.x >> 6] = s;
  }
  const ListStats l = threadIdx.x < LONG_THREADS ? ListStats{0.f, 0.f} : fill_list(a, row, z, 0, a.v, list);
  __syncthreads();
  if (threadIdx.x < LONG_THREADS) return;
  s = lane < LONG_THREADS / 64 ? wave_stats[lane] : Stats{-INFINITY, 0.f};
  s = merge_wave(s, a.c);
  if (a.splits > 1) {
    // Parts and tickets are written and read past the XCDs' own caches (agent scope).  A part has arrived before its ticket is taken; whoever
    // takes the last one reads all parts, and leaves the counter at zero.
    uint64_t* parts = reinterpret_cast<uint64_t*>(a.parts) + row * a.splits;
    uint32_t ticket = 0;
    if (lane == 0) {
      __hip_atomic_store(parts + split, __builtin_bit_cast(uint64_t, s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      ticket = __hip_atomic_fetch_add(&a.tickets[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__shfl((int)ticket, 0) != (int)a.splits - 1) return;
    asm volatile("" ::: "memory");
    if (lane == 0) __hip_atomic_store(&a.tickets[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = Stats{-INFINITY, 0.f};
    for (uint32_t i = lane; i < a.splits; i += 64)
      s = merge(s, __builtin_bit_cast(Stats, __hip_atomic_load(parts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)), a.c);
    s = merge_wave(s, a.c);
  }
  const float loss = l.top == -INFINITY ? 0.f : a.temperature * a.temperature * divergence(a, row, list, l, s);
  if (lane == 0) {
    a.loss[row] = loss;
    if (a.lse) a.lse[row] = lse_of(s, a.inv_t);
    if (a.row_stats) a.row_stats[row] = s;
  }
}

// FROM: FromStats after k_distill_long of the same call, FromLse where the caller kept an lse.
template <typename T, typename FROM>
__global__ __launch_bounds__(LONG_THREADS) void k_distill_long_grad(const DistillArgs a) {
  __shared__ List list;
  __shared__ float shared_list_top;
  const int64_t row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
  const T* z = static_cast<const T*>(a.Z) + row * a.ldz;
  const int64_t from = split * a.per_split, to = from + a.per_split < a.v ? from + a.per_split : a.v;
  T* dz = static_cast<T*>(a.dZ) + row * a.lddz;
  if (threadIdx.x < 64) {
    const ListStats l = fill_list(a, row, z, from, to, list);
    if (threadIdx.x == 0) shared_list_top = l.top;
  }
  const float weight = a.weights[row] * a.temperature;
  const FROM weighted_q(a, FROM::of_row(a, row), weight);
  __syncthreads();  // (the entries' scores are read before any is overwritten: dZ may be Z)
  if (shared_list_top == -INFINITY) {  // no entry: zeros
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t at = from + threadIdx.x * 8; at < to; at += LONG_THREADS * 8) store8(dz + at, to - at < 8 ? (int)(to - at) : 8, zero);
    return;
  }
  for (int64_t at = from + threadIdx.x * 8; at < to; at += 2 * LONG_THREADS * 8) {
    float x[2][8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t here = at + j * LONG_THREADS * 8, left = to - here;
      load8(z + here, left < 0 ? 0 : (left < 8 ? (int)left : 8), x[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t here = at + j * LONG_THREADS * 8, left = to - here;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = weighted_q(x[j][i]);
      store8(dz + here, left < 0 ? 0 : (left < 8 ? (int)left : 8), x[j]);
    }
  }
  __syncthreads();
  put_entries(a, dz, from, to, list, weighted_q, weight, LONG_THREADS);
}

// ------------------------------------------------------------------------------------------ host side
// log2(e) / T: exp(x / T) = 2^(c x).
float base2(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

bool bad_args(const ejoin_ctx* ctx, int32_t ztype, int64_t t, int64_t v, int64_t ldz, int32_t id_type, int32_t k, int64_t ldi, float temperature) {
  if (!ctx || bad_type(ztype) || (id_type != EJOIN_I32 && id_type != EJOIN_I64) || t < 0 || t >= (1ll << 31) || v < 1 || v >= (1ll << 31) || ldz < v) return true;
  return k < 0 || k > MOST_ENTRIES || ldi < k || !(temperature > 0.f) || !isfinite(temperature) || !isfinite(base2(temperature));
}

typedef void (*DistillKernel)(DistillArgs);
// The kernel that holds a row of v scores in registers (at most 64 of a thread), and its threads; null where none does.
template <typename T, bool FORWARD, bool GRAD>
DistillKernel row_kernel(int64_t v, int& threads) {
  threads = v <= 4096 ? 256 : (v <= 512 * 8 * (sizeof(T) == 2 ? 16 : 8) ? 512 : 1024);
  if (v <= 2048) return &k_distill_row<T, 256, 1, FORWARD, GRAD>;
  if (v <= 4096) return &k_distill_row<T, 256, 2, FORWARD, GRAD>;
  if (v <= 8192) return &k_distill_row<T, 512, 2, FORWARD, GRAD>;
  if (v <= 16384) return &k_distill_row<T, 512, 4, FORWARD, GRAD>;
  if (v <= 32768) return &k_distill_row<T, 512, 8, FORWARD, GRAD>;
  if constexpr (sizeof(T) == 4) {
    if (v <= 65536) return &k_distill_row<T, 1024, 8, FORWARD, GRAD>;
  } else {
    if (v <= 40960) return &k_distill_row<T, 512, 10, FORWARD, GRAD>;
    if (v <= 53248) return &k_distill_row<T, 512, 13, FORWARD, GRAD>;
    if (v <= 65536) return &k_distill_row<T, 512, 16, FORWARD, GRAD>;
    if (v <= 98304) return &k_distill_row<T, 1024, 12, FORWARD, GRAD>;
    if (v <= 131072) return &k_distill_row<T, 1024, 16, FORWARD, GRAD>;
  }
  return nullptr;
}

// Pieces of a long row: so many that the rows' pieces fill the CUs several times over, of 16,384 scores at least (what a workgroup has under way).
void split_rows(const ejoin_ctx* ctx, DistillArgs& a) {
  int64_t s = (3 * (int64_t)ctx->num_cu + a.t - 1) / a.t;
  const int64_t most = (a.v + 16383) / 16384;
  s = s < most ? s : most;
  s = s < MOST_SPLITS ? s : MOST_SPLITS;
  if (a.t > MOST_TICKETS) s = 1;
  a.per_split = up((a.v + s - 1) / s, 8);
  a.splits = (uint32_t)((a.v + a.per_split - 1) / a.per_split);
}

// Whether rows that would fit the registers of a workgroup are cut into pieces all the same: few long ones leave most CUs idle.
// 16-bit scores, whole and in pieces: forward, 128 rows of 20,011 8.9 and 8.7 us, of 40,009 9.7 and 8.9, of 130,003 20.9 and
// 16.8, 256 of 40,009 10.7 and 12.0; gradient, 128 of 40,009 12.7 and 10.6, of 130,003 24.7 and 16.5; both, where pieces are read twice, 32 of 40,009 13.8 and
// 16.1, of 65,521 20.0 and 16.5, 128 of 90,001 23.5 and 26.2.
// FP32 ones, in graphs, which adds 6 us: forward, 1 row of 33,001 13.0 and 12.2, 128 of 33,001 16.7 and 14.9, of 65,521 17.3 and 16.5, 256 of 40,009 17.3 and 18.3;
// gradient, 128 of 33,001 19.6 and 18.6, of 65,521 26.1 and 23.2; both, 32 of 33,001 18.2 and 20.6, of 65,521 23.3 and 21.7, 64 of 65,521 25.8 and 25.7, 128 29.0 and 31.9.
template <bool BOTH>
bool few_long(const ejoin_ctx* ctx, int64_t t, int64_t v) {
  return BOTH ? v > 53248 && t <= ctx->num_cu / 4 : v > 32768 && t <= ctx->num_cu / 2;
}

template <bool FORWARD, bool GRAD>
int launch_distill(ejoin_ctx* ctx, DistillArgs& a, int32_t ztype, hipStream_t st) {
  int rc = EJOIN_OK;
  with_type(ztype, [&](auto z) {
    typedef decltype(z) T;
    int threads;
    const DistillKernel kernel = row_kernel<T, FORWARD, GRAD>(a.v, threads);
    if (kernel && !few_long<FORWARD && GRAD>(ctx, a.t, a.v)) {
      in_launches(a.t, [&](int64_t first, unsigned rows) {
        a.first = first;
        hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), 0, st, a);
      });
      return;
    }
    split_rows(ctx, a);
    if (a.t * a.splits > MOST_GROUPS) {  // (more than 2^21 rows of more than 32,768 scores)
      rc = EJOIN_EUNSUPPORTED;
      return;
    }
    const dim3 grid((unsigned)(a.t * a.splits));
    if (FORWARD) {
      const int64_t parts = up(a.t * a.splits * (int64_t)sizeof(Stats), 256);
      rc = ensure_embed(ctx, parts + (GRAD ? a.t * (int64_t)sizeof(Stats) : 0), st);
      if (rc != EJOIN_OK) return;
      a.parts = reinterpret_cast<Stats*>(ctx->embed);
      a.tickets = ctx->tickets;
      if (GRAD) a.row_stats = reinterpret_cast<Stats*>(ctx->embed + parts);
      hipLaunchKernelGGL(k_distill_long<T>, grid, dim3(LONG_THREADS + 64), 0, st, a);
    }
    if constexpr (GRAD) hipLaunchKernelGGL((k_distill_long_grad<T, std::conditional_t<FORWARD, FromStats, FromLse>>), grid, dim3(LONG_THREADS), 0, st, a);
  });
  if (rc != EJOIN_OK) return rc;
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

DistillArgs distill_args(ejoin_ctx* ctx, const void* Z, int64_t t, int64_t v, int64_t ldz, const void* ids, int32_t id_type, const float* teacher, int32_t k,
                         int64_t ldi, float temperature) {
  DistillArgs a;
  memset(&a, 0, sizeof(a));
  a.Z = Z, a.t = t, a.v = v, a.ldz = ldz, a.ids = ids, a.id_type = id_type, a.teacher = teacher, a.k = k, a.ldi = ldi;
  a.inv_t = 1.f / temperature;
  a.c = base2(temperature);
  a.temperature = temperature;
  a.status = ctx->token_status;
  return a;
}

}  // namespace

extern "C" {

int ejoin_distill(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const void* ids, int32_t id_type, const float* teacher,
                  int32_t k, int64_t ldi, float temperature, float* loss, float* lse, void* stream) {
  if (bad_args(ctx, ztype, t, v, ldz, id_type, k, ldi, temperature)) return EJOIN_EINVAL;
  if (t == 0) return EJOIN_OK;
  if (!Z || !loss || !lse || (k > 0 && (!ids || !teacher))) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  DistillArgs a = distill_args(ctx, Z, t, v, ldz, ids, id_type, teacher, k, ldi, temperature);
  a.loss = loss;
  a.lse = lse;
  return launch_distill<true, false>(ctx, a, ztype, static_cast<hipStream_t>(stream));
}

int ejoin_distill_grad(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const float* lse, const void* ids, int32_t id_type,
                       const float* teacher, int32_t k, int64_t ldi, const float* weights, float temperature, void* dZ, int64_t lddz, void* stream) {
  if (bad_args(ctx, ztype, t, v, ldz, id_type, k, ldi, temperature) || lddz < v) return EJOIN_EINVAL;
  if (t == 0) return EJOIN_OK;
  if (!Z || !lse || !weights || !dZ || (dZ == Z && lddz != ldz) || (k > 0 && (!ids || !teacher))) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  DistillArgs a = distill_args(ctx, Z, t, v, ldz, ids, id_type, teacher, k, ldi, temperature);
  a.lse_in = lse;
  a.weights = weights;
  a.dZ = dZ;
  a.lddz = lddz;
  return launch_distill<false, true>(ctx, a, ztype, static_cast<hipStream_t>(stream));
}

int ejoin_distill_with_grad(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const void* ids, int32_t id_type,
                            const float* teacher, int32_t k, int64_t ldi, const float* weights, float temperature, float* loss, void* dZ, int64_t lddz,
                            void* stream) {
  if (bad_args(ctx, ztype, t, v, ldz, id_type, k, ldi, temperature) || lddz < v) return EJOIN_EINVAL;
  if (t == 0) return EJOIN_OK;
  if (!Z || !loss || !weights || !dZ || (dZ == Z && lddz != ldz) || (k > 0 && (!ids || !teacher))) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  DistillArgs a = distill_args(ctx, Z, t, v, ldz, ids, id_type, teacher, k, ldi, temperature);
  a.loss = loss;
  a.weights = weights;
  a.dZ = dZ;
  a.lddz = lddz;
  return launch_distill<true, true>(ctx, a, ztype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
