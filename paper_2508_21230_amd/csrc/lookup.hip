// Rows of a table by token, and the gradient of that: the rows' gradients summed by token.
#include <type_traits>

#include "embed.h"

namespace {

// A token as a row of the table; -1 for none and for one outside the table, which is reported.
template <typename I>
__device__ __forceinline__ int64_t row_of(I token, int64_t v, uint32_t* status) {
  const int64_t x = (int64_t)token;
  if (x >= 0 && x < v) return x;
  if (x != -1) *status = EJOIN_STATUS_TOKEN;  // (every lane that writes writes this)
  return -1;
}

// ------------------------------------------------------------------------------------------
// Lookup
// ------------------------------------------------------------------------------------------
struct LookupArgs {
  const void* table;
  int64_t v, ldt;
  int32_t d;
  const void* tokens;
  int64_t t;
  float scale;
  void* Y;
  int64_t ldy;
  uint32_t chunks;  // pieces of eight of a row, padding included
  uint32_t* status;
};

// Y[t] = scale * table[token t], rounded once to FP32 and once to Y's type.  Bound by the memory, whole rows of a kilobyte or so wherever they are:
// 400,003 FP32 rows of 384 into FP16 107 us, 4.6 TB/s; 300 of 96 4.6 us, a launch.  Four pieces a thread hide the token's load and the row's, one after the
// other (one piece a thread: 126 us).  A thread has LOOKUP_PIECES pieces of eight under way.  WIDE: more pieces than 32 bits count.  PASSING: the result goes past the caches.
constexpr int LOOKUP_PIECES = 4;
template <typename T, typename O, typename I, bool WIDE, bool PASSING>
__global__ __launch_bounds__(256) void k_lookup(const LookupArgs a) {
  typedef std::conditional_t<WIDE, uint64_t, uint32_t> Unit;
  const Unit first = (Unit)blockIdx.x * (256 * LOOKUP_PIECES) + threadIdx.x, units = (Unit)a.t * a.chunks;
  int64_t row[LOOKUP_PIECES];
  uint32_t t[LOOKUP_PIECES];
  int c[LOOKUP_PIECES];
#pragma unroll
  for (int q = 0; q < LOOKUP_PIECES; ++q) {
    const Unit unit = first + q * 256 < units ? first + q * 256 : units - 1;  // (past the end: the last one again)
    t[q] = (uint32_t)(unit / a.chunks);
    c[q] = (int)(unit - (Unit)t[q] * a.chunks) * 8;
    row[q] = row_of(static_cast<const I*>(a.tokens)[t[q]], a.v, a.status);
  }
  float x[LOOKUP_PIECES][8];
#pragma unroll
  for (int q = 0; q < LOOKUP_PIECES; ++q) {
    const int left = a.d - c[q];
    load8(static_cast<const T*>(a.table) + (row[q] < 0 ? 0 : row[q] * a.ldt + c[q]), row[q] < 0 || left < 0 ? 0 : (left < 8 ? left : 8), x[q]);
  }
#pragma unroll
  for (int q = 0; q < LOOKUP_PIECES; ++q) {
    if (first + q * 256 >= units) break;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[q][i] = row[q] < 0 || c[q] + i >= a.d ? 0.f : x[q][i] * a.scale;  // (a scale of either sign gives zeros of its sign)
      asm("" : "+v"(x[q][i]));  // (rounded to FP32 here: there is an instruction that would multiply and round to FP16 at once)
    }
    store8<O, PASSING>(static_cast<O*>(a.Y) + (int64_t)t[q] * a.ldy + c[q], x[q]);
  }
}

// ------------------------------------------------------------------------------------------
// Gradient
// ------------------------------------------------------------------------------------------
// The tokens are sorted (stable, by digits of up to DIGIT_BITS bits, least first), so that the places of a row stand together in
// ascending order.  Then pieces of CHUNK sorted places are summed side by side, whatever rows they belong to: frequent tokens make no
// workgroup's work longer.  A row whose places lie in one piece is written at once; one that goes on in the next piece leaves sums
// that k_grad_join adds up in their order.
// 300,007 tokens, frequencies as 1 / rank, of 100,000 rows of 384, FP16 into FP32: 157 us; of that the sort 34, the sums 102 (385 MB, 3.8 TB/s: rows of 768 bytes
// in the order of the table), the long runs 22.  Pieces of 16, 32 and 64 places, in graphs: 183, 161 and 160 us; 20,000 of 50,000 x 128: 50, 57, 76; even
// frequencies 127, 127, 137 and 43, 43, 57.  Few tens of thousands of tokens are bound by the six launches that wait for each other.
// Places without a token sort last and are read like others, their sum is dropped: 300,000 tokens of which half are none take as long as if all were there.
constexpr int DIGIT_BITS = 9;
constexpr int DIGITS = 1 << DIGIT_BITS;
constexpr int SORT_THREADS = 512;  // (as many as there are digits)
constexpr int SORT_ITEMS = 4;
constexpr int SORT_BLOCK = SORT_THREADS * SORT_ITEMS;
constexpr int CHUNK = 32;
// (4,000,000 tokens, traced: counts 8 and 12 us, running sums 9 + 5 a pass, scatters 30 and 19.)
// From SCAN_FROM blocks on their counts are turned into running sums first, in groups of SCAN_BLOCKS; below, every block adds up the counts of all
// others for itself, which is two launches less but grows as their square.  The gradient of 400,000, 500,000, 600,000 and 4,000,000 tokens of 100,000
// rows of 64 with running sums 74, 77, 84 and 404 us, without 71, 77, 92 and 963; of 300 rows of 16 57, 60, 64, 169 and 54, 59, 67, 444.
constexpr int SCAN_BLOCKS = 128;
constexpr int SCAN_FROM = 256;

struct SortArgs {
  const void* tokens;  // first pass
  const uint2* items;  // (key, place)
  uint2* items_out;
  uint32_t* counts;  // of the blocks, DIGITS each; scanned: what the blocks before each in its group have
  uint32_t* groups;  // what the groups before each have, and last where each digit's places begin; null where counts are not scanned
  uint32_t t, v, blocks;
  int shift;
  uint32_t mask;
  uint32_t* status;
};

// Key of place i: its row, v for none.
template <typename I, bool FIRST>
__device__ __forceinline__ uint32_t key_at(const SortArgs& a, uint32_t i) {
  if (!FIRST) return a.items[i].x;
  const int64_t row = row_of(static_cast<const I*>(a.tokens)[i], (int64_t)a.v, a.status);
  return row < 0 ? a.v : (uint32_t)row;
}

template <typename I, bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_count(const SortArgs a) {
  __shared__ uint32_t count[DIGITS];
  count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < SORT_ITEMS; ++q) {
    const uint32_t i = blockIdx.x * SORT_BLOCK + q * SORT_THREADS + threadIdx.x;
    if (i < a.t) atomicAdd(&count[(key_at<I, FIRST>(a, i) >> a.shift) & a.mask], 1u);
  }
  __syncthreads();
  a.counts[(int64_t)blockIdx.x * DIGITS + threadIdx.x] = count[threadIdx.x];
}

// Exclusive sum over the 512 threads of a workgroup.
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t x, uint32_t* scratch /* 8 */) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = x;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)sum, s);
    if (lane >= s) sum += y;
  }
  if (lane == 63) scratch[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += scratch[w];
  return before + sum - x;
}

// A column of `rows` counts into running sums (what the rows before each have); what all of them have.  Thread = digit, 32 loads under way at a time.
__device__ __forceinline__ uint32_t scan_column(uint32_t* counts, uint32_t rows) {
  uint32_t sum = 0;
  for (uint32_t b = 0; b < rows; b += 32) {
    uint32_t c[32];
#pragma unroll
    for (int q = 0; q < 32; ++q) c[q] = b + q < rows ? counts[(int64_t)(b + q) * DIGITS + threadIdx.x] : 0;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      if (b + q < rows) counts[(int64_t)(b + q) * DIGITS + threadIdx.x] = sum;
      sum += c[q];
    }
  }
  return sum;
}

__global__ __launch_bounds__(SORT_THREADS) void k_sort_scan(const SortArgs a) {
  const uint32_t first = blockIdx.x * SCAN_BLOCKS;
  a.groups[(int64_t)blockIdx.x * DIGITS + threadIdx.x] = scan_column(a.counts + (int64_t)first * DIGITS, min((uint32_t)SCAN_BLOCKS, a.blocks - first));
}

// One workgroup: the groups' sums, and where each digit's places begin.
__global__ __launch_bounds__(SORT_THREADS) void k_sort_scan_groups(const SortArgs a, const uint32_t groups) {
  __shared__ uint32_t scratch[SORT_THREADS / 64];
  const uint32_t all = scan_column(a.groups, groups);
  a.groups[(int64_t)groups * DIGITS + threadIdx.x] = exclusive_sum(all, scratch);
}

template <typename I, bool FIRST, bool SCANNED>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_scatter(const SortArgs a) {
  constexpr int WAVES = SORT_THREADS / 64;
  __shared__ uint32_t at[WAVES][DIGITS];  // a wavefront's count of a digit so far, then where its first one goes
  __shared__ uint32_t scratch[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) at[w][threadIdx.x] = 0;
  __syncthreads();
  // a wavefront takes 256 consecutive places, 64 at a time: its equal digits are ranked by their lanes
  uint32_t key[SORT_ITEMS], place[SORT_ITEMS], rank[SORT_ITEMS];
#pragma unroll
  for (int q = 0; q < SORT_ITEMS; ++q) {
    const uint32_t i = blockIdx.x * SORT_BLOCK + wave * (64 * SORT_ITEMS) + q * 64 + lane;
    const bool there = i < a.t;
    if (FIRST) {
      key[q] = there ? key_at<I, FIRST>(a, i) : 0;
    } else {
      const uint2 item = there ? a.items[i] : uint2{0, 0};
      key[q] = item.x;
      place[q] = item.y;
    }
    const uint32_t digit = (key[q] >> a.shift) & a.mask;
    uint64_t same = __ballot(there);
#pragma unroll
    for (int b = 0; b < DIGIT_BITS; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same &= ((digit >> b) & 1) ? set : ~set;
    }
    const uint32_t below = __popcll(same & ((1ull << lane) - 1));
    uint32_t seen = 0;
    // (the lanes of a wavefront read, then write: its LDS accesses are done in order, the fences keep the compiler from moving them)
    if (there) seen = at[wave][digit];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (there && below == 0) at[wave][digit] = seen + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    rank[q] = seen + below;
  }
  __syncthreads();
  // thread = digit: its places in all blocks and in those before this one, and in the block's wavefronts
  uint32_t to;
  if (SCANNED) {
    const uint32_t groups = (a.blocks + SCAN_BLOCKS - 1) / SCAN_BLOCKS;
    to = a.counts[(int64_t)blockIdx.x * DIGITS + threadIdx.x] + a.groups[(int64_t)(blockIdx.x / SCAN_BLOCKS) * DIGITS + threadIdx.x] +
         a.groups[(int64_t)groups * DIGITS + threadIdx.x];
  } else {
    uint32_t all = 0, before = 0;
    for (uint32_t b = 0; b < a.blocks; b += 32) {  // (thirty-two loads under way at a time)
      uint32_t c[32];
#pragma unroll
      for (int q = 0; q < 32; ++q) c[q] = b + q < a.blocks ? a.counts[(b + q) * DIGITS + threadIdx.x] : 0;
#pragma unroll
      for (int q = 0; q < 32; ++q) {
        all += c[q];
        before += b + q < blockIdx.x ? c[q] : 0;
      }
    }
    to = exclusive_sum(all, scratch) + before;
  }
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const uint32_t c = at[w][threadIdx.x];
    at[w][threadIdx.x] = to;
    to += c;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < SORT_ITEMS; ++q) {
    const uint32_t i = blockIdx.x * SORT_BLOCK + wave * (64 * SORT_ITEMS) + q * 64 + lane;
    if (i >= a.t) continue;
    const uint32_t p = at[wave][(key[q] >> a.shift) & a.mask] + rank[q];
    a.items_out[p] = uint2{key[q], FIRST ? i : place[q]};
  }
}

struct GradArgs {
  const void* dY;
  int64_t ldy;
  int32_t d;
  uint32_t t, v;
  const uint2* items;  // (row, place), sorted by row
  float scale;
  void* G;
  int64_t ldg;
  float* parts;    // of each piece: the sum of a row that began before it, and of one that begins in it and goes on
  int32_t width;   // of a row of parts
  int lanes_log2;  // that share a row, eight columns each
  uint32_t sum_groups;   // workgroups of k_grad_sum that sum; the others zero rows
  uint32_t zero_rows;    // of each of those
  uint32_t* status;
};

// Sum of the rows' gradients at places[from, to), their columns c .. c + have - 1: eight loads under way at a time, added up in order.
template <typename T, typename P>
__device__ __forceinline__ void add_rows(const GradArgs& a, const P* places, uint32_t from, uint32_t to, int c, int have, float (&sum)[8]) {
  const T* dY = static_cast<const T*>(a.dY) + c;
  uint32_t p = from;
  for (; p + 8 <= to; p += 8) {
    float x[8][8];
#pragma unroll
    for (int q = 0; q < 8; ++q) load8(dY + (int64_t)places[p + q] * a.ldy, have, x[q]);
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += x[q][i];
  }
  if (p < to) {  // the rest: places past the end are the last one again, left out of the sum
    float x[7][8];
#pragma unroll
    for (int q = 0; q < 7; ++q) load8(dY + (int64_t)places[p + q < to ? p + q : to - 1] * a.ldy, have, x[q]);
#pragma unroll
    for (int q = 0; q < 7; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += p + q < to ? x[q][i] : 0.f;
  }
}

template <typename O>
__device__ __forceinline__ void put_row(const GradArgs& a, uint32_t row, int c, int have, float (&sum)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] *= a.scale;
  store8(static_cast<O*>(a.G) + (int64_t)row * a.ldg + c, have, sum);
}

// The first of the sorted keys that is not below `row`.
__device__ __forceinline__ uint32_t lower_bound(const uint2* items, uint32_t n, uint32_t row) {
  uint32_t at = 0;
  while (n) {
    const uint32_t half = n >> 1;
    if (items[at + half].x < row) {
      at += half + 1;
      n -= half + 1;
    } else {
      n = half;
    }
  }
  return at;
}

// Zero rows of the table that no place names: a lane looks for each row, the wavefront writes them.
template <typename O>
__device__ __forceinline__ void zero_rows(const GradArgs& a, uint32_t group) {
  const uint32_t lane = threadIdx.x & 63, per_wave = a.zero_rows / 4, first = group * a.zero_rows + (threadIdx.x >> 6) * per_wave;
  const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (uint32_t r0 = first; r0 < first + per_wave && r0 < a.v; r0 += 64) {
    const uint32_t row = r0 + lane;
    bool empty = row < first + per_wave && row < a.v;
    if (empty) {
      const uint32_t p = lower_bound(a.items, a.t, row);
      empty = p >= a.t || a.items[p].x != row;
    }
    for (uint64_t left = __ballot(empty); left; left &= left - 1) {
      O* g = static_cast<O*>(a.G) + (int64_t)(r0 + __builtin_ctzll(left)) * a.ldg;
      for (int c = lane * 8; c < a.d; c += 512) store8(g + c, a.d - c < 8 ? a.d - c : 8, zero);
    }
  }
}

// Piece `group` sums the runs of equal keys that begin in it.  A run that ends in the piece after it, it follows to its end (and that
// piece leaves it out): two pieces' places at most.  Runs of three pieces or more are long: each piece leaves the sum of its part.
// Eight rows are under way at a time, whichever runs they belong to.
constexpr int SUM_LANES_LOG2 = 3;  // at least: eight lanes a row, 32 groups a workgroup
constexpr int SUM_BATCH = 8;
template <typename T, typename O>
__global__ __launch_bounds__(256) void k_grad_sum(const GradArgs a) {
  constexpr int STRIDE = 2 * CHUNK + SUM_BATCH + 1;
  __shared__ uint32_t key_list[(256 >> SUM_LANES_LOG2) * STRIDE], place_list[(256 >> SUM_LANES_LOG2) * STRIDE];
  if (blockIdx.x >= a.sum_groups) {
    zero_rows<O>(a, blockIdx.x - a.sum_groups);
    return;
  }
  const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1), mine = threadIdx.x >> a.lanes_log2;
  const uint32_t group = blockIdx.x * (256 >> a.lanes_log2) + mine;
  const bool active = (uint64_t)group * CHUNK < a.t;
  const uint32_t p0 = active ? group * CHUNK : 0, most = min(a.t - p0, 2u * CHUNK), here = min(a.t - p0, (uint32_t)CHUNK);
  // the keys and places of this piece and the next
  uint32_t* keys = key_list + mine * STRIDE;
  uint32_t* places = place_list + mine * STRIDE;
  if (active)
    for (uint32_t i = lane; i < most; i += lanes) {
      const uint2 item = a.items[p0 + i];
      keys[i] = item.x;
      places[i] = item.y;
    }
  const uint32_t before = active && p0 ? a.items[p0 - 1].x : 0xFFFFFFFFu, before_that = active && p0 > CHUNK ? a.items[p0 - CHUNK - 1].x : 0xFFFFFFFFu;
  const uint32_t after = active && a.t - p0 > 2 * CHUNK ? a.items[p0 + 2 * CHUNK].x : 0xFFFFFFFFu;
  __syncthreads();
  if (!active) return;
  const uint32_t head = keys[0];
  uint32_t first = 0, stop = here;
  float* head_part = nullptr;
  float* tail_part = nullptr;
  if (before == head) {  // the run began before
    uint32_t end = 1;
    while (end < here && keys[end] == head) ++end;
    const bool ends_here = end < here || here == most || keys[here] != head;
    if (ends_here && before_that != head) first = end;  // it began in the piece before, which follows it
    else head_part = a.parts + (int64_t)group * 2 * a.width;
  }
  const uint32_t tail = keys[here - 1];
  if (here < most && keys[here] == tail && tail < a.v && !(head_part && tail == head)) {
    // the last run, which begins here, goes on: to its end, if the next piece holds it
    while (stop < most && keys[stop] == tail) ++stop;
    if (stop == 2 * CHUNK && after == tail) {
      stop = here;
      tail_part = a.parts + ((int64_t)group * 2 + 1) * a.width;
    }
  }
  if (first >= stop) return;
  const T* dY = static_cast<const T*>(a.dY);
  for (int c = (int)lane * 8; c < a.d; c += 8 * lanes) {
    const int have = a.d - c < 8 ? a.d - c : 8;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float* part = head_part;
    uint32_t row = keys[first];
    auto leave = [&](bool last) {
      if (row >= a.v) return;
      if (last && tail_part) part = tail_part;
      if (part) store8(part + c, sum);
      else put_row<O>(a, row, c, have, sum);
    };
    for (uint32_t p = first; p < stop; p += SUM_BATCH) {
      Eight<T> x[SUM_BATCH];
      if (have == 8) {
#pragma unroll
        for (int q = 0; q < SUM_BATCH; ++q) x[q] = *reinterpret_cast<const Eight<T>*>(dY + (int64_t)places[p + q < stop ? p + q : stop - 1] * a.ldy + c);
      } else {
#pragma unroll
        for (int q = 0; q < SUM_BATCH; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[q].x[i] = i < have ? dY[(int64_t)places[p + q < stop ? p + q : stop - 1] * a.ldy + c + i] : T(0.f);
      }
#pragma unroll
      for (int q = 0; q < SUM_BATCH; ++q) {
        if (p + q < stop) {
          const uint32_t key = keys[p + q];
          if (key != row) {
            leave(false);
            part = nullptr;
            row = key;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] += Element<T>::get(x[q].x[i]);
        }
      }
    }
    leave(true);
  }
}

// Long runs: a workgroup looks through JOIN_PIECES pieces for runs that begin in them, and adds up the parts of each, every
// group of lanes those of some consecutive pieces, then their sums in order.
// 256 threads and four pieces, 512 and eight, 1,024 and sixteen, whole gradients in graphs, frequencies even or as 1 / rank: 400,000 tokens of 2,000 x 64 71, 78,
// 87 and 81, 87, 95 us; 1,000,000 of 5,000 x 128 131, 148, 173 and 146, 146, 166; 200,000 of 1,000 x 300 89, 96, 104 and 117, 113, 118; 100,000 of 100,000 x 256
// 64, 64, 64 and 75, 77, 81; 300,007 of 100,000 x 384 127, 127, 127 and 162, 158, 161.
constexpr int JOIN_THREADS = 256;
constexpr int JOIN_PIECES = 4;
template <typename O>
__global__ __launch_bounds__(JOIN_THREADS) void k_grad_join(const GradArgs a, const uint32_t first_block) {
  __shared__ float sums[JOIN_THREADS * 8];
  __shared__ uint64_t found;
  const uint32_t lane = threadIdx.x & ((1u << a.lanes_log2) - 1), mine = threadIdx.x >> a.lanes_log2, groups = JOIN_THREADS >> a.lanes_log2;
  const uint32_t pieces = (uint32_t)(((uint64_t)a.t + CHUNK - 1) / CHUNK);
  if (threadIdx.x < 64) {
    const uint32_t group = (first_block + blockIdx.x) * JOIN_PIECES + threadIdx.x, p0 = group * CHUNK, p1 = p0 + CHUNK;
    bool begins = threadIdx.x < JOIN_PIECES && (uint64_t)group + 2 < pieces;
    if (begins) {
      const uint32_t row = a.items[p1 - 1].x, third = a.items[p1 + CHUNK].x, first = a.items[p0].x, before = p0 ? a.items[p0 - 1].x : 0xFFFFFFFFu;
      begins = row < a.v && third == row && !(first == row && before == row);  // through the next piece into a third, and did begin here
    }
    const uint64_t mask = __ballot(begins);
    if (threadIdx.x == 0) found = mask;
  }
  __syncthreads();
  for (uint64_t left = found; left; left &= left - 1) {
    const uint32_t group = (first_block + blockIdx.x) * JOIN_PIECES + __builtin_ctzll(left), row = a.items[group * CHUNK + CHUNK - 1].x;
    // parts: of this piece, and of those after it whose first key is the row's (a thread looks at each: a search would wait for the memory some twenty times)
    uint32_t number = 1;
    for (int more = JOIN_THREADS; more == JOIN_THREADS; number += more) {
      const uint64_t p = ((uint64_t)group + number + threadIdx.x) * CHUNK;
      more = __syncthreads_count(p < a.t && a.items[p].x == row);
    }
    const uint32_t per = (number + groups - 1) / groups;
    for (int c0 = 0; c0 < a.d; c0 += 8 << a.lanes_log2) {
      const int c = c0 + (int)lane * 8;
      float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (c < a.d) {
        const uint32_t to = min(number, (mine + 1) * per);
        for (uint32_t i = mine * per; i < to; i += 8) {
          float x[8][8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const uint32_t n = min(i + q, to - 1);
            load8(a.parts + ((int64_t)(group + n) * 2 + (n == 0 ? 1 : 0)) * a.width + c, x[q]);
          }
#pragma unroll
          for (int q = 0; q < 8; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += i + q < to ? x[q][k] : 0.f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) sums[(k * groups + mine) * (1u << a.lanes_log2) + lane] = sum[k];
      __syncthreads();
      // a thread adds up one column of the groups
      const uint32_t columns = 8u << a.lanes_log2;
      for (uint32_t x = threadIdx.x; x < columns; x += JOIN_THREADS) {
        const uint32_t k = x >> a.lanes_log2, l = x & ((1u << a.lanes_log2) - 1), col = c0 + l * 8 + k;
        float total = 0.f;
        for (uint32_t g = 0; g < groups && g * per < number; ++g) total += sums[(k * groups + g) * (1u << a.lanes_log2) + l];
        if ((int)col < a.d) static_cast<O*>(a.G)[(int64_t)row * a.ldg + col] = Element<O>::put(total * a.scale);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Few places: one launch
// ------------------------------------------------------------------------------------------
// A workgroup owns SMALL_ROWS rows of the table or fewer.  It reads all tokens (from the L2: there are few), keeps those of its
// rows in the LDS, puts them in the order of (row, place) and writes its rows.  A row of few places is one group of lanes'; one of
// many is shared by all of them, whose sums are added up in order.  Bound by the launch and the latency of three dependent reads: 2,011 tokens of
// 4,096 rows of 128 11 us.  8,000 tokens of 100,000 x 256 57 to 62 us, by the sort 67; of 2,000 x 96 25 and 49.  Larger tables: every workgroup looks
// through all tokens before it writes its rows, most of them zeros (1,000 of 50,000 x 300 38 us for 61 MB).
constexpr int SMALL_ROWS = 64;
constexpr int SMALL_ALONE = 32;  // places of a row that one group sums
constexpr int SMALL_PLACES = 8192;  // at most

struct SmallArgs {
  GradArgs g;
  const void* tokens;
  uint32_t rows;   // of a workgroup
  uint32_t first;  // workgroup that the launch begins with
};

template <typename T, typename O, typename I, int PLACES, int THREADS>
__global__ __launch_bounds__(THREADS) void k_grad_small(const SmallArgs s) {
  constexpr int WAVES = THREADS / 64;
  __shared__ uint32_t found[PLACES];   // (row << 16 | place) in the order of places
  __shared__ uint16_t sorted[PLACES];  // places in the order of rows
  __shared__ uint32_t begin[SMALL_ROWS + 1], cursor[SMALL_ROWS], scratch[WAVES];
  __shared__ float sums[THREADS * 8];
  const GradArgs& a = s.g;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t row0 = (s.first + blockIdx.x) * s.rows, rows = min(s.rows, a.v - row0);
  if (threadIdx.x < SMALL_ROWS) cursor[threadIdx.x] = 0;
  // each wavefront: its share of the tokens, all under way together
  constexpr int TOKENS = PLACES / THREADS;  // of a lane
  const uint32_t per_wave = (a.t + WAVES * 64 - 1) / (WAVES * 64) * 64, from = wave * per_wave, to = min(a.t, from + per_wave);
  const I* tokens = static_cast<const I*>(s.tokens);
  I token[TOKENS];
#pragma unroll
  for (int q = 0; q < TOKENS; ++q) {
    const uint32_t p = from + q * 64 + lane;
    token[q] = p < to ? tokens[p] : I(-1);
  }
  uint8_t row[TOKENS];  // of the workgroup's, SMALL_ROWS: another's
  uint32_t count = 0;
#pragma unroll
  for (int q = 0; q < TOKENS; ++q) {
    const int64_t r = row_of(token[q], (int64_t)a.v, a.status) - (int64_t)row0;
    row[q] = r >= 0 && r < (int64_t)rows ? (uint8_t)r : (uint8_t)SMALL_ROWS;
    count += __popcll(__ballot(row[q] < SMALL_ROWS));
  }
  if (lane == 0) scratch[wave] = count;
  __syncthreads();
  uint32_t at = 0, total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) at += scratch[w];
    total += scratch[w];
  }
  if (count) {
#pragma unroll
    for (int q = 0; q < TOKENS; ++q) {
      const uint64_t hit = __ballot(row[q] < SMALL_ROWS);
      if (row[q] < SMALL_ROWS) {
        found[at + __popcll(hit & ((1ull << lane) - 1))] = (uint32_t)row[q] << 16 | (from + q * 64 + lane);
        atomicAdd(&cursor[row[q]], 1u);
      }
      at += __popcll(hit);
    }
  }
  __syncthreads();
  if (wave == 0) {
    // where each row's places begin, then the places in order: equal rows of 64 are ranked by their lanes
    const uint32_t n = cursor[lane];
    uint32_t sum = n;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)sum, k);
      if (lane >= k) sum += y;
    }
    begin[lane + 1] = sum;
    if (lane == 0) begin[0] = 0;
    cursor[lane] = sum - n;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (uint32_t p = 0; p < total; p += 64) {
      const bool there = p + lane < total;
      const uint32_t x = there ? found[p + lane] : 0, r = x >> 16;
      uint64_t same = __ballot(there);
#pragma unroll
      for (int b = 0; b < 6; ++b) {
        const uint64_t set = __ballot((r >> b) & 1);
        same &= ((r >> b) & 1) ? set : ~set;
      }
      const uint32_t below = __popcll(same & ((1ull << lane) - 1));
      uint32_t first = 0;
      if (there) first = cursor[r];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (there && below == 0) cursor[r] = first + __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (there) sorted[first + below] = (uint16_t)x;
    }
  }
  __syncthreads();
  const uint32_t l = threadIdx.x & ((1u << a.lanes_log2) - 1), mine = threadIdx.x >> a.lanes_log2, groups = THREADS >> a.lanes_log2;
  const int step = 8 << a.lanes_log2;
  for (uint32_t r = mine; r < rows; r += groups) {
    const uint32_t b = begin[r], e = begin[r + 1];
    if (e - b > SMALL_ALONE) continue;
    for (int c = (int)l * 8; c < a.d; c += step) {
      const int have = a.d - c < 8 ? a.d - c : 8;
      float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      add_rows<T>(a, sorted, b, e, c, have, sum);
      put_row<O>(a, row0 + r, c, have, sum);
    }
  }
  for (uint32_t r = 0; r < rows; ++r) {
    const uint32_t b = begin[r], e = begin[r + 1];
    if (e - b <= SMALL_ALONE) continue;
    const uint32_t per = (e - b + groups - 1) / groups, p0 = min(e, b + mine * per), p1 = min(e, p0 + per);
    for (int c0 = 0; c0 < a.d; c0 += step) {
      const int c = c0 + (int)l * 8;
      float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (c < a.d) add_rows<T>(a, sorted, p0, p1, c, a.d - c < 8 ? a.d - c : 8, sum);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) sums[(k * groups + mine) * (1u << a.lanes_log2) + l] = sum[k];
      __syncthreads();
      for (uint32_t x = threadIdx.x; x < (uint32_t)step; x += THREADS) {
        const uint32_t k = x >> a.lanes_log2, m = x & ((1u << a.lanes_log2) - 1), col = c0 + m * 8 + k;
        float all = 0.f;
        for (uint32_t g = 0; g < groups; ++g) all += sums[(k * groups + g) * (1u << a.lanes_log2) + m];
        if ((int)col < a.d) static_cast<O*>(a.G)[(int64_t)(row0 + r) * a.ldg + col] = Element<O>::put(all * a.scale);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------ host side
bool bad_tokens(const void* tokens, int32_t token_type) { return !tokens || (token_type != EJOIN_I32 && token_type != EJOIN_I64); }

template <typename F>
auto with_index(int32_t type, F f) {
  return type == EJOIN_I64 ? f(int64_t()) : f(int32_t());
}

}  // namespace

extern "C" {

int ejoin_lookup(ejoin_ctx* ctx, const void* table, int32_t type, int64_t v, int32_t d, int64_t ldt, const void* tokens, int32_t token_type, int64_t t,
                 float scale, void* Y, int32_t ytype, int64_t ldy, void* stream) {
  if (!ctx || !table || bad_type(type) || bad_type(ytype) || v < 1 || v >= (1ll << 31) || d < 1 || d > 65536 || ldt < d) return EJOIN_EINVAL;
  if (t < 0 || t >= (1ll << 31) || !isfinite(scale) || ldy < up(d, 64)) return EJOIN_EINVAL;
  if (t == 0) return EJOIN_OK;
  if (!Y || bad_tokens(tokens, token_type)) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  LookupArgs a{table, v, ldt, d, tokens, t, scale, Y, ldy, (uint32_t)(up(d, 64) / 8), ctx->token_status};
  const int64_t units = t * a.chunks, groups = (units + 256 * LOOKUP_PIECES - 1) / (256 * LOOKUP_PIECES);
  if (groups >= 1ll << 24) return EJOIN_EUNSUPPORTED;  // (of 256 threads: Y would be 2^37 values)
  const bool wide = units + 256 * LOOKUP_PIECES >= (1ll << 32);
  // 16-bit results that the memory-side cache does not hold, 307 MB of 400,003 rows of 384, tokens evenly spread over 1,000,000 FP32 rows: 166 us through the
  // caches, 142 past them.  (FP32 ones, whose pieces are two stores, are the slower for it: 102 MB 28 and 40 us.)
  const bool passing = ytype != EJOIN_F32 && t * ldy * 2 > (256ll << 20);
  with_type(type, [&](auto x) {
    with_type(ytype, [&](auto y) {
      with_index(token_type, [&](auto i) {
        typedef decltype(x) X;
        typedef decltype(y) Y;
        typedef decltype(i) I;
        void (*kernel)(LookupArgs) = k_lookup<X, Y, I, false, false>;
        if constexpr (sizeof(Y) == 2) {
          if (passing) kernel = wide ? k_lookup<X, Y, I, true, true> : k_lookup<X, Y, I, false, true>;  // (wide ones are 68 GB)
        } else {
          if (wide) kernel = k_lookup<X, Y, I, true, false>;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream), a);
      });
    });
  });
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

int ejoin_lookup_grad(ejoin_ctx* ctx, const void* dY, int32_t type, int64_t t, int32_t d, int64_t ldy, const void* tokens, int32_t token_type, int64_t v,
                      float scale, void* G, int32_t gtype, int64_t ldg, void* stream) {
  if (!ctx || !G || bad_type(type) || bad_type(gtype) || v < 1 || v >= (1ll << 31) || d < 1 || d > 65536 || ldg < d) return EJOIN_EINVAL;
  if (t < 0 || t >= (1ll << 31) || !isfinite(scale) || ldy < d) return EJOIN_EINVAL;
  if (t > 0 && (!dY || bad_tokens(tokens, token_type))) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int bits = 1;
  while ((v >> bits) != 0) ++bits;  // of v, the key of no token
  const int passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS, digit = (bits + passes - 1) / passes;
  const int64_t blocks = (t + SORT_BLOCK - 1) / SORT_BLOCK, pieces = (t + CHUNK - 1) / CHUNK, width = up(d, 8);
  const int64_t list = up(8 * t, 256), groups = blocks >= SCAN_FROM ? (blocks + SCAN_BLOCKS - 1) / SCAN_BLOCKS : 0;
  const int64_t counts = blocks * DIGITS * 4, group_counts = groups ? (groups + 1) * DIGITS * 4 : 0;
  GradArgs g;
  memset(&g, 0, sizeof(g));
  g.dY = dY, g.ldy = ldy, g.d = d, g.t = (uint32_t)t, g.v = (uint32_t)v, g.scale = scale, g.G = G, g.ldg = ldg;
  g.width = (int32_t)width;
  g.status = ctx->token_status;
  g.lanes_log2 = SUM_LANES_LOG2;
  while (g.lanes_log2 < 6 && (8 << g.lanes_log2) < d) ++g.lanes_log2;

  if (t <= SMALL_PLACES) {
    // some 1,024 workgroups, where there are rows enough
    int64_t rows = (v + 1023) / 1024;
    rows = rows < 8 ? 8 : (rows < SMALL_ROWS ? rows : SMALL_ROWS);
    SmallArgs a{g, tokens, (uint32_t)rows, 0};
    with_type(gtype, [&](auto o) {
      with_type(type, [&](auto x) {
        with_index(token_type, [&](auto i) {
          typedef decltype(x) X;
          typedef decltype(o) O;
          typedef decltype(i) I;
          // (room for no more places than there may be: 1,000 tokens of 50,000 rows of 300 32 us with room for 1,024, 49 with room for 8,192)
          void (*kernel)(SmallArgs) = t <= 1024   ? &k_grad_small<X, O, I, 1024, 256>
                                      : t <= 4096 ? &k_grad_small<X, O, I, 4096, 512>
                                                  : &k_grad_small<X, O, I, SMALL_PLACES, 512>;
          in_launches((v + rows - 1) / rows, [&](int64_t first, unsigned groups) {
            a.first = (uint32_t)first;
            hipLaunchKernelGGL(kernel, dim3(groups), dim3(t <= 1024 ? 256 : 512), 0, st, a);
          });
        });
      });
    });
    EJ_TRY(hipGetLastError());
    return EJOIN_OK;
  }
  EJ_RC(ensure_embed(ctx, 2 * list + counts + group_counts + pieces * 2 * width * 4, st));
  uint2* lists[2] = {reinterpret_cast<uint2*>(ctx->embed), reinterpret_cast<uint2*>(ctx->embed + list)};
  g.parts = reinterpret_cast<float*>(ctx->embed + 2 * list + counts + group_counts);
  SortArgs s;
  memset(&s, 0, sizeof(s));
  s.tokens = tokens, s.counts = reinterpret_cast<uint32_t*>(ctx->embed + 2 * list), s.t = (uint32_t)t, s.v = (uint32_t)v, s.blocks = (uint32_t)blocks;
  s.groups = groups ? s.counts + blocks * DIGITS : nullptr;
  s.mask = (1u << digit) - 1, s.status = ctx->token_status;
  for (int pass = 0; pass < passes; ++pass) {
    s.items = lists[pass & 1], s.items_out = lists[1 - (pass & 1)];
    s.shift = pass * digit;
    const dim3 grid((unsigned)blocks), block(SORT_THREADS);
    auto sort = [&](auto count, auto scatter, auto scatter_scanned) {
      hipLaunchKernelGGL(count, grid, block, 0, st, s);
      if (groups) {
        hipLaunchKernelGGL(k_sort_scan, dim3((unsigned)groups), block, 0, st, s);
        hipLaunchKernelGGL(k_sort_scan_groups, dim3(1), block, 0, st, s, (uint32_t)groups);
      }
      hipLaunchKernelGGL(groups ? scatter_scanned : scatter, grid, block, 0, st, s);
    };
    if (pass == 0) {
      with_index(token_type, [&](auto i) {
        typedef decltype(i) I;
        sort(&k_sort_count<I, true>, &k_sort_scatter<I, true, false>, &k_sort_scatter<I, true, true>);
      });
    } else {
      sort(&k_sort_count<int32_t, false>, &k_sort_scatter<int32_t, false, false>, &k_sort_scatter<int32_t, false, true>);
    }
    EJ_TRY(hipGetLastError());
    g.items = s.items_out;
  }
  g.sum_groups = (uint32_t)(((pieces << g.lanes_log2) + 255) / 256);
  g.zero_rows = 256;
  // (one launch: 2^23 workgroups of zeros at most, and rows of 64 columns, the most that 2^31 places may have, take 2^21 of sums)
  const dim3 grid((unsigned)(g.sum_groups + (v + g.zero_rows - 1) / g.zero_rows));
  with_type(gtype, [&](auto o) {
    typedef decltype(o) O;
    with_type(type, [&](auto x) { hipLaunchKernelGGL((k_grad_sum<decltype(x), O>), grid, dim3(256), 0, st, g); });
    in_launches((pieces + JOIN_PIECES - 1) / JOIN_PIECES,
                [&](int64_t first, unsigned groups) { hipLaunchKernelGGL(k_grad_join<O>, dim3(groups), dim3(JOIN_THREADS), 0, st, g, (uint32_t)first); });
  });
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

int ejoin_embed_status(ejoin_ctx* ctx, int* status) {
  if (!ctx || !status) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  EJ_TRY(hipDeviceSynchronize());
  uint32_t st = 0;
  EJ_TRY(hipMemcpy(&st, ctx->token_status, sizeof(st), hipMemcpyDeviceToHost));
  if (st != 0) {
    const uint32_t none = 0;
    EJ_TRY(hipMemcpy(ctx->token_status, &none, sizeof(none), hipMemcpyHostToDevice));
  }
  *status = (int)st;
  return EJOIN_OK;
}

}  // extern "C"
