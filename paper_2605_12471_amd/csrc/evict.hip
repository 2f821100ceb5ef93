// Eviction by weight: per KV head the first n_sink rows, the last n_recent and, between them, the heaviest, in their order, to the front of this
// layer or to another one.
//
// First what is kept is found: the order of fp32 numbers is that of unsigned ones after a change of the upper bits, so that the smallest kept
// weight is found digit by digit, eight bits at a time, by counting the digit's values among the rows that have the digits so far; then every
// wavefront numbers the rows that it keeps by ballots.  Up to 8192 rows are one workgroup's, whose weights stay in registers; a longer head is
// shared out in pieces, a launch per digit (one workgroup alone is bound by its vector instructions: 128K rows 163 us).  Then the rows are
// moved: memory-bound, each kept row read and written once, a workgroup's 64 rows of K and V all in flight at once.
//
// In place a row goes to a place in front of it, where another row may lie that is kept as well.  A workgroup therefore has all its rows in
// registers, and says so, before it waits for those whose rows lie where it is going to write: their chunks come in front of its own (a kept row is at
// least as far back as its new place), so that they were handed out before it and say so without waiting for anyone.  Chunks are
// handed out by a counter.  What is ordered is a read before a write, so that no cache has to be written back or dropped for it.
#include "weigh.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) unsigned uintx4;

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;

// Turns of 64 rows that each of a workgroup's wavefronts has
__host__ __device__ inline int evict_turns(int len) { return (len + kSelect - 1) / kSelect; }

// Larger weights have larger numbers: NaN above everything, both zeros alike.
__device__ __forceinline__ unsigned weight_order(float w) {
  if (w != w) return 0xffffffffu;
  const unsigned x = __float_as_uint(w + 0.f);
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// The weights of a workgroup's rows begin .. begin + 1024 TURNS - 1, as their order, in registers: wavefront w, lane l, turn i has row begin + 64 (w turns + i) + l.
template <int TURNS>
struct Held {
  unsigned x[TURNS] = {};
  int turns, first;
  const float* weights;
  __device__ __forceinline__ Held(const EvictParams& p, int g, int begin, int turns_, bool load) : turns(turns_) {
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    weights = p.weights + (int64_t)g * p.from_capacity;
    first = begin + 64 * w * turns + l;
    if (!load) return;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int j = first + 64 * i;
      if (i < turns) x[i] = weight_order(weights[j < p.len ? j : p.len - 1]);
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
      if (i < turns) f(first + 64 * i, x[i]);
  }
};

// Counts of a digit's 256 values, COPIES of each, a bank's own: the weights of a cache have few exponents, and all lanes would ask for the same counter.
template <int COPIES>
struct Histogram {
  unsigned n[256 * COPIES];
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < 256 * COPIES; i += kSelect) n[i] = 0;
  }
  __device__ __forceinline__ void add(unsigned value) { atomicAdd(&n[value * COPIES + (threadIdx.x & (COPIES - 1))], 1u); }
  __device__ __forceinline__ unsigned total(unsigned value) const {
    unsigned sum = 0;
#pragma unroll 8
    for (int i = 0; i < COPIES; ++i) sum += n[value * COPIES + ((i + value) & (COPIES - 1))];
    return sum;
  }
};

// The largest value of the digit of which, with those above it, there are at least `want`; how many are above it.  By the first wavefront, from the
// counts of all values in LDS.
__device__ __forceinline__ void find_digit(const unsigned* count, unsigned want, unsigned* digit, unsigned* above) {
  const int tid = threadIdx.x;
  if (tid >= 64) return;
  unsigned n[4], sum = 0;  // lane l has values 255 - 4 l and the three below
#pragma unroll
  for (int i = 0; i < 4; ++i) sum += n[i] = count[255 - 4 * tid - i];
  unsigned before = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const unsigned x = (unsigned)__shfl_up((int)before, off);
    if (tid >= off) before += x;
  }
  before -= sum;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (before < want && want <= before + n[i]) {
      *digit = 255u - 4u * (unsigned)tid - (unsigned)i;
      *above = before;
    }
    before += n[i];
  }
}

// What is kept between the first and the last rows: all rows, or those above `found` and the first `want` of those that are it (none: want = 0).
struct Bound {
  int lo, hi;
  unsigned want, found;
  bool all, some;
  __device__ __forceinline__ Bound(const EvictParams& p) : lo(p.n_sink), hi(p.len - p.n_recent), want((unsigned)(p.n_keep - p.n_sink - p.n_recent)), found(0) {
    all = want == (unsigned)(hi - lo);
    some = want > 0 && !all;
  }
  __device__ __forceinline__ bool between(int j) const { return j >= lo && j < hi; }
};

// Writes down the kept rows of a workgroup, whose first has the number at[0]; same[0]: rows in front that are `found`.
template <int TURNS>
__device__ __forceinline__ void number_rows(const EvictParams& p, int g, const Held<TURNS>& rows, const Bound& b, unsigned kept_in_front, unsigned same_in_front,
                                            unsigned* wave_more, unsigned* wave_same) {
  const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto classify = [&](int j, unsigned x, bool& more, bool& same) __attribute__((always_inline)) {
    const bool between = b.between(j) && !b.all;
    more = j < p.len && (!between || (b.some && x > b.found));
    same = between && b.some && x == b.found;
  };
  unsigned n_more = 0, n_same = 0;
  rows.each([&](int j, unsigned x) __attribute__((always_inline)) {
    bool more, same;
    classify(j, x, more, same);
    n_more += (unsigned)__popcll(__ballot(more));
    n_same += (unsigned)__popcll(__ballot(same));
  });
  if (l == 0) wave_more[w] = n_more, wave_same[w] = n_same;
  __syncthreads();
  n_more = kept_in_front;
  n_same = same_in_front;
  for (int i = 0; i < w; ++i) n_more += wave_more[i], n_same += wave_same[i];
  unsigned at = n_more + (n_same < b.want ? n_same : b.want);
  int32_t* kept = p.kept + (int64_t)g * p.n_keep;
  float* kept_weights = reinterpret_cast<float*>(p.workspace + p.ws.weights) + (int64_t)g * p.n_keep;
  uint32_t* before = p.workspace + p.ws.before + (int64_t)g * (p.ws.chunks + 1);
  const uint64_t lower = (1ull << l) - 1;
  static_assert(kEvictRows == 64, "a chunk begins where a wavefront's turn does");
  rows.each([&](int j, unsigned x) __attribute__((always_inline)) {
    bool more, same;
    classify(j, x, more, same);
    const uint64_t equal = __ballot(same);
    const bool keep = more || (same && n_same + (unsigned)__popcll(equal & lower) < b.want);
    const uint64_t kept_here = __ballot(keep);
    if (l == 0 && j < p.len && j / kEvictRows <= p.ws.chunks) before[j / kEvictRows] = at;
    if (keep) {
      const unsigned i = at + (unsigned)__popcll(kept_here & lower);
      kept[i] = j;
      kept_weights[i] = rows.weights[j];
    }
    at += (unsigned)__popcll(kept_here);
    n_same += (unsigned)__popcll(equal);
  });
}

// What the moving workgroups begin with, a share of it for each of the head's `n` workgroups
__device__ __forceinline__ void begin_moving(const EvictParams& p, int g, int part, int n) {
  uint32_t* read = p.workspace + p.ws.read + (int64_t)g * p.ws.chunks;
  for (int i = part * kSelect + (int)threadIdx.x; i < p.ws.chunks; i += n * kSelect) read[i] = 0;
  if (threadIdx.x || part) return;
  if (p.ws.chunks * kEvictRows >= p.len) p.workspace[p.ws.before + (int64_t)g * (p.ws.chunks + 1) + p.ws.chunks] = (uint32_t)p.n_keep;
  if (g == 0) p.workspace[p.ws.next] = 0;
}

// A workgroup per KV head, whose weights stay in its registers.
template <int TURNS, int COPIES>
__global__ void __launch_bounds__(kSelect) evict_select_kernel(EvictParams p) {
  __shared__ Histogram<COPIES> hist;
  __shared__ unsigned count[256], digit, above, wave_more[kSelectWaves], wave_same[kSelectWaves];
  const int tid = threadIdx.x, g = blockIdx.x;
  Bound b(p);
  const Held<TURNS> rows(p, g, 0, evict_turns(p.len), b.some);
  if (b.some) {
    unsigned mask = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist.clear();
      __syncthreads();
      rows.each([&](int j, unsigned x) __attribute__((always_inline)) {
        if (b.between(j) && (x & mask) == b.found) hist.add(x >> shift & 255u);
      });
      __syncthreads();
      if (tid < 256) count[tid] = hist.total(tid);
      __syncthreads();
      find_digit(count, b.want, &digit, &above);
      __syncthreads();
      b.found |= digit << shift;
      mask |= 255u << shift;
      b.want -= above;
    }
  }
  number_rows(p, g, rows, b, 0, 0, wave_more, wave_same);
  begin_moving(p, g, 0, 1);
}

// Long caches: a workgroup per piece of kEvictPiece rows, a launch per digit.  Each counts the digit's values among its rows that have the digits found
// so far, and begins with the pieces' counts of the digit before, from which it finds that digit by itself; the last launch has all
// it needs to number its rows: what the pieces in front keep follows from the same counts.
//   DIGIT 0 .. 3: count that digit (after finding the one before); 4: number the rows.
template <int DIGIT>
__global__ void __launch_bounds__(kSelect) evict_digit_kernel(EvictParams p) {
  constexpr int COPIES = 32, PARTS = kSelect / 256;
  __shared__ Histogram<COPIES> hist;
  __shared__ unsigned sums[PARTS][256], front[PARTS][256], count[256], digit, above, mine, more_in_front, same_in_front;
  const int tid = threadIdx.x, l = tid & 63, piece = blockIdx.x, g = blockIdx.y, pieces = gridDim.x, value = tid & 255, part = tid >> 8;
  Bound b(p);
  const Held<kEvictPiece / kSelect> rows(p, g, piece * kEvictPiece, kEvictPiece / kSelect, b.some);
  const size_t set = 256 * (size_t)p.n_kv_heads * (size_t)p.ws.pieces;
  uint32_t* counts = p.workspace + p.ws.counts;
  const uint32_t* last = counts + (DIGIT + 1) % 2 * set + 256 * ((size_t)g * (size_t)p.ws.pieces);
  uint32_t* state = p.workspace + p.ws.state;  // what was known when the digit before was counted
  uint32_t* more = p.workspace + p.ws.more + (size_t)g * (size_t)p.ws.pieces;
  unsigned mask = 0;
  if (b.some && DIGIT > 0) {
    if (DIGIT > 1) {
      b.found = state[(DIGIT % 2 * p.n_kv_heads + g) * 2];
      b.want = state[(DIGIT % 2 * p.n_kv_heads + g) * 2 + 1];
    }
    unsigned sum = 0, in_front = 0;
#pragma unroll 4
    for (int i = part; i < pieces; i += PARTS) {
      const unsigned n = last[256 * (size_t)i + value];
      sum += n;
      if (i < piece) in_front += n;
    }
    sums[part][value] = sum;
    front[part][value] = in_front;
    if (tid == 0) mine = more_in_front = same_in_front = 0;
    __syncthreads();
    if (tid < 256) {
      unsigned n = 0;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) n += sums[i][tid];
      count[tid] = n;
    }
    __syncthreads();
    find_digit(count, b.want, &digit, &above);
    __syncthreads();
    const unsigned d = digit;
    b.found |= d << (32 - 8 * DIGIT);
    b.want -= above;
    mask = ~0u << (32 - 8 * DIGIT);
    // the piece's own rows above the digit found, and in the end those in front
    if (DIGIT < 4 && tid < 256) {
      unsigned n = value > (int)d ? last[256 * (size_t)piece + value] : 0;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) n += (unsigned)__shfl_xor((int)n, off);
      if (l == 0) atomicAdd(&mine, n);
    }
    if (DIGIT == 4) {
      unsigned n = value > (int)d ? front[part][value] : 0;
      for (int i = tid; i < piece; i += kSelect) n += more[i];
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) n += (unsigned)__shfl_xor((int)n, off);
      if (l == 0) atomicAdd(&more_in_front, n);
      if (value == (int)d) atomicAdd(&same_in_front, front[part][value]);
    }
    __syncthreads();
    if (DIGIT < 4 && tid == 0) {
      more[piece] = (DIGIT > 1 ? more[piece] : 0) + mine;
      if (piece == 0) {
        state[((DIGIT + 1) % 2 * p.n_kv_heads + g) * 2] = b.found;
        state[((DIGIT + 1) % 2 * p.n_kv_heads + g) * 2 + 1] = b.want;
      }
    }
  }
  if constexpr (DIGIT < 4) {
    if (!b.some) return;
    hist.clear();
    __syncthreads();
    rows.each([&](int j, unsigned x) __attribute__((always_inline)) {
      if (b.between(j) && (x & mask) == b.found) hist.add(x >> (24 - 8 * DIGIT) & 255u);
    });
    __syncthreads();
    if (tid < 256) counts[DIGIT % 2 * set + 256 * ((size_t)g * (size_t)p.ws.pieces + (size_t)piece) + tid] = hist.total(tid);
  } else {
    __shared__ unsigned wave_more[kSelectWaves], wave_same[kSelectWaves];
    // rows in front that are kept whatever they weigh
    const int begin = piece * kEvictPiece;
    unsigned in_front = b.all ? (unsigned)begin : (unsigned)((begin < b.lo ? begin : b.lo) + (begin > b.hi ? begin - b.hi : 0));
    number_rows(p, g, rows, b, in_front + (b.some ? more_in_front : 0), b.some ? same_in_front : 0, wave_more, wave_same);
    begin_moving(p, g, piece, pieces);
  }
}

template <int ROW>  // bytes of a row
__global__ void __launch_bounds__(256) evict_move_kernel(EvictParams p) {
  constexpr int V = ROW / 16, T = kEvictRows * V / 256;  // vectors of a row, and of a thread's share of K (of V)
  __shared__ unsigned turn;
  const int tid = threadIdx.x;
  unsigned t = blockIdx.x;
  if (p.in_place) {
    if (tid == 0) turn = atomicAdd(p.workspace + p.ws.next, 1u);
    __syncthreads();
    t = turn;
  }
  const int chunk = (int)(t / (unsigned)p.n_kv_heads), g = (int)(t % (unsigned)p.n_kv_heads);
  const int row0 = chunk * kEvictRows, n = p.n_keep - row0 < kEvictRows ? p.n_keep - row0 : kEvictRows;
  const int32_t* kept = p.kept + (int64_t)g * p.n_keep + row0;

  uintx4 x[2][T];
  bool move[T];
#pragma unroll
  for (int j = 0; j < T; ++j) {
    const int i = tid + 256 * j, r = i / V, c = i % V, src = kept[r < n ? r : n - 1];
    move[j] = r < n && !(p.in_place && src == row0 + r);
    const int64_t from = ((int64_t)g * p.from_capacity + src) * ROW + c * 16;
#pragma unroll
    for (int v = 0; v < 2; ++v) x[v][j] = *reinterpret_cast<const uintx4*>(p.from[v] + from);
  }
  if (p.in_place) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
      uint32_t* read = p.workspace + p.ws.read + (int64_t)g * p.ws.chunks;
      __hip_atomic_store(read + chunk, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const uint32_t* before = p.workspace + p.ws.before + (int64_t)g * (p.ws.chunks + 1) + chunk;
      const EvictWaits others = evict_waits(before[0], before[1], chunk);
      for (int other = others.from; other < others.to; ++other)
        while (__hip_atomic_load(read + other, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0) __builtin_amdgcn_s_sleep(1);
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < T; ++j) {
    if (!move[j]) continue;
    const int i = tid + 256 * j, r = i / V, c = i % V;
    const int64_t to = ((int64_t)g * p.to_capacity + row0 + r) * ROW + c * 16;
#pragma unroll
    for (int v = 0; v < 2; ++v) *reinterpret_cast<uintx4*>(p.to[v] + to) = x[v][j];
  }
  if (p.to_weights) {
    float* to = p.to_weights + (int64_t)g * p.to_capacity;
    if (tid < n) to[row0 + tid] = reinterpret_cast<const float*>(p.workspace + p.ws.weights)[(int64_t)g * p.n_keep + row0 + tid];
    // the places behind the kept rows begin at nothing, a share of them for every chunk
    const int64_t rest = p.to_capacity - p.n_keep, share = (rest + p.ws.chunks - 1) / p.ws.chunks, b = share * chunk, e = b + share < rest ? b + share : rest;
    for (int64_t i = b + tid; i < e; i += 256) to[p.n_keep + i] = 0.f;
  }
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const dim3 heads((unsigned)p.n_kv_heads), threads(kSelect);
  const int turns = evict_turns(p.len);
  if (turns <= 4) {
    hipLaunchKernelGGL((evict_select_kernel<4, 8>), heads, threads, 0, s, p);
  } else if (turns <= kEvictPiece / kSelect) {
    hipLaunchKernelGGL((evict_select_kernel<kEvictPiece / kSelect, 32>), heads, threads, 0, s, p);
  } else {
    const dim3 pieces((unsigned)((p.len + kEvictPiece - 1) / kEvictPiece), (unsigned)p.n_kv_heads);
    if (p.n_keep > p.n_sink + p.n_recent && p.n_keep < p.len) {
      hipLaunchKernelGGL(evict_digit_kernel<0>, pieces, threads, 0, s, p);
      hipLaunchKernelGGL(evict_digit_kernel<1>, pieces, threads, 0, s, p);
      hipLaunchKernelGGL(evict_digit_kernel<2>, pieces, threads, 0, s, p);
      hipLaunchKernelGGL(evict_digit_kernel<3>, pieces, threads, 0, s, p);
    }
    hipLaunchKernelGGL(evict_digit_kernel<4>, pieces, threads, 0, s, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(p.ws.chunks * p.n_kv_heads)), block(256);
  if (p.row_bytes == 128)
    hipLaunchKernelGGL(evict_move_kernel<128>, grid, block, 0, s, p);
  else if (p.row_bytes == 256)
    hipLaunchKernelGGL(evict_move_kernel<256>, grid, block, 0, s, p);
  else
    hipLaunchKernelGGL(evict_move_kernel<512>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
