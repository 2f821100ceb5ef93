// Eviction by weight: per KV head the first n_sink rows, the last n_recent and, between them, the heaviest, in their order, to the front of this
// layer or to another one.
//
// Two kernels.  The first finds what is kept, a workgroup per KV head: the order of fp32 numbers is that of unsigned ones after a change of the
// upper bits, so that the smallest kept weight is found digit by digit, eight bits at a time, in histograms (32 copies of each, a bank's
// own, as the weights of a cache have few exponents and all lanes would ask for the same counters); then every wavefront walks a piece of the rows
// and numbers those it keeps by ballots.  The second moves the rows: memory-bound, each kept row read and written once, a workgroup's
// 64 rows of K and V all in flight at once.
//
// In place a row goes to a place in front of it, where another row may lie that is kept as well.  A workgroup therefore has all its rows in
// registers, and says so, before it waits for those whose rows lie where it is going to write: their chunks come in front of its own (a kept row is at
// least as far back as its new place), so that they were handed out before it and say so without waiting for anyone.  Chunks are
// handed out by a counter.  What is ordered is a read before a write, so that no cache has to be written back or dropped for it.
#include "weigh.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) unsigned uintx4;

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64, kCopies = 32;

// Larger weights have larger numbers: NaN above everything, both zeros alike.
__device__ __forceinline__ unsigned weight_order(float w) {
  if (w != w) return 0xffffffffu;
  const unsigned x = __float_as_uint(w + 0.f);
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}

__global__ void __launch_bounds__(kSelect) evict_select_kernel(EvictParams p) {
  __shared__ unsigned hist[256 * kCopies];
  __shared__ unsigned count[256];
  __shared__ unsigned digit, above, wave_more[kSelectWaves], wave_same[kSelectWaves];
  const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = blockIdx.x;
  const float* weights = p.weights + (int64_t)g * p.from_capacity;
  const int lo = p.n_sink, hi = p.len - p.n_recent;
  unsigned want = (unsigned)(p.n_keep - p.n_sink - p.n_recent);  // of those that have the digits found so far
  const bool all = want == (unsigned)(hi - lo);

  unsigned found = 0, mask = 0;
  if (want > 0 && !all) {
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256 * kCopies; i += kSelect) hist[i] = 0;
      __syncthreads();
#pragma unroll 4
      for (int j = lo + tid; j < hi; j += kSelect) {
        const unsigned x = weight_order(weights[j]);
        if ((x & mask) == found) atomicAdd(&hist[(x >> shift & 255u) * kCopies + (tid & (kCopies - 1))], 1u);
      }
      __syncthreads();
      if (tid < 256) {
        unsigned n = 0;
        for (int i = 0; i < kCopies; ++i) n += hist[tid * kCopies + ((i + tid) & (kCopies - 1))];
        count[tid] = n;
      }
      __syncthreads();
      if (tid < 64) {  // lane l has digits 255 - 4 l and the three below
        unsigned n[4], sum = 0;
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
            digit = 255u - 4u * (unsigned)tid - (unsigned)i;
            above = before;
          }
          before += n[i];
        }
      }
      __syncthreads();
      found |= digit << shift;
      mask |= 255u << shift;
      want -= above;
      __syncthreads();
    }
  }
  // Kept between the first and the last rows: all above `found`, and the first `want` of those that are it.
  const bool some = want > 0 && !all;
  auto classify = [&](int j, bool& more, bool& same) __attribute__((always_inline)) {
    more = same = false;
    if (j >= p.len) return;
    if (j < lo || j >= hi || all) {
      more = true;
    } else if (some) {
      const unsigned x = weight_order(weights[j]);
      more = x > found;
      same = x == found;
    }
  };
  const int piece = ((p.len + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, begin = w * piece, end = begin + piece < p.len ? begin + piece : p.len;
  unsigned n_more = 0, n_same = 0;
#pragma unroll 4
  for (int j0 = begin; j0 < end; j0 += 64) {
    bool more, same;
    classify(j0 + l, more, same);
    n_more += (unsigned)__popcll(__ballot(more));
    n_same += (unsigned)__popcll(__ballot(same));
  }
  if (l == 0) wave_more[w] = n_more, wave_same[w] = n_same;
  __syncthreads();
  n_more = n_same = 0;
  for (int i = 0; i < w; ++i) n_more += wave_more[i], n_same += wave_same[i];
  unsigned at = n_more + (n_same < want ? n_same : want);
  int32_t* kept = p.kept + (int64_t)g * p.n_keep;
  float* kept_weights = reinterpret_cast<float*>(p.workspace + p.ws.weights) + (int64_t)g * p.n_keep;
  uint32_t* before = p.workspace + p.ws.before + (int64_t)g * (p.ws.chunks + 1);
  const uint64_t lower = (1ull << l) - 1;
#pragma unroll 4
  for (int j0 = begin; j0 < end; j0 += 64) {
    const int j = j0 + l;
    bool more, same;
    classify(j, more, same);
    const uint64_t equal = __ballot(same);
    const bool keep = more || (same && n_same + (unsigned)__popcll(equal & lower) < want);
    const uint64_t kept_here = __ballot(keep);
    static_assert(kEvictRows == 64, "a chunk begins where a wavefront's turn does");
    if (l == 0 && j0 / kEvictRows <= p.ws.chunks) before[j0 / kEvictRows] = at;
    if (keep) {
      const unsigned i = at + (unsigned)__popcll(kept_here & lower);
      kept[i] = j;
      kept_weights[i] = weights[j];
    }
    at += (unsigned)__popcll(kept_here);
    n_same += (unsigned)__popcll(equal);
  }
  uint32_t* read = p.workspace + p.ws.read + (int64_t)g * p.ws.chunks;
  for (int i = tid; i < p.ws.chunks; i += kSelect) read[i] = 0;
  if (tid == 0 && p.ws.chunks * kEvictRows >= p.len) before[p.ws.chunks] = (uint32_t)p.n_keep;
  if (tid == 0 && g == 0) p.workspace[p.ws.next] = 0;
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
      // the kept rows that lie in places row0 .. row0 + n - 1: their numbers, and the chunks that these are in
      const uint32_t* before = p.workspace + p.ws.before + (int64_t)g * (p.ws.chunks + 1) + chunk;
      const uint32_t first = before[0], end = before[1];
      for (int other = (int)(first / kEvictRows); other < chunk && (uint32_t)other * kEvictRows < end; ++other)
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
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)p.n_kv_heads), dim3(kSelect), 0, s, p);
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
