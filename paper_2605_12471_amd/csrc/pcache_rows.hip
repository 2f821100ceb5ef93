// The cache in pages: where new tokens go (assign), and rows to their places (append).
#include "pcache.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) unsigned uintx4;

// ---- assign ------------------------------------------------------------------------------------------------------------
// A few thousand numbers: bound by the chain inside one launch.  Every workgroup goes through all requests for itself, twice: for the totals, which say
// whether anything is assigned at all, and for the running sums, from which it takes the tokens that are its share of the places (a long prompt's are shared
// out like any others').  So nobody waits for another workgroup, there is one launch and no memory of its own.  A page is written into its table by the thread
// whose token is the page's first.
constexpr int kAssignThreads = 256;

struct Sums {
  int64_t tokens, pages;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return Sums{a.tokens + b.tokens, a.pages + b.pages}; }
__device__ __forceinline__ Sums from_lane(const Sums& a, int lane) { return Sums{(int64_t)__shfl(a.tokens, lane), (int64_t)__shfl(a.pages, lane)}; }

// The sum of the block's values in front of the thread's own; *total: of all.  red: a wavefront's sums.
__device__ __forceinline__ Sums scan(const Sums& mine, Sums* red, Sums* total) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  Sums x = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const Sums y = from_lane(x, l < d ? l : l - d);
    if (l >= d) x = x + y;
  }
  __syncthreads();  // (red may still be read)
  if (l == 63) red[w] = x;
  __syncthreads();
  Sums front = {0, 0}, all = {0, 0};
#pragma unroll
  for (int i = 0; i < kAssignThreads / 64; ++i) {
    if (i < w) front = front + red[i];
    all = all + red[i];
  }
  *total = all;
  return Sums{front.tokens + x.tokens - mine.tokens, front.pages + x.pages - mine.pages};
}

__global__ void __launch_bounds__(kAssignThreads) assign_kernel(AssignParams p) {
  constexpr int NT = kAssignThreads;
  __shared__ Sums red[NT / 64];
  __shared__ int wrong;
  __shared__ int64_t cu[NT + 1], first_page[NT];
  __shared__ int held[NT], before[NT];  // pages, tokens
  const int tid = threadIdx.x, lg = p.page_log2, page = 1 << lg;
  const int64_t t0 = p.n_slots * (int64_t)blockIdx.x / gridDim.x, t1 = p.n_slots * (int64_t)(blockIdx.x + 1) / gridDim.x;

  auto pages_of = [&](int64_t n) -> int64_t { return (n + page - 1) >> lg; };
  // ---- the totals
  if (tid == 0) wrong = 0;
  __syncthreads();
  Sums mine = {0, 0}, total;
  int flags = 0;
  for (int s = tid; s < p.n_seqs; s += NT) {
    const int64_t len = p.lens[s], more = p.n_new[s];
    if (len < 0 || more < 0) {
      flags |= 8;
      continue;
    }
    const int64_t after = pages_of(len + more);
    if (after > p.table_stride || len + more > 0x7fffffff) flags |= 2;
    mine = mine + Sums{more, after - pages_of(len)};
  }
  if (flags) atomicOr(&wrong, flags);
  (void)scan(mine, red, &total);
  int n_free = *p.n_free;
  n_free = n_free < 0 ? 0 : n_free > p.n_pages ? p.n_pages : n_free;
  int status = wrong;
  if (total.pages > n_free) status |= 1;
  if (total.tokens > p.n_slots) status |= 4;
  const bool ok = status == 0;
  if (blockIdx.x == 0 && tid == 0) {
    *p.status = status;
    *p.n_free_after = ok ? n_free - (int)total.pages : *p.n_free;
    p.cu_new[0] = 0;
  }

  // ---- the requests in order, NT at a time
  int64_t tokens = 0, pages = 0;
  for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
    const int s = s0 + tid, n_here = p.n_seqs - s0 < NT ? p.n_seqs - s0 : NT;
    int64_t len = 0, more = 0;
    if (s < p.n_seqs) {
      len = p.lens[s];
      more = ok ? p.n_new[s] : 0;
    }
    const Sums own = {more, ok ? pages_of(len + more) - pages_of(len) : 0};
    const Sums front = scan(own, red, &total);
    cu[tid] = tokens + front.tokens;
    first_page[tid] = pages + front.pages;
    held[tid] = ok ? (int)pages_of(len) : 0;
    before[tid] = (int)len;
    if (tid == 0) cu[NT] = tokens + total.tokens;
    if (blockIdx.x == (unsigned)(s0 / NT) % gridDim.x && s < p.n_seqs) {
      p.lens_after[s] = (int32_t)(len + more);
      p.cu_new[s + 1] = (int32_t)(tokens + front.tokens + more);
    }
    __syncthreads();
    const int64_t from = t0 > tokens ? t0 : tokens, to = t1 < tokens + total.tokens ? t1 : tokens + total.tokens;
    for (int64_t t = from + tid; t < to; t += NT) {
      int lo = 0, hi = n_here;  // the last request with cu <= t, which has tokens
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t)
          lo = mid;
        else
          hi = mid;
      }
      const int64_t at = before[lo] + (t - cu[lo]), column = at >> lg, lacking = column - held[lo];
      int32_t* row = p.tables + (int64_t)(s0 + lo) * p.table_stride;
      int32_t number;
      if (lacking < 0) {
        number = row[column];
      } else {
        number = p.free_pages[n_free - 1 - first_page[lo] - lacking];
        if ((at & (page - 1)) == 0) row[column] = number;
      }
      p.slots[t] = (int64_t)number * page + (at & (page - 1));
      if (p.positions) p.positions[t] = (int32_t)at;
    }
    tokens += total.tokens;
    pages += total.pages;
    __syncthreads();
  }
  for (int64_t t = (t0 > tokens ? t0 : tokens) + tid; t < t1; t += NT) {
    p.slots[t] = -1;
    if (p.positions) p.positions[t] = -1;
  }
}

hipError_t launch_assign(const AssignParams& p, int n_cu, hipStream_t s) {
  int64_t wgs = (p.n_slots + 4 * kAssignThreads - 1) / (4 * kAssignThreads);
  wgs = wgs < 1 ? 1 : wgs > n_cu ? n_cu : wgs;
  hipLaunchKernelGGL(assign_kernel, dim3((unsigned)wgs), dim3(kAssignThreads), 0, s, p);
  return hipGetLastError();
}

// ---- append ------------------------------------------------------------------------------------------------------------
// 16 bytes a thread and turn, neighbours side by side in a row: bound by memory, every row read and written once.
__global__ void __launch_bounds__(256) pappend_kernel(PAppendParams p, int per_row_log2, unsigned per_token, FastDiv by_token) {
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  const unsigned t = quot(i, by_token);
  if (t >= (unsigned)p.n_tokens) return;
  const unsigned c = i - t * per_token, g = c >> per_row_log2, at = (c & ((1u << per_row_log2) - 1)) * 16;
  const int64_t slot = p.slots[t];
  if ((uint64_t)slot >= (uint64_t)p.n_places) return;
  const uint64_t from = (uint64_t)t * (uint64_t)p.token_bytes + (uint64_t)g * (unsigned)p.row_bytes + at;
  const uint64_t row = ((((uint64_t)slot >> p.page_log2) * (unsigned)p.n_kv_heads + g) << p.page_log2) + ((uint64_t)slot & ((1u << p.page_log2) - 1));
  const uint64_t to = row * (unsigned)p.row_bytes + at;
  const uintx4 k = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.k) + from);
  const uintx4 v = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.v) + from);
  *reinterpret_cast<uintx4*>(static_cast<unsigned char*>(p.k_pages) + to) = k;
  *reinterpret_cast<uintx4*>(static_cast<unsigned char*>(p.v_pages) + to) = v;
}

hipError_t launch_pappend(const PAppendParams& p, hipStream_t s) {
  const int chunks = p.row_bytes / 16;  // 8, 16 or 32
  int lg = 0;
  while ((1 << lg) < chunks) ++lg;
  const unsigned per_token = (unsigned)(p.n_kv_heads * chunks);
  // (a launch has at most 2^31 threads' worth of 16 bytes: quot()'s range)
  const int64_t most = ((int64_t)1 << 30) / per_token;
  PAppendParams q = p;
  for (int64_t t = 0; t < p.n_tokens; t += most) {
    q.k = static_cast<const unsigned char*>(p.k) + t * p.token_bytes;
    q.v = static_cast<const unsigned char*>(p.v) + t * p.token_bytes;
    q.slots = p.slots + t;
    q.n_tokens = (int32_t)(p.n_tokens - t < most ? p.n_tokens - t : most);
    const int64_t threads = (int64_t)q.n_tokens * per_token;
    hipLaunchKernelGGL(pappend_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, q, lg, per_token, fast_div((int)per_token));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace kvfold
