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

// ---- the list of a batch's work ------------------------------------------------------------------------------------------
// Every sequence's packed rows in blocks, and each block's keys in pieces where that fills the GPU more evenly: it has room for so many workgroups at a time, and
// sequences differ.  With W tiles in all and N workgroups, pieces of a place's share of them, W / places, or a half ... a sixth of it, are compared with none at
// all, by the time of (in tiles)
//   the longest piece and what a workgroup does once, where all are there at the same time; else W and N times what it does once over the places, and half of the
//   longest for the last round's gaps; and for pieces what they cost besides.
// The longest come first (five classes).  One workgroup, beside the others that bring the new rows to their places: bound by its chain.  It takes as long as they
// do for a few hundred tokens.
constexpr int kPlanThreads = 256;
constexpr int kPlanClasses = 5, kPlanCounts = kPlanClasses + 1;  // (the last: blocks that are to be merged)

// The block's sums of N values each, for all threads
template <int N>
__device__ __forceinline__ void block_sums(int64_t (&x)[N], int64_t (*red)[kPlanThreads / 64]) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x[i] += __shfl_xor(x[i], d);
  __syncthreads();
  if (l == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[i][w] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = 0;
#pragma unroll
    for (int j = 0; j < kPlanThreads / 64; ++j) x[i] += red[i][j];
  }
}
// The sums of what stands in front of the thread's own values; all[i]: of all
template <int N>
__device__ __forceinline__ void block_scan(int (&x)[N], int (&all)[N], int64_t (*red)[kPlanThreads / 64]) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  int y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    y[i] = x[i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int z = __shfl_up(y[i], d);
      if (l >= d) y[i] += z;
    }
  }
  __syncthreads();
  if (l == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) red[i][w] = y[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int before = 0;
    all[i] = 0;
#pragma unroll
    for (int j = 0; j < kPlanThreads / 64; ++j) {
      const int z = (int)red[i][j];
      if (j < w) before += z;
      all[i] += z;
    }
    x[i] = before + y[i] - x[i];
  }
}

__device__ void prompt_plan(const PromptPlanParams& p) {
  constexpr int NT = kPlanThreads;
  __shared__ int64_t red[kPromptShares > kPlanCounts ? kPromptShares : kPlanCounts][NT / 64];
  __shared__ int front[NT];  // items in front of a sequence's
  __shared__ PagedSeq held[NT];
  const int tid = threadIdx.x;
  const bool once = p.n_seqs <= NT;  // each thread has one sequence, for good
  auto fetch = [&](int s) -> PagedSeq {
    if (s >= p.n_seqs) return PagedSeq{0, 0, 0};
    return paged_seq(p.cu_new ? p.cu_new[s] : s, p.cu_new ? p.cu_new[s + 1] : s + 1, p.lens[s], p.n_tokens, p.max_new, p.max_len);
  };
  const PagedSeq own = fetch(tid);
  auto seq_at = [&](int s0) -> PagedSeq { return s0 ? fetch(s0 + tid) : own; };
  auto blocks_of = [&](const PagedSeq& q) -> int { return (int)((unsigned)(q.n * p.group + p.unit_rows - 1) / (unsigned)p.unit_rows); };
  auto tiles_of = [&](const PagedSeq& q) -> int { return (q.len + 63) / 64; };

  // ---- the pieces' length, in tiles
  int64_t sums[2] = {0, 0};  // tiles, blocks
  int most = 2;
  for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
    const PagedSeq q = seq_at(s0);
    const int nb = blocks_of(q), keys = q.len - q.n / 2;
    sums[0] += (int64_t)nb * ((keys > 0 ? keys : 0) / 64 + 1);
    sums[1] += nb;
    if (nb && tiles_of(q) > most) most = tiles_of(q);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) {
    const int y = __shfl_xor(most, d);
    most = y > most ? y : most;
  }
  if ((tid & 63) == 0) front[tid >> 6] = most;
  block_sums(sums, red);
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) most = front[i] > most ? front[i] : most;
  most = (most + 1) / 2 * 2;  // (pieces are whole steps of 128 keys)
  const int64_t work = sums[0] * p.n_kv_heads;
  int piece = most;
  if (p.n_pieces > 1) {
    int len[kPromptShares];
    int64_t n[kPromptShares];
    const int64_t share = (work + p.n_places - 1) / p.n_places;
    const int least = (most + p.n_pieces - 1) / p.n_pieces;
#pragma unroll
    for (int k = 0; k < kPromptShares; ++k) {
      int64_t x = (share + k) / (k + 1);
      x = x < least ? least : x;
      x = x < p.shortest ? p.shortest : x;
      len[k] = x < most ? ((int)x + 1) / 2 * 2 : most;
      n[k] = 0;
    }
    for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
      const PagedSeq q = seq_at(s0);
      const int nb = blocks_of(q), tiles = tiles_of(q);
#pragma unroll
      for (int k = 0; k < kPromptShares; ++k) n[k] += (int64_t)nb * (int)((unsigned)(tiles + len[k] - 1) / (unsigned)len[k]);
    }
    block_sums(n, red);
    auto cost = [&](int longest, int64_t wgs, int each) -> int64_t {
      return wgs <= p.n_places ? longest + each : (work + wgs * each) / p.n_places + (longest + each) / 2;
    };
    int64_t best = cost(most, sums[1] * p.n_kv_heads, p.cost_once);
#pragma unroll
    for (int k = 0; k < kPromptShares; ++k) {
      const int64_t wgs = n[k] * p.n_kv_heads, t = cost(len[k], wgs, p.cost_once + p.cost_split) + p.cost_split;
      if (k < p.n_shares && len[k] < most && t < best && n[k] <= p.max_items) {
        best = t;
        piece = len[k];
      }
    }
  }
  const int keys = piece * 64;

  // ---- the items: counted by classes, then written, each thread's behind those of the threads before it
  int at[kPlanCounts] = {}, total[kPlanCounts] = {};
  auto walk = [&](int s0, bool write) {
    const PagedSeq q = seq_at(s0);
    int x[1] = {blocks_of(q) * paged_pieces(q.len, keys)}, all[1];  // every block's pieces, of the sequence's last row (those that a block does not see are passed over)
    __syncthreads();  // (what is read of front and held is read)
    block_scan(x, all, red);
    front[tid] = x[0];
    held[tid] = q;
    __syncthreads();
    const int n_here = p.n_seqs - s0 < NT ? p.n_seqs - s0 : NT;
    for (int i = tid; i < all[0]; i += NT) {
      int lo = 0, hi = n_here;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (front[mid] <= i)
          lo = mid;
        else
          hi = mid;
      }
      const PagedSeq t = held[lo];
      const int nb = blocks_of(t), n_of = paged_pieces(t.len, keys), j = i - front[lo];
      const int back = (int)((unsigned)j / (unsigned)nb), pc = n_of - 1 - back, b = nb - 1 - (j - back * nb);  // (the blocks of a piece side by side)
      int last = (b + 1) * p.unit_rows;  // (below 2^29)
      last = last < t.n * p.group ? last : t.n * p.group;
      int seen = t.len - t.n + (int)((unsigned)(last - 1) / (unsigned)p.group) + 1;  // keys that the block's last row sees
      seen = seen < 0 ? 0 : seen;
      const int n_pieces = paged_pieces(seen, keys);
      if (pc >= n_pieces) continue;
      const int begin = pc * keys, end = begin + keys < seen ? begin + keys : seen, size = end > begin ? end - begin : 0;
      const int kind = size >= keys ? 0 : kPlanClasses - 1 - (int)((unsigned)((size >> 6) * 4) / (unsigned)piece);
      const bool merge = n_pieces > 1 && pc == 0;
      int to = 0;
#pragma unroll
      for (int c = 0; c < kPlanClasses; ++c)
        if (c == kind) to = at[c]++;
      if (write && to < p.max_items) {
        p.items[to] = PromptItem{s0 + lo, t.first, t.n, t.len, b * p.unit_rows, begin, begin + size, pc | n_pieces << 16};
        if (merge && at[kPlanClasses] < p.max_merges) p.merges[at[kPlanClasses]] = to;
      }
      at[kPlanClasses] += merge;
    }
  };
  if (!once) {  // (all chunks' counts, for where the classes begin)
    for (int s0 = 0; s0 < p.n_seqs; s0 += NT) walk(s0, false);
    block_scan(at, total, red);
  }
  int base[kPlanCounts] = {};
  for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
    int here[kPlanCounts];
#pragma unroll
    for (int c = 0; c < kPlanCounts; ++c) at[c] = 0;
    walk(s0, false);
    block_scan(at, here, red);
    if (once)
#pragma unroll
      for (int c = 0; c < kPlanCounts; ++c) total[c] = here[c];
    int begin = 0;
#pragma unroll
    for (int c = 0; c < kPlanCounts; ++c) {
      at[c] += base[c] + (c < kPlanClasses ? begin : 0);
      begin += total[c];
      base[c] += here[c];
    }
    walk(s0, true);
  }
  if (tid == 0) {
    int count = 0;
#pragma unroll
    for (int c = 0; c < kPlanClasses; ++c) count += total[c];
    p.head[0] = count < p.max_items ? count : p.max_items;
    p.head[1] = total[kPlanClasses] < p.max_merges ? total[kPlanClasses] : p.max_merges;
    p.head[2] = keys;
  }
}

// ---- append ------------------------------------------------------------------------------------------------------------
// 16 bytes a thread and turn, neighbours side by side in a row: bound by memory, every row read and written once.
__global__ void __launch_bounds__(kPlanThreads) pappend_kernel(PAppendParams p, PromptPlanParams plan, int per_row_log2, unsigned per_token, FastDiv by_token) {
  unsigned block = blockIdx.x;
  if (plan.items) {
    if (block == 0) return prompt_plan(plan);
    --block;
  }
  const unsigned i = block * kPlanThreads + threadIdx.x;
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

hipError_t launch_pappend(const PAppendParams& p, const PromptPlanParams& plan, hipStream_t s) {
  const int chunks = p.row_bytes / 16;  // 8, 16 or 32
  int lg = 0;
  while ((1 << lg) < chunks) ++lg;
  const unsigned per_token = (unsigned)(p.n_kv_heads * chunks);
  // (a launch has at most 2^30 threads' worth of 16 bytes, well inside quot()'s range)
  const int64_t most = ((int64_t)1 << 30) / per_token;
  PAppendParams q = p;
  PromptPlanParams with = plan;
  int64_t t = 0;
  do {
    q.k = static_cast<const unsigned char*>(p.k) + t * p.token_bytes;
    q.v = static_cast<const unsigned char*>(p.v) + t * p.token_bytes;
    q.slots = p.slots + t;
    q.n_tokens = (int32_t)(p.n_tokens - t < most ? p.n_tokens - t : most);
    const int64_t threads = (int64_t)q.n_tokens * per_token;
    const int64_t blocks = (threads + kPlanThreads - 1) / kPlanThreads + (with.items ? 1 : 0);
    if (blocks) hipLaunchKernelGGL(pappend_kernel, dim3((unsigned)blocks), dim3(kPlanThreads), 0, s, q, with, lg, per_token, fast_div((int)per_token));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    with.items = nullptr;
    t += most;
  } while (t < p.n_tokens);
  return hipSuccess;
}

}  // namespace kvfold
