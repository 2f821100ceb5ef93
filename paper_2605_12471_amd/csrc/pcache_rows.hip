// The cache in pages: where new tokens go (assign), and rows to their places (append).
#include "pcache.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) unsigned uintx4;

// ---- assign ------------------------------------------------------------------------------------------------------------
// A few thousand numbers: bound by the chain inside one launch.  Every workgroup goes through all requests for itself: for the totals, which say whether
// anything is assigned at all, and for the running sums, from which it takes the tokens that are its share of the places (a long prompt's are shared out like
// any others').  So nobody waits for another workgroup, there is one launch and no memory of its own.  Up to 1024 requests are gone through once, four a thread, more
// of them twice.  A page is written into its table by the thread whose token is the page's first.  64 requests of a token each 3.5 us, 300 with 145220 tokens 6.3 (twice through, four tokens
// a thread one behind the other: 3.8 and 9.3).
constexpr int kAssignThreads = 256, kAssignEach = 4, kAssignChunk = kAssignThreads * kAssignEach;

struct Sums {
  int64_t tokens, pages;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return Sums{a.tokens + b.tokens, a.pages + b.pages}; }

// x and what the lane that CTRL names holds, in the rows (of 16 lanes) of the mask; nothing where there is no such lane
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t plus_lane(int64_t x) {
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, true);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)x >> 32), CTRL, ROWS, 0xf, true);
  return x + (int64_t)((uint64_t)hi << 32 | lo);
}
// The wavefront's running sum, each lane's own value included
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  x = plus_lane<0x111, 0xf>(x);  // lanes 1, 2, 4 and 8 down in the row,
  x = plus_lane<0x112, 0xf>(x);
  x = plus_lane<0x114, 0xf>(x);
  x = plus_lane<0x118, 0xf>(x);
  x = plus_lane<0x142, 0xa>(x);  // a row's last lane to the next row, of two
  return plus_lane<0x143, 0xc>(x);  // and lane 31 to the upper half
}

struct WaveSums {
  Sums sums;
  int flags;
};
// The sum of the block's values in front of the thread's own; *total, *flags: of all
__device__ __forceinline__ Sums scan(const Sums& mine, WaveSums* red, Sums* total, int* flags) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Sums x = {wave_scan(mine.tokens), wave_scan(mine.pages)};
  const int any = (__any(*flags & 2) ? 2 : 0) | (__any(*flags & 8) ? 8 : 0);
  __syncthreads();  // (red may still be read)
  if (l == 63) red[w] = WaveSums{x, any};
  __syncthreads();
  Sums front = {0, 0}, all = {0, 0};
#pragma unroll
  for (int i = 0; i < kAssignThreads / 64; ++i) {
    const WaveSums y = red[i];
    if (i < w) front = front + y.sums;
    all = all + y.sums;
    *flags |= y.flags;
  }
  *total = all;
  return Sums{front.tokens + x.tokens - mine.tokens, front.pages + x.pages - mine.pages};
}

__global__ void __launch_bounds__(kAssignThreads) assign_kernel(AssignParams p) {
  constexpr int NT = kAssignThreads, EACH = kAssignEach, CHUNK = kAssignChunk;
  __shared__ WaveSums red[NT / 64];
  // Of a chunk's requests: what stands in front (below 2^31 where anything is assigned), and the pages and tokens that they hold
  __shared__ int cu[CHUNK], first_page[CHUNK], held[CHUNK], before[CHUNK];
  const int tid = threadIdx.x, lg = p.page_log2, page = 1 << lg;
  const int64_t t0 = p.n_slots * (int64_t)blockIdx.x / gridDim.x, t1 = p.n_slots * (int64_t)(blockIdx.x + 1) / gridDim.x;
  const int free_was = *p.n_free;

  auto pages_of = [&](int64_t n) -> int64_t { return (n + page - 1) >> lg; };
  int len[EACH], more[EACH];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int s = s0 + tid * EACH + i;
      len[i] = s < p.n_seqs ? p.lens[s] : 0;
      more[i] = s < p.n_seqs ? p.n_new[s] : 0;
    }
  };
  auto needs = [&](int i) -> Sums { return Sums{more[i], pages_of((int64_t)len[i] + more[i]) - pages_of(len[i])}; };

  // ---- the totals
  Sums mine = {0, 0}, total;
  int flags = 0;
  for (int s0 = 0; s0 < p.n_seqs; s0 += CHUNK) {
    fetch(s0);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t after = (int64_t)len[i] + more[i];
      if (len[i] < 0 || more[i] < 0) {
        flags |= 8;
        continue;
      }
      if (pages_of(after) > p.table_stride || after > 0x7fffffff) flags |= 2;
      mine = mine + needs(i);
    }
  }
  Sums front = scan(mine, red, &total, &flags);
  const int n_free = free_was < 0 ? 0 : free_was > p.n_pages ? p.n_pages : free_was;
  int status = flags;
  if (total.pages > n_free) status |= 1;
  if (total.tokens > p.n_slots) status |= 4;
  const bool ok = status == 0;
  if (blockIdx.x == 0 && tid == 0) {
    *p.status = status;
    *p.n_free_after = ok ? n_free - (int)total.pages : free_was;
    p.cu_new[0] = 0;
  }

  // ---- the requests in order, a chunk at a time
  int64_t tokens = 0;
  int pages = 0;
  for (int s0 = 0; s0 < p.n_seqs; s0 += CHUNK) {
    const int n_here = p.n_seqs - s0 < CHUNK ? p.n_seqs - s0 : CHUNK;
    if (p.n_seqs > CHUNK) {
      fetch(s0);
      mine = Sums{0, 0};
#pragma unroll
      for (int i = 0; i < EACH; ++i) mine = mine + needs(i);
      front = scan(mine, red, &total, &flags);  // (whose barriers end the chunk before this one)
    }
    int in_front = ok ? (int)(tokens + front.tokens) : 0, pages_in_front = ok ? pages + (int)front.pages : 0;
    const bool writes = blockIdx.x == (unsigned)(s0 / CHUNK) % gridDim.x;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int at = tid * EACH + i, s = s0 + at;
      const Sums own = needs(i);
      cu[at] = in_front;
      first_page[at] = pages_in_front;
      held[at] = (int)pages_of(len[i]);
      before[at] = len[i];
      if (ok) {
        in_front += (int)own.tokens;
        pages_in_front += (int)own.pages;
      }
      if (writes && s < p.n_seqs) {
        p.lens_after[s] = ok ? len[i] + more[i] : len[i];
        p.cu_new[s + 1] = in_front;
      }
    }
    if (!ok) continue;
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
      const int at = before[lo] + ((int)t - cu[lo]), column = at >> lg, lacking = column - held[lo];
      int32_t* row = p.tables + (int64_t)(s0 + lo) * p.table_stride;
      const int32_t* from_where = lacking < 0 ? row + column : p.free_pages + (n_free - 1 - first_page[lo] - lacking);
      const int32_t number = *from_where;
      if (lacking >= 0 && (at & (page - 1)) == 0) row[column] = number;
      p.slots[t] = (int64_t)number * page + (at & (page - 1));
      if (p.positions) p.positions[t] = at;
    }
    tokens += total.tokens;
    pages += (int)total.pages;
  }
  for (int64_t t = (t0 > tokens ? t0 : tokens) + tid; t < t1; t += NT) {
    p.slots[t] = -1;
    if (p.positions) p.positions[t] = -1;
  }
}

hipError_t launch_assign(const AssignParams& p, int n_cu, hipStream_t s) {
  // A token a thread, up to two workgroups a CU: a thread's tokens are looked up one behind the other
  int64_t wgs = (p.n_slots + kAssignThreads - 1) / kAssignThreads;
  wgs = wgs < 1 ? 1 : wgs > 2 * n_cu ? 2 * n_cu : wgs;
  hipLaunchKernelGGL(assign_kernel, dim3((unsigned)wgs), dim3(kAssignThreads), 0, s, p);
  return hipGetLastError();
}

// ---- the list of a batch's work ------------------------------------------------------------------------------------------
// Every sequence's packed rows in blocks, and each block's keys in pieces where that fills the GPU more evenly: it has room for so many workgroups at a time, and
// sequences differ.  With W tiles in all, pieces of a place's share of them, W / places, or an eighth to three more, are compared with none at
// all, by the time of (in tiles at the rate of a full GPU)
//   the longest piece and what a workgroup does once, where all are there at the same time (less where each has a CU for itself); else W and N times what each of N
//   does once over the places, and an eighth of the longest for the last round's gaps (of whole blocks: a half); and for pieces what they cost besides.
// A sequence's blocks are cut at the same keys and stand side by side in the list: they read the same rows at about the same time.  The longest come first (five classes).  One workgroup,
// beside the others that bring the new rows to their places: bound by its chain, 6 us for eight sequences in 364 pieces (with a launch), of which each pass over the sequences, a running
// sum and two barriers, is 1.
constexpr int kPlanThreads = 256;
constexpr int kPlanClasses = 5;
constexpr int kPlanLengths = 4;  // of a piece that are looked at, an eighth of a share apart

struct PlanSums {
  int64_t tiles, blocks;
  int most;
};

__device__ void prompt_plan(const PromptPlanParams& p) {
  constexpr int NT = kPlanThreads, COUNTS = kPlanClasses + 1;  // (the last: blocks that are to be merged)
  __shared__ PlanSums red[NT / 64];
  __shared__ int front[NT];  // of a chunk's sequences: the blocks in front of theirs,
  __shared__ PagedSeq held[NT];  // and themselves
  __shared__ int counts[2][COUNTS];
  __shared__ int64_t lengths[kPlanLengths][NT / 64];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const bool once = p.n_seqs <= NT;  // each thread has one sequence, for good
  if (tid < 2 * COUNTS) counts[0][tid] = 0;
  auto blocks_of = [&](const PagedSeq& q) -> int { return (int)((unsigned)(q.n * p.group + p.unit_rows - 1) / (unsigned)p.unit_rows); };
  // A chunk's sequences into LDS, with what stands in front of them in the chunk; returns the chunk's sums
  auto chunk = [&](int s0) -> PlanSums {
    const int s = s0 + tid;
    PagedSeq q = {0, 0, 0};
    if (s < p.n_seqs) q = paged_seq(p.cu_new ? p.cu_new[s] : s, p.cu_new ? p.cu_new[s + 1] : paged_one(p.slots, p.all_places, s), p.lens[s], p.n_tokens, p.max_new, p.max_len);
    const int nb = blocks_of(q);
    const int keys = q.len - q.n / 2;  // of a block, about
    const int64_t tiles = wave_scan((int64_t)nb * ((keys > 0 ? keys : 0) / 64 + 1)), blocks = wave_scan((int64_t)nb);
    int most = nb ? (q.len + 63) / 64 : 0;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
      const int y = __shfl_xor(most, d);
      most = y > most ? y : most;
    }
    __syncthreads();  // (what is read of LDS is read)
    if (l == 63) red[w] = PlanSums{tiles, blocks, most};
    __syncthreads();
    int64_t before = 0;
    PlanSums all = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      const PlanSums y = red[i];
      if (i < w) before += y.blocks;
      all.tiles += y.tiles;
      all.blocks += y.blocks;
      all.most = y.most > all.most ? y.most : all.most;
    }
    front[tid] = (int)(before + blocks) - nb;
    held[tid] = q;
    __syncthreads();
    return all;
  };

  // ---- all of the work, and whether it is cut
  PlanSums all = chunk(0);
  for (int s0 = NT; s0 < p.n_seqs; s0 += NT) {
    const PlanSums y = chunk(s0);
    all.tiles += y.tiles;
    all.blocks += y.blocks;
    all.most = y.most > all.most ? y.most : all.most;
  }
  if (all.blocks > p.max_merges) {  // sequences that overlap: no work at all, rather than more than there can be
    if (tid < 2) p.head[tid] = 0;
    return;
  }
  const int most = all.most > 1 ? all.most : 1;
  int piece = most;
  if (p.n_pieces > 1) {
    const float work = (float)(all.tiles * p.n_kv_heads), places = (float)p.n_places, alone = (float)p.n_cu;
    auto cost = [&](float longest, float wgs, float each, float gaps) -> float {
      return wgs <= alone ? longest * alone / places + each : wgs <= places ? longest + each : (work + wgs * each) / places + (longest + each) * gaps;
    };
    const int least = (most + p.n_pieces - 1) / p.n_pieces;
    int len[kPlanLengths];
    int64_t pieces[kPlanLengths];
#pragma unroll
    for (int k = 0; k < kPlanLengths; ++k) {
      int x = (int)fminf(ceilf(work * (1.f + 0.125f * (float)k) / places), 1e9f);
      x = x < least ? least : x;
      x = x < p.shortest ? p.shortest : x;
      len[k] = (x + p.step - 1) / p.step * p.step;
      pieces[k] = 0;
    }
    for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
      if (!once) (void)chunk(s0);
      const PagedSeq q = held[tid];
      const int nb = blocks_of(q), sees = (q.len > q.n ? q.len - q.n : 0) + p.unit_rows / p.group, first = ((sees < q.len ? sees : q.len) + 63) / 64, last = (q.len + 63) / 64;
#pragma unroll
      for (int k = 0; k < kPlanLengths; ++k)  // (of the first block and the last, halved below)
        pieces[k] += (int64_t)nb * ((int)((unsigned)(first + len[k] - 1) / (unsigned)len[k]) + (int)((unsigned)(last + len[k] - 1) / (unsigned)len[k]));
    }
    // (each length's sum in a lane of its own from here on)
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPlanLengths; ++k) {
      const int64_t sum = wave_scan(pieces[k]);
      if (l == 63) lengths[k][w] = sum;
    }
    __syncthreads();
    const int k0 = l & (kPlanLengths - 1);
    int64_t wgs = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) wgs += lengths[k0][i];
    wgs = (wgs + 1) / 2;
    int best = len[0];
#pragma unroll
    for (int k = 1; k < kPlanLengths; ++k) best = k == k0 ? len[k] : best;
    float t = cost((float)best, (float)(wgs * p.n_kv_heads), p.cost_once + p.cost_piece, 0.125f) + p.cost_merge;
    if (best >= most || wgs > p.max_items) t = INFINITY;
#pragma unroll
    for (int d = kPlanLengths / 2; d > 0; d /= 2) {
      const float t2 = __shfl_xor(t, d);
      const int best2 = __shfl_xor(best, d);
      if (t2 < t || (t2 == t && best2 > best)) t = t2, best = best2;
    }
    const float whole = cost((float)most, (float)(all.blocks * p.n_kv_heads), p.cost_once, 0.5f);
    if (t < whole) piece = best;
  }

  // ---- the items: counted by classes, then written
  auto items = [&](int n_here, int s0, bool write) {
    const int n_most = (most + piece - 1) / piece;
    for (int i = tid; i < n_here * n_most; i += NT) {  // (below 2^28; the blocks of a piece side by side)
      const int pc = (int)((unsigned)i / (unsigned)n_here), block = i - pc * n_here;
      int lo = 0, hi = p.n_seqs - s0 < NT ? p.n_seqs - s0 : NT;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (front[mid] <= block)
          lo = mid;
        else
          hi = mid;
      }
      const PagedSeq t = held[lo];
      const int b = block - front[lo];
      int last = (b + 1) * p.unit_rows;  // (below 2^29)
      last = last < t.n * p.group ? last : t.n * p.group;
      int seen = t.len - t.n + (int)((unsigned)(last - 1) / (unsigned)p.group) + 1;  // keys that the block's last row sees
      seen = seen < 0 ? 0 : seen;
      const int n = paged_pieces(seen, piece * 64);
      if (pc >= n) continue;
      const int from = pc * piece * 64, to = pc + 1 < n ? from + piece * 64 : seen, size = (to - from) >> 6;
      const int kind = size >= piece ? 0 : kPlanClasses - 1 - (int)((unsigned)(size * 4) / (unsigned)piece);
      const unsigned slot = (unsigned)atomicAdd(&counts[write][kind], 1);
      if (!write || slot >= (unsigned)p.max_items) continue;
      p.items[slot] = PromptItem{s0 + lo, t.first, t.n, t.len, b * p.unit_rows, from, to, pc | n << 16};
      if (n > 1 && pc == 0) {
        const unsigned at = (unsigned)atomicAdd(&counts[1][kPlanClasses], 1);
        if (at < (unsigned)p.max_merges) p.merges[at] = (int)slot;
      }
    }
  };
  int total;
  for (;;) {
    for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
      PlanSums y = all;
      if (!once) y = chunk(s0);
      items((int)y.blocks, s0, false);
    }
    __syncthreads();
    total = 0;
#pragma unroll
    for (int c = 0; c < kPlanClasses; ++c) total += counts[0][c];
    if (piece == most || total <= p.max_items) break;
    piece = most;  // more than the list has room for
    __syncthreads();
    if (tid < COUNTS) counts[0][tid] = 0;
    __syncthreads();
  }
  if (tid < kPlanClasses) {
    int begin = 0;
    for (int c = 0; c < tid; ++c) begin += counts[0][c];
    counts[1][tid] = begin;
  }
  __syncthreads();
  for (int s0 = 0; s0 < p.n_seqs; s0 += NT) {
    PlanSums y = all;
    if (!once) y = chunk(s0);
    items((int)y.blocks, s0, true);
  }
  __syncthreads();
  if (tid == 0) {
    p.head[0] = total < p.max_items ? total : p.max_items;
    p.head[1] = counts[1][kPlanClasses] < p.max_merges ? counts[1][kPlanClasses] : p.max_merges;
  }
}

// ---- append ------------------------------------------------------------------------------------------------------------
// 16 bytes a thread, neighbours side by side in a row: bound by memory, every row read and written once (24K tokens of 8 KV heads, 128 wide: 33 us, 6.0 TB/s).
// A step's rows are stored where they belong to a sequence.  A wavefront, which has few tokens, mostly one, looks among the running sums for 64 at a time, while
// the places are on their way, and each thread among what is left, while its rows are (1500 prompts of 20 to 40 tokens, the whole step: 332 us, as without a look; by a binary
// search from the start 350).
__device__ __forceinline__ void narrow(const int32_t* cu_new, int t_first, int t_last, int l, int& lo, int& hi) {
  for (int step = 0x7fffffff; step > 1 && hi - lo > 1;) {
    const int now = (int)((unsigned)(hi - lo + 63) / 64u);
    if (now >= step) return;  // (tokens of many sequences: no fewer of them)
    step = now;
    const int64_t at = lo + (int64_t)l * step;
    const int32_t sum = at < hi ? cu_new[at] : 0x7fffffff;
    const int a = __builtin_popcountll(__ballot(at < hi && sum <= t_first)), b = __builtin_popcountll(__ballot(at < hi && sum <= t_last));
    const int64_t end = lo + (int64_t)(b < 1 ? 1 : b) * step;
    lo += a < 1 ? 0 : (a - 1) * step;
    hi = end < hi ? (int)end : hi;
    if (hi <= lo) hi = lo + 1;  // (running sums that do not ascend)
  }
}
__global__ void __launch_bounds__(kPlanThreads) pappend_kernel(PAppendParams p, PromptPlanParams plan, int per_row_log2, unsigned per_token, FastDiv by_token) {
  unsigned block = blockIdx.x;
  if (plan.items) {
    if (block == 0) return prompt_plan(plan);
    --block;
  }
  const unsigned i = block * kPlanThreads + threadIdx.x, asked = quot(i, by_token);
  const unsigned t = asked < (unsigned)p.n_tokens ? asked : (unsigned)p.n_tokens - 1;
  const int64_t slot = p.slots[t];
  const int token = p.first + (int)t;
  int seq = p.cu_new ? 0 : token, end = p.cu_new ? p.n_seqs : token + 1;
  if (p.lens && p.cu_new)
    narrow(p.cu_new, __builtin_amdgcn_readfirstlane(token), __builtin_amdgcn_readlane(token, 63), threadIdx.x & 63, seq, end);
  if (asked != t || (uint64_t)slot >= (uint64_t)p.n_places) return;
  const unsigned c = i - t * per_token, g = c >> per_row_log2, at = (c & ((1u << per_row_log2) - 1)) * 16;
  const uint64_t from = (uint64_t)t * (uint64_t)p.token_bytes + (uint64_t)g * (unsigned)p.row_bytes + at;
  const uint64_t row = ((((uint64_t)slot >> p.page_log2) * (unsigned)p.n_kv_heads + g) << p.page_log2) + ((uint64_t)slot & ((1u << p.page_log2) - 1));
  const uint64_t to = row * (unsigned)p.row_bytes + at;
  const uintx4 k = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.k) + from);
  const uintx4 v = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.v) + from);
  if (p.lens && !paged_token(p.cu_new, p.lens, seq, end, p.all_tokens, p.max_new, p.max_len, token)) return;
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
    q.first = (int32_t)t;
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
