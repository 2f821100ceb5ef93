// Attention of whole prompts, and of chunks of them, of many sequences on a cache in pages, bf16.  The new rows are in the pages already.  A work unit is 32
// consecutive packed (token, query head) rows of a sequence and KV head; a wavefront has QB of them, a workgroup four wavefronts and a piece of the keys that
// its rows see.
//
// Bound by the matrix instructions, and by issue beside them.  64 keys' rows of K and V (a tile) come by copies into LDS, a ring of tiles ahead: each wavefront
// brings 16 keys of each, which lie in one page.  S^T = K Q^T and O^T = V^T P^T on the 32x32x16 shapes, swizzles and transpose reads as in attn_bf16.hip, whose
// P never leaves its lane.  Queries are not rounded on the way: the scale is part of the exponent's multiply-add.
#include <type_traits>

#include "meet.h"
#include "prompt.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short short4_;
typedef __attribute__((ext_vector_type(8))) short short8_;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((ext_vector_type(4))) unsigned uintx4;

constexpr int kPromptRing = 3;  // tiles in LDS
template <int D>
constexpr int prompt_lds = kPromptRing * 2 * kTileKeys * D * 2;

__device__ __forceinline__ void prompt_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D, int QB>
__global__ void __launch_bounds__(256, QB == 2 ? 1 : 2) attn_prompt_kernel(PAttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned lds0 = (unsigned)(uintptr_t)((unsigned char __attribute__((address_space(3)))*)smem);
  constexpr int CH = D / 8, ROWB = D * 2, KS = D / 16, DB = D / 32;  // 16-byte chunks and bytes of a row; contraction steps of S^T; tiles of O^T
  constexpr int BN = kTileKeys, TILEB = BN * ROWB;
  constexpr int RPS = 64 / CH, SLABS = 16 / RPS;  // rows of a 1 KiB copy; copies of a wavefront's 16 rows
  constexpr int KSW = CH < 16 ? CH : 16, VSW = CH / 4;
  constexpr int NS = kPromptRing;
  constexpr float kStale = 16.0f;  // log2 units

  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PromptWork wk = prompt_work(p, blockIdx.x, l);
  if (!wk.any) return;
  const int G = p.group, Hq = p.n_q_heads, prev = wk.sq.len - wk.sq.n;

  // ---- the wavefront's rows
  int my_vis[QB], vis_first[QB], vis_last[QB];
  bf16x8 qf[QB][KS];
  const int unit0 = wk.row0 + w * 32 * QB;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int first = unit0 + 32 * qb, r = first + c32, row = r < wk.rows ? r : wk.rows - 1, tok = (int)quot((unsigned)row, p.by_group);
    const int last = first + 31 < wk.rows ? first + 31 : wk.rows - 1;
    my_vis[qb] = prev + tok + 1;
    vis_first[qb] = first < wk.rows ? prev + (int)quot((unsigned)first, p.by_group) + 1 : 0;
    vis_last[qb] = first < wk.rows ? prev + (int)quot((unsigned)last, p.by_group) + 1 : 0;
    const __bf16* qrow = static_cast<const __bf16*>(p.q) + (int64_t)(wk.sq.first + tok) * p.q_stride + (wk.g * G + row - tok * G) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = *reinterpret_cast<const bf16x8*>(qrow + 16 * ks + 8 * h);
  }

  // ---- tiles on their way
  const int32_t* table = p.tables + (int64_t)wk.seq * p.table_stride;
  const int t_begin = wk.key_begin / BN, t_end = (wk.key_end + BN - 1) / BN;
  const uint64_t head = (uint64_t)(unsigned)wk.g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  PageWindow win;      // of tiles [16 n, 16 n + 16): those of the tile asked for last
  unsigned k_off[SLABS], v_off[SLABS];  // the lane's place in 16 rows of a page
  unsigned in_row[SLABS];
#pragma unroll
  for (int i = 0; i < SLABS; ++i) {
    const int r = i * RPS + l / CH;  // (16 w is a multiple of either swizzle)
    in_row[i] = (unsigned)r;
    k_off[i] = (unsigned)(r * ROWB + (((l % CH) ^ (r % KSW)) * 16));
    v_off[i] = (unsigned)(r * ROWB + (((l % CH) ^ ((r & 3) * VSW)) * 16));
  }
  // Whether 64 rows of a tile are all there: then its copies are 2 SLABS a wavefront
  auto whole = [&](int t) __attribute__((always_inline)) -> bool { return t * BN + BN <= wk.sq.len && (win.there >> (4 * (t & 15)) & 15) == 15; };
  auto issue = [&](int t) __attribute__((always_inline)) -> bool {
    if (t >= t_end) return false;
    if ((t & 15) == 0 || t == t_begin) win.fetch(p, table, (t & ~15) * BN, wk.sq.len, l);
    const int at = 4 * (t & 15) + w, key0 = t * BN + 16 * w;
    const int number = __builtin_amdgcn_readlane(win.number, at);
    const bool there = win.there >> at & 1;
    const uint64_t from = (uint64_t)(unsigned)(there ? number : 0) * p.page_bytes + head + (unsigned)((key0 & ((1 << p.page_log2) - 1)) * ROWB);
    const unsigned char *kf = static_cast<const unsigned char*>(p.k_pages) + from, *vf = static_cast<const unsigned char*>(p.v_pages) + from;
    const unsigned slot = lds0 + (unsigned)((t % NS) * 2 * TILEB + 16 * w * ROWB);
    if (__builtin_expect(whole(t), 1)) {
#pragma unroll
      for (int i = 0; i < SLABS; ++i) {
        dma16(kf, k_off[i], slot + i * 1024);
        dma16(vf, v_off[i], slot + TILEB + i * 1024);
      }
      return true;
    }
    // rows that are not there become zeros, so that 0 times them is 0
    const int n = there ? wk.sq.len - key0 : 0;
#pragma unroll 1
    for (int i = 0; i < SLABS; ++i) {
      const unsigned at_lane = slot + (unsigned)(i * 1024 + l * 16);
      unsigned r = 0, ko = 0, vo = 0;
#pragma unroll
      for (int j = 0; j < SLABS; ++j)
        if (j == i) {
          r = in_row[j];
          ko = k_off[j];
          vo = v_off[j];
        }
      if ((int)r < n) {
        dma16(kf, ko, slot + i * 1024);
        dma16(vf, vo, slot + TILEB + i * 1024);
      } else {
        *LDS_PTR(uintx4, at_lane) = uintx4{0u, 0u, 0u, 0u};
        *LDS_PTR(uintx4, at_lane + TILEB) = uintx4{0u, 0u, 0u, 0u};
      }
    }
    return false;
  };

  // ---- LDS read offsets of a lane in a tile
  unsigned kaddr[KS], vaddr[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = lds0 + (unsigned)(c32 * ROWB + (((ks * 2 + h) ^ (c32 % KSW)) * 16));
  {
    const int i16 = l & 15, b2 = (l >> 4) & 1, v_row = 4 * h + (i16 >> 2);
#pragma unroll
    for (int db = 0; db < DB; ++db)
      vaddr[db] = lds0 + (unsigned)(TILEB + v_row * ROWB + (((4 * db + 2 * b2 + ((i16 & 3) >> 1)) ^ ((v_row & 3) * VSW)) * 16) + 8 * (i16 & 1));
  }
  auto v_frag = [&](unsigned slot, int tt, int db) __attribute__((always_inline)) -> short8_ {  // keys 16 tt .. 16 tt + 15, columns 32 db ..
    const short4_ lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, vaddr[db] + slot + (unsigned)(16 * tt * ROWB)));
    const short4_ hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, vaddr[db] + slot + (unsigned)(16 * tt * ROWB + 8 * ROWB)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  floatx16 o[QB][DB];
  float m_run[QB], l_run[QB];
  constexpr floatx16 zero = {};

  // A tile: `careful`, where values that are not finite may stand in rows that some of the unit's rows do not see (0 times them is not 0): each row then
  // takes the 16 keys' values with those that it does not see as zeros.
  auto attend = [&](int t, uint64_t gone, bool careful) __attribute__((always_inline)) {
    const unsigned slot = (unsigned)((t % NS) * 2 * TILEB);
    floatx16 s[QB][2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const bf16x8 k = *LDS_PTR(const bf16x8, kaddr[ks] + slot + (unsigned)(tt * 32 * ROWB));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[qb][tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[qb][ks], ks == 0 ? zero : s[qb][tt], 0, 0, 0);
      }
    const int key0 = t * BN;
    bf16x8 pf[QB][2][2];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (key0 + BN > vis_first[qb] || gone) {  // wave-uniform
        const int rel = my_vis[qb] - key0 - 4 * h;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * tt + 8 * (i >> 2) + (i & 3) >= rel || (gone >> (2 * tt + (i >> 3)) & 1)) s[qb][tt][i] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[qb][tt][i]);
      mx = pair_max(mx) * p.scale_log2e;
      const bool mine = mx > m_run[qb] + kStale || (m_run[qb] == -INFINITY && mx > -INFINITY);
      if (__any(mine)) {
        const float m2 = mine ? mx : m_run[qb];
        const float alpha = m_run[qb] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[qb] - m2);
        m_run[qb] = m2;
        l_run[qb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[qb][db][i] *= alpha;
      }
      const float ref = m_run[qb] == -INFINITY ? 0.f : m_run[qb];
      float sum = 0.f;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qb][tt][i], p.scale_log2e, -ref));
          sum += a;
          pf[qb][tt][i >> 3][i & 7] = (__bf16)a;
        }
      l_run[qb] += sum;
    }
    if (__builtin_expect(!careful, 1)) {
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const short8_ v = v_frag(slot, tt, db);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            o[qb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pf[qb][tt >> 1][tt & 1], o[qb][db], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll 1
        for (int n = 1; n <= 16; ++n) {  // rows that see n of the 16 keys, and the last time those that see them all
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            short8_ v = v_frag(slot, tt, db);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (8 * (e >> 2) + 4 * h + (e & 3) >= n) v[e] = 0;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
              const floatx16 part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pf[qb][tt >> 1][tt & 1], zero, 0, 0, 0);
              const int sees = my_vis[qb] - key0 - 16 * tt;
              if ((sees > 16 ? 16 : sees) == n)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[qb][db][i] += part[i];
            }
          }
        }
    }
  };

#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[qb][ks]));  // (waited for here, not in the loop)
#pragma unroll 1
  for (bool careful = false;; careful = true) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m_run[qb] = -INFINITY;
      l_run[qb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[qb][db] = zero;
    }
    issue(t_begin);
    uint64_t gone = ~win.there >> (4 * (t_begin & 15)) & 15;  // runs of 16 keys of tile t that are in no page
    bool ahead = issue(t_begin + 1);
#pragma unroll 1
    for (int t = t_begin; t < t_end; ++t) {
      const uint64_t gone_next = ~win.there >> (4 * ((t + 1) & 15)) & 15;
      if (ahead)
        wait_vm<2 * SLABS>();
      else
        wait_vm<0>();
      prompt_barrier();  // the tile is there for all, and the slot of the one before is free
      ahead = issue(t + 2);
      bool live = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) live |= t * BN < vis_last[qb];
      if (live) attend(t, gone, careful);
      gone = gone_next;
    }
    // Outputs that are not finite may come from values that their rows do not see: once more, then, with care.
    bool odd = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(__builtin_fabsf(o[qb][db][i]) < INFINITY);
    wait_vm<0>();
    prompt_barrier();
    if (careful) break;
    if (l == 0) *LDS_PTR(int, lds0 + 4 * w) = 0;
    if (__any(odd) && l == 0) *LDS_PTR(int, lds0 + 4 * w) = 1;
    prompt_barrier();
    int again = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) again |= *LDS_PTR(const int, lds0 + 4 * i);
    prompt_barrier();
    if (!__builtin_amdgcn_readfirstlane(again)) break;
  }

  // ---- out, or what the piece leaves for the merge
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float l_tot = pair_sum(l_run[qb]);
    const int r = unit0 + 32 * qb + c32;
    if (r >= wk.rows) continue;
    const int t = (int)quot((unsigned)r, p.by_group), head_q = wk.g * G + r - t * G;
    const int64_t at = (int64_t)(wk.sq.first + t) * Hq + head_q;
    if (wk.n_pieces == 1) {
      const float inv = 1.f / l_tot;
      __bf16* out = static_cast<__bf16*>(p.out) + at * D + 4 * h;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (__bf16)(l_tot == 0.f ? 0.f : o[qb][db][i + e] * inv);
          *reinterpret_cast<bf16x4*>(out + 32 * db + 2 * i) = v;
        }
      if (p.lse && h == 0)
        p.lse[(int64_t)head_q * p.n_tokens + wk.sq.first + t] = l_tot == 0.f ? -INFINITY : (m_run[qb] + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
    } else {
      const int64_t part = (int64_t)wk.piece * p.n_tokens * Hq + at;
      float* out = p.part_o + part * D + 4 * h;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<floatx4*>(out + 32 * db + 2 * i) = floatx4{o[qb][db][i], o[qb][db][i + 1], o[qb][db][i + 2], o[qb][db][i + 3]};
      if (h == 0) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{m_run[qb], l_tot};
    }
  }
}

template <int D, int QB>
static hipError_t prepare_one() {
  static bool done[64] = {};  // (idempotent; two threads at worst set it twice)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!done[dev]) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_prompt_kernel<D, QB>), hipFuncAttributeMaxDynamicSharedMemorySize, prompt_lds<D>);
    if (e != hipSuccess) return e;
    done[dev] = true;
  }
  return hipSuccess;
}
template <int D, int QB>
static hipError_t launch_one(const PAttnParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.n_units * (unsigned)p.n_pieces * (unsigned)p.n_kv_heads), block(256);
  hipLaunchKernelGGL((attn_prompt_kernel<D, QB>), grid, block, prompt_lds<D>, s, p);
  return hipGetLastError();
}

hipError_t prepare_attn_prompt(int head_dim, bool bf16) {
  if (!bf16) return prepare_attn_prompt_f32(head_dim);
  return head_dim == 128 ? prepare_one<128, 1>() : prepare_one<64, 1>();
}
hipError_t launch_attn_prompt(const PAttnParams& p, int head_dim, bool bf16, int units_per_wave, hipStream_t s) {
  if (!bf16) return launch_attn_prompt_f32(p, head_dim, s);
  (void)units_per_wave;
  return head_dim == 128 ? launch_one<128, 1>(p, s) : launch_one<64, 1>(p, s);
}

// ---- the merge of pieces ---------------------------------------------------------------------------------------------------
// A thread has 16 bytes of a row and goes through its pieces, eight in flight; rows of one piece have been written.  Bound by memory.
template <class T, int D>
__global__ void __launch_bounds__(256) pmerge_kernel(PAttnParams p, int parts_log2) {
  constexpr int V = D / 4, ROWS = 256 / V;  // (rows of a workgroup: unit_rows / ROWS = 2^parts_log2 of them share a block's)
  const PromptWork wk = prompt_work(p, blockIdx.x >> parts_log2, threadIdx.x & 63);
  const int c = threadIdx.x % V, r = wk.row0 + (int)(blockIdx.x & ((1u << parts_log2) - 1)) * ROWS + threadIdx.x / V, n = wk.n_pieces;
  if (!wk.any || n < 2 || r >= wk.rows) return;
  const int tok = (int)quot((unsigned)r, p.by_group), head = wk.g * p.group + r - tok * p.group;
  const int64_t n_rows = (int64_t)p.n_tokens * p.n_q_heads, token = wk.sq.first + tok, at = token * p.n_q_heads + head;
  float M = -INFINITY, L = 0.f;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int N = 8;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += N) {
    floatx2 ml[N];
    floatx4 o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t part = (int64_t)(i0 + i < n ? i0 + i : n - 1) * n_rows + at;
      ml[i] = *reinterpret_cast<const floatx2*>(p.part_ml + part * 2);
      o[i] = *reinterpret_cast<const floatx4*>(p.part_o + part * D + c * 4);
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i0 + i >= n || ml[i].y == 0.f) {  // no key for the row in this piece
        ml[i] = floatx2{-INFINITY, 0.f};
        o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      top = fmaxf(top, ml[i].x);
    }
    const float ref = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(M - ref);
    M = top;
    L *= f0;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float f = __builtin_amdgcn_exp2f(ml[i].x - ref);
      L = __builtin_fmaf(ml[i].y, f, L);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(o[i][e], f, acc[e]);
    }
  }
  const float inv = 1.f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = L == 0.f ? 0.f : acc[e] * inv;
  if constexpr (sizeof(T) == 2) {
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)acc[e];
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + at * D + c * 4) = v;
  } else {
    *reinterpret_cast<floatx4*>(static_cast<float*>(p.out) + at * D + c * 4) = acc;
  }
  if (p.lse && c == 0) p.lse[(int64_t)head * p.n_tokens + token] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

hipError_t launch_pmerge(const PAttnParams& p, int head_dim, bool bf16, hipStream_t s) {
  int lg = 0;
  while ((256 / (head_dim / 4)) << lg < p.unit_rows) ++lg;
  const dim3 grid(((unsigned)p.n_units * (unsigned)p.n_kv_heads) << lg), block(256);
  if (bf16 && head_dim == 128)
    hipLaunchKernelGGL((pmerge_kernel<__bf16, 128>), grid, block, 0, s, p, lg);
  else if (bf16)
    hipLaunchKernelGGL((pmerge_kernel<__bf16, 64>), grid, block, 0, s, p, lg);
  else if (head_dim == 128)
    hipLaunchKernelGGL((pmerge_kernel<float, 128>), grid, block, 0, s, p, lg);
  else
    hipLaunchKernelGGL((pmerge_kernel<float, 64>), grid, block, 0, s, p, lg);
  return hipGetLastError();
}

}  // namespace kvfold
