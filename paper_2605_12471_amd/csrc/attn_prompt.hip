// Attention of whole prompts, and of chunks of them, of many sequences on a cache in pages, bf16.  The new rows are in the pages already.  A work unit is 32
// consecutive packed (token, query head) rows of a sequence and KV head; a wavefront has QB of them, a workgroup four wavefronts and a piece of the keys that
// its rows see.
//
// Bound by the matrix instructions under the power cap, and by issue beside them: one prompt of 16K tokens, 32 heads on 8, 128 wide 1.75 ms, 1.26 PFLOP/s, matrix pipes 0.61 busy.  Tiles, rings, swizzles and the software pipeline are those of attn_bf16.hip (two
// units a wavefront: every fragment read from LDS feeds two matrix instructions, and no row maximum is taken below the causal horizon).  What differs:
//  * A tile's 64 rows come from the pages: a wavefront brings 16 keys of K and of V, which lie in one (page_tokens is a multiple of 16).  Its number is a scalar
//    load half a tile ahead of the copies, and V's copies of a tile go to the place where K's went a step before.
//  * Queries are not rounded on the way: S^T is formed from them as they are, starts from -m in its own units, and a weight is 2^(S scale log2 e), a
//    multiplication more a logit.
//  * Rows that do not exist (of pages that are none, behind the sequence's end) become zeros in LDS, so that 0 times them is 0; their tiles are masked.
//  * Outputs that are not finite may come from values that their rows do not see (0 times them is not 0): the workgroup then does its work once more, slowly, each
//    row with the values that it does not see as zeros.
#include <type_traits>

#include "prompt.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short short4_;
typedef __attribute__((ext_vector_type(8))) short short8_;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) unsigned uintx4;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

// Wait until at most N LDS reads are outstanding (compiler-visible, so that it adds none of its own
// for fragments covered by this wait).  gfx9 encoding: vmcnt and expcnt left at their maxima.
template <int N>
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_s_waitcnt(0xC07F | (N << 8));
}

// MFMA issued by hand so that the register files are under control: S^T accumulates in VGPRs (the vector ALU reads it next), O^T in AGPRs, and the Q fragments (B
// operands) and the K fragments (A operands, loaded from LDS straight into AGPRs) sit in AGPRs too.  The compiler does not see these as matrix instructions, so the
// distances the hardware needs, ahead of them and behind them (mfma_settle_*()), are kept by construction.
__device__ __forceinline__ void mfma_qk_first(floatx16& s, const bf16x8& a, const bf16x8& q, const floatx16& c0) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %3" : "=&v"(s) : "a"(a), "a"(q), "v"(c0));
}
__device__ __forceinline__ void mfma_qk(floatx16& s, const bf16x8& a, const bf16x8& q) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "a"(a), "a"(q));
}
__device__ __forceinline__ void mfma_pv(floatx16& o, const bf16x8& a, const bf16x8& pfrag) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(a), "v"(pfrag));
}
// 48 idle issue cycles tied to a register tuple: everything that reads or writes `x` afterwards
// is ordered behind a finished matrix pipe (an 8-pass MFMA result is readable 19 cycles after issue).
__device__ __forceinline__ void mfma_settle_v(floatx16& x) {
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" : "+v"(x));
}
__device__ __forceinline__ void mfma_settle_a(floatx16& x) {
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" : "+a"(x));
}
constexpr float kRescaleThreshold = 16.0f;                // log2 units: stale running max tolerated up to 2^16
constexpr float kSumThreshold = 1048576.0f;               // 2^20: row sum of a half that moves the reference up
constexpr float kRedoThreshold = 1152921504606846976.0f;  // 2^60: beyond this the workgroup starts over

// Slot schedule of one pipeline step of a wavefront with QA active units (QA = QB in the ordinary
// step; QA = 1 in a two-unit wavefront whose first unit has passed its causal horizon).  A step
// handles one 32-key half hh and consists of M MFMA slots: M1 slots forming S^T of half hh+1 (phase
// 1), then M2 slots accumulating O^T += V^T P^T of half hh (phase 2).  A single wavefront hides only
// about 16-20 cycles of other instructions under one 32-cycle MFMA (an exp2 costs 8, plain vector
// instructions 4), so everything else is dealt out evenly, a fixed share behind every MFMA:
//   * exp2 / pack / row-sum "events" of half hh (one event = one exp2; the second event of a logit
//     pair also packs the pair, and each event adds the exp2 before it to the row sum): events
//     [NEAR, NE) in slots [0, EW) of the half's own step, so that slab 0 of P is packed before phase
//     2 and slab 1 before its second half; the first NEAR events (all in slab 0) are
//     taken EARLY, in the tail slots [EW, M) of the step before, as soon as that S^T is complete;
//   * LDS fragment reads one batch ahead, in slots [0, RW), RW half way into the tail, one wait per batch;
//   * the test of the row sums against 2^20 right after the last event (no row maximum is taken below the causal horizon);
//   * in odd steps the workgroup barrier and the ring refill (DMA) in the tail [EW, M).
template <int D, int QA, int LPG>
struct PromptSched {
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int M1 = KS * QA;       // MFMAs of phase 1 (K fragment ks feeds QA of them)
  static constexpr int M2 = 2 * DB * QA;   // MFMAs of phase 2 (V^T fragment (tt, db) feeds QA of them)
  static constexpr int M = M1 + M2;
  static constexpr int NP = QA * 8;        // logit pairs per step; pair k: slab k / (4 QA), unit (k / 4) % QA
  static constexpr int NE = 2 * NP;        // exp events
  static constexpr int EW = M1 + M2 / 2;
  static constexpr int NEAR = (NE * (M - EW) / M) & ~1;
  static constexpr int NMAIN = NE - NEAR;
  static_assert(NEAR <= NE / 2, "early events must stay inside slab 0");
  static_assert(NEAR + (M1 * NMAIN + EW - 1) / EW >= NE / 2, "slab 0 would not be complete at the start of phase 2");
  static constexpr int GK = KS / 2;        // K fragments per batch (two batches per step)
  static constexpr int GV = DB;            // V^T fragments per batch (two batches per step, 2 reads each)
  static constexpr int R = 2 * GK + 4 * GV;  // LDS read instructions per step, in issue order:
                                             //   kg[1] (GK) | vg[0] (2 GV) | vg[1] (2 GV) | kg[0] of the next step (GK)
  static constexpr int RW = EW + (M - EW) / 2;  // (measured: spreading the reads a little into the tail beats stopping at EW)
  static_assert(EW + 1 < M, "no slot for the row-sum test");
  static_assert(LPG <= (M - EW) * 4, "ring refill does not fit the tail");
  // read r is issued in slot r * RW / R; reads issued before slot sl:
  static constexpr int rd_before(int sl) {
    int n = 0;
    for (int r = 0; r < R; ++r) n += (r * RW / R) < sl;
    return n;
  }
};

// Place of packed row r of the work's sequence and KV head among the batch's [token][query head] rows
__device__ __forceinline__ unsigned prompt_place(const PAttnParams& p, const PromptWork& wk, int r) {
  const int tok = (int)quot((unsigned)r, p.by_group);
  return (unsigned)(wk.sq.first + tok) * (unsigned)p.n_q_heads + (unsigned)(wk.g * p.group + r - tok * p.group);
}
// A row's log-sum-exp, or what its piece leaves for the merge; m in log2 units
__device__ __forceinline__ void prompt_sums(const PAttnParams& p, const PromptWork& wk, unsigned place, float m, float l_tot) {
  const unsigned Hq = (unsigned)p.n_q_heads, token = place / Hq;
  if (wk.n_pieces > 1)
    *reinterpret_cast<floatx2*>(p.part_ml + ((int64_t)wk.piece * p.n_tokens * Hq + place) * 2) = floatx2{m, l_tot};
  else if (p.lse)
    p.lse[(int64_t)(place - token * Hq) * p.n_tokens + token] = l_tot == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
}

// Where a wavefront of the workgroup has outputs that are not finite (`odd`), which may come from values that their rows do not see: everything once more, 64 keys and
// 32 columns of a unit at a time, each row with the values that it does not see as zeros.  For all four wavefronts, behind their last use of LDS.
template <int D, int QB>
__device__ __forceinline__ void prompt_again(const PAttnParams& p, const PromptWork& wk, unsigned lds0, int w, bool odd) {
  constexpr int CH = D / 8, ROWB = D * 2, KS = D / 16, DB = D / 32, BN = kTileKeys, TILEB = BN * ROWB;
  constexpr int RPS = 64 / CH, SLABS = 16 / RPS, KSW = CH < 16 ? CH : 16, VSW = CH / 4;
  constexpr floatx16 zero = {};
  __syncthreads();
  const int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), hi = l >> 5, m = l & 31;
  const int vote = __any(odd) ? 1 : 0;
  if (l == 0) *LDS_PTR(int, lds0 + 4u * (unsigned)w) = vote;
  __syncthreads();
  int again = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) again |= *LDS_PTR(const int, lds0 + 4u * (unsigned)i);
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(again) == 0, 1)) return;
  __syncthreads();
  const int32_t* table = p.tables + (int64_t)wk.seq * p.table_stride;
  const int len = wk.sq.len, prev = len - wk.sq.n;
  const uint64_t head = (uint64_t)(unsigned)wk.g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  const bool alone = wk.n_pieces == 1;
  auto none = [&](int key) __attribute__((always_inline)) -> bool { return key >= len || (unsigned)table[(unsigned)key >> p.page_log2] >= (unsigned)p.n_pages; };
#pragma unroll 1
  for (int pass = 0; pass < QB * DB; ++pass) {
    const int db = pass % DB, row = wk.row0 + (w * QB + pass / DB) * 32 + m, row_q = row < wk.rows ? row : wk.rows - 1;
    const int tok = (int)quot((unsigned)row_q, p.by_group), vis = prev + tok + 1;
    const __bf16* qrow = static_cast<const __bf16*>(p.q) + (int64_t)(wk.sq.first + tok) * p.q_stride + (wk.g * p.group + row_q - tok * p.group) * D + 8 * hi;
    floatx16 acc = zero;
    float top = -INFINITY, sum = 0.f;
#pragma unroll 1
    for (int key0 = wk.key_begin; key0 < wk.key_end; key0 += BN) {
#pragma unroll 1
      for (int i = 0; i < SLABS; ++i) {  // K, then V, with zeros where there is no row
        const int r = 16 * w + i * RPS + l / CH, key = key0 + r, c = l % CH;
        uintx4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
        if (!none(key)) {
          const uint64_t from = (uint64_t)(unsigned)table[(unsigned)key >> p.page_log2] * p.page_bytes + head + ((unsigned)key & ((1u << p.page_log2) - 1)) * (unsigned)ROWB + (unsigned)(c * 16);
          k = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.k_pages) + from);
          v = *reinterpret_cast<const uintx4*>(static_cast<const unsigned char*>(p.v_pages) + from);
        }
        *LDS_PTR(uintx4, lds0 + (unsigned)(r * ROWB + ((c ^ (r % KSW)) * 16))) = k;
        *LDS_PTR(uintx4, lds0 + (unsigned)(TILEB + r * ROWB + ((c ^ ((r & 3) * VSW)) * 16))) = v;
      }
      __syncthreads();
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        floatx16 s = zero;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 k = *LDS_PTR(const bf16x8, lds0 + (unsigned)((32 * half + m) * ROWB + (((ks * 2 + hi) ^ (m % KSW)) * 16)));
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, *reinterpret_cast<const bf16x8*>(qrow + 16 * ks), s, 0, 0, 0);
        }
        const int first = key0 + 32 * half;
        const bool gone[2] = {none(first), none(first + 16)};
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (8 * (r >> 2) + 4 * hi + (r & 3) >= vis - first || gone[r >> 3]) s[r] = -INFINITY;
          mx = fmaxf(mx, s[r]);
        }
        mx = pair_max(mx) * p.scale_log2e;
        if (mx > top) {
          const float alpha = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - mx);
          top = mx;
          sum *= alpha;
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[r] *= alpha;
        }
        const float ref = top == -INFINITY ? 0.f : top;
        bf16x8 pf[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2e, -ref));
          sum += a;
          pf[r >> 3][r & 7] = (__bf16)a;
        }
        const int i16 = l & 15, b2 = (l >> 4) & 1, v_row = 4 * hi + (i16 >> 2);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const unsigned at = lds0 + (unsigned)(TILEB + (32 * half + 16 * tt + v_row) * ROWB + (((4 * db + 2 * b2 + ((i16 & 3) >> 1)) ^ ((v_row & 3) * VSW)) * 16) + 8 * (i16 & 1));
          const short4_ lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, at)), up = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, at + 8 * ROWB));
          const int sees = vis - first - 16 * tt;
#pragma unroll 1
          for (int n = __all(sees >= 16) ? 16 : 1; n <= 16; ++n) {  // rows that see n of these 16 keys, at last those that see them all
            short8_ v = __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (8 * (e >> 2) + 4 * hi + (e & 3) >= n) v[e] = 0;
            const floatx16 part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pf[tt], zero, 0, 0, 0);
            if ((sees > 16 ? 16 : sees) == n)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[r] += part[r];
          }
        }
      }
      __syncthreads();
    }
    const float l_tot = pair_sum(sum);
    if (row < wk.rows) {
      const unsigned place = prompt_place(p, wk, row);
      if (hi == 0 && db == 0) prompt_sums(p, wk, place, top, l_tot);
      const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int c = 32 * db + 2 * r + 4 * hi;
        if (alone) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[r + e] * inv);
          *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + (int64_t)place * D + c) = v;
        } else {
          *reinterpret_cast<floatx4*>(p.part_o + ((int64_t)wk.piece * p.n_tokens * p.n_q_heads + place) * D + c) = floatx4{acc[r], acc[r + 1], acc[r + 2], acc[r + 3]};
        }
      }
    }
  }
}

constexpr int kPromptRing = 3;  // V slots; K has one more
template <int D>
constexpr int prompt_lds = (2 * kPromptRing + 1) * kTileKeys * D * 2;

template <int D>
__global__ void __launch_bounds__(256, 1) attn_prompt_kernel(PAttnParams p) {
  constexpr int QB = 2, NV = kPromptRing;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned lds0 = (unsigned)(uintptr_t)((unsigned char __attribute__((address_space(3)))*)smem);
  constexpr int NK = NV + 1;         // K ring slots (K runs half a tile ahead of V in the pipeline)
  constexpr int CH = D / 8;          // 16-byte chunks per row
  constexpr int ROWB = D * 2;        // bytes per row
  constexpr int BN = kTileKeys;      // 64
  constexpr int KS = D / 16;         // contraction steps of S^T = K Q^T
  constexpr int DB = D / 32;         // 32-wide blocks of the head dim in O^T
  constexpr int TILEB = BN * ROWB;   // bytes of one K (or V) tile
  constexpr int HALFB = 32 * ROWB;   // bytes of a 32-key half tile
  constexpr int RPS = 64 / CH;       // rows covered by one 1 KiB copy
  constexpr int SLABS = 16 / RPS;    // copies of a wavefront's 16 rows of a tile, K or V
  constexpr int LPG = 2 * SLABS;     // copies per wavefront per tile
  constexpr int KSW = CH < 16 ? CH : 16;  // K swizzle: chunk ^= row % KSW
  constexpr int VSW = CH / 4;             // V swizzle: chunk ^= (row & 3) * VSW

  const int tid = threadIdx.x, l = tid & 63, hi = l >> 5, m = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PromptWork wk = prompt_work(p, blockIdx.x);
  if (!wk.any) return;
  // The lane, found again where it is rarely needed, not held through the main loop
  auto lane_now = []() __attribute__((always_inline)) -> int {
    int x = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(x));
    return x;
  };
  const int g = wk.g, G = p.group, Hq = p.n_q_heads, len = wk.sq.len, prev = wk.sq.len - wk.sq.n;
  const float to_log2 = p.scale_log2e, from_log2 = p.from_log2, stale = p.stale;

  // ---- my units
  const int n_units = (wk.rows + 31) / 32, unit0 = wk.row0 / 32 + w * QB;
  unsigned q_at[QB];    // of this lane's row (the last one where the unit runs past it), in eighths of a row's elements from the batch's first
  int vis_first[QB];    // keys visible to the unit's first row (key blocks entirely below need no mask)
  int vis_last0 = 0;    // keys visible to the last row of unit 0: tiles entirely beyond are dead for it
  auto row_at = [&](int row) __attribute__((always_inline)) -> unsigned {
    const int tok = (int)quot((unsigned)row, p.by_group);
    return (unsigned)(wk.sq.first + tok) * (unsigned)(p.q_stride >> 3) + (unsigned)((g * G + row - tok * G) * (D / 8));
  };
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int u = unit0 + qb < n_units ? unit0 + qb : n_units - 1, last = 32 * u + 31 < wk.rows ? 32 * u + 31 : wk.rows - 1;
    const int row = 32 * u + m < wk.rows ? 32 * u + m : wk.rows - 1;
    q_at[qb] = row_at(row);
    vis_first[qb] = prev + (int)quot((unsigned)(32 * u), p.by_group) + 1;
    if (qb == 0) vis_last0 = prev + (int)quot((unsigned)last, p.by_group) + 1;
  }
  const bool idle = unit0 >= n_units;  // (then the second unit does not exist either)
  const int vis_min = vis_first[0];

  // ---- the piece's tiles
  const int t_begin = wk.key_begin / BN, t_end = (wk.key_end + BN - 1) / BN, t_last = t_end - 1;
  const ConstPtr<int32_t> table = (ConstPtr<int32_t>)(uintptr_t)(p.tables + (int64_t)wk.seq * p.table_stride);
  const uint64_t head = (uint64_t)(unsigned)g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  const unsigned in_page = (1u << p.page_log2) - 1;

  // ---- the Q rows, through LDS like the tiles: the K slots from the third on, then the V slots from the second on
  constexpr int QAREA = QB * HALFB;
  static_assert(4 * QAREA <= (NK - 2 + NV - 1) * TILEB && (NK - 2) * TILEB % QAREA == 0, "Q does not fit the free slots");
  const unsigned q_lds = lds0 + (unsigned)(2 * TILEB + w * QAREA) + (w * QAREA >= (NK - 2) * TILEB ? (unsigned)TILEB : 0u);
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    unsigned place[32 / RPS];  // of the rows that the lane fetches from: held by the lanes whose rows they are
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) place[i] = (unsigned)__builtin_amdgcn_ds_bpermute(4 * (i * RPS + l / CH), (int)q_at[qb]);
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) {
      const unsigned char* qrow = static_cast<const unsigned char*>(p.q) + (uint64_t)place[i] * 16 + (unsigned)(((l % CH) ^ ((i * RPS + l / CH) % KSW)) * 16);
      dma16_at(qrow, q_lds + (unsigned)(qb * HALFB + i * 1024));
    }
  }

  // ---- the first tile with keys of a page that is none: each wavefront looks through the piece's part of the table, 64 pages at a time
  int t_bad = 0x7fffffff;
  if (t_begin < t_end) {
    const int last = ((t_end * BN < len ? t_end * BN : len) - 1) >> p.page_log2;  // (tiles are brought whole, also the piece's last one)
#pragma unroll 1
    for (int i = wk.key_begin >> p.page_log2; i <= last; i += 64) {
      const int32_t number = i + l <= last ? p.tables[(int64_t)wk.seq * p.table_stride + i + l] : 0;
      const uint64_t bad = __ballot((unsigned)number >= (unsigned)p.n_pages);
      if (bad && t_bad == 0x7fffffff) t_bad = ((i + __builtin_ctzll(bad)) << p.page_log2) / BN;
    }
    if (t_bad < t_begin) t_bad = t_begin;
  }
  const int t_whole = len / BN < t_bad ? len / BN : t_bad;  // tiles before it have 64 rows

  // ---- tiles on their way: a wavefront's 16 rows of K and of V, lane l at chunk l % CH of row i RPS + l / CH of copy i, which the swizzle maps elsewhere
  // (the swizzle of row i RPS + r is that of row r and that of row i RPS, which have no bit in common)
  const unsigned dma_k = (unsigned)((l / CH) * ROWB + (((l % CH) ^ (l / CH)) * 16));
  auto k_off = [&](int i) __attribute__((always_inline)) -> unsigned { return dma_k ^ (unsigned)(i * RPS % KSW * 16); };
  const unsigned dma_v = (unsigned)((l / CH) * ROWB + (((l % CH) ^ ((l / CH & 3) * VSW)) * 16));
  auto place_of = [&](unsigned number, int key0) __attribute__((always_inline)) -> uint64_t {
    return (uint64_t)number * p.page_bytes + head + ((unsigned)key0 & in_page) * (unsigned)ROWB;
  };
  // The main loop's copies: K of a tile NV + 1 ahead, V of the one before it.  The ring knows no end: past the piece its last tile is fetched again (an L2
  // hit), so that pieces below the causal horizon never leave the main loop.
  uint64_t k_from = 0, v_from = 0;
  int32_t number_next = 0;
  int key_next = 0;
  auto ask_page = [&](int t) __attribute__((always_inline)) {
    key_next = (t < t_last ? t : t_last) * BN + 16 * w;
    number_next = table[(unsigned)key_next >> p.page_log2];
  };
  auto from_page = [&]() __attribute__((always_inline)) -> uint64_t { return place_of((unsigned)number_next, key_next); };
  auto issue_slab = [&](bool is_v, uint64_t from, int slot, int i) __attribute__((always_inline)) {
    const unsigned lds = lds0 + (unsigned)(((is_v ? NK : 0) + slot) * TILEB + (w * SLABS + i) * 1024);
    dma16(static_cast<const unsigned char*>(is_v ? p.v_pages : p.k_pages) + from + i * 1024, is_v ? dma_v : k_off(i), lds);
  };
  // A whole tile outside the slot schedule; nothing past the piece.  Where rows do not exist zeros are written in their stead.
  auto issue_tile = [&](bool is_v, int t, int slot) __attribute__((always_inline)) {
    if (t >= t_end) return;
    const int key0 = t * BN + 16 * w;
    const unsigned lds = lds0 + (unsigned)(((is_v ? NK : 0) + slot) * TILEB + w * SLABS * 1024);
    const unsigned char* pages = static_cast<const unsigned char*>(is_v ? p.v_pages : p.k_pages);
    if (__builtin_expect(t < t_whole, 1)) {
      const unsigned char* base = pages + place_of((unsigned)table[(unsigned)key0 >> p.page_log2], key0);
#pragma unroll
      for (int i = 0; i < SLABS; ++i) dma16(base + i * 1024, is_v ? dma_v : k_off(i), lds + i * 1024);
    } else {
      int n = len - key0;
      unsigned number = 0;
      if (n > 0) number = (unsigned)table[(unsigned)key0 >> p.page_log2];
      if (number >= (unsigned)p.n_pages) n = 0;
      const unsigned char* base = pages + place_of(n > 0 ? number : 0, key0);
      const int l2 = lane_now();
#pragma unroll 1
      for (int i = 0; i < SLABS; ++i) {
        const int r = i * RPS + l2 / CH;
        const unsigned off = (unsigned)((l2 / CH) * ROWB + (((l2 % CH) ^ (is_v ? (r & 3) * VSW : r % KSW)) * 16));
        if (r < n)
          dma16(base + i * 1024, off, lds + i * 1024);
        else
          *LDS_PTR(uintx4, lds + (unsigned)(i * 1024 + l2 * 16)) = uintx4{0u, 0u, 0u, 0u};
      }
    }
  };
  auto prefill = [&](int j0, int j1) __attribute__((always_inline)) {
    // Steady state at the top of the even step of tile t: K[t], K[t+1], V[t] are in LDS and visible, the
    // groups {K[t+1+j], V[t+j]}, j = 1 .. NV-1, are in flight.  Tile t_begin + j takes ring slot j.
#pragma unroll 1
    for (int j = j0; j <= j1; ++j) {
      issue_tile(false, t_begin + j, j);
      if (j > 0) issue_tile(true, t_begin + j - 1, j - 1);
    }
  };
  wait_vm<0>();  // (Q: in front of the table, which has been waited for)
  prefill(0, 1);
  bf16x8 qf[QB][KS];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[qb][ks] = *LDS_PTR(const bf16x8, q_lds + (unsigned)(qb * HALFB + m * ROWB + (((ks * 2 + hi) ^ (m % KSW)) * 16)));
      asm volatile("" : "+a"(qf[qb][ks]));  // park the fragment in the AGPR file, where the MFMAs read it
    }
  wait_lds<0>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();  // every wavefront has its Q out of the slots that are filled now
  asm volatile("" ::: "memory");
  prefill(2, NV);

  // ---- LDS read offsets (per lane) of the tile currently being read, ring slot included; moved from slot to slot once per tile
  int kslot, vslot;  // ring slots of tile t (wave-uniform)
  unsigned kaddr[KS];
  unsigned vaddr[DB];

  // ---- running state, in S^T's own units (before the scale)
  floatx16 o[QB][DB];   // O^T accumulators (AGPRs)
  floatx16 negm[QB];    // -m (0 while no key has been seen) in every element: start value of S^T
  float m_run[QB], l_run[QB];
  int overflowed = 0;   // wave-uniform: a row sum left the range the sum-driven rescale can repair
  auto reset_state = [&]() __attribute__((always_inline)) {
    kslot = 0;
    vslot = 0;
    const int l2 = lane_now();  // (nothing computed here is kept in registers across the main loop for the sake of a restart that almost never happens)
    const int hi2 = l2 >> 5, m2 = l2 & 31;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      kaddr[ks] = lds0 + (unsigned)(m2 * ROWB + (((ks * 2 + hi2) ^ (m2 % KSW)) * 16)) + (unsigned)(kslot * TILEB);
    // V^T fragment via transpose read: lane i of a 16-lane block supplies row (i/4) of a 4-row group and 4 columns
    const int i16 = l2 & 15, b2 = (l2 >> 4) & 1;
    const int v_row = 4 * hi2 + (i16 >> 2);  // + 16*tt (+8)
#pragma unroll
    for (int db = 0; db < DB; ++db)
      vaddr[db] = lds0 + (unsigned)(v_row * ROWB + (((4 * db + 2 * b2 + ((i16 & 3) >> 1)) ^ ((v_row & 3) * VSW)) * 16) + 8 * (i16 & 1)) +
                  (unsigned)((NK + vslot) * TILEB);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m_run[qb] = -INFINITY;
      l_run[qb] = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) negm[qb][r] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[qb][db][r] = 0.f;
    }
  };

  // ---- building blocks of the software pipeline --------------------------------------------
  // K fragment ks of the current K tile (imm = 0) or of its second half (imm = HALFB), read from LDS
  // straight into AGPRs.  The compiler does not see an LDS access here: every use is covered by one
  // of the wait_lds<>() calls of the pipeline.
  auto k_frag = [&](int ks, int imm) __attribute__((always_inline)) -> bf16x8 {
    bf16x8 f;
    if (imm == 0)
      asm volatile("ds_read_b128 %0, %1" : "=a"(f) : "v"(kaddr[ks]));
    else
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=a"(f) : "v"(kaddr[ks]), "n"(HALFB));
    return f;
  };
  // The mask of the 32-key half hh: the causal one, and keys of pages that are none.
  auto mask_half = [&](floatx16 (&s)[QB], int hh, int q0 = 0) __attribute__((always_inline)) {
    const int l2 = lane_now(), hi_here = l2 >> 5;
    const int key0 = hh * 32;
    unsigned gone = 0;  // of its two runs of 16 keys
    if (__builtin_expect((hh >> 1) >= t_bad, 0)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (key0 + 16 * i < len) gone |= (unsigned)((unsigned)table[(unsigned)(key0 + 16 * i) >> p.page_log2] >= (unsigned)p.n_pages) << i;
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (qb < q0) continue;
      if (key0 + 32 > vis_first[qb]) {  // wave-uniform
        const int row = 32 * (unit0 + qb) + (l2 & 31);  // (those behind the last see what they like)
        const int rel = prev + (int)quot((unsigned)row, p.by_group) + 1 - key0;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + 4 * hi_here + (r & 3) >= rel) s[qb][r] = -INFINITY;
      }
      if (__builtin_expect(gone, 0)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (gone >> (r >> 3) & 1) s[qb][r] = -INFINITY;
      }
    }
  };
  // mx[] holds the row maxima of a half whose logits are already relative to the running max, i.e.
  // by how much the max would grow.  The running max is raised only when it lags by more than
  // 2^16 (or has never been set).  The decision (cross-lane max, compare) is taken early, under
  // the matrix pipe; the branch comes later.
  auto rescale_need = [&](const float (&dm)[QB], int q0 = 0) __attribute__((always_inline)) -> bool {
    int need = 0;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)  // no short-circuit: plain lane-wise compares, one wave-wide reduction at the end
      if (qb >= q0) need |= (int)(dm[qb] > stale) | ((int)(m_run[qb] == -INFINITY) & (int)(dm[qb] > -INFINITY));
    return __any(need);
  };
  auto rescale_decide = [&](const float (&mx)[QB], float (&dm)[QB], int q0 = 0) __attribute__((always_inline)) -> bool {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
      if (qb >= q0) dm[qb] = pair_max(mx[qb]);
    return rescale_need(dm, q0);
  };
  // s holds the logits of the half the maxima came from: they were formed against the old max
  auto rescale_apply = [&](const float (&dm)[QB], floatx16 (&s)[QB], int q0 = 0) __attribute__((always_inline)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (qb < q0) continue;
      const float cur = (m_run[qb] == -INFINITY) ? 0.f : m_run[qb];
      // only rows that asked for it move, so a row's arithmetic never depends on its wave neighbours
      const bool mine = (dm[qb] > stale) || (m_run[qb] == -INFINITY && dm[qb] > -INFINITY);
      const float m2 = mine ? fmaxf(m_run[qb], cur + dm[qb]) : m_run[qb];
      const float use = (m2 == -INFINITY) ? 0.f : m2;
      const float delta = use - cur;
      // a row without history (l = 0, O = 0) has nothing to scale, and its first reference may lie far enough
      // below zero for 2^-delta to overflow
      const float alpha = (m_run[qb] == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(-delta * to_log2);
      m_run[qb] = m2;
      l_run[qb] *= alpha;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        negm[qb][r] = -use;
        s[qb][r] -= delta;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        mfma_settle_a(o[qb][db]);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[qb][db][r] *= alpha;
      }
    }
  };
  // The first half of a pass: no history, so the row max of the half is the reference (0 for a row that sees
  // none of its keys) and neither l nor O needs touching.
  auto reference_first = [&](const float (&mx)[QB], floatx16 (&s)[QB]) __attribute__((always_inline)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float dm = pair_max(mx[qb]);
      const float use = (dm > -INFINITY) ? dm : 0.f;
      m_run[qb] = dm;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        negm[qb][r] = -use;
        s[qb][r] -= use;
      }
      asm volatile("" : "+v"(negm[qb]));  // 16 registers from here on, not one value splatted anew ahead of every MFMA chain
    }
  };
  // ls[] holds the row sums of the half just exponentiated (per lane: the 16 keys it owns).  A sum
  // above 2^20 moves the reference up by the power of two just above it (to the rounding of the reference); s holds
  // the in-flight logits of the next half, formed against the old reference.  Both lanes of a row
  // decide on the larger of their two sums, so a row never depends on its wave neighbours.
  auto rescale_from_sum = [&](const float (&ls)[QB], floatx16 (&s)[QB], int q0 = 0) __attribute__((always_inline)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (qb < q0) continue;
      const float tot = pair_max(ls[qb]);
      const bool bad = !(tot <= kRedoThreshold);  // also infinite or NaN
      overflowed |= __any((int)bad);
      const bool mine = !(tot <= kSumThreshold) && !bad;
      const int e = mine ? __builtin_amdgcn_frexp_expf(tot) : 0;  // tot < 2^e
      const float delta = (float)e * from_log2;
      const float alpha = __builtin_ldexpf(1.0f, -e);
      const float cur = (m_run[qb] == -INFINITY) ? 0.f : m_run[qb];
      const float use = cur + delta;
      if (mine) m_run[qb] = use;
      l_run[qb] *= alpha;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        negm[qb][r] = -use;
        s[qb][r] -= delta;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        mfma_settle_a(o[qb][db]);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[qb][db][r] *= alpha;
      }
    }
  };
  auto rowmax_all = [&](floatx16 (&s)[QB], float (&mx)[QB], int q0 = 0) __attribute__((always_inline)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (qb < q0) continue;
      float a = fmaxf(s[qb][0], s[qb][1]);
#pragma unroll
      for (int r = 2; r < 16; r += 2) a = fmaxf(fmaxf(a, s[qb][r]), s[qb][r + 1]);
      mx[qb] = a;
    }
  };

  // ---- the software pipeline (slot schedule: struct PromptSched) -----------------------------------
  constexpr int GK = KS / 2, GV = DB;  // fragments per batch, whatever the number of active units

  floatx16 sA[QB], sB[QB];
  uintx4 pb[QB][2];      // P^T fragments: 8 bf16 per 16-key slab, as packed pairs
  float lsum_early[QB];  // row sums of the early events of the half that the next step finishes
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) lsum_early[qb] = 0.f;
  // One exp event of a half whose logits are in s: event j covers logit j of the half's 2 NP, in
  // pairs; the second event of a pair also packs the pair into its P^T slot and the first adds the
  // previous pair's second exp to the row sum (`first`: there is none pending).
  float ev_a = 0.f, ev_b = 0.f;  // first exp of the pair in flight; second exp not yet in its row sum
  // unit that event j of a step with units Q0 .. QB-1 belongs to
  auto ev_unit = [](int j, int Q0, int QA) constexpr { return Q0 + (((j >> 1) % (QA * 4)) >> 2); };
  auto exp_event = [&](const floatx16 (&s)[QB], float (&ls)[QB], int j, bool first, auto q0_tag) __attribute__((always_inline)) {
    constexpr int Q0 = decltype(q0_tag)::value, QA = QB - Q0;  // active units Q0 .. QB-1
    const int k = j >> 1, slab = k / (QA * 4), kk = k % (QA * 4);
    const int qb = Q0 + (kk >> 2), jj = kk & 3, r = 8 * slab + 2 * jj;
    if ((j & 1) == 0) {
      if (first)
        asm volatile(
            "v_mul_f32_e32 %0, %2, %1\n\t"
            "v_exp_f32_e32 %0, %0"
            : "=&v"(ev_a)
            : "v"(s[qb][r]), "s"(to_log2));
      else
        asm volatile(
            "v_mul_f32_e32 %0, %4, %2\n\t"
            "v_exp_f32_e32 %0, %0\n\t"
            "v_add_f32_e32 %1, %3, %1"
            : "=&v"(ev_a), "+v"(ls[ev_unit(j - 1, Q0, QA)])
            : "v"(s[qb][r]), "v"(ev_b), "s"(to_log2));
    } else {
      float eb;
      unsigned pku;
      asm volatile(
          "v_mul_f32_e32 %0, %5, %3\n\t"
          "v_exp_f32_e32 %0, %0\n\t"
          "v_add_f32_e32 %2, %4, %2\n\t"
          "v_cvt_pk_bf16_f32 %1, %4, %0"
          : "=&v"(eb), "=v"(pku), "+v"(ls[qb])
          : "v"(s[qb][r + 1]), "v"(ev_a), "s"(to_log2));
      pb[qb][slab][jj] = pku;
      ev_b = eb;
    }
  };
  // the early events of a half all at once (prologue, masked steps, and again after a sum-driven shift)
  auto early_events = [&](const floatx16 (&s)[QB], auto q0_tag) __attribute__((always_inline)) {
    constexpr int Q0 = decltype(q0_tag)::value, QA = QB - Q0;
    constexpr int NEAR = PromptSched<D, QA, LPG>::NEAR;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) lsum_early[qb] = 0.f;
    if (NEAR > 0) {
#pragma unroll
      for (int j = 0; j < NEAR; ++j) exp_event(s, lsum_early, j, j == 0, q0_tag);
      lsum_early[ev_unit(NEAR - 1, Q0, QA)] += ev_b;
    }
  };
  bf16x8 kg[2][GK];          // K fragment batches
  short4_ vh[2][GV][2];      // V^T fragment batches, as the two transpose-read halves of each fragment
  auto v_half = [&](int tt, int db, int half, int imm) __attribute__((always_inline)) -> short4_ {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, vaddr[db] + (unsigned)(imm + 16 * tt * ROWB + half * 8 * ROWB)));
  };

  // One pipeline step for half hh.  On entry s_cur holds S^T of half hh (masked, relative to the
  // running max), kg[0] the first batch of K fragments of half hh+1, and kaddr/vaddr point at the
  // tiles of halves hh+1 / hh.  ODD steps (second half of a tile) end with the workgroup barrier
  // and the ring refill for the tiles after next; MASKED selects the variant for halves hh+1 that
  // reach past the causal horizon, and for every half once a row sum has overflowed (mask, then the
  // exact row max, after the matrix work); PLAIN the variant whose refill consists of cache tiles only, slab by slab in
  // the slot schedule, where the others refill whole tiles after the matrix work.  q0_tag = 1 (two-unit kernel only):
  // unit 0 has passed its causal horizon for good and only unit 1 is worked on, with the schedule of a one-unit step; a
  // masked step of both units that is followed by such a step (next_unit1_only) leaves the early events in that step's
  // numbering.  Past the piece's last tile the ring need not hold keys: the last step forms an S^T of stale LDS
  // contents, on which nothing may be decided.
  auto step = [&](floatx16 (&s_cur)[QB], floatx16 (&s_next)[QB], int hh, auto odd_tag, auto masked_tag, auto plain_tag,
                  auto q0_tag, bool next_unit1_only = false) __attribute__((always_inline)) {
    constexpr bool PLAIN = decltype(plain_tag)::value;
    constexpr bool ODD = decltype(odd_tag)::value;
    constexpr bool MASKED = decltype(masked_tag)::value;
    constexpr int Q0 = decltype(q0_tag)::value, QA = QB - Q0;
    using S = PromptSched<D, QA, LPG>;
    constexpr int M1 = S::M1, M = S::M, EW = S::EW, NE = S::NE, NEAR = S::NEAR, NMAIN = S::NMAIN;
    constexpr int R = S::R, RW = S::RW;
    const int t = hh >> 1;
    constexpr int KIMM = ODD ? 0 : HALFB;  // even hh: half hh+1 is the second half of tile t
    constexpr int VIMM = ODD ? HALFB : 0;  // even hh: half hh is the first half of tile t
    float lsum[QB], lsum_next[QB];  // row sums of half hh (early part included) and of the early part of hh+1
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      lsum[qb] = lsum_early[qb];
      lsum_next[qb] = 0.f;
    }  // (entries of units before Q0 are carried along untouched and never added anywhere)
    float mx[QB], dm[QB];
    bool need_rescale = false;
    int sum_flag = 0;      // per lane: a row sum of this half passed 2^20 (or is not a number)
    int kslot_prev = 0, vslot_prev = 0;
    const bool more = PLAIN || hh + 1 < 2 * t_end;  // half hh + 1 is there (or nothing is decided on it)

    wait_lds<0>();  // kg[0] (fetched at the end of the previous step) has landed
    // the page that the next (odd) step's copies of K come from: there by its own wait
    if (PLAIN && !ODD) ask_page(t + 1 + NV);
    if (PLAIN && ODD) k_from = from_page();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      // ---- waits and the barrier come before the MFMA of the slot
      if (i == GK * QA) wait_lds<(S::rd_before(GK * QA) - GK)>();                 // kg[1]
      if (i == M1) wait_lds<(S::rd_before(M1) - GK - 2 * GV)>();                  // vg[0]
      if (i == EW) wait_lds<(S::rd_before(EW) - GK - 4 * GV)>();                  // vg[1]
      if (ODD && i == EW) {
        // Every read of K[t] and V[t] by this wave has returned.  K[t+2] and V[t+1] were issued
        // NV-1 tiles ago: they are the oldest group in flight.
        if (PLAIN || (t + NV < t_end && t + NV < t_whole))
          wait_vm<(NV - 2) * LPG>();
        else
          wait_vm<0>();  // the group issued last is not whole
        __builtin_amdgcn_s_barrier();  // ... and this holds for every wave of the workgroup
        kslot_prev = kslot == 0 ? NK - 1 : kslot - 1;  // K[t]'s slot (kslot already names K[t+1]) takes K[t+1+NV]
        vslot_prev = vslot;                            // V[t]'s slot takes V[t+NV]
      }
      // (one unit: the last weights have just been packed, two instructions ahead of the matrix instruction that reads them, which is asm)
      if (QA == 1 && i == EW) asm volatile("s_nop 1" : "+v"(pb[Q0][1]));
      // ---- the MFMA
      if (i < M1) {
        const int ks = i / QA, qb = Q0 + i % QA;
        if (ks == 0)
          mfma_qk_first(s_next[qb], kg[0][0], qf[qb][0], negm[qb]);
        else
          mfma_qk(s_next[qb], kg[ks / GK][ks % GK], qf[qb][ks]);
      } else {
        const int sl = (i - M1) / QA, qb = Q0 + (i - M1) % QA, tt = sl / DB, db = sl % DB;
        const short8_ a8 = __builtin_shufflevector(vh[sl / GV][sl % GV][0], vh[sl / GV][sl % GV][1], 0, 1, 2, 3, 4, 5, 6, 7);
        mfma_pv(o[qb][db], __builtin_bit_cast(bf16x8, a8), __builtin_bit_cast(bf16x8, pb[qb][tt]));
      }
      __builtin_amdgcn_sched_barrier(0);
      // ---- its share of everything else
      // LDS reads
#pragma unroll
      for (int r = (i * R + RW - 1) / RW; r < ((i + 1) * R + RW - 1) / RW && r < R; ++r) {  // rd_slot(r) == i
        if (r < GK) {
          kg[1][r] = k_frag(GK + r, KIMM);
        } else if (r < GK + 4 * GV) {
          const int q = r - GK, f = q / 2, half = q % 2;  // fragment f = (tt, db) of the half, in use order
          vh[f / GV][f % GV][half] = v_half(f / DB, f % DB, half, VIMM);
        } else {
          const int j = r - GK - 4 * GV;
          kg[0][j] = k_frag(j, ODD ? HALFB : 0);  // kg[0] of the NEXT step (half hh+2)
        }
      }
      // after an even step the next K half starts a new tile: move the K read offsets to its ring
      // slot, a few per slot, between the last read of this tile's K and the first of the next
      if (!ODD && i >= GK * QA && i < GK * QA + (KS + 1) / 2) {
        const int kn = kslot + 1 == NK ? 0 : kslot + 1;
        const unsigned dk = (unsigned)((kn - kslot) * TILEB);
        const int a = (i - GK * QA) * 2;
        kaddr[a] += dk;
        if (a + 1 < KS) kaddr[a + 1] += dk;
        if (i == GK * QA + (KS + 1) / 2 - 1) kslot = kn;
      }
      // exp events of half hh ...
      if (i == EW) lsum[ev_unit(NE - 1, Q0, QA)] += ev_b;
#pragma unroll
      for (int j = NEAR + (i * NMAIN + EW - 1) / EW; j < NEAR + ((i + 1) * NMAIN + EW - 1) / EW && j < NE; ++j)
        exp_event(s_cur, lsum, j, j == NEAR, q0_tag);
      // ... and, below the causal horizon, the early ones of half hh+1, whose S^T is complete by now
      if (!MASKED && NEAR > 0 && i >= EW) {
#pragma unroll
        for (int j = ((i - EW) * NEAR + (M - EW) - 1) / (M - EW); j < ((i - EW + 1) * NEAR + (M - EW) - 1) / (M - EW) && j < NEAR; ++j)
          exp_event(s_next, lsum_next, j, j == 0, q0_tag);
        if (i == M - 1) lsum_next[ev_unit(NEAR - 1, Q0, QA)] += ev_b;
      }
      if (i == EW + 1) {
#pragma unroll
        for (int qb = Q0; qb < QB; ++qb) sum_flag |= (int)!(lsum[qb] <= kSumThreshold);
      }
      // ring refill and the V address of the next tile (odd steps, after the barrier)
      if (ODD && i >= EW) {
        if (PLAIN) {
#pragma unroll
          for (int d = ((i - EW) * LPG) / (M - EW); d < ((i - EW + 1) * LPG) / (M - EW); ++d) {
            if (d < SLABS) issue_slab(false, k_from, kslot_prev, d);
            else issue_slab(true, v_from, vslot_prev, d - SLABS);
          }
        }
        if (i == M - 1) {
          const int vn = vslot + 1 == NV ? 0 : vslot + 1;
          const unsigned dv = (unsigned)((vn - vslot) * TILEB);
#pragma unroll
          for (int d2 = 0; d2 < DB; ++d2) vaddr[d2] += dv;
          vslot = vn;
          if (PLAIN) v_from = k_from;  // (tile t + 1 + NV: V's of the next turn)
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int qb = Q0; qb < QB; ++qb) {
      l_run[qb] += lsum[qb];
      lsum_early[qb] = lsum_next[qb];
    }
    if (__builtin_expect(__any(sum_flag), 0)) {
#pragma unroll
      for (int qb = Q0; qb < QB; ++qb) mfma_settle_v(s_next[qb]);
      rescale_from_sum(lsum, s_next, Q0);  // (past the last half s_next is stale, and merely moved)
      if (!MASKED) early_events(s_next, q0_tag);  // they were formed against the old reference: once more
    }
    if (!PLAIN && ODD) {
      issue_tile(false, t + 1 + NV, kslot_prev);
      issue_tile(true, t + NV, vslot_prev);
    }
    if (MASKED && more) {
#pragma unroll
      for (int qb = Q0; qb < QB; ++qb) mfma_settle_v(s_next[qb]);
      mask_half(s_next, hh + 1, Q0);
      rowmax_all(s_next, mx, Q0);
      need_rescale = rescale_decide(mx, dm, Q0);
    }
    if (__builtin_expect(need_rescale, 0)) {
#pragma unroll
      for (int qb = Q0; qb < QB; ++qb) mfma_settle_v(s_next[qb]);
      rescale_apply(dm, s_next, Q0);
    }
    if (MASKED) {
      if (Q0 == 0 && next_unit1_only)
        early_events(s_next, std::integral_constant<int, QB - 1>{});
      else
        early_events(s_next, q0_tag);
    }
  };

  if (t_begin < t_end) {
    // A second pass (exact = true) follows only if a row sum overflowed in the first.
    for (bool exact = false;; exact = true) {
      reset_state();
      // Tiles whose two steps only produce halves entirely below the nearest causal horizon take the
      // fast variant: step 2t+1 produces half 2t+2 = keys [64t+64, 64t+96), so it needs 64t+96 <= vis_min.
      int t_fast = (vis_min - 96) / BN + 1;  // first tile that is not fast
      if (vis_min < 96 || exact) t_fast = 0;
      if (!exact && t_end * BN <= vis_min) t_fast = t_end;  // the piece ends below every horizon
      if (t_fast > t_end) t_fast = t_end;
      if (t_fast > t_bad - 1) t_fast = t_bad - 1;  // (pages that are none are masked)
      // From tile t_dead on every key is beyond the last row of unit 0 and only unit 1
      // is worked on, fast up to its own horizon (t_fast1), masked from there.
      int t_dead = vis_last0 > 0 ? (vis_last0 + BN - 1) / BN : 0;
      if (exact || t_dead > t_end) t_dead = t_end;
      int t_fast1 = (vis_first[QB - 1] - 96) / BN + 1;
      if (vis_first[QB - 1] < 96 || exact) t_fast1 = 0;
      if (t_fast1 > t_end) t_fast1 = t_end;
      if (t_fast1 > t_bad - 1) t_fast1 = t_bad - 1;
      // ... and tiles whose refill (tile t + 1 + NV) has all its rows take the main loop (every tile of a piece that has nothing else).
      int t_plain = t_whole >= t_end ? t_end : t_whole - NV - 1;
      if (t_plain > t_fast) t_plain = t_fast;
      // Prologue.  The first pass finds the ring's fill under way; a second pass fills it again.
      if (exact) prefill(0, NV);
      if (t_begin + NV < t_end && t_begin + NV < t_whole)  // every group of the fill is whole
        wait_vm<(NV - 1) * LPG>();
      else
        wait_vm<0>();
      wait_lds<0>();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (idle) {
        // no rows of its own: this wavefront only moves its share of the tiles
        for (int t = t_begin, ks = 0, vs = 0; t < t_end; ++t) {
          if (t + NV < t_end && t + NV < t_whole)
            wait_vm<(NV - 2) * LPG>();
          else
            wait_vm<0>();
          wait_lds<0>();
          asm volatile("" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          issue_tile(false, t + 1 + NV, ks);
          issue_tile(true, t + NV, vs);
          ks = ks + 1 == NK ? 0 : ks + 1;
          vs = vs + 1 == NV ? 0 : vs + 1;
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kg[ks / GK][ks % GK] = k_frag(ks, 0);
        wait_lds<0>();
        // (the matrix instructions are asm: what they start from has to be written two instructions ahead of them)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) asm volatile("s_nop 3" : "+v"(negm[qb]));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            if (ks == 0)
              mfma_qk_first(sA[qb], kg[0][0], qf[qb][ks], negm[qb]);
            else
              mfma_qk(sA[qb], kg[ks / GK][ks % GK], qf[qb][ks]);
          }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) mfma_settle_v(sA[qb]);
        const bool whole = t_begin * BN + 32 <= vis_min && t_begin < t_bad;
        if (!whole) mask_half(sA, 2 * t_begin);
        float mx[QB];
        rowmax_all(sA, mx);
        reference_first(mx, sA);
        // A row whose 32 logits are all -inf, none of them masked, has no reference, and the main loop finds none: the exact pass does.
        if (whole) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) overflowed |= __any((int)(m_run[qb] == -INFINITY));
        }
        if (t_begin >= t_dead && t_dead < t_end)
          early_events(sA, std::integral_constant<int, QB - 1>{});  // the first step already works on unit 1 alone
        else
          early_events(sA, std::integral_constant<int, 0>{});
        // first K batch of the first step: second half of tile t_begin
#pragma unroll
        for (int j = 0; j < GK; ++j) kg[0][j] = k_frag(j, HALFB);
        constexpr std::integral_constant<int, 0> both{};
        constexpr std::false_type even{}, unmasked{}, mixed{};
        constexpr std::true_type odd{}, masked{}, plain{};
        int t = t_begin;
        if (t < t_plain) {
          ask_page(t + NV);
          v_from = from_page();
        }
        asm volatile(".p2align 5\n\ts_nop 0");
        for (; t < t_plain; ++t) {
          step(sA, sB, 2 * t, even, unmasked, plain, both);
          step(sB, sA, 2 * t + 1, odd, unmasked, plain, both);
        }
        for (; t < t_fast; ++t) {
          step(sA, sB, 2 * t, even, unmasked, mixed, both);
          step(sB, sA, 2 * t + 1, odd, unmasked, mixed, both);
        }
        for (; t < t_dead; ++t) {
          step(sA, sB, 2 * t, even, masked, mixed, both);
          step(sB, sA, 2 * t + 1, odd, masked, mixed, both, t + 1 == t_dead && t_dead < t_end);
        }
        // unit 0 is done for good (every further key is beyond its last row): unit 1 alone
        constexpr std::integral_constant<int, 1> second{};
        for (; t < t_fast1; ++t) {
          step(sA, sB, 2 * t, even, unmasked, mixed, second);
          step(sB, sA, 2 * t + 1, odd, unmasked, mixed, second);
        }
        for (; t < t_end; ++t) {
          step(sA, sB, 2 * t, even, masked, mixed, second);
          step(sB, sA, 2 * t + 1, odd, masked, mixed, second);
        }
      }
      wait_vm<0>();  // nothing of ours may still be writing LDS when the workgroup retires or starts over
      wait_lds<0>();
      __syncthreads();  // every wavefront of the workgroup is through with the rings
      if (exact) break;
      // Did a row sum of any wavefront overflow?
      if (lane_now() == 0) *LDS_PTR(int, lds0 + 4u * (unsigned)w) = overflowed;
      __syncthreads();
      int any_overflow = 0;
#pragma unroll
      for (int ww = 0; ww < 4; ++ww) any_overflow |= *LDS_PTR(const int, lds0 + 4u * (unsigned)ww);
      any_overflow = __builtin_amdgcn_readfirstlane(any_overflow);
      __syncthreads();
      if (__builtin_expect(any_overflow == 0, 1)) break;
    }
    mfma_settle_a(o[0][0]);  // (one wait for all; the others are tied behind it)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db) asm volatile("" : "+a"(o[qb][db]));
  } else {
    reset_state();
  }

  // ---- out, or what the piece leaves for the merge, turned in LDS (the rings are dead by now): every store instruction writes whole rows, 16 bytes per lane.
  // (the lane's place and its row's token and head are formed anew: nothing is held for them through the main loop)
  const int le = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), hie = le >> 5, me = le & 31;
  constexpr int OROWF = D * 4 + 16;  // padded LDS row: fp32 partials
  constexpr int OROWH = D * 2 + 16;  // padded LDS row: bf16 output
  const unsigned obase = lds0 + (unsigned)(w * kRowsPerUnit * OROWF);  // this wavefront's staging area, reused by its units
  const bool alone = wk.n_pieces == 1;
  const int64_t n_rows = (int64_t)p.n_tokens * Hq;
  float odd = 0.f;  // 0 as long as all outputs are finite
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float l_tot = pair_sum(l_run[qb]);
    const int row0 = (unit0 + qb) * kRowsPerUnit, left = wk.rows - row0;
    const int n_live = left < 0 ? 0 : left < kRowsPerUnit ? left : kRowsPerUnit;  // rows of the unit that exist
    const unsigned my_place = prompt_place(p, wk, row0 + me);
    // `rows` whole rows of `chunks` 16-byte pieces, turned in LDS, to dst (the batch's first row), in a loop of few instructions
    auto store_rows = [&](unsigned char* dst, auto bytes_tag, unsigned lds_row) __attribute__((always_inline)) {
      constexpr int BYTES = decltype(bytes_tag)::value, CPR = BYTES / 16, RPI = 64 / CPR;
      const unsigned r_lane = (unsigned)le / CPR, c = (unsigned)le % CPR * 16u;
      unsigned char* lane_dst = dst + c;
      unsigned at = obase + r_lane * lds_row + c;
#pragma unroll 1
      for (unsigned i = r_lane; i < (unsigned)kRowsPerUnit; i += 4 * RPI) {
        uintx4 x[4];
#pragma unroll
        for (unsigned j = 0; j < 4; ++j) x[j] = *LDS_PTR(const uintx4, at + j * RPI * lds_row);
#pragma unroll
        for (unsigned j = 0; j < 4; ++j) asm volatile("" : "+v"(x[j]));
#pragma unroll
        for (unsigned j = 0; j < 4; ++j) {
          const unsigned r = i + j * RPI;
          const unsigned at_row = (unsigned)__builtin_amdgcn_ds_bpermute((int)(4 * r), (int)my_place);
          if ((int)r < n_live) __builtin_nontemporal_store(x[j], reinterpret_cast<uintx4*>(lane_dst + (uint64_t)at_row * BYTES));
        }
        at += 4 * RPI * lds_row;
      }
    };
    if (hie == 0 && me < n_live) prompt_sums(p, wk, my_place, m_run[qb] * to_log2, l_tot);
    float check = 0.f;
    if (alone) {
      const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = o[qb][db][rg * 4 + e] * inv;
            check = __builtin_fmaf(x, 0.f, check);
            v[e] = (__bf16)x;
          }
          *LDS_PTR(bf16x4, obase + (unsigned)(me * OROWH + (db * 32 + 8 * rg + 4 * hie) * 2)) = v;
        }
      store_rows(static_cast<unsigned char*>(p.out), std::integral_constant<int, D * 2>{}, OROWH);
    } else {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          floatx4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = o[qb][db][rg * 4 + e];
            check = __builtin_fmaf(v[e], 0.f, check);
          }
          *LDS_PTR(floatx4, obase + (unsigned)(me * OROWF + (db * 32 + 8 * rg + 4 * hie) * 4)) = v;
        }
      store_rows(reinterpret_cast<unsigned char*>(p.part_o) + (uint64_t)wk.piece * (uint64_t)n_rows * (D * 4), std::integral_constant<int, D * 4>{}, OROWF);
    }
    if (me < n_live) odd += check;
  }

  prompt_again<D, QB>(p, wk, lds0, w, odd != 0.f);  // (NaN)
}

// Short prompts and chunks: a unit a wavefront, two workgroups a CU, tiles one ahead, a turn's matrix instructions, exponentials and outputs one after the other (the
// other workgroup's fill the gaps).  Sequences of fewer rows than a workgroup of the kernel above has are bound by what a launch does once.  32 heads on 8, 128 wide, with the launch in front:
// 1000 tokens 33 us, 33 12.3; tiles three ahead, where a CU has one workgroup, were no gain (37 and 13).
constexpr int kFewRing = 2;
template <int D>
constexpr int prompt_few_lds = kFewRing * 2 * kTileKeys * D * 2;

template <int D>
__global__ void __launch_bounds__(256, 2) attn_prompt_few_kernel(PAttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned lds0 = (unsigned)(uintptr_t)((unsigned char __attribute__((address_space(3)))*)smem);
  constexpr int CH = D / 8, ROWB = D * 2, KS = D / 16, DB = D / 32;  // 16-byte chunks and bytes of a row; contraction steps of S^T; tiles of O^T
  constexpr int BN = kTileKeys, TILEB = BN * ROWB;
  constexpr int RPS = 64 / CH, SLABS = 16 / RPS;  // rows of a 1 KiB copy; copies of a wavefront's 16 rows
  constexpr int KSW = CH < 16 ? CH : 16, VSW = CH / 4;
  constexpr float kStale = 16.0f;  // log2 units
  constexpr floatx16 zero = {};

  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PromptWork wk = prompt_work(p, blockIdx.x);
  if (!wk.any) return;
  const int prev = wk.sq.len - wk.sq.n;

  // ---- the wavefront's rows
  const int first = wk.row0 + w * 32, r = first + c32, row = r < wk.rows ? r : wk.rows - 1, tok = (int)quot((unsigned)row, p.by_group);
  const int last = first + 31 < wk.rows ? first + 31 : wk.rows - 1, my_vis = prev + tok + 1;
  const int vis_first = prev + (int)quot((unsigned)first, p.by_group) + 1, vis_last = first < wk.rows ? prev + (int)quot((unsigned)last, p.by_group) + 1 : 0;
  bf16x8 qf[KS];
  {
    const __bf16* qrow = static_cast<const __bf16*>(p.q) + (int64_t)(wk.sq.first + tok) * p.q_stride + (wk.g * p.group + row - tok * p.group) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + 16 * ks + 8 * h);
  }

  // ---- tiles on their way
  const int32_t* table = p.tables + (int64_t)wk.seq * p.table_stride;
  const int t_begin = wk.key_begin / BN, t_end = (wk.key_end + BN - 1) / BN;
  const uint64_t head = (uint64_t)(unsigned)wk.g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  PageWindow win;  // of tiles [16 n, 16 n + 16): those of the tile asked for last
  const unsigned dma_k = (unsigned)((l / CH) * ROWB + (((l % CH) ^ (l / CH)) * 16)), dma_v = (unsigned)((l / CH) * ROWB + (((l % CH) ^ ((l / CH & 3) * VSW)) * 16));
  auto k_off = [&](int i) __attribute__((always_inline)) -> unsigned { return dma_k ^ (unsigned)(i * RPS % KSW * 16); };
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= t_end) return;
    if ((t & 15) == 0 || t == t_begin) win.fetch(p, table, (t & ~15) * BN, wk.sq.len, l);
    const int at = 4 * (t & 15) + w, key0 = t * BN + 16 * w;
    const int number = __builtin_amdgcn_readlane(win.number, at);
    const bool there = win.there >> at & 1;
    const uint64_t from = (uint64_t)(unsigned)(there ? number : 0) * p.page_bytes + head + (unsigned)((key0 & ((1 << p.page_log2) - 1)) * ROWB);
    const unsigned char *kf = static_cast<const unsigned char*>(p.k_pages) + from, *vf = static_cast<const unsigned char*>(p.v_pages) + from;
    const unsigned slot = lds0 + (unsigned)((t % kFewRing) * 2 * TILEB + 16 * w * ROWB);
    const int n = there ? wk.sq.len - key0 : 0;  // rows that are not there become zeros, so that 0 times them is 0
    if (__builtin_expect(n >= 16, 1)) {
#pragma unroll
      for (int i = 0; i < SLABS; ++i) {
        dma16(kf + i * 1024, k_off(i), slot + i * 1024);
        dma16(vf + i * 1024, dma_v, slot + TILEB + i * 1024);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < SLABS; ++i) {
        if (i * RPS + l / CH < n) {
          dma16(kf + i * 1024, k_off(i), slot + i * 1024);
          dma16(vf + i * 1024, dma_v, slot + TILEB + i * 1024);
        } else {
          *LDS_PTR(uintx4, slot + (unsigned)(i * 1024 + l * 16)) = uintx4{0u, 0u, 0u, 0u};
          *LDS_PTR(uintx4, slot + (unsigned)(TILEB + i * 1024 + l * 16)) = uintx4{0u, 0u, 0u, 0u};
        }
      }
    }
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

  floatx16 o[DB];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero;
  auto attend = [&](int t, unsigned gone) __attribute__((always_inline)) {
    const unsigned slot = (unsigned)((t % kFewRing) * 2 * TILEB);
    floatx16 s[2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*LDS_PTR(const bf16x8, kaddr[ks] + slot + (unsigned)(tt * 32 * ROWB)), qf[ks], ks == 0 ? zero : s[tt], 0, 0, 0);
    const int key0 = t * BN;
    if (key0 + BN > vis_first || gone) {  // wave-uniform
      const int rel = my_vis - key0 - 4 * h;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * tt + 8 * (i >> 2) + (i & 3) >= rel || (gone >> (2 * tt + (i >> 3)) & 1)) s[tt][i] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[tt][i]);
    mx = pair_max(mx) * p.scale_log2e;
    // only rows that ask for it move, so a row's arithmetic never depends on its wave neighbours
    const bool mine = mx > m_run + kStale || (m_run == -INFINITY && mx > -INFINITY);
    if (__any(mine)) {
      const float m2 = mine ? mx : m_run;
      const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m2);
      m_run = m2;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    bf16x8 pf[2][2];
    float sum = 0.f;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i], p.scale_log2e, -ref));
        sum += a;
        pf[tt][i >> 3][i & 7] = (__bf16)a;
      }
    l_run += sum;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const unsigned at = vaddr[db] + slot + (unsigned)(16 * tt * ROWB);
        const short4_ lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, at)), up = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4_, at + 8 * ROWB));
        const short8_ v = __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pf[tt >> 1][tt & 1], o[db], 0, 0, 0);
      }
  };

#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));  // (waited for here, not in the loop)
  issue(t_begin);
#pragma unroll 1
  for (int t = t_begin; t < t_end; ++t) {
    const unsigned gone = (unsigned)(~win.there >> (4 * (t & 15))) & 15;  // runs of 16 keys that are in no page, or do not exist
    wait_vm<0>();
    wait_lds<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // the tile is there for all, and the slot of the one before is free
    asm volatile("" ::: "memory");
    issue(t + 1);
    if (t * BN < vis_last) attend(t, gone);
  }

  // ---- out, or what the piece leaves for the merge
  float check = 0.f;  // 0 as long as all outputs are finite
  const float l_tot = pair_sum(l_run);
  if (r < wk.rows) {
    const unsigned place = prompt_place(p, wk, r);
    if (h == 0) prompt_sums(p, wk, place, m_run, l_tot);
    const bool alone = wk.n_pieces == 1;
    const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int c = 32 * db + 2 * i + 4 * h;
#pragma unroll
        for (int e = 0; e < 4; ++e) check = __builtin_fmaf(o[db][i + e], 0.f, check);
        if (alone) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[db][i + e] * inv);
          *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + (int64_t)place * D + c) = v;
        } else {
          *reinterpret_cast<floatx4*>(p.part_o + ((int64_t)wk.piece * p.n_tokens * p.n_q_heads + place) * D + c) = floatx4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]};
        }
      }
  }
  prompt_again<D, 1>(p, wk, lds0, w, check != 0.f);  // (NaN)
}

template <class K>
static hipError_t prepare_one(K* kernel, int lds, bool* done) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!done[dev]) {  // (idempotent; two threads at worst set it twice)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    done[dev] = true;
  }
  return hipSuccess;
}
template <int D>
static hipError_t prepare_both() {
  static bool done[2][64] = {};
  const hipError_t e = prepare_one(&attn_prompt_kernel<D>, prompt_lds<D>, done[0]);
  return e == hipSuccess ? prepare_one(&attn_prompt_few_kernel<D>, prompt_few_lds<D>, done[1]) : e;
}
template <int D>
static hipError_t launch_one(const PAttnParams& p, int units_per_wave, hipStream_t s) {
  const dim3 grid((unsigned)p.n_units * (unsigned)p.n_kv_heads), block(256);
  if (units_per_wave == 2)
    hipLaunchKernelGGL(attn_prompt_kernel<D>, grid, block, prompt_lds<D>, s, p);
  else
    hipLaunchKernelGGL(attn_prompt_few_kernel<D>, grid, block, prompt_few_lds<D>, s, p);
  return hipGetLastError();
}

hipError_t prepare_attn_prompt(int head_dim, bool bf16) { return !bf16 ? prepare_attn_prompt_f32(head_dim) : head_dim == 128 ? prepare_both<128>() : prepare_both<64>(); }
hipError_t launch_attn_prompt(const PAttnParams& p, int head_dim, bool bf16, int units_per_wave, hipStream_t s) {
  return !bf16 ? launch_attn_prompt_f32(p, head_dim, s) : head_dim == 128 ? launch_one<128>(p, units_per_wave, s) : launch_one<64>(p, units_per_wave, s);
}

// ---- the merge of pieces ---------------------------------------------------------------------------------------------------
// A thread has 16 bytes of a row and goes through its pieces, eight in flight; rows of one piece have been written.  Bound by memory, and by the way to the first bytes: a
// workgroup has no second rows, which would wait for its first (chunks of 45 tokens of 8 sequences in 16 pieces: 8.5 us, with four rows a thread 17.4; of 256 tokens of
// 28 heads on 4: 13.2 and 21.1, which is 3.4 TB/s of partial results).
template <class T, int D>
__global__ void __launch_bounds__(256) pmerge_kernel(PAttnParams p, int parts_log2) {
  constexpr int V = D / 4, ROWS = 256 / V, N = 8;  // (unit_rows / ROWS = 2^parts_log2 workgroups share a block's rows)
  const unsigned todo = ((unsigned)((ConstPtr<int32_t>)(uintptr_t)p.list_head)[1] * (unsigned)p.n_kv_heads) << parts_log2;
#pragma unroll 1
  for (unsigned id = blockIdx.x; id < todo; id += gridDim.x) {
    const int at_block = (int)quot(id >> parts_log2, p.by_kv_heads);
    const PromptWork wk = prompt_item(p, ((ConstPtr<int32_t>)(uintptr_t)p.merges)[at_block], (int)(id >> parts_log2) - at_block * p.n_kv_heads);
    const int n = wk.n_pieces, c = threadIdx.x % V, r = wk.row0 + (int)(id & ((1u << parts_log2) - 1)) * ROWS + (int)threadIdx.x / V;
    if (r >= wk.rows) continue;
    const unsigned place = prompt_place(p, wk, r), Hq = (unsigned)p.n_q_heads;
    const int64_t n_rows = (int64_t)p.n_tokens * Hq;
    float M = -INFINITY, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += N) {
      floatx2 ml[N];
      floatx4 o[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t part = (int64_t)(i0 + i < n ? i0 + i : n - 1) * n_rows + place;
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
    const uint64_t at = (uint64_t)place * D + (unsigned)c * 4u;
    if constexpr (sizeof(T) == 2) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)acc[e];
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + at) = v;
    } else {
      *reinterpret_cast<floatx4*>(static_cast<float*>(p.out) + at) = acc;
    }
    const unsigned token = place / Hq;
    if (p.lse && c == 0) p.lse[(int64_t)(place - token * Hq) * p.n_tokens + token] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
  }
}

hipError_t launch_pmerge(const PAttnParams& p, int head_dim, bool bf16, hipStream_t s) {
  const int rows = 256 / (head_dim / 4);
  int lg = 0;
  while (rows << lg < p.unit_rows) ++lg;
  // (how many blocks there are to merge only the device knows: no more workgroups than find out at once, 32 a CU)
  const unsigned most = ((unsigned)p.n_blocks * (unsigned)p.n_kv_heads) << lg, cap = 32u * (unsigned)p.n_cu;
  const dim3 grid(most < cap ? most : cap), block(256);
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

