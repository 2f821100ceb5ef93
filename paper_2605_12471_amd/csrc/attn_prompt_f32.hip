// Attention of whole prompts, and of chunks of them, of many sequences on a cache in pages, fp32: attn_prompt.hip's shape with one unit a wavefront and tiles of
// 32 keys, on the fp32 matrix instructions.
//
// Bound by these: 32x32x2, 4 kFLOP in 64 cycles.  S^T = K Q^T: a lane has 16 bytes of a K row and of its query's, four contraction steps whose columns are
// whichever these are.  O^T = V^T P^T: step i's two keys are those whose logits the two lanes of a row hold in register i, and a lane's 16 (64 wide: 8)
// bytes of such a V row are its columns of all tiles of O^T (tile j has every fourth, or second, column of the head), so that V needs no transpose.
#include "prompt.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kF32Ring = 3, kF32Tile = 32;
template <int D>
constexpr int prompt_f32_lds = kF32Ring * 2 * kF32Tile * D * 4;

template <int D>
__global__ void __launch_bounds__(256, 1) attn_prompt_f32_kernel(PAttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned lds0 = (unsigned)(uintptr_t)((unsigned char __attribute__((address_space(3)))*)smem);
  constexpr int CH = D / 4, ROWB = D * 4, KS = D / 8, JT = D / 32;  // 16-byte chunks and bytes of a row; 16-byte shares of a lane; tiles of O^T
  constexpr int BN = kF32Tile, TILEB = BN * ROWB, NS = kF32Ring;
  constexpr int RPS = 64 / CH, SLABS = 8 / RPS;  // rows of a 1 KiB copy; copies of a wavefront's 8 rows
  constexpr float kStale = 16.0f;
  typedef __attribute__((ext_vector_type(JT))) float vvec;

  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PromptWork wk = prompt_work(p, blockIdx.x, l);
  if (!wk.any) return;
  const int G = p.group, Hq = p.n_q_heads, prev = wk.sq.len - wk.sq.n;

  // ---- the wavefront's rows: lane (c32, h) holds the columns 8 j + 4 h .. + 3 of row c32
  const int unit0 = wk.row0 + w * 32;
  int my_vis, vis_first, vis_last;
  floatx4 qf[KS];
  {
    const int r = unit0 + c32, row = r < wk.rows ? r : wk.rows - 1, tok = (int)quot((unsigned)row, p.by_group);
    const int last = unit0 + 31 < wk.rows ? unit0 + 31 : wk.rows - 1;
    my_vis = prev + tok + 1;
    vis_first = unit0 < wk.rows ? prev + (int)quot((unsigned)unit0, p.by_group) + 1 : 0;
    vis_last = unit0 < wk.rows ? prev + (int)quot((unsigned)last, p.by_group) + 1 : 0;
    const float* qrow = static_cast<const float*>(p.q) + (int64_t)(wk.sq.first + tok) * p.q_stride + (wk.g * G + row - tok * G) * D;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[j] = *reinterpret_cast<const floatx4*>(qrow + 8 * j + 4 * h);
  }

  // ---- tiles on their way, eight rows a wavefront
  const int32_t* table = p.tables + (int64_t)wk.seq * p.table_stride;
  const int t_begin = wk.key_begin / BN, t_end = (wk.key_end + BN - 1) / BN;
  const uint64_t head = (uint64_t)(unsigned)wk.g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  PageWindow win;  // of tiles [32 n, 32 n + 32)
  unsigned k_off[SLABS];
#pragma unroll
  for (int i = 0; i < SLABS; ++i) {
    const int r = i * RPS + l / CH, in_tile = 8 * w + r;
    k_off[i] = (unsigned)(r * ROWB + (((l % CH) ^ (in_tile % 16)) * 16));
  }
  const unsigned v_off = (unsigned)(l * 16);
  auto issue = [&](int t) __attribute__((always_inline)) -> bool {
    if (t >= t_end) return false;
    if ((t & 31) == 0 || t == t_begin) win.fetch(p, table, (t & ~31) * BN, wk.sq.len, l);
    const int at = 2 * (t & 31) + (w >> 1), key0 = t * BN + 8 * w;
    const int number = __builtin_amdgcn_readlane(win.number, at);
    const bool there = win.there >> at & 1;
    const uint64_t from = (uint64_t)(unsigned)(there ? number : 0) * p.page_bytes + head + (unsigned)((key0 & ((1 << p.page_log2) - 1)) * ROWB);
    const unsigned char *kf = static_cast<const unsigned char*>(p.k_pages) + from, *vf = static_cast<const unsigned char*>(p.v_pages) + from;
    const unsigned slot = lds0 + (unsigned)((t % NS) * 2 * TILEB + 8 * w * ROWB);
    if (__builtin_expect(t * BN + BN <= wk.sq.len && (win.there >> (2 * (t & 31)) & 3) == 3, 1)) {
#pragma unroll
      for (int i = 0; i < SLABS; ++i) {
        dma16(kf, k_off[i], slot + i * 1024);
        dma16(vf, v_off + i * 1024, slot + TILEB + i * 1024);
      }
      return true;
    }
    const int n = there ? wk.sq.len - key0 : 0;  // rows that are not there become zeros
#pragma unroll
    for (int i = 0; i < SLABS; ++i) {
      if (i * RPS + l / CH < n) {
        dma16(kf, k_off[i], slot + i * 1024);
        dma16(vf, v_off + i * 1024, slot + TILEB + i * 1024);
      } else {
        *LDS_PTR(floatx4, slot + (unsigned)(i * 1024 + l * 16)) = floatx4{0.f, 0.f, 0.f, 0.f};
        *LDS_PTR(floatx4, slot + (unsigned)(TILEB + i * 1024 + l * 16)) = floatx4{0.f, 0.f, 0.f, 0.f};
      }
    }
    return false;
  };

  const unsigned krow = lds0 + (unsigned)(c32 * ROWB), vrow = lds0 + (unsigned)(TILEB + 4 * h * ROWB + c32 * (JT * 4));
  floatx16 o[JT];
  float m_run, l_run;
  constexpr floatx16 zero = {};

  auto attend = [&](int t, uint64_t gone, bool careful) __attribute__((always_inline)) {
    const unsigned slot = (unsigned)((t % NS) * 2 * TILEB);
    floatx16 s = zero;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const floatx4 k = *LDS_PTR(const floatx4, krow + slot + (unsigned)(((2 * j + h) ^ (c32 % 16)) * 16));
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[j][e], s, 0, 0, 0);
    }
    const int key0 = t * BN, rel = my_vis - key0 - 4 * h;
    if (key0 + BN > vis_first || gone) {  // wave-uniform
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) >= rel || (gone >> (i >> 3) & 1)) s[i] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx) * p.scale_log2e;
    const bool mine = mx > m_run + kStale || (m_run == -INFINITY && mx > -INFINITY);
    if (__any(mine)) {
      const float m2 = mine ? mx : m_run;
      const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m2);
      m_run = m2;
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2e, -ref));
      l_run += s[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      vvec v = *LDS_PTR(const vvec, vrow + slot + (unsigned)((8 * (i >> 2) + (i & 3)) * ROWB));
      if (__builtin_expect(!careful, 1)) {
#pragma unroll
        for (int j = 0; j < JT; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[j], s[i], o[j], 0, 0, 0);
      } else {
        // (values that are not finite, of keys that some rows do not see: rows that see the first of the two keys alone take the other's as zeros, rows that
        // see neither take nothing)
        const int sees = my_vis - key0 - (8 * (i >> 2) + (i & 3));
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          const floatx16 both = __builtin_amdgcn_mfma_f32_32x32x2f32(v[j], s[i], zero, 0, 0, 0);
          const floatx16 one = __builtin_amdgcn_mfma_f32_32x32x2f32(h ? 0.f : v[j], s[i], zero, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[j][e] += sees > 4 ? both[e] : sees > 0 ? one[e] : 0.f;
        }
      }
    }
  };

  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int j = 0; j < KS; ++j) asm volatile("" : "+v"(qf[j]));  // (waited for here, not in the loop)
#pragma unroll 1
  for (bool careful = false;; careful = true) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int j = 0; j < JT; ++j) o[j] = zero;
    issue(t_begin);
    uint64_t gone = ~win.there >> (2 * (t_begin & 31)) & 3;
    bool ahead = issue(t_begin + 1);
#pragma unroll 1
    for (int t = t_begin; t < t_end; ++t) {
      const uint64_t gone_next = ~win.there >> (2 * ((t + 1) & 31)) & 3;
      if (ahead)
        wait_vm<2 * SLABS>();
      else
        wait_vm<0>();
      barrier();
      ahead = issue(t + 2);
      if (t * BN < vis_last) attend(t, gone, careful);
      gone = gone_next;
    }
    bool odd = false;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= !(__builtin_fabsf(o[j][i]) < INFINITY);
    wait_vm<0>();
    barrier();
    if (careful) break;
    const int mine = __any(odd) ? 1 : 0;
    if (l == 0) *LDS_PTR(int, lds0 + 4 * w) = mine;
    barrier();
    int again = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) again |= *LDS_PTR(const int, lds0 + 4 * i);
    barrier();
    if (!__builtin_amdgcn_readfirstlane(again)) break;
  }

  const float l_tot = pair_sum(l_run);
  const int r = unit0 + c32;
  if (r >= wk.rows) return;
  const int t = (int)quot((unsigned)r, p.by_group), head_q = wk.g * G + r - t * G;
  const int64_t at = (int64_t)(wk.sq.first + t) * Hq + head_q, part = (int64_t)wk.piece * p.n_tokens * Hq + at;
  const bool alone = wk.n_pieces == 1;
  const float inv = !alone ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
  float* out = (alone ? static_cast<float*>(p.out) + at * D : p.part_o + part * D) + 4 * h * JT;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    vvec v;
#pragma unroll
    for (int j = 0; j < JT; ++j) v[j] = alone && l_tot == 0.f ? 0.f : o[j][i] * inv;
    *reinterpret_cast<vvec*>(out + (8 * (i >> 2) + (i & 3)) * JT) = v;
  }
  if (h == 0) {
    if (!alone)
      *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{m_run, l_tot};
    else if (p.lse)
      p.lse[(int64_t)head_q * p.n_tokens + wk.sq.first + t] = l_tot == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
  }
}

template <int D>
static hipError_t prepare_one() {
  static bool done[64] = {};  // (idempotent; two threads at worst set it twice)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!done[dev]) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_prompt_f32_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, prompt_f32_lds<D>);
    if (e != hipSuccess) return e;
    done[dev] = true;
  }
  return hipSuccess;
}
hipError_t prepare_attn_prompt_f32(int head_dim) { return head_dim == 128 ? prepare_one<128>() : prepare_one<64>(); }

hipError_t launch_attn_prompt_f32(const PAttnParams& p, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)p.n_units * (unsigned)p.n_pieces * (unsigned)p.n_kv_heads), block(256);
  if (head_dim == 128)
    hipLaunchKernelGGL(attn_prompt_f32_kernel<128>, grid, block, prompt_f32_lds<128>, s, p);
  else
    hipLaunchKernelGGL(attn_prompt_f32_kernel<64>, grid, block, prompt_f32_lds<64>, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
