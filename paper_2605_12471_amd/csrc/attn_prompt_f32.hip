// Attention of whole prompts, and of chunks of them, of many sequences on a cache in pages, fp32: attn_prompt.hip's shape with one unit a wavefront and tiles of
// 32 keys, on the fp32 matrix instructions.
//
// Bound by these: 32x32x2, 4 kFLOP in 64 cycles (3000 tokens, 32 heads on 8, 128 wide: 666 us, 111 TFLOP/s; six prompts of 47 to 725, 8 heads on 2, 64 wide: 20 us, two tiles a CU).  S^T = K Q^T: a lane has 16 bytes of a K row and of its query's, four contraction steps whose columns are
// whichever these are.  O^T = V^T P^T: step i's two keys are those whose logits the two lanes of a row hold in register i, and a lane's 16 (64 wide: 8)
// bytes of such a V row are its columns of all tiles of O^T (tile j has every fourth, or second, column of the head), so that V needs no transpose.
#include "prompt.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kF32Ring = 2, kF32Tile = 32;
template <int D>
constexpr int prompt_f32_lds = kF32Ring * 2 * kF32Tile * D * 4;

template <int D>
__global__ void __launch_bounds__(256, 2) attn_prompt_f32_kernel(PAttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned lds0 = (unsigned)(uintptr_t)((unsigned char __attribute__((address_space(3)))*)smem);
  constexpr int CH = D / 4, ROWB = D * 4, KS = D / 8, JT = D / 32;  // 16-byte chunks and bytes of a row; 16-byte shares of a lane; tiles of O^T
  constexpr int BN = kF32Tile, TILEB = BN * ROWB, NS = kF32Ring;
  constexpr int RPS = 64 / CH, SLABS = 8 / RPS;  // rows of a 1 KiB copy; copies of a wavefront's 8 rows
  constexpr float kStale = 16.0f;
  typedef __attribute__((ext_vector_type(JT))) float vvec;

  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PromptWork wk = prompt_work(p, blockIdx.x);
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
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= t_end) return;
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
      return;
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
  };

  const unsigned krow = lds0 + (unsigned)(c32 * ROWB), vrow = lds0 + (unsigned)(TILEB + 4 * h * ROWB + c32 * (JT * 4));
  constexpr floatx16 zero = {};
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A tile's S^T, masked; then the reference of a row, and what a row's results are to be multiplied by (1 but for a wavefront that moves one); then weights, and their sum
  auto logits = [&](int t) __attribute__((always_inline)) -> floatx16 {
    const unsigned slot = (unsigned)((t % NS) * 2 * TILEB);
    const uint64_t gone = ~win.there >> (2 * (t & 31)) & 3;  // of the tile's two runs of 16 keys, those of no page
    issue(t + 1);
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
    return s;
  };
  auto reference = [&](const floatx16& s, float& m_run, float& alpha) __attribute__((always_inline)) -> bool {
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx) * p.scale_log2e;
    // only rows that ask for it move, so a row's arithmetic never depends on its wave neighbours
    const bool mine = mx > m_run + kStale || (m_run == -INFINITY && mx > -INFINITY);
    if (!__any(mine)) return false;
    const float m2 = mine ? mx : m_run;
    alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m2);
    m_run = m2;
    return true;
  };
  auto weights = [&](floatx16& s, float m_run) __attribute__((always_inline)) -> float {
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2e, -ref));
      sum += s[i];
    }
    return sum;
  };

#pragma unroll
  for (int j = 0; j < KS; ++j) asm volatile("" : "+v"(qf[j]));  // (waited for here, not in the loop)
  floatx16 o[JT];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int j = 0; j < JT; ++j) o[j] = zero;
  issue(t_begin);
#pragma unroll 1
  for (int t = t_begin; t < t_end; ++t) {
    wait_vm<0>();
    barrier();  // the tile is there for all, and the slot of the one before is free
    if (t * BN >= vis_last) {
      issue(t + 1);
      continue;
    }
    floatx16 s = logits(t);
    float alpha;
    if (reference(s, m_run, alpha)) {
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= alpha;
    }
    l_run += weights(s, m_run);
    const unsigned at = vrow + (unsigned)((t % NS) * 2 * TILEB);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const vvec v = *LDS_PTR(const vvec, at + (unsigned)((8 * (i >> 2) + (i & 3)) * ROWB));
#pragma unroll
      for (int j = 0; j < JT; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[j], s[i], o[j], 0, 0, 0);
    }
  }

  // ---- out, or what the piece leaves for the merge
  const int r = unit0 + c32;
  const bool alone = wk.n_pieces == 1;
  int64_t at = 0, part = 0;
  int head_q = 0, tok_out = 0;
  if (r < wk.rows) {
    tok_out = (int)quot((unsigned)r, p.by_group);
    head_q = wk.g * G + r - tok_out * G;
    at = (int64_t)(wk.sq.first + tok_out) * Hq + head_q;
    part = (int64_t)wk.piece * p.n_tokens * Hq + at;
  }
  auto sums = [&](float m, float l_tot) __attribute__((always_inline)) {
    if (h || r >= wk.rows) return;
    if (!alone)
      *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{m, l_tot};
    else if (p.lse)
      p.lse[(int64_t)head_q * p.n_tokens + wk.sq.first + tok_out] = l_tot == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
  };
  float* out = (alone ? static_cast<float*>(p.out) + at * D : p.part_o + part * D) + 4 * h * JT;
  float check = 0.f;  // 0 as long as all outputs are finite
  {
    const float l_tot = pair_sum(l_run), inv = !alone ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
    sums(m_run, l_tot);
    if (r < wk.rows) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        vvec v;
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          check = __builtin_fmaf(o[j][i], 0.f, check);
          v[j] = o[j][i] * inv;
        }
        *reinterpret_cast<vvec*>(out + (8 * (i >> 2) + (i & 3)) * JT) = v;
      }
    }
  }
  // Outputs that are not finite may come from values that their rows do not see (0 times them is not 0): everything once more, then, a tile of O^T at a time; of a
  // step's two keys, rows that see the first alone take the other's values as zeros, rows that see neither take nothing.
  wait_vm<0>();
  __syncthreads();
  const int vote = __any(check != 0.f) ? 1 : 0;  // (NaN)
  if (l == 0) *LDS_PTR(int, lds0 + 4 * w) = vote;
  __syncthreads();
  int again = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) again |= *LDS_PTR(const int, lds0 + 4 * i);
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(again) == 0, 1)) return;
#pragma unroll 1
  for (int j = 0; j < JT; ++j) {
    floatx16 acc = zero;
    float m = -INFINITY, total = 0.f;
    __syncthreads();
    issue(t_begin);
#pragma unroll 1
    for (int t = t_begin; t < t_end; ++t) {
      wait_vm<0>();
      barrier();
      floatx16 s = logits(t);
      float alpha;
      if (reference(s, m, alpha)) {
        total *= alpha;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] *= alpha;
      }
      total += weights(s, m);
      const unsigned from = vrow + (unsigned)((t % NS) * 2 * TILEB + j * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k0 = 8 * (i >> 2) + (i & 3), sees = my_vis - t * BN - k0;
        const float v = *LDS_PTR(const float, from + (unsigned)(k0 * ROWB));
        floatx16 x = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], zero, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] += sees > 4 ? x[e] : 0.f;
        x = __builtin_amdgcn_mfma_f32_32x32x2f32(h ? 0.f : v, s[i], zero, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] += sees > 0 && sees <= 4 ? x[e] : 0.f;
      }
    }
    const float l_tot = pair_sum(total), inv = !alone ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
    if (j == 0) sums(m, l_tot);
    if (r < wk.rows) {
#pragma unroll
      for (int i = 0; i < 16; ++i) out[(8 * (i >> 2) + (i & 3)) * JT + j] = acc[i] * inv;
    }
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
  const dim3 grid((unsigned)p.n_units * (unsigned)p.n_kv_heads), block(256);
  if (head_dim == 128)
    hipLaunchKernelGGL(attn_prompt_f32_kernel<128>, grid, block, prompt_f32_lds<128>, s, p);
  else
    hipLaunchKernelGGL(attn_prompt_f32_kernel<64>, grid, block, prompt_f32_lds<64>, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
