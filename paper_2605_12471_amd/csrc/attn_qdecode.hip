// Attention of at most 16 packed rows per KV head on a cache held in 8 bits: decoding, one token or a few at a time.  A workgroup owns the KV
// head's rows and a piece of its blocks, dealt to four wavefronts in turn.
//
// Bound by memory when the cache is long, half the bytes of the bf16 cache, and by the chain of what a launch does once when it is short.  The
// codes come straight into registers, 16 bytes a lane and instruction (the layout is made for that, qcache.h), a block ahead, and are
// widened to bf16 there, which holds them exactly: three instructions a pair, 384 a block of 16 KB and wavefront, a third of the time that memory
// takes for it.  On the 16x16x32 shapes, S^T = K Q^T has 16 keys as its rows, O^T = V^T P^T 16 columns.
//
// The scales cost nothing per logit.  With s the product of the query as handed in and the codes, a weight of a block with scales k and v is
//     P' = 2^(s (k scale log2 e) - (m - log2 v)),
// its share of O the codes times P', rounded to bf16 for the matrix instruction as in the other kernels, and its share of the row sum P' / v,
// whose factor is taken out of the block's sum.  So neither the queries nor the keys are rounded on the way.  Where v is so small that P' leaves fp32's
// range (zero rows are held with 2^-100), the row sum's share is summed up from weights without it, a second exponential a logit (three
// quarters of the values zero: 128K keys 45.8 us for 45.5).  m is the row's maximum, stale by at most 2^16, or above it where v is
// so large that O would leave the range (an infinity among the values is held as the largest number, v = 2^121); O, m and l are fp32.
//
// A step whose rows fill no block is one launch: the wavefront that has the incomplete block writes the new rows into it, waits for its own stores and
// reads them back; nobody else reads them.  (The append as a launch in front takes 4.7 us.)  One token, 32 heads on 8, 128 wide, captured steps: 300
// keys 6.7 us, 4187 7.6, 16K 11.1, 128K 46 (268 MB of codes, 5.8 TB/s).
#include "meet.h"
#include "qcache.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kWaves = 4;

template <int D>
__global__ void __launch_bounds__(kWaves * 64, 2) attn_qdecode_kernel(QAttnParams qp) {
  const AttnParams& p = qp.a;
  constexpr int NW = kWaves, NT = NW * 64;
  constexpr int H = D / 64;           // pieces of a lane's share of a K row, each two contraction steps
  constexpr int J = D / 16;           // tiles of O^T
  constexpr int BLOCK = kQBlock * D;  // codes of a block
  constexpr float kStale = 16.0f;     // log2 units
  constexpr int ROWS = 16, OROW = D * 4 + 16;
  __shared__ __attribute__((aligned(16))) unsigned char red_o[NW * ROWS * OROW];
  __shared__ floatx2 red_ml[NW * ROWS];
  __shared__ int last;

  const int lid = logical_workgroup(blockIdx.x, gridDim.x, p);
  if (lid >= p.n_wgs) return;
  const int g = (int)quot((unsigned)lid, p.by_wgs_per_kvh);
  const int split = lid - g * p.n_splits;

  const int tid = threadIdx.x, l = tid & 63, kg = l >> 4, c16 = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int C = p.n_tokens, Hq = p.n_q_heads, G = p.group;
  const int rows = C * G;

  // ---- Q: lane (c16, kg) holds columns 64 h + 16 kg .. + 15 of row c16
  const int row = c16 < rows ? c16 : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
  const int my_vis = (int)p.len_prev + tok + 1;
  qbf16x8 qf[2 * H];
  {
    const __bf16* qrow = reinterpret_cast<const __bf16*>(p.q) + (uint64_t)(unsigned)(row + tok * (Hq - G) + g * G) * D;
    const float* cs = p.rope_cos ? p.rope_cos + tok * (D / 2) : nullptr;
    const float* sn = p.rope_cos ? p.rope_sin + tok * (D / 2) : nullptr;
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) qf[i] = q_query<D>(qrow, 64 * (i >> 1) + 16 * kg + 8 * (i & 1), cs, sn);
  }

  const int vis_first = (int)p.len_prev + 1, len = (int)p.len_prev + C;
  const int n_whole = len / kQBlock, n_all = (len + kQBlock - 1) / kQBlock;
  const int b_begin = split * p.tiles_per_split;
  int b_end = b_begin + p.tiles_per_split;
  if (b_end > n_all) b_end = n_all;
  const int b_codes = b_end < n_whole ? b_end : n_whole;  // blocks before it are held as codes

  const unsigned char* kcodes = qp.c.codes[0] + (uint64_t)g * (uint64_t)qp.c.blocks * BLOCK;
  const unsigned char* vcodes = qp.c.codes[1] + (uint64_t)g * (uint64_t)qp.c.blocks * BLOCK;
  const float* scales = qp.c.scales + 2 * (uint64_t)g * (uint64_t)qp.c.blocks;

  // Rows of S^T's tile t are keys 32 (r / 8) + 4 (r / 4 % 2) + 8 t + r % 4, of which a lane's four are those of its group (qcache.h)
  const int key_row = 32 * (c16 >> 3) + 4 * (c16 >> 2 & 1) + (c16 & 3), key_mine = 32 * (kg >> 1) + 4 * (kg & 1);
  const unsigned k_lane = (unsigned)q_k_piece(kg, key_row) * 16, v_lane = (unsigned)q_v_piece(D, kg, c16) * 16;

  // Blocks come by buffer loads: a lane's place in a block is fixed, the block's is a scalar, and a block that does not exist (past the last) is asked for in
  // an empty buffer, which costs no traffic, so that the loads in flight are the same on every path and the compiler can count them.
  struct Codes {
    quintx4 k[4][H], v[J];
    floatx2 scale;
  };
  const unsigned head_bytes = (unsigned)qp.c.blocks * (unsigned)BLOCK;  // (at most 2^31: half of what the rows may take in bf16)
  auto load = [&](Codes& x, int b, bool there) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(kcodes), 0, there ? head_bytes : 0u, kRawBuffer);
    const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(vcodes), 0, there ? head_bytes : 0u, kRawBuffer);
    const __amdgpu_buffer_rsrc_t sb = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(scales), 0, there ? (unsigned)qp.c.blocks * 8u : 0u, kRawBuffer);
    const unsigned at = (unsigned)b * (unsigned)BLOCK;
    x.scale = __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(sb, 0, (unsigned)b * 8u, 0));
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < H; ++h)
        x.k[t][h] = __builtin_bit_cast(quintx4, __builtin_amdgcn_raw_buffer_load_b128(kb, k_lane + (unsigned)(q_k_piece(4 * h, 8 * t) * 16), at, 0));
#pragma unroll
    for (int j = 0; j < J; ++j) x.v[j] = __builtin_bit_cast(quintx4, __builtin_amdgcn_raw_buffer_load_b128(vb, v_lane + (unsigned)(q_v_piece(D, 0, 16 * j) * 16), at, 0));
  };

  floatx4 o[J];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};

  // P' of a block from its S^T, masked
  auto weights = [&](floatx4 (&s)[4], int b, float k_scale, float v_scale, qbf16x8 (&pf)[2]) __attribute__((always_inline)) {
    const int key0 = b * kQBlock;
    if (key0 + kQBlock > vis_first) {  // wave-uniform: some row does not see the whole block
      const int rel = my_vis - key0 - key_mine;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (8 * t + e >= rel) s[t][e] = -INFINITY;
    }
    const float to_log2 = q_to_log2(k_scale, p.scale_log2e);
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t) mx = fmaxf(mx, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
    mx = pair_max(row16_max(mx));
    mx = __builtin_fmaf(mx, to_log2, q_above(v_scale));
    // only rows that ask for it move, so a row's arithmetic never depends on its wave neighbours
    const bool mine = mx > m_run + kStale || (m_run == -INFINITY && mx > -INFINITY);
    if (__any(mine)) {
      const float m2 = mine ? mx : m_run;
      const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m2);  // (without history: l = 0, O = 0)
      m_run = m2;
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][r] *= alpha;
    }
    const float ref = (m_run == -INFINITY ? 0.f : m_run) - __builtin_amdgcn_logf(v_scale);
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], to_log2, -ref));
        sum += a;
        pf[t >> 1][4 * (t & 1) + e] = (__bf16)a;
      }
    if (__builtin_expect(q_tiny(v_scale), 0)) {
      sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], to_log2, m_run == -INFINITY ? 0.f : -m_run));
      l_run += sum;
    } else {
      l_run = __builtin_fmaf(sum, __builtin_amdgcn_rcpf(v_scale), l_run);
    }
  };
  auto block = [&](const Codes& x, int b) __attribute__((always_inline)) {
    floatx4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        qbf16x8 lo, up;
        q_widen(x.k[t][h], lo, up);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, qf[2 * h], s[t], 0, 0, 0);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(up, qf[2 * h + 1], s[t], 0, 0, 0);
      }
    qbf16x8 pf[2];
    weights(s, b, x.scale.x, x.scale.y, pf);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      qbf16x8 lo, up;
      q_widen(x.v[j], lo, up);
      o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, pf[0], o[j], 0, 0, 0);
      o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(up, pf[1], o[j], 0, 0, 0);
    }
  };

  // ---- the wavefront's blocks, every NW-th of the piece's, two in flight: in cyclic order from a place that differs from piece to piece and head to
  // head, as pieces and heads lie powers of two apart, and workgroups in step would ask the same few memory channels for their rows
  const int b_first = b_begin + w, n = b_first < b_codes ? (int)((unsigned)(b_codes - b_first + NW - 1) / (unsigned)NW) : 0, b_rest = b_first + NW * n;
  auto next = [&](int b) __attribute__((always_inline)) -> int { return b + NW < b_rest ? b + NW : b_first; };
  Codes x, y;
  int b = b_first + NW * (int)(((((unsigned)(split * 8 + g) * 40503u) & 0xffffu) * (unsigned)n) >> 16), left = n;
  if (n > 0) load(x, b, true);

  // ---- The rows that are not a whole block, in bf16, are the wavefront's whose turn it is, the only one to read them: it also appends the new ones
  if (b_rest == n_whole && n_whole < b_end) {
    const int b = n_whole, n = len - b * kQBlock;
    const uint64_t slot = ((uint64_t)g * kQRing + (unsigned)b % kQRing) * BLOCK;
    if (qp.k_new) q_fill_block<D>(qp, g, slot, n, l, 64);
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(qp.c.ring[0] + slot) + 2 * k_lane;
    const unsigned char* vb = reinterpret_cast<const unsigned char*>(qp.c.ring[1] + slot) + 2 * v_lane;
    floatx4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const qbf16x8* at = reinterpret_cast<const qbf16x8*>(kb + (unsigned)(q_k_piece(4 * h, 8 * t) * 32));
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(at[0], qf[2 * h], s[t], 0, 0, 0);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(at[1], qf[2 * h + 1], s[t], 0, 0, 0);
      }
    }
    qbf16x8 pf[2];
    weights(s, b, 1.f, 1.f, pf);
    auto outputs = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const qbf16x8* at = reinterpret_cast<const qbf16x8*>(vb + (unsigned)(q_v_piece(D, 0, 16 * j) * 32));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          qbf16x8 v = at[u];
#pragma unroll
          for (int e = 0; e < 8; ++e)  // (places without a row hold anything: 0 times it has to be 0)
            if (key_mine + 16 * u + 8 * (e >> 2) + (e & 3) >= n) v[e] = (__bf16)0.f;
          o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[u], o[j], 0, 0, 0);
        }
      }
    };
    outputs();
    if (__builtin_expect(__any(q_large<4>(o)), 0)) {  // (the wavefront's first results, from weights of at most 1)
#pragma unroll
      for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = (__bf16)((float)pf[e >> 3][e & 7] * kQLower);
#pragma unroll
      for (int j = 0; j < J; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};
      outputs();
      m_run += kQAboveRows;
      l_run *= kQLower;
    }
  }

  if (n > 0) {
#pragma unroll 1
    while (true) {
      const int b1 = next(b), b2 = next(b1);
      load(y, b1, left > 1);
      asm volatile("" ::: "memory");
      block(x, b);
      if (--left == 0) break;
      load(x, b2, left > 1);
      asm volatile("" ::: "memory");
      block(y, b1);
      if (--left == 0) break;
      b = b2;
    }
  }
  // ---- the wavefronts' results meet in LDS: [wavefront][row][D] and [wavefront][row] (m, l)
  const float l_tot = pair_sum(row16_sum(l_run));
  if (c16 < rows) {
#pragma unroll
    for (int j = 0; j < J; ++j) *reinterpret_cast<floatx4*>(red_o + (w * ROWS + c16) * OROW + (16 * j + 4 * kg) * 4) = o[j];
    if (kg == 0) red_ml[w * ROWS + c16] = floatx2{m_run, l_tot};
  }
  __syncthreads();

  constexpr int V = D / 4;  // 16-byte column vectors of a row
  const int c = tid % V;
  const int64_t n_rows = (int64_t)C * Hq;
  const Partials<D> parts(p);
#pragma unroll 1
  for (int r = tid / V; r < rows; r += NT / V) {
    floatx2 ml[NW];
    float M = -INFINITY;
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) {
      ml[ww] = red_ml[ww * ROWS + r];
      M = fmaxf(M, ml[ww].x);
    }
    float L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) {
      const floatx4 x = *reinterpret_cast<const floatx4*>(red_o + (ww * ROWS + r) * OROW + c * 16);
      const float f = ml[ww].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[ww].x - M);  // (0: it saw no visible key)
      L += f * ml[ww].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += f * x[e];
    }
    const int t = (int)quot((unsigned)r, p.by_group), h = g * G + r - t * G;
    const int64_t at = (int64_t)t * Hq + h;
    if (p.n_splits == 1) {
      const float inv = 1.f / L;
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[e] * inv);
      *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(p.out) + at * D + c * 4) = v;
      if (p.lse && c == 0) p.lse[(int64_t)h * C + t] = (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
    } else if (p.meet_count) {
      parts.store(split, (unsigned)at, c, acc, M, L);
    } else {
      *reinterpret_cast<floatx4*>(p.part_o + ((int64_t)split * n_rows + at) * D + c * 4) = acc;
      if (c == 0) *reinterpret_cast<float2*>(p.part_ml + ((int64_t)split * n_rows + at) * 2) = make_float2(M, L);
    }
  }
  if (!p.meet_count || !last_to_meet(p, g, &last)) return;
  // the last of the head's pieces merges them, a row or two per wavefront
  const int cv = l % V, part = l / V;
  constexpr int N = kMeetSplits * V / 64;
#pragma unroll 1
  for (int r = w; r < rows; r += NW) {
    const int t = (int)quot((unsigned)r, p.by_group), h = g * G + r - t * G;
    const unsigned at[1] = {(unsigned)(t * Hq + h)};
    floatx4 acc[1];
    float M[1], L[1];
    parts.template merge<N, 1>(at, part, cv, acc, M, L);
    if (part != 0) continue;
    const float inv = 1.f / L[0];
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[0][e] * inv);
    *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(p.out) + (int64_t)at[0] * D + cv * 4) = v;
    if (p.lse && cv == 0) p.lse[(int64_t)h * C + t] = (M[0] + __builtin_amdgcn_logf(L[0])) * 0.6931471805599453f;
  }
}

hipError_t launch_attn_qdecode(const QAttnParams& p, int head_dim, hipStream_t s) {
  const dim3 grid(padded_grid(p.a.n_wgs)), block(kWaves * 64);
  if (head_dim == 128)
    hipLaunchKernelGGL(attn_qdecode_kernel<128>, grid, block, 0, s, p);
  else
    hipLaunchKernelGGL(attn_qdecode_kernel<64>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
