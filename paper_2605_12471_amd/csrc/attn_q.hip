// Chunk-prefix attention on a cache held in 8 bits, any number of rows.  A work unit is 32 consecutive packed (token, head of the group) rows
// of a KV head, a wavefront owns U of them, a workgroup four wavefronts of one KV head and a piece of its blocks.
//
// Bound by the matrix instructions where rows are many.  A block of 64 keys is brought in as codes, half the bytes of bf16, a block
// ahead, 64 bytes a thread (32 where heads are 64 wide); each thread widens its own to bf16, which holds them exactly, and puts them into LDS in the
// order of the matrix instructions' operands, so that they are widened once for the workgroup's 128 U rows and every LDS access
// is 16 bytes a lane, neighbours side by side.  V needs no transpose on the way: the layout (qcache.h) has its keys side by side.  Two
// buffers, one barrier a block.
//
// S^T = K Q^T and O^T = V^T P^T on the 32x32x16 shapes: a lane holds 32 logits of one query, whose weights are its operand of the second product
// as they stand.  Scales, rounding points and the stale maximum as in the decoding kernel (attn_qdecode.hip).
#include "qcache.h"
#include "wave_ops.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((ext_vector_type(16))) float floatx16;

template <int D, int U>
__global__ void __launch_bounds__(256, U == 1 ? 2 : 1) attn_q_kernel(QAttnParams qp) {
  const AttnParams& p = qp.a;
  constexpr int KS = D / 16, JT = D / 32;    // contraction steps of S^T, tiles of O^T
  constexpr int BLOCK = kQBlock * D;         // codes of a block
  constexpr int T = BLOCK / 16 / 256;        // pieces of K, and of V, per thread
  constexpr int KLDS = BLOCK * 2, BUF = 2 * KLDS;
  constexpr float kStale = 16.0f;            // log2 units
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * BUF];

  const int lid = logical_workgroup(blockIdx.x, gridDim.x, p);
  if (lid >= p.n_wgs) return;
  const int g = (int)quot((unsigned)lid, p.by_wgs_per_kvh);
  const int in_head = lid - g * p.wgs_per_head * p.n_splits;
  const int split = (int)quot((unsigned)in_head, p.by_wgs_per_head);
  const int wg = p.wgs_per_head - 1 - (in_head - split * p.wgs_per_head);  // heaviest first

  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int C = p.n_tokens, Hq = p.n_q_heads, G = p.group, rows = C * G;
  const int len = (int)p.len_prev + C, n_whole = len / kQBlock;

  // ---- the wavefront's rows
  const int unit0 = (wg * 4 + w) * U;
  int tok[U], row[U];
  qbf16x8 qf[U][KS];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = (unit0 + u) * kRowsPerUnit + c32;
    row[u] = r < rows ? r : rows - 1;
    tok[u] = (int)quot((unsigned)row[u], p.by_group);
    const __bf16* qrow = reinterpret_cast<const __bf16*>(p.q) + (uint64_t)(unsigned)(row[u] + tok[u] * (Hq - G) + g * G) * D;
    const float* cs = p.rope_cos ? p.rope_cos + (int64_t)tok[u] * (D / 2) : nullptr;
    const float* sn = p.rope_cos ? p.rope_sin + (int64_t)tok[u] * (D / 2) : nullptr;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[u][ks] = q_query<D>(qrow, 16 * ks + 8 * h, cs, sn);
  }
  // Keys that the wavefront's first row sees, and its last one; that the workgroup's last row sees
  auto seen_by = [&](int r) __attribute__((always_inline)) -> int {
    r = r < rows ? r : rows - 1;
    return (int)p.len_prev + (int)quot((unsigned)r, p.by_group) + 1;
  };
  const bool live = unit0 * kRowsPerUnit < rows;
  const int vis_first = seen_by(unit0 * kRowsPerUnit), vis_last = live ? seen_by((unit0 + U) * kRowsPerUnit - 1) : 0;
  const int vis_wg = seen_by((wg * 4 + 4) * U * kRowsPerUnit - 1);
  const int b_begin = split * p.tiles_per_split;
  int b_end = b_begin + p.tiles_per_split;
  const int b_seen = (vis_wg + kQBlock - 1) / kQBlock;
  if (b_end > b_seen) b_end = b_seen;

  const unsigned char* codes[2];
  codes[0] = qp.c.codes[0] + (uint64_t)g * (uint64_t)qp.c.blocks * BLOCK;
  codes[1] = qp.c.codes[1] + (uint64_t)g * (uint64_t)qp.c.blocks * BLOCK;
  const float* scales = qp.c.scales + 2 * (uint64_t)g * (uint64_t)qp.c.blocks;

  // ---- a block on its way: K fragment (tile t, step, half) at ((t KS + step) 2 + half) 512, V's (tile t, step, tile of O^T, half) behind them
  quintx4 raw[2][T];
  auto load = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int j = 0; j < T; ++j) raw[v][j] = *reinterpret_cast<const quintx4*>(codes[v] + (uint64_t)(unsigned)b * BLOCK + (unsigned)(tid + 256 * j) * 16);
  };
  auto put = [&](unsigned char* buf, int v, int piece, const qbf16x8& lo, const qbf16x8& up) __attribute__((always_inline)) {
    unsigned char* at;
    int next;
    if (v == 0) {
      const int c = piece >> 6, key = piece & 63;
      at = buf + (((key >> 5) * KS + c) * 2 * 32 + (key & 31)) * 16;
      next = 32 * 16;  // the other half
    } else {
      const int kg = piece / D, col = piece % D;
      at = buf + KLDS + ((((kg >> 1) * 2 * JT + (col >> 5)) * 2 + (kg & 1)) * 32 + (col & 31)) * 16;
      next = JT * 2 * 32 * 16;  // the other step
    }
    *reinterpret_cast<qbf16x8*>(at) = lo;
    *reinterpret_cast<qbf16x8*>(at + next) = up;
  };
  auto store = [&](unsigned char* buf) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int j = 0; j < T; ++j) {
        qbf16x8 lo, up;
        q_widen(raw[v][j], lo, up);
        put(buf, v, tid + 256 * j, lo, up);
      }
  };
  // The rows that are not a whole block yet, in bf16; places without a row hold anything, in V they become 0 (0 times it has to be 0)
  auto store_rest = [&](unsigned char* buf, int b) __attribute__((always_inline)) {
    const int n = len - b * kQBlock;
    const uint64_t slot = ((uint64_t)g * kQRing + (unsigned)b % kQRing) * BLOCK;
#pragma unroll 1
    for (int j = 0; j < T; ++j) {
      const int piece = tid + 256 * j, kg = piece / D;
      const qbf16x8* k = reinterpret_cast<const qbf16x8*>(qp.c.ring[0] + slot + piece * 16);
      const qbf16x8* v = reinterpret_cast<const qbf16x8*>(qp.c.ring[1] + slot + piece * 16);
      put(buf, 0, piece, k[0], k[1]);
      qbf16x8 x[2] = {v[0], v[1]};
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (32 * (kg >> 1) + 4 * (kg & 1) + 8 * (e >> 2) + (e & 3) >= n) x[e >> 3][e & 7] = (__bf16)0.f;
      put(buf, 1, piece, x[0], x[1]);
    }
  };

  floatx16 o[U][JT];
  float m_run[U], l_run[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    m_run[u] = -INFINITY;
    l_run[u] = 0.f;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[u][j][i] = 0.f;
  }

  auto attend = [&](const unsigned char* buf, int b, float k_scale, float v_scale) __attribute__((always_inline)) {
    floatx16 s[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][t][i] = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const qbf16x8 k = *reinterpret_cast<const qbf16x8*>(buf + ((t * KS + ks) * 64 + l) * 16);
#pragma unroll
        for (int u = 0; u < U; ++u) s[u][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[u][ks], s[u][t], 0, 0, 0);
      }
    const int key0 = b * kQBlock;
    if (key0 + kQBlock > vis_first) {  // wave-uniform: some row does not see the whole block
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int rel = (int)p.len_prev + tok[u] + 1 - key0 - 4 * h;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * t + 8 * (i >> 2) + (i & 3) >= rel) s[u][t][i] = -INFINITY;
      }
    }
    const float to_log2 = q_to_log2(k_scale, p.scale_log2e);
    float mx[U];
    bool mine[U], any = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      mx[u] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx[u] = fmaxf(mx[u], s[u][t][i]);
      mx[u] = pair_max(mx[u]);
      mx[u] *= to_log2;
      mine[u] = mx[u] > m_run[u] + kStale || (m_run[u] == -INFINITY && mx[u] > -INFINITY);
      any |= mine[u];
    }
    if (__any(any)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float m2 = mine[u] ? mx[u] : m_run[u];
        const float alpha = m_run[u] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[u] - m2);
        m_run[u] = m2;
        l_run[u] *= alpha;
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[u][j][i] *= alpha;
      }
    }
    qbf16x8 pf[U][2][2];
    const float log2_v = __builtin_amdgcn_logf(v_scale), inv_v = __builtin_amdgcn_rcpf(v_scale);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float ref = (m_run[u] == -INFINITY ? 0.f : m_run[u]) - log2_v;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][t][i], to_log2, -ref));
          sum += a;
          pf[u][t][i >> 3][i & 7] = (__bf16)a;
        }
      l_run[u] = __builtin_fmaf(sum, inv_v, l_run[u]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          const qbf16x8 v = *reinterpret_cast<const qbf16x8*>(buf + KLDS + (((t * 2 + st) * JT + j) * 64 + l) * 16);
#pragma unroll
          for (int u = 0; u < U; ++u) o[u][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[u][t][st], o[u][j], 0, 0, 0);
        }
  };

  if (b_begin < b_end) {
    int at = 0;
    floatx2 scale = {1.f, 1.f}, next = {1.f, 1.f};
    if (b_begin < n_whole) {
      load(b_begin);
      scale = *reinterpret_cast<const floatx2*>(scales + 2 * (unsigned)b_begin);
      store(lds);
    } else {
      store_rest(lds, b_begin);
    }
    __syncthreads();
#pragma unroll 1
    for (int b = b_begin; b < b_end; ++b) {
      const bool more = b + 1 < b_end, more_codes = more && b + 1 < n_whole;
      if (more_codes) {
        load(b + 1);
        next = *reinterpret_cast<const floatx2*>(scales + 2 * (unsigned)(b + 1));
      }
      if (b * kQBlock < vis_last) attend(lds + at, b, scale.x, scale.y);
      if (more_codes) {
        store(lds + (at ^ BUF));
        scale = next;
      } else if (more) {
        store_rest(lds + (at ^ BUF), b + 1);
        scale = floatx2{1.f, 1.f};
      }
      at ^= BUF;
      __syncthreads();
    }
  }

  // ---- out, or what the piece leaves for the merge
  const int64_t n_rows = (int64_t)C * Hq;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float l_tot = pair_sum(l_run[u]);
    if ((unit0 + u) * kRowsPerUnit + c32 >= rows) continue;
    const int head = g * G + row[u] - tok[u] * G;
    const int64_t at = (int64_t)tok[u] * Hq + head;
    if (p.n_splits == 1) {
      const float inv = 1.f / l_tot;
      __bf16* out = reinterpret_cast<__bf16*>(p.out) + at * D + 4 * h;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[u][j][i + e] * inv);
          *reinterpret_cast<bf16x4*>(out + 32 * j + 2 * i) = v;
        }
      if (p.lse && h == 0) p.lse[(int64_t)head * C + tok[u]] = (m_run[u] + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
    } else {
      float* out = p.part_o + ((int64_t)split * n_rows + at) * D + 4 * h;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<floatx4*>(out + 32 * j + 2 * i) = floatx4{o[u][j][i], o[u][j][i + 1], o[u][j][i + 2], o[u][j][i + 3]};
      if (h == 0) *reinterpret_cast<floatx2*>(p.part_ml + ((int64_t)split * n_rows + at) * 2) = floatx2{m_run[u], l_tot};
    }
  }
}

hipError_t launch_attn_q(const QAttnParams& p, int head_dim, int units_per_wave, hipStream_t s) {
  const dim3 grid(padded_grid(p.a.n_wgs)), block(256);
  if (head_dim == 128 && units_per_wave == 2)
    hipLaunchKernelGGL((attn_q_kernel<128, 2>), grid, block, 0, s, p);
  else if (head_dim == 128)
    hipLaunchKernelGGL((attn_q_kernel<128, 1>), grid, block, 0, s, p);
  else if (units_per_wave == 2)
    hipLaunchKernelGGL((attn_q_kernel<64, 2>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attn_q_kernel<64, 1>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
