// The softmax weight that a chunk's queries gave to each cached key, summed over the rows and the query heads of the KV head's group:
//     w[g][j] = sum over rows (i, h) of the group with j <= len - n + i of 2^(s scale log2 e - lse[h][i] log2 e),   s = q . k_j.
// The step has left the log-sum-exps, so that one product is all there is: no maximum, no second pass, and every weight's sum belongs to one lane.
//
// S = Q K^T with the queries as the matrix instruction's rows: a lane holds the logits of one key, which it adds up without a word to other lanes
// until the end.  The keys stay in registers and the queries stream past, through LDS, units of 32 packed rows at a time, two buffers, one
// barrier.  What a logit's sum begins with is the row's -lse / (scale log2 e), so that a multiplication, an exponential and an addition are
// all that is left to do to it; the product's sums are rounded at that size for it, 5.8e-7 of a weight (2-norm; 9e-8 where it is added last).  Bound by
// issue: a 32x32x16 matrix instruction keeps its pipe busy for 32 cycles, 128 wide 16 a logit and lane, and the vector port for 16 of them; a logit's own
// instructions take it for 16 more, of which no more than half go beside matrix instructions, and of the 11 vector instructions beside each of these
// a third finds the rows (ten for a piece of a query, fourteen for a log-sum-exp).  256 tokens on 64K keys, 28 heads on 4, 158 us, 762 TFLOP/s: matrix
// pipes 0.33 busy, the vector port 0.72 of the time that a CU has work.  Two or three blocks of
// 32 keys a wavefront (fewer wavefronts a SIMD), queries two stages ahead, and a schedule written out gained nothing.
//
// Few rows (at most 16 a KV head) are bound by reading the keys: the wavefronts take 64 keys at a time straight into registers, on the 16x16x32
// shapes, whole 64-byte pieces of rows an instruction.
//
// A row whose log-sum-exp is -inf gave no weight to any key, whatever its query is: it sees no key.  (Many rows, bf16: its sums begin with -inf, which a
// query that is not finite makes NaN.  A wavefront with such a weight goes through its rows again, straight from memory, with zeros for these queries.)
#include "append_rows.h"
#include "qcache.h"
#include "wave_ops.h"
#include "weigh.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(16))) float floatx16;

// log2 units; rows that do not count, and those that gave no weight, get +inf: 2^(x - inf) = 0
__device__ __forceinline__ float lse_log2(const WeighParams& p, int g, int row, int rows) {
  if (row >= rows) return INFINITY;
  const int tok = (int)quot((unsigned)row, p.by_group), head = g * p.group + row - tok * p.group;
  const float x = p.lse[(int64_t)head * p.n_tokens + tok] * 1.4426950408889634f;
  return x == -INFINITY ? INFINITY : x;
}

__device__ __forceinline__ void give(const WeighParams& p, int g, int key, float w) {
  if (key >= p.len) return;
  float* at = p.weights + (int64_t)g * p.capacity + key;
  *at = p.add ? *at + w : w;
}

// Many rows, bf16.  A workgroup has 32 KW keys of one KV head, a wavefront 32 of them and, of the UB RW units that are in LDS at a time, every RW-th: RW
// wavefronts share keys where there are too few keys for the chip, and add up what they have in the end.
template <int D, int KW, int RW, int UB>
__global__ void __launch_bounds__(64 * KW * RW, 2) weigh_bf16_kernel(WeighParams p) {
  constexpr int KS = D / 16, CH = D / 8, NT = 64 * KW * RW, STAGE = RW * UB, T = STAGE * 32 * CH / NT, ROW = D * 2 + 16, UNIT = 32 * ROW;
  __shared__ __attribute__((aligned(16))) unsigned char q_lds[2 * STAGE * UNIT];
  __shared__ __attribute__((aligned(16))) float lse_lds[2 * STAGE * 32];
  static_assert(STAGE * 32 <= NT && T * NT == STAGE * 32 * CH, "a thread has the same share of every stage");
  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31, w = __builtin_amdgcn_readfirstlane(tid >> 6), kw = w % KW, rw = w / KW;
  const int g = blockIdx.y, rows = p.n_tokens * p.group, units = (rows + 31) / 32, prev = p.len - p.n_tokens;
  const int wg_key = blockIdx.x * (KW * 32), key0 = wg_key + kw * 32, key = key0 + c32;

  // ---- the keys: lane (key, h) holds columns 16 ks + 8 h .. + 7
  const __bf16* k_head = reinterpret_cast<const __bf16*>(p.k) + (int64_t)g * p.capacity * D;
  qbf16x8 kf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const qbf16x8*>(k_head + (int64_t)(key < p.len ? key : p.len - 1) * D + 16 * ks + 8 * h);

  // ---- a stage on its way: its rows, ROW bytes apart (no two of sixteen in the same banks), and what the logits' sums begin with
  qbf16x8 q_in[T];
  float lse_in = 0.f;
  const __bf16* q_all = reinterpret_cast<const __bf16*>(p.q) + (unsigned)(g * p.group * D);
  const float to_logit = 1.f / p.scale_log2e;
  auto load = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int i = tid + NT * j, r = i / CH, c = i % CH;
      int row = u * 32 + r;
      if (row >= rows) row = rows - 1;
      const int tok = (int)quot((unsigned)row, p.by_group);
      const __bf16* q_row = q_all + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group)) * D;
      q_in[j] = q_query<D>(q_row, 8 * c, p.rope_cos ? p.rope_cos + (int64_t)tok * (D / 2) : nullptr, p.rope_cos ? p.rope_sin + (int64_t)tok * (D / 2) : nullptr);
    }
    if (tid < STAGE * 32) lse_in = -lse_log2(p, g, u * 32 + tid, rows) * to_logit;
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int i = tid + NT * j, r = i / CH, c = i % CH;
      *reinterpret_cast<qbf16x8*>(q_lds + buf * STAGE * UNIT + r * ROW + c * 16) = q_in[j];
    }
    if (tid < STAGE * 32) lse_lds[buf * STAGE * 32 + tid] = lse_in;
  };

  // The first unit with a row that sees the workgroup's first key: row i of the chunk sees keys up to prev + i
  const int first_tok = wg_key > prev ? wg_key - prev : 0, u_begin = (int)((int64_t)first_tok * p.group / 32);
  float sum = 0.f;
  // S - lse of a unit, in units of the logits before their scale; -inf where a row does not see the key
  floatx16 s;
  auto logits = [&](int slot, floatx16& x) __attribute__((always_inline)) {
    floatx16 from;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const floatx4 m = *reinterpret_cast<const floatx4*>(lse_lds + slot * 32 + 2 * i + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) from[i + e] = m[e];
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const qbf16x8 q = *reinterpret_cast<const qbf16x8*>(q_lds + slot * UNIT + c32 * ROW + h * 16 + ks * 32);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, kf[ks], ks == 0 ? from : x, 0, 0, 0);
    }
  };
  auto mask = [&](int u) __attribute__((always_inline)) {
    if (prev + (int)quot((unsigned)(u * 32), p.by_group) < key0 + 31) {  // some row does not see all of the wavefront's keys
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (key > prev + (int)quot((unsigned)(u * 32 + 8 * (i >> 2) + 4 * h + (i & 3)), p.by_group)) s[i] = -INFINITY;
      }
    }
  };
  auto add_up = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(s[i] * p.scale_log2e);
  };
  // A unit's exponentials stand among the next one's matrix instructions
  load(u_begin);
  store(0);
  __syncthreads();
  int u_last = -1;
#pragma unroll 1
  for (int u0 = u_begin, buf = 0; u0 < units; u0 += STAGE, buf ^= 1) {
    const bool more = u0 + STAGE < units;
    if (more) load(u0 + STAGE);
#pragma unroll
    for (int i = 0; i < UB; ++i) {
      const int u = u0 + i * RW + rw;
      if (u >= units) continue;
      if (u_last < 0) {
        logits(buf * STAGE + i * RW + rw, s);
      } else {
        mask(u_last);
        floatx16 x;
        logits(buf * STAGE + i * RW + rw, x);
        add_up();
        s = x;
      }
      u_last = u;
    }
    if (more) store(buf ^ 1);
    __syncthreads();
  }
  if (u_last >= 0) {
    mask(u_last);
    add_up();
  }
  if (__builtin_expect(__any(sum != sum), 0)) {
    sum = 0.f;
#pragma unroll 1
    for (int u = u_begin + rw; u < units; u += RW) {
      const int row = u * 32 + c32 < rows ? u * 32 + c32 : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
      const __bf16* q_row = q_all + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group)) * D;
      const bool off = lse_log2(p, g, row, rows) == INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = -lse_log2(p, g, u * 32 + 8 * (i >> 2) + 4 * h + (i & 3), rows) * to_logit;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qbf16x8 q = q_query<D>(q_row, 16 * ks + 8 * h, p.rope_cos ? p.rope_cos + (int64_t)tok * (D / 2) : nullptr, p.rope_cos ? p.rope_sin + (int64_t)tok * (D / 2) : nullptr);
        if (off) q = qbf16x8{};
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, kf[ks], s, 0, 0, 0);
      }
      mask(u);
      add_up();
    }
  }
  sum = pair_sum(sum);
  if constexpr (RW > 1) {
    float* part = reinterpret_cast<float*>(q_lds);  // (behind the last barrier)
    if (h == 0) part[(rw * KW + kw) * 32 + c32] = sum;
    __syncthreads();
    if (tid < KW * 32) {
      float x = part[tid];
#pragma unroll
      for (int i = 1; i < RW; ++i) x += part[i * (KW * 32) + tid];
      give(p, g, wg_key + tid, x);
    }
  } else if (h == 0) {
    give(p, g, key, sum);
  }
}

template <int D, int KW, int RW, int UB>
static void launch_many(const WeighParams& p, hipStream_t s) {
  constexpr int keys = 32 * KW;
  const dim3 grid((unsigned)((p.len + keys - 1) / keys), (unsigned)p.n_kv_heads), block(64 * KW * RW);
  hipLaunchKernelGGL((weigh_bf16_kernel<D, KW, RW, UB>), grid, block, 0, s, p);
}

// At most 16 rows, bf16: every wavefront takes strips of 64 keys.
template <int D>
__global__ void __launch_bounds__(256, 4) weigh_few_bf16_kernel(WeighParams p) {
  constexpr int KS = D / 32;
  const int tid = threadIdx.x, l = tid & 63, kg = l >> 4, c16 = l & 15;
  const int g = blockIdx.y, rows = p.n_tokens * p.group, prev = p.len - p.n_tokens;
  const __bf16* k_head = reinterpret_cast<const __bf16*>(p.k) + (int64_t)g * p.capacity * D;
  const int row = c16 < rows ? c16 : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
  const __bf16* q_row = reinterpret_cast<const __bf16*>(p.q) + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group) + g * p.group) * D;
  qbf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = q_query<D>(q_row, 32 * ks + 8 * kg, p.rope_cos ? p.rope_cos + (int64_t)tok * (D / 2) : nullptr, p.rope_cos ? p.rope_sin + (int64_t)tok * (D / 2) : nullptr);
  float m[4];
  int at[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = lse_log2(p, g, 4 * kg + e, rows);
    at[e] = m[e] == INFINITY ? -1 : prev + (int)quot((unsigned)(4 * kg + e), p.by_group);
  }
  for (int strip = blockIdx.x * 4 + (tid >> 6); strip * 64 < p.len; strip += gridDim.x * 4) {
    qbf16x8 kf[4][KS];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      int key = strip * 64 + 16 * t + c16;
      if (key >= p.len) key = p.len - 1;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[t][ks] = *reinterpret_cast<const qbf16x8*>(k_head + (int64_t)key * D + 32 * ks + 8 * kg);
    }
    float sum[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], kf[t][ks], s, 0, 0, 0);
      const int key = strip * 64 + 16 * t + c16;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) x += __builtin_amdgcn_exp2f(__builtin_fmaf(key > at[e] ? -INFINITY : s[e], p.scale_log2e, -m[e]));
      sum[t] = pair_sum(row16_sum(x));
    }
    // lane (kg, c16) has key 16 kg + c16 of the strip to write
    const float mine = kg == 0 ? sum[0] : kg == 1 ? sum[1] : kg == 2 ? sum[2] : sum[3];
    give(p, g, strip * 64 + l, mine);
  }
}

// fp32, on the fp32 matrix instructions, which take 64 cycles for two columns of 32 rows and keys: the queries come straight from memory and nothing else
// matters much.  A wavefront has 32 keys and every RW-th unit, KW of them neighbouring keys.
template <int D, int KW, int RW>
__global__ void __launch_bounds__(64 * KW * RW, 2) weigh_f32_kernel(WeighParams p) {
  constexpr int CH = D / 8;  // pieces of a lane's share of a row: columns 8 i + 4 h .. + 3
  __shared__ float part[KW * RW * 32];
  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31, w = __builtin_amdgcn_readfirstlane(tid >> 6), kw = w % KW, rw = w / KW;
  const int g = blockIdx.y, rows = p.n_tokens * p.group, units = (rows + 31) / 32, prev = p.len - p.n_tokens;
  const int wg_key = blockIdx.x * (32 * KW), key = wg_key + kw * 32 + c32;
  const float* k_head = reinterpret_cast<const float*>(p.k) + (int64_t)g * p.capacity * D;
  floatx4 kf[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) kf[i] = *reinterpret_cast<const floatx4*>(k_head + (int64_t)(key < p.len ? key : p.len - 1) * D + 8 * i + 4 * h);
  const float* q_all = reinterpret_cast<const float*>(p.q) + (unsigned)(g * p.group * D);
  const int first_tok = wg_key > prev ? wg_key - prev : 0;
  float sum = 0.f;
#pragma unroll 1
  for (int u = (int)((int64_t)first_tok * p.group / 32) + rw; u < units; u += RW) {
    const int row = u * 32 + c32 < rows ? u * 32 + c32 : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
    const float* q_row = q_all + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group)) * D;
    floatx4 q[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) q[i] = *reinterpret_cast<const floatx4*>(q_row + 8 * i + 4 * h);
    // lane r of the wavefront's first 32 finds row r's log-sum-exp, and the last key that it sees
    const float lse = lse_log2(p, g, u * 32 + c32, rows);
    const int last = lse == INFINITY ? -1 : prev + (int)quot((unsigned)(u * 32 + c32), p.by_group);
    if (p.rope_cos) {
#pragma unroll
      for (int i = 0; i < CH / 2; ++i) {  // (a lane holds both elements of its pairs)
        const floatx4 c = *reinterpret_cast<const floatx4*>(p.rope_cos + (int64_t)tok * (D / 2) + 8 * i + 4 * h);
        const floatx4 sn = *reinterpret_cast<const floatx4*>(p.rope_sin + (int64_t)tok * (D / 2) + 8 * i + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = q[i][e], up = q[i + CH / 2][e], tl = up * sn[e], tu = lo * sn[e];
          q[i][e] = __builtin_fmaf(lo, c[e], -tl);
          q[i + CH / 2][e] = __builtin_fmaf(up, c[e], tu);
        }
      }
    }
    floatx16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q[i][e], kf[i][e], s, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 8 * (i >> 2) + 4 * h + (i & 3);
      const float x = key <= __shfl(last, r) ? s[i] : -INFINITY;
      sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x, p.scale_log2e, -__shfl(lse, r)));
    }
  }
  sum = pair_sum(sum);
  if (h == 0) part[w * 32 + c32] = sum;
  __syncthreads();
  if (tid < 32 * KW) {
    float x = part[tid];
#pragma unroll
    for (int i = 1; i < RW; ++i) x += part[i * (32 * KW) + tid];
    give(p, g, wg_key + tid, x);
  }
}

template <int D, int KW, int RW>
static void launch_f32(const WeighParams& p, hipStream_t s) {
  constexpr int keys = 32 * KW;
  const dim3 grid((unsigned)((p.len + keys - 1) / keys), (unsigned)p.n_kv_heads), block(64 * KW * RW);
  hipLaunchKernelGGL((weigh_f32_kernel<D, KW, RW>), grid, block, 0, s, p);
}

// How a workgroup's wavefronts are shared out between keys and rows.  Neighbouring keys share what is read of the queries; rows are shared out
// where there are too few keys to fill the chip, of 256 CUs where this was measured, with workgroups of 128.  bf16, 128 keys a workgroup / 64 keys and four shares of the rows: 256 tokens on 4096 keys,
// 32 heads on 8 (256 workgroups of 128 keys) 21.9 / 17.7 us, 1024 on 1024 84.2 / 39.2, 64 wide 128 on 512, 4 on 1, 11.1 / 6.0; 256 on 32K 92.9 / 115, 32 on
// 8192 (four units of rows) 7.5 / 11.5.  fp32, 128 keys and two shares / 32 keys and eight: 128 on 4096, 28 on 4, 75.6 / 50.7, 128 on 512, 64 wide, 24.6 / 9.4; 512 on
// 16K, 8 on 2 (256 workgroups) 159 / 188; one unit of rows has nothing to share out.
template <int D>
static void launch_width(const WeighParams& p, bool bf16, int n_cu, hipStream_t s) {
  const int64_t wgs = (int64_t)p.n_kv_heads * ((p.len + 127) / 128);
  const int units = (int)(((int64_t)p.n_tokens * p.group + 31) / 32);
  if (!bf16) {
    if (units == 1)
      launch_f32<D, 8, 1>(p, s);
    else if (weigh_shares_rows(bf16, n_cu, wgs, units))
      launch_f32<D, 1, 8>(p, s);
    else
      launch_f32<D, 4, 2>(p, s);
  } else if (p.n_tokens * p.group <= 16) {
    const dim3 grid((unsigned)((p.len + 255) / 256), (unsigned)p.n_kv_heads);
    hipLaunchKernelGGL(weigh_few_bf16_kernel<D>, grid, dim3(256), 0, s, p);
  } else if (weigh_shares_rows(bf16, n_cu, wgs, units)) {
    launch_many<D, 2, 4, 1>(p, s);
  } else {
    launch_many<D, 4, 1, 2>(p, s);
  }
}

hipError_t launch_weigh(const WeighParams& p, int head_dim, bool bf16, int n_cu, hipStream_t s) {
  if (head_dim == 128)
    launch_width<128>(p, bf16, n_cu, s);
  else
    launch_width<64>(p, bf16, n_cu, s);
  return hipGetLastError();
}

}  // namespace kvfold
