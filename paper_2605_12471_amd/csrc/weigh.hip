// The softmax weight that a chunk's queries gave to each cached key, summed over the rows and the query heads of the KV head's group:
//     w[g][j] = sum over rows (i, h) of the group with j <= len - n + i of 2^(s scale log2 e - lse[h][i] log2 e),   s = q . k_j.
// The step has left the log-sum-exps, so that one product is all there is: no maximum, no second pass, and every weight's sum belongs to one lane.
//
// S = Q K^T with the queries as the matrix instruction's rows: a lane holds the logits of one key, which it adds up without a word to other lanes
// until the end.  The keys stay in registers and the queries stream past, through LDS in operand order, a unit of 32 packed rows at a time,
// two buffers, one barrier.  Bound by matrix instructions and exponentials alike: 128 wide a unit on 32 keys takes eight of 32 cycles,
// and 16 exponentials a lane of 8 with a multiply-add and an add.
//
// Few rows (at most 16 a KV head) are bound by reading the keys: the wavefronts take 64 keys at a time straight into registers, on the 16x16x32
// shapes, whole 64-byte pieces of rows an instruction.
//
// A row whose log-sum-exp is -inf gave no weight to any key.
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

// Many rows, bf16: a workgroup has 4 x 32 KB keys of one KV head.
template <int D, int KB>
__global__ void __launch_bounds__(256, 2) weigh_bf16_kernel(WeighParams p) {
  constexpr int KS = D / 16, CH = D / 8, T = 32 * CH / 256, UNIT = 32 * D * 2;
  __shared__ __attribute__((aligned(16))) unsigned char q_lds[2 * UNIT];
  __shared__ __attribute__((aligned(16))) float lse_lds[2 * 32];
  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.y, rows = p.n_tokens * p.group, units = (rows + 31) / 32, prev = p.len - p.n_tokens;
  const int wg_key = blockIdx.x * (4 * 32 * KB), key0 = wg_key + w * (32 * KB);

  // ---- the keys: lane (key, h) holds columns 16 ks + 8 h .. + 7
  const __bf16* k_head = reinterpret_cast<const __bf16*>(p.k) + (int64_t)g * p.capacity * D;
  qbf16x8 kf[KB][KS];
#pragma unroll
  for (int b = 0; b < KB; ++b) {
    int key = key0 + 32 * b + c32;
    if (key >= p.len) key = p.len - 1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[b][ks] = *reinterpret_cast<const qbf16x8*>(k_head + (int64_t)key * D + 16 * ks + 8 * h);
  }

  // ---- a unit on its way: 16-byte piece c of row r at (32 c + (r ^ c % 32)) 16
  qbf16x8 q_in[T];
  float lse_in = 0.f;
  const __bf16* q_all = reinterpret_cast<const __bf16*>(p.q);
  auto load = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int i = tid + 256 * j, r = i / CH, c = i % CH;
      int row = u * 32 + r;
      if (row >= rows) row = rows - 1;
      const int tok = (int)quot((unsigned)row, p.by_group);
      const __bf16* q_row = q_all + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group) + g * p.group) * D;
      q_in[j] = q_query<D>(q_row, 8 * c, p.rope_cos ? p.rope_cos + (int64_t)tok * (D / 2) : nullptr, p.rope_cos ? p.rope_sin + (int64_t)tok * (D / 2) : nullptr);
    }
    if (tid < 32) lse_in = lse_log2(p, g, u * 32 + tid, rows);
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int i = tid + 256 * j, r = i / CH, c = i % CH;
      *reinterpret_cast<qbf16x8*>(q_lds + buf * UNIT + (32 * c + (r ^ c)) * 16) = q_in[j];
    }
    if (tid < 32) lse_lds[buf * 32 + tid] = lse_in;
  };

  // The first unit with a row that sees the workgroup's first key: row i of the chunk sees keys up to prev + i
  const int first_tok = wg_key > prev ? wg_key - prev : 0, u_begin = (int)((int64_t)first_tok * p.group / 32);
  float sum[KB];
#pragma unroll
  for (int b = 0; b < KB; ++b) sum[b] = 0.f;
  load(u_begin);
  store(0);
  __syncthreads();
#pragma unroll 1
  for (int u = u_begin; u < units; ++u) {
    const int buf = (u - u_begin) & 1;
    if (u + 1 < units) load(u + 1);
    floatx16 s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int c = 2 * ks + h;
      const qbf16x8 q = *reinterpret_cast<const qbf16x8*>(q_lds + buf * UNIT + (32 * c + (c32 ^ c)) * 16);
#pragma unroll
      for (int b = 0; b < KB; ++b) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, kf[b][ks], s[b], 0, 0, 0);
    }
    if (prev + (int)quot((unsigned)(u * 32), p.by_group) < key0 + 32 * KB - 1) {  // some row does not see all of the wavefront's keys
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = prev + (int)quot((unsigned)(u * 32 + 8 * (i >> 2) + 4 * h + (i & 3)), p.by_group);
#pragma unroll
        for (int b = 0; b < KB; ++b)
          if (key0 + 32 * b + c32 > at) s[b][i] = -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const floatx4 m = *reinterpret_cast<const floatx4*>(lse_lds + buf * 32 + 2 * i + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int b = 0; b < KB; ++b) sum[b] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i + e], p.scale_log2e, -m[e]));
    }
    if (u + 1 < units) store(buf ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < KB; ++b) {
    const float x = pair_sum(sum[b]);
    if (h == 0) give(p, g, key0 + 32 * b + c32, x);
  }
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
    at[e] = prev + (int)quot((unsigned)(4 * kg + e), p.by_group);
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

// fp32: 32 keys a wavefront, on the fp32 matrix instructions.
template <int D>
__global__ void __launch_bounds__(256, 2) weigh_f32_kernel(WeighParams p) {
  constexpr int CH = D / 4, T = 32 * CH / 256, UNIT = 32 * D * 4;
  __shared__ __attribute__((aligned(16))) unsigned char q_lds[UNIT];
  __shared__ __attribute__((aligned(16))) float lse_lds[32];
  const int tid = threadIdx.x, l = tid & 63, h = l >> 5, c32 = l & 31, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.y, rows = p.n_tokens * p.group, units = (rows + 31) / 32, prev = p.len - p.n_tokens;
  const int wg_key = blockIdx.x * 128, key0 = wg_key + w * 32;
  const float* k_head = reinterpret_cast<const float*>(p.k) + (int64_t)g * p.capacity * D;
  const int key = key0 + c32;
  floatx4 kf[CH / 2];  // columns 8 i + 4 h .. + 3
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) kf[i] = *reinterpret_cast<const floatx4*>(k_head + (int64_t)(key < p.len ? key : p.len - 1) * D + 8 * i + 4 * h);
  const float* q_all = reinterpret_cast<const float*>(p.q);
  const int first_tok = wg_key > prev ? wg_key - prev : 0;
  float sum = 0.f;
#pragma unroll 1
  for (int u = (int)((int64_t)first_tok * p.group / 32); u < units; ++u) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int i = tid + 256 * j, r = i / CH, c = i % CH;
      int row = u * 32 + r;
      if (row >= rows) row = rows - 1;
      const int tok = (int)quot((unsigned)row, p.by_group);
      const float* q_row = q_all + (uint64_t)(unsigned)(row + tok * (p.n_q_heads - p.group) + g * p.group) * D;
      row_vec<float, 4> x = *reinterpret_cast<const row_vec<float, 4>*>(q_row + 4 * c);
      if (p.rope_cos) {
        const int a = 4 * c % (D / 2);
        const row_vec<float, 4> other = *reinterpret_cast<const row_vec<float, 4>*>(q_row + ((4 * c) ^ (D / 2)));
        rotate_vec<float, 4>(x, other, p.rope_cos + (int64_t)tok * (D / 2) + a, p.rope_sin + (int64_t)tok * (D / 2) + a, 4 * c < D / 2);
      }
      *reinterpret_cast<row_vec<float, 4>*>(q_lds + (32 * c + (r ^ (c & 31))) * 16) = x;
    }
    if (tid < 32) lse_lds[tid] = lse_log2(p, g, u * 32 + tid, rows);
    __syncthreads();
    floatx16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const int c = 2 * i + h;
      const floatx4 q = *reinterpret_cast<const floatx4*>(q_lds + (32 * c + (c32 ^ (c & 31))) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q[e], kf[i][e], s, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 8 * (i >> 2) + 4 * h + (i & 3);
      const bool seen = key <= prev + (int)quot((unsigned)(u * 32 + r), p.by_group);
      sum += __builtin_amdgcn_exp2f(__builtin_fmaf(seen ? s[i] : -INFINITY, p.scale_log2e, -lse_lds[r]));
    }
  }
  sum = pair_sum(sum);
  if (h == 0) give(p, g, key, sum);
}

hipError_t launch_weigh(const WeighParams& p, int head_dim, bool bf16, hipStream_t s) {
  const unsigned heads = (unsigned)p.n_kv_heads;
  const dim3 block(256);
  if (!bf16) {
    const dim3 grid((unsigned)((p.len + 127) / 128), heads);
    if (head_dim == 128)
      hipLaunchKernelGGL(weigh_f32_kernel<128>, grid, block, 0, s, p);
    else
      hipLaunchKernelGGL(weigh_f32_kernel<64>, grid, block, 0, s, p);
  } else if (p.n_tokens * p.group <= 16) {
    const dim3 grid((unsigned)((p.len + 255) / 256), heads);
    if (head_dim == 128)
      hipLaunchKernelGGL(weigh_few_bf16_kernel<128>, grid, block, 0, s, p);
    else
      hipLaunchKernelGGL(weigh_few_bf16_kernel<64>, grid, block, 0, s, p);
  } else {
    const dim3 grid((unsigned)((p.len + 255) / 256), heads);
    if (head_dim == 128)
      hipLaunchKernelGGL((weigh_bf16_kernel<128, 2>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((weigh_bf16_kernel<64, 2>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace kvfold
