// Rows on their way into the cache that is held in 8 bits, and back (the layout and the arithmetic are described in qcache.h).
//
// Append: a workgroup has a block of 64 rows of one KV head, K or V.  Rows that were there already come from the ring, the others as handed
// in; the block's largest magnitude is found, and the codes leave 16 bytes a lane.  Memory-bound where many rows come at once (8 heads, 128 wide: 65536 rows 108 us,
// 3.7 TB/s), else one launch's latency (up to 64 rows 4.7 us, 256 6.0, 2048 8.3).  Reading
// back is memory-bound as well, four bytes written for a code: 65536 rows 133 to 137 us, 5.0 TB/s.
#include "qcache.h"

namespace kvfold {

constexpr int kThreads = 256;

// Elements of a piece as they come in (fresh: bit e, row of element e is one of the new ones), bf16 bits.
template <int D, bool V>
struct Piece {
  unsigned x[16];
  unsigned fresh;
};

template <int D, bool V>
__device__ __forceinline__ void piece_place(int i, int& c, int& key) {  // c: column block (K) or column (V); key: the row, or the key group
  if (V) {
    c = i % D;
    key = i / D;
  } else {
    c = i % (D / 16);
    key = i / (D / 16);
  }
}

template <int D, bool V>
__device__ __forceinline__ Piece<D, V> piece_in(const QAppendParams& p, int64_t block, int g, int i) {
  Piece<D, V> q;
  int c, key;
  piece_place<D, V>(i, c, key);
  const __bf16* rows = p.rows[V] + (int64_t)g * p.head_stride;
  const int64_t t0 = block * kQBlock - p.len_prev;  // the block's first row, among the new ones
  q.fresh = 0;
  if (V) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t t = t0 + q_key(key, e);
      const bool in = t >= 0 && t < p.n;
      q.fresh |= in ? 1u << e : 0u;
      q.x[e] = finite_bf16(in ? __builtin_bit_cast(unsigned short, rows[t * p.token_stride + c]) : 0u);
    }
  } else {
    const int64_t t = t0 + key;
    if (t >= 0 && t < p.n) {
      q.fresh = 0xffffu;
      const __bf16* row = rows + t * p.token_stride;
      const float* cs = p.rope_cos ? p.rope_cos + t * (D / 2) : nullptr;
      const float* sn = p.rope_cos ? p.rope_sin + t * (D / 2) : nullptr;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const qbf16x8 v = q_query<D>(row, 16 * c + 8 * h, cs, sn);
#pragma unroll
        for (int e = 0; e < 8; ++e) q.x[8 * h + e] = finite_bf16(__builtin_bit_cast(unsigned short, (__bf16)v[e]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) q.x[e] = 0;
    }
  }
  return q;
}

template <int D, bool V>
__device__ __forceinline__ int piece_index(int i) {
  int c, key;
  piece_place<D, V>(i, c, key);
  return V ? q_v_piece(D, key, c) : q_k_piece(c, key);
}

template <int D, bool V>
__device__ __forceinline__ void to_ring(__bf16* slot, int i, const Piece<D, V>& q) {
  unsigned short* at = reinterpret_cast<unsigned short*>(slot) + piece_index<D, V>(i) * 16;
  if (q.fresh == 0xffffu) {
    quintx4 w[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2][e & 3] = q.x[2 * e] | q.x[2 * e + 1] << 16;
    reinterpret_cast<quintx4*>(at)[0] = w[0];
    reinterpret_cast<quintx4*>(at)[1] = w[1];
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (q.fresh >> e & 1) at[e] = (unsigned short)q.x[e];
  }
}

template <int D, bool V>
__device__ __forceinline__ void append_block(const QAppendParams& p, int g) {
  constexpr int N = kQBlock * D / 16, T = N / kThreads;  // pieces, and those of a thread
  __shared__ float wave_max[kThreads / 64];
  const int tid = threadIdx.x;
  const QRingWriters writers(p.len_prev, p.n);
  const int64_t end = p.len_prev + p.n, block = writers.first + blockIdx.x;
  __bf16* ring = p.to.ring[V] + (int64_t)g * (kQRing * kQBlock * D);
  Piece<D, V> q[T];
#pragma unroll
  for (int j = 0; j < T; ++j) q[j] = piece_in<D, V>(p, block, g, tid + j * kThreads);
  if (writers.itself(block)) {
#pragma unroll
    for (int j = 0; j < T; ++j) to_ring<D, V>(ring + (block % kQRing) * (kQBlock * D), tid + j * kThreads, q[j]);
  }
  const bool whole = (block + 1) * kQBlock <= end;
  if (whole) {
    if (block == writers.first && writers.earlier) {
      const unsigned short* slot = reinterpret_cast<const unsigned short*>(ring) + (block % kQRing) * (kQBlock * D);
#pragma unroll
      for (int j = 0; j < T; ++j) {
        const quintx4* at = reinterpret_cast<const quintx4*>(slot + piece_index<D, V>(tid + j * kThreads) * 16);
        const quintx4 w[2] = {at[0], at[1]};
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(q[j].fresh >> e & 1)) q[j].x[e] = w[e >> 3][e >> 1 & 3] >> 16 * (e & 1) & 0xffffu;
      }
    }
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, q[j].x[e] & 0x7fffu);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, off));
    if ((tid & 63) == 0) wave_max[tid >> 6] = __uint_as_float(top << 16);
    __syncthreads();
    float amax = wave_max[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) amax = fmaxf(amax, wave_max[w]);
    const float scale = fmaxf(amax / 127.f, 0x1p-100f);
    const int64_t at = (int64_t)g * p.to.blocks + block;
    if (tid == 0) p.to.scales[2 * at + V] = scale;
    quintx4* codes = reinterpret_cast<quintx4*>(p.to.codes[V] + at * (kQBlock * D));
#pragma unroll
    for (int j = 0; j < T; ++j) {
      quintx4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        unsigned r = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = rintf(__uint_as_float(q[j].x[4 * k + e] << 16) / scale);
          r |= ((unsigned)(int)fminf(fmaxf(y, -127.f), 127.f) & 0xffu) << (8 * e);
        }
        w[k] = r;
      }
      codes[piece_index<D, V>(tid + j * kThreads)] = w;
    }
  }
  // The block whose rows take the place of the first block's in the ring
  const int64_t over = writers.taken_over();
  if (block == writers.first && over > block) {
    __syncthreads();  // (the block's earlier rows have been read: their values went into the codes' scale)
#pragma unroll 1
    for (int j = 0; j < T; ++j) to_ring<D, V>(ring + (over % kQRing) * (kQBlock * D), tid + j * kThreads, piece_in<D, V>(p, over, g, tid + j * kThreads));
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads) qappend_kernel(QAppendParams p) {
  const int g = blockIdx.y >> 1;
  if (blockIdx.y & 1)
    append_block<D, true>(p, g);
  else
    append_block<D, false>(p, g);
}

hipError_t launch_qappend(const QAppendParams& p, int head_dim, hipStream_t s) {
  if (p.n <= 0) return hipSuccess;
  const int64_t blocks = (p.len_prev + p.n - 1) / kQBlock - p.len_prev / kQBlock + 1;
  const dim3 grid((unsigned)blocks, (unsigned)(2 * p.n_kv_heads)), block(kThreads);
  if (head_dim == 128)
    hipLaunchKernelGGL(qappend_kernel<128>, grid, block, 0, s, p);
  else
    hipLaunchKernelGGL(qappend_kernel<64>, grid, block, 0, s, p);
  return hipGetLastError();
}

// Rows as numbers: a thread has four columns of four rows, which are whole words of K (a row's) and of V (a column's) alike.
template <int D>
__global__ void __launch_bounds__(kThreads) qread_kernel(QReadParams p) {
  typedef __attribute__((ext_vector_type(4))) float floatx4;
  const bool v = blockIdx.y & 1;
  const int g = blockIdx.y >> 1;
  float* out = p.out[v];
  if (!out) return;
  const int64_t quad0 = p.first / 4, end = p.first + p.n, n = ((end - 1) / 4 - quad0 + 1) * (D / 4), whole = p.len / kQBlock * kQBlock;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row0 = 4 * (quad0 + i / (D / 4)), block = row0 / kQBlock;
    const int c = (int)(i % (D / 4)) * 4, key = (int)(row0 % kQBlock);
    const int at = v ? q_v_piece(D, q_key_group(key), c) * 16 + q_key_element(key) : q_k_piece(c >> 4, key) * 16 + (c & 15);
    floatx4 x[4];
    if (row0 < whole) {
      const int64_t b = (int64_t)g * p.from.blocks + block;
      const unsigned char* codes = p.from.codes[v] + b * (kQBlock * D) + at;
      const float scale = p.from.scales[2 * b + v];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const unsigned w = *reinterpret_cast<const unsigned*>(codes + 16 * u);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = (float)(int)(signed char)(w >> (8 * e)) * scale;
      }
    } else {
      const __bf16* slot = p.from.ring[v] + ((int64_t)g * kQRing + block % kQRing) * (kQBlock * D) + at;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = (float)slot[16 * u + e];
    }
    if (v) {  // (came by columns)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < u; ++e) {
          const float y = x[u][e];
          x[u][e] = x[e][u];
          x[e][u] = y;
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = row0 + u;
      if (row >= p.first && row < end) *reinterpret_cast<floatx4*>(out + ((row - p.first) * p.n_kv_heads + g) * D + c) = x[u];
    }
  }
}

hipError_t launch_qread(const QReadParams& p, int head_dim, hipStream_t s) {
  if (p.n <= 0) return hipSuccess;
  int64_t bx = ((p.n + 6) / 4 * (head_dim / 4) + kThreads - 1) / kThreads;
  if (bx > 4096) bx = 4096;
  const dim3 grid((unsigned)bx, (unsigned)(2 * p.n_kv_heads)), block(kThreads);
  if (head_dim == 128)
    hipLaunchKernelGGL(qread_kernel<128>, grid, block, 0, s, p);
  else
    hipLaunchKernelGGL(qread_kernel<64>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
