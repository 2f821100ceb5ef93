// The cache held in 8 bits: how a layer lies in memory, and what the rows go through on their way in.  The layout part has no HIP types, so that
// host-only tests are built on it.
//
// Rows come in blocks of 64 (block b of a KV head: rows 64 b .. 64 b + 63).  A block whose rows are all there is held as codes, whole numbers from
// -127 to 127, with one scale for K and one for V:
//     scale = max(max |x| / 127, 2^-100),   code = x / scale rounded to the nearest whole number (ties to even),
// both quotients rounded to fp32 first; the row that a code stands for is code * scale.  The floor keeps scale and 1 / scale inside the range of
// fp32 (a weight times a small scale may leave it: q_tiny()); a block below 127 * 2^-100 loses at most 2^-101 an element by it.  Rows of the last,
// incomplete block are held as they came, in bf16, in a ring of two blocks (row r in slot r / 64 % 2), so that what a block is held as
// does not depend on the chunks that it came in, and behind an append the last 64 rows can be taken back, but for those that a rewind has left as codes (QLength).  What comes in is made finite: infinities become
// the largest bf16 number, NaN 0.  (A masked weight is 0, and 0 times infinity is NaN, in rows that do not see the key.)
//
// A block lies as the matrix instructions want it, in pieces of 16 elements, codes (16 bytes) or bf16 (32 bytes) alike:
//   K: piece (column block c, key) = columns 16 c .. 16 c + 15 of the key's row, at piece 64 c + key;
//   V: piece (key group kg, column) = the column at the group's 16 keys, at piece d kg + column.  Key 32 (kg / 2) + 4 (kg % 2) + 8 j + e (j, e < 4)
//      is element 4 j + e: the keys whose logits a lane holds, of the 32x32 shapes (lane half kg % 2, S^T's tile kg / 2) and of the 16x16
//      ones alike (lane group kg, where S^T's tile j has these keys as its rows), so that a weight never leaves its lane.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/kvfold.h"
#include "kvfold_consts.h"

namespace kvfold {

constexpr int kQBlock = kTileKeys;  // rows that share a scale
constexpr int kQRing = 2;           // blocks held in bf16

KVFOLD_HD int q_k_piece(int c, int key) { return kQBlock * c + key; }
KVFOLD_HD int q_v_piece(int d, int kg, int column) { return d * kg + column; }
KVFOLD_HD int q_key_group(int key) { return 2 * (key >> 5) + (key >> 2 & 1); }
KVFOLD_HD int q_key_element(int key) { return 4 * (key >> 3 & 3) + (key & 3); }
KVFOLD_HD int q_key(int kg, int element) { return 32 * (kg >> 1) + 4 * (kg & 1) + 8 * (element >> 2) + (element & 3); }

// Bytes of a layer, each part's a multiple of 256: codes of K, codes of V, [Hkv][blocks][64 d]; scales [Hkv][blocks][2]; ring of K, ring of V,
// [Hkv][2][64 d] bf16.
struct QLayout {
  int64_t blocks;  // of a KV head
  size_t codes, scales, ring, layer;
};
inline QLayout q_layout(const kvfold_config_t& c) {
  auto whole = [](size_t n) { return (n + 255) / 256 * 256; };
  QLayout l;
  l.blocks = (c.capacity_tokens + kQBlock - 1) / kQBlock;
  const size_t block = (size_t)kQBlock * (size_t)c.head_dim, heads = (size_t)c.n_kv_heads;
  l.codes = whole(heads * (size_t)l.blocks * block);
  l.scales = whole(heads * (size_t)l.blocks * 2 * sizeof(float));
  l.ring = whole(heads * kQRing * block * 2);
  l.layer = 2 * l.codes + l.scales + 2 * l.ring;
  return l;
}

// Who writes the ring when rows [prev, prev + n) are appended, a workgroup a block (and KV head, K or V).  The ring takes the rows of the last two
// blocks.  Whose slot the first block's earlier rows lie in, if it has any, is written by the first block's workgroup, once it has read them.
struct QRingWriters {
  int64_t first, last;  // the blocks that get rows
  bool earlier;         // the first one has rows already
  KVFOLD_HD QRingWriters(int64_t prev, int64_t n) : first(prev / kQBlock), last((prev + n - 1) / kQBlock), earlier(prev % kQBlock != 0) {}
  // The block's workgroup writes its new rows, before all else.
  KVFOLD_HD bool itself(int64_t block) const { return block + kQRing > last && !(earlier && block != first && (block - first) % kQRing == 0); }
  // The block whose new rows the first block's workgroup writes at its end; first: none
  KVFOLD_HD int64_t taken_over() const { return earlier ? last - (last - first) % kQRing : first; }
};

// What the host knows of a layer.  Rows [ring_from, len) are in the ring, but for those of blocks that begin before ring_from.
struct QLength {
  int64_t len = 0, ring_from = 0;
  void append(int64_t n) {
    len += n;
    const int64_t last = (len - 1) / kQBlock, oldest = (last - (kQRing - 1)) * kQBlock;
    if (ring_from < oldest) ring_from = oldest;
  }
  // Rows of an incomplete block have to be in the ring.
  bool can_truncate(int64_t n) const { return n >= 0 && n <= len && (n % kQBlock == 0 || n / kQBlock * kQBlock >= ring_from); }
  void truncate(int64_t n) {
    len = n;
    if (ring_from > n) ring_from = n;
  }
};

int validate_qconfig(const kvfold_config_t* c);
// Pieces that the keys of a step are cut into, and blocks of each; the kernel (decode: at most 16 packed rows a KV head); whether the
// pieces meet in it.
struct QPlan {
  bool decode, meet;
  int waves_per_wg, units_per_head, wgs_per_head, n_splits, blocks_per_split, n_wgs;  // a wavefront has a unit of 32 rows
};
QPlan make_qplan(const kvfold_config_t& c, int n_cu, int64_t ws_rows, int n_tokens, int64_t len_after);

}  // namespace kvfold

#if defined(__HIP__)
#include "append_rows.h"
#include "kvfold_internal.h"

namespace kvfold {

struct QRows {  // one layer
  unsigned char* codes[2];  // K, V
  float* scales;
  __bf16* ring[2];
  int64_t blocks;
};

struct QAppendParams {
  QRows to;
  const __bf16* rows[2];  // K, V: row t of KV head g at t * token_stride + g * head_stride
  int64_t token_stride, head_stride;
  int64_t len_prev, n;
  const float *rope_cos, *rope_sin;  // of the K rows, [n][d/2], or nullptr
  int n_kv_heads;
};
hipError_t launch_qappend(const QAppendParams& p, int head_dim, hipStream_t s);

struct QReadParams {
  QRows from;
  float* out[2];  // [n][Hkv][d]
  int64_t first, n, len;
  int n_kv_heads;
};
hipError_t launch_qread(const QReadParams& p, int head_dim, hipStream_t s);

struct QAttnParams {
  AttnParams a;  // k_cache, v_cache: unused; tiles_per_split: blocks
  QRows c;
  // Rows of the chunk that fill no block are appended by whom alone reads them, the workgroup with the head's last block (nullptr: the cache holds them
  // already): as handed in, [C][Hkv][d]
  const __bf16 *k_new, *v_new;
};
hipError_t launch_attn_qdecode(const QAttnParams& p, int head_dim, hipStream_t s);
hipError_t launch_attn_q(const QAttnParams& p, int head_dim, int waves, hipStream_t s);  // waves: of a workgroup, as planned

typedef __attribute__((ext_vector_type(8))) __bf16 qbf16x8;
typedef __attribute__((ext_vector_type(4))) unsigned quintx4;

__device__ __forceinline__ unsigned finite_bf16(unsigned x) {
  const unsigned m = x & 0x7fffu;
  return m < 0x7f80u ? x : m == 0x7f80u ? (x & 0x8000u) | 0x7f7fu : 0u;
}
__device__ __forceinline__ qbf16x8 finite_row(qbf16x8 x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(__bf16, (unsigned short)finite_bf16(__builtin_bit_cast(unsigned short, (__bf16)x[e])));
  return x;
}

// Two of 16 codes as bf16, which holds them exactly: two conversions that pick their byte, and a byte permutation that takes the upper halves of both.
__device__ __forceinline__ unsigned q_widen_word(const quintx4& codes, int w) {
  const unsigned x = codes[w >> 1];
  const float f0 = (float)(int)(signed char)(x >> (w & 1 ? 16 : 0)), f1 = (float)(int)(signed char)(x >> (w & 1 ? 24 : 8));
  return __builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u);
}
__device__ __forceinline__ qbf16x8 q_widen_half(const quintx4& codes, int half) {
  quintx4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) r[w] = q_widen_word(codes, 4 * half + w);
  return __builtin_bit_cast(qbf16x8, r);
}
__device__ __forceinline__ void q_widen(const quintx4& codes, qbf16x8& lo, qbf16x8& up) {
  lo = q_widen_half(codes, 0);
  up = q_widen_half(codes, 1);
}

// What a block's logits are multiplied by; above 0, so that a masked logit, -inf, stays that.
__device__ __forceinline__ float q_to_log2(float k_scale, float scale_log2e) { return fmaxf(k_scale * scale_log2e, 0x1p-126f); }

// The weights of a block come multiplied by its scale of V.  One as small as this takes them out of fp32's range: what the output
// loses by that is less than 2^-119 a key, but of the row sum it may be a good part, which is taken from the weights by themselves.  (The scale is the
// wavefront's; numbers above 0 compare like whole ones.)
__device__ __forceinline__ bool q_tiny(float v_scale) { return __builtin_amdgcn_readfirstlane((int)__float_as_uint(v_scale)) < (int)__builtin_bit_cast(unsigned, 0x1p-20f); }

// One as large as 2^64 and more would take the outputs out of it, which are not divided by the row sum before the end: a row's reference then is this much
// (log2 units) above its maximum.  (Weights of 2^16 above the reference, 127 times a scale and 2^25 blocks of 64 keys: 2^118.
// Such a row's weights and outputs are held up to 2^57 smaller for it: weights below 2^-69 of the largest are lost, and outputs below 2^-69.)
__device__ __forceinline__ float q_above(float v_scale) { return fmaxf(__builtin_amdgcn_logf(v_scale) - 64.f, 0.f); }
// Rows held as they came may be as large, without a scale that tells.  They are done again with the reference this much above where an output
// reaches 2^100: 63 numbers of 2^128 and weights of 2^(16 - 32) are 2^118.
constexpr float kQAboveRows = 32.f, kQLower = 0x1p-32f;  // log2 units, and as a factor
template <int E, class V, int N>
__device__ __forceinline__ bool q_large(const V (&o)[N]) {
  float all = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < E; ++i) all = __builtin_fmaf(o[j][i], 0x1p28f, all);
  return !(fabsf(all) < INFINITY);  // (what is infinite on the way, or NaN, stays so)
}

// Columns c0 .. c0 + 7 of a query row, rotated if there are angles (the arithmetic of append_rows.h, bit for bit that of a caller who rotates and
// stores bf16).
template <int D>
__device__ __forceinline__ qbf16x8 q_query(const __bf16* row, int c0, const float* cs, const float* sn) {
  qbf16x8 x = *reinterpret_cast<const qbf16x8*>(row + c0);
  if (cs) {
    typedef __attribute__((ext_vector_type(4))) float floatx4;
    const qbf16x8 other = *reinterpret_cast<const qbf16x8*>(row + (c0 ^ (D / 2)));
    const int at = c0 & (D / 2 - 1);
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const floatx4 a = *reinterpret_cast<const floatx4*>(cs + at + e), b = *reinterpret_cast<const floatx4*>(sn + at + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[e + i] = a[i], s[e + i] = b[i];
    }
    rotate_vec<__bf16, 8>(x, other, c, s, c0 < D / 2);
  }
  return x;
}

// The chunk's rows of KV head g into its incomplete block, in place `slot` of the ring, whose last rows they are of n: share i0, i0 + step, ...
template <int D>
__device__ __forceinline__ void q_fill_block(const QAttnParams& qp, int g, uint64_t slot, int n, int i0, int step) {
  const AttnParams& p = qp.a;
  const int C = p.n_tokens;
  const int64_t stride = (int64_t)p.n_kv_heads * D;
  const __bf16 *k_new = qp.k_new + g * D, *v_new = qp.v_new + g * D;
  unsigned short* v_slot = reinterpret_cast<unsigned short*>(qp.c.ring[1] + slot);
  for (int i = i0; i < C * (D / 8); i += step) {
    const int t = i / (D / 8), c = i % (D / 8), key = n - C + t;
    const qbf16x8 k = finite_row(q_query<D>(k_new + t * stride, 8 * c, p.rope_cos ? p.rope_cos + t * (D / 2) : nullptr, p.rope_cos ? p.rope_sin + t * (D / 2) : nullptr));
    const qbf16x8 v = finite_row(*reinterpret_cast<const qbf16x8*>(v_new + t * stride + 8 * c));
    *reinterpret_cast<qbf16x8*>(qp.c.ring[0] + slot + q_k_piece(c >> 1, key) * 16 + (c & 1) * 8) = k;
#pragma unroll
    for (int e = 0; e < 8; ++e) v_slot[q_v_piece(D, q_key_group(key), 8 * c + e) * 16 + q_key_element(key)] = __builtin_bit_cast(unsigned short, (__bf16)v[e]);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

}  // namespace kvfold
#endif
