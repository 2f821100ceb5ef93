// Chunk-prefix attention on a cache held in 8 bits, any number of rows.  A work unit is 32 consecutive packed (token, head of the group) rows
// of a KV head, the work of one wavefront; a workgroup has NW of them of one KV head, and a piece of its blocks.
//
// Bound by the matrix instructions and by issue.  A block of 64 keys is brought in as codes, half the bytes of bf16; each thread widens its own to
// bf16, which holds them exactly, and puts them into LDS in the order of the matrix instructions' operands, so that they are widened once for
// the workgroup's rows and every LDS access is 16 bytes a lane, neighbours side by side.  V needs no transpose on the way: the layout
// (qcache.h) has its keys side by side.
//
// S^T = K Q^T and O^T = V^T P^T on the 32x32x16 shapes: a lane holds 32 logits of one query, whose weights are its operand of the second product
// as they stand.  Scales and rounding points as in the decoding kernel (attn_qdecode.hip), the second exponential for a tiny scale of V included (three
// quarters of the values zero: 2048 tokens on 32K keys 1067 us for 996).  The reference m of a row only has to keep the weights
// inside the range of fp32.  It is the first block's maximum, and is not compared with another's while the row sees all of a block: the sum of a
// block's weights, needed anyway, tells when it is far behind, and it follows by a power of two.  Logits that rise by more than fp32 holds
// within one block, or values so large that outputs might, lose the piece, which the workgroup then does again, with every block's maximum taken.
//
// A turn of a SIMD's two wavefronts, 64 matrix instructions of 32 cycles, takes 1.9 us, 0.59 of what the pipes do alone; the rest is issue, 5.8 vector
// instructions beside each: per logit a multiplication, an exponential, an addition and half a rounding, and the widening.  Steps of 32 heads on 8, 128
// wide: 256 tokens on 64K keys 269 us (1.02 PFLOP/s), 2048 on 32K 1008 us (1.12); 64 wide, 1000 on 8K, where a logit has half the products, 100 us
// (0.71).  Codes three turns ahead by copies to LDS took as long as without, and so did codes of one place for every block: it is not the memory
// that is waited for.
#include "qcache.h"
#include "wave_ops.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((ext_vector_type(16))) float floatx16;

template <int D, int NW>
__global__ void __launch_bounds__(NW * 64, 2) attn_q_kernel(QAttnParams qp) {
  const AttnParams& p = qp.a;
  constexpr int KS = D / 16, JT = D / 32;            // contraction steps of S^T, tiles of O^T
  constexpr int BLOCK = kQBlock * D;                 // codes of a block
  constexpr int NT = NW * 64, T = 2 * BLOCK / 16 / NT;  // threads; pieces of each: one of K and one of V, or of either
  constexpr int SLOT = BLOCK * 2;                    // bytes of a block's K, or V, in LDS
  constexpr float kStale = 16.0f;                    // log2 units
  constexpr float kFar = 0x1p60f, kLost = 0x1p100f;  // sums of a lane's weights in a block
  constexpr float kMost = 0x1p90f;                   // the same times the scale of V: 2^8 of it, in 2^25 blocks, are outputs
  static_assert(T * NT * 16 == 2 * BLOCK && (T == 1 || T == 2), "every thread has the same share of a block");
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * SLOT];  // K, K, V, V

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

  // Keys that a row sees; that the workgroup's last row sees
  auto seen_by = [&](int r) __attribute__((always_inline)) -> int {
    r = r < rows ? r : rows - 1;
    return (int)p.len_prev + (int)quot((unsigned)r, p.by_group) + 1;
  };
  const int vis_wg = seen_by((wg + 1) * NW * kRowsPerUnit - 1);
  const int b_begin = split * p.tiles_per_split, b_seen = (vis_wg + kQBlock - 1) / kQBlock;
  const int b_end = b_begin + p.tiles_per_split < b_seen ? b_begin + p.tiles_per_split : b_seen;
  const int b_codes = b_end < n_whole ? b_end : n_whole;  // blocks before it are held as codes

  // ---- the chunk's rows, where they are appended here: the head's only workgroup with its last block writes them, and reads them back behind a barrier
  if (qp.k_new && b_begin <= n_whole && n_whole < b_end) {
    q_fill_block<D>(qp, g, ((uint64_t)g * kQRing + (unsigned)n_whole % kQRing) * BLOCK, len - n_whole * kQBlock, tid, NT);
    __syncthreads();
  }

  // ---- the wavefront's rows: lane (c32, h) holds columns 16 ks + 8 h .. + 7 of row c32
  const int unit = wg * NW + w;
  int my_vis;  // keys that the lane's row sees, counted from the lane's first of a block
  qbf16x8 qf[KS];
  {
    const int r = unit * kRowsPerUnit + c32, row = r < rows ? r : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
    my_vis = (int)p.len_prev + tok + 1 - 4 * h;
    const __bf16* qrow = reinterpret_cast<const __bf16*>(p.q) + (uint64_t)(unsigned)(row + tok * (Hq - G) + g * G) * D;
    const float* cs = p.rope_cos ? p.rope_cos + (int64_t)tok * (D / 2) : nullptr;
    const float* sn = p.rope_cos ? p.rope_sin + (int64_t)tok * (D / 2) : nullptr;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = q_query<D>(qrow, 16 * ks + 8 * h, cs, sn);
  }
  // Keys that the wavefront's first row sees, and its last one
  const int vis_first = seen_by(unit * kRowsPerUnit), vis_last = unit * kRowsPerUnit < rows ? seen_by((unit + 1) * kRowsPerUnit - 1) : 0;

  // ---- a block on its way: K fragment (tile t, step, half) at ((t KS + step) 2 + half) 512, V fragment (tile t, step, tile of O^T, half) at
  // (((t 2 + step) JT + tile) 2 + half) 512, in two slots of each.  (By buffer accesses: a lane's place in a block is fixed and the
  // block's is a scalar.  A head's codes take at most 2^31 bytes.)
  // Piece j of a thread is K's (v = 0) or V's (v = 1), number `mine` of the block.
  auto v_of = [&](int j) __attribute__((always_inline)) -> int { return T == 2 ? j : w / (NW / 2); };
  const unsigned mine = T == 2 ? (unsigned)tid : (unsigned)tid % (NT / 2);
  __amdgpu_buffer_rsrc_t codes[T];
#pragma unroll
  for (int j = 0; j < T; ++j)
    codes[j] = __builtin_amdgcn_make_buffer_rsrc(qp.c.codes[v_of(j)] + (uint64_t)g * (uint64_t)qp.c.blocks * BLOCK, 0, (unsigned)qp.c.blocks * (unsigned)BLOCK, 0x00020000);
  // (scales by scalar loads: nobody writes them meanwhile)
  typedef const __attribute__((address_space(4))) floatx2* constants;
  const constants scales = (constants)(uintptr_t)(qp.c.scales + 2 * (uint64_t)g * (uint64_t)qp.c.blocks);
  quintx4 raw[T];
  auto load = [&](int j, int b) __attribute__((always_inline)) {
    raw[j] = __builtin_bit_cast(quintx4, __builtin_amdgcn_raw_buffer_load_b128(codes[j], mine * 16, (unsigned)b * (unsigned)BLOCK, 0));
  };
  auto put_half = [&](int j, int b, unsigned piece, int half, const qbf16x8& x) __attribute__((always_inline)) {
    const int v = v_of(j);
    const unsigned c = piece >> 6, key = piece & 63, kg = piece / D, col = piece % D;
    const unsigned in_k = (((key >> 5) * KS + c) * 2 * 32 + (key & 31)) * 16, in_v = ((((kg >> 1) * 2 * JT + (col >> 5)) * 2 + (kg & 1)) * 32 + (col & 31)) * 16;
    *reinterpret_cast<qbf16x8*>(lds + ((v ? in_v : in_k) + (unsigned)((2 * v + (b & 1)) * SLOT + half * (v ? JT * 1024 : 512)))) = x;
  };
  // Asks for block b, and puts what was asked for into LDS, as far as there is such a block
  auto load_any = [&](int j, int b) __attribute__((always_inline)) {
    if (b < b_codes) load(j, b);
  };
  auto store_any = [&](int j, int b) __attribute__((always_inline)) {
    unsigned me = mine;
    asm volatile("" : "+v"(me));  // (or what follows from it would be held in registers all the while)
    if (b < b_codes) {
#pragma unroll
      for (int half = 0; half < 2; ++half) put_half(j, b, me, half, q_widen_half(raw[j], half));
    } else if (b < b_end) {
      // the rows that are not a whole block, in bf16; places without a row hold anything, in V they become 0 (0 times it has to be 0)
      const int n = len - b * kQBlock, kg = (int)(me / D);
      const qbf16x8* at = reinterpret_cast<const qbf16x8*>(qp.c.ring[v_of(j)] + ((uint64_t)g * kQRing + (unsigned)b % kQRing) * BLOCK + me * 16);
      qbf16x8 x[2] = {at[0], at[1]};
      if (v_of(j) == 1) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * (kg >> 1) + 4 * (kg & 1) + 8 * (e >> 2) + (e & 3) >= n) x[e >> 3][e & 7] = (__bf16)0.f;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) put_half(j, b, me, half, x[half]);
    }
  };

  floatx16 o[JT];
  float m_run, l_run;
  auto clear = [&]() __attribute__((always_inline)) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
  };
  clear();

  constexpr floatx16 zero = {};
  // S^T of a block
  auto logits = [&](floatx16 (&s)[2], int b) __attribute__((always_inline)) {
    const unsigned char* buf = lds + (b & 1) * SLOT + l * 16;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const qbf16x8*>(buf + (t * KS + ks) * 1024), qf[ks], ks == 0 ? zero : s[t], 0, 0, 0);
      if (ks % 2) __builtin_amdgcn_sched_barrier(0);  // (four operands on their way at a time, for want of registers)
    }
  };
  // The reference, before a block's exponentials: masks S^T, and moves rows whose maximum, and what they have to be above it, asks for it.  (Whether it is looked at
  // depends on the wavefront's other rows, and whether a piece is done again on the workgroup's: a row among other rows may be rounded otherwise, the
  // same call gives the same bits.)
  auto reference = [&](floatx16 (&s)[2], int b, float to_log2, float above) __attribute__((always_inline)) {
    const int key0 = b * kQBlock;
    if (key0 + kQBlock > vis_first) {  // wave-uniform: some row does not see the whole block
      const int rel = my_vis - key0;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * t + 8 * (i >> 2) + (i & 3) >= rel) s[t][i] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
    mx = __builtin_fmaf(pair_max(mx), to_log2, above);
    const bool mine = mx > m_run + kStale || (m_run == -INFINITY && mx > -INFINITY);
    if (__any(mine)) {
      const float m2 = mine ? mx : m_run;
      const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m2);  // (without history: l = 0, O = 0)
      m_run = m2;
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= alpha;
    }
  };
  // The sum of a block's weights without the scale of V, which else comes with them
  auto plain_sum = [&](const floatx16 (&s)[2], float to_log2) __attribute__((always_inline)) -> float {
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], to_log2, -ref));
    return sum;
  };
  // A block's exponentials and outputs, one after the other
  auto attend = [&](const floatx16 (&s)[2], int b, float to_log2, float v_scale) __attribute__((always_inline)) {
    const float ref = (m_run == -INFINITY ? 0.f : m_run) - __builtin_amdgcn_logf(v_scale);
    qbf16x8 pf[2][2];
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], to_log2, -ref));
        sum += a;
        pf[t][i >> 3][i & 7] = (__bf16)a;
      }
    if (__builtin_expect(q_tiny(v_scale), 0))
      l_run += plain_sum(s, to_log2);
    else
      l_run = __builtin_fmaf(sum, __builtin_amdgcn_rcpf(v_scale), l_run);
    const unsigned char* buf = lds + (2 + (b & 1)) * SLOT + l * 16;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
#pragma unroll
        for (int j = 0; j < JT; ++j)
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const qbf16x8*>(buf + ((t * 2 + st) * JT + j) * 1024), pf[t][st], o[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // The same, laid out by hand, with S^T of the next block: 2 KS slots with a matrix instruction of S^T, 4 JT with one of O^T.  Behind each stands
  // an even share of what else there is to do: this block's exponentials, done by the time that O^T asks for them (after 7/8 of the slots), and the
  // codes of K of block b + 2 and V of block b + 1 that go into LDS.  Operands are read kAhead slots ahead.
  bool lost = false;
  auto turn = [&](const floatx16 (&s)[2], floatx16 (&x)[2], int b, float to_log2, float v_scale) __attribute__((always_inline)) {
    constexpr int SM = 2 * KS, OM = 4 * JT, NS = SM + OM, kAhead = 2;
    constexpr int WORDS = T * 8, E = NS - NS / 8;  // words of widened codes; slots with exponentials
    const unsigned char *kbuf = lds + ((b + 1) & 1) * SLOT + l * 16, *vbuf = lds + (2 + (b & 1)) * SLOT + l * 16;
    auto operand = [&](int i) __attribute__((always_inline)) -> qbf16x8 {  // of slot i
      return *reinterpret_cast<const qbf16x8*>(i < SM ? kbuf + ((i & 1) * KS + (i >> 1)) * 1024 : vbuf + (i - SM) * 1024);
    };
    qbf16x8 f[kAhead + 1];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) f[i] = operand(i);
    const float inv_v = __builtin_amdgcn_rcpf(v_scale), ref = (m_run == -INFINITY ? 0.f : m_run) - __builtin_amdgcn_logf(v_scale);
    const float far = fminf(kFar * v_scale, kMost);
    float sum = 0.f, last = 0.f;
    quintx4 pb[2][2], wide;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (i + kAhead < NS) f[(i + kAhead) % (kAhead + 1)] = operand(i + kAhead);
      const qbf16x8 a = f[i % (kAhead + 1)];
      const int j = i - SM;
      if (i < SM)
        x[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[i >> 1], i < 2 ? zero : x[i & 1], 0, 0, 0);
      else
        o[j % JT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(qbf16x8, pb[j / JT / 2][j / JT % 2]), o[j % JT], 0, 0, 0);
      if (i < E) {
#pragma unroll
        for (int e = 32 * i / E; e < 32 * (i + 1) / E; ++e) {
          const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], to_log2, -ref));
          sum += weight;
          if (e & 1) {
            bf16x2 pk;
            pk[0] = (__bf16)last;
            pk[1] = (__bf16)weight;
            pb[e >> 4][e >> 3 & 1][e >> 1 & 3] = __builtin_bit_cast(unsigned, pk);
          }
          last = weight;
        }
      }
#pragma unroll
      for (int k = WORDS * i / NS; k < WORDS * (i + 1) / NS; ++k) {
        wide[k % 4] = q_widen_word(raw[k / 8], k % 8);
        if (k % 4 == 3) put_half(k / 8, b + 2 - v_of(k / 8), mine, k / 4 % 2, __builtin_bit_cast(qbf16x8, wide));
      }
      if (T == 2 && i == NS / 2) load(0, b + 3);
      __builtin_amdgcn_sched_barrier(0);
    }
    load(T - 1, b + 3 - v_of(T - 1));
    l_run = __builtin_fmaf(sum, q_tiny(v_scale) ? 0.f : inv_v, l_run);
    if (__builtin_expect(__any(!(sum < far)), 0)) {
      // Logits far above their row's reference: it follows by a power of two.  Beyond what fp32 holds, of weights or, with V, of outputs, all is to be done
      // again.
      const float top = pair_max(sum * inv_v);
      lost |= !(pair_sum(sum * inv_v) < kLost && pair_sum(sum) < kMost);
      const int by = top >= kFar && top < kLost ? __builtin_amdgcn_frexp_expf(top) : 0;
      const float alpha = __builtin_amdgcn_ldexpf(1.f, -by);
      m_run += (float)by;
      l_run *= alpha;
#pragma unroll
      for (int jj = 0; jj < JT; ++jj)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[jj][i] *= alpha;
    }
  };

  // (Waited for here: in the loop the compiler would wait for the block that has just been asked for.)
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  floatx16 s[2], x[2];
  floatx2 scale;
  auto step = [&](floatx16 (&now)[2], floatx16 (&next)[2], int b) __attribute__((always_inline)) {
    const floatx2 scale_next = scales[(unsigned)(b + 1)];
    const float to_log2 = q_to_log2(scale.x, p.scale_log2e);
    // every row sees all of the block, and has a reference
    if (!__all(b * kQBlock + kQBlock <= vis_first && m_run != -INFINITY)) reference(now, b, to_log2, q_above(scale.y));
    if (__builtin_expect(q_tiny(scale.y), 0)) l_run += plain_sum(now, to_log2);
    turn(now, next, b, to_log2, scale.y);
    scale = scale_next;
    __syncthreads();
  };
  auto scale_of = [&](int b) __attribute__((always_inline)) -> floatx2 {
    return b < b_codes ? scales[(unsigned)b] : floatx2{1.f, 1.f};
  };
#pragma unroll 1
  for (bool again = false; b_begin < b_end; again = true) {  // the second time, if there is one, with every block's maximum
    int b = b_begin;
    asm volatile("" : "+s"(b));  // (or what follows from it would be held in registers for a second time)
#pragma unroll
    for (int j = 0; j < T; ++j) load_any(j, b);
#pragma unroll
    for (int j = 0; j < T; ++j) {
      store_any(j, b);
      if (v_of(j) == 0) {
        load_any(j, b + 1);
        store_any(j, b + 1);
      }
      load_any(j, b + 2 - v_of(j));
    }
    scale = scale_of(b);
    __syncthreads();
    logits(s, b);
    __syncthreads();  // (K of block b + 2 is going to take its place)
    // Turns laid out by hand: a wavefront's that has rows, as long as K of block b + 2 is codes or nobody's.  (Past the piece's end they ask for, and
    // widen, what is never used: what lies behind the piece, at most three blocks further on, which is the layer's own storage: its ring lies behind the codes and scales.)
    // Wavefronts without rows only widen: 37 tokens on 32K keys, five of eight with rows, 47.5 us a step; 4.5 more when they all multiplied.
    const int b_fast = again || !vis_last ? b : b_codes == b_end ? b_end : b_codes - 2;
#pragma unroll 1
    for (; b + 1 < b_fast; b += 2) {
      step(s, x, b);
      step(x, s, b + 1);
    }
#pragma unroll 1
    for (; b < b_end; ++b) {
#pragma unroll
      for (int j = 0; j < T; ++j) {
        store_any(j, b + 2 - v_of(j));
        load_any(j, b + 3 - v_of(j));
      }
      if (b * kQBlock < vis_last) {
        const float to_log2 = q_to_log2(scale.x, p.scale_log2e);
        reference(s, b, to_log2, b < b_codes ? q_above(scale.y) : again ? kQAboveRows : 0.f);
        attend(s, b, to_log2, scale.y);
        if (b >= b_codes) lost |= q_large<16>(o);
        if (b + 1 < b_end) logits(s, b + 1);
      }
      scale = scale_of(b + 1);
      __syncthreads();
    }
    if (again) break;
    int* flag = reinterpret_cast<int*>(lds);  // (behind the last barrier)
    if (tid == 0) *flag = 0;
    __syncthreads();
    if (lost) *flag = 1;
    __syncthreads();
    const int redo = *flag;
    __syncthreads();
    if (!redo) break;
    clear();
  }

  // ---- out, or what the piece leaves for the merge
  const float l_tot = pair_sum(l_run);
  int lane = threadIdx.x;
  asm volatile("" : "+v"(lane));  // (found again, not held through the loop)
  const int half = lane >> 5 & 1, r = unit * kRowsPerUnit + (lane & 31);
  if (r >= rows) return;
  const int t = (int)quot((unsigned)r, p.by_group), head = g * G + r - t * G;
  const int64_t at = (int64_t)t * Hq + head;
  if (p.n_splits == 1) {
    const float inv = 1.f / l_tot;
    __bf16* out = reinterpret_cast<__bf16*>(p.out) + at * D + 4 * half;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[j][i + e] * inv);
        *reinterpret_cast<bf16x4*>(out + 32 * j + 2 * i) = v;
      }
    if (p.lse && half == 0) p.lse[(int64_t)head * C + t] = (m_run + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f;
  } else {
    const int64_t piece = (int64_t)split * C * Hq + at;
    float* out = p.part_o + piece * D + 4 * half;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < 16; i += 4) *reinterpret_cast<floatx4*>(out + 32 * j + 2 * i) = floatx4{o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]};
    if (half == 0) *reinterpret_cast<floatx2*>(p.part_ml + piece * 2) = floatx2{m_run, l_tot};
  }
}

hipError_t launch_attn_q(const QAttnParams& p, int head_dim, int waves, hipStream_t s) {
  const dim3 grid(padded_grid(p.a.n_wgs)), block(waves * 64);
  if (head_dim == 128)
    hipLaunchKernelGGL((attn_q_kernel<128, 8>), grid, block, 0, s, p);
  else if (waves == 8)
    hipLaunchKernelGGL((attn_q_kernel<64, 8>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attn_q_kernel<64, 4>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
