// Attention of at most 16 packed (token, query head) rows per sequence and KV head on a cache in pages: decoding a batch of sequences.  A workgroup owns one
// sequence's rows of one KV head and a piece of its keys; the pieces of a sequence, as many as its length asks for, meet in the one that ends last.
//
// Every key is read once and next to nothing computed: bound by memory where there are many keys, by the chain of what a launch does once where there are few.
// So keys are dealt to four wavefronts in blocks (32, fp32 16) that run alone until their results meet in LDS, K and V come straight into registers, two
// blocks in flight a wavefront, on the 16x16x32 bf16 and 16x16x4 fp32 shapes (layouts as in attn_decode.hip: S^T = K Q^T has 16 keys as its rows; O^T = V^T P^T
// takes columns of V, a lane holding four keys of 16, those whose S^T it has).  fp32 is the fp32 instructions' own: 16 rows are an eighth of their time per byte.
//
// Pages: 16 keys lie in one (page_tokens is a multiple of 16), so that a tile's page is a scalar and its rows one buffer descriptor: the page's, with as many
// bytes as the tile has rows.  Rows that do not exist, of a page that is none or past the sequence's end, come back as zeros without traffic, so that nothing that
// lies there is ever multiplied; their logits are -inf.  64 blocks' page numbers are held by the wavefront's lanes.
//
// The step's new rows are not read from the cache: the one wavefront whose block they fall into takes them from k_new and v_new and stores them.
//
// 32 heads on 8, 128 wide: 256 sequences of 3000 to 5000 tokens on pages of 16 732 us, 5.7 TB/s; 64 of 16 to 16K 127, 4.8 TB/s; 4 of 128K 366, 5.8 TB/s; one of 300 tokens 7.3.
//
// bf16: neither queries nor keys are rounded on the way, P = 2^(S scale log2 e - m) is for P V (attn_decode.hip's rounding points but for the query's), row sums are
// fp32 from the unrounded P, m is stale by at most 2^16.
#include "meet.h"
#include "pcache.h"

namespace kvfold {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) unsigned uintx4;
typedef __attribute__((ext_vector_type(2))) unsigned uintx2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kPDecodeWaves = 4;  // (eight: never better, 300 keys 9.6 us for 8.8, 64 sequences of 500 31 for 26)

// The sum of the wavefront's values, for all its lanes
__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // lanes 1, 2, 4 and 8 down in the row of 16,
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);  // a row's last lane to the next row, of two
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);  // and lane 31 to the upper half
  return __builtin_amdgcn_readlane(x, 63);
}

template <class T, int D>
__global__ void __launch_bounds__(kPDecodeWaves * 64, 2) attn_pdecode_kernel(PAttnParams p) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int NW = kPDecodeWaves, NT = NW * 64;
  constexpr int ROWB = D * (int)sizeof(T), TILES = BF16 ? 2 : 1, BK = 16 * TILES;
  constexpr int KV = ROWB / 64;                // 16-byte vectors of a lane's share of a K row
  constexpr int J = D / 16;                    // matrix instructions of P V, each with 16 columns
  constexpr int CW = BF16 ? J : 4;             // columns side by side of a lane's share of a V row
  constexpr int VV = J / CW;                   // such shares
  constexpr int VWORDS = CW * (int)sizeof(T) / 4;
  constexpr float kStale = 16.0f;              // log2 units
  constexpr int ROWS = 16, OROW = D * 4 + 16;
  typedef __attribute__((ext_vector_type(VWORDS))) unsigned vvec;
  __shared__ __attribute__((aligned(16))) unsigned char red_o[NW * ROWS * OROW];
  __shared__ floatx2 red_ml[NW * ROWS];
  __shared__ int last;

  // (every line of the arguments is fetched now, in one round trip)
  asm volatile("" ::"s"(p.q), "s"(p.out), "s"(p.slots), "s"(p.table_stride), "s"(p.n_seqs), "s"(p.n_pieces), "s"(p.by_kv_heads.mul));
  // The longest sequences' last pieces first (from_end), which are whole; everybody's first one, which is what is left of its length, at the end.  Else everybody's first piece, and so
  // on: pieces that are not there, of which there are many where lengths decide, would hold up the others in front of them (8 equal sequences of 4000 keys 31.0 us, so 26.7).
  const int n_before = (int)quot(blockIdx.x, p.by_units), unit = (int)blockIdx.x - n_before * p.n_units, piece = p.from_end ? p.n_pieces - 1 - n_before : n_before;
  const int seq = (int)quot((unsigned)unit, p.by_kv_heads), g = unit - seq * p.n_kv_heads;
  const int tid = threadIdx.x, l = tid & 63, kg = l >> 4, c16 = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* table = p.tables + (int64_t)seq * p.table_stride;
  int pages[TILES];  // lane l: of the wavefront's block (the last multiple of 64) + l
  const bool known = !p.from_end && p.shared == 0.f;
  if (known) {  // where a piece begins is known: its pages are asked for together with the lengths (a tenth of the time of a short sequence's step)
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int64_t column = (((int64_t)piece * (p.piece / BK) + w + NW * l) * BK + 16 * t) >> p.page_log2;
      pages[t] = column < p.table_stride ? table[column] : -1;
    }
  }
  PagedSeq sq;
  {
    const int len = ((ConstPtr<int32_t>)(uintptr_t)p.lens)[seq];
    int from = seq, to = seq + 1;
    if (p.cu_new) {
      from = ((ConstPtr<int32_t>)(uintptr_t)p.cu_new)[seq];
      to = ((ConstPtr<int32_t>)(uintptr_t)p.cu_new)[seq + 1];
    }
    sq = paged_seq(from, to, len, p.n_tokens, p.max_new, p.max_len);
  }
  // The place of the one token, where there are no running sums (paged_one): asked for behind the lengths, and not waited for before it is needed (16 unlike sequences 24.2 us, in front of the
  // lengths' use 26.5, without it 23.9).
  int64_t place = 0;
  if (!p.cu_new && p.slots) place = ((ConstPtr<int64_t>)(uintptr_t)p.slots)[seq];
  int piece_keys = p.piece;
  if (p.shared != 0.f) {  // a workgroup's share of all keys: every workgroup adds up all lengths, which come with its own
    int steps = 0;        // (of 128 keys: a sum of fewer than 2^31)
    for (int s = l; s < p.n_seqs; s += 64) {
      const int len = p.lens[s];
      steps += (int)((unsigned)(len < 0 ? 0 : len > p.max_len ? p.max_len : len) + 127u) / 128;
    }
    const int share = (int)fminf(ceilf((float)wave_sum(steps) * p.shared), (float)(kPagedLongestPiece / 128)) * 128;
    piece_keys = share > piece_keys ? share : piece_keys;
  }
  const int n_pieces = paged_pieces(sq.len, piece_keys);
  if (sq.n == 0 || piece >= n_pieces || (uint64_t)place >= (uint64_t)p.n_places) return;

  const int Hq = p.n_q_heads, G = p.group, rows = sq.n * G, prev = sq.len - sq.n;

  // ---- the wavefront's blocks: every NW-th of the piece's.  New rows lie in the sequence's last two at most, so that a wavefront has at most one with new
  // rows, its last.
  const int b_all = (sq.len + BK - 1) / BK, per_piece = piece_keys / BK;
  int b_begin = piece * per_piece, b_end = b_begin + per_piece < b_all ? b_begin + per_piece : b_all;
  if (p.from_end) {  // what is left of the length is the first piece's
    b_end = b_all - (n_pieces - 1 - piece) * per_piece;
    b_begin = piece == 0 ? 0 : b_end - per_piece;
  }
  const int b_first = b_begin + w, n_blocks = b_first < b_end ? (int)((unsigned)(b_end - b_first + NW - 1) / (unsigned)NW) : 0;
  const bool fresh = p.k_new != nullptr;
  const int old = !fresh ? sq.len : prev > 0 ? prev : 0;  // rows that are read from the pages
  const int b_last = b_first + NW * (n_blocks - 1);
  const bool special = n_blocks > 0 && (b_last + 1) * BK > old && fresh;
  const int n_plain = n_blocks - (special ? 1 : 0);

  const int key_end = b_end * BK < sq.len ? b_end * BK : sq.len;
  auto fetch_pages = [&](int i0, bool there) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int key = (b_first + NW * (i0 + l)) * BK + 16 * t;
      const bool mine = i0 + l < n_blocks && key < key_end;
      if (!there && mine) pages[t] = table[(unsigned)key >> p.page_log2];
      if (!mine) pages[t] = -1;
    }
  };
  fetch_pages(0, known);

  // ---- Q: lane (c16, kg) holds the columns of row c16 that its shares of the K rows have
  const int row = c16 < rows ? c16 : rows - 1, tok = (int)quot((unsigned)row, p.by_group);
  const int my_vis = prev + tok + 1;
  uintx4 qf[KV];
  {
    const T* qrow = static_cast<const T*>(p.q) + (int64_t)(sq.first + tok) * p.q_stride + (g * G + row - tok * G) * D;
#pragma unroll
    for (int v = 0; v < KV; ++v) qf[v] = *reinterpret_cast<const uintx4*>(reinterpret_cast<const unsigned char*>(qrow) + v * 64 + kg * 16);
  }

  int limit = sq.len;  // keys from it on are taken as zeros
  struct Block {
    uintx4 k[TILES][KV];
    vvec v[TILES][4][VV];
    int gone;  // tiles of no page, a bit each
  };
  const unsigned k_lane = (unsigned)c16 * ROWB + (unsigned)kg * 16, v_lane = (unsigned)(4 * kg) * ROWB + (unsigned)c16 * (VWORDS * 4);
  const uint64_t head = (uint64_t)(unsigned)g * ((uint64_t)(unsigned)ROWB << p.page_log2);
  auto load_tile = [&](Block& x, int t, int page, int key0) __attribute__((always_inline)) {
    int n = (old < limit ? old : limit) - key0;
    n = n < 0 ? 0 : n > 16 ? 16 : n;
    const bool there = (unsigned)page < (unsigned)p.n_pages;
    const uint64_t at = (uint64_t)(unsigned)(there ? page : 0) * p.page_bytes + head + (unsigned)((key0 & ((1 << p.page_log2) - 1)) * ROWB);
    const unsigned bytes = there ? (unsigned)(n * ROWB) : 0u;
    const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(static_cast<unsigned char*>(p.k_pages) + at, 0, bytes, kRawBuffer);
    const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(static_cast<unsigned char*>(p.v_pages) + at, 0, bytes, kRawBuffer);
#pragma unroll
    for (int v = 0; v < KV; ++v) x.k[t][v] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(kb, k_lane + v * 64, 0, 0));
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VV; ++j) {
        if constexpr (VWORDS == 4)
          x.v[t][r][j] = __builtin_bit_cast(vvec, __builtin_amdgcn_raw_buffer_load_b128(vb, v_lane + r * ROWB + j * 256, 0, 0));
        else
          x.v[t][r][j] = __builtin_bit_cast(vvec, __builtin_amdgcn_raw_buffer_load_b64(vb, v_lane + r * ROWB + j * 256, 0, 0));
      }
    x.gone |= (int)!there << t;
  };
  // Block i of the wavefront's; past the plain ones there is nothing to ask for, and nothing is
  auto load = [&](Block& x, int i) __attribute__((always_inline)) {
    if ((i & 63) == 0 && i > 0 && i < n_plain) fetch_pages(i, false);
    x.gone = 0;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int page = __builtin_amdgcn_readlane(pages[t], i & 63);
      load_tile(x, t, i < n_plain ? page : -1, (b_first + NW * i) * BK + 16 * t);
    }
  };

  floatx4 o[J];
  float m_run, l_run;

  auto outputs = [&](const Block& x, const floatx4 (&pw)[TILES]) __attribute__((always_inline)) {
    if constexpr (BF16) {
      uintx4 pb;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          bf16x2 pk;
          pk[0] = (__bf16)pw[t][2 * e];
          pk[1] = (__bf16)pw[t][2 * e + 1];
          pb[2 * t + e] = __builtin_bit_cast(unsigned, pk);
        }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        uintx4 a;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          a[k] = __builtin_amdgcn_perm(x.v[k >> 1][2 * (k & 1) + 1][0][j >> 1], x.v[k >> 1][2 * (k & 1)][0][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, pb), o[j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[0][r][j / 4][j % 4]), pw[0][r], o[j], 0, 0, 0);
    }
  };
  auto block = [&](const Block& x, int b) __attribute__((always_inline)) {
    floatx4 s[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < KV; ++v)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        if constexpr (BF16) {
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[t][v]), __builtin_bit_cast(bf16x8, qf[v]), s[t], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.k[t][v][e]), __uint_as_float(qf[v][e]), s[t], 0, 0, 0);
        }
      }
    const int key0 = b * BK;
    const bool masked = key0 + BK > prev + 1 || x.gone;  // wave-uniform: some row does not see the whole block
    if (masked) {
      const int rel = my_vis - key0 - 4 * kg;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * t + e >= rel || x.gone >> t & 1) s[t][e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < TILES; ++t) mx = fmaxf(mx, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
    mx = pair_max(row16_max(mx)) * p.scale_log2e;
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
    const float ref = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], p.scale_log2e, -ref));
        l_run += s[t][e];
      }
    outputs(x, s);
  };

  // Once; and where outputs are not finite, which may come from values that their rows do not see (0 times them is not 0), once more for each token, with what it does not
  // see as zeros.
#pragma unroll 1
  for (int pass = -1; pass < sq.n; ++pass) {
    if (pass >= 0) {
      limit = prev + pass + 1;
      fetch_pages(0, false);
    }
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    Block x, y;
    load(x, 0);
    if (special) {
      // ---- the block with new rows: what lies in the pages, zeros from there on, and the new rows in their stead, which are stored (16 bytes of a row's K or V a lane)
      const int key0 = b_last * BK;
      y.gone = 0;
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int key = key0 + 16 * t;
        int page = __builtin_amdgcn_readlane(pages[t], (n_blocks - 1) & 63);
        if (__builtin_expect(n_blocks > 64, 0)) {
          page = -1;
          if (key < sq.len) page = __builtin_amdgcn_readfirstlane(table[(unsigned)key >> p.page_log2]);
        }
        load_tile(y, t, page, key);
      }
      const int64_t new_row = p.kv_stride * (int64_t)sizeof(T);
      const unsigned char* knew = static_cast<const unsigned char*>(p.k_new) + (int64_t)(sq.first - prev) * new_row + g * ROWB;
      const unsigned char* vnew = static_cast<const unsigned char*>(p.v_new) + (int64_t)(sq.first - prev) * new_row + g * ROWB;
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int key = key0 + 16 * t + c16, vkey = key0 + 16 * t + 4 * kg;
        if (y.gone >> t & 1) continue;  // (seen by nobody)
        if (key >= old && key < limit)
#pragma unroll
          for (int v = 0; v < KV; ++v) y.k[t][v] = *reinterpret_cast<const uintx4*>(knew + (int64_t)key * new_row + v * 64 + kg * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vkey + r >= old && vkey + r < limit)
#pragma unroll
            for (int v = 0; v < VV; ++v)
              y.v[t][r][v] = *reinterpret_cast<const vvec*>(vnew + (int64_t)(vkey + r) * new_row + (unsigned)c16 * (VWORDS * 4) + v * 256);
      }
      constexpr int CH = ROWB / 16;
      const int from = old > key0 ? old : key0, to = key0 + BK < sq.len ? key0 + BK : sq.len;
#pragma unroll 1
      for (int e = l; pass < 0 && e < (to - from) * (2 * CH); e += 64) {
        const int key = from + e / (2 * CH), c = e % CH * 16;
        const bool is_v = e / CH & 1;
        const int64_t slot = p.slots[sq.first + key - prev];
        const uintx4 row16 = *reinterpret_cast<const uintx4*>((is_v ? vnew : knew) + (int64_t)key * new_row + c);
        const uint64_t at = ((uint64_t)slot >> p.page_log2) * p.page_bytes + head + ((uint64_t)slot & ((1u << p.page_log2) - 1)) * ROWB + (unsigned)c;
        if ((uint64_t)slot < (uint64_t)p.n_places) *reinterpret_cast<uintx4*>(static_cast<unsigned char*>(is_v ? p.v_pages : p.k_pages) + at) = row16;
      }
      block(y, b_last);
    }
    if (n_plain > 0) {
      int i = 0;
#pragma unroll 1
      while (true) {
        load(y, i + 1);
        asm volatile("" ::: "memory");
        block(x, b_first + NW * i);
        if (++i >= n_plain) break;
        load(x, i + 1);
        asm volatile("" ::: "memory");
        block(y, b_first + NW * i);
        if (++i >= n_plain) break;
      }
    }

    // ---- the wavefronts' results meet in LDS: [wavefront][row][D] and [wavefront][row] (m, l)
    const float l_tot = pair_sum(row16_sum(l_run));
    if (c16 < rows && (pass < 0 || tok == pass)) {
      float* mine = reinterpret_cast<float*>(red_o + (w * ROWS + c16) * OROW);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < J; j += 4)  // columns CW m + j of share 0, or 64 (j / 4) + 4 m + j % 4, m = 4 kg + r
          *reinterpret_cast<floatx4*>(mine + (BF16 ? CW * (4 * kg + r) + j : 16 * j + 4 * (4 * kg + r))) = floatx4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
      if (kg == 0) red_ml[w * ROWS + c16] = floatx2{m_run, l_tot};
    }
    if (pass < 0) {
      if (sq.n == 1) break;
      float check = 0.f;  // (0 as long as all are finite)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) check = __builtin_fmaf(o[j][r], 0.f, check);
      if (__builtin_expect(!__any(check != 0.f), 1)) break;
    }
  }
  __syncthreads();

  constexpr int V = D / 4;  // 16-byte column vectors of a row
  const int c = tid % V;
  const uint64_t part = (uint64_t)(unsigned)unit * (unsigned)p.n_pieces;
  const unsigned part_rows = (unsigned)(n_pieces * p.unit_rows);
  const __amdgpu_buffer_rsrc_t po = __builtin_amdgcn_make_buffer_rsrc(p.part_o + part * (unsigned)(p.unit_rows * D), 0, part_rows * (D * 4u), kRawBuffer);
  const __amdgpu_buffer_rsrc_t pml = __builtin_amdgcn_make_buffer_rsrc(p.part_ml + part * (unsigned)(p.unit_rows * 2), 0, part_rows * 8u, kRawBuffer);
  auto result = [&](int r, const floatx4& acc, float M, float L) __attribute__((always_inline)) {
    const int t = (int)quot((unsigned)r, p.by_group), h = g * G + r - t * G;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T* out = static_cast<T*>(p.out) + ((int64_t)(sq.first + t) * Hq + h) * D + c * 4;
    if constexpr (BF16) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(L == 0.f ? 0.f : acc[e] * inv);
      *reinterpret_cast<bf16x4*>(out) = v;
    } else {
      floatx4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = L == 0.f ? 0.f : acc[e] * inv;
      *reinterpret_cast<floatx4*>(out) = v;
    }
    if (p.lse && c == 0) p.lse[(int64_t)h * p.n_tokens + sq.first + t] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
  };
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
      const floatx4 from = *reinterpret_cast<const floatx4*>(red_o + (ww * ROWS + r) * OROW + c * 16);
      if (ml[ww].y == 0.f) continue;  // it saw no key
      const float f = __builtin_amdgcn_exp2f(ml[ww].x - M);
      L += f * ml[ww].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += f * from[e];
    }
    if (n_pieces == 1) {
      result(r, acc, M, L);
    } else {
      const unsigned at = (unsigned)(piece * p.unit_rows + r);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, acc), po, at * (D * 4u) + (unsigned)c * 16u, 0, kDeviceScope);
      if (c == 0) __builtin_amdgcn_raw_buffer_store_b64(uintx2{__float_as_uint(M), __float_as_uint(L)}, pml, at * 8u, 0, kDeviceScope);
    }
  }
  if (n_pieces == 1) return;
  // ---- the last of the sequence's pieces to have stored its results merges them, in their order (its counter is back at zero then)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) last = atomicInc(p.counters + (uint64_t)(unsigned)unit * kPagedMeetStride, (unsigned)n_pieces - 1u) == (unsigned)n_pieces - 1u;
  __syncthreads();
  if (!last) return;
#pragma unroll 1
  for (int r = tid / V; r < rows; r += NT / V) {
    float M = -INFINITY, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int N = 8;  // pieces in flight; those past the last lie outside the buffer and bring zeros: no keys
#pragma unroll 1
    for (int i0 = 0; i0 < n_pieces; i0 += N) {
      uintx4 from[N];
      uintx2 ml[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned at = (unsigned)((i0 + i) * p.unit_rows + r);
        ml[i] = __builtin_bit_cast(uintx2, __builtin_amdgcn_raw_buffer_load_b64(pml, at * 8u, 0, kDeviceScope));
        from[i] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(po, at * (D * 4u) + (unsigned)c * 16u, 0, kDeviceScope));
      }
      float top = M;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (ml[i][1] == 0u) {
          ml[i][0] = __float_as_uint(-INFINITY);
          from[i] = uintx4{0u, 0u, 0u, 0u};
        }
        top = fmaxf(top, __uint_as_float(ml[i][0]));
      }
      const float ref = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(M - ref);
      M = top;
      L *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float f = __builtin_amdgcn_exp2f(__uint_as_float(ml[i][0]) - ref);
        L = __builtin_fmaf(__uint_as_float(ml[i][1]), f, L);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(__uint_as_float(from[i][e]), f, acc[e]);
      }
    }
    result(r, acc, M, L);
  }
}

hipError_t launch_attn_pdecode(const PAttnParams& p, int head_dim, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)p.n_units * (unsigned)p.n_pieces), block(kPDecodeWaves * 64);
  if (bf16 && head_dim == 128)
    hipLaunchKernelGGL((attn_pdecode_kernel<__bf16, 128>), grid, block, 0, s, p);
  else if (bf16)
    hipLaunchKernelGGL((attn_pdecode_kernel<__bf16, 64>), grid, block, 0, s, p);
  else if (head_dim == 128)
    hipLaunchKernelGGL((attn_pdecode_kernel<float, 128>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attn_pdecode_kernel<float, 64>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace kvfold
