// Attention of a chunk of new tokens over a paged cache.
//
// A query head's rows and those of the other heads that share its kv head are COLUMNS of one problem (column c of a sequence: token c / g, head c % g of the group of g): they
// read the same keys and values.  Scores and outputs are computed transposed on v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T = V^T P^T, so a lane owns one column: its running
// maximum and sum and the rescaling are lane-local, and a score's place in the accumulator is where the second product wants its weight.  One pass over the keys with the running
// maximum and sum of the softmax; everything but the operands of the matrix instructions is fp32.
//
// fp32 operands are exact sums of three bf16 pieces (8 bits each of the 24), and of the nine products of two such sums the six of at least 2^-15 of the largest are kept: what is
// left out is 2^-22 of a product at most.  The cache's first pieces are cut off and not rounded, since the largest numbers would round to infinity (and their other pieces to NaN).  bf16
// operands are one piece.  Weights are three pieces for fp32 queries and one for bf16: that rounds a weight by at most 2^-8 of itself, as the output rounds (their sum takes them unrounded).  The
// error against 64 bits is 0.0022 to 0.0023 of the result's norm, 0.0017 of which is the output's rounding alone; a second piece would be half as many products again.
//
// Two shapes.  WIDE (more than 32 columns a sequence and kv head): four waves of 32 columns share tiles of tokens in LDS.  Narrow: one block of 32 columns, the four waves take every
// fourth tile and join at the end.  Where sequences, kv heads and column blocks do not fill the chip, the token range is split over work-groups and k_chunk_attn_join adds the parts up.
//
// What bounds it, and what it reaches (us a call, joining with it).  A batch of 64 tokens over 1k to 16k tokens each, 64 / 8 heads of 128, bf16: 406, the cache once at 5.6 TB/s (a bare read in
// the same order reaches 6.0); tiles go to LDS without registers, a wave's next keys under way while it works on the values.  1536 and 509 rows behind a window of 4096 and a cap, 32 / 8 heads, bf16:
// 191, 0.63 PFLOP/s of visible products: per tile 32 matrix instructions beside 460 vector ones (mask, cap, exponent, sums), which share a SIMD's two waves; the matrix unit is busy a quarter of the
// time.  2011 fp32 rows, 32 heads of 80: 171: 72 matrix and 630 vector instructions a tile (making the pieces, also in waves that have nothing to multiply: a third), the matrix unit busy a third of the
// time, and the last rows' blocks, which see 63 tiles, alone on their CU at the end.  Four trees of 26 nodes, fp32 over bf16, about 2000 tokens: 29, five tiles of 3.4 one after the other, 6 until the
// first tile is there, 6 for joining.  One token over 701, fp32: 19, all of it latency.
//
// 8-bit codes are exact in bf16, so the products are those of a bf16 cache.  A block has at least 16 tokens: 16 scores share a key scale, which stands in the constant that takes scores to powers of
// two (or to the cap's tangent), and their weights a value scale.  fp32 weights are multiplied with it before they become pieces; a bf16 weight takes it as log2 in its exponent, so that it is rounded
// once (scales below 2^-96 count as 2^-96, or below 2^-64 as 2^-64 beside one above 2^96: none is lost to the least exponent).  The sum takes weights as they are: with rounded ones a row of
// few tokens can be off by 2^-7 of its weights, twice what a weight's rounding is.  The maximum stands where the largest weight times its scale is a power of two, and is not rounded: 0.0019
// of the result's norm off where some hundred tokens are seen, 0.0017 of which is the output's rounding, and 0.0022 to 0.0023 where thousands weigh about alike; standing at the largest score
// 0.0022 to 0.0026 and 0.0025, with rounded weights in the sum 0.0020 to 0.0024 and 0.0023 (and two instructions a pair of weights more: 2045 rows 221 us for 214); weights of two pieces
// 0.0017, 254 us.  The narrow shape brings codes to LDS as they are and makes bf16 of what each wave reads (RAW); in the wide one four waves would do so four times, so a tile's codes are
// parked in LDS and become bf16 between the products of the tile before.  64 tokens over 1k to 16k each, 64 / 8 heads, e4m3: 222 us, 5.1 TB/s of cache (lengths all alike 5.4 to 5.8); 510
// vector instructions a tile beside 32 products, the matrix unit busy 14 %.  1536 and 509 rows behind a window and a cap, bf16: 217, 760 vector instructions a tile, 128 of them what makes
// bf16 of the codes; busy 22 %.  Four trees of 26 nodes, fp32 over int8: 33, 5 of it joining.  One token over 701, fp32: 12.6.
//
// Registers: fp32 queries over a bf16 cache of 128 hold all 256 and spill (3 and, with cap or slopes, 17 of the wide shape, 7 and 6 of the narrow), which is a few of their loads a tile; over codes of 128
// three at most; no other shape spills vector registers.
//
// A wave issues a vector instruction every 4.75 cycles and a matrix instruction takes the matrix unit 33, in whose shadow seven vector instructions fit if they stand between the matrix
// instructions: the compiler does not put them there, so the order in which pieces and weights are made is written out, a step a product.
#pragma once
#include "rows.h"
#include "rope.h"
#include "codes.h"
#include <type_traits>

typedef short s16x4 __attribute__((ext_vector_type(4)));

struct ChunkAttnDev {
  const void* q; void* out;
  long long q_row, q_head, out_row, out_head;
  int H, window;
  float scale, softcap;                    // scale >= 0: the sign is q_flip's
  uint32_t q_flip;                         // 0x8000 in both halves: the queries change sign
  const float* slopes; const int* prefix;
  ChunkDev chunk; PagedDev kv;
  int col_blocks, splits, split_tiles;     // parts of the token range at most, tiles of one
  int turn;                                // column blocks in descending order before the others ascend
  int lane_pages;                          // pages of fewer than 8 tokens: every lane looks its own up
  float* part_o; float* part_ml;           // [row][head][split][DH], [row][head][split][maximum, sum]
  const float *k_scale, *v_scale;          // a cache of codes: scale of block b of a page's kv head at page * scale_page + head * scale_head + b
  long long scale_page, scale_head;
  int block_shift;
};
// Types of a cache of 8-bit codes.
struct e4m3_t { uint8_t bits; };
struct int8_code_t { int8_t bits; };

// What a column block of a sequence has to visit: tiles [0, n_prefix) and from first on, n_tiles in all; and what its rows have in common.
struct ColumnRange {
  int row0, n, keys, base, prefix, own0;   // first row, rows, tokens, tokens in front of the tree, prefix, index of row 0
  bool tree;
  int n_prefix, first, n_tiles;
  int full_to, full_from;                  // tokens below full_to are in order for every row, tokens from full_from on inside every row's window
};
template <int KT>
__device__ inline ColumnRange column_range(const ChunkAttnDev& A, int s, int col0, int cols, int g) {
  ColumnRange c;
  const int r0 = min(max(0, A.chunk.row_start[s]), A.chunk.n_rows), r1 = min(A.chunk.row_start[s + 1], A.chunk.n_rows);
  const int n_all = max(0, r1 - r0);
  c.row0 = r0;
  c.n = min(n_all, A.chunk.max_rows);
  c.keys = chunk_keys(A.chunk, A.kv, s);
  c.tree = A.chunk.tree_mask != nullptr;
  c.base = c.tree ? min(max(0, A.chunk.tree_base[s]), 1 << 30) : 0;   // (positions count from it, also where fewer tokens may be read)
  c.own0 = c.tree ? c.base : min(max(0, A.chunk.key_len[s]), 1 << 30) - n_all;
  c.prefix = A.prefix ? min(A.prefix[s], c.tree ? c.base : c.keys) : 0;
  c.prefix = max(0, c.prefix);
  const int i_lo = col0 / g, i_hi = min(c.n - 1, (col0 + cols - 1) / g);
  const int own_lo = c.tree ? c.base : c.own0 + i_lo, own_hi = c.tree ? c.base + 63 : c.own0 + i_hi;
  const int end = min(c.keys, max(own_hi + 1, c.prefix));
  const int lo = A.window > 0 ? max(0, own_lo - A.window + 1) : 0;
  c.n_prefix = lo > 0 ? (min(c.prefix, end) + KT - 1) / KT : 0;
  c.first = max(c.n_prefix, lo / KT);
  c.n_tiles = i_lo >= c.n || end <= 0 ? 0 : c.n_prefix + max(0, (end + KT - 1) / KT - c.first);
  c.full_to = min(c.keys, max(c.tree ? c.base : own_lo + 1, c.prefix));
  c.full_from = A.window > 0 ? own_hi - A.window + 1 : 0;
  return c;
}

__device__ __forceinline__ uint64_t low_ones(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1ull; }

// The upper halves of two fp32 numbers: their first pieces.
__device__ __forceinline__ uint32_t upper_pair(float a, float b) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u); }
// Eight numbers as exact sums of three bf16 pieces, the first of which is cut off (NEAREST: rounded, but where that is infinite).  (Of what is not finite the first is the same, but for a signalling
// NaN, which may become infinite; the others are NaN.)
template <bool NEAREST> __device__ __forceinline__ void pieces(const float* x, bf16x8* p) {
  u32x4 h[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
    h[0][i] = upper_pair(a, b);
    if constexpr (NEAREST) {
      const uint32_t n = bf16_pair(a, b);
      if ((n & 0x7F80u) != 0x7F80u) h[0][i] = (h[0][i] & 0xFFFF0000u) | (n & 0xFFFFu);
      if ((n & 0x7F800000u) != 0x7F800000u) h[0][i] = (h[0][i] & 0xFFFFu) | (n & 0xFFFF0000u);
    }
#pragma unroll
    for (int j = 1; j < 3; ++j) {
      a -= __builtin_bit_cast(float, h[j - 1][i] << 16);
      b -= __builtin_bit_cast(float, h[j - 1][i] & 0xFFFF0000u);
      h[j][i] = bf16_pair(a, b);
    }
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) p[j] = __builtin_bit_cast(bf16x8, h[j]);
}
__device__ __forceinline__ bool not_finite(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) == 0x7F800000u; }
// Not 0 if one of the eight bf16 numbers is not finite: an exponent of ones carries into the sign's place.
__device__ __forceinline__ uint32_t exponents(u32x4 v) {
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7F807F80u) + 0x00800080u;
  return any & 0x80008000u;
}
__device__ __forceinline__ uint32_t not_finite_any(f32x4 x) {
  const u32x4 u = __builtin_bit_cast(u32x4, x);
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (u[i] & 0x7F800000u) + 0x00800000u;
  return any & 0x80000000u;
}
// Eight elements of a token in flight, and their pieces.
template <typename CT> struct Raw8;
template <> struct Raw8<bf16_t> {
  u32x4 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = *(const u32x4*)p; }
  __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
  template <bool NEAREST = false> __device__ __forceinline__ void split(bf16x8* p) const { p[0] = __builtin_bit_cast(bf16x8, v); }
};
template <> struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ uint32_t bad() const { return not_finite_any(a) | not_finite_any(b); }
  template <bool NEAREST = false> __device__ __forceinline__ void split(bf16x8* p) const {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    pieces<NEAREST>(x, p);
  }
};

// Eight codes as bf16 numbers: exact (at most four or seven significant bits).
__device__ __forceinline__ bf16x8 coded8(u32x2 u, e4m3_t) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 h;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    h[2 * i] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.f, false));
    h[2 * i + 1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.f, true));
  }
  return __builtin_bit_cast(bf16x8, h);
}
__device__ __forceinline__ bf16x8 coded8(u32x2 u, int8_code_t) {
  u32x4 h;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = u[i >> 1] >> (i & 1 ? 16 : 0);
    h[i] = upper_pair((float)(int)(int8_t)w, (float)(int)(int8_t)(w >> 8));
  }
  return __builtin_bit_cast(bf16x8, h);
}

// Where 16 bytes (8 elements, piece c) of token t lie in a tile in LDS, in units of 8 elements.  Keys are read a token a lane: eight consecutive tokens' pieces lie in eight different
// 16-byte columns.  Values are read transposed, four tokens by 64 bytes at a time: those lie in four different 64-byte columns.  (Rows of 96 elements, 3/4 of the banks, put four tokens into
// four different 64-byte columns by themselves.)
template <int ROW> __device__ __forceinline__ int k_place(int t, int c) { return t * (ROW / 8) + (c ^ (ROW == 96 ? t >> 2 & 3 : t & 7)); }
template <int ROW> __device__ __forceinline__ int v_place(int t, int c) { return t * (ROW / 8) + (c ^ (ROW == 128 ? (t & 3) << 2 : ROW == 64 ? (t & 2) << 1 : 0)); }

// RAW: 16 codes (piece c) of token t lie in piece c ^ turn(t) of its row.  Keys are read a token a lane, 16 lanes at a time: 16 tokens' pieces lie in 16 different 16-byte columns; values
// transposed, 16 tokens by 32 bytes at a time: twice in each of the 64 banks.
template <int ROW> __device__ __forceinline__ int raw_k_turn(int t) { return ROW == 128 ? t >> 1 & 7 : t >> 2 & 3; }
template <int ROW> __device__ __forceinline__ int raw_v_turn(int t) { return ROW == 128 ? (t >> 1 & 3) << 1 : (t >> 2 & 1) << 1; }
// Lane l of 16 gets code l of the eight 16-code rows whose l / 2-th this address is in.
__device__ __forceinline__ u32x2 read_transposed8(const char* p) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p));
}
// Not 0 if one of the e4m3 codes is NaN: seven ones carry into the sign's place.
__device__ __forceinline__ uint32_t nan_codes(u32x4 v) {
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7F7F7F7Fu) + 0x01010101u;
  return any & 0x80808080u;
}

__device__ __forceinline__ s16x4 read_transposed(const bf16_t* p) {   // lane l of 16 gets element l of the four 16-element rows whose l / 4-th this address is in
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

// Tokens of a tile, by shape, whether queries are fp32, and bytes of an element of the cache.
constexpr int tile_tokens(bool wide, bool fp32, int bytes) { return (bytes == 1 && !fp32) || (bytes == 2 && wide) ? 64 : 32; }

template <typename T, typename CT, int DH_, bool WIDE_, bool MODS_>
struct ChunkAttn {
  static constexpr int DH = DH_, NQ = sizeof(T) == 4 ? 3 : 1, NK = sizeof(CT) == 4 ? 3 : 1, NP = NQ > NK ? NQ : NK;
  static constexpr bool WIDE = WIDE_, MODS = MODS_, CODED = sizeof(CT) == 1;
  // bf16 caches go from memory to LDS without passing through registers (DIRECT); fp32 ones are split into their pieces on the way.  The narrow shape has fp32 keys in registers.
  // Codes do so in the narrow shape, as they are (RAW: a wave has its tile for itself, and makes bf16 of what it reads); in the wide one they become bf16 on the way, once for four waves.
  static constexpr bool DIRECT = sizeof(CT) == 2, RAW = CODED && !WIDE, KEYS_IN_LDS = WIDE || NK == 1;
  static constexpr int KT = tile_tokens(WIDE, NQ == 3, sizeof(CT)), KB = KT / 32, KSN = DH / 16, DB = DH / 32;
  static constexpr int COLS = WIDE ? 128 : 32;
  static constexpr int ROW = (DIRECT || RAW) && DH == 96 ? 128 : DH;   // elements of a token in LDS (a DIRECT load fills 1 KiB: whole tokens)
  static constexpr int PART = DH <= 64 ? 64 : 128;                // and in the workspace
  static constexpr int TILE = RAW ? KT * ROW / 2 : KT * ROW;      // elements (of 2 bytes) of a piece of a tile
  static constexpr int OWNERS = WIDE ? 1 : 4;                     // waves with a tile of their own
  static constexpr int K_ELTS = KEYS_IN_LDS ? OWNERS * NK * TILE : 8, V_ELTS = OWNERS * NK * TILE;   // of one buffer
  static constexpr bool TWO = WIDE;                               // buffers
  static constexpr int JOIN = WIDE ? 0 : 2 * (16 * DB + 2) * 64 * 2;   // elements (of 2 bytes) that joining the waves takes
  static constexpr int V0_ELTS = V_ELTS > JOIN ? V_ELTS : JOIN;
  static constexpr int LDS = 2 * ((TWO ? 2 : 1) * K_ELTS + V0_ELTS + (TWO ? V_ELTS : 0));
  // The products of pieces that are kept, n-th of them: a piece of the cache, one of the columns (queries, weights).  Small ones come first, and of three cache pieces each is done with as soon
  // as can be, so that the next one's can take its registers.
  static constexpr int PRODUCTS = NQ * NK == 9 ? 6 : NQ * NK;
  static constexpr int cache_piece(int n) { return NK == 1 ? 0 : n == 0 ? 2 : n < 3 ? 1 : 0; }
  static constexpr int column_piece(int n) { return NQ == 1 ? 0 : NK == 1 ? 2 - n : n == 0 ? 0 : n < 3 ? 2 - n : 5 - n; }
  static constexpr bool done_with(int n) { return NK == 3 ? n == 0 || n == 2 || n == 5 : n == PRODUCTS - 1; }   // the cache piece of product n
  static constexpr int WAVES = NK == 3 && (DH == 128 || (DH == 96 && !WIDE)) ? 1 : 2;      // a SIMD holds (by registers)
  static constexpr bool SPLIT = WIDE && NK == 3;                   // fp32 keys and values go through LDS in pieces
  static constexpr int RUNS = DH == 64 ? 4 : 8;                   // CODED, WIDE: runs of 16 codes of a token
  static constexpr int PARKED = CODED && WIDE ? 2 * 8 * 256 * ((KT * RUNS + 255) / 256) : 8;
  static constexpr int ITEMS = SPLIT ? KT * DH / 4 / 256 : CODED ? (KT * RUNS + 255) / 256 : KT * DH / 8 / 64;   // runs of 4 (SPLIT) or 8 elements a thread fetches of the values, and of the keys if they go through LDS
};

struct ScoreRow {
  float v[16];
  __device__ __forceinline__ float& operator[](int i) { return v[i]; }
};
template <bool FIRST, typename A, typename B> __device__ __forceinline__ auto& one_of(A& a, B& b) {
  if constexpr (FIRST) return a;
  else return b;
}

typedef __attribute__((address_space(3))) bf16_t* lds_ptr;
// At most N vector-memory operations of this wave under way; all of its LDS operations done.  No access to memory moves across.
template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}

template <typename P, typename T, typename CT>
__global__ __launch_bounds__(256, P::WAVES) void k_chunk_attn(const ChunkAttnDev A) {
  constexpr int DH = P::DH, ROW = P::ROW, NQ = P::NQ, NK = P::NK, KT = P::KT, KB = P::KB, KSN = P::KSN, DB = P::DB, COLS = P::COLS, TILE = P::TILE, ITEMS = P::ITEMS;
  constexpr bool WIDE = P::WIDE, MODS = P::MODS, DIRECT = P::DIRECT, CODED = P::CODED, RAW = P::RAW;
  // (arrays of their own: the compiler tells reads of one from loads on their way into another)
  __shared__ __attribute__((aligned(16))) bf16_t k_lds0[P::K_ELTS], k_lds1[P::TWO ? P::K_ELTS : 8], v_lds0[P::V0_ELTS], v_lds1[P::TWO ? P::V_ELTS : 8];
  __shared__ __attribute__((aligned(16))) bf16_t parked[P::PARKED];  // CODED, WIDE: the codes of the tile after the next
  __shared__ int s_bad[2];                                        // WIDE, not DIRECT: number of the last tile in a buffer whose values are not all finite
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane & 31, hh = lane >> 5;
  // The lane, worked out anew: inside the loop, what can be had from the thread's number in an instruction or two is not kept (the widest shapes hold all 256 registers).
  auto lane_now = []() -> int { int l = threadIdx.x; asm volatile("" : "+v"(l)); return l & 63; };
  const int kvh = blockIdx.x % A.kv.n_kv_heads, part = blockIdx.x / A.kv.n_kv_heads, s = blockIdx.y, g = A.H / A.kv.n_kv_heads, dh = A.kv.head_dim;
  // Blocks of the last rows see most and go first.  Where all work-groups are resident at once, two a CU, the second half ascends, so that a CU's two see as much as another's.
  const int nth = part % A.col_blocks, split = part / A.col_blocks, cb = nth < A.turn ? A.col_blocks - 1 - nth : nth - A.turn;
  const int col0 = cb * COLS;
  const ColumnRange R = column_range<KT>(A, s, col0, COLS, g);
  if (col0 >= R.n * g) return;
  const int t_begin = split * A.split_tiles, t_end = min(R.n_tiles, t_begin + A.split_tiles);
  if (t_begin >= t_end && split > 0) return;
  const bool whole = R.n_tiles <= A.split_tiles;

  // this lane's column
  const int wave_col = col0 + (WIDE ? 32 * w : 0);
  struct Column { int tok, head, row; bool live; };
  auto column = [&]() -> Column {                                 // (asked for again where it is needed: kept, it costs registers of the loop)
    const int col = wave_col + (lane_now() & 31);
    const int tok = min(col / g, R.n - 1);
    return Column{tok, kvh * g + col % g, R.row0 + tok, col < R.n * g};
  };
  auto near_path = [&](int row) -> unsigned long long {           // nodes of the row's path inside the window
    unsigned long long m = A.chunk.tree_mask[row];
    if (A.window > 0) for (int i = __popcll(m) - A.window; i > 0; --i) m &= m - 1;
    return m;
  };
  unsigned long long kept_path = 0;                               // (SPLIT has no registers for it)
  int own;                                                        // position (and, for consecutive tokens, index)
  float slope;
  {
    const Column c = column();
    own = R.own0 + c.tok;
    if (R.tree) own = R.base + __popcll(A.chunk.tree_mask[c.row]) - 1;
    if (R.tree && !P::SPLIT) kept_path = near_path(c.row);
    slope = MODS && A.slopes ? A.slopes[c.head] * 1.44269504088896341f : 0.f;
  }

  // tile number -> first token
  auto tile_token = [&](int it) { return (it < R.n_prefix ? it : it - R.n_prefix + R.first) * KT; };
  // The table's entry for token k0 + lane (KT 32: lane % 32) of a tile, requested a tile and a half before it is looked at: looked at at once it would wait for every load in flight.
  const int* table = A.kv.page_table + (size_t)s * A.kv.table_stride;
  auto entry_of = [&](int it) -> int { return table[max(0, min(tile_token(it) + (lane_now() & (KT - 1)), R.keys - 1)) >> A.kv.page_shift]; };
  // the page itself, -1: not there, or the token is behind the last
  auto page_of = [&](int it, int entry) -> int {
    return (unsigned)entry < (unsigned)A.kv.n_pages && tile_token(it) + (lane_now() & (KT - 1)) < R.keys ? entry : -1;
  };
  constexpr int STEP = WIDE ? 1 : 4;
  const int in_page = (1 << A.kv.page_shift) - 1;
  const CT *kb = (const CT*)A.kv.k + kvh * A.kv.head_stride, *vb = (const CT*)A.kv.v + kvh * A.kv.head_stride;
  // Narrow and DIRECT or RAW: a wave has one buffer for keys and one for values; the next keys are on their way from the end of the scores on, the next values from the end of the products on.
  constexpr bool STAGGERED = !WIDE && (DIRECT || RAW);
  constexpr int MINE = WIDE ? 0 : NK * TILE;                      // a wave's place in a buffer: w * MINE

  // ---- DIRECT: a load instruction fills 1 KiB of LDS, RPI tokens of DH elements; lane -> (token, place), and the piece of 8 elements that belongs in the place.  What is not there (a page, a
  // token behind the last, elements from head_dim on) is whatever lies in page 0, or in the head's first piece: finite or not, it is masked like what a column may not see.
  constexpr int RPI = (RAW ? 1024 : 512) / ROW, RUNS = ROW * (int)sizeof(CT) / 16, INSTS = DIRECT || RAW ? KT / RPI / (WIDE ? 4 : 1) : 1, ORDERS = DIRECT ? 8 / RPI : RAW ? 16 / RPI : 1;
  const int tr = lane / RUNS, place = lane % RUNS;
  // bytes from an instruction's first token to what this lane loads (the keys' order of pieces repeats every eight tokens (RAW: 16), the values' every RPI)
  uint32_t k_off[ORDERS], v_off;
  if constexpr (RAW) {
#pragma unroll
    for (int i = 0; i < ORDERS; ++i) {
      const int kc = place ^ raw_k_turn<ROW>(i * RPI + tr);
      k_off[i] = (uint32_t)(tr * (int)A.kv.token_stride + (kc * 16 < dh ? kc * 16 : 0));
    }
    const int vc = place ^ raw_v_turn<ROW>(tr);
    v_off = (uint32_t)(tr * (int)A.kv.token_stride + (vc * 16 < dh ? vc * 16 : 0));
  } else {
    const int vc = place ^ (v_place<ROW>(tr, 0) - tr * (ROW / 8));
#pragma unroll
    for (int i = 0; i < ORDERS; ++i) {
      const int t = i * RPI + tr, kc = place ^ (k_place<ROW>(t, 0) - t * (ROW / 8));
      k_off[i] = (uint32_t)(tr * (int)A.kv.token_stride + (kc * 8 < dh ? kc * 8 : 0)) * (uint32_t)sizeof(CT);
    }
    v_off = (uint32_t)(tr * (int)A.kv.token_stride + (vc * 8 < dh ? vc * 8 : 0)) * (uint32_t)sizeof(CT);
  }
  typedef std::integral_constant<int, 1> KEYS;
  typedef std::integral_constant<int, 2> VALUES;
  typedef std::integral_constant<int, 3> BOTH;
  auto load_lds = [&](const void* from, lds_ptr to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  auto dma = [&](lds_ptr kd, lds_ptr vd, int it, int pages, auto what) {
    constexpr bool K = decltype(what)::value & 1, V = decltype(what)::value & 2;
    const int k0 = tile_token(it), first = WIDE ? w * INSTS : 0;
    if (!A.lane_pages) {                                          // the tokens of an instruction lie in one page, whose place stays in scalar registers
      long long at[INSTS];
      if (in_page >= KT - 1) {                                    // (and those of the tile: one product does)
        at[0] = max(0, __builtin_amdgcn_readfirstlane(pages)) * A.kv.page_stride + ((k0 & in_page) + first * RPI) * A.kv.token_stride;
#pragma unroll
        for (int u = 1; u < INSTS; ++u) at[u] = at[u - 1] + RPI * A.kv.token_stride;
      } else {
#pragma unroll
        for (int u = 0; u < INSTS; ++u) {
          const int t0 = (first + u) * RPI;
          at[u] = max(0, __builtin_amdgcn_readlane(pages, t0)) * A.kv.page_stride + ((k0 + t0) & in_page) * A.kv.token_stride;
        }
      }
#pragma unroll
      for (int u = 0; u < INSTS; ++u) {
        const int t0 = (first + u) * RPI;
        if constexpr (K) load_lds((const char*)(kb + at[u]) + k_off[u % ORDERS], kd + t0 * (RAW ? ROW / 2 : ROW));
        if constexpr (V) load_lds((const char*)(vb + at[u]) + v_off, vd + t0 * (RAW ? ROW / 2 : ROW));
      }
    } else {
#pragma unroll
      for (int u = 0; u < INSTS; ++u) {
        const int t0 = (first + u) * RPI, page = max(0, __shfl(pages, t0 + tr, 64));
        const long long at = page * A.kv.page_stride + (((k0 + t0 + tr) & in_page) - tr) * A.kv.token_stride;
        if constexpr (K) load_lds((const char*)(kb + at) + k_off[u % ORDERS], kd + t0 * (RAW ? ROW / 2 : ROW));
        if constexpr (V) load_lds((const char*)(vb + at) + v_off, vd + t0 * (RAW ? ROW / 2 : ROW));
      }
    }
  };

  // ---- not DIRECT: through registers
  f32x4 k4[P::SPLIT ? ITEMS : 1], v4[P::SPLIT ? ITEMS : 1];
  typedef Raw8<std::conditional_t<CODED, bf16_t, CT>> Raw;
  Raw kr[DIRECT || CODED || WIDE ? 1 : KSN], vr[DIRECT || CODED || WIDE ? 1 : ITEMS];
  float2 sc_next = {1.f, 1.f};                                    // CODED: scales of the keys and values of the lane's token of the next tile
  const uint32_t run_off = CODED && WIDE ? lane / P::RUNS * (uint32_t)A.kv.token_stride + (lane % P::RUNS * 16 < dh ? lane % P::RUNS * 16u : 0u) : 0u;   // from a wave's first token to this lane's run
  auto scales = [&](int it, int pages) -> float2 {                // CODED: of the keys and values of the lane's token
    if (pages < 0) return float2{1.f, 1.f};
    const long long at = pages * A.scale_page + kvh * A.scale_head + (((tile_token(it) + (lane_now() & (KT - 1))) & in_page) >> A.block_shift);
    return float2{fabsf(A.k_scale[at]), fabsf(A.v_scale[at])};
  };
  auto fetch = [&](int it, int pages) {
    const int k0 = tile_token(it);
    if constexpr (CODED && WIDE) {                                // (the tokens of a wave's 64 runs lie in one page, whose place stays in scalar registers; what is not there: as for DIRECT)
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int t0 = (i * 256 + 64 * w) / P::RUNS;
        if (t0 >= KT) break;
        const long long at = max(0, __builtin_amdgcn_readlane(pages, t0 & (KT - 1))) * A.kv.page_stride + ((k0 + t0) & in_page) * A.kv.token_stride;
        load_lds((const char*)kb + at + run_off, (lds_ptr)parked + (2 * i * 256 + 64 * w) * 8);
        load_lds((const char*)vb + at + run_off, (lds_ptr)parked + ((2 * i + 1) * 256 + 64 * w) * 8);
      }
    } else if constexpr (P::SPLIT) {                              // a token is eight threads': every eighth run of 4 elements
      const int l = lane_now(), t = 8 * w + (l >> 3), c = l & 7, page = __shfl(pages, t, 64);
      const long long at = page * A.kv.page_stride + ((k0 + t) & in_page) * A.kv.token_stride + 4 * c;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        f32x4 k = {0.f, 0.f, 0.f, 0.f}, v = k;
        if (page >= 0 && 4 * c + 32 * i < dh) { k = *(const f32x4*)(kb + at + 32 * i); v = *(const f32x4*)(vb + at + 32 * i); }
        k4[i] = k;
        v4[i] = v;
      }
    } else if constexpr (!WIDE && !CODED) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int item = i * 64 + lane, t = item / (DH / 8), c = item % (DH / 8);
        const int page = __shfl(pages, t, 64);
        const long long at = page * A.kv.page_stride + ((k0 + t) & in_page) * A.kv.token_stride + c * 8;
        vr[i].zero();
        if (page >= 0 && c * 8 < dh) vr[i].load(vb + at);
      }
    }
    if constexpr (!WIDE && !CODED) {
      const int page = pages;                                     // (KT = 32: the lane's own token)
      const long long at = page * A.kv.page_stride + ((k0 + q) & in_page) * A.kv.token_stride;
#pragma unroll
      for (int ks = 0; ks < KSN; ++ks) {
        const int d = 16 * ks + 8 * hh;
        kr[ks].zero();
        if (page >= 0 && d < dh) kr[ks].load(kb + at + d);
      }
    }
  };
  // SPLIT: a step of bringing the fetched tile to LDS, of as many as there are products of a tile's scores: three for two elements, six for a run.
  auto put_step = [&](bf16_t* kd, bf16_t* vd, int n, u32x2* pk) -> uint32_t {
    const int run = n / 6, i = run >> 1, pair = n % 6 / 3, j = n % 3;
    const bool values = run & 1;
    f32x4& x = values ? v4[i] : k4[i];
    const uint32_t bad = values && pair == 0 && j == 0 ? not_finite_any(x) : 0;
    uint32_t h = j == 0 ? upper_pair(x[2 * pair], x[2 * pair + 1]) : bf16_pair(x[2 * pair], x[2 * pair + 1]);
    if (j == 0) asm volatile("" : "+v"(h));                       // (the remainders come from it: the compiler would take them from the numbers, in more registers than there are)
    pk[j][pair] = h;
    if (j < 2) {
      x[2 * pair] -= __builtin_bit_cast(float, h << 16);
      x[2 * pair + 1] -= __builtin_bit_cast(float, h & 0xFFFF0000u);
    } else if (pair == 1) {
      const int t = tid >> 3, c = (tid & 7) + 8 * i;
      bf16_t* d = (values ? vd + 8 * v_place<ROW>(t, c >> 1) : kd + 8 * k_place<ROW>(t, c >> 1)) + 4 * (c & 1);
#pragma unroll
      for (int u = 0; u < 3; ++u) *(u32x2*)(d + u * TILE) = pk[u];
    }
    return bad;
  };
  // CODED, WIDE: the parked codes, and a step of 4 ITEMS that make bf16 of them: eight elements of the keys or values.
  u32x4 held[CODED && WIDE ? 2 * ITEMS : 1];
  auto take = [&]() {
#pragma unroll
    for (int i = 0; i < 2 * ITEMS; ++i) held[i] = *(const u32x4*)(parked + (i * 256 + tid) * 8);
  };
  auto code_step = [&](bf16_t* kd, bf16_t* vd, int n) {
    const int i = n >> 2, h = n & 1, item = i * 256 + tid, t = item / P::RUNS, c = item % P::RUNS;
    const bool values = n & 2;
    const u32x4 u = held[2 * i + values];
    if constexpr (CODED) {
      const bf16x8 x = coded8(u32x2{u[2 * h], u[2 * h + 1]}, CT());
      if (t < KT && c * 16 < DH) *(bf16x8*)(values ? vd + 8 * v_place<ROW>(t, 2 * c + h) : kd + 8 * k_place<ROW>(t, 2 * c + h)) = x;
    }
  };
  // the fetched tile to LDS; returns not 0 if a value is not finite (to this thread's knowledge)
  auto put = [&](bf16_t* kd, bf16_t* vd) -> uint32_t {
    uint32_t bad = 0;
    if constexpr (P::SPLIT) {
      u32x2 pk[3];
#pragma unroll
      for (int n = 0; n < 12 * ITEMS; ++n) bad |= put_step(kd, vd, n, pk);
    } else if constexpr (!CODED) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int item = i * 64 + lane, t = item / (DH / 8), c = item % (DH / 8);
        bf16x8 p[3];
        vr[i].split(p);
        if constexpr (!DIRECT) bad |= vr[i].bad();
#pragma unroll
        for (int j = 0; j < NK; ++j) *(bf16x8*)(vd + j * TILE + 8 * v_place<ROW>(t, c)) = p[j];
      }
    }
    return bad;
  };

  constexpr bool AHEAD2 = P::SPLIT || (CODED && WIDE);           // through registers into the other of two buffers: fetched two tiles ahead
  int it = t_begin + (WIDE ? 0 : w);
  int pages = -1, entry_next = 0, pages1 = -1;                    // (AHEAD2: pages1 are the next tile's, entry_next is the one's behind it)
  if (it < t_end) {
    pages = page_of(it, entry_of(it));
    entry_next = entry_of(it + STEP);
    if constexpr (AHEAD2) {
      if (it + 1 < t_end) pages1 = page_of(it + 1, entry_next);
      entry_next = entry_of(it + 2);
    }
  }
  if constexpr (STAGGERED) {
    if (it < t_end) {
      if constexpr (RAW) sc_next = scales(it, pages);
      dma((lds_ptr)k_lds0 + w * MINE, (lds_ptr)v_lds0, it, pages, KEYS());
      dma((lds_ptr)k_lds0, (lds_ptr)v_lds0 + w * MINE, it, pages, VALUES());
    }
  } else if constexpr (DIRECT) {
    if (it < t_end) dma((lds_ptr)k_lds0, (lds_ptr)v_lds0, it, pages, BOTH());
  } else if (it < t_end) fetch(it, pages);

  bf16x8 qf[NQ][KSN];
  {
    const Column c = column();
    const T* qp = (const T*)A.q + c.row * A.q_row + c.head * A.q_head;
#pragma unroll
    for (int ks = 0; ks < KSN; ++ks) {
      const int d = RAW ? 32 * (ks >> 1) + 16 * hh + 8 * (ks & 1) : 16 * ks + 8 * hh;   // (RAW: a lane reads 16 codes of a key at once, for two steps)
      Raw8<T> x;
      x.zero();
      if (c.live && d < dh) x.load(qp + d);
      bf16x8 p[3];
      x.template split<true>(p);
#pragma unroll
      for (int i = 0; i < NQ; ++i) qf[i][ks] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, p[i]) ^ A.q_flip);
    }
  }
  if constexpr (P::SPLIT) {
    if (tid < 2) s_bad[tid] = -1;
    __syncthreads();
    if (it < t_end && __any(put(k_lds0, v_lds0) != 0) && lane == 0) s_bad[0] = it;
    __syncthreads();
    fetch(it + 1, pages1);
  }
  if constexpr (CODED && WIDE) {
    wait_loads<0>();
    take();
#pragma unroll
    for (int n = 0; n < 4 * ITEMS; ++n) code_step(k_lds0, v_lds0, n);
    sc_next = scales(it, pages);
    wait_lds();
    if (it + 1 < t_end) fetch(it + 1, pages1);
    __syncthreads();
  }

  auto uniform = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); };
  const float c2 = uniform(A.scale * 1.44269504088896341f);       // scores to powers of two
  const float cap_in = uniform(MODS && A.softcap > 0.f ? 2.f * c2 / A.softcap : 0.f), cap_out = uniform(A.softcap * 1.44269504088896341f);
  const float cap_y = uniform(cap_in * 0.34657359027997264f);     // scale / cap
  constexpr float V_FAR = 0x1p96f, V_LIFT = 32.f, V_LEAST = 0x1p-96f;
  float v_least = V_LEAST;                                        // CODED, bf16 queries: the least value scale that is told from smaller ones
  float m_run = -INFINITY, l_run = 0.f;                           // maximum (in powers of two) of the column, sum of this lane's half of the tokens
  f32x16 oacc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[b][r] = 0.f;

  // Byte offsets in a buffer of what this lane reads of a tile: the keys' k-steps 0..3 (the others, and the second 32 tokens, lie a constant further on), the values' 32-wide blocks.
  // RAW: of a key's pieces hh, 2 + hh, ..; of the values' blocks, a pair of 16-wide columns each.
  uint32_t k_at[4], v_at[DB];                                     // (rows of 96 elements: pieces 4 to 7 lie behind 0 to 3 in the same order)
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = RAW ? (uint32_t)(q * ROW + 16 * (((2 * i + hh) ^ raw_k_turn<ROW>(q)) & (RUNS - 1))) : ROW == 96 && i > 1 ? k_at[i - 2] + 64 : 16 * k_place<ROW>(q, 2 * i + hh);
#pragma unroll
  for (int b = 0; b < DB; ++b) {
    if constexpr (RAW) {
      const int r8 = (lane & 15) >> 1, t = 4 * hh + (r8 & 3) + 8 * (r8 >> 2), c = 2 * b + ((lane >> 4) & 1);
      v_at[b] = t * ROW + 16 * ((c ^ raw_v_turn<ROW>(t)) & (RUNS - 1)) + 8 * (lane & 1);
      continue;
    }
    const int t = 4 * hh + ((lane & 15) >> 2), c = 4 * b + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    v_at[b] = 16 * v_place<ROW>(t, c) + 8 * (lane & 1);
  }
  const int wave_last = R.tree ? R.keys : max(R.own0 + min(R.n - 1, (wave_col + 31) / g), R.prefix - 1);   // last token a column of this wave may see
  const bool wave_live = wave_col < R.n * g;

  // One tile, its keys and values in kt, vt; the next goes to kn, vn.
  auto tile = [&](bf16_t* kt, bf16_t* vt, bf16_t* kn, bf16_t* vn, int which, auto last) {
    constexpr bool LAST = decltype(last)::value;                  // STAGGERED: nothing follows (known ahead, so that the loads in flight can be counted)
    const int k0 = tile_token(it);
    const uint64_t there = __ballot(pages >= 0) & low_ones(KT);
    const bool full = k0 + KT <= R.full_to && (k0 >= R.full_from || k0 + KT <= R.prefix) && there == low_ones(KT);
    bool bad = false;
    const int pages_next = AHEAD2 ? pages1 : page_of(it + STEP, entry_next);
    const float2 sc = sc_next;                                    // CODED: scales of the lane's token of this tile
    if constexpr (STAGGERED) {
      wait_loads<INSTS>();                   // the keys have landed (the values are behind them)
    } else if constexpr (DIRECT) {
      // this tile has landed (for WIDE: everyone's part of it, and everyone is done with the other buffer)
      wait_loads<0>();
      if constexpr (WIDE) { __builtin_amdgcn_s_barrier(); asm volatile("" ::: "memory"); }
      if (it + STEP < t_end) dma((lds_ptr)kn, (lds_ptr)vn, it + STEP, pages_next, BOTH());
    } else if constexpr (CODED) {
      wait_loads<0>();
      take();                                                     // (a wave's parked codes are its own; behind the last tile they are whatever they are)
      sc_next = scales(it + 1, pages_next);
    } else if constexpr (WIDE) {
      bad = s_bad[which] == it;
    } else {
      bad = __any(put(kt, vt) != 0);
    }
    const bool idle = WIDE && (!wave_live || k0 > wave_last);     // (the wave's part of moving data and the barriers stay)
    auto ask_next = [&]() {                                       // CODED, WIDE: the parked codes have been read, the tile after the next may take their place
      pages1 = it + 2 < t_end ? page_of(it + 2, entry_next) : -1;
      wait_lds();
      if (it + 2 < t_end) fetch(it + 2, pages1);
      entry_next = entry_of(it + 3);
    };
    f32x16 sacc[KB];
    uint32_t next_bad = 0;
    if (idle) {
      if constexpr (P::SPLIT) next_bad = put(kn, vn);
      if constexpr (CODED && WIDE)
#pragma unroll
        for (int n = 0; n < 4 * ITEMS; ++n) code_step(kn, vn, n);
      if constexpr (CODED && WIDE) ask_next();
    } else {
      auto key = [&](int a, int ks, int j) -> bf16x8 { return *(const bf16x8*)((const char*)kt + k_at[ks & 3] + (2 * j * TILE + 64 * ROW * a + 128 * (ks >> 2))); };
#pragma unroll
      for (int a = 0; a < KB; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[a][r] = 0.f;
      if constexpr (P::SPLIT) {
        // The next tile's pieces are made between this one's products (behind the last tile they are zeros): a step of it while the matrix unit works, in this order.
        bf16x8 kf[NK];
        u32x2 pk[3];
#pragma unroll
        for (int j = NK - 1; j >= 0; --j) kf[j] = key(0, 0, j);
#pragma unroll
        for (int n = 0; n < KSN * P::PRODUCTS; ++n) {
          const int ks = n / P::PRODUCTS, u = n % P::PRODUCTS, j = P::cache_piece(u);
          sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[P::column_piece(u)][ks], sacc[0], 0, 0, 0);
          if (P::done_with(u) && ks + 1 < KSN) kf[j] = key(0, ks + 1, j);
          next_bad |= put_step(kn, vn, n, pk);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else if constexpr (RAW) {                                 // a read is two k-steps; as below
        constexpr int PAIRS = KSN / 2, READS = KB * PAIRS, AHEAD = 2;
        auto raw = [&](int n) -> u32x4 { return *(const u32x4*)((const char*)kt + k_at[n % PAIRS] + 32 * ROW * (n / PAIRS)); };
        u32x4 kr[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) kr[n] = raw(n);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < READS; ++n) {
          const u32x4 k = kr[n % AHEAD];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bf16x8 kf = coded8(u32x2{k[2 * h], k[2 * h + 1]}, CT());
#pragma unroll
            for (int u = 0; u < P::PRODUCTS; ++u)
              sacc[n / PAIRS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[P::column_piece(u)][2 * (n % PAIRS) + h], sacc[n / PAIRS], 0, 0, 0);
          }
          if (n + AHEAD < READS) kr[n % AHEAD] = raw(n + AHEAD);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else if constexpr (P::KEYS_IN_LDS) {                      // reads some k-steps ahead of their products: LDS answers in the time of about four products
        constexpr int STEPS = KB * KSN, AHEAD = NQ == 3 ? 2 : 4;
        bf16x8 kf[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) kf[n] = key(n / KSN, n % KSN, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < STEPS; ++n) {
#pragma unroll
          for (int u = 0; u < P::PRODUCTS; ++u) sacc[n / KSN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n % AHEAD], qf[P::column_piece(u)][n % KSN], sacc[n / KSN], 0, 0, 0);
          if (n + AHEAD < STEPS) kf[n % AHEAD] = key((n + AHEAD) / KSN, (n + AHEAD) % KSN, 0);
          if constexpr (CODED)                                    // the next tile's codes, while the matrix unit works
#pragma unroll
            for (int i = n * 4 * ITEMS / STEPS; i < (n + 1) * 4 * ITEMS / STEPS; ++i) code_step(kn, vn, i);
          if (CODED && n == 3) ask_next();
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KSN; ++ks) {
          bf16x8 kf[3];
          kr[ks].split(kf);
#pragma unroll
          for (int u = 0; u < P::PRODUCTS; ++u) sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[P::cache_piece(u)], qf[P::column_piece(u)][ks], sacc[0], 0, 0, 0);
        }
      }
    }
    if constexpr (!WIDE && !DIRECT && !CODED) {
      if (it + STEP < t_end) fetch(it + STEP, pages_next);        // (the keys' registers are free now)
    }
    if constexpr (STAGGERED && !LAST) {
      if constexpr (RAW) sc_next = scales(it + STEP, pages_next);
      wait_lds();                                                 // the keys have been read
      dma((lds_ptr)kt, (lds_ptr)vt, it + STEP, pages_next, KEYS());
    }
    pages = pages_next;
    if constexpr (P::SPLIT) {
      if (__any(next_bad != 0) && lane_now() == 0) s_bad[which ^ 1] = it + 1;
      pages1 = it + 2 < t_end ? page_of(it + 2, entry_next) : -1;
      fetch(it + 2, pages1);
      entry_next = entry_of(it + 3);
    } else if constexpr (!STAGGERED && !CODED) entry_next = entry_of(it + 2 * STEP);
    const int lane = lane_now(), hh = lane >> 5;
    // CODED: numbers of their own, since parts of an accumulator are moved about as a whole where branches meet (with a cap, 31 registers spilled less); for the others it costs more than it gives.
    ScoreRow own_scores[CODED ? KB : 1];
    auto& score = one_of<CODED>(own_scores, sacc);
    if constexpr (CODED)
#pragma unroll
      for (int a = 0; a < KB; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) score[a][r] = sacc[a][r];
    uint64_t vis = ~0ull;                                         // tokens of the tile that the column sees
    // CODED: a block is at least 16 tokens and begins at a multiple of 16, so each 16 tokens of a tile have one scale: the first one's.  k_by: to powers of two, or to what the cap's tanh is taken of.
    constexpr int GROUPS16 = CODED ? KT / 16 : 1;
    float k_by[GROUPS16], v_by[GROUPS16], v_out[GROUPS16];
    // A value scale above V_FAR (or none that is a number) is in this tile.  It stands inside the weights, of up to 2^8, and would take them and their sums out of range.  So the maximum is put
    // V_LIFT above what it is, which makes all weights so much smaller and changes nothing else; the least scale of bf16 queries is as much larger from then on.
    bool far = false;
    if constexpr (CODED) {
      far = __any(!(sc.y <= V_FAR));
      const float x = sc.x * (MODS && A.softcap > 0.f ? cap_y : c2);
#pragma unroll
      for (int i = 0; i < GROUPS16; ++i) {
        k_by[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 16 * i));
      }
      // a score of -inf must not meet a scale that is 0 or not finite: such a block's scores (not its neighbours', whose rows' bits are theirs) take it before the mask
      if (!idle && (MODS || __any(!(x > 0.f && x < INFINITY)))) {
#pragma unroll
        for (int i = 0; i < GROUPS16; ++i) {
          if (!MODS && k_by[i] > 0.f && k_by[i] < INFINITY) continue;
#pragma unroll
          for (int r = 0; r < 8; ++r) score[i >> 1][8 * (i & 1) + r] *= k_by[i];
          k_by[i] = 1.f;
        }
      }
    }
    if (!idle) {
    // cap and slopes
    if constexpr (MODS && CODED) {                                // (as below, of what is the cap's y already)
      if (A.softcap > 0.f) {
        auto bent = [&](float y) -> float {
          const float z = y * y;
          float t = fmaf(cap_out * 0.01359966f, z, cap_out * -0.05067464f);
          t = fmaf(t, z, cap_out * 0.13276915f);
          t = fmaf(t, z, cap_out * -0.33330065f);
          return y * fmaf(t, z, cap_out);
        };
        bool small = false;
        if constexpr (NQ == 1) {
          float far = 0.f;
#pragma unroll
          for (int a = 0; a < KB; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) far = fmaxf(far, fabsf(score[a][r]));
          small = !__any(far > 0.7f);
        }
        if (small) {
#pragma unroll
          for (int a = 0; a < KB; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) { score[a][r] = bent(score[a][r]); asm volatile("" : "+v"(score[a][r])); }
        } else {
#pragma unroll
          for (int a = 0; a < KB; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float y = score[a][r], e = __builtin_amdgcn_exp2f(y * 2.88539008f);
              float x = fmaf(-2.f * cap_out, __builtin_amdgcn_rcpf(e + 1.f), cap_out);
              if constexpr (NQ == 3) {
                const float z = y * y;
                float t = 3.59212803657248102e-3f;
                t = fmaf(t, z, -8.86323552990219657e-3f);
                t = fmaf(t, z, 2.18694885361552028e-2f);
                t = fmaf(t, z, -5.39682539682539683e-2f);
                t = fmaf(t, z, 0.133333333333333333f);
                t = fmaf(t, z, -0.333333333333333333f);
                t = fmaf(t * z, y, y);
                x = fabsf(y) < 0.35f ? cap_out * t : x;
              } else {
                x = fabsf(y) > 0.7f ? x : bent(y);
              }
              score[a][r] = x;
              asm volatile("" : "+v"(score[a][r]));
            }
        }
      }
    } else if constexpr (MODS) {
      // bf16 queries: a score up to 0.7 of the cap takes a polynomial, one beyond it the exponential, each by its own size alone; where no score of the wave is beyond (of those that no row sees
      // neither), the exponential is left out.
      const float k = cap_out * cap_y;
      auto bent = [&](float x) -> float {
        // tanh(y) = y (1 + z (a1 + z (a2 + z (a3 + z a4)))), z = y^2: the coefficients of the least largest error up to 0.7, which is 1.34 * 10^-7.  Seven operations at the full rate for five of
        // which two take four times as long.
        const float y = x * cap_y, z = y * y;
        float t = fmaf(k * 0.01359966f, z, k * -0.05067464f);
        t = fmaf(t, z, k * 0.13276915f);
        t = fmaf(t, z, k * -0.33330065f);
        return x * fmaf(t, z, k);
      };
      bool small = false;
      if (NQ == 1 && A.softcap > 0.f) {
        float far = 0.f;
#pragma unroll
        for (int a = 0; a < KB; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r) far = fmaxf(far, fabsf(score[a][r]));
        small = !__any(far * cap_y > 0.7f);
      }
      if (small) {
#pragma unroll
        for (int a = 0; a < KB; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r) score[a][r] = bent(score[a][r]);
      } else if (A.softcap > 0.f) {
#pragma unroll
        for (int a = 0; a < KB; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(score[a][r] * cap_in);   // e^(2 x / cap); tanh = 1 - 2 / (e + 1)
            float x = fmaf(-2.f * cap_out, __builtin_amdgcn_rcpf(e + 1.f), cap_out);
            if constexpr (NQ == 3) {                              // fp32: near 0 that cancels; the Taylor polynomial to y^13 is within 10^-9 below 0.35
              const float y = score[a][r] * cap_y, z = y * y;
              float t = 3.59212803657248102e-3f;
              t = fmaf(t, z, -8.86323552990219657e-3f);
              t = fmaf(t, z, 2.18694885361552028e-2f);
              t = fmaf(t, z, -5.39682539682539683e-2f);
              t = fmaf(t, z, 0.133333333333333333f);
              t = fmaf(t, z, -0.333333333333333333f);
              t = fmaf(t * z, y, y);
              x = fabsf(y) < 0.35f ? cap_out * t : x;
            } else {
              x = fabsf(score[a][r]) * cap_y > 0.7f ? x : bent(score[a][r]);
            }
            score[a][r] = x;
          }
      } else {
#pragma unroll
        for (int a = 0; a < KB; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r) score[a][r] *= c2;
      }
    }
    if constexpr (MODS) {
      if (A.slopes) {
        if (R.tree && k0 + KT > R.base) {
          const unsigned long long tmask = A.chunk.tree_mask[column().row];
#pragma unroll
          for (int a = 0; a < KB; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = k0 + 32 * a + 8 * (r >> 2) + 4 * hh + (r & 3);
              const int pos = j > R.base ? R.base + __popcll(tmask & low_ones(j - R.base)) : j;
              score[a][r] = fmaf(-slope, (float)abs(own - pos), score[a][r]);
            }
        } else {
          const float d = (float)(own - k0 - 4 * hh);
#pragma unroll
          for (int a = 0; a < KB; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) score[a][r] = fmaf(-slope, fabsf(d - (float)(32 * a + 8 * (r >> 2) + (r & 3))), score[a][r]);
        }
      }
    }
    // what the column does not see
    if (!full) {
      if (R.tree) {
        const int sh = k0 - R.base;                               // bit u of the path is token base + u
        vis = low_ones(-sh) & ~(A.window > 0 ? low_ones(own - A.window + 1 - k0) : 0ull);
        const unsigned long long tnear = P::SPLIT ? near_path(column().row) : kept_path;
        vis |= sh >= 64 || sh <= -64 ? 0ull : sh >= 0 ? tnear >> sh : tnear << -sh;
      } else {
        vis = low_ones(own + 1 - k0);
        if (A.window > 0) vis &= ~low_ones(own - A.window + 1 - k0);
      }
      vis |= low_ones(R.prefix - k0);
      vis &= there;
      const uint64_t mine = vis >> (4 * hh);
#pragma unroll
      for (int a = 0; a < KB; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) score[a][r] = (uint32_t)(mine >> (32 * a)) >> (8 * (r >> 2) + (r & 3)) & 1u ? score[a][r] : -INFINITY;
    }
    float top = score[0][0];
    if constexpr (CODED && !MODS) {
      top = -INFINITY;
#pragma unroll
      for (int a = 0; a < KB; ++a)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = score[a][8 * h];
#pragma unroll
          for (int r = 1; r < 8; ++r) x = fmaxf(x, score[a][8 * h + r]);
          top = fmaxf(top, x * k_by[2 * a + h]);
        }
    } else {
#pragma unroll
      for (int a = 0; a < KB; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, score[a][r]);
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if constexpr (!MODS && !CODED) top *= c2;
    const float top_seen = top;
    if constexpr (CODED) {
      if (far) {                                                  // the columns that see a token of such a block
        bool lifted = false;
#pragma unroll
        for (int i = 0; i < GROUPS16; ++i) {
          const float y = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sc.y), 16 * i));
          lifted |= y > V_FAR && (vis & there) >> (16 * i) & 0xFFFFu;
        }
        top += lifted ? V_LIFT : 0.f;
        if (__any(lifted)) v_least = V_LEAST * 0x1p32f;
      }
    }
    // The maximum moves only when it grows by more than 8 (weights up to 2^8 lose nothing in fp32 or bf16), and lane by lane, so that a column's bits are its own.
    const bool moved = top > m_run + 8.f || (m_run == -INFINITY && top > -INFINITY);
    if (__any(moved)) {
      if constexpr (CODED && NQ == 1) {
        // With the scale of its block the largest weight is no power of two, as it is without, and would be rounded.  So the maximum is put up to 1 higher, where it is one.
        const float in_block = __builtin_amdgcn_fractf(__builtin_amdgcn_logf(not_finite(sc.y) ? 1.f : fmaxf(sc.y, V_LEAST)));
        float up = 0.f;
#pragma unroll
        for (int i = 0; i < GROUPS16; ++i) {
          float x = score[i >> 1][8 * (i & 1)];
#pragma unroll
          for (int r = 1; r < 8; ++r) x = fmaxf(x, score[i >> 1][8 * (i & 1) + r]);
          if ((MODS ? x : x * k_by[i]) >= top_seen) up = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, in_block), 16 * i));
        }
        top += fmaxf(up, __shfl_xor(up, 32, 64));
      }
      const float f = moved ? __builtin_amdgcn_exp2f(m_run - top) : 1.f;
      m_run = moved ? top : m_run;
      l_run *= f;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[b][r] *= f;
    }
    }
    if constexpr (STAGGERED) wait_loads<LAST ? 0 : INSTS>();   // the values have landed
    if (RAW && !full && std::is_same<CT, e4m3_t>::value) {        // is there a NaN among the values?
      uint32_t any = 0;
#pragma unroll 4
      for (int i = 0; i < TILE / 512; ++i) any |= nan_codes(*(const u32x4*)(vt + i * 512 + lane * 8));
      bad = __any(any != 0);
    }
    if (NK == 1 && !RAW && !full) {                                       // is there anything that is not finite among the values?
      uint32_t any = 0;
#pragma unroll 4
      for (int i = 0; i < TILE / 512; ++i) any |= exponents(*(const u32x4*)(vt + i * 512 + lane * 8));
      bad = __any(any != 0);
    }
    if (RAW && bad) {
      // 0 times NaN is not 0.  So it is added to the columns that see it, and zeroed for the product.
      uint64_t spoilt = 0;
#pragma unroll 1
      for (int i = 0; i < TILE / 512; ++i) {
        if (nan_codes(*(const u32x4*)(vt + i * 512 + lane * 8)) != 0) spoilt |= 1ull << ((i * 64 + lane) / RUNS);
      }
      for (int o = 32; o; o >>= 1) spoilt |= __shfl_xor((unsigned long long)spoilt, o, 64);
      for (uint64_t left = spoilt & there; left; left &= left - 1) {
        const int t = __builtin_ctzll(left);
        const bool seen = vis >> t & 1;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = 32 * b + 8 * i + 4 * hh;
            const uint32_t v = *(const uint32_t*)((const char*)vt + t * ROW + 16 * (((d >> 4) ^ raw_v_turn<ROW>(t)) & (RUNS - 1)) + (d & 15));
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[b][4 * i + e] += seen && (v >> (8 * e) & 0x7Fu) == 0x7Fu ? NAN : 0.f;
            __builtin_amdgcn_sched_barrier(0);
          }
      }
#pragma unroll 1
      for (int i = 0; i < TILE / 512; ++i) {
        u32x4 v = *(const u32x4*)(vt + i * 512 + lane * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] &= ~((((v[e] & 0x7F7F7F7Fu) + 0x01010101u & 0x80808080u) >> 7) * 0xFFu);
        *(u32x4*)(vt + i * 512 + lane * 8) = v;
      }
    } else if (bad) {
      // 0 times what is not finite is not 0.  So it is added to the columns that see it, and zeroed for the product.
      uint64_t spoilt = 0;
#pragma unroll 1
      for (int i = 0; i < TILE / 512; ++i) {
        if (exponents(*(const u32x4*)(vt + i * 512 + lane * 8)) != 0) spoilt |= 1ull << ((i * 64 + lane) / (ROW / 8));
      }
      for (int o = 32; o; o >>= 1) spoilt |= __shfl_xor((unsigned long long)spoilt, o, 64);
      for (uint64_t left = spoilt & there; left && !idle; left &= left - 1) {
        const int t = __builtin_ctzll(left);
        const bool seen = vis >> t & 1;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = 32 * b + 8 * i + 4 * hh;
            const u32x2 v = *(const u32x2*)(vt + 8 * v_place<ROW>(t, d >> 3) + (d & 7));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = __builtin_bit_cast(float, e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
              oacc[b][4 * i + e] += seen && not_finite(x) ? x : 0.f;
            }
            __builtin_amdgcn_sched_barrier(0);                    // (one read at a time: all of them at once would take registers that the loop keeps)
          }
      }
      if constexpr (WIDE) __syncthreads();
#pragma unroll 1
      for (int i = WIDE ? w : 0; i < NK * TILE / 512; i += WIDE ? 4 : 1) {   // (all pieces)
        u32x4 v = *(const u32x4*)(vt + i * 512 + lane * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((v[e] & 0x7F80u) == 0x7F80u) v[e] &= 0xFFFF0000u;
          if ((v[e] & 0x7F800000u) == 0x7F800000u) v[e] &= 0xFFFFu;
        }
        *(u32x4*)(vt + i * 512 + lane * 8) = v;
      }
      if constexpr (WIDE) __syncthreads();
    }
    if constexpr (CODED) {                                        // a block of values whose scale is not finite: nothing finite for the columns that see one of them
      const bool odd_here = not_finite(sc.y);
      if (far && !idle && __any(odd_here)) {
#pragma unroll
        for (int i = 0; i < GROUPS16; ++i) {
          const bool odd = not_finite(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sc.y), 16 * i)));
          const float add = odd && (vis & there) >> (16 * i) & 0xFFFFu ? NAN : 0.f;
#pragma unroll
          for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[b][r] += add;
        }
      }
      // Weights take their block's value scale.  fp32 queries: by a product; bf16: in the exponent, as its logarithm (off by 2^-24 of it, the scale v_least at least), and it is taken out of their sum again.
      const float x = odd_here ? (NQ == 3 ? 0.f : 1.f) : NQ == 3 ? sc.y : fmaxf(sc.y, v_least), y = NQ == 3 ? x : __builtin_amdgcn_logf(x);
      float z = NQ == 3 ? 0.f : __builtin_amdgcn_rcpf(x);
      if (NQ == 1 && far) z = x > V_FAR ? __builtin_amdgcn_rcpf(x * 0x1p-32f) * 0x1p-32f : z;   // (the instruction makes 0 of what is below the least normal number)
#pragma unroll
      for (int i = 0; i < GROUPS16; ++i) {
        v_by[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, y), 16 * i));
        v_out[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, z), 16 * i));
      }
    }
    if (!idle) {
    const float m_sub = m_run == -INFINITY ? 0.f : m_run;
    // 16 tokens at a time: their values are read a block ahead, and the weights of the next 16 are made between the products, in this order.
    constexpr int GROUPS = KT / 16 * DB, SLOTS = DB * P::PRODUCTS, WORK = NQ == 3 ? 12 : 4;
    u32x4 pf[2][NQ];
    constexpr int AHEAD = NK == 3 ? 1 : NQ == 3 ? 2 : 4;          // (of three pieces each is read again as soon as it is done with)
    bf16x8 vf[AHEAD][NK];
    u32x2 vraw[AHEAD];                                            // RAW
    float sum = 0.f, block_sum = 0.f;
    auto weights = [&](int jj, int n) {                           // n of WORK steps: a pair's weights and their first piece, its second, its third
      const int pair = NQ == 3 ? n / 3 : n, j = NQ == 3 ? n % 3 : 0, a = jj >> 1, r = 8 * (jj & 1) + 2 * pair;
      float x = score[a][r], y = score[a][r + 1];
      if (j == 0) {
        const float by = CODED ? k_by[CODED ? jj : 0] : c2, off = CODED && NQ == 1 ? m_sub - v_by[CODED ? jj : 0] : m_sub;
        x = __builtin_amdgcn_exp2f(MODS ? x - off : fmaf(x, by, -off));
        y = __builtin_amdgcn_exp2f(MODS ? y - off : fmaf(y, by, -off));
        if constexpr (CODED && NQ == 1) {
          block_sum = pair == 0 ? x : block_sum + x;
          block_sum += y;
          if (pair == 3) sum = fmaf(block_sum, v_out[jj], sum);
        } else {
          sum += x;
          sum += y;
          if constexpr (CODED) { x *= v_by[jj]; y *= v_by[jj]; }
        }
      }
      const uint32_t h = bf16_pair(x, y);
      pf[jj & 1][j][pair] = h;
      if (j + 1 < NQ) {
        score[a][r] = x - __builtin_bit_cast(float, h << 16);
        score[a][r + 1] = y - __builtin_bit_cast(float, h & 0xFFFF0000u);
      }
    };
    auto value = [&](int i, int j) {                              // piece j of block i % DB of 16 tokens
      if constexpr (RAW) {
        vraw[i % AHEAD] = read_transposed8((const char*)vt + v_at[i % DB] + 16 * ROW * (i / DB));
        return;
      }
      const char* p = (const char*)vt + v_at[i % DB] + (2 * j * TILE + 32 * ROW * (i / DB));
      const s16x4 lo = read_transposed((const bf16_t*)p), hi = read_transposed((const bf16_t*)(p + 16 * ROW));
      vf[i % AHEAD][j] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int j = NK - 1; j >= 0; --j) value(i, j);
#pragma unroll
    for (int n = 0; n < WORK; ++n) weights(0, n);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int jj = i / DB, b = i % DB;
      if constexpr (RAW) vf[i % AHEAD][0] = coded8(vraw[i % AHEAD], CT());
#pragma unroll
      for (int u = 0; u < P::PRODUCTS; ++u) {
        const int j = P::cache_piece(u), slot = b * P::PRODUCTS + u;
        oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % AHEAD][j], __builtin_bit_cast(bf16x8, pf[jj & 1][P::column_piece(u)]), oacc[b], 0, 0, 0);
        if (P::done_with(u) && i + AHEAD < GROUPS) value(i + AHEAD, j);
        if (jj + 1 < KT / 16)
#pragma unroll
          for (int n = slot * WORK / SLOTS; n < (slot + 1) * WORK / SLOTS; ++n) weights(jj + 1, n);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l_run += sum;
    }
    if constexpr (STAGGERED && !LAST) {
      entry_next = entry_of(it + 2 * STEP);
      wait_lds();                                                 // the values have been read
      dma((lds_ptr)kt, (lds_ptr)vt, it + STEP, pages, VALUES());
    }
    if constexpr (CODED && WIDE) {                                // (not __syncthreads, which would wait for the codes on their way)
      wait_lds();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    } else if constexpr (AHEAD2) __syncthreads();
    it += STEP;
  };
  if constexpr (P::TWO) {
    while (it < t_end) {
      tile(k_lds0, v_lds0, k_lds1, v_lds1, 0, std::false_type());
      if (it >= t_end) break;
      tile(k_lds1, v_lds1, k_lds0, v_lds0, 1, std::false_type());
    }
  } else {
    bf16_t *kt = k_lds0 + w * (P::KEYS_IN_LDS ? MINE : 0), *vt = v_lds0 + w * MINE;
    if constexpr (STAGGERED) {
      while (it + STEP < t_end) tile(kt, vt, kt, vt, 0, std::false_type());
      if (it < t_end) tile(kt, vt, kt, vt, 0, std::true_type());
    } else
      while (it < t_end) tile(kt, vt, kt, vt, 0, std::false_type());
  }
  l_run += __shfl_xor(l_run, 32, 64);
  if constexpr (!WIDE) {
    // waves 2 and 3 into 0 and 1, then 1 into 0
    float* st = (float*)v_lds0 + lane_now();
#pragma unroll
    for (int half = 2; half > 0; half >>= 1) {
      __syncthreads();
      float* mine = st + (w & (half - 1)) * (16 * DB + 2) * 64;
      if (w >= half && w < 2 * half) {
        mine[0] = m_run; mine[64] = l_run;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) mine[(2 + 16 * b + r) * 64] = oacc[b][r];
      }
      __syncthreads();
      if (w < half) {
        const float m1 = mine[0], m = fmaxf(m_run, m1);
        const float w0 = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m), w1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - m);
        l_run = l_run * w0 + mine[64] * w1;
        m_run = m;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[b][r] = oacc[b][r] * w0 + mine[(2 + 16 * b + r) * 64] * w1;
      }
    }
    if (w > 0) return;
  }
  const Column c = column();
  if (!c.live) return;
  const int half = lane_now() >> 5;
  if (whole) {
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    T* o = (T*)A.out + c.row * A.out_row + c.head * A.out_head;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = 32 * b + 8 * i + 4 * half;
        if (d >= dh) continue;
        const float x[4] = {oacc[b][4 * i] * inv, oacc[b][4 * i + 1] * inv, oacc[b][4 * i + 2] * inv, oacc[b][4 * i + 3] * inv};
        store_run<4>(o + d, x);
      }
  } else {
    const size_t at = ((size_t)c.row * A.H + c.head) * A.splits + split;
    if (half == 0) { A.part_ml[2 * at] = m_run; A.part_ml[2 * at + 1] = l_run; }
    float* o = A.part_o + at * P::PART;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x[4] = {oacc[b][4 * i], oacc[b][4 * i + 1], oacc[b][4 * i + 2], oacc[b][4 * i + 3]};
        store_run<4>(o + 32 * b + 8 * i + 4 * half, x);
      }
  }
}

// Adds up the parts (at most 64) of the (row, head) pairs whose tokens were split; a wave a pair.  Its time is one chain of loads, so the first parts are requested before it is known how many
// there are: they lie in the workspace whatever they hold.
template <typename P, typename T>
__global__ __launch_bounds__(256) void k_chunk_attn_join(const ChunkAttnDev A) {
  constexpr int PART = P::PART, E = PART / 64, AHEAD = 8;
  const int row = blockIdx.x, head = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, dh = A.kv.head_dim;
  if (head >= A.H) return;
  const size_t at = ((size_t)row * A.H + head) * A.splits;
  const float* po = A.part_o + at * PART + lane * E;
  float ov[AHEAD][E];
  auto request = [&](int k0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) ov[u][e] = po[(size_t)min(k0 + u, A.splits - 1) * PART + e];
  };
  const float2 ml = *(const float2*)(A.part_ml + 2 * (at + min(lane, A.splits - 1)));
  request(0);
  const int s = wave_row_seq(A.chunk.row_start, A.chunk.n_seqs, row);
  if (s < 0) return;
  const int g = A.H / A.kv.n_kv_heads, i = row - max(0, A.chunk.row_start[s]), col = i * g + head % g;
  const ColumnRange R = column_range<P::KT>(A, s, col / P::COLS * P::COLS, P::COLS, g);
  if (i >= R.n || R.n_tiles <= A.split_tiles) return;
  const int n = (R.n_tiles + A.split_tiles - 1) / A.split_tiles;   // at most A.splits
  const float mine = lane < n ? ml.x : -INFINITY;
  float m = mine;
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  // A part without a maximum saw nothing (its sum is 0), or nothing but scores that are NaN: then its sum is NaN, and so is the row.
  const float sum = lane < n ? ml.y : 0.f, f = mine == -INFINITY ? (sum == 0.f ? 0.f : sum) : __builtin_amdgcn_exp2f(mine - m);
  float l = f * sum, x[E];
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o, 64);
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  for (int k0 = 0; k0 < n; k0 += AHEAD) {
    if (k0 > 0) request(k0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const bool there = k0 + u < n;                              // (what lies behind the parts may be anything)
      const float fk = there ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), k0 + u)) : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = there ? fmaf(fk, ov[u][e], x[e]) : x[e];   // (0 times an infinity that a row sees is NaN, as it is within a part)
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)A.out + row * A.out_row + head * A.out_head;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (lane * E + e < dh) { x[e] *= inv; store_run<1>(o + lane * E + e, x + e); }
}
