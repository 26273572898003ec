// Dense attention of new tokens, bf16, many rows per tile: chunks of prompts and whole ones, on the matrix cores.
//
// A tile is 256 rows (256 / G tokens times the G heads of a KV head).  Four waves, one per SIMD, own 64 rows each and walk the same
// 64-key tiles, which arrive in LDS directly, requested two tiles ahead; every fragment read from LDS serves 64 rows.  In one piece of
// straight-line code a wave forms the weights of one block of 32 keys on the vector ALU while the matrix cores form the
// scores of the next and add the output of the last one:
//   * A wave issues in order, so the vector instructions are shared out behind every single product (two of those in a row make
//     what follows wait until the first has left the matrix cores).  Four of them fit a product of 32 cycles with room: fma, exp, the weight's sum
//     and half a conversion.
//   * The softmax's reference is not a running maximum.  In tiles with masks, the first one among them, it is raised, with what has
//     been added up so far, when a weight of 2 or more shows up, which the first visible key of
//     a row does.  Tiles that every row sees in full take a copy of the code without masks and without that: weights may grow to 2^64
//     there, which costs no precision.  Should they grow further (logits 44 above all of the first tile's), the output not be finite (values of V beyond 2^64 may
//     overflow with such weights), or the reference be so large that logits have to be rounded first, the workgroup does the piece again with the former code throughout.  (With the
//     code for raising in the loop the compiler moves accumulators about: 1000 instructions a tile instead of 560.)
// Weights keep their 24 bits: V is multiplied with each of the three bf16 numbers that a weight is the sum of, and nothing is rounded before the result is; four
// units of matrix work instead of two.  The caller may choose weights rounded to bf16 (half a step, 2^-8 of each; the relative error of results against 64 bits
// is then 1.8e-3 instead of 1.7e-3, which is the results' own rounding); their sum is of the floats before that rounding, so that the log-sum-exp keeps 24 bits.
//
// Measured (H 32/8, D 128): a prompt of 8192 tokens 835 to 883 us from card to card, 512 tokens over 131072 keys 1650 to 1715, up to 1.32 and 1.33 PFLOP/s of
// products with the three parts counted; a bf16 product of 8192^3 by the library reaches 1.22 on such a card.  64 keys take 6300 cycles, of which the matrix cores
// work 4096, at a clock of 2.0 GHz (2.4 with little work).  D 64, 8192 tokens: 523 us, 4040 cycles where the matrix cores work 2048: the vector ALU is the bound.
// Rounded weights: 470 to 505 us, 904 to 966, up to 1.17 and 1.22 PFLOP/s: 3350 cycles for 64 keys, of which the matrix cores work 2048 and 2500 go to issuing,
// at 1.8 to 2.0 GHz.  A tile's start and end cost 13000 cycles (page ids and queries 2100, the first tile and its scores 3700, the first block's weights
// 2200, results 4400): what short prompts are bound by.  D 64: 298 us, 2150 cycles where the matrix cores work 1024; exponentials, sums and
// conversions are as many as for D 128, so the vector ALU is the bound.
#include "paged_shares.h"
#include <limits.h>
#include <type_traits>

namespace ts {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int kPtTile = 64;                   // keys per tile
constexpr int kPtRows = 256;                  // rows per tile of the share
constexpr int kPtBuf = 3;                     // tiles of K, and of V, in LDS
constexpr int kPtRing = 4;                    // tiles whose page ids are in LDS
constexpr float kPtUnset = -3.40282347e38f;   // reference exponent of a row that has seen no key: no finite logit lies below it
constexpr uint32_t kPtTwo = 0x40004000u;      // bits that only bf16 numbers of 2 and more have (and infinities and NaN)
constexpr float kPtMost = 1.8446744e19f;      // 2^64: sums of a block's weights that leave room for all others
constexpr float kPtHead = 8.f;                // a raised reference lies this far above the largest exponent so far
constexpr float kPtBig = 1048576.f;           // references beyond this: the logits are rounded before it is taken off them

// place of a row's 16-byte pieces in LDS: 16 rows x one piece (K fragments) and 4 rows x 4 pieces (V^T) each fall on all banks
template <int D> __device__ __forceinline__ int pt_swz(int key) {
  return D == 128 ? (((key & 3) << 2) | ((key >> 2) & 3)) : ((((key >> 1) & 1) << 2) | (((key >> 2) & 1) << 1) | ((key >> 3) & 1));
}

template <int D, bool FULL>                   // FULL: weights of 24 bits, else rounded to bf16
__global__ __launch_bounds__(256, 1) void paged_tall_kernel(PagedAttnArgs a, ShareArgs sh) {
  constexpr int KS = D / 16;                  // k-steps of Q K^T
  constexpr int NBO = D / 32;                 // 32-row blocks of the transposed output
  constexpr int RB = D * 2, PPR = RB / 16;    // bytes and 16-byte pieces of a K/V row
  constexpr int KPI = 64 / PPR;               // keys per wave load
  constexpr int WK = kPtTile / 4;             // keys of a tile that a wave stages
  constexpr int NLD = WK / KPI;               // loads per wave, tile and pool
  constexpr int TILE_B = kPtTile * RB;
  constexpr int VH = D == 128 ? 32 : 16;      // what eight keys more flip of a piece's place
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];   // [buffer][K tile, V tile], page ids [wave][ring][64], the share's ends, a flag
  // (nothing else is in LDS: places of pieces are flipped in the address, so the tiles have to begin at a multiple of a row)
  ShareScratch* s_share = reinterpret_cast<ShareScratch*>(smem + 2 * kPtBuf * TILE_B + 4 * kPtRing * 256);
  int* s_bad = reinterpret_cast<int*>(s_share + 1);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int H = a.H, G = a.H / a.H_kv;
  const int wg = share_of(blockIdx.x, sh.wgs);
  SharePlace from, to;
  SeqShape first;
  find_share<kPtTile>(a, sh, G, wg, s_share, &from, &to, &first);
  int32_t* desc = sh.desc + (size_t)wg * 8;
  if (!sh.whole && threadIdx.x == 0) { desc[3] = kPieceNone; desc[7] = kPieceNone; }

  const uint32_t g_inv = 65536u / (uint32_t)G + 1u;             // exact for rows below 256
  const uint32_t reach = a.window > 0 ? (uint32_t)a.window : 0x7fffffffu;
  float c2 = a.sm_scale * 1.44269504088896340736f;
  if (c2 == 0.f) c2 = 1e-37f;                                   // the same weights (all 1), and a hidden key still gets 0
  const float hidden = c2 > 0.f ? -INFINITY : INFINITY;         // c2 * hidden = -inf

  typedef const __attribute__((address_space(3))) bf16x8_t lds_bf16x8;
  typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
  // K fragment ks of key block kb: row 32 * kb + col, piece (2 * ks + half) ^ swz(col) -- ks flips bits of the address only
  const uint32_t ka0 = lds_base + (uint32_t)(col * RB + ((half ^ pt_swz<D>(col)) * 16));
  // V^T: 16 lanes read 4 keys x 16 columns; lane i of them reads key i / 4, columns 4 * (i % 4) ..; the output block nb and
  // the upper eight keys of a k-step flip bits of the piece
  const int vt_key = 4 * half + ((lane & 15) >> 2), vt_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const uint32_t va0 = lds_base + (uint32_t)(vt_key * RB + (((vt_col >> 3) ^ pt_swz<D>(vt_key)) * 16) + (vt_col & 7) * 2);
  // staging: this wave's 16 keys of a tile, load i covering keys 16 * wave + i * KPI + lane / PPR
  const int st_key = lane / PPR, st_pos = lane % PPR;
  const uint32_t lds_st = __builtin_amdgcn_readfirstlane(lds_base + (uint32_t)(wave * WK * RB));
  const uint32_t look = __builtin_amdgcn_readfirstlane(lds_base + (uint32_t)(2 * kPtBuf * TILE_B + wave * kPtRing * 256));
  const int row_shift = 31 - __builtin_clz((uint32_t)(a.H_kv * RB));   // H_kv is a power of two

  walk_share<kPtTile>(a, sh, G, from, to, first, [&](int kvh, const SeqShape& sq, int r, const TileKeys& keys, int ua, int ub, bool again) __attribute__((always_inline)) -> bool {
    const int c0 = r * sh.tpt, ntok = min(sh.tpt, sq.n - c0), nrows = ntok * G;
    const int row0 = sq.row0 + c0, x0 = sq.N - sq.n + c0, x1 = x0 + ntok - 1;   // first row; places of the first and last token
    const bool whole = ua == 0 && ub == keys.units;
    const int tmax = keys.end - 1;
    auto token_of = [&](uint32_t j) -> uint32_t { return __umul24(j, g_inv) >> 16; };   // j / G
    // the tile's row j in q, out and lse: a uniform first row and 32 bits behind it (j / G tokens of H rows, then j % G)
    const size_t tile_row = (size_t)row0 * H + kvh * G;
    auto row_at = [&](uint32_t j) -> uint32_t { return __umul24(token_of(j), (uint32_t)(H - G)) + j; };
    if (keys.end <= keys.first) {                                  // no row sees a token (one unit: the tile is not cut)
      for (int i = threadIdx.x; i < nrows * D; i += 256) {
        const size_t o = tile_row + row_at(i / D);
        reinterpret_cast<uint16_t*>(a.out)[o * D + i % D] = 0;
        if (i % D == 0 && a.lse != nullptr) a.lse[o] = -INFINITY;
      }
      return false;
    }
    const int slot = ua > 0 ? 0 : 1;
    if (!whole && threadIdx.x == 0) {
      int32_t* d = desc + slot * 4;
      d[0] = row0; d[1] = kvh; d[2] = ntok; d[3] = ub == keys.units ? kPieceEnds : kPieceGoesOn;
    }
    const int32_t* pages = a.page_indices + sq.page0;
    const int key0 = (keys.u0 + ua) * kPtTile, nt = ub - ua;       // first key and number of tiles
    // tiles [f0, f1) are seen in full by every row
    const int f0 = again ? nt : a.window > 0 ? max((x1 - key0 - a.window + kPtTile) / kPtTile, 0) : 0;
    int f1 = again ? 0 : x0 >= key0 ? min((x0 + 1 - key0) / kPtTile, nt) : 0;       // (INT_MIN once the logits are rounded before the reference is taken off)
    bool bad = false;                                              // a weight beyond what the code without raising can take

    // ---- Memory to LDS, 16 bytes per lane: the wave's 64 lanes fill 1 KiB from the (uniform) LDS address.  Written in assembly because the
    // compiler, which cannot tell the buffers apart, makes every later LDS read wait for the builtin form; completion is awaited by the
    // vmcnt before a tile's barrier.  Page ids come the same way, three tiles earlier.
    // Keys past the end or in front of the tile's first window stand for the nearest that some row sees: no other place of the pools is read.
    auto seen = [&](int t) __attribute__((always_inline)) -> int { return min(max(t, keys.first), tmax); };
    auto fetch_look = [&](int it) __attribute__((always_inline)) {
      const int t = seen(key0 + it * kPtTile + wave * WK + (lane & (WK - 1)));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(look + (it & (kPtRing - 1)) * 256), "v"(pages + (t >> a.p_shift)) : "memory", "m0");
    };
    uint64_t at_k[NLD], at_v[NLD];                                 // places in a pool (this lane's) of the K tile's and the V tile's rows that are requested next
    const uint8_t* const k_head = a.k_pool + kvh * RB;
    const uint8_t* const v_head = a.v_pool + kvh * RB;
    int page[NLD];
    auto pages_of = [&](int it) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NLD; ++i)
        page[i] = *(const volatile __attribute__((address_space(3))) int*)(look + (uint32_t)((it & (kPtRing - 1)) * 256 + (i * KPI + st_key) * 4));
    };
    auto rows_at = [&](int it) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const int key = i * KPI + st_key, t = seen(key0 + it * kPtTile + wave * WK + key);
        at_v[i] = at_k[i];
        at_k[i] = ((uint64_t)(((uint32_t)page[i] << a.p_shift) + (uint32_t)(t & (a.P - 1))) << row_shift) | (uint32_t)((st_pos ^ pt_swz<D>((wave * WK + key) & 15)) * 16);
      }
    };
    auto rows_of = [&](int it) __attribute__((always_inline)) { pages_of(it); rows_at(it); };
    auto load_row = [&](const uint8_t* pool, uint64_t at, int i, uint32_t place) __attribute__((always_inline)) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_st + place + (uint32_t)(i * 1024)), "v"(pool + at) : "memory", "m0");
    };
    // places of tiles it, it + 1 and it + 2 in LDS (of K; V lies TILE_B behind), handed on from tile to tile
    uint32_t p0 = 0, p1 = 2 * TILE_B, p2 = 4 * TILE_B;

    // ---- queries: the wave's 64 rows by way of the last four tiles' places (one each), 1 KiB of neighbouring bytes per load.  (Read as fragments from
    // memory, 16 bytes of 32 rows at a time, it took 8000 cycles until they were there; now 2100.)  Rows past the
    // last are copies of it.
    __syncthreads();                                               // the tiles of the piece before have been read
    if (threadIdx.x == 0) *s_bad = 0;
    fetch_look(0); fetch_look(1); fetch_look(2); fetch_look(3);
    const uint32_t lds_q = __builtin_amdgcn_readfirstlane(lds_base + (uint32_t)((2 + wave) * TILE_B));
    constexpr int NLQ = 64 / KPI;
    const uint8_t* q_base = a.q + tile_row * RB;
    int q_key = st_key;
    asm volatile("" : "+v"(q_key));                                // (formed anew for every tile: the compiler would keep all of these addresses)
    const int q_pos = st_pos ^ pt_swz<D>(q_key);                   // (the load's own part of the row's number flips other bits)
#pragma unroll
    for (int i = 0; i < NLQ; ++i) {
      const uint32_t off = row_at((uint32_t)min(wave * 64 + i * KPI + q_key, nrows - 1)) * RB + (uint32_t)((q_pos ^ pt_swz<D>(i * KPI & 15)) * 16);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_q + i * 1024), "v"(off), "s"(q_base) : "memory", "m0");
    }
    uint32_t low[2];                                               // first of the `reach` keys that the row sees (modulo 2^32: it may lie before key 0)
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const int j = wave * 64 + rb * 32 + col;
      low[rb] = (uint32_t)(j < nrows ? x0 + token_of(j) : x1) - (reach - 1u);
    }
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NLQ) : "memory");    // page ids
    rows_of(0);
#pragma unroll
    for (int i = 0; i < NLD; ++i) load_row(k_head, at_k[i], i, p0);
    rows_of(1);
#pragma unroll
    for (int i = 0; i < NLD; ++i) load_row(v_head, at_v[i], i, p0 + TILE_B);
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * NLD) : "memory");
    // fragments (B operand of K Q^T): of the wave's two blocks of 32 rows, lane holds row = col, k = 16 * ks + 8 * half .. + 8
    bf16x8_t qfrag[2][KS];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qfrag[rb][ks] = *(lds_bf16x8*)((ka0 + (uint32_t)((2 + wave) * TILE_B + rb * 32 * RB)) ^ (uint32_t)(ks * 32));
        asm volatile("" : "+a"(qfrag[rb][ks]));                    // (in accumulation registers, where matrix products can take them; elsewhere the compiler spills)
      }
    float ref[2] = {kPtUnset, kPtUnset};                           // the rows' reference exponents
    float lsum[2] = {0.f, 0.f};                                    // this lane's keys' weights
    float factor = c2;                                             // 1 once the logits are rounded first
    f32x16_t oacc[2][NBO];                                         // O^T: d = 32 * nb + 8 * (e / 4) + 4 * half + e % 4
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int nb = 0; nb < NBO; ++nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[rb][nb][e] = 0.f;


    // ---- blocks of 32 keys, two to a tile.  While the vector ALU forms the weights of block j, the matrix cores form the scores of
    // block j + 1 and add the output of block j - 1.
    f32x16_t s[2][2];                                              // [block parity][row block] S^T: key 8 * (e / 4) + 4 * half + e % 4
    uint32_t pk[FULL ? 3 : 2][2][8];                               // [part][row block] the last block's weights; rounded ones [block parity][row block]
    auto round_logits = [&](f32x16_t (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[rb][e] *= c2;
    };
    // Raises the rows' references above the logits x of a block, with what has been added up so far
    auto raise = [&](f32x16_t (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        float m = ref[rb];
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, factor * x[rb][e] + kPtHead);
        m = fmaxf(m, __shfl_xor(m, 32));                         // both halves of a row raise its reference together
        const float f = __builtin_amdgcn_exp2f(ref[rb] - m);     // 1 where nothing changes, 0 while the reference is unset
        lsum[rb] *= f;
#pragma unroll
        for (int nb = 0; nb < NBO; ++nb)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[rb][nb][e] *= f;
        ref[rb] = m;
      }
      const bool big = (fabsf(ref[0]) > kPtBig && ref[0] != kPtUnset) || (fabsf(ref[1]) > kPtBig && ref[1] != kPtUnset);
      if (__builtin_expect(f1 != INT_MIN && __builtin_amdgcn_ballot_w64(big) != 0, 0)) {
        // An fma's exact product is off by up to 2^-24 of the logit from the rounded one that the reference came from, and with logits of 2^31 that
        // alone would over- or underflow the exponential: from here on the logits are rounded first.
        factor = 1.f; f1 = INT_MIN;
        round_logits(x);                                         // (later blocks round their own)
      }
    };
    constexpr int AHEAD = 3;
    bf16x8_t carry[AHEAD];
    auto body_rounded = [&](auto half_c, int it, uint32_t k_at, uint32_t v_at, auto with_scores, auto with_output, auto with_loads, auto masked_c) __attribute__((always_inline)) {
      constexpr int CUR = decltype(half_c)::value, NXT = 1 - CUR;  // this block is half CUR of tile `it`
      constexpr bool SC = decltype(with_scores)::value, OUT = decltype(with_output)::value, LD = decltype(with_loads)::value;
      constexpr bool MASKED = decltype(masked_c)::value;
      f32x16_t (&x)[2] = s[CUR];
      const int j0 = key0 + it * kPtTile + CUR * 32 + 4 * half;    // key of element 0
      if constexpr (MASKED) {
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t key = (uint32_t)(j0 + 8 * (e >> 2) + (e & 3)) - low[rb];   // counted from the first that the row sees
            x[rb][e] = key < reach ? x[rb][e] : hidden;
          }
        if (__builtin_expect(f1 == INT_MIN, 0)) round_logits(x);
      }
      const uint32_t kt = ka0 + k_at + (uint32_t)(NXT * 32 * RB), vt = va0 + v_at + (uint32_t)(TILE_B + NXT * 32 * RB);
      constexpr int NS = KS + 2 * NBO, T0 = SC ? 0 : KS, T1 = OUT ? NS : KS; // steps: scores, then output; two products each
      constexpr int PPS = 16 / NS;                                 // pairs of weights per step
      constexpr bool CIN = CUR == 0 && OUT;                        // this block's first fragments were read at the end of the one before
      bf16x8_t frag[NS];                                           // of step t: K rows of the next block (t < KS), V^T of the last one
      auto fetch = [&](int t) __attribute__((always_inline)) {
        if (t < KS) { frag[t] = *(lds_bf16x8*)(kt ^ (uint32_t)(t * 32)); return; }
        const int k2 = (t - KS) / NBO, nb = (t - KS) % NBO;        // k-step k2 takes keys 16 * k2 + 4 * half + {0..3, 8..11}, the keys of x[8 * k2 ..]
        s16x4_t v[2];
#pragma unroll
        for (int h8 = 0; h8 < 2; ++h8)
          v[h8] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((vt ^ (uint32_t)(nb * 64 + h8 * VH)) + (uint32_t)((k2 * 16 + h8 * 8) * RB)));
        const uint2 v0 = __builtin_bit_cast(uint2, v[0]), v1 = __builtin_bit_cast(uint2, v[1]);
        frag[t] = __builtin_bit_cast(bf16x8_t, make_uint4(v0.x, v0.y, v1.x, v1.y));
      };
      auto weights_of = [&](int rb, int k2) __attribute__((always_inline)) -> bf16x8_t {
        const uint32_t (&pw)[8] = pk[NXT][rb];
        return __builtin_bit_cast(bf16x8_t, make_uint4(pw[4 * k2], pw[4 * k2 + 1], pw[4 * k2 + 2], pw[4 * k2 + 3]));
      };
      uint32_t any = 0u;
      float y[16][2], w[16][2], sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
      // pair i of the 16 pairs of weights, in three stages a step apart: none of a step's instructions waits for another of them
      auto exponent = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) y[i][u] = fmaf(factor, x[i >> 3][2 * (i & 7) + u], -ref[i >> 3]);
      };
      auto power = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) w[i][u] = __builtin_amdgcn_exp2f(y[i][u]);
      };
      auto pack = [&](int i) __attribute__((always_inline)) {
        const bf16x2_t p = {(__bf16)w[i][0], (__bf16)w[i][1]};
        pk[CUR][i >> 3][i & 7] = __builtin_bit_cast(uint32_t, p);
        if (MASKED) any |= pk[CUR][i >> 3][i & 7];
#pragma unroll
        for (int u = 0; u < 2; ++u) sum[i >> 3][u] += w[i][u];
      };
#pragma unroll
      for (int t = T0; t < T1 && t < T0 + AHEAD; ++t) { if (CIN) frag[t] = carry[t - T0]; else fetch(t); }
      auto product = [&](int t, int rb) __attribute__((always_inline)) {
        if (t < T0 || t >= T1) return;
        if (t < KS) s[NXT][rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[t], qfrag[rb][t < KS ? t : 0], t == 0 ? (f32x16_t){} : s[NXT][rb], 0, 0, 0);
        else oacc[rb][(t - KS) % NBO] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[t], weights_of(rb, (t - KS) / NBO), oacc[rb][(t - KS) % NBO], 0, 0, 0);
      };
      // A step: two products, a fragment read AHEAD steps before its use, a row load, pairs of weights
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        product(t, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (t >= T0 && t + AHEAD < T1) fetch(t + AHEAD);
        if (CUR == 1 && SC && t + AHEAD >= NS)                     // of K tile it + 1, second half
          carry[t + AHEAD - NS] = *(lds_bf16x8*)((ka0 + p1 + (uint32_t)(32 * RB)) ^ (uint32_t)((t + AHEAD - NS) * 32));
#pragma unroll
        for (int i = t * PPS; i < (t + 1) * PPS; ++i) { if (i >= 2 * PPS) pack(i - 2 * PPS); exponent(i); }
        __builtin_amdgcn_sched_barrier(0);
        product(t, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (LD && t < NLD) {                                       // rows of K tile it + 3 and V tile it + 2
          load_row(k_head, at_k[t < NLD ? t : 0], t, p0);
          load_row(v_head, at_v[t < NLD ? t : 0], t, p2 + TILE_B);
        }
        if (LD && t == NLD) { pages_of(it + 4); fetch_look(it + 6); }
        if (CUR == 0 && OUT && t == 2) rows_at(it + 3);            // (of the ids that the block before has read: no wait stands between)
#pragma unroll
        for (int i = t * PPS; i < (t + 1) * PPS; ++i) if (i >= PPS) power(i - PPS);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 16 - PPS; i < 16; ++i) power(i);
#pragma unroll
      for (int i = 16 - 2 * PPS; i < 16; ++i) pack(i);
      if (!MASKED) bad = bad || !(fmaxf(sum[0][0] + sum[0][1], sum[1][0] + sum[1][1]) <= kPtMost);
      if (MASKED && __builtin_amdgcn_ballot_w64((any & kPtTwo) != 0u) != 0) {
        // first visible key of a row, or a logit far above the reference.  Straight-line code: a branch per lane here
        // makes the compiler copy the accumulators on the common path too.
        raise(x);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) sum[rb][0] = sum[rb][1] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) { exponent(i); power(i); pack(i); }
      }
      lsum[0] += sum[0][0] + sum[0][1];
      lsum[1] += sum[1][0] + sum[1][1];
    };
    // The same with weights of 24 bits, each the sum of three bf16 numbers that V is multiplied with.  The output takes three of four products then, and the order
    // changes: first the output of block j - 1 while the weights of block j are formed in the place of its scores, then the scores of block
    // j + 1; the weights of a k-step are split once the former block's weights of that k-step have been multiplied.  With masks the reference is raised
    // before the weights are formed, when both the output of block j - 1 and the block's largest logit are there.
    auto body_full = [&](auto half_c, int it, uint32_t k_at, uint32_t v_at, auto with_scores, auto with_output, auto with_loads, auto masked_c) __attribute__((always_inline)) {
      constexpr int CUR = decltype(half_c)::value, NXT = 1 - CUR;
      constexpr bool SC = decltype(with_scores)::value, OUT = decltype(with_output)::value, LD = decltype(with_loads)::value;
      constexpr bool MASKED = decltype(masked_c)::value;
      f32x16_t (&x)[2] = s[CUR];
      const int j0 = key0 + it * kPtTile + CUR * 32 + 4 * half;
      const uint32_t kt = ka0 + k_at + (uint32_t)(NXT * 32 * RB), vt = va0 + v_at + (uint32_t)(TILE_B + NXT * 32 * RB);
      constexpr int VS = 2 * NBO, NS = VS + KS, G0 = OUT ? 0 : VS, G1 = SC ? NS : VS;   // steps: output (six products each), then scores (two)
      constexpr bool CIN = CUR == 0 && OUT;
      bf16x8_t frag[NS];
      auto read_v = [&](uint32_t at, int g) __attribute__((always_inline)) -> bf16x8_t {
        const int k2 = g / NBO, nb = g % NBO;
        s16x4_t v[2];
#pragma unroll
        for (int h8 = 0; h8 < 2; ++h8)
          v[h8] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((at ^ (uint32_t)(nb * 64 + h8 * VH)) + (uint32_t)((k2 * 16 + h8 * 8) * RB)));
        const uint2 v0 = __builtin_bit_cast(uint2, v[0]), v1 = __builtin_bit_cast(uint2, v[1]);
        return __builtin_bit_cast(bf16x8_t, make_uint4(v0.x, v0.y, v1.x, v1.y));
      };
      auto fetch = [&](int g) __attribute__((always_inline)) {
        if (g < VS) frag[g] = read_v(vt, g);
        else frag[g] = *(lds_bf16x8*)(kt ^ (uint32_t)((g - VS) * 32));
      };
      auto ahead = [&](int g) __attribute__((always_inline)) {
        if (g >= G0 && g + AHEAD < G1) fetch(g + AHEAD);
        if (CUR == 1 && SC && g + AHEAD >= NS) carry[g + AHEAD - NS] = read_v(va0 + p0 + (uint32_t)(TILE_B + 32 * RB), g + AHEAD - NS);   // of V tile it, second half
      };
      auto loads = [&](int g) __attribute__((always_inline)) {
        if (LD && g < NLD) {                                       // rows of K tile it + 3 and V tile it + 2
          load_row(k_head, at_k[g < NLD ? g : 0], g, p0);
          load_row(v_head, at_v[g < NLD ? g : 0], g, p2 + TILE_B);
        }
        if (LD && g == NLD) { pages_of(it + 4); fetch_look(it + 6); }
        if (CUR == 0 && OUT && g == 2) rows_at(it + 3);
      };
      // pair q of the 16 pairs of weights, those of k-step 0 first: elements 2 i and 2 i + 1 of row block rb
      float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
      auto rb_of = [](int q) { return (q >> 2) & 1; };
      auto i_of = [](int q) { return (q & 3) + 4 * (q >> 3); };
      auto exponent = [&](int q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) { float e = x[rb_of(q)][2 * i_of(q) + u]; x[rb_of(q)][2 * i_of(q) + u] = fmaf(factor, e, -ref[rb_of(q)]); }
      };
      auto power = [&](int q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) x[rb_of(q)][2 * i_of(q) + u] = __builtin_amdgcn_exp2f(x[rb_of(q)][2 * i_of(q) + u]);
      };
      auto add = [&](int q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) sum[rb_of(q)][u] += x[rb_of(q)][2 * i_of(q) + u];
      };
      // Parts are cut off, not rounded; the third holds the last 8 bits.  With masks the lower two are kept above 2^-30 of the weight, so that an infinite V row
      // comes out infinite (0 * inf would be NaN); without, a result that is not finite has the piece done again.
      auto split = [&](int q) __attribute__((always_inline)) {
        float y0 = x[rb_of(q)][2 * i_of(q)], y1 = x[rb_of(q)][2 * i_of(q) + 1];
        const float l0 = y0 * 9.3132257e-10f, l1 = y1 * 9.3132257e-10f;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
          pk[c][rb_of(q)][i_of(q)] = __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(y0), 0x07060302u);   // the high halves
          if (c < 2) {
            y0 -= __uint_as_float(__float_as_uint(y0) & 0xffff0000u);                    // (exact)
            y1 -= __uint_as_float(__float_as_uint(y1) & 0xffff0000u);
            if (MASKED) { y0 = fmaxf(y0, l0); y1 = fmaxf(y1, l1); }
          }
        }
      };
      auto output = [&](int g, int c, int rb) __attribute__((always_inline)) {
        if (!OUT) return;
        const int k2 = g / NBO, nb = g % NBO;
        const uint32_t (&pw)[8] = pk[c][rb];
        oacc[rb][nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[g], __builtin_bit_cast(bf16x8_t, make_uint4(pw[4 * k2], pw[4 * k2 + 1], pw[4 * k2 + 2], pw[4 * k2 + 3])),
                                                               oacc[rb][nb], 0, 0, 0);
      };
      auto score = [&](int t, int rb) __attribute__((always_inline)) {
        if (SC) s[NXT][rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[VS + t], qfrag[rb][t], t == 0 ? (f32x16_t){} : s[NXT][rb], 0, 0, 0);
      };
#pragma unroll
      for (int g = G0; g < G1 && g < G0 + AHEAD; ++g) { if (CIN) frag[g] = carry[g - G0]; else fetch(g); }
      constexpr int FORM = 16 / VS, SPLIT = 8 / NBO, LATE = 8 / KS;   // pairs formed per output step, split per output step of k-step 1, split per score step
      if constexpr (MASKED) {
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t key = (uint32_t)(j0 + 8 * (e >> 2) + (e & 3)) - low[rb];
            x[rb][e] = key < reach ? x[rb][e] : hidden;
          }
        if (__builtin_expect(f1 == INT_MIN, 0)) round_logits(x);
#pragma unroll
        for (int g = 0; g < VS; ++g) {
          ahead(g);
          loads(g);
#pragma unroll
          for (int c = 0; c < 3; ++c) { output(g, c, 0); output(g, c, 1); }
        }
        float most[2] = {-INFINITY, -INFINITY};                    // exponents
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
          for (int e = 0; e < 16; ++e) most[rb] = fmaxf(most[rb], fmaf(factor, x[rb][e], -ref[rb]));
        if (__builtin_amdgcn_ballot_w64(fmaxf(most[0], most[1]) >= 1.f) != 0) raise(x);
#pragma unroll
        for (int q = 0; q < 16; ++q) { exponent(q); power(q); add(q); }
#pragma unroll
        for (int t = 0; t < KS; ++t) { ahead(VS + t); score(t, 0); score(t, 1); }
#pragma unroll
        for (int q = 0; q < 16; ++q) split(q);
      } else {
#pragma unroll
        for (int g = 0; g < VS; ++g) {
#pragma unroll
          for (int p = 0; p < 6; ++p) {
            output(g, p >> 1, p & 1);
            __builtin_amdgcn_sched_barrier(0);
            if (p == 0) {
              ahead(g);
#pragma unroll
              for (int q = g * FORM; q < (g + 1) * FORM; ++q) exponent(q);
            }
            if (p == 3) loads(g);
            if (p >= 1 && p <= 4) {
#pragma unroll
              for (int k = (p - 1) * FORM / 4; k < p * FORM / 4; ++k) power(g * FORM + k);
              if (g >= NBO) {
#pragma unroll
                for (int k = (p - 1) * SPLIT / 4; k < p * SPLIT / 4; ++k) split((g - NBO) * SPLIT + k);
              }
            }
            if (p == 5) {
#pragma unroll
              for (int q = g * FORM; q < (g + 1) * FORM; ++q) add(q);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
#pragma unroll
        for (int t = 0; t < KS; ++t) {
          score(t, 0);
          __builtin_amdgcn_sched_barrier(0);
          ahead(VS + t);
#pragma unroll
          for (int q = 8 + t * LATE; q < 8 + (t + 1) * LATE; ++q) split(q);
          __builtin_amdgcn_sched_barrier(0);
          score(t, 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        bad = bad || !(fmaxf(sum[0][0] + sum[0][1], sum[1][0] + sum[1][1]) <= kPtMost);
      }
      lsum[0] += sum[0][0] + sum[0][1];
      lsum[1] += sum[1][0] + sum[1][1];
    };
    auto body = [&](auto... args) __attribute__((always_inline)) { if constexpr (FULL) body_full(args...); else body_rounded(args...); };
    // Buffers: the barrier between the blocks of tile `it` says that K tile it + 1 and V tile `it` have arrived (and the page ids of tile
    // it + 4) and that K tile `it` and V tile it - 1 have been read, whose places K tile it + 3 and V tile it + 2 then take.  What tile it - 1
    // requested -- K tile it + 2, V tile it + 1, page ids -- stays in flight.
    constexpr int BATCH = 2 * NLD + 1;
    auto tile_barrier = [&](auto in_flight) __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(decltype(in_flight)::value) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    auto next_tile = [&]() __attribute__((always_inline)) { const uint32_t p = p0; p0 = p1; p1 = p2; p2 = p; };
    using One = std::integral_constant<int, BATCH>;
    using B0 = std::integral_constant<int, 0>;
    using B1 = std::integral_constant<int, 1>;
    using Yes = std::true_type;
    using No = std::false_type;
    tile_barrier(std::integral_constant<int, NLD>{});              // K tile 0 has arrived, and every wave has read its queries
    // the scores of the first block; K tiles 1 and 2 and V tile 1 are requested meanwhile, in the queries' places
    bf16x8_t k_first[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) k_first[ks] = *(lds_bf16x8*)((ka0 + p0) ^ (uint32_t)(ks * 32));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) s[0][rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_first[ks], qfrag[rb][ks], ks == 0 ? (f32x16_t){} : s[0][rb], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NLD; ++i) load_row(k_head, at_k[i], i, p1);
    fetch_look(4);
    rows_of(2);
#pragma unroll
    for (int i = 0; i < NLD; ++i) { load_row(k_head, at_k[i], i, p2); load_row(v_head, at_v[i], i, p1 + TILE_B); }
    fetch_look(5);
    rows_of(3);
    // the first reference: above the block's largest exponent (a row that sees none of its keys, or one with large logits, gets its own later)
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      float m = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, (uint32_t)(key0 + 4 * half + 8 * (e >> 2) + (e & 3)) - low[rb] < reach ? c2 * s[0][rb][e] : -INFINITY);
      m = fmaxf(m, __shfl_xor(m, 32)) + kPtHead;
      ref[rb] = fabsf(m) <= kPtBig ? m : kPtUnset;
    }
    body(B0{}, 0, p0, p0, Yes{}, No{}, No{}, Yes{});
    // tiles in turn: second half of tile `it`, first half of tile it + 1.  (Three loops and not one: with both copies of the code in one loop
    // the compiler spills registers.)
    int it = 0;
    for (; it + 1 < nt && it < f0; ++it) {
      tile_barrier(One{});
      body(B1{}, it, p1, p0, Yes{}, Yes{}, Yes{}, Yes{});
      body(B0{}, it + 1, p1, p0, Yes{}, Yes{}, No{}, Yes{});
      next_tile();
    }
    for (; it + 1 < f1; ++it) {
      tile_barrier(One{});
      body(B1{}, it, p1, p0, Yes{}, Yes{}, Yes{}, No{});
      body(B0{}, it + 1, p1, p0, Yes{}, Yes{}, No{}, No{});
      next_tile();
    }
    for (; it + 1 < nt; ++it) {
      tile_barrier(One{});
      body(B1{}, it, p1, p0, Yes{}, Yes{}, Yes{}, Yes{});
      body(B0{}, it + 1, p1, p0, Yes{}, Yes{}, No{}, Yes{});
      next_tile();
    }
    tile_barrier(One{});
    body(B1{}, nt - 1, p1, p0, No{}, Yes{}, No{}, Yes{});
    // the output of the last block
    const uint32_t vt = va0 + p0 + (uint32_t)(TILE_B + 32 * RB);
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int nb = 0; nb < NBO; ++nb) {
        s16x4_t v[2];
#pragma unroll
        for (int h8 = 0; h8 < 2; ++h8)
          v[h8] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((vt ^ (uint32_t)(nb * 64 + h8 * VH)) + (uint32_t)((k2 * 16 + h8 * 8) * RB)));
        const uint2 v0 = __builtin_bit_cast(uint2, v[0]), v1 = __builtin_bit_cast(uint2, v[1]);
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(v0.x, v0.y, v1.x, v1.y));
#pragma unroll
        for (int c = FULL ? 0 : 1; c < (FULL ? 3 : 2); ++c)
#pragma unroll
          for (int rb = 0; rb < 2; ++rb) {
            const uint32_t (&pw)[8] = pk[c][rb];
            oacc[rb][nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8_t, make_uint4(pw[4 * k2], pw[4 * k2 + 1], pw[4 * k2 + 2], pw[4 * k2 + 3])),
                                                                   oacc[rb][nb], 0, 0, 0);
          }
      }
    if (!again) {                                                  // large values of V times large weights, or an infinite one times a part that is 0
      float x = 0.f;
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int nb = 0; nb < NBO; ++nb)
#pragma unroll
          for (int e = 0; e < 16; ++e) x = fmaf(oacc[rb][nb][e], 0.f, x);
      bad = bad || !(x == 0.f);
    }
    if (__builtin_amdgcn_ballot_w64(bad) != 0) *s_bad = 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // tiles past the end that were requested: their places are used below
    __syncthreads();
    if (*s_bad != 0) return true;

    // ---- results: whole tiles by way of LDS, 16 bytes of a row per lane; pieces as they lie in the registers (the merge knows)
    uint8_t* mine = smem + wave * 64 * RB;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const int jw = rb * 32 + col, j = wave * 64 + jw;
      const float l = lsum[rb] + __shfl_xor(lsum[rb], 32);
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;             // (a sum that is no number stays one)
#pragma unroll
        for (int nb = 0; nb < NBO; ++nb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const bf16x2_t y0 = {(__bf16)(oacc[rb][nb][q4 * 4] * inv), (__bf16)(oacc[rb][nb][q4 * 4 + 1] * inv)};
            const bf16x2_t y1 = {(__bf16)(oacc[rb][nb][q4 * 4 + 2] * inv), (__bf16)(oacc[rb][nb][q4 * 4 + 3] * inv)};
            *reinterpret_cast<uint2*>(mine + jw * RB + (((nb * 4 + q4) ^ (jw & (PPR - 1))) * 16) + half * 8) =
                make_uint2(__builtin_bit_cast(uint32_t, y0), __builtin_bit_cast(uint32_t, y1));
          }
        if (half == 0 && j < nrows && a.lse != nullptr) a.lse[tile_row + row_at(j)] = l == 0.f ? -INFINITY : (ref[rb] + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
      } else {
        float4* po = reinterpret_cast<float4*>(sh.part_o + ((size_t)wg * 2 + slot) * kPtRows * D) + (wave * 2 + rb) * (NBO * 4 * 64) + lane;
#pragma unroll
        for (int nb = 0; nb < NBO; ++nb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            po[(nb * 4 + q4) * 64] = make_float4(oacc[rb][nb][q4 * 4], oacc[rb][nb][q4 * 4 + 1], oacc[rb][nb][q4 * 4 + 2], oacc[rb][nb][q4 * 4 + 3]);
        if (half == 0) {
          float* pm = sh.part_ml + (((size_t)wg * 2 + slot) * kPtRows + j) * 2;
          pm[0] = l == 0.f ? -INFINITY : ref[rb] * 0.69314718055994530942f; pm[1] = l;      // in units of the logits
        }
      }
    }
    if (whole) {
      uint8_t* o_base = a.out + tile_row * RB;
      int o_key = st_key;
      asm volatile("" : "+v"(o_key));
      u32x4_t y[64 / KPI];                                         // (all of them are read first: with a read and a store in turn, each would wait for the other)
#pragma unroll
      for (int i = 0; i < 64 / KPI; ++i) {
        const int jw = i * KPI + o_key;
        y[i] = *reinterpret_cast<const u32x4_t*>(mine + jw * RB + ((st_pos ^ (jw & (PPR - 1))) * 16));
      }
#pragma unroll
      for (int i = 0; i < 64 / KPI; ++i) {
        const int j = wave * 64 + i * KPI + o_key;
        if (j < nrows) *reinterpret_cast<u32x4_t*>(o_base + (row_at((uint32_t)j) * RB + (uint32_t)(st_pos * 16))) = y[i];
      }
    }
    return false;
  });
}

template <int D, bool FULL>
static hipError_t tall_one(const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s) {
  constexpr int lds = 2 * kPtBuf * kPtTile * D * 2 + 4 * kPtRing * 256 + sizeof(ShareScratch) + 16;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_tall_kernel<D, FULL>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((paged_tall_kernel<D, FULL>), dim3(sh.wgs), dim3(256), lds, s, a, sh);
  return hipGetLastError();
}

hipError_t launch_paged_tall(int D, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s) {
  if (a.round_weights) return D == 64 ? tall_one<64, false>(a, sh, s) : tall_one<128, false>(a, sh, s);
  return D == 64 ? tall_one<64, true>(a, sh, s) : tall_one<128, true>(a, sh, s);
}

}  // namespace ts
