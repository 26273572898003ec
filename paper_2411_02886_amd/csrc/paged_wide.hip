// Dense attention of many new tokens, bf16 queries, over a cache in 8 bits, and of drafted trees over one in bf16: on the matrix cores.
//
// A tile is 256 rows (256 / G tokens times the G heads of a KV head) in eight waves of 32, two to a SIMD (or 128 rows, see below): while one of them forms weights on the vector
// ALU the other one's matrix products run.  All walk the same tiles of 64 keys, which the workgroup widens to bf16 (codes are small numbers that bf16
// holds) and puts into LDS, a tile ahead of their use and requested another one ahead; one barrier a tile.  Scores get their key's scale, weights their
// value's.  A weight is multiplied with V as the sum of two bf16 numbers, each rounded to nearest (8 bits): what the first leaves is at most half its last bit, 2^-8 of the weight,
// and the second leaves at most 2^-9 of that, so that 2^-17 of a weight is lost where the result is rounded by up to 2^-8.  (Three parts, all 24 bits: a third product for every
// two.  The kernel is bound by the power of the matrix cores: 512 bf16 tokens, 28/4 heads, over 65536 keys 703 us = 1030 TFLOP/s of products, where a product of two square matrices of 8192 reaches 1225; by the stream kernel's tiles of 64 rows 1356.)
#include "paged_shares.h"
#include "ts_codes.h"
#include <limits.h>
#include <type_traits>

namespace ts {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int kPwTile = 64;                   // keys per tile
constexpr int kPwThreads = 512;
constexpr int kPwRing = 4;                    // tiles whose scales are in LDS
constexpr float kPwUnset = -3.40282347e38f;   // reference exponent before the first key: no finite one lies below it
constexpr float kPwHead = 6.f;                // a raised reference lies this far above the largest exponent so far ...
constexpr float kPwRaise = 2.f;               // ... and is raised again when a lane's weights of a block exceed this together
constexpr int kRows16 = 2;                    // beside ts_code: rows of bf16 numbers

// place of a row's 16-byte pieces in LDS: 16 rows x one piece (K fragments) and 4 rows x 4 pieces (V^T) each fall on all banks
template <int D> __device__ __forceinline__ int pw_swz(int key) {
  return D == 128 ? (((key & 3) << 2) | ((key >> 2) & 3)) : ((((key >> 1) & 1) << 2) | (((key >> 2) & 1) << 1) | ((key >> 3) & 1));
}

// BLOCKS: blocks of 32 keys of a tile that a wave has.  2: waves of 32 rows each, 256 in all.  1: 128 rows, the second four waves have the rows of the first four and the other half of
// each tile's keys; the two halves of a row are joined in LDS behind the last tile.  (With up to 128 rows in tiles of 256 half of the waves would only stage, and the matrix cores rest while the
// other half forms its weights.)
template <int KIND, int D, int BLOCKS>
__global__ __launch_bounds__(kPwThreads, 2) void paged_wide_kernel(PagedAttnArgs a, QuantPools c, ShareArgs sh) {
  constexpr int ROWS = 128 * BLOCKS;
  constexpr int AHEAD = BLOCKS == 1 ? 2 : 1;  // tiles that loads are ahead of their way to LDS (those of 128 rows take hardly more time than a load: 24 sequences over 3000 bf16 keys, 32/8 heads, 96 rows 94 us, one ahead 102)
  constexpr int KS = D / 16, NB = D / 32;     // k-steps of K Q^T, 32-row blocks of the transposed output
  constexpr int RB = D * 2, TILE_B = kPwTile * RB;
  constexpr int SB = KIND == kRows16 ? RB : D;        // bytes of a row in the cache
  constexpr int NL = SB / 8 > 16 ? 2 : 1;     // loads per thread and row: eight threads have a row
  constexpr int LB = SB / 8 / NL;             // bytes of a load
  constexpr int VH = D == 128 ? 32 : 16;      // what eight keys more flip of a piece's place
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];   // K tiles [2], V tiles [2], scales [kPwRing][K's, V's], the share's ends
  float* const s_scale = reinterpret_cast<float*>(smem + 4 * TILE_B);
  ShareScratch* s_share = reinterpret_cast<ShareScratch*>(s_scale + kPwRing * 2 * kPwTile);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int H = a.H, G = a.H / a.H_kv;
  const bool tree = a.mask != nullptr;
  const int wg = share_of(blockIdx.x, sh.wgs);
  SharePlace from, to;
  SeqShape first;
  find_share<kPwTile, kPwThreads>(a, sh, G, wg, s_share, &from, &to, &first, tree);
  int32_t* desc = sh.desc + (size_t)wg * 8;
  if (!sh.whole && threadIdx.x == 0) { desc[3] = kPieceNone; desc[7] = kPieceNone; }
  const uint32_t g_inv = 65536u / (uint32_t)G + 1u;             // exact for rows below 256
  const float c2 = a.sm_scale * 1.44269504088896340736f;        // logits are exponents of two here
  const int row_shift = 31 - __builtin_clz((uint32_t)(a.H_kv * SB));   // H_kv is a power of two

  typedef const __attribute__((address_space(3))) bf16x8_t lds_bf16x8;
  typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
  // K fragment ks of block kb: row 32 kb + col, piece (2 ks + half) ^ swz(col) -- ks flips bits of the address only
  const uint32_t ka0 = lds_base + (uint32_t)(col * RB + ((half ^ pw_swz<D>(col)) * 16));
  // V^T: 16 lanes read 4 keys x 16 columns; lane i of them reads key i / 4, columns 4 (i % 4) ..; the output block and the upper eight
  // keys of a k-step flip bits of the piece
  const int vt_key = 4 * half + ((lane & 15) >> 2), vt_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const uint32_t va0 = lds_base + (uint32_t)(2 * TILE_B + vt_key * RB + (((vt_col >> 3) ^ pw_swz<D>(vt_key)) * 16) + (vt_col & 7) * 2);
  // staging: eight threads to a key
  const int st_key = threadIdx.x >> 3, st_part = threadIdx.x & 7;

  walk_share<kPwTile>(a, sh, G, from, to, first, [&](int kvh, const SeqShape& sq, int r, const TileKeys& keys, int ua, int ub, bool) -> bool {
    const int c0 = r * sh.tpt, ntok = min(sh.tpt, sq.n - c0), nrows = ntok * G;
    const int row0 = sq.row0 + c0, base = sq.N - sq.n;
    const bool whole = ua == 0 && ub == keys.units;
    const int tmax = keys.end - 1;
    auto token_of = [&](uint32_t j) -> int { return (int)min(__umul24(j, g_inv) >> 16, (uint32_t)(ntok - 1)); };   // j / G; rows past the last stand for it
    const size_t tile_row = (size_t)row0 * H + kvh * G;
    auto row_at = [&](uint32_t j) -> uint32_t { return __umul24(__umul24(j, g_inv) >> 16, (uint32_t)(H - G)) + j; };
    if (keys.end <= keys.first) {                                  // no row sees a token (one unit: the tile is not cut)
      for (int i = threadIdx.x; i < nrows * D; i += kPwThreads) {
        const size_t o = tile_row + row_at((uint32_t)(i / D));
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
    const int key0 = (keys.u0 + ua) * kPwTile, nt = ub - ua;       // first key and number of tiles
    const int late = wave >> 2, row_block = BLOCKS == 2 ? wave : wave & 3, key_block = BLOCKS == 2 ? 0 : late;   // (first block of the tile's keys)
    const int j = row_block * 32 + col;                            // the lane's row
    const bool there = j < nrows, busy = row_block * 32 < nrows;   // (a wave without rows only stages)

    // ---- a tile's keys from memory to LDS
    // (keys past the end or in front of the tile's first window stand for the nearest that some row sees: no other place of the cache is read)
    auto key_of = [&](int it) -> int { return min(max(key0 + it * kPwTile + st_key, keys.first), tmax); };
    auto page_of = [&](int it) -> int { return pages[key_of(it) >> a.p_shift]; };
    typedef typename std::conditional<LB == 16, u32x4_t, u32x2_t>::type load_t;   // (vectors: structs that are written under a condition would go by way of memory)
    load_t kr[AHEAD][NL], vr[AHEAD][NL];                           // requested: tiles of K, and the ones before of V (tile t in t % AHEAD)
    float scale[AHEAD] = {};                                       // of the tiles of K
    uint64_t at = 0;                                               // the place of the last tile of K in the pools
    const uint8_t* const k_head = (KIND == kRows16 ? a.k_pool : c.k_codes) + kvh * SB;
    const uint8_t* const v_head = (KIND == kRows16 ? a.v_pool : c.v_codes) + kvh * SB;
    // (formed anew in each turn: the compiler would keep dozens of addresses, and spill)
    auto fresh = [](uint32_t x) -> uint32_t { asm volatile("" : "+v"(x)); return x; };
    uint64_t before = 0;                                           // and of the one before
    int in_page = 0;
    auto locate = [&](int it, int page) __attribute__((always_inline)) {
      in_page = key_of(it) & (a.P - 1);
      before = at;
      at = ((uint64_t)(((uint32_t)page << a.p_shift) + (uint32_t)in_page) << row_shift) + (uint32_t)(st_part * LB);
    };
    auto request_k = [&](int i) __attribute__((always_inline)) {
#pragma unroll
      for (int l = 0; l < NL; ++l) kr[i][l] = *reinterpret_cast<const load_t*>(k_head + at + l * 8 * LB);
    };
    auto request_v = [&](int i) __attribute__((always_inline)) {
#pragma unroll
      for (int l = 0; l < NL; ++l) vr[i][l] = *reinterpret_cast<const load_t*>(v_head + before + l * 8 * LB);
    };
    auto request_scale = [&](int page, int i) __attribute__((always_inline)) {
      if (KIND != kRows16 && st_part < 2) scale[i] = (st_part == 0 ? c.k_scale : c.v_scale)[(((int64_t)page * a.H_kv + kvh) << a.p_shift) + in_page];
    };
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
    auto put = [&](uint32_t tile, const load_t (&x)[NL]) {
      const uint32_t key = fresh((uint32_t)st_key), row = lds_base + tile + key * RB, swz = (uint32_t)pw_swz<D>((int)(key & 15u)), part = (uint32_t)st_part;
      if constexpr (KIND == kRows16) {
#pragma unroll
        for (int l = 0; l < NL; ++l) *(lds_u32x4*)(row + (((part + 8 * l) ^ swz) * 16)) = x[l];
      } else {
#pragma unroll
        for (int p = 0; p < LB / 8; ++p) {
          const uint2 y = widen<KIND>(x[0][2 * p]), z = widen<KIND>(x[0][2 * p + 1]);
          *(lds_u32x4*)(row + (((part * (LB / 8) + p) ^ swz) * 16)) = u32x4_t{y.x, y.y, z.x, z.y};
        }
      }
    };
    auto put_k = [&](int it, int i) __attribute__((always_inline)) { put((uint32_t)((it & 1) * TILE_B), kr[i]); };
    auto put_v = [&](int it, int i) __attribute__((always_inline)) { put((uint32_t)((2 + (it & 1)) * TILE_B), vr[i]); };
    auto put_scale = [&](int it, int i) __attribute__((always_inline)) {
      if (KIND != kRows16 && st_part < 2) s_scale[((it & (kPwRing - 1)) * 2 + st_part) * kPwTile + st_key] = st_part == 0 ? scale[i] * c2 : scale[i];
    };
    int page = 0, page_then = 0;                                   // of the tile of K that is requested next, and the one after it
    // K tile it + 1 and V tile `it` to LDS, K tile it + 1 + AHEAD and V tile it + AHEAD requested: in steps, which stand between matrix products (parity: it % AHEAD)
    auto staging = [&](int it, auto parity, int part) __attribute__((always_inline)) {
      constexpr int v = decltype(parity)::value, k = AHEAD - 1 - v;
      if (part == 0) put_k(it + 1, k);
      if (part == 1) put_v(it, v);
      if (part == 2) { put_scale(it + 1, k); page_then = page_of(it + 2 + AHEAD); locate(it + 1 + AHEAD, page); }
      if (part == 3) request_k(k);
      if (part == 4) request_v(v);
      if (part == 5) { request_scale(page, k); page = page_then; }
    };

    // ---- queries: lane holds row col, elements 16 ks + 8 half ..
    bf16x8_t qf[KS];
    {
      const uint8_t* q = a.q + (tile_row + (there ? row_at((uint32_t)j) : 0u)) * (size_t)RB + half * 16;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        uint4 w = *reinterpret_cast<const uint4*>(q + ks * 32);
        if (!there) w = make_uint4(0u, 0u, 0u, 0u);
        qf[ks] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
    const int place = base + c0 + token_of((uint32_t)j);
    const int low = tree ? tree_low(a, row0 + token_of((uint32_t)j), sq.n, base) : a.window > 0 ? place - a.window + 1 : 0;
    float ref = kPwUnset, lsum = 0.f;                              // reference exponent of the row (the same in both of its lanes), this lane's keys' sum
    f32x16_t o[NB];                                                // O^T: d = 32 nb + 8 (e / 4) + 4 half + e % 4
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[nb][e] = 0.f;

    // ---- Waves 0 .. 3 and 4 .. 7, one of each to a SIMD, take turns: while the first form weights the others multiply, then the other way round. Between two
    // barriers a wave either adds the output of tile it - 1 and forms the scores of tile `it` (the matrix cores), its part of the staging between the products, or forms
    // the weights of tile `it` (the vector ALU); the second four do what the first did a turn before.  K tile `it` and V tile it - 1 are read in turns 2 it and
    // 2 it + 1, and those that follow staged in the same turns into the places of those before, which have been read by then.
    f32x16_t s[BLOCKS];                                            // S^T of the wave's blocks of 32 keys: key 8 (e / 4) + 4 half + e % 4
    uint32_t w[BLOCKS][2][8];                                      // [block][part] their weights; k-step k2 takes elements 8 k2 ..
    // weights 2 i and 2 i + 1 of a block, as the sums of two bf16 numbers each
    auto split = [&](int kb, int i) __attribute__((always_inline)) {
      const float y0 = s[kb][2 * i], y1 = s[kb][2 * i + 1];
      const uint32_t hi = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)y0, (__bf16)y1});
      w[kb][0][i] = hi;
      w[kb][1][i] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)(y0 - bf16_lo(hi)), (__bf16)(y1 - bf16_hi(hi))});
    };
    // O^T += V^T P^T of a tile, by pairs of blocks (the two products of a block stand a block apart: the second waits for the first), fragments a pair ahead
    auto output = [&](int it, auto stages, auto parity) __attribute__((always_inline)) {
      const uint32_t vt = fresh(va0 + (uint32_t)((it & 1) * TILE_B + key_block * 32 * RB));
      bf16x8_t vf[2][2];
      auto fetch = [&](int t) __attribute__((always_inline)) {      // pair t: keys 16 (2 t / NB) .. of the wave's, blocks 2 t % NB and the next
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int k4 = 2 * t / NB, nb = 2 * t % NB + u;
          s16x4_t v[2];
#pragma unroll
          for (int h8 = 0; h8 < 2; ++h8)
            v[h8] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((vt ^ (uint32_t)(nb * 64 + h8 * VH)) + (uint32_t)((k4 * 16 + h8 * 8) * RB)));
          const uint2 v0 = __builtin_bit_cast(uint2, v[0]), v1 = __builtin_bit_cast(uint2, v[1]);
          vf[t & 1][u] = __builtin_bit_cast(bf16x8_t, make_uint4(v0.x, v0.y, v1.x, v1.y));
        }
      };
      fetch(0);
#pragma unroll
      for (int t = 0; t < BLOCKS * NB; ++t) {
        if (t + 1 < BLOCKS * NB) fetch(t + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int k4 = 2 * t / NB, nb = 2 * t % NB + u, k2 = k4 & 1;
            const uint32_t (&y)[8] = w[k4 >> 1][part];
            o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t & 1][u], __builtin_bit_cast(bf16x8_t, make_uint4(y[4 * k2], y[4 * k2 + 1], y[4 * k2 + 2], y[4 * k2 + 3])), o[nb], 0, 0, 0);
          }
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(stages)::value) {
          constexpr int EACH = 8 / (BLOCKS * NB);
#pragma unroll
          for (int i = t * EACH; i < (t + 1) * EACH; ++i) staging(it + 1, parity, i);
        }
        if (BLOCKS == 2 && t < NB) {                               // the second block's weights, while the first one's are multiplied
#pragma unroll
          for (int i = t * (8 / NB); i < (t + 1) * (8 / NB); ++i) split(BLOCKS - 1, i);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto scores = [&](int it) __attribute__((always_inline)) {
      const uint32_t kt = fresh(ka0 + (uint32_t)((it & 1) * TILE_B + key_block * 32 * RB));
      bf16x8_t kf[KS][BLOCKS];
      auto fetch = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < BLOCKS; ++kb) kf[ks][kb] = *(lds_bf16x8*)((kt ^ (uint32_t)(ks * 32)) + (uint32_t)(kb * 32 * RB));
      };
      fetch(0);
      fetch(1);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 2 < KS) fetch(ks + 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < BLOCKS; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks][kb], qf[ks], ks == 0 ? (f32x16_t){} : s[kb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto weights = [&](int it) __attribute__((always_inline)) {
      const float* const scales = s_scale + (it & (kPwRing - 1)) * 2 * kPwTile + key_block * 32;
      const int k0 = key0 + it * kPwTile + key_block * 32;
      const bool masked = k0 + 32 * BLOCKS - 1 > (tree ? base - 1 : base + c0) || (a.window > 0 && k0 <= (tree ? base + sq.n - 1 : base + c0 + ntok - 1) - a.window);
#pragma unroll
      for (int kb = 0; kb < BLOCKS; ++kb) {
        f32x16_t& x = s[kb];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {                           // (rounded before the reference is taken off: a fused product of large logits would be off by more than a weight)
          const float4 k4 = KIND == kRows16 ? make_float4(c2, c2, c2, c2) : *reinterpret_cast<const float4*>(scales + kb * 32 + 8 * q4 + 4 * half);
          x[4 * q4] *= k4.x; x[4 * q4 + 1] *= k4.y; x[4 * q4 + 2] *= k4.z; x[4 * q4 + 3] *= k4.w;
        }
      }
      uint32_t bits[BLOCKS];                                // the keys that the row sees
#pragma unroll
      for (int kb = 0; kb < BLOCKS; ++kb) bits[kb] = ~0u;
      if (__builtin_expect(masked, 0)) {
#pragma unroll
        for (int kb = 0; kb < BLOCKS; ++kb) {
          const int b0 = k0 + kb * 32;
          if (tree) bits[kb] = tree_bits(a, row0 + token_of((uint32_t)j), sq.n, base, low, b0);
          else {
            const int many = min(max(place + 1 - b0, 0), 32), cut = min(max(low - b0, 0), 32);
            bits[kb] = (uint32_t)(((1ull << many) - 1ull) & ~((1ull << cut) - 1ull));
          }
          bits[kb] >>= 4 * half;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[kb][e] = (bits[kb] >> (8 * (e >> 2) + (e & 3)) & 1u) != 0u ? s[kb][e] : -INFINITY;
        }
      }
      auto sum_of = [&](f32x16_t& p, const f32x16_t& x) __attribute__((always_inline)) -> float {
        float sum = 0.f, more = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          p[e] = __builtin_amdgcn_exp2f(x[e] - ref); p[e + 1] = __builtin_amdgcn_exp2f(x[e + 1] - ref);
          sum += p[e]; more += p[e + 1];
        }
        return sum + more;
      };
#pragma unroll
      for (int kb = 0; kb < BLOCKS; ++kb) {
        f32x16_t p;
        float sum = sum_of(p, s[kb]);
        if (__builtin_amdgcn_ballot_w64(!(sum <= kPwRaise)) != 0) {            // a key far above the reference, such as a row's first
          float m = s[kb][0];
#pragma unroll
          for (int e = 1; e < 16; ++e) m = fmaxf(m, s[kb][e]);
          m = fmaxf(m, __shfl_xor(m, 32)) + kPwHead;
          m = fmaxf(m, ref);
          const float f = __builtin_amdgcn_exp2f(ref - m);         // 0 while the reference is unset, 1 where it stays
          lsum *= f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[nb][e] *= f;
          if (kb == 1) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[0][e] *= f;
          }
          ref = m;
          sum = sum_of(p, s[kb]);
        }
        lsum += sum;
        s[kb] = p;
      }
      if constexpr (KIND != kRows16) {
#pragma unroll
        for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            float4 v4 = *reinterpret_cast<const float4*>(scales + kPwTile + kb * 32 + 8 * q4 + 4 * half);
            if (__builtin_expect(masked, 0)) {                     // (a scale may be no number)
              const uint32_t b4 = bits[kb] >> (8 * q4);
              v4 = make_float4((b4 & 1u) != 0u ? v4.x : 0.f, (b4 & 2u) != 0u ? v4.y : 0.f, (b4 & 4u) != 0u ? v4.z : 0.f, (b4 & 8u) != 0u ? v4.w : 0.f);
            }
            s[kb][4 * q4] *= v4.x; s[kb][4 * q4 + 1] *= v4.y; s[kb][4 * q4 + 2] *= v4.z; s[kb][4 * q4 + 3] *= v4.w;
          }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) split(0, i);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, AHEAD - 1>;
    __syncthreads();                                               // the tiles of the piece before have been read
    {
      const int p0 = page_of(0), p1 = page_of(1), p2 = page_of(2);
      page = AHEAD == 2 ? page_of(3) : p2;
      locate(0, p0);
      request_k(0);
      request_scale(p0, 0);
      if (AHEAD == 1) { put_k(0, 0); put_scale(0, 0); }
      locate(1, p1);
      request_k(AHEAD - 1);
      request_v(0);
      request_scale(p1, AHEAD - 1);
      if (AHEAD == 2) {
        put_k(0, 0);
        put_scale(0, 0);
        locate(2, p2);
        request_k(0);
        request_v(AHEAD - 1);
        request_scale(p2, 0);
      }
    }
    __syncthreads();
    if (late) __syncthreads();
    auto turn = [&](int it, auto parity) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
      if (busy && it > 0) output(it - 1, Yes{}, parity);
      else {
#pragma unroll
        for (int i = 0; i < 6; ++i) staging(it, parity, i);
      }
      if (busy) scores(it);
      __builtin_amdgcn_s_setprio(0);
      __syncthreads();
      if (busy) weights(it);
      __syncthreads();
    };
    for (int it = 0; it < nt; it += AHEAD) {
      turn(it, Even{});
      if (AHEAD == 2 && it + 1 < nt) turn(it + 1, Odd{});
    }
    if (busy) output(nt - 1, No{}, Even{});
    if (!late) __syncthreads();

    // ---- results: whole tiles are written, pieces left as they lie in the registers (the merge knows)
    if (!busy && BLOCKS == 2) return false;
    if constexpr (BLOCKS == 1) {                                   // the second four waves' sums to the first, in the place of the tiles and scales
      float4* const half_o = reinterpret_cast<float4*>(smem) + row_block * (NB * 4 * 64) + lane;
      float2* const half_ml = reinterpret_cast<float2*>(s_scale) + row_block * 64 + lane;
      __syncthreads();                                             // which have been read
      if (busy && late) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) half_o[(nb * 4 + q4) * 64] = make_float4(o[nb][q4 * 4], o[nb][q4 * 4 + 1], o[nb][q4 * 4 + 2], o[nb][q4 * 4 + 3]);
        *half_ml = make_float2(ref, lsum);
      }
      __syncthreads();
      if (!busy || late) return false;
      const float2 ml = *half_ml;
      const float m = fmaxf(ref, ml.x), f = __builtin_amdgcn_exp2f(ref - m), g = __builtin_amdgcn_exp2f(ml.x - m);   // (a half without keys of the row: its sums are 0)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 x = half_o[(nb * 4 + q4) * 64];
          o[nb][q4 * 4] = fmaf(f, o[nb][q4 * 4], g * x.x); o[nb][q4 * 4 + 1] = fmaf(f, o[nb][q4 * 4 + 1], g * x.y);
          o[nb][q4 * 4 + 2] = fmaf(f, o[nb][q4 * 4 + 2], g * x.z); o[nb][q4 * 4 + 3] = fmaf(f, o[nb][q4 * 4 + 3], g * x.w);
        }
      lsum = fmaf(f, lsum, g * ml.y);
      ref = m;
    }
    const float l = lsum + __shfl_xor(lsum, 32);
    constexpr float kLn2 = 0.69314718055994530942f;
    if (whole) {
      if (there) {
        const size_t hb = tile_row + row_at((uint32_t)j);
        const float inv = l == 0.f ? 0.f : 1.f / l;                // (a sum that is no number stays one)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const bf16x2_t y0 = {(__bf16)(o[nb][q4 * 4] * inv), (__bf16)(o[nb][q4 * 4 + 1] * inv)}, y1 = {(__bf16)(o[nb][q4 * 4 + 2] * inv), (__bf16)(o[nb][q4 * 4 + 3] * inv)};
            *reinterpret_cast<uint2*>(a.out + hb * RB + (nb * 32 + q4 * 8 + half * 4) * 2) = make_uint2(__builtin_bit_cast(uint32_t, y0), __builtin_bit_cast(uint32_t, y1));
          }
        if (half == 0 && a.lse != nullptr) a.lse[hb] = l == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l)) * kLn2;
      }
    } else {
      float4* po = reinterpret_cast<float4*>(sh.part_o + ((size_t)wg * 2 + slot) * ROWS * D) + row_block * (NB * 4 * 64) + lane;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) po[(nb * 4 + q4) * 64] = make_float4(o[nb][q4 * 4], o[nb][q4 * 4 + 1], o[nb][q4 * 4 + 2], o[nb][q4 * 4 + 3]);
      if (half == 0) {
        float* pm = sh.part_ml + (((size_t)wg * 2 + slot) * ROWS + j) * 2;
        pm[0] = l == 0.f ? -INFINITY : ref * kLn2; pm[1] = l;      // in units of the logits
      }
    }
    return false;
  }, tree);
}

template <int KIND, int D, int BLOCKS>
static hipError_t wide_one(const PagedAttnArgs& a, const QuantPools& c, const ShareArgs& sh, hipStream_t s) {
  constexpr int lds = 4 * kPwTile * D * 2 + kPwRing * 2 * kPwTile * 4 + sizeof(ShareScratch);
  static_assert(4 * D / 8 * 64 * 16 <= 4 * kPwTile * D * 2 && 4 * 64 * 8 <= kPwRing * 2 * kPwTile * 4, "the halves' sums");
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_wide_kernel<KIND, D, BLOCKS>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((paged_wide_kernel<KIND, D, BLOCKS>), dim3(sh.wgs), dim3(kPwThreads), lds, s, a, c, sh);
  return hipGetLastError();
}
template <int KIND>
static hipError_t wide_some(int D, int rows, const PagedAttnArgs& a, const QuantPools& c, const ShareArgs& sh, hipStream_t s) {
  if (rows == 128) return D == 64 ? wide_one<KIND, 64, 1>(a, c, sh, s) : wide_one<KIND, 128, 1>(a, c, sh, s);
  return D == 64 ? wide_one<KIND, 64, 2>(a, c, sh, s) : wide_one<KIND, 128, 2>(a, c, sh, s);
}

// Tiles of 128 rows where a sequence has no more of them on average (trees, 28/4 heads, int8, 24 sequences over 3000 keys: 84 rows 59 us, by tiles of 256 69, 119 rows 65 and 74; 32 over
// 700: 33 and 37; a single sequence, whose keys are few for every workgroup, 40 and 40 to 42).  More rows: their keys would be staged twice (320 and 384 rows, 24 sequences over 3000 keys, 32/8 heads, bf16: 262 and 280 us
// instead of 222 and 239, 512 tokens over 65536 keys 820 instead of 710).
int wide_rows(const PagedAttnArgs& a) {
  const long tokens = a.q_indptr != nullptr ? ((long)a.T + a.B - 1) / a.B : a.C;
  return tokens * (a.H / a.H_kv) <= 128 ? 128 : kWideRows;
}

// A packed batch whose sequences all fit a tile and have half of the most on average: those with few rows take the wide kernel too.  A launch of their own and its merge cost 5 to 10 us where there
// are none, 10 to 20 where there are some (28/4 heads, int8, drafts of 18 tokens and of one or two: 24 sequences of up to 500 keys 27 us, with a launch for the few 42, of 4000 62 and 83, of 16000 169 and
// 175), and save at most a twentieth of a long call (64 sequences of up to 4000 bf16 keys, 32/8 heads, a third of them with few rows: 242 us instead of 228).
bool wide_alone(const PagedAttnArgs& a) {
  return a.q_indptr == nullptr || ((long)a.C * (a.H / a.H_kv) <= kWideRows && 2l * a.T >= (long)a.B * a.C);
}

// rows: of a tile, 128 or 256; c null: the pools of `a`, rows of bf16
hipError_t launch_paged_wide(int D, int rows, const PagedAttnArgs& a, const QuantPools* c, const ShareArgs& sh, hipStream_t s) {
  if (c == nullptr) return wide_some<kRows16>(D, rows, a, QuantPools{}, sh, s);
  return c->code == TS_INT8 ? wide_some<TS_INT8>(D, rows, a, *c, sh, s) : wide_some<TS_E4M3>(D, rows, a, *c, sh, s);
}

}  // namespace ts
