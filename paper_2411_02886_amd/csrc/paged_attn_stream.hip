// Dense attention of new tokens, few rows per tile: single tokens, short drafts, and all of fp32.
//
// The rows are the columns of 16-column matrix products.  What bounds it (bf16 always, fp32 up to 16 rows) is the memory: every K and V row
// is read once, and what counts is how many bytes are in flight.  The four waves of a workgroup walk wave tiles of their own
// (32 keys bf16, 16 keys fp32; a unit of the share is one of each wave) without any barrier: rows go from memory to the wave's part of
// the LDS directly, 16 bytes per lane; K is requested again as soon as its scores are formed, V as soon as it has been
// multiplied.  Page ids pass through LDS too, two tiles ahead, because the compiler would wait for a register's load with a
// count that knows nothing of the rows in flight.
// bf16 weights keep their 24 bits: each is the sum of three bf16 numbers, and V is multiplied with each of them.  The
// softmax's reference is raised only when a weight exceeds what it allows, so that no maximum is taken in the loop.
// Measured: 8 bf16 tokens (H 32/8, D 128) over 16384 to 65536 keys 241 us, 6.4 TB/s; one over 1000 keys 10.8 us, over 131072 90 (5.9 TB/s); 64 packed sequences
// of 300 keys 15; one fp32 token (8/2, 64) over 4096 keys 11.4.  The fixed part of a call is about 10 us: two launches, the search for the share 1.5 us, page ids and queries 1.2, the first rows
// 1, the waves' meeting 1.5.  fp32 with 64 rows a tile: 512 tokens (32/8, 128) over 4000 keys 351 us, 66 % of what a product by the library
// reaches (154 TFLOP/s); a weight's exponential and its neighbours stand between the products of 16 x 16 x 4.
#include "paged_shares.h"

namespace ts {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

constexpr float kPsUnset = -3.40282347e38f;   // reference logit before the first key: no finite logit lies below it
constexpr float kPsHead = 4.f;                // a raised reference lies this far above the largest logit so far ...
constexpr float kPsRaise = 1.f;               // ... and is raised again when a lane's weights of a tile exceed this together
constexpr float kPsBig = 1048576.f;           // references beyond this: the logits are rounded before it is taken off them (an fma's exact product is off by
                                              // up to 2^-24 of a logit from the rounded one that the reference came from)
constexpr float kPsLog2e = 1.44269504088896340736f;

// place of a row's 16-byte pieces in LDS: the 16 rows of one K piece, and the rows and pieces of a V read, fall on all banks
template <int ES, int D> __device__ __forceinline__ int ps_swz(int key) {
  if (ES == 4) return key & 15;
  return D == 128 ? (((key & 7) << 1) | ((key >> 3) & 1)) : ((((key >> 1) & 3) << 1) | ((key >> 3) & 1));
}

template <int ES, int D, int CB>              // bytes per element, head size, blocks of 16 rows
struct StreamShape {
  static constexpr int TK = ES == 2 ? 32 : 16;     // keys per wave tile
  static constexpr int KT = 4 * TK;                // keys per unit
  static constexpr int RB = D * ES, PPR = RB / 16, RPI = 64 / PPR, NLD = TK / RPI;
  static constexpr int TILE_B = TK * RB;
  static constexpr int LDS = 4 * (2 * TILE_B + 512);   // the waves' tiles and look-ups; the waves' results fit the same place
  static constexpr int PER_CU = CB == 4 ? 1 : 2;
  static_assert(4 * 16 * (D + 4) * 4 <= LDS, "the waves' results");
};

template <int ES, int D, int CB>
__global__ __launch_bounds__(256, (StreamShape<ES, D, CB>::PER_CU)) void paged_stream_kernel(PagedAttnArgs a, ShareArgs sh) {
  using S = StreamShape<ES, D, CB>;
  constexpr int TK = S::TK, KT = S::KT, RB = S::RB, PPR = S::PPR, RPI = S::RPI, NLD = S::NLD, TILE_B = S::TILE_B;
  constexpr int NE = TK / 4;                  // weights per lane and block of rows
  constexpr int DB = D / 16;                  // 16-row blocks of the transposed output
  constexpr int NQ = D / (ES == 2 ? 32 : 16); // 16-byte pieces of a query row per lane
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  __shared__ ShareScratch s_share;
  __shared__ float s_ml[4][16][2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kgrp = lane >> 4;
  const int H = a.H, G = a.H / a.H_kv;
  const int wg = share_of(blockIdx.x, sh.wgs);
  SharePlace from, to;
  SeqShape first;
  find_share<KT>(a, sh, G, wg, &s_share, &from, &to, &first);
  int32_t* desc = sh.desc + (size_t)wg * 8;
  if (!sh.whole && threadIdx.x == 0) { desc[3] = kPieceNone; desc[7] = kPieceNone; }

  uint8_t* kt = smem + wave * (2 * TILE_B + 512);
  uint8_t* vt = kt + TILE_B;
  const uint32_t lds_k = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)kt);
  // two places of 64 page ids (as an LDS pointer: a flat load would wait for every row in flight)
  const volatile __attribute__((address_space(3))) int32_t* look = (const volatile __attribute__((address_space(3))) int32_t*)(vt + TILE_B);
  const int st_row = lane / PPR, st_pos = lane % PPR;
  typedef const __attribute__((address_space(3))) u32x4_t lds_u32x4;
  const float sm = a.sm_scale;
  const int row_shift = 31 - __builtin_clz((uint32_t)(a.H_kv * RB));   // H_kv is a power of two
  const uint32_t g_inv = 65536u / (uint32_t)G + 1u;             // exact for rows below 256
  const uint32_t reach = a.window > 0 ? (uint32_t)a.window : 0x7fffffffu;

  walk_share<KT>(a, sh, G, from, to, first, [&](int kvh, const SeqShape& sq, int r, const TileKeys& keys, int ua, int ub, bool) -> bool {
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
        const size_t o = tile_row + row_at((uint32_t)(i / D));
        if (ES == 2) reinterpret_cast<uint16_t*>(a.out)[o * D + i % D] = 0; else reinterpret_cast<float*>(a.out)[o * D + i % D] = 0.f;
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

    // the wave's tiles: tile i holds keys key0 + i * KT .. + TK; a last one without a key is left out
    const int key0 = (keys.u0 + ua) * KT + wave * TK;
    int nt = ub - ua;
    if (key0 + (nt - 1) * KT > tmax) --nt;
    uint32_t at[NLD];                                              // a tile's rows (this lane's of each load) in the pools
    // (keys past the end or in front of the tile's first window stand for the nearest that some row sees: no other place of the pools is read)
    auto seen = [&](int t) -> int { return min(max(t, keys.first), tmax); };
    auto fetch_look = [&](int i, int place) {
      const int t = seen(key0 + i * KT + (lane & (TK - 1)));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(lds_k + 2 * TILE_B + place * 256), "v"(pages + (t >> a.p_shift)) : "memory", "m0");
    };
    // (fresh(): the compiler forms the address anew in each turn of the loop.  It would keep all of them, dozens of registers, and spill.)
    auto fresh = [](uint32_t x) -> uint32_t { if (CB > 1) asm volatile("" : "+v"(x)); return x; };
    __syncthreads();                                               // the tiles' place is free
    if (nt > 0) fetch_look(0, 0);
    // query rows (zero past the last): 16-byte pieces 4 i + kgrp of row cb * 16 + col
    const uint8_t* q_base = a.q + tile_row * RB;
    uint4 qf[CB][NQ];
    uint32_t low[CB];                                              // first of the `reach` keys that the row sees (modulo 2^32: it may lie before key 0)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int j = cb * 16 + col;
      low[cb] = (uint32_t)(j < nrows ? x0 + token_of((uint32_t)j) : x1) - (reach - 1u);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        qf[cb][i] = make_uint4(0u, 0u, 0u, 0u);
        if (j < nrows) qf[cb][i] = *reinterpret_cast<const uint4*>(q_base + (row_at((uint32_t)j) * RB + (uint32_t)((4 * i + kgrp) * 16)));
      }
    }
    auto rows_of = [&](int i, int place) {
      const int my_row = (int)fresh(st_row);
#pragma unroll
      for (int l = 0; l < NLD; ++l) {
        const int row = l * RPI + my_row, t = seen(key0 + i * KT + row);
        at[l] = ((uint32_t)look[place * 64 + row] << a.p_shift) + (uint32_t)(t & (a.P - 1));
      }
    };
    // 1 KiB per load: the wave's lanes fill LDS from `dst` on.  In assembly, so that the compiler does not make every LDS read wait for
    // it; the waits stand below.  Non-temporal: with few rows per tile nobody else reads them (a batch of 64 over 6000 keys 257 us, else
    // 286; where tiles share rows it makes no difference).
    auto load_rows = [&](const uint8_t* pool, uint32_t dst) {
      const int my_row = (int)fresh(st_row);
#pragma unroll
      for (int l = 0; l < NLD; ++l) {
        const uint64_t off = ((uint64_t)at[l] << row_shift) + (uint32_t)(kvh * RB + ((st_pos ^ ps_swz<ES, D>((l * RPI + my_row) & 15)) * 16));
        asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" :: "s"(dst), "v"(pool + off), "i"(l * 1024) : "memory", "m0", "scc");
      }
    };
    float ref[CB], lsum[CB];                  // of row cb * 16 + col: reference logit (the same in its four lanes), this lane's keys' sum
    bool big = false;                         // some row's reference is large (the same for the whole wave)
    f32x4_t o[CB][DB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      ref[cb] = kPsUnset; lsum[cb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[cb][db] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                            // vmcnt(0): from here on only the row and page loads are outstanding
    asm volatile("" ::: "memory");
    if (nt > 0) {
      rows_of(0, 0);
      fetch_look(1, 1);
      load_rows(a.k_pool, lds_k);
      load_rows(a.v_pool, lds_k + TILE_B);
    }
    for (int i = 0; i < nt; ++i) {
      const bool more = i + 1 < nt;
      const int k0 = key0 + i * KT;
      asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NLD) : "memory");            // this tile's K rows and the next one's page ids (its V rows follow them)
      // ---- scores, element e: key 16 * (e / 4) + 4 * kgrp + e % 4.  Products are added up in four chains, which loses less than one (two where the
      // registers hold no more)
      float s[CB][NE];
      constexpr int NB = TK / 16, NC = CB == 1 ? 4 : 2;              // blocks of 16 keys, chains
      f32x4_t part[CB][NC][NB];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int kb = 0; kb < NB; ++kb) part[cb][c][kb] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
      const uint32_t k_at = fresh(lds_k + (uint32_t)(col * RB)), k_piece = fresh((uint32_t)(kgrp ^ ps_swz<ES, D>(col)));
#pragma unroll
      for (int ks = 0; ks < NQ; ++ks)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
          const uint4 kf = __builtin_bit_cast(uint4, *(lds_u32x4*)(k_at + (uint32_t)(kb * 16 * RB) + ((k_piece ^ (uint32_t)(ks * 4)) * 16)));
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            if constexpr (ES == 2) {
              f32x4_t& acc = part[cb][ks % NC][kb];
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qf[cb][ks]), acc, 0, 0, 0);
            } else {
              const uint32_t kw[4] = {kf.x, kf.y, kf.z, kf.w}, qw[4] = {qf[cb][ks].x, qf[cb][ks].y, qf[cb][ks].z, qf[cb][ks].w};
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                f32x4_t& acc = part[cb][c % NC][kb];
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[c]), __uint_as_float(qw[c]), acc, 0, 0, 0);
              }
            }
          }
        }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          s[cb][e] = part[cb][0][e >> 2][e & 3] + part[cb][1][e >> 2][e & 3];
          if constexpr (NC == 4) s[cb][e] += part[cb][2][e >> 2][e & 3] + part[cb][3][e >> 2][e & 3];
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                     // the K tile has been read
      if (more) { rows_of(i + 1, (i + 1) & 1); fetch_look(i + 2, i & 1); load_rows(a.k_pool, lds_k); }
      // ---- weights against the reference: exp(logit - reference)
      const bool masked = k0 + TK - 1 > x0 || (a.window > 0 && k0 <= x1 - a.window);   // some row does not see some key
      float p[CB][NE];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        float sum = 0.f;
        for (int tries = 0; tries < 2; ++tries) {
          sum = 0.f;
          if (masked || big) {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              const float y = (uint32_t)(k0 + 16 * (e >> 2) + 4 * kgrp + (e & 3)) - low[cb] < reach ? s[cb][e] * sm : -INFINITY;
              p[cb][e] = __builtin_amdgcn_exp2f((y - ref[cb]) * kPsLog2e);
              sum += p[cb][e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              p[cb][e] = __builtin_amdgcn_exp2f(fmaf(s[cb][e], sm, -ref[cb]) * kPsLog2e);
              sum += p[cb][e];
            }
          }
          if (__builtin_amdgcn_ballot_w64(!(sum <= kPsRaise)) == 0) break;
          float m = ref[cb];                                                 // first keys, or a logit far above the reference
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            m = fmaxf(m, (uint32_t)(k0 + 16 * (e >> 2) + 4 * kgrp + (e & 3)) - low[cb] < reach ? s[cb][e] * sm + kPsHead : -INFINITY);
          }
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m, __shfl_xor(m, 32));
          big = big || __builtin_amdgcn_ballot_w64(fabsf(m) > kPsBig && m != kPsUnset) != 0;
          const float f = __builtin_amdgcn_exp2f((ref[cb] - m) * kPsLog2e);  // 0 while the reference is unset, 1 where it stays
          lsum[cb] *= f;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[cb][db][e] *= f;
          ref[cb] = m;
        }
        lsum[cb] += sum;
      }
      // ---- O^T += V^T P^T
      if constexpr (ES == 2) {
        // each weight as three bf16 numbers whose sum is the weight; k-slot 8 * kgrp + e of the product is p[e]'s key.  The parts are cut
        // off, not rounded, and the lower two are kept above 2^-30 of the weight: all three have its sign and none is zero beside
        // it, so that an infinite V row comes out infinite (inf - inf and 0 * inf would make it NaN)
        uint32_t w[CB][3][4];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int e = 0; e < NE; e += 2) {
            const float q0 = p[cb][e] * 9.3132257e-10f, q1 = p[cb][e + 1] * 9.3132257e-10f;
            float y0 = p[cb][e], y1 = p[cb][e + 1];
#pragma unroll
            for (int c = 0; c < 3; ++c) {
              w[cb][c][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(y0), 0x07060302u);   // the high halves
              if (c < 2) {
                y0 = fmaxf(y0 - bf16_lo(w[cb][c][e >> 1]), q0);              // the differences are exact
                y1 = fmaxf(y1 - bf16_hi(w[cb][c][e >> 1]), q1);
              }
            }
          }
        if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NLD + 1) : "memory");   // this tile's V rows (page ids and the next K rows follow them)
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // V^T read: key, piece of the pair, half
        const int vt_key = 4 * kgrp + (col >> 2);
        const uint32_t v_at = fresh(lds_k + (uint32_t)(TILE_B + vt_key * RB + (col & 1) * 8)), v_piece = fresh((uint32_t)(((col & 3) >> 1) ^ ps_swz<ES, D>(vt_key)));
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          uint2 v[2];
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const uint32_t vp = v_at + (uint32_t)(kb * 16 * RB) + ((v_piece ^ (uint32_t)(db * 2)) * 16);
            v[kb] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)vp));
          }
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(v[0].x, v[0].y, v[1].x, v[1].y));
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int c = 0; c < 3; ++c)
              o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8_t, make_uint4(w[cb][c][0], w[cb][c][1], w[cb][c][2], w[cb][c][3])),
                                                                  o[cb][db], 0, 0, 0);
        }
      } else {
        if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NLD + 1) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint32_t v_at = fresh(lds_k + (uint32_t)(TILE_B + 4 * kgrp * RB)), v_piece = fresh((uint32_t)(col ^ (4 * kgrp)));
        // product e takes keys 4 * kgrp + e; a read of 16 bytes serves four blocks of the output, row i of block 4 q + c is d = 64 q + 4 i + c
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            const uint32_t vp = v_at + (uint32_t)(e * RB) + (((uint32_t)(16 * q) + (v_piece ^ (uint32_t)e)) * 16);   // key 4 * kgrp + e: its piece is flipped by itself
            const uint4 vf = __builtin_bit_cast(uint4, *(lds_u32x4*)vp);
            const float vw[4] = {__uint_as_float(vf.x), __uint_as_float(vf.y), __uint_as_float(vf.z), __uint_as_float(vf.w)};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int cb = 0; cb < CB; ++cb) o[cb][4 * q + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[c], p[cb][e], o[cb][4 * q + c], 0, 0, 0);
          }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                     // the V tile has been read
      if (more) load_rows(a.v_pool, lds_k + TILE_B);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                         // a look-up past the end may be outstanding

    // ---- the four waves meet, sixteen rows at a time
    float* so = reinterpret_cast<float*>(smem);                              // [wave][row][D + 4]
    float* part_o = sh.part_o + ((size_t)wg * 2 + slot) * (16 * CB) * D;
    float* part_ml = sh.part_ml + ((size_t)wg * 2 + slot) * (16 * CB) * 2;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      if (cb * 16 >= nrows) break;
      float l = lsum[cb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      __syncthreads();                                                       // every wave is done with its tiles, or with the last rows
      float* mine = so + (wave * 16 + col) * (D + 4);
      if constexpr (ES == 2) {
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<float4*>(mine + db * 16 + kgrp * 4) = make_float4(o[cb][db][0], o[cb][db][1], o[cb][db][2], o[cb][db][3]);
      } else {
#pragma unroll
        for (int q = 0; q < D / 64; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float4*>(mine + 64 * q + 16 * kgrp + 4 * e) = make_float4(o[cb][4 * q][e], o[cb][4 * q + 1][e], o[cb][4 * q + 2][e], o[cb][4 * q + 3][e]);
      }
      if (kgrp == 0) { s_ml[wave][col][0] = ref[cb]; s_ml[wave][col][1] = l; }
      __syncthreads();
#pragma unroll
      for (int it = 0; it < 16 * D / 4 / 256; ++it) {
        const int i = it * 256 + threadIdx.x, jj = i / (D / 4), d = i % (D / 4) * 4, j = cb * 16 + jj;
        if (j >= nrows) continue;
        const float m = fmaxf(fmaxf(s_ml[0][jj][0], s_ml[1][jj][0]), fmaxf(s_ml[2][jj][0], s_ml[3][jj][0]));
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float L = 0.f;
#pragma unroll
        for (int w4 = 0; w4 < 4; ++w4) {
          const float f = __builtin_amdgcn_exp2f((s_ml[w4][jj][0] - m) * kPsLog2e);   // a wave without keys of the row: its sums are 0
          const float4 z = *reinterpret_cast<const float4*>(so + (w4 * 16 + jj) * (D + 4) + d);
          y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
          L = fmaf(f, s_ml[w4][jj][1], L);
        }
        if (whole) {
          const size_t hb = tile_row + row_at((uint32_t)j);
          const float inv = L == 0.f ? 0.f : 1.f / L;       // (a sum that is no number stays one)
          y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
          if (ES == 2)
            *reinterpret_cast<uint2*>(a.out + (hb * D + d) * 2) = make_uint2(f32_to_bf16_bits(y.x) | (f32_to_bf16_bits(y.y) << 16), f32_to_bf16_bits(y.z) | (f32_to_bf16_bits(y.w) << 16));
          else *reinterpret_cast<float4*>(a.out + (hb * D + d) * 4) = y;
          if (d == 0 && a.lse != nullptr) a.lse[hb] = L == 0.f ? -INFINITY : m + logf(L);
        } else {
          *reinterpret_cast<float4*>(part_o + j * D + d) = y;
          if (d == 0) { part_ml[2 * j] = L == 0.f ? -INFINITY : m; part_ml[2 * j + 1] = L; }
        }
      }
    }
    return false;
  });
}

template <int ES, int D, int CB>
static hipError_t stream_one(const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s) {
  using S = StreamShape<ES, D, CB>;
  if (S::LDS > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_stream_kernel<ES, D, CB>), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((paged_stream_kernel<ES, D, CB>), dim3(sh.wgs), dim3(256), S::LDS, s, a, sh);
  return hipGetLastError();
}

hipError_t launch_paged_stream(int dtype, int D, int blocks, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s) {
  if (dtype == TS_BF16) {
    if (D == 64) return blocks == 1 ? stream_one<2, 64, 1>(a, sh, s) : stream_one<2, 64, 2>(a, sh, s);
    return blocks == 1 ? stream_one<2, 128, 1>(a, sh, s) : stream_one<2, 128, 2>(a, sh, s);
  }
  if (D == 64) return blocks == 1 ? stream_one<4, 64, 1>(a, sh, s) : blocks == 2 ? stream_one<4, 64, 2>(a, sh, s) : stream_one<4, 64, 4>(a, sh, s);
  return blocks == 1 ? stream_one<4, 128, 1>(a, sh, s) : blocks == 2 ? stream_one<4, 128, 2>(a, sh, s) : stream_one<4, 128, 4>(a, sh, s);
}

}  // namespace ts
