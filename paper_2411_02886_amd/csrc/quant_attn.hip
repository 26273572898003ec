// Dense attention of new tokens over a cache in 8 bits: single tokens, drafts and their trees, chunks, prompts.
//
// The rows (a tile: some tokens of a sequence times the query heads of one KV head) are the columns of 16-column matrix products.  Codes are small
// numbers that bf16 holds exactly, so scores are bf16 products of queries and codes, summed in float, times the key's scale; a weight is multiplied
// with the value's scale and cut into three bf16 numbers that add up to it, each of which multiplies the codes of V: nothing is rounded that float
// arithmetic would not round.  fp32 queries are three bf16 numbers as well.
// This is the kernel of few rows, bound by the bytes it reads: a workgroup's four waves have four KV heads side by side, or share the keys of one.  Many rows: paged_wide.hip.
// The waves walk wave tiles of 32 keys of their own without barriers, rows in registers: K as the matrix product wants it (a lane has a key's 16 bytes), V as rows too (a
// lane has the same bytes of its eight keys), whose bytes are transposed in the lane by byte permutations before they are widened.  A tile's rows, scales and page ids
// are requested a tile ahead.
// Eight sequences of 16384 to 65536 keys, 8 KV heads of 128, int8, a token each: 148 us, 5.4 TB/s with the joining of the pieces; the same read pattern without arithmetic
// reaches 5.8 to 6.1 TB/s, one head per workgroup 5.35.
#include "paged_shares.h"
#include "ts_codes.h"
#include <algorithm>

namespace ts {

hipError_t launch_paged_merge(int dtype, int D, const PagedAttnArgs& a, const ShareArgs& sh, int rows, PieceOrder order, long tiles, hipStream_t s);

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

constexpr int kQaTile = 32;                   // keys of a wave tile
constexpr float kQaUnset = -3.40282347e38f;   // reference exponent before the first key: no finite one lies below it
constexpr float kQaHead = 6.f;                // a raised reference lies this far above the largest exponent so far ...
constexpr float kQaRaise = 2.f;               // ... and is raised again when a lane's weights of a tile exceed this together

// byte c of each of four words, as word c
__device__ __forceinline__ void transpose4(uint32_t (&v)[4]) {
  const uint32_t lo01 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);
  const uint32_t lo23 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
  v[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
  v[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
  v[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
  v[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
}
__device__ __forceinline__ bf16x8_t frag_of(uint2 a, uint2 b) { return __builtin_bit_cast(bf16x8_t, make_uint4(a.x, a.y, b.x, b.y)); }
__device__ __forceinline__ uint32_t high_halves(float y1, float y0) { return __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(y0), 0x07060302u); }
__device__ __forceinline__ float low_part(float y) { return y - __uint_as_float(__float_as_uint(y) & 0xffff0000u); }   // (exact)

template <int CODE, int ES, int D, int CB>    // ES: bytes of a query's and an output's element; CB: blocks of 16 rows
__global__ __launch_bounds__(256, CB == 1 ? 2 : 1) void quant_attn_kernel(PagedAttnArgs a, QuantPools c, ShareArgs sh) {
  constexpr int TK = kQaTile;
  constexpr int QP = ES == 2 ? 1 : 3;         // bf16 numbers that a query element is the sum of
  constexpr int NP = D / 64;                  // 16-byte pieces of a key per lane
  constexpr int VB = D / 16;                  // bytes of a value per lane, and 16-row blocks of the transposed output
  __shared__ ShareScratch s_share;
  __shared__ __attribute__((aligned(16))) float s_o[4][16][D + 4];
  __shared__ float s_ml[4][16][2];
  __shared__ __attribute__((aligned(16))) uint32_t s_slot[4][TK];
  __shared__ __attribute__((aligned(16))) float s_scale[4][2 * TK];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kgrp = lane >> 4;
  // The waves have one, two or four KV heads side by side, and share the keys of a head if it is fewer than four.  To the shares and the merge the heads of a
  // workgroup are one with all of their query heads (`line`).
  const int heads_shift = sh.heads_shift, heads = 1 << heads_shift, parts = 4 >> heads_shift;
  const int my_head = wave & (heads - 1), my_part = wave >> heads_shift;
  const int H = a.H, G = a.H / a.H_kv, GW = G << heads_shift;
  PagedAttnArgs line = a;
  line.H_kv = a.H_kv >> heads_shift;
  const bool tree = a.mask != nullptr;
  const int wg = share_of(blockIdx.x, sh.wgs);
  SharePlace from, to;
  SeqShape first;
  find_share<TK>(line, sh, G, wg, &s_share, &from, &to, &first, tree);
  int32_t* desc = sh.desc + (size_t)wg * 8;
  if (!sh.whole && threadIdx.x == 0) { desc[3] = kPieceNone; desc[7] = kPieceNone; }
  const uint32_t g_inv = 65536u / (uint32_t)G + 1u;             // exact for rows below 256
  const float c2 = a.sm_scale * 1.44269504088896340736f;        // logits are exponents of two here
  const int row_shift = 31 - __builtin_clz((uint32_t)(a.H_kv * D));   // H_kv is a power of two

  walk_share<TK>(line, sh, G, from, to, first, [&](int group, const SeqShape& sq, int r, const TileKeys& keys, int ua, int ub, bool) -> bool {
    const int c0 = r * sh.tpt, ntok = min(sh.tpt, sq.n - c0), nrows = ntok * G;
    const int row0 = sq.row0 + c0, base = sq.N - sq.n;
    const bool whole = ua == 0 && ub == keys.units;
    const int tmax = keys.end - 1;
    auto token_of = [&](uint32_t j) -> int { return (int)min(__umul24(j, g_inv) >> 16, (uint32_t)(ntok - 1)); };   // j / G; rows past the last stand for it
    const int kvh = (group << heads_shift) + my_head;
    // row j of a wave's head in q, out and lse, and in a piece: its token's rows, the workgroup's heads side by side
    const size_t tile_row = (size_t)row0 * H + group * GW;
    auto row_at = [&](uint32_t j, int h) -> uint32_t { return __umul24(__umul24(j, g_inv) >> 16, (uint32_t)(H - G)) + j + (uint32_t)(h * G); };
    auto piece_at = [&](uint32_t j, int h) -> uint32_t { return __umul24(__umul24(j, g_inv) >> 16, (uint32_t)(GW - G)) + j + (uint32_t)(h * G); };
    if (keys.end <= keys.first) {                                  // no row sees a token (one unit: the tile is not cut)
      for (int i = threadIdx.x; i < (nrows << heads_shift) * D; i += 256) {
        const int j = i / D;
        const size_t o = tile_row + row_at((uint32_t)(j >> heads_shift), j & (heads - 1));
        if (ES == 2) reinterpret_cast<uint16_t*>(a.out)[o * D + i % D] = 0; else reinterpret_cast<float*>(a.out)[o * D + i % D] = 0.f;
        if (i % D == 0 && a.lse != nullptr) a.lse[o] = -INFINITY;
      }
      return false;
    }
    const int slot = ua > 0 ? 0 : 1;
    if (!whole && threadIdx.x == 0) {
      int32_t* d = desc + slot * 4;
      d[0] = row0; d[1] = group; d[2] = ntok; d[3] = ub == keys.units ? kPieceEnds : kPieceGoesOn;
    }
    const int32_t* pages = a.page_indices + sq.page0;
    // the wave's tiles: tile i holds keys key0 + i * KT .. + TK
    const int KT = TK * parts, key0 = (keys.u0 + ua) * TK + my_part * TK, nt = (ub - ua - my_part + parts - 1) >> (2 - heads_shift);
    // (keys past the end or in front of the tile's first window stand for the nearest that some row sees: no other place of the cache is read)
    const int my_key = lane & (TK - 1);
    auto key_of = [&](int i) -> int { return min(max(key0 + i * KT + my_key, keys.first), tmax); };
    auto page_of = [&](int i) -> int { return pages[key_of(i) >> a.p_shift]; };

    // queries: pieces of 16 elements, two products each; element 64 i + 16 kgrp + 8 h + .. of row cb * 16 + col (zero past the last)
    bf16x8_t qf[CB][QP][2 * NP];
    int low[CB], place[CB];                                        // first key of the row's window; its place
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const uint32_t j = (uint32_t)(cb * 16 + col);
      const bool there = (int)j < nrows;
      place[cb] = base + c0 + token_of(j);
      low[cb] = tree ? tree_low(a, row0 + token_of(j), sq.n, base) : a.window > 0 ? place[cb] - a.window + 1 : 0;
      const uint8_t* q = a.q + (tile_row + (there ? row_at(j, my_head) : 0u)) * (size_t)(D * ES);
#pragma unroll
      for (int x = 0; x < 2 * NP; ++x) {
        const int d = 64 * (x >> 1) + 16 * kgrp + 8 * (x & 1);
        if constexpr (ES == 2) {
          uint4 w = *reinterpret_cast<const uint4*>(q + d * 2);
          if (!there) w = make_uint4(0u, 0u, 0u, 0u);
          qf[cb][0][x] = __builtin_bit_cast(bf16x8_t, w);
        } else {
          float y[8];
          const float4 y0 = *reinterpret_cast<const float4*>(q + d * 4), y1 = *reinterpret_cast<const float4*>(q + d * 4 + 16);
          y[0] = y0.x; y[1] = y0.y; y[2] = y0.z; y[3] = y0.w; y[4] = y1.x; y[5] = y1.y; y[6] = y1.z; y[7] = y1.w;
#pragma unroll
          for (int part = 0; part < QP; ++part) {                  // cut off, not rounded: the third part holds the last 8 bits
            uint32_t w[4];
#pragma unroll
            for (int u = 0; u < 8; u += 2) {
              w[u >> 1] = there ? high_halves(y[u + 1], y[u]) : 0u;
              y[u] = low_part(y[u]); y[u + 1] = low_part(y[u + 1]);
            }
            qf[cb][part][x] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
          }
        }
      }
    }

    u32x4_t kr[2][NP];                                             // the next tile's keys 16 kb + col
    uint32_t vr[8][VB / 4];                                        // its values of keys 16 (j / 4) + 4 kgrp + j % 4, bytes VB col ..
    float scale;                                                   // of key my_key: K's in lanes 0 .. 31, V's in the others
    const uint8_t* const k_head = c.k_codes + kvh * D + kgrp * 16;
    const uint8_t* const v_head = c.v_codes + kvh * D + col * VB;
    const float* const scales = lane < TK ? c.k_scale : c.v_scale;
    auto request = [&](int i, int page) {
      const int in_page = key_of(i) & (a.P - 1);
      scale = scales[((((int64_t)page * a.H_kv + kvh) << a.p_shift) + in_page)];
      __builtin_amdgcn_wave_barrier();
      if (lane < TK) s_slot[wave][lane] = ((uint32_t)page << a.p_shift) + (uint32_t)in_page;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint8_t* row = k_head + ((uint64_t)s_slot[wave][kb * 16 + col] << row_shift);
#pragma unroll
        for (int x = 0; x < NP; ++x) kr[kb][x] = *reinterpret_cast<const u32x4_t*>(row + x * 64);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint8_t* row = v_head + ((uint64_t)s_slot[wave][(j >> 2) * 16 + 4 * kgrp + (j & 3)] << row_shift);
        if constexpr (VB == 8) {
          const uint2 w = *reinterpret_cast<const uint2*>(row);
          vr[j][0] = w.x; vr[j][1] = w.y;
        } else vr[j][0] = *reinterpret_cast<const uint32_t*>(row);
      }
    };

    float ref[CB], lsum[CB];                  // of row cb * 16 + col: reference exponent (the same in its four lanes), this lane's keys' sum
    f32x4_t o[CB][VB];                        // O^T: block x, element e is d = VB (4 kgrp + e) + x
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      ref[cb] = kQaUnset; lsum[cb] = 0.f;
#pragma unroll
      for (int x = 0; x < VB; ++x) o[cb][x] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    int page = 0;
    if (nt > 0) {
      const int now = page_of(0);
      page = page_of(1);
      request(0, now);
    }
    for (int i = 0; i < nt; ++i) {
      const int k0 = key0 + i * KT;
      u32x4_t k_now[2][NP];
      uint32_t v_now[8][VB / 4];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < NP; ++x) k_now[kb][x] = kr[kb][x];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int x = 0; x < VB / 4; ++x) v_now[j][x] = vr[j][x];
      __builtin_amdgcn_wave_barrier();
      s_scale[wave][lane] = scale;
      __builtin_amdgcn_wave_barrier();
      if (i + 1 < nt) {
        const int now = page;
        page = page_of(i + 2);
        request(i + 1, now);
      }
      // ---- scores: element 4 kb + e is key 16 kb + 4 kgrp + e
      f32x4_t s[CB][2];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) s[cb][0] = s[cb][1] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 2 * NP; ++x) {
          const u32x4_t w = k_now[kb][x >> 1];
          const bf16x8_t kf = frag_of(widen<CODE>(w[2 * (x & 1)]), widen<CODE>(w[2 * (x & 1) + 1]));
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int part = 0; part < QP; ++part) s[cb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[cb][part][x], s[cb][kb], 0, 0, 0);
        }
      float ks[8], vs[8];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const float4 x = *reinterpret_cast<const float4*>(&s_scale[wave][kb * 16 + 4 * kgrp]), y = *reinterpret_cast<const float4*>(&s_scale[wave][TK + kb * 16 + 4 * kgrp]);
        ks[4 * kb] = x.x * c2; ks[4 * kb + 1] = x.y * c2; ks[4 * kb + 2] = x.z * c2; ks[4 * kb + 3] = x.w * c2;
        vs[4 * kb] = y.x; vs[4 * kb + 1] = y.y; vs[4 * kb + 2] = y.z; vs[4 * kb + 3] = y.w;
      }
      // ---- weights against the reference
      const bool masked = k0 + TK - 1 > (tree ? base - 1 : base + c0) || (a.window > 0 && k0 <= (tree ? base + sq.n - 1 : base + c0 + ntok - 1) - a.window);
      uint32_t w[CB][3][4];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        float y[8], p[8], sum = 0.f, seen_vs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { y[e] = s[cb][e >> 2][e & 3] * ks[e]; seen_vs[e] = vs[e]; }
        if (masked) {                                                        // (a scale may be no number: it concerns the rows that see the key, those too whose weight for it is 0)
          uint32_t bits;                                                     // the keys that the row sees
          if (tree) bits = tree_bits(a, row0 + token_of((uint32_t)(cb * 16 + col)), sq.n, base, low[cb], k0);
          else {
            const int many = min(max(place[cb] + 1 - k0, 0), 32), cut = min(max(low[cb] - k0, 0), 32);
            bits = (uint32_t)(((1ull << many) - 1ull) & ~((1ull << cut) - 1ull));
          }
          bits >>= 4 * kgrp;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((bits >> (16 * (e >> 2) + (e & 3)) & 1u) == 0u) { y[e] = -INFINITY; seen_vs[e] = 0.f; }
        }
        for (int tries = 0; tries < 2; ++tries) {
          sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) { p[e] = __builtin_amdgcn_exp2f(y[e] - ref[cb]); sum += p[e]; }
          if (__builtin_amdgcn_ballot_w64(!(sum <= kQaRaise)) == 0) break;
          float m = ref[cb];                                                 // first keys, or a logit far above the reference
#pragma unroll
          for (int e = 0; e < 8; ++e) m = fmaxf(m, y[e] + kQaHead);
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m, __shfl_xor(m, 32));
          const float f = __builtin_amdgcn_exp2f(ref[cb] - m);               // 0 while the reference is unset, 1 where it stays
          lsum[cb] *= f;
#pragma unroll
          for (int x = 0; x < VB; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[cb][x][e] *= f;
          ref[cb] = m;
        }
        lsum[cb] += sum;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float y0 = p[e] * seen_vs[e], y1 = p[e + 1] * seen_vs[e + 1];
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            w[cb][part][e >> 1] = high_halves(y1, y0);
            y0 = low_part(y0); y1 = low_part(y1);
          }
        }
      }
      // ---- O^T += V^T P^T
#pragma unroll
      for (int x4 = 0; x4 < VB / 4; ++x4) {
        uint32_t t0[4] = {v_now[0][x4], v_now[1][x4], v_now[2][x4], v_now[3][x4]}, t1[4] = {v_now[4][x4], v_now[5][x4], v_now[6][x4], v_now[7][x4]};
        transpose4(t0);
        transpose4(t1);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const bf16x8_t vf = frag_of(widen<CODE>(t0[x]), widen<CODE>(t1[x]));
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int part = 0; part < 3; ++part)
              o[cb][4 * x4 + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  vf, __builtin_bit_cast(bf16x8_t, make_uint4(w[cb][part][0], w[cb][part][1], w[cb][part][2], w[cb][part][3])), o[cb][4 * x4 + x], 0, 0, 0);
        }
      }
    }

    // ---- the waves of a head meet, sixteen rows of each head at a time
    const int rows = 16 * CB << heads_shift;
    float* part_o = sh.part_o + ((size_t)wg * 2 + slot) * rows * D;
    float* part_ml = sh.part_ml + ((size_t)wg * 2 + slot) * rows * 2;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      if (cb * 16 >= nrows) break;
      float l = lsum[cb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      __syncthreads();                                                       // every wave is done with the last rows
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int x = 0; x < VB; x += 4)
          *reinterpret_cast<float4*>(&s_o[wave][col][VB * (4 * kgrp + e) + x]) = make_float4(o[cb][x][e], o[cb][x + 1][e], o[cb][x + 2][e], o[cb][x + 3][e]);
      if (kgrp == 0) { s_ml[wave][col][0] = ref[cb]; s_ml[wave][col][1] = l; }
      __syncthreads();
      for (int i = threadIdx.x; i < (16 * D / 4) << heads_shift; i += 256) {
        const int jw = i / (D / 4), h = jw >> 4, jj = jw & 15, d = i % (D / 4) * 4, j = cb * 16 + jj;
        if (j >= nrows) continue;
        float m = kQaUnset;
#pragma unroll
        for (int w4 = 0; w4 < 4; ++w4) m = fmaxf(m, (w4 & (heads - 1)) == h ? s_ml[w4][jj][0] : kQaUnset);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float L = 0.f;
#pragma unroll
        for (int w4 = 0; w4 < 4; ++w4) {
          const float4 z = *reinterpret_cast<const float4*>(&s_o[w4][jj][d]);
          const float l = s_ml[w4][jj][1], f = __builtin_amdgcn_exp2f(s_ml[w4][jj][0] - m);       // a wave without keys of the row: its sums are 0
          if ((w4 & (heads - 1)) != h) continue;
          y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
          L = fmaf(f, l, L);
        }
        constexpr float kLn2 = 0.69314718055994530942f;
        if (whole) {
          const size_t hb = tile_row + row_at((uint32_t)j, h);
          const float inv = L == 0.f ? 0.f : 1.f / L;                        // (a sum that is no number stays one)
          y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
          if (ES == 2) {
            const bf16x2_t z0 = {(__bf16)y.x, (__bf16)y.y}, z1 = {(__bf16)y.z, (__bf16)y.w};
            *reinterpret_cast<uint2*>(a.out + (hb * D + d) * 2) = make_uint2(__builtin_bit_cast(uint32_t, z0), __builtin_bit_cast(uint32_t, z1));
          } else *reinterpret_cast<float4*>(a.out + (hb * D + d) * 4) = y;
          if (d == 0 && a.lse != nullptr) a.lse[hb] = L == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(L)) * kLn2;
        } else {
          const uint32_t pr = piece_at((uint32_t)j, h);
          *reinterpret_cast<float4*>(part_o + (size_t)pr * D + d) = y;
          if (d == 0) { part_ml[2 * pr] = L == 0.f ? -INFINITY : m * kLn2; part_ml[2 * pr + 1] = L; }   // in units of the logits
        }
      }
    }
    return false;
  }, tree);
}

template <int CODE, int ES, int D, int CB>
static hipError_t quant_one(const PagedAttnArgs& a, const QuantPools& c, const ShareArgs& sh, hipStream_t s) {
  hipLaunchKernelGGL((quant_attn_kernel<CODE, ES, D, CB>), dim3(sh.wgs), dim3(256), 0, s, a, c, sh);
  return hipGetLastError();
}
template <int CODE, int D>
static hipError_t quant_some(int dtype, int blocks, const PagedAttnArgs& a, const QuantPools& c, const ShareArgs& sh, hipStream_t s) {
  if (dtype == TS_F32) return blocks == 1 ? quant_one<CODE, 4, D, 1>(a, c, sh, s) : quant_one<CODE, 4, D, 2>(a, c, sh, s);
  return blocks == 1 ? quant_one<CODE, 2, D, 1>(a, c, sh, s) : quant_one<CODE, 2, D, 2>(a, c, sh, s);
}

// KV heads that a workgroup may have side by side
static int most_beside(int H_kv) { return H_kv < 4 ? H_kv : 4; }
// Heads side by side read four times as many bytes of a token at once, one head has its keys divided among four waves.  A call with much to read for
// every workgroup is bound by the bytes (int8, 8 KV heads of 128, one token each; side by side against one: 64 sequences of 6000 keys 147 against 165 us, 8 of up
// to 65536 147 against 165, 32 of 8000 with D 64 45 against 51), others by the way through the keys (one of 8000 22.9 against 17.4, 8 of 4000 26.5 against
// 20.8, 64 of 500 24.7 against 17.6, drafts of four tokens over 16 of 8000 79 against 58).  The host knows the bound, not the lengths: a bound far above them chooses heads side by side where
// one would be quicker, at these costs.
static int heads_beside(const PagedAttnArgs& a, int D) {
  const long keys = std::min((long)a.max_seq_len, a.window > 0 ? (long)a.window + a.C : LONG_MAX);
  return (double)a.B * keys * a.H_kv / kShareWgs >= 50. * D ? most_beside(a.H_kv) : 1;
}

// bytes that tiles of `rows` rows leave pieces in
static size_t quant_piece_bytes(int wgs, int rows, int D) {
  return align_up((size_t)wgs * 32, 256) + align_up((size_t)wgs * 2 * rows * 2 * 4, 256) + (size_t)wgs * 2 * rows * D * 4;
}

// A sequence's rows n * G decide.  Up to 32 are a tile of the stream kernel, up to 64 two (28/4 heads: over 2000 keys 18 us, by the wide
// kernel 24, 8 times 8000 keys 97 and 89); more are tiles of the wide kernel in bf16, which reads and widens a key once for 256, of 32 rows in fp32, whose products
// are three times as many and need the registers.
struct QuantPlan { int few_rows, many_rows; };   // rows of the tiles of sequences with few rows, and of those with more (0: there are none)
static QuantPlan quant_plan(int dtype, int G, int chunk) {
  const long rows = (long)chunk * G;
  if (rows <= 16) return QuantPlan{16, 0};
  if (rows <= 64) return QuantPlan{32, 0};
  return dtype == TS_F32 ? QuantPlan{16, 32} : QuantPlan{32, kWideRows};
}

size_t quant_attn_workspace(int dtype, int D, int G, int H_kv, int chunk) {
  const QuantPlan pl = quant_plan(dtype, G, chunk);
  size_t bytes = quant_piece_bytes(kShareWgs, pl.few_rows * most_beside(H_kv), D);
  if (pl.many_rows == kWideRows) bytes += quant_piece_bytes(kShareWgs, kWideRows, D);
  else if (pl.many_rows) bytes += quant_piece_bytes(kShareWgs, pl.many_rows * most_beside(H_kv), D);
  return align_up(bytes, 256);
}

hipError_t launch_quant_attn(int dtype, int D, const PagedAttnArgs& a, const QuantPools& c, void* ws, hipStream_t s) {
  const int G = a.H / a.H_kv, heads = heads_beside(a, D);
  const QuantPlan pl = quant_plan(dtype, G, a.C);
  uint8_t* at = (uint8_t*)ws;
  auto run = [&](int rows, int more_rows, int most_rows) -> hipError_t {
    const bool wide = rows == kWideRows;
    PagedAttnArgs line = a;                                // what the merge sees: the heads that a workgroup has side by side are one
    if (!wide) line.H_kv = a.H_kv / heads;
    if (wide) rows = wide_rows(a);
    const int held = wide ? rows : rows * heads, wgs = kShareWgs;
    ShareArgs sh{};
    sh.heads_shift = wide ? 0 : ilog2(heads);
    sh.together = wide ? 0 : 4 / heads - 1;                // a unit for each wave (else the cuts fall so that one workgroup has two short pieces, one after the other: 4095 keys 13.1 us instead of 10.2)
    sh.tpt = rows / G;
    sh.more_rows = more_rows;
    sh.most_rows = most_rows;
    const bool beside = most_rows < INT_MAX;
    // tiles of every sequence (0: not as many), and bounds on all tiles and on the keys of one
    sh.each = beside ? 1 : a.q_indptr != nullptr ? 0 : (a.C + sh.tpt - 1) / sh.tpt;
    const long tiles = (sh.each > 0 ? (long)a.B * sh.each : (long)a.T / sh.tpt + a.B) * line.H_kv;
    const long keys = std::min((long)a.max_seq_len, a.window > 0 ? (long)a.window + a.C : LONG_MAX);
    // A workgroup per tile and no merge where that is no longer a way than the pieces' and their joining (one bf16 token, D 128, 8 KV heads: 400 keys 9.2 us, cut
    // 13.8; 1000 keys 14.0 and 13.9; 2000 keys 23.3 and 14.0; fp32 over 500 keys 7.0 and 12.7)
    sh.whole = wide ? tiles <= wgs * (a.q_indptr != nullptr ? 2 : 1) && keys <= 1024
                    : tiles < (1l << 23) && (keys <= 512 || (tiles >= kShareWgs && keys <= 2048));
    sh.min_keys = wide ? 128 : kQaTile * 4 / heads;
    sh.tile_cost = wide ? 256 : 64;
    sh.wgs = sh.whole ? (int)tiles : wgs;
    sh.desc = (int32_t*)at;
    sh.part_ml = (float*)(at + align_up((size_t)wgs * 32, 256));
    sh.part_o = (float*)((uint8_t*)sh.part_ml + align_up((size_t)wgs * 2 * held * 2 * 4, 256));
    at += quant_piece_bytes(wgs, held, D);
    hipError_t e;
    if (wide) e = launch_paged_wide(D, rows, a, &c, sh, s);
    else if (c.code == TS_INT8) e = D == 64 ? quant_some<TS_INT8, 64>(dtype, rows / 16, a, c, sh, s) : quant_some<TS_INT8, 128>(dtype, rows / 16, a, c, sh, s);
    else e = D == 64 ? quant_some<TS_E4M3, 64>(dtype, rows / 16, a, c, sh, s) : quant_some<TS_E4M3, 128>(dtype, rows / 16, a, c, sh, s);
    if (e != hipSuccess || sh.whole) return e;
    return launch_paged_merge(dtype, D, line, sh, held, wide ? kWideBlocks : kRowByRow, tiles, s);
  };
  if (!pl.many_rows) return run(pl.few_rows, 0, INT_MAX);
  const bool alone = pl.many_rows == kWideRows ? wide_alone(a) : a.q_indptr == nullptr;   // (without q_indptr every sequence has as many)
  if (!alone) {
    const hipError_t e = run(pl.few_rows, 0, pl.few_rows);
    if (e != hipSuccess) return e;
  }
  return run(pl.many_rows, alone ? 0 : pl.few_rows, INT_MAX);
}

}  // namespace ts
