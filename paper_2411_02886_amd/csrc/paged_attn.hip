// Dense attention of new tokens over their whole sequence through the page table: which kernel takes which sequences, and the
// merge of the tiles that shares have cut.
#include "paged_shares.h"
#include <limits.h>
#include <algorithm>

namespace ts {

hipError_t launch_paged_stream(int dtype, int D, int blocks, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);
hipError_t launch_paged_tall(int D, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);

constexpr int kTallRows = 256;
// Workgroups that cut the line into shares: one per CU (128 / 192 / 256 / 512 of the stream kernel: a bf16 token over 131072 keys 129, 98, 91, 95 us, over
// 1000 keys 10.9, 11.0, 11.1, 13.5, 16 drafts of 8 over 3000 keys 66, 51, 46, 49: fewer start, and fewer pieces are joined).
constexpr int kShareWgs = 256;

// Pieces of the tile that workgroup w's share began: its own and those of workgroups w + 1 .. w + count - 1, up to the one that ends the tile; a
// share in between may hold no unit of it.  The states of the first 64 are loaded beside w's own.
struct Pieces {
  int count;
  uint64_t some;                                // of workgroups w + 1 .. w + 64: those that left a piece
  __device__ __forceinline__ bool there(const ShareArgs& sh, int w, int p) const {
    if (p == 0) return true;
    return p <= 64 ? ((some >> (p - 1)) & 1) != 0 : sh.desc[(size_t)(w + p) * 8 + 3] != kPieceNone;
  }
};
__device__ __forceinline__ int next_piece(const ShareArgs& sh, int w, int lane) {
  return w + 1 + lane < sh.wgs ? sh.desc[(size_t)(w + 1 + lane) * 8 + 3] : kPieceEnds;
}
__device__ __forceinline__ Pieces find_pieces(const ShareArgs& sh, int w, int lane, int state) {
  Pieces p{1, __builtin_amdgcn_ballot_w64(state != kPieceNone)};
  for (;; state = next_piece(sh, w + p.count - 1, lane)) {
    const uint64_t end = __builtin_amdgcn_ballot_w64(state == kPieceEnds);
    if (end != 0) { p.count += __builtin_ctzll(end) + 1; break; }
    p.count += 64;
  }
  p.count = min(p.count, sh.wgs - w);
  return p;
}

// Joins the pieces of the tiles that were cut: blockIdx.y stands for the workgroup whose share began the tile, the
// pieces that follow lie in the workgroups behind it, up to the one that ends the tile: many of which may belong to a tile.  A workgroup per row: D / 4
// lanes hold it, PG groups of them take the pieces in turn, with US in flight each, and meet in LDS.  Latency is all it costs (one token over 4096
// keys, fp32: 13 us with the attention; with four rows per workgroup and two pieces in flight per group it was 18).
template <int ES, int D, int THREADS, int US>
__global__ __launch_bounds__(THREADS) void paged_merge_kernel(PagedAttnArgs a, ShareArgs sh, int rows) {
  constexpr int LPR = D / 4, PG = THREADS / LPR;
  __shared__ float4 s_o[PG][LPR];
  __shared__ float s_ml[PG][2];
  const int w = blockIdx.y, G = a.H / a.H_kv;     // (rows first: the tiles that were cut may all be every fourth workgroup's, and so on two XCDs)
  const int32_t* d1 = sh.desc + (size_t)w * 8 + 4;
  const int lane = threadIdx.x & 63, next = next_piece(sh, w, lane);
  if (d1[3] == kPieceNone) return;
  const int row0 = d1[0], kvh = d1[1], nrows = d1[2] * G;
  const int sub = threadIdx.x % LPR, pg = threadIdx.x / LPR;
  const Pieces pc = find_pieces(sh, w, lane, next);
  const int pieces = pc.count;
  for (int j = blockIdx.x; j < nrows; j += gridDim.x) {
    float M = -INFINITY, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = pg; p0 < pieces; p0 += PG * US) {
      float2 v[US];
      float4 x[US];
#pragma unroll
      for (int u = 0; u < US; ++u) {
        const int p = p0 + u * PG;
        const size_t slot = (size_t)(w + p) * 2 + (p == 0 ? 1 : 0);
        v[u] = make_float2(-INFINITY, 0.f);
        x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p >= pieces || !pc.there(sh, w, p)) continue;
        v[u] = *reinterpret_cast<const float2*>(sh.part_ml + (slot * rows + j) * 2);
        x[u] = *reinterpret_cast<const float4*>(sh.part_o + (slot * rows + j) * D + sub * 4);
      }
      float m = M;
#pragma unroll
      for (int u = 0; u < US; ++u) m = fmaxf(m, v[u].x);
      if (m == -INFINITY) continue;
      const float f = expf(M - m);
      L *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
      for (int u = 0; u < US; ++u) {
        const float g = expf(v[u].x - m);
        L = fmaf(g, v[u].y, L);
        o.x = fmaf(g, x[u].x, o.x); o.y = fmaf(g, x[u].y, o.y);
        o.z = fmaf(g, x[u].z, o.z); o.w = fmaf(g, x[u].w, o.w);
      }
      M = m;
    }
    s_o[pg][sub] = o;
    if (sub == 0) { s_ml[pg][0] = M; s_ml[pg][1] = L; }
    __syncthreads();
    if (pg == 0) {
#pragma unroll
      for (int g = 1; g < PG; ++g) M = fmaxf(M, s_ml[g][0]);
      L = 0.f; o = make_float4(0.f, 0.f, 0.f, 0.f);
      if (M != -INFINITY)
#pragma unroll
        for (int g = 0; g < PG; ++g) {
          const float f = expf(s_ml[g][0] - M);
          const float4 x = s_o[g][sub];
          L = fmaf(f, s_ml[g][1], L);
          o.x = fmaf(f, x.x, o.x); o.y = fmaf(f, x.y, o.y); o.z = fmaf(f, x.z, o.z); o.w = fmaf(f, x.w, o.w);
        }
      const size_t hb = (size_t)(row0 + j / G) * a.H + kvh * G + j % G;
      const float4 y = L == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x / L, o.y / L, o.z / L, o.w / L);   // (a sum that is no number stays one)
      if (ES == 2)
        *reinterpret_cast<uint2*>(a.out + (hb * D + sub * 4) * 2) = make_uint2(f32_to_bf16_bits(y.x) | (f32_to_bf16_bits(y.y) << 16), f32_to_bf16_bits(y.z) | (f32_to_bf16_bits(y.w) << 16));
      else *reinterpret_cast<float4*>(a.out + (hb * D + sub * 4) * 4) = y;
      if (sub == 0 && a.lse != nullptr) a.lse[hb] = L == 0.f ? -INFINITY : M + logf(L);
    }
    __syncthreads();                                    // the next row takes the same place
  }
}

// The same for the tall kernel, whose pieces lie as in its registers: of each block of 32 rows 16 bytes of the output [D / 8][64 lanes], the
// lane's row lane % 32, its elements 8 i + 4 (lane / 32) .. + 3.  A wave of a workgroup (blockIdx.x: block of rows, then i / 4) has one i.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_tall_kernel(PagedAttnArgs a, ShareArgs sh) {
  constexpr int PB = D / 32, US = 6;                    // workgroups per block of rows; partial results in flight
  const int w = blockIdx.y, G = a.H / a.H_kv;
  const int32_t* d1 = sh.desc + (size_t)w * 8 + 4;
  const int lane = threadIdx.x & 63, next = next_piece(sh, w, lane);
  if (d1[3] == kPieceNone) return;
  const int row0 = d1[0], kvh = d1[1], nrows = d1[2] * G;
  const int block = blockIdx.x / PB, i = blockIdx.x % PB * 4 + (threadIdx.x >> 6), j = block * 32 + (lane & 31);
  if (block * 32 >= nrows) return;
  const Pieces pc = find_pieces(sh, w, lane, next);
  const int pieces = pc.count;
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < pieces; p0 += US) {
    float2 v[US];
    float4 x[US];
#pragma unroll
    for (int u = 0; u < US; ++u) {
      const int p = p0 + u;
      const size_t slot = (size_t)(w + p) * 2 + (p == 0 ? 1 : 0);
      v[u] = make_float2(-INFINITY, 0.f);
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p >= pieces || !pc.there(sh, w, p)) continue;
      v[u] = *reinterpret_cast<const float2*>(sh.part_ml + (slot * kTallRows + j) * 2);
      x[u] = reinterpret_cast<const float4*>(sh.part_o + slot * kTallRows * D)[(block * (D / 8) + i) * 64 + lane];
    }
    float m = M;
#pragma unroll
    for (int u = 0; u < US; ++u) m = fmaxf(m, v[u].x);
    if (m == -INFINITY) continue;
    const float f = expf(M - m);
    L *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
    for (int u = 0; u < US; ++u) {
      const float g = expf(v[u].x - m);
      L = fmaf(g, v[u].y, L);
      o.x = fmaf(g, x[u].x, o.x); o.y = fmaf(g, x[u].y, o.y); o.z = fmaf(g, x[u].z, o.z); o.w = fmaf(g, x[u].w, o.w);
    }
    M = m;
  }
  if (j >= nrows) return;
  const size_t hb = (size_t)(row0 + j / G) * a.H + kvh * G + j % G;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  *reinterpret_cast<uint2*>(a.out + (hb * D + 8 * i + 4 * (lane >> 5)) * 2) =
      make_uint2(f32_to_bf16_bits(o.x * inv) | (f32_to_bf16_bits(o.y * inv) << 16), f32_to_bf16_bits(o.z * inv) | (f32_to_bf16_bits(o.w * inv) << 16));
  if (i == 0 && lane < 32 && a.lse != nullptr) a.lse[hb] = L == 0.f ? -INFINITY : M + logf(L);
}

template <int ES, int D>
static hipError_t merge(const PagedAttnArgs& a, const ShareArgs& sh, int rows, long tiles, hipStream_t s) {
  if (rows == kTallRows) {                       // (tiles are short only where their sequence is)
    hipLaunchKernelGGL(paged_merge_tall_kernel<D>, dim3(kTallRows / 32 * (D / 32), sh.wgs), dim3(256), 0, s, a, sh);
    return hipGetLastError();
  }
  // A workgroup per row that a tile may have; where only the sequences with few rows are meant, as many as one token has (12 mixed ones, 28 heads: 4 us
  // less, as most workgroups find nothing).  More rows take turns.  Where there are many tiles, of few pieces then, a wave per row (16 drafts of 8 tokens
  // over 3000 keys 38.9 us, by 256 threads 42.3; one token over 4000, 32 pieces a tile, 14.5 and 12.2).
  const int G = a.H / a.H_kv;
  const dim3 grid(sh.most_rows < INT_MAX ? G : std::min(sh.tpt, a.C) * G, sh.wgs);
  if (tiles * 4 >= sh.wgs) hipLaunchKernelGGL((paged_merge_kernel<ES, D, 64, 4>), grid, dim3(64), 0, s, a, sh, rows);
  else hipLaunchKernelGGL((paged_merge_kernel<ES, D, 256, 4>), grid, dim3(256), 0, s, a, sh, rows);
  return hipGetLastError();
}

// bytes that tiles of `rows` rows leave pieces in
static size_t piece_bytes(int rows, int D) {
  return align_up((size_t)kShareWgs * 32, 256) + align_up((size_t)kShareWgs * 2 * rows * 2 * 4, 256) + (size_t)kShareWgs * 2 * rows * D * 4;
}

// The rows of a sequence and KV head, n * G, decide: up to 16 (one block of columns) or 32 by the stream kernel, which is bound by the memory (8 tokens times
// 4 heads over 2000 keys, one sequence 17 us, eight of them 25; by the tall kernel 32 and 47), bf16 up to 128 by four of its tiles (32 tokens over 2000 keys 21 us,
// by the tall kernel 33, 8 times 2000 keys 38 and 48, 8 times 8000 145 and 128; with 192 rows these are 28 and 34, 51 and 48, 224 and 135); more by the tall one (bf16), or by
// the stream kernel with 64 rows a tile (fp32, whose matrix products it is then bound by: 512 tokens over 4000 keys 362 us, with 32 rows 412).  A packed batch may hold both kinds:
// two launches, each takes the sequences that are its.  fp32: as a packed batch's bound says little about most of its sequences, twice as many rows go without the second
// (12 tokens over 3000 keys 28.7 us, else 42.8; 8 times 87 and 84).
// Rounded weights, for which the tall kernel needs half the time: up to 64 rows by the stream kernel (16 tokens over 2000 keys 18.6 us, by the tall kernel 27.7, 8
// times 4000 47 and 53; with 96 rows it would be 75 and 52), twice that where a packed batch's sequences are
// shorter than the bound (loose: less than three quarters of it on average; 8 of 1 to 30 tokens over up to 4000 keys 42 us, else 76; but 8 of 24 each 73 and 57).
struct PagedPlan { int few_rows, many_rows; };   // rows of the tiles of sequences with few rows, and of those with more (0: there are none)
static PagedPlan paged_plan(int dtype, int G, int chunk, bool packed, bool loose, bool rounded) {
  const long rows = (long)chunk * G;
  if (rows <= 16) return PagedPlan{16, 0};
  if (rows <= (dtype == TS_F32 ? (packed ? 64 : 32) : rounded && !loose ? 64 : 128)) return PagedPlan{32, 0};
  return dtype == TS_BF16 ? PagedPlan{32, kTallRows} : PagedPlan{16, 64};
}

size_t paged_attn_workspace(int dtype, int D, int G, int chunk) {
  size_t most = 0;
  for (int form = 0; form < 4; ++form) {
    const PagedPlan pl = paged_plan(dtype, G, chunk, (form & 1) != 0, (form & 1) != 0, (form & 2) != 0);
    most = std::max(most, align_up(piece_bytes(pl.few_rows, D) + (pl.many_rows ? piece_bytes(pl.many_rows, D) : 0), 256));
  }
  return most;
}

hipError_t launch_paged_attn(int dtype, int D, const PagedAttnArgs& a, void* ws, hipStream_t s) {
  const int G = a.H / a.H_kv;
  const PagedPlan pl = paged_plan(dtype, G, a.C, a.q_indptr != nullptr, (long)a.T * 4 <= (long)a.B * a.C * 3, a.round_weights != 0);
  uint8_t* at = (uint8_t*)ws;
  // tiles of every sequence (0: not as many), and bounds on all tiles and on the keys of one.  A tile of few rows beside large ones is its whole sequence.
  auto each_of = [&](int tpt, bool beside) -> int { return beside ? 1 : a.q_indptr != nullptr ? 0 : (a.C + tpt - 1) / tpt; };
  auto tiles_of = [&](int tpt, bool beside) -> long {
    const int each = each_of(tpt, beside);
    return (each > 0 ? (long)a.B * each : (long)a.T / tpt + a.B) * a.H_kv;
  };
  auto keys_of = [&](int tpt) -> long { return std::min((long)a.max_seq_len, a.window > 0 ? (long)a.window + tpt : LONG_MAX); };
  auto run = [&](int rows, int more_rows, int most_rows, bool whole) -> hipError_t {
    const bool tall = rows == kTallRows;
    const int kt = tall || dtype == TS_F32 ? 64 : 128;
    ShareArgs sh{};
    sh.tpt = rows / G;
    sh.more_rows = more_rows;
    sh.most_rows = most_rows;
    sh.whole = whole ? 1 : 0;
    const bool beside = most_rows < INT_MAX;
    sh.each = each_of(sh.tpt, beside);
    // The smallest share (twice as much: a token over 1000 keys 1.4 us more, 64 tokens over 4000 keys 4 us), and what a tile's start and end cost (a quarter
    // of it: 12 mixed chunks 273 us instead of 245; twice: 243, but 2048 tokens 82 instead of 78).
    sh.min_keys = tall ? 2 * kt : kt;
    sh.tile_cost = tall ? 256 : 64;
    sh.wgs = whole ? (int)tiles_of(sh.tpt, beside) : kShareWgs;
    sh.desc = (int32_t*)at;
    sh.part_ml = (float*)(at + align_up((size_t)kShareWgs * 32, 256));
    sh.part_o = (float*)((uint8_t*)sh.part_ml + align_up((size_t)kShareWgs * 2 * rows * 2 * 4, 256));
    at += piece_bytes(rows, D);
    const hipError_t e = tall ? launch_paged_tall(D, a, sh, s) : launch_paged_stream(dtype, D, rows / 16, a, sh, s);
    if (e != hipSuccess || whole) return e;
    if (dtype == TS_BF16) return D == 64 ? merge<2, 64>(a, sh, rows, tiles_of(sh.tpt, beside), s) : merge<2, 128>(a, sh, rows, tiles_of(sh.tpt, beside), s);
    return D == 64 ? merge<4, 64>(a, sh, rows, tiles_of(sh.tpt, beside), s) : merge<4, 128>(a, sh, rows, tiles_of(sh.tpt, beside), s);
  };
  // A workgroup per tile, and no merge, where tiles are short, or where there are enough of them that are not long.  (200 keys: 8.2 us, in shares 10.3; 64
  // sequences of 250 to 500 keys, 512 tiles: 22.8 and 29; but 16 fp32 sequences of 1000 to 2000 keys, 32 tiles, 42 us instead of 17.)  Beside large
  // tiles a second merge costs more, up to 1024 keys (14 chunks of 1 to 197 tokens over up to 770 keys 52 us, in shares 64; one to four single tokens beside a prompt of
  // 512: over 300 keys 42 and 44 to 48, over 600 45.5 and 44.5, over 1000 53 and 47, 16 of them over 1000 52 and 53; but one to four over 1500 keys 59 and 47, over 2000 66 and 48).
  auto few_whole = [&](int rows, bool beside) -> bool {
    const long tiles = tiles_of(rows / G, beside), keys = keys_of(rows / G);
    return tiles < (1l << 23) && (keys <= (beside ? 1024 : 512) || (tiles >= kShareWgs && keys <= 16 * (dtype == TS_F32 ? 64 : 128)));
  };
  if (!pl.many_rows) return run(pl.few_rows, 0, INT_MAX, few_whole(pl.few_rows, false));
  // Short prompts have too few tiles for the chip: there 32 rows a tile for all sequences, at most two workgroups per CU.  (256 tokens 10.6 us, by 256 rows a
  // tile 20.7, 512 tokens 17 and 29, with rounded weights 20.8; 768, more tiles than that, 33 and 38, rounded 27, and 4 of 256 25 and 22.  fp32: 256 tokens 20.5, by 64 rows a tile 33, 400 39 and 48.)
  // (fp32, whose larger tiles save less, also with more tiles of few keys: 16 sequences of 64 tokens 33 and 45, 4 of 256 60 and 60.)
  const long small = tiles_of(32 / G, false), small_keys = keys_of(32 / G);
  if (small_keys <= 1024 && (small <= 2 * kShareWgs || (dtype == TS_F32 && small * small_keys <= 1l << 18))) return run(32, 0, INT_MAX, true);
  if (a.q_indptr != nullptr) {                             // (without, every sequence has as many)
    const hipError_t e = run(pl.few_rows, 0, pl.few_rows, few_whole(pl.few_rows, true));
    if (e != hipSuccess) return e;
  }
  // (4 prompts of 512 tokens 35 us, in shares 40, 8 of 256 24.6 and 30.4; but one of 1024 52 and 44, 2 of 512 over 500 keys more 54 and 49.  With rounded weights
  // 1024 tokens take 33.4 us, in shares 35.7, 2048 59 and 54.  A packed batch's bound counts up to a tile per sequence too many: there twice the tiles, 24 of 1
  // to 100 tokens 36 us, in shares 41, 8 of 1 to 600 68 and 75; four times would cost 64 of 64 tokens over 900 119 instead of 98 (rounded).)
  const long tiles = tiles_of(pl.many_rows / G, false);
  return run(pl.many_rows, a.q_indptr != nullptr ? pl.few_rows : 0, INT_MAX,
             tiles <= kShareWgs * (a.q_indptr != nullptr ? 2 : 1) && keys_of(pl.many_rows / G) <= (a.round_weights ? 1024 : 768));
}

}  // namespace ts
