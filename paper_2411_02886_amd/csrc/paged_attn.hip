// Dense attention of new tokens over their whole sequence through the page table: which kernel takes which sequences, and the
// merge of the tiles that shares have cut.
#include "paged_shares.h"
#include <limits.h>
#include <algorithm>

namespace ts {

hipError_t launch_paged_stream(int dtype, int D, int blocks, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);
hipError_t launch_paged_tall(int D, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);

constexpr int kStreamWgs = 512, kTallWgs = 256, kTallRows = 256;

// Joins the pieces of the tiles that were cut: blockIdx.y stands for the workgroup whose share began the tile, the
// pieces that follow lie in the workgroups behind it, up to the one that ends the tile.  D / 4 lanes per row, RPT rows per lane, PG
// groups of lanes that share the pieces, US of which a lane has in flight: many of which may belong to a tile.
template <int ES, int D, int THREADS, int RPT, int PG, int US>
__global__ __launch_bounds__(THREADS) void paged_merge_kernel(PagedAttnArgs a, ShareArgs sh, int rows) {
  constexpr int LPR = D / 4, LR = THREADS / (LPR * PG), RPB = LR * RPT;   // rows side by side, rows per workgroup
  __shared__ float4 s_o[PG][RPB][LPR];
  __shared__ float s_ml[PG][RPB][2];
  const int w = blockIdx.y, G = a.H / a.H_kv;     // (rows first: the tiles that were cut may all be every fourth workgroup's, and so on two XCDs)
  const int32_t* d1 = sh.desc + (size_t)w * 8 + 4;
  if (d1[3] == kPieceNone) return;
  const int row0 = d1[0], kvh = d1[1], nrows = d1[2] * G;
  const int lane = threadIdx.x & 63, sub = threadIdx.x % LPR, rr = threadIdx.x / LPR % LR, pg = threadIdx.x / (LPR * LR);
  int pieces = 1;                                       // this workgroup's, and those of the workgroups w + 1 .. w + pieces - 1
  for (;; pieces += 64) {
    const int i = w + pieces + lane;
    const uint64_t end = __builtin_amdgcn_ballot_w64(i >= sh.wgs || sh.desc[(size_t)i * 8 + 3] == kPieceEnds);
    if (end != 0) { pieces += __builtin_ctzll(end) + 1; break; }
  }
  pieces = min(pieces, sh.wgs - w);
  for (int j0 = blockIdx.x * RPB; j0 < nrows; j0 += gridDim.x * RPB) {
    float M[RPT], L[RPT];
    float4 o[RPT];
#pragma unroll
    for (int t = 0; t < RPT; ++t) { M[t] = -INFINITY; L[t] = 0.f; o[t] = make_float4(0.f, 0.f, 0.f, 0.f); }
    for (int p0 = pg; p0 < pieces; p0 += PG * US) {
      float2 v[RPT][US];
      float4 x[RPT][US];
#pragma unroll
      for (int u = 0; u < US; ++u) {
        const int p = p0 + u * PG;
        const size_t slot = (size_t)(w + p) * 2 + (p == 0 ? 1 : 0);
        const bool there = p < pieces && (p == 0 || sh.desc[slot * 4 + 3] != kPieceNone);   // a share may hold no unit
#pragma unroll
        for (int t = 0; t < RPT; ++t) {
          const int j = j0 + t * LR + rr;
          v[t][u] = make_float2(-INFINITY, 0.f);
          x[t][u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (!there || j >= nrows) continue;
          v[t][u] = *reinterpret_cast<const float2*>(sh.part_ml + (slot * rows + j) * 2);
          x[t][u] = *reinterpret_cast<const float4*>(sh.part_o + (slot * rows + j) * D + sub * 4);
        }
      }
#pragma unroll
      for (int t = 0; t < RPT; ++t) {
        float m = M[t];
#pragma unroll
        for (int u = 0; u < US; ++u) m = fmaxf(m, v[t][u].x);
        if (m == -INFINITY) continue;
        const float f = expf(M[t] - m);
        L[t] *= f; o[t].x *= f; o[t].y *= f; o[t].z *= f; o[t].w *= f;
#pragma unroll
        for (int u = 0; u < US; ++u) {
          const float g = expf(v[t][u].x - m);
          L[t] = fmaf(g, v[t][u].y, L[t]);
          o[t].x = fmaf(g, x[t][u].x, o[t].x); o[t].y = fmaf(g, x[t][u].y, o[t].y);
          o[t].z = fmaf(g, x[t][u].z, o[t].z); o[t].w = fmaf(g, x[t][u].w, o[t].w);
        }
        M[t] = m;
      }
    }
    if constexpr (PG > 1) {
#pragma unroll
      for (int t = 0; t < RPT; ++t) {
        s_o[pg][t * LR + rr][sub] = o[t];
        if (sub == 0) { s_ml[pg][t * LR + rr][0] = M[t]; s_ml[pg][t * LR + rr][1] = L[t]; }
      }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < RPT; ++t) {
        float m = -INFINITY;
#pragma unroll
        for (int g = 0; g < PG; ++g) m = fmaxf(m, s_ml[g][t * LR + rr][0]);
        L[t] = 0.f; o[t] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (m != -INFINITY)
#pragma unroll
          for (int g = 0; g < PG; ++g) {
            const float f = expf(s_ml[g][t * LR + rr][0] - m);
            const float4 x = s_o[g][t * LR + rr][sub];
            L[t] = fmaf(f, s_ml[g][t * LR + rr][1], L[t]);
            o[t].x = fmaf(f, x.x, o[t].x); o[t].y = fmaf(f, x.y, o[t].y); o[t].z = fmaf(f, x.z, o[t].z); o[t].w = fmaf(f, x.w, o[t].w);
          }
        M[t] = m;
      }
    }
#pragma unroll
    for (int t = 0; t < RPT; ++t) {
      const int j = j0 + t * LR + rr;
      if (j >= nrows || pg != 0) continue;
      const size_t hb = (size_t)(row0 + j / G) * a.H + kvh * G + j % G;
      const float4 y = L[t] > 0.f ? make_float4(o[t].x / L[t], o[t].y / L[t], o[t].z / L[t], o[t].w / L[t]) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (ES == 2)
        *reinterpret_cast<uint2*>(a.out + (hb * D + sub * 4) * 2) = make_uint2(f32_to_bf16_bits(y.x) | (f32_to_bf16_bits(y.y) << 16), f32_to_bf16_bits(y.z) | (f32_to_bf16_bits(y.w) << 16));
      else *reinterpret_cast<float4*>(a.out + (hb * D + sub * 4) * 4) = y;
      if (sub == 0 && a.lse != nullptr) a.lse[hb] = L[t] > 0.f ? M[t] + logf(L[t]) : -INFINITY;
    }
    if (PG > 1) __syncthreads();                        // the next rows take the same place
  }
}

// The same for the tall kernel, whose pieces lie as in its registers: of each block of 32 rows (blockIdx.x), 16 bytes of the output
// [D / 8][64 lanes], the lane's row lane % 32, its elements 8 i + 4 (lane / 32) .. + 3.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_tall_kernel(PagedAttnArgs a, ShareArgs sh) {
  constexpr int NT = D / 32, US = 3;                    // 16-byte pieces per thread, partial results in flight
  const int w = blockIdx.y, G = a.H / a.H_kv;
  const int32_t* d1 = sh.desc + (size_t)w * 8 + 4;
  if (d1[3] == kPieceNone) return;
  const int row0 = d1[0], kvh = d1[1], nrows = d1[2] * G;
  const int lane = threadIdx.x & 63, j = blockIdx.x * 32 + (lane & 31);
  if ((int)blockIdx.x * 32 >= nrows) return;
  int pieces = 1;
  for (;; pieces += 64) {
    const int i = w + pieces + lane;
    const uint64_t end = __builtin_amdgcn_ballot_w64(i >= sh.wgs || sh.desc[(size_t)i * 8 + 3] == kPieceEnds);
    if (end != 0) { pieces += __builtin_ctzll(end) + 1; break; }
  }
  pieces = min(pieces, sh.wgs - w);
  float M = -INFINITY, L = 0.f;
  float4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < pieces; p0 += US) {
    float2 v[US];
    float4 x[US][NT];
#pragma unroll
    for (int u = 0; u < US; ++u) {
      const int p = p0 + u;
      const size_t slot = (size_t)(w + p) * 2 + (p == 0 ? 1 : 0);
      const bool there = p < pieces && (p == 0 || sh.desc[slot * 4 + 3] != kPieceNone);   // a share may hold no unit
      v[u] = make_float2(-INFINITY, 0.f);
      if (there) v[u] = *reinterpret_cast<const float2*>(sh.part_ml + (slot * kTallRows + j) * 2);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        x[u][t] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (there) x[u][t] = *(reinterpret_cast<const float4*>(sh.part_o + slot * kTallRows * D) + (size_t)blockIdx.x * (D / 8 * 64) + t * 256 + threadIdx.x);
      }
    }
    float m = M;
#pragma unroll
    for (int u = 0; u < US; ++u) m = fmaxf(m, v[u].x);
    if (m == -INFINITY) continue;
    const float f = expf(M - m);
    L *= f;
#pragma unroll
    for (int t = 0; t < NT; ++t) { o[t].x *= f; o[t].y *= f; o[t].z *= f; o[t].w *= f; }
#pragma unroll
    for (int u = 0; u < US; ++u) {
      const float g = expf(v[u].x - m);
      L = fmaf(g, v[u].y, L);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        o[t].x = fmaf(g, x[u][t].x, o[t].x); o[t].y = fmaf(g, x[u][t].y, o[t].y);
        o[t].z = fmaf(g, x[u][t].z, o[t].z); o[t].w = fmaf(g, x[u][t].w, o[t].w);
      }
    }
    M = m;
  }
  if (j >= nrows) return;
  const size_t hb = (size_t)(row0 + j / G) * a.H + kvh * G + j % G;
  const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int d = 8 * (t * 4 + (threadIdx.x >> 6)) + 4 * (lane >> 5);
    *reinterpret_cast<uint2*>(a.out + (hb * D + d) * 2) = make_uint2(f32_to_bf16_bits(o[t].x * inv) | (f32_to_bf16_bits(o[t].y * inv) << 16),
                                                                     f32_to_bf16_bits(o[t].z * inv) | (f32_to_bf16_bits(o[t].w * inv) << 16));
  }
  if (threadIdx.x < 32 && a.lse != nullptr) a.lse[hb] = L > 0.f ? M + logf(L) : -INFINITY;
}

template <int ES, int D>
static hipError_t merge(const PagedAttnArgs& a, const ShareArgs& sh, int rows, hipStream_t s) {
  // (a tile with more rows than the bound says takes turns; the tall kernel's tiles are short only where their sequence is)
  if (rows != kTallRows) hipLaunchKernelGGL((paged_merge_kernel<ES, D, D * 8, 1, 8, 4>), dim3((std::min(sh.tpt, a.C) * (a.H / a.H_kv) + 3) / 4, sh.wgs), dim3(D * 8), 0, s, a, sh, rows);
  else hipLaunchKernelGGL(paged_merge_tall_kernel<D>, dim3(kTallRows / 32, sh.wgs), dim3(256), 0, s, a, sh);
  return hipGetLastError();
}

// bytes that a kernel of `wgs` workgroups and tiles of `rows` rows leaves pieces in
static size_t piece_bytes(int wgs, int rows, int D) {
  return align_up((size_t)wgs * 32, 256) + align_up((size_t)wgs * 2 * rows * 2 * 4, 256) + (size_t)wgs * 2 * rows * D * 4;
}

// The rows of a sequence and KV head, n * G, decide: up to 16 (one block of columns) or 32 by the stream kernel, which is bound by the memory; more by
// the tall one (bf16), or by the stream kernel with 64 rows a tile (fp32, whose matrix products it is then bound by).  A packed batch may hold both kinds:
// two launches, each takes the sequences that are its.
struct PagedPlan { int few_blocks, many; };   // blocks of 16 rows of the stream kernel for few rows; whether a sequence may have more
static PagedPlan paged_plan(int dtype, int G, int chunk) {
  const long rows = (long)chunk * G;
  if (rows <= 16) return PagedPlan{1, 0};
  if (rows <= 32) return PagedPlan{2, 0};
  return PagedPlan{dtype == TS_BF16 ? 2 : 1, 1};
}
static int many_rows(int dtype) { return dtype == TS_BF16 ? kTallRows : 64; }
static int many_wgs(int dtype, int D) { return dtype == TS_BF16 || D == 128 ? kTallWgs : kStreamWgs; }

size_t paged_attn_workspace(int dtype, int D, int G, int chunk) {
  const PagedPlan pl = paged_plan(dtype, G, chunk);
  return align_up(piece_bytes(kStreamWgs, 16 * pl.few_blocks, D) + (pl.many ? piece_bytes(many_wgs(dtype, D), many_rows(dtype), D) : 0), 256);
}

hipError_t launch_paged_attn(int dtype, int D, const PagedAttnArgs& a, void* ws, hipStream_t s) {
  const int G = a.H / a.H_kv;
  const PagedPlan pl = paged_plan(dtype, G, a.C);
  uint8_t* at = (uint8_t*)ws;
  for (int kind = 0; kind < 2; ++kind) {                 // few rows, many rows
    const bool few = kind == 0;
    const int rows = few ? 16 * pl.few_blocks : many_rows(dtype), most_wgs = few ? kStreamWgs : many_wgs(dtype, D);
    if (!few && !pl.many) break;
    ShareArgs sh{};
    sh.tpt = rows / G;
    sh.more_rows = few || a.q_indptr == nullptr ? 0 : 16 * pl.few_blocks;
    sh.most_rows = few && pl.many ? 16 * pl.few_blocks : INT_MAX;
    sh.desc = (int32_t*)at;
    sh.part_ml = (float*)(at + align_up((size_t)most_wgs * 32, 256));
    sh.part_o = (float*)((uint8_t*)sh.part_ml + align_up((size_t)most_wgs * 2 * rows * 2 * 4, 256));
    at += piece_bytes(most_wgs, rows, D);
    if (few && pl.many && a.q_indptr == nullptr) continue;   // every sequence has as many
    const bool tall = !few && dtype == TS_BF16;
    const int kt = tall ? 64 : dtype == TS_BF16 ? 128 : 64;
    sh.min_keys = 2 * kt;
    sh.tile_cost = tall ? 256 : 64;
    sh.wgs = most_wgs;
    hipError_t e;
    if (tall) e = launch_paged_tall(D, a, sh, s);
    else e = launch_paged_stream(dtype, D, rows / 16, a, sh, s);
    if (e != hipSuccess) return e;
    if (sh.whole) continue;
    if (dtype == TS_BF16) e = D == 64 ? merge<2, 64>(a, sh, rows, s) : merge<2, 128>(a, sh, rows, s);
    else e = D == 64 ? merge<4, 64>(a, sh, rows, s) : merge<4, 128>(a, sh, rows, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ts
