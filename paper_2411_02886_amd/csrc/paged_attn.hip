// Dense attention of new tokens over their whole sequence through the page table: which kernel takes which sequences, and the
// merge of the tiles that shares have cut.
#include "paged_shares.h"
#include <limits.h>

namespace ts {

hipError_t launch_paged_stream(int dtype, int D, int blocks, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);
hipError_t launch_paged_tall(int D, const PagedAttnArgs& a, const ShareArgs& sh, hipStream_t s);

constexpr int kStreamWgs = 512, kTallWgs = 256, kTallRows = 256;

// Joins the pieces of the tiles that were cut: a workgroup column stands for the workgroup whose share began the tile, the
// pieces that follow lie in the workgroups behind it, up to the one that ends the tile.  RPB rows per workgroup, D / 4 lanes per
// row, PG groups of lanes that share the pieces.
template <int ES, int D, int RPB, int PG>
__global__ __launch_bounds__((D / 4) * RPB * PG) void paged_merge_kernel(PagedAttnArgs a, ShareArgs sh, int rows) {
  constexpr int LPR = D / 4;
  __shared__ float4 s_o[PG][RPB][LPR];
  __shared__ float s_ml[PG][RPB][2];
  const int w = blockIdx.x, G = a.H / a.H_kv;
  const int32_t* d1 = sh.desc + (size_t)w * 8 + 4;
  if (d1[3] == kPieceNone) return;
  const int row0 = d1[0], kvh = d1[1], nrows = d1[2] * G;
  const int lane = threadIdx.x & 63, sub = threadIdx.x % LPR, rr = threadIdx.x / LPR % RPB, pg = threadIdx.x / (LPR * RPB);
  const int j = blockIdx.y * RPB + rr;
  if ((int)blockIdx.y * RPB >= nrows) return;
  int pieces = 1;                                       // this workgroup's, and those of the workgroups w + 1 .. w + pieces - 1
  for (;; pieces += 64) {
    const int i = w + pieces + lane;
    const uint64_t end = __builtin_amdgcn_ballot_w64(i >= sh.wgs || sh.desc[(size_t)i * 8 + 3] == kPieceEnds);
    if (end != 0) { pieces += __builtin_ctzll(end) + 1; break; }
  }
  pieces = min(pieces, sh.wgs - w);
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int US = 4;                                 // pieces in flight per lane
  for (int p0 = pg; p0 < pieces; p0 += PG * US) {
    float2 v[US];
    float4 x[US];
#pragma unroll
    for (int u = 0; u < US; ++u) {
      const int p = p0 + u * PG;
      v[u] = make_float2(-INFINITY, 0.f);
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p >= pieces || j >= nrows) continue;
      const size_t slot = (size_t)(w + p) * 2 + (p == 0 ? 1 : 0);
      if (p > 0 && sh.desc[slot * 4 + 3] == kPieceNone) continue;      // a share without a unit
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
      o.x = fmaf(g, x[u].x, o.x); o.y = fmaf(g, x[u].y, o.y); o.z = fmaf(g, x[u].z, o.z); o.w = fmaf(g, x[u].w, o.w);
    }
    M = m;
  }
  if constexpr (PG > 1) {
    s_o[pg][rr][sub] = o;
    if (sub == 0) { s_ml[pg][rr][0] = M; s_ml[pg][rr][1] = L; }
    __syncthreads();
    if (pg != 0) return;
    float m = -INFINITY;
#pragma unroll
    for (int g = 0; g < PG; ++g) m = fmaxf(m, s_ml[g][rr][0]);
    L = 0.f; o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m != -INFINITY)
#pragma unroll
      for (int g = 0; g < PG; ++g) {
        const float f = expf(s_ml[g][rr][0] - m);
        const float4 x = s_o[g][rr][sub];
        L = fmaf(f, s_ml[g][rr][1], L);
        o.x = fmaf(f, x.x, o.x); o.y = fmaf(f, x.y, o.y); o.z = fmaf(f, x.z, o.z); o.w = fmaf(f, x.w, o.w);
      }
    M = m;
  }
  if (j >= nrows) return;
  const size_t hb = (size_t)(row0 + j / G) * a.H + kvh * G + j % G;
  o = L > 0.f ? make_float4(o.x / L, o.y / L, o.z / L, o.w / L) : make_float4(0.f, 0.f, 0.f, 0.f);
  if (ES == 2)
    *reinterpret_cast<uint2*>(a.out + (hb * D + sub * 4) * 2) = make_uint2(f32_to_bf16_bits(o.x) | (f32_to_bf16_bits(o.y) << 16), f32_to_bf16_bits(o.z) | (f32_to_bf16_bits(o.w) << 16));
  else *reinterpret_cast<float4*>(a.out + (hb * D + sub * 4) * 4) = o;
  if (sub == 0 && a.lse != nullptr) a.lse[hb] = L > 0.f ? M + logf(L) : -INFINITY;
}

template <int ES, int D>
static hipError_t merge(const PagedAttnArgs& a, const ShareArgs& sh, int rows, hipStream_t s) {
  if (rows <= 64) hipLaunchKernelGGL((paged_merge_kernel<ES, D, 4, 8>), dim3(sh.wgs, rows / 4), dim3(D * 8), 0, s, a, sh, rows);
  else hipLaunchKernelGGL((paged_merge_kernel<ES, D, 8, 1>), dim3(sh.wgs, rows / 8), dim3(D * 2), 0, s, a, sh, rows);
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
