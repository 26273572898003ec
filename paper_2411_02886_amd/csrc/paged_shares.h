// How the work of a dense attention call is cut into equal shares, on the device, from the lengths themselves.
//
// A tile is up to `tpt` tokens of one sequence times the query heads of one KV head: its rows share every key.  The tiles stand in
// one line -- KV head, sequence, tile -- and take as much room in it as they have keys (closed form: without a window a
// sequence's tiles grow by tpt keys from one to the next).  Each workgroup gets an equal piece of that line.  A cut inside a tile
// falls between two units of KT keys; the tile's pieces leave partial results, which a merge launch joins.  Workgroups of one XCD get
// neighbouring pieces, so that its L2 fetches the keys of a KV head once.
#pragma once
#include "ts_kernels.h"

namespace ts {

// words that a workgroup leaves in the workspace about its (at most two) cut tiles, eight each
constexpr int kPieceNone = 0, kPieceGoesOn = 1, kPieceEnds = 2;

struct ShareArgs {
  int tpt;          // tokens per tile
  int more_rows, most_rows;   // sequences with more_rows < n * G <= most_rows take part
  int whole;        // a workgroup per tile, nothing is cut
  int min_keys;     // smallest share
  int wgs;          // workgroups of the launch
  int32_t* desc;    // [wgs][2][4]: first row, KV head and number of tokens of the tile, kPiece*; [0]: the piece goes on from the workgroup before, [1]: it begins the tile
  float* part_o;    // [wgs][2][rows][D] not normalised
  float* part_ml;   // [wgs][2][rows][2] (reference, sum)
};

#ifdef __HIPCC__

struct SeqShape { int b, row0, n, N, tiles; };   // sequence, first row, new tokens, length, tiles (0: takes no part)

__device__ __forceinline__ SeqShape seq_shape(const PagedAttnArgs& a, const ShareArgs& sh, int G, int b) {
  SeqShape s;
  s.b = b;
  const int r0 = a.q_indptr != nullptr ? min(max(a.q_indptr[b], 0), a.T) : b * a.C;
  const int r1 = a.q_indptr != nullptr ? min(max(a.q_indptr[b + 1], 0), a.T) : r0 + a.C;
  s.row0 = r0;
  s.n = max(r1 - r0, 0);
  s.N = min(max(a.seq_lens[b], 0), a.max_seq_len);
  const long rows = (long)s.n * G;
  s.tiles = rows > sh.more_rows && rows <= sh.most_rows ? (s.n + sh.tpt - 1) / sh.tpt : 0;
  return s;
}

constexpr int kTileCost = 64;                 // keys that a tile's start and end cost

// room in the line of a sequence's first r tiles
__device__ __forceinline__ long tiles_room(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, long r) {
  if (sh.whole) return r;
  const long first = max(s.N - s.n, 0) + kTileCost, tpt = sh.tpt;
  if (a.window == 0) return r * first + tpt * (r * (r + 1) / 2);
  const long cap = min((long)a.window, (long)a.max_seq_len) + tpt + kTileCost;   // where the window cuts a tile's keys
  const long grow = cap > first ? min(r, (cap - first - 1) / tpt) : 0;           // tiles that it does not cut
  return grow * first + tpt * (grow * (grow + 1) / 2) + (r - grow) * cap;
}

// keys that a tile's rows see, in units of KT keys from u0 on; at least one unit, though it may hold no visible key
struct TileKeys { int first, end, u0, units; };
template <int KT>
__device__ __forceinline__ TileKeys tile_keys(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int r) {
  TileKeys k;
  const int c0 = r * sh.tpt, c1 = min(c0 + sh.tpt, s.n) - 1;
  k.end = max(s.N - s.n + c1 + 1, 0);
  k.first = a.window > 0 ? max(s.N - s.n + c0 - a.window + 1, 0) : 0;
  k.u0 = k.first / KT;
  k.units = max((k.end + KT - 1) / KT - k.u0, 1);
  return k;
}

struct SharePlace { int kvh, b, r, u; };

// All threads of the workgroup (NT of them): begin and end of this workgroup's share, in scalar registers.  lds: 2, scratch: NT / 64.
template <int KT, int NT>
__device__ __forceinline__ void find_share(const PagedAttnArgs& a, const ShareArgs& sh, int G, int wg, SharePlace* lds, long* scratch,
                                           SharePlace* from, SharePlace* to) {
  const int tid = threadIdx.x, lane = tid & 63, per = (a.B + NT - 1) / NT;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  long mine = 0;
  SeqShape only{0, 0, 0, 0, 0};
  for (int b = b0; b < b1; ++b) { only = seq_shape(a, sh, G, b); mine += tiles_room(a, sh, only, only.tiles); }
  long upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) { const long x = __shfl_up(upto, d); if (lane >= d) upto += x; }
  if (lane == 63) scratch[tid >> 6] = upto;
  if (tid == 0) lds[0] = lds[1] = SharePlace{a.H_kv, 0, 0, 0};   // the end of the line; also where lengths that change under the call lead nowhere
  __syncthreads();
  long before = upto - mine, line = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { if (w < (tid >> 6)) before += scratch[w]; line += scratch[w]; }
  const long all = line * a.H_kv;
  const long share = sh.whole ? 1 : max((long)sh.min_keys, (all + sh.wgs - 1) / sh.wgs);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const long x = min((long)(wg + e) * share, all);
    if (x >= all) continue;
    const int kvh = (int)(x / line);
    long y = x - kvh * line - before;
    if (y < 0 || y >= mine) continue;          // another thread's sequences
    SeqShape s = only;
    int b = b0;
    if (per > 1)
      for (; b < b1; ++b) {
        s = seq_shape(a, sh, G, b);
        const long room = tiles_room(a, sh, s, s.tiles);
        if (y < room) break;
        y -= room;
      }
    int lo = 0, hi = s.tiles - 1;              // the last tile that begins at or before y
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (tiles_room(a, sh, s, mid) <= y) lo = mid; else hi = mid - 1; }
    const long at = tiles_room(a, sh, s, lo), room = tiles_room(a, sh, s, lo + 1) - at;
    const TileKeys k = tile_keys<KT>(a, sh, s, lo);
    lds[e] = SharePlace{kvh, b, lo, (int)((y - at) * k.units / room)};
  }
  __syncthreads();
  auto scalar = [](const SharePlace& p) {
    return SharePlace{__builtin_amdgcn_readfirstlane(p.kvh), __builtin_amdgcn_readfirstlane(p.b), __builtin_amdgcn_readfirstlane(p.r),
                      __builtin_amdgcn_readfirstlane(p.u)};
  };
  *from = scalar(lds[0]); *to = scalar(lds[1]);
}

// next sequence from b on that takes part (a.B: none); every wave by itself, 64 sequences at a time
__device__ __forceinline__ int next_sequence(const PagedAttnArgs& a, const ShareArgs& sh, int G, int b) {
  const int lane = threadIdx.x & 63;
  for (; b < a.B; b += 64) {
    const bool in = b + lane < a.B && seq_shape(a, sh, G, b + lane).tiles > 0;
    const uint64_t any = __builtin_amdgcn_ballot_w64(in);
    if (any != 0) return b + __builtin_ctzll(any);
  }
  return a.B;
}

// A workgroup's walk over its share: fn(kvh, shape, r, keys, ua, ub, again) for units [ua, ub) of every tile in it; where it returns true it is
// called again, with `again` set.
template <int KT, typename F>
__device__ __forceinline__ void walk_share(const PagedAttnArgs& a, const ShareArgs& sh, int G, const SharePlace& from, const SharePlace& to, F&& fn) {
  int kvh = from.kvh, b = from.b, r = from.r, ua = from.u;
  if (kvh >= a.H_kv) return;
  SeqShape s = seq_shape(a, sh, G, b);
  bool again = false;
  for (;;) {
    const bool last = kvh == to.kvh && b == to.b && r == to.r;
    const TileKeys k = tile_keys<KT>(a, sh, s, r);
    const int ub = last ? to.u : k.units;
    if (ub > ua) { again = fn(kvh, s, r, k, ua, ub, again); if (again) continue; }
    if (last) return;
    ua = 0;
    if (++r < s.tiles) continue;
    r = 0;
    b = next_sequence(a, sh, G, b + 1);
    if (b >= a.B) { if (++kvh >= a.H_kv) return; b = next_sequence(a, sh, G, 0); }
    s = seq_shape(a, sh, G, b);
  }
}

// which piece a workgroup stands for: those of an XCD (workgroup L runs on XCD L % 8) follow each other
__device__ __forceinline__ int share_of(int block, int wgs) {
  return (wgs & 7) == 0 ? (block & 7) * (wgs >> 3) + (block >> 3) : block;
}

#endif  // __HIPCC__
}  // namespace ts
