// How the work of a dense attention call is cut into equal shares, on the device, from the lengths themselves.
//
// A tile is up to `tpt` tokens of one sequence times the query heads of one KV head: its rows share every key.  The tiles stand in
// one line -- KV head, sequence, tile -- and take as much room in it as they have keys (closed form: without a window a
// sequence's tiles grow by tpt keys from one to the next) and their start and end cost.  A sequence's tiles stand as first, last,
// second, last but one, ...: two neighbours together are as long as any other two, and the cuts of a prompt often fall between tiles.  Each
// workgroup gets an equal piece of that line.  A cut inside a tile falls between two units of KT keys (near an end of the tile it moves
// there); the tile's pieces leave partial results, which a merge launch joins.  Workgroups of one XCD get
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
  int tile_cost;    // keys that a tile's start and end cost
  int wgs;          // workgroups of the launch
  int32_t* desc;    // [wgs][2][4]: first row, KV head and number of tokens of the tile, kPiece*; [0]: the piece goes on from the workgroup before, [1]: it begins the tile
  float* part_o;    // [wgs][2][rows][D] not normalised
  float* part_ml;   // [wgs][2][rows][2] (reference, sum)
};

#ifdef __HIPCC__

// floor(a / b) for 0 <= a < 2^53, 0 < b: a division of doubles and its correction (of 64-bit integers the compiler makes 150 instructions)
__device__ __forceinline__ long floor_div(long a, long b) {
  long q = (long)((double)a / (double)b);
  const long r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

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

// room of a sequence's first r tiles
__device__ __forceinline__ long tiles_room(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, long r) {
  if (sh.whole) return r;
  const long first = max(s.N - s.n, 0) + sh.tile_cost, tpt = sh.tpt;
  if (a.window == 0) return r * first + tpt * (r * (r + 1) / 2);
  const long cap = min((long)a.window, (long)a.max_seq_len) + tpt + sh.tile_cost;   // where the window cuts a tile's keys
  const long grow = cap > first ? min(r, floor_div(cap - first - 1, tpt)) : 0;           // tiles that it does not cut
  return grow * first + tpt * (grow * (grow + 1) / 2) + (r - grow) * cap;
}

// The i-th tile of a sequence in the line, and the room of the first i.
__device__ __forceinline__ int tile_at(const SeqShape& s, int i) { return (i & 1) != 0 ? s.tiles - 1 - (i >> 1) : i >> 1; }
__device__ __forceinline__ long line_room(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int i) {
  return tiles_room(a, sh, s, (i + 1) >> 1) + tiles_room(a, sh, s, s.tiles) - tiles_room(a, sh, s, s.tiles - (i >> 1));
}

// keys that a tile's rows see, in units of KT keys from u0 on; at least one unit, though it may hold no visible key
struct TileKeys { int first, end, u0, units; };
template <int KT>
__device__ __forceinline__ TileKeys tile_keys(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int r) {
  TileKeys k;
  const int c0 = r * sh.tpt, c1 = min(c0 + sh.tpt, s.n) - 1;
  k.end = max(s.N - s.n + c1 + 1, 0);
  k.first = a.window > 0 ? max(s.N - s.n + c0 - a.window + 1, 0) : 0;
  k.u0 = (int)((uint32_t)k.first / KT);
  k.units = max((int)(((uint32_t)k.end + KT - 1) / KT) - k.u0, 1);
  return k;
}

struct SharePlace { int kvh, b, i, u; };       // i: the tile's turn in its sequence

// All threads of the workgroup (NT of them): begin and end of this workgroup's share, in scalar registers.
struct ShareScratch { long sums[4], y[2]; int kvh[2], b[2]; SharePlace place[2]; };
template <int KT, int NT>
__device__ __forceinline__ void find_share(const PagedAttnArgs& a, const ShareArgs& sh, int G, int wg, ShareScratch* lds, SharePlace* from,
                                           SharePlace* to) {
  static_assert(NT == 256, "four waves");
  // which sequences the two ends lie in: a thread has `per` neighbouring ones
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (a.B + NT - 1) / NT;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  long mine = 0;
  for (int b = b0; b < b1; ++b) {
    const SeqShape s = seq_shape(a, sh, G, b);
    mine += tiles_room(a, sh, s, s.tiles);
  }
  long upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) { const long x = __shfl_up(upto, d); if (lane >= d) upto += x; }
  if (lane == 63) lds->sums[wave] = upto;
  if (tid < 2) lds->kvh[tid] = a.H_kv;         // the end of the line; also where lengths that change under the call lead nowhere
  __syncthreads();
  long before = upto - mine, line = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { if (w < wave) before += lds->sums[w]; line += lds->sums[w]; }
  const long all = line * a.H_kv;
  const long share = sh.whole ? 1 : max((long)sh.min_keys, floor_div(all + sh.wgs - 1, sh.wgs));
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const long x = (long)(wg + e) * share;
    if (x >= all) continue;
    const int kvh = (int)floor_div(x, line);
    long y = x - kvh * line - before;
    if (y < 0 || y >= mine) continue;          // another thread's sequences
    int b = b0;
    for (; b + 1 < b1; ++b) {
      const SeqShape s = seq_shape(a, sh, G, b);
      const long room = tiles_room(a, sh, s, s.tiles);
      if (y < room) break;
      y -= room;
    }
    lds->kvh[e] = kvh; lds->b[e] = b; lds->y[e] = y;
  }
  __syncthreads();
  // where in the sequence: a wave per end, 64 tiles (or steps of tiles) at a time
  if (wave < 2) {
    SharePlace at{lds->kvh[wave], 0, 0, 0};
    if (at.kvh < a.H_kv) {
      at.b = __builtin_amdgcn_readfirstlane(lds->b[wave]);
      const long y = lds->y[wave];
      const SeqShape s = seq_shape(a, sh, G, at.b);
      int lo = 0, n = s.tiles;                 // the last tile that begins at or before y is one of lo .. lo + n - 1
      while (n > 1) {
        const int step = (n + 63) >> 6, i = lo + lane * step;
        const uint64_t past = __builtin_amdgcn_ballot_w64(lane * step >= n || line_room(a, sh, s, i) > y);   // the first lane's tile begins before it
        const int k = (past == 0 ? 64 : __builtin_ctzll(past)) - 1;
        n = min(step, n - k * step);
        lo += k * step;
      }
      const long begin = line_room(a, sh, s, lo), room = line_room(a, sh, s, lo + 1) - begin;
      const TileKeys k = tile_keys<KT>(a, sh, s, tile_at(s, lo));
      const int u = (int)floor_div((y - begin) * k.units, room);
      const int near = (int)min(share / (KT * 24), (long)k.units);    // a cut so near an end would cost more than it evens out
      at.i = lo; at.u = u < near ? 0 : k.units - u < near ? k.units : u;
    }
    if (lane == 0) lds->place[wave] = at;
  }
  __syncthreads();
  auto scalar = [](const SharePlace& p) {
    return SharePlace{__builtin_amdgcn_readfirstlane(p.kvh), __builtin_amdgcn_readfirstlane(p.b), __builtin_amdgcn_readfirstlane(p.i),
                      __builtin_amdgcn_readfirstlane(p.u)};
  };
  *from = scalar(lds->place[0]); *to = scalar(lds->place[1]);
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
  int kvh = from.kvh, b = from.b, i = from.i, ua = from.u;
  if (kvh >= a.H_kv) return;
  SeqShape s = seq_shape(a, sh, G, b);
  bool again = false;
  for (;;) {
    const bool last = kvh == to.kvh && b == to.b && i == to.i;
    const int r = tile_at(s, i);
    const TileKeys k = tile_keys<KT>(a, sh, s, r);
    const int ub = last ? to.u : k.units;
    if (ub > ua) { again = fn(kvh, s, r, k, ua, ub, again); if (again) continue; }
    if (last) return;
    ua = 0;
    if (++i < s.tiles) continue;
    i = 0;
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
