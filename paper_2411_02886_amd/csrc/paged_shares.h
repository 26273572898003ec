// How the work of a dense attention call is cut into equal shares, on the device, from the lengths themselves.
//
// A tile is up to `tpt` tokens of one sequence times the query heads of one KV head: its rows share every key.  The tiles stand in
// one line -- KV head, sequence, tile -- and take as much room in it as they have keys (closed form: without a window a
// sequence's tiles grow by tpt keys from one to the next) and their start and end cost.  A sequence's tiles stand as first, last,
// second, last but one, ...: two neighbours together are as long as any other two, and the cuts of a prompt often fall between tiles.  Each
// workgroup gets an equal piece of that line.  A cut inside a tile falls between two units of KT keys (near an end of the tile it moves
// there); the tile's pieces leave partial results, which a merge launch joins.  Workgroups of one XCD get
// neighbouring pieces, so that its L2 fetches the keys of a KV head once.
// The search costs 3700 cycles (1.5 us), half of it the latency of the lengths; nothing where every tile is a workgroup's and all sequences have as many (64 new
// tokens 10.2 -> 8.5 us), little where it is a workgroup's in a packed batch.  Measured: 8192 tokens of one sequence, four tiles a workgroup, 490 us at the time; with the tiles in their natural order, nearly all of them cut, 660.
#pragma once
#include "ts_kernels.h"
#include <limits.h>

namespace ts {

// words that a workgroup leaves in the workspace about its (at most two) cut tiles, eight each
constexpr int kPieceNone = 0, kPieceGoesOn = 1, kPieceEnds = 2;

struct ShareArgs {
  int tpt;          // tokens per tile
  int more_rows, most_rows;   // sequences with more_rows < n * G <= most_rows take part
  int whole;        // a workgroup per tile, nothing is cut
  int each;         // whole: tiles of every sequence that takes part, where they have as many; or 0
  int min_keys;     // smallest share
  int tile_cost;    // keys that a tile's start and end cost
  int wgs;          // workgroups of the launch
  int32_t* desc;    // [wgs][2][4]: first row, KV head and number of tokens of the tile, kPiece*; [0]: the piece goes on from the workgroup before, [1]: it begins the tile
  float* part_o;    // [wgs][2][rows][D] not normalised
  float* part_ml;   // [wgs][2][rows][2] (reference, sum)
};

#ifdef __HIPCC__

// Rooms are whole numbers held in doubles: exact below 2^53 (lines of 10^15 keys), and the double unit has a product in one instruction where
// 64-bit integers take six.
__device__ __forceinline__ double floor_div(double a, double b) {
  const double q = floor(a / b), r = fma(-q, b, a);
  return r < 0. ? q - 1. : r >= b ? q + 1. : q;
}

struct SeqShape { int b, row0, n, N, tiles, page0; };   // sequence, first row, new tokens, length, tiles (0: takes no part), first page's place

__device__ __forceinline__ SeqShape seq_shape(const PagedAttnArgs& a, const ShareArgs& sh, int G, int b) {
  SeqShape s;
  s.b = b;
  const int r0 = a.q_indptr != nullptr ? min(max(a.q_indptr[b], 0), a.T) : b * a.C;
  const int r1 = a.q_indptr != nullptr ? min(max(a.q_indptr[b + 1], 0), a.T) : r0 + a.C;
  s.page0 = a.page_indptr[b];
  s.row0 = r0;
  s.n = max(r1 - r0, 0);
  s.N = min(max(a.seq_lens[b], 0), a.max_seq_len);
  const long rows = (long)s.n * G;
  s.tiles = rows > sh.more_rows && rows <= sh.most_rows ? (int)((uint32_t)(s.n + sh.tpt - 1) / (uint32_t)sh.tpt) : 0;
  return s;
}

// room of a sequence's first r tiles
__device__ __forceinline__ double tiles_room(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int tiles) {
  const double r = tiles;
  const double first = max(s.N - s.n, 0) + sh.tile_cost, tpt = sh.tpt;
  if (a.window == 0) return fma(r, first, tpt * (r * (r + 1.) * 0.5));
  const double cap = (double)a.window + tpt + sh.tile_cost;                     // where the window cuts a tile's keys
  const double grow = cap > first ? fmin(r, floor_div(cap - first - 1., tpt)) : 0.;   // tiles that it does not cut
  return fma(grow, first, tpt * (grow * (grow + 1.) * 0.5)) + (r - grow) * cap;
}

// The i-th tile of a sequence in the line, and the room of the first i.
__device__ __forceinline__ int tile_at(const SeqShape& s, int i) { return (i & 1) != 0 ? s.tiles - 1 - (i >> 1) : i >> 1; }
__device__ __forceinline__ double line_room(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int i) {
  return tiles_room(a, sh, s, (i + 1) >> 1) + (tiles_room(a, sh, s, s.tiles) - tiles_room(a, sh, s, s.tiles - (i >> 1)));
}

// keys that a tile's rows see, in units of KT keys from u0 on; at least one unit, though it may hold no visible key
struct TileKeys { int first, end, u0, units; };
template <int KT>
__device__ __forceinline__ TileKeys tile_keys(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& s, int r) {
  TileKeys k;
  const int c0 = r * sh.tpt, c1 = min(c0 + sh.tpt, s.n) - 1;
  k.end = max(s.N - s.n + c1 + 1, 0);
  k.first = a.window > 0 ? (int)max((long)s.N - s.n + c0 - a.window + 1, 0l) : 0;
  k.u0 = (int)((uint32_t)k.first / KT);
  k.units = max((int)(((uint32_t)k.end + KT - 1) / KT) - k.u0, 1);
  return k;
}

struct SharePlace { int kvh, b, i, u; };       // i: the tile's turn in its sequence

// The tile of a sequence that place y of its part of the line lies in, and the unit: by 32 or 64 lanes that have the same q and y (`first`:
// the lowest of them, `many` of them), a step of tiles per lane and turn.
template <int KT>
__device__ __forceinline__ void find_unit(const PagedAttnArgs& a, const ShareArgs& sh, const SeqShape& q, double y, double share, int first, int many,
                                          int* tile, int* unit) {
  const int lane = (threadIdx.x & 63) - first;
  int lo = 0, n = q.tiles;                     // the last tile that begins at or before y is one of lo .. lo + n - 1
  while (__builtin_amdgcn_ballot_w64(n > 1) != 0) {
    const int step = (n + many - 1) / many;
    uint64_t past = __builtin_amdgcn_ballot_w64(lane * step >= n || line_room(a, sh, q, min(lo + lane * step, q.tiles)) > y) >> first;
    past = (many == 32 ? past & 0xffffffffull : past) & ~1ull;
    const int k = (past == 0 ? many : __builtin_ctzll(past)) - 1;
    n = min(step, n - k * step);
    lo += k * step;
  }
  const double begin = line_room(a, sh, q, lo), room = line_room(a, sh, q, lo + 1) - begin;
  const TileKeys k = tile_keys<KT>(a, sh, q, tile_at(q, lo));
  const int u = max((int)fmin(floor_div((y - begin) * k.units, room), (double)k.units), 0);
  const int near = (int)fmin(share * (1. / (KT * 24)), (double)k.units);   // a cut so near an end would cost more than it evens out
  *tile = lo;
  *unit = u < near ? 0 : k.units - u < near ? k.units : u;
}

// Begin and end of this workgroup's share, in scalar registers, and the sequence that it begins in.  Called by all threads of the workgroup (256).
struct ShareScratch { double sums[4], y[2]; int kvh[2]; SeqShape shape[2]; SharePlace place[2]; };
template <int KT>
__device__ __forceinline__ void find_share(const PagedAttnArgs& a, const ShareArgs& sh, int G, int wg, ShareScratch* lds, SharePlace* from,
                                           SharePlace* to, SeqShape* first) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (sh.whole && sh.each > 0) {                           // no search
    const uint32_t at = (uint32_t)wg / (uint32_t)sh.each;
    const int b = (int)(at % (uint32_t)a.B), i = (int)((uint32_t)wg - at * (uint32_t)sh.each);
    *first = seq_shape(a, sh, G, b);
    *from = SharePlace{i < first->tiles ? (int)(at / (uint32_t)a.B) : a.H_kv, b, i, 0};
    *to = SharePlace{from->kvh, b, i, INT_MAX};
    return;
  }
  if (sh.whole) {
    // Sequence b has the tiles from (its first row) / tpt + b on: more places than tiles, but one that is found in a search by every wave for itself, 64
    // sequences at a time.  (In the line below each of the workgroups would add up all sequences: 4096 of 100 keys 2159 us.)
    const int each = sh.wgs / a.H_kv, kvh = wg / each, at = wg - kvh * each;
    auto begin_of = [&](int b) -> int { return (int)((uint32_t)min(max(a.q_indptr[b], 0), a.T) / (uint32_t)sh.tpt) + b; };
    *from = *to = SharePlace{a.H_kv, 0, 0, 0};             // nothing, unless a sequence is found
    for (int lo = 0, n = a.B;;) {                          // of the places lo .. lo + n - 1 those that begin at or before `at` come first
      const int step = (n + 63) >> 6, i = lane * step, begin = i < n ? begin_of(lo + i) : INT_MAX;
      const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && begin <= at));
      if (k == 0) return;
      if (step == 1) {
        const int b = lo + k - 1, turn = at - __builtin_amdgcn_readlane(begin, k - 1);
        *first = seq_shape(a, sh, G, b);
        if (turn < first->tiles) { *from = SharePlace{kvh, b, turn, 0}; *to = SharePlace{kvh, b, turn, INT_MAX}; }
        return;
      }
      lo += (k - 1) * step;
      n = min(step, n - (k - 1) * step);
    }
  }
  auto share_of_line = [&](double all) { return fmax((double)sh.min_keys, floor_div(all + (sh.wgs - 1), sh.wgs)); };
  if (a.B <= 64) {
    // a lane per sequence, every wave for itself, both ends at once in the halves of the wave: no barrier, and half the time
    SeqShape s{0, 0, 0, 0, 0, 0};
    if (lane < a.B) s = seq_shape(a, sh, G, lane);
    const double mine = tiles_room(a, sh, s, s.tiles);
    double upto = mine;
    for (int d = 1; d < a.B; d <<= 1) {
      const double x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    const double line = __shfl(upto, a.B - 1), all = line * a.H_kv, share = share_of_line(all);
    const int e = lane >> 5;                   // the end that this lane works on
    const double x = (wg + e) * share;
    const bool there = x < all;
    const double kvh = there ? floor_div(x, line) : a.H_kv, y = fma(-kvh, line, x);
    // its sequence: the first whose part of the line ends behind y
    const uint64_t behind[2] = {__builtin_amdgcn_ballot_w64(upto > __shfl(y, 0)), __builtin_amdgcn_ballot_w64(upto > __shfl(y, 32))};
    const int own = min((e == 0 ? behind[0] : behind[1]) != 0 ? __builtin_ctzll(e == 0 ? behind[0] : behind[1]) : 0, a.B - 1);
    const int own_tiles = __shfl(s.tiles, own);         // (by all lanes: one that takes no part gives nothing)
    const SeqShape q{own, __shfl(s.row0, own), __shfl(s.n, own), __shfl(s.N, own), there ? own_tiles : 0, __shfl(s.page0, own)};
    int tile = 0, unit = 0;
    find_unit<KT>(a, sh, q, y - __shfl(upto - mine, own), share, e * 32, 32, &tile, &unit);
    auto at = [](int x, int l) { return __builtin_amdgcn_readlane(x, l); };
    const int kv = (int)kvh;
    *from = SharePlace{at(kv, 0), at(own, 0), at(tile, 0), at(unit, 0)};
    *to = SharePlace{at(kv, 32), at(own, 32), at(tile, 32), at(unit, 32)};
    *first = SeqShape{at(q.b, 0), at(q.row0, 0), at(q.n, 0), at(q.N, 0), at(q.tiles, 0), at(q.page0, 0)};
    return;
  }
  // which sequences the two ends lie in: a thread has `per` neighbouring ones
  const int per = (a.B + 255) >> 8, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  SeqShape s{0, 0, 0, 0, 0, 0};
  double mine = 0.;
  for (int b = b0; b < b1; ++b) {
    s = seq_shape(a, sh, G, b);
    mine += tiles_room(a, sh, s, s.tiles);
  }
  double upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) { const double x = __shfl_up(upto, d); if (lane >= d) upto += x; }
  if (lane == 63) lds->sums[wave] = upto;
  if (tid < 2) lds->kvh[tid] = a.H_kv;         // the end of the line; also where lengths that change under the call lead nowhere
  __syncthreads();
  double before = upto - mine, line = 0.;
#pragma unroll
  for (int w = 0; w < 4; ++w) { if (w < wave) before += lds->sums[w]; line += lds->sums[w]; }
  const double all = line * a.H_kv, share = share_of_line(all);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const double x = (wg + e) * share;
    if (!(x < all)) continue;
    const double kvh = floor_div(x, line);
    double y = fma(-kvh, line, x) - before;
    if (!(y >= 0. && y < mine)) continue;      // another thread's sequences
    for (int b = b0; b + 1 < b1; ++b) {
      s = seq_shape(a, sh, G, b);
      const double room = tiles_room(a, sh, s, s.tiles);
      if (y < room) break;
      y -= room;
      s = seq_shape(a, sh, G, b + 1);
    }
    lds->kvh[e] = (int)kvh; lds->shape[e] = s; lds->y[e] = y;
  }
  __syncthreads();
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto shape_of = [&](int e) {
    const SeqShape& x = lds->shape[e];
    return SeqShape{scalar(x.b), scalar(x.row0), scalar(x.n), scalar(x.N), scalar(x.tiles), scalar(x.page0)};
  };
  if (wave < 2) {                              // a wave per end
    SharePlace at{scalar(lds->kvh[wave]), 0, 0, 0};
    if (at.kvh < a.H_kv) {
      const SeqShape q = shape_of(wave);
      at.b = q.b;
      find_unit<KT>(a, sh, q, lds->y[wave], share, 0, 64, &at.i, &at.u);
    }
    if (lane == 0) lds->place[wave] = at;
  }
  __syncthreads();
  auto place_of = [&](int e) { const SharePlace& p = lds->place[e]; return SharePlace{scalar(p.kvh), scalar(p.b), scalar(p.i), scalar(p.u)}; };
  *from = place_of(0); *to = place_of(1);
  *first = shape_of(0);
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
__device__ __forceinline__ void walk_share(const PagedAttnArgs& a, const ShareArgs& sh, int G, const SharePlace& from, const SharePlace& to, SeqShape s, F&& fn) {
  int kvh = from.kvh, b = from.b, i = from.i, ua = from.u;
  if (kvh >= a.H_kv) return;
  bool again = false;
  for (;;) {
    const bool last = kvh == to.kvh && b == to.b && i == to.i;
    const int r = tile_at(s, i);
    const TileKeys k = tile_keys<KT>(a, sh, s, r);
    const int ub = last ? min(to.u, k.units) : k.units;
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
