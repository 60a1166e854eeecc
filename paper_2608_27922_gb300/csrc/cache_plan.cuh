// The attention of chunks over the paged cache (k_cache_tc.cu): which items a call consists of and which partial
// results belong together.  Every CTA works this out for itself, a warp at a time.
#pragma once

#include "cache_internal.h"

namespace dkv {
namespace cache {
namespace chunk {

// What the lanes of a warp do together.  (The arithmetic below also compiles for the host, where a test walks the plans
// with 32 lanes of its own: host_lane, and host_warp, which takes a word of every lane and returns all 32.)
#ifndef __CUDA_ARCH__
int host_lane();
const unsigned* host_warp(unsigned mine);
#endif

__host__ __device__ __forceinline__ int lane_of() {
#ifdef __CUDA_ARCH__
  return threadIdx.x & 31;
#else
  return host_lane();
#endif
}
__host__ __device__ __forceinline__ int shfl(int x, int from) {
#ifdef __CUDA_ARCH__
  return __shfl_sync(0xffffffffu, x, from);
#else
  return (int)host_warp((unsigned)x)[from & 31];
#endif
}
__host__ __device__ __forceinline__ int shfl_up(int x, int by) {
#ifdef __CUDA_ARCH__
  return __shfl_up_sync(0xffffffffu, x, by);
#else
  const unsigned* all = host_warp((unsigned)x);
  return (int)all[host_lane() >= by ? host_lane() - by : host_lane()];
#endif
}
__host__ __device__ __forceinline__ float shfl_xor(float x, int with) {
#ifdef __CUDA_ARCH__
  return __shfl_xor_sync(0xffffffffu, x, with);
#else
  union { float f; unsigned u; } a;
  a.f = x;
  a.u = host_warp(a.u)[host_lane() ^ with];
  return a.f;
#endif
}
__host__ __device__ __forceinline__ unsigned ballot(bool x) {
#ifdef __CUDA_ARCH__
  return __ballot_sync(0xffffffffu, x);
#else
  const unsigned* all = host_warp(x);
  unsigned bits = 0;
  for (int i = 0; i < 32; ++i) bits |= all[i] << i;
  return bits;
#endif
}
__host__ __device__ __forceinline__ bool all_of(bool x) { return ballot(x) == 0xffffffffu; }
__host__ __device__ __forceinline__ int sum_of(int x) {
#ifdef __CUDA_ARCH__
  return __reduce_add_sync(0xffffffffu, x);
#else
  const unsigned* all = host_warp((unsigned)x);
  unsigned y = 0;
  for (int i = 0; i < 32; ++i) y += all[i];
  return (int)y;
#endif
}
__host__ __device__ __forceinline__ int max_of(int x) {
#ifdef __CUDA_ARCH__
  return __reduce_max_sync(0xffffffffu, x);
#else
  const unsigned* all = host_warp((unsigned)x);
  int y = x;
  for (int i = 0; i < 32; ++i) y = max(y, (int)all[i]);
  return y;
#endif
}
__host__ __device__ __forceinline__ unsigned min_of(unsigned x) {
#ifdef __CUDA_ARCH__
  return __reduce_min_sync(0xffffffffu, x);
#else
  const unsigned* all = host_warp(x);
  unsigned y = x;
  for (int i = 0; i < 32; ++i) y = min(y, all[i]);
  return y;
#endif
}
__host__ __device__ __forceinline__ int first_bit(unsigned x) {
#ifdef __CUDA_ARCH__
  return __ffs(x);
#else
  return __builtin_ffs((int)x);
#endif
}

constexpr int BQ = 128, BK = 128;        // query rows of a tile, keys of a tile
constexpr int MAX_CTAS = 152;            // persistent CTAs (the SMs of the GPU): sizes the scratch
// This many units a CTA, or more, are not cut: little is left to even out (prompts with 5.5 a CTA 257 us, cut 260; with 3
// a CTA 167 cut and 164 not, but units of one length would then go 3 rounds where 2.1 are due).
constexpr int CUT_ROUNDS = 4;
constexpr int MAX_PARTS = 4 * MAX_CTAS;  // partial results
constexpr int MAX_ITEMS = 16 * MAX_CTAS; // items of a call that cuts units
// Whole units go round the heads, last tokens first, where a sequence's keys and values are no more than this, else head
// by head, which reads them from L2.  Round the heads the last items to be handed out are the shortest ones: causal
// prompts over 98 MB (24 heads) of keys and values 233 us against 250, over 164 MB (40 heads) 441 against 478; over 490 MB
// 2,102 against 2,058.
constexpr int64_t NEAR = 192 << 20;
constexpr int MAX_CUT = 32;              // parts of one unit
constexpr int MIN_PART = 4;              // key tiles of a part, at least (256 tokens over 2,256 keys, 8 heads: with 4 27 us, 2 28, 8 32)
// What an item costs beside its key tiles, a part (which stores its outputs in 32 bits) more than that, and the joining of
// parts, in key tiles (1.6 us each at two query tiles of 128 dimensions; with 64 a tile takes about two thirds of that, and
// the same numbers are used)
constexpr int ITEM_TILES = 2, PART_TILES = 2, JOIN_TILES = 6;

struct Job {
  Pool c;
  Seqs s;
  Mask m;
  Packed o;
  int G, TQ, max_rows;
  int cut;                     // units may be cut: cache_merge follows
  int wide;                    // every output row is 32-byte aligned
  unsigned long long call;     // the call's number
  unsigned long long* count;   // [3] items taken beside each CTA's first, CTAs done, partial results: call << CHUNK_COUNT_BITS | count (see take)
  int4* plan;                  // stored_plan, for cache_merge
  int* slot;                   // [MAX_ITEMS] place of an item's partial result
  float* parts;                // [MAX_PARTS][(D + 1) * 256]
};

// One item: a unit's key tiles [i0, i1) of its list.
struct Item {
  int state;          // 1: an item, 0: no more
  int b, h, r0;       // sequence, key head, packed row of the first token
  int n, p0, len;     // tokens, position of the first, length of the sequence
  int ns, w0;         // the list: tiles 0 .. ns - 1, then w0, w0 + 1, ..
  int i0, i1, part;   // part: slot of the partial result, -1: a whole unit
};

__host__ __device__ __forceinline__ int tile_of(const Item& it, int i) { return i < it.ns ? i : it.w0 + (i - it.ns); }

// What the tokens of one query tile see, in key tiles: tile kt has a key that some row sees if
// kt < any_end and (kt >= any_lo or kt < any_sk), and every row sees all of it if
// kt < all_end and (kt >= all_lo or kt < all_sk).
struct Span {
  int n;                          // tokens with a position among them, 0: none
  int any_end, any_lo, any_sk;
  int all_end, all_lo, all_sk;
  int lo, end, sk;                // in positions: the first token's window, the last one's end and sinks
};

__host__ __device__ __forceinline__ Span span_of(const Mask& m, int tokens, int p0, int len, int g, int TQ) {
  Span s{};
  const int at = g * TQ, n = min(tokens - at, TQ), pf = p0 + at, pl = pf + n - 1;
  if (n <= 0 || pl < 0) return s;
  s.n = n;
  const int e0 = visible_end(m, max(pf, 0), len), l1 = window_first(m, visible_end(m, pl, len));
  s.end = visible_end(m, pl, len);
  s.lo = window_first(m, e0);
  s.sk = m.window ? min(m.sinks, s.end) : 0;
  s.any_end = (s.end + BK - 1) / BK;
  s.any_lo = s.lo / BK;
  s.any_sk = (s.sk + BK - 1) / BK;
  s.all_end = pf >= 0 ? e0 / BK : 0;
  s.all_lo = (l1 + BK - 1) / BK;
  s.all_sk = m.window ? m.sinks / BK : 0;
  return s;
}

__host__ __device__ __forceinline__ bool active(const Span& s, int kt) {
  return kt < s.any_end && (kt >= s.any_lo || kt < s.any_sk);
}
__host__ __device__ __forceinline__ bool all_seen(const Span& s, int kt) {
  return kt < s.all_end && (kt >= s.all_lo || kt < s.all_sk);
}

// Key tiles that one query tile of a unit sees whole and in which the other one does not: the kernel treats values that are
// not finite there as in a tile that both see partly, so that what becomes of them is no matter of who comes first.  (The
// second tile's tokens lie behind the first one's, and so do the ends of their windows: seen whole by the second, it is the
// first one's ends that cut a tile; by the first, the beginning of the second one's window and its last sinks.)
struct Edges {
  int from, to, sink;   // tiles [from, to) and sink
};
__host__ __device__ __forceinline__ Edges edges_of(const Span& other, int g) {   // other: of tile 1 - g
  if (other.n == 0) return Edges{0, 0, -1};
  if (g == 1) return Edges{other.all_end, other.any_end, -1};
  return Edges{max(other.any_lo, other.all_sk), other.all_lo,
               other.any_sk > other.all_sk && other.all_lo > other.all_sk ? other.all_sk : -1};
}
__host__ __device__ __forceinline__ bool in(const Edges& e, int kt) { return (kt >= e.from && kt < e.to) || kt == e.sink; }

// The list of a unit's key tiles: ns, w0 and how many in all; lo and end of what its rows see beside the sinks.
struct List {
  int ns, w0, n, lo, end, sk;
};
__host__ __device__ __forceinline__ List list_of(const Mask& m, int tokens, int p0, int len) {
  List l{};
  const int pl = p0 + tokens - 1;
  if (tokens <= 0 || pl < 0) return l;
  l.end = visible_end(m, pl, len);
  l.lo = window_first(m, visible_end(m, max(p0, 0), len));
  l.sk = m.window ? min(m.sinks, l.end) : 0;
  l.ns = (l.sk + BK - 1) / BK;
  l.w0 = max(l.ns, l.lo / BK);
  l.n = l.ns + max(0, (l.end + BK - 1) / BK - l.w0);
  return l;
}

// Units: sequence by sequence, key head by key head, last tokens first (where none is cut, see also NEAR and order).
// Items are the units, or, where those are few:
//   all of one length (each sequence's first and last unit are looked at): as many whole units as go round the CTAs evenly,
//   then the others in S equal parts (part s of all of them before part s + 1: those that read the same keys run side by
//   side).  A unit between the two may be a few tiles longer, where it straddles a block or its window another tile: the last
//   of its S parts takes them;
//   else: parts of C tiles of every unit that is longer; S is the sequence's, from its last unit (a head's parts s before
//   its parts s + 1), and shorter units have empty parts, which are passed over.
struct Plan {
  int units, items;
  int C;       // tiles of a part, 0: no unit is cut
  int whole;   // units of one length: how many are whole; else -1
  int S;       // units of one length: parts of each of the others
};

__host__ __device__ __forceinline__ int tiles_at(const Job& j, const Seq& q, int t) {
  const int t0 = t * 2 * j.TQ;
  return list_of(j.m, min(q.n - t0, 2 * j.TQ), q.len - q.n + t0, q.len).n;
}
__host__ __device__ __forceinline__ int parts_of(int tiles, int C) {
  return C == 0 || tiles <= C ? 1 : min((int)((unsigned)(tiles + C - 1) / (unsigned)C), MAX_CUT);
}

// A sequence with its units (of a key head) and the tiles of the first and the last one.
struct Known {
  Seq q;
  int b, nu, first, last;
};
__host__ __device__ __forceinline__ Known known(const Job& j, int b) {
  Known k{};
  k.b = b;
  if (b >= j.s.n) return k;
  k.q = seq_at(j.c, j.s, b);
  if (k.q.n == 0) return k;
  k.nu = (int)((unsigned)(k.q.n + 2 * j.TQ - 1) / (unsigned)(2 * j.TQ));
  k.first = tiles_at(j, k.q, 0);
  k.last = k.nu > 1 ? tiles_at(j, k.q, k.nu - 1) : k.first;
  return k;
}

// All lanes of one warp; mine: sequence `lane`.
__host__ __device__ __forceinline__ Plan make_plan(const Job& j, int ctas, Known& mine) {
  const int lane = lane_of();
  int units = 0, longest = 0;
  unsigned claimed = 0;  // rows of all sequences
  bool even = true;      // units of one length
  float tiles = 0.f;     // of all units, about
  mine = known(j, lane);
  for (int b = lane; b < j.s.n; b += 32) {
    const Known k = b == lane ? mine : known(j, b);
    if (k.q.n > j.max_rows) fail(j.c.status, DEV_INCONSISTENT, SITE_CHUNK);
    if (k.nu == 0) continue;
    claimed += (unsigned)k.q.n;
    units += k.nu * j.c.H;
    tiles += 0.5f * (k.first + k.last) * k.nu * j.c.H;
    even &= k.first == k.last && (longest == 0 || longest == k.last);
    longest = max(longest, k.last);
  }
  const int most = longest;
  units = sum_of(units);
  longest = max_of(longest);
  even = all_of(even && (most == 0 || most == longest));
  Plan p{units, units, 0, 0, 1};
  // (a row_start that goes back and forth: the work would be that of up to n_seq / 2 times the call's rows)
  if ((unsigned)sum_of((int)claimed) > (unsigned)j.s.rows) {
    fail(j.c.status, DEV_INCONSISTENT, SITE_ROWS);
    return Plan{0, 0, 0, 0, 1};
  }
  // (the choice below looks at every sequence in turn: many sequences are many units anyway)
  if (units == 0 || !j.cut || units >= CUT_ROUNDS * ctas || (!even && j.s.n > 64)) return p;
  // (uneven units:) no cut gains more than its joining costs
  if (!even) {
#pragma unroll
    for (int o = 16; o; o >>= 1) tiles += shfl_xor(tiles, o);
    const float least = (tiles + (float)(units * ITEM_TILES)) / ctas;
    if (fmaxf((float)(longest + ITEM_TILES), least + 0.35f * longest) <= least + 0.35f * MIN_PART + JOIN_TILES) return p;
  }
  // lane: the longest unit in S = lane + 1 parts
  const int S = lane + 1, C = (int)((unsigned)(longest + S - 1) / (unsigned)S);
  const int rounds = (int)((unsigned)units / (unsigned)ctas), rest = units - rounds * ctas;
  int length = 0;
  float est;
  bool fits;
  if (even) {
    length = rounds * ctas + rest * S;
    fits = S == 1 || (C >= MIN_PART && rest * S <= MAX_PARTS);
    est = (float)(rounds * (longest + ITEM_TILES));
    if (rest > 0)
      est += S == 1 ? (float)(longest + ITEM_TILES)
                    : (float)((rest * S + ctas - 1) / ctas) * (C + ITEM_TILES + PART_TILES) + JOIN_TILES;
  } else {
    int parts = 0, most_parts = 0;
#pragma unroll 1
    for (int b = 0; b < j.s.n; ++b) {
      Known k = mine;
      if (b >= 32) k = known(j, b);
      const int nu = shfl(k.nu, b & 31) * j.c.H, first = shfl(k.first, b & 31),
                last = shfl(k.last, b & 31);
      const int sb = parts_of(last, C), mid = parts_of((first + last + 1) / 2, C);
      length += nu * sb;                                         // with empty ones
      most_parts += sb > 1 ? nu * sb : 0;
      parts += sb == 1 ? 0 : mid > 1 ? nu * mid : nu / 2;
    }
    fits = S == 1 || (C >= MIN_PART && most_parts <= MAX_PARTS && length <= MAX_ITEMS);
    // the CTAs are busy to the end but for about a third of the longest item, and at least as long as it
    est = fmaxf((float)(C + ITEM_TILES), (tiles + (float)(units * ITEM_TILES + parts * (ITEM_TILES + PART_TILES))) / ctas + 0.35f * C) +
          (S > 1 ? JOIN_TILES : 0);
  }
  const unsigned best = min_of(fits ? ((unsigned)min((int)(est * 4.f), 1 << 24) << 6) | S : 0xffffffffu);
  const int s = best & 63;
  if (s > 1) {
    p.C = shfl(C, s - 1);
    p.items = shfl(length, s - 1);
    p.whole = even ? rounds * ctas : -1;
    p.S = s;
  }
  return p;
}

// Item (or, with C = 0, unit) i -> its sequence and place; before: items of earlier sequences.  All lanes of one warp; the
// search goes on from the 32 sequences where the last one ended (items are mostly taken in order), this lane's in k.
struct Unit {
  int b, h, t, s, S, nu, before;
  Seq q;
};
struct Cursor {
  int b0, before;
  Known k;
};
__host__ __device__ __forceinline__ Unit find_unit(const Job& j, int i, int C, Cursor& c) {
  const int lane = lane_of();
  if (i < c.before) {
    c.b0 = c.before = 0;
    c.k = known(j, lane);
  }
  for (;;) {
    const int S = parts_of(c.k.last, C), here = c.k.nu * j.c.H * S;
    int incl = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    const unsigned past = ballot(c.before + incl > i);
    if (past || c.b0 + 32 >= j.s.n) {
      const int w = past ? first_bit(past) - 1 : 31;   // (i is below the sum of all)
      Unit r;
      r.b = min(shfl(c.k.b, w), j.s.n - 1);
      r.before = c.before + shfl(incl - here, w);
      r.S = shfl(S, w);
      r.nu = max(1, shfl(c.k.nu, w));
      r.q.r0 = shfl(c.k.q.r0, w);
      r.q.n = shfl(c.k.q.n, w);
      r.q.len = shfl(c.k.q.len, w);
      const unsigned rem = (unsigned)(i - r.before);
      if (C == 0 && (int64_t)r.q.len * j.c.H * (j.c.d * 4 >> j.c.e4m3) <= NEAR) {
        const unsigned back = rem / (unsigned)j.c.H;
        r.t = max(0, r.nu - 1 - (int)back);
        r.h = (int)(rem - back * j.c.H);
        r.s = 0;
        return r;
      }
      const unsigned hs = rem / (unsigned)r.nu, h = r.S == 1 ? hs : hs / (unsigned)r.S;
      r.t = max(0, r.nu - 1 - (int)(rem - hs * r.nu));
      r.h = min((int)h, j.c.H - 1);
      r.s = (int)(hs - h * r.S);
      return r;
    }
    c.before += shfl(incl, 31);
    c.b0 += 32;
    c.k = known(j, c.b0 + lane);
  }
}

// The sequences of the 32 that the lanes hold (n of them) by the length of their first units, longest first: the last
// items are short ones (ragged prompts of three sequences 185 us for 196, 177 for 185, 257 for 262).
__host__ __device__ __forceinline__ void order(Known& k, int n) {
  const int lane = lane_of();
  int rank = 0, from = lane;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const int f = shfl(k.first, i);
    rank += f > k.first || (f == k.first && i < lane);
  }
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const int to = shfl(rank, i);
    if (to == lane) from = i;
  }
  int* const w = reinterpret_cast<int*>(&k);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(Known) / 4); ++i) w[i] = shfl(w[i], from);
}

// Item i and its list; state 0 where it is an empty part.  (Its partial result's place is taken when it is handed out.)
__host__ __device__ __forceinline__ Item make_item(const Job& j, const Plan& p, int i, Cursor& cursor, List& l) {
  // (units of one length: part s of the R that are cut)
  int unit = i, s = 0, S = 1;
  if (p.C > 0 && p.whole >= 0 && i >= p.whole) {
    const int R = p.units - p.whole, k = i - p.whole;
    s = (int)((unsigned)k / (unsigned)R);
    unit = p.whole + k - s * R;
    S = p.S;
  }
  const Unit u = find_unit(j, unit, p.whole < 0 ? p.C : 0, cursor);
  if (p.whole < 0) {
    s = u.s;
    S = u.S;
  }
  const int t0 = u.t * 2 * j.TQ;
  Item x;
  x.b = u.b;
  x.h = u.h;
  x.r0 = u.q.r0 + t0;
  x.n = min(u.q.n - t0, 2 * j.TQ);
  x.p0 = u.q.len - u.q.n + t0;
  x.len = u.q.len;
  l = list_of(j.m, x.n, x.p0, x.len);
  x.ns = l.ns;
  x.w0 = l.w0;
  S = min(S, parts_of(l.n, p.C));
  x.i0 = s * p.C;
  x.i1 = s + 1 < S ? x.i0 + p.C : l.n;
  x.part = S > 1 ? 0 : -1;
  x.state = s < S;
  return x;
}

// The plan as *j.plan holds it: units (0: none is cut), tiles of a part, whole ones (-1), parts of the others.
__host__ __device__ __forceinline__ int4 stored_plan(const Plan& p) { return make_int4(p.C > 0 ? p.units : 0, p.C, p.whole, p.S); }

// What cache_merge joins of a unit: the partial results of the items at, at + step, .. (n of them; 1: none, it is whole).
// p: stored_plan.  All lanes of one warp.
struct Joined {
  Unit u;
  int n, at, step;
};
__host__ __device__ __forceinline__ Joined joined(const Job& j, const int4& p, int unit) {
  const int lane = lane_of();
  const Known mine = known(j, lane);
  Cursor cursor{0, 0, mine};
  Joined x;
  x.u = find_unit(j, unit, 0, cursor);
  x.n = parts_of(tiles_at(j, x.u.q, x.u.t), p.y);
  if (p.z >= 0) {
    x.n = min(x.n, p.w);
    x.at = unit;
    x.step = p.x - p.z;
  } else {   // those of the sequences before it, then (head, part, unit)
    int before = 0;
    for (int b = lane; b < x.u.b; b += 32) {
      const Known k = b == lane ? mine : known(j, b);
      before += k.nu * j.c.H * parts_of(k.last, p.y);
    }
    before = sum_of(before);
    const int SB = parts_of(tiles_at(j, x.u.q, x.u.nu - 1), p.y);
    x.n = min(x.n, SB);
    x.at = before + x.u.h * SB * x.u.nu + (x.u.nu - 1 - x.u.t);
    x.step = x.u.nu;
  }
  return x;
}

// Place of item i's partial result, -1: none.  (Where a CTA gave up waiting, its items have stored no place, and what
// the uncleared scratch holds in its stead is any number.)
__host__ __device__ __forceinline__ int slot_of(const int* slot, int i) {
  if (i < 0 || i >= MAX_ITEMS) return -1;
  const int at = slot[i];
  return at >= 0 && at < MAX_PARTS ? at : -1;
}

}  // namespace chunk
}  // namespace cache
}  // namespace dkv
