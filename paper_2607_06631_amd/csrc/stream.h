// Device-side view of a batch of sequences: which sequence a row belongs to, where
// a key lies.  Whatever the tables hold, no access leaves its operand: row and key
// ranges are clamped to the call's, page numbers to the cache's.
#pragma once
#include "common.h"
#include "kernels.h"

namespace dif {

// Rows [lo, hi) of sequence s, within the call's.
__device__ __forceinline__ void seq_rows(const KeyView& kv, int s, int* lo, int* hi) {
  *lo = min(max(kv.row_off[s], 0), kv.rows);
  *hi = min(max(kv.row_off[s + 1], *lo), kv.rows);
}

// The sequence that row `row` belongs to (ascending offsets): the last one whose rows
// begin at or before it, found by the 64 lanes together, 64 offsets a step.
__device__ __forceinline__ int seq_of_row(const KeyView& kv, int row) {
  const int lane = threadIdx.x & 63;
  int base = 0, n = kv.n_seqs;
  while (n > 64) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool before = at < n && kv.row_off[base + at] <= row;
    const int last = max((int)__popcll(__ballot(before)) - 1, 0);
    base += last * step;
    n = min(step, n - last * step);
  }
  const bool before = lane < n && kv.row_off[base + lane] <= row;
  return base + max((int)__popcll(__ballot(before)) - 1, 0);
}

// What the row at position p sees: keys below sinks and from start to end.
struct Seen {
  int start, end;
};
__host__ __device__ __forceinline__ Seen seen_by(const SeenMask& m, int p, int length) {
  if (m.block > 0 && p < 0) return {0, 0};
  // (p + block may pass 2^31)
  const int64_t e = m.block > 0 ? ((int64_t)(p / m.block) + 1) * m.block : length;
  const int end = (int)min(e, (int64_t)length);
  const int start = m.window > 0 ? (int)min(max(e - m.window, (int64_t)0), (int64_t)end) : 0;
  return {start, end};
}

// Sequence s: its rows and keys.
struct Sequence {
  int row0, rows, keys, key0;
};
__device__ __forceinline__ Sequence sequence(const KeyView& kv, int s) {
  Sequence q;
  int hi;
  seq_rows(kv, s, &q.row0, &hi);
  q.rows = hi - q.row0;
  q.key0 = 0;
  if (kv.table) {
    q.keys = min(max(kv.lengths[s], 0), kv.max_keys);
  } else {
    q.key0 = min(max(kv.key_off[s], 0), kv.max_keys);
    q.keys = min(max(kv.key_off[s + 1], q.key0), kv.max_keys) - q.key0;
  }
  return q;
}

// The key tiles, BN keys each, of rows at positions p0 to p1 of a sequence: those that hold
// keys below sinks, then those of keys from lo, the first of a window, to hi.  GAP: windows
// shorter than the blocks lie apart, and no row sees the first `gap` keys of a block.
template <int BN, bool GAP>
struct Extent {
  int lo, hi, sinks;
  int nsink, w0, ntiles;
  int block, gap;
  __host__ __device__ __forceinline__ int tile(int i) const { return i < nsink ? i : w0 + i - nsink; }
  // every key of tile i is seen by some row
  __host__ __device__ __forceinline__ bool whole(int i) const {
    const int k0 = i * BN, k1 = k0 + BN;
    const bool in = i < w0 ? k1 <= sinks : (k0 >= lo || k1 <= sinks) && k1 <= hi;
    if constexpr (GAP) {
      if (gap > 0 && in && k1 > sinks) return k0 % block >= gap && BN <= block - k0 % block;
    }
    return in;
  }
  // the key of tile i nearest to k that lies between the ends of what rows see
  __host__ __device__ __forceinline__ int nearest(int i, int k) const {
    if (i < w0) return min(k, sinks - 1);
    if (k >= sinks) k = max(k, lo);
    return min(k, hi - 1);
  }
  // some row sees key k (of one of the tiles)
  __host__ __device__ __forceinline__ bool sees(int k) const {
    bool in = k < sinks || (k >= lo && k < hi);
    if constexpr (GAP) {
      if (gap > 0) in = in && (k < sinks || k % block >= gap);
    }
    return in;
  }
  // a key that some row sees, before tile i, none of whose keys is seen by any
  __host__ __device__ __forceinline__ int before(int i) const { return i * BN - (GAP ? i * BN % block : 0) - 1; }
};
template <int BN, bool GAP>
__host__ __device__ __forceinline__ Extent<BN, GAP> extent(const SeenMask& m, int p0, int p1, int keys) {
  Extent<BN, GAP> e;
  e.block = m.block;
  e.gap = m.window > 0 && m.block > m.window ? m.block - m.window : 0;
  // (rows before the sequence's first token see nothing, or as it does; without gaps it sees key 0)
  e.lo = seen_by(m, GAP ? max(p0, 0) : p0, keys).start;
  e.hi = seen_by(m, p1, keys).end;
  e.sinks = m.window > 0 ? min(m.sinks, e.hi) : 0;
  const int end = (e.hi + BN - 1) / BN;
  e.w0 = e.lo < e.hi ? e.lo / BN : end;   // (no tiles of an empty window)
  e.nsink = min((e.sinks + BN - 1) / BN, e.w0);
  e.ntiles = e.nsink + end - e.w0;
  return e;
}

// Sums over the lanes below, this one included.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int t = __shfl_up(v, d);
    if (lane >= d) v += t;
  }
  return v;
}

// Work split.  An item is a tile of bmq rows (tokens times shared heads) of one
// sequence, for one key head.  When items are few or uneven, the key tiles of an item
// are cut into pieces of about `most` tiles, all tiles of a sequence's rows into as
// many; a second launch joins the pieces.  Every wave works the plan out for itself
// from the tables, a lane per sequence.
struct Plan {
  int most;      // key tiles of a piece (kWhole: items stay whole)
  int items;     // row tiles of all sequences
  int pieces;    // and pieces of them, for one key head
};
constexpr int kWhole = 0x7fffffff;
struct SplitRule {
  int slots;     // workgroups that run at once
  int limit;     // most pieces, all key heads together (the workspace's)
  int least;     // fewest tiles of a piece
  int cost;      // of a piece, in tiles: its start and its share of the second launch
};
struct Load {
  int tiles, keys;   // row tiles of a sequence; key tiles that its last one sees
  float mean;        // and that one sees on average (of first and last)
  Sequence sq;
};
// Row tiles of a sequence of `rows`; none where they are another launch's.
__device__ __forceinline__ int row_tiles(const KeyView& kv, int rows, int group, int bmq) {
  return rows >= kv.least_rows && rows <= kv.most_rows ? (int)(((int64_t)rows * group + bmq - 1) / bmq) : 0;
}
template <int BN>
__device__ __forceinline__ Load load_of(const KeyView& kv, const SeenMask& m, int s, int group, int bmq) {
  Load l{0, 0, 0.f, {0, 0, 0, 0}};
  if (s >= kv.n_seqs) return l;
  l.sq = sequence(kv, s);
  const int rows = l.sq.rows, keys = l.sq.keys;
  l.tiles = row_tiles(kv, rows, group, bmq);
  if (l.tiles == 0) return l;
  const int few = min(rows, (bmq + group - 1) / group);   // tokens of a row tile
  l.keys = extent<BN, false>(m, keys - few, keys - 1, keys).ntiles;
  l.mean = 0.5f * (l.keys + extent<BN, false>(m, keys - rows, keys - rows + few - 1, keys).ntiles);
  return l;
}
__device__ __forceinline__ int pieces_of(int keys, int most) { return keys > most ? (keys + most - 1) / most : 1; }
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// What a lane keeps of the sequences: its first one, or, for many that stay whole, the row
// tiles of a run of `per` (run, and with those of the lanes before, upto).
struct Sequences {
  Load first;
  int per, run, upto;
};
template <int BN>
__device__ __forceinline__ Plan make_plan(const KeyView& kv, const SeenMask& m, int group, int bmq, bool split,
                                          const SplitRule& rule, Sequences* q) {
  const int lane = threadIdx.x & 63, n = kv.n_seqs;
  q->per = 0;
  if (!split && n > 64) {
    q->per = (n + 63) / 64;
    q->run = 0;
    for (int s = lane * q->per; s < min((lane + 1) * q->per, n); ++s) {
      int lo, hi;
      seq_rows(kv, s, &lo, &hi);
      q->run += row_tiles(kv, hi - lo, group, bmq);
    }
    q->upto = wave_scan(q->run);
    const int all = __builtin_amdgcn_readlane(q->upto, 63);
    return {kWhole, all, all};
  }
  q->first = load_of<BN>(kv, m, lane, group, bmq);
  const Load& mine = q->first;
  float work = 0.f, items = 0.f, longest = 0.f;   // (counts below 2^24 where they decide)
  for (int s = lane; s < n; s += 64) {
    const Load l = s < 64 ? mine : load_of<BN>(kv, m, s, group, bmq);
    items += l.tiles;
    work += l.tiles * l.mean;
    if (l.tiles) longest = fmaxf(longest, l.keys);
  }
  Plan p;
  p.items = p.pieces = (int)wave_sum(items);
  p.most = kWhole;
  const int64_t all_items = (int64_t)p.items * kv.kv_heads;
  if (!split || all_items >= rule.limit) return p;   // (no piece more would fit)
  work = wave_sum(work) * kv.kv_heads;
  longest = wave_max(longest);
  // Two rounds and more level out by themselves, unless an item is much longer than a slot's share:
  // one cache of 131072 keys among 128 streams of 690 on average, 8 heads of 64, takes 103 us,
  // 1388 as one piece; 1200 uneven streams of one head 157 us, 209 with the candidates weighed.
  if (all_items >= 2 * rule.slots && longest * rule.slots <= 2.f * work) return p;
  // the estimate: one round ends with its longest piece, several level out but for three
  // quarters of one (that share, and a piece's cost, as measured over causal batches of 1024 to
  // 32768 tokens)
  auto estimate = [&](float count, float piece) __attribute__((always_inline)) {
    return count <= rule.slots ? piece + rule.cost : (work + count * rule.cost) / rule.slots + 0.75f * piece;
  };
  float best = estimate((float)p.items * kv.kv_heads, longest) - rule.cost;
  const int fair = max(rule.least, (int)(work / rule.slots) + 1);
  // pieces of half the fair share to three times that
  constexpr int NC = 10;
  const int eighths[NC] = {4, 8, 9, 10, 11, 12, 14, 16, 20, 24};
  float count[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) count[c] = 0.f;
  for (int s = lane; s < n; s += 64) {
    const Load l = s < 64 ? mine : load_of<BN>(kv, m, s, group, bmq);
#pragma unroll
    for (int c = 0; c < NC; ++c) count[c] += (float)l.tiles * pieces_of(l.keys, max(rule.least, (int)((int64_t)fair * eighths[c] / 8)));
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const float one = wave_sum(count[c]), all = one * kv.kv_heads;
    const int most = max(rule.least, (int)((int64_t)fair * eighths[c] / 8));
    const float e = estimate(all, (float)most);
    if (all <= rule.limit && most < longest && e < best) {
      best = e;
      p.most = most;
      p.pieces = (int)one;
    }
  }
  p.most = __builtin_amdgcn_readfirstlane(p.most);
  p.pieces = __builtin_amdgcn_readfirstlane(p.pieces);
  return p;
}

// Where piece i of the plan is.
struct Place {
  int seq, tile;       // sequence, and which of its row tiles
  int part, parts;     // which piece of how many
  Sequence sq;
};
template <int BN>
__device__ __forceinline__ Place find_place(const KeyView& kv, const SeenMask& m, int group, int bmq, const Plan& p,
                                            const Sequences& q, int i) {
  const int lane = threadIdx.x & 63, n = kv.n_seqs;
  if (q.per > 0) {   // the lane whose run holds row tile i, then the sequence in that run (of 64 at most)
    uint64_t past = __ballot(q.upto > i);
    int at = past ? __builtin_ctzll(past) : 0;
    const int s0 = at * q.per, left = i - __builtin_amdgcn_readlane(q.upto - q.run, at);
    int lo = 0, hi = 0;
    if (lane < q.per && s0 + lane < n) seq_rows(kv, s0 + lane, &lo, &hi);
    const int mine = row_tiles(kv, hi - lo, group, bmq), upto = wave_scan(mine);
    past = __ballot(upto > left);
    at = past ? __builtin_ctzll(past) : 0;
    Place r{s0 + at, left - __builtin_amdgcn_readlane(upto - mine, at), 0, 1, {}};
    const Sequence sq = sequence(kv, min(r.seq, n - 1));
    r.sq = {__builtin_amdgcn_readfirstlane(sq.row0), __builtin_amdgcn_readfirstlane(sq.rows),
            __builtin_amdgcn_readfirstlane(sq.keys), __builtin_amdgcn_readfirstlane(sq.key0)};
    return r;
  }
  int before = 0;   // pieces of the sequences passed
  for (int s0 = 0;; s0 += 64) {
    const Load l = s0 == 0 ? q.first : load_of<BN>(kv, m, s0 + lane, group, bmq);
    const int parts = p.most == kWhole ? 1 : pieces_of(l.keys, p.most);
    const int mine = l.tiles * parts, upto = wave_scan(mine);
    const uint64_t past = __ballot(before + upto > i);
    if (past || s0 + 64 >= n) {
      const int at = past ? __builtin_ctzll(past) : 0;
      Place r;
      r.seq = s0 + at;
      r.parts = __builtin_amdgcn_readlane(parts, at);
      const int local = i - before - __builtin_amdgcn_readlane(upto - mine, at);
      r.tile = local / r.parts;
      r.part = local - r.tile * r.parts;
      r.sq.row0 = __builtin_amdgcn_readlane(l.sq.row0, at);
      r.sq.rows = __builtin_amdgcn_readlane(l.sq.rows, at);
      r.sq.keys = __builtin_amdgcn_readlane(l.sq.keys, at);
      r.sq.key0 = __builtin_amdgcn_readlane(l.sq.key0, at);
      return r;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
}

// The piece (of a key head) and the head of workgroup b in the chunks' kernels; false: none.
// The heaviest row tiles of all heads come first, so that light ones even out the end
// (with heads outermost a clip of 32760 tokens under a window took 30 % longer).  From 1024 on,
// runs of up to 16 row tiles of a head go to one XCD, workgroup b running on XCD b % 8, so
// that they share its tiles in that XCD's L2.  Against the plain order, 7488 rows over 32760 keys:
// 40 heads 4.29 ms and 4.40 (packed 3.99 and 4.14), 41 heads, whose runs are uneven over the XCDs,
// 4.78 and 4.36; the clip of 12 heads 2.56 and 2.47.
__host__ __device__ __forceinline__ bool turn_of(int b, int pieces, int heads, int* i, int* h) {
  if ((int64_t)pieces * heads < 1024) {
    *i = b / heads;
    *h = b - *i * heads;
    return *i < pieces;
  }
  const int bands = (pieces + 15) / 16, size = (pieces + bands - 1) / bands;
  const int local = b / kXcds, unit = local / size * kXcds + b % kXcds;
  const int band = unit / heads;
  *h = unit - band * heads;
  *i = band * size + local % size;
  return band < bands && *i < pieces;
}
// Workgroups for `pieces` of all heads together.
inline int64_t turns(int64_t pieces, int64_t heads) {
  return pieces < 1024 ? pieces : pieces + pieces / 16 + heads + kXcds * 16;
}

// Workspace of pieces: the plan, a note on each piece, unnormalised sums [slot][row][head_dim],
// (m, l) of each row.  Slots: all pieces of a key head, head by head.
struct Note {
  int row0, rows;   // first row of the sequence; its rows times shared heads
  int r0, parts;    // the row tile's first; its pieces, 0 on all but the first of them
};
constexpr int kMostSlots = 2048;
constexpr int kNoteFloats = 64 + kMostSlots * (int)(sizeof(Note) / sizeof(float));
__device__ __forceinline__ Note* part_note(float* part, int slot) { return reinterpret_cast<Note*>(part + 64) + slot; }
__device__ __forceinline__ float* part_sums(float* part, int slot, int row, int bmq, int dh) {
  return part + kNoteFloats + ((int64_t)slot * bmq + row) * dh;
}
__device__ __forceinline__ float* part_stats(float* part, int limit, int slot, int row, int bmq, int dh) {
  return part + kNoteFloats + (int64_t)limit * bmq * dh + ((int64_t)slot * bmq + row) * 2;
}
// For the launch that joins the pieces: the plan, from the first workgroup, and each
// piece's note.
__device__ __forceinline__ void leave_plan(float* part, const Plan& p) {
  if (part && blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<Plan*>(part) = p;
}
__device__ __forceinline__ void leave_note(float* part, const Plan& p, const Place& at, int slot, int r0, int rows) {
  if (p.most != kWhole && threadIdx.x == 0)
    *part_note(part, slot) = Note{at.sq.row0, rows, r0, at.part == 0 && r0 >= 0 && r0 < rows ? at.parts : 0};
}

constexpr float kRowsSlack = 8.f;      // log2 headroom of the lazy rescale
constexpr float kNoBase = -1e38f;      // base before a row's first key: any key's score moves it
constexpr int kRowsTile = 128;         // rows of a workgroup of the chunks' kernel
constexpr int kTokensTile = 16;        // and of the single tokens'
constexpr int kTokensShort = 1024;     // most keys of a sequence in whole pieces of eight waves

// Rows and pieces of the two kernels: chunks (two workgroups a CU; a tile of 64 keys
// takes 1.5 us), single tokens (tiles of 32 keys).
constexpr SplitRule kRowsRule{512, 1024, 8, 8};
constexpr SplitRule kTokensRule{512, 1536, 8, 4};

template <typename T>
struct RowsParams {
  KeyView kv;
  const T* q;
  T* out;
  int64_t ldq, ldo;
  int heads, group;    // query heads, and how many share a key head
  SeenMask mask;
  float c;             // scores to base-2 exponents: log2(e) / sqrt(head_dim), 1 for scaled queries
  float* part;         // null: nothing is split
};

}  // namespace dif
