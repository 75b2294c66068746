// How the work of new tokens on a paged cache is shared out: plain integer code, compiled for the kernels and for the host, where
// the CPU tests replay every workgroup and check that each block of keys is taken exactly once, and how even the shares are.
//
// Work is a list of tiles (rows of one KV head of a sequence that see about the same keys), each with its blocks of kKeys keys.
// Laid end to end the tiles form one line; every workgroup takes an equal stretch of it, whatever tiles lie there, so that a
// long tile is shared by many and short ones are taken many at a time.  A block counts what it takes, `each` of its tile, and a tile
// start_cost besides, what it takes to begin and end one.  Ends of stretches that lie closer than kLeast blocks to an end of their tile
// move there.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define L2A_PLAN_FN __host__ __device__ inline __attribute__((always_inline))
#else
#define L2A_PLAN_FN inline
#endif

namespace l2a {
namespace plan {

constexpr int kKeys = 64;   // keys of a block
constexpr int kLeast = 2;   // blocks of a piece

// A sequence of the call: new tokens start .. start + n - 1 of the packed ones, at positions pos .. pos + n - 1.  Device data that is
// out of range is clamped: any values give rows inside the tensors and positions inside the table.
struct Seq {
    int start, n, pos;
};
L2A_PLAN_FN int clamp(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
L2A_PLAN_FN Seq make_seq(int start, int end, int pos, int tokens, int max_new, int capacity) {
    Seq s;
    s.start = clamp(start, 0, tokens);
    const int most = max_new < capacity ? max_new : capacity;
    const int room = tokens - s.start < most ? tokens - s.start : most;
    const long long n = (long long)end - s.start;
    s.n = n < 0 ? 0 : n > room ? room : (int)n;
    s.pos = clamp(pos, 0, capacity - s.n);
    return s;
}

// The keys a row at position t takes part in with, by the kind of its tile: the window's, or those before it.  W = -1: there is
// no window, all keys are before it.
enum { kWindow = 0, kPrefix = 1 };
struct Range {
    int lo, hi;
};
L2A_PLAN_FN Range row_keys(int kind, int t, int W) {
    if (kind == kWindow) return Range{t - W > 0 ? t - W : 0, t};
    return Range{0, t - W - 1};
}
// The keys of a tile whose first and last rows are at t0 and t1.
L2A_PLAN_FN Range tile_keys(int kind, int t0, int t1, int W) { return Range{row_keys(kind, t0, W).lo, row_keys(kind, t1, W).hi}; }
L2A_PLAN_FN int tile_blocks(const Range& k) { return k.hi < k.lo ? 0 : k.hi / kKeys - k.lo / kKeys + 1; }
// Rows of a sequence before the first one with keys before the window.
L2A_PLAN_FN int rows_without_prefix(const Seq& s, int G, int W) { return clamp(W + 1 - s.pos, 0, s.n) * G; }

// What a block takes, in quarters of a microsecond, and what a tile does besides.  Measured, us: 2.1 a block of many rows and 2.35 in e4m3, 1.15 and
// 1.55 of up to 128, 0.75 and 0.5 of few, which wait for their loads; 7.5 a tile.  (In calls of few rows alone the
// waits of one workgroup are time for another's loads, and a tile counts half as much.)
constexpr int kFewRows = 32, kManyRows = 128;
L2A_PLAN_FN int block_cost(int rows, bool fp8) { return rows <= kFewRows ? (fp8 ? 2 : 3) : rows <= kManyRows ? (fp8 ? 6 : 5) : fp8 ? 9 : 8; }
L2A_PLAN_FN int start_cost(int each) { return each <= 3 ? 16 : 30; }

// Tiles of keys before the window all begin at key 0.  Where those of many rows are longer than a stretch, segments of its length, rounded up to whole
// blocks, are cut off their beginnings, as many for each such tile of a KV head as its first and shortest has, so that a block remains; each is the
// work of one workgroup.  The same segments of all tiles lie side by side, for workgroups on one XCD, which then read the same keys at the same time.
// What remains of the tiles is the line, for the workgroups that remain.  There are some, and their stretches are no longer than `per` was: a line no
// longer than 256 per, less s segments none of which is shorter than per, is no longer than (256 - s) per, and it is not empty.
// (Rounded down, segments left more of the line than the remaining workgroups' share: 128 tokens of 28 / 4 heads behind 64K, window 512,
// 20 % routed, were 252 segments and four stretches 3.7 times as long as the others' work: 174 us for 98.  313 of 12 / 1 heads behind 17548, all
// routed: 427 for 77.)
constexpr int kSegmentLeast = 16;  // blocks
L2A_PLAN_FN int segment_blocks(int per, int dearest) {  // 0: none are cut
    const int x = (per + dearest - 1) / dearest;
    return x >= kSegmentLeast ? x : 0;
}
L2A_PLAN_FN int segments(int blocks, int segment) { return blocks > 0 && segment > 0 ? (blocks - 1) / segment : 0; }
L2A_PLAN_FN int many_tiles(int rows, int tile_rows) { return rows / tile_rows + (rows % tile_rows > kManyRows ? 1 : 0); }
// The workgroup of segment k of the j-th of a KV head's `of` tiles that have some.
L2A_PLAN_FN int segment_workgroup(int first_segment, int of, int k, int j) { return first_segment + k * of + j; }

// A tile's place in the line.
struct Place {
    long long start;
    int blocks, each;
    L2A_PLAN_FN int length() const { return start_cost(each) + blocks * each; }
    L2A_PLAN_FN long long end() const { return start + length(); }
    // ends of stretches before `begun` move to the tile's beginning, those behind it from `ended` on to its end
    L2A_PLAN_FN int begun() const { return clamp(start_cost(each) + kLeast * each, 0, length()); }
    L2A_PLAN_FN int ended() const {
        const int x = start_cost(each) + (blocks - kLeast + 1) * each;
        return clamp(x, begun(), length());
    }
};
// The stretch of workgroup w: [w per, (w + 1) per).  No shorter than the dearest block, so that no two ends of stretches fall on the same block.
L2A_PLAN_FN int stretch(long long total, int workgroups, int dearest) {
    const int per = (int)((total + workgroups - 1) / workgroups);
    return per > dearest ? per : dearest;
}
// The workgroup in whose stretch x lies.  (A division of 64 bits takes the GPU several times as long as one of 32.)
L2A_PLAN_FN int workgroup_at(long long x, int per) { return (x >> 31) == 0 ? (int)x / per : (int)(x / per); }
// The stretch's end x, in the tile it lies in, moved: how many blocks from the tile's beginning.
L2A_PLAN_FN int moved(const Place& t, long long x) {
    const int at = (int)(x - t.start);
    return at < t.begun() ? 0 : at >= t.ended() ? t.blocks : (at - start_cost(t.each)) / t.each;
}
// Workgroup w's blocks of a tile [from, to), none: from == to.  The tile must overlap its stretch.
struct Piece {
    int from, to;
    int first, last;  // whether it holds the tile's first and last block
};
L2A_PLAN_FN Piece piece(const Place& t, int per, int w) {
    const long long x0 = (long long)w * per, x1 = x0 + per;
    Piece p;
    p.from = x0 <= t.start ? 0 : moved(t, x0), p.to = x1 >= t.end() ? t.blocks : moved(t, x1);
    p.first = p.from == 0, p.last = p.to == t.blocks;
    if (p.from >= p.to) p.from = p.to = 0;
    return p;
}
// The workgroups that have pieces of a tile, from first_of to last_of.
L2A_PLAN_FN int first_of(const Place& t, int per) { return workgroup_at(t.start + t.begun() - 1, per); }
L2A_PLAN_FN int last_of(const Place& t, int per) { return workgroup_at(t.start + t.ended() - 1, per); }
// Where a piece that is not the whole tile leaves its sums: every workgroup has a place for a tile that it does not begin and
// one for a tile that it does not end.
L2A_PLAN_FN int slot(int w, int first) { return 2 * w + (first ? 1 : 0); }
// The pieces whose sums a tile's rows have: its segments, then those of its stretch of the line.
struct Pieces {
    int segments, first_segment, of;  // segment k: workgroup first_segment + k of
    int first, last, line;            // workgroups on the line, of which the first is workgroup number `line`
    L2A_PLAN_FN bool whole() const { return first >= last; }
    L2A_PLAN_FN int count() const { return segments + (whole() ? 1 : last - first + 1); }
    L2A_PLAN_FN bool in_parts(int i) const { return i >= segments && whole(); }  // the i-th: no slot, every row has a place for it
    L2A_PLAN_FN int slot_of(int i) const {
        const int k = i - segments;
        return i < segments ? slot(segment_workgroup(first_segment, of, i, 0), 0) : slot(line + first + k, k == 0);
    }
};
L2A_PLAN_FN Pieces pieces_of(const Place& t, int per, int line) { return Pieces{0, 0, 0, first_of(t, per), last_of(t, per), line}; }

}  // namespace plan
}  // namespace l2a
