// How the work of new tokens on a paged cache is shared out: plain integer code, compiled for the kernels and for the host, where
// the CPU test replays every workgroup and checks that each block of keys is taken exactly once.
//
// Work is a list of tiles (rows of one KV head of a sequence that see about the same keys), each with its blocks of kKeys keys.
// Laid end to end the tiles form one line; every workgroup takes an equal stretch of it, whatever tiles lie there, so that a
// long tile is shared by many and short ones are taken many at a time.  A block counts what it takes, `each` of its tile; a tile
// counts kStart more blocks than it has, what it costs to begin and end one.  Ends of stretches that lie closer than kLeast blocks to
// an end of their tile move there.
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
constexpr int kStart = 3;   // what a tile costs besides its blocks, in blocks
constexpr int kLeast = 5;   // > kStart: a piece of a tile has at least a block

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

// What a block takes, in units of about half a microsecond: tiles of few rows wait for their loads (e4m3 half as long), those of many for the
// matrix cores.
constexpr int kFewRows = 32, kManyRows = 128;
L2A_PLAN_FN int block_cost(int rows, bool fp8) { return (rows <= kFewRows ? 1 : rows <= kManyRows ? 2 : 3) + (fp8 ? 0 : 1); }

// Tiles of keys before the window all begin at key 0.  Where those of many rows are longer than a stretch, segments of its length are cut off their
// beginnings, as many for each such tile of a KV head as its first and shortest has, so that a block remains; each is the work of one
// workgroup.  The same segments of all tiles lie side by side, for workgroups on one XCD, which then read the same keys at the same time.
// What remains of the tiles is the line, for the workgroups that remain: there are some, since every segment has a stretch's length.
constexpr int kSegmentLeast = 16;  // blocks
L2A_PLAN_FN int segments(int blocks, int segment) { return blocks > 0 && segment >= kSegmentLeast ? (blocks - 1) / segment : 0; }
L2A_PLAN_FN int many_tiles(int rows, int tile_rows) { return rows / tile_rows + (rows % tile_rows > kManyRows ? 1 : 0); }

// A tile's place in the line.
struct Place {
    long long start;
    int blocks, each;
    L2A_PLAN_FN int steps() const { return blocks + kStart; }
    L2A_PLAN_FN long long end() const { return start + (long long)steps() * each; }
};
// The stretch of workgroup w: [w per, (w + 1) per).  No shorter than the dearest block, so that no two ends of stretches fall on the same block.
L2A_PLAN_FN int stretch(long long total, int workgroups, int dearest) {
    const int per = (int)((total + workgroups - 1) / workgroups);
    return per > dearest ? per : dearest;
}
// The stretch's end x, in the tile it lies in, moved: how many steps from the tile's beginning.
L2A_PLAN_FN int moved(const Place& t, long long x) {
    const int at = (int)(x - t.start) / t.each, len = t.steps();
    if (at < kLeast) return 0;
    return len - at < kLeast ? len : at;
}
// Workgroup w's blocks of a tile [from, to), none: from == to.  The tile must overlap its stretch.
struct Piece {
    int from, to;
    int first, last;  // whether it holds the tile's first and last block
};
L2A_PLAN_FN Piece piece(const Place& t, int per, int w) {
    const long long x0 = (long long)w * per, x1 = x0 + per;
    const int a = x0 <= t.start ? 0 : moved(t, x0), b = x1 >= t.end() ? t.steps() : moved(t, x1);
    Piece p;
    p.first = a == 0, p.last = b == t.steps();
    p.from = a > kStart ? a - kStart : 0;
    p.to = b > kStart ? b - kStart : 0;
    if (a >= b) p.from = p.to = 0;
    return p;
}
// The workgroups that have pieces of a tile, from first_of to last_of: ends of stretches before `begun` move to its beginning or
// lie before it, those from `ended` on to its end or lie behind it.
L2A_PLAN_FN int first_of(const Place& t, int per) {
    const long long begun = t.start + (long long)(t.steps() < kLeast ? t.steps() : kLeast) * t.each;
    return (int)((begun - 1) / per);
}
L2A_PLAN_FN int last_of(const Place& t, int per) {
    const int n = t.steps(), b = n - kLeast + 1, c = kLeast > b ? kLeast : b, ended = c < n ? c : n;
    return (int)((t.start + (long long)ended * t.each - 1) / per);
}
// Where a piece that is not the whole tile leaves its sums: every workgroup has a place for a tile that it does not begin and
// one for a tile that it does not end.
L2A_PLAN_FN int slot(int w, int first) { return 2 * w + (first ? 1 : 0); }

}  // namespace plan
}  // namespace l2a
