// Replays the whole division of a call with lists (extend_plan.hpp): the tiles of every KV head of every sequence, the segments cut off the long
// ones, the line that remains, what every workgroup does of them, and where the last kernel looks for the sums.  Every block of every tile in exactly
// one piece, every slot written once, the closed forms for a tile's pieces agreeing with the walk, and no workgroup with more than its share.
#include <cstdio>
#include <cstdint>
#include <set>
#include <vector>

#include "../paper_2603_17484_amd/csrc/extend_plan.hpp"

using namespace l2a::plan;

namespace {
struct Tile {
    int pair, kind, j, rows, blocks, skip;
    Place place(bool fp8, long long start) const { return Place{start, blocks, block_cost(rows, fp8)}; }
    long long start;
    std::vector<int> done;       // by block, counted from the tile's first key on
    std::vector<int> slots;      // of its pieces, in the order of its keys
    bool parts = false;          // a piece that is the whole tile on the line
};
struct Pair {
    int first_tile, windows, listed, segments, first_segment;
};
}  // namespace

// n, cached: of B sequences, whose rows are routed where a hash says so, in routed of 100 cases.  workgroups: of the call.
// out: segments, the longest work of a workgroup, what each would have if the line were divided evenly without segments (per).
extern "C" int segments_check(const int* n, const int* cached, int B, int Hkv, int G, int W, int routed, int fp8, int do_local, int workgroups, int* out, char* msg, int len) {
    const int tile_rows = 256;
    std::vector<Tile> tiles;
    std::vector<Pair> pairs;
    if (!do_local) W = -1;
    for (int b = 0; b < B; ++b)
        for (int hk = 0; hk < Hkv; ++hk) {
            const Seq s{0, n[b], cached[b]};
            std::vector<int> list;
            for (int code = rows_without_prefix(s, 1, W) * G; code < s.n * G; ++code) {
                const uint32_t h = (uint32_t)(code / G * 2654435761u + b * 40503u) >> 8;  // (a decision per token)
                if ((int)(h % 100) < routed) list.push_back(code);
            }
            Pair p{(int)tiles.size(), 0, (int)list.size(), 0, 0};
            auto add = [&](int kind, int first, int of, auto&& code) {
                Tile t{};
                t.pair = (int)pairs.size(), t.kind = kind, t.j = first / tile_rows, t.rows = of - first < tile_rows ? of - first : tile_rows;
                t.blocks = tile_blocks(tile_keys(kind, s.pos + code(first) / G, s.pos + code(first + t.rows - 1) / G, W));
                t.done.assign(t.blocks, 0);
                tiles.push_back(t);
            };
            if (do_local)
                for (int i = 0; i < s.n * G; i += tile_rows) add(kWindow, i, s.n * G, [](int i) { return i; }), ++p.windows;
            for (int i = 0; i < (int)list.size(); i += tile_rows) add(kPrefix, i, (int)list.size(), [&](int i) { return list[i]; });
            pairs.push_back(p);
        }
    long long line = 0;
    auto lay = [&] {
        line = 0;
        for (Tile& t : tiles) t.start = line, line = t.place(fp8, line).end();
    };
    lay();
    if (tiles.empty()) return 0;
    const int dearest = block_cost(tile_rows, fp8);
    const int whole = stretch(line, workgroups, dearest);
    int per = whole, all = 0;
    const int segment = segment_blocks(per, dearest);
    std::vector<long long> load(workgroups, 0);
    std::set<int> slots;
    if (segment) {
        for (Pair& p : pairs) {
            const int of = many_tiles(p.listed, tile_rows);
            p.first_segment = all;
            if (of) p.segments = segments(tiles[p.first_tile + p.windows].blocks, segment);
            all += p.segments * of;
        }
        if (all >= workgroups) return snprintf(msg, len, "%d segments", all), 1;
        std::vector<int> taken(workgroups, 0);
        for (Tile& t : tiles) {
            const Pair& p = pairs[t.pair];
            const int of = many_tiles(p.listed, tile_rows);
            if (t.kind != kPrefix || t.j >= of || !p.segments) continue;
            t.skip = p.segments * segment;
            t.blocks -= t.skip;
            if (t.blocks < 1) return snprintf(msg, len, "a tile of %d blocks, %d of them in segments", t.blocks + t.skip, t.skip), 1;
            for (int k = 0; k < p.segments; ++k) {
                const int w = segment_workgroup(p.first_segment, of, k, t.j);
                if (w < 0 || w >= all || taken[w]++) return snprintf(msg, len, "segment of workgroup %d", w), 1;
                for (int i = k * segment; i < (k + 1) * segment; ++i) ++t.done[i];
                load[w] += segment * block_cost(t.rows, fp8);
                t.slots.push_back(slot(w, 0));
                if (!slots.insert(slot(w, 0)).second) return snprintf(msg, len, "slot of segment %d", w), 1;
            }
        }
        lay();
        per = stretch(line, workgroups - all, dearest);
    }
    size_t T = 0;
    for (int x = 0; x < workgroups - all && (long long)x * per < line; ++x) {
        const int w = all + x;
        while (tiles[T].place(fp8, tiles[T].start).end() <= (long long)x * per) ++T;
        for (size_t i = T; i < tiles.size() && tiles[i].start < (long long)(x + 1) * per; ++i) {
            Tile& t = tiles[i];
            const Place place = t.place(fp8, t.start);
            const Piece p = piece(place, per, x);
            if (p.from == p.to) continue;
            for (int j = p.from; j < p.to; ++j) ++t.done[t.skip + j];
            load[w] += (p.to - p.from) * place.each + (p.first ? start_cost(place.each) : 0);
            if (p.first && p.last) {
                t.parts = true;
            } else {
                t.slots.push_back(slot(w, p.first));
                if (!slots.insert(slot(w, p.first)).second) return snprintf(msg, len, "slot of workgroup %d", w), 1;
            }
        }
    }
    for (size_t i = 0; i < tiles.size(); ++i) {
        const Tile& t = tiles[i];
        const Pair& p = pairs[t.pair];
        for (size_t j = 0; j < t.done.size(); ++j)
            if (t.done[j] != 1) return snprintf(msg, len, "tile %zu: block %zu taken %d times", i, j, t.done[j]), 1;
        Pieces where = pieces_of(t.place(fp8, t.start), per, all);
        const int of = many_tiles(p.listed, tile_rows);
        if (t.kind == kPrefix && t.j < of) where.segments = p.segments, where.first_segment = segment_workgroup(p.first_segment, of, 0, t.j), where.of = of;
        if (where.whole() != t.parts || where.count() != (int)t.slots.size() + (t.parts ? 1 : 0)) return snprintf(msg, len, "tile %zu: pieces", i), 1;
        for (int k = 0; k < where.count(); ++k)
            if (where.in_parts(k) ? k + 1 != where.count() : where.slot_of(k) != t.slots[k]) return snprintf(msg, len, "tile %zu: piece %d", i, k), 1;
    }
    out[0] = all, out[1] = 0, out[2] = whole;
    for (long long x : load) out[1] = x > out[1] ? (int)x : out[1];
    // A segment passes `per` by less than a block.  A stretch is no longer than per, and its ends move to the ends of tiles that are near: at most the
    // tile's beginning and kLeast blocks at its front, kLeast - 1 behind.
    const int most = whole + start_cost(dearest) + (2 * kLeast - 1) * dearest;
    if (per > whole || out[1] > most) return snprintf(msg, len, "%d segments, a workgroup with %d of work; %d is even, stretches are %d", all, out[1], whole, per), 1;
    return 0;
}
