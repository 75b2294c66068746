// Replays the division of work of extend_plan.hpp: every block of every tile in exactly one workgroup's piece, pieces in the
// order of the workgroups, and the closed forms for a tile's workgroups and the slots agreeing with the walk.
#include <cstdio>
#include <vector>

#include "../paper_2603_17484_amd/csrc/extend_plan.hpp"

using namespace l2a::plan;

extern "C" int plan_check(const int* blocks, const int* each, int tiles, int workgroups, char* msg, int n) {
    std::vector<Place> at;
    long long total = 0;
    for (int i = 0; i < tiles; ++i) {
        at.push_back(Place{total, blocks[i], each[i]});
        total = at.back().end();
    }
    int dearest = 1;
    for (int i = 0; i < tiles; ++i) dearest = each[i] > dearest ? each[i] : dearest;
    const int per = stretch(total, workgroups, dearest);
    std::vector<int> done(tiles, 0), first(tiles, -1), last(tiles, -1);
    std::vector<int> used(2 * workgroups, 0);
    int T = 0;
    for (int w = 0; w < workgroups; ++w) {
        if ((long long)w * per >= total) break;
        while (at[T].end() <= (long long)w * per) ++T;  // the tile the stretch begins in
        for (int t = T; t < tiles && at[t].start < (long long)(w + 1) * per; ++t) {
            const Piece p = piece(at[t], per, w);
            if (p.from == p.to) continue;
            if (p.from != done[t]) return snprintf(msg, n, "tile %d: workgroup %d begins at %d, %d were done", t, w, p.from, done[t]), 1;
            if (p.to <= p.from || p.to > blocks[t]) return snprintf(msg, n, "tile %d: piece %d..%d", t, p.from, p.to), 1;
            if ((p.from == 0) != (p.first != 0) || (p.to == blocks[t]) != (p.last != 0)) return snprintf(msg, n, "tile %d: flags of %d..%d", t, p.from, p.to), 1;
            if (first[t] < 0) first[t] = w;
            else if (last[t] != w - 1) return snprintf(msg, n, "tile %d: nothing from workgroup %d", t, w - 1), 1;
            last[t] = w;
            done[t] = p.to;
            if (!(p.first && p.last) && used[slot(w, p.first)]++) return snprintf(msg, n, "slot of workgroup %d used twice", w), 1;
        }
    }
    for (int t = 0; t < tiles; ++t) {
        if (done[t] != blocks[t]) return snprintf(msg, n, "tile %d: %d of %d blocks", t, done[t], blocks[t]), 1;
        if (first[t] != first_of(at[t], per) || last[t] != last_of(at[t], per))
            return snprintf(msg, n, "tile %d: workgroups %d..%d, closed form %d..%d", t, first[t], last[t], first_of(at[t], per), last_of(at[t], per)), 1;
    }
    return 0;
}

extern "C" int seq_check(int start, int end, int pos, int tokens, int max_new, int capacity) {
    const Seq s = make_seq(start, end, pos, tokens, max_new, capacity);
    return s.start >= 0 && s.n >= 0 && s.n <= max_new && s.start + s.n <= tokens && s.pos >= 0 && (long long)s.pos + s.n <= capacity;
}
