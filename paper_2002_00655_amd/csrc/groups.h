// Rows grouped by the matrix that they use (group_rows): where a group's rows stand in the order, and the tiles of rows of one group.
#pragma once
#include "token_ids.h"

// What a call is given of the groups.  order: the rows, group by group, those of no group behind; offsets: groups + 1 places where they start.  Both come
// from the caller's memory, so whatever is read from them is brought into range before it is used.
struct RowGroups {
    const int32_t *order = nullptr, *offsets = nullptr;
    int32_t groups = 0;
    int32_t n = 0;                               // rows
    __device__ __forceinline__ int start(int e) const {
        const int o = offsets[e];
        return o < 0 ? 0 : o > n ? n : o;
    }
};

// The rows of one group from place `first` on, `rows` of them.  group == groups: rows of no group.
struct RowTile { int group, first, rows, start, end; };        // start, end: the group's places

// Tiles of BM places that hold rows of one group only.  Group e's tiles have the numbers from floor(start_e / BM) + e on: as ceil(c / BM) is at most
// floor((s + c) / BM) + 1 - floor(s / BM), they end before the next group's, and no tile's number has to be looked up in a sum over the groups.
// Numbers that belong to no tile have no rows.
inline int64_t row_tiles(int64_t n, int32_t groups, int BM) { return n / BM + groups + 1; }
__device__ __forceinline__ RowTile row_tile(const RowGroups &g, int tile, int BM) {
    // the last e with floor(start_e / BM) + e <= tile: the rows of no group, or what the wavefront's lanes find, 64 groups at once
    const int lane = threadIdx.x & 63, none = g.start(g.groups);
    int lo = 0, hi = g.groups - 1, s, end, c, step;
    do {
        step = (hi - lo) / 64 + 1;
        const int e = lo + lane * step;
        s = e < g.groups ? g.start(e) : none;
        const bool at = e <= hi && s / BM + e <= tile;
        c = __popcll(__ballot(at));
        c = c > 1 ? c - 1 : 0;
        lo += c * step;
        hi = hi < lo + step - 1 ? hi : lo + step - 1;
    } while (step > 1);
    RowTile t;
    if (none / BM + g.groups <= tile) {
        t.group = g.groups;
        s = none;
        end = g.n;
    } else {
        // (where the group's places start and end, the lanes have seen: another trip to memory only where it was the last one)
        t.group = __builtin_amdgcn_readfirstlane(lo);
        c = __builtin_amdgcn_readfirstlane(c);
        end = t.group + 1 == g.groups ? none : c < 63 ? __builtin_amdgcn_readlane(s, c + 1) : g.start(t.group + 1);
        s = __builtin_amdgcn_readlane(s, c);
    }
    // (a number that is none of the group's, where offsets do not rise, is not multiplied: it could pass 32 bits)
    const int turn = tile - s / BM - t.group, last = (end - s) / BM;
    t.first = s + (turn < 0 || turn > last ? 0 : turn) * BM;
    t.rows = turn < 0 || turn > last || end < t.first ? 0 : end - t.first;
    if (t.rows > BM) t.rows = BM;
    t.start = s;
    t.end = end;
    return t;
}

// group_rows.hip: the statistics of a pull of the groups' keys: those of a matrix for all (`shared` keys from `first` on, shared_keys may be 0), and for every
// group that has rows, `each` keys from first_a + group * each on and, if first_b >= 0, from first_b + group * each on
struct GroupKeys { int64_t first = 0, shared = 0, first_a = 0, first_b = -1; int32_t each = 0; };
int dpaps_route_groups(dpaps_ps *ps, int32_t worker, const RowGroups &g, const GroupKeys &k, hipStream_t st);
// group_rows.hip: what all calls check of the groups that they are given
int dpaps_row_groups(dpaps_ps *ps, const int32_t *order, const int32_t *offsets, int32_t groups, int64_t n, RowGroups *g);
bool dpaps_strides_fit(dpaps_ps *ps, int64_t a, int64_t b);      // below 2^31
