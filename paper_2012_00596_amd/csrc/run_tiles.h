// Which rows a workgroup has, where a call's rows are runs of new tokens of several sequences.
#pragma once
#include "device_util.h"

namespace npas {

// Tile of a workgroup: BM rows (token, query head of the key head) of one sequence.
struct RunTile {
    int s, token0, row0, rows; // sequence, its first row of q, first row of the tile and rows from there on within the run
    int at0;                   // position of the run's first token
    int length;
};
// Sequence s owns the places [start G / BM] + s .. of the grid: as many as its rows need, whatever the parting.
template <int BM, typename Args> __device__ __forceinline__ bool find_run_tile(const Args &a, int place, int group, RunTile &t)
{
    auto bounded = [&](int start) { return max(0, min(start, a.T)); };
    auto first = [&](int start, int s) { return (int)((long)start * group / BM) + s; };
    const int lane = threadIdx.x & 63;
    int begin = 0, after = 0, n = 0; // of the last sequence that begins at or before this place
    t.s = -1;
    for (int s0 = 0; s0 < a.c.sequences; s0 += 64) {
        const int s = min(s0 + lane, a.c.sequences - 1), b = bounded(a.start[s]), e = bounded(a.start[s + 1]), len = a.length[s];
        const int here = __popcll(__ballot(s0 + lane < a.c.sequences && first(b, s) <= place));
        if (here) {
            t.s = s0 + here - 1;
            begin = __builtin_amdgcn_readlane(b, here - 1);
            after = __builtin_amdgcn_readlane(e, here - 1);
            n = __builtin_amdgcn_readlane(len, here - 1);
        }
        if (here < 64) break;
    }
    if (t.s < 0) return false;
    t.token0 = begin;
    const int run = max(0, after - begin);
    t.row0 = (place - first(begin, t.s)) * BM;
    t.rows = run * group - t.row0;
    const long room = (long)a.c.table_stride * a.c.page_size;
    n = max(0, min(n, a.max_length));
    if (n > room) n = (int)room;
    t.length = n;
    t.at0 = n - run;
    return t.rows > 0 && t.row0 >= 0; // (starts that fall, which no call has, lead to places before a run's first)
}

} // namespace npas
