// How dynakv_attend_chunk on tcgen05 cuts its work.
//
// A tile is 256 query rows of one sequence, row = token * G + head of the group; a unit is a tile and a KV head; its work is the
// stages of 128 rows (4 pages) between the first and the last row that one of its tokens sees.  A first launch writes down every
// tile's stages, their prefix sums and where every CTA of the main kernel begins, because that depends on lengths and ranges that only the
// device has.  All units' stages, in the order sequence, KV head, tile (so that CTAs side by side read the same rows), form one
// list that the CTAs share out evenly; a unit cut by a border leaves records that a last launch merges, as in tree_plan.cuh.
#pragma once

#include "tree_plan.cuh"

namespace dkv {

constexpr int CT_ROWS = 256, CT_KEYS = 128, CT_PAGES = CT_KEYS / PAGE;

struct ChunkTile { int seq, tile, from, stages; };
struct ChunkSeq { int q0, T, n, first; };          // first packed token, tokens, rows, first tile
struct ChunkStart { int tile, head, off, left; };  // where a CTA begins: tile, KV head, stage of the unit; stages it has in all
struct ChunkPlan {
    ChunkTile* tiles;                              // [most tiles]
    long long* before;                             // [most tiles + 1] stages of the tiles before, for one KV head
    ChunkSeq* seqs;                                // [n_seqs + 1]; of the last only `first` counts: the number of tiles
    ChunkStart* starts;                            // [CTAs]
    long long* total;                              // [2] stages of one KV head, CTAs that have work
};

struct ChunkSeg {
    int seq, h, tile, s0, s1;                      // stages [s0, s1) of the sequence
    int q0, T, n;
    bool first, last;                              // holds the unit's first / last stage
    long long unit_start;                          // flat index of the unit's first stage
};

struct ChunkWalk {
    int e, h, off, left;
    ChunkTile t;
    ChunkSeq s;
    int next_first;
    __device__ __forceinline__ void look(const ChunkPlan& p) {
        t = p.tiles[e];
        s = p.seqs[t.seq];
        next_first = p.seqs[t.seq + 1].first;
    }
    __device__ __forceinline__ void start(const ChunkPlan& p) {
        const ChunkStart c = p.starts[blockIdx.x];
        e = c.tile; h = c.head; off = c.off; left = c.left;
        if (left > 0) look(p);
    }
    __device__ __forceinline__ bool next(const TreeArgs& a, const ChunkPlan& p, ChunkSeg& g) {
        if (left <= 0) return false;
        if (off == t.stages) {                     // the next tile, or the sequence's next head, or the next sequence
            off = 0;
            e++;
            if (e == next_first && h + 1 < a.Hk) { h++; e = s.first; }
            else if (e == next_first) h = 0;
            look(p);
        }
        const int here = min(left, t.stages - off);
        g.seq = t.seq; g.h = h; g.tile = t.tile;
        g.s0 = t.from + off; g.s1 = g.s0 + here;
        g.q0 = s.q0; g.T = s.T; g.n = s.n;
        g.first = off == 0; g.last = off + here == t.stages;
        if (!(g.first && g.last)) {
            const long long lead = p.before[s.first], all = p.before[next_first] - lead;
            g.unit_start = lead * a.Hk + h * all + p.before[e] - lead;
        }
        off += here; left -= here;
        return true;
    }
};

}  // namespace dkv
