// How dynakv_attend_chunk cuts the work of its kernels for many query rows.
//
// A tile is the query rows, row = token * G + head of the group, of so many consecutive tokens of one sequence: of 128 / G, or on tcgen05 of
// two streams of as many, which begin with a token's first head, so that the TMA can fetch them.  A unit is a tile and a KV head; its work
// is the stages of 64 or 128 rows between the first and the last row that one of its tokens sees.  A first launch writes down
// every tile's stages, their prefix sums and where every CTA of the main kernel begins, because that depends on lengths and ranges that
// only the device has.  All units' stages, in the order sequence, KV head, tile (so that CTAs side by side read the same
// rows), form one list that the CTAs share out evenly, a unit's beginning counted as ChunkCut::unit stages more; a unit cut by a border leaves
// records that a last launch merges, as in tree_plan.cuh.
#pragma once

#include "tree_plan.cuh"

namespace dkv {

constexpr int CT_ROWS = 256, CT_KEYS = 128, CT_PAGES = CT_KEYS / PAGE;       // rows of a tile and of a stage: tcgen05
constexpr int CF_ROWS = 128, CF_KEYS = 64;                                    // fp32 rows
// How a kernel's work is cut: tokens of a tile, rows of a stage, what a unit costs beside its stages (in stages), stages up to which a unit is not cut.
struct ChunkCut { int per, keys, unit, whole; };
constexpr int CT_UNIT_COST = 2, CT_WHOLE = 12;                                // tcgen05
// fp32 rows, whose stages are half as many rows and take longer.  In us, (1, 4) / (2, 12), as the tcgen05 kernel has it / (1, 0) / (0, 0) / (3, 0): one prompt of 2000
// tokens, 32 heads over 8 of 128, 829 / 871 / 824 / 909 / 903; 8 x 300 over 1000 567 / 651 / 567 / 579 / 621; documents 2 x 3001 789 / 890 / 788 / 881 / 900;
// 3 x 777 with prefixes, 8 heads of 64, 90 / 99 / 90 / 96 / 105; 64 x 100 205 / 206 / 207 / 240 / 208.
constexpr int CF_UNIT_COST = 1, CF_WHOLE = 4;

struct __align__(16) ChunkTile {
    int seq, tile, from, stages;                   // 2 * tile of the sequence, + 1 the last; first stage, stages
    int q0, T, n, first;                           // the sequence's first packed token, tokens, rows and first tile
};
struct __align__(16) ChunkPlace { int tile, head, off, left; };        // tile, KV head, stage of the unit; stages from there on
struct __align__(16) ChunkStart {
    ChunkPlace first, late;                        // what a CTA begins with; the end of a unit that comes last (left = 0: none)
    long long at;                                  // place of its stages in the list of all stages
};
struct ChunkPlan {
    ChunkTile* tiles;                              // [most tiles]
    long long* before;                             // [most tiles + 1] stages of the tiles before, for one KV head
    ChunkStart* starts;                            // [CTAs]
    int* first;                                    // [n_seqs + 1] first tile of every sequence
    // long chunks over FP8 rows (else NULL): where a sequence's pages lie when they are turned into bf16, and whether all find room
    int* wide_base;                                // [n_seqs] column 0's page
    int* wide_fits;                                // [1]
    long long wide_pages;                          // pages there is room for
};

__device__ __host__ __forceinline__ int tile_tokens(int G) { return 2 * (128 / G); }

struct ChunkSeg {
    int seq, h, tile, s0, s1;                      // stages [s0, s1) of the sequence
    int q0, T, n;
    int tokens;                                    // of the tile
    bool first, last;                              // holds the unit's first / last stage
    long long unit_start;                          // place of the unit's first stage in the list of all stages
};

// A CTA's segments in order, but the end of a unit that another CTA begins comes last: CTAs then begin with a unit's beginning all at once, and
// those of one KV head, which read the same rows, stay side by side.  (Cut anywhere they would be some tens of stages apart, which for sequences that L2
// does not hold means that every tile reads HBM: 4 x 512 tokens over 16384, 490 -> 454 us, with caps and one after the other 751 -> 694; documents 2 x 4001,
// where nothing is cut, 114 -> 116.)  The next tile's record is on its way while this one's is worked on.
struct ChunkWalk {
    int e, h, off, left, late;
    long long at;
    ChunkTile t, ahead;
    __device__ __forceinline__ void start(const ChunkPlan& p) {
        const ChunkStart& c = p.starts[blockIdx.x];
        e = c.first.tile; h = c.first.head; off = c.first.off; left = c.first.left; late = c.late.left; at = c.at + late;
        if (left > 0) ahead = p.tiles[e];
    }
    __device__ __forceinline__ bool next(int heads, int per, const ChunkPlan& p, ChunkSeg& g) {
        if (left <= 0) return false;
        t = ahead;
        const int here = min(left, t.stages - off);
        g.seq = t.seq; g.h = h; g.tile = t.tile >> 1;
        g.s0 = t.from + off; g.s1 = g.s0 + here;
        g.q0 = t.q0; g.T = t.T; g.n = t.n;
        g.tokens = min(per, t.T - g.tile * per);
        g.first = off == 0; g.last = off + here == t.stages;
        g.unit_start = at - off;
        at += here; left -= here; off = 0;
        if (left > 0) {                            // the next tile, or the sequence's next head, or the next sequence
            e++;
            if (t.tile & 1) {
                if (h + 1 < heads) { h++; e = t.first; }
                else h = 0;
            }
        } else if (late > 0) {
            const ChunkStart& c = p.starts[blockIdx.x];
            e = c.late.tile; h = c.late.head; off = c.late.off; left = late; at = c.at; late = 0;
        }
        if (left > 0) ahead = p.tiles[e];
        return true;
    }
};

// Host side.
int chunk_plan_launch(const TreeArgs& a, const ChunkPlan& plan, int sms, const ChunkCut& cut, cudaStream_t st);
// The bytes up to the end of the plan in a workspace whose first `at` are taken.
// wide_pages > 0: FP8 rows are turned into bf16.
size_t chunk_plan_space(int64_t n_tokens, int per, int n_seqs, int ctas, long long wide_pages, size_t at, char* base, ChunkPlan* plan);
// The kernels: chunk_tc.cu (bf16 and FP8 rows, tcgen05), chunk_f32.cu.
// wide: where FP8 rows are turned into bf16 first (plan.wide_pages pages, 128-byte aligned), NULL: they are not.  always: there is room for whatever the table names.
int chunk_tc_launch(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, void* wide, bool always, int sms, cudaStream_t st);
// Bytes of a page's K and V as bf16.
static inline size_t chunk_wide_page(const dynakv_row_cache* c) { return (size_t)c->n_kv_heads * PAGE * c->head_dim * 2 * 2; }
int chunk_f32_launch(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st);

}  // namespace dkv
