// The launch that plans dynakv_attend_chunk's work (chunk_plan.cuh).
#include "chunk_plan.cuh"
#include "tree_host.cuh"

namespace dkv {

constexpr int PLAN_THREADS = 1024, PLAN_NEAR = 2048;            // prefix sums of so many tiles are kept in shared memory as well

__global__ void __launch_bounds__(PLAN_THREADS) k_chunk_plan(const TreeArgs a, const ChunkPlan p, int ctas, long long most, const ChunkCut cut) {
    __shared__ long long sums[32];
    __shared__ long long near_s[PLAN_NEAR + 1];
    __shared__ long long at_s[PLAN_THREADS + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = cut.per, keys = cut.keys, unit = cut.unit;
    pdl_wait();
    pdl_trigger();
    auto scan = [&](long long x, long long& total) {           // inclusive, over the block
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
        __syncthreads();
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        long long w = sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += y; }
        total = __shfl_sync(0xffffffffu, w, 31);
        const long long before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
        return x + (warp ? before : 0);
    };
    // ---- sequences and their tiles; where pages lie that are turned into bf16: from the first that a token may see to the last
    long long tiles = 0, wide = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        SeqInfo s = {};
        if (b < a.n_seqs) s = seq_info<CT_ROWS, false>(a, b, true);
        int count = (s.T + per - 1) / per;
        long long total, incl = scan(count, total);
        if (tiles + total > most) {                            // ranges of q that overlap: the workspace has no room for more tiles than tokens make
            if (tiles + incl > most) { count = 0; s.T = 0; tree_status(a, DYNAKV_ST_BOUNDS); }
            incl = scan(count, total);
        }
        const int first = (int)(tiles + incl - count);
        if (b < a.n_seqs) p.first[b] = first;
        if (p.wide_base) {
            const int from = a.rows_from || a.rows_to || a.window == 0 ? 0 : max(0, s.n - s.T + 1 - a.window) / CT_KEYS * CT_PAGES, pages = count > 0 ? (s.n + PAGE - 1) / PAGE - from : 0;
            long long all;
            const long long upto = scan(pages, all);
            if (b < a.n_seqs) p.wide_base[b] = (int)min(wide + upto - pages, p.wide_pages) - from;         // (looked at only when all fit)
            wide += all;
        }
        for (unsigned left = __ballot_sync(0xffffffffu, count > 0); left; left &= left - 1) {      // few sequences have many tiles, so a warp writes a sequence's
            const int src = __ffs(left) - 1;
            const int c = __shfl_sync(0xffffffffu, count, src), f = __shfl_sync(0xffffffffu, first, src), q0 = __shfl_sync(0xffffffffu, s.q0, src),
                      T = __shfl_sync(0xffffffffu, s.T, src), n = __shfl_sync(0xffffffffu, s.n, src);
            for (int i = lane; i < c; i += 32) {
                const int from = i * per, to = min(T, from + per), place = n - T;
                int lo = n, hi = 0;
                if (!a.rows_from && !a.rows_to) {
                    lo = a.window > 0 ? max(0, place + from + 1 - a.window) : 0;
                    hi = place + to;
                }
                p.tiles[f + i] = {b0 + warp * 32 + src, 2 * i + (i == c - 1 ? 1 : 0), lo, hi, q0, T, n, f};
            }
        }
        tiles += total;
    }
    if (tid == 0) { p.first[a.n_seqs] = (int)tiles; if (p.wide_base) *p.wide_fits = wide <= p.wide_pages ? 1 : 0; }
    __syncthreads();
    // ---- stages of every tile; where the tokens' ranges have to be read, 8 lanes per tile find the first and the last row
    if (a.rows_from || a.rows_to) {
        for (int i0 = warp * 4; i0 < tiles; i0 += PLAN_THREADS / 8) {
            const int i = i0 + (lane >> 3);
            int lo = 0x7fffffff, hi = 0;
            if (i < tiles) {
                const ChunkTile t = p.tiles[i];
                const int from = (t.tile >> 1) * per, to = min(t.T, from + per);
#pragma unroll 4
                for (int x = from + (lane & 7); x < to; x += 8) {
                    int l, h;
                    chunk_sees(a, t.q0 + x, t.n - t.T + x, t.n, l, h);
                    if (l < h) { lo = min(lo, max(l, 0)); hi = max(hi, h); }
                }
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) { lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o)); hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o)); }
            if (i < tiles && (lane & 7) == 0) { p.tiles[i].from = lo; p.tiles[i].stages = hi; }
        }
        __syncthreads();
    }
    long long run = 0;
    for (int t0 = 0; t0 < tiles; t0 += PLAN_THREADS) {
        const int i = t0 + tid;
        long long mine = 0;
        if (i < tiles) {
            const int lo = p.tiles[i].from, hi = p.tiles[i].stages, from = lo < hi ? lo / keys : 0;
            mine = lo < hi ? (hi + keys - 1) / keys - from : 1;
            p.tiles[i].from = from;
            p.tiles[i].stages = (int)mine;
        }
        long long total;
        const long long incl = scan(mine, total);
        if (i < tiles) { p.before[i] = run + incl - mine; if (i < PLAN_NEAR) near_s[i] = run + incl - mine; }
        run += total;
    }
    if (tid == 0) { p.before[tiles] = run; if (tiles <= PLAN_NEAR) near_s[tiles] = run; }
    __syncthreads();
    // ---- where every CTA begins: cost x is stage x of the list in which every unit has unit stages more
    const long long* before = tiles <= PLAN_NEAR ? near_s : p.before;
    const long long W = (run + tiles * unit) * a.Hk;
    const int C = (int)max(1ll, min((long long)ctas, run * a.Hk));
    for (int c0 = 0; c0 < ctas; c0 += PLAN_THREADS) {
        // the CTA's place, and that of the one behind it
        ChunkStart st = {{0, 0, 0, 0}, {0, 0, 0, 0}, run * a.Hk};
        ChunkPlace& to = st.first;
        int rest = 0, e0 = 0, e1 = 0;                          // stages of the unit from the place on; the sequence's tiles
        const int c = c0 + tid;
        const long long x = c < C ? mul_div(c, W, C) : W;
        auto behind = [&]() {                                  // the unit behind
            to.off = 0;
            if (++to.tile == e1) {
                if (to.head + 1 < a.Hk) { to.head++; to.tile = e0; }
                else to.head = 0;
            }
        };
        if (c <= ctas && x < W) {
            auto find = [&](long long y, int lo, int hi) {     // last tile of [lo, hi) whose cost before it is <= y
                while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (before[mid] + (long long)mid * unit <= y) lo = mid; else hi = mid; }
                return lo;
            };
            const ChunkTile t = p.tiles[find(x / a.Hk, 0, (int)tiles)];
            e0 = t.first; e1 = e0 + (t.T + per - 1) / per;
            const long long lead = before[e0] + (long long)e0 * unit, all = before[e1] + (long long)e1 * unit - lead, cost = x - lead * a.Hk;
            to.head = (int)(cost / all);
            const long long y = lead + cost - to.head * all;
            to.tile = find(y, e0, e1);
            to.off = (int)max(0ll, y - before[to.tile] - (long long)(to.tile + 1) * unit);
            // a short unit is not cut where a CTA has several: two records and their merge cost more than what it adds to one side
            const int whole = (int)(before[to.tile + 1] - before[to.tile]);
            if (whole <= cut.whole && (whole + unit) * 3ll * C <= W) to.off = to.off * 2 >= whole ? whole : 0;
            st.at = before[e0] * a.Hk + to.head * (before[e1] - before[e0]) + before[to.tile] - before[e0] + to.off;
            if (to.off == whole) behind();
            else rest = whole - to.off;
        }
        at_s[tid] = st.at;
        __syncthreads();
        if (c < ctas) {
            // up to where the next one begins; the last of a batch of CTAs (more than 1024: none has been built) finds its end in the list's
            to.left = (int)((tid + 1 < PLAN_THREADS ? at_s[tid + 1] : run * a.Hk) - st.at);
            if (to.off > 0 && to.left > rest) {                // the end of a unit, and more: it comes last
                st.late = {to.tile, to.head, to.off, rest};
                to.left -= rest;
                behind();
            }
            p.starts[c] = st;
        }
        __syncthreads();
    }
}

static long long chunk_most_tiles(int64_t n_tokens, int per, int n_seqs) { return n_tokens / per + n_seqs; }

int chunk_plan_launch(const TreeArgs& a, const ChunkPlan& plan, int sms, const ChunkCut& cut, cudaStream_t st) {
    return launch_pdl(k_chunk_plan, dim3(1), dim3(PLAN_THREADS), 0, st, a, plan, sms, chunk_most_tiles(a.n_tokens, cut.per, a.n_seqs), cut) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

// The plan's part of the workspace behind the records'.
size_t chunk_plan_space(int64_t n_tokens, int per, int n_seqs, int ctas, long long wide_pages, size_t at, char* base, ChunkPlan* plan) {
    const size_t tiles = (size_t)chunk_most_tiles(n_tokens, per, n_seqs);
    auto take = [&](size_t bytes) { const size_t x = (at + 15) / 16 * 16; at = x + bytes; return base + x; };
    ChunkPlan p;
    p.tiles = reinterpret_cast<ChunkTile*>(take(tiles * sizeof(ChunkTile)));
    p.before = reinterpret_cast<long long*>(take((tiles + 1) * 8));
    p.starts = reinterpret_cast<ChunkStart*>(take((size_t)ctas * sizeof(ChunkStart)));
    p.first = reinterpret_cast<int*>(take(((size_t)n_seqs + 1) * 4));
    p.wide_base = wide_pages > 0 ? reinterpret_cast<int*>(take((size_t)n_seqs * 4)) : nullptr;
    p.wide_fits = wide_pages > 0 ? reinterpret_cast<int*>(take(4)) : nullptr;
    p.wide_pages = wide_pages;
    if (plan) *plan = p;
    return at;
}

}  // namespace dkv
