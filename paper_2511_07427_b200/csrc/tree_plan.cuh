// How dynakv_attend_tree cuts its work, shared by its kernels.
//
// A unit is one (sequence, KV head, tile of RT query rows); a query row is one (drafted token, query head of the group),
// row = token * G + head, and its work is the sequence's pages.  All units' pages form one flat list that C persistent
// CTAs share out evenly, CTA c taking [c W / C, (c + 1) W / C): every length is read on the device, so neither the host nor
// a captured graph has to know them, and a ragged batch costs what its rows cost.  A CTA walks over its segments (the
// part of a unit that lies in its range).  A unit inside one CTA is normalised and written by it; of a unit cut by range
// boundaries every CTA leaves one unnormalised record (acc, m, l): in its slot 1 if the unit begins there, else in its
// slot 0 (only the first segment of a CTA can have begun earlier).  The CTA that holds the unit's last page describes the
// unit for a second launch, which merges the records in order, so results do not depend on timing.
#pragma once

#include "common.cuh"

namespace dkv {

constexpr int TREE_MAX = 256;              // drafted tokens per sequence

struct TreeArgs {
    const void* q;                         // [n_tokens][Hq][d]
    const int* q_start;                    // [n_seqs + 1]
    const int* page_table;                 // [n_seqs][pages_per_seq]
    const int* kv_len;                     // [n_seqs]
    const unsigned long long* mask;        // [n_tokens][mask_words], NULL: a chain
    void* out;                             // [n_tokens][Hq][d]
    float* lse;                            // [n_tokens][Hq], may be NULL
    float* acc;                            // records: [CTA][2][RT][d], from the tcgen05 kernel [CTA][2][d / 4][RT][4]
    float2* ml;                            //          [CTA][2][RT] (m, l)
    int* desc;                             // [CTA][8] the cut unit that ends in the CTA
    unsigned* status;
    const unsigned char* kpool;
    const unsigned char* vpool;
    const signed char* kexp;
    const signed char* vexp;
    long long n_tokens, n_pages;
    int n_seqs, max_tree, pages_per_seq, mask_words, G, Hq, Hk;
    float scale;                           // logits are q . k * scale
};
enum { DESC_VALID = 0, DESC_FIRST = 1, DESC_Q0 = 2, DESC_T = 3, DESC_H = 4, DESC_RT = 5 };

__device__ __forceinline__ void tree_status(const TreeArgs& a, unsigned bit) {
    if (a.status) atomicOr(a.status, bit);
}

struct SeqInfo {
    int q0, T, n, pages, tiles;            // first packed token, drafted tokens, rows, pages (at least 1), row tiles
    long long work;                        // pages of all the sequence's units
};
template <int RT>
__device__ __forceinline__ SeqInfo seq_work(const TreeArgs& a, int q0, int T, int n) {
    SeqInfo s;
    s.q0 = q0; s.T = T; s.n = n;
    s.pages = max(1, (n + PAGE - 1) / PAGE);
    s.tiles = (T * a.G + RT - 1) / RT;
    s.work = (long long)s.pages * s.tiles * a.Hk;
    return s;
}
template <int RT>
__device__ __forceinline__ SeqInfo seq_info(const TreeArgs& a, int b, bool report) {
    const int q0 = a.q_start[b], q1 = a.q_start[b + 1], n = a.kv_len[b];
    long long T = (long long)q1 - q0;
    const long long rows = (long long)a.pages_per_seq * PAGE;
    const bool bad_q = q0 < 0 || T < 0 || T > a.max_tree || q1 > a.n_tokens, bad_n = n < 0 || n > rows;
    if (bad_q) {                           // what is out of range is left out
        if (q0 < 0 || T < 0) T = 0;
        T = max(0ll, min(T, min((long long)a.max_tree, a.n_tokens - q0)));
    }
    if (report && (bad_q || bad_n)) tree_status(a, DYNAKV_ST_BOUNDS);
    return seq_work<RT>(a, q0, (int)T, (int)max(0ll, min((long long)n, rows)));
}

struct Segment {
    int b, h, tile, p0, p1;                // sequence, KV head, row tile, pages [p0, p1)
    int q0, T, n;
    bool first, last;                      // holds the unit's first / last page
    long long unit_start;                  // flat index of the unit's first page
};

// The CTA's range of the flat list, and the sequence it begins in.
struct Range {
    long long x, end, base, W;
    int b, C;
};

// a * b / c for non-negative values, in 32 bits when they fit: the 64-bit division costs some hundred cycles.
__device__ __forceinline__ long long mul_div(long long a, long long b, long long c) {
    const long long p = a * b;
    return p < (1ll << 32) && c < (1ll << 32) ? (long long)((unsigned)p / (unsigned)c) : p / c;
}

// Which range of the list the CTA has.  Every thread of the block (a multiple of 32, at most 1024) calls it; sh: 48 long longs.
// Up to 32 sequences: a lane takes one each, which needs one trip to memory and no block barrier, and what the walk will
// look up is left in sh (the caller synchronises the block); more: the block scans them, and the walk loads them again.
template <int RT>
__device__ __forceinline__ Range tree_range(const TreeArgs& a, int min_pages, long long* sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, nw = nt >> 5, c = blockIdx.x;
    auto warp_scan = [&](long long x) {                    // inclusive
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
        return x;
    };
    Range r;
    r.W = 0;
    auto share = [&]() {
        r.C = (int)max(1ll, min((long long)gridDim.x, r.W / min_pages));
        r.x = c < r.C ? mul_div(c, r.W, r.C) : r.W;
        r.end = c < r.C ? mul_div(c + 1, r.W, r.C) : r.W;
    };
    if (a.n_seqs <= 32) {
        SeqInfo mine;
        mine.work = 0;
        if (lane < a.n_seqs) {
            mine = seq_info<RT>(a, lane, c == 0 && warp == 0);
            if (warp == 0) { int* to = reinterpret_cast<int*>(sh); to[lane] = mine.q0; to[32 + lane] = mine.T; to[64 + lane] = mine.n; }
        }
        const long long incl = warp_scan(mine.work);
        r.W = __shfl_sync(0xffffffffu, incl, 31);
        share();
        const unsigned has = __ballot_sync(0xffffffffu, incl - mine.work <= r.x && r.x < incl);
        r.b = has ? __ffs(has) - 1 : 0;
        r.base = __shfl_sync(0xffffffffu, incl - mine.work, r.b);
        return r;
    }
    auto scan = [&](long long v, long long& total) {       // inclusive, over the block
        const long long x = warp_scan(v);
        __syncthreads();
        if (lane == 31) sh[warp] = x;
        __syncthreads();
        long long before = 0;
        total = 0;
        for (int w = 0; w < nw; w++) { if (w < warp) before += sh[w]; total += sh[w]; }
        return x + before;
    };
    const bool one = a.n_seqs <= nt;
    long long v = 0, incl = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += nt) {
        v = b0 + tid < a.n_seqs ? seq_info<RT>(a, b0 + tid, c == 0).work : 0;
        long long total;
        incl = scan(v, total);
        r.W += total;
    }
    share();
    if (tid == 0) { sh[34] = 0; sh[35] = 0; }
    __syncthreads();
    if (r.x < r.end) {                     // uniform in the block
        long long run = 0;
        for (int b0 = 0; b0 < a.n_seqs; b0 += nt) {
            long long total = r.W;
            if (!one) {
                v = b0 + tid < a.n_seqs ? seq_info<RT>(a, b0 + tid, false).work : 0;
                incl = scan(v, total);
            }
            const long long lo = run + incl - v, hi = run + incl;
            if (lo <= r.x && r.x < hi) { sh[34] = b0 + tid; sh[35] = lo; }
            run += total;
        }
    }
    __syncthreads();
    r.b = (int)sh[34];
    r.base = sh[35];
    return r;
}

// The CTA's segments in order.
template <int RT>
struct SegmentWalk {
    Range r;
    const long long* sh;
    __device__ __forceinline__ SegmentWalk(const Range& range, const long long* shared) : r(range), sh(shared) {}
    __device__ __forceinline__ SeqInfo look(const TreeArgs& a) const {
        if (a.n_seqs > 32) return seq_info<RT>(a, r.b, false);
        const int* from = reinterpret_cast<const int*>(sh);
        return seq_work<RT>(a, from[r.b], from[32 + r.b], from[64 + r.b]);
    }
    __device__ __forceinline__ bool next(const TreeArgs& a, Segment& g) {
        if (r.x >= r.end) return false;
        SeqInfo s = look(a);
        while (r.x - r.base >= s.work) { r.base += s.work; r.b++; s = look(a); }
        const long long off = r.x - r.base;
        const long long unit = off < (1ll << 31) ? (long long)((unsigned)off / (unsigned)s.pages) : off / s.pages;
        g.p0 = (int)(off - unit * s.pages);
        g.p1 = (int)min((long long)s.pages, g.p0 + (r.end - r.x));
        g.b = r.b; g.h = (int)((unsigned)unit / (unsigned)s.tiles); g.tile = (int)(unit - (long long)g.h * s.tiles);     // heads times tiles fit 32 bits
        g.q0 = s.q0; g.T = s.T; g.n = s.n;
        g.first = g.p0 == 0; g.last = g.p1 == s.pages;
        g.unit_start = r.base + unit * s.pages;
        r.x += g.p1 - g.p0;
        return true;
    }
};

// next() as a call of its own: the walk's state stays in (local) memory between segments instead of in registers of the loops
// over pages.  Measured both ways: the tcgen05 kernel, whose softmax fills its 168 registers, gains (113 -> 111 us and 121 -> 118 us on
// trees of 16 and of 64), the mma.sync kernel loses (90 -> 95 us on one token over 4 x 32768 rows).
template <int RT>
__device__ __noinline__ bool next_segment(SegmentWalk<RT>& walk, const TreeArgs& a, Segment& g) { return walk.next(a, g); }

// The CTA whose range holds flat index x.
__device__ __forceinline__ int range_owner(long long x, long long W, int C) { return (int)(((x + 1) * C - 1) / W); }

// Called once per CTA when it has walked its range: what the second launch has to merge here.
__device__ __forceinline__ void describe_cut_unit(const TreeArgs& a, const Segment& g, const Range& r) {
    int* d = a.desc + (size_t)blockIdx.x * 8;
    d[DESC_FIRST] = range_owner(g.unit_start, r.W, r.C);
    d[DESC_Q0] = g.q0; d[DESC_T] = g.T; d[DESC_H] = g.h; d[DESC_RT] = g.tile;
}

// Which of the 32 rows of a page (first row key0) token t of the tree sees, as bits.  All rows before the tree; of the tree
// the tokens its mask names, or without a mask itself and those before it; nothing past the sequence's length.
__device__ __forceinline__ unsigned tree_window(const TreeArgs& a, const Segment& g, int t, int key0) {
    const int cnt = g.n - key0;
    if (cnt <= 0) return 0u;
    const int j0 = key0 - (g.n - g.T);          // tree index of the page's first row
    unsigned win = 0u;
    if (j0 + 31 >= 0) {
        if (a.mask) {
            const unsigned long long* m = a.mask + (size_t)(g.q0 + t) * a.mask_words;
            const int w = j0 >> 6, sh = j0 & 63;
            const unsigned long long lo = w >= 0 && w < a.mask_words ? m[w] : 0ull, hi = w + 1 >= 0 && w + 1 < a.mask_words ? m[w + 1] : 0ull;
            win = (unsigned)((lo >> sh) | (sh ? hi << (64 - sh) : 0ull));
        } else {
            const int vis = t - j0 + 1;
            win = vis >= 32 ? ~0u : vis <= 0 ? 0u : (1u << vis) - 1u;
        }
    }
    if (j0 < 0) win |= j0 <= -32 ? ~0u : (1u << -j0) - 1u;
    if (cnt < 32) win &= (1u << cnt) - 1u;
    return win;
}
__device__ __forceinline__ bool tree_sees(const TreeArgs& a, const Segment& g, int t, int j) {       // token j of the tree
    if (!a.mask) return j <= t;
    return (j >> 6) < a.mask_words && ((a.mask[(size_t)(g.q0 + t) * a.mask_words + (j >> 6)] >> (j & 63)) & 1ull);
}

}  // namespace dkv
