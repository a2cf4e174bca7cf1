// Tree attention on the tcgen05 tensor cores: bf16 rows, tiles of 128 query rows (token, head of the group).
//
// With R query rows per KV head a bf16 row of K and V (512 bytes at d = 128) meets 4 d R flops: from a few dozen rows on the
// mma.sync kernel is bound by the legacy tensor pipe (one m16n8k16 per 8.2 cycles and scheduler), while tcgen05 keeps
// the call on the HBM side up to R = 256.
//
// One CTA per SM walks over its range of pages (tree_plan.cuh) in tiles of up to four pages (128 keys).  Even and odd tiles
// belong to two independent streams, each with its own K and V stage, logits S, running softmax and output sum O in
// tensor memory, so that one stream's softmax runs while the other's products do; the streams meet once per segment.
//   warp 0 / warp 3     TMA loads of K / of V, one 32-row panel of 128 bytes per copy, 128-byte swizzle
//   warp 1 / warp 2     tcgen05.mma of stream 0 / 1: S = Q K^T (M = 128, N = keys of the tile), then O += P V with P from
//                       tensor memory and V read with its rows as the contraction index, no transposed copy anywhere
//   warps 4-7 / 8-11    softmax of stream 0 / 1: a query row per thread
// Tensor memory (512 columns): S of the streams at 0 and 128, O at 256 and 384.  The weights replace the logits in place:
// 32 logits of a row become 16 columns of bf16 hi pairs and 16 of lo pairs (the two MMAs of the split keep fp32 weights to 2^-17;
// bf16 weights alone would add an error as large as the output's own rounding).  The softmax's reference moves only when
// the maximum has grown by 2^8, which is when O has to be rescaled.
// A K stage is free when its S is complete, a V stage when its O is: the loads wait on the MMAs' own commits.  Stages, S and
// O belong to one stream each, so no waiter can be two phases away from a barrier.  All waits are bounded.
#include <cuda.h>
#include <float.h>

#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_ops.cuh"
#include "tree_host.cuh"
#include "tree_plan.cuh"

namespace dkv {

constexpr int TT_KEYS = 128, TT_PAGES = TT_KEYS / PAGE;        // keys and pages of a tile
constexpr int TT_THREADS = 384;
constexpr float TT_LOG2E = 1.4426950408889634f, TT_LN2 = 0.6931471805599453f, TT_LAZY = 8.f;

template <int HD>
struct TcTree {
    static constexpr int panels = HD / 64;                     // 128-byte column panels of a row
    static constexpr int panel_bytes = 128 * 128;              // 128 rows of 128 bytes
    static constexpr int tile_bytes = panels * panel_bytes;
    static constexpr int smem = 5 * tile_bytes + 2 * 128 * 8 + 36 * 8 + 16 * 8 + 2 * 8 * 4 + 2 * 2 * 2 * TT_PAGES * 4 + 64;   // Q, two K, two V stages
    // kind::f16, fp32 accumulate, bf16 operands, M = 128
    static constexpr unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
    static constexpr unsigned idesc_pv = idesc | (1u << 16) | ((unsigned)(HD >> 3) << 17);      // B's contraction index is its outer one
};
enum { TB_KFULL = 0, TB_VFULL = 2, TB_SFULL = 4, TB_PFULL = 6, TB_ODONE = 8, TB_QFULL = 10, TB_DRAIN = 12, TB_COUNT = 14 };

__device__ __forceinline__ void tt_load(unsigned dst, const CUtensorMap* map, int row, int panel, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n"
                 ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(panel), "r"(bar) : "memory");
}
__device__ __forceinline__ float tt_max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void sts16(unsigned addr, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void tt_proxy_fence() { asm volatile("fence.proxy.async;\n" ::: "memory"); }

template <int HD>
__global__ void __launch_bounds__(TT_THREADS, 1) k_tree_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                           const TreeArgs a) {
    using C = TcTree<HD>;
    extern __shared__ __align__(1024) unsigned char tt_smem[];
    unsigned char* at = tt_smem + 5 * C::tile_bytes;
    float2* ml_s = reinterpret_cast<float2*>(at); at += 2 * 128 * 8;               // [stream][row] (m, l)
    long long* sh = reinterpret_cast<long long*>(at); at += 36 * 8;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(at); at += 16 * 8;
    unsigned* odd = reinterpret_cast<unsigned*>(at); at += 2 * 8 * 4;              // [segment parity][8]
    // [K, V][stream][tile parity][page]: the page was loaded.  By parity, because the next K is on its way while the softmax reads
    volatile int* meta = reinterpret_cast<volatile int*>(at); at += 2 * 2 * 2 * TT_PAGES * 4;
    volatile unsigned* s_tmem = reinterpret_cast<volatile unsigned*>(at);
    volatile int* s_abort = reinterpret_cast<volatile int*>(at + 4);
    const unsigned sQ = tc_smem_u32(tt_smem);
    auto sK = [&](int s) { return sQ + (1 + s) * C::tile_bytes; };
    auto sV = [&](int s) { return sQ + (3 + s) * C::tile_bytes; };
    auto bar = [&](int i) { return tc_smem_u32(&bars[i]); };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int i = 0; i < TB_COUNT; i++) tc_mbar_init(bar(i), 1);
        for (int s = 0; s < 2; s++) { tc_mbar_init(bar(TB_PFULL + s), 4); tc_mbar_init(bar(TB_QFULL + s), 8); }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (tid < 16) odd[tid] = 0u;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tc_smem_u32((const void*)s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    const Range range = tree_range<TREE_TC_ROWS>(a, TT_PAGES, sh);                 // holds block barriers
    tc_fence_after();
    pdl_trigger();
    const unsigned tmem = *s_tmem;
    SegmentWalk<TREE_TC_ROWS> walk(a, range);
    Segment g;
    auto give_up = [&]() { *s_abort = 1; };

    if (warp == 0 || warp == 3) {
        // =============================== loads: warp 0 K, warp 3 V ===============================
        const bool is_v = warp == 3;
        const CUtensorMap* map = is_v ? &map_v : &map_k;
        const int full = is_v ? TB_VFULL : TB_KFULL, freed = is_v ? TB_ODONE : TB_SFULL;
        int n = 0;                                             // tile number in the CTA
        bool ok = true;
        while (ok && walk.next(a, g)) {
            for (int pc = g.p0; ok && pc < g.p1; pc += 32) {
                const int cnt = min(32, g.p1 - pc);
                int id = -1;
                if (lane < cnt && g.n > 0) {
                    id = a.page_table[(size_t)g.b * a.pages_per_seq + pc + lane];
                    if (id < 0 || id >= a.n_pages) { id = -1; tree_status(a, DYNAKV_ST_BOUNDS); }
                }
                for (int j = 0; j < cnt && ok; j += TT_PAGES, n++) {
                    const int s = n & 1, i = n >> 1;
                    int page[TT_PAGES], there = 0;
#pragma unroll
                    for (int x = 0; x < TT_PAGES; x++) { page[x] = __shfl_sync(0xffffffffu, id, (j + x) & 31); if (j + x >= cnt) page[x] = -1; there += page[x] >= 0; }
                    if (lane == 0) {
                        ok = !*s_abort && (i == 0 || tc_mbar_wait(bar(freed + s), (unsigned)(i - 1) & 1u));
                        if (ok) {
#pragma unroll
                            for (int x = 0; x < TT_PAGES; x++) meta[((is_v * 2 + s) * 2 + (i & 1)) * TT_PAGES + x] = page[x] >= 0;
                            if (there) tc_mbar_expect_tx(bar(full + s), there * PAGE * HD * 2);
                            else tc_mbar_arrive(bar(full + s));
                            const unsigned dst = is_v ? sV(s) : sK(s);
#pragma unroll
                            for (int x = 0; x < TT_PAGES; x++) {
                                if (page[x] < 0) continue;
#pragma unroll
                                for (int p = 0; p < C::panels; p++)
                                    tt_load(dst + p * C::panel_bytes + x * PAGE * 128, map, (page[x] * a.Hk + g.h) * PAGE, p, bar(full + s));
                            }
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                }
            }
        }
        if (!ok && lane == 0) {
            give_up();
            // let the copies under way land before the block ends
            for (int s = 0; s < 2; s++) {
                // tile n - 1 was not issued; the stream's last one before it
                if (n - 2 >= s) tc_mbar_wait(bar(full + s), (unsigned)((n - 2 - s) >> 1) & 1u);
            }
        }
    } else if (warp == 1 || warp == 2) {
        // =============================== MMAs of one stream ===============================
        const int s = warp - 1;
        if (lane == 0) {
            int n = 0, segs = 0;                               // segments in which the stream had a tile
            bool ok = true;
            while (ok && walk.next(a, g)) {
                const int tiles = (g.p1 - g.p0 + TT_PAGES - 1) / TT_PAGES;
                bool first = true;
                for (int j = (n & 1) == s ? 0 : 1; j < tiles && ok; j += 2) {
                    const int i = (n + j) >> 1;
                    const unsigned ph = (unsigned)i & 1u;
                    if (first) ok = tc_mbar_wait(bar(TB_QFULL + s), (unsigned)segs & 1u);
                    ok = ok && !*s_abort && tc_mbar_wait(bar(TB_KFULL + s), ph);
                    if (!ok) break;
                    tc_fence_after();
                    const int pages = min(TT_PAGES, g.p1 - g.p0 - j * TT_PAGES);
                    const unsigned idesc = C::idesc | ((unsigned)(pages * PAGE >> 3) << 17);
#pragma unroll
                    for (int k = 0; k < HD / 16; k++) {
                        const unsigned off = (k >> 2) * C::panel_bytes + (k & 3) * 32;
                        tc_mma_f16(tmem + s * 128, tc_panel_desc(sQ + off), tc_panel_desc(sK(s) + off), idesc, k > 0 ? 1u : 0u);
                    }
                    tc_commit(bar(TB_SFULL + s));
                    ok = tc_mbar_wait(bar(TB_VFULL + s), ph) && tc_mbar_wait(bar(TB_PFULL + s), ph);
                    if (!ok) break;
                    tc_fence_after();
                    for (int k = 0; k < pages * 2; k++) {
                        const unsigned long long d = tc_rows_desc(sV(s) + k * 2048, C::panel_bytes);
                        const unsigned p = tmem + s * 128 + (k >> 1) * 32 + (k & 1) * 8;
                        tc_mma_f16_ta(tmem + 256 + s * 128, p, d, C::idesc_pv, !first || k > 0 ? 1u : 0u);
                        tc_mma_f16_ta(tmem + 256 + s * 128, p + 16, d, C::idesc_pv, 1u);
                    }
                    tc_commit(bar(TB_ODONE + s));
                    ok = tc_mbar_wait(bar(TB_ODONE + s), ph);
                    if (first) { first = false; segs++; }
                }
                n += tiles;
            }
            if (!ok) {
                give_up();
                tc_commit(bar(TB_DRAIN + s));                  // whatever was issued ends before the tensor memory is freed
                tc_mbar_wait(bar(TB_DRAIN + s), 0u);
            }
        }
    } else {
        // =============================== softmax of one stream ===============================
        const int s = (warp - 4) >> 2, row = (warp & 3) * 32 + lane, wt = tid - 128;       // wt: thread of the 256
        const unsigned lane_base = (unsigned)((warp & 3) * 32) << 16;
        const unsigned tS = tmem + s * 128 + lane_base;
        const bool flip = a.scale < 0.f;                       // q changes sign, so that the largest product is the largest logit
        const float qs = fabsf(a.scale) * TT_LOG2E;
        auto both_sync = [&]() { asm volatile("bar.sync 3, 256;\n" ::: "memory"); };
        int n = 0, seg = 0;
        bool dead = false, cut_end = false;
        Segment cut;
        auto wait = [&](int b, unsigned ph) {
            if (!dead && (*s_abort || !tc_mbar_wait(bar(b), ph))) { dead = true; give_up(); }
            dead = __any_sync(0xffffffffu, dead);
        };
        while (walk.next(a, g)) {
            const int tiles = (g.p1 - g.p0 + TT_PAGES - 1) / TT_PAGES, prefix = g.n - g.T;
            unsigned* odd_now = odd + (seg & 1) * 8;
            const int r = g.tile * TREE_TC_ROWS + row, t = r < g.T * a.G ? r / a.G : -1;
            const size_t q_row = (size_t)(g.q0 + max(t, 0)) * a.Hq + g.h * a.G + (t < 0 ? 0 : r - t * a.G);
            // ---- Q: row `row`, the panel of this thread's stream (d = 64: half a panel), rows that do not exist as zeros
            {
                constexpr int CH = HD / 16;                    // 16-byte chunks per thread
                const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD) + s * CH;
                uint4 v[CH];
#pragma unroll
                for (int c = 0; c < CH; c++) v[c] = t >= 0 ? src[c] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int c = 0; c < CH; c++) {
                    if (flip) { v[c].x ^= 0x80008000u; v[c].y ^= 0x80008000u; v[c].z ^= 0x80008000u; v[c].w ^= 0x80008000u; }
                    const int ch = s * CH + c;
                    sts16(sQ + (ch >> 3) * C::panel_bytes + row * 128 + (((ch & 7) ^ (row & 7)) << 4), v[c]);
                }
                tt_proxy_fence();
                __syncwarp();
                if (lane == 0) {
#pragma unroll
                    for (int x = 0; x < 2; x++) if (tiles > 1 || (n & 1) == x) tc_mbar_arrive(bar(TB_QFULL + x));
                }
            }
            float m = -INFINITY, l = 0.f;
            bool first = true;
            const bool idle = __all_sync(0xffffffffu, t < 0);  // no row of this warp exists
            for (int j = (n & 1) == s ? 0 : 1; j < tiles; j += 2) {
                const int i = (n + j) >> 1, key0 = (g.p0 + j * TT_PAGES) * PAGE, pages = min(TT_PAGES, g.p1 - g.p0 - j * TT_PAGES);
                const unsigned ph = (unsigned)i & 1u;
                wait(TB_SFULL + s, ph);
                tc_fence_after();
                const bool edge = key0 + pages * PAGE > prefix;
                bool gap = false;                              // a page of the tile was not there
                if (!dead)
                    for (int x = 0; x < pages; x++) gap |= meta[(s * 2 + (i & 1)) * TT_PAGES + x] == 0;
                if (edge || gap) {
                    // V rows that must not reach the MMAs (see tree_attn.cu): one row of the tile per thread
                    wait(TB_VFULL + s, ph);
                    if (!dead && row < pages * PAGE) {
                        const int pos = key0 + row;
                        const unsigned v = sV(s) + row * 128;
                        bool zero = pos >= g.n || meta[((2 + s) * 2 + (i & 1)) * TT_PAGES + row / PAGE] == 0;
                        if (!zero && pos >= prefix) {
                            bool wild = false;
#pragma unroll
                            for (int c = 0; c < HD / 8; c++) {
                                const uint4 u = lds16(v + (c >> 3) * C::panel_bytes + (c & 7) * 16);
                                const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                                for (int y = 0; y < 4; y++) wild |= (w[y] & 0x7f80u) == 0x7f80u || (w[y] & 0x7f800000u) == 0x7f800000u;
                            }
                            if (wild) { zero = true; atomicOr(&odd_now[(pos - prefix) >> 5], 1u << ((pos - prefix) & 31)); }
                        }
                        if (zero) {
#pragma unroll
                            for (int c = 0; c < HD / 8; c++) sts16(v + (c >> 3) * C::panel_bytes + (c & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
                            tt_proxy_fence();
                        }
                    }
                    __syncwarp();
                }
                if (!dead && !idle) {
                    unsigned win[TT_PAGES];
#pragma unroll
                    for (int c = 0; c < TT_PAGES; c++) win[c] = ~0u;
                    if (edge || gap) {
#pragma unroll
                        for (int c = 0; c < TT_PAGES; c++)
                            win[c] = t < 0 || c >= pages || meta[(s * 2 + (i & 1)) * TT_PAGES + c] == 0 ? 0u : tree_window(a, g, t, key0 + c * PAGE);
                    }
                    // ---- the largest logit of the row in this tile
                    float mx = -INFINITY;
                    unsigned x[2][32];
                    tc_ld32(tS, x[0]);
#pragma unroll
                    for (int c = 0; c < TT_PAGES; c++) {
                        if (c < pages) {
                            tc_ld_wait();
                            if (c + 1 < TT_PAGES && c + 1 < pages) tc_ld32(tS + (c + 1) * 32, x[(c + 1) & 1]);
                            const unsigned (&y)[32] = x[c & 1];
                            if (edge || gap) {
#pragma unroll
                                for (int e = 0; e < 32; e++) mx = fmaxf(mx, (win[c] >> e) & 1u ? __uint_as_float(y[e]) : -INFINITY);
                            } else {
#pragma unroll
                                for (int e = 0; e < 32; e += 2) mx = tt_max3(mx, __uint_as_float(y[e]), __uint_as_float(y[e + 1]));
                            }
                        }
                    }
                    mx *= qs;                                  // -inf * 0 is NaN, which the comparison below takes as "no growth"
                    if (mx != mx) mx = 0.f;
                    const bool move = mx > m + TT_LAZY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = move ? mx : m, f = to == -INFINITY ? 1.f : ex2(m - to);
                        m = to; l *= f;
                        if (!first) {                          // the stream's last product is complete: its successor S is
#pragma unroll
                            for (int c = 0; c < HD / 32; c++) {
                                unsigned o[32];
                                tc_ld32(tmem + 256 + s * 128 + lane_base + c * 32, o);
                                tc_ld_wait();
#pragma unroll
                                for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tc_st32(tmem + 256 + s * 128 + lane_base + c * 32, o);
                            }
                        }
                    }
                    // ---- weights, in place: 32 logits become 16 columns of hi pairs and 16 of lo pairs
                    const float ref = m == -INFINITY ? 0.f : m;
                    float l0 = 0.f, l1 = 0.f;
                    tc_ld32(tS, x[0]);
#pragma unroll
                    for (int c = 0; c < TT_PAGES; c++) {
                        if (c < pages) {
                            tc_ld_wait();
                            if (c + 1 < TT_PAGES && c + 1 < pages) tc_ld32(tS + (c + 1) * 32, x[(c + 1) & 1]);
                            const unsigned (&y)[32] = x[c & 1];
                            unsigned w[32];
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                float u = fmaf(__uint_as_float(y[e]), qs, -ref), v = fmaf(__uint_as_float(y[e + 1]), qs, -ref);
                                if (edge || gap) {
                                    if (!((win[c] >> e) & 1u)) u = -INFINITY;
                                    if (!((win[c] >> (e + 1)) & 1u)) v = -INFINITY;
                                }
                                u = ex2(u); v = ex2(v);
                                l0 += u; l1 += v;
                                split2(u, v, w[e / 2], w[16 + e / 2]);
                            }
                            tc_st32(tS + c * 32, w);
                        }
                    }
                    l += l0 + l1;
                    tc_st_wait();
                }
                first = false;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_mbar_arrive(bar(TB_PFULL + s));
            }
            // ---- the streams meet: both sums are complete, both halves of the columns are merged and written
            n += tiles;
            const int last = n - 1 - (((n - 1) & 1) != s);     // the stream's last tile so far
            if (!first) wait(TB_ODONE + s, (unsigned)(last >> 1) & 1u);
            ml_s[s * 128 + row] = make_float2(m, first ? -1.f : l);
            tc_fence_before();
            both_sync();
            tc_fence_after();
            if (wt < 8) odd[((seg + 1) & 1) * 8 + wt] = 0u;
            const float2 o0 = ml_s[row], o1 = ml_s[128 + row];
            const bool have0 = o0.y >= 0.f || o0.y != o0.y, have1 = o1.y >= 0.f || o1.y != o1.y;      // the stream had a tile (l may be NaN)
            const float top = fmaxf(have0 ? o0.x : -INFINITY, have1 ? o1.x : -INFINITY), ref = top == -INFINITY ? 0.f : top;
            const float f0 = have0 ? ex2(o0.x - ref) : 0.f, f1 = have1 ? ex2(o1.x - ref) : 0.f;
            const float lt = (have0 ? o0.y * f0 : 0.f) + (have1 ? o1.y * f1 : 0.f);
            const bool whole = g.first && g.last;
            if (!dead && !idle) {
                const float norm = !whole ? 1.f : lt == 0.f ? 0.f : 1.f / lt;
                unsigned any_odd = 0u;
#pragma unroll
                for (int w = 0; w < 8; w++) any_odd |= odd_now[w];
#pragma unroll
                for (int c = 0; c < HD / 64; c++) {
                    const int col = s * (HD / 2) + c * 32;     // this stream's half of the columns
                    float o[32];
                    unsigned u[32];
#pragma unroll
                    for (int e = 0; e < 32; e++) o[e] = 0.f;
                    if (have0) {                               // the same in all lanes
                        tc_ld32(tmem + 256 + lane_base + col, u);
                        tc_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; e++) o[e] = __uint_as_float(u[e]) * f0;
                    }
                    if (have1) {
                        tc_ld32(tmem + 384 + lane_base + col, u);
                        tc_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; e++) o[e] = fmaf(__uint_as_float(u[e]), f1, o[e]);
                    }
                    if (any_odd && t >= 0) {                   // drafted rows that were left out of the products
                        for (int w = 0; w < 8; w++) {
                            unsigned bits = odd_now[w];
                            while (bits) {
                                const int jj = w * 32 + __ffs(bits) - 1, pos = prefix + jj;
                                bits &= bits - 1;
                                if (!tree_sees(a, g, t, jj)) continue;
                                const int page = a.page_table[(size_t)g.b * a.pages_per_seq + pos / PAGE];
                                const size_t key = ((size_t)page * a.Hk + g.h) * PAGE + pos % PAGE;
                                const __nv_bfloat16* kr = reinterpret_cast<const __nv_bfloat16*>(a.kpool) + key * HD;
                                const __nv_bfloat16* vr = reinterpret_cast<const __nv_bfloat16*>(a.vpool) + key * HD + col;
                                const __nv_bfloat16* qr = reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD;
                                float d = 0.f;
                                for (int e = 0; e < HD; e++) d = fmaf(__bfloat162float(qr[e]), __bfloat162float(kr[e]), d);
                                const float p = ex2(d * (a.scale * TT_LOG2E) - ref);
#pragma unroll
                                for (int e = 0; e < 32; e++) o[e] = fmaf(p, __bfloat162float(vr[e]), o[e]);
                            }
                        }
                    }
                    if (t >= 0) {
                        if (whole) {
                            uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + q_row * HD + col);
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                to[e] = make_uint4(pack_bf16(o[8 * e] * norm, o[8 * e + 1] * norm), pack_bf16(o[8 * e + 2] * norm, o[8 * e + 3] * norm),
                                                   pack_bf16(o[8 * e + 4] * norm, o[8 * e + 5] * norm), pack_bf16(o[8 * e + 6] * norm, o[8 * e + 7] * norm));
                        } else {
                            const size_t slot = (size_t)blockIdx.x * 2 + (g.first ? 1 : 0);
                            float4* to = reinterpret_cast<float4*>(a.acc + (slot * TREE_TC_ROWS + row) * HD + col);
#pragma unroll
                            for (int e = 0; e < 8; e++) to[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    }
                }
                if (t >= 0 && s == 0) {
                    if (!whole) a.ml[((size_t)blockIdx.x * 2 + (g.first ? 1 : 0)) * TREE_TC_ROWS + row] = make_float2(top, lt);
                    else if (a.lse) a.lse[q_row] = lt == 0.f ? -INFINITY : (top + log2f(lt)) * TT_LN2;
                }
            }
            tc_fence_before();
            both_sync();                                       // Q, O and the records are free again
            tc_fence_after();
            if (g.last && !g.first) { cut = g; cut_end = true; }
            seg++;
        }
        if (wt == 0) {
            if (cut_end) describe_cut_unit(a, cut, range);
            a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
        }
    }
    // ---- everyone meets here, on every path; then the allocating warp frees the tensor memory
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && *s_abort) tree_status(a, DYNAKV_ST_INTERNAL);
}

template <int HD>
static int tree_tc_launch_hd(const dynakv_row_cache* cache, const TreeArgs& a, int sms, cudaStream_t st) {
    CUtensorMap mk, mv;
    if (!tree_page_map(&mk, cache, cache->k, false) || !tree_page_map(&mv, cache, cache->v, false)) return DYNAKV_ERR_CUDA;
    if (cudaFuncSetAttribute(k_tree_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcTree<HD>::smem) != cudaSuccess) return DYNAKV_ERR_CUDA;
    k_tree_tc<HD><<<sms, TT_THREADS, TcTree<HD>::smem, st>>>(mk, mv, a);
    if (cudaGetLastError() != cudaSuccess) return DYNAKV_ERR_CUDA;
    return tree_merge_launch(HD, TREE_TC_ROWS, false, a, sms, st);
}

int tree_tc_launch(const dynakv_row_cache* cache, const TreeArgs& a, int sms, cudaStream_t st) {
    return cache->head_dim == 128 ? tree_tc_launch_hd<128>(cache, a, sms, st) : tree_tc_launch_hd<64>(cache, a, sms, st);
}

}  // namespace dkv
