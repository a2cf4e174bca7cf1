// Tree attention on the tcgen05 tensor cores: bf16 and FP8 rows, tiles of 128 or 256 query rows (token, head of the group).
//
// With R query rows per KV head a bf16 row of K and V (512 bytes at d = 128) meets 4 d R flops: from a few dozen rows on the
// mma.sync kernel is bound by the legacy tensor pipe (one m16n8k16 per 8.2 cycles and scheduler).  On tcgen05 the softmax's
// instructions per logit set the pace: bf16 trees of 16 (R = 64) over 4 x 32768 rows take 105 us in a burst and 120 when run for long, of 64
// (R = 256) over 2 x 34816 rows 115 and 132, with all pages read from L2 still 91 and 114; the bytes alone would take 79 and 43.
// FP8 rows: 244 us at R = 80 and 259 at R = 128 over 4 x 32768 rows, whose bytes take 40, because four warps convert every
// element and the softmax has 128 registers a thread (282 to 298 bytes spilled; bf16 rows: 168 registers, 18 to 26 bytes).
//
// One CTA per SM walks over its range of pages (tree_plan.cuh) in stages of four pages (128 keys) of K and of V.  Two streams
// work on every stage, each with logits S, a running softmax and an output sum O of its own in tensor memory: with up to
// 128 rows (PAIR = false) both have the same rows and take two pages of the stage each, and meet at a segment's
// end; with more (PAIR = true) each has 128 rows of the tile of 256 and takes the stage in two halves, so that a row of
// K and V is read once for 256 query rows.  S is kept twice: the next half's logits are multiplied while the softmax works
// on this one's, and the sum of products follows behind (a first version with one S of 128 keys per stream left tensor
// pipe and softmax waiting for each other: 4 450 cycles per 128 keys, 1 536 of them in the tensor pipe).
//   warp 0 / warp 3     TMA loads of K / of V, one 32-row panel of 128 bytes per copy, 128-byte swizzle
//   warp 1 / warp 2     tcgen05.mma of stream 0 / 1: S = Q K^T (M = 128, N = 64 keys), then O += P V with P from tensor
//                       memory and V read with its rows as the contraction index, no transposed copy anywhere
//   warps 4-7 / 8-11    softmax of stream 0 / 1: a query row per thread
//   warps 12-15         FP8 rows only: they fetch the rows and turn them into bf16 stages (warps 0 and 3 then rest)
// Tensor memory (512 columns): S of stream s at 128 s and 128 s + 64, O at 256 + 128 s.  The weights replace the logits in
// place: 32 logits of a row become 16 columns of bf16 hi pairs and 16 of lo pairs (the two MMAs of the split keep fp32 weights to
// 2^-17; bf16 weights alone would add an error as large as the output's own rounding).  The softmax's reference moves
// only when the maximum has grown by 2^8, which is when O has to be rescaled.
// Barriers: a half u of a stream uses buffer u mod 2 and its barriers' phase u div 2, so that no waiter can be two
// phases away from a barrier although logits, weights and sums run up to two halves apart.  All waits are bounded.
#include <cuda.h>
#include <float.h>

#include "bulk_copy.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"
#include "tree_plan.cuh"

namespace dkv {

constexpr int TT_PAGES = 4, TT_HALF = 2;                       // pages of a stage and of the half a stream works on
constexpr int TT_CONVERT = 128;                                // FP8: threads that load rows and convert them
constexpr float TT_LOG2E = 1.4426950408889634f, TT_LN2 = 0.6931471805599453f, TT_LAZY = 8.f;

template <int HD, bool PAIR, bool F8>
struct TcTree {
    static constexpr int threads = 384 + (F8 ? TT_CONVERT : 0);
    static constexpr int rows = PAIR ? 256 : 128;              // query rows of a tile
    static constexpr int panels = HD / 64;                     // 128-byte column panels of a row
    static constexpr int panel_bytes = 128 * 128;              // 128 rows of 128 bytes
    static constexpr int tile_bytes = panels * panel_bytes;
    static constexpr int q_tiles = PAIR ? 2 : 1;
    static constexpr int stages = 2;                           // of K and V each: with Q 160 or 192 KB at d = 128 (three: 3 to 8 % slower,
                                                               // three of only one of them: no difference)
    static constexpr int fixed = 2 * 128 * 8 + 48 * 8 + 32 * 8 + 2 * 8 * 4 + 8 * 4 + 16;
    static constexpr int smem = (q_tiles + 2 * stages) * tile_bytes + fixed;
    static_assert(smem + 1024 <= 233472, "shared memory of an SM");
    // kind::f16, fp32 accumulate, bf16 operands, M = 128
    static constexpr unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
    static constexpr unsigned idesc_pv = idesc | (1u << 16) | ((unsigned)(HD >> 3) << 17);      // B's contraction index is its outer one
    // barriers; those of a stream: + 2 * stream + buffer
    static constexpr int KFULL = 0, KEMPTY = stages, VFULL = 2 * stages, VEMPTY = 3 * stages, SFULL = 4 * stages, PFULL = SFULL + 4,
                         ODONE = PFULL + 4, QFULL = ODONE + 4, DRAIN = QFULL + 2, count = DRAIN + 2;
    static_assert(count <= 32, "barrier block");
};

// Pages of half h of stage j of a segment of `pages` pages.
__device__ __forceinline__ int half_pages(int pages, int j, int h) { return max(0, min(TT_HALF, pages - j * TT_PAGES - h * TT_HALF)); }

template <int HD, bool PAIR, bool F8>
__global__ void __launch_bounds__((TcTree<HD, PAIR, F8>::threads), 1) k_tree_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                           const __grid_constant__ TreeArgs a) {
    using C = TcTree<HD, PAIR, F8>;
    constexpr int NS = C::stages;
    extern __shared__ __align__(1024) unsigned char tt_smem[];
    unsigned char* at = tt_smem + (C::q_tiles + 2 * NS) * C::tile_bytes;
    float2* ml_s = reinterpret_cast<float2*>(at); at += 2 * 128 * 8;               // [stream][row] (m, l)
    long long* sh = reinterpret_cast<long long*>(at); at += 48 * 8;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(at); at += 32 * 8;
    unsigned* odd = reinterpret_cast<unsigned*>(at); at += 2 * 8 * 4;              // [segment parity][8]
    volatile int* meta = reinterpret_cast<volatile int*>(at); at += 8 * 4;         // [stage number mod 8] bit per page: it was loaded
    volatile unsigned* s_tmem = reinterpret_cast<volatile unsigned*>(at);
    volatile int* s_abort = reinterpret_cast<volatile int*>(at + 4);
    const unsigned sQ = tc_smem_u32(tt_smem);
    auto sK = [&](int st) { return sQ + (C::q_tiles + st) * C::tile_bytes; };
    auto sV = [&](int st) { return sQ + (C::q_tiles + NS + st) * C::tile_bytes; };
    const unsigned bar0 = tc_smem_u32(bars);
    auto bar = [&](int i) { return bar0 + i * 8; };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int i = 0; i < C::count; i++) {
            const bool empty = (i >= C::KEMPTY && i < C::VFULL) || (i >= C::VEMPTY && i < C::SFULL);
            const bool full = (i >= C::KFULL && i < C::KEMPTY) || (i >= C::VFULL && i < C::VEMPTY);
            tc_mbar_init(bar(i), empty ? 2 : full && F8 ? TT_CONVERT / 32 : i >= C::PFULL && i < C::ODONE ? 4 : i >= C::QFULL && i < C::DRAIN ? 8 : 1);
        }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (tid < 16) odd[tid] = 0u;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tc_smem_u32((const void*)s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    pdl_wait();                                                // from here on the results of earlier kernels are read
    const Range range = tree_range<C::rows>(a, TT_PAGES, sh);
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const unsigned tmem = *s_tmem;
    SegmentWalk<C::rows> walk(range, sh);
    Segment g;
    auto give_up = [&]() { *s_abort = 1; };

    if (F8 && (warp == 0 || warp == 3)) {
        // nothing to load by TMA: the converting warps fetch the rows themselves
    } else if (warp == 0 || warp == 3) {
        // =============================== loads: warp 0 K, warp 3 V ===============================
        const bool is_v = warp == 3;
        const CUtensorMap* map = is_v ? &map_v : &map_k;
        const int full = is_v ? C::VFULL : C::KFULL, empty = is_v ? C::VEMPTY : C::KEMPTY;
        int n = 0;                                             // stage number in the CTA
        bool ok = true;
        while (ok && next_segment(walk, a, g)) {
            for (int pc = g.p0; ok && pc < g.p1; pc += 32) {
                const int cnt = min(32, g.p1 - pc);
                int id = -1;
                if (lane < cnt && g.n > 0) {
                    id = a.page_table[(size_t)g.b * a.pages_per_seq + pc + lane];
                    if (id < 0 || id >= a.n_pages) { id = -1; tree_status(a, DYNAKV_ST_BOUNDS); }
                }
                const unsigned there = __ballot_sync(0xffffffffu, id >= 0);
                for (int j = 0; j < cnt && ok; j += TT_PAGES, n++) {
                    const int st = n % NS, use = n / NS;
                    int page[TT_PAGES];
#pragma unroll
                    for (int x = 0; x < TT_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, id, j + x);      // -1 past the segment's end
                    const int bits = (there >> j) & 15;
                    if (lane == 0) {
                        ok = !*s_abort && (use == 0 || mbar_wait(bar(empty + st), (unsigned)(use - 1) & 1u));
                        if (ok) {
                            if (!is_v) meta[n & 7] = bits;
                            if (bits) tc_mbar_expect_tx(bar(full + st), __popc(bits) * PAGE * HD * 2);
                            else tc_mbar_arrive(bar(full + st));
                            const unsigned dst = is_v ? sV(st) : sK(st);
#pragma unroll
                            for (int x = 0; x < TT_PAGES; x++) {
                                if (page[x] < 0) continue;
#pragma unroll
                                for (int p = 0; p < C::panels; p++)
                                    tt_load(dst + p * C::panel_bytes + x * PAGE * 128, map, (page[x] * a.Hk + g.h) * PAGE, p, bar(full + st));
                            }
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                }
            }
        }
        if (!ok && lane == 0) {
            give_up();
            // stage n - 1 was not issued; let the copies of the ones before it land before the block ends
            for (int x = max(0, n - 1 - NS); x < n - 1; x++) mbar_wait(bar(full + x % NS), (unsigned)(x / NS) & 1u);
        }
    } else if (warp == 1 || warp == 2) {
        // =============================== MMAs of one stream ===============================
        // The whole warp walks and waits, one elected lane issues: addresses and descriptors then stay in uniform registers, where
        // the instructions want them.
        const int s = warp - 1;
        int n = 0, u = 0, segs = 0;                            // stages so far, halves so far, segments in which the stream had a half
        bool ok = true;
        // operand descriptors of the first step; the address field counts 16 bytes
        const unsigned long long dq = tc_panel_desc(sQ + (PAIR ? s * C::tile_bytes : 0)), dk = tc_panel_desc(sK(0)), dv = tc_rows_desc(sV(0), C::panel_bytes);
        const unsigned tO = tmem + 256 + s * 128;
        auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
        while (ok && next_segment(walk, a, g)) {
            const int pages = g.p1 - g.p0, stages = (pages + TT_PAGES - 1) / TT_PAGES;
            const int halves = PAIR ? (pages + TT_HALF - 1) / TT_HALF : stages - (s == 1 && half_pages(pages, stages - 1, 1) == 0 ? 1 : 0);
            const int u0 = u;
            // logits of half i of the segment
            auto logits = [&](int i) {
                const int j = PAIR ? i >> 1 : i, h = PAIR ? i & 1 : s, st = (n + j) % NS, use = (n + j) / NS, v = u0 + i;
                if (i == 0) wait(C::QFULL + s, segs);
                if (!PAIR || h == 0) wait(C::KFULL + st, use);
                if (v >= 2) wait(C::ODONE + 2 * s + (v & 1), (v >> 1) - 1);            // the buffer's last weights have been used
                if (!ok) return;
                tc_fence_after();
                const unsigned idesc = C::idesc | ((unsigned)(half_pages(pages, j, h) * PAGE >> 3) << 17);
                const unsigned long long k0 = dk + ((st * C::tile_bytes + h * TT_HALF * PAGE * 128) >> 4);
                const unsigned tS = tmem + s * 128 + (v & 1) * 64;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < HD / 16; k++) {
                        const unsigned off = ((k >> 2) * C::panel_bytes + (k & 3) * 32) >> 4;
                        tc_mma_f16(tS, dq + off, k0 + off, idesc, k > 0 ? 1u : 0u);
                    }
                    tc_commit(bar(C::SFULL + 2 * s + (v & 1)));
                    if (!PAIR || h == 1 || i == halves - 1) tc_commit(bar(C::KEMPTY + st));
                }
                __syncwarp();
            };
            if (halves > 0) logits(0);
            for (int i = 0; i < halves && ok; i++, u++) {
                if (i + 1 < halves) logits(i + 1);
                const int j = PAIR ? i >> 1 : i, h = PAIR ? i & 1 : s, st = (n + j) % NS, use = (n + j) / NS;
                if (!PAIR || h == 0) wait(C::VFULL + st, use);
                wait(C::PFULL + 2 * s + (u & 1), u >> 1);
                if (!ok) break;
                tc_fence_after();
                const unsigned tP = tmem + s * 128 + (u & 1) * 64;
                const unsigned long long v0 = dv + ((st * C::tile_bytes + h * TT_HALF * PAGE * 128) >> 4);
                const int steps = half_pages(pages, j, h) * 2;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < TT_HALF * 2; k++) {
                        if (k >= steps) break;
                        const unsigned p = tP + (k >> 1) * 32 + (k & 1) * 8;
                        tc_mma_f16_ta(tO, p, v0 + k * (2048 >> 4), C::idesc_pv, i > 0 || k > 0 ? 1u : 0u);
                        tc_mma_f16_ta(tO, p + 16, v0 + k * (2048 >> 4), C::idesc_pv, 1u);
                    }
                    tc_commit(bar(C::ODONE + 2 * s + (u & 1)));
                    if (!PAIR || h == 1 || i == halves - 1) tc_commit(bar(C::VEMPTY + st));
                }
                __syncwarp();
            }
            if (!PAIR && halves < stages && ok) {              // the last stage has no half for this stream: give it back
                const int st = (n + stages - 1) % NS, use = (n + stages - 1) / NS;
                wait(C::KFULL + st, use);
                wait(C::VFULL + st, use);
                if (ok && lane == 0) { tc_mbar_arrive(bar(C::KEMPTY + st)); tc_mbar_arrive(bar(C::VEMPTY + st)); }
            }
            if (halves > 0) segs++;
            n += stages;
        }
        if (!ok) {
            if (elect_one()) {
                give_up();
                tc_commit(bar(C::DRAIN + s));                  // whatever was issued ends before the tensor memory is freed
            }
            __syncwarp();
            mbar_wait(bar(C::DRAIN + s), 0u);
        }
    } else if (F8 && warp >= 12) {
        // =============================== FP8 rows to bf16 stages ===============================
        // A thread takes the same 16 bytes of every RPP-th row of a stage.  K and V alternate: while one is converted (exactly: e4m3
        // times a power of two is a bf16 value) and stored where the TMA would have put it, the other's loads are under way.
        constexpr int CPR = HD / 16, RPP = TT_CONVERT / CPR, NP = TT_PAGES * PAGE / RPP;
        const int ct = tid - 384, chunk = ct % CPR, row0 = ct / CPR;
        int n = 0, pc = 0, id = -1;
        bool ok = true, more = false;
        int page[TT_PAGES], bits = 0, h = 0;                   // the stage to load next
        auto advance = [&](bool first) {                       // all lanes together
            if (!first) pc += TT_PAGES;
            if (first || pc >= g.p1) { more = next_segment(walk, a, g); pc = more ? g.p0 : 0; }
            if (!more) return;
            if (((pc - g.p0) & 31) == 0) {
                id = -1;
                if (pc + lane < g.p1 && g.n > 0) {
                    id = a.page_table[(size_t)g.b * a.pages_per_seq + pc + lane];
                    if (id < 0 || id >= a.n_pages) { id = -1; tree_status(a, DYNAKV_ST_BOUNDS); }
                }
            }
            const int j = (pc - g.p0) & 31;
            const unsigned there = __ballot_sync(0xffffffffu, id >= 0);
            bits = (there >> j) & 15;
#pragma unroll
            for (int x = 0; x < TT_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, id, j + x);
            h = g.h;
        };
        uint4 raw[2][NP];                                      // K, V
        int ex[2][NP];
        auto fetch = [&](int kv) {
            const unsigned char* pool = kv ? a.vpool : a.kpool;
            const signed char* exps = kv ? a.vexp : a.kexp;
#pragma unroll
            for (int i = 0; i < NP; i++) {
                const int pg = page[i * RPP / PAGE];
                const size_t r = ((size_t)(pg < 0 ? 0 : pg) * a.Hk + h) * PAGE + (i * RPP + row0) % PAGE;
                raw[kv][i] = pg >= 0 ? __ldg(reinterpret_cast<const uint4*>(pool + r * HD) + chunk) : make_uint4(0u, 0u, 0u, 0u);
                ex[kv][i] = pg >= 0 ? (int)__ldg(reinterpret_cast<const signed char*>(exps) + r) : 0;
            }
        };
        auto convert = [&](int kv, unsigned dst) {
#pragma unroll
            for (int i = 0; i < NP; i++) {
                const int row = i * RPP + row0;
                const float sc = pow2f(ex[kv][i]);
                const float2 sc2 = make_float2(sc, sc);
                const unsigned w[4] = {raw[kv][i].x, raw[kv][i].y, raw[kv][i].z, raw[kv][i].w};
                unsigned o[8];
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    unsigned lo, hi;
                    e4m3x4_to_f16x2(w[x], lo, hi);
                    const float2 p = mul2(__half22float2(*reinterpret_cast<const __half2*>(&lo)), sc2), q = mul2(__half22float2(*reinterpret_cast<const __half2*>(&hi)), sc2);
                    o[2 * x] = pack_bf16(p.x, p.y);
                    o[2 * x + 1] = pack_bf16(q.x, q.y);
                }
                const unsigned to = dst + (chunk >> 2) * C::panel_bytes + row * 128, ch = (2 * chunk) & 7;
                sts16(to + ((ch ^ (row & 7)) << 4), make_uint4(o[0], o[1], o[2], o[3]));
                sts16(to + (((ch + 1) ^ (row & 7)) << 4), make_uint4(o[4], o[5], o[6], o[7]));
            }
            tt_proxy_fence();
            __syncwarp();
        };
        auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
        advance(true);
        if (more) fetch(0);
        while (more && ok) {
            const int st = n % NS, use = n / NS, bits_now = bits;
            fetch(1);
            if (use > 0) wait(C::KEMPTY + st, use - 1);
            if (!ok) break;
            if (ct == 0) meta[n & 7] = bits_now;
            convert(0, sK(st));
            if (lane == 0) tc_mbar_arrive(bar(C::KFULL + st));
            advance(false);
            if (more) fetch(0);
            if (use > 0) wait(C::VEMPTY + st, use - 1);
            if (!ok) break;
            convert(1, sV(st));
            if (lane == 0) tc_mbar_arrive(bar(C::VFULL + st));
            n++;
        }
        if (!ok && lane == 0) give_up();
    } else {
        // =============================== softmax of one stream ===============================
        const int s = (warp - 4) >> 2, row = (warp & 3) * 32 + lane, wt = tid - 128;       // wt: thread of the 256
        const unsigned lane_base = (unsigned)((warp & 3) * 32) << 16;
        const unsigned tO = tmem + 256 + s * 128 + lane_base;
        const bool flip = a.scale < 0.f;                       // q changes sign, so that the largest product is the largest logit
        const float qs = a.scale == 0.f ? 1.f : fabsf(a.scale) * TT_LOG2E;     // scale 0: q is taken as zero, so that a masked -inf stays one
        auto both_sync = [&]() { asm volatile("bar.sync 3, 256;\n" ::: "memory"); };
        int n = 0, u = 0, seg = 0;
        bool dead = false, cut_end = false;
        auto wait = [&](int b, int phase) {
            if (!dead && !mbar_wait(bar(b), (unsigned)phase & 1u)) { dead = true; give_up(); }
            dead = __any_sync(0xffffffffu, dead);
        };
        while (next_segment(walk, a, g)) {
            const int pages = g.p1 - g.p0, stages = (pages + TT_PAGES - 1) / TT_PAGES, prefix = g.n - g.T;
            const int halves = PAIR ? (pages + TT_HALF - 1) / TT_HALF : stages - (s == 1 && half_pages(pages, stages - 1, 1) == 0 ? 1 : 0);
            unsigned* odd_now = odd + (seg & 1) * 8;
            const int rl = (PAIR ? s * 128 : 0) + row, r = g.tile * C::rows + rl, t = r < g.T * a.G ? r / a.G : -1;
            const size_t q_row = (size_t)(g.q0 + max(t, 0)) * a.Hq + g.h * a.G + (t < 0 ? 0 : r - t * a.G);
            // ---- Q: this thread's row, or with the same rows in both streams half of it; rows that do not exist as zeros
            {
                constexpr int CH = PAIR ? HD / 8 : HD / 16;    // 16-byte chunks per thread
                const int c0 = PAIR ? 0 : s * CH;
                const unsigned to = sQ + (PAIR ? s * C::tile_bytes : 0) + row * 128;
                const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD) + c0;
                uint4 v[CH];                                   // all loads before the first store
#pragma unroll
                for (int c = 0; c < CH; c++) v[c] = t >= 0 && a.scale != 0.f ? src[c] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int c = 0; c < CH; c++) {
                    if (flip) { v[c].x ^= 0x80008000u; v[c].y ^= 0x80008000u; v[c].z ^= 0x80008000u; v[c].w ^= 0x80008000u; }
                    const int ch = c0 + c;
                    sts16(to + (ch >> 3) * C::panel_bytes + (((ch & 7) ^ (row & 7)) << 4), v[c]);
                }
                tt_proxy_fence();
                __syncwarp();
                if (lane == 0) {
                    tc_mbar_arrive(bar(C::QFULL));
                    if (PAIR || pages > TT_HALF) tc_mbar_arrive(bar(C::QFULL + 1));
                }
            }
            float m = -INFINITY, l = 0.f;
            const bool idle = __all_sync(0xffffffffu, t < 0);  // no row of this warp exists
            for (int i = 0; i < halves; i++, u++) {
                const int j = PAIR ? i >> 1 : i, h = PAIR ? i & 1 : s, st = (n + j) % NS, use = (n + j) / NS;
                const int key0 = (g.p0 + j * TT_PAGES + h * TT_HALF) * PAGE, cnt = half_pages(pages, j, h), b = 2 * s + (u & 1);
                const unsigned tS = tmem + s * 128 + (u & 1) * 64 + lane_base;
                wait(C::SFULL + b, u >> 1);
                tc_fence_after();
                const int want = (1 << cnt) - 1, have = (meta[(n + j) & 7] >> (h * TT_HALF)) & want;       // pages of the half that were there
                const bool edge = key0 + cnt * PAGE > prefix;  // holds drafted rows or the end of the sequence: a matter of lengths alone
                const bool mask = edge || (have != want && !dead);
                if (mask) {
                    // V rows that must not reach the MMAs (see tree_attn.cu), one row of the half per thread.  Of a stage that both
                    // streams use, stream 0's threads look at the rows; those of a page that was not there are zeroed by both
                    wait(C::VFULL + st, use);
                    if (!dead && row < cnt * PAGE) {
                        const int pos = key0 + row;
                        const unsigned v = sV(st) + (h * TT_HALF * PAGE + row) * 128;
                        bool zero = !((have >> (row / PAGE)) & 1);
                        if (!zero && edge && (!PAIR || s == 0)) {
                            if (pos >= g.n) zero = true;
                            else if (pos >= prefix) {
                                bool wild = false;
#pragma unroll
                                for (int c = 0; c < HD / 8; c++) {
                                    const uint4 x = lds16(v + (c >> 3) * C::panel_bytes + (c & 7) * 16);
                                    const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                    for (int y = 0; y < 4; y++) wild |= (w[y] & 0x7f80u) == 0x7f80u || (w[y] & 0x7f800000u) == 0x7f800000u;
                                }
                                if (wild) { zero = true; atomicOr(&odd_now[(pos - prefix) >> 5], 1u << ((pos - prefix) & 31)); }
                            }
                        }
                        if (zero) {
#pragma unroll
                            for (int c = 0; c < HD / 8; c++) sts16(v + (c >> 3) * C::panel_bytes + (c & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
                            tt_proxy_fence();
                        }
                    }
                    __syncwarp();
                }
                if (PAIR && edge) both_sync();                 // both streams come by the same halves
                if (!dead && !idle) {
                    // ---- the row's logits, and the largest
                    unsigned x[TT_HALF][32];
#pragma unroll
                    for (int c = 0; c < TT_HALF; c++) if (c < cnt) tc_ld32(tS + c * 32, x[c]);
                    tc_ld_wait();
                    if (mask) {
#pragma unroll
                        for (int c = 0; c < TT_HALF; c++) {
                            const unsigned win = t >= 0 && ((have >> c) & 1) ? tree_window(a, g, t, key0 + c * PAGE) : 0u;
#pragma unroll
                            for (int e = 0; e < 32; e++) if (!((win >> e) & 1u)) x[c][e] = 0xff800000u;
                        }
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < TT_HALF; c++)
                        if (c < cnt) {
#pragma unroll
                            for (int e = 0; e < 32; e += 2) m4[(e >> 1) & 3] = tt_max3(m4[(e >> 1) & 3], __uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1]));
                        }
                    const float mx = tt_max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]) * qs;
                    const bool move = mx > m + TT_LAZY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = move ? mx : m, f = to == -INFINITY ? 1.f : ex2(m - to);
                        m = to; l *= f;
                        if (i > 0) {                           // O as it is after the last half's products
                            wait(C::ODONE + 2 * s + ((u - 1) & 1), (u - 1) >> 1);
                            tc_fence_after();
                            if (!dead) {
#pragma unroll
                                for (int c = 0; c < HD / 32; c++) {
                                    unsigned o[32];
                                    tc_ld32(tO + c * 32, o);
                                    tc_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                    tc_st32(tO + c * 32, o);
                                }
                            }
                        }
                    }
                    // ---- weights, in place: 32 logits become 16 columns of hi pairs and 16 of lo pairs
                    const float ref = m == -INFINITY ? 0.f : m;
                    float2 sum = make_float2(0.f, 0.f);
                    const float2 qs2 = make_float2(qs, qs), ref2 = make_float2(-ref, -ref), neg = make_float2(-1.f, -1.f), one = make_float2(1.f, 1.f);
#pragma unroll
                    for (int c = 0; c < TT_HALF; c++)
                        if (c < cnt) {
#pragma unroll
                            for (int part = 0; part < 2; part++) {             // 16 keys at a time: fewer registers
                                unsigned hi[8], lo[8];
#pragma unroll
                                for (int e = 0; e < 8; e++) {
                                    float2 y = fma2(make_float2(__uint_as_float(x[c][part * 16 + 2 * e]), __uint_as_float(x[c][part * 16 + 2 * e + 1])), qs2, ref2);
                                    y = make_float2(ex2(y.x), ex2(y.y));
                                    sum = fma2(y, one, sum);
                                    hi[e] = pack_bf16(y.x, y.y);
                                    const float2 z = fma2(make_float2(__uint_as_float(hi[e] << 16), __uint_as_float(hi[e] & 0xffff0000u)), neg, y);
                                    lo[e] = pack_bf16(z.x, z.y);
                                }
                                tc_st8(tS + c * 32 + part * 8, hi);
                                tc_st8(tS + c * 32 + 16 + part * 8, lo);
                            }
                        }
                    l += sum.x + sum.y;
                    tc_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_mbar_arrive(bar(C::PFULL + b));
            }
            n += stages;
            if (halves > 0) wait(C::ODONE + 2 * s + ((u - 1) & 1), (u - 1) >> 1);
            // ---- with the same rows in both streams: they meet, and each merges and writes half of the columns
            if (!PAIR) ml_s[s * 128 + row] = make_float2(m, l);
            tc_fence_before();
            both_sync();
            tc_fence_after();
            if (wt < 8) odd[((seg + 1) & 1) * 8 + wt] = 0u;
            float2 o0 = make_float2(m, l), o1 = make_float2(-INFINITY, 0.f);
            const bool have1 = !PAIR && pages > TT_HALF;       // stream 1 had a half: the same in all threads, as the warp-wide loads need it
            if (!PAIR) { o0 = ml_s[row]; if (have1) o1 = ml_s[128 + row]; }
            const float top = fmaxf(o0.x, o1.x), ref = top == -INFINITY ? 0.f : top;
            const float f0 = ex2(o0.x - ref), f1 = ex2(o1.x - ref), lt = o0.y * f0 + o1.y * f1;
            const bool whole = g.first && g.last;
            const size_t slot = (size_t)blockIdx.x * 2 + (g.first ? 1 : 0);
            if (!dead && !idle) {
                const float norm = !whole ? 1.f : lt == 0.f ? 0.f : 1.f / lt;
                unsigned any_odd = 0u;
#pragma unroll
                for (int w = 0; w < 8; w++) any_odd |= odd_now[w];
#pragma unroll 1
                for (int c = 0; c < (PAIR ? HD / 32 : HD / 64); c++) {
                    const int col = (PAIR ? 0 : s * (HD / 2)) + c * 32;
                    float o[32];
                    unsigned v[32];
                    tc_ld32((PAIR ? tO : tmem + 256 + lane_base) + col, v);
                    tc_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; e++) o[e] = __uint_as_float(v[e]) * f0;
                    if (have1) {
                        tc_ld32(tmem + 384 + lane_base + col, v);
                        tc_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; e++) o[e] = fmaf(__uint_as_float(v[e]), f1, o[e]);
                    }
                    if (any_odd && t >= 0) {                   // drafted rows that were left out of the products
                        for (int w = 0; w < 8; w++) {
                            unsigned bits = odd_now[w];
                            while (bits) {
                                const int jj = w * 32 + __ffs(bits) - 1, pos = prefix + jj;
                                bits &= bits - 1;
                                if (!tree_sees(a, g, t, jj)) continue;
                                const int page = a.page_table[(size_t)g.b * a.pages_per_seq + pos / PAGE];
                                const long long key = ((long long)page * a.Hk + g.h) * PAGE + pos % PAGE;
                                constexpr int DT = F8 ? DYNAKV_FP8 : DYNAKV_BF16;
                                const __nv_bfloat16* qr = reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD;
                                float d = 0.f;
                                for (int e = 0; e < HD; e++) d = fmaf(__bfloat162float(qr[e]), cache_elem<DT>(a.kpool, a.kexp, key, HD, e), d);
                                const float p = ex2(d * (a.scale * TT_LOG2E) - ref);
#pragma unroll
                                for (int e = 0; e < 32; e++) o[e] = fmaf(p, cache_elem<DT>(a.vpool, a.vexp, key, HD, col + e), o[e]);
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
                            // four columns of all rows side by side: the lanes' stores join
                            float4* to = reinterpret_cast<float4*>(a.acc) + (slot * (HD / 4) + col / 4) * C::rows + rl;
#pragma unroll
                            for (int e = 0; e < 8; e++) to[e * C::rows] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    }
                }
                if (t >= 0 && (PAIR || s == 0)) {
                    if (!whole) a.ml[slot * C::rows + rl] = make_float2(top, lt);
                    else if (a.lse) a.lse[q_row] = lt == 0.f ? -INFINITY : (top + log2f(lt)) * TT_LN2;
                }
            }
            tc_fence_before();
            both_sync();                                       // Q, O and the records are free again
            tc_fence_after();
            if (g.last && !g.first) { cut_end = true; if (wt == 0) describe_cut_unit(a, g, walk.r); }
            seg++;
        }
        if (wt == 0) a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
    }
    // ---- everyone meets here, on every path; then the allocating warp frees the tensor memory
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && *s_abort) tree_status(a, DYNAKV_ST_INTERNAL);
}

template <int HD, bool PAIR, bool F8>
static int tree_tc_launch_as(const dynakv_row_cache* cache, const TreeArgs& a, int sms, cudaStream_t st) {
    using C = TcTree<HD, PAIR, F8>;
    CUtensorMap mk = {}, mv = {};              // FP8 rows are fetched by plain loads: that kernel looks at neither
    if (!F8 && (!tree_page_map(&mk, cache, cache->k, false) || !tree_page_map(&mv, cache, cache->v, false))) return DYNAKV_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_tree_tc<HD, PAIR, F8>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    if (launch_pdl(k_tree_tc<HD, PAIR, F8>, dim3(sms), dim3(C::threads), C::smem, st, mk, mv, a) != cudaSuccess) return DYNAKV_ERR_CUDA;
    return tree_merge_launch(HD, C::rows, false, a, sms, st);
}
template <int HD>
static int tree_tc_launch_hd(const dynakv_row_cache* cache, int rows, const TreeArgs& a, int sms, cudaStream_t st) {
    if (cache->kv_dtype == DYNAKV_FP8) return rows == 128 ? tree_tc_launch_as<HD, false, true>(cache, a, sms, st) : tree_tc_launch_as<HD, true, true>(cache, a, sms, st);
    return rows == 128 ? tree_tc_launch_as<HD, false, false>(cache, a, sms, st) : tree_tc_launch_as<HD, true, false>(cache, a, sms, st);
}

int tree_tc_launch(const dynakv_row_cache* cache, int rows, const TreeArgs& a, int sms, cudaStream_t st) {
    return cache->head_dim == 128 ? tree_tc_launch_hd<128>(cache, rows, a, sms, st) : tree_tc_launch_hd<64>(cache, rows, a, sms, st);
}

}  // namespace dkv
