// Attention of chunks on the tcgen05 tensor cores: bf16 and FP8 rows, tiles of 256 query rows (token, head of the group).
//
// One CTA per SM walks over its share of the stages (chunk_plan.cuh).  A stage is 128 rows of K and of V; two streams of 128 query rows
// work on every stage, each with its logits S and sums O in tensor memory, and take turns in the tensor pipe:
//   ... O0 += P0 V, S0 = Q0 K' | O1 += P1 V, S1 = Q1 K' | O0 += P0' V', ...
// so that one stream's softmax runs while the other's products do.  A stream's weights P replace its logits in place (bf16 pairs in the
// first half of the columns); the next logits overwrite them, in the tensor pipe's own order, after the products that read them.
//   warp 0 / warp 2      TMA loads of K / of V, one 32-row panel of 128 bytes per copy, 128-byte swizzle
//   warp 1               tcgen05.mma of both streams
//   warps 4-7 / 8-11     softmax of stream 0 / 1: a query row per thread
//   warps 12-15          FP8 rows only: they fetch the rows and turn them into bf16 stages (warps 0 and 2 then rest)
// Weights enter the products as bf16 (2^-9 of each).
#include <cuda.h>
#include <float.h>

#include "bulk_copy.cuh"
#include "chunk_plan.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"

namespace dkv {

constexpr int CT_CONVERT = 128;                                // FP8: threads that load rows and convert them
constexpr float CT_LOG2E = 1.4426950408889634f, CT_LN2 = 0.6931471805599453f;
constexpr float CT_LAZY = 8.f;                                 // the softmax's reference moves when the maximum has outgrown it by 2^8

// ---------------------------------------------------------------------------------- the plan

constexpr int PLAN_THREADS = 1024;

__device__ __forceinline__ ChunkSeq chunk_seq(const TreeArgs& a, int b, bool report) {
    const SeqInfo s = seq_info<CT_ROWS, false>(a, b, report);
    return {s.q0, s.T, s.n, s.tiles};
}

__global__ void __launch_bounds__(PLAN_THREADS) k_chunk_plan(const TreeArgs a, const ChunkPlan p, int ctas, int min_stages, long long most) {
    __shared__ long long sums[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
    // ---- sequences, and where their tiles begin
    long long tiles = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        ChunkSeq s = {0, 0, 0, 0};
        if (b < a.n_seqs) s = chunk_seq(a, b, true);
        long long total, incl = scan(s.first, total);
        int count = s.first;
        if (tiles + total > most) {                            // ranges of q that overlap: the workspace has no room for more tiles than tokens make
            if (tiles + incl > most) { count = 0; s.T = 0; tree_status(a, DYNAKV_ST_BOUNDS); }
            incl = scan(count, total);
        }
        s.first = (int)(tiles + incl - count);
        if (b < a.n_seqs) p.seqs[b] = s;
        // the tiles' sequences: few sequences have many tiles, so a warp writes a sequence's
        for (int src = 0; src < 32; src++) {
            const int c = __shfl_sync(0xffffffffu, count, src), f = __shfl_sync(0xffffffffu, s.first, src);
            for (int i = lane; i < c; i += 32) { p.tiles[f + i].seq = b0 + warp * 32 + src; p.tiles[f + i].tile = i; }
        }
        tiles += total;
    }
    if (tid == 0) p.seqs[a.n_seqs].first = (int)tiles;
    __syncthreads();
    // ---- stages of every tile: a thread per tile, or a warp where the tokens' ranges have to be read
    const bool ranges = a.rows_from || a.rows_to;
    long long run = 0;
    for (int t0 = 0; t0 < tiles; t0 += PLAN_THREADS) {
        const int n_here = (int)min((long long)PLAN_THREADS, tiles - t0);
        if (ranges) {
            for (int i = warp; i < n_here; i += 32) {
                ChunkTile& t = p.tiles[t0 + i];
                const ChunkSeq s = p.seqs[t.seq];
                const int from = t.tile * CT_ROWS / a.G, to = min(s.T, ((t.tile + 1) * CT_ROWS + a.G - 1) / a.G);
                int lo = s.n, hi = 0;
                for (int x = from + lane; x < to; x += 32) {
                    int l, h;
                    chunk_sees(a, s.q0 + x, s.n - s.T + x, s.n, l, h);
                    if (l < h) { lo = min(lo, max(l, 0)); hi = max(hi, h); }
                }
                lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi);
                if (lane == 0) { t.from = lo < hi ? lo / CT_KEYS : 0; t.stages = lo < hi ? (hi + CT_KEYS - 1) / CT_KEYS - t.from : 1; }
            }
            __syncthreads();
        }
        long long mine = 0;
        if (tid < n_here) {
            ChunkTile& t = p.tiles[t0 + tid];
            if (!ranges) {
                const ChunkSeq s = p.seqs[t.seq];
                const int from = t.tile * CT_ROWS / a.G, to = min(s.T, ((t.tile + 1) * CT_ROWS + a.G - 1) / a.G), place = s.n - s.T;
                const int lo = a.window > 0 ? max(0, place + from + 1 - a.window) : 0, hi = place + to;
                t.from = lo < hi ? lo / CT_KEYS : 0;
                t.stages = lo < hi ? (hi + CT_KEYS - 1) / CT_KEYS - t.from : 1;
            }
            mine = t.stages;
        }
        long long total;
        const long long incl = scan(mine, total);
        if (tid < n_here) p.before[t0 + tid] = run + incl - mine;
        run += total;
    }
    if (tid == 0) p.before[tiles] = run;
    __syncthreads();
    // ---- where every CTA begins
    const long long W = run * a.Hk;
    const int C = (int)max(1ll, min((long long)ctas, W / min_stages));
    if (tid == 0) { p.total[0] = run; p.total[1] = C; }
    for (int c = tid; c < ctas; c += PLAN_THREADS) {
        ChunkStart st = {0, 0, 0, 0};
        const long long x = c < C ? mul_div(c, W, C) : W, end = c < C ? mul_div(c + 1, W, C) : W;
        if (x < end) {
            auto find = [&](long long y, int lo, int hi) {     // last tile of [lo, hi) with before <= y
                while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (p.before[mid] <= y) lo = mid; else hi = mid; }
                return lo;
            };
            const int any = find(x / a.Hk, 0, (int)tiles), b = p.tiles[any].seq, e0 = p.seqs[b].first, e1 = p.seqs[b + 1].first;
            const long long lead = p.before[e0], all = p.before[e1] - lead, off = x - lead * a.Hk;
            st.head = (int)(off / all);
            st.tile = find(lead + off - st.head * all, e0, e1);
            st.off = (int)(lead + off - st.head * all - p.before[st.tile]);
            st.left = (int)(end - x);
        }
        p.starts[c] = st;
    }
}

// ---------------------------------------------------------------------------------- the kernel

template <int HD, bool F8>
struct TcChunk {
    static constexpr int threads = 384 + (F8 ? CT_CONVERT : 0);
    static constexpr int panels = HD / 64;                     // 128-byte column panels of a row
    static constexpr int panel_bytes = 128 * 128;              // 128 rows of 128 bytes
    static constexpr int tile_bytes = panels * panel_bytes;
    static constexpr int stages = 2;                           // of K and V each
    static constexpr int fixed = 32 * 8 + 8 * 4 + 16;
    static constexpr int smem = (2 + 2 * stages) * tile_bytes + fixed;
    static_assert(smem + 1024 <= 233472, "shared memory of an SM");
    // registers a thread: what the launch gives (64 K over all threads, in steps of 8) is shared out anew among the warpgroups
    static constexpr int regs_rest = F8 ? 64 : 104, regs_softmax = F8 ? 184 : 200, regs_convert = 80;
    static_assert(F8 ? 2 * regs_softmax + regs_rest + regs_convert <= 4 * 128 : 2 * regs_softmax + regs_rest <= 3 * 168, "registers of the launch");
    // kind::f16, fp32 accumulate, bf16 operands, M = 128
    static constexpr unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
    static constexpr unsigned idesc_qk = idesc | ((unsigned)(CT_KEYS >> 3) << 17);
    static constexpr unsigned idesc_pv = idesc | (1u << 16) | ((unsigned)(HD >> 3) << 17);      // B's contraction index is its outer one
    static constexpr int KFULL = 0, KEMPTY = stages, VFULL = 2 * stages, VEMPTY = 3 * stages, SFULL = 4 * stages, PFULL = SFULL + 2,
                         OFULL = PFULL + 2, QFULL = OFULL + 2, DRAIN = QFULL + 2, count = DRAIN + 1;
    static_assert(count <= 32, "barrier block");
};

template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(N)); }

// A query row: what it sees, and how its logits become scores (log2 units).
struct ChunkRow {
    int lo, hi, place;
    float slope;
};
__device__ __forceinline__ float chunk_score(const TreeArgs& a, const ChunkRow& w, float x, int key) {
    if (a.cap > 0.f) x = a.cap * CT_LOG2E * tanhf(x);
    if (a.slopes) x = fmaf(-w.slope, fabsf((float)(w.place - key)), x);
    return x;
}

// Columns [col, col + 32) of a row's sums taken again, row by row with the rows that it sees: a row of V with a value that is no number
// has reached them (0 * NaN where the row is not seen).
template <int HD, bool F8>
__device__ __noinline__ void chunk_again(const TreeArgs& a, const ChunkSeg& g, const ChunkRow& w, size_t q_row, float factor, float ref, int col, float* o) {
    constexpr int DT = F8 ? DYNAKV_FP8 : DYNAKV_BF16;
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD;
    for (int e = 0; e < 32; e++) o[e] = 0.f;
    for (int pos = max(w.lo, g.s0 * CT_KEYS); pos < min(w.hi, g.s1 * CT_KEYS); pos++) {
        const int page = a.page_table[(size_t)g.seq * a.pages_per_seq + pos / PAGE];
        if (page < 0 || page >= a.n_pages) continue;
        const long long key = ((long long)page * a.Hk + g.h) * PAGE + pos % PAGE;
        float d = 0.f;
        for (int e = 0; e < HD; e++) d = fmaf(__bfloat162float(q[e]), cache_elem<DT>(a.kpool, a.kexp, key, HD, e), d);
        const float x = ex2(chunk_score(a, w, d * factor, pos) - ref);
        for (int e = 0; e < 32; e++) o[e] = fmaf(x, cache_elem<DT>(a.vpool, a.vexp, key, HD, col + e), o[e]);
    }
}

template <int HD, bool F8, bool MODS>
__global__ void __launch_bounds__((TcChunk<HD, F8>::threads), 1) k_chunk_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                           const __grid_constant__ TreeArgs a, const __grid_constant__ ChunkPlan plan) {
    using C = TcChunk<HD, F8>;
    constexpr int NS = C::stages;
    extern __shared__ __align__(1024) unsigned char ct_smem[];
    unsigned char* at = ct_smem + (2 + 2 * NS) * C::tile_bytes;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(at); at += 32 * 8;
    volatile int* meta = reinterpret_cast<volatile int*>(at); at += 8 * 4;         // [stage number mod 8] bit per page: it was loaded
    volatile unsigned* s_tmem = reinterpret_cast<volatile unsigned*>(at);
    volatile int* s_abort = reinterpret_cast<volatile int*>(at + 4);
    const unsigned sQ = tc_smem_u32(ct_smem);
    auto sK = [&](int st) { return sQ + (2 + st) * C::tile_bytes; };
    auto sV = [&](int st) { return sQ + (2 + NS + st) * C::tile_bytes; };
    const unsigned bar0 = tc_smem_u32(bars);
    auto bar = [&](int i) { return bar0 + i * 8; };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int i = 0; i < C::count; i++) {
            const bool full = (i >= C::KFULL && i < C::KEMPTY) || (i >= C::VFULL && i < C::VEMPTY);
            tc_mbar_init(bar(i), full && F8 ? CT_CONVERT / 32 : (i >= C::PFULL && i < C::OFULL) || (i >= C::QFULL && i < C::DRAIN) ? 4 : 1);
        }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tc_smem_u32((const void*)s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *s_tmem;
    pdl_wait();                                                // from here on the results of earlier kernels are read
    pdl_trigger();
    ChunkWalk walk;
    walk.start(plan);
    ChunkSeg g;
    auto give_up = [&]() { *s_abort = 1; };
    // pages of stage s of the walk's segment that exist and are known to the table, as bits; ids by lane (4 lanes)
    auto page_of = [&](int s) {
        int id = -1;
        const int pg = s * CT_PAGES + lane;
        if (lane < CT_PAGES && pg * PAGE < g.n) {
            id = a.page_table[(size_t)g.seq * a.pages_per_seq + pg];
            if (id < 0 || id >= a.n_pages) { id = -1; tree_status(a, DYNAKV_ST_BOUNDS); }
        }
        return id;
    };

    if (warp < 4) {
        regs_down<C::regs_rest>();
        if (!F8 && (warp == 0 || warp == 2)) {
            // =============================== loads: warp 0 K, warp 2 V ===============================
            const bool is_v = warp == 2;
            const CUtensorMap* map = is_v ? &map_v : &map_k;
            const int full = is_v ? C::VFULL : C::KFULL, empty = is_v ? C::VEMPTY : C::KEMPTY;
            int n = 0;                                         // stage number in the CTA
            bool ok = true;
            while (ok && walk.next(a, plan, g)) {
                int id = page_of(g.s0);
                for (int s = g.s0; s < g.s1 && ok; s++, n++) {
                    const int st = n % NS, use = n / NS, now = id;
                    if (s + 1 < g.s1) id = page_of(s + 1);
                    const int bits = (int)__ballot_sync(0xffffffffu, now >= 0);
                    int page[CT_PAGES];
#pragma unroll
                    for (int x = 0; x < CT_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, now, x);
                    if (lane == 0) {
                        ok = !*s_abort && (use == 0 || mbar_wait(bar(empty + st), (unsigned)(use - 1) & 1u));
                        if (ok) {
                            if (!is_v) meta[n & 7] = bits;
                            if (bits) tc_mbar_expect_tx(bar(full + st), __popc(bits) * PAGE * HD * 2);
                            else tc_mbar_arrive(bar(full + st));
                            const unsigned dst = is_v ? sV(st) : sK(st);
#pragma unroll
                            for (int x = 0; x < CT_PAGES; x++) {
                                if (page[x] < 0) continue;
#pragma unroll
                                for (int q = 0; q < C::panels; q++)
                                    tt_load(dst + q * C::panel_bytes + x * PAGE * 128, map, (page[x] * a.Hk + g.h) * PAGE, q, bar(full + st));
                            }
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                }
            }
            if (!ok && lane == 0) {
                give_up();
                // stage n - 1 was not issued; let the copies of the ones before it land before the block ends
                for (int x = max(0, n - 1 - NS); x < n - 1; x++) mbar_wait(bar(full + x % NS), (unsigned)(x / NS) & 1u);
            }
        } else if (warp == 1) {
            // =============================== MMAs ===============================
            // The whole warp walks and waits, one elected lane issues.
            int n = 0, u[2] = {0, 0}, segs[2] = {0, 0};        // stages so far; stages and segments of a stream so far
            bool ok = true;
            const unsigned long long dq[2] = {tc_panel_desc(sQ), tc_panel_desc(sQ + C::tile_bytes)}, dk = tc_panel_desc(sK(0)), dv = tc_rows_desc(sV(0), C::panel_bytes);
            auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
            while (ok && walk.next(a, plan, g)) {
                const int stages = g.s1 - g.s0, active = g.T * a.G - g.tile * CT_ROWS > 128 ? 2 : 1;
                auto logits = [&](int s, int j) {              // of stage j of the segment
                    const int st = (n + j) % NS;
                    if (s == 0) wait(C::KFULL + st, (n + j) / NS);
                    if (j == 0) { wait(C::QFULL + s, segs[s]); segs[s]++; }
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < HD / 16; k++) {
                            const unsigned off = ((k >> 2) * C::panel_bytes + (k & 3) * 32) >> 4;
                            tc_mma_f16(tmem + s * 128, dq[s] + off, dk + ((st * C::tile_bytes) >> 4) + off, C::idesc_qk, k > 0 ? 1u : 0u);
                        }
                        tc_commit(bar(C::SFULL + s));
                        if (s == active - 1) tc_commit(bar(C::KEMPTY + st));
                    }
                    __syncwarp();
                };
                for (int s = 0; s < active && ok; s++) logits(s, 0);
                for (int j = 0; j < stages && ok; j++) {
                    const int st = (n + j) % NS;
                    for (int s = 0; s < active && ok; s++) {
                        if (s == 0) wait(C::VFULL + st, (n + j) / NS);
                        wait(C::PFULL + s, u[s]);
                        if (!ok) break;
                        u[s]++;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < CT_KEYS / 16; k++)
                                tc_mma_f16_ta(tmem + 256 + s * 128, tmem + s * 128 + k * 8, dv + ((st * C::tile_bytes + k * 2048) >> 4), C::idesc_pv, j > 0 || k > 0 ? 1u : 0u);
                            if (s == active - 1) tc_commit(bar(C::VEMPTY + st));
                            if (j + 1 == stages) tc_commit(bar(C::OFULL + s));
                        }
                        __syncwarp();
                        if (j + 1 < stages) logits(s, j + 1);
                    }
                }
                n += stages;
            }
            if (!ok) {
                if (elect_one()) {
                    give_up();
                    tc_commit(bar(C::DRAIN));                  // whatever was issued ends before the tensor memory is freed
                }
                __syncwarp();
                mbar_wait(bar(C::DRAIN), 0u);
            }
        }
    } else if (F8 && warp >= 12) {
        // =============================== FP8 rows to bf16 stages ===============================
        // A thread takes the same 16 bytes of every RPP-th row of a stage.  K and V alternate: while one is converted (exactly: e4m3
        // times a power of two is a bf16 value) and stored where the TMA would have put it, the other's loads are under way.
        regs_down<C::regs_convert>();
        constexpr int CPR = HD / 16, RPP = CT_CONVERT / CPR, NP = CT_KEYS / RPP;
        const int ct = tid - 384, chunk = ct % CPR, row0 = ct / CPR;
        int n = 0;
        bool ok = true;
        auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
        while (ok && walk.next(a, plan, g)) {
            for (int s = g.s0; s < g.s1 && ok; s++, n++) {
                const int st = n % NS, use = n / NS, id = page_of(s);
                const int bits = (int)__ballot_sync(0xffffffffu, id >= 0);
                int page[CT_PAGES];
#pragma unroll
                for (int x = 0; x < CT_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, id, x);
#pragma unroll 1
                for (int kv = 0; kv < 2; kv++) {
                    const unsigned char* pool = kv ? a.vpool : a.kpool;
                    const signed char* exps = kv ? a.vexp : a.kexp;
                    uint4 raw[NP];
                    int ex[NP];
#pragma unroll
                    for (int i = 0; i < NP; i++) {
                        const int pg = page[i * RPP / PAGE];
                        const size_t r = ((size_t)(pg < 0 ? 0 : pg) * a.Hk + g.h) * PAGE + (i * RPP + row0) % PAGE;
                        raw[i] = pg >= 0 ? __ldg(reinterpret_cast<const uint4*>(pool + r * HD) + chunk) : make_uint4(0u, 0u, 0u, 0u);
                        ex[i] = pg >= 0 ? (int)__ldg(exps + r) : 0;
                    }
                    if (use > 0) wait((kv ? C::VEMPTY : C::KEMPTY) + st, use - 1);
                    if (!ok) break;
                    if (ct == 0 && kv == 0) meta[n & 7] = bits;
                    const unsigned dst = kv ? sV(st) : sK(st);
#pragma unroll
                    for (int i = 0; i < NP; i++) {
                        const int row = i * RPP + row0;
                        const float sc = pow2f(ex[i]);
                        const float2 sc2 = make_float2(sc, sc);
                        const unsigned w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                        unsigned o[8];
#pragma unroll
                        for (int x = 0; x < 4; x++) {
                            unsigned lo, hi;
                            e4m3x4_to_f16x2(w[x], lo, hi);
                            const float2 y = mul2(__half22float2(*reinterpret_cast<const __half2*>(&lo)), sc2), z = mul2(__half22float2(*reinterpret_cast<const __half2*>(&hi)), sc2);
                            o[2 * x] = pack_bf16(y.x, y.y);
                            o[2 * x + 1] = pack_bf16(z.x, z.y);
                        }
                        const unsigned to = dst + (chunk >> 2) * C::panel_bytes + row * 128, ch = (2 * chunk) & 7;
                        sts16(to + ((ch ^ (row & 7)) << 4), make_uint4(o[0], o[1], o[2], o[3]));
                        sts16(to + (((ch + 1) ^ (row & 7)) << 4), make_uint4(o[4], o[5], o[6], o[7]));
                    }
                    tt_proxy_fence();
                    __syncwarp();
                    if (lane == 0) tc_mbar_arrive(bar((kv ? C::VFULL : C::KFULL) + st));
                }
            }
        }
        if (!ok && lane == 0) give_up();
    } else {
        // =============================== softmax of one stream ===============================
        regs_up<C::regs_softmax>();
        const int s = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const unsigned lane_base = (unsigned)((warp & 3) * 32) << 16;
        const unsigned tS = tmem + s * 128 + lane_base, tO = tmem + 256 + s * 128 + lane_base;
        const bool flip = a.scale < 0.f;                       // q changes sign, so that the largest product is the largest logit
        // scale 0: q is taken as zero, so that a masked -inf stays one
        const float qs = a.scale == 0.f ? 1.f : fabsf(a.scale) * (MODS && a.cap > 0.f ? 1.f / a.cap : CT_LOG2E);
        int n = 0, u = 0, seg = 0;
        bool dead = false, cut_end = false;
        auto wait = [&](int b, int phase) {
            if (!dead && !mbar_wait(bar(b), (unsigned)phase & 1u)) { dead = true; give_up(); }
            dead = __any_sync(0xffffffffu, dead);
        };
        while (walk.next(a, plan, g)) {
            const int stages = g.s1 - g.s0, r = g.tile * CT_ROWS + s * 128 + row, t = r < g.T * a.G ? r / a.G : -1;
            if (s == 1 && g.T * a.G - g.tile * CT_ROWS <= 128) {           // no rows for this stream
                n += stages;
                continue;
            }
            const size_t q_row = (size_t)(g.q0 + max(t, 0)) * a.Hq + g.h * a.G + (t < 0 ? 0 : r - t * a.G);
            ChunkRow w = {0, g.n, g.n - g.T + max(t, 0), 0.f};
            if (t >= 0) chunk_sees(a, g.q0 + t, w.place, g.n, w.lo, w.hi);
            if (MODS && a.slopes && t >= 0) w.slope = a.slopes[g.h * a.G + r - t * a.G] * CT_LOG2E;
            // ---- Q: this thread's row; rows that do not exist as zeros
            {
                const unsigned to = sQ + s * C::tile_bytes + row * 128;
                const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + q_row * HD);
                uint4 v[HD / 8];                               // all loads before the first store
#pragma unroll
                for (int c = 0; c < HD / 8; c++) v[c] = t >= 0 && a.scale != 0.f ? src[c] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int c = 0; c < HD / 8; c++) {
                    if (flip) { v[c].x ^= 0x80008000u; v[c].y ^= 0x80008000u; v[c].z ^= 0x80008000u; v[c].w ^= 0x80008000u; }
                    sts16(to + (c >> 3) * C::panel_bytes + (((c & 7) ^ (row & 7)) << 4), v[c]);
                }
                tt_proxy_fence();
                __syncwarp();
                if (lane == 0) tc_mbar_arrive(bar(C::QFULL + s));
            }
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < stages; j++, u++) {
                const int key0 = (g.s0 + j) * CT_KEYS, st = (n + j) % NS;
                wait(C::SFULL + s, u);                         // the stream's products so far are done as well
                tc_fence_after();
                const int have = meta[(n + j) & 7];
                if (have != (1 << CT_PAGES) - 1 || key0 + CT_KEYS > g.n) {
                    // rows of V that no page holds, or past the sequence's end, must not reach the MMAs: a row per thread, by both streams
                    wait(C::VFULL + st, (n + j) / NS);
                    if (!dead && (key0 + row >= g.n || !((have >> (row / PAGE)) & 1))) {
#pragma unroll
                        for (int c = 0; c < HD / 8; c++) sts16(sV(st) + row * 128 + (c >> 3) * C::panel_bytes + (c & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
                        tt_proxy_fence();
                    }
                    __syncwarp();
                }
                if (!dead) {
                    unsigned x[4][32];
#pragma unroll
                    for (int c = 0; c < 4; c++) tc_ld32(tS + c * 32, x[c]);
                    tc_ld_wait();
                    float f = qs;                              // what is left to do to the logits
                    if constexpr (MODS) {
#pragma unroll
                        for (int e = 0; e < CT_KEYS; e++) x[e >> 5][e & 31] = __float_as_uint(chunk_score(a, w, __uint_as_float(x[e >> 5][e & 31]) * qs, key0 + e));
                        f = 1.f;
                    }
                    if (__any_sync(0xffffffffu, w.lo > key0 || w.hi < key0 + CT_KEYS) || have != (1 << CT_PAGES) - 1) {
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const int from = w.lo - key0 - c * 32, to = ((have >> c) & 1) ? w.hi - key0 - c * 32 : 0;
#pragma unroll
                            for (int e = 0; e < 32; e++) if (e < from || e >= to) x[c][e] = 0xff800000u;
                        }
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int e = 0; e < CT_KEYS; e += 2) m4[(e >> 1) & 3] = tt_max3(m4[(e >> 1) & 3], __uint_as_float(x[e >> 5][e & 31]), __uint_as_float(x[e >> 5][(e & 31) + 1]));
                    const float mx = tt_max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]) * f;
                    const bool move = mx > m + CT_LAZY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = move ? mx : m, down = to == -INFINITY ? 1.f : ex2(m - to);
                        m = to; l *= down;
                        if (j > 0) {
#pragma unroll 1
                            for (int c = 0; c < HD / 16; c++) {
                                unsigned o[16];
                                tc_ld16(tO + c * 16, o);
                                tc_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * down);
                                tc_st16(tO + c * 16, o);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    const float2 f2 = make_float2(f, f), ref2 = make_float2(-ref, -ref);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < CT_KEYS / 32; c++) {
                        unsigned p[16];
#pragma unroll
                        for (int e = 0; e < 16; e++) {
                            float2 y = fma2(make_float2(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), f2, ref2);
                            y = make_float2(ex2(y.x), ex2(y.y));
                            sum[e & 1] = add2(sum[e & 1], y);
                            p[e] = pack_bf16(y.x, y.y);
                        }
                        tc_st16(tS + c * 16, p);
                    }
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    tc_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_mbar_arrive(bar(C::PFULL + s));
            }
            n += stages;
            wait(C::OFULL + s, seg);
            seg++;
            tc_fence_after();
            // ---- the row, or its record
            const bool whole = g.first && g.last;
            const size_t slot = (size_t)blockIdx.x * 2 + (g.first ? 1 : 0);
            if (!dead) {
                const float norm = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
                for (int c = 0; c < HD / 32; c++) {
                    float o[32];
                    unsigned v[32];
                    tc_ld32(tO + c * 32, v);
                    tc_ld_wait();
                    bool wild = false;
#pragma unroll
                    for (int e = 0; e < 32; e++) { o[e] = __uint_as_float(v[e]); wild |= !(fabsf(o[e]) <= FLT_MAX); }
                    if (wild && t >= 0) {
                        float again[32];
                        chunk_again<HD, F8>(a, g, w, q_row, a.cap > 0.f ? a.scale / a.cap : a.scale * CT_LOG2E, m == -INFINITY ? 0.f : m, c * 32, again);
#pragma unroll
                        for (int e = 0; e < 32; e++) o[e] = again[e];
                    }
                    __syncwarp();
                    if (t >= 0) {
                        if (whole) {
                            uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + q_row * HD + c * 32);
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                to[e] = make_uint4(pack_bf16(o[8 * e] * norm, o[8 * e + 1] * norm), pack_bf16(o[8 * e + 2] * norm, o[8 * e + 3] * norm),
                                                   pack_bf16(o[8 * e + 4] * norm, o[8 * e + 5] * norm), pack_bf16(o[8 * e + 6] * norm, o[8 * e + 7] * norm));
                        } else {
                            // four columns of all rows side by side: the lanes' stores join
                            float4* to = reinterpret_cast<float4*>(a.acc) + (slot * (HD / 4) + c * 8) * CT_ROWS + s * 128 + row;
#pragma unroll
                            for (int e = 0; e < 8; e++) to[e * CT_ROWS] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    }
                }
                if (t >= 0) {
                    if (!whole) a.ml[slot * CT_ROWS + s * 128 + row] = make_float2(m, l);
                    else if (a.lse) a.lse[q_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * CT_LN2;
                }
            }
            tc_fence_before();                                 // O has been read: the next segment's products may overwrite it
            if (g.last && !g.first) {
                cut_end = true;
                if (tid == 128) {
                    int* d = a.desc + (size_t)blockIdx.x * 8;
                    d[DESC_FIRST] = range_owner(g.unit_start, plan.total[0] * a.Hk, (int)plan.total[1]);
                    d[DESC_Q0] = g.q0; d[DESC_T] = g.T; d[DESC_H] = g.h; d[DESC_RT] = g.tile;
                }
            }
        }
        if (tid == 128) a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
    }
    // ---- everyone meets here, on every path; then the allocating warp frees the tensor memory
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && *s_abort) tree_status(a, DYNAKV_ST_INTERNAL);
}

template <int HD, bool F8, bool MODS>
static int chunk_tc_launch_as(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    using C = TcChunk<HD, F8>;
    CUtensorMap mk = {}, mv = {};              // FP8 rows are fetched by plain loads: that kernel looks at neither
    if (!F8 && (!tree_page_map(&mk, cache, cache->k, false) || !tree_page_map(&mv, cache, cache->v, false))) return DYNAKV_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_chunk_tc<HD, F8, MODS>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    // the warpgroups' shares of the registers add up to what the launch gets, or the kernel would wait for them forever
    static const int regs = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, k_chunk_tc<HD, F8, MODS>) == cudaSuccess ? f.numRegs : 0;
    }();
    if (regs * (C::threads / 128) < 2 * C::regs_softmax + C::regs_rest + (F8 ? C::regs_convert : 0)) return DYNAKV_ERR_CUDA;
    const long long most = a.n_tokens * a.G / CT_ROWS + a.n_seqs;
    if (launch_pdl(k_chunk_plan, dim3(1), dim3(PLAN_THREADS), 0, st, a, plan, sms, 1, most) != cudaSuccess) return DYNAKV_ERR_CUDA;
    if (launch_pdl(k_chunk_tc<HD, F8, MODS>, dim3(sms), dim3(C::threads), C::smem, st, mk, mv, a, plan) != cudaSuccess) return DYNAKV_ERR_CUDA;
    return tree_merge_launch(HD, CT_ROWS, false, a, sms, st);
}
template <int HD, bool F8>
static int chunk_tc_launch_mods(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    return a.cap > 0.f || a.slopes ? chunk_tc_launch_as<HD, F8, true>(cache, a, plan, sms, st) : chunk_tc_launch_as<HD, F8, false>(cache, a, plan, sms, st);
}
template <int HD>
static int chunk_tc_launch_hd(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    return cache->kv_dtype == DYNAKV_FP8 ? chunk_tc_launch_mods<HD, true>(cache, a, plan, sms, st) : chunk_tc_launch_mods<HD, false>(cache, a, plan, sms, st);
}

// The plan's part of the workspace behind the records'.
size_t chunk_plan_space(int64_t n_tokens, int G, int n_seqs, int ctas, size_t at, char* base, ChunkPlan* plan) {
    const size_t tiles = (size_t)(n_tokens * G / CT_ROWS) + n_seqs;
    auto take = [&](size_t bytes) { const size_t x = (at + 15) / 16 * 16; at = x + bytes; return base + x; };
    ChunkPlan p;
    p.tiles = reinterpret_cast<ChunkTile*>(take(tiles * sizeof(ChunkTile)));
    p.before = reinterpret_cast<long long*>(take((tiles + 1) * 8));
    p.seqs = reinterpret_cast<ChunkSeq*>(take(((size_t)n_seqs + 1) * sizeof(ChunkSeq)));
    p.starts = reinterpret_cast<ChunkStart*>(take((size_t)ctas * sizeof(ChunkStart)));
    p.total = reinterpret_cast<long long*>(take(16));
    if (plan) *plan = p;
    return at;
}

int chunk_tc_launch(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    return cache->head_dim == 128 ? chunk_tc_launch_hd<128>(cache, a, plan, sms, st) : chunk_tc_launch_hd<64>(cache, a, plan, sms, st);
}

}  // namespace dkv
