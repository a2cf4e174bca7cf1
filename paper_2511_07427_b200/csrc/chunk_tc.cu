// Attention of chunks on the tcgen05 tensor cores: bf16 and FP8 rows, tiles of 256 query rows (token, head of the group).
//
// One CTA per SM walks over its share of the stages (chunk_plan.cuh).  A stage is 128 rows of K and of V; two streams of 128 query rows
// work on every stage, each with its logits S and sums O in tensor memory, and take turns in the tensor pipe:
//   ... O0 += P0 V, S0 = Q0 K' | O1 += P1 V, S1 = Q1 K' | O0 += P0' V', ...
// so that one stream's softmax runs while the other's products do.  A stream's weights P replace its logits in place (bf16 pairs in the
// first half of the columns); the next logits overwrite them, in the tensor pipe's own order, after the products that read them.
//   warp 0 / warp 2      TMA loads of K / of V, one 32-row panel of 128 bytes per copy, 128-byte swizzle
//   warp 1               tcgen05.mma of both streams
//   warp 3               TMA loads of the next unit's queries, when the last logits of this one have been multiplied
//   warps 4-7 / 8-11     softmax of stream 0 / 1: a query row per thread
//   warps 12-15          FP8 rows only: they turn the rows, which warps 0 and 2 then fetch as they are, into bf16 stages
// Weights enter the products as bf16 (2^-8 of each): bf16 hi + lo, as the kernel for few rows has them, would add half to the tensor pipe's work, which here is
// what the power limit leaves time for.  The error of the results is 1.4 times that of rounding alone (2.3e-3 of their size against 1.7e-3).
//
// 4096 tokens over 16384 rows, 32 heads over 8 of 128 (962 GFLOP): 842 us in bursts (1142 TFLOP/s), 945 in a stream of them (1.70 GHz at the 1000 W
// limit; cuBLAS gets 1386 TFLOP/s there).  A stage takes 3800 cycles: 2048 in the tensor pipe (52 % busy), as many for the exponentials (52 %), the
// rest what a stream waits for the other's products and for barriers.  280 to 332 bytes a thread are spilled (FP8 rows: 396 to 596).  Tried and not kept: weights handed over in halves (830 -> 888 us), a part of the
// exponentials as polynomials on the FMA pipe (a quarter 832, a third 862 against 827: the power that this takes), waits that poll
// (876), logits read twice instead of kept (caps: 694 -> 912), two threads per query row (815 -> 932, caps 1265 -> 1879: 96 registers do not hold half a
// row), weights taken before the stage's maximum is known and thrown away if it moves (818 -> 847; caps on long rows 1265 -> 1150, but documents 166 -> 183
// and windows 268 -> 288).  A unit costs 4.8 us more than its stages, two stages' worth (CT_UNIT_COST).
// FP8 rows turned into bf16 in the kernel: 1330 us; with their conversion left out 990.
#include <cuda.h>
#include <float.h>

#include <type_traits>

#include "bulk_copy.cuh"
#include "chunk_again.cuh"
#include "chunk_plan.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"

namespace dkv {

constexpr int CT_CONVERT = 128;                                // FP8: threads that turn rows into bf16
constexpr float CT_LOG2E = 1.4426950408889634f, CT_LN2 = 0.6931471805599453f;
// The softmax's reference moves when the maximum has outgrown it by 2^24, so that O is rescaled next to never: weights have the range of
// fp32, and sums of 2^24 rows' weights times V stay below its end up to |V| = 2^79 (what does not is taken again).
constexpr float CT_LAZY = 24.f;

// ---------------------------------------------------------------------------------- the kernel

template <int HD, bool F8>
struct TcChunk {
    static constexpr int threads = 384 + (F8 ? CT_CONVERT : 0);
    static constexpr int panels = HD / 64;                     // 128-byte column panels of a row
    static constexpr int panel_bytes = 128 * 128;              // 128 rows of 128 bytes
    static constexpr int tile_bytes = panels * panel_bytes;
    static constexpr int stages = 2;                           // of K and V each
    static constexpr int raw_bytes = F8 ? CT_KEYS * HD : 0;    // FP8 rows as they come, one stage of K and of V, then their exponents
    static constexpr int exp_bytes = F8 ? CT_KEYS : 0;
    static constexpr int fixed = 32 * 8 + 8 * 4 + 16;
    static constexpr int smem = (2 + 2 * stages) * tile_bytes + 2 * (raw_bytes + exp_bytes) + fixed;
    static_assert(smem + 1024 <= 233472, "shared memory of an SM");
    // registers a thread: what the launch gives (64 K over all threads, in steps of 8) is shared out anew among the warpgroups
    static constexpr int regs_rest = F8 ? 64 : 104, regs_softmax = F8 ? 184 : 200, regs_convert = 80;
    static_assert(F8 ? 2 * regs_softmax + regs_rest + regs_convert <= 4 * 128 : 2 * regs_softmax + regs_rest <= 3 * 168, "registers of the launch");
    // kind::f16, fp32 accumulate, bf16 operands, M = 128
    static constexpr unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
    static constexpr unsigned idesc_qk = idesc | ((unsigned)(CT_KEYS >> 3) << 17);
    static constexpr unsigned idesc_pv = idesc | (1u << 16) | ((unsigned)(HD >> 3) << 17);      // B's contraction index is its outer one
    static constexpr int KFULL = 0, KEMPTY = stages, VFULL = 2 * stages, VEMPTY = 3 * stages, SFULL = 4 * stages, OFULL = SFULL + 2,
                         QFULL = OFULL + 2, QEMPTY = QFULL + 2, DRAIN = QEMPTY + 2, PFULL = DRAIN + 1, RAWEMPTY = PFULL + 2, RAWFULL = RAWEMPTY + 2, count = RAWFULL + 2;
    static_assert(count <= 32, "barrier block");
};

// 32 bytes in one store where the address allows.
__device__ __forceinline__ void store32(void* to, const unsigned (&p)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(to), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]), "r"(p[4]), "r"(p[5]), "r"(p[6]), "r"(p[7]) : "memory");
    } else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(p[0], p[1], p[2], p[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(p[4], p[5], p[6], p[7]);
    }
}

// A query row: what it sees, and how its logits become scores (log2 units).
struct ChunkRow {
    int lo, hi, place;
    float slope;
};
__device__ __forceinline__ int lds_s8(unsigned addr) {
    int v;
    asm volatile("ld.shared.s8 %0, [%1];\n" : "=r"(v) : "r"(addr));
    return v;
}
// 16 e4m3 values times 2^e as bf16 pairs (exact).
__device__ __forceinline__ void widen16(uint4 raw, int e, unsigned (&o)[8]) {
    const float sc = pow2f(e);
    const float2 sc2 = make_float2(sc, sc);
    const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int x = 0; x < 4; x++) {
        unsigned lo, hi;
        e4m3x4_to_f16x2(w[x], lo, hi);
        const float2 y = mul2(__half22float2(*reinterpret_cast<const __half2*>(&lo)), sc2), z = mul2(__half22float2(*reinterpret_cast<const __half2*>(&hi)), sc2);
        o[2 * x] = pack_bf16(y.x, y.y);
        o[2 * x + 1] = pack_bf16(z.x, z.y);
    }
}
// What the scores need beside the factor and the mask.
enum { PLAIN = 0, BIASED = 1, CAPPED = 2 };
// tanh(y) / y as a polynomial of y^2 (interpolated at Chebyshev nodes; tanh is off by 1e-7 at most): for |y| <= 0.4, which is what a cap well above
// the logits gives, and for |y| <= 1.  The FMA pipe is what this costs, 5 and 9 instructions' worth per logit.  N pairs step by step: one after
// the other they would wait for their own results.
constexpr float CT_TANH_SHORT = 0.4f, CT_TANH_LONG = 1.f;
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
struct TanhShort { float k0, k1, k2, k3; };                    // x (k0 + k1 x^2 + k2 x^4 + k3 x^6) = f tanh(x s)
__device__ __forceinline__ TanhShort tanh_short(float s, float f) {
    const float z = s * s, k = s * f;
    return {k, -0.3333137333f * z * k, 0.1327115595f * (z * z) * k, -0.0475610755f * (z * z) * (z * k)};
}
template <int N>
__device__ __forceinline__ void tanh_short2(float2 (&x)[N], const TanhShort& k) {
    float2 z[N], p[N];
#pragma unroll
    for (int i = 0; i < N; i++) z[i] = mul2(x[i], x[i]);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma2(both(k.k3), z[i], both(k.k2));
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma2(p[i], z[i], both(k.k1));
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma2(p[i], z[i], both(k.k0));
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = mul2(p[i], x[i]);
}
template <int N>
__device__ __forceinline__ void tanh_long2(float2 (&x)[N], float s) {
    constexpr float c[8] = {1.f, -0.3333328068f, 0.1333219111f, -0.0538727380f, 0.0214699805f, -0.0079249460f, 0.0022876456f, -0.0003548834f};
    float2 z[N], p[N];
#pragma unroll
    for (int i = 0; i < N; i++) { x[i] = mul2(x[i], both(s)); z[i] = mul2(x[i], x[i]); p[i] = both(c[7]); }
#pragma unroll
    for (int k = 6; k >= 0; k--)
#pragma unroll
        for (int i = 0; i < N; i++) p[i] = fma2(p[i], z[i], both(c[k]));
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = mul2(p[i], x[i]);
}
// tanh(y) = 1 - 2 / (1 + e^2y) for any y: off by 2e-7 at most.
__device__ __forceinline__ float tanh_far(float y) { return fmaf(-2.f, __fdividef(1.f, 1.f + ex2(2.f * CT_LOG2E * (y > 40.f ? 40.f : y))), 1.f); }

// The CTA's segments once more, by the eight softmax warps (chunk_again.cuh).
template <int HD, bool F8>
__device__ __noinline__ void chunk_tc_again(const TreeArgs& a, const ChunkPlan& plan, int warp, int* shared) {
    const int step = 128 / a.G;
    ChunkWalk walk;
    walk.start(plan);
    for (ChunkSeg g; walk.next(a.Hk, 2 * step, plan, g);) {
        const AgainSeg part = {g.seq, g.h, g.s0 * CT_KEYS, min(g.n, g.s1 * CT_KEYS), g.q0, g.T, g.n, CT_ROWS, g.first && g.last, (size_t)blockIdx.x * 2 + (g.first ? 1 : 0)};
        chunk_segment_again<HD, F8 ? DYNAKV_FP8 : DYNAKV_BF16, CT_ROWS, true, 8>(a, part, warp, shared,
            [&](int r) {
                const int mine = (r & 127) / a.G + (r >> 7) * step;
                return (r & 127) >= step * a.G || mine >= g.tokens ? -1ll : (long long)(g.q0 + g.tile * 2 * step + mine) * a.Hq + g.h * a.G + (r & 127) % a.G;
            }, [] { asm volatile("bar.sync 1, 256;\n" ::: "memory"); });
    }
}

template <int HD, bool F8, int MODE>
__global__ void __launch_bounds__((TcChunk<HD, F8>::threads), 1) k_chunk_tc(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                           const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TreeArgs a, const __grid_constant__ ChunkPlan plan) {
    using C = TcChunk<HD, F8>;
    constexpr int NS = C::stages;
    extern __shared__ __align__(1024) unsigned char ct_smem[];
    unsigned char* at = ct_smem + (2 + 2 * NS) * C::tile_bytes;
    const unsigned sRaw = tc_smem_u32(at); at += 2 * C::raw_bytes;                 // K, V
    const unsigned sExp = tc_smem_u32(at); at += 2 * C::exp_bytes;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(at); at += 32 * 8;
    volatile int* meta = reinterpret_cast<volatile int*>(at); at += 8 * 4;         // [stage number mod 8] bit per page: it was loaded
    volatile unsigned* s_tmem = reinterpret_cast<volatile unsigned*>(at);
    volatile int* s_abort = reinterpret_cast<volatile int*>(at + 4);
    volatile int* s_odd = s_abort + 1;                                             // rows are to be taken again
    const unsigned sQ = tc_smem_u32(ct_smem);
    auto sK = [&](int st) { return sQ + (2 + st) * C::tile_bytes; };
    auto sV = [&](int st) { return sQ + (2 + NS + st) * C::tile_bytes; };
    const unsigned bar0 = tc_smem_u32(bars);
    auto bar = [&](int i) { return bar0 + i * 8; };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (a.wide_fits) {                                         // both kernels are launched, and one of them has nothing to do
        pdl_wait();
        if (*a.wide_fits != (F8 ? 0 : 1)) return;
    }
    if (tid == 0) {
        for (int i = 0; i < C::count; i++) {
            const bool full = (i >= C::KFULL && i < C::KEMPTY) || (i >= C::VFULL && i < C::VEMPTY);
            tc_mbar_init(bar(i), (full && F8) || (i >= C::PFULL && i < C::RAWFULL) ? 4 : 1);             // 4: warps
        }
        *s_abort = 0; *s_odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tc_smem_u32((const void*)s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    if (tid < 256 && (tid & 127) >= 128 / a.G * a.G) {         // rows that no query is loaded into
#pragma unroll
        for (int c = 0; c < HD / 8; c++) sts16(sQ + (tid >> 7) * C::tile_bytes + (c >> 3) * C::panel_bytes + (tid & 127) * 128 + (c & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
        tt_proxy_fence();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *s_tmem;
    pdl_wait();                                                // from here on the results of earlier kernels are read
    pdl_trigger();
    const int tokens = tile_tokens(a.G);
    ChunkWalk walk;
    walk.start(plan);
    ChunkSeg g = {};
    auto give_up = [&]() { *s_abort = 1; };
    // pages of stage s of the walk's segment that exist and are known to the table, as bits; ids by lane (4 lanes)
    auto page_of = [&](int s) {
        int id = -1;
        const int pg = s * CT_PAGES + lane;
        if (lane < CT_PAGES && pg * PAGE < g.n) {
            id = chunk_page(a, g.seq, pg);
            if (id < 0) tree_status(a, DYNAKV_ST_BOUNDS);
        }
        return id;
    };

    if (warp < 4) {
        regs_down<C::regs_rest>();
        if (warp == 0 || warp == 2) {
            // =============================== loads: warp 0 K, warp 2 V ===============================
            const bool is_v = warp == 2;
            const CUtensorMap* map = is_v ? &map_v : &map_k;
            constexpr int RING = F8 ? 1 : NS;
            const int full = F8 ? C::RAWFULL + is_v : is_v ? C::VFULL : C::KFULL, empty = F8 ? C::RAWEMPTY + is_v : is_v ? C::VEMPTY : C::KEMPTY;
            int n = 0;                                         // stage number in the CTA
            bool ok = true;
            while (ok && walk.next(a.Hk, tokens, plan, g)) {
                int id = page_of(g.s0);
                for (int s = g.s0; s < g.s1 && ok; s++, n++) {
                    const int st = n % RING, use = n / RING, now = id;
                    if (s + 1 < g.s1) id = page_of(s + 1);
                    const int bits = (int)__ballot_sync(0xffffffffu, now >= 0);
                    int page[CT_PAGES];
#pragma unroll
                    for (int x = 0; x < CT_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, now, x);
                    if (lane == 0) {
                        ok = !*s_abort && (use == 0 || mbar_wait(bar(empty + st), (unsigned)(use - 1) & 1u));
                        if (ok) {
                            if (!is_v) meta[n & 7] = bits;
                            if (bits) tc_mbar_expect_tx(bar(full + st), __popc(bits) * PAGE * (F8 ? HD + 1 : HD * 2));
                            else tc_mbar_arrive(bar(full + st));
                            const unsigned dst = F8 ? sRaw + is_v * C::raw_bytes : is_v ? sV(st) : sK(st);
#pragma unroll
                            for (int x = 0; x < CT_PAGES; x++) {
                                if (page[x] < 0) continue;
                                const int r = (page[x] * a.Hk + g.h) * PAGE;
                                if constexpr (F8) {
                                    tt_load(dst + x * PAGE * HD, map, r, 0, bar(full));
                                    bulk_g2s(sExp + is_v * C::exp_bytes + x * PAGE, (is_v ? a.vexp : a.kexp) + r, PAGE, bar(full));
                                } else {
#pragma unroll
                                    for (int q = 0; q < C::panels; q++) tt_load(dst + q * C::panel_bytes + x * PAGE * 128, map, r, q, bar(full + st));
                                }
                            }
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                }
            }
            if (!ok && lane == 0) {
                give_up();
                // stage n - 1 was not issued; let the copies of the ones before it land before the block ends
                for (int x = max(0, n - 1 - RING); x < n - 1; x++) mbar_wait(bar(full + x % RING), (unsigned)(x / RING) & 1u);
            }
        } else if (warp == 3) {
            // =============================== queries ===============================
            // A stream's rows are the heads of the group of 128 / G tokens; tokens behind the chunk's last come along and are not used.
            const int step = tokens / 2;
            int segs[2] = {0, 0};
            bool ok = true;
            while (ok && walk.next(a.Hk, tokens, plan, g)) {
                for (int s = 0; s < (g.tokens > step ? 2 : 1) && ok; s++, __syncwarp()) {
                    if (lane == 0) {
                        ok = !*s_abort && (segs[s] == 0 || mbar_wait(bar(C::QEMPTY + s), (unsigned)(segs[s] - 1) & 1u));
                        if (ok) {
                            tc_mbar_expect_tx(bar(C::QFULL + s), step * a.G * HD * 2);
#pragma unroll
                            for (int q = 0; q < C::panels; q++)
                                tt_load3(sQ + s * C::tile_bytes + q * C::panel_bytes, &map_q, q * 64, g.h * a.G, g.q0 + g.tile * 2 * step + s * step, bar(C::QFULL + s));
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                    if (ok) segs[s]++;
                }
            }
            if (!ok && lane == 0) {
                give_up();
                for (int s = 0; s < 2; s++) if (segs[s] > 0) mbar_wait(bar(C::QFULL + s), (unsigned)(segs[s] - 1) & 1u);     // copies under way land first
            }
        } else if (warp == 1) {
            // =============================== MMAs ===============================
            // The whole warp walks and waits, one elected lane issues.
            int n = 0, u[2] = {0, 0}, segs[2] = {0, 0};        // stages so far; stages and segments of a stream so far
            bool ok = true;
            const unsigned long long dq[2] = {tc_panel_desc(sQ), tc_panel_desc(sQ + C::tile_bytes)}, dk = tc_panel_desc(sK(0)), dv = tc_rows_desc(sV(0), C::panel_bytes);
            auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
            while (ok && walk.next(a.Hk, tokens, plan, g)) {
                const int stages = g.s1 - g.s0, active = g.tokens > tokens / 2 ? 2 : 1;
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
                        if (j + 1 == stages) tc_commit(bar(C::QEMPTY + s));
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
        // A thread takes the same 16 bytes of every RPP-th row of a stage, as the TMA has put them, and stores them where it would put
        // bf16 rows (exactly: e4m3 times a power of two is a bf16 value).
        regs_down<C::regs_convert>();
        constexpr int CPR = HD / 16, RPP = CT_CONVERT / CPR, NP = CT_KEYS / RPP;
        const int ct = tid - 384, chunk = ct % CPR, row0 = ct / CPR;
        int n = 0;
        bool ok = true;
        auto wait = [&](int b, int phase) { ok = ok && mbar_wait(bar(b), (unsigned)phase & 1u); ok = __all_sync(0xffffffffu, ok); };
        while (ok && walk.next(a.Hk, tokens, plan, g)) {
            for (int s = g.s0; s < g.s1 && ok; s++, n++) {
                const int st = n % NS, use = n / NS;
#pragma unroll 1
                for (int kv = 0; kv < 2; kv++) {
                    wait(C::RAWFULL + kv, n);
                    if (use > 0) wait((kv ? C::VEMPTY : C::KEMPTY) + st, use - 1);
                    if (!ok) break;
                    const unsigned dst = kv ? sV(st) : sK(st), from = sRaw + kv * C::raw_bytes, exps = sExp + kv * C::exp_bytes;
#pragma unroll
                    for (int i = 0; i < NP; i++) {
                        const int row = i * RPP + row0;
                        const uint4 raw = lds16(from + row * HD + ((HD == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3)) << 4));
                        unsigned o[8];
                        widen16(raw, lds_s8(exps + row), o);
                        const unsigned to = dst + (chunk >> 2) * C::panel_bytes + row * 128, ch = (2 * chunk) & 7;
                        sts16(to + ((ch ^ (row & 7)) << 4), make_uint4(o[0], o[1], o[2], o[3]));
                        sts16(to + (((ch + 1) ^ (row & 7)) << 4), make_uint4(o[4], o[5], o[6], o[7]));
                    }
                    tt_proxy_fence();
                    __syncwarp();
                    if (lane == 0) { tc_mbar_arrive(bar(C::RAWEMPTY + kv)); tc_mbar_arrive(bar((kv ? C::VFULL : C::KFULL) + st)); }
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
        const int step = tokens / 2, my_token = row / a.G + s * step, my_head = row % a.G;          // token of the tile
        const float qs = a.scale * (MODE == CAPPED ? 1.f / a.cap : CT_LOG2E);                      // PLAIN: positive
        const float top = a.cap * CT_LOG2E;
        const TanhShort k_short = tanh_short(qs, top);
        // where the powers leave fp32's range: not taken
        const bool powers = fabsf(qs) > 1e-6f && fabsf(k_short.k0) + fabsf(k_short.k1) + fabsf(k_short.k2) + fabsf(k_short.k3) <= FLT_MAX;
        const float short_range = powers ? CT_TANH_SHORT / fabsf(qs) : -1.f;
        const bool wide = ((uintptr_t)a.out & 31) == 0;
        int n = 0, u = 0, seg = 0;
        bool dead = false, cut_end = false;
        auto wait = [&](int b, int phase) {
            if (!dead && !mbar_wait(bar(b), (unsigned)phase & 1u)) { dead = true; give_up(); }
            dead = __any_sync(0xffffffffu, dead);
        };
        while (walk.next(a.Hk, tokens, plan, g)) {
            const int stages = g.s1 - g.s0, t = row < step * a.G && my_token < g.tokens ? g.tile * 2 * step + my_token : -1;
            if (s == 1 && g.tokens <= step) {                  // no rows for this stream
                n += stages;
                continue;
            }
            const size_t q_row = (size_t)(g.q0 + max(t, 0)) * a.Hq + g.h * a.G + my_head;
            ChunkRow w = {0, g.n, g.n - g.T + max(t, 0), 0.f};
            if (t >= 0) chunk_sees(a, g.q0 + t, w.place, g.n, w.lo, w.hi);
            if (MODE != PLAIN && a.slopes) w.slope = a.slopes[g.h * a.G + my_head] * CT_LOG2E;
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
                    // Which rows of the stage this query sees, and (none) which pages nobody in the warp does: those are left out
                    const bool edge = __any_sync(0xffffffffu, w.lo > key0 || w.hi < key0 + CT_KEYS) || have != (1 << CT_PAGES) - 1;
                    unsigned win[4] = {~0u, ~0u, ~0u, ~0u}, none = 0u;
                    if (edge) {
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const int z = max(w.lo - key0 - c * 32, 0), y = ((have >> c) & 1) ? min(w.hi - key0 - c * 32, 32) : 0;
                            win[c] = z >= y ? 0u : (y == 32 ? ~0u : (1u << y) - 1u) & ~((1u << z) - 1u);
                        }
                    }
                    float f = qs;                              // what is left to do to the logits
                    if constexpr (MODE == CAPPED) {
                        if (edge) {                            // what is not seen has no say in which of the tanh is taken: it may be anything
#pragma unroll
                            for (int e = 0; e < CT_KEYS; e++) if (!((win[e >> 5] >> (e & 31)) & 1u)) x[e >> 5][e & 31] = 0u;
                        }
                        float hi = 0.f;
#pragma unroll
                        for (int e = 0; e < CT_KEYS; e += 2) hi = tt_max3(hi, fabsf(__uint_as_float(x[e >> 5][e & 31])), fabsf(__uint_as_float(x[e >> 5][(e & 31) + 1])));
                        hi = t < 0 ? 0.f : hi;                 // nor have rows that do not exist
                        auto groups = [&](auto work) {
                            constexpr int N = 8;
#pragma unroll
                            for (int b = 0; b < CT_KEYS; b += 2 * N) {
                                float2 y[N];
#pragma unroll
                                for (int e = 0; e < N; e++) y[e] = make_float2(__uint_as_float(x[(b + 2 * e) >> 5][(b + 2 * e) & 31]), __uint_as_float(x[(b + 2 * e) >> 5][(b + 2 * e + 1) & 31]));
                                work(y);
#pragma unroll
                                for (int e = 0; e < N; e++) { x[(b + 2 * e) >> 5][(b + 2 * e) & 31] = __float_as_uint(y[e].x); x[(b + 2 * e) >> 5][(b + 2 * e + 1) & 31] = __float_as_uint(y[e].y); }
                            }
                        };
                        f = 1.f;
                        if (__all_sync(0xffffffffu, hi <= short_range)) groups([&](float2 (&y)[8]) { tanh_short2(y, k_short); });
                        else {
                            f = top;
                            if (__all_sync(0xffffffffu, hi * fabsf(qs) <= CT_TANH_LONG)) groups([&](float2 (&y)[8]) { tanh_long2(y, qs); });
                            else {
#pragma unroll
                                for (int e = 0; e < CT_KEYS; e++) x[e >> 5][e & 31] = __float_as_uint(tanh_far(__uint_as_float(x[e >> 5][e & 31]) * qs));
                            }
                        }
                    }
                    if (MODE == BIASED || (MODE == CAPPED && a.slopes)) {
                        const float2 f2 = both(f);
                        if (__all_sync(0xffffffffu, w.place >= key0 + CT_KEYS - 1)) {              // the distance falls from row to row
                            // a base for every 8 rows, and what the rows inside them add
                            float2 more[4];
#pragma unroll
                            for (int e = 0; e < 4; e++) more[e] = make_float2(w.slope * (float)(2 * e), w.slope * (float)(2 * e + 1));
#pragma unroll
                            for (int b = 0; b < CT_KEYS; b += 8) {
                                const float base = w.slope * (float)(key0 + b - w.place);
                                const float2 base2 = both(base);
#pragma unroll
                                for (int e = 0; e < 4; e++) {
                                    unsigned& lo = x[b >> 5][(b & 31) + 2 * e];
                                    unsigned& hi = x[b >> 5][(b & 31) + 2 * e + 1];
                                    const float2 y = fma2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), f2, add2(base2, more[e]));
                                    lo = __float_as_uint(y.x); hi = __float_as_uint(y.y);
                                }
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < CT_KEYS; e++) x[e >> 5][e & 31] = __float_as_uint(fmaf(__uint_as_float(x[e >> 5][e & 31]), f, -w.slope * fabsf((float)(w.place - key0 - e))));
                        }
                        f = 1.f;
                    }
                    if (edge) {
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            if (__all_sync(0xffffffffu, win[c] == ~0u)) continue;
                            if (__all_sync(0xffffffffu, win[c] == 0u)) none |= 1u << c;
#pragma unroll
                            for (int e = 0; e < 32; e++) if (!((win[c] >> e) & 1u)) x[c][e] = 0xff800000u;
                        }
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int e = 0; e < CT_KEYS; e += 2) m4[(e >> 1) & 3] = tt_max3(m4[(e >> 1) & 3], __uint_as_float(x[e >> 5][e & 31]), __uint_as_float(x[e >> 5][(e & 31) + 1]));
                    const float mx = tt_max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]) * f;
                    const bool move = mx > m + CT_LAZY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = move ? mx : m, down = to == -INFINITY ? 1.f : ex2(m - to);
                        const bool carry = move && l > 0.f;    // without weights so far O is zero
                        m = to; l *= down;
                        if (__any_sync(0xffffffffu, carry)) {
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
                    const float2 f2 = both(f), ref2 = make_float2(-ref, -ref);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    auto weights = [&](int c) {
                        unsigned p[16];
#pragma unroll
                        for (int e = 0; e < 16; e++) {
                            float2 y = fma2(make_float2(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), f2, ref2);
                            y = make_float2(ex2(y.x), ex2(y.y));
                            sum[e & 1] = add2(sum[e & 1], y);
                            p[e] = pack_bf16(y.x, y.y);
                        }
                        tc_st16(tS + c * 16, p);
                    };
                    if (none == 0u) {                          // one run of instructions without a branch
#pragma unroll
                        for (int c = 0; c < 4; c++) weights(c);
                    } else {
                        const unsigned zero[16] = {};
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            if ((none >> c) & 1u) tc_st16(tS + c * 16, zero);
                            else weights(c);
                        }
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
                bool wild = false;
#pragma unroll 1
                for (int c = 0; c < HD / 32; c++) {
                    float o[32];
                    unsigned v[32];
                    tc_ld32(tO + c * 32, v);
                    tc_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; e++) { o[e] = __uint_as_float(v[e]); wild |= far_out(o[e]); }
                    if (t >= 0) {
                        if (whole) {
                            __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(a.out) + q_row * HD + c * 32;
#pragma unroll
                            for (int e = 0; e < 2; e++) {
                                unsigned p[8];
#pragma unroll
                                for (int i = 0; i < 8; i++) p[i] = pack_bf16(o[16 * e + 2 * i] * norm, o[16 * e + 2 * i + 1] * norm);
                                store32(to + 16 * e, p, wide);
                            }
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
                    if (wild && is_number(l)) *s_odd = 1;
                }
            }
            tc_fence_before();                                 // O has been read: the next segment's products may overwrite it
            if (g.last && !g.first) {
                cut_end = true;
                if (tid == 128) {
                    int* d = a.desc + (size_t)blockIdx.x * 8;
                    int c = blockIdx.x;
                    while (c > 0 && plan.starts[c].at > g.unit_start) c--;
                    d[DESC_FIRST] = c;
                    d[DESC_Q0] = g.q0 + g.tile * 2 * step; d[DESC_T] = g.tokens; d[DESC_H] = g.h;
                }
            }
        }
        if (tid == 128) a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
        // ---- all is done: rows whose sums are no numbers are taken again
        asm volatile("bar.sync 1, 256;\n" ::: "memory");
        if (*s_odd && !*s_abort) chunk_tc_again<HD, F8>(a, plan, warp - 4, reinterpret_cast<int*>(ct_smem));
    }
    // ---- everyone meets here, on every path; then the allocating warp frees the tensor memory
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && *s_abort) tree_status(a, DYNAKV_ST_INTERNAL);
}

// Merges the records of the units that were cut: block (x = CTA in which the unit ends, y = 16 columns), a thread per row.
template <int HD>
__global__ void __launch_bounds__(CT_ROWS) k_chunk_merge(const TreeArgs a) {
    pdl_wait();
    const int* d = a.desc + (size_t)blockIdx.x * 8;
    if (!d[DESC_VALID]) return;
    const int step = 128 / a.G, rl = threadIdx.x, row = rl & 127, t = (rl >> 7) * step + row / a.G, c0 = d[DESC_FIRST], n = blockIdx.x - c0 + 1;
    if (row >= step * a.G || t >= d[DESC_T]) return;
    auto slot = [&](int i) { return (size_t)(c0 + i) * 2 + (i == 0 ? 1 : 0); };
    const float4* acc = reinterpret_cast<const float4*>(a.acc) + (size_t)blockIdx.y * 4 * CT_ROWS + rl;
    float m = -INFINITY, l = 0.f;
    float4 o[4];
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < n; i++) {
        const float2 x = a.ml[slot(i) * CT_ROWS + rl];
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = acc[(slot(i) * (HD / 4) + e) * CT_ROWS];
        const float to = fmaxf(m, x.x), ref = to == -INFINITY ? 0.f : to, f0 = ex2(m - ref), f1 = ex2(x.x - ref);
        m = to;
        l = l * f0 + x.y * f1;
#pragma unroll
        for (int e = 0; e < 4; e++)
            o[e] = make_float4(o[e].x * f0 + v[e].x * f1, o[e].y * f0 + v[e].y * f1, o[e].z * f0 + v[e].z * f1, o[e].w * f0 + v[e].w * f1);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const size_t at = (size_t)(d[DESC_Q0] + t) * a.Hq + d[DESC_H] * a.G + row % a.G;
    uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at * HD + blockIdx.y * 16);
#pragma unroll
    for (int e = 0; e < 4; e += 2)
        out[e / 2] = make_uint4(pack_bf16(o[e].x * f, o[e].y * f), pack_bf16(o[e].z * f, o[e].w * f), pack_bf16(o[e + 1].x * f, o[e + 1].y * f), pack_bf16(o[e + 1].z * f, o[e + 1].w * f));
    if (a.lse && blockIdx.y == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * CT_LN2;
}

// ---------------------------------------------------------------------------------- FP8 rows as bf16
//
// Every tile of a sequence reads the same rows, and what turns a stage into bf16 inside the kernel competes with its softmax for the same
// pipes: 4096 tokens over 16384 rows, 8 KV heads, take 1330 us that way, 826 as bf16 rows.  So from three tiles per sequence on (two would break
// even) the stages that any tile needs are turned once, into the workspace, sequence by sequence.  Block (x: every gridDim.x-th stage, y = KV head, z = sequence).
constexpr int CW_THREADS = 256, CW_BLOCKS = 8192;

template <int HD>
__global__ void __launch_bounds__(CW_THREADS) k_chunk_widen(const TreeArgs a, const ChunkPlan p, uint4* k_out, uint4* v_out) {
    constexpr int CPR = HD / 16, RPP = CW_THREADS / CPR, NP = CT_KEYS / RPP;               // 16-byte chunks of a row, rows and passes
    const int h = blockIdx.y, seq = blockIdx.z, tid = threadIdx.x, chunk = tid % CPR, row0 = tid / CPR;
    pdl_wait();
    pdl_trigger();
    const int t0 = p.first[seq], t1 = p.first[seq + 1], n = t0 < t1 ? p.tiles[t0].n : 0;
    if (!*p.wide_fits) return;
    const int base = p.wide_base[seq];
    for (int stage = blockIdx.x; stage * CT_KEYS < n; stage += gridDim.x) {
        bool need = false;
        for (int i = t0 + tid; i < t1; i += CW_THREADS) { const ChunkTile& t = p.tiles[i]; need |= t.from <= stage && stage < t.from + t.stages; }
        if (!__syncthreads_or(need)) continue;
        uint4 raw[2][NP];
        int ex[2][NP];
        size_t to[NP];
        bool there[NP];
#pragma unroll
        for (int i = 0; i < NP; i++) {
            const int row = i * RPP + row0, column = stage * CT_PAGES + row / PAGE, page = column * PAGE < n ? chunk_page(a, seq, column) : -1;
            there[i] = page >= 0;
            const size_t r = ((size_t)(there[i] ? page : 0) * a.Hk + h) * PAGE + row % PAGE;
            to[i] = ((size_t)(base + column) * a.Hk + h) * PAGE + row % PAGE;
            raw[0][i] = __ldg(reinterpret_cast<const uint4*>(a.kpool + r * HD) + chunk); ex[0][i] = __ldg(a.kexp + r);
            raw[1][i] = __ldg(reinterpret_cast<const uint4*>(a.vpool + r * HD) + chunk); ex[1][i] = __ldg(a.vexp + r);
        }
#pragma unroll
        for (int kv = 0; kv < 2; kv++)
#pragma unroll
            for (int i = 0; i < NP; i++) {
                unsigned o[8];
                widen16(raw[kv][i], ex[kv][i], o);
                uint4* out = (kv ? v_out : k_out) + to[i] * (HD / 8) + 2 * chunk;
                if (there[i]) { out[0] = make_uint4(o[0], o[1], o[2], o[3]); out[1] = make_uint4(o[4], o[5], o[6], o[7]); }
            }
    }
}

// ---------------------------------------------------------------------------------- host side

// q [tokens][heads][HD]: a box is 64 elements of a group's heads of a stream's tokens.
static bool chunk_query_map(CUtensorMap* map, const TreeArgs& a, int hd) {
    const tree_encode_fn enc = tree_encode();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)a.Hq, (cuuint64_t)a.n_tokens}, strides[2] = {(cuuint64_t)hd * 2, (cuuint64_t)a.Hq * hd * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)(128 / a.G)}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, bool F8, int MODE>
static int chunk_tc_launch_as(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    using C = TcChunk<HD, F8>;
    CUtensorMap mq, mk, mv;
    if (!chunk_query_map(&mq, a, HD) || !tree_page_map(&mk, cache, cache->k, false) || !tree_page_map(&mv, cache, cache->v, false)) return DYNAKV_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_chunk_tc<HD, F8, MODE>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    // the warpgroups' shares of the registers add up to what the launch gets, or the kernel would wait for them forever
    static const int regs = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, k_chunk_tc<HD, F8, MODE>) == cudaSuccess ? f.numRegs : 0;
    }();
    if (regs * (C::threads / 128) < 2 * C::regs_softmax + C::regs_rest + (F8 ? C::regs_convert : 0)) return DYNAKV_ERR_CUDA;
    return launch_pdl(k_chunk_tc<HD, F8, MODE>, dim3(sms), dim3(C::threads), C::smem, st, mq, mk, mv, a, plan) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}
template <int HD, bool F8>
static int chunk_tc_launch_mode(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    // PLAIN takes the largest product for the largest logit, and -infinity times the factor for what is not seen; BIASED multiplies first
    if (a.cap > 0.f) return chunk_tc_launch_as<HD, F8, CAPPED>(cache, a, plan, sms, st);
    return a.slopes || !(a.scale >= FLT_MIN) ? chunk_tc_launch_as<HD, F8, BIASED>(cache, a, plan, sms, st) : chunk_tc_launch_as<HD, F8, PLAIN>(cache, a, plan, sms, st);
}
template <int HD>
static int chunk_tc_launch_hd(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, void* wide, bool always, int sms, cudaStream_t st) {
    int rc = DYNAKV_OK;
    TreeArgs own = a;
    if (wide) {
        // FP8 rows turned into bf16 once, then the kernel of bf16 rows; where they may not all find room, that of FP8 rows behind it, of which one has the call
        dynakv_row_cache c = *cache;
        c.n_pages = plan.wide_pages;
        c.k = wide; c.v = reinterpret_cast<char*>(wide) + plan.wide_pages * chunk_wide_page(cache) / 2;
        c.k_exp = c.v_exp = nullptr; c.kv_dtype = DYNAKV_BF16;
        const int stages = (a.pages_per_seq + CT_PAGES - 1) / CT_PAGES;
        const dim3 grid(max(1, min(stages, CW_BLOCKS / a.Hk / a.n_seqs)), a.Hk, a.n_seqs);
        if (launch_pdl(k_chunk_widen<HD>, grid, dim3(CW_THREADS), 0, st, a, plan, reinterpret_cast<uint4*>(c.k), reinterpret_cast<uint4*>(c.v)) != cudaSuccess) return DYNAKV_ERR_CUDA;
        TreeArgs w = a;
        w.kpool = reinterpret_cast<const unsigned char*>(c.k); w.vpool = reinterpret_cast<const unsigned char*>(c.v);
        w.kexp = w.vexp = nullptr; w.wide_base = plan.wide_base;
        if (!always) own.wide_fits = w.wide_fits = plan.wide_fits;
        rc = chunk_tc_launch_mode<HD, false>(&c, w, plan, sms, st);
    }
    if (rc == DYNAKV_OK && !(wide && always)) rc = cache->kv_dtype == DYNAKV_FP8 ? chunk_tc_launch_mode<HD, true>(cache, own, plan, sms, st) : chunk_tc_launch_mode<HD, false>(cache, own, plan, sms, st);
    if (rc != DYNAKV_OK) return rc;
    return launch_pdl(k_chunk_merge<HD>, dim3(sms, HD / 16), dim3(CT_ROWS), 0, st, a) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

int chunk_tc_launch(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, void* wide, bool always, int sms, cudaStream_t st) {
    const int rc = chunk_plan_launch(a, plan, sms, {tile_tokens(a.G), CT_KEYS, CT_UNIT_COST, CT_WHOLE}, st);
    if (rc != DYNAKV_OK) return rc;
    return cache->head_dim == 128 ? chunk_tc_launch_hd<128>(cache, a, plan, wide, always, sms, st) : chunk_tc_launch_hd<64>(cache, a, plan, wide, always, sms, st);
}

}  // namespace dkv
