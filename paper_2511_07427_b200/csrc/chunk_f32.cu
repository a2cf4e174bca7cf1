// Attention of chunks over fp32 rows: fp32 FMAs, tiles of 128 query rows (token, head of the group).
//
// fp32 products to fp32 accuracy have no tensor pipe, so the FMA pipe bounds the call: 4 d flops per pair of a query row and a row
// at 128 FMAs per cycle and SM.  What matters is then how few shared-memory reads feed them: a thread has 8 query rows times 4 keys of a stage of 64
// for the logits, and 8 query rows times 8 columns for the sums, in packed pairs.  16 lanes share a row, so a warp has 16 rows to itself, and
// warps meet only at the barriers of the one stage of K and of V: the next K comes in while this one's weights are multiplied with V, the next V
// while the next logits are.
//   warp 8         (with three that rest) TMA loads, a page of K or V per copy (128-byte swizzle: the 8 lanes of a 16-byte read meet in no bank)
//   warps 0-7      16 query rows each
// Work is shared out as for the tcgen05 kernel (chunk_plan.cuh).  Weights go through shared memory twice side by side, as the packed products want them.
// Measured: 2000 tokens of one prompt, 32 heads over 8 of 128, 825 us, 40 TFLOP/s; 3 x 777 with prefixes and distances, 8 heads of 64, 88 us, the FMA pipe busy
// 56 % of the time: two warps per scheduler wait for their own results and for reads of shared memory.  Rows of 128 spill 134 bytes.
#include <cuda.h>
#include <float.h>

#include "bulk_copy.cuh"
#include "chunk_again.cuh"
#include "chunk_plan.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"

namespace dkv {

constexpr float CF_LOG2E = 1.4426950408889634f, CF_LN2 = 0.6931471805599453f, CF_LAZY = 24.f;
constexpr int CF_WARPS = 8, CF_PAGES = CF_KEYS / PAGE;

template <int HD>
struct F32Chunk {
    static constexpr int threads = CF_WARPS * 32 + 128;        // a whole warpgroup for the loads, because registers are shared out by warpgroups
    static constexpr int regs_sums = 232, regs_loads = 40;
    static_assert(2 * regs_sums + regs_loads <= 3 * 168, "registers of the launch");
    static constexpr int row_bytes = HD * 4, page_bytes = PAGE * row_bytes, tile_bytes = CF_KEYS * row_bytes;
    static constexpr int q_bytes = CF_ROWS * row_bytes, p_bytes = CF_ROWS * CF_KEYS * 8;
    static constexpr int smem = 2 * tile_bytes + q_bytes + p_bytes + CF_ROWS * 16 + 8 * 8 + 16;
    static constexpr int cols = HD / 64;                       // 16-byte column chunks of a thread
    static_assert(smem + 1024 <= 233472, "shared memory of an SM");
};
// Byte offset of 16-byte chunk c of row r of a page, as the TMA swizzle placed it.
__device__ __forceinline__ int cf_chunk(int r, int c) { return (c >> 3) * (PAGE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4); }
__device__ __forceinline__ float2 lo2(uint4 v) { return make_float2(__uint_as_float(v.x), __uint_as_float(v.y)); }
__device__ __forceinline__ float2 hi2(uint4 v) { return make_float2(__uint_as_float(v.z), __uint_as_float(v.w)); }

// The CTA's segments once more, by the warps that have query rows (chunk_again.cuh).
template <int HD>
__device__ __noinline__ void chunk_f32_again(const TreeArgs& a, const ChunkPlan& plan, int warp, int* shared) {
    const int tokens = CF_ROWS / a.G;
    ChunkWalk walk;
    walk.start(plan);
    for (ChunkSeg g; walk.next(a.Hk, tokens, plan, g);) {
        const AgainSeg part = {g.seq, g.h, g.s0 * CF_KEYS, min(g.n, g.s1 * CF_KEYS), g.q0, g.T, g.n, g.tokens * a.G, g.first && g.last, (size_t)blockIdx.x * 2 + (g.first ? 1 : 0)};
        chunk_segment_again<HD, DYNAKV_F32, CF_ROWS, false, CF_WARPS>(a, part, warp, shared,
            [&](int r) { return (long long)(g.q0 + g.tile * tokens + r / a.G) * a.Hq + g.h * a.G + r % a.G; },
            [] { asm volatile("bar.sync 1, %0;\n" ::"n"(CF_WARPS * 32) : "memory"); });
    }
}

template <int HD>
__global__ void __launch_bounds__(F32Chunk<HD>::threads, 1) k_chunk_f32(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                         const __grid_constant__ TreeArgs a, const __grid_constant__ ChunkPlan plan) {
    using C = F32Chunk<HD>;
    extern __shared__ __align__(1024) unsigned char cf_smem[];
    const unsigned sK = smem_u32(cf_smem), sV = sK + C::tile_bytes, sQ = sV + C::tile_bytes, sP = sQ + C::q_bytes;
    int4* row_s = reinterpret_cast<int4*>(cf_smem + 2 * C::tile_bytes + C::q_bytes + C::p_bytes);       // of every query row: lo, hi, place, slope
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(row_s + CF_ROWS);
    volatile int* meta = reinterpret_cast<volatile int*>(bars + 4);                                      // [stage number mod 4] bit per page: it was loaded
    volatile int* s_abort = meta + 4;
    volatile int* s_odd = s_abort + 1;                                                                   // rows are to be taken again
    const unsigned KFULL = smem_u32(bars), KEMPTY = KFULL + 8, VFULL = KFULL + 16, VEMPTY = KFULL + 24;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        mbar_init(KFULL, 1); mbar_init(KEMPTY, CF_WARPS); mbar_init(VFULL, 1); mbar_init(VEMPTY, CF_WARPS);
        *s_abort = 0; *s_odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    __syncthreads();
    pdl_wait();                                                // from here on the results of earlier kernels are read
    pdl_trigger();
    const int tokens = CF_ROWS / a.G;
    ChunkWalk walk;
    walk.start(plan);
    ChunkSeg g = {};

    if (warp >= CF_WARPS) {
        regs_down<C::regs_loads>();
        if (warp > CF_WARPS) return;
        // =============================== loads ===============================
        int n = 0;
        bool ok = true;
        while (ok && walk.next(a.Hk, tokens, plan, g)) {
            for (int s = g.s0; s < g.s1 && ok; s++, n++) {
                int id = -1;
                const int pg = s * CF_PAGES + lane;
                if (lane < CF_PAGES && pg * PAGE < g.n) {
                    id = a.page_table[(size_t)g.seq * a.pages_per_seq + pg];
                    if (id < 0 || id >= a.n_pages) { id = -1; tree_status(a, DYNAKV_ST_BOUNDS); }
                }
                const int bits = (int)__ballot_sync(0xffffffffu, id >= 0);
                int page[CF_PAGES];
#pragma unroll
                for (int x = 0; x < CF_PAGES; x++) page[x] = __shfl_sync(0xffffffffu, id, x);
                if (lane == 0) {
                    for (int kv = 0; kv < 2 && ok; kv++) {
                        const unsigned full = kv ? VFULL : KFULL, empty = kv ? VEMPTY : KEMPTY, dst = kv ? sV : sK;
                        ok = !*s_abort && (n == 0 || mbar_wait(empty, (unsigned)(n - 1) & 1u));
                        if (!ok) break;
                        if (kv == 0) meta[n & 3] = bits;
                        if (bits) mbar_arrive_expect_tx(full, __popc(bits) * C::page_bytes);
                        else mbar_arrive(full);
#pragma unroll
                        for (int x = 0; x < CF_PAGES; x++)
                            if (page[x] >= 0) tt_load(dst + x * C::page_bytes, kv ? &map_v : &map_k, (page[x] * a.Hk + g.h) * PAGE, 0, full);
                    }
                }
                ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            }
        }
        if (!ok && lane == 0) {                                // what was issued lands before the block ends
            *s_abort = 1;
            tree_status(a, DYNAKV_ST_INTERNAL);
            if (n > 1) { mbar_wait(KFULL, (unsigned)(n - 2) & 1u); mbar_wait(VFULL, (unsigned)(n - 2) & 1u); }
            if (n > 0) mbar_wait(KFULL, (unsigned)(n - 1) & 1u, 1 << 12);
        }
        return;
    }
    // =============================== 16 query rows per warp ===============================
    regs_up<C::regs_sums>();
    const int tx = lane & 15, row0 = warp * 16 + (lane >> 4) * 8;               // this thread's 8 rows; keys tx + 16 j; columns 4 tx and 64 + 4 tx
    const float2 factors = chunk_factor(a);
    const float factor = factors.x;
    int n = 0;
    bool dead = false, cut_end = false;
    auto wait = [&](unsigned b, int phase) {
        if (!dead && !mbar_wait(b, (unsigned)phase & 1u)) { dead = true; *s_abort = 1; tree_status(a, DYNAKV_ST_INTERNAL); }
        dead = __any_sync(0xffffffffu, dead);
    };
    while (walk.next(a.Hk, tokens, plan, g)) {
        // ---- the warp's queries, scaled, and what they see
        __syncwarp();
        int wlo = 0, whi = g.n;                                // rows that all of the warp's queries see
        if (lane < 16) {
            const int row = warp * 16 + lane, mine = row / a.G, t = row < tokens * a.G && mine < g.tokens ? g.tile * tokens + mine : -1;
            int lo = 0, hi = g.n;
            const int place = g.n - g.T + max(t, 0);
            if (t >= 0) chunk_sees(a, g.q0 + t, place, g.n, lo, hi);
            const float slope = a.slopes ? a.slopes[g.h * a.G + row % a.G] * CF_LOG2E : 0.f;
            row_s[row] = make_int4(lo, hi, place, __float_as_int(slope));
            wlo = lo; whi = hi;
        }
        wlo = __reduce_max_sync(0xffffffffu, wlo); whi = __reduce_min_sync(0xffffffffu, whi);
        auto q_row = [&](int row) { return (size_t)(g.q0 + g.tile * tokens + row / a.G) * a.Hq + g.h * a.G + row % a.G; };
        auto exists = [&](int row) { return row < tokens * a.G && row / a.G < g.tokens; };
#pragma unroll 4
        for (int x = lane; x < 16 * HD / 4; x += 32) {
            const int row = warp * 16 + x / (HD / 4), c = x % (HD / 4);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (exists(row)) v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + q_row(row) * HD + c * 4);
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(sQ + row * C::row_bytes + c * 16), "f"(v.x * factor), "f"(v.y * factor), "f"(v.z * factor), "f"(v.w * factor) : "memory");
        }
        __syncwarp();
        float2 o[8][2 * C::cols];
        float m[8], l[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
            for (int d = 0; d < 2 * C::cols; d++) o[i][d] = make_float2(0.f, 0.f);
        }
        for (int st = g.s0; st < g.s1; st++, n++) {
            const int key0 = st * CF_KEYS;
            wait(KFULL, n);
            const int have = meta[n & 3];
            // ---- logits
            float2 s[8][4];
#pragma unroll
            for (int i = 0; i < 8; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) s[i][j] = make_float2(0.f, 0.f);
            if (!dead) {
#pragma unroll 4
                for (int c = 0; c < HD / 4; c++) {
                    uint4 k[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) k[j] = lds16(sK + (j >> 1) * C::page_bytes + cf_chunk((j & 1) * 16 + tx, c));
                    uint4 q[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) q[i] = lds16(sQ + (row0 + i) * C::row_bytes + c * 16);
#pragma unroll
                    for (int i = 0; i < 8; i++)
#pragma unroll
                        for (int j = 0; j < 4; j++) s[i][j] = fma2(lo2(q[i]), lo2(k[j]), s[i][j]);
#pragma unroll
                    for (int i = 0; i < 8; i++)
#pragma unroll
                        for (int j = 0; j < 4; j++) s[i][j] = fma2(hi2(q[i]), hi2(k[j]), s[i][j]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(KEMPTY);
            const bool edge = wlo > key0 || whi < key0 + CF_KEYS || have != (1 << CF_PAGES) - 1;          // the same in the whole warp
            bool move = false;
            float mx[8], x[8][4];
#pragma unroll
            for (int i = 0; i < 8; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) x[i][j] = s[i][j].x + s[i][j].y;
            if (a.cap > 0.f) {
#pragma unroll
                for (int i = 0; i < 8; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) x[i][j] = a.cap * CF_LOG2E * tanhf(x[i][j] * factors.y);
            }
            if (a.slopes) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float away = (float)(row_s[row0 + i].z - key0 - tx), slope = __int_as_float(row_s[row0 + i].w);     // whole numbers below 2^24: exact
#pragma unroll
                    for (int j = 0; j < 4; j++) x[i][j] = fmaf(-slope, fabsf(away - 16.f * j), x[i][j]);
                }
            }
            if (edge) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int lo = row_s[row0 + i].x - key0 - tx, hi = row_s[row0 + i].y - key0 - tx;
#pragma unroll
                    for (int j = 0; j < 4; j++) if (16 * j < lo || 16 * j >= hi || !((have >> (j >> 1)) & 1)) x[i][j] = -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                mx[i] = fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]));
#pragma unroll
                for (int b = 1; b < 16; b <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], b));
                move |= mx[i] > m[i] + CF_LAZY;
            }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float to = mx[i] > m[i] + CF_LAZY ? mx[i] : m[i], f = to == -INFINITY ? 1.f : ex2(m[i] - to);
                    m[i] = to; l[i] *= f;
#pragma unroll
                    for (int d = 0; d < 2 * C::cols; d++) o[i][d] = mul2(o[i][d], make_float2(f, f));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float p = ex2(x[i][j] - ref);
                    l[i] += p;
                    asm volatile("st.shared.v2.f32 [%0], {%1, %1};\n" ::"r"(sP + ((row0 + i) * CF_KEYS + j * 16 + tx) * 8), "f"(p) : "memory");
                }
            }
            __syncwarp();
            // ---- sums
            wait(VFULL, n);
            if (!dead && (have != (1 << CF_PAGES) - 1 || key0 + CF_KEYS > g.n)) {
                // rows of V that no page holds, or past the sequence's end: every warp zeroes them for itself
                for (int e = lane; e < CF_KEYS * HD / 4; e += 32) {
                    const int r = e / (HD / 4);
                    if (key0 + r >= g.n || !((have >> (r / PAGE)) & 1))
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};\n" ::"r"(sV + r / PAGE * C::page_bytes + cf_chunk(r % PAGE, e % (HD / 4))), "r"(0u) : "memory");
                }
                fence_proxy_async();
                __syncwarp();
            }
            if (!dead) {
#pragma unroll 4
                for (int k2 = 0; k2 < CF_KEYS / 2; k2++) {
                    uint4 v[2][C::cols];
#pragma unroll
                    for (int y = 0; y < 2; y++)
#pragma unroll
                        for (int d = 0; d < C::cols; d++) v[y][d] = lds16(sV + (k2 >> 4) * C::page_bytes + cf_chunk((k2 & 15) * 2 + y, tx + d * 16));
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const uint4 p = lds16(sP + ((row0 + i) * CF_KEYS + k2 * 2) * 8);
#pragma unroll
                        for (int d = 0; d < C::cols; d++) { o[i][2 * d] = fma2(lo2(p), lo2(v[0][d]), o[i][2 * d]); o[i][2 * d + 1] = fma2(lo2(p), hi2(v[0][d]), o[i][2 * d + 1]); }
#pragma unroll
                        for (int d = 0; d < C::cols; d++) { o[i][2 * d] = fma2(hi2(p), lo2(v[1][d]), o[i][2 * d]); o[i][2 * d + 1] = fma2(hi2(p), hi2(v[1][d]), o[i][2 * d + 1]); }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(VEMPTY);
        }
        // ---- the rows, or their records
        const bool whole = g.first && g.last;
        const size_t slot = (size_t)blockIdx.x * 2 + (g.first ? 1 : 0);
        bool wild = false;
#pragma unroll
        for (int i = 0; i < 8; i++) {
#pragma unroll
            for (int b = 1; b < 16; b <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], b);
#pragma unroll
            for (int d = 0; d < 2 * C::cols; d++) wild |= (far_out(o[i][d].x) || far_out(o[i][d].y)) && is_number(l[i]);
        }
        if (wild) *s_odd = 1;
        if (!dead) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int row = row0 + i;
                if (!exists(row)) continue;
                const float f = !whole ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
                float* to = whole ? reinterpret_cast<float*>(a.out) + q_row(row) * HD : a.acc + (slot * CF_ROWS + row) * HD;
#pragma unroll
                for (int c = 0; c < C::cols; c++)
                    *reinterpret_cast<float4*>(to + 64 * c + 4 * tx) = make_float4(o[i][2 * c].x * f, o[i][2 * c].y * f, o[i][2 * c + 1].x * f, o[i][2 * c + 1].y * f);
                if (tx == 0) {
                    if (!whole) a.ml[slot * CF_ROWS + row] = make_float2(m[i], l[i]);
                    else if (a.lse) a.lse[q_row(row)] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * CF_LN2;
                }
            }
        }
        if (g.last && !g.first) {
            cut_end = true;
            if (tid == 0) {
                int* d = a.desc + (size_t)blockIdx.x * 8;
                int c = blockIdx.x;
                while (c > 0 && plan.starts[c].at > g.unit_start) c--;
                d[DESC_FIRST] = c;
                d[DESC_Q0] = g.q0 + g.tile * tokens; d[DESC_T] = g.tokens; d[DESC_H] = g.h;
            }
        }
    }
    if (tid == 0) a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
    // ---- all is done: rows whose sums are no numbers are taken again
    asm volatile("bar.sync 1, %0;\n" ::"n"(CF_WARPS * 32) : "memory");
    if (*s_odd && !*s_abort) chunk_f32_again<HD>(a, plan, warp, reinterpret_cast<int*>(cf_smem));
}

// Merges the records of the units that were cut: block (x = CTA in which the unit ends, y = 8 rows), a warp per row.
template <int HD>
__global__ void __launch_bounds__(256) k_chunk_merge_f32(const TreeArgs a) {
    constexpr int EPL = HD / 32;
    pdl_wait();
    const int* d = a.desc + (size_t)blockIdx.x * 8;
    if (!d[DESC_VALID]) return;
    const int lane = threadIdx.x & 31, row = blockIdx.y * 8 + (threadIdx.x >> 5), t = row / a.G, c0 = d[DESC_FIRST], n = blockIdx.x - c0 + 1;
    if (row >= CF_ROWS / a.G * a.G || t >= d[DESC_T]) return;
    auto slot = [&](int i) { return ((size_t)(c0 + i) * 2 + (i == 0 ? 1 : 0)) * CF_ROWS + row; };
    float m = -INFINITY, l = 0.f, o[EPL] = {};
    for (int i = 0; i < n; i++) {
        const float2 x = a.ml[slot(i)];
        const float to = fmaxf(m, x.x), ref = to == -INFINITY ? 0.f : to, f0 = exp2f(m - ref), f1 = exp2f(x.x - ref);
        m = to;
        l = l * f0 + x.y * f1;
        const float* v = a.acc + slot(i) * HD + lane * EPL;
#pragma unroll
        for (int e = 0; e < EPL; e++) o[e] = o[e] * f0 + v[e] * f1;
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const size_t at = (size_t)(d[DESC_Q0] + t) * a.Hq + d[DESC_H] * a.G + row % a.G;
    float* out = reinterpret_cast<float*>(a.out) + at * HD + lane * EPL;
#pragma unroll
    for (int e = 0; e < EPL; e++) out[e] = o[e] * f;
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * CF_LN2;
}

template <int HD>
static int chunk_f32_launch_hd(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    using C = F32Chunk<HD>;
    CUtensorMap mk, mv;
    if (!tree_page_map(&mk, cache, cache->k, true) || !tree_page_map(&mv, cache, cache->v, true)) return DYNAKV_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_chunk_f32<HD>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    // the warpgroups' shares of the registers add up to what the launch gets, or the kernel would wait for them forever
    static const int regs = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, k_chunk_f32<HD>) == cudaSuccess ? f.numRegs : 0;
    }();
    if (3 * regs < 2 * C::regs_sums + C::regs_loads) return DYNAKV_ERR_CUDA;
    const int rc = chunk_plan_launch(a, plan, sms, {CF_ROWS / a.G, CF_KEYS, CF_UNIT_COST, CF_WHOLE}, st);
    if (rc != DYNAKV_OK) return rc;
    if (launch_pdl(k_chunk_f32<HD>, dim3(sms), dim3(C::threads), C::smem, st, mk, mv, a, plan) != cudaSuccess) return DYNAKV_ERR_CUDA;
    return launch_pdl(k_chunk_merge_f32<HD>, dim3(sms, CF_ROWS / 8), dim3(256), 0, st, a) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

int chunk_f32_launch(const dynakv_row_cache* cache, const TreeArgs& a, const ChunkPlan& plan, int sms, cudaStream_t st) {
    return cache->head_dim == 128 ? chunk_f32_launch_hd<128>(cache, a, plan, sms, st) : chunk_f32_launch_hd<64>(cache, a, plan, sms, st);
}

}  // namespace dkv
