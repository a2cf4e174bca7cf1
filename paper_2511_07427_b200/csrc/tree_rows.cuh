// The kernel for few query rows behind dynakv_attend_tree and dynakv_attend_chunk: attention of one new token, a tree of drafted
// tokens or a short chunk over the rows of a paged cache.
//
//   out[i] = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(q_i . k_j * scale) where token i sees row j, else 0
//
// All G query heads of a KV head and all tokens of the tree share every row that is read, so a CTA works on a tile of
// query rows (token, head of the group) at once: with R rows per KV head a row of K and V (512 bytes in bf16, d = 128) meets
// 4 d R flops, and HBM bounds the call until R is in the tens.  tree_plan.cuh says how the pages are shared out.
//
// Kernel shape.  One producer warp streams whole 32-row pages, K and V, into a shared-memory ring with tiled TMA loads
// (128-byte swizzle, so that the fragment loads below meet no bank conflicts; FP8 rows' exponents come by cp.async, because the two
// bulk copies of 32 bytes cost as much issue time as the pages: 4 x 32768 rows of 64, 8 KV heads, 52 -> 46 us without them).
// The consumer warps are RG row groups x KG page groups: a row group holds 16 query rows, a page group takes every KG-th
// page of the CTA's range with a softmax state of its own, merged through shared memory at a segment's end.
// Few rows: three page groups hide the latency of a page's chain of dependent steps; 64 rows: four row groups share a
// page, which divides its shared-memory traffic.  A ring stage is always consumed by the same page group (a parity
// wait cannot tell a phase from the one after the next).
//
// The consumers.  bf16 rows: mma.sync m16n8k16, fragments by ldmatrix; the weights are split into bf16 hi + lo (two MMAs),
// because bf16 weights alone would add an error as large as the output's own rounding.  FP8 rows: the bytes become f16
// operands (exact), q is divided by a power of two per row so that it fits f16, the K row's scale multiplies the logit, and
// the V row's scale is folded into the softmax (running maximum over logit + exponent) as in the gather-attention kernel;
// f16 weights round to 2^-12 of themselves down to 2^-26 of the largest weight times scale, below to 2^-37 of it (F16_BELOW); with
// few query rows of 128 elements the products are turned round.  fp32 rows: fp32 FMAs, one
// lane per key for the logits, one lane per 4 columns for the sums.
//
// Masked rows never reach a sum.  Logits of rows that a token does not see are replaced by -inf.  Rows of V past the
// sequence's length (whatever an earlier sequence left there) are zeroed in shared memory, and so are drafted rows that hold
// a NaN or an infinity, because 0 * NaN would leak them into the tokens that do not see them; tokens that do see them get
// their share added in fp32 at the end of the segment.  For dynakv_attend_chunk, where any row may be one that some tokens do not see, query rows whose sums
// came out as no numbers are taken again at the end (chunk_again.cuh).
#pragma once

#include <cuda.h>
#include <float.h>

#include <type_traits>

#include "bulk_copy.cuh"
#include "chunk_again.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tree_host.cuh"
#include "tree_plan.cuh"

namespace dkv {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int PLAN_RANGE = 80;
constexpr float VE_LOW = -60.f;            // FP8: V rows with a smaller scale take part in the reference as if they had this one
// l * 2^d, d <= 0, where 2^d by itself may lie below fp32's range: FP8 rows' sums of weights are kept relative to a maximum that
// has the V rows' exponents in it, so they are as far from 1 as those exponents are from another.
__device__ __forceinline__ float scaled_sum(float l, float d) {
    const float h = exp2f(0.5f * d);
    return l * h * h;
}
// The softmax's reference moves when the maximum has outgrown it by 2^LAZY, to the maximum.  FP8 rows, whose weights become f16
// values (65504 at most, subnormal below 2^-14): to 2^F16_BELOW below the maximum, and again when that has grown by 2^F16_LAZY, so
// that weights stay below 2^15.8 and those down to 2^-26 of the largest are normal.  With the reference at the maximum they were
// subnormal from 2^-14 on and lost below 2^-25, which a column sees where a dominant row holds a zero: it came out as 0.  The
// lower reference and earlier moves cost up to 2 % (4 x 32768 rows, 8 KV heads: 32 query rows 104 -> 106 us, 64 rows 187 -> 190 us).
constexpr float LAZY = 8.f, F16_BELOW = 12.f, F16_LAZY = 3.75f;

__device__ __forceinline__ void tma_page(unsigned dst, const CUtensorMap* map, int row, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n"
                 ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(0), "r"(bar) : "memory");
}
// Two 16-byte copies global -> shared that arrive at `bar` (one arrival) together with all earlier ones of the thread.
__device__ __forceinline__ void copy32(unsigned dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n cp.async.cg.shared.global [%0 + 16], [%1 + 16], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_arrive(unsigned bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float lds_f32(unsigned addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}

template <int HD, int DT, int RG, bool MOD>
struct TreeCfg {
    static constexpr int esize = DT == DYNAKV_F32 ? 4 : DT == DYNAKV_BF16 ? 2 : 1;
    static constexpr int row_bytes = HD * esize;
    static constexpr int panel_w = row_bytes < 128 ? row_bytes : 128;        // bytes of a row in one swizzle panel
    static constexpr int panels = row_bytes / panel_w;
    static constexpr int page_bytes = PAGE * row_bytes;
    static constexpr int stage_bytes = 2 * page_bytes;
    static constexpr int groups = RG == 0 ? 1 : RG;                          // row groups; RG = 0: one, of few rows
    static constexpr int rows = RG > 0 ? 16 : DT == DYNAKV_F32 ? 4 : 8;      // rows of a group
    static constexpr int RT = groups * rows;
    static constexpr int dump_bytes = rows * HD * 4 + rows * 8;              // one warp's sums, then (m, l) of its rows
    // page groups; fp32 rows have one CTA per SM and a long way through a page, so more of them
    static constexpr int KG = DT == DYNAKV_F32 ? (RG == 0 ? 6 : RG == 1 ? 4 : RG == 2 ? 2 : 1) : RG <= 1 ? 3 : RG == 2 ? 2 : 1;
    static constexpr int consumers = groups * KG;
    static constexpr int merge_bytes = (KG - 1) * groups * dump_bytes;
    // the ring takes what the merge leaves of 112 KB per CTA (fp32: of 224 KB, with q and the weights), in a multiple of the page groups, at most 12 stages
    static constexpr int ring_bytes = (DT == DYNAKV_F32 ? 224 * 1024 - RT * HD * 4 - consumers * rows * 128 : 112 * 1024) - merge_bytes;
    static constexpr int most = (ring_bytes - consumers * 512) / (stage_bytes + 80) < 12 ? (ring_bytes - consumers * 512) / (stage_bytes + 80) : 12;
    static constexpr int stages = most / KG * KG;
    static constexpr int threads = 32 * (consumers + 1);
    static constexpr int per_sm = DT == DYNAKV_F32 ? 1 : 2;
    static constexpr int exp_bytes = DT == DYNAKV_FP8 ? stages * 64 + consumers * 32 * 16 : 0;   // and a table of scales per warp
    static constexpr int q_bytes = DT == DYNAKV_F32 ? RT * HD * 4 : 0;
    static constexpr int p_bytes = DT == DYNAKV_F32 ? consumers * rows * 32 * 4 : 0;
    static constexpr int plan_words = MOD ? PLAN_RANGE + sizeof(Range) / 8 : 48;       // what tree_range leaves for the walk, and (MOD) the range itself
    static constexpr int fixed_bytes = 32 * 4 + 2 * stages * 8 + stages * 4 + 3 * 8 * 4 + 16 + plan_words * 8;
    static constexpr int smem = stages * stage_bytes + exp_bytes + q_bytes + p_bytes + merge_bytes + fixed_bytes;
    static_assert(stages % KG == 0, "each ring stage belongs to one page group");
    static_assert(per_sm * (smem + 1024) <= 233472, "shared memory of an SM");
};

// What a consumer warp needs to know of the page it is handed.
struct PageIn {
    unsigned k, v;                 // shared-memory addresses
    const signed char* exps;       // FP8: scale exponents of the 32 K rows, then of the 32 V rows
    float4* scales;                // FP8: this warp's table of what they come to (shared memory)
    int key0;                      // first row's place in the sequence
    bool mask;                     // rows of the page may be invisible
};

// Byte offset of 16-byte chunk c of row r inside a page of the ring, as the TMA swizzle placed it.
template <typename C>
__device__ __forceinline__ unsigned chunk_at(int r, int c) {
    if constexpr (C::panel_w == 128) return (c >> 3) * (PAGE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    else return r * 64 + (((c & 3) ^ ((r >> 1) & 3)) << 4);
}

// ---------------------------------------------------------------------------------- which rows a token sees, and its scores
//
// MOD = false (dynakv_attend_tree): a context that every token sees and a tree with its mask.  MOD = true (dynakv_attend_chunk): every
// token sees one range of rows, and its logits may be capped and lowered with the distance.
template <bool MOD>
__device__ __forceinline__ float logit_factor(const TreeArgs& a) { return MOD && a.cap > 0.f ? a.scale / a.cap : a.scale * LOG2E; }

template <bool MOD>
struct RowScore {
    __device__ __forceinline__ void start(const TreeArgs&, const Segment&, int, int) {}
    __device__ __forceinline__ float logit(const TreeArgs&, float x, int) const { return x; }
    __device__ __forceinline__ RowScore from_lane(int) const { return *this; }
};
template <>
struct RowScore<true> {
    int lo, hi, place;                 // rows [lo, hi) are seen; the token's own row
    float slope;                       // log2 units
    // token t (-1: the row does not exist) and query row r of the unit
    __device__ __forceinline__ void start(const TreeArgs& a, const Segment& g, int t, int r) {
        place = g.n - g.T + max(t, 0);
        lo = 0; hi = g.n; slope = 0.f;
        if (t < 0) return;
        chunk_sees(a, g.q0 + t, place, g.n, lo, hi);
        if (a.slopes) slope = a.slopes[g.h * a.G + r - t * a.G] * LOG2E;
    }
    __device__ __forceinline__ float logit(const TreeArgs& a, float x, int key) const {
        if (a.cap > 0.f) x = a.cap * LOG2E * tanhf(x);
        if (a.slopes) x = fmaf(-slope, fabsf((float)(place - key)), x);
        return x;
    }
    __device__ __forceinline__ RowScore from_lane(int r) const {
        RowScore o;
        o.lo = __shfl_sync(0xffffffffu, lo, r); o.hi = __shfl_sync(0xffffffffu, hi, r);
        o.place = __shfl_sync(0xffffffffu, place, r); o.slope = __shfl_sync(0xffffffffu, slope, r);
        return o;
    }
    // the rows of a page (first row key0) in [lo, hi), as bits
    __device__ __forceinline__ unsigned window(int key0) const {
        const int x = max(lo - key0, 0), y = min(hi - key0, PAGE);
        return x >= y ? 0u : (y == 32 ? ~0u : (1u << y) - 1u) & ~((1u << x) - 1u);
    }
};
template <bool MOD>
__device__ __forceinline__ unsigned page_window(const TreeArgs& a, const Segment& g, const PageIn& p, int t, const RowScore<MOD>& s) {
    if constexpr (MOD) return s.window(p.key0);
    else return !p.mask ? ~0u : t >= 0 ? tree_window(a, g, t, p.key0) : 0u;
}

// ---------------------------------------------------------------------------------- mma.sync consumers (bf16, FP8)
//
// The MMAs are plain functions of their registers to the compiler (no volatile), and a group's operands are loaded before its
// first product: independent chains then overlap, which is what few warps per scheduler need (two; 254 registers each).
template <bool F16>
__device__ __forceinline__ void tree_mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
    if constexpr (F16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Lane (g = lane / 4, c = lane % 4) owns rows g and g + 8 of the warp's 16 and the columns of its fragments.  With at most 8
// rows (RG = 0: plain decoding of a group of up to 8 heads) rows 8 to 15 of the weights' tile hold the lo parts of rows 0 to 7, so
// that one MMA does for both, and only one row per lane goes through the softmax.
template <int HD, int DT, int RG, bool MOD>
struct MmaRows {
    using C = TreeCfg<HD, DT, RG, MOD>;
    static constexpr bool F8 = DT == DYNAKV_FP8;
    static constexpr bool HALF = RG == 0;
    static constexpr int KS = HD / 16, NT = HD / 8, NR = HALF ? 1 : 2;       // rows per lane
    static constexpr float BELOW = F8 ? F16_BELOW : 0.f, GROW = F8 ? F16_BELOW + F16_LAZY : LAZY;
    static constexpr bool PERM = F8 && HD == 128;       // key order inside a tile that keeps FP8 loads free of conflicts
    unsigned qf[KS][4];
    float qs[NR];                                       // logit factor (log2 units) of the rows
    float acc[NT][4], m[NR], l[NR];
    int t[NR];                                          // token of the rows, -1: no such row
    RowScore<MOD> score[NR];

    static __device__ __forceinline__ int key_of(int n) { return PERM ? (n & 1) * 4 + (n >> 1) : n; }       // column n of an 8-key tile
    // element of the output that acc[nt][i] (i = 0, 1) of lane column c holds
    static __device__ __forceinline__ int elem(int nt, int i, int c) {
        if constexpr (!F8) return nt * 8 + 2 * c + i;
        else if constexpr (HD == 128) return 16 * (c + 4 * i) + nt;
        else return 8 * (2 * c + i) + nt;
    }

    __device__ __forceinline__ void start(const TreeArgs& a, const Segment& g, int rg, int lane) {
        const int c = lane & 3;
#pragma unroll
        for (int i = 0; i < NR; i++) {
            const int r = g.tile * C::RT + rg * 16 + (lane >> 2) + 8 * i;
            t[i] = r < g.T * a.G ? r / a.G : -1;
            const unsigned* q = reinterpret_cast<const unsigned*>(
                reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)(g.q0 + max(t[i], 0)) * a.Hq + g.h * a.G + (t[i] < 0 ? 0 : r - t[i] * a.G)) * HD);
            float mx = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ks++) {
                if constexpr (!F8) {
                    qf[ks][i] = t[i] >= 0 ? q[ks * 8 + c] : 0u;
                    qf[ks][i + 2] = t[i] >= 0 ? q[ks * 8 + c + 4] : 0u;
                } else {             // four neighbouring elements: the lane's bytes of a K chunk are its fragments of four steps
                    const int e = ((ks >> 2) * 4 + c) * 16 + (ks & 3) * 4;
                    const uint2 w = t[i] >= 0 ? *reinterpret_cast<const uint2*>(q + e / 2) : make_uint2(0u, 0u);
                    qf[ks][i] = w.x; qf[ks][i + 2] = w.y;
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        const unsigned u = x ? w.y : w.x;
                        mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(u << 16)), fabsf(__uint_as_float(u & 0xffff0000u))));
                    }
                }
            }
            qs[i] = logit_factor<MOD>(a);
            score[i].start(a, g, t[i], r);
            if constexpr (F8) {      // q / 2^e with the largest element in [2^14, 2^15): exact in f16 down to 2^-29 of it
                mx = quad_max(mx);
                const int e = mx > 0.f ? max(-100, min(112, (int)(__float_as_uint(mx) >> 23) - 127 - 14)) : 0;
                const float down = pow2f(-e);
#pragma unroll
                for (int ks = 0; ks < KS; ks++)
#pragma unroll
                    for (int x = 0; x < 4; x += 2) {
                        const unsigned u = qf[ks][i + x];
                        const __half2 h = __floats2half2_rn(__uint_as_float(u << 16) * down, __uint_as_float(u & 0xffff0000u) * down);
                        qf[ks][i + x] = *reinterpret_cast<const unsigned*>(&h);
                    }
                qs[i] *= pow2f(e);
            }
            m[i] = -INFINITY; l[i] = 0.f;
        }
        if constexpr (HALF) {
#pragma unroll
            for (int ks = 0; ks < KS; ks++) qf[ks][1] = qf[ks][3] = 0u;
        }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int x = 0; x < 4; x++) acc[nt][x] = 0.f;
    }

    __device__ __forceinline__ void page(const TreeArgs& a, const Segment& g, const PageIn& p, int lane) {
        const int c = lane & 3, n = lane >> 2;
        // FP8: one lane per row turns its exponents into factors, and all lanes read what they need behind the products: the logit's
        // factor, the exponent that takes part in the softmax, and what a V row below 2^VE_LOW is still to be scaled by
        bool low = false;
        if constexpr (F8) {
            const float ve = (float)p.exps[32 + lane], vr = fmaxf(ve, VE_LOW);
            p.scales[lane] = make_float4(pow2f(p.exps[lane]), vr, ex2(fminf(ve - VE_LOW, 0.f)), 0.f);
            low = __any_sync(0xffffffffu, ve < VE_LOW);
            __syncwarp();
        }
        float s[4][4];
#pragma unroll
        for (int kt = 0; kt < 4; kt++)
#pragma unroll
            for (int x = 0; x < 4; x++) s[kt][x] = 0.f;
        if constexpr (!F8) {
            const int mt = lane >> 3, r8 = lane & 7;
#pragma unroll
            for (int k2 = 0; k2 < KS / 2; k2++) {
                unsigned b[4][4];
#pragma unroll
                for (int kt = 0; kt < 4; kt++) ldmatrix_x4(p.k + chunk_at<C>(kt * 8 + r8, k2 * 4 + mt), b[kt]);
#pragma unroll
                for (int kt = 0; kt < 4; kt++) tree_mma<false>(s[kt], qf[2 * k2], b[kt][0], b[kt][1]);
#pragma unroll
                for (int kt = 0; kt < 4; kt++) tree_mma<false>(s[kt], qf[2 * k2 + 1], b[kt][2], b[kt][3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < HD / 64; j++) {
                uint4 w[4];
#pragma unroll
                for (int kt = 0; kt < 4; kt++) w[kt] = lds16(p.k + chunk_at<C>(kt * 8 + key_of(n), c + 4 * j));
#pragma unroll
                for (int x = 0; x < 4; x++)
#pragma unroll
                    for (int kt = 0; kt < 4; kt++) {
                        const unsigned ww[4] = {w[kt].x, w[kt].y, w[kt].z, w[kt].w};
                        unsigned b0, b1;
                        e4m3x4_to_f16x2(ww[x], b0, b1);
                        tree_mma<true>(s[kt], qf[j * 4 + x], b0, b1);
                    }
            }
        }
        // logits in log2 units, FP8 with the K row's scale; the running maximum is over logit + exponent of the V row
        unsigned win[NR];
#pragma unroll
        for (int i = 0; i < NR; i++) win[i] = page_window<MOD>(a, g, p, t[i], score[i]);
        const bool mask = MOD ? __any_sync(0xffffffffu, (win[0] & win[NR - 1]) != ~0u) : p.mask;
        float4 sc[4][2];
        float mx[NR];
#pragma unroll
        for (int i = 0; i < NR; i++) mx[i] = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 4; kt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int key = kt * 8 + key_of(2 * c + e);
                if constexpr (F8) sc[kt][e] = p.scales[key];
#pragma unroll
                for (int i = 0; i < NR; i++) {
                    float& x = s[kt][2 * i + e];
                    x *= F8 ? qs[i] * sc[kt][e].x : qs[i];
                    if constexpr (MOD) x = score[i].logit(a, x, p.key0 + key);
                    if (mask && !((win[i] >> key) & 1u)) x = -INFINITY;
                    if constexpr (F8) x += sc[kt][e].y;
                    mx[i] = fmaxf(mx[i], x);
                }
            }
        float ref[NR];
        bool move = false;
#pragma unroll
        for (int i = 0; i < NR; i++) { mx[i] = quad_max(mx[i]); move |= mx[i] > m[i] + GROW; }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int i = 0; i < NR; i++) {
                const float to = mx[i] > m[i] + GROW ? mx[i] - BELOW : m[i];
                const float f = to == -INFINITY ? 1.f : ex2(m[i] - to);
                l[i] = !F8 ? l[i] * f : to == -INFINITY ? l[i] : scaled_sum(l[i], m[i] - to);
                m[i] = to;
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int x = 0; x < (HALF ? 4 : 2); x++) acc[nt][2 * i + x] *= f;
            }
        }
#pragma unroll
        for (int i = 0; i < NR; i++) ref[i] = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
        for (int kt = 0; kt < 4; kt++)
#pragma unroll
            for (int e = 0; e < 2; e++)
#pragma unroll
                for (int i = 0; i < NR; i++) {
                    float& x = s[kt][2 * i + e];
                    const float y = x - ref[i];
                    x = ex2(y);
                    // not x / 2^exponent: x is 0 where this V row's scale is far below another's, its weight is not
                    if constexpr (F8) l[i] += ex2(y - sc[kt][e].y);
                    else l[i] += x;
                }
        if constexpr (F8) {
            if (low) {
#pragma unroll
                for (int kt = 0; kt < 4; kt++)
#pragma unroll
                    for (int e = 0; e < 2; e++)
#pragma unroll
                        for (int i = 0; i < NR; i++) s[kt][2 * i + e] *= sc[kt][e].z;
            }
        }
        // weights as A fragments: two 8-key tiles of the logits are the 16 keys of a step
        if constexpr (!F8) {
            const int mt = lane >> 3, r8 = lane & 7;
#pragma unroll
            for (int kk = 0; kk < 2; kk++) {
                unsigned hi[4], lo[4];
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    if constexpr (HALF) split2(s[2 * kk + x][0], s[2 * kk + x][1], hi[2 * x], hi[2 * x + 1]);
                    else {
                        split2(s[2 * kk + x][0], s[2 * kk + x][1], hi[2 * x], lo[2 * x]);
                        split2(s[2 * kk + x][2], s[2 * kk + x][3], hi[2 * x + 1], lo[2 * x + 1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt += 4) {
                    unsigned b[2][4];
#pragma unroll
                    for (int x = 0; x < 2; x++) ldmatrix_x4_trans(p.v + chunk_at<C>(kk * 16 + (mt & 1) * 8 + r8, nt + 2 * x + (mt >> 1)), b[x]);
#pragma unroll
                    for (int x = 0; x < 4; x++) tree_mma<false>(acc[nt + x], hi, b[x >> 1][2 * (x & 1)], b[x >> 1][2 * (x & 1) + 1]);
#pragma unroll
                    for (int x = 0; x < (HALF ? 0 : 4); x++) tree_mma<false>(acc[nt + x], lo, b[x >> 1][2 * (x & 1)], b[x >> 1][2 * (x & 1) + 1]);
                }
            }
        } else {
            constexpr int VB = HD / 8;               // bytes of a V row a lane loads: columns n of all tiles
            const int chunk = HD == 128 ? (n & 1) * 4 + (n >> 1) : 0;
#pragma unroll
            for (int kk = 0; kk < 2; kk++) {
                unsigned pa[4];
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    if constexpr (HALF) split2h(s[2 * kk + x][0], s[2 * kk + x][1], pa[2 * x], pa[2 * x + 1]);
                    else {
                        const __half2 h0 = __floats2half2_rn(s[2 * kk + x][0], s[2 * kk + x][1]), h1 = __floats2half2_rn(s[2 * kk + x][2], s[2 * kk + x][3]);
                        pa[2 * x] = *reinterpret_cast<const unsigned*>(&h0);
                        pa[2 * x + 1] = *reinterpret_cast<const unsigned*>(&h1);
                    }
                }
                unsigned w[4][VB / 4];
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const int key = kk * 16 + (y >> 1) * 8 + key_of(2 * c + (y & 1));
                    if constexpr (HD == 128) {
                        const uint4 v = lds16(p.v + chunk_at<C>(key, chunk));
                        w[y][0] = v.x; w[y][1] = v.y; w[y][2] = v.z; w[y][3] = v.w;
                    } else {
                        unsigned x0, x1;
                        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(x0), "=r"(x1) : "r"(p.v + chunk_at<C>(key, n >> 1) + (n & 1) * 8));
                        w[y][0] = x0; w[y][1] = x1;
                    }
                }
#pragma unroll
                for (int x = 0; x < VB / 4; x++)
#pragma unroll
                    for (int half = 0; half < 2; half++) {
                        const unsigned sel = half ? 0x7362u : 0x5140u;        // bytes (2, 6, 3, 7) or (0, 4, 1, 5) of two keys
                        unsigned b0, b1, d0, d1;
                        e4m3x4_to_f16x2(__byte_perm(w[0][x], w[1][x], sel), b0, d0);
                        e4m3x4_to_f16x2(__byte_perm(w[2][x], w[3][x], sel), b1, d1);
                        tree_mma<true>(acc[4 * x + 2 * half], pa, b0, b1);
                        tree_mma<true>(acc[4 * x + 2 * half + 1], pa, d0, d1);
                    }
            }
        }
    }

    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int i = 0; i < NR; i++) l[i] = quad_sum(l[i]);
        if constexpr (HALF) {                      // the lo parts join the hi parts
#pragma unroll
            for (int nt = 0; nt < NT; nt++) { acc[nt][0] += acc[nt][2]; acc[nt][1] += acc[nt][3]; }
        }
    }
    // This warp's state into shared memory, and another's into this one's.
    __device__ __forceinline__ void dump(float* to, int lane) const {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int x = 0; x < 2 * NR; x++) to[(nt * 2 * NR + x) * 32 + lane] = acc[nt][x];
        if ((lane & 3) == 0) {
#pragma unroll
            for (int i = 0; i < NR; i++) reinterpret_cast<float2*>(to + NT * 64 * NR)[(lane >> 2) + 8 * i] = make_float2(m[i], l[i]);
        }
    }
    __device__ __forceinline__ void merge(const float* from, int lane) {
        float f0[NR], f1[NR];
#pragma unroll
        for (int i = 0; i < NR; i++) {
            const float2 o = reinterpret_cast<const float2*>(from + NT * 64 * NR)[(lane >> 2) + 8 * i];
            const float to = fmaxf(m[i], o.x), ref = to == -INFINITY ? 0.f : to;
            f0[i] = ex2(m[i] - ref); f1[i] = ex2(o.x - ref);
            l[i] = F8 ? scaled_sum(l[i], m[i] - ref) + scaled_sum(o.y, o.x - ref) : l[i] * f0[i] + o.y * f1[i];
            m[i] = to;
        }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int x = 0; x < 2 * NR; x++) acc[nt][x] = acc[nt][x] * f0[x >> 1] + from[(nt * 2 * NR + x) * 32 + lane] * f1[x >> 1];
    }
    // Whether a sum of this lane's rows is no number, or near the end of fp32, while the sum of the row's weights is one (MOD).
    __device__ __forceinline__ bool wild() const {
        bool bad = false;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int x = 0; x < 2 * NR; x++) bad |= far_out(acc[nt][x]) && is_number(l[x >> 1]);
        return bad;
    }
    // The share of a row that was left out of the MMAs: key row `row` of the pool, token j of the tree.
    __device__ __forceinline__ void add_row(const TreeArgs& a, const Segment& g, int rg, long long row, int j, int lane) {
        const int c = lane & 3;
        float d[NR];
#pragma unroll
        for (int i = 0; i < NR; i++) {
            d[i] = 0.f;
            const int r = g.tile * C::RT + rg * 16 + (lane >> 2) + 8 * i;
            if (t[i] >= 0) {
                const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)(g.q0 + t[i]) * a.Hq + g.h * a.G + r - t[i] * a.G) * HD;
                for (int e = c; e < HD; e += 4) d[i] = fmaf(__bfloat162float(q[e]), cache_elem<DT>(a.kpool, a.kexp, row, HD, e), d[i]);
            }
            d[i] = quad_sum(d[i]);
        }
#pragma unroll
        for (int i = 0; i < NR; i++)
            if (t[i] >= 0 && tree_sees(a, g, t[i], j)) {
                const float w = ex2(d[i] * (a.scale * LOG2E) - (m[i] == -INFINITY ? 0.f : m[i]));
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int x = 0; x < 2; x++) acc[nt][2 * i + x] = fmaf(w, cache_elem<DT>(a.vpool, a.vexp, row, HD, elem(nt, x, c)), acc[nt][2 * i + x]);
            }
    }
    __device__ __forceinline__ void write(const TreeArgs& a, const Segment& g, int rg, int lane, bool whole, size_t slot) const {
        const int c = lane & 3;
#pragma unroll
        for (int i = 0; i < NR; i++) {
            if (t[i] < 0) continue;
            const int rl = rg * 16 + (lane >> 2) + 8 * i, r = g.tile * C::RT + rl;
            const size_t at = (size_t)(g.q0 + t[i]) * a.Hq + g.h * a.G + r - t[i] * a.G;
            if (whole) {
                const float f = l[i] == 0.f ? 0.f : 1.f / l[i];
                __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(a.out) + at * HD;
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    if constexpr (!F8) *reinterpret_cast<unsigned*>(o + elem(nt, 0, c)) = pack_bf16(acc[nt][2 * i] * f, acc[nt][2 * i + 1] * f);
                    else if ((nt & 1) == 0) {
#pragma unroll
                        for (int x = 0; x < 2; x++)
                            *reinterpret_cast<unsigned*>(o + elem(nt, x, c)) = pack_bf16(acc[nt][2 * i + x] * f, acc[nt + 1][2 * i + x] * f);
                    }
                }
                if (a.lse && c == 0) a.lse[at] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * LN2;
            } else {
                float* o = a.acc + (slot * C::RT + rl) * HD;
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    if constexpr (!F8) *reinterpret_cast<float2*>(o + elem(nt, 0, c)) = make_float2(acc[nt][2 * i], acc[nt][2 * i + 1]);
                    else if ((nt & 3) == 0) {
#pragma unroll
                        for (int x = 0; x < 2; x++)
                            *reinterpret_cast<float4*>(o + elem(nt, x, c)) = make_float4(acc[nt][2 * i + x], acc[nt + 1][2 * i + x], acc[nt + 2][2 * i + x], acc[nt + 3][2 * i + x]);
                    }
                }
                if (c == 0) a.ml[slot * C::RT + rl] = make_float2(m[i], l[i]);
            }
        }
    }
};

// ---------------------------------------------------------------------------------- FP8 rows of 128, few queries
//
// With at most 8 query rows of 128 elements (RG = 0) the products are turned round: the rows of K and of V are the 16-row operand
// and the queries the 8-column one, S^T = K Q^T and O^T = V^T P^T, so that no MMA works on empty rows; MmaRows fills those rows
// with the lo parts of the weights, which bf16 weights need and f16 weights do not, and bytes turned into f16 come at a price.
// Lane (n = lane / 4, c = lane % 4) has query rows 2 c and 2 c + 1, of the logits the keys 8 y + key_of(n), of the sums the
// columns elem() names.  The weights become the second product's operand by four 8 x 8 transpositions.  Measured on 16 sequences
// of up to 20480 rows: 55 us, MmaRows 60; rows of 64: 47 us, MmaRows 45, and 0.5 to 1 us more for short bf16 caches, so that
// MmaRows has those.
template <bool MOD>
struct TurnedRows {
    static constexpr int HD = 128, KS = HD / 16, MT = HD / 16;
    using C = TreeCfg<HD, DYNAKV_FP8, 0, MOD>;
    unsigned qb[KS][2];
    float qs[2];                                        // logit factor (log2 units) of the two rows
    float acc[MT][4], m[2], l[2];                       // acc[mt][x]: query row 2 c + (x & 1)
    int t[2];                                           // token of the two rows, -1: no such row
    RowScore<MOD> score[2];

    // key order inside 8 keys that keeps the loads free of bank conflicts
    static __device__ __forceinline__ int key_of(int n) { return (n & 1) * 4 + (n >> 1); }
    // element of the output that acc[mt][2 * half], acc[mt][2 * half + 1] hold: the 16 bytes of a lane are neighbours
    static __device__ __forceinline__ int elem(int mt, int half, int n) { return 16 * key_of(n) + 2 * mt + half; }
    static __device__ __forceinline__ float max_over_keys(float v) {               // over the 8 lanes that share c
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    }
    static __device__ __forceinline__ float sum_over_keys(float v) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    static __device__ __forceinline__ unsigned transposed(unsigned v) {            // of an 8 x 8 matrix of 16-bit values
        unsigned r;
        asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(v));
        return r;
    }
    static __device__ __forceinline__ const __nv_bfloat16* q_row(const TreeArgs& a, const Segment& g, int r, int token) {
        return reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)(g.q0 + token) * a.Hq + g.h * a.G + r - token * a.G) * HD;
    }

    __device__ __forceinline__ void start(const TreeArgs& a, const Segment& g, int, int lane) {
        const int c = lane & 3, r0 = g.tile * C::RT, rows = g.T * a.G;
        // the lane loads for row n: four neighbouring elements per step, divided by a power of two per row, as in MmaRows
        const int rq = r0 + (lane >> 2);
        const unsigned* q = reinterpret_cast<const unsigned*>(rq < rows ? q_row(a, g, rq, rq / a.G) : nullptr);
        float mx = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
            const int e = ((ks >> 2) * 4 + c) * 16 + (ks & 3) * 4;
            const uint2 w = q ? *reinterpret_cast<const uint2*>(q + e / 2) : make_uint2(0u, 0u);
            qb[ks][0] = w.x; qb[ks][1] = w.y;
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const unsigned u = qb[ks][x];
                mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(u << 16)), fabsf(__uint_as_float(u & 0xffff0000u))));
            }
        }
        mx = quad_max(mx);
        const int e = mx > 0.f ? max(-100, min(112, (int)(__float_as_uint(mx) >> 23) - 127 - 14)) : 0;
        const float down = pow2f(-e), mine = logit_factor<MOD>(a) * pow2f(e);
#pragma unroll
        for (int ks = 0; ks < KS; ks++)
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const unsigned u = qb[ks][x];
                const __half2 h = __floats2half2_rn(__uint_as_float(u << 16) * down, __uint_as_float(u & 0xffff0000u) * down);
                qb[ks][x] = *reinterpret_cast<const unsigned*>(&h);
            }
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int r = r0 + 2 * c + i;
            t[i] = r < rows ? r / a.G : -1;
            score[i].start(a, g, t[i], r);
            qs[i] = __shfl_sync(0xffffffffu, mine, (2 * c + i) * 4);
            m[i] = -INFINITY; l[i] = 0.f;
        }
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int x = 0; x < 4; x++) acc[mt][x] = 0.f;
    }

    __device__ __forceinline__ void page(const TreeArgs& a, const Segment& g, const PageIn& p, int lane) {
        const int c = lane & 3, n = lane >> 2;
        // the scales of the 32 rows, one row per lane, as in MmaRows
        const float ve = (float)p.exps[32 + lane], vr = fmaxf(ve, VE_LOW);
        p.scales[lane] = make_float4(pow2f(p.exps[lane]), vr, ex2(fminf(ve - VE_LOW, 0.f)), 0.f);
        const bool low = __any_sync(0xffffffffu, ve < VE_LOW);
        __syncwarp();
        float s[2][4];               // [16 keys][(key n, row 2 c), (n, 2 c + 1), (n + 8, 2 c), (n + 8, 2 c + 1)]
#pragma unroll
        for (int k16 = 0; k16 < 2; k16++)
#pragma unroll
            for (int x = 0; x < 4; x++) s[k16][x] = 0.f;
#pragma unroll
        for (int j = 0; j < 2; j++) {
            unsigned w[4][4];
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const uint4 u = lds16(p.k + chunk_at<C>(y * 8 + key_of(n), c + 4 * j));
                w[y][0] = u.x; w[y][1] = u.y; w[y][2] = u.z; w[y][3] = u.w;
            }
#pragma unroll
            for (int x = 0; x < 4; x++)
#pragma unroll
                for (int k16 = 0; k16 < 2; k16++) {
                    unsigned k[4];
                    e4m3x4_to_f16x2(w[2 * k16][x], k[0], k[2]);
                    e4m3x4_to_f16x2(w[2 * k16 + 1][x], k[1], k[3]);
                    tree_mma<true>(s[k16], k, qb[j * 4 + x][0], qb[j * 4 + x][1]);
                }
        }
        unsigned win[2];
#pragma unroll
        for (int i = 0; i < 2; i++) win[i] = page_window<MOD>(a, g, p, t[i], score[i]);
        const bool mask = MOD ? __any_sync(0xffffffffu, (win[0] & win[1]) != ~0u) : p.mask;
        float4 sc[2][2];
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int k16 = 0; k16 < 2; k16++)
#pragma unroll
            for (int y = 0; y < 2; y++) {
                const int key = k16 * 16 + y * 8 + key_of(n);
                sc[k16][y] = p.scales[key];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    float& x = s[k16][2 * y + i];
                    x *= qs[i] * sc[k16][y].x;
                    if constexpr (MOD) x = score[i].logit(a, x, p.key0 + key);
                    if (mask && !((win[i] >> key) & 1u)) x = -INFINITY;
                    x += sc[k16][y].y;
                    mx[i] = fmaxf(mx[i], x);
                }
            }
        bool move = false;
#pragma unroll
        for (int i = 0; i < 2; i++) { mx[i] = max_over_keys(mx[i]); move |= mx[i] > m[i] + (F16_BELOW + F16_LAZY); }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float to = mx[i] > m[i] + (F16_BELOW + F16_LAZY) ? mx[i] - F16_BELOW : m[i];
                const float f = to == -INFINITY ? 1.f : ex2(m[i] - to);
                l[i] = to == -INFINITY ? l[i] : scaled_sum(l[i], m[i] - to);
                m[i] = to;
#pragma unroll
                for (int mt = 0; mt < MT; mt++) { acc[mt][i] *= f; acc[mt][2 + i] *= f; }
            }
        }
        unsigned b[2][2];            // [16 keys][half]: the weights as the second product's operand
#pragma unroll
        for (int k16 = 0; k16 < 2; k16++)
#pragma unroll
            for (int y = 0; y < 2; y++) {
                float w[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const float z = s[k16][2 * y + i] - (m[i] == -INFINITY ? 0.f : m[i]);
                    w[i] = ex2(z);
                    l[i] += ex2(z - sc[k16][y].y);             // as in MmaRows
                    if (low) w[i] *= sc[k16][y].z;
                }
                const __half2 h = __floats2half2_rn(w[0], w[1]);
                b[k16][y] = transposed(*reinterpret_cast<const unsigned*>(&h));
            }
#pragma unroll
        for (int k16 = 0; k16 < 2; k16++) {
            unsigned w[4][4];
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const uint4 v = lds16(p.v + chunk_at<C>(k16 * 16 + (y >> 1) * 8 + key_of(2 * c + (y & 1)), key_of(n)));
                w[y][0] = v.x; w[y][1] = v.y; w[y][2] = v.z; w[y][3] = v.w;
            }
#pragma unroll
            for (int x = 0; x < 4; x++)
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    const unsigned sel = half ? 0x7362u : 0x5140u;        // bytes (2, 6, 3, 7) or (0, 4, 1, 5) of two keys
                    unsigned v[4];
                    e4m3x4_to_f16x2(__byte_perm(w[0][x], w[1][x], sel), v[0], v[1]);
                    e4m3x4_to_f16x2(__byte_perm(w[2][x], w[3][x], sel), v[2], v[3]);
                    tree_mma<true>(acc[2 * x + half], v, b[k16][0], b[k16][1]);
                }
        }
    }

    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int i = 0; i < 2; i++) l[i] = sum_over_keys(l[i]);
    }
    __device__ __forceinline__ void dump(float* to, int lane) const {
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int x = 0; x < 4; x++) to[(mt * 4 + x) * 32 + lane] = acc[mt][x];
        if (lane < 4) {
#pragma unroll
            for (int i = 0; i < 2; i++) reinterpret_cast<float2*>(to + MT * 128)[2 * lane + i] = make_float2(m[i], l[i]);
        }
    }
    __device__ __forceinline__ void merge(const float* from, int lane) {
        float f0[2], f1[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const float2 o = reinterpret_cast<const float2*>(from + MT * 128)[2 * (lane & 3) + i];
            const float to = fmaxf(m[i], o.x), ref = to == -INFINITY ? 0.f : to;
            f0[i] = ex2(m[i] - ref); f1[i] = ex2(o.x - ref);
            l[i] = scaled_sum(l[i], m[i] - ref) + scaled_sum(o.y, o.x - ref);
            m[i] = to;
        }
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int x = 0; x < 4; x++) acc[mt][x] = acc[mt][x] * f0[x & 1] + from[(mt * 4 + x) * 32 + lane] * f1[x & 1];
    }
    __device__ __forceinline__ bool wild() const {
        bool bad = false;
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int x = 0; x < 4; x++) bad |= far_out(acc[mt][x]) && is_number(l[x & 1]);
        return bad;
    }
    // As in MmaRows.
    __device__ __forceinline__ void add_row(const TreeArgs& a, const Segment& g, int, long long row, int j, int lane) {
        const int c = lane & 3, n = lane >> 2;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            float d = 0.f;
            if (t[i] >= 0) {
                const __nv_bfloat16* q = q_row(a, g, g.tile * C::RT + 2 * c + i, t[i]);
                for (int e = n; e < HD; e += 8) d = fmaf(__bfloat162float(q[e]), cache_elem<DYNAKV_FP8>(a.kpool, a.kexp, row, HD, e), d);
            }
            d = sum_over_keys(d);
            if (t[i] >= 0 && tree_sees(a, g, t[i], j)) {
                const float w = ex2(d * (a.scale * LOG2E) - (m[i] == -INFINITY ? 0.f : m[i]));
#pragma unroll
                for (int mt = 0; mt < MT; mt++)
#pragma unroll
                    for (int half = 0; half < 2; half++)
                        acc[mt][2 * half + i] = fmaf(w, cache_elem<DYNAKV_FP8>(a.vpool, a.vexp, row, HD, elem(mt, half, n)), acc[mt][2 * half + i]);
            }
        }
    }
    __device__ __forceinline__ void write(const TreeArgs& a, const Segment& g, int, int lane, bool whole, size_t slot) const {
        const int c = lane & 3, n = lane >> 2;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            if (t[i] < 0) continue;
            const int rl = 2 * c + i, r = g.tile * C::RT + rl;
            const size_t at = (size_t)(g.q0 + t[i]) * a.Hq + g.h * a.G + (r - t[i] * a.G);
            const float f = !whole ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
            __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(a.out) + at * HD;
            float* part = a.acc + (slot * C::RT + rl) * HD;
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const float x = acc[mt][i] * f, y = acc[mt][2 + i] * f;
                const int e = elem(mt, 0, n);
                if (whole) *reinterpret_cast<unsigned*>(o + e) = pack_bf16(x, y);
                else *reinterpret_cast<float2*>(part + e) = make_float2(x, y);
            }
            if (n == 0) {
                if (!whole) a.ml[slot * C::RT + rl] = make_float2(m[i], l[i]);
                else if (a.lse) a.lse[at] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * LN2;
            }
        }
    }
};

// ---------------------------------------------------------------------------------- fp32 consumers
//
// Lane = key for the logits (q is read from shared memory, the same word for all lanes), lane = HD / 32 columns for the
// sums (the weights go through shared memory).  Every lane keeps all rows' running maxima; the sums l stay split
// over the lanes until the end.  16 rows per warp, or 4 (plain decoding of a small group), which is a quarter of the code and of
// the latency.
template <int HD, int RG, bool MOD>
struct F32Rows {
    using C = TreeCfg<HD, DYNAKV_F32, RG, MOD>;
    static constexpr int DPL = HD / 32, NR = C::rows;
    float acc[NR][DPL], m[NR], l[NR];
    unsigned q_s, p_s;             // shared memory: this row group's q [NR][HD], this warp's weights [NR][32]
    int rows;                      // rows of the warp that exist
    RowScore<MOD> score;           // lane r < NR: of row r

    __device__ __forceinline__ void start(const TreeArgs& a, const Segment& g, int rg, int lane) {
        rows = max(0, min(NR, g.T * a.G - (g.tile * C::RT + rg * NR)));
        if constexpr (MOD) {
            const int x = g.tile * C::RT + rg * NR + (lane & (NR - 1)), t = x / a.G;
            score.start(a, g, t < g.T ? t : -1, x);
        }
#pragma unroll
        for (int r = 0; r < NR; r++) {
            m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
            for (int d = 0; d < DPL; d++) acc[r][d] = 0.f;
        }
        (void)lane;
    }
    // q of the group's rows, scaled; rows that do not exist as zeros.  One warp, the loads of eight steps side by side.
    static __device__ __forceinline__ void load_q(const TreeArgs& a, const Segment& g, int rg, float* q_s, int lane) {
#pragma unroll 8
        for (int x = lane; x < NR * HD; x += 32) {
            const int r = g.tile * C::RT + rg * NR + x / HD, t = r / a.G;
            const float* q = reinterpret_cast<const float*>(a.q) + ((size_t)(g.q0 + t) * a.Hq + g.h * a.G + r - t * a.G) * HD;
            q_s[x] = t < g.T ? __ldg(q + x % HD) * (MOD ? chunk_factor(a).x : a.scale * LOG2E) : 0.f;
        }
    }
    __device__ __forceinline__ void page(const TreeArgs& a, const Segment& g, const PageIn& p, int lane, int rg) {
        // Four chains per logit, in pairs that share an instruction: one chain of 64 carries the sum of a few large channels through
        // all the rest.  Output error on such keys (one sequence of 2048 rows, logits up to 40): 1.4e-6 of its size with one
        // chain, 2e-7 to 8e-7 with four.  16 rows have registers for two steps at a time, not four.
        float2 s4[NR][2];
#pragma unroll
        for (int r = 0; r < NR; r++) s4[r][0] = s4[r][1] = make_float2(0.f, 0.f);
#pragma unroll (NR == 16 ? 2 : 4)
        for (int ch = 0; ch < HD / 4; ch++) {
            const uint4 k = lds16(p.k + chunk_at<C>(lane, ch));
#pragma unroll
            for (int r = 0; r < NR; r++) {
                const uint4 q = lds16(q_s + (r * HD + ch * 4) * 4);
                s4[r][0] = fma2(make_float2(__uint_as_float(q.x), __uint_as_float(q.y)), make_float2(__uint_as_float(k.x), __uint_as_float(k.y)), s4[r][0]);
                s4[r][1] = fma2(make_float2(__uint_as_float(q.z), __uint_as_float(q.w)), make_float2(__uint_as_float(k.z), __uint_as_float(k.w)), s4[r][1]);
            }
        }
        float s[NR];
#pragma unroll
        for (int r = 0; r < NR; r++) s[r] = (s4[r][0].x + s4[r][0].y) + (s4[r][1].x + s4[r][1].y);
        unsigned win = ~0u;                        // lane r < NR: the window of row r
        bool mask = p.mask;
        if constexpr (MOD) {
            win = page_window<MOD>(a, g, p, 0, score);
            mask = __any_sync(0xffffffffu, win != ~0u);
            if (a.cap > 0.f || a.slopes) {
                const float rest = chunk_factor(a).y;
#pragma unroll
                for (int r = 0; r < NR; r++) s[r] = score.from_lane(r).logit(a, s[r] * rest, p.key0 + lane);
            }
        } else if (p.mask) {
            const int x = g.tile * C::RT + rg * NR + (lane & (NR - 1)), t = x / a.G;
            win = t < g.T ? tree_window(a, g, t, p.key0) : 0u;
        }
#pragma unroll
        for (int r = 0; r < NR; r++) {
            if (mask && !((__shfl_sync(0xffffffffu, win, r) >> lane) & 1u)) s[r] = -INFINITY;
            float mx = s[r];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            if (mx > m[r] + LAZY) {                // the same in all lanes
                const float f = ex2(m[r] - mx);
                m[r] = mx; l[r] *= f;
#pragma unroll
                for (int d = 0; d < DPL; d++) acc[r][d] *= f;
            }
            const float w = exp2f(s[r] - (m[r] == -INFINITY ? 0.f : m[r]));
            l[r] += w;
            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(p_s + (r * 32 + lane) * 4), "f"(w) : "memory");
        }
        __syncwarp();
        // (MOD, rows of 128: two steps at a time find no registers, 32 query rows over 4 x 4096: 190 us, one at a time 145)
#pragma unroll (MOD && HD == 128 && NR == 16 ? 1 : 2)
        for (int k4 = 0; k4 < 8; k4++) {
            float v[4][DPL];
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const int key = k4 * 4 + y;
                if constexpr (DPL == 4) {
                    const uint4 u = lds16(p.v + chunk_at<C>(key, lane));
                    v[y][0] = __uint_as_float(u.x); v[y][1] = __uint_as_float(u.y); v[y][2] = __uint_as_float(u.z); v[y][3] = __uint_as_float(u.w);
                } else {
                    const unsigned at = p.v + chunk_at<C>(key, lane >> 1) + (lane & 1) * 8;
                    v[y][0] = lds_f32(at); v[y][1] = lds_f32(at + 4);
                }
            }
#pragma unroll
            for (int r = 0; r < NR; r++) {
                const uint4 u = lds16(p_s + (r * 32 + k4 * 4) * 4);
                const float w[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
#pragma unroll
                for (int y = 0; y < 4; y++)
#pragma unroll
                    for (int d = 0; d < DPL; d += 2) {
                        const float2 x = fma2(make_float2(w[y], w[y]), make_float2(v[y][d], v[y][d + 1]), make_float2(acc[r][d], acc[r][d + 1]));
                        acc[r][d] = x.x; acc[r][d + 1] = x.y;
                    }
            }
        }
        __syncwarp();
    }
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int r = 0; r < NR; r++) l[r] = warp_sum(l[r]);
    }
    __device__ __forceinline__ void dump(float* to, int lane) const {
#pragma unroll
        for (int r = 0; r < NR; r++) {
#pragma unroll
            for (int d = 0; d < DPL; d++) to[(r * DPL + d) * 32 + lane] = acc[r][d];
            if (lane == r) reinterpret_cast<float2*>(to + NR * HD)[r] = make_float2(m[r], l[r]);
        }
    }
    __device__ __forceinline__ void merge(const float* from, int lane) {
#pragma unroll
        for (int r = 0; r < NR; r++) {
            const float2 o = reinterpret_cast<const float2*>(from + NR * HD)[r];
            const float to = fmaxf(m[r], o.x), ref = to == -INFINITY ? 0.f : to;
            const float f0 = exp2f(m[r] - ref), f1 = exp2f(o.x - ref);
            l[r] = l[r] * f0 + o.y * f1;
            m[r] = to;
#pragma unroll
            for (int d = 0; d < DPL; d++) acc[r][d] = acc[r][d] * f0 + from[(r * DPL + d) * 32 + lane] * f1;
        }
    }
    __device__ __forceinline__ bool wild() const {
        bool bad = false;
#pragma unroll
        for (int r = 0; r < NR; r++)
#pragma unroll
            for (int d = 0; d < DPL; d++) bad |= far_out(acc[r][d]) && is_number(l[r]);
        return bad;
    }
    __device__ __forceinline__ void add_row(const TreeArgs& a, const Segment& g, int rg, long long row, int j, int lane) {
        const float* k = reinterpret_cast<const float*>(a.kpool) + row * HD;
        const float* v = reinterpret_cast<const float*>(a.vpool) + row * HD;
#pragma unroll
        for (int r = 0; r < NR; r++) {
            float d = 0.f;
            for (int e = lane; e < HD; e += 32) d = fmaf(lds_f32(q_s + (r * HD + e) * 4), k[e], d);
            d = warp_sum(d);
            const int x = g.tile * C::RT + rg * NR + r, t = x / a.G;
            if (r < rows && tree_sees(a, g, t, j)) {
                const float w = exp2f(d - (m[r] == -INFINITY ? 0.f : m[r]));
#pragma unroll
                for (int e = 0; e < DPL; e++) acc[r][e] = fmaf(w, v[lane * DPL + e], acc[r][e]);
            }
        }
    }
    __device__ __forceinline__ void write(const TreeArgs& a, const Segment& g, int rg, int lane, bool whole, size_t slot) const {
#pragma unroll
        for (int r = 0; r < NR; r++) {
            if (r >= rows) continue;
            const int rl = rg * NR + r, x = g.tile * C::RT + rl, t = x / a.G;
            const size_t at = (size_t)(g.q0 + t) * a.Hq + g.h * a.G + x - t * a.G;
            const float f = !whole ? 1.f : l[r] == 0.f ? 0.f : 1.f / l[r];
            float* o = whole ? reinterpret_cast<float*>(a.out) + at * HD : a.acc + (slot * C::RT + rl) * HD;
#pragma unroll
            for (int d = 0; d < DPL; d++) o[lane * DPL + d] = acc[r][d] * f;
            if (lane == 0) {
                if (!whole) a.ml[slot * C::RT + rl] = make_float2(m[r], l[r]);
                else if (a.lse) a.lse[at] = l[r] == 0.f ? -INFINITY : (m[r] + log2f(l[r])) * LN2;
            }
        }
    }
};

// ---------------------------------------------------------------------------------- the kernel

// Rows of a V page that must not reach the MMAs: those at or past the sequence's end are zeroed, and so are drafted rows
// that hold a NaN or an infinity, which are noted in `odd` (bit j: token j of the tree).  MOD: only the former.  One warp.
template <typename C, int DT, bool MOD>
__device__ __forceinline__ void mend_page(unsigned v, const Segment& g, int key0, unsigned* odd, int lane) {
    const int prefix = MOD ? g.n : g.n - g.T;
    unsigned wild = 0u;                                    // rows of the page with a value that is no number
    constexpr int chunks = C::page_bytes / 16;
    for (int x = lane; x < chunks; x += 32) {
        const unsigned at = v + x * 16;
        const int row = (x * 16 % (PAGE * C::panel_w)) / C::panel_w, pos = key0 + row;
        if (pos < prefix) continue;
        if (pos >= g.n) {
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};\n" ::"r"(at), "r"(0u) : "memory");
        } else {
            const uint4 u = lds16(at);
            const unsigned w[4] = {u.x, u.y, u.z, u.w};
            bool bad = false;
#pragma unroll
            for (int y = 0; y < 4; y++) {
                if constexpr (DT == DYNAKV_F32) bad |= (w[y] & 0x7f800000u) == 0x7f800000u;
                else if constexpr (DT == DYNAKV_BF16) bad |= (w[y] & 0x7f80u) == 0x7f80u || (w[y] & 0x7f800000u) == 0x7f800000u;
                else {
#pragma unroll
                    for (int z = 0; z < 4; z++) bad |= ((w[y] >> (8 * z)) & 0x7fu) == 0x7fu;
                }
            }
            if (bad) wild |= 1u << row;
        }
    }
    wild = __reduce_or_sync(0xffffffffu, wild);
    if (wild) {
        for (int x = lane; x < chunks; x += 32) {
            const int row = (x * 16 % (PAGE * C::panel_w)) / C::panel_w;
            if ((wild >> row) & 1u) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};\n" ::"r"(v + x * 16), "r"(0u) : "memory");
        }
        const int j = key0 + lane - prefix;
        if (((wild >> lane) & 1u) && j >= 0 && j < TREE_MAX) atomicOr(&odd[j >> 5], 1u << (j & 31));
    }
    fence_proxy_async();               // the copies that refill the stage come after these stores
    __syncwarp();
}

// The CTA's segments once more, by the consuming warps (chunk_again.cuh).
template <int HD, int DT, int RG>
__device__ __forceinline__ void tree_rows_again(const TreeArgs& a, const long long* sh, int warp, int* shared) {
    using C = TreeCfg<HD, DT, RG, true>;
    SegmentWalk<C::RT, true> walk(*reinterpret_cast<const Range*>(sh + PLAN_RANGE), sh);
    for (Segment g; walk.next(a, g);) {
        const AgainSeg part = {g.b, g.h, g.p0 * PAGE, min(g.n, g.p1 * PAGE), g.q0, g.T, g.n, min(C::RT, g.T * a.G - g.tile * C::RT), g.first && g.last, (size_t)blockIdx.x * 2 + (g.first ? 1 : 0)};
        chunk_segment_again<HD, DT, C::RT, false, C::consumers>(a, part, warp, shared,
            [&](int r) { const int x = g.tile * C::RT + r; return (long long)(g.q0 + x / a.G) * a.Hq + g.h * a.G + x % a.G; },
            [] { asm volatile("bar.sync 5, %0;\n" ::"n"(C::consumers * 32) : "memory"); });
    }
}
// As a call of its own, so that what it needs does not weigh on the kernel's registers.  Not for fp32 rows: with a call in it that kernel becomes slower (rows of 64,
// 4 x 4096, 16, 32 and 64 query rows: 58, 75 and 110 us without, 63, 85 and 127 with one).
template <int HD, int DT, int RG>
__device__ __noinline__ void tree_rows_again_call(const TreeArgs& a, const long long* sh, int warp, int* shared) { tree_rows_again<HD, DT, RG>(a, sh, warp, shared); }

template <int HD, int DT, int RG, bool MOD>
__global__ void __launch_bounds__((TreeCfg<HD, DT, RG, MOD>::threads), (TreeCfg<HD, DT, RG, MOD>::per_sm))
k_tree_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TreeArgs a) {
    using C = TreeCfg<HD, DT, RG, MOD>;
    constexpr int S = C::stages, KG = C::KG;
    extern __shared__ __align__(1024) unsigned char tree_smem[];
    unsigned char* at = tree_smem + S * C::stage_bytes;
    signed char* exps = reinterpret_cast<signed char*>(at); at += C::exp_bytes;
    float* q_s = reinterpret_cast<float*>(at); at += C::q_bytes;
    float* p_s = reinterpret_cast<float*>(at); at += C::p_bytes;
    float* dump = reinterpret_cast<float*>(at); at += C::merge_bytes;
    long long* sh = reinterpret_cast<long long*>(at); at += C::plan_words * 8;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(at); at += 2 * S * 8;
    int* rows_s = reinterpret_cast<int*>(at); at += 32 * 4;
    int* s_abort = reinterpret_cast<int*>(at); at += 16;
    unsigned* odd = reinterpret_cast<unsigned*>(at); at += 3 * 8 * 4;
    volatile int* meta = reinterpret_cast<volatile int*>(at);
    const unsigned ring = smem_u32(tree_smem);
    auto full = [&](int s) { return smem_u32(&bars[s]); };
    auto empty = [&](int s) { return smem_u32(&bars[S + s]); };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int s = 0; s < S; s++) { mbar_init(full(s), DT == DYNAKV_FP8 ? 2 : 1); mbar_init(empty(s), C::groups); }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (tid < 24) odd[tid] = 0u;
    pdl_wait();                                            // from here on the results of earlier kernels are read
    const Range range = tree_range<C::RT, MOD>(a, KG, sh);
    if (MOD && tid == 0) *reinterpret_cast<Range*>(sh + PLAN_RANGE) = range;
    __syncthreads();
    pdl_trigger();
    SegmentWalk<C::RT, MOD> walk(range, sh);
    Segment g;

    if (warp == C::consumers) {
        // =============================== producer ===============================
        // One lane issues, and walks through up to 32 pages without the others: with small pages its time per page sets the pace
        // (FP8 rows of 64: 500 cycles when the warp met at every page; 4 x 32768 rows 54 -> 52 us with this).
        int st = 0, items = 0;
        unsigned ph = 1;
        bool ok = true;
        while (ok && walk.next(a, g)) {
            for (int pc = g.p0; ok && pc < g.p1; pc += 32) {
                const int cnt = min(32, g.p1 - pc);
                int row = -1;
                if (lane < cnt && g.n > 0) {
                    const int id = a.page_table[(size_t)g.b * a.pages_per_seq + pc + lane];
                    if (id < 0 || id >= a.n_pages) tree_status(a, DYNAKV_ST_BOUNDS);
                    else row = (id * a.Hk + g.h) * PAGE;
                }
                rows_s[lane] = row;
                __syncwarp();
                if (lane == 0) {
                    for (int j = 0; j < cnt; j++) {
                        const int at_row = rows_s[j];
                        ok = mbar_wait(empty(st), ph);
                        if (!ok) break;
                        meta[st] = at_row >= 0;
                        if (at_row >= 0) {
                            mbar_arrive_expect_tx(full(st), C::stage_bytes);
                            tma_page(ring + st * C::stage_bytes, &map_k, at_row, full(st));
                            tma_page(ring + st * C::stage_bytes + C::page_bytes, &map_v, at_row, full(st));
                            if constexpr (DT == DYNAKV_FP8) {
                                copy32(smem_u32(exps + st * 64), a.kexp + at_row);
                                copy32(smem_u32(exps + st * 64 + 32), a.vexp + at_row);
                                copies_arrive(full(st));
                            }
                        } else {
                            mbar_arrive(full(st));
                            if constexpr (DT == DYNAKV_FP8) mbar_arrive(full(st));
                        }
                        items++;
                        if (++st == S) { st = 0; ph ^= 1; }
                    }
                }
                ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            }
        }
        if (!ok && lane == 0) {
            // a stage was not given back in time: report it and let the copies under way land before the block ends
            *s_abort = 1;
            tree_status(a, DYNAKV_ST_INTERNAL);
            for (int x = max(0, items - S); x < items; x++) mbar_wait(full(x % S), (x / S) & 1);
        }
    } else {
        // =============================== consumers ===============================
        const int rg = warp % C::groups, kg = warp / C::groups;
        constexpr bool F32 = DT == DYNAKV_F32;
        constexpr bool TURNED = DT == DYNAKV_FP8 && HD == 128 && RG == 0;
        typename std::conditional<F32, F32Rows<HD, RG, MOD>, typename std::conditional<TURNED, TurnedRows<MOD>, MmaRows<HD, F32 ? DYNAKV_BF16 : DT, RG, MOD>>::type>::type rows;
        auto all_sync = [&]() { asm volatile("bar.sync 5, %0;\n" ::"n"(C::consumers * 32) : "memory"); };
        auto group_sync = [&]() { asm volatile("bar.sync %0, %1;\n" ::"r"(6 + kg), "n"(C::groups * 32) : "memory"); };
        if constexpr (F32) { rows.q_s = smem_u32(q_s + rg * C::rows * HD); rows.p_s = smem_u32(p_s + warp * C::rows * 32); }
        // This group's items are every KG-th of the CTA: `ahead` items pass before its next one, which lies in stage `st` in phase `ph`.
        int ahead = kg, st = kg, seg = 0;
        unsigned ph = 0;
        bool dead = false, cut_end = false;
        while (walk.next(a, g)) {
            const int prefix = MOD ? g.n : g.n - g.T;
            unsigned* odd_now = odd + (seg % 3) * 8;
            if constexpr (F32) {
                all_sync();                            // nobody still reads the last segment's q
                if (kg == 0) F32Rows<HD, RG, MOD>::load_q(a, g, rg, q_s + rg * C::rows * HD, lane);
                all_sync();
            }
            rows.start(a, g, rg, lane);
            int pg = g.p0 + ahead;
            for (; pg < g.p1; pg += KG) {
                if (!dead && !__all_sync(0xffffffffu, mbar_try_wait(full(st), ph))) {
                    if (!__all_sync(0xffffffffu, !*reinterpret_cast<volatile int*>(s_abort) && mbar_wait(full(st), ph))) {
                        dead = true;
                        *reinterpret_cast<volatile int*>(s_abort) = 1;
                        tree_status(a, DYNAKV_ST_INTERNAL);
                    }
                }
                PageIn p;
                p.k = ring + st * C::stage_bytes; p.v = p.k + C::page_bytes; p.exps = exps + st * 64;
                p.scales = reinterpret_cast<float4*>(exps + S * 64) + warp * 32;
                p.key0 = pg * PAGE;
                p.mask = p.key0 + PAGE > prefix;       // holds drafted rows or the end of the sequence
                // a page that the table does not name was not copied: the stage holds an older one
                const bool there = !dead && meta[st] != 0;
                if (p.mask) {                          // the same in all warps of the group, dead or not
                    if (rg == 0 && there) mend_page<C, DT, MOD>(p.v, g, p.key0, odd_now, lane);
                    if (C::groups > 1) group_sync();
                }
                if (there) {
                    if constexpr (F32) rows.page(a, g, p, lane, rg);
                    else rows.page(a, g, p, lane);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(st));
                st += KG;
                if (st >= S) { st = kg; ph ^= 1; }
            }
            ahead = pg - g.p1;
            rows.finish();
            if (!MOD && tid < 8) odd[((seg + 1) % 3) * 8 + tid] = 0u;      // last read before the previous segment's barrier
            if (kg > 0) rows.dump(dump + ((kg - 1) * C::groups + rg) * (C::dump_bytes / 4), lane);
            all_sync();
            if (kg == 0) {
#pragma unroll
                for (int src = 1; src < KG; src++) rows.merge(dump + ((src - 1) * C::groups + rg) * (C::dump_bytes / 4), lane);
            }
            if (KG > 1) all_sync();                    // the boxes may be filled again
            if (kg == 0) {
                if constexpr (MOD) {
                    if (rows.wild()) odd[0] = 1u;      // seen to when all is done
                }
                for (int w = 0; w < (MOD ? 0 : TREE_MAX / 32); w++) {
                    unsigned bits = odd_now[w];
                    while (bits) {
                        const int j = w * 32 + __ffs(bits) - 1;
                        bits &= bits - 1;
                        const int pos = prefix + j, page = a.page_table[(size_t)g.b * a.pages_per_seq + pos / PAGE];
                        rows.add_row(a, g, rg, ((long long)page * a.Hk + g.h) * PAGE + pos % PAGE, j, lane);
                    }
                }
                rows.write(a, g, rg, lane, g.first && g.last, (size_t)blockIdx.x * 2 + (g.first ? 1 : 0));
            }
            if (g.last && !g.first) { cut_end = true; if (tid == 0) describe_cut_unit(a, g, walk.r); }
            seg++;
        }
        if (tid == 0) a.desc[(size_t)blockIdx.x * 8 + DESC_VALID] = cut_end ? 1 : 0;
        if constexpr (MOD) {
            // all is done: rows whose sums are no numbers are taken again
            all_sync();
            if (odd[0] && !*reinterpret_cast<volatile int*>(s_abort)) {
                if constexpr (F32) tree_rows_again<HD, DT, RG>(a, sh, warp, reinterpret_cast<int*>(tree_smem));
                else tree_rows_again_call<HD, DT, RG>(a, sh, warp, reinterpret_cast<int*>(tree_smem));
            }
        }
    }
}

}  // namespace dkv
