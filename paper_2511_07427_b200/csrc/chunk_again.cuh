// Query rows of dynakv_attend_chunk that are taken again by themselves.
//
// The kernels multiply a tile's weights with all rows of V of a stage, so that 0 * NaN reaches the sums of query rows that do not see
// the row of V in which the NaN lies.  (0 * infinity does too, and sums of large values may leave fp32 although the result fits it.)  While they walk over their
// segments they only note that it happened.  A CTA that has a note goes over its segments once more when all of them are done and no copy, product or
// wait is left: rows whose values are no numbers, in out or in a record, and need not be, are taken again, a warp per row, from the rows that the query sees
// alone.  (Done between two units it kept the warps that load and multiply waiting beyond the limit of their waits, from some tens of thousands
// of rows on.  Done by the launch that merges, whose registers it trebles, it cost calls without any such row 7 to 16 us.)
// Rows whose sum of weights is no number (a NaN in the query, or in a key that it sees) are not taken again: their result is NaN.
#pragma once

#include <float.h>

#include "chunk_plan.cuh"
#include "fp8_rows.cuh"
#include "head_rows.cuh"

namespace dkv {

__device__ __forceinline__ bool is_number(float x) { return fabsf(x) <= FLT_MAX; }
// A record's sums are as good as none from here on, because those of all records of a unit together might leave fp32's range.
constexpr float AGAIN_FAR = 0x1p100f;
__device__ __forceinline__ bool far_out(float x) { return !(fabsf(x) <= AGAIN_FAR); }

// This lane's HD / 32 consecutive elements of a row of the pool, FP8 without the row's scale.
template <int HD, int DT>
__device__ __forceinline__ void row_part(const unsigned char* pool, long long row, int lane, float (&x)[HD / 32]) {
    constexpr int E = HD / 32;
    if constexpr (DT == DYNAKV_F32) {
        const float* p = reinterpret_cast<const float*>(pool) + row * HD + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) { const float2 v = *reinterpret_cast<const float2*>(p + e); x[e] = v.x; x[e + 1] = v.y; }
    } else if constexpr (DT == DYNAKV_BF16) {
        const unsigned* p = reinterpret_cast<const unsigned*>(reinterpret_cast<const __nv_bfloat16*>(pool) + row * HD + lane * E);
#pragma unroll
        for (int e = 0; e < E; e += 2) { const unsigned v = p[e / 2]; x[e] = __uint_as_float(v << 16); x[e + 1] = __uint_as_float(v & 0xffff0000u); }
    } else {
        const unsigned short* p = reinterpret_cast<const unsigned short*>(pool + row * HD + lane * E);
#pragma unroll
        for (int e = 0; e < E; e += 2) { const float2 v = fp8_unpack2(p[e / 2], 1.f); x[e] = v.x; x[e + 1] = v.y; }
    }
}

// What is taken again: a segment of a unit, KV head h of sequence seq with rows [k0, k1).
struct AgainSeg {
    int seq, h, k0, k1, q0, T, n;
    int rows;                                      // of the tile
    bool whole;                                    // written to out, or (else) to the record `slot`
    size_t slot;
};
// Where the segment's query rows lie.  RT, COLS: how the kernel lays out its records, four columns of all rows side by side or row by row.
template <int HD, int RT, bool COLS>
__device__ __forceinline__ float* record_part(const TreeArgs& a, size_t slot, int row, int lane) {
    constexpr int E = HD / 32;
    return COLS ? a.acc + ((slot * (HD / 4) + lane * E / 4) * RT + row) * 4 + lane * E % 4 : a.acc + (slot * RT + row) * HD + lane * E;
}
// This lane's values of a row of out or of a record that are no numbers, as bits.
template <int HD, int DT, int RT, bool COLS>
__device__ __forceinline__ unsigned odd_values(const TreeArgs& a, const AgainSeg& g, long long place, int row, int lane) {
    constexpr int E = HD / 32;
    unsigned bits = 0u;
#pragma unroll
    for (int e = 0; e < E; e++) {
        const size_t at = (size_t)place * HD + lane * E + e;
        const float x = !g.whole ? record_part<HD, RT, COLS>(a, g.slot, row, lane)[e] : DT == DYNAKV_F32 ? reinterpret_cast<const float*>(a.out)[at] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(a.out)[at]);
        if (g.whole ? !is_number(x) : far_out(x)) bits |= 1u << e;
    }
    return bits;
}

// A warp's sums of 32 values per lane, of the j-th ones in lane j: 31 exchanges instead of 160.
__device__ __forceinline__ float transpose_sum(float (&d)[32], int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < o; j++) {
            const bool up = lane & o;
            const float keep = up ? d[j + o] : d[j], give = up ? d[j] : d[j + o];
            d[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    return d[0];
}

// Packed token `token` and query head hq by one warp, row `row` of the tile: two passes over the rows that it sees, a page at a time, lane j with the
// score of the page's row j.  Weights add up to 1 before they meet V.
template <int HD, int DT, int RT, bool COLS>
__device__ __forceinline__ void chunk_row_again(const TreeArgs& a, const AgainSeg& g, int token, int hq, int row) {
    constexpr int E = HD / 32;
    constexpr float LOG2_E = 1.4426950408889634f;
    const int lane = threadIdx.x & 31, place = g.n - g.T + token - g.q0;
    const size_t at = ((size_t)token * a.Hq + hq) * HD + lane * E;
    int lo, hi;
    chunk_sees(a, token, place, g.n, lo, hi);
    lo = max(lo, g.k0); hi = min(hi, g.k1);
    const float slope = a.slopes ? a.slopes[hq] * LOG2_E : 0.f, factor = a.cap > 0.f ? a.scale / a.cap : a.scale * LOG2_E;
    float q[E];
#pragma unroll
    for (int e = 0; e < E; e++) q[e] = DT == DYNAKV_F32 ? reinterpret_cast<const float*>(a.q)[at + e] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(a.q)[at + e]);
    auto first_row = [&](int column) {                         // of the page in the pool, -1: there is none
        const int page = chunk_page(a, g.seq, column);
        return page < 0 ? -1ll : ((long long)page * a.Hk + g.h) * PAGE;
    };
    auto score = [&](int column, long long first) {
        float d[PAGE];
#pragma unroll
        for (int j = 0; j < PAGE; j++) {
            float k[E];
            row_part<HD, DT>(a.kpool, first + j, lane, k);
            d[j] = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) d[j] = fmaf(q[e], k[e], d[j]);
        }
        float x = transpose_sum(d, lane);
        if constexpr (DT == DYNAKV_FP8) x *= pow2f(a.kexp[first + lane]);
        x *= factor;
        if (a.cap > 0.f) x = a.cap * LOG2_E * tanhf(x);
        const int pos = column * PAGE + lane;
        if (a.slopes) x = fmaf(-slope, fabsf((float)(place - pos)), x);
        return pos >= lo && pos < hi ? x : -INFINITY;
    };
    float m = -INFINITY, l = 0.f;                              // of this lane's rows
#pragma unroll 1
    for (int column = lo / PAGE; column * PAGE < hi; column++) {
        const long long first = first_row(column);
        if (first < 0) continue;
        const float x = score(column, first), to = fmaxf(m, x), ref = to == -INFINITY ? 0.f : to;
        l = l * exp2f(m - ref) + exp2f(x - ref);
        m = to;
    }
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = top == -INFINITY ? 0.f : top, total = warp_sum(l * exp2f(m - ref));
    const float norm = total == 0.f ? 0.f : 1.f / total;
    float o[E];
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = 0.f;
#pragma unroll 1
    for (int column = lo / PAGE; column * PAGE < hi && total != 0.f; column++) {
        const long long first = first_row(column);
        if (first < 0) continue;
        float w = exp2f(score(column, first) - ref) * norm;
        if constexpr (DT == DYNAKV_FP8) w *= pow2f(a.vexp[first + lane]);
        const int from = max(lo - column * PAGE, 0), to = min(hi - column * PAGE, PAGE);
#pragma unroll 8
        for (int j = from; j < to; j++) {
            const float p = __shfl_sync(0xffffffffu, w, j);
            float v[E];
            row_part<HD, DT>(a.vpool, first + j, lane, v);
#pragma unroll
            for (int e = 0; e < E; e++) o[e] = fmaf(p, v[e], o[e]);
        }
    }
    if (!g.whole) {
        // relative to the record's own reference, which stays (and with it every bit of lse); or where that leaves fp32's range, to one 2^10 above the sum
        float2* ml = a.ml + g.slot * RT + row;
        const float2 was = *ml;
        float by = 0.f;
        bool far = false;
#pragma unroll
        for (int e = 0; e < E; e++) far |= is_number(o[e]) && far_out(o[e] * was.y);
        if (__any_sync(0xffffffffu, far) && was.y > 0.f) by = (float)(ilogbf(was.y) + 11);
        const float sum = was.y * exp2f(-by);
        float* to = record_part<HD, RT, COLS>(a, g.slot, row, lane);
#pragma unroll
        for (int e = 0; e < E; e++) to[e] = o[e] * sum;
        __syncwarp();
        if (lane == 0 && by != 0.f) *ml = make_float2(was.x + by, sum);
    } else if constexpr (DT == DYNAKV_F32) {
#pragma unroll
        for (int e = 0; e < E; e++) reinterpret_cast<float*>(a.out)[at + e] = o[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) *reinterpret_cast<unsigned*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at + e) = pack_bf16(o[e], o[e + 1]);
    }
}

// A segment, by WARPS warps (this one: `warp`) that all call it.  What a row of V that holds no number does to a column of a query row that sees it needs no sums: the column
// is NaN, or infinite where all that it sees of this kind are infinities of one sign.  So the segment's rows of V are looked through once, for the first and the last NaN and
// infinity of either sign in every column, and a query row is taken again only where a column's value has no such reason.  (A row of V between the first and the last leaves
// it open, which counts as none.)
// place_of(row): packed token * heads + query head, -1: there is none.  shared: AGAIN_SHARED HD + 1 ints; sync: a barrier of those warps.
constexpr int AGAIN_SHARED = 6;
template <int HD, int DT, int RT, bool COLS, int WARPS, typename PLACE, typename SYNC>
__device__ __forceinline__ void chunk_segment_again(const TreeArgs& a, const AgainSeg& g, int warp, int* shared, PLACE place_of, SYNC sync) {
    constexpr int E = HD / 32;
    const int lane = threadIdx.x & 31;
    int* any = shared + AGAIN_SHARED * HD;                     // a row of the segment has such a value
    for (int c = warp * 32 + lane; c <= AGAIN_SHARED * HD; c += WARPS * 32) shared[c] = c == AGAIN_SHARED * HD ? 0 : c / HD % 2 == 0 ? 0x7fffffff : -1;
    sync();
    for (int r = warp; r < g.rows; r += WARPS) {
        const long long place = place_of(r);
        if (place >= 0 && odd_values<HD, DT, RT, COLS>(a, g, place, r, lane)) *any = 1;
    }
    sync();
    if (!*any) { sync(); return; }
#pragma unroll 1
    for (int column = g.k0 / PAGE; column * PAGE < g.k1; column++) {
        const int page = chunk_page(a, g.seq, column);
        if (page < 0) continue;
        for (int j = warp; j < PAGE; j += WARPS) {
            float v[E];
            row_part<HD, DT>(a.vpool, ((long long)page * a.Hk + g.h) * PAGE + j, lane, v);
            const int pos = column * PAGE + j;
#pragma unroll
            for (int e = 0; e < E; e++)
                if (!is_number(v[e]) && pos < g.k1) {
                    int* at = shared + (v[e] != v[e] ? 0 : v[e] > 0.f ? 2 : 4) * HD + lane * E + e;
                    atomicMin(at, pos); atomicMax(at + HD, pos);
                }
        }
    }
    sync();
#pragma unroll 1
    for (int r = warp; r < g.rows; r += WARPS) {
        const long long place = place_of(r);
        if (place < 0) continue;                               // the same in the whole warp
        const unsigned bits = odd_values<HD, DT, RT, COLS>(a, g, place, r, lane);
        const int token = (int)(place / a.Hq);
        int lo, hi;
        chunk_sees(a, token, g.n - g.T + token - g.q0, g.n, lo, hi);
        lo = max(lo, g.k0); hi = min(hi, g.k1);
        const bool nothing = g.whole ? a.lse && a.lse[place] != a.lse[place] : !is_number(a.ml[g.slot * RT + r].y);
        if (nothing) continue;                                 // the same in the whole warp
        bool need = false;
        float value[E];                                        // 0: to be taken again
#pragma unroll
        for (int e = 0; e < E; e++) {
            bool sees[3], open[3];
#pragma unroll
            for (int k = 0; k < 3; k++) {
                const int first = shared[2 * k * HD + lane * E + e], last = shared[(2 * k + 1) * HD + lane * E + e];
                sees[k] = (first >= lo && first < hi) || (last >= lo && last < hi);
                open[k] = !sees[k] && first < lo && last >= hi;
            }
            value[e] = 0.f;
            if (sees[0]) value[e] = NAN;
            else if (!open[0] && !open[1] && !open[2]) value[e] = sees[1] ? sees[2] ? NAN : INFINITY : sees[2] ? -INFINITY : 0.f;
            if (!((bits >> e) & 1u)) value[e] = 0.f;
            else need |= value[e] == 0.f;
        }
        if (__any_sync(0xffffffffu, need)) chunk_row_again<HD, DT, RT, COLS>(a, g, token, (int)(place - (long long)token * a.Hq), r);
#pragma unroll
        for (int e = 0; e < E; e++) {
            if (value[e] == 0.f) continue;
            const size_t at = (size_t)place * HD + lane * E + e;
            if (!g.whole) record_part<HD, RT, COLS>(a, g.slot, r, lane)[e] = value[e];
            else if (DT == DYNAKV_F32) reinterpret_cast<float*>(a.out)[at] = value[e];
            else reinterpret_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16(value[e]);
        }
    }
    sync();
}

}  // namespace dkv
