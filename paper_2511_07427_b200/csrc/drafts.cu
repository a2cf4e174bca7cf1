// What follows the attention of drafted tokens: which of them are accepted (dynakv_verify_drafts), and their rows moved
// together (dynakv_rows_keep).
//
// Verification.  With p the target's distribution behind a kept token (softmax of its logits over the temperature, or all of it on the first
// largest logit), a drafted child x is accepted when u q(x) < p(x); refused, it leaves max(p - q, 0) to its younger siblings and to
// the token that is drawn at the end, all up to a factor that is carried along.  A draft that was not drawn has q = 1 at x, so that what is
// left is p without x.
//   k_row_stats: the one pass over the logits, HBM bound: (largest, first place of it, sum of exp) of every row, in pieces.
//   k_verify, a cluster of CTAs per sequence: every draft's test from those and one logit, at once for all drafts; the walk in shared
//     memory; then the drawing from the last kept token's row, which is by inverse sums in 64 bits: among 10^5 tokens fp32 sums
//     misplace the draw with a chance of about 10^-3, and the same numbers have to give the same token however the sums are split.
// Measured, calls one after the other: 64 sequences of 6 tokens over 128256, drafts drawn, 72 us: 22 for the rows, 8 until the walk is done, 15
// each for the target's sum and for what is left of it (64-bit operations and the loads that feed them, 128 CTAs), 3 for the place of the draw.
// 16 trees of 32 over 50257: 31 us.  One sequence of 5 over 32000: 14 us on the device, a chain of dependent loads; 22 us of host time.
#include <cooperative_groups.h>
#include <float.h>

#include "bulk_copy.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"

namespace dkv {

namespace cg = cooperative_groups;

constexpr int RS_THREADS = 128, RS_VECS = 4, RS_BYTES = RS_THREADS * RS_VECS * 16;     // a block's piece of a row
constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32, VF_CLUSTER = 8;

struct VerifyArgs {
    const void* logits; long long stride;  // row stride, elements
    const int* tokens; const int* q_start; const int* parent;
    const float* uniform; const float* heat;
    const float* draft; long long draft_stride;
    int* kept; int* dropped; int* path; int* next;
    float4* stats;                         // [n_tokens][pieces]: largest, its place (bits of an int), sum of exp
    int n_tokens, n_seqs, vocab, most, pieces;
};

// Tokens of sequence b; none where its range is not one.
__device__ __forceinline__ bool verify_range(const VerifyArgs& a, int b, int& q0, int& T) {
    q0 = a.q_start[b];
    const int q1 = a.q_start[b + 1];
    const bool ok = q0 >= 0 && q1 >= q0 && q1 <= a.n_tokens && q1 - q0 <= a.most;
    T = ok ? q1 - q0 : 0;
    return ok;
}

// A sequence's temperature, 0: the first largest logit.  Beyond 2^-100 and 2^100 the distribution stays the same, while quotients would leave fp32's range.
__device__ __forceinline__ float heat_of(const VerifyArgs& a, int b) { const float h = a.heat[b]; return h > 0.f ? fminf(fmaxf(h, 0x1p-100f), 0x1p100f) : 0.f; }

struct Best { float top; int at; };
__device__ __forceinline__ Best better(Best a, Best b) { return b.top > a.top || (b.top == a.top && b.at < a.at) ? b : a; }

// A piece is loaded whole, every thread's 64 bytes on their way before anything is looked at: then the largest, then the sum relative to
// it.  98 MB of bf16 logits take 22 us (4.4 TB/s; pieces of 32 KB in blocks of 256 threads 24 us; a running maximum with two loads under way 31 us).
template <typename T>
__global__ void __launch_bounds__(RS_THREADS, 12) k_row_stats(const VerifyArgs a) {
    constexpr int N = 16 / sizeof(T);      // elements of a load
    const int row = blockIdx.x, piece = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ float heat_s;
    __shared__ float top_s[RS_THREADS / 32], sum_s[RS_THREADS / 32];
    __shared__ int at_s;
    pdl_wait();
    const T* p = reinterpret_cast<const T*>(a.logits) + (long long)row * a.stride;
    // elements before the first 16-byte boundary, whole vectors, and what is left
    const int head = min(a.vocab, (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T))), vecs = (a.vocab - head) / N, tail = a.vocab - head - vecs * N;
    const int v0 = piece * (RS_THREADS * RS_VECS) + tid;
    const uint4* pv = reinterpret_cast<const uint4*>(p + head);
    const unsigned low = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;                   // -infinity
    uint4 w[RS_VECS];
#pragma unroll
    for (int i = 0; i < RS_VECS; i++) w[i] = v0 + i * RS_THREADS < vecs ? __ldg(pv + v0 + i * RS_THREADS) : make_uint4(low, low, low, low);
    // the first piece's threads have the elements around the vectors
    float x_odd = -INFINITY;
    int at_odd = 0x7fffffff;
    if (piece == 0 && tid < head + tail) { at_odd = tid < head ? tid : vecs * N + tid; x_odd = to_f(p[at_odd]); }
    if (tid == 0) { heat_s = -1.f; at_s = 0x7fffffff; }
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += RS_THREADS)       // at most one sequence has the row
        if (a.q_start[b] <= row && row < a.q_start[b + 1]) heat_s = heat_of(a, b);
    auto elem = [&](int i, int e) {
        const unsigned u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[e]);
        else return __uint_as_float(e & 1 ? u[e >> 1] & 0xffff0000u : u[e >> 1] << 16);
    };
    float m = x_odd;
#pragma unroll
    for (int i = 0; i < RS_VECS; i++)
#pragma unroll
        for (int e = 0; e < N; e++) m = fmaxf(m, elem(i, e));
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) top_s[warp] = top;
    __syncthreads();
    pdl_trigger();
    const float heat = heat_s;
    if (heat < 0.f) return;                                // a row of no sequence
    top = top_s[0];
#pragma unroll
    for (int k = 1; k < RS_THREADS / 32; k++) top = fmaxf(top, top_s[k]);
    if (m == top) {                                        // the few threads that have the largest look for its place
        int at = x_odd == m ? at_odd : 0x7fffffff;
#pragma unroll
        for (int i = 0; i < RS_VECS; i++)
#pragma unroll
            for (int e = 0; e < N; e++) if (elem(i, e) == m && v0 + i * RS_THREADS < vecs) at = min(at, head + (v0 + i * RS_THREADS) * N + e);
        atomicMin(&at_s, at);
    }
    float sum = 0.f;
    if (heat > 0.f && top > -INFINITY) {
        const float f = 1.4426950408889634f / heat;
        const float2 f2 = make_float2(f, f), less = make_float2(-top, -top);
        float2 part = make_float2(x_odd > -INFINITY ? ex2((x_odd - top) * f) : 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < RS_VECS; i++)
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const float2 y = mul2(add2(make_float2(elem(i, e), elem(i, e + 1)), less), f2);        // not x f - m f, which is off by the rounding of m f
                part = add2(part, make_float2(ex2(y.x), ex2(y.y)));
            }
        sum = warp_sum(part.x + part.y);
    }
    if (lane == 0) sum_s[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        float total = 0.f;
#pragma unroll
        for (int k = 0; k < RS_THREADS / 32; k++) total += sum_s[k];
        a.stats[(size_t)row * a.pieces + piece] = make_float4(top, __int_as_float(at_s), total, 0.f);
    }
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Bytes [p, p + n) into L2, as far as whole 16-byte pieces go.
__device__ __forceinline__ void prefetch_l2(const void* p, size_t n) {
    const uintptr_t from = ((uintptr_t)p + 15) & ~(uintptr_t)15, end = ((uintptr_t)p + n) & ~(uintptr_t)15;
    for (uintptr_t at = from; at < end; at += 65536)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(at), "r"((unsigned)(end - at < 65536 ? end - at : 65536)) : "memory");
}

constexpr int EXP_TABLE = 16;
__device__ const double two_to[EXP_TABLE] = {      // 2^(j / 16)
    1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927,
    1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543, 1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};
// N values of 2^((l - top) * scale) in 64 bits, l <= top: the exponent is n + j / 16 + r with |r| <= 1 / 32, the factor of j comes from a table
// (in shared memory once per pair of lanes, so that no two meet in a bank) and that of r from its series up to r^5 (what is left out is
// below 2^-42 of the value, far below what could misplace a draw).  Values below 2^-1000 are 0.  Step by step for all N, because a 64-bit operation's result is a long time in coming: one value after the other,
// the 8 M of a large call took 140 us.
template <int N>
__device__ __forceinline__ void exp2_64(const float (&l)[N], double top, double scale, float lowest, const double* table, double (&w)[N]) {
    const double shift = 6755399441055744.0 / EXP_TABLE;   // 1.5 * 2^52 in units of 1 / 16: the sum's last bits are round(16 x)
    int k[N];
    double r[N], p[N];
#pragma unroll
    for (int i = 0; i < N; i++) w[i] = (double)l[i] - top;
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(w[i], scale, shift);
#pragma unroll
    for (int i = 0; i < N; i++) { k[i] = __double2loint(p[i]); p[i] -= shift; }
#pragma unroll
    for (int i = 0; i < N; i++) { r[i] = fma(w[i], scale, -p[i]); w[i] = table[(k[i] & (EXP_TABLE - 1)) * 16]; }
    // (ln 2)^k / k!
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(r[i], 0.0013333558146428441, 0.0096181291076284769);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], r[i], 0.055504108664821576);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], r[i], 0.24022650695910069);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], r[i], 0.69314718055994529);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] *= r[i];
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], w[i], w[i]);
#pragma unroll
    for (int i = 0; i < N; i++) w[i] = l[i] >= lowest ? __hiloint2double(__double2hiint(p[i]) + ((k[i] >> 4) << 20), __double2loint(p[i])) : 0.0;
}
// The logit below which a weight is 0: rounded up, to the largest one at most, so that no weight is below 2^-1000, the largest never left out, and -infinity always.
__device__ __forceinline__ float lowest_logit(double top, double scale) { return __double2float_ru(top - 1000.0 / scale); }

constexpr int LEFT_STEPS = 8;                      // loads of so many steps side by side

struct VerifyShared {
    double weight[TREE_MAX], sum[TREE_MAX];        // of a draft: its token's weight behind its parent; [a row]: sum of the row's weights
    float top[TREE_MAX];                           // [a row] largest logit
    int best[TREE_MAX];                            //         first place of it
    int token[TREE_MAX], up[TREE_MAX], first[TREE_MAX];
    unsigned char again[TREE_MAX];                 // an older sibling has the same token
    double table[EXP_TABLE * 16];
    double slices[VF_CLUSTER * VF_WARPS], part[VF_WARPS];
    double held[32 * LEFT_STEPS];                  // weights of the run in which the drawn token lies
    int last, refused, found;
};

// What is left of a row's distribution: its weights, or (norm > 0) weight * norm - q, without the tokens of `refused` children.
template <typename T>
struct RowLeft {
    const T* row;
    const float* q;
    double top, scale, norm;
    int refused;
};
// The sum over elements [from, end), by one warp; `held`: the weights of up to 32 LEFT_STEPS of them are kept there.  One function,
// not inlined: the code is run once or twice, and fetching it is what it would cost.
template <typename T>
__device__ __noinline__ double left_sum(const RowLeft<T> a, const VerifyShared& sh, int from, int end, double* held) {
    const int lane = threadIdx.x & 31;
    const bool less = a.norm > 0.0;
    const float lowest = lowest_logit(a.top, a.scale);
    double s[2] = {0.0, 0.0};
    T l[LEFT_STEPS];
    float q[LEFT_STEPS] = {};
    // The next elements, while these are worked on.  Every lane loads, those behind the end the last one again: loads under conditions of their
    // own wait for one another.
    auto fetch = [&](int base) {
#pragma unroll
        for (int k = 0; k < LEFT_STEPS; k++) l[k] = a.row[min(base + k * 32, end - 1)];
        if (less) {
#pragma unroll
            for (int k = 0; k < LEFT_STEPS; k++) q[k] = a.q[min(base + k * 32, end - 1)];
        }
    };
    if (from < end) fetch(from + lane);
    for (int base = from + lane; base - lane < end; base += 32 * LEFT_STEPS) {
        double w[LEFT_STEPS];
        float now[LEFT_STEPS], minus[LEFT_STEPS];
#pragma unroll
        for (int k = 0; k < LEFT_STEPS; k++) { now[k] = base + k * 32 < end ? to_f(l[k]) : -INFINITY; minus[k] = q[k]; }
        for (int r = 0; r < a.refused; r++) {              // a refused token weighs nothing
            const int off = sh.token[sh.first[r]] - base;
            if ((unsigned)(off + lane) >= 32u * LEFT_STEPS) continue;          // the same in the whole warp
#pragma unroll
            for (int k = 0; k < LEFT_STEPS; k++) if (off == k * 32) now[k] = -INFINITY;
        }
        if (base - lane + 32 * LEFT_STEPS < end) fetch(base + 32 * LEFT_STEPS);
        exp2_64(now, a.top, a.scale, lowest, sh.table + (lane & 15), w);
        if (less) {
#pragma unroll
            for (int k = 0; k < LEFT_STEPS; k++) w[k] = fma(w[k], a.norm, -(double)minus[k]);
#pragma unroll
            for (int k = 0; k < LEFT_STEPS; k++) w[k] = w[k] > 0.0 ? w[k] : 0.0;
        }
        if (held) {
#pragma unroll
            for (int k = 0; k < LEFT_STEPS; k++) held[k * 32 + lane] = w[k];
        }
#pragma unroll
        for (int k = 0; k < LEFT_STEPS; k += 2) { s[0] += w[k]; s[1] += w[k + 1]; }
    }
    return warp_sum64(s[0] + s[1]);
}

// 512 threads per CTA, one slice of the vocabulary per warp.
template <typename T>
__global__ void __launch_bounds__(VF_THREADS) k_verify(const VerifyArgs a) {
    __shared__ VerifyShared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = gridDim.x, cta = blockIdx.x, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    int q0, n;
    const bool ok = verify_range(a, b, q0, n);
    const T* logits = reinterpret_cast<const T*>(a.logits);
    if (n == 0) {                                          // the same in the whole cluster
        if (cta == 0) {
            for (int i = tid; i < a.most; i += VF_THREADS) a.path[(size_t)b * a.most + i] = -1;
            if (tid == 0) { a.kept[b] = 0; a.dropped[b] = ok ? 0 : -1; a.next[b] = -1; }
        }
        return;
    }
    const float heat = heat_of(a, b);
    const bool draws = heat > 0.f;
    const double scale = 1.4426950408889634074 / (double)heat;             // weights are 2^((logit - largest) * scale)
    if (tid < EXP_TABLE * 16) sh.table[tid] = two_to[tid / 16];
    __syncthreads();
    auto weight_of = [&](float l, float top) {
        const float x[1] = {l};
        double w[1];
        exp2_64(x, (double)top, scale, lowest_logit((double)top, scale), sh.table + (lane & 15), w);
        return w[0];
    };
    // ---- every row's largest logit and sum, a warp per row
    for (int i = warp; i < n; i += VF_WARPS) {
        const float4* st = a.stats + (size_t)(q0 + i) * a.pieces;
        Best best = {-INFINITY, 0x7fffffff};
        for (int k = lane; k < a.pieces; k += 32) best = better(best, Best{st[k].x, __float_as_int(st[k].y)});
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = better(best, Best{__shfl_xor_sync(0xffffffffu, best.top, o), __shfl_xor_sync(0xffffffffu, best.at, o)});
        double sum = 0.0;
        for (int k = lane; k < a.pieces; k += 32)
            if (draws && st[k].x > -INFINITY) sum += (double)st[k].z * weight_of(st[k].x, best.top);
        sum = warp_sum64(sum);
        if (lane == 0) { sh.top[i] = best.top; sh.best[i] = best.at; sh.sum[i] = sum; }
    }
    for (int i = tid; i < n; i += VF_THREADS) {
        sh.token[i] = a.tokens[q0 + i];
        const int up = i == 0 ? -1 : a.parent ? a.parent[q0 + i] : i - 1;
        sh.up[i] = up >= 0 && up < i ? up : -1;            // a draft without a parent before it is never reached
        sh.first[i] = n;
    }
    __syncthreads();
    auto weight = [&](int row, int x) {                    // of token x behind row `row`, relative to the row's largest
        if (x < 0 || x >= a.vocab || sh.top[row] == -INFINITY) return 0.0;
        return weight_of(to_f(logits[(long long)(q0 + row) * a.stride + x]), sh.top[row]);
    };
    for (int i = tid; i < n; i += VF_THREADS) {
        const int up = sh.up[i];
        sh.weight[i] = draws && up >= 0 ? weight(up, sh.token[i]) : 0.0;
        bool again = false;
        if (a.parent && up >= 0) for (int s = up + 1; s < i; s++) again |= sh.up[s] == up && sh.token[s] == sh.token[i];
        sh.again[i] = again;
    }
    __syncthreads();
    // ---- every draft's test, against what its older siblings leave
    for (int i = tid; i < n; i += VF_THREADS) {
        const int up = sh.up[i], x = sh.token[i];
        if (up < 0) continue;
        bool pass;
        if (!draws) pass = sh.best[up] == x && sh.top[up] > -INFINITY;
        else if (a.draft) pass = x >= 0 && x < a.vocab && (double)a.uniform[q0 + i] * (double)a.draft[(long long)(q0 + i) * a.draft_stride + x] * sh.sum[up] < sh.weight[i];
        else {
            double left = sh.sum[up];
            if (a.parent) for (int s = up + 1; s < i; s++) if (sh.up[s] == up && !sh.again[s]) left -= sh.weight[s];
            pass = !sh.again[i] && (double)a.uniform[q0 + i] * left < sh.weight[i];
        }
        if (pass) atomicMin(&sh.first[up], i);
    }
    __syncthreads();
    // ---- the walk
    if (tid == 0) {
        int at = 0, kept = 1;
        if (cta == 0) a.path[(size_t)b * a.most] = 0;
        while (sh.first[at] < n) {
            at = sh.first[at];
            if (cta == 0) a.path[(size_t)b * a.most + kept] = at;
            kept++;
        }
        sh.last = at; sh.found = kept;
        if (cta == 0) { a.kept[b] = kept; a.dropped[b] = n - kept; }
    }
    __syncthreads();
    const int last = sh.last;
    if (cta == 0) for (int i = sh.found + tid; i < a.most; i += VF_THREADS) a.path[(size_t)b * a.most + i] = -1;
    if (!draws || sh.top[last] == -INFINITY) {             // the same in the whole cluster
        if (cta == 0 && tid == 0) a.next[b] = sh.top[last] == -INFINITY ? -1 : sh.best[last];
        return;
    }
    // ---- the token behind the last kept one.  Its refused children: their tokens are out, or (drawn) the one child's distribution is taken off
    __syncthreads();
    if (tid == 0) sh.refused = 0;
    __syncthreads();
    for (int i = last + 1 + tid; i < n; i += VF_THREADS) if (sh.up[i] == last) sh.first[atomicAdd(&sh.refused, 1)] = i;       // the links are not needed any more
    __syncthreads();
    const int refused = sh.refused;
    const bool taken = a.draft && refused > 0;
    const int slice = cta * VF_WARPS + warp, slices = ctas * VF_WARPS, e0 = (int)((long long)a.vocab * slice / slices), e1 = (int)((long long)a.vocab * (slice + 1) / slices);
    RowLeft<T> left = {logits + (long long)(q0 + last) * a.stride, taken ? a.draft + (long long)(q0 + sh.first[0]) * a.draft_stride : nullptr,
                       (double)sh.top[last], scale, 0.0, a.draft ? 0 : refused};
    if (lane == 0) {                                       // both rows on their way: the sums have too few loads under way to wait for HBM
        prefetch_l2(left.row + e0, (size_t)(e1 - e0) * sizeof(T));
        if (taken) prefetch_l2(left.q + e0, (size_t)(e1 - e0) * 4);
    }
    // Sums of all slices, the same in all CTAs: every lane has those of `mine` consecutive ones, `before` those ahead of them; returns the total.
    constexpr int MOST = VF_CLUSTER * VF_WARPS / 32;
    const int mine = (slices + 31) / 32;
    double held[MOST], before = 0.0;
    auto sum_all = [&]() {
        const double all = left_sum(left, sh, e0, e1, nullptr);
        cluster.sync();                                    // nobody reads the last sums any more
        if (lane < ctas) cluster.map_shared_rank(sh.slices, lane)[slice] = all;
        cluster.sync();
        double incl = 0.0;
#pragma unroll
        for (int k = 0; k < MOST; k++) {
            held[k] = k < mine && lane * mine + k < slices ? sh.slices[lane * mine + k] : 0.0;
            incl += held[k];
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
        before = __shfl_up_sync(0xffffffffu, incl, 1);
        if (lane == 0) before = 0.0;
        return __shfl_sync(0xffffffffu, incl, 31);
    };
    double total;
    for (int round = 0;; round++) {
        total = sum_all();
        if (round == 0 && taken && total > 0.0) left.norm = 1.0 / total;               // now what the refused draft leaves
        else if (round == 1 && !(total > 0.0)) left.norm = 0.0;                        // nothing: its distribution covers the target's
        else break;
    }
    // ---- the first element whose running sum exceeds u * total
    if (!(total > 0.0)) {
        if (cta == 0 && tid == 0) a.next[b] = -1;
    } else {
        const double goal = (double)a.uniform[q0] * total;
        int pick = -1, some = -1;                          // this lane's slice that holds it; its last with a weight
        double ahead = before, start = 0.0;
#pragma unroll
        for (int k = 0; k < MOST; k++) {
            if (held[k] > 0.0) {
                some = lane * mine + k;
                if (pick < 0 && ahead + held[k] > goal) { pick = some; start = ahead; }
            }
            ahead += held[k];
        }
        const unsigned hits = __ballot_sync(0xffffffffu, pick >= 0), any = __ballot_sync(0xffffffffu, some >= 0);
        if (hits) { const int src = __ffs(hits) - 1; pick = __shfl_sync(0xffffffffu, pick, src); start = __shfl_sync(0xffffffffu, start, src); }
        else { pick = __shfl_sync(0xffffffffu, some, 31 - __clz(any)); start = -INFINITY; }        // rounding leaves none: the last with a weight
        if (pick / VF_WARPS == cta) {                      // the same in the whole CTA: its warps share the slice out
            const int p0 = (int)((long long)a.vocab * pick / slices), p1 = (int)((long long)a.vocab * (pick + 1) / slices);
            const int f0 = p0 + (int)((long long)(p1 - p0) * warp / VF_WARPS), f1 = p0 + (int)((long long)(p1 - p0) * (warp + 1) / VF_WARPS);
            const double part = left_sum(left, sh, f0, f1, nullptr);
            if (lane == 0) sh.part[warp] = part;
            __syncthreads();
            double incl = lane < VF_WARPS ? sh.part[lane] : 0.0;
            const bool weighs = incl > 0.0;
#pragma unroll
            for (int o = 1; o < VF_WARPS; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
            const unsigned over = __ballot_sync(0xffffffffu, weighs && start + incl > goal), has = __ballot_sync(0xffffffffu, weighs);
            const int sub = over ? __ffs(over) - 1 : 31 - __clz(has);
            const double ahead_of = __shfl_sync(0xffffffffu, incl, max(sub - 1, 0));
            if (warp == sub) {
                double run = sub > 0 ? start + ahead_of : start;
                int found = -1, last_one = -1;
                for (int base = f0; base < f1 && found < 0; base += 32 * LEFT_STEPS) {
                    left_sum(left, sh, base, min(f1, base + 32 * LEFT_STEPS), sh.held);
                    __syncwarp();
#pragma unroll 1
                    for (int k = 0; k < LEFT_STEPS && found < 0; k++) {
                        const double v = sh.held[k * 32 + lane];
                        double x = v;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
                        const unsigned hit = __ballot_sync(0xffffffffu, v > 0.0 && run + x > goal), some_here = __ballot_sync(0xffffffffu, v > 0.0);
                        if (hit) found = base + k * 32 + __ffs(hit) - 1;
                        if (some_here) last_one = base + k * 32 + 31 - __clz(some_here);
                        run += __shfl_sync(0xffffffffu, x, 31);
                    }
                    __syncwarp();
                }
                if (lane == 0) a.next[b] = found >= 0 ? found : last_one;
            }
        }
    }
    cluster.sync();                                        // no CTA leaves while others write to its shared memory
}

// ---------------------------------------------------------------------------------- rows of accepted drafts
//
// Block (x = sequence, y = KV head): kept rows are copied in batches, first all rows of a batch are read, then they are written.  A path
// goes upward, path[i] >= i, so that no batch overwrites what a later one reads.
constexpr int KEEP_THREADS = 256;

struct KeepArgs {
    dynakv_row_cache c;
    const int* table; const int* len; const int* q_start; const int* path; const int* kept;
    unsigned* status;
    int per, width, n_seqs;
};

__global__ void __launch_bounds__(KEEP_THREADS) k_rows_keep(const KeepArgs a, int row_bytes) {
    const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    pdl_wait();
    const long long rows = (long long)a.per * PAGE, T = (long long)a.q_start[b + 1] - a.q_start[b];
    const int n = a.len[b], kept = a.kept[b];
    if (T < 0 || n < 0 || n > rows || T > n || kept < 0 || kept > T || kept > a.width) {
        if (tid == 0 && h == 0 && a.status) atomicOr(a.status, DYNAKV_ST_BOUNDS);
        return;
    }
    const int lanes = row_bytes / 16, batch = KEEP_THREADS / lanes, l = tid % lanes, mine = tid / lanes, base = n - (int)T;
    uint4* pools[2] = {reinterpret_cast<uint4*>(a.c.k), reinterpret_cast<uint4*>(a.c.v)};
    int8_t* exps[2] = {a.c.k_exp, a.c.v_exp};
    auto at = [&](int place) {                             // the row's index in the pool, -1: no such page
        const int page = a.table[(size_t)b * a.per + place / PAGE];
        return page >= 0 && page < a.c.n_pages ? ((long long)page * a.c.n_kv_heads + h) * PAGE + place % PAGE : -1ll;
    };
    bool trouble = false;
    for (int i0 = 1; i0 < kept; i0 += batch) {             // the root stays where it is
        const int i = i0 + mine;
        long long to = -1, from = -1;
        uint4 v[2];
        int8_t e[2] = {0, 0};
        if (i < kept) {
            const int p = a.path[(size_t)b * a.width + i];
            if (p < i || p >= T) trouble = true;
            else if (p != i) {
                to = at(base + i); from = at(base + p);
                if (to < 0 || from < 0) { trouble = true; to = -1; }
            }
        }
        if (to >= 0) {
#pragma unroll
            for (int x = 0; x < 2; x++) {
                v[x] = pools[x][from * lanes + l];
                if (exps[x] && l == 0) e[x] = exps[x][from];
            }
        }
        __syncthreads();
        if (to >= 0) {
#pragma unroll
            for (int x = 0; x < 2; x++) {
                pools[x][to * lanes + l] = v[x];
                if (exps[x] && l == 0) exps[x][to] = e[x];
            }
        }
        __syncthreads();
    }
    if (trouble && a.status) atomicOr(a.status, DYNAKV_ST_BOUNDS);
}

static int verify_pieces(int vocab, int es) { return (int)(((long long)vocab * es + RS_BYTES - 1) / RS_BYTES); }

template <typename T>
static int verify_launch(const VerifyArgs& a, int sms, cudaStream_t st) {
    if (a.n_tokens > 0 && launch_pdl(k_row_stats<T>, dim3(a.n_tokens, a.pieces), dim3(RS_THREADS), 0, st, a) != cudaSuccess) return DYNAKV_ERR_CUDA;
    // CTAs of a sequence: as many as keep all of them on the device at once, down to 4 K elements each
    int ctas = 1;
    while (ctas < VF_CLUSTER && 2ll * ctas * a.n_seqs <= sms && a.vocab > 4096 * ctas) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(ctas, a.n_seqs); cfg.blockDim = dim3(VF_THREADS); cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_verify<T>, a) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

}  // namespace dkv

using namespace dkv;

static bool verify_shape_ok(int32_t dtype, int64_t n_tokens, int32_t vocab, int32_t n_seqs, int32_t max_tree) {
    return (dtype == DYNAKV_F32 || dtype == DYNAKV_BF16) && n_tokens >= 0 && n_tokens < (1ll << 24) && vocab >= 1 && vocab <= (1 << 26) && n_seqs >= 0 &&
           n_seqs <= 65535 && max_tree >= 1 && max_tree <= TREE_MAX;
}

extern "C" int64_t dynakv_verify_drafts_workspace(int32_t logits_dtype, int64_t n_tokens, int32_t vocab, int32_t n_seqs, int32_t max_tree) {
    if (!verify_shape_ok(logits_dtype, n_tokens, vocab, n_seqs, max_tree)) return DYNAKV_ERR_ARG;
    return (int64_t)max(1ll, (long long)n_tokens) * verify_pieces(vocab, logits_dtype == DYNAKV_F32 ? 4 : 2) * 16;
}

extern "C" int dynakv_verify_drafts(const void* logits, int64_t logits_stride, int32_t logits_dtype, int64_t n_tokens, int32_t vocab, const int32_t* tokens,
                                    const int32_t* q_start, int32_t n_seqs, int32_t max_tree, const float* uniform, const float* temperature,
                                    const int32_t* parent, const float* draft_probs, int64_t draft_stride, int32_t* kept, int32_t* dropped,
                                    int32_t* path, int32_t* next_token, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (!verify_shape_ok(logits_dtype, n_tokens, vocab, n_seqs, max_tree) || (draft_probs && parent)) return DYNAKV_ERR_ARG;
    if (n_seqs == 0) return DYNAKV_OK;
    if (!q_start || !temperature || !kept || !dropped || !path || !next_token || !workspace || ((uintptr_t)workspace & 15)) return DYNAKV_ERR_ARG;
    const int es = logits_dtype == DYNAKV_F32 ? 4 : 2;
    if (n_tokens > 0 && (!logits || !tokens || !uniform || ((uintptr_t)logits & (es - 1)) || ((uintptr_t)draft_probs & 3) || logits_stride < 0 || draft_stride < 0)) return DYNAKV_ERR_ARG;
    int rc;
    const int sms = sm_count(&rc);
    if (rc != DYNAKV_OK) return rc;
    VerifyArgs a;
    a.logits = logits; a.stride = logits_stride; a.tokens = tokens; a.q_start = q_start; a.parent = parent; a.uniform = uniform; a.heat = temperature;
    a.draft = draft_probs; a.draft_stride = draft_stride; a.kept = kept; a.dropped = dropped; a.path = path; a.next = next_token;
    a.stats = reinterpret_cast<float4*>(workspace);
    a.n_tokens = (int)n_tokens; a.n_seqs = n_seqs; a.vocab = vocab; a.most = max_tree;
    a.pieces = verify_pieces(vocab, es);
    if (workspace_bytes < max(1ll, (long long)n_tokens) * a.pieces * 16) return DYNAKV_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    // an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
    cudaGetLastError();
    return logits_dtype == DYNAKV_F32 ? verify_launch<float>(a, sms, st) : verify_launch<__nv_bfloat16>(a, sms, st);
}

extern "C" int dynakv_rows_keep(const dynakv_row_cache* cache, const int32_t* page_table, int32_t pages_per_seq, const int32_t* kv_len,
                                const int32_t* q_start, int32_t n_seqs, const int32_t* path, int32_t path_width, const int32_t* kept,
                                uint32_t* status, void* cuda_stream) {
    if (!row_cache_ok(cache) || pages_per_seq < 0 || pages_per_seq >= (1 << 26) || n_seqs < 0 || path_width < 0 || cache->n_kv_heads > 65535) return DYNAKV_ERR_ARG;
    if (n_seqs == 0 || path_width == 0) return DYNAKV_OK;
    if ((!page_table && pages_per_seq > 0) || !kv_len || !q_start || !path || !kept) return DYNAKV_ERR_ARG;
    KeepArgs a;
    a.c = *cache; a.table = page_table; a.len = kv_len; a.q_start = q_start; a.path = path; a.kept = kept; a.status = status;
    a.per = pages_per_seq; a.width = path_width; a.n_seqs = n_seqs;
    const int row_bytes = cache->head_dim * (cache->kv_dtype == DYNAKV_F32 ? 4 : cache->kv_dtype == DYNAKV_BF16 ? 2 : 1);
    if (cache->kv_dtype != DYNAKV_FP8) a.c.k_exp = a.c.v_exp = nullptr;
    // an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
    cudaGetLastError();
    return launch_pdl(k_rows_keep, dim3(n_seqs, cache->n_kv_heads), dim3(KEEP_THREADS), 0, reinterpret_cast<cudaStream_t>(cuda_stream), a, row_bytes) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}
