// What follows the attention of drafted tokens: which of them are accepted (dynakv_verify_drafts), and their rows moved
// together (dynakv_rows_keep).
//
// Verification.  With p the target's distribution behind a kept token (softmax of its logits over the temperature, or all of it on the first
// largest logit), a drafted child x is accepted when u q(x) < p(x); refused, it leaves max(p - q, 0) to its younger siblings and to
// the token that is drawn at the end, all up to a factor that is carried along.  A draft that was not drawn has q = 1 at x, so that what is
// left is p without x.
//   k_row_stats: the one pass over the logits, HBM bound: (largest, first place of it, sum of exp) of every row, in pieces.
//   k_verify, a cluster of CTAs per sequence: every draft's test from those and one logit, at once for all drafts (and from sums in 64 bits where
//     they leave it open); the walk in shared memory; then the drawing from the last kept token's row, which is by inverse sums in 64 bits: among 10^5 tokens fp32 sums
//     misplace the draw with a chance of about 10^-3, and the same numbers have to give the same token however the sums are split.
// Measured, calls one after the other: 64 sequences of 6 tokens over 128256, drafts drawn, 52 us: 22 for the rows, 6 until the walk is done, 16
// for the sums (36 instructions an element, 11 of them in 64 bits; 128 CTAs; in two passes, the target's sum first, 31), 6 for the place of
// the draw.  16 trees of 32 over 50257: 26 us.  One sequence of 5 over 32000: 12 us on the device, a chain of dependent loads; 19 us of host time.
// 512 sequences of one token over 128256: 169 us, of which 36 without the draw (one CTA of 512 threads per SM 176).
#include <cooperative_groups.h>
#include <float.h>

#include <utility>

#include "bulk_copy.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tc_rows.cuh"
#include "tree_host.cuh"

namespace dkv {

namespace cg = cooperative_groups;

constexpr int RS_THREADS = 128, RS_VECS = 4, RS_BYTES = RS_THREADS * RS_VECS * 16;     // a block's piece of a row
constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32, VF_CLUSTER = 8;            // at most

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
    pdl_trigger();
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
    if (tid == 0) at_s = 0x7fffffff;
    if (warp == 0) {
        // the last sequence that begins at or before the row: 32 of them are looked at a time
        int lo = 0;
        for (int n = a.n_seqs; n > 1;) {
            const int step = (n + 31) / 32, at = lane * step;
            const unsigned before = __ballot_sync(0xffffffffu, at < n && a.q_start[lo + min(at, n - 1)] <= row);
            const int skip = max(0, __popc(before) - 1) * step;
            lo += skip; n = min(step, n - skip);
        }
        auto has = [&](int b) { return a.q_start[b] <= row && row < a.q_start[b + 1]; };
        int mine = has(lo) ? lo : -1;
        if (mine < 0)                                      // a row of no sequence, or ranges out of order, of which some may be sound
            for (int b = lane; b < a.n_seqs; b += 32) if (has(b)) mine = b;
        mine = __reduce_max_sync(0xffffffffu, mine);
        if (lane == 0) heat_s = mine >= 0 ? heat_of(a, mine) : -1.f;
    }
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

constexpr int EXP_TABLE = 256;
__device__ const double two_to[32] = {             // 2^(j / 16), 2^(j / 256)
    1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484, 1.2968395546510096,
    1.3542555469368927, 1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543, 1.681792830507429, 1.7562521603732995,
    1.8340080864093424, 1.9152065613971474, 1.0, 1.0027112750502025, 1.0054299011128027, 1.0081558981184175, 1.0108892860517005,
    1.0136300849514894, 1.016378314910953, 1.019133996077738, 1.0218971486541166, 1.0246677928971357, 1.0274459491187637, 1.030231637686041,
    1.0330248790212284, 1.0358256936019572, 1.0386341019613787, 1.041450124688316};
// N values of 2^((l - top) * scale) in 64 bits, l <= top: the exponent is n + j / 256 + r with |r| <= 1 / 512, the factor of j comes from a table
// (in shared memory once per pair of lanes, so that no two meet in a bank) and that of r from its series up to r^3 (what is left out is
// below 2^-42 of the value, far below what could misplace a draw).  Values below 2^-1000 are 0.  Step by step for all N, because a 64-bit operation's result is a long time in coming: one value after the other,
// the 8 M of a large call took 140 us.
template <int N>
__device__ __forceinline__ void exp2_64(const float (&l)[N], double top, double scale, float lowest, const double* table, double (&w)[N]) {
    const double shift = 6755399441055744.0 / EXP_TABLE;   // 1.5 * 2^52 in units of 1 / 256: the sum's last bits are round(256 x)
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
    for (int i = 0; i < N; i++) p[i] = fma(r[i], 0.055504108664821576, 0.24022650695910069);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], r[i], 0.69314718055994529);
#pragma unroll
    for (int i = 0; i < N; i++) p[i] *= r[i];
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = fma(p[i], w[i], w[i]);
#pragma unroll
    for (int i = 0; i < N; i++) w[i] = l[i] >= lowest ? __hiloint2double(__double2hiint(p[i]) + ((k[i] >> 8) << 20), __double2loint(p[i])) : 0.0;
}
// The logit below which a weight is 0: rounded up, to the largest one at most, so that no weight is below 2^-1000, the largest never left out, and -infinity always.
__device__ __forceinline__ float lowest_logit(double top, double scale_inv) { return __double2float_ru(top - 1000.0 * scale_inv); }

// What a row's sum of fp32 exponentials may be off by, relative to it: logits minus the largest times 1 / temperature carry three roundings and the factor's own,
// 4 2^-24 of an exponent of at most 26 where the weight of up to 2^26 tokens lies (times ln 2: 72 2^-24), ex2 2^-22 and some 50 additions 2^-24 each.
constexpr double SUM_OFF = 0x1p-16;

constexpr int LEFT_EACH = 8, LEFT_RUN = 32 * LEFT_EACH;     // elements of a lane and of a warp at a time

struct VerifyShared {
    double weight[TREE_MAX], sum[TREE_MAX];        // of a draft: its token's weight behind its parent; [a row]: sum of the row's weights
    float top[TREE_MAX];                           // [a row] largest logit
    int best[TREE_MAX];                            //         first place of it
    int token[TREE_MAX], up[TREE_MAX], first[TREE_MAX];
    unsigned char again[TREE_MAX];                 // an older sibling has the same token
    unsigned char out[TREE_MAX];                   // drafts whose tokens are refused
    unsigned unsure[TREE_MAX / 32];                // bit per draft: its test needs the sum in 64 bits
    double table[EXP_TABLE * 16];
    double slices[3][VF_CLUSTER * VF_WARPS], part[VF_WARPS];
    double held[LEFT_RUN];                  // weights of the run in which the drawn token lies
    int last, refused, found;
};

// What is left of a row's distribution: its weights without the tokens of `refused` children, or (a refused draft that was drawn from q)
// max(weight / S - q, 0), S the sum of the weights.  Which elements of the latter are not 0 is decided with S as fp32 sums give it (near = 1 / S): the
// others' sums P and Q can then be taken in the pass that finds S in 64 bits, and P / S - Q is off by what such elements as lie within 1e-6 of 0 add,
// where each adds next to nothing.  Where what is left is itself little (LEFT_LITTLE: a draft drawn from nearly the target's distribution, which is refused as seldom) that is
// not nothing, and the elements are gone over once more with S in 64 bits.
constexpr double LEFT_LITTLE = 0x1p-10;
enum { LEFT_ALL = 0, LEFT_LESS = 1, LEFT_SUMS = 2 };       // weights; max(weight norm - q, 0); all three sums
template <typename T>
struct RowLeft {
    const T* row;
    const float* q;
    double top, scale, scale_inv, near, norm;
    int refused, what;
};
struct LeftSums { double all, p, q; };
// The largest element <= x at which the row has a 16-byte boundary (it may lie before the row).
template <typename T>
__device__ __forceinline__ int left_aligned(const T* row, int x) { return x - (int)(((uintptr_t)(row + x) & 15) / sizeof(T)); }
// The sum over elements [from, end), by one warp, each lane LEFT_EACH elements side by side, from 16-byte boundaries on; `held`: the weights of one
// run are kept there, in their order from the boundary on.  One function, not inlined: the code is run once or twice, and fetching it is what it would cost.
template <typename T>
__device__ __noinline__ LeftSums left_sum(const RowLeft<T> a, const VerifyShared& sh, int vocab, int from, int end, double* held) {
    constexpr int WORDS = LEFT_EACH * sizeof(T) / 16;
    const int lane = threadIdx.x & 31;
    const bool less = a.what != LEFT_ALL, less16 = less && (((uintptr_t)(a.q + left_aligned(a.row, from)) & 15) == 0);
    const float lowest = lowest_logit(a.top, a.scale_inv);
    double s[2] = {0.0, 0.0}, p[2] = {0.0, 0.0}, m[2] = {0.0, 0.0};
    uint4 l[WORDS];
    float q[LEFT_EACH] = {};
    // The next elements, while these are worked on.  Whole vectors but at the row's ends.
    auto fetch = [&](int at) {
        if (at >= 0 && at + LEFT_EACH <= vocab) {
#pragma unroll
            for (int k = 0; k < WORDS; k++) l[k] = __ldg(reinterpret_cast<const uint4*>(a.row + at) + k);
            if (less16) {
#pragma unroll
                for (int k = 0; k < LEFT_EACH; k += 4) {
                    const float4 v = __ldg(reinterpret_cast<const float4*>(a.q + at + k));
                    q[k] = v.x; q[k + 1] = v.y; q[k + 2] = v.z; q[k + 3] = v.w;
                }
            } else if (less) {
#pragma unroll
                for (int k = 0; k < LEFT_EACH; k++) q[k] = __ldg(a.q + at + k);
            }
            return;
        }
        unsigned u[4 * WORDS];
#pragma unroll
        for (int k = 0; k < 4 * WORDS; k++) u[k] = 0u;
#pragma unroll
        for (int k = 0; k < LEFT_EACH; k++) {
            if ((unsigned)(at + k) >= (unsigned)vocab) continue;
            if constexpr (sizeof(T) == 4) u[k] = __float_as_uint(a.row[at + k]);
            else u[k >> 1] |= (unsigned)__bfloat16_as_ushort(a.row[at + k]) << (16 * (k & 1));
            if (less) q[k] = a.q[at + k];
        }
#pragma unroll
        for (int k = 0; k < WORDS; k++) l[k] = make_uint4(u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]);
    };
    int at = left_aligned(a.row, from) + lane * LEFT_EACH;         // this lane's elements
    if (from < end) fetch(at);
    for (; at - lane * LEFT_EACH < end; at += LEFT_RUN) {
        double w[LEFT_EACH];
        float now[LEFT_EACH], minus[LEFT_EACH];
#pragma unroll
        for (int k = 0; k < LEFT_EACH; k++) {
            const uint4 v = l[k * sizeof(T) / 16];
            const unsigned u[4] = {v.x, v.y, v.z, v.w};
            if constexpr (sizeof(T) == 4) now[k] = __uint_as_float(u[k & 3]);
            else now[k] = __uint_as_float(k & 1 ? u[k >> 1] & 0xffff0000u : u[k >> 1] << 16);
            minus[k] = q[k];
        }
        if (__any_sync(0xffffffffu, at < from || at + LEFT_EACH > end)) {
#pragma unroll
            for (int k = 0; k < LEFT_EACH; k++) if (at + k < from || at + k >= end) { now[k] = -INFINITY; minus[k] = 0.f; }
        }
        for (int r = 0; r < a.refused; r++) {              // a refused token weighs nothing
            const int off = sh.token[sh.out[r]] - at;
            if (!__any_sync(0xffffffffu, (unsigned)off < (unsigned)LEFT_EACH)) continue;
#pragma unroll
            for (int k = 0; k < LEFT_EACH; k++) if (off == k) now[k] = -INFINITY;
        }
        if (at - lane * LEFT_EACH + LEFT_RUN < end) fetch(at + LEFT_RUN);
        exp2_64(now, a.top, a.scale, lowest, sh.table + (lane & 15), w);
        if (a.what == LEFT_SUMS) {
#pragma unroll
            for (int k = 0; k < LEFT_EACH; k++) {
                const double x = (double)minus[k];
                const bool more = w[k] * a.near > x;
                p[k & 1] += more ? w[k] : 0.0;
                m[k & 1] += more ? x : 0.0;
            }
        } else if (less) {
#pragma unroll
            for (int k = 0; k < LEFT_EACH; k++) {
                const double x = (double)minus[k];
                w[k] = w[k] * a.near > x ? fmax(fma(w[k], a.norm, -x), 1e-300) : 0.0;
            }
        }
        if (held) {
#pragma unroll
            for (int k = 0; k < LEFT_EACH; k++) held[lane * LEFT_EACH + k] = w[k];
        }
#pragma unroll
        for (int k = 0; k < LEFT_EACH; k += 2) { s[0] += w[k]; s[1] += w[k + 1]; }
    }
    LeftSums sums = {warp_sum64(s[0] + s[1]), 0.0, 0.0};
    if (a.what == LEFT_SUMS) { sums.p = warp_sum64(p[0] + p[1]); sums.q = warp_sum64(m[0] + m[1]); }
    return sums;
}

// One slice of the vocabulary per warp.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_verify(const VerifyArgs a) {
    constexpr int WARPS = THREADS / 32, EACH = (TREE_MAX + THREADS - 1) / THREADS;
    __shared__ VerifyShared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = gridDim.x, cta = blockIdx.x, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < EXP_TABLE * 16; i += THREADS) sh.table[i] = two_to[i >> 8] * two_to[16 + ((i >> 4) & 15)];
    pdl_wait();
    int q0, n;
    const bool ok = verify_range(a, b, q0, n);
    const T* logits = reinterpret_cast<const T*>(a.logits);
    if (n == 0) {                                          // the same in the whole cluster
        if (cta == 0) {
            for (int i = tid; i < a.most; i += THREADS) a.path[(size_t)b * a.most + i] = -1;
            if (tid == 0) { a.kept[b] = 0; a.dropped[b] = ok ? 0 : -1; a.next[b] = -1; }
        }
        return;
    }
    cg::cluster_group::arrival_token begun = cluster.barrier_arrive();
    const float heat = heat_of(a, b);
    const bool draws = heat > 0.f;
    const double scale = 1.4426950408889634074 / (double)heat, scale_inv = 0.69314718055994530942 * (double)heat;         // weights are 2^((logit - largest) * scale)
    // what the tests will need is on its way before anything is waited for
    int token[EACH], up[EACH];
    float chance[EACH];
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int i = tid + e * THREADS;
        token[e] = i < n ? a.tokens[q0 + i] : -1;
        up[e] = i < n && i > 0 ? a.parent ? a.parent[q0 + i] : i - 1 : -1;
        chance[e] = i < n ? a.uniform[q0 + i] : 0.f;
    }
    __syncthreads();
    auto weight_of = [&](float l, float top) {
        const float x[1] = {l};
        double w[1];
        exp2_64(x, (double)top, scale, lowest_logit((double)top, scale_inv), sh.table + (lane & 15), w);
        return w[0];
    };
    // ---- every row's largest logit and sum, a warp per row
    for (int i = warp; i < n; i += WARPS) {
        const float4* st = a.stats + (size_t)(q0 + i) * a.pieces;
        const float4 mine = lane < a.pieces ? st[lane] : make_float4(-INFINITY, __int_as_float(0x7fffffff), 0.f, 0.f);
        Best best = {mine.x, __float_as_int(mine.y)};
        for (int k = lane + 32; k < a.pieces; k += 32) best = better(best, Best{st[k].x, __float_as_int(st[k].y)});
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = better(best, Best{__shfl_xor_sync(0xffffffffu, best.top, o), __shfl_xor_sync(0xffffffffu, best.at, o)});
        double sum = draws && mine.x > -INFINITY ? (double)mine.z * weight_of(mine.x, best.top) : 0.0;
        for (int k = lane + 32; k < a.pieces; k += 32)
            if (draws && st[k].x > -INFINITY) sum += (double)st[k].z * weight_of(st[k].x, best.top);
        sum = warp_sum64(sum);
        if (lane == 0) { sh.top[i] = best.top; sh.best[i] = best.at; sh.sum[i] = sum; }
    }
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int i = tid + e * THREADS;
        if (up[e] < 0 || up[e] >= i) up[e] = -1;           // a draft without a parent before it is never reached
        if (i < n) { sh.token[i] = token[e]; sh.up[i] = up[e]; sh.first[i] = n; }
    }
    if (tid < TREE_MAX / 32) sh.unsure[tid] = 0u;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int i = tid + e * THREADS, x = token[e];
        if (i >= n) continue;
        // of token x behind row up, relative to the row's largest
        sh.weight[i] = draws && up[e] >= 0 && x >= 0 && x < a.vocab && sh.top[up[e]] > -INFINITY ? weight_of(to_f(logits[(long long)(q0 + up[e]) * a.stride + x]), sh.top[up[e]]) : 0.0;
        bool again = false;
        if (a.parent && up[e] >= 0) for (int s = up[e] + 1; s < i; s++) again |= sh.up[s] == up[e] && sh.token[s] == x;
        sh.again[i] = again;
    }
    __syncthreads();
    // ---- every draft's test, against what its older siblings leave
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int i = tid + e * THREADS, x = token[e], above = up[e];
        if (above < 0) continue;
        bool pass = false;
        if (!draws) pass = sh.best[above] == x && sh.top[above] > -INFINITY;
        else if (sh.weight[i] > 0.0 && !sh.again[i]) {
            double left = sh.sum[above], part = (double)chance[e];
            const double off = left * SUM_OFF;
            if (a.draft) part *= (double)a.draft[(long long)(q0 + i) * a.draft_stride + x];
            else if (a.parent) for (int s = above + 1; s < i; s++) if (sh.up[s] == above && !sh.again[s]) left -= sh.weight[s];
            pass = part * (left + off) < sh.weight[i];
            if (!pass && part * (left - off) < sh.weight[i]) atomicOr(&sh.unsure[i >> 5], 1u << (i & 31));
        }
        if (pass) atomicMin(&sh.first[above], i);
    }
    if (tid == 0) sh.refused = 0;
    __syncthreads();
    // ---- tests that lie within the error of the sums (next to never; or where older siblings have nearly all of the weight): the row once more in 64 bits, without
    // the older siblings' tokens, by every CTA for itself
    for (int k = 0; k < n; k += 32) for (unsigned open = sh.unsure[k >> 5]; open; open &= open - 1) {          // the same in the whole cluster
        const int i = k + __ffs(open) - 1, above = sh.up[i];
        if (tid == 0) {
            int count = 0;
            if (!a.draft) for (int s = above + 1; s < i; s++) if (sh.up[s] == above && !sh.again[s]) sh.out[count++] = (unsigned char)s;
            sh.found = count;
        }
        __syncthreads();
        const RowLeft<T> row = {logits + (long long)(q0 + above) * a.stride, nullptr, (double)sh.top[above], scale, scale_inv, 0.0, 0.0, sh.found, LEFT_ALL};
        const double mine = left_sum(row, sh, a.vocab, (int)((long long)a.vocab * warp / WARPS), (int)((long long)a.vocab * (warp + 1) / WARPS), nullptr).all;
        if (lane == 0) sh.part[warp] = mine;
        __syncthreads();
        if (tid == 0) {
            double left = 0.0, part = (double)a.uniform[q0 + i];
            for (int k = 0; k < WARPS; k++) left += sh.part[k];
            if (a.draft) part *= (double)a.draft[(long long)(q0 + i) * a.draft_stride + sh.token[i]];
            if (part * left < sh.weight[i]) sh.first[above] = min(sh.first[above], i);
        }
        __syncthreads();
    }
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
    if (cta == 0) for (int i = sh.found + tid; i < a.most; i += THREADS) a.path[(size_t)b * a.most + i] = -1;
    if (!draws || sh.top[last] == -INFINITY) {             // the same in the whole cluster
        if (cta == 0 && tid == 0) a.next[b] = sh.top[last] == -INFINITY ? -1 : sh.best[last];
        cluster.barrier_wait(std::move(begun));
        return;
    }
    // ---- the token behind the last kept one.  Its refused children: their tokens are out, or (drawn) the one child's distribution is taken off
#pragma unroll
    for (int e = 0; e < EACH; e++) if (up[e] == last) sh.out[atomicAdd(&sh.refused, 1)] = (unsigned char)(tid + e * THREADS);
    __syncthreads();
    const int refused = sh.refused;
    const bool taken = a.draft && refused > 0;
    const int slice = cta * WARPS + warp, slices = ctas * WARPS, shift = __ffs(slices) - 1;         // a power of two
    auto begin = [&](int x) { return (int)((long long)a.vocab * x >> shift); };
    const int e0 = begin(slice), e1 = begin(slice + 1);
    RowLeft<T> left = {logits + (long long)(q0 + last) * a.stride, taken ? a.draft + (long long)(q0 + sh.out[0]) * a.draft_stride : nullptr,
                       (double)sh.top[last], scale, scale_inv, taken ? 1.0 / sh.sum[last] : 0.0, 0.0, a.draft ? 0 : refused, taken ? LEFT_SUMS : LEFT_ALL};
    if (lane == 0) {                                       // both rows on their way: the sums have too few loads under way to wait for HBM
        prefetch_l2(left.row + e0, (size_t)(e1 - e0) * sizeof(T));
        if (taken) prefetch_l2(left.q + e0, (size_t)(e1 - e0) * 4);
    }
    {
        const LeftSums mine = left_sum(left, sh, a.vocab, e0, e1, nullptr);
        cluster.barrier_wait(std::move(begun));            // all CTAs have begun
        if (lane < ctas) {
            VerifyShared* to = cluster.map_shared_rank(&sh, lane);
            to->slices[0][slice] = mine.all;
            if (taken) { to->slices[1][slice] = mine.p; to->slices[2][slice] = mine.q; }
        }
        cluster.sync();
    }
    // Sums of all slices, the same in all CTAs: every lane has those of `mine` consecutive ones, `before` those ahead of them
    constexpr int MOST = VF_CLUSTER * VF_WARPS / 32;
    const int mine = (slices + 31) / 32;
    double held[MOST], before = 0.0;
    // kind LEFT_ALL: the weights, LEFT_LESS: P / S - Q, LEFT_SUMS: what the slices hold in place of P
    auto sum_all = [&](int kind) {
        double incl = 0.0;
#pragma unroll
        for (int k = 0; k < MOST; k++) {
            const int at = lane * mine + k;
            held[k] = k >= mine || at >= slices ? 0.0 : kind == LEFT_LESS ? fmax(fma(sh.slices[1][at], left.norm, -sh.slices[2][at]), 0.0) : sh.slices[kind == LEFT_ALL ? 0 : 1][at];
            incl += held[k];
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
        before = __shfl_up_sync(0xffffffffu, incl, 1);
        if (lane == 0) before = 0.0;
        return __shfl_sync(0xffffffffu, incl, 31);
    };
    left.what = LEFT_ALL;
    double total = sum_all(LEFT_ALL);
    if (taken && total > 0.0) {
        left.norm = 1.0 / total; left.what = LEFT_LESS;
        double less = sum_all(LEFT_LESS);
        if (less < LEFT_LITTLE) {                          // the same in the whole cluster
            left.near = left.norm;
            const double exact = left_sum(left, sh, a.vocab, e0, e1, nullptr).all;
            cluster.sync();                                // the sums have been read
            if (lane < ctas) cluster.map_shared_rank(&sh, lane)->slices[1][slice] = exact;
            cluster.sync();
            less = sum_all(LEFT_SUMS);
        }
        if (less > 0.0) total = less;
        else { left.what = LEFT_ALL; sum_all(LEFT_ALL); }  // nothing: its distribution covers the target's
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
        if (pick / WARPS == cta) {                      // the same in the whole CTA: its warps share the slice out
            const int p0 = begin(pick), p1 = begin(pick + 1);
            const bool share = p1 - p0 > 2 * LEFT_RUN;         // or the first warp has it alone
            const int f0 = share ? p0 + (int)((long long)(p1 - p0) * warp / WARPS) : p0, f1 = share ? p0 + (int)((long long)(p1 - p0) * (warp + 1) / WARPS) : p1;
            if (share) {
                const double part = left_sum(left, sh, a.vocab, f0, f1, nullptr).all;
                if (lane == 0) sh.part[warp] = part;
                __syncthreads();
            }
            double incl = share && lane < WARPS ? sh.part[lane] : 0.0;
            const bool weighs = incl > 0.0;
#pragma unroll
            for (int o = 1; o < WARPS; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
            const unsigned over = __ballot_sync(0xffffffffu, weighs && start + incl > goal), has = __ballot_sync(0xffffffffu, weighs);
            const int sub = !share ? 0 : over ? __ffs(over) - 1 : 31 - __clz(has);
            const double ahead_of = __shfl_sync(0xffffffffu, incl, max(sub - 1, 0));
            if (warp == sub) {
                double run = sub > 0 ? start + ahead_of : start;
                int found = -1, last_one = -1;
                for (int base = left_aligned(left.row, f0); base < f1 && found < 0; base += LEFT_RUN) {
                    left_sum(left, sh, a.vocab, max(base, f0), min(f1, base + LEFT_RUN), sh.held);
                    __syncwarp();
                    // a lane's elements one after the other, behind those of the lanes before it
                    double v[LEFT_EACH], x = 0.0;
#pragma unroll
                    for (int k = 0; k < LEFT_EACH; k++) { v[k] = sh.held[lane * LEFT_EACH + k]; x += v[k]; }
                    double upto = x;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += y; }
                    double ahead_here = __shfl_up_sync(0xffffffffu, upto, 1);
                    if (lane == 0) ahead_here = 0.0;
                    int hit = -1, some_here = -1;
                    double sum = run + ahead_here;
#pragma unroll
                    for (int k = 0; k < LEFT_EACH; k++) {
                        sum += v[k];
                        if (v[k] > 0.0) { some_here = k; if (hit < 0 && sum > goal) hit = k; }
                    }
                    const unsigned hits_here = __ballot_sync(0xffffffffu, hit >= 0), any_here = __ballot_sync(0xffffffffu, some_here >= 0);
                    if (hits_here) { const int src = __ffs(hits_here) - 1; found = base + src * LEFT_EACH + __shfl_sync(0xffffffffu, hit, src); }
                    if (any_here) { const int src = 31 - __clz(any_here); last_one = base + src * LEFT_EACH + __shfl_sync(0xffffffffu, some_here, src); }
                    run += __shfl_sync(0xffffffffu, upto, 31);
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
    // more sequences than SMs: two smaller CTAs per SM, of which one sums while the other waits
    const bool few = a.n_seqs <= sms;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(ctas, a.n_seqs); cfg.blockDim = dim3(few ? VF_THREADS : VF_THREADS / 2); cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    const cudaError_t e = few ? cudaLaunchKernelEx(&cfg, k_verify<T, VF_THREADS>, a) : cudaLaunchKernelEx(&cfg, k_verify<T, VF_THREADS / 2>, a);
    return e == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
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
