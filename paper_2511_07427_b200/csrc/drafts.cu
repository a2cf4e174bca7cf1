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
#include <cooperative_groups.h>
#include <float.h>

#include "bulk_copy.cuh"
#include "head_rows.cuh"
#include "mma_ops.cuh"
#include "tree_host.cuh"

namespace dkv {

namespace cg = cooperative_groups;

constexpr int RS_THREADS = 256, RS_VECS = 8, RS_BYTES = RS_THREADS * RS_VECS * 16;     // a block's piece of a row
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

struct Best { float top; int at; };
__device__ __forceinline__ Best better(Best a, Best b) { return b.top > a.top || (b.top == a.top && b.at < a.at) ? b : a; }

// A piece is loaded whole, every thread's 128 bytes on their way before anything is looked at: then the largest, then the sum
// relative to it.  (A running maximum with two loads under way took 31 us for 98 MB, this takes RS_TIME.)
template <typename T>
__global__ void __launch_bounds__(RS_THREADS) k_row_stats(const VerifyArgs a) {
    constexpr int N = 16 / sizeof(T);      // elements of a load
    const int row = blockIdx.x, piece = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ float heat_s;
    __shared__ Best best_s[RS_THREADS / 32];
    __shared__ float sum_s[RS_THREADS / 32];
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
    if (tid == 0) heat_s = -1.f;
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += RS_THREADS)       // at most one sequence has the row
        if (a.q_start[b] <= row && row < a.q_start[b + 1]) heat_s = fmaxf(a.heat[b], 0.f);
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
    Best best = {m, 0x7fffffff};
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (m == top) {                        // few threads look for the place of the warp's largest
        if (x_odd == m) best.at = at_odd;
#pragma unroll
        for (int i = RS_VECS - 1; i >= 0; i--)
#pragma unroll
            for (int e = N - 1; e >= 0; e--) if (elem(i, e) == m && v0 + i * RS_THREADS < vecs) best.at = min(best.at, head + (v0 + i * RS_THREADS) * N + e);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = better(best, Best{__shfl_xor_sync(0xffffffffu, best.top, o), __shfl_xor_sync(0xffffffffu, best.at, o)});
    if (lane == 0) best_s[warp] = best;
    __syncthreads();
    pdl_trigger();
    const float heat = heat_s;
    if (heat < 0.f) return;                                // a row of no sequence
    best = best_s[0];
#pragma unroll
    for (int k = 1; k < RS_THREADS / 32; k++) best = better(best, best_s[k]);
    float sum = 0.f;
    if (heat > 0.f && best.top > -INFINITY) {
        const float f = 1.4426950408889634f / heat, shift = best.top;
        float part[2] = {0.f, 0.f};
        if (x_odd > -INFINITY) part[0] = ex2((x_odd - shift) * f);
#pragma unroll
        for (int i = 0; i < RS_VECS; i++)
#pragma unroll
            for (int e = 0; e < N; e++) part[e & 1] += ex2((elem(i, e) - shift) * f);      // not x f - m f, which is off by the rounding of m f
        sum = warp_sum(part[0] + part[1]);
    }
    if (lane == 0) sum_s[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        float total = 0.f;
#pragma unroll
        for (int k = 0; k < RS_THREADS / 32; k++) total += sum_s[k];
        a.stats[(size_t)row * a.pieces + piece] = make_float4(best.top, __int_as_float(best.at), total, 0.f);
    }
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// 2^x in 64 bits for x <= 0: 2^x = 2^n * 2^(j / 32) * 2^r with |r| <= 1 / 64, the middle factor from a table and the last from its
// series up to r^6 (what is left out is below 2^-57).  Results below 2^-1000 are 0.
__device__ __forceinline__ double exp2_64(double x, const double* table) {
    if (!(x > -1000.0)) return 0.0;
    const double shift = 6755399441055744.0 / 32.0;        // 1.5 * 2^52 in units of 1 / 32: the sum's last bits are round(32 x)
    const double t = x + shift, r = x - (t - shift);
    const int k = __double2loint(t);
    const double y = r * 0.69314718055994530942;
    double p = fma(y, 1.0 / 720.0, 1.0 / 120.0);
    p = fma(p, y, 1.0 / 24.0);
    p = fma(p, y, 1.0 / 6.0);
    p = fma(p, y, 0.5);
    p = fma(p, y, 1.0);
    const double z = table[k & 31];
    p = fma(p * y, z, z);
    return __hiloint2double(__double2hiint(p) + ((k >> 5) << 20), __double2loint(p));
}

struct VerifyShared {
    double weight[TREE_MAX], sum[TREE_MAX];        // of a draft: its token's weight behind its parent; [a row]: sum of the row's weights
    float top[TREE_MAX];                           // [a row] largest logit
    int best[TREE_MAX];                            //         first place of it
    int token[TREE_MAX], up[TREE_MAX], first[TREE_MAX];
    unsigned char again[TREE_MAX];                 // an older sibling has the same token
    double table[32];                              // 2^(j / 32)
    double slices[VF_CLUSTER * VF_WARPS];
    int last, refused, found;
};

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
    const float heat = a.heat[b];
    const bool draws = heat > 0.f;
    const double scale = 1.4426950408889634074 / (double)heat;             // weights are 2^((logit - largest) * scale)
    if (tid < 32) sh.table[tid] = exp2((double)tid / 32.0);
    // ---- every row's largest logit and sum, a warp per row
    for (int i = warp; i < n; i += VF_WARPS) {
        const float4* st = a.stats + (size_t)(q0 + i) * a.pieces;
        Best best = {-INFINITY, 0x7fffffff};
        for (int k = lane; k < a.pieces; k += 32) best = better(best, Best{st[k].x, __float_as_int(st[k].y)});
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = better(best, Best{__shfl_xor_sync(0xffffffffu, best.top, o), __shfl_xor_sync(0xffffffffu, best.at, o)});
        double sum = 0.0;
        for (int k = lane; k < a.pieces; k += 32)
            if (draws && st[k].x > -INFINITY) sum += (double)st[k].z * exp2(((double)st[k].x - (double)best.top) * scale);
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
        return exp2_64(((double)to_f(logits[(long long)(q0 + row) * a.stride + x]) - (double)sh.top[row]) * scale, sh.table);
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
    const T* row = logits + (long long)(q0 + last) * a.stride;
    const float* q = taken ? a.draft + (long long)(q0 + sh.first[0]) * a.draft_stride : nullptr;
    const double top = (double)sh.top[last];
    const int slice = cta * VF_WARPS + warp, slices = ctas * VF_WARPS, e0 = (int)((long long)a.vocab * slice / slices), e1 = (int)((long long)a.vocab * (slice + 1) / slices);
    double norm = 0.0;                                     // 1 / sum of weights; 0: nothing is taken off
    auto value = [&](int i, float l, float minus) {
        double w = exp2_64(((double)l - top) * scale, sh.table);
        if (norm > 0.0) return fmax(fma(w, norm, -(double)minus), 0.0);
        if (!a.draft) for (int r = 0; r < refused; r++) if (sh.token[sh.first[r]] == i) w = 0.0;
        return w;
    };
    // Sums of all slices, the same in all CTAs: every lane has those of `mine` consecutive ones, `before` those ahead of them; returns the total.
    constexpr int MOST = VF_CLUSTER * VF_WARPS / 32;
    const int mine = (slices + 31) / 32;
    double held[MOST], before = 0.0;
    auto sum_all = [&]() {
        double s[2] = {0.0, 0.0};
        constexpr int U = 8;                               // loads of so many steps side by side
        for (int base = e0 + lane; base < e1; base += 32 * U) {
            float l[U], minus[U];
#pragma unroll
            for (int k = 0; k < U; k++) {
                const bool in = base + k * 32 < e1;
                l[k] = in ? to_f(row[base + k * 32]) : -INFINITY;
                minus[k] = in && norm > 0.0 ? q[base + k * 32] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < U; k++) s[k & 1] += value(base + k * 32, l[k], minus[k]);
        }
        const double all = warp_sum64(s[0] + s[1]);
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
    double total = sum_all();
    if (taken && total > 0.0) {
        norm = 1.0 / total;
        total = sum_all();
        if (!(total > 0.0)) { norm = 0.0; total = sum_all(); }     // nothing left: the draft's distribution covers the target's
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
        if (pick == slice) {
            int found = -1, fallback = -1;
            double run = start;
            for (int base = e0; base < e1 && found < 0; base += 32) {
                const int i = base + lane;
                const double v = i < e1 ? value(i, to_f(row[i]), norm > 0.0 ? q[i] : 0.f) : 0.0;
                double x = v;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
                const unsigned hit = __ballot_sync(0xffffffffu, v > 0.0 && run + x > goal), weighs = __ballot_sync(0xffffffffu, v > 0.0);
                if (hit) found = base + __ffs(hit) - 1;
                if (weighs) fallback = base + 31 - __clz(weighs);
                run += __shfl_sync(0xffffffffu, x, 31);
            }
            if (lane == 0) a.next[b] = found >= 0 ? found : fallback;
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
    return (dtype == DYNAKV_F32 || dtype == DYNAKV_BF16) && n_tokens >= 0 && n_tokens < (1ll << 24) && vocab >= 1 && vocab <= (1 << 28) && n_seqs >= 0 &&
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
