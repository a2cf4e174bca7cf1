// Norm and rotary embedding of single heads, and rows written to and read from a paged cache
// (dynakv_norm_rope, dynakv_norm_rope_store, dynakv_rows_write, dynakv_rows_read).
//
// All four move rows of one head: read once, a few operations per element, written once, so HBM bounds them when there
// are many rows and the launch when there are few.  A row is held by head_dim / 8 lanes, eight elements (16 bytes of
// bf16) each: the mean of squares and an FP8 row's maximum are 3 or 4 shuffles, and the partner of an element in the
// rotation is in the same lane (interleaved pairs) or in one other lane of the group (half-split pairs, because
// rotary_dim / 2 is a multiple of 8).  Nothing goes through shared memory but the sines and cosines of a token.
#include "head_rows.cuh"

namespace dkv {

struct HeadRowsDev {
    const void* p;
    long long ts, hs;      // strides in elements
};

constexpr int ROW_THREADS = 128;

// ---------------------------------------------------------------------------------- norm + rotary embedding
//
// Block (x = token, y = chunk of its rows): a group of lanes walks over the token's rows, q heads first, then k heads, then
// (store) v heads, the next row on its way while this one is normed, turned and stored.  The call is bound by the
// instructions per row as much as by HBM (a first version that normed, turned and weighted in separate steps issued 310
// per warp and pass and moved 2.4 TB/s), so the constants of a lane's eight elements are folded once per kind of
// row and block: with a = weight * cos, b = weight of the partner * (+-) sin,
//     out = f * (x * a + x_partner * b),   f = rsqrt(mean(x^2) + eps)  (1 without a norm),
// in packed fp32 pairs; rows of v stay as they are.
//
// The angle in half turns, position * (inv_freq / pi), is one 64-bit product, and its whole turns are removed in 64 bits: at
// position 2^20 the fp32 product alone would be off by 0.06 rad.  What the rest loses when it is rounded to fp32 (up to pi 2^-25 rad, more
// than the sine's own rounding) is put back with the first term of the addition formulas; the next one is below 2^-47.
__device__ __forceinline__ void head_angle(int position, float inv_freq, float* sine, float* cosine) {
    const double turns = (double)position * ((double)inv_freq * 0.31830988618379067154);   // half turns
    const double part = turns - 2.0 * rint(turns * 0.5);
    const float f = (float)part, left = (float)(part - (double)f) * 3.14159265f;
    float s, c;
    sincospif(f, &s, &c);
    *sine = fmaf(left, c, s);
    *cosine = fmaf(-left, s, c);
}

constexpr int ROPE_THREADS = 64;           // two warps: the fold below is shared by twice as many rows as with four
template <int HD, typename T, bool STORE, bool INTER>
__global__ void __launch_bounds__(ROPE_THREADS) k_norm_rope(HeadRowsDev q, HeadRowsDev k, HeadRowsDev v, int vec, dynakv_rotary ro,
                                                           const int* __restrict__ positions, void* q_out, int q_f32,
                                                           void* k_out, int k_f32, dynakv_row_cache cache,
                                                           const int* __restrict__ slots, int passes, unsigned* status) {
    constexpr int LG = HD / 8, RPP = ROPE_THREADS / LG;    // lanes per row, rows per pass
    __shared__ __align__(16) float cos_s[HD / 2], sin_s[HD / 2];
    const long long t = blockIdx.x;
    const int l = threadIdx.x % LG;
    const int n_q = ro.n_heads, n_k = ro.n_kv_heads, n_rows = n_q + n_k + (STORE ? n_k : 0);
    int r = blockIdx.y * passes * RPP + threadIdx.x / LG;
    const T* qp = reinterpret_cast<const T*>(q.p) + t * q.ts + l * 8;
    const T* kp = reinterpret_cast<const T*>(k.p) + t * k.ts + l * 8;
    const T* vp = STORE ? reinterpret_cast<const T*>(v.p) + t * v.ts + l * 8 : nullptr;
    auto load_row = [&](int r) {
        if (r >= n_rows) return zero_raw8<T>();
        return load_raw8(r < n_q ? qp + r * q.hs : !STORE || r < n_q + n_k ? kp + (r - n_q) * k.hs : vp + (r - n_q - n_k) * v.hs, vec);
    };
    Raw8<T> next = load_row(r);
    const int slot = STORE ? slots[t] : 0;
    const bool slot_ok = slot >= 0 && slot < cache.n_pages * PAGE;
    if (STORE && slot >= 0 && !slot_ok && status && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
    const int half = ro.rotary_dim / 2;
    if ((int)threadIdx.x < half) {                         // half <= 64
        head_angle(positions[t], ro.inv_freq[threadIdx.x], &sin_s[threadIdx.x], &cos_s[threadIdx.x]);
    }
    __syncthreads();
    const bool turned = l * 8 < ro.rotary_dim;             // rotary_dim is a multiple of 16: a lane is wholly in or out
    const bool upper = !INTER && l * 8 >= half;
    // half-split pairs: the lane with the partners of this lane's elements, half being a multiple of 8
    const int step = INTER || !turned ? 0 : upper ? -(half / 8) : half / 8;
    const int partner = (threadIdx.x & 31) + step;

    float2 a[4], b[4];                                     // the constants of a kind of row
    int kind = -1;                                         // 0: q, 1: k, 2: v
    bool norm = false;
    auto fold = [&]() {
        const float* w = kind == 0 ? ro.q_weight : ro.k_weight;
        norm = w != nullptr;
        float own[8], other[8];
        if (norm) {
            const bool wide = ((uintptr_t)w & 15) == 0;
            load8(w + l * 8, wide, own);
            load8(w + (l + step) * 8, wide, other);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) own[i] = other[i] = 1.f;
        }
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; i++) { c[i] = 1.f; s[i] = 0.f; }
        if (turned) {
            if constexpr (INTER) {
                const float4 cv = *reinterpret_cast<const float4*>(cos_s + l * 4), sv = *reinterpret_cast<const float4*>(sin_s + l * 4);
                c[0] = c[1] = cv.x; c[2] = c[3] = cv.y; c[4] = c[5] = cv.z; c[6] = c[7] = cv.w;
                s[0] = -sv.x; s[1] = sv.x; s[2] = -sv.y; s[3] = sv.y; s[4] = -sv.z; s[5] = sv.z; s[6] = -sv.w; s[7] = sv.w;
            } else {
                const int j = l * 8 - (upper ? half : 0);
                load8(cos_s + j, true, c);
                load8(sin_s + j, true, s);
                if (!upper) {
#pragma unroll
                    for (int i = 0; i < 8; i++) s[i] = -s[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            a[i] = make_float2(own[2 * i] * c[2 * i], own[2 * i + 1] * c[2 * i + 1]);
            b[i] = INTER ? make_float2(own[2 * i + 1] * s[2 * i], own[2 * i] * s[2 * i + 1]) : make_float2(other[2 * i] * s[2 * i], other[2 * i + 1] * s[2 * i + 1]);
        }
    };

    for (int p = 0; p < passes; p++, r += RPP) {
        float x[8], y[8];                                  // the row's elements and their partners
        unpack8(next, x);
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = x[i ^ 1];
        } else {
            Raw8<T> other;                                 // exchanged as they lie in memory: half the shuffles for bf16
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) {
                other.w[i].x = __shfl_sync(0xffffffffu, next.w[i].x, partner); other.w[i].y = __shfl_sync(0xffffffffu, next.w[i].y, partner);
                other.w[i].z = __shfl_sync(0xffffffffu, next.w[i].z, partner); other.w[i].w = __shfl_sync(0xffffffffu, next.w[i].w, partner);
            }
            unpack8(other, y);
        }
        if (p + 1 < passes) next = load_row(r + RPP);
        const bool live = r < n_rows;
        const int now = r < n_q ? 0 : !STORE || r < n_q + n_k ? 1 : 2;
        if (now != kind) { kind = now; if (kind < 2) fold(); }
        float2 sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; i++) { const float2 y = make_float2(x[2 * i], x[2 * i + 1]); sq = fma2(y, y, sq); }
        float ss = sq.x + sq.y;
#pragma unroll
        for (int o = LG / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float f = norm ? rsqrtf(ss * (1.f / HD) + ro.eps) : 1.f;
        if (!turned) {                                     // no partner: an infinity there would make 0 * inf
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = 0.f;
        }
        const float2 ff = make_float2(f, f);
        if (kind < 2) {                                    // rows of v stay as they are, signs of zeros too
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float2 o = mul2(make_float2(y[2 * i], y[2 * i + 1]), b[i]);
                o = mul2(fma2(make_float2(x[2 * i], x[2 * i + 1]), a[i], o), ff);
                x[2 * i] = o.x; x[2 * i + 1] = o.y;
            }
        }
        if (kind == 0) {
            if (live) {
                const size_t at = ((size_t)t * n_q + r) * HD + l * 8;
                if (q_f32) store8(reinterpret_cast<float*>(q_out) + at, x);
                else store8(reinterpret_cast<__nv_bfloat16*>(q_out) + at, x);
            }
        } else if (!STORE) {
            if (live) {
                const size_t at = ((size_t)t * n_k + r - n_q) * HD + l * 8;
                if (k_f32) store8(reinterpret_cast<float*>(k_out) + at, x);
                else store8(reinterpret_cast<__nv_bfloat16*>(k_out) + at, x);
            }
        }
        if (STORE && __any_sync(0xffffffffu, kind != 0)) {     // the whole warp: an FP8 row's maximum is exchanged by shuffles
            const int h = kind == 2 ? r - n_q - n_k : r - n_q;
            const long long row = ((long long)(slot >> 5) * n_k + h) * PAGE + (slot & 31);
            const float (&xs)[1][8] = reinterpret_cast<const float (&)[1][8]>(x);
            store_cache<HD, 1>(cache, kind == 2, row, live && kind != 0 && slot_ok, l, xs);
        }
    }
}

// The same for the usual case, whole heads rotated in half-split pairs (rotary_dim = head_dim): a lane takes the eight elements
// at l * 8 and the eight at l * 8 + head_dim / 2, so that every pair lies inside it.  No exchange of partners, half the
// lanes per row and half the per-row instructions (8192 tokens of 32 + 8 heads: 43 us with the kernel above, 34 us with
// this one, against 26 us at the measured copy rate).  72 registers, 40 to 68 bytes spilled in most variants: 13 blocks per SM
// (96 registers: 37 us; 64: 37 us).
template <int HD, typename T, bool STORE>
__global__ void __launch_bounds__(ROPE_THREADS, 13) k_norm_rope_whole(HeadRowsDev q, HeadRowsDev k, HeadRowsDev v, int vec, dynakv_rotary ro,
                                                                  const int* __restrict__ positions, void* q_out, int q_f32,
                                                                  void* k_out, int k_f32, dynakv_row_cache cache,
                                                                  const int* __restrict__ slots, int passes, unsigned* status) {
    constexpr int LG = HD / 16, RPP = ROPE_THREADS / LG, H2 = HD / 2;
    __shared__ __align__(16) float cos_s[H2], sin_s[H2];
    const long long t = blockIdx.x;
    const int l = threadIdx.x % LG;
    const int n_q = ro.n_heads, n_k = ro.n_kv_heads, n_rows = n_q + n_k + (STORE ? n_k : 0);
    int r = blockIdx.y * passes * RPP + threadIdx.x / LG;
    const T* qp = reinterpret_cast<const T*>(q.p) + t * q.ts + l * 8;
    const T* kp = reinterpret_cast<const T*>(k.p) + t * k.ts + l * 8;
    const T* vp = STORE ? reinterpret_cast<const T*>(v.p) + t * v.ts + l * 8 : nullptr;
    Raw8<T> next[2];
    auto load_row = [&](int r) {
        next[0] = next[1] = zero_raw8<T>();
        if (r >= n_rows) return;
        const T* p = r < n_q ? qp + r * q.hs : !STORE || r < n_q + n_k ? kp + (r - n_q) * k.hs : vp + (r - n_q - n_k) * v.hs;
        next[0] = load_raw8(p, vec);
        next[1] = load_raw8(p + H2, vec);
    };
    load_row(r);
    const int slot = STORE ? slots[t] : 0;
    const bool slot_ok = slot >= 0 && slot < cache.n_pages * PAGE;
    if (STORE && slot >= 0 && !slot_ok && status && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
    if ((int)threadIdx.x < H2) {
        head_angle(positions[t], ro.inv_freq[threadIdx.x], &sin_s[threadIdx.x], &cos_s[threadIdx.x]);
    }
    __syncthreads();
    // lo' = lo * (w_lo cos) - hi * (w_hi sin), hi' = hi * (w_hi cos) + lo * (w_lo sin)
    float2 lc[4], hs[4], hc[4], ls[4];
    int kind = -1;                                         // 0: q, 1: k, 2: v
    bool norm = false;
    auto fold = [&]() {
        const float* w = kind == 0 ? ro.q_weight : kind == 1 ? ro.k_weight : nullptr;
        norm = w != nullptr;
        float wl[8], wh[8], c[8], s[8];
        if (norm) {
            const bool wide = ((uintptr_t)w & 15) == 0;
            load8(w + l * 8, wide, wl);
            load8(w + l * 8 + H2, wide, wh);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) wl[i] = wh[i] = 1.f;
        }
        if (kind < 2) {
            load8(cos_s + l * 8, true, c);
            load8(sin_s + l * 8, true, s);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) { c[i] = 1.f; s[i] = 0.f; }
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            lc[i] = make_float2(wl[2 * i] * c[2 * i], wl[2 * i + 1] * c[2 * i + 1]);
            ls[i] = make_float2(wl[2 * i] * s[2 * i], wl[2 * i + 1] * s[2 * i + 1]);
            hc[i] = make_float2(wh[2 * i] * c[2 * i], wh[2 * i + 1] * c[2 * i + 1]);
            hs[i] = make_float2(-(wh[2 * i] * s[2 * i]), -(wh[2 * i + 1] * s[2 * i + 1]));
        }
    };
    for (int p = 0; p < passes; p++, r += RPP) {
        float x[2][8];
        unpack8(next[0], x[0]);
        unpack8(next[1], x[1]);
        if (p + 1 < passes) load_row(r + RPP);
        const bool live = r < n_rows;
        const int now = r < n_q ? 0 : !STORE || r < n_q + n_k ? 1 : 2;
        if (now != kind) { kind = now; fold(); }
        float2 sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int y = 0; y < 2; y++)
#pragma unroll
            for (int i = 0; i < 4; i++) { const float2 z = make_float2(x[y][2 * i], x[y][2 * i + 1]); sq = fma2(z, z, sq); }
        float ss = sq.x + sq.y;
#pragma unroll
        for (int o = LG / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float f = norm ? rsqrtf(ss * (1.f / HD) + ro.eps) : 1.f;
        const float2 ff = make_float2(f, f);
        if (kind < 2) {                                    // rows of v stay as they are
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 lo = make_float2(x[0][2 * i], x[0][2 * i + 1]), hi = make_float2(x[1][2 * i], x[1][2 * i + 1]);
                const float2 a = mul2(fma2(lo, lc[i], mul2(hi, hs[i])), ff), b = mul2(fma2(hi, hc[i], mul2(lo, ls[i])), ff);
                x[0][2 * i] = a.x; x[0][2 * i + 1] = a.y;
                x[1][2 * i] = b.x; x[1][2 * i + 1] = b.y;
            }
        }
        if (kind == 0 || !STORE) {
            if (live) {
                const bool wide = kind == 0 ? q_f32 : k_f32;
                void* out = kind == 0 ? q_out : k_out;
                const size_t at = (kind == 0 ? (size_t)t * n_q + r : (size_t)t * n_k + r - n_q) * HD + l * 8;
                if (wide) { store8(reinterpret_cast<float*>(out) + at, x[0]); store8(reinterpret_cast<float*>(out) + at + H2, x[1]); }
                else { store8(reinterpret_cast<__nv_bfloat16*>(out) + at, x[0]); store8(reinterpret_cast<__nv_bfloat16*>(out) + at + H2, x[1]); }
            }
        }
        if (STORE && __any_sync(0xffffffffu, kind != 0)) {     // the whole warp: an FP8 row's maximum is exchanged by shuffles
            const int h = kind == 2 ? r - n_q - n_k : r - n_q;
            const long long row = ((long long)(slot >> 5) * n_k + h) * PAGE + (slot & 31);
            store_cache<HD, 2>(cache, kind == 2, row, live && kind != 0 && slot_ok, l, x);
        }
    }
}

// ---------------------------------------------------------------------------------- rows into the cache
//
// A token's 2 * n_kv_heads rows (k heads, then v heads) side by side in a block's groups of lanes, as many tokens as fit
// (or, with many heads, part of a token: blockIdx.y); each group takes the same row of `per` <= WR tokens, all loads before
// the first store.  Which row that is takes one division per thread.
constexpr int WR = 4;
template <int HD, typename T>
__global__ void __launch_bounds__(ROW_THREADS) k_rows_write(HeadRowsDev k, HeadRowsDev v, int vec, dynakv_row_cache cache,
                                                            const int* __restrict__ slots, long long n, int per, unsigned* status) {
    constexpr int LG = HD / 8, RPP = ROW_THREADS / LG;
    const int l = threadIdx.x % LG, grp = threadIdx.x / LG;
    const int nk = cache.n_kv_heads, tp = 2 * nk <= RPP ? RPP / (2 * nk) : 1;      // tokens side by side
    const int dt = tp > 1 ? grp / (2 * nk) : 0;
    const int h2 = blockIdx.y * RPP + grp - dt * 2 * nk;
    const bool there = dt < tp && h2 < 2 * nk, is_v = h2 >= nk;
    const int h = is_v ? h2 - nk : h2;
    const HeadRowsDev& from = is_v ? v : k;
    const T* p = reinterpret_cast<const T*>(from.p) + h * from.hs + l * 8;
    const long long t0 = (long long)blockIdx.x * (tp * per) + dt;
    Raw8<T> raw[WR];
    int slot[WR];
#pragma unroll
    for (int i = 0; i < WR; i++) {
        const long long t = t0 + i * tp;
        raw[i] = zero_raw8<T>();
        slot[i] = -1;
        if (i < per && there && t < n) {
            raw[i] = load_raw8(p + t * from.ts, vec);
            slot[i] = slots[t];
        }
    }
#pragma unroll
    for (int i = 0; i < WR; i++) {
        if (i >= per) break;
        const bool live = slot[i] >= 0 && slot[i] < cache.n_pages * PAGE;
        if (slot[i] >= 0 && !live && status && l == 0 && h2 == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
        float x[1][8];
        unpack8(raw[i], x[0]);
        store_cache<HD, 1>(cache, is_v, ((long long)(slot[i] >> 5) * nk + h) * PAGE + (slot[i] & 31), live, l, x);
    }
}

// ---------------------------------------------------------------------------------- rows out of the cache
//
// Block (x = 32 output rows, y = KV head, z = sequence), K and V; each group of lanes takes every RPP-th row, the loads of
// all its rows before the first store.
template <int HD, int DT>
__global__ void __launch_bounds__(ROW_THREADS) k_rows_read(dynakv_row_cache cache, const int* __restrict__ page_table, int pages_per_seq,
                                                           const int* __restrict__ lengths, long long first, long long n,
                                                           void* K_out, void* V_out, unsigned* status) {
    constexpr int LG = HD / 8, RPP = ROW_THREADS / LG, NR = PAGE / RPP;
    const int l = threadIdx.x % LG, grp = threadIdx.x / LG;
    const int h = blockIdx.y, b = blockIdx.z, nk = cache.n_kv_heads;
    const long long len = lengths[b];
    const int* table = page_table + (size_t)b * pages_per_seq;
    if (len < 0 && status && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
    uint4 raw[2][NR][DT == DYNAKV_F32 ? 2 : 1];
    float scale[2][NR];
    bool there[NR];
#pragma unroll
    for (int i = 0; i < NR; i++) {
        const long long o = (long long)blockIdx.x * PAGE + i * RPP + grp, r = first + o;
        there[i] = false;
        if (o < n && r < len) {
            const long long at = r / PAGE;
            const int page = at < pages_per_seq ? table[at] : -1;
            there[i] = page >= 0 && page < cache.n_pages;
            if (!there[i] && status && l == 0 && h == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
            const long long row = ((long long)page * nk + h) * PAGE + (r & (PAGE - 1));
            if (there[i]) {
#pragma unroll
                for (int kv = 0; kv < 2; kv++) {
                    const unsigned char* pool = reinterpret_cast<const unsigned char*>(kv ? cache.v : cache.k);
                    if constexpr (DT == DYNAKV_F32) {
                        const uint4* p = reinterpret_cast<const uint4*>(pool + ((size_t)row * HD + l * 8) * 4);
                        raw[kv][i][0] = p[0]; raw[kv][i][1] = p[1];
                    } else if constexpr (DT == DYNAKV_BF16) {
                        raw[kv][i][0] = *reinterpret_cast<const uint4*>(pool + ((size_t)row * HD + l * 8) * 2);
                    } else {
                        const uint2 w = *reinterpret_cast<const uint2*>(pool + (size_t)row * HD + l * 8);
                        raw[kv][i][0].x = w.x; raw[kv][i][0].y = w.y;
                        scale[kv][i] = pow2f((kv ? cache.v_exp : cache.k_exp)[row]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NR; i++) {
        const long long o = (long long)blockIdx.x * PAGE + i * RPP + grp;
        if (o >= n) continue;
        const size_t at = (((size_t)b * nk + h) * n + o) * HD + l * 8;
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            void* out = kv ? V_out : K_out;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (DT == DYNAKV_F32) {
                uint4* p = reinterpret_cast<uint4*>(reinterpret_cast<float*>(out) + at);
                p[0] = there[i] ? raw[kv][i][0] : zero;
                p[1] = there[i] ? raw[kv][i][1] : zero;
            } else if constexpr (DT == DYNAKV_BF16) {
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = there[i] ? raw[kv][i][0] : zero;
            } else {
                uint4 w = zero;
                if (there[i]) {
                    const float2 a = fp8_unpack2((unsigned short)(raw[kv][i][0].x & 0xffffu), scale[kv][i]);
                    const float2 c = fp8_unpack2((unsigned short)(raw[kv][i][0].x >> 16), scale[kv][i]);
                    const float2 e = fp8_unpack2((unsigned short)(raw[kv][i][0].y & 0xffffu), scale[kv][i]);
                    const float2 g = fp8_unpack2((unsigned short)(raw[kv][i][0].y >> 16), scale[kv][i]);
                    w = make_uint4(pack_bf16(a.x, a.y), pack_bf16(c.x, c.y), pack_bf16(e.x, e.y), pack_bf16(g.x, g.y));
                }
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = w;
            }
        }
    }
}

}  // namespace dkv

using namespace dkv;

static bool head_rows_ok(const dynakv_head_rows* a, int dtype) {
    return a && a->data && a->dtype == dtype && ((uintptr_t)a->data & (dtype == DYNAKV_F32 ? 3 : 1)) == 0;
}
static bool head_rows_vec(const dynakv_head_rows* a) {
    const int es = a->dtype == DYNAKV_F32 ? 4 : 2;
    return ((uintptr_t)a->data & 15) == 0 && (a->token_stride * es) % 16 == 0 && (a->head_stride * es) % 16 == 0;
}
static HeadRowsDev head_rows_dev(const dynakv_head_rows* a) { return HeadRowsDev{a->data, a->token_stride, a->head_stride}; }
static bool float_type(int dtype) { return dtype == DYNAKV_F32 || dtype == DYNAKV_BF16; }
// an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
static void forget_errors() { cudaGetLastError(); }
static int launched() { return cudaGetLastError() == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA; }

static int norm_rope(const dynakv_rotary* ro, const dynakv_head_rows* q, const dynakv_head_rows* k, const dynakv_head_rows* v,
                     const int32_t* positions, int64_t n, void* q_out, int32_t q_dtype, void* k_out, int32_t k_dtype,
                     const dynakv_row_cache* cache, const int32_t* slots, uint32_t* status, cudaStream_t st) {
    if (!ro || !q || !k || n < 0 || n >= (1ll << 31) || ro->n_heads < 1 || ro->n_kv_heads < 1 || ro->n_heads > 65536 || ro->n_kv_heads > 65536 ||
        (ro->head_dim != 64 && ro->head_dim != 128) || ro->rotary_dim < 0 || ro->rotary_dim > ro->head_dim || ro->rotary_dim % 16 != 0 ||
        !(ro->eps >= 0.f) || (ro->rotary_dim > 0 && !ro->inv_freq) || !float_type(q_dtype)) return DYNAKV_ERR_ARG;
    if (n == 0) return DYNAKV_OK;
    if (!float_type(q->dtype) || !head_rows_ok(q, q->dtype) || !head_rows_ok(k, q->dtype) || (v && !head_rows_ok(v, q->dtype)) || !positions ||
        !q_out || ((uintptr_t)q_out & 15) || (k_out && ((uintptr_t)k_out & 15))) return DYNAKV_ERR_ARG;
    const bool whole = !ro->interleaved && ro->rotary_dim == ro->head_dim;
    const int rpp = ROPE_THREADS / (ro->head_dim / (whole ? 16 : 8));
    const int rows = ro->n_heads + ro->n_kv_heads * (cache ? 2 : 1), chunks = (rows + rpp - 1) / rpp;
    // a whole token per block once there are two blocks for every SM of a B200 (148), which shares the sines and the folded constants by all
    // of its rows; fewer tokens (a decode step) spread over the SMs, one pass per block
    const int passes = n >= 148 * 2 ? chunks : 1;
    const dim3 grid((unsigned)n, (unsigned)((chunks + passes - 1) / passes));
    const int vec = head_rows_vec(q) && head_rows_vec(k) && (!v || head_rows_vec(v));
    const HeadRowsDev dq = head_rows_dev(q), dk = head_rows_dev(k), dv = v ? head_rows_dev(v) : HeadRowsDev{nullptr, 0, 0};
    const dynakv_row_cache c = cache ? *cache : dynakv_row_cache{};
    const int qf = q_dtype == DYNAKV_F32, kf = k_dtype == DYNAKV_F32;
    forget_errors();
#define DKV_ROPE(HD, T, STORE, INTER) \
    k_norm_rope<HD, T, STORE, INTER><<<grid, ROPE_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status)
#define DKV_ROPE_WHOLE(HD, T, STORE) \
    k_norm_rope_whole<HD, T, STORE><<<grid, ROPE_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status)
#define DKV_ROPE_KIND(HD, T) \
    do { \
        if (whole) { if (cache) DKV_ROPE_WHOLE(HD, T, true); else DKV_ROPE_WHOLE(HD, T, false); } \
        else if (cache) { if (ro->interleaved) DKV_ROPE(HD, T, true, true); else DKV_ROPE(HD, T, true, false); } \
        else { if (ro->interleaved) DKV_ROPE(HD, T, false, true); else DKV_ROPE(HD, T, false, false); } \
    } while (0)
    if (ro->head_dim == 128) {
        if (q->dtype == DYNAKV_F32) DKV_ROPE_KIND(128, float);
        else DKV_ROPE_KIND(128, __nv_bfloat16);
    } else {
        if (q->dtype == DYNAKV_F32) DKV_ROPE_KIND(64, float);
        else DKV_ROPE_KIND(64, __nv_bfloat16);
    }
#undef DKV_ROPE_KIND
#undef DKV_ROPE_WHOLE
#undef DKV_ROPE
    return launched();
}

extern "C" int dynakv_norm_rope(const dynakv_rotary* rotary, const dynakv_head_rows* q, const dynakv_head_rows* k,
                                const int32_t* positions, int64_t n, void* q_out, int32_t q_dtype, void* k_out, int32_t k_dtype,
                                void* cuda_stream) {
    if (!float_type(k_dtype) || (n > 0 && !k_out)) return DYNAKV_ERR_ARG;
    return norm_rope(rotary, q, k, nullptr, positions, n, q_out, q_dtype, k_out, k_dtype, nullptr, nullptr, nullptr,
                     reinterpret_cast<cudaStream_t>(cuda_stream));
}

extern "C" int dynakv_norm_rope_store(const dynakv_rotary* rotary, const dynakv_head_rows* q, const dynakv_head_rows* k,
                                      const dynakv_head_rows* v, const int32_t* positions, int64_t n, void* q_out, int32_t q_dtype,
                                      const dynakv_row_cache* cache, const int32_t* slots, uint32_t* status, void* cuda_stream) {
    if (!rotary || !row_cache_ok(cache) || cache->head_dim != rotary->head_dim || cache->n_kv_heads != rotary->n_kv_heads ||
        !v || (n > 0 && !slots)) return DYNAKV_ERR_ARG;
    return norm_rope(rotary, q, k, v, positions, n, q_out, q_dtype, nullptr, DYNAKV_F32, cache, slots, status,
                     reinterpret_cast<cudaStream_t>(cuda_stream));
}

extern "C" int dynakv_rows_write(const dynakv_row_cache* cache, const dynakv_head_rows* k, const dynakv_head_rows* v,
                                 const int32_t* slots, int64_t n, uint32_t* status, void* cuda_stream) {
    if (!row_cache_ok(cache) || !k || !v || n < 0 || n >= (1ll << 31)) return DYNAKV_ERR_ARG;
    if (n == 0) return DYNAKV_OK;
    if (!float_type(k->dtype) || !head_rows_ok(k, k->dtype) || !head_rows_ok(v, k->dtype) || !slots) return DYNAKV_ERR_ARG;
    const int rpp = ROW_THREADS / (cache->head_dim / 8), rows = 2 * cache->n_kv_heads;
    const int tp = rows <= rpp ? rpp / rows : 1, chunks = (rows + rpp - 1) / rpp;
    if (chunks > 65535) return DYNAKV_ERR_TOO_LARGE;
    // few tokens: one per group of lanes, over as many blocks as that gives; many: four, for the loads in flight
    const int per = n * chunks >= 148ll * 8 * tp * WR ? WR : 1;
    const dim3 g((unsigned)((n + tp * per - 1) / (tp * per)), (unsigned)chunks);
    const int vec = head_rows_vec(k) && head_rows_vec(v);
    const HeadRowsDev dk = head_rows_dev(k), dv = head_rows_dev(v);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    forget_errors();
    if (cache->head_dim == 128) {
        if (k->dtype == DYNAKV_F32) k_rows_write<128, float><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, n, per, status);
        else k_rows_write<128, __nv_bfloat16><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, n, per, status);
    } else {
        if (k->dtype == DYNAKV_F32) k_rows_write<64, float><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, n, per, status);
        else k_rows_write<64, __nv_bfloat16><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, n, per, status);
    }
    return launched();
}

extern "C" int dynakv_rows_read(const dynakv_row_cache* cache, const int32_t* page_table, int32_t pages_per_seq, const int32_t* lengths,
                                int32_t n_seqs, int64_t first, int64_t n, void* K_out, void* V_out, uint32_t* status, void* cuda_stream) {
    if (!row_cache_ok(cache) || pages_per_seq < 0 || n_seqs < 0 || n_seqs > 65535 || cache->n_kv_heads > 65535 || first < 0 || n < 0 ||
        n >= (1ll << 31) || first >= (1ll << 31)) return DYNAKV_ERR_ARG;
    if (n == 0 || n_seqs == 0) return DYNAKV_OK;
    if ((!page_table && pages_per_seq > 0) || !lengths || !K_out || !V_out || (((uintptr_t)K_out | (uintptr_t)V_out) & 15)) return DYNAKV_ERR_ARG;
    const dim3 grid((unsigned)((n + PAGE - 1) / PAGE), (unsigned)cache->n_kv_heads, (unsigned)n_seqs);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    forget_errors();
#define DKV_READ(HD, DT) k_rows_read<HD, DT><<<grid, ROW_THREADS, 0, st>>>(*cache, page_table, pages_per_seq, lengths, first, n, K_out, V_out, status)
    if (cache->head_dim == 128) {
        if (cache->kv_dtype == DYNAKV_F32) DKV_READ(128, DYNAKV_F32);
        else if (cache->kv_dtype == DYNAKV_BF16) DKV_READ(128, DYNAKV_BF16);
        else DKV_READ(128, DYNAKV_FP8);
    } else {
        if (cache->kv_dtype == DYNAKV_F32) DKV_READ(64, DYNAKV_F32);
        else if (cache->kv_dtype == DYNAKV_BF16) DKV_READ(64, DYNAKV_BF16);
        else DKV_READ(64, DYNAKV_FP8);
    }
#undef DKV_READ
    return launched();
}
