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
// Block (x = token, y = chunk of its rows): the token's sines and cosines are taken once per block, each thread keeps the
// eight pairs of its own elements in registers and walks over the heads, q heads first, then k heads, then (store) v
// heads.  A decode step has few tokens, so a token is cut into chunks of one pass over the block; a prompt's tokens are
// taken whole, which shares the sines by all heads.
//
// The angle in half turns, position * (inv_freq / pi), is one 64-bit product, and its whole turns are removed in 64 bits
// before the rest is rounded to fp32: at position 2^20 the fp32 product alone would be off by 0.06 rad.
template <int HD, typename T>
__global__ void __launch_bounds__(ROW_THREADS) k_norm_rope(HeadRowsDev q, HeadRowsDev k, HeadRowsDev v, int vec, dynakv_rotary ro,
                                                           const int* __restrict__ positions, void* q_out, int q_f32,
                                                           void* k_out, int k_f32, dynakv_row_cache cache,
                                                           const int* __restrict__ slots, int passes, unsigned* status) {
    constexpr int LG = HD / 8, RPP = ROW_THREADS / LG;     // lanes per row, rows per pass
    __shared__ float2 sc[HD / 2];
    const long long t = blockIdx.x;
    const int l = threadIdx.x % LG, grp = threadIdx.x / LG;
    const bool store = slots != nullptr;
    const int n_q = ro.n_heads, n_k = ro.n_kv_heads, n_rows = n_q + n_k + (store ? n_k : 0);
    const int first = blockIdx.y * passes * RPP;
    const int slot = store ? slots[t] : 0;
    const bool slot_ok = slot >= 0 && slot < cache.n_pages * PAGE;
    if (store && slot >= 0 && !slot_ok && status && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(status, DYNAKV_ST_BOUNDS);

    if ((int)threadIdx.x < ro.rotary_dim / 2) {
        const double turns = (double)positions[t] * ((double)ro.inv_freq[threadIdx.x] * 0.31830988618379067154);   // half turns
        const float r = (float)(turns - 2.0 * rint(turns * 0.5));
        float s, c;
        sincospif(r, &s, &c);
        sc[threadIdx.x] = make_float2(c, s);
    }
    __syncthreads();
    // the rotation of this lane's eight elements: x' = x * cs + partner * sn, the sign of the pair's half in sn
    float cs[8], sn[8];
    const bool turned = l * 8 < ro.rotary_dim;             // rotary_dim is a multiple of 16: a lane is wholly in or out
    const int half = ro.rotary_dim / 2;
    int partner = l;
    if (turned) {
        if (ro.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; i++) { const float2 a = sc[l * 4 + i / 2]; cs[i] = a.x; sn[i] = (i & 1) ? a.y : -a.y; }
        } else {
            const bool upper = l * 8 >= half;
            partner = upper ? l - half / 8 : l + half / 8;
#pragma unroll
            for (int i = 0; i < 8; i++) { const float2 a = sc[l * 8 + i - (upper ? half : 0)]; cs[i] = a.x; sn[i] = upper ? a.y : -a.y; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) { cs[i] = 1.f; sn[i] = 0.f; }
    }
    float wq[8], wk[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        wq[i] = ro.q_weight ? ro.q_weight[l * 8 + i] : 1.f;
        wk[i] = ro.k_weight ? ro.k_weight[l * 8 + i] : 1.f;
    }

    auto row_ptr = [&](int r) -> const T* {
        const HeadRowsDev& a = r < n_q ? q : r < n_q + n_k ? k : v;
        const int h = r < n_q ? r : r < n_q + n_k ? r - n_q : r - n_q - n_k;
        return reinterpret_cast<const T*>(a.p) + t * a.ts + h * a.hs + l * 8;
    };
    // the next row is on its way while this one is normed, turned and stored; every lane takes part in the shuffles
    float nx[8];
    {
        const int r = first + grp;
        if (r < n_rows) load8(row_ptr(r), vec, nx);
        else {
#pragma unroll
            for (int i = 0; i < 8; i++) nx[i] = 0.f;
        }
    }
    for (int p = 0; p < passes; p++) {
        const int r = first + p * RPP + grp;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = nx[i];
        if (p + 1 < passes && r + RPP < n_rows) load8(row_ptr(r + RPP), vec, nx);
        const bool live = r < n_rows, is_q = r < n_q, is_v = r >= n_q + n_k;
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = LG / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const bool norm = !is_v && (is_q ? ro.q_weight != nullptr : ro.k_weight != nullptr);
        const float f = norm ? 1.f / sqrtf(ss * (1.f / HD) + ro.eps) : 1.f;
        if (norm) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = x[i] * f * (is_q ? wq[i] : wk[i]);
        }
        float y[8];
        if (ro.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = x[i ^ 1];
        } else {
            const int src = (threadIdx.x & 31) - l + partner;
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = __shfl_sync(0xffffffffu, x[i], src);
        }
        if (turned && !is_v) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = fmaf(x[i], cs[i], y[i] * sn[i]);
        }
        if (is_q) {
            if (live) {
                const size_t at = ((size_t)t * n_q + r) * HD + l * 8;
                if (q_f32) store8(reinterpret_cast<float*>(q_out) + at, x);
                else store8(reinterpret_cast<__nv_bfloat16*>(q_out) + at, x);
            }
        } else if (!store) {
            if (live) {
                const size_t at = ((size_t)t * n_k + r - n_q) * HD + l * 8;
                if (k_f32) store8(reinterpret_cast<float*>(k_out) + at, x);
                else store8(reinterpret_cast<__nv_bfloat16*>(k_out) + at, x);
            }
        }
        if (store) {         // all lanes of the warp come here: an FP8 row's maximum is exchanged by shuffles
            const int h = is_v ? r - n_q - n_k : r - n_q;
            const long long row = ((long long)(slot >> 5) * n_k + h) * PAGE + (slot & 31);
            store_cache8<HD>(cache, is_v, row, live && !is_q && slot_ok, l, x);
        }
    }
}

// ---------------------------------------------------------------------------------- rows into the cache
//
// One flat list of rows, (token, k or v, head); a group of lanes takes WR of them, all loads before the first store.
constexpr int WR = 4;
template <int HD, typename T>
__global__ void __launch_bounds__(ROW_THREADS) k_rows_write(HeadRowsDev k, HeadRowsDev v, int vec, dynakv_row_cache cache,
                                                            const int* __restrict__ slots, long long n_rows, int per, unsigned* status) {
    constexpr int LG = HD / 8, RPP = ROW_THREADS / LG;
    const int l = threadIdx.x % LG, grp = threadIdx.x / LG;
    const int nk = cache.n_kv_heads;
    float x[WR][8];
    long long row[WR];
    bool live[WR], is_v[WR];
    const long long r0 = (long long)blockIdx.x * (RPP * per) + grp;
#pragma unroll
    for (int i = 0; i < WR; i++) {
        const long long r = r0 + i * RPP;
        live[i] = i < per && r < n_rows;
        is_v[i] = false;
        row[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) x[i][j] = 0.f;
        if (live[i]) {
            const long long t = r / (2 * nk);
            const int h2 = (int)(r - t * (2 * nk));
            is_v[i] = h2 >= nk;
            const int h = is_v[i] ? h2 - nk : h2;
            const int slot = slots[t];
            const HeadRowsDev& a = is_v[i] ? v : k;
            load8(reinterpret_cast<const T*>(a.p) + t * a.ts + h * a.hs + l * 8, vec, x[i]);
            live[i] = slot >= 0 && slot < cache.n_pages * PAGE;
            if (slot >= 0 && !live[i] && status && l == 0 && h2 == 0) atomicOr(status, DYNAKV_ST_BOUNDS);
            row[i] = ((long long)(slot >> 5) * nk + h) * PAGE + (slot & 31);
        }
    }
#pragma unroll
    for (int i = 0; i < WR; i++) if (i < per) store_cache8<HD>(cache, is_v[i], row[i], live[i], l, x[i]);
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
    const int rpp = ROW_THREADS / (ro->head_dim / 8);
    const int rows = ro->n_heads + ro->n_kv_heads * (cache ? 2 : 1);
    const int chunks = (rows + rpp - 1) / rpp;
    // a whole token per block once that gives every SM (148) its 16 resident blocks; below that one pass per block, so
    // that a decode step spreads over the SMs (16 tokens x 32 rows: 64 blocks of one pass against 16 blocks of four)
    const int passes = n >= 148 * 16 ? chunks : 1;
    const dim3 grid((unsigned)n, (unsigned)((chunks + passes - 1) / passes));
    const int vec = head_rows_vec(q) && head_rows_vec(k) && (!v || head_rows_vec(v));
    const HeadRowsDev dq = head_rows_dev(q), dk = head_rows_dev(k), dv = v ? head_rows_dev(v) : HeadRowsDev{nullptr, 0, 0};
    const dynakv_row_cache c = cache ? *cache : dynakv_row_cache{};
    const int qf = q_dtype == DYNAKV_F32, kf = k_dtype == DYNAKV_F32;
    forget_errors();
    if (ro->head_dim == 128) {
        if (q->dtype == DYNAKV_F32) k_norm_rope<128, float><<<grid, ROW_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status);
        else k_norm_rope<128, __nv_bfloat16><<<grid, ROW_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status);
    } else {
        if (q->dtype == DYNAKV_F32) k_norm_rope<64, float><<<grid, ROW_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status);
        else k_norm_rope<64, __nv_bfloat16><<<grid, ROW_THREADS, 0, st>>>(dq, dk, dv, vec, *ro, positions, q_out, qf, k_out, kf, c, slots, passes, status);
    }
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
    const long long rows = n * 2 * cache->n_kv_heads;
    const int rpp = ROW_THREADS / (cache->head_dim / 8);
    // few rows: one per group of lanes, over as many blocks as there are; many: four, for the loads in flight
    const int per = rows >= 148ll * 8 * rpp * WR ? WR : 1;
    const long long blocks = (rows + rpp * per - 1) / (rpp * per);
    if (blocks >= (1ll << 31)) return DYNAKV_ERR_TOO_LARGE;
    const int vec = head_rows_vec(k) && head_rows_vec(v);
    const HeadRowsDev dk = head_rows_dev(k), dv = head_rows_dev(v);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const unsigned g = (unsigned)blocks;
    forget_errors();
    if (cache->head_dim == 128) {
        if (k->dtype == DYNAKV_F32) k_rows_write<128, float><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, rows, per, status);
        else k_rows_write<128, __nv_bfloat16><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, rows, per, status);
    } else {
        if (k->dtype == DYNAKV_F32) k_rows_write<64, float><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, rows, per, status);
        else k_rows_write<64, __nv_bfloat16><<<g, ROW_THREADS, 0, st>>>(dk, dv, vec, *cache, slots, rows, per, status);
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
