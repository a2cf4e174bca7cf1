// dynakv_attend_tree: which kernel a call takes, and its launch.
#include "tree_rows.cuh"

namespace dkv {

// Merges the records of the units that were cut: block (x = CTA of the first launch in which the unit ends, y = 8 of its rows).
// A unit of few rows may have dozens of records (one sequence of 8192 rows: 37), so the block's 8 warps share its rows out, up
// to all eight of them taking every eighth record of one row.
template <int HD, int RT, typename OUT>
__global__ void __launch_bounds__(256) k_tree_merge(const TreeArgs a) {
    constexpr int EPL = HD / 32;
    __shared__ float part[8][HD];
    pdl_wait();
    const int* d = a.desc + (size_t)blockIdx.x * 8;
    if (!d[DESC_VALID]) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int first = d[DESC_RT] * RT + blockIdx.y * 8, here = min(RT < 8 ? RT : 8, d[DESC_T] * a.G - first);
    if (here <= 0) return;
    const int share = here > 4 ? 1 : here > 2 ? 2 : here > 1 ? 4 : 8;        // warps per row
    const int rb = warp / share, mine = warp % share, r = first + rb, rl = blockIdx.y * 8 + rb, t = r / a.G;
    const bool live = rb < here;
    const int c0 = d[DESC_FIRST], n = live ? blockIdx.x - c0 + 1 : 0;        // records: slot 1 of CTA c0, slot 0 of the others
    auto slot = [&](int i) { return ((size_t)(c0 + i) * 2 + (i == 0 ? 1 : 0)) * RT + rl; };
    float m = -INFINITY;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, a.ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    float acc[EPL], l = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; e++) acc[e] = 0.f;
    for (int i0 = 0; i0 < n; i0 += 32) {
        float f = 0.f, fl = 0.f;
        if (i0 + lane < n) { const float2 x = a.ml[slot(i0 + lane)]; f = exp2f(x.x - ref); fl = x.x - ref < -100.f ? scaled_sum(x.y, x.x - ref) : f * x.y; }
        l += warp_sum(fl);
        const int cnt = min(32, n - i0);
#pragma unroll 8
        for (int i = mine; i < cnt; i += share) {
            const float w = __shfl_sync(0xffffffffu, f, i);
            const float* p = a.acc + slot(i0 + i) * HD + lane * EPL;
            float v[EPL];
            if constexpr (EPL == 4) { const float4 x = *reinterpret_cast<const float4*>(p); v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
            else { const float2 x = *reinterpret_cast<const float2*>(p); v[0] = x.x; v[1] = x.y; }
#pragma unroll
            for (int e = 0; e < EPL; e++) acc[e] = fmaf(w, v[e], acc[e]);
        }
    }
    if (share > 1) {                               // the same in the whole block
#pragma unroll
        for (int e = 0; e < EPL; e++) part[warp][lane * EPL + e] = acc[e];
        __syncthreads();
        if (mine != 0) return;
        for (int w = 1; w < share; w++)
#pragma unroll
            for (int e = 0; e < EPL; e++) acc[e] += part[warp + w][lane * EPL + e];
    }
    if (!live) return;
    const float f = l == 0.f ? 0.f : 1.f / l;
    const size_t at = (size_t)(d[DESC_Q0] + t) * a.Hq + d[DESC_H] * a.G + r - t * a.G;
    OUT* o = reinterpret_cast<OUT*>(a.out) + at * HD + lane * EPL;
    if constexpr (sizeof(OUT) == 4) {
#pragma unroll
        for (int e = 0; e < EPL; e++) o[e] = acc[e] * f;
    } else {
#pragma unroll
        for (int e = 0; e < EPL; e += 2) reinterpret_cast<unsigned*>(o)[e / 2] = pack_bf16(acc[e] * f, acc[e + 1] * f);
    }
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// The same for the tcgen05 kernel's records, four columns of all rows side by side: a thread per row and 16 columns,
// block (x = CTA, y = 16 columns), so that the lanes' loads join.
template <int HD, int RT>
__global__ void __launch_bounds__(RT) k_tree_merge_cols(const TreeArgs a) {
    pdl_wait();
    const int* d = a.desc + (size_t)blockIdx.x * 8;
    if (!d[DESC_VALID]) return;
    const int rl = threadIdx.x, r = d[DESC_RT] * RT + rl, t = r / a.G, c0 = d[DESC_FIRST], n = blockIdx.x - c0 + 1;
    if (t >= d[DESC_T]) return;
    auto slot = [&](int i) { return (size_t)(c0 + i) * 2 + (i == 0 ? 1 : 0); };
    const float4* acc = reinterpret_cast<const float4*>(a.acc) + (size_t)blockIdx.y * 4 * RT + rl;
    float m = -INFINITY, l = 0.f;
    float4 o[4];
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < n; i++) {
        const float2 x = a.ml[slot(i) * RT + rl];
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = acc[(slot(i) * (HD / 4) + e) * RT];
        const float to = fmaxf(m, x.x), ref = to == -INFINITY ? 0.f : to, f0 = exp2f(m - ref), f1 = exp2f(x.x - ref);
        m = to;
        l = l * f0 + x.y * f1;
#pragma unroll
        for (int e = 0; e < 4; e++)
            o[e] = make_float4(o[e].x * f0 + v[e].x * f1, o[e].y * f0 + v[e].y * f1, o[e].z * f0 + v[e].z * f1, o[e].w * f0 + v[e].w * f1);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const size_t at = (size_t)(d[DESC_Q0] + t) * a.Hq + d[DESC_H] * a.G + r - t * a.G;
    uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at * HD + blockIdx.y * 16);
#pragma unroll
    for (int e = 0; e < 4; e += 2)
        out[e / 2] = make_uint4(pack_bf16(o[e].x * f, o[e].y * f), pack_bf16(o[e].z * f, o[e].w * f), pack_bf16(o[e + 1].x * f, o[e + 1].y * f), pack_bf16(o[e + 1].z * f, o[e + 1].w * f));
    if (a.lse && blockIdx.y == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// ---------------------------------------------------------------------------------- host side

template <int HD, int RT>
static cudaError_t merge_launch(bool f32, const TreeArgs& a, dim3 grid, cudaStream_t st) {
    return f32 ? launch_pdl(k_tree_merge<HD, RT, float>, grid, dim3(256), 0, st, a) : launch_pdl(k_tree_merge<HD, RT, __nv_bfloat16>, grid, dim3(256), 0, st, a);
}
template <int HD>
static cudaError_t merge_launch_rows(int rt, bool f32, const TreeArgs& a, dim3 grid, cudaStream_t st) {
    if (rt >= 128) {           // the tcgen05 kernel's tiles
        const dim3 cols(grid.x, HD / 16);
        return rt == 128 ? launch_pdl(k_tree_merge_cols<HD, 128>, cols, dim3(128), 0, st, a) : launch_pdl(k_tree_merge_cols<HD, 256>, cols, dim3(256), 0, st, a);
    }
    return rt == 4 ? merge_launch<HD, 4>(f32, a, grid, st) : rt == 8 ? merge_launch<HD, 8>(f32, a, grid, st) : rt == 16 ? merge_launch<HD, 16>(f32, a, grid, st) : rt == 32 ? merge_launch<HD, 32>(f32, a, grid, st) : merge_launch<HD, 64>(f32, a, grid, st);
}
int tree_merge_launch(int hd, int rt, bool f32, const TreeArgs& a, int ctas, cudaStream_t st) {
    const dim3 grid(ctas, (rt + 7) / 8);
    return (hd == 128 ? merge_launch_rows<128>(rt, f32, a, grid, st) : merge_launch_rows<64>(rt, f32, a, grid, st)) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

template <int HD, int DT, int RG>
static int tree_launch(const CUtensorMap& mk, const CUtensorMap& mv, const TreeArgs& a, int sms, cudaStream_t st) {
    using C = TreeCfg<HD, DT, RG, false>;
    const int grid = sms * C::per_sm;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_tree_attn<HD, DT, RG, false>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    if (launch_pdl(k_tree_attn<HD, DT, RG, false>, dim3(grid), dim3(C::threads), C::smem, st, mk, mv, a) != cudaSuccess) return DYNAKV_ERR_CUDA;
    return tree_merge_launch(HD, C::RT, DT == DYNAKV_F32, a, grid, st);
}

template <int HD, int DT>
static int tree_launch_rows(int rg, const CUtensorMap& mk, const CUtensorMap& mv, const TreeArgs& a, int sms, cudaStream_t st) {
    return rg == 0 ? tree_launch<HD, DT, 0>(mk, mv, a, sms, st) : rg == 1 ? tree_launch<HD, DT, 1>(mk, mv, a, sms, st) : rg == 2 ? tree_launch<HD, DT, 2>(mk, mv, a, sms, st) : tree_launch<HD, DT, 4>(mk, mv, a, sms, st);
}

// Which kernel, and how many CTAs with how many rows per tile.  The tcgen05 kernel pays from so many query rows per KV head on;
// mma.sync / tcgen05 in us, 8 KV heads:
//                   bf16: 16 rows   32 rows    40 rows    64 rows | FP8: 48 rows   64 rows    80 rows    128 rows
//   4 x 32768, d = 128   93 / 100  100 / 101  176 / 104  177 / 104 |  188 / 241  191 / 241  274 / 245  356 / 258
//   16 x 4096, d = 128   46 / 53    51 / 54    83 / 56    86 / 58  |   88 / 113   91 / 114  120 / 116  161 / 122
//   1 x 2048, d = 128    17 / 19    18 / 20    22 / 20    23 / 20  |   24 / 23    25 / 24    26 / 24    28 / 25
//   4 x 32768, d = 64    53 / 84    63 / 84   109 / 84   109 / 85  |  130 / 171  131 / 172  188 / 178  243 / 189
// (FP8 rows have to be converted in shared memory there.)  Spilled on mma.sync with 32 and 64 rows of 128 elements: FP8 134 to
// 138 bytes a thread, bf16 54, fp32 78.
#ifndef DKV_TREE_TC_BF16
#define DKV_TREE_TC_BF16 33
#endif
#ifndef DKV_TREE_TC_FP8
#define DKV_TREE_TC_FP8 65
#endif
struct TreeKind { bool tc; int rg, rows, ctas; };
static TreeKind tree_kind(const dynakv_row_cache* c, int n_heads, int max_tree, int sms) {
    const int most = max_tree * (n_heads / c->n_kv_heads);
    if (c->kv_dtype != DYNAKV_F32 && most >= (c->kv_dtype == DYNAKV_FP8 ? DKV_TREE_TC_FP8 : DKV_TREE_TC_BF16)) return {true, 0, most <= 128 ? 128 : 256, sms};
    const int rg = row_groups(most, c->kv_dtype == DYNAKV_F32);
    return {false, rg, rg > 0 ? 16 * rg : c->kv_dtype == DYNAKV_F32 ? 4 : 8, sms * (c->kv_dtype == DYNAKV_F32 ? 1 : 2)};
}

static bool tree_shape_ok(const dynakv_row_cache* c, int n_heads, int max_tree) {
    return row_cache_ok(c) && n_heads >= 1 && n_heads % c->n_kv_heads == 0 && n_heads / c->n_kv_heads <= MAX_G && max_tree >= 1 && max_tree <= TREE_MAX;
}

}  // namespace dkv

using namespace dkv;

extern "C" int64_t dynakv_attend_tree_workspace(const dynakv_row_cache* cache, int32_t n_heads, int32_t max_tree) {
    if (!tree_shape_ok(cache, n_heads, max_tree)) return DYNAKV_ERR_ARG;
    int rc;
    const int sms = sm_count(&rc);
    if (rc != DYNAKV_OK) return rc;
    const TreeKind k = tree_kind(cache, n_heads, max_tree, sms);
    return (int64_t)tree_space(k.ctas, k.rows, cache->head_dim).bytes;
}

extern "C" int dynakv_attend_tree(const dynakv_row_cache* cache, const void* q, int32_t n_heads, int64_t n_tokens, const int32_t* q_start,
                                  int32_t n_seqs, int32_t max_tree, const int32_t* page_table, int32_t pages_per_seq, const int32_t* kv_len,
                                  const uint64_t* tree_mask, int32_t mask_words, float scale, void* out, float* lse, void* workspace,
                                  int64_t workspace_bytes, uint32_t* status, void* cuda_stream) {
    if (!tree_shape_ok(cache, n_heads, max_tree) || n_tokens < 0 || n_tokens >= (1ll << 31) || n_seqs < 0 || pages_per_seq < 0 ||
        pages_per_seq >= (1 << 26) || !(fabsf(scale) <= FLT_MAX) || (tree_mask && (mask_words < 1 || mask_words > TREE_MAX / 64))) return DYNAKV_ERR_ARG;
    if (n_tokens == 0 || n_seqs == 0) return DYNAKV_OK;
    if (!q || !q_start || (!page_table && pages_per_seq > 0) || !kv_len || !out || !workspace) return DYNAKV_ERR_ARG;
    if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)workspace) & 15) return DYNAKV_ERR_ARG;
    int rc;
    const int sms = sm_count(&rc);
    if (rc != DYNAKV_OK) return rc;
    const TreeKind kind = tree_kind(cache, n_heads, max_tree, sms);
    const TreeSpace sp = tree_space(kind.ctas, kind.rows, cache->head_dim);
    if (workspace_bytes < (int64_t)sp.bytes) return DYNAKV_ERR_ARG;
    TreeArgs a = tree_args(cache, q, n_heads, n_tokens, q_start, n_seqs, max_tree, page_table, pages_per_seq, kv_len, out, lse, workspace, sp, status);
    a.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
    a.mask_words = tree_mask ? mask_words : 0;
    a.scale = scale;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    // an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
    cudaGetLastError();
    if (kind.tc) return tree_tc_launch(cache, kind.rows, a, sms, st);
    CUtensorMap mk, mv;
    if (!tree_page_map(&mk, cache, cache->k, true) || !tree_page_map(&mv, cache, cache->v, true)) return DYNAKV_ERR_CUDA;
    const int rg = kind.rg;
    if (cache->head_dim == 128) {
        if (cache->kv_dtype == DYNAKV_F32) return tree_launch_rows<128, DYNAKV_F32>(rg, mk, mv, a, sms, st);
        if (cache->kv_dtype == DYNAKV_BF16) return tree_launch_rows<128, DYNAKV_BF16>(rg, mk, mv, a, sms, st);
        return tree_launch_rows<128, DYNAKV_FP8>(rg, mk, mv, a, sms, st);
    }
    if (cache->kv_dtype == DYNAKV_F32) return tree_launch_rows<64, DYNAKV_F32>(rg, mk, mv, a, sms, st);
    if (cache->kv_dtype == DYNAKV_BF16) return tree_launch_rows<64, DYNAKV_BF16>(rg, mk, mv, a, sms, st);
    return tree_launch_rows<64, DYNAKV_FP8>(rg, mk, mv, a, sms, st);
}
