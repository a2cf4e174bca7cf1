// dynakv_attend_chunk: which kernel a call takes, and its launch.
#include "chunk_plan.cuh"
#include "tree_rows.cuh"

namespace dkv {

template <int HD, int DT, int RG>
static int chunk_launch(const CUtensorMap& mk, const CUtensorMap& mv, const TreeArgs& a, int sms, cudaStream_t st) {
    using C = TreeCfg<HD, DT, RG, true>;
    const int grid = sms * C::per_sm;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(k_tree_attn<HD, DT, RG, true>, C::smem, allowed)) return DYNAKV_ERR_CUDA;
    if (launch_pdl(k_tree_attn<HD, DT, RG, true>, dim3(grid), dim3(C::threads), C::smem, st, mk, mv, a) != cudaSuccess) return DYNAKV_ERR_CUDA;
    return tree_merge_launch(HD, C::RT, DT == DYNAKV_F32, a, grid, st);
}
template <int HD, int DT>
static int chunk_launch_rows(int rg, const CUtensorMap& mk, const CUtensorMap& mv, const TreeArgs& a, int sms, cudaStream_t st) {
    if constexpr (HD == 64) { if (rg == 4) return chunk_launch<HD, DT, 4>(mk, mv, a, sms, st); }     // rows of 128: 32 at most come here
    return rg == 0 ? chunk_launch<HD, DT, 0>(mk, mv, a, sms, st) : rg == 1 ? chunk_launch<HD, DT, 1>(mk, mv, a, sms, st) : chunk_launch<HD, DT, 2>(mk, mv, a, sms, st);
}

// From so many query rows per KV head on the kernels for many rows pay (rows of 128 elements, of 64).  In us, 8 KV heads, the kernel for few
// rows / tcgen05 (bf16, FP8) or the 128-row tiles (fp32):
//                             bf16: 32 rows  40 rows   64 rows   128 rows | FP8: 32 rows  40 rows   64 rows  128 rows | fp32: 32 rows   64 rows   128 rows
//   4 x 16384 (fp32: 4096), d = 128  66 / 70  104 / 70  105 / 71  183 / 72 |    69 / 87  112 / 87  113 / 88  197 / 89 |     151 / 191  230 / 192  401 / 195
//   16 x 2048, d = 128               38 / 46   54 / 46   57 / 46   91 / 48 |    38 / 51   55 / 52   59 / 52   99 / 54 |     249 / 334  402 / 334  756 / 339
//   1 x 1024, d = 128                20 / 22   20 / 22   21 / 22   20 / 23 |    20 / 23   21 / 24   23 / 24   22 / 24 |      37 / 49    41 / 50    62 / 52
//   4 x 16384 (fp32: 4096), d = 64   40 / 61   64 / 61   65 / 61  112 / 62 |    43 / 71   70 / 71   72 / 71  126 / 72 |      76 / 112  112 / 112  190 / 114
//   16 x 2048, d = 64                24 / 38   33 / 38   35 / 38   57 / 39 |    26 / 43   37 / 43   40 / 43   64 / 44 |     126 / 192  200 / 192  360 / 195
static int chunk_few(const dynakv_row_cache* c) { return c->head_dim == 128 ? 32 : 64; }
// From three tiles per sequence on FP8 rows are turned into bf16 first (chunk_tc.cu).  There is room for as many pages as the table can name or the cache has, in
// CHUNK_WIDE bytes at most; the plan counts how many the sequences have, and where those are more (the same page in many sequences; long caches) the rows are turned
// into bf16 as they are read.
constexpr size_t CHUNK_WIDE = (size_t)2 << 30;
struct ChunkKind { bool planned; int rg, rows, ctas, per; long long wide; };        // per: tokens of a planned tile; wide: pages turned into bf16 at most, 0: none
static ChunkKind chunk_kind(const dynakv_row_cache* c, int n_heads, int n_seqs, int max_chunk, int pages_per_seq, int sms) {
    const bool f32 = c->kv_dtype == DYNAKV_F32;
    const int most = (int)min(1000ll, (long long)max_chunk * (n_heads / c->n_kv_heads));
    if (most > chunk_few(c)) {
        const int G = n_heads / c->n_kv_heads;
        const long long table = (long long)n_seqs * pages_per_seq;
        const bool wide = c->kv_dtype == DYNAKV_FP8 && max_chunk > 2 * tile_tokens(G) && n_seqs <= 65535 && c->n_kv_heads <= 65535;
        return {true, 0, f32 ? CF_ROWS : CT_ROWS, sms, f32 ? CF_ROWS / G : tile_tokens(G), wide ? min(min(table, (long long)c->n_pages), (long long)(CHUNK_WIDE / chunk_wide_page(c))) : 0};
    }
    const int rg = row_groups(most, f32);
    return {false, rg, rg > 0 ? 16 * rg : f32 ? 4 : 8, sms * (f32 ? 1 : 2), 0, 0};
}

// Workspace: records, the plan, rows as bf16.
struct ChunkSpace { TreeSpace records; size_t wide, bytes; };
static ChunkSpace chunk_space(const dynakv_row_cache* c, const ChunkKind& k, int64_t n_tokens, int n_seqs, char* base, ChunkPlan* plan) {
    ChunkSpace s;
    s.records = tree_space(k.ctas, k.rows, c->head_dim);
    s.wide = 0;
    s.bytes = s.records.bytes;
    if (k.planned) s.bytes = chunk_plan_space(n_tokens, k.per, n_seqs, k.ctas, k.wide, s.bytes, base, plan);
    if (k.wide > 0) {
        s.wide = (s.bytes + 127) / 128 * 128;
        s.bytes = s.wide + k.wide * chunk_wide_page(c) + 128;       // the workspace itself is aligned to 16 bytes
    }
    return s;
}

// Rows of a sequence and windows up to 2^30, so that sums of two of them, and of a stage more, stay in 32 bits.
constexpr int CHUNK_COLUMNS = (1 << 30) / PAGE;

static bool chunk_shape_ok(const dynakv_row_cache* c, int n_heads, int64_t n_tokens, int n_seqs, int max_chunk, int pages_per_seq) {
    return row_cache_ok(c) && n_heads >= 1 && n_heads % c->n_kv_heads == 0 && n_heads / c->n_kv_heads <= MAX_G && max_chunk >= 1 && max_chunk <= (1 << 24) &&
           n_tokens >= 0 && n_tokens < (1ll << 31) && n_seqs >= 0 && pages_per_seq >= 0 && pages_per_seq <= CHUNK_COLUMNS;
}

}  // namespace dkv

using namespace dkv;

extern "C" int64_t dynakv_attend_chunk_workspace(const dynakv_row_cache* cache, int32_t n_heads, int64_t n_tokens, int32_t n_seqs, int32_t max_chunk,
                                                 int32_t pages_per_seq) {
    if (!chunk_shape_ok(cache, n_heads, n_tokens, n_seqs, max_chunk, pages_per_seq)) return DYNAKV_ERR_ARG;
    int rc;
    const int sms = sm_count(&rc);
    if (rc != DYNAKV_OK) return rc;
    return (int64_t)chunk_space(cache, chunk_kind(cache, n_heads, n_seqs, max_chunk, pages_per_seq, sms), n_tokens, n_seqs, nullptr, nullptr).bytes;
}

extern "C" int dynakv_attend_chunk(const dynakv_row_cache* cache, const void* q, int32_t n_heads, int64_t n_tokens, const int32_t* q_start,
                                   int32_t n_seqs, int32_t max_chunk, const int32_t* page_table, int32_t pages_per_seq, const int32_t* kv_len,
                                   const dynakv_scores* scores, void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                   uint32_t* status, void* cuda_stream) {
    if (!chunk_shape_ok(cache, n_heads, n_tokens, n_seqs, max_chunk, pages_per_seq) || !scores ||
        !(fabsf(scores->scale) <= FLT_MAX) || scores->window < 0) return DYNAKV_ERR_ARG;
    const float cap = scores->softcap;
    if (cap != 0.f && !(cap >= 0x1p-100f && cap <= 0x1p100f && fabsf(scores->scale / cap) <= FLT_MAX)) return DYNAKV_ERR_ARG;
    if (n_tokens == 0 || n_seqs == 0) return DYNAKV_OK;
    if (!q || !q_start || (!page_table && pages_per_seq > 0) || !kv_len || !out || !workspace) return DYNAKV_ERR_ARG;
    if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)workspace) & 15) return DYNAKV_ERR_ARG;
    int rc;
    const int sms = sm_count(&rc);
    if (rc != DYNAKV_OK) return rc;
    const ChunkKind kind = chunk_kind(cache, n_heads, n_seqs, max_chunk, pages_per_seq, sms);
    ChunkPlan plan = {};
    const ChunkSpace sp = chunk_space(cache, kind, n_tokens, n_seqs, reinterpret_cast<char*>(workspace), &plan);
    if (workspace_bytes < (int64_t)sp.bytes) return DYNAKV_ERR_ARG;
    TreeArgs a = tree_args(cache, q, n_heads, n_tokens, q_start, n_seqs, max_chunk, page_table, pages_per_seq, kv_len, out, lse, workspace, sp.records, status);
    a.scale = scores->scale;
    a.cap = scores->softcap;
    a.slopes = scores->slopes;
    a.window = min(scores->window, 1 << 30);
    a.rows_from = scores->rows_from; a.rows_to = scores->rows_to;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    // an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
    cudaGetLastError();
    if (kind.planned && cache->kv_dtype == DYNAKV_F32) return chunk_f32_launch(cache, a, plan, sms, st);
    if (kind.planned) {
        void* wide = reinterpret_cast<void*>(((uintptr_t)workspace + sp.wide + 127) / 128 * 128);
        return chunk_tc_launch(cache, a, plan, kind.wide > 0 ? wide : nullptr, kind.wide >= (long long)n_seqs * pages_per_seq, sms, st);
    }
    CUtensorMap mk, mv;
    if (!tree_page_map(&mk, cache, cache->k, true) || !tree_page_map(&mv, cache, cache->v, true)) return DYNAKV_ERR_CUDA;
    const int rg = kind.rg;
    if (cache->head_dim == 128) {
        if (cache->kv_dtype == DYNAKV_F32) return chunk_launch_rows<128, DYNAKV_F32>(rg, mk, mv, a, sms, st);
        if (cache->kv_dtype == DYNAKV_BF16) return chunk_launch_rows<128, DYNAKV_BF16>(rg, mk, mv, a, sms, st);
        return chunk_launch_rows<128, DYNAKV_FP8>(rg, mk, mv, a, sms, st);
    }
    if (cache->kv_dtype == DYNAKV_F32) return chunk_launch_rows<64, DYNAKV_F32>(rg, mk, mv, a, sms, st);
    if (cache->kv_dtype == DYNAKV_BF16) return chunk_launch_rows<64, DYNAKV_BF16>(rg, mk, mv, a, sms, st);
    return chunk_launch_rows<64, DYNAKV_FP8>(rg, mk, mv, a, sms, st);
}
