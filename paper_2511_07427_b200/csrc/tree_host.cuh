// Host side of the kernels behind dynakv_attend_tree and dynakv_attend_chunk: tensor maps of a row cache, the device's SM count, the workspace.
#pragma once

#include <cuda.h>

#include <atomic>

#include "head_rows.cuh"
#include "tree_plan.cuh"

namespace dkv {

typedef CUresult (*tree_encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// Looked up through the runtime: the library carries no link-time dependency on the driver library.
static tree_encode_fn tree_encode() {
    static std::atomic<tree_encode_fn> fn{nullptr};
    tree_encode_fn f = fn.load(std::memory_order_acquire);
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qr) == cudaSuccess && qr == cudaDriverEntryPointSuccess)
            fn.store(f = reinterpret_cast<tree_encode_fn>(p), std::memory_order_release);
        else
            cudaGetLastError();
    }
    return f;
}

// Pool [rows][HD] as [panel][row][128 bytes]: a box is one page, laid out panel by panel, or (whole_rows = false) one panel of
// one page.
static bool tree_page_map(CUtensorMap* map, const dynakv_row_cache* c, void* pool, bool whole_rows) {
    const tree_encode_fn enc = tree_encode();
    if (!enc) return false;
    const int es = c->kv_dtype == DYNAKV_F32 ? 4 : c->kv_dtype == DYNAKV_BF16 ? 2 : 1;
    const int row = c->head_dim * es, w = row < 128 ? row : 128;
    const cuuint64_t dims[3] = {(cuuint64_t)(w / es), (cuuint64_t)(c->n_pages * c->n_kv_heads * PAGE), (cuuint64_t)(row / w)};
    const cuuint64_t strides[2] = {(cuuint64_t)row, (cuuint64_t)w};
    const cuuint32_t box[3] = {(cuuint32_t)(w / es), PAGE, (cuuint32_t)(whole_rows ? row / w : 1)}, estr[3] = {1, 1, 1};
    const CUtensorMapDataType dt = es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    return enc(map, dt, 3, pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               w == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_count(int* rc) {
    constexpr int MAX_DEV = 64;
    static std::atomic<int> sms[MAX_DEV];
    int dev = -1;
    *rc = DYNAKV_ERR_CUDA;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEV) { cudaGetLastError(); return 0; }
    int n = sms[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) { cudaGetLastError(); return 0; }
        sms[dev].store(n, std::memory_order_relaxed);
    }
    *rc = DYNAKV_OK;
    return n;
}

// More than 48 KB of dynamic shared memory, asked for once per device; `done`: the kernel's own word, a bit per device.
template <typename K>
static bool allow_smem(K kernel, int bytes, std::atomic<unsigned long long>& done) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if ((done.load(std::memory_order_acquire) >> dev) & 1ull) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(1ull << dev, std::memory_order_release);
    return true;
}

// 16 rows of a tile per row group; the groups needed for all rows of a sequence in one tile, up to four (0: one of few rows)
static inline int row_groups(int max_rows, bool f32) { return max_rows <= (f32 ? 4 : 8) ? 0 : max_rows <= 16 ? 1 : max_rows <= 32 ? 2 : 4; }

struct TreeSpace { size_t acc, ml, desc, bytes; };
static inline TreeSpace tree_space(int ctas, int rt, int hd) {
    TreeSpace s;
    s.acc = 0;
    s.ml = (size_t)ctas * 2 * rt * hd * 4;
    s.desc = s.ml + (size_t)ctas * 2 * rt * 8;
    s.bytes = s.desc + (size_t)ctas * 8 * 4;
    return s;
}


static inline TreeArgs tree_args(const dynakv_row_cache* cache, const void* q, int n_heads, int64_t n_tokens, const int* q_start, int n_seqs, int max_tokens,
                                 const int* page_table, int pages_per_seq, const int* kv_len, void* out, float* lse, void* workspace, const TreeSpace& sp,
                                 unsigned* status) {
    TreeArgs a = {};
    a.q = q; a.q_start = q_start; a.page_table = page_table; a.kv_len = kv_len;
    a.out = out; a.lse = lse;
    char* ws = reinterpret_cast<char*>(workspace);
    a.acc = reinterpret_cast<float*>(ws + sp.acc);
    a.ml = reinterpret_cast<float2*>(ws + sp.ml);
    a.desc = reinterpret_cast<int*>(ws + sp.desc);
    a.status = status;
    a.kpool = reinterpret_cast<const unsigned char*>(cache->k); a.vpool = reinterpret_cast<const unsigned char*>(cache->v);
    a.kexp = reinterpret_cast<const signed char*>(cache->k_exp); a.vexp = reinterpret_cast<const signed char*>(cache->v_exp);
    a.n_tokens = n_tokens; a.n_pages = cache->n_pages;
    a.n_seqs = n_seqs; a.max_tree = max_tokens; a.pages_per_seq = pages_per_seq;
    a.G = n_heads / cache->n_kv_heads; a.Hq = n_heads; a.Hk = cache->n_kv_heads;
    return a;
}

// tcgen05 kernel (tree_tc.cu): bf16 and FP8 rows, tiles of 128 or 256 query rows, one CTA per SM.
int tree_tc_launch(const dynakv_row_cache* cache, int rows, const TreeArgs& a, int sms, cudaStream_t st);
// Merge of cut units (tree_attn.cu).
int tree_merge_launch(int hd, int rt, bool f32, const TreeArgs& a, int ctas, cudaStream_t st);

}  // namespace dkv
