// Host side of dynakv_attend_tree's kernels: tensor maps of a row cache, the device's SM count, the workspace.
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

// tcgen05 kernel (tree_tc.cu): bf16 and FP8 rows, tiles of 128 or 256 query rows, one CTA per SM.
int tree_tc_launch(const dynakv_row_cache* cache, int rows, const TreeArgs& a, int sms, cudaStream_t st);
// Merge of cut units (tree_attn.cu).
int tree_merge_launch(int hd, int rt, bool f32, const TreeArgs& a, int ctas, cudaStream_t st);

}  // namespace dkv
