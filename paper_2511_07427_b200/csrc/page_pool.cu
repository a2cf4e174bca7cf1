// Pages for the rows of new tokens, and pages given back (dynakv_pages_extend, dynakv_pages_trim).
//
// Everything follows from prefix sums over the sequences: of tokens (places in the packed batch) and of pages (places on the stack of
// free ones).  A few bytes per sequence and 8 per token are all that moves, so a call is a chain of dependent steps: lengths are
// read, summed, and looked up again by every token.  One cluster of CTAs does it in one launch: each CTA reads and sums all
// lengths for itself (1024 sequences at a time), the cluster meets, which is when the old lengths may be overwritten, and the
// tokens and pages are then shared out evenly.  A token finds its sequence by bisection in shared memory.
// Measured on the device: 64 sequences of one token 5 us, 512 prompts with places for 131072 tokens 14 us; giving the pages back 4 and 7 us.  A call takes
// 5 to 12 us of host time, so that is what it costs in a stream of calls.
#include <cooperative_groups.h>

#include "common.cuh"

namespace dkv {

namespace cg = cooperative_groups;

constexpr int PP_THREADS = 1024;           // sequences summed at a time
constexpr int PP_CLUSTER = 8;              // CTAs of a large call; the portable limit

struct PoolArgs {
    int* free; int* count;                 // [n_pages] page ids, the first *count of them free
    int* table; int* len;                  // [n_seqs][per], [n_seqs]
    const int* change;                     // [n_seqs] rows to add / to drop
    int* q_start; int* positions; int* slots;
    unsigned* status;
    long long n_tokens;
    int n_pages, n_seqs, per;
};

__device__ __forceinline__ int pages_of(int rows) { return (int)(((long long)rows + PAGE - 1) / PAGE); }

struct Two { long long x, y; };
// Inclusive sums of both numbers over the block, and their totals.  sh: 64 long longs.
__device__ __forceinline__ Two block_sums(long long x, long long y, long long* sh, Two& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) { x += u; y += v; }
    }
    __syncthreads();
    if (lane == 31) { sh[warp] = x; sh[32 + warp] = y; }
    __syncthreads();
    long long a = sh[lane], b = sh[32 + lane];             // every warp sums the warps' totals
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, a, o), v = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) { a += u; b += v; }
    }
    total = {__shfl_sync(0xffffffffu, a, 31), __shfl_sync(0xffffffffu, b, 31)};
    const long long ba = __shfl_sync(0xffffffffu, a, (warp + 31) & 31), bb = __shfl_sync(0xffffffffu, b, (warp + 31) & 31);
    return {x + (warp ? ba : 0), y + (warp ? bb : 0)};
}

// Index of the last of ends[0 .. n) that is <= x: ends are non-decreasing and ends[0] <= x.
__device__ __forceinline__ int last_at_most(const int* ends, int n, int x) {
    int lo = 0;
    for (int step = PP_THREADS / 2; step > 0; step >>= 1)
        if (lo + step < n && ends[lo + step] <= x) lo += step;
    return lo;
}

// What the lengths of up to 1024 sequences come to, in shared memory: where their tokens and pages begin, their old lengths.
struct PoolShared {
    long long sums[64];
    int tokens[PP_THREADS + 1], pages[PP_THREADS + 1], old[PP_THREADS];
    int stop;                              // first sequence of the batch that is not served
};

// What one sequence asks for; y: in pages.  ok = false: out of range, left as it is.
template <bool GROW>
__device__ __forceinline__ Two asked(const PoolArgs& a, int old, int change, bool& ok) {
    const long long rows = (long long)a.per * PAGE, then = GROW ? (long long)old + change : (long long)old - change;
    ok = old >= 0 && change >= 0 && old <= rows && then >= 0 && then <= rows;
    if (!ok) return {0, 0};
    return {change, GROW ? pages_of((int)then) - pages_of(old) : pages_of(old) - pages_of((int)then)};
}

template <bool GROW>
__global__ void __launch_bounds__(PP_THREADS) k_page_pool(const PoolArgs a) {
    __shared__ PoolShared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, ctas = gridDim.x, cta = blockIdx.x;
    const bool first = cta == 0;
    pdl_wait();
    unsigned trouble = 0;
    int count = *a.count;
    if (count < 0 || count > a.n_pages) { trouble |= DYNAKV_ST_BOUNDS; count = max(0, min(count, a.n_pages)); }
    const long long room = GROW ? count : a.n_pages - count;       // pages that can change hands
    long long total = 0;                                           // trimming: pages that will, over all sequences
    int last = a.n_seqs;                                           // sequences from here on are not served
    // The sums of sequences b0 .. b0 + 1023, after `done` of those before them.
    auto sum = [&](int b0, Two done, Two& here, int& old, int& change, Two& end) {
        const int b = b0 + tid;
        bool ok = true;
        Two want = {0, 0};
        old = 0; change = 0;
        if (b < a.n_seqs) {
            old = a.len[b]; change = a.change[b];
            want = asked<GROW>(a, old, change, ok);
            if (!ok) trouble |= DYNAKV_ST_BOUNDS;
        }
        end = block_sums(want.x, want.y, sh.sums, here);
        here = {here.x + done.x, here.y + done.y};
        end = {end.x + done.x, end.y + done.y};
        // in order up to the first that finds too few pages, or too few places in the packed batch
        const bool short_pages = end.y > room, short_places = GROW && end.x > a.n_tokens;
        if (tid == 0) sh.stop = PP_THREADS;
        __syncthreads();
        if (b < a.n_seqs && (short_pages || short_places)) atomicMin(&sh.stop, tid);
        __syncthreads();
        const int stop = sh.stop;
        if (stop < PP_THREADS) {
            if (tid == stop) trouble |= short_pages ? DYNAKV_ST_PAGE_POOL : DYNAKV_ST_BOUNDS;
            if (tid == stop) { sh.sums[0] = end.x - want.x; sh.sums[1] = end.y - want.y; }
            __syncthreads();
            here = {sh.sums[0], sh.sums[1]};
            if (tid >= stop) { end = here; change = 0; }
        }
        if (!ok) change = 0;
        return stop;
    };
    if (!GROW && a.n_seqs > PP_THREADS) {                          // where the last page comes to lie depends on all
        Two done = {0, 0}, here, end;
        int old, change;
        for (int b0 = 0; b0 < a.n_seqs; b0 += PP_THREADS) {
            const int stop = sum(b0, done, here, old, change, end);
            done = here;
            if (stop < PP_THREADS) break;
        }
        total = done.y;
    }
    Two done = {0, 0};
    if (GROW && first && tid == 0) a.q_start[0] = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += PP_THREADS) {
        Two here = done, end = done;
        int old = 0, change = 0;
        if (b0 < last) {
            const int stop = sum(b0, done, here, old, change, end);
            if (stop < PP_THREADS) last = b0 + stop;
        }
        if (!GROW && a.n_seqs <= PP_THREADS) total = here.y;
        const int b = b0 + tid, n = min(PP_THREADS, a.n_seqs - b0);
        sh.tokens[tid + 1] = (int)(end.x - done.x); sh.pages[tid + 1] = (int)(end.y - done.y); sh.old[tid] = old;
        if (tid == 0) { sh.tokens[0] = 0; sh.pages[0] = 0; }
        cluster.sync();                                            // all have read the old lengths of these sequences
        if (first && b < a.n_seqs) {
            if (GROW) a.q_start[b + 1] = (int)end.x;
            if (change != 0) a.len[b] = GROW ? old + change : old - change;
        }
        if (GROW) {
            const int tokens = (int)(here.x - done.x);
            for (int i = cta * PP_THREADS + tid; i < tokens; i += ctas * PP_THREADS) {
                const int s = last_at_most(sh.tokens, n, i), was = sh.old[s], place = was + i - sh.tokens[s], column = place / PAGE;
                const int fresh = column - pages_of(was);          // number among the sequence's new pages
                const size_t cell = (size_t)(b0 + s) * a.per + column;
                const int page = fresh >= 0 ? a.free[count - 1 - (done.y + sh.pages[s] + fresh)] : a.table[cell];
                if (fresh >= 0 && place % PAGE == 0) a.table[cell] = page;
                const bool known = page >= 0 && page < a.n_pages;
                if (!known) trouble |= DYNAKV_ST_BOUNDS;
                a.positions[done.x + i] = place;
                a.slots[done.x + i] = known ? page * PAGE + place % PAGE : -1;
            }
        } else {
            const int pages = (int)(here.y - done.y);
            for (int i = cta * PP_THREADS + tid; i < pages; i += ctas * PP_THREADS) {
                const int s = last_at_most(sh.pages, n, i);
                const int column = pages_of(sh.old[s]) - (sh.pages[s + 1] - sh.pages[s]) + i - sh.pages[s];
                const size_t cell = (size_t)(b0 + s) * a.per + column;
                const int page = a.table[cell];
                if (page < 0 || page >= a.n_pages) trouble |= DYNAKV_ST_BOUNDS;
                a.free[count + total - 1 - (done.y + i)] = page;
                a.table[cell] = -1;
            }
        }
        __syncthreads();
        done = here;
    }
    if (GROW) {
        for (long long i = done.x + (long long)cta * PP_THREADS + tid; i < a.n_tokens; i += (long long)ctas * PP_THREADS) { a.positions[i] = 0; a.slots[i] = -1; }
    }
    cluster.sync();                                                // the old count has been read
    if (first && tid == 0 && done.y != 0) *a.count = GROW ? count - (int)done.y : count + (int)done.y;
    if (trouble && a.status) atomicOr(a.status, trouble);
}

template <bool GROW>
static int page_pool_launch(const PoolArgs& a, long long work, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    const int ctas = work > 4 * PP_THREADS ? PP_CLUSTER : 1;
    cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(PP_THREADS); cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    // an error left behind by an earlier, unrelated call on this thread must not be reported as this call's
    cudaGetLastError();
    return cudaLaunchKernelEx(&cfg, k_page_pool<GROW>, a) == cudaSuccess ? DYNAKV_OK : DYNAKV_ERR_CUDA;
}

static bool pool_ok(const dynakv_page_pool* p, const int* table, int per, const int* len, const int* change, int n_seqs) {
    return p && p->free_pages && p->count && p->n_pages >= 1 && p->n_pages < (1 << 26) && per >= 0 && per < (1 << 26) && n_seqs >= 0 &&
           (n_seqs == 0 || (len && change && (table || per == 0)));
}
static PoolArgs pool_args(const dynakv_page_pool* p, int* table, int per, int* len, const int* change, int n_seqs, unsigned* status) {
    PoolArgs a = {};
    a.free = p->free_pages; a.count = p->count; a.n_pages = (int)p->n_pages;
    a.table = table; a.per = per; a.len = len; a.change = change; a.n_seqs = n_seqs; a.status = status;
    return a;
}

}  // namespace dkv

using namespace dkv;

extern "C" int dynakv_pages_extend(const dynakv_page_pool* pool, int32_t* page_table, int32_t pages_per_seq, int32_t* kv_len, const int32_t* new_len,
                                   int32_t n_seqs, int64_t n_tokens, int32_t* q_start, int32_t* positions, int32_t* slots, uint32_t* status, void* cuda_stream) {
    if (!pool_ok(pool, page_table, pages_per_seq, kv_len, new_len, n_seqs) || n_tokens < 0 || n_tokens >= (1ll << 31) || !q_start ||
        (n_tokens > 0 && (!positions || !slots))) return DYNAKV_ERR_ARG;
    PoolArgs a = pool_args(pool, page_table, pages_per_seq, kv_len, new_len, n_seqs, status);
    a.q_start = q_start; a.positions = positions; a.slots = slots; a.n_tokens = n_tokens;
    return page_pool_launch<true>(a, n_tokens, reinterpret_cast<cudaStream_t>(cuda_stream));
}

extern "C" int dynakv_pages_trim(const dynakv_page_pool* pool, int32_t* page_table, int32_t pages_per_seq, int32_t* kv_len, const int32_t* drop,
                                 int32_t n_seqs, uint32_t* status, void* cuda_stream) {
    if (!pool_ok(pool, page_table, pages_per_seq, kv_len, drop, n_seqs)) return DYNAKV_ERR_ARG;
    if (n_seqs == 0) return DYNAKV_OK;
    return page_pool_launch<false>(pool_args(pool, page_table, pages_per_seq, kv_len, drop, n_seqs, status), n_seqs, reinterpret_cast<cudaStream_t>(cuda_stream));
}
