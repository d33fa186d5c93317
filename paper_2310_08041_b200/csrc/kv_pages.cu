// Pages of the 4-bit key/value cache: taking, sharing, returning, moving and copying them.
//
// The pool is its reference counts: a page is free when its count is 0, and pages are taken lowest index first, so what
// a call does depends on its arguments alone.  Each call runs its bookkeeping in one CTA (a list of requests is ordered by
// prefix sums, duplicates are settled by an atomic minimum over list positions or an exchange), which costs a pass over refs; the page
// contents then move in a second kernel over (page, layer) that reads the bookkeeping's result.  Contents: 2 * page_size * kv_heads * (head_dim / 2 + 8) bytes a page and layer, read and written
// once in 16-byte accesses, four in flight per thread.  Measured: 43 pages of 32 layers (100 MB copied) 29 us, 6.9 TB/s; 1.25 GB moved
// by a compaction of 40 layers in 184 us, 6.8 TB/s; the bookkeeping 4 to 8 us.  Making room: 7 us for one more token of 64 sequences, 8
// of 512, 12 of 4096; 10 for a prompt of 2048 tokens in pages of 64, 240 for one of 131072 in pages of 16, whose 8192 counts one
// thread sets.

#include "device_utils.cuh"
#include "kv_cache.cuh"

namespace qllm {
namespace {

using kv::raise_page;

constexpr int kPoolMax = 8192;                             // sequences of a pool, entries of a list
constexpr int kThreads = 1024;
constexpr int kMaxLayers = 65534;                        // layers are a grid dimension (one more for the tables)

struct Pool {
    int32_t *refs, *table, *lens;
    int pages, seqs, width, page_log2;
};

// The four arrays of the cache, as 16-byte pieces of one page in one layer.
struct Store {
    uint4* a[4];
    int64_t n[4];                                          // pieces of a page: codes, parameters, codes, parameters
    int pages, layers;
};

// CTA-wide exclusive prefix sum of one number per thread (kThreads threads); total in *sum.
template <typename I>
__device__ __forceinline__ I block_prefix(I v, I* s_warp, I* sum) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    I x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const I y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                                       // s_warp is free again
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        I w = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const I y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    *sum = s_warp[31];
    return x - v + (warp ? s_warp[warp - 1] : I(0));
}

// Calls f(rank, page) for the free pages of ranks [0, want), in order of their index.  Whole CTA.
template <typename F>
__device__ __forceinline__ int free_pages(const Pool& p, int want, int* s_warp, F f) {
    int seen = 0;
    for (int base = 0; base < p.pages && seen < want; base += 4 * kThreads) {
        int at[4], k = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = base + 4 * int(threadIdx.x) + i;
            at[i] = page < p.pages && p.refs[page] == 0;
            k += at[i];
        }
        int total, r = seen + block_prefix(k, s_warp, &total);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at[i]) {
                if (r < want) f(r, base + 4 * int(threadIdx.x) + i);
                ++r;
            }
        seen += total;
    }
    __syncthreads();
    return seen < want ? seen : want;
}

// ---- extend: seq_lens += add ---------------------------------------------------------------------------------------
// Pages of sequence s now and with add[s] more tokens; false when the request can never be served.
__device__ __forceinline__ bool extend_need(const Pool& p, const int32_t* add, int s, int& have, int& need) {
    const int64_t len = p.lens[s], more = add[s], P = int64_t(1) << p.page_log2;
    const int64_t h = (len + P - 1) >> p.page_log2, w = (len + more + P - 1) >> p.page_log2;
    if (len < 0 || more < 0 || len + more > 0x7fffffff || w > p.width || w - h > p.pages) return false;
    have = int(h);
    need = int(w - h);
    return true;
}

__global__ void __launch_bounds__(kThreads) kv_extend_kernel(Pool p, const int32_t* __restrict__ add, int* status) {
    __shared__ int64_t s_warp64[32];
    __shared__ int s_warp[32], s_at[kPoolMax + 1];          // pages asked for by the sequences in front
    constexpr int64_t kTop = 0x3fffffff;                   // more than there can be
    int64_t asked = 0;
    for (int base = 0; base < p.seqs; base += kThreads) {
        const int s = base + threadIdx.x;
        int have = 0, need = 0;
        if (s < p.seqs && !extend_need(p, add, s, have, need)) {
            need = 0;
            raise_page(status);
        }
        int64_t total;
        const int64_t before = asked + block_prefix<int64_t>(need, s_warp64, &total);
        if (s < p.seqs) s_at[s] = int(before < kTop ? before : kTop);
        asked += total;
    }
    const int want = int(asked < kTop ? asked : kTop);
    if (threadIdx.x == 0) s_at[p.seqs] = want;
    __syncthreads();
    // the r-th free page is shown to the sequence whose range of requests holds r
    const int got = free_pages(p, want, s_warp, [&](int r, int page) {
        int lo = 0, hi = p.seqs;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_at[mid + 1] <= r) lo = mid + 1; else hi = mid;
        }
        int have = 0, need = 0;
        if (extend_need(p, add, lo, have, need)) p.table[int64_t(lo) * p.width + have + (r - s_at[lo])] = page;
    });
    for (int s = threadIdx.x; s < p.seqs; s += kThreads) {
        int have, need;
        if (!extend_need(p, add, s, have, need)) continue;
        int32_t* row = p.table + int64_t(s) * p.width + have;
        if (need == 0 || s_at[s + 1] <= got) {
            for (int j = 0; j < need; ++j) p.refs[row[j]] = 1;
            p.lens[s] += add[s];
        } else {                                           // not served: the pages it was shown stay free
            for (int j = 0; j < need && s_at[s] + j < got; ++j) row[j] = -1;
            raise_page(status);
        }
    }
}

// ---- fork ----------------------------------------------------------------------------------------------------------
// An entry is served when its indices exist, its child is unused, not named earlier in the list and no parent of it, and its parent's
// pages exist.
__global__ void __launch_bounds__(kThreads)
kv_fork_kernel(Pool p, const int32_t* __restrict__ parent, const int32_t* __restrict__ child, int n, int32_t* __restrict__ fresh,
               int* status) {
    extern __shared__ int s_dyn[];
    int* s_first = s_dyn;                                  // [seqs] first entry that names the sequence as a child, or one of:
    constexpr int kNobody = 0x7fffffff, kParent = 0x7ffffffe, kBroken = 0x7ffffffd;      // no child; a parent; one that cannot be copied
    int* s_rank = s_dyn + p.seqs;                          // [n] the parents, then pages asked for by the entries in front; -1: not served
    __shared__ int s_warp[32];
    const int P = 1 << p.page_log2;
    for (int s = threadIdx.x; s < p.seqs; s += kThreads) s_first[s] = kNobody;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int early = warp + 32 * lane < p.seqs ? p.lens[warp + 32 * lane] : 0;      // under the loads below
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int c = child[i];
        s_rank[i] = parent[i];
        if (c >= 0 && c < p.seqs) atomicMin(&s_first[c], i);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int a = s_rank[i];
        if (a >= 0 && a < p.seqs && s_first[a] >= kParent) s_first[a] = kParent;
    }
    __syncthreads();
    // each parent's pages are looked at once, however many children it gets (7000 entries of 1000 parents: entry by entry 376 us), and
    // neighbours by different warps
    for (int base = warp; base < p.seqs; base += kThreads) {
        const int mine = base + 32 * lane;
        const bool marked = mine < p.seqs && s_first[mine] == kParent;
        const int length = base == warp ? early : marked ? p.lens[mine] : 0;
        for (unsigned left = __ballot_sync(0xffffffffu, marked); left; left &= left - 1) {
            const int l = __ffs(left) - 1, s = base + 32 * l, len = __shfl_sync(0xffffffffu, length, l);
            bool ok = len >= 0 && int64_t(len) <= int64_t(p.width) << p.page_log2;
            const int used = ok ? int((int64_t(len) + P - 1) >> p.page_log2) : 0;
            for (int j = lane; j < used; j += 32) {
                const int page = p.table[int64_t(s) * p.width + j];
                ok &= page >= 0 && page < p.pages;
            }
            if (!__all_sync(0xffffffffu, ok) && lane == 0) s_first[s] = kBroken;
        }
    }
    __syncthreads();
    int asked = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + threadIdx.x;
        int need = 0, ok = 0;
        if (i < n) {
            const int a = s_rank[i], c = child[i];
            ok = a >= 0 && a < p.seqs && c >= 0 && c < p.seqs && s_first[c] == i && s_first[a] == kParent && p.lens[c] == 0;
            need = ok && (p.lens[a] & (P - 1)) != 0;
            if (!ok) raise_page(status);
        }
        int total;
        const int before = asked + block_prefix(need, s_warp, &total);
        if (i < n) s_rank[i] = ok ? (need ? before : 0x40000000) : -1;
        asked += total;
    }
    __syncthreads();
    int* s_page = s_dyn + p.seqs + n;                      // [asked] the page of rank r
    const int got = free_pages(p, asked, s_warp, [&](int r, int page) { s_page[r] = page; });
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (s_rank[i] >= 0 && s_rank[i] != 0x40000000) {
            if (s_rank[i] < got) p.refs[s_page[s_rank[i]]] = 1;
            else { s_rank[i] = -1; raise_page(status); }
        }
    __syncthreads();
    for (int i = warp; i < n; i += kThreads / 32) {
        const int r = s_rank[i];
        if (lane == 0) fresh[i] = r < 0 ? -2 : (r == 0x40000000 ? -1 : s_page[r]);
        if (r < 0) continue;
        const int a = parent[i], c = child[i], len = p.lens[a], full = len >> p.page_log2;
        const int32_t* from = p.table + int64_t(a) * p.width;
        int32_t* to = p.table + int64_t(c) * p.width;
        for (int j = lane; j < full; j += 32) {
            const int page = from[j];
            to[j] = page;
            if (page >= 0 && page < p.pages) atomicAdd(&p.refs[page], 1);    // (looked at above; a table that changes meanwhile faults nothing)
        }
        if (lane == 0) {
            if (len & (P - 1)) to[full] = s_page[r];
            p.lens[c] = len;
        }
    }
}

// ---- free ----------------------------------------------------------------------------------------------------------
// A CTA per entry.  Each table entry is taken by an exchange, so of two equal list entries exactly one returns a page.
__global__ void __launch_bounds__(256) kv_free_kernel(Pool p, const int32_t* __restrict__ seqs, int* status) {
    const int s = seqs[blockIdx.x];
    if (s < 0 || s >= p.seqs) {
        if (threadIdx.x == 0) raise_page(status);
        return;
    }
    int32_t* row = p.table + int64_t(s) * p.width;
    for (int j = threadIdx.x; j < p.width; j += blockDim.x) {
        if (row[j] == -1) continue;
        const int page = atomicExch(&row[j], -1);
        if (page >= 0 && page < p.pages) atomicSub(&p.refs[page], 1);
        else if (page != -1) raise_page(status);
    }
    if (threadIdx.x == 0) p.lens[s] = 0;
}

// ---- copies --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void copy_page(const Store& s, int src, int dst, int layer) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint4* from = s.a[k] + (int64_t(layer) * s.pages + src) * s.n[k];
        uint4* to = s.a[k] + (int64_t(layer) * s.pages + dst) * s.n[k];
        const int64_t step = blockDim.x;
        for (int64_t i = threadIdx.x; i < s.n[k]; i += 4 * step) {
            uint4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j * step < s.n[k]) v[j] = from[i + j * step];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j * step < s.n[k]) to[i + j * step] = v[j];
        }
    }
}

// blockIdx.x = entry, blockIdx.y = layer
__global__ void __launch_bounds__(256)
kv_copy_kernel(Store st, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int* status) {
    const int a = src[blockIdx.x], b = dst[blockIdx.x];
    if (a < 0 || a >= st.pages || b < 0 || b >= st.pages) {
        if (threadIdx.x == 0) raise_page(status);
        return;
    }
    if (a != b) copy_page(st, a, b, blockIdx.y);
}

// The last pages of forked sequences: the parent's partly filled one into the fresh one of entry i's child.
__global__ void __launch_bounds__(256)
kv_fork_copy_kernel(Store st, Pool p, const int32_t* __restrict__ parent, const int32_t* __restrict__ fresh) {
    const int to = fresh[blockIdx.x];
    if (to < 0) return;                                    // nothing to copy, or the entry was not served
    const int a = parent[blockIdx.x];
    const int from = p.table[int64_t(a) * p.width + (p.lens[a] >> p.page_log2)];
    if (from >= 0 && from < st.pages) copy_page(st, from, to, blockIdx.y);
}

// ---- compact -------------------------------------------------------------------------------------------------------
// remap: a used page below the number of used pages stays; the k-th used page behind it takes the k-th hole.
__global__ void __launch_bounds__(kThreads) kv_compact_plan_kernel(Pool p, int32_t* __restrict__ remap) {
    __shared__ int s_warp[32];
    int used = 0;
    for (int base = 0; base < p.pages; base += kThreads) {
        const int i = base + threadIdx.x;
        used += __syncthreads_count(i < p.pages && p.refs[i] > 0);
    }
    // holes go, in order, to the end of remap (entries >= used, where the pages that move are found next)
    int holes = 0;
    for (int base = 0; base < used; base += kThreads) {
        const int i = base + threadIdx.x;
        const bool hole = i < used && p.refs[i] <= 0;
        int total;
        const int r = holes + block_prefix(int(hole), s_warp, &total);
        if (i < used) remap[i] = hole ? -1 : i;
        if (hole) remap[used + r] = i;                     // there are at most pages - used holes
        holes += total;
    }
    __syncthreads();
    // the k-th used page behind `used` reads hole k from entry used + k, which lies at or in front of its own entry: taken
    // from the back, an entry is overwritten only after everything that lies behind it has been read
    int behind = 0;                                        // used pages behind the chunk
    const int chunks = (p.pages - used + kThreads - 1) / kThreads;
    for (int ch = chunks - 1; ch >= 0; --ch) {
        const int i = used + ch * kThreads + threadIdx.x;
        const bool live = i < p.pages && p.refs[i] > 0;
        int total;
        const int before = block_prefix(int(live), s_warp, &total);
        const int to = live ? remap[used + holes - behind - total + before] : -1;
        __syncthreads();
        if (i < p.pages) remap[i] = to;
        __syncthreads();
        behind += total;
    }
}

// blockIdx.y < layers: the contents of that layer's pages; blockIdx.y = layers: the new names in table and refs.
__global__ void __launch_bounds__(256) kv_compact_move_kernel(Store st, Pool p, const int32_t* __restrict__ remap, int* status) {
    if (int(blockIdx.y) < st.layers) {
        for (int page = blockIdx.x; page < st.pages; page += gridDim.x) {
            const int to = remap[page];
            if (to >= 0 && to != page) copy_page(st, page, to, blockIdx.y);
        }
        return;
    }
    const int64_t n = int64_t(p.seqs) * p.width, step = int64_t(gridDim.x) * blockDim.x;
    const int64_t first = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
    for (int64_t i = first; i < n; i += step) {
        const int page = p.table[i];
        if (page == -1) continue;
        if (page >= 0 && page < p.pages && remap[page] >= 0) p.table[i] = remap[page];
        else raise_page(status);
    }
    // counts follow their page: a page that moves lands on a hole, whose count is 0 and which no other page moves to
    for (int64_t i = first; i < p.pages; i += step) {
        const int to = remap[i];
        if (to >= 0 && to != i) {
            p.refs[to] = p.refs[i];
            p.refs[i] = 0;
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
Store store_of(const qllm_kv_cache_t* c) {
    Store s;
    const int64_t rows = int64_t(c->kv_heads) * c->page_size;
    s.a[0] = reinterpret_cast<uint4*>(c->k_codes); s.a[1] = reinterpret_cast<uint4*>(c->k_param);
    s.a[2] = reinterpret_cast<uint4*>(c->v_codes); s.a[3] = reinterpret_cast<uint4*>(c->v_param);
    s.n[0] = s.n[2] = rows * (c->head_dim / 2) / 16;
    s.n[1] = s.n[3] = rows * 8 / 16;
    s.pages = c->pages;
    s.layers = c->layers;
    return s;
}
int check_pool(const qllm_kv_pool_t* p) {
    if (!p) return QLLM_ERR_NULL;
    if (p->pages <= 0 || p->seqs <= 0 || p->table_width <= 0) return QLLM_ERR_SHAPE;
    if (p->seqs > kPoolMax || p->table_width > (1 << 23) || p->pages > (1 << 29)) return QLLM_ERR_UNSUPPORTED;
    if (!p->refs || !p->table || !p->seq_lens) return QLLM_ERR_NULL;
    return QLLM_OK;
}
int check_both(const qllm_kv_cache_t* c, const qllm_kv_pool_t* p) {
    int rc = kv::check_cache(c);
    if (rc == QLLM_OK) rc = check_pool(p);
    if (rc != QLLM_OK) return rc;
    if (c->pages != p->pages) return QLLM_ERR_SHAPE;
    if (int64_t(p->table_width) * c->page_size > (int64_t(1) << 30)) return QLLM_ERR_UNSUPPORTED;
    return c->layers > kMaxLayers ? QLLM_ERR_UNSUPPORTED : QLLM_OK;
}
Pool pool_of(const qllm_kv_pool_t* p, int log2) {
    return Pool{p->refs, p->table, p->seq_lens, p->pages, p->seqs, p->table_width, log2};
}

}  // namespace
}  // namespace qllm

extern "C" int qllm_kv_pages_extend(const qllm_kv_cache_t* cache, const qllm_kv_pool_t* pool, const int32_t* add, void* stream) {
    using namespace qllm;
    const int rc = check_both(cache, pool);
    if (rc != QLLM_OK) return rc;
    if (!add) return QLLM_ERR_NULL;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    kv_extend_kernel<<<1, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(pool_of(pool, kv::page_log2(cache->page_size)), add, status);
    return after_launch();
}

extern "C" int qllm_kv_pages_fork(const qllm_kv_cache_t* cache, const qllm_kv_pool_t* pool, const int32_t* parent,
                                  const int32_t* child, int n, int32_t* fresh, void* stream) {
    using namespace qllm;
    const int rc = check_both(cache, pool);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (n > kPoolMax) return QLLM_ERR_UNSUPPORTED;
    if (n == 0) return QLLM_OK;
    if (!parent || !child || !fresh) return QLLM_ERR_NULL;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Pool p = pool_of(pool, kv::page_log2(cache->page_size));
    const size_t smem = (size_t(pool->seqs) + 2 * size_t(n)) * 4;
    QLLM_CUDA_TRY(allow_smem<&kv_fork_kernel>(3 * kPoolMax * 4));
    kv_fork_kernel<<<1, kThreads, smem, st>>>(p, parent, child, n, fresh, status);
    const int rc1 = after_launch();
    if (rc1 != QLLM_OK) return rc1;
    kv_fork_copy_kernel<<<dim3(n, cache->layers), 256, 0, st>>>(store_of(cache), p, parent, fresh);
    return after_launch();
}

extern "C" int qllm_kv_pages_free(const qllm_kv_pool_t* pool, const int32_t* seqs, int n, void* stream) {
    using namespace qllm;
    const int rc = check_pool(pool);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (n > kPoolMax) return QLLM_ERR_UNSUPPORTED;
    if (n == 0) return QLLM_OK;
    if (!seqs) return QLLM_ERR_NULL;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    kv_free_kernel<<<n, 256, 0, static_cast<cudaStream_t>(stream)>>>(pool_of(pool, 0), seqs, status);
    return after_launch();
}

extern "C" int qllm_kv_pages_compact(const qllm_kv_cache_t* cache, const qllm_kv_pool_t* pool, int32_t* remap, void* stream) {
    using namespace qllm;
    const int rc = check_both(cache, pool);
    if (rc != QLLM_OK) return rc;
    if (!remap) return QLLM_ERR_NULL;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Pool p = pool_of(pool, kv::page_log2(cache->page_size));
    kv_compact_plan_kernel<<<1, kThreads, 0, st>>>(p, remap);
    const int rc1 = after_launch();
    if (rc1 != QLLM_OK) return rc1;
    const int x = cache->pages < 1024 ? cache->pages : 1024;
    kv_compact_move_kernel<<<dim3(x, cache->layers + 1), 256, 0, st>>>(store_of(cache), p, remap, status);
    return after_launch();
}

extern "C" int qllm_kv_pages_copy(const qllm_kv_cache_t* cache, const int32_t* src, const int32_t* dst, int n, void* stream) {
    using namespace qllm;
    const int rc = kv::check_cache(cache);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (cache->layers > kMaxLayers) return QLLM_ERR_UNSUPPORTED;
    if (n == 0) return QLLM_OK;
    if (!src || !dst) return QLLM_ERR_NULL;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    kv_copy_kernel<<<dim3(n, cache->layers), 256, 0, static_cast<cudaStream_t>(stream)>>>(store_of(cache), src, dst, status);
    return after_launch();
}
