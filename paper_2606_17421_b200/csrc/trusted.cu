// The trusted half: its context, and the pages of the 4-bit cache (growing, forking, freeing, compacting).
#include <new>

#include "bf_trusted.h"

using namespace bft;

static constexpr size_t HEAD_BYTES = 256 + ARRIVALS * sizeof(unsigned);

extern "C" int bf_trusted_create(bf_trusted** out, uint64_t workspace_bytes, void* cuda_stream) {
    if (!out) return BF_ERR_INVALID_ARG;
    *out = nullptr;
    if (workspace_bytes == 0) workspace_bytes = 32ull << 20;
    if (workspace_bytes < (1ull << 20) || workspace_bytes > (1ull << 40)) return BF_ERR_INVALID_ARG;
    bf_trusted* t = new (std::nothrow) bf_trusted();
    if (!t) return BF_ERR_OOM;
    t->stream = static_cast<cudaStream_t>(cuda_stream);
    t->ws_bytes = workspace_bytes;
    auto fail = [&](int code) {
        cudaGetLastError();
        cudaFree(t->base);
        delete t;
        return code;
    };
    if (cudaGetDevice(&t->device) != cudaSuccess) return fail(BF_ERR_CUDA);
    if (cudaDeviceGetAttribute(&t->n_sm, cudaDevAttrMultiProcessorCount, t->device) != cudaSuccess) return fail(BF_ERR_CUDA);
    cudaError_t e = cudaMalloc(&t->base, HEAD_BYTES + workspace_bytes);
    if (e != cudaSuccess) return fail(e == cudaErrorMemoryAllocation ? BF_ERR_OOM : BF_ERR_CUDA);
    t->status = reinterpret_cast<int*>(t->base);
    t->arrivals = reinterpret_cast<unsigned*>(t->base + 256);
    t->ws = t->base + HEAD_BYTES;
    if (cudaMemset(t->base, 0, HEAD_BYTES) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) return fail(BF_ERR_CUDA);
    *out = t;
    return BF_OK;
}

extern "C" void bf_trusted_destroy(bf_trusted* t) {
    if (!t) return;
    {
        OnDevice on(t->device);
        cudaStreamSynchronize(t->stream);
        cudaFree(t->base);
        cudaGetLastError();
    }
    delete t;
}

extern "C" const char* bf_trusted_last_cuda_error(const bf_trusted* t) { return t ? t->cuda_msg : ""; }

extern "C" int bf_trusted_status(bf_trusted* t) {
    if (!t) return BF_ERR_INVALID_ARG;
    OnDevice on(t->device);
    if (!on.ok) return cuda_failed(t, "cudaSetDevice", cudaErrorInvalidDevice);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(t->stream, &cap);
    if (e != cudaSuccess) return cuda_failed(t, "cudaStreamIsCapturing", e);
    if (cap != cudaStreamCaptureStatusNone) return BF_ERR_INVALID_ARG;
    int found = 0;
    e = cudaMemcpyAsync(&found, t->status, sizeof(int), cudaMemcpyDeviceToHost, t->stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(t->status, 0, sizeof(int), t->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(t->stream);
    if (e != cudaSuccess) return cuda_failed(t, "bf_trusted_status", e);
    return found & ST_TIMEOUT ? BF_ERR_TIMEOUT : found & ST_RANGE ? BF_ERR_RANGE : found & ST_OOM ? BF_ERR_OOM : BF_OK;
}

extern "C" uint64_t bf_kv4_block_bytes(uint32_t head_dim, uint32_t group, uint32_t page_tokens) {
    if (head_dim != 64 && head_dim != 128) return 0;
    if ((group != 32 && group != 64 && group != 128) || group > head_dim) return 0;
    if (page_tokens < 16 || page_tokens > 256 || page_tokens % 16) return 0;
    return (uint64_t)(16 * head_dim + 128 * (head_dim / group)) * (page_tokens / 16);
}

int bft::cache_check(const bf_kv4_cache* c, Cache* out) {
    if (!c || !c->pool || !c->tables || !c->lengths || !c->refs) return BF_ERR_INVALID_ARG;
    if (!c->n_layers || !c->n_pages || !c->n_kv_heads || !c->n_seqs || !c->max_pages) return BF_ERR_INVALID_ARG;
    if ((uintptr_t)c->pool % 16 || (uintptr_t)c->tables % 4 || (uintptr_t)c->lengths % 4 || (uintptr_t)c->refs % 4) return BF_ERR_INVALID_ARG;
    const uint64_t block = bf_kv4_block_bytes(c->head_dim, c->group, c->page_tokens);
    if (!block) return BF_ERR_SHAPE;
    // positions, pages and table entries are counted in 31 bits
    if ((uint64_t)c->max_pages * c->page_tokens >= (1ull << 31) - 512 || c->n_pages >= (1u << 31) || c->n_seqs >= (1u << 31) ||
        c->n_kv_heads > 1024 || c->n_layers > (1u << 16) || (uint64_t)c->n_seqs * c->max_pages >= (1ull << 40)) return BF_ERR_SHAPE;
    const unsigned __int128 bytes = (unsigned __int128)c->n_pages * c->n_kv_heads * block * c->n_layers;
    if (bytes >> 48 || bytes / c->n_layers >= ((unsigned __int128)1 << 36)) return BF_ERR_SHAPE;    // (a layer's bytes / 16 are counted in 32 bits)
    out->pool = static_cast<unsigned char*>(c->pool);
    out->tables = c->tables;
    out->lengths = c->lengths;
    out->refs = c->refs;
    out->n_layers = c->n_layers;
    out->n_pages = c->n_pages;
    out->heads = c->n_kv_heads;
    out->page_tokens = c->page_tokens;
    out->n_seqs = c->n_seqs;
    out->max_pages = c->max_pages;
    out->sub_bytes = 16 * c->head_dim + 128 * (c->head_dim / c->group);
    out->block_bytes = (unsigned)block;
    out->layer_bytes = (size_t)c->n_pages * c->n_kv_heads * block;
    return BF_OK;
}

// ------------------------------------------------------------------------------------------------
// Handing out pages.  One block decides for the whole list (its work is a scan of the reference counts, a few
// microseconds up to tens of thousands of pages), so that which page goes where depends on the list alone.
namespace {

constexpr unsigned ONE = 1024;                  // threads of a kernel that is one block

// exclusive sum over the ONE threads of a block
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* warp_sums, unsigned long long& total) {
    const unsigned lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    unsigned long long inc = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(~0u, inc, d);
        if (lane >= d) inc += o;
    }
    __syncthreads();
    if (lane == 31) warp_sums[w] = inc;
    __syncthreads();
    unsigned long long s = warp_sums[lane], sum = s;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(~0u, sum, d);
        if (lane >= d) sum += o;
    }
    total = __shfl_sync(~0u, sum, 31);
    return __shfl_sync(~0u, sum - s, w) + inc - v;
}

struct HandOut {
    Cache c;
    const int* seqs;      // grow: sequences; fork: parents
    const int* other;     // grow: counts or null; fork: children
    unsigned n;
    int fork;
    int* owner;           // [n_seqs]
    int* off;             // [n] first of a sequence's new pages in `page`, or a mark
    int* page;            // [n_pages] pages handed out
    int* status;
};
constexpr int OFF_REFUSED = -1;

__device__ __forceinline__ int pages_of(int tokens, unsigned page_tokens) { return (int)((tokens + page_tokens - 1) / page_tokens); }

__global__ void __launch_bounds__(ONE) hand_out_kernel(HandOut h) {
    __shared__ unsigned long long sums[32];
    const Cache& c = h.c;
    const int most = (int)(c.max_pages * c.page_tokens);
    // whom a name belongs to: the first in the list
    for (unsigned i = threadIdx.x; i < h.n; i += ONE) {
        const int a = h.seqs ? h.seqs[i] : (int)i;
        if (a >= 0 && a < (int)c.n_seqs) h.owner[a] = 0x7fffffff;
        if (h.fork) {
            const int b = h.other[i];
            if (b >= 0 && b < (int)c.n_seqs) h.owner[b] = 0x7fffffff;
        }
    }
    __syncthreads();
    for (unsigned i = threadIdx.x; i < h.n; i += ONE) {
        const int a = h.fork ? h.other[i] : h.seqs ? h.seqs[i] : (int)i;
        if (a >= 0 && a < (int)c.n_seqs) atomicMin(&h.owner[a], (int)i);
    }
    __syncthreads();
    unsigned long long wanted = 0, total;
    for (unsigned i0 = 0; i0 < h.n; i0 += ONE) {
        const unsigned i = i0 + threadIdx.x;
        unsigned need = 0;
        bool ok = false;
        if (i < h.n) {
            const int a = h.seqs ? h.seqs[i] : (int)i;
            ok = a >= 0 && a < (int)c.n_seqs;
            const int len = ok ? c.lengths[a] : 0;
            ok = ok && len >= 0 && len <= most;
            if (h.fork) {
                const int b = h.other[i];
                ok = ok && b >= 0 && b < (int)c.n_seqs && h.owner[b] == (int)i && h.owner[a] == 0x7fffffff && c.lengths[b] == 0;
                if (ok) need = len % c.page_tokens ? 1 : 0;
            } else {
                const int more = h.other ? h.other[i] : 1;
                ok = ok && h.owner[a] == (int)i && more >= 0 && more <= most - len;
                if (ok) need = pages_of(len + more, c.page_tokens) - pages_of(len, c.page_tokens);
            }
            if (!ok) atomicOr(h.status, ST_RANGE);
        }
        const unsigned long long at = wanted + block_scan(need, sums, total);
        if (i < h.n) h.off[i] = ok ? (int)min(at, 0x7ffffffeull) : OFF_REFUSED;    // (as high: behind every page there is)
        wanted += total;
    }
    unsigned long long found = 0;
    for (unsigned p0 = 0; p0 < c.n_pages && found < wanted; p0 += ONE) {
        const unsigned p = p0 + threadIdx.x;
        const bool is_free = p < c.n_pages && c.refs[p] == 0;
        const unsigned long long r = found + block_scan(is_free, sums, total);
        if (is_free) h.page[r] = (int)p;
        found += total;
    }
    __syncthreads();
    // (each entry of the list is read and written by the one warp that serves it)
    const unsigned lane = threadIdx.x & 31;
    for (unsigned i = threadIdx.x >> 5; i < h.n; i += ONE / 32) {
        const int at = h.off[i];
        if (at == OFF_REFUSED) continue;
        const int a = h.seqs ? h.seqs[i] : (int)i;
        const int len = c.lengths[a];
        const int more = h.fork ? 0 : h.other ? h.other[i] : 1;
        const int have = pages_of(len, c.page_tokens);
        const unsigned need = h.fork ? (len % c.page_tokens ? 1 : 0) : pages_of(len + more, c.page_tokens) - have;
        __syncwarp();
        if (need && (unsigned long long)at + need > found) {
            if (lane == 0) {
                atomicOr(h.status, ST_OOM);
                h.off[i] = OFF_REFUSED;
            }
            continue;
        }
        for (unsigned k = lane; k < need; k += 32) {
            const int p = h.page[at + k];
            c.refs[p] = 1;
            if (!h.fork) c.tables[(size_t)a * c.max_pages + have + k] = p;
        }
        if (!h.fork && lane == 0) c.lengths[a] = len + more;
    }
}

// ------------------------------------------------------------------------------------------------
// Copies of pages: bound by HBM, 16 bytes a lane, COPY_CHUNK bytes a block so that many are in flight.
constexpr unsigned COPY_THREADS = 256, COPY_CHUNK = 32768;

__device__ __forceinline__ void copy_chunk(const unsigned char* from, unsigned char* to, unsigned bytes) {
    const uint4* a = reinterpret_cast<const uint4*>(from);
    uint4* b = reinterpret_cast<uint4*>(to);
    const unsigned n = bytes / 16;
    unsigned i = threadIdx.x;
    for (; i + 7 * COPY_THREADS < n; i += 8 * COPY_THREADS) {
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __ldcs(a + i + k * COPY_THREADS);
#pragma unroll
        for (int k = 0; k < 8; ++k) __stcs(b + i + k * COPY_THREADS, v[k]);
    }
    for (; i < n; i += COPY_THREADS) __stcs(b + i, __ldcs(a + i));
}

// block (part, i): child i's table and counts (part 0), and its share of the last page's copy in every layer
__global__ void __launch_bounds__(COPY_THREADS) fork_kernel(HandOut h, unsigned parts_per_layer) {
    const Cache& c = h.c;
    const unsigned i = blockIdx.y;
    const int at = h.off[i];
    if (at == OFF_REFUSED) return;
    const int a = h.seqs[i], b = h.other[i];
    const int len = c.lengths[a];
    const unsigned full = len / c.page_tokens;
    const int* src = c.tables + (size_t)a * c.max_pages;
    if (blockIdx.x == 0) {
        int* dst = c.tables + (size_t)b * c.max_pages;
        for (unsigned k = threadIdx.x; k < c.max_pages; k += COPY_THREADS) {
            int p = -1;
            if (k < full) {
                p = src[k];
                if (p >= 0 && p < (int)c.n_pages) atomicAdd(&c.refs[p], 1);
                else {
                    p = -1;
                    atomicOr(h.status, ST_RANGE);
                }
            } else if (k == full && len % c.page_tokens) {
                p = h.page[at];
            }
            dst[k] = p;
        }
        if (threadIdx.x == 0) c.lengths[b] = len;
    }
    if (len % c.page_tokens == 0) return;
    const int from = src[full], to = h.page[at];
    if (from < 0 || from >= (int)c.n_pages) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(h.status, ST_RANGE);
        return;
    }
    const size_t page_bytes = (size_t)c.heads * c.block_bytes;
    const unsigned layer = blockIdx.x / parts_per_layer;
    const size_t o = (size_t)(blockIdx.x % parts_per_layer) * COPY_CHUNK;
    unsigned char* base = c.pool + layer * c.layer_bytes + o;
    copy_chunk(base + from * page_bytes, base + to * page_bytes, (unsigned)min(page_bytes - o, (size_t)COPY_CHUNK));
}

__global__ void __launch_bounds__(COPY_THREADS) free_kernel(Cache c, const int* seqs, int* status) {
    __shared__ int claimed;
    const int a = seqs[blockIdx.x];
    if (a < 0 || a >= (int)c.n_seqs) {
        if (threadIdx.x == 0) atomicOr(status, ST_RANGE);
        return;
    }
    if (threadIdx.x == 0) {
        const int len = *static_cast<volatile int*>(c.lengths + a);
        claimed = 0;
        if (len < 0 || len > (int)(c.max_pages * c.page_tokens)) atomicOr(status, ST_RANGE);
        else if (atomicCAS(&c.lengths[a], len, 0) == len) claimed = len;     // one block takes the sequence, others find it empty
    }
    __syncthreads();
    const int len = claimed;
    int* table = c.tables + (size_t)a * c.max_pages;
    for (int k = threadIdx.x; k < pages_of(len, c.page_tokens); k += COPY_THREADS) {
        const int p = table[k];
        table[k] = -1;
        if (p < 0 || p >= (int)c.n_pages) atomicOr(status, ST_RANGE);
        else if (atomicSub(&c.refs[p], 1) <= 0) {
            atomicAdd(&c.refs[p], 1);
            atomicOr(status, ST_RANGE);
        }
    }
}

// ------------------------------------------------------------------------------------------------
struct Compact {
    Cache c;
    int *tables_out, *refs_out, *n_live_out;
    int *holes, *movers, *to;     // [n_pages] each; to[p]: where page p goes, -1 if it is free
    int* counts;                  // n_live, movers
    int* status;
};

__global__ void __launch_bounds__(ONE) compact_plan_kernel(Compact h) {
    __shared__ unsigned long long sums[32];
    const Cache& c = h.c;
    unsigned long long live = 0, n_live, t1, t2;
    for (unsigned p = threadIdx.x; p < c.n_pages; p += ONE) live += c.refs[p] > 0;
    block_scan(live, sums, n_live);
    unsigned long long holes = 0, movers = 0;
    for (unsigned p0 = 0; p0 < c.n_pages; p0 += ONE) {
        const unsigned p = p0 + threadIdx.x;
        const bool is_live = p < c.n_pages && c.refs[p] > 0;
        const bool hole = p < n_live && !is_live, mover = p >= n_live && is_live;
        const unsigned long long a = block_scan(hole, sums, t1), b = block_scan(mover, sums, t2);
        if (hole) h.holes[holes + a] = (int)p;
        if (mover) h.movers[movers + b] = (int)p;
        if (p < c.n_pages) h.to[p] = is_live && !mover ? (int)p : -1;
        holes += t1;
        movers += t2;
    }
    __syncthreads();
    for (unsigned k = threadIdx.x; k < movers; k += ONE) h.to[h.movers[k]] = h.holes[k];
    if (threadIdx.x == 0) {
        h.counts[0] = (int)n_live;
        h.counts[1] = (int)movers;
        if (h.n_live_out) *h.n_live_out = (int)n_live;
    }
}

__global__ void __launch_bounds__(COPY_THREADS) compact_move_kernel(Compact h, unsigned parts_per_layer) {
    const Cache& c = h.c;
    const int n_live = h.counts[0];
    const unsigned movers = h.counts[1];
    const size_t page_bytes = (size_t)c.heads * c.block_bytes;
    const size_t per_page = (size_t)c.n_layers * parts_per_layer;
    for (size_t u = blockIdx.x; u < movers * per_page; u += gridDim.x) {
        const unsigned k = (unsigned)(u / per_page), rest = (unsigned)(u % per_page);
        const unsigned layer = rest / parts_per_layer;
        const size_t o = (size_t)(rest % parts_per_layer) * COPY_CHUNK;
        unsigned char* base = c.pool + layer * c.layer_bytes + o;
        copy_chunk(base + h.movers[k] * page_bytes, base + h.holes[k] * page_bytes, (unsigned)min(page_bytes - o, (size_t)COPY_CHUNK));
    }
    const size_t me = (size_t)blockIdx.x * COPY_THREADS + threadIdx.x, all = (size_t)gridDim.x * COPY_THREADS;
    for (size_t e = me; e < (size_t)c.n_seqs * c.max_pages; e += all) {
        const int p = c.tables[e];
        int q = -1;
        if (p >= 0) {
            if (p < (int)c.n_pages) q = h.to[p];
            if (q < 0) atomicOr(h.status, ST_RANGE);        // a table that names a page which is free, or none
        }
        h.tables_out[e] = q;
    }
    for (size_t k = me; k < movers; k += all) {
        const int m = h.movers[k];
        h.refs_out[h.holes[k]] = c.refs[m];
        h.refs_out[m] = 0;
    }
    if (h.refs_out != c.refs)
        for (size_t p = me; p < c.n_pages; p += all) {
            const int r = c.refs[p];
            if (p < (size_t)n_live ? r > 0 : r <= 0) h.refs_out[p] = p < (size_t)n_live ? r : 0;
        }
}

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

bool hand_out_fits(const bf_trusted* t, const Cache& c, uint32_t n) {
    return up((size_t)c.n_seqs * 4) + up((size_t)n * 4) + up((size_t)c.n_pages * 4) <= t->ws_bytes;
}
int hand_out(bf_trusted* t, const Cache& cache, const int* seqs, const int* other, uint32_t n, int fork, HandOut* h) {
    const size_t owner = up((size_t)cache.n_seqs * 4), off = up((size_t)n * 4);
    *h = HandOut{cache, seqs, other, n, fork, (int*)t->ws, (int*)(t->ws + owner), (int*)(t->ws + owner + off), t->status};
    hand_out_kernel<<<1, ONE, 0, t->stream>>>(*h);
    return launched(t, "hand_out_kernel");
}

}  // namespace

#define ON_DEVICE(t)                \
    OnDevice on((t)->device);       \
    if (!on.ok) return cuda_failed(t, "cudaSetDevice", cudaErrorInvalidDevice)

extern "C" int bf_kv4_grow(bf_trusted* t, const bf_kv4_cache* c, const int32_t* seqs, const int32_t* counts, uint32_t n) {
    Cache cache;
    if (!t || !n) return BF_ERR_INVALID_ARG;
    if (int rc = cache_check(c, &cache)) return rc;
    if (!seqs && n > c->n_seqs) return BF_ERR_SHAPE;
    if (n >= (1u << 31) || !hand_out_fits(t, cache, n)) return BF_ERR_TOO_LARGE;
    ON_DEVICE(t);
    HandOut h;
    return hand_out(t, cache, seqs, counts, n, 0, &h);
}

extern "C" int bf_kv4_fork(bf_trusted* t, const bf_kv4_cache* c, const int32_t* src, const int32_t* dst, uint32_t n) {
    Cache cache;
    if (!t || !src || !dst || !n) return BF_ERR_INVALID_ARG;
    if (int rc = cache_check(c, &cache)) return rc;
    const size_t parts = ((size_t)cache.heads * cache.block_bytes + COPY_CHUNK - 1) / COPY_CHUNK;
    if (parts * cache.n_layers >= (1u << 31) || n > 65535 || !hand_out_fits(t, cache, n)) return BF_ERR_TOO_LARGE;
    ON_DEVICE(t);
    HandOut h;
    if (int rc = hand_out(t, cache, src, dst, n, 1, &h)) return rc;
    fork_kernel<<<dim3((unsigned)(parts * cache.n_layers), n), COPY_THREADS, 0, t->stream>>>(h, (unsigned)parts);
    return launched(t, "fork_kernel");
}

extern "C" int bf_kv4_free(bf_trusted* t, const bf_kv4_cache* c, const int32_t* seqs, uint32_t n) {
    Cache cache;
    if (!t || !seqs || !n || n >= (1u << 31)) return BF_ERR_INVALID_ARG;
    if (int rc = cache_check(c, &cache)) return rc;
    ON_DEVICE(t);
    free_kernel<<<n, COPY_THREADS, 0, t->stream>>>(cache, seqs, t->status);
    return launched(t, "free_kernel");
}

extern "C" int bf_kv4_compact(bf_trusted* t, const bf_kv4_cache* c, int32_t* tables_out, int32_t* refs_out, int32_t* n_live) {
    Cache cache;
    if (!t) return BF_ERR_INVALID_ARG;
    if (int rc = cache_check(c, &cache)) return rc;
    const size_t list = up((size_t)cache.n_pages * 4);
    if (3 * list + 256 > t->ws_bytes) return BF_ERR_TOO_LARGE;
    ON_DEVICE(t);
    int* ws = (int*)t->ws;
    Compact h{cache, tables_out ? tables_out : cache.tables, refs_out ? refs_out : cache.refs, n_live,
              ws + 64, ws + 64 + list / 4, ws + 64 + 2 * (list / 4), ws, t->status};
    compact_plan_kernel<<<1, ONE, 0, t->stream>>>(h);
    if (int rc = launched(t, "compact_plan_kernel")) return rc;
    const size_t parts = ((size_t)cache.heads * cache.block_bytes + COPY_CHUNK - 1) / COPY_CHUNK;
    compact_move_kernel<<<t->n_sm * 8, COPY_THREADS, 0, t->stream>>>(h, (unsigned)parts);
    return launched(t, "compact_move_kernel");
}
