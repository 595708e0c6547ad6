// The cache in 4 bits: writing it, reading it back, and attention over it.
#include <math_constants.h>

#include "bf_trusted.h"

using namespace bft;

namespace {

// Sequence i of a list, its rows and its tokens; ok: every index is in range and the rows fit.
struct Span {
    int seq, row0, rows, len;
    bool ok;
};
struct List {
    const int *seqs, *starts;
    unsigned n, most;              // most: bound on the rows of a sequence
};
__device__ __forceinline__ Span span_of(const Cache& c, const List& l, unsigned i) {
    Span s;
    s.seq = l.seqs ? l.seqs[i] : (int)i;
    s.row0 = l.starts ? l.starts[i] : (int)i;
    s.rows = l.starts ? l.starts[i + 1] - s.row0 : 1;
    s.len = 0;
    s.ok = s.seq >= 0 && s.seq < (int)c.n_seqs && s.row0 >= 0 && s.rows >= 0 && s.rows <= (int)l.most;
    if (s.ok) {
        s.len = c.lengths[s.seq];
        s.ok = s.len >= 0 && s.len <= (int)(c.max_pages * c.page_tokens);
    }
    return s;
}

// Places within a sub-block of 16 tokens, see bifrost.h
template <int D, int G> struct Sub {
    static constexpr int DIM = D, GROUP = G;
    static constexpr int E = D / G;                       // groups
    static constexpr int K_PAR = 8 * D, V_CODE = 8 * D + 64 * E, V_PAR = 16 * D + 64 * E, BYTES = 16 * D + 128 * E;
};

constexpr unsigned IO_THREADS = 128;

// One block a (sub-block, head): a warp takes a (token, group) at a time, finds its range, leaves the codes in shared memory;
// then whole words of codes are put together, since a word of value codes holds four tokens of two channels.
template <int D, int G>
__global__ void __launch_bounds__(IO_THREADS) append_kernel(Cache c, unsigned layer, List l, unsigned subs, bf_rows k, bf_rows v, int* status) {
    using S = Sub<D, G>;
    __shared__ unsigned char code[2][16][D];
    const unsigned i = blockIdx.x / subs, head = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Span s = span_of(c, l, i);
    bool twice = false;
    if (l.seqs)
        for (unsigned j = threadIdx.x; j < i; j += IO_THREADS) twice |= l.seqs[j] == s.seq;
    twice = __syncthreads_or(twice);
    if (!s.ok || s.rows > s.len || twice) {
        if (threadIdx.x == 0 && s.rows != 0) atomicOr(status, ST_RANGE);
        return;
    }
    const int base = s.len - s.rows, sub = base / 16 + (int)(blockIdx.x % subs), t0 = sub * 16;
    const int from = max(t0, base) - t0, to = min(t0 + 16, s.len) - t0;
    if (from >= to) return;
    const int page = c.tables[(size_t)s.seq * c.max_pages + t0 / c.page_tokens];
    if (page < 0 || page >= (int)c.n_pages) {
        if (threadIdx.x == 0) atomicOr(status, ST_RANGE);
        return;
    }
    unsigned char* out = c.pool + layer * c.layer_bytes + ((size_t)page * c.heads + head) * c.block_bytes + (t0 % c.page_tokens) / 16 * S::BYTES;
    for (int u = warp; u < 2 * (to - from) * S::E; u += IO_THREADS / 32) {
        const int e = u % S::E, kind = u / S::E % 2, tok = from + u / (2 * S::E);
        const bf_rows& r = kind ? v : k;
        const int64_t at = (int64_t)(s.row0 + t0 + tok - base) * r.row_stride + head * r.head_stride + e * G + lane;
        float x[G / 32], low = CUDART_INF_F, high = -CUDART_INF_F;
        bool nan = false;
#pragma unroll
        for (int m = 0; m < G / 32; ++m) {
            x[m] = load_as_float(r.data, r.type, at + 32 * m);
            nan |= isnan(x[m]);
            x[m] = fminf(fmaxf(x[m], -61440.f), 61440.f);
            low = fminf(low, x[m]);
            high = fmaxf(high, x[m]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            low = fminf(low, __shfl_xor_sync(~0u, low, d));
            high = fmaxf(high, __shfl_xor_sync(~0u, high, d));
        }
        nan = __any_sync(~0u, nan);
        __half hs = __float2half_rn(__double2float_rn(((double)high - (double)low) / 15.0)), hm = __float2half_rn(low);
        if (nan) hs = hm = __float2half_rn(CUDART_NAN_F);
        const float sc = __half2float(hs), m0 = __half2float(hm), inv = 1.0f / sc;
#pragma unroll
        for (int m = 0; m < G / 32; ++m) {
            int q = 0;
            if (sc > 0) {
                // the quotient in 32 bits is off by a few parts in 2^22 of at most 15 (or far above 15.5, where the code is 15 either
                // way); only next to a border of two codes does that matter, and there it is made in 64 bits
                const float a = (x[m] - m0) * inv, n = rintf(a);
                q = (int)fminf(fmaxf(n, 0.f), 15.f);
                if (fabsf(a - n) > 0.499f && a < 16.f) q = (int)fmin(fmax(rint(((double)x[m] - (double)m0) / (double)sc), 0.0), 15.0);
            }
            code[kind][tok][e * G + 32 * m + lane] = (unsigned char)q;
        }
        if (lane == 0) {
            if (kind == 0) {
                __half* p = reinterpret_cast<__half*>(out + S::K_PAR) + 2 * (e + S::E * (tok / 8 + 2 * (tok % 8)));
                p[0] = hs;
                p[1] = hm;
            } else {
                __half* p = reinterpret_cast<__half*>(out + S::V_PAR) + (tok % 2 + 2 * (tok / 8) + 8 * (tok / 2 % 4) + 32 * e);
                p[0] = hs;
                p[4] = hm;
            }
        }
    }
    __syncthreads();
    for (int w = threadIdx.x; w < 2 * D; w += IO_THREADS) {
        // key word w: eight channels of one token
        const int tok = (w >> 4 & 7) + 8 * (w & 1), ch = 64 * (w >> 7) + 32 * (w >> 1 & 1) + 8 * (w >> 2 & 3);
        if (tok >= from && tok < to) {
            uint32_t word = 0;
#pragma unroll
            for (int b = 0; b < 8; ++b) word |= (uint32_t)code[0][tok][ch + b] << (4 * b);
            reinterpret_cast<uint32_t*>(out)[w] = word;
        }
        // value word w: tokens 2j, 2j+1, 2j+8, 2j+9 of channels c and c+8
        const int c0 = 16 * (w & 3) + 64 * (w >> 7) + (w >> 4 & 7), j = w >> 2 & 3;
        uint32_t word = 0, mask = 0;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const int u = 2 * j + 8 * (b >> 1 & 1) + (b >> 2);
            if (u >= from && u < to) {
                word |= (uint32_t)code[1][u][c0 + 8 * (b & 1)] << (4 * b);
                mask |= 15u << (4 * b);
            }
        }
        uint32_t* p = reinterpret_cast<uint32_t*>(out + S::V_CODE) + w;
        if (mask) *p = mask == ~0u ? word : (*p & ~mask) | word;
    }
}

template <int D, int G> __device__ __forceinline__ float key_at(const unsigned char* sub, int u, int ch) {
    using S = Sub<D, G>;
    const int nib = ch % 8 + 8 * (u / 8 + 2 * (ch / 32 % 2 + 2 * (ch / 8 % 4 + 4 * (u % 8 + 8 * (ch / 64)))));
    const __half2 p = reinterpret_cast<const __half2*>(sub + S::K_PAR)[ch / G + S::E * (u / 8 + 2 * (u % 8))];
    return fmaf(__low2float(p), (float)(sub[nib / 2] >> (4 * (nib % 2)) & 15), __high2float(p));
}
template <int D, int G> __device__ __forceinline__ float value_at(const unsigned char* sub, int u, int ch) {
    using S = Sub<D, G>;
    const int nib = ch / 8 % 2 + 2 * (u / 8) + 4 * (u % 2) + 8 * (ch / 16 % 4 + 4 * (u / 2 % 4 + 4 * (ch % 8 + 8 * (ch / 64))));
    const __half* p = reinterpret_cast<const __half*>(sub + S::V_PAR) + (u % 2 + 2 * (u / 8) + 8 * (u / 2 % 4) + 32 * (ch / G));
    return fmaf(__half2float(p[0]), (float)(sub[S::V_CODE + nib / 2] >> (4 * (nib % 2)) & 15), __half2float(p[4]));
}

// One block a (sub-block, head): the sub-block by way of shared memory, its tokens out in rows.
template <int D, int G>
__global__ void __launch_bounds__(IO_THREADS) read_kernel(Cache c, unsigned layer, List l, const int* first, unsigned subs, bf_rows k, bf_rows v,
                                                          int* status) {
    using S = Sub<D, G>;
    __shared__ __align__(16) unsigned char in[S::BYTES];
    const unsigned i = blockIdx.x / subs, head = blockIdx.y;
    const Span s = span_of(c, l, i);
    const int base = first ? first[i] : s.len - s.rows;
    if (!s.ok || base < 0 || base > s.len - s.rows) {
        if (threadIdx.x == 0 && s.rows != 0) atomicOr(status, ST_RANGE);
        return;
    }
    const int end = base + s.rows, sub = base / 16 + (int)(blockIdx.x % subs), t0 = sub * 16;
    const int from = max(t0, base) - t0, to = min(t0 + 16, end) - t0;
    if (from >= to) return;
    const int page = c.tables[(size_t)s.seq * c.max_pages + t0 / c.page_tokens];
    if (page < 0 || page >= (int)c.n_pages) {
        if (threadIdx.x == 0) atomicOr(status, ST_RANGE);
        return;
    }
    const uint4* src = reinterpret_cast<const uint4*>(c.pool + layer * c.layer_bytes + ((size_t)page * c.heads + head) * c.block_bytes +
                                                      (t0 % c.page_tokens) / 16 * S::BYTES);
    for (int w = threadIdx.x; w < S::BYTES / 16; w += IO_THREADS) reinterpret_cast<uint4*>(in)[w] = src[w];
    __syncthreads();
    for (int u = threadIdx.x; u < (to - from) * D; u += IO_THREADS) {
        const int tok = from + u / D, ch = u % D;
        const int64_t row = s.row0 + t0 + tok - base;
        store_from_float(k.data, k.type, row * k.row_stride + head * k.head_stride + ch, key_at<D, G>(in, tok, ch));
        store_from_float(v.data, v.type, row * v.row_stride + head * v.head_stride + ch, value_at<D, G>(in, tok, ch));
    }
}

// One block a (query head, row of a sequence, sequence); a warp takes a token at a time.
template <int D, int G>
__global__ void __launch_bounds__(128) attention_kernel(Cache c, unsigned layer, List l, bf_rows q, unsigned q_heads, bf_rows out, float scale,
                                                        unsigned window, float* lse, int* status) {
    using S = Sub<D, G>;
    __shared__ float acc[4][D], stat[4][2];
    const unsigned head = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kv = head / (q_heads / c.heads);
    const int i = blockIdx.z, j = blockIdx.y;
    const Span s = span_of(c, l, i);
    if (!s.ok) {
        if (threadIdx.x == 0 && s.rows != 0) atomicOr(status, ST_RANGE);
        return;
    }
    if (j >= s.rows) return;
    const int pos = s.len - s.rows + j, first = window && pos >= (int)window ? pos - (int)window + 1 : 0;
    const int64_t row = s.row0 + j;
    float x[D / 32], o[D / 32] = {}, m = -CUDART_INF_F, sum = 0;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) x[e] = load_as_float(q.data, q.type, row * q.row_stride + head * q.head_stride + lane + 32 * e) * scale;
    for (int t = first + warp; t <= pos; t += 4) {
        const int page = c.tables[(size_t)s.seq * c.max_pages + t / c.page_tokens];
        if (page < 0 || page >= (int)c.n_pages) {
            if (lane == 0) atomicOr(status, ST_RANGE);
            continue;
        }
        const unsigned char* sub = c.pool + layer * c.layer_bytes + ((size_t)page * c.heads + kv) * c.block_bytes + (t % c.page_tokens) / 16 * S::BYTES;
        float a = 0;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) a += x[e] * key_at<D, G>(sub, t % 16, lane + 32 * e);
        for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(~0u, a, d);
        const float m2 = fmaxf(m, a), f = m == m2 ? 1.f : expf(m - m2), p = expf(a - m2);
        sum = sum * f + p;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = o[e] * f + p * value_at<D, G>(sub, t % 16, lane + 32 * e);
        m = m2;
    }
#pragma unroll
    for (int e = 0; e < D / 32; ++e) acc[warp][lane + 32 * e] = o[e];
    stat[warp][0] = m;
    stat[warp][1] = sum;
    __syncthreads();
    float top = -CUDART_INF_F, all = 0, y = 0;
    for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w][0]);
    for (int w = 0; w < 4; ++w) {
        if (stat[w][1] == 0) continue;
        const float f = expf(stat[w][0] - top);
        all += f * stat[w][1];
        if (threadIdx.x < D) y += f * acc[w][threadIdx.x];
    }
    if (threadIdx.x < D) store_from_float(out.data, out.type, row * out.row_stride + head * out.head_stride + threadIdx.x, all == 0 ? 0 : y / all);
    if (lse && threadIdx.x == 0) lse[row * q_heads + head] = all == 0 ? -CUDART_INF_F : top + logf(all);
}

template <typename F> void with_shape(const bf_kv4_cache* c, F f) {
    if (c->head_dim == 64) c->group == 32 ? f(Sub<64, 32>{}) : f(Sub<64, 64>{});
    else if (c->group == 32) f(Sub<128, 32>{});
    else if (c->group == 64) f(Sub<128, 64>{});
    else f(Sub<128, 128>{});
}

// rows of k and v of `most` tokens at most touch so many sub-blocks
unsigned subs_of(unsigned most) { return (unsigned)(((uint64_t)most + 14) / 16 + 1); }

int io_check(bf_trusted* t, const bf_kv4_cache* c, Cache* cache, uint32_t layer, const int32_t* seqs, uint32_t n, uint32_t most, const bf_rows* k,
             const bf_rows* v) {
    if (!t || !n || !most || !rows_ok(k) || !rows_ok(v)) return BF_ERR_INVALID_ARG;
    if (int rc = cache_check(c, cache)) return rc;
    if (layer >= c->n_layers || (!seqs && n > c->n_seqs)) return BF_ERR_SHAPE;
    return most >= (1u << 31) || (uint64_t)n * subs_of(most) >= (1u << 31) ? BF_ERR_TOO_LARGE : BF_OK;
}

}  // namespace

#define ON_DEVICE(t)                \
    OnDevice on((t)->device);       \
    if (!on.ok) return cuda_failed(t, "cudaSetDevice", cudaErrorInvalidDevice)

extern "C" int bf_kv4_append(bf_trusted* t, const bf_kv4_cache* c, uint32_t layer, const int32_t* seqs, const int32_t* starts, uint32_t n,
                             uint32_t max_new, const bf_rows* k, const bf_rows* v) {
    Cache cache;
    if (int rc = io_check(t, c, &cache, layer, seqs, n, max_new, k, v)) return rc;
    ON_DEVICE(t);
    const List l{seqs, starts, n, max_new};
    const unsigned subs = subs_of(max_new);
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        append_kernel<S::DIM, S::GROUP><<<dim3(n * subs, c->n_kv_heads), IO_THREADS, 0, t->stream>>>(cache, layer, l, subs, *k, *v, t->status);
    });
    return launched(t, "append_kernel");
}

extern "C" int bf_kv4_read(bf_trusted* t, const bf_kv4_cache* c, uint32_t layer, const int32_t* seqs, const int32_t* starts, const int32_t* first,
                           uint32_t n, uint32_t max_tokens, const bf_rows* k, const bf_rows* v) {
    Cache cache;
    if (int rc = io_check(t, c, &cache, layer, seqs, n, max_tokens, k, v)) return rc;
    ON_DEVICE(t);
    const List l{seqs, starts, n, max_tokens};
    const unsigned subs = subs_of(max_tokens);
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        read_kernel<S::DIM, S::GROUP><<<dim3(n * subs, c->n_kv_heads), IO_THREADS, 0, t->stream>>>(cache, layer, l, first, subs, *k, *v, t->status);
    });
    return launched(t, "read_kernel");
}

extern "C" int bf_kv4_attention(bf_trusted* t, const bf_kv4_cache* c, uint32_t layer, const int32_t* seqs, const int32_t* starts, uint32_t n,
                                uint32_t max_q, uint32_t max_len, const bf_rows* q, uint32_t n_q_heads, const bf_rows* out, float scale,
                                uint32_t window, float* lse) {
    Cache cache;
    if (int rc = io_check(t, c, &cache, layer, seqs, n, max_q, q, out)) return rc;
    if (q->type == BF_F32 || out->type != q->type || !max_len || !isfinite(scale)) return BF_ERR_INVALID_ARG;
    if (!n_q_heads || n_q_heads % c->n_kv_heads) return BF_ERR_SHAPE;
    if (n > 65535 || max_q > 65535 || n_q_heads > 65535) return BF_ERR_TOO_LARGE;
    ON_DEVICE(t);
    const List l{seqs, starts, n, max_q};
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        attention_kernel<S::DIM, S::GROUP><<<dim3(n_q_heads, max_q, n), 128, 0, t->stream>>>(cache, layer, l, *q, n_q_heads, *out, scale, window, lse, t->status);
    });
    return launched(t, "attention_kernel");
}
