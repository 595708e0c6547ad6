// The cache in 4 bits: writing it, reading it back, and attention over it.
#include <math_constants.h>

#include <algorithm>


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

// ------------------------------------------------------------------------------------------------
// Writing and reading.  One block a (sub-block, head); D / 8 lanes a token, 8 channels a lane, 16 or 32 bytes to a load or store.  Both are
// bound by issue (two prompts of 4001 tokens, 8 key heads of 128: 55 instructions an element and 64 % of the slots writing, 27 and 76 % reading, 46 us
// together for 94 MB); what a sub-block holds is put together in, or taken from, shared memory, so that the cache sees whole lines.
constexpr int IO_THREADS = 128;

__device__ __forceinline__ void load8(float (&x)[8], const bf_rows& r, int64_t at, bool wide) {
    if (wide && r.type == BF_F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(r.data) + at);
        const float4 a = p[0], b = p[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else if (wide) {
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.data) + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (r.type == BF_BF16) {
                x[2 * k] = __uint_as_float(w[k] << 16);
                x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                x[2 * k] = f.x, x[2 * k + 1] = f.y;
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = load_as_float(r.data, r.type, at + k);
    }
}
__device__ __forceinline__ void store8(const float (&x)[8], const bf_rows& r, int64_t at, bool wide) {
    if (wide && r.type == BF_F32) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(r.data) + at);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else if (wide) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (r.type == BF_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __half2 h = __floats2half2_rn(x[2 * k], x[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(r.data) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) store_from_float(r.data, r.type, at + k, x[k]);
    }
}
// eight bytes below 16, the first in the lowest bits -> eight nibbles
__device__ __forceinline__ uint32_t nibbles_of(uint2 v) {
    const uint32_t a = (v.x | v.x >> 4) & 0x00ff00ffu, b = (v.y | v.y >> 4) & 0x00ff00ffu;
    return __byte_perm(a, b, 0x6420);
}

template <int D, int G>
__global__ void __launch_bounds__(IO_THREADS, 8) append_kernel(Cache c, unsigned layer, List l, unsigned subs, bf_rows k, bf_rows v, int wide, int* status) {
    using S = Sub<D, G>;
    constexpr int LANES = D / 8, UNITS = IO_THREADS / LANES;                 // lanes of a token; tokens at once
    __shared__ __align__(16) unsigned char image[S::BYTES], code[16 * D];    // code: a byte a nibble of the value words
    const unsigned i = blockIdx.x / subs, head = blockIdx.y;
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
    const int names = threadIdx.x == 0 ? c.refs[page] : 0;                   // (asked for here, needed where the page is written)
    unsigned char* out = c.pool + layer * c.layer_bytes + ((size_t)page * c.heads + head) * c.block_bytes + (t0 % c.page_tokens) / 16 * S::BYTES;
    const int ch = (int)threadIdx.x % LANES * 8, unit = (int)threadIdx.x / LANES;
#pragma unroll 4
    for (int u0 = 2 * from; u0 < 2 * to; u0 += UNITS) {                      // key of token u / 2, value of it
        const int u = u0 + unit, kind = u & 1, tok = u >> 1, e = ch / G;
        const bool here = tok < to;
        float x[8] = {}, low = CUDART_INF_F, high = -CUDART_INF_F;
        if (here) load8(x, kind ? v : k, (int64_t)(s.row0 + t0 + tok - base) * (kind ? v : k).row_stride + head * (kind ? v : k).head_stride + ch, wide >> kind & 1);
        bool nan = false;
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            nan |= isnan(x[m]);
            x[m] = fminf(fmaxf(x[m], -61440.f), 61440.f);
            low = fminf(low, x[m]);
            high = fmaxf(high, x[m]);
        }
#pragma unroll
        for (int d = G / 16; d; d >>= 1) {
            low = fminf(low, __shfl_xor_sync(~0u, low, d));
            high = fmaxf(high, __shfl_xor_sync(~0u, high, d));
            nan |= (bool)__shfl_xor_sync(~0u, (int)nan, d);
        }
        __half hs = __float2half_rn(__double2float_rn(((double)high - (double)low) / 15.0)), hm = __float2half_rn(low);
        if (nan) hs = hm = __float2half_rn(CUDART_NAN_F);
        const float sc = __half2float(hs), m0 = __half2float(hm), inv = 1.0f / sc;
        unsigned q[8] = {};
        if (sc > 0)
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                // the quotient in 32 bits is off by a few parts in 2^22 of at most 15 (or far above 15.5, where the code is 15 either
                // way); only next to a border of two codes does that matter, and there it is made in 64 bits
                const float a = (x[m] - m0) * inv, n = rintf(a);
                q[m] = (unsigned)fminf(fmaxf(n, 0.f), 15.f);
                if (fabsf(a - n) > 0.499f && a < 16.f) q[m] = (unsigned)fmin(fmax(rint(((double)x[m] - (double)m0) / (double)sc), 0.0), 15.0);
            }
        if (!here) continue;
        if (kind == 0) {
            uint32_t word = 0;
#pragma unroll
            for (int m = 0; m < 8; ++m) word |= q[m] << (4 * m);
            reinterpret_cast<uint32_t*>(image)[tok / 8 + 2 * (ch / 32 % 2) + 4 * (ch / 8 % 4) + 16 * (tok % 8) + 128 * (ch / 64)] = word;
        } else {
#pragma unroll
            for (int m = 0; m < 8; ++m)
                code[8 * (ch / 16 % 4 + 4 * (tok / 2 % 4) + 16 * m + 128 * (ch / 64)) + ch / 8 % 2 + 2 * (tok / 8) + 4 * (tok % 2)] = (unsigned char)q[m];
        }
        if (ch % G == 0) {
            __half* p = reinterpret_cast<__half*>(image + (kind ? S::V_PAR : S::K_PAR)) + (kind ? tok % 2 + 2 * (tok / 8) + 8 * (tok / 2 % 4) + 32 * e : 2 * (e + S::E * (tok / 8 + 2 * (tok % 8))));
            p[0] = hs;
            p[kind ? 4 : 1] = hm;
        }
    }
    if (__syncthreads_or(names > 1)) {                                       // other sequences have it too
        if (threadIdx.x == 0) atomicOr(status, ST_RANGE);
        return;
    }
    if (from == 0 && to == 16) {
        for (int w = threadIdx.x; w < 2 * D; w += IO_THREADS) reinterpret_cast<uint32_t*>(image + S::V_CODE)[w] = nibbles_of(reinterpret_cast<const uint2*>(code)[w]);
        __syncthreads();
        for (int w = threadIdx.x; w < S::BYTES / 16; w += IO_THREADS) reinterpret_cast<uint4*>(out)[w] = reinterpret_cast<const uint4*>(image)[w];
        return;
    }
    // in part: the words and parameters of the tokens that are new; a value word keeps the others' nibbles
    for (int w = threadIdx.x; w < 2 * D; w += IO_THREADS) {
        const int tok = (w >> 4 & 7) + 8 * (w & 1);
        if (tok >= from && tok < to) reinterpret_cast<uint32_t*>(out)[w] = reinterpret_cast<const uint32_t*>(image)[w];
        const int j = w >> 2 & 3;
        uint32_t mask = 0;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const int u = 2 * j + 8 * (b >> 1 & 1) + (b >> 2);
            if (u >= from && u < to) mask |= 15u << (4 * b);
        }
        uint32_t* p = reinterpret_cast<uint32_t*>(out + S::V_CODE) + w;
        if (mask) *p = (*p & ~mask) | (nibbles_of(reinterpret_cast<const uint2*>(code)[w]) & mask);
    }
    for (int w = threadIdx.x; w < 16 * S::E; w += IO_THREADS) {
        const int kt = w / S::E % 2 * 8 + w / (2 * S::E);                    // key pair w: (scale, low)
        if (kt >= from && kt < to) reinterpret_cast<uint32_t*>(out + S::K_PAR)[w] = reinterpret_cast<const uint32_t*>(image + S::K_PAR)[w];
    }
    for (int w = threadIdx.x; w < 32 * S::E; w += IO_THREADS) {
        const int vt = 2 * (w >> 3 & 3) + (w & 1) + (w >> 1 & 1) * 8;        // value parameter w, scale or low
        if (vt >= from && vt < to) reinterpret_cast<__half*>(out + S::V_PAR)[w] = reinterpret_cast<const __half*>(image + S::V_PAR)[w];
    }
}

template <int D, int G>
__global__ void __launch_bounds__(IO_THREADS) read_kernel(Cache c, unsigned layer, List l, const int* first, unsigned subs, bf_rows k, bf_rows v,
                                                          int wide, int* status) {
    using S = Sub<D, G>;
    constexpr int LANES = D / 8, UNITS = IO_THREADS / LANES;
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
    const int ch = (int)threadIdx.x % LANES * 8, unit = (int)threadIdx.x / LANES, e = ch / G;
#pragma unroll 4
    for (int u = 2 * from + unit; u < 2 * to; u += UNITS) {
        const int kind = u & 1, tok = u >> 1;
        float x[8];
        if (kind == 0) {
            const uint32_t word = reinterpret_cast<const uint32_t*>(in)[tok / 8 + 2 * (ch / 32 % 2) + 4 * (ch / 8 % 4) + 16 * (tok % 8) + 128 * (ch / 64)];
            const __half2 p = reinterpret_cast<const __half2*>(in + S::K_PAR)[e + S::E * (tok / 8 + 2 * (tok % 8))];
#pragma unroll
            for (int m = 0; m < 8; ++m) x[m] = fmaf(__low2float(p), (float)(word >> (4 * m) & 15), __high2float(p));
        } else {
            const __half* p = reinterpret_cast<const __half*>(in + S::V_PAR) + (tok % 2 + 2 * (tok / 8) + 8 * (tok / 2 % 4) + 32 * e);
            const float sc = __half2float(p[0]), lo = __half2float(p[4]);
            const int nib = ch / 8 % 2 + 2 * (tok / 8) + 4 * (tok % 2), w0 = ch / 16 % 4 + 4 * (tok / 2 % 4) + 128 * (ch / 64);
#pragma unroll
            for (int m = 0; m < 8; ++m) x[m] = fmaf(sc, (float)(reinterpret_cast<const uint32_t*>(in + S::V_CODE)[w0 + 16 * m] >> (4 * nib) & 15), lo);
        }
        const bf_rows& r = kind ? v : k;
        store8(x, r, (int64_t)(s.row0 + t0 + tok - base) * r.row_stride + head * r.head_stride + ch, wide >> kind & 1);
    }
}

// ------------------------------------------------------------------------------------------------
// Attention.  A block has the rows of one key head (its query heads, the tokens of a chunk) that fill NT columns of eight and a share of
// the tokens; a warp takes every 8th sub-block of 16 tokens of that share, so that nothing but the end is shared in the block.
//   S^T = K q^T: tokens x rows, codes as fp16 numbers below the normal range (code * 2^-24, or 2^-20 with q * 2^-4), so that an AND makes
//         two operands; q relative to the largest of its row.  Per group of channels: score += scale_t * sum + low_t * (sum of q).
//   softmax over tokens with a maximum per row that is only moved when a score exceeds it by 2^8: a vote a sub-block in the
//         place of three exchanges.  p is held 2^6 up, so that fp16 takes what lies down to 2^-30 of the largest.
//   O^T = V^T (p scale): channels x rows, codes taken the same way; p^T by a transposition in registers, times the scale of each
//         token and group relative to a power of two that follows them (follow_scales).  The lows are a product of their own, a row a group.
// Codes lie in the cache as the instructions take them, 16 bytes a lane; asynchronous copies run ATT_STAGES - 1 sub-blocks ahead.
// Single tokens are bound by issue: 325 instructions a sub-block of 2.2 KB at D = 128 with one group, 436 with four, half of them unpacking and
// scores, in 54 % of the slots (131072 tokens, 32 query heads: 42 us, 3.4 TB/s); few tokens by the chain of length, table, first copy and joining.
// Chunks: one block of 8 warps an SM by registers, 39 % of the slots (two chunks of 40 and 64 tokens over 4096, 32 heads).
constexpr int ATT_WARPS = 8, ATT_STAGES = 4, P_UP = 6;
constexpr float P_SLACK = 8.f, NO_BASE = __builtin_huge_valf();
constexpr unsigned PIECE = 128, MOST_SPLITS = 160;          // (what 8 NT rows of them count for fits where the copies were)

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 half2_of(uint32_t b) { return *reinterpret_cast<__half2*>(&b); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// n / d by a multiplication where that is exact: m = 2^32 / d + 1 exceeds 2^32 / d by 1 at most, so that n m / 2^32 is off by less than
// 1 / d while n d < 2^32
struct Divisor {
    unsigned d, m, below;
    Divisor() = default;
    explicit Divisor(unsigned by) : d(by), m(by > 1 ? (unsigned)((1ull << 32) / by + 1) : 0), below(by > 1 ? 0xffffffffu / by : 0) {}
    __device__ __forceinline__ unsigned quotient(unsigned n) const { return n < below ? __umulhi(n, m) : d == 1 ? n : n / d; }
    __device__ __forceinline__ unsigned split(unsigned n, unsigned& rest) const {
        const unsigned q = quotient(n);
        rest = n - q * d;
        return q;
    }
};

struct Att {
    Cache c;
    List l;
    bf_rows q, out;
    const unsigned char* layer;    // of the pool
    float* lse;
    float* parts;                  // [block] rows x (D + 2) where a row's tokens are split
    unsigned* arrivals;            // one for every set of splits
    int* status;
    Divisor per, row_tiles, splits, heads, spp;
    unsigned q_heads, window;
    int each;                      // sub-blocks of a split, where that is enough
    float scale;
    int wide;
};

// The first token that a row at `pos` sees.  (A window may be as large as it likes, and a position below zero.)
__device__ __forceinline__ int first_seen(int pos, unsigned window) { return window ? (int)max(0ll, (long long)pos + 1 - window) : 0; }

// Parameters of values where some row does not see some token.  What no row sees may be anything; a NaN that some rows see and others
// do not is taken out of the product, and given to the channels of those that do.
template <int D, int G, int NT>
__device__ __forceinline__ void give_nan(unsigned odd, int e, float (&o)[D / 16][NT][4], int t0, const int (&pos)[NT][2], unsigned window) {
#pragma unroll 1
    for (int u = 0; u < 16; ++u) {
        const unsigned theirs = __shfl_sync(~0u, odd, u / 2 % 4);
        if (!(theirs >> (u % 2 + u / 8 * 2) & 1)) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (t0 + u <= pos[n][h] && t0 + u >= first_seen(pos[n][h], window))
#pragma unroll
                    for (int t = 0; t < D / 16; ++t)
                        if (t * 16 / G == e) o[t][n][h] = o[t][n][h + 2] = CUDART_NAN_F;
    }
}
template <int D, int G, int NT>
__device__ __forceinline__ void open_values(uint4 (&par)[D / G], float (&o)[D / 16][NT][4], int t0, int from, int to, const int (&pos)[NT][2], unsigned window, int j4) {
#pragma unroll
    for (int e = 0; e < D / G; ++e) {
        uint32_t w[4] = {par[e].x, par[e].y, par[e].z, par[e].w};
        unsigned odd = 0;                                                    // which of the four tokens
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = t0 + 2 * j4 + k % 2 + k / 2 * 8;
            const unsigned sh = 16 * (k % 2), sc = w[k / 2] >> sh & 0x7fff, lo = w[2 + k / 2] >> sh & 0x7fff;
            const bool seen = t >= from && t < to, off = sc >= 0x7c00 || lo >= 0x7c00;
            if (!seen || off) {
                w[k / 2] &= ~(0xffffu << sh);
                w[2 + k / 2] &= ~(0xffffu << sh);
            }
            if (seen && off) odd |= 1u << k;
        }
        par[e] = make_uint4(w[0], w[1], w[2], w[3]);
        if (__any_sync(~0u, odd)) give_nan<D, G, NT>(odd, e, o, t0, pos, window);
    }
}

// Scales of the values of 16 tokens in one group as the products take them: two a register (every lane with the same j4 has the same),
// relative to a power of two, 2^-14 .. 2^15, of which `inv` is the inverse.  It is 1 at first, which suits scales from 2^-7 to 2, and 2 to 4 times
// the largest when it is set; and it is set when one exceeds it twice (with p < 2^14 fp16 holds that) or one falls below 2^-7 of
// it: fp16 would lose bits of a smaller one, alone (below 2^-14) or with a probability.  What is small beside others is left out, as 0,
// for products of its own.  Returns whether there is any; `f` is what earlier sums are to be multiplied by.
constexpr float LEAST_RATIO = 0x1p-7f, MOST_RATIO = 2.f, LEAST_REF = 0x1p-14f;   // (relative to the least nothing is below 2^-10)
__device__ __forceinline__ float below_of(__half2 inv) {
    const float i = __low2float(inv);
    return i < 1.f / LEAST_REF ? LEAST_RATIO / i : 0.f;
}
__device__ __forceinline__ bool follow_scales(uint32_t (&s)[2], __half2& inv, float& f) {
    float v[4], top = 0, least = CUDART_INF_F;                               // of what is not 0; both pass over a NaN
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 h = half2_of(s[k / 2]);
        v[k] = fabsf(k % 2 ? __high2float(h) : __low2float(h));
        top = fmaxf(top, v[k]);
        if (v[k] > 0) least = fminf(least, v[k]);
    }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        least = fminf(least, __shfl_xor_sync(~0u, least, d));
    }
    const float old = 1.f / __low2float(inv);
    f = 1.f;
    if (top > MOST_RATIO * old || least < below_of(inv)) {
        const float now = fminf(fmaxf(__uint_as_float((__float_as_uint(fminf(top, 32768.f)) & 0x7f800000u) + 0x01000000u), LEAST_REF), 32768.f);
        f = old / now;
        inv = __float2half2_rn(1.f / now);
    }
    const float below = below_of(inv);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (v[k] < below) s[k / 2] &= ~(0xffffu << (16 * (k % 2)));
#pragma unroll
    for (int k = 0; k < 2; ++k) s[k] = bits(__hmul2(half2_of(s[k]), inv));
    return least < below;
}

template <int D, int G, int NT>
__global__ void __launch_bounds__(ATT_WARPS * 32, NT == 1 ? 2 : 1) attention_kernel(const __grid_constant__ Att p) {
    using S = Sub<D, G>;
    constexpr int E = D / G, RW = 8 * NT, BLOCKS = D / 32, MT = D / 16;
    constexpr bool HOLD = NT <= 2;                                           // operands of q in registers
    // one column of rows: scales go to p, 5 instructions for 8 codes.  More: values are made once for all, 13 for 8.
    constexpr bool SCALE_P = NT == 1;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float sh_m[ATT_WARPS][RW], sh_l[ATT_WARPS][RW], row_scale[RW], row_lift[RW];
    __shared__ unsigned last;
    uint4* qf = reinterpret_cast<uint4*>(smem);                              // [BLOCKS][RW][4]
    float* qs = reinterpret_cast<float*>(smem + BLOCKS * RW * 64);           // [E][RW] sums of q * 2^-24
    unsigned char* ring = smem + BLOCKS * RW * 64 + E * RW * 4;              // [warp][stage][S::BYTES]; at the end [warp][8][D + 4] floats
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, j4 = lane & 3;
    unsigned split, tile, kv;
    const unsigned set = p.splits.split(blockIdx.x, split), i = p.heads.split(p.row_tiles.split(set, tile), kv), per = p.per.d;
    const Span s = span_of(p.c, p.l, i);
    if (!s.ok) {
        if (threadIdx.x == 0 && s.rows != 0) atomicOr(p.status, ST_RANGE);
        return;
    }
    const int rows = s.rows * (int)per, r0 = (int)(tile * RW);
    if (r0 >= rows) return;
    // tokens that some row of this block sees, those that every row sees, and this block's share of the sub-blocks
    const int before = s.len - s.rows;                                       // position of the sequence's first row
    const int pos_first = before + (int)p.per.quotient(r0), pos_last = before + (int)p.per.quotient(min(r0 + RW, rows) - 1);
    const int from = first_seen(pos_first, p.window), to = pos_last + 1, all_from = first_seen(pos_last, p.window), all_to = pos_first + 1;
    const int sb0 = from / 16, n_sb = to > from ? (to + 15) / 16 - sb0 : 0, each = max(p.each, (int)p.splits.quotient(n_sb + p.splits.d - 1));
    const unsigned n_splits = max(1, (n_sb + each - 1) / each);              // of this row's tokens
    if (split >= n_splits) return;
    const int sb_a = sb0 + (int)split * each, sb_b = sb0 + min(n_sb, ((int)split + 1) * each);

    // q of this block's rows, a row a warp at a time: asked for before the copies, which wait for lengths and tables
    auto q_row = [&](float (&x)[8], int r) {
        const int rr = r0 + r;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 0;
        if (rr < rows && lane < D / 8) {
            unsigned h;
            const unsigned j = p.per.split(rr, h);
            const int64_t at = (int64_t)(s.row0 + (int)j) * p.q.row_stride + (int64_t)(kv * per + h) * p.q.head_stride + 8 * lane;
            if (p.wide) {
                const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.q.data) + at);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (p.q.type == BF_BF16) {
                        x[2 * k] = __uint_as_float(w[k] << 16);
                        x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                    } else {
                        const float2 f = __half22float2(half2_of(w[k]));
                        x[2 * k] = f.x, x[2 * k + 1] = f.y;
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = load_as_float(p.q.data, p.q.type, at + k);
            }
        }
    };
    float q_first[8];
    q_row(q_first, warp);

    // copies of this warp's sub-blocks.  Where they lie is looked up 32 at a time, by one lane each
    const int mine = sb_b - sb_a > (int)warp ? (sb_b - sb_a - (int)warp + ATT_WARPS - 1) / ATT_WARPS : 0;
    const int* table = p.c.tables + (size_t)s.seq * p.c.max_pages;
    unsigned char* my_ring = ring + warp * (ATT_STAGES * S::BYTES);
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(my_ring) + lane * 16;
    const unsigned char* my_layer = p.layer + lane * 16;
    constexpr unsigned NOWHERE = 0xffffffffu;
    unsigned where = NOWHERE, bad = 0;                                       // in the layer, in units of 16 bytes
    int next = 0, next_slot = 0;
    auto fetch = [&]() {
        bad <<= 1;
        if (next < mine) {
            if (next % 32 == 0) {
                where = NOWHERE;
                if (next + (int)lane < mine) {
                    const int sb = sb_a + (int)warp + ATT_WARPS * (next + (int)lane);
                    unsigned in_page;
                    const int page = table[p.spp.split(sb, in_page)];
                    if (page >= 0 && page < (int)p.c.n_pages)
                        where = (unsigned)((((size_t)page * p.c.heads + kv) * p.c.block_bytes + in_page * S::BYTES) / 16);
                    else atomicOr(p.status, ST_RANGE);
                }
            }
            const unsigned at = __shfl_sync(~0u, where, next % 32);
            if (at != NOWHERE) {
                const unsigned char* src = my_layer + (size_t)at * 16;
                const uint32_t dst = ring_at + next_slot * S::BYTES;
#pragma unroll
                for (int o = 0; o < S::BYTES; o += 512)
                    if (o + 512 <= S::BYTES || (int)lane * 16 < S::BYTES - o)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + o), "l"(src + o));
            } else {
                bad |= 1;
            }
            ++next;
            next_slot = next_slot + 1 == ATT_STAGES ? 0 : next_slot + 1;
        }
        asm volatile("cp.async.commit_group;");
    };
#pragma unroll
    for (int k = 0; k < ATT_STAGES - 1; ++k) fetch();

    // q as operands
    for (int r = warp; r < RW; r += ATT_WARPS) {
        float x[8];
        if (r == (int)warp) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = q_first[k];
        } else {
            q_row(x, r);
        }
        float big = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) big = fmaxf(big, fabsf(x[k]));
#pragma unroll
        for (int d = 16; d; d >>= 1) big = fmaxf(big, __shfl_xor_sync(~0u, big, d));
        // 2^k with 2^14 <= big 2^k < 2^15, where 2^k is a float
        const int e = max(1, (int)(__float_as_uint(big) >> 23));
        const float up = __uint_as_float((unsigned)min(253, 268 - e) << 23);
        float h[8], sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[k] = __half2float(__float2half_rn(x[k] * up));
            sum += h[k];
        }
        if (lane < D / 8) {
            uint4 o;
            o.x = bits(__floats2half2_rn(h[0], h[4]));
            o.y = bits(__floats2half2_rn(h[1] * 0.0625f, h[5] * 0.0625f));
            o.z = bits(__floats2half2_rn(h[2], h[6]));
            o.w = bits(__floats2half2_rn(h[3] * 0.0625f, h[7] * 0.0625f));
            qf[(lane / 4 * RW + r) * 4 + lane % 4] = o;
        }
#pragma unroll
        for (int d = G / 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (lane < D / 8 && lane % (G / 8) == 0) qs[lane / (G / 8) * RW + r] = sum * 0x1p-24f;
        if (lane == 0) {
            // Scores are x times this, below 2^101: with more, x of 2^14 leaves the range before the score does.  What is taken off makes a difference
            // to none but the log-sum-exp, since scores that differ at all are then 2^20 and more apart.
            const float c = p.scale * 1.4426950408889634f;
            const int by = max(1, e - 14) - 127 + 24, off = min(127, max(0, (int)(__float_as_uint(c) >> 23 & 255) - 127 + by - 100));
            const int half = (by - off) / 2, rest = by - off - half;        // (all of it may be above 2^127)
            row_scale[r] = c * __int_as_float((127 + rest) << 23) * __int_as_float((127 + half) << 23);
            row_lift[r] = __int_as_float((127 + off) << 23);
        }
    }
    __syncthreads();

    uint4 held[HOLD ? BLOCKS : 1][HOLD ? NT : 1];
    float held_sum[HOLD ? E : 1][HOLD ? NT : 1][2];
    float coef[NT][2], base[NT][2], l[NT][2] = {}, o[MT][NT][4] = {};   // base: P_UP - the maximum that is held
    float low[NT][4] = {};                                                   // of group g's lows
    __half2 inv_ref[E];                                                      // see follow_scales
#pragma unroll
    for (int e = 0; e < E; ++e) inv_ref[e] = __float2half2_rn(1.f);
    __half2 my_inv = inv_ref[0];                                             // of group g % E
    int pos[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 8 * n + 2 * (int)j4 + h;
            coef[n][h] = row_scale[r];
            base[n][h] = NO_BASE;
            pos[n][h] = r0 + r < rows ? before + (int)p.per.quotient(r0 + r) : -1;
        }
        if (HOLD) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) held[b][n] = qf[(b * RW + 8 * n + g) * 4 + j4];
#pragma unroll
            for (int e = 0; e < E; ++e) held_sum[e][n][0] = qs[e * RW + 8 * n + 2 * j4], held_sum[e][n][1] = qs[e * RW + 8 * n + 2 * j4 + 1];
        }
    }

    int slot = 0;
    for (int it = 0; it < mine; ++it) {
        fetch();
        asm volatile("cp.async.wait_group %0;" ::"n"(ATT_STAGES - 1));
        __syncwarp();
        const unsigned char* sub = my_ring + slot * S::BYTES;
        slot = slot + 1 == ATT_STAGES ? 0 : slot + 1;
        if (bad >> (ATT_STAGES - 1) & 1) continue;
        const int t0 = (sb_a + (int)warp + ATT_WARPS * it) * 16;
        const bool masked = t0 < all_from || t0 + 16 > all_to;

        // scores of tokens g, g + 8 and rows 2 j4, 2 j4 + 1
        float x[NT][4] = {};
        {
            uint32_t word[BLOCKS][2];
#pragma unroll
            for (int b = 0; b < BLOCKS; b += 2) {
                const uint4 w = reinterpret_cast<const uint4*>(sub)[b * 16 + lane];
                word[b][0] = w.x, word[b][1] = w.y, word[b + 1][0] = w.z, word[b + 1][1] = w.w;
            }
            uint32_t par[2][E];
            {
                const uint32_t* at = reinterpret_cast<const uint32_t*>(sub + S::K_PAR) + 2 * E * g;
                if (E == 1) {
                    const uint2 v = *reinterpret_cast<const uint2*>(at);
                    par[0][0] = v.x, par[1][0] = v.y;
                } else {
#pragma unroll
                    for (int k = 0; k < 2 * E; k += 4) {
                        const uint4 v = *reinterpret_cast<const uint4*>(at + k);
                        par[k / E][k % E] = v.x, par[(k + 1) / E][(k + 1) % E] = v.y, par[(k + 2) / E][(k + 2) % E] = v.z, par[(k + 3) / E][(k + 3) % E] = v.w;
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float acc[NT][4] = {}, acc2[NT][4] = {};
#pragma unroll
                for (int bb = 0; bb < G / 32; ++bb) {
                    const int b = e * (G / 32) + bb;
                    const uint32_t w0 = word[b][0], w1 = word[b][1], v0 = w0 >> 8, v1 = w1 >> 8;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 f = HOLD ? held[HOLD ? b : 0][HOLD ? n : 0] : qf[(b * RW + 8 * n + g) * 4 + j4];
                        mma(acc[n], w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u, f.x, f.y);
                        mma(G == D ? acc2[n] : acc[n], v0 & 0x000f000fu, v1 & 0x000f000fu, v0 & 0x00f000f0u, v1 & 0x00f000f0u, f.z, f.w);
                    }
                }
                const float2 a = __half22float2(half2_of(par[0][e])), b = __half22float2(half2_of(par[1][e]));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float s0 = HOLD ? held_sum[HOLD ? e : 0][HOLD ? n : 0][0] : qs[e * RW + 8 * n + 2 * j4];
                    const float s1 = HOLD ? held_sum[HOLD ? e : 0][HOLD ? n : 0][1] : qs[e * RW + 8 * n + 2 * j4 + 1];
#pragma unroll
                    for (int k = 0; k < 4 && G == D; ++k) acc[n][k] += acc2[n][k];
                    x[n][0] = fmaf(a.x, acc[n][0], fmaf(a.y, s0, x[n][0]));
                    x[n][1] = fmaf(a.x, acc[n][1], fmaf(a.y, s1, x[n][1]));
                    x[n][2] = fmaf(b.x, acc[n][2], fmaf(b.y, s0, x[n][2]));
                    x[n][3] = fmaf(b.x, acc[n][3], fmaf(b.y, s1, x[n][3]));
                }
            }
        }
        uint4 par[E];                                                        // of the values, for later
#pragma unroll
        for (int e = 0; e < E; ++e) par[e] = reinterpret_cast<const uint4*>(sub + S::V_PAR)[e * 4 + j4];
        if (masked) open_values<D, G, NT>(par, o, t0, from, to, pos, p.window, (int)j4);
        bool apart = false;                                                  // scales too far from what they are held relative to
        if (SCALE_P) {
#pragma unroll
            for (int e = 0; e < E; ++e) par[e].x = bits(__hmul2(half2_of(par[e].x), inv_ref[e])), par[e].y = bits(__hmul2(half2_of(par[e].y), inv_ref[e]));
            // each group is looked at by the lanes whose g is its number, not by all.  (Behind a border that may be anything: a look too many)
            __half2 s01 = half2_of(par[0].x), s89 = half2_of(par[0].y);
            if (E > 1) {
                const uint2 w = *reinterpret_cast<const uint2*>(sub + S::V_PAR + (g % E * 4 + j4) * 16);
                s01 = __hmul2(half2_of(w.x), my_inv), s89 = __hmul2(half2_of(w.y), my_inv);
            }
            apart = __any_sync(~0u, !__hbge2(__hmin2(s01, s89), __float2half2_rn(LEAST_RATIO)) || !__hble2(__hmax2(s01, s89), __float2half2_rn(MOST_RATIO)));
        }
        bool over = false, left = false;                                     // left: scales of values that the products leave out for now
        auto take_scales = [&](bool again) {                                 // of all tokens, or of those that were left out
            left = false;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint2 w = *reinterpret_cast<const uint2*>(sub + S::V_PAR + (e * 4 + j4) * 16);
                uint32_t s[2] = {w.x, w.y};
                const float below = again ? below_of(inv_ref[e]) : CUDART_INF_F;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned sh = 16 * (k % 2), a = s[k / 2] >> sh & 0x7fff;
                    const int t = t0 + 2 * (int)j4 + k % 2 + k / 2 * 8;
                    const bool in = (!masked || (t >= from && t < to && a < 0x7c00)) && (!again || __half2float(__ushort_as_half((unsigned short)a)) < below);
                    if (!in) s[k / 2] &= ~(0xffffu << sh);
                }
                float f;
                left |= follow_scales(s, inv_ref[e], f);
                par[e].x = s[0], par[e].y = s[1];
                if ((int)g % E == e) my_inv = inv_ref[e];
                if (f != 1.f)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int t = e * (G / 16); t < (e + 1) * (G / 16); ++t)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[t][n][k] *= f;
            }
        };
        float y[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                y[n][k] = fmaf(x[n][k], coef[n][k % 2], base[n][k % 2]);
                if (masked) {
                    const int t = t0 + (int)g + k / 2 * 8;
                    if (t > pos[n][k % 2] || t < first_seen(pos[n][k % 2], p.window)) y[n][k] = -CUDART_INF_F;
                }
            }
            over |= fmaxf(y[n][0], y[n][2]) > P_UP + P_SLACK;
            over |= fmaxf(y[n][1], y[n][3]) > P_UP + P_SLACK;
        }
        if (__any_sync(~0u, over)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (scores are masked where y is; what is not masked is not -inf in y unless it is in x)
                    const float u = y[n][h] == -CUDART_INF_F ? y[n][h] : x[n][h] * coef[n][h], v = y[n][h + 2] == -CUDART_INF_F ? y[n][h + 2] : x[n][h + 2] * coef[n][h];
                    float top = fmaxf(u, v);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
                    if (P_UP - top < base[n][h]) {
                        const float f = base[n][h] == NO_BASE ? 0.f : exp2_fast(P_UP - top - base[n][h]);
                        base[n][h] = P_UP - top;
                        l[n][h] *= f;
#pragma unroll
                        for (int t = 0; t < MT; ++t) o[t][n][h] *= f, o[t][n][h + 2] *= f;
                        low[n][h] *= f;
                        y[n][h] = u + base[n][h];
                        y[n][h + 2] = v + base[n][h];
                    }
                }
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int k = 0; k < 4; ++k) y[n][k] = exp2_fast(y[n][k]);
            l[n][0] += y[n][0] + y[n][2];
            l[n][1] += y[n][1] + y[n][3];
            pb[n][0] = transposed(bits(__floats2half2_rn(y[n][0], y[n][1])));
            pb[n][1] = transposed(bits(__floats2half2_rn(y[n][2], y[n][3])));
        }

        // values of tokens 2 j4, 2 j4 + 1 and those 8 behind, channels g and g + 8 of 16
        if (SCALE_P) {
            uint32_t m01 = 0, m89 = 0;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if ((int)g == e) m01 = par[e].z, m89 = par[e].w;
#pragma unroll
            for (int n = 0; n < NT; ++n) mma(low[n], m01, 0u, m89, 0u, pb[n][0], pb[n][1]);
        }
        auto add_values = [&]() {
            uint32_t ps[SCALE_P ? E : 1][NT][2];
            if (SCALE_P) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        ps[SCALE_P ? e : 0][n][0] = bits(__hmul2(half2_of(pb[n][0]), half2_of(par[e].x)));
                        ps[SCALE_P ? e : 0][n][1] = bits(__hmul2(half2_of(pb[n][1]), half2_of(par[e].y)));
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                const uint4 w4 = reinterpret_cast<const uint4*>(sub + S::V_CODE)[c * 32 + lane];
                const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = 4 * c + k, e = t * 16 / G;
                    const uint32_t w = word[k], v = w >> 8;
                    if (SCALE_P) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma(o[t][n], w & 0x000f000fu, w & 0x00f000f0u, v & 0x000f000fu, v & 0x00f000f0u, ps[SCALE_P ? e : 0][n][0], ps[SCALE_P ? e : 0][n][1]);
                    } else {
                        const __half2 k1024 = __floats2half2_rn(1024.f, 1024.f), k16 = __floats2half2_rn(0.0625f, 0.0625f), k64 = __floats2half2_rn(-64.f, -64.f);
                        const __half2 s01 = half2_of(par[e].x), s89 = half2_of(par[e].y), m01 = half2_of(par[e].z), m89 = half2_of(par[e].w);
                        const __half2 c0 = __hsub2(half2_of((w & 0x000f000fu) | 0x64006400u), k1024), c1 = __hfma2(half2_of((w & 0x00f000f0u) | 0x64006400u), k16, k64);
                        const __half2 c2 = __hsub2(half2_of((v & 0x000f000fu) | 0x64006400u), k1024), c3 = __hfma2(half2_of((v & 0x00f000f0u) | 0x64006400u), k16, k64);
                        const uint32_t a0 = bits(__hfma2(c0, s01, m01)), a1 = bits(__hfma2(c1, s01, m01)), a2 = bits(__hfma2(c2, s89, m89)), a3 = bits(__hfma2(c3, s89, m89));
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma(o[t][n], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                    }
                }
            }
        };
        if (!SCALE_P || !apart) {
            add_values();
        } else {
            uint2* stash = reinterpret_cast<uint2*>(my_ring + (sub - my_ring)) + lane;   // where the codes of keys were: no registers for what is rare
            __syncwarp();
            *stash = make_uint2(pb[0][0], pb[0][1]);
            for (bool again = false;; again = true) {
                take_scales(again);
                add_values();
                if (!left) break;
                const uint2 kept = *stash;
                pb[0][0] = kept.x, pb[0][1] = kept.y;
            }
        }
        __syncwarp();                                                        // the slot is free for the next copy
    }
    asm volatile("cp.async.wait_all;");

    if (SCALE_P)
    // codes were taken as 2^-24 (channels g) and 2^-20 (g + 8) of themselves, scales relative to ref
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float f = 1.f / __low2float(inv_ref[e]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float add = __shfl_sync(~0u, low[n][h], 4 * e + j4);
#pragma unroll
                for (int t = e * (G / 16); t < (e + 1) * (G / 16); ++t) o[t][n][h] = o[t][n][h] * (f * 0x1p24f) + add, o[t][n][h + 2] = o[t][n][h + 2] * (f * 0x1p20f) + add;
            }
    }
    // the block's rows: maxima and sums of the warps, then their products, eight rows at a time where the copies were
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[n][h] += __shfl_xor_sync(~0u, l[n][h], d);
            if (g == 0) {
                sh_m[warp][8 * n + 2 * j4 + h] = base[n][h] == NO_BASE ? -CUDART_INF_F : (float)P_UP - base[n][h];
                sh_l[warp][8 * n + 2 * j4 + h] = l[n][h];
            }
        }
    float* red = reinterpret_cast<float*>(ring);
    constexpr int PITCH = D + 4;
    constexpr int PART = RW * (D + 2);                                       // rows' products, then their maxima and sums
    float* part = p.parts + (size_t)blockIdx.x * PART;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) red[(warp * 8 + 2 * j4 + k % 2) * PITCH + 16 * t + k / 2 * 8 + g] = o[t][n][k];
        __syncthreads();
        const int r = 8 * n + warp, rr = r0 + r;                             // a warp puts a row together
        if (rr >= rows) continue;
        float top = -CUDART_INF_F, sum = 0, y[D / 32] = {};
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) top = fmaxf(top, sh_m[w][r]);
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) {
            if (sh_l[w][r] == 0) continue;
            const float f = sh_m[w][r] == top ? 1.f : exp2_fast(sh_m[w][r] - top);
            sum += f * sh_l[w][r];
#pragma unroll
            for (int k = 0; k < D / 32; ++k) y[k] += f * red[(w * 8 + warp) * PITCH + lane + 32 * k];
        }
        if (n_splits == 1) {
            unsigned h;
            const unsigned j = p.per.split(rr, h);
            const int64_t row = s.row0 + (int)j, head = kv * per + h;
            const float inv = sum == 0 ? 0.f : 1.f / sum;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) store_from_float(p.out.data, p.out.type, row * p.out.row_stride + head * p.out.head_stride + lane + 32 * k, y[k] * inv);
            if (p.lse && lane == 0) p.lse[row * p.q_heads + head] = sum == 0 ? -CUDART_INF_F : (top * row_lift[r] + log2f(sum) - (float)P_UP) * 0.69314718055994531f;
        } else {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) part[r * D + lane + 32 * k] = y[k];
            if (lane == 0) part[RW * D + 2 * r] = top, part[RW * D + 2 * r + 1] = sum;
        }
    }
    if (n_splits == 1) return;
    // the last block of a row's splits joins them, in their order
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&p.arrivals[set], 1) == n_splits - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (threadIdx.x == 0) p.arrivals[set] = 0;
    const float* first = p.parts + (size_t)(blockIdx.x - split) * PART;
    float* f_of = reinterpret_cast<float*>(smem);                            // [rows][splits] what a split's part counts for
    const int n_rows = min(RW, rows - r0);
    for (int r = warp; r < n_rows; r += ATT_WARPS) {
        float top = -CUDART_INF_F, sum = 0;
        for (unsigned k = lane; k < n_splits; k += 32) top = fmaxf(top, __ldcg(first + (size_t)k * PART + RW * D + 2 * r));
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        for (unsigned k = lane; k < n_splits; k += 32) {
            const float2 a = __ldcg(reinterpret_cast<const float2*>(first + (size_t)k * PART + RW * D + 2 * r));
            const float ml = a.x, ll = a.y, f = ll == 0 ? 0.f : ml == top ? 1.f : exp2_fast(ml - top);
            f_of[r * n_splits + k] = f;
            sum += ll == 0 ? 0.f : f * ll;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (lane == 0) {
            sh_l[0][r] = sum == 0 ? 0.f : 1.f / sum;
            if (p.lse) {
                unsigned h;
                const unsigned j = p.per.split(r0 + r, h);
                const int64_t row = s.row0 + (int)j, head = kv * per + h;
                p.lse[row * p.q_heads + head] = sum == 0 ? -CUDART_INF_F : (top * row_lift[r] + log2f(sum) - (float)P_UP) * 0.69314718055994531f;
            }
        }
    }
    __syncthreads();
    // four channels a thread; where the rows are few, threads share the splits out, so that many loads are on their way
    const int n_vec = n_rows * (D / 4), groups = max(1, ATT_WARPS * 32 / n_vec), mine_k = (int)threadIdx.x / n_vec;
    float4* sum_of = reinterpret_cast<float4*>(smem + (RW * MOST_SPLITS * 4));
    for (int v0 = 0; v0 < n_vec; v0 += ATT_WARPS * 32) {
        const int v = v0 + (groups > 1 ? (int)threadIdx.x % n_vec : (int)threadIdx.x), r = v / (D / 4), c = v % (D / 4) * 4, rr = r0 + r;
        float4 y = make_float4(0, 0, 0, 0);
        if (v < n_vec && mine_k < groups) {
            const float* a = first + r * D + c;
#pragma unroll 8
            for (int k = groups > 1 ? mine_k : 0; k < (int)n_splits; k += groups) {
                const float4 u = __ldcg(reinterpret_cast<const float4*>(a + (size_t)k * PART));
                const float f = f_of[r * n_splits + k];
                if (f != 0) y.x += f * u.x, y.y += f * u.y, y.z += f * u.z, y.w += f * u.w;    // (nothing was seen where it is 0)
            }
        }
        if (groups > 1) {
            sum_of[threadIdx.x] = y;
            __syncthreads();
            if (mine_k == 0)
                for (int k = 1; k < groups; ++k) {
                    const float4 u = sum_of[threadIdx.x + k * n_vec];
                    y.x += u.x, y.y += u.y, y.z += u.z, y.w += u.w;
                }
        }
        if (v < n_vec && (groups == 1 || mine_k == 0)) {
            unsigned h;
            const unsigned j = p.per.split(rr, h);
            const int64_t at = (int64_t)(s.row0 + (int)j) * p.out.row_stride + (int64_t)(kv * per + h) * p.out.head_stride + c;
            const float inv = sh_l[0][r], z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) store_from_float(p.out.data, p.out.type, at + k, z[k] * inv);
        }
    }
}

template <int D, int G, int NT> int attention(bf_trusted* t, Att p, unsigned n, unsigned max_q, unsigned max_len) {
    using S = Sub<D, G>;
    constexpr unsigned RW = 8 * NT;
    const uint64_t row_tiles = ((uint64_t)max_q * p.per.d + RW - 1) / RW, sets = (uint64_t)n * p.c.heads * row_tiles;
    if (sets >= (1u << 31) / 64) return BF_ERR_TOO_LARGE;
    // A row's tokens are split while all blocks run at once, as long as a warp keeps eight sub-blocks (four, where that leaves SMs
    // without a block and the tokens are many); and of many sequences, which may differ in length, the long ones into pieces of 128
    // sub-blocks.  (4096 tokens, 8 key heads: one sequence 13.2 us with four, 15.8 with eight; eight of them 18.2 with either.  700 tokens,
    // 12 heads: 9.3 and 7.8.  131072 tokens in one wave of blocks 42, in two 55.  32 sequences of 160 to 8000 tokens, 8 key heads: 79 us
    // with a block each, 62 in pieces of 128, 67 in pieces of 64.)
    const uint64_t n_sb = ((p.window && (uint64_t)p.window + max_q < max_len ? (uint64_t)p.window + max_q : max_len) + 15) / 16;
    const uint64_t slots = (uint64_t)t->n_sm * (NT == 1 ? 2 : 1), wanted = std::max<uint64_t>(1, slots / sets);
    uint64_t splits = std::min(wanted, (n_sb + 8 * ATT_WARPS - 1) / (8 * ATT_WARPS));
    if (splits * sets < (uint64_t)t->n_sm && n_sb >= 16 * ATT_WARPS)
        splits = std::max(splits, std::min(t->n_sm / sets, (n_sb + 4 * ATT_WARPS - 1) / (4 * ATT_WARPS)));
    if (n > 1 && NT == 1) splits = std::max(splits, (n_sb + PIECE - 1) / PIECE);
    const uint64_t fit = t->ws_bytes / (sets * RW * (D + 2) * sizeof(float));
    if (splits > MOST_SPLITS) splits = MOST_SPLITS;
    if (splits > fit) splits = fit;
    if (splits < 1 || sets > ARRIVALS) splits = 1;
    p.row_tiles = Divisor((unsigned)row_tiles);
    p.splits = Divisor((unsigned)splits);
    p.each = (int)((n_sb + splits - 1) / splits);
    constexpr size_t ring = (size_t)ATT_WARPS * ATT_STAGES * S::BYTES, red = (size_t)ATT_WARPS * 8 * (D + 4) * 4;
    constexpr size_t first = (D / 32) * RW * 64 + (D / G) * RW * 4 + (ring > red ? ring : red), join = RW * MOST_SPLITS * 4 + ATT_WARPS * 32 * 16;
    constexpr size_t smem = first > join ? first : join;
    const cudaError_t e = room_for<attention_kernel<D, G, NT>>(t, smem);
    if (e != cudaSuccess) return cuda_failed(t, "cudaFuncSetAttribute", e);
    attention_kernel<D, G, NT><<<(unsigned)(sets * splits), ATT_WARPS * 32, smem, t->stream>>>(p);
    return launched(t, "attention_kernel");
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
    const int wide = rows_wide(k, true) | rows_wide(v, true) << 1;
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        append_kernel<S::DIM, S::GROUP><<<dim3(n * subs, c->n_kv_heads), IO_THREADS, 0, t->stream>>>(cache, layer, l, subs, *k, *v, wide, t->status);
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
    const int wide = rows_wide(k, true) | rows_wide(v, true) << 1;
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        read_kernel<S::DIM, S::GROUP><<<dim3(n * subs, c->n_kv_heads), IO_THREADS, 0, t->stream>>>(cache, layer, l, first, subs, *k, *v, wide, t->status);
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
    ON_DEVICE(t);
    Att p{cache, List{seqs, starts, n, max_q}, *q, *out, cache.pool + layer * cache.layer_bytes, lse, (float*)t->ws, t->arrivals, t->status,
          Divisor(n_q_heads / c->n_kv_heads), Divisor(1), Divisor(1), Divisor(c->n_kv_heads), Divisor(c->page_tokens / 16), n_q_heads, window, 0, scale,
          rows_wide(q, true)};
    const uint64_t rows = (uint64_t)max_q * p.per.d;
    int rc = BF_OK;
    with_shape(c, [&](auto s) {
        using S = decltype(s);
        rc = rows <= 8 ? attention<S::DIM, S::GROUP, 1>(t, p, n, max_q, max_len)
             : rows <= 16 ? attention<S::DIM, S::GROUP, 2>(t, p, n, max_q, max_len)
                          : attention<S::DIM, S::GROUP, 4>(t, p, n, max_q, max_len);
    });
    return rc;
}
