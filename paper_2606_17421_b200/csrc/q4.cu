// Products with 4-bit weights: y[i] = W x[i], W[o][c] = s (code - 8) + z with s, z per row and group of columns.
#include "bf_trusted.h"

using namespace bft;

namespace {

struct Q4 {
    const uint8_t* codes;
    const __half *scales, *offsets;
    size_t row_bytes;
    unsigned group_stride, d_out, d_in, group;
};

// Codes go into the matrix instruction as they are.  A nibble at bits 0..3 or 4..7 of a 16-bit half IS an fp16 number, code * 2^-24 or
// code * 2^-20 (both below the normal range, both exact), so that one AND makes two operands, against three instructions
// for a conversion: 5 per 8 codes.  x carries the 2^-4 that the second kind is too large by.  Products of 11-bit x and 4-bit codes are
// exact, sums are fp32; the 8 that a code is offset by enters as the accumulator's start, -8 sum x, and the scale of a
// group multiplies the 32 to 128 columns' sum in fp32.
//
// x is held as fp16 relative to the largest of 256 columns, or of its row where it is laid out once (2^14 .. 2^15), which loses nothing of
// bf16 or fp16 above 2^-24 of that, and at most 2^-35 of it below; fp32 takes two columns of the instruction, x = hi + 2^-11 lo, 22 bits.
// Three would hold all 24 and cost half as much again in instructions that are the bound.
constexpr unsigned SEG = 256, SEG_BLOCKS = SEG / 32;          // columns of a stage; blocks of 32 columns in it
constexpr unsigned CODE_BYTES = 16 * SEG / 2;                 // 16 rows of a stage

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t smem, const void* p) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p)); }
__device__ __forceinline__ void copy16(uint32_t smem, const void* p, bool some) {       // zeros where not
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(p), "r"(some ? 16 : 0));
}
template <int BYTES> __device__ __forceinline__ void copy_par(uint32_t smem, const void* p) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p));
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem), "l"(p), "n"(BYTES));
}
// four 8 x 16-byte tiles: lane l names row l % 8 of tile l / 8 and gets word l % 4 of row l / 4 of each
__device__ __forceinline__ void load_words(uint32_t (&w)[4], uint32_t smem) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(smem) : "memory");
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// 256 columns of one row of x (a warp; 8 a lane), zero behind d_in
__device__ __forceinline__ void x_load(float (&v)[8], const bf_rows& x, unsigned row, unsigned c0, unsigned d_in, bool wide) {
    const unsigned c = c0 + 8 * (threadIdx.x & 31);
    const int64_t at = (int64_t)row * x.row_stride + c;
    if (wide && c + 8 <= d_in) {
        if (x.type == BF_F32) {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x.data) + at);
            const float4 a = p[0], b = p[1];
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x.data) + at);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (x.type == BF_BF16) {
                    v[2 * i] = __uint_as_float(w[i] << 16);
                    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    v[2 * i] = f.x;
                    v[2 * i + 1] = f.y;
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < d_in ? load_as_float(x.data, x.type, at + i) : 0.f;
    }
}

__device__ __forceinline__ float largest(const float (&v)[8], float big = 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(v[i]));
    return big;
}
__device__ __forceinline__ float warp_largest(float big) {
#pragma unroll
    for (int d = 16; d; d >>= 1) big = fmaxf(big, __shfl_xor_sync(~0u, big, d));
    return big;
}

// The same as operands, relative to `big`: a lane's 16 bytes at *place(col), the sums of the groups times 2^-24 at sums[group * sums_step
// + col], and what undoes the scaling at undo[col] (from one lane where `tell`); fp32 fills two columns.
template <int G, typename Place>
__device__ __forceinline__ void x_unit(float (&v)[8], float big, bool two, Place place, float* sums, unsigned sums_step, float* undo, bool tell,
                                       unsigned col) {
    const unsigned lane = threadIdx.x & 31;
    // 2^k with 2^14 <= big 2^k < 2^15, where 2^k is a float
    const int e = max(1, (int)(__float_as_uint(big) >> 23));
    const float up = __uint_as_float((unsigned)min(253, 268 - e) << 23), down = __uint_as_float((unsigned)max(1, e - 14) << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= up;
    for (int part = 0; part < (two ? 2 : 1); ++part, ++col) {
        __half h[8];
        float s = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = __float2half_rn(v[i]);
            s += __half2float(h[i]);
        }
        const float q = 0.0625f;
        uint4 o;
        o.x = half2_bits(__half2float(h[0]), __half2float(h[4]));
        o.y = half2_bits(__half2float(h[1]) * q, __half2float(h[5]) * q);
        o.z = half2_bits(__half2float(h[2]), __half2float(h[6]));
        o.w = half2_bits(__half2float(h[3]) * q, __half2float(h[7]) * q);
        *place(col) = o;
#pragma unroll
        for (int d = G / 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        if (lane % (G / 8) == 0) sums[lane / (G / 8) * sums_step + col] = s * 0x1p-24f;
        if (tell && lane == 0) undo[col] = part ? down * 0x1p-11f : down;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] - __half2float(h[i])) * 2048.f;
    }
}

// Up to 8 columns of x that fit shared memory whole.  A warp takes 16 rows of W and every KW-th stage of 256 columns, brings the codes in by
// asynchronous copies, STAGES - 1 ahead and without a barrier of the block, and multiplies them from there.
// 4096 x 128256, one row: 54 us (5.0 TB/s of the 6.5 that a copy reaches); half of the issue slots, 250 instructions a stage of 2.1 KB, are
// what is next.  With the eight 16-byte pieces of a row's stage in eight lines of shared memory instead of one it took 87, with 32
// warps a block of 64 registers 61.  Small matrices are a launch, x and one or two stages.
constexpr unsigned STAGES = 4, X_AT_ONCE = 4, MOST_WARPS = 16;
static_assert((MOST_WARPS & (MOST_WARPS - 1)) == 0, "warps along the columns, a power of two, have to divide a block's");
template <int G, bool OFFSETS> struct Stage { static constexpr unsigned BYTES = CODE_BYTES + 16 * (SEG / G) * 2 * (OFFSETS ? 2 : 1); };

// the parameters that a row has in a stage: 2, 4 or 8 fp16 numbers
template <int N> struct Pars {
    uint32_t w[N / 2];
    __device__ __forceinline__ void load(const void* p) {
        if (N == 2) w[0] = *static_cast<const uint32_t*>(p);
        if (N == 4) *reinterpret_cast<uint2*>(w) = *static_cast<const uint2*>(p);
        if (N == 8) *reinterpret_cast<uint4*>(w) = *static_cast<const uint4*>(p);
    }
    __device__ __forceinline__ float get(int i) const {
        const __half2 h = *reinterpret_cast<const __half2*>(&w[i / 2]);
        return i % 2 ? __high2float(h) : __low2float(h);
    }
};

template <int G, bool OFFSETS>
__global__ void __launch_bounds__(MOST_WARPS * 32) q4_few_kernel(Q4 w, bf_rows x, unsigned n, bf_rows y, unsigned cols, unsigned kw, bool wide) {
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr unsigned STAGE = Stage<G, OFFSETS>::BYTES, GROUPS = SEG / G, PAR = GROUPS * 2;
    const unsigned warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, j = lane % 4;
    const unsigned segs = (w.d_in + SEG - 1) / SEG, per_block = warps / kw, mine = warp / kw, k0 = warp % kw;
    const unsigned tiles = (w.d_out + 15) / 16, rounds = (tiles + gridDim.x * per_block - 1) / (gridDim.x * per_block);
    unsigned char* ring = smem + warp * (STAGES * STAGE);
    uint4* frag = reinterpret_cast<uint4*>(smem + warps * (STAGES * STAGE));
    float* sums = reinterpret_cast<float*>(frag + (size_t)segs * SEG_BLOCKS * cols * 4);
    float* undo = sums + segs * GROUPS * 8;
    float* red = undo + segs * 8;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const unsigned per_tile = k0 < segs ? (segs - k0 + kw - 1) / kw : 0;       // stages of a tile that are this warp's

    // the sequence of stages: tiles of this warp, in each its stages.  A lane copies 16 bytes of row lane / 8 and of the rows 4, 8, 12 below;
    // block b of row r lies at 128 r + 16 (b ^ r % 8): a row's copies fill one line, and eight rows are read without conflicts
    unsigned in_tile = mine * gridDim.x + blockIdx.x, in_seg = k0, in_slot = 0;
    const unsigned cr = lane / 8, cb = lane % 8;
    const uint32_t to_lo = ring_at + cr * 128 + ((cr ^ cb) * 16), to_hi = ring_at + (cr + 4) * 128 + (((cr + 4) ^ cb) * 16);
    const uint32_t to_par = ring_at + CODE_BYTES + lane * PAR;
    const size_t four_rows = 4 * w.row_bytes;
    const uint8_t* from = nullptr;
    const __half* from_par = nullptr;
    auto at_tile = [&]() {
        from = w.codes + (size_t)(in_tile * 16 + cr) * w.row_bytes + cb * 16 + (size_t)in_seg * (SEG / 2);
        const unsigned o = min(in_tile * 16 + lane % 16, w.d_out - 1);
        from_par = (OFFSETS && lane >= 16 ? w.offsets : w.scales) + (size_t)o * w.group_stride + in_seg * GROUPS;
    };
    at_tile();
    auto fetch = [&]() {
        if (in_tile < tiles && per_tile) {
            const uint32_t slot_at = in_slot * STAGE;
            if (in_tile * 16 + 16 <= w.d_out && (size_t)(in_seg + 1) * (SEG / 2) <= w.row_bytes) {
                copy16(to_lo + slot_at, from);
                copy16(to_hi + slot_at, from + four_rows);
                copy16(to_lo + slot_at + 1024, from + 2 * four_rows);
                copy16(to_hi + slot_at + 1024, from + 3 * four_rows);
            } else {                                             // rows behind the last and bytes behind a row's: zeros
                const bool in_row = (size_t)in_seg * (SEG / 2) + cb * 16 < w.row_bytes;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool some = in_row && in_tile * 16 + cr + 4 * i < w.d_out;
                    copy16((i % 2 ? to_hi : to_lo) + slot_at + i / 2 * 1024, some ? from + i * four_rows : w.codes, some);
                }
            }
            if (OFFSETS || lane < 16) copy_par<PAR>(to_par + slot_at, from_par);
            in_slot = in_slot + 1 == STAGES ? 0 : in_slot + 1;
            in_seg += kw;
            from += kw * (SEG / 2);
            from_par += kw * GROUPS;
            if (in_seg >= segs) {
                in_seg = k0;
                in_tile += gridDim.x * per_block;
                at_tile();
            }
        }
        asm volatile("cp.async.commit_group;");
    };
#pragma unroll
    for (unsigned i = 0; i + 1 < STAGES; ++i) fetch();

    // (the rows of x come from L2 a few at a time: one after the other they would wait for it as often)
    const bool two = x.type == BF_F32;
    for (unsigned u0 = warp; u0 < segs * n; u0 += X_AT_ONCE * warps) {
        float v[X_AT_ONCE][8];
#pragma unroll
        for (unsigned i = 0; i < X_AT_ONCE; ++i)
            if (u0 + i * warps < segs * n) x_load(v[i], x, (u0 + i * warps) / segs, (u0 + i * warps) % segs * SEG, w.d_in, wide);
#pragma unroll
        for (unsigned i = 0; i < X_AT_ONCE; ++i) {
            const unsigned seg = (u0 + i * warps) % segs, row = (u0 + i * warps) / segs;
            if (u0 + i * warps < segs * n)
                x_unit<G>(v[i], warp_largest(largest(v[i])), two, [&](unsigned c) { return frag + (((size_t)seg * SEG_BLOCKS + lane / 4) * cols + c) * 4 + lane % 4; },
                          sums + seg * GROUPS * 8, 8, undo + seg * 8, true, two ? 2 * row : row);
        }
    }
    __syncthreads();

    // (columns of the instruction behind the last of x repeat one; nobody reads their sums)
    const uint4* my_frag = frag + min(g, cols - 1) * 4 + j;
    const unsigned fr_step = cols * 4;
    uint32_t rows_at[SEG_BLOCKS / 2];                            // this lane's row of the two blocks 2 p, 2 p + 1, for load_words
#pragma unroll
    for (unsigned p = 0; p < SEG_BLOCKS / 2; ++p) {
        const unsigned b = 2 * p + lane / 16, row = lane % 16;
        rows_at[p] = row * 128 + ((b ^ row % 8) * 16);
    }
    unsigned slot = 0;
    for (unsigned r = 0; r < rounds; ++r) {
        const unsigned tile = (r * per_block + mine) * gridDim.x + blockIdx.x;   // (a last round in part falls to all blocks alike)
        float total[4] = {};
        if (tile < tiles)
            for (unsigned seg = k0; seg < segs; seg += kw) {
                fetch();
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1));
                __syncwarp();
                const unsigned char* st = ring + slot * STAGE;
                const uint4* fr = my_frag + (size_t)seg * SEG_BLOCKS * cols * 4;
                const float* xs_at = sums + seg * GROUPS * 8 + 2 * j;
                const unsigned groups = (w.d_in - seg * SEG + G - 1) / G;      // (x is zero behind d_in, a scale may be anything)
                Pars<GROUPS> s0, s1, z0, z1;
                s0.load(st + CODE_BYTES + g * PAR);
                s1.load(st + CODE_BYTES + (g + 8) * PAR);
                if (OFFSETS) {
                    z0.load(st + CODE_BYTES + (g + 16) * PAR);
                    z1.load(st + CODE_BYTES + (g + 24) * PAR);
                }
                float part[4] = {};
                const uint32_t stage_at = ring_at + slot * STAGE;
#pragma unroll
                for (int e = 0; e < (int)GROUPS; ++e) {
                    const float2 xs = *reinterpret_cast<const float2*>(xs_at + e * 8);
                    float acc[4] = {-8.f * xs.x, -8.f * xs.y, -8.f * xs.x, -8.f * xs.y}, acc2[4] = {};
                    uint32_t word[4];                            // of rows g, g + 8 in an even block, and in the one behind it
#pragma unroll
                    for (int bb = 0; bb < G / 32; ++bb) {
                        const int b = e * (G / 32) + bb;
                        if (b % 2 == 0 || bb == 0) load_words(word, stage_at + rows_at[b / 2]);
                        const uint32_t w0 = word[b % 2 * 2], w1 = word[b % 2 * 2 + 1];
                        const uint4 f = fr[b * fr_step];
                        const uint32_t a0[4] = {w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u};
                        mma(acc, a0, f.x, f.y);
                        const uint32_t v0 = w0 >> 8, v1 = w1 >> 8;
                        const uint32_t a1[4] = {v0 & 0x000f000fu, v1 & 0x000f000fu, v0 & 0x00f000f0u, v1 & 0x00f000f0u};
                        mma(acc2, a1, f.z, f.w);
                    }
                    const float f0 = e < (int)groups ? s0.get(e) : 0.f, f1 = e < (int)groups ? s1.get(e) : 0.f;
                    part[0] += f0 * (acc[0] + acc2[0]), part[1] += f0 * (acc[1] + acc2[1]);
                    part[2] += f1 * (acc[2] + acc2[2]), part[3] += f1 * (acc[3] + acc2[3]);
                    if (OFFSETS) {
                        const float h0 = e < (int)groups ? z0.get(e) : 0.f, h1 = e < (int)groups ? z1.get(e) : 0.f;
                        part[0] += h0 * xs.x, part[1] += h0 * xs.y, part[2] += h1 * xs.x, part[3] += h1 * xs.y;
                    }
                }
                const float2 un = *reinterpret_cast<const float2*>(undo + seg * 8 + 2 * j);
                // (2^24 first: with x near the end of the range on either side, what is undone by itself would leave it)
                total[0] += un.x * (part[0] * 0x1p24f), total[1] += un.y * (part[1] * 0x1p24f);
                total[2] += un.x * (part[2] * 0x1p24f), total[3] += un.y * (part[3] * 0x1p24f);
                __syncwarp();                                    // the slot is free for the next copy
                slot = slot + 1 == STAGES ? 0 : slot + 1;
            }
        if (kw > 1) {                                            // the shares of a tile, in the order of the warps
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) red[warp * 128 + i * 32 + lane] = total[i];
            __syncthreads();
            if (k0 == 0)
                for (unsigned k = 1; k < kw; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[i] += red[(warp + k) * 128 + i * 32 + lane];
        }
        if (tile < tiles && k0 == 0) {
            const unsigned o = tile * 16 + g;
            if (x.type == BF_F32) {
                if (2 * j < cols) {
                    if (o < w.d_out) store_from_float(y.data, y.type, (int64_t)j * y.row_stride + o, total[0] + total[1]);
                    if (o + 8 < w.d_out) store_from_float(y.data, y.type, (int64_t)j * y.row_stride + o + 8, total[2] + total[3]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned col = 2 * j + i % 2, row = o + i / 2 * 8;
                    if (col < cols && row < w.d_out) store_from_float(y.data, y.type, (int64_t)col * y.row_stride + row, total[i]);
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;");
}

constexpr unsigned SMEM_MAX = 227 * 1024;

struct FewPlan { unsigned warps, kw, grid, smem; bool ok; };
template <int G> FewPlan few_plan(const Q4& w, unsigned cols, unsigned n_sm) {
    FewPlan p{};
    const size_t segs = (w.d_in + SEG - 1) / SEG;
    const size_t x_bytes = segs * SEG * 2 * cols + segs * (SEG / G) * 32 + segs * 32;
    const unsigned tiles = (w.d_out + 15) / 16;
    // warps along the columns: what leaves the longest-working warp the fewest stages, a round of joining counted as one
    p.kw = 1;
    size_t least = ~(size_t)0;
    for (unsigned kw = 1; kw <= MOST_WARPS && (kw == 1 || kw / 2 < segs); kw *= 2) {
        const size_t at_once = (size_t)n_sm * (MOST_WARPS / kw), cost = (tiles + at_once - 1) / at_once * ((segs + kw - 1) / kw + (kw > 1));
        if (cost < least) least = cost, p.kw = kw;
    }
    // small matrices: blocks of as few warps as spread them over all SMs
    p.warps = MOST_WARPS;
    while (p.warps > p.kw && p.warps > 1 && (size_t)tiles * p.kw * 2 <= (size_t)n_sm * p.warps) p.warps /= 2;
    const size_t bytes = x_bytes + p.warps * ((size_t)STAGES * (w.offsets ? Stage<G, true>::BYTES : Stage<G, false>::BYTES) + 512);
    p.ok = bytes <= SMEM_MAX;
    p.smem = (unsigned)bytes;
    const unsigned per_block = p.warps / p.kw, blocks = (tiles + per_block - 1) / per_block;
    p.grid = blocks < n_sm ? blocks : n_sm;
    return p;
}

template <int G, bool OFFSETS> int few_launch(bf_trusted* t, const Q4& w, const bf_rows& x, unsigned n, const bf_rows& y, unsigned cols) {
    const FewPlan p = few_plan<G>(w, cols, t->n_sm);
    const cudaError_t e = room_for<q4_few_kernel<G, OFFSETS>>(t, SMEM_MAX);
    if (e != cudaSuccess) return cuda_failed(t, "cudaFuncSetAttribute", e);
    q4_few_kernel<G, OFFSETS><<<p.grid, p.warps * 32, p.smem, t->stream>>>(w, x, n, y, cols, p.kw, rows_wide(&x, false));
    return launched(t, "q4_few_kernel");
}

// ------------------------------------------------------------------------------------------------
// More columns, or more than shared memory holds.  x is laid out once, by a kernel of its own, and streamed with the weights.
struct Prepared {
    unsigned char* at;            // [column chunk][seg]: operands of `width` columns, then the sums of their groups
    float* undo;                  // [columns]
    unsigned width, segs;
    bool tiled;                   // as q4_wide_kernel takes it
    size_t seg_bytes, chunk_bytes;
};

// One block a row of x: the largest of it, then its operands.  What the warps' first PREP_HELD segments read stays in registers.
constexpr unsigned PREP_WARPS = 32, PREP_HELD = 2;

template <int G>
__global__ void __launch_bounds__(PREP_WARPS * 32) q4_prepare_kernel(bf_rows x, unsigned row0, unsigned d_in, bool wide, Prepared p) {
    asm volatile("griddepcontrol.launch_dependents;");
    __shared__ float most[PREP_WARPS];
    const unsigned warp = threadIdx.x / 32, row = blockIdx.x;
    const bool two = x.type == BF_F32;
    float held[PREP_HELD][8], v[8], big = 0;
#pragma unroll
    for (unsigned i = 0; i < PREP_HELD; ++i)
        if (warp + i * PREP_WARPS < p.segs) x_load(held[i], x, row0 + row, (warp + i * PREP_WARPS) * SEG, d_in, wide);
#pragma unroll
    for (unsigned i = 0; i < PREP_HELD; ++i)
        if (warp + i * PREP_WARPS < p.segs) big = largest(held[i], big);
    for (unsigned seg = warp + PREP_HELD * PREP_WARPS; seg < p.segs; seg += PREP_WARPS) {
        x_load(v, x, row0 + row, seg * SEG, d_in, wide);
        big = largest(v, big);
    }
    big = warp_largest(big);
    if (threadIdx.x % 32 == 0) most[warp] = big;
    __syncthreads();
    big = warp_largest(most[threadIdx.x % 32]);
    const unsigned col = two ? 2 * row : row, chunk = col / p.width;          // (a chunk's width is even)
    auto make = [&](float (&u)[8], unsigned seg) {
        unsigned char* at = p.at + chunk * p.chunk_bytes + seg * p.seg_bytes;
        const unsigned lane = threadIdx.x % 32;
        x_unit<G>(u, big, two, [&](unsigned c) {
            // rows of 128 bytes, 64 columns of x each, their 16-byte pieces exchanged by the row's number; or fragments side by side
            return reinterpret_cast<uint4*>(at) + (p.tiled ? (lane / 8 * p.width + c) * 8 + (lane % 8 ^ c % 8) : (lane / 4 * p.width + c) * 4 + lane % 4);
        }, reinterpret_cast<float*>(at + p.width * 512), p.width, p.undo + chunk * p.width, seg == 0, col % p.width);
    };
#pragma unroll
    for (unsigned i = 0; i < PREP_HELD; ++i)
        if (warp + i * PREP_WARPS < p.segs) make(held[i], warp + i * PREP_WARPS);
    for (unsigned seg = warp + PREP_HELD * PREP_WARPS; seg < p.segs; seg += PREP_WARPS) {
        x_load(v, x, row0 + row, seg * SEG, d_in, wide);
        make(v, seg);
    }
}

// A block of 8 warps, kw of them along the columns; a warp has 32 rows of W, 8 NT columns.  All warps go through the stages together: a
// stage holds kw times 256 columns of the rows and of x.  14336 x 4096, 8 rows: 18 us with the kernel before it, 7 steps of 2 us: the
// latency of a step with its barrier.  32 rows of x and 128256 of W: 144 us, the matrix instructions busy in half of them.
constexpr unsigned MANY_WARPS = 8, ROWS = 32;
template <int G, bool OFFSETS> struct Many {
    static constexpr unsigned GROUPS = SEG / G, PAR = GROUPS * 2, CODES = ROWS * SEG / 2, WARP = CODES + ROWS * PAR * (OFFSETS ? 2 : 1);
};

template <int G, bool OFFSETS, int NT>
__global__ void __launch_bounds__(MANY_WARPS * 32, NT <= 4 ? 2 : 1) q4_many_kernel(Q4 w, Prepared p, unsigned cols, unsigned kw, unsigned stages, bf_rows y, unsigned row0) {
    using M = Many<G, OFFSETS>;
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr unsigned GROUPS = M::GROUPS, PAR = M::PAR, WIDTH = 8 * NT, X_SEG = WIDTH * 512 + GROUPS * WIDTH * 4;
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, j = lane % 4;
    const unsigned per_block = MANY_WARPS / kw, mine = warp / kw, k0 = warp % kw;
    const unsigned tiles = (w.d_out + ROWS - 1) / ROWS, steps = (p.segs + kw - 1) / kw;
    const unsigned rounds = (tiles + gridDim.x * per_block - 1) / (gridDim.x * per_block);
    const unsigned stage_bytes = MANY_WARPS * M::WARP + kw * X_SEG;
    const uint32_t smem_at = (uint32_t)__cvta_generic_to_shared(smem);
    float* red = reinterpret_cast<float*>(smem + stages * stage_bytes);
    const unsigned char* x_from = p.at + blockIdx.y * p.chunk_bytes;

    // the next stage to bring in
    unsigned in_round = 0, in_step = 0, in_slot = 0;
    const unsigned cr = lane / 8, cb = lane % 8;
    auto fetch_weights = [&]() {
        if (in_round >= rounds) return;
        const unsigned tile = (in_round * per_block + mine) * gridDim.x + blockIdx.x, seg = in_step * kw + k0;
        if (tile >= tiles || seg >= p.segs) return;
        const uint32_t to = smem_at + in_slot * stage_bytes + warp * M::WARP;
        const size_t at = (size_t)seg * (SEG / 2) + cb * 16;
        const uint8_t* from = w.codes + (size_t)(tile * ROWS + cr) * w.row_bytes + at;
        if (tile * ROWS + ROWS <= w.d_out && (size_t)(seg + 1) * (SEG / 2) <= w.row_bytes) {
#pragma unroll
            for (int i = 0; i < 8; ++i) copy16(to + (cr + 4 * i) * 128 + ((cb ^ ((cr + 4 * i) & 7)) * 16), from + (size_t)(4 * i) * w.row_bytes);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool some = at < w.row_bytes && tile * ROWS + cr + 4 * i < w.d_out;
                copy16(to + (cr + 4 * i) * 128 + ((cb ^ ((cr + 4 * i) & 7)) * 16), some ? from + (size_t)(4 * i) * w.row_bytes : w.codes, some);
            }
        }
        const size_t par = (size_t)min(tile * ROWS + lane, w.d_out - 1) * w.group_stride + seg * GROUPS;
        copy_par<PAR>(to + M::CODES + lane * PAR, w.scales + par);
        if (OFFSETS) copy_par<PAR>(to + M::CODES + (ROWS + lane) * PAR, w.offsets + par);
    };
    auto fetch_x = [&]() {
        if (in_round < rounds) {
            const unsigned segs = min(kw, p.segs - in_step * kw);
            const uint32_t to = smem_at + in_slot * stage_bytes + MANY_WARPS * M::WARP;
            const unsigned char* from = x_from + (size_t)in_step * kw * X_SEG;
            for (unsigned o = threadIdx.x * 16; o < segs * X_SEG; o += MANY_WARPS * 32 * 16) copy16(to + o, from + o);
        }
        asm volatile("cp.async.commit_group;");
        in_slot = in_slot + 1 == stages ? 0 : in_slot + 1;
        if (++in_step == steps) in_step = 0, ++in_round;
    };
    // the first stages' weights do not wait for the kernel before this one, which writes x
    for (unsigned i = 0; i + 1 < stages; ++i) {
        fetch_weights();
        in_slot = in_slot + 1 == stages ? 0 : in_slot + 1;
        if (++in_step == steps) in_step = 0, ++in_round;
    }
    in_round = in_step = in_slot = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (unsigned i = 0; i + 1 < stages; ++i) fetch_x();

    uint32_t rows_at[SEG_BLOCKS / 2];
#pragma unroll
    for (unsigned q = 0; q < SEG_BLOCKS / 2; ++q) rows_at[q] = lane % 16 * 128 + (((2 * q + lane / 16) ^ (lane & 7)) * 16);
    unsigned slot = 0;
    for (unsigned r = 0; r < rounds; ++r) {
        const unsigned tile = (r * per_block + mine) * gridDim.x + blockIdx.x;
        float total[2][NT][4] = {};
        for (unsigned step = 0; step < steps; ++step) {
            if (stages == 4) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else if (stages == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();                                     // this stage is there, and all are done with the one before
            fetch_weights();
            fetch_x();
            const unsigned seg = step * kw + k0;
            if (tile < tiles && seg < p.segs) {
                const unsigned char* st = smem + slot * stage_bytes + warp * M::WARP;
                const uint32_t st_at = smem_at + slot * stage_bytes + warp * M::WARP;
                const unsigned char* xs_seg = smem + slot * stage_bytes + MANY_WARPS * M::WARP + k0 * X_SEG;
                const uint4* fr = reinterpret_cast<const uint4*>(xs_seg) + lane;
                const float* sums = reinterpret_cast<const float*>(xs_seg + WIDTH * 512) + 2 * j;
                const unsigned groups = (w.d_in - seg * SEG + G - 1) / G;      // (x is zero behind d_in, a scale may be anything)
#pragma unroll
                for (int e = 0; e < (int)GROUPS; ++e) {
                    float acc[2][NT][4];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float2 xs = *reinterpret_cast<const float2*>(sums + e * WIDTH + 8 * t);
#pragma unroll
                        for (int m = 0; m < 2; ++m) acc[m][t][0] = acc[m][t][2] = -8.f * xs.x, acc[m][t][1] = acc[m][t][3] = -8.f * xs.y;
                    }
                    uint32_t word[2][4];
#pragma unroll
                    for (int bb = 0; bb < G / 32; ++bb) {
                        const int b = e * (G / 32) + bb;
                        if (b % 2 == 0 || bb == 0) {
                            load_words(word[0], st_at + rows_at[b / 2]);
                            load_words(word[1], st_at + 2048 + rows_at[b / 2]);
                        }
                        uint32_t a0[2][4], a1[2][4];
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const uint32_t w0 = word[m][b % 2 * 2], w1 = word[m][b % 2 * 2 + 1], v0 = w0 >> 8, v1 = w1 >> 8;
                            a0[m][0] = w0 & 0x000f000fu, a0[m][1] = w1 & 0x000f000fu, a0[m][2] = w0 & 0x00f000f0u, a0[m][3] = w1 & 0x00f000f0u;
                            a1[m][0] = v0 & 0x000f000fu, a1[m][1] = v1 & 0x000f000fu, a1[m][2] = v0 & 0x00f000f0u, a1[m][3] = v1 & 0x00f000f0u;
                        }
                        // (all of the first half, then all of the second: two that add to the same sums would wait for each other)
                        uint4 f[NT];
#pragma unroll
                        for (int t = 0; t < NT; ++t) f[t] = fr[(b * WIDTH + 8 * t) * 4];
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int m = 0; m < 2; ++m) mma(acc[m][t], a0[m], f[t].x, f[t].y);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int m = 0; m < 2; ++m) mma(acc[m][t], a1[m], f[t].z, f[t].w);
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const __half* par = reinterpret_cast<const __half*>(st + M::CODES) + (16 * m + g) * GROUPS + e;
                        const float f0 = e < (int)groups ? __half2float(par[0]) : 0.f, f1 = e < (int)groups ? __half2float(par[8 * GROUPS]) : 0.f;
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            total[m][t][0] += f0 * acc[m][t][0], total[m][t][1] += f0 * acc[m][t][1];
                            total[m][t][2] += f1 * acc[m][t][2], total[m][t][3] += f1 * acc[m][t][3];
                        }
                        if (OFFSETS) {
                            const float h0 = e < (int)groups ? __half2float(par[ROWS * GROUPS]) : 0.f, h1 = e < (int)groups ? __half2float(par[(ROWS + 8) * GROUPS]) : 0.f;
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                const float2 xs = *reinterpret_cast<const float2*>(sums + e * WIDTH + 8 * t);
                                total[m][t][0] += h0 * xs.x, total[m][t][1] += h0 * xs.y, total[m][t][2] += h1 * xs.x, total[m][t][3] += h1 * xs.y;
                            }
                        }
                    }
                }
            }
            slot = slot + 1 == stages ? 0 : slot + 1;
        }
        if (kw > 1) {                                            // the shares of a tile, in the order of the warps
            __syncthreads();
            float* to = red + warp * (2 * NT * 128) + lane;
#pragma unroll
            for (int i = 0; i < 2 * NT * 4; ++i) to[i * 32] = total[i / (4 * NT)][i / 4 % NT][i % 4];
            __syncthreads();
            if (k0 == 0)
                for (unsigned k = 1; k < kw; ++k)
#pragma unroll
                    for (int i = 0; i < 2 * NT * 4; ++i) total[i / (4 * NT)][i / 4 % NT][i % 4] += to[k * (2 * NT * 128) + i * 32];
        }
        if (tile < tiles && k0 == 0) {
            const bool two = cols >> 31;                         // (fp32: pairs of columns are one row of x)
            const unsigned n_cols = cols & 0x7fffffffu;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const unsigned col = blockIdx.y * WIDTH + 8 * t + 2 * j;
                if (col >= n_cols) continue;
                const float u0 = p.undo[col], u1 = col + 1 < n_cols ? p.undo[col + 1] : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // four rows of 16 m + 8 h + g
                    const unsigned o = tile * ROWS + 8 * i + g;
                    if (o >= w.d_out) continue;
                    const float a = total[i / 2][t][i % 2 * 2] * 0x1p24f * u0, b = total[i / 2][t][i % 2 * 2 + 1] * 0x1p24f * u1;
                    if (two) {
                        store_from_float(y.data, y.type, (int64_t)(row0 + col / 2) * y.row_stride + o, a + b);
                    } else {
                        store_from_float(y.data, y.type, (int64_t)(row0 + col) * y.row_stride + o, a);
                        if (col + 1 < n_cols) store_from_float(y.data, y.type, (int64_t)(row0 + col + 1) * y.row_stride + o, b);
                    }
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;");
}

template <int G, bool OFFSETS, int NT>
int many_launch(bf_trusted* t, const Q4& w, const bf_rows& x, unsigned row0, unsigned rows, const bf_rows& y, Prepared p) {
    using M = Many<G, OFFSETS>;
    const bool two = x.type == BF_F32;
    const unsigned cols = rows * (two ? 2 : 1), chunks = (cols + p.width - 1) / p.width, tiles = (w.d_out + ROWS - 1) / ROWS;
    q4_prepare_kernel<G><<<rows, PREP_WARPS * 32, 0, t->stream>>>(x, row0, w.d_in, rows_wide(&x, false), p);
    if (int rc = launched(t, "q4_prepare_kernel")) return rc;
    // warps along the columns: what leaves the longest-working SM the fewest steps, a round of joining counted as one; the x of a
    // stage is at most 32 KB.  Two blocks an SM where there is room and work for two.
    unsigned kw = 1, per_sm = 1;
    size_t least = ~(size_t)0;
    for (unsigned k = 1; k <= MANY_WARPS && k * p.width <= 64 && (k == 1 || k / 2 < p.segs); k *= 2) {
        const size_t bytes = 2 * (MANY_WARPS * M::WARP + k * p.seg_bytes) + (k > 1 ? MANY_WARPS * 2 * NT * 512 : 0);
        const size_t blocks = (tiles + MANY_WARPS / k - 1) / (MANY_WARPS / k) * (size_t)chunks;
        const unsigned two_fit = NT <= 4 && bytes <= SMEM_MAX / 2 - 1024 && blocks > (size_t)t->n_sm ? 2 : 1;
        const size_t at_once = (size_t)t->n_sm * two_fit, cost = (blocks + at_once - 1) / at_once * ((p.segs + k - 1) / k + (k > 1)) * two_fit;
        if (cost < least) least = cost, kw = k, per_sm = two_fit;
    }
    const unsigned stage = MANY_WARPS * M::WARP + kw * (unsigned)p.seg_bytes, red = kw > 1 ? MANY_WARPS * 2 * NT * 512 : 0;
    unsigned stages = 4;
    while (stages > 2 && stages * stage + red > (per_sm == 2 ? SMEM_MAX / 2 - 1024 : SMEM_MAX)) --stages;
    const unsigned per_block = MANY_WARPS / kw, blocks = (tiles + per_block - 1) / per_block, most_blocks = t->n_sm * per_sm;
    cudaError_t e = room_for<q4_many_kernel<G, OFFSETS, NT>>(t, SMEM_MAX);
    if (e != cudaSuccess) return cuda_failed(t, "cudaFuncSetAttribute", e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks < most_blocks ? blocks : most_blocks, chunks);
    cfg.blockDim = MANY_WARPS * 32;
    cfg.dynamicSmemBytes = stages * stage + red;
    cfg.stream = t->stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, q4_many_kernel<G, OFFSETS, NT>, w, p, cols | (two ? 1u << 31 : 0), kw, stages, y, row0);
    return e == cudaSuccess ? launched(t, "q4_many_kernel") : cuda_failed(t, "q4_many_kernel", e);
}

// Segments of x that every block makes operands of by itself; more are made once, which costs a launch.  4096 x 4096, 1 / 2 / 4 rows
// (16 segments each): in every block 6.0 / 6.8 / 8.6 us, by a kernel of its own 6.6 / 6.7 / 6.6.  Of 14336 columns (56 segments a row) one row: 4096
// outputs 13.3 either way, 1024 outputs 9.3 and 13.1, 16384 outputs 30.6 and 33.6: there the line is drawn too low.
constexpr unsigned FEW_UNITS = 32;
// ------------------------------------------------------------------------------------------------
// Many rows of W as well: the fifth-generation matrix instructions.  A block of 128 threads has 128 rows of W, a thread a row.  Codes go from
// shared memory through registers (the same ANDs) to TMEM, 128 columns of W at a time, as operand A (K pairs in 32-bit columns, K in
// the order in which a word unpacks); x is operand B in shared memory, rows of 128 bytes in the 128-byte swizzle; one thread issues
// the products of a group of columns into its own accumulators, and each thread multiplies its row's sums by the group's scale.
// While the products run, the next 128 columns are unpacked.  Waits are bounded; one that gives up is BF_ERR_TIMEOUT.
// 4096 x 128256, 32 rows: 104 us (2.7 TB/s); three blocks an SM, which shared memory allows, keep 46 % of the issue slots busy, and 1002
// tiles are 2.3 rounds of them.  With two blocks (210 registers a thread) 138.
constexpr unsigned TILE = 128;

__device__ __forceinline__ bool wait_for(uint32_t bar, unsigned parity) {
    for (int i = 0; i < (1 << 17); ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                 "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t (&r)[16], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
}

template <int G, bool OFFSETS, int N> struct Wide {
    static constexpr unsigned GROUPS = SEG / G, PAR = GROUPS * 2, IN_UNIT = TILE / G;      // groups of a stage, of a unit of 128 columns
    static constexpr unsigned X = N * 512, CODES = TILE * SEG / 2, PARS = TILE * PAR * (OFFSETS ? 2 : 1), SUMS = GROUPS * N * 4;
    static constexpr unsigned STAGE = X + CODES + PARS;                      // (sums have a slot more: they are read for one stage longer)
    static constexpr unsigned TMEM = 64 + IN_UNIT * N <= 128 ? 128 : 64 + IN_UNIT * N <= 256 ? 256 : 512;   // columns: A, then the sums
};

template <int G, bool OFFSETS, int N>
__global__ void __launch_bounds__(TILE, N == 64 || Wide<G, OFFSETS, N>::TMEM > 128 ? 2 : TILE / G * N > 32 || N == 32 ? 3 : 4) q4_wide_kernel(Q4 w, Prepared p, unsigned cols, unsigned stages, bf_rows y, unsigned row0, int* status) {
    using M = Wide<G, OFFSETS, N>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long bar_word;
    __shared__ uint32_t tmem_word;
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32, row = threadIdx.x;
    const unsigned tiles = (w.d_out + TILE - 1) / TILE, steps = p.segs;
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(smem) + 1023) & ~1023u;                   // operand B lies on 1024 bytes
    unsigned char* at_base = smem + (base - (uint32_t)__cvta_generic_to_shared(smem));
    const uint32_t codes_at = base + stages * M::X, pars_at = codes_at + stages * M::CODES, sums_at = pars_at + stages * M::PARS;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&bar_word);
    const unsigned char* x_from = p.at + blockIdx.y * p.chunk_bytes;
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_word)), "n"(M::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (threadIdx.x == 0) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    // stages to bring in: a warp its own 32 rows of codes and parameters, all of them x
    unsigned in_tile = blockIdx.x, in_step = 0, in_slot = 0, in_sums = 0;
    const unsigned cr = lane / 8, cb = lane % 8;
    auto fetch_weights = [&]() {
        if (in_tile >= tiles) return;
        const unsigned r0 = in_tile * TILE + warp * 32;
        const uint32_t to = codes_at + in_slot * M::CODES + warp * 32 * 128;
        const size_t at = (size_t)in_step * (SEG / 2) + cb * 16;
        const uint8_t* from = w.codes + (size_t)(r0 + cr) * w.row_bytes + at;
        if (r0 + 32 <= w.d_out && (size_t)(in_step + 1) * (SEG / 2) <= w.row_bytes) {
#pragma unroll
            for (int i = 0; i < 8; ++i) copy16(to + (cr + 4 * i) * 128 + ((cb ^ ((cr + 4 * i) & 7)) * 16), from + (size_t)(4 * i) * w.row_bytes);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool some = at < w.row_bytes && r0 + cr + 4 * i < w.d_out;
                copy16(to + (cr + 4 * i) * 128 + ((cb ^ ((cr + 4 * i) & 7)) * 16), some ? from + (size_t)(4 * i) * w.row_bytes : w.codes, some);
            }
        }
        const size_t par = (size_t)min(in_tile * TILE + row, w.d_out - 1) * w.group_stride + in_step * M::GROUPS;
        copy_par<M::PAR>(pars_at + in_slot * M::PARS + row * M::PAR, w.scales + par);
        if (OFFSETS) copy_par<M::PAR>(pars_at + in_slot * M::PARS + (TILE + row) * M::PAR, w.offsets + par);
    };
    auto step_on = [&]() {
        in_slot = in_slot + 1 == stages ? 0 : in_slot + 1;
        if (++in_step == steps) in_step = 0, in_tile += gridDim.x;
    };
    auto fetch_x = [&]() {
        if (in_tile < tiles) {
            const unsigned char* from = x_from + (size_t)in_step * (M::X + M::SUMS);
            for (unsigned o = threadIdx.x * 16; o < M::X; o += TILE * 16) copy16(base + in_slot * M::X + o, from + o);
            for (unsigned o = threadIdx.x * 16; o < M::SUMS; o += TILE * 16) copy16(sums_at + in_sums * M::SUMS + o, from + M::X + o);
        }
        asm volatile("cp.async.commit_group;");
        in_sums = in_sums == stages ? 0 : in_sums + 1;
        step_on();
    };
    for (unsigned i = 0; i + 1 < stages; ++i) {
        fetch_weights();
        step_on();
    }
    in_tile = blockIdx.x, in_step = in_slot = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (unsigned i = 0; i + 1 < stages; ++i) fetch_x();
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_word, mine = tmem + (warp * 32 << 16);        // this warp's 32 lanes of it
    // f16 operands, both K-major, f32 sums, 128 x N; operand B: 128-byte swizzle, 1024 bytes from 8 rows to the next
    constexpr uint32_t IDESC = 1u << 4 | (N / 8) << 17 | (TILE / 16) << 24;
    constexpr unsigned long long BDESC = 2ull << 61 | 1ull << 46 | (1024ull >> 4) << 32 | 1ull << 16;

    bool dead = false;
    unsigned slot = 0, sums_slot = 0, parity = 0;
    for (unsigned tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        float total[N] = {};
        // the sums of a unit: of the groups of columns whose scales are s (and z), times what x was summed to
        uint32_t acc[M::IN_UNIT][N / 16][16];
        Pars<M::GROUPS> s, z, s_old, z_old;
        unsigned old_sums = 0, old_unit = 0, old_groups = 0;
        auto take = [&]() {                                      // (what was loaded before)
            const float* xs = reinterpret_cast<const float*>(at_base + (sums_at - base) + old_sums * M::SUMS) + old_unit * M::IN_UNIT * N;
#pragma unroll
            for (int e = 0; e < (int)M::IN_UNIT; ++e) {
                const int ge = old_unit * M::IN_UNIT + e;
                const float f = ge < (int)old_groups ? s_old.get(old_unit ? M::IN_UNIT + e : e) : 0.f;
                const float h = ge < (int)old_groups ? (OFFSETS ? z_old.get(old_unit ? M::IN_UNIT + e : e) : 0.f) - 8.f * f : 0.f;
#pragma unroll
                for (int c = 0; c < N; c += 4) {
                    const float4 v = *reinterpret_cast<const float4*>(xs + e * N + c);
                    total[c] += f * __uint_as_float(acc[e][c / 16][c % 16]) + h * v.x;
                    total[c + 1] += f * __uint_as_float(acc[e][c / 16][c % 16 + 1]) + h * v.y;
                    total[c + 2] += f * __uint_as_float(acc[e][c / 16][c % 16 + 2]) + h * v.z;
                    total[c + 3] += f * __uint_as_float(acc[e][c / 16][c % 16 + 3]) + h * v.w;
                }
            }
        };
        auto load_sums = [&]() {
#pragma unroll
            for (int e = 0; e < (int)M::IN_UNIT; ++e)
#pragma unroll
                for (int c = 0; c < N / 16; ++c) tmem_load16(acc[e][c], mine + 64 + e * N + c * 16);
        };
        for (unsigned step = 0; step < steps; ++step) {
            if (stages == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // x, for the matrix instructions
            __syncwarp();
            const unsigned char* st = at_base + (codes_at - base) + slot * M::CODES + row * 128;
            const unsigned char* pr = at_base + (pars_at - base) + slot * M::PARS + row * M::PAR;
            s.load(pr);
            if (OFFSETS) z.load(pr + TILE * M::PAR);
            const unsigned groups = (w.d_in - step * SEG + G - 1) / G;
#pragma unroll
            for (unsigned unit = 0; unit < 2; ++unit) {
                uint32_t a[64];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint4 v = *reinterpret_cast<const uint4*>(st + (((unit * 4 + c) ^ (row & 7)) * 16));
                    const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t u = word[k], h = u >> 8;
                        a[c * 16 + k * 4] = u & 0x000f000fu, a[c * 16 + k * 4 + 1] = u & 0x00f000f0u;
                        a[c * 16 + k * 4 + 2] = h & 0x000f000fu, a[c * 16 + k * 4 + 3] = h & 0x00f000f0u;
                    }
                }
                const bool before = step || unit;                // products are under way: their end, their sums
                if (before) {
                    if (!dead && !wait_for(bar, parity)) dead = true;
                    parity ^= 1;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    load_sums();
                }
                tmem_store32(mine, a);
                tmem_store32(mine + 32, a + 32);
                if (before) asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) {
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t b_at = base + slot * M::X + unit * 2 * (N * 128);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const unsigned long long desc = BDESC | ((b_at + k / 4 * (N * 128) + k % 4 * 32) >> 4 & 0x3fff);
                        const uint32_t more = k % (G / 16) != 0;
                        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                                     ::"r"(tmem + 64 + k / (G / 16) * N), "r"(tmem + k * 8), "l"(desc), "r"(IDESC), "r"(more) : "memory");
                    }
                    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
                }
                __syncwarp();
                if (unit == 0) {                                 // the stage before this one is free
                    fetch_weights();
                    fetch_x();
                }
                if (before) take();
                s_old = s;
                if (OFFSETS) z_old = z;
                old_sums = sums_slot, old_unit = unit, old_groups = groups;
            }
            slot = slot + 1 == stages ? 0 : slot + 1;
            sums_slot = sums_slot == stages ? 0 : sums_slot + 1;
        }
        if (!dead && !wait_for(bar, parity)) dead = true;
        parity ^= 1;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        load_sums();
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        take();
        const unsigned o = tile * TILE + row;
        const bool two = cols >> 31;                             // (fp32: pairs of columns are one row of x)
        const unsigned n_cols = cols & 0x7fffffffu;
        if (o < w.d_out) {
#pragma unroll
            for (int c = 0; c < N; c += 2) {
                const unsigned col = blockIdx.y * N + c;
                if (col >= n_cols) break;
                const float u = total[c] * 0x1p24f * p.undo[col], v = col + 1 < n_cols ? total[c + 1] * 0x1p24f * p.undo[col + 1] : 0.f;
                if (two) {
                    store_from_float(y.data, y.type, (int64_t)(row0 + col / 2) * y.row_stride + o, u + v);
                } else {
                    store_from_float(y.data, y.type, (int64_t)(row0 + col) * y.row_stride + o, u);
                    if (col + 1 < n_cols) store_from_float(y.data, y.type, (int64_t)(row0 + col + 1) * y.row_stride + o, v);
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (dead) atomicOr(status, ST_TIMEOUT);
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(M::TMEM));
}

template <int G, bool OFFSETS, int N>
int wide_launch(bf_trusted* t, const Q4& w, const bf_rows& x, unsigned row0, unsigned rows, const bf_rows& y, Prepared p) {
    using M = Wide<G, OFFSETS, N>;
    const bool two = x.type == BF_F32;
    const unsigned cols = rows * (two ? 2 : 1), chunks = (cols + N - 1) / N, tiles = (w.d_out + TILE - 1) / TILE;
    q4_prepare_kernel<G><<<rows, PREP_WARPS * 32, 0, t->stream>>>(x, row0, w.d_in, rows_wide(&x, false), p);
    if (int rc = launched(t, "q4_prepare_kernel")) return rc;
    const unsigned stages = 2, bytes = stages * M::STAGE + (stages + 1) * M::SUMS + 1024;
    unsigned per_sm = SMEM_MAX / (bytes + 1024 + 256);
    if (per_sm > 512 / M::TMEM) per_sm = 512 / M::TMEM;          // (a block that finds no TMEM would wait for one that ends)
    cudaError_t e = room_for<q4_wide_kernel<G, OFFSETS, N>>(t, SMEM_MAX - 1024);
    if (e != cudaSuccess) return cuda_failed(t, "cudaFuncSetAttribute", e);
    cudaLaunchConfig_t cfg = {};
    const unsigned most = t->n_sm * per_sm / (chunks < per_sm ? chunks : per_sm);
    cfg.gridDim = dim3(tiles < most ? tiles : most, chunks);
    cfg.blockDim = TILE;
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = t->stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, q4_wide_kernel<G, OFFSETS, N>, w, p, cols | (two ? 1u << 31 : 0), stages, y, row0, t->status);
    return e == cudaSuccess ? launched(t, "q4_wide_kernel") : cuda_failed(t, "q4_wide_kernel", e);
}

// Rows of W from which products take blocks of 128 of them, in the place of blocks that share the columns out as well.  4096 columns, us with the former and
// the latter, for 4096 / 19072 / 32768 / 65536 / 128256 rows:
//   groups of 128  16 rows of x  29, 11 / 34, 23 / 34, 27 / 47, 41 / 80, 89      32  33, 24 / 38, 41 / 39, 42 / 69, 77 / 105, 147
//                  64            36, 63 / 43, 63 / 44, 64 / 83, 122 / 159, 223
//   groups of 64   16            37, 11 / 56, 26 / 56, 31 / 72, 49 / 128, 104    32  37, 26 / 58, 56 / 58, 56 / 102, 94 / 163, 165
//                  64            54, 82 / 73, 84 / 73, 86 / 143, 163 / 275, 304
//   groups of 32   16            34, 12 / 42, 28 / 43, 34 / 78, 53 / 122, 111    32  40, 29 / 51, 53 / 52, 55 / 100, 93 / 180, 190
// So the line holds for 64 rows of x, and for 32 but for groups of 64 (4 to 9 % slower than the other up to 65536 rows, 6 to 23 with offsets).  For 16 it
// is drawn too low: groups of 128 gain from somewhere above 65536 rows only, groups of 64 and 32 nowhere here (up to twice the time).
// (Groups of 32 with 64 columns would need more registers for sums than there are.)
template <int G> bool wide_pays(const bf_trusted* t, unsigned d_out, unsigned width) {
    if (width < 16 || TILE / G * width > 128) return false;
    return (d_out + TILE - 1) / TILE >= (unsigned)t->n_sm / (width == 64 ? 8 : 1);
}
template <int G, bool OFFSETS> int linear(bf_trusted* t, const Q4& w, const bf_rows& x, unsigned n, const bf_rows& y) {
    const unsigned per_row = x.type == BF_F32 ? 2 : 1, segs = (w.d_in + SEG - 1) / SEG;
    // every block of the first kernel makes the operands of x itself
    if ((uint64_t)n * per_row <= 8 && (uint64_t)n * segs <= FEW_UNITS && few_plan<G>(w, n * per_row, t->n_sm).ok) return few_launch<G, OFFSETS>(t, w, x, n, y, n * per_row);
    // rows of x whose operands the workspace holds, in chunks of 8 to 64 columns; 65535 chunks at most
    Prepared p{};
    p.segs = segs;
    const uint64_t all = (uint64_t)n * per_row;
    p.width = all <= 8 ? 8 : all <= 16 ? 16 : all <= 32 ? 32 : 64;
    uint64_t chunks = 0;
    for (;; p.width /= 2) {                                      // (narrower where the workspace does not hold one chunk)
        p.seg_bytes = p.width * (512 + SEG / G * 4);
        p.chunk_bytes = p.seg_bytes * segs;
        chunks = t->ws_bytes / (p.chunk_bytes + p.width * 4 + 256);
        if (chunks || p.width == 8) break;
    }
    if (chunks == 0) return BF_ERR_TOO_LARGE;
    p.tiled = wide_pays<G>(t, w.d_out, p.width);
    if (chunks > 1024) chunks = 1024;
    const unsigned rows_at_once = (unsigned)(chunks * p.width / per_row);
    for (unsigned r = 0; r < n; r += rows_at_once) {
        const unsigned rows = n - r < rows_at_once ? n - r : rows_at_once;
        p.undo = reinterpret_cast<float*>(t->ws);
        p.at = t->ws + (((size_t)rows * per_row + p.width) * 4 + 255) / 256 * 256;
        if (p.tiled) {
            int rc;
            if (p.width == 16) rc = wide_launch<G, OFFSETS, 16>(t, w, x, r, rows, y, p);
            else if (p.width == 32) rc = wide_launch<G, OFFSETS, 32>(t, w, x, r, rows, y, p);
            else rc = wide_launch<G, OFFSETS, G == 32 ? 32 : 64>(t, w, x, r, rows, y, p);       // (groups of 32 do not come here)
            if (rc) return rc;
            continue;
        }
        int rc = p.width == 8    ? many_launch<G, OFFSETS, 1>(t, w, x, r, rows, y, p)
                 : p.width == 16 ? many_launch<G, OFFSETS, 2>(t, w, x, r, rows, y, p)
                 : p.width == 32 ? many_launch<G, OFFSETS, 4>(t, w, x, r, rows, y, p)
                                 : many_launch<G, OFFSETS, 8>(t, w, x, r, rows, y, p);
        if (rc) return rc;
    }
    return BF_OK;
}

}  // namespace

// One thread an element; read from L2 and L1, bound by the writes.
static __global__ void __launch_bounds__(256) q4_expand_kernel(Q4 w, float* out) {
    const unsigned c = blockIdx.x * 256 + threadIdx.x;
    if (c >= w.d_in) return;
    for (unsigned o = blockIdx.y; o < w.d_out; o += gridDim.y) {
        const int code = w.codes[o * w.row_bytes + c / 2] >> (4 * (c % 2)) & 15;
        const size_t g = (size_t)o * w.group_stride + c / w.group;
        out[(size_t)o * w.d_in + c] = fmaf(__half2float(w.scales[g]), (float)(code - 8), w.offsets ? __half2float(w.offsets[g]) : 0.f);
    }
}

static Q4 q4_of(const bf_q4_matrix& W) {
    return Q4{W.codes, (const __half*)W.scales, (const __half*)W.offsets, W.row_bytes, W.group_stride, W.d_out, W.d_in, W.group};
}

cudaError_t bft::launch_q4_expand(const bf_q4_matrix& W, float* out, cudaStream_t stream) {
    q4_expand_kernel<<<dim3((W.d_in + 255) / 256, W.d_out < 65535 ? W.d_out : 65535), 256, 0, stream>>>(q4_of(W), out);
    return cudaGetLastError();
}

int bft::q4_check(const bf_q4_matrix* W) {
    if (!W || !W->codes || !W->scales || !W->d_out || !W->d_in) return BF_ERR_INVALID_ARG;
    if ((uintptr_t)W->codes % 16 || (uintptr_t)W->scales % 16 || (uintptr_t)W->offsets % 16) return BF_ERR_INVALID_ARG;
    if (W->group != 32 && W->group != 64 && W->group != 128) return BF_ERR_SHAPE;
    const uint32_t groups = W->d_in / W->group + (W->d_in % W->group != 0);
    if (W->row_bytes % 16 || W->row_bytes < W->d_in / 2 + W->d_in % 2 || W->group_stride % 8 || W->group_stride < groups) return BF_ERR_SHAPE;
    // rows are counted in 31 bits, and the tail of a stage of columns behind d_in stays in them too
    return W->d_out >= (1u << 31) - 4096 || W->d_in >= (1u << 31) - 4096 || W->row_bytes >= (1ull << 32) ? BF_ERR_SHAPE : BF_OK;
}

extern "C" int bf_q4_linear(bf_trusted* t, const bf_q4_matrix* W, const bf_rows* x, uint32_t n, const bf_rows* y) {
    if (!t || !n || !rows_ok(x) || !rows_ok(y)) return BF_ERR_INVALID_ARG;
    if (int rc = q4_check(W)) return rc;
    if (n >= (1u << 31)) return BF_ERR_SHAPE;
    OnDevice on(t->device);
    if (!on.ok) return cuda_failed(t, "cudaSetDevice", cudaErrorInvalidDevice);
    const Q4 w = q4_of(*W);
    switch (W->group) {
        case 32: return W->offsets ? linear<32, true>(t, w, *x, n, *y) : linear<32, false>(t, w, *x, n, *y);
        case 64: return W->offsets ? linear<64, true>(t, w, *x, n, *y) : linear<64, false>(t, w, *x, n, *y);
        default: return W->offsets ? linear<128, true>(t, w, *x, n, *y) : linear<128, false>(t, w, *x, n, *y);
    }
}
