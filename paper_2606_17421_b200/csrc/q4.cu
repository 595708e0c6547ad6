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

constexpr unsigned WARPS = 8;

// One warp a row of W and row of x: sum_g s_g sum_c x_c (code_c - 8) + z_g sum_c x_c, in fp32.
__global__ void __launch_bounds__(WARPS * 32) q4_linear_kernel(Q4 w, bf_rows x, unsigned n, bf_rows y) {
    const unsigned o = blockIdx.x * WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (o >= w.d_out) return;
    for (unsigned i = blockIdx.y; i < n; i += gridDim.y) {
        float sum = 0;
        for (unsigned c0 = lane * 8; c0 < w.d_in; c0 += 256) {
            const uint32_t word = *reinterpret_cast<const uint32_t*>(w.codes + o * w.row_bytes + c0 / 2);
            const size_t g = (size_t)o * w.group_stride + c0 / w.group;
            float a = 0, b = 0;
            for (unsigned k = 0; k < 8 && c0 + k < w.d_in; ++k) {
                const float v = load_as_float(x.data, x.type, (int64_t)i * x.row_stride + c0 + k);
                a += v * (float)((int)(word >> (4 * k) & 15) - 8);
                b += v;
            }
            sum += __half2float(w.scales[g]) * a;
            if (w.offsets) sum += __half2float(w.offsets[g]) * b;
        }
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (lane == 0) store_from_float(y.data, y.type, (int64_t)i * y.row_stride + o, sum);
    }
}

}  // namespace

extern "C" int bf_q4_linear(bf_trusted* t, const bf_q4_matrix* W, const bf_rows* x, uint32_t n, const bf_rows* y) {
    if (!t || !W || !n || !rows_ok(x) || !rows_ok(y) || !W->codes || !W->scales || !W->d_out || !W->d_in) return BF_ERR_INVALID_ARG;
    if ((uintptr_t)W->codes % 16 || (uintptr_t)W->scales % 16 || (uintptr_t)W->offsets % 16) return BF_ERR_INVALID_ARG;
    if (W->group != 32 && W->group != 64 && W->group != 128) return BF_ERR_SHAPE;
    const uint32_t groups = W->d_in / W->group + (W->d_in % W->group != 0);
    if (W->row_bytes % 16 || W->row_bytes < W->d_in / 2 + W->d_in % 2 || W->group_stride % 8 || W->group_stride < groups) return BF_ERR_SHAPE;
    // rows are counted in 31 bits, and the tail of a stage of columns behind d_in stays in them too
    if (n >= (1u << 31) || W->d_out >= (1u << 31) - 4096 || W->d_in >= (1u << 31) - 4096 || W->row_bytes >= (1ull << 32)) return BF_ERR_SHAPE;
    OnDevice on(t->device);
    if (!on.ok) return cuda_failed(t, "cudaSetDevice", cudaErrorInvalidDevice);
    const Q4 w{W->codes, (const __half*)W->scales, (const __half*)W->offsets, W->row_bytes, W->group_stride, W->d_out, W->d_in, W->group};
    q4_linear_kernel<<<dim3((W->d_out + WARPS - 1) / WARPS, n < 65535 ? n : 65535), WARPS * 32, 0, t->stream>>>(w, *x, n, *y);
    return launched(t, "q4_linear_kernel");
}
