// Quantising to blocks of 8-bit floating point: rows on their way to the experts (pgmoe_quantize_rows) and the experts
// themselves (pgmoe_quantize_weights).  Both read and write each byte once and are bound by memory.
#include "fp8.h"

namespace pgmoe {

struct QuantizeRowsArgs {
    const void *x;
    size_t x_stride;
    int T, cols;
    const int32_t *row_of;
    int copies;
    uint8_t *q;
    size_t q_stride;
    float *scale;
    size_t scale_stride;
    int rows;
};

// Sixteen lanes take the 128 columns of one block, eight each; a workgroup takes the same block of 16 consecutive rows, whose
// scales are neighbours in memory.  The hardware deals workgroups out to the eight dies in turn: every eighth one goes through the blocks
// of the same rows, so that one L2 holds what neighbouring blocks share of a line.  8191 x 4096 float32 take 30.0 us (5.6 TB/s read
// and written; a plain copy on this chip 4.8), 4097 x 3000 10.8.  In the grid's order, all rows of a block first: 37.2 and 12.4; all
// blocks of 16 rows first: 29.5 and 12.2.
constexpr int QR_THREADS = 256, QR_ROWS = QR_THREADS / 16;
template <typename L, int Q, bool VEC>
__global__ __launch_bounds__(QR_THREADS) void quantize_rows_kernel(const QuantizeRowsArgs a) {
    const unsigned blocks = fp8_blocks(a.cols), n = blockIdx.x / 8, eighth = n / blocks;
    const int lane = threadIdx.x & 15, b = n - eighth * blocks;
    const int64_t t = (int64_t)(eighth * 8 + blockIdx.x % 8) * QR_ROWS + (threadIdx.x >> 4);
    if (t >= a.T) return;  // whole groups of 16 lanes
    float v[8];
    load_eight<L, VEC>(reinterpret_cast<const L *>(a.x) + t * a.x_stride, b * FP8_BLOCK + lane * 8, a.cols, v);
    auto largest = [&](auto of) {
        float l = of(v[0]);
#pragma unroll
        for (int j = 1; j < 8; ++j) l = maximum(l, of(v[j]));
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) l = maximum(l, __shfl_xor(l, m));
        return l;
    };
    float amax = largest([](float x) { return fabsf(x); });
    const bool unusual = fp8_unusual<Q>(amax);
    if (unusual) amax = largest(finite_magnitude);
    const float scale = fp8_scale<Q>(amax);
    auto quantise = [&](auto by) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = by(v[j]);
    };
    if (unusual) quantise(Fp8CarefulDivisor(scale));
    else quantise(Fp8Divisor(scale));
    const uint2 codes = make_uint2(fp8_pack<Q>(v[0], v[1], v[2], v[3]), fp8_pack<Q>(v[4], v[5], v[6], v[7]));
    for (int j = 0; j < a.copies; ++j) {
        const int r = a.row_of ? a.row_of[t * a.copies + j] : (int)t;
        if (r < 0 || r >= a.rows) continue;
        *reinterpret_cast<uint2 *>(a.q + (size_t)r * a.q_stride + b * FP8_BLOCK + lane * 8) = codes;
        if (lane == 0) a.scale[(size_t)b * a.scale_stride + r] = scale;
    }
}

struct QuantizeWeightsArgs {
    const void *w;
    int n_in, n_out;
    uint8_t *fwd_q, *bwd_q;
    float *fwd_scale, *bwd_scale;
};

// One workgroup takes one 128 x 128 block of one expert and keeps it in registers: a thread has two patches of four inputs by
// eight outputs, so that four inputs of an output are one dword of the forward tiles, and eight outputs of an input two of the
// backward ones.  Both go out through LDS as whole tiles.  The forward image has 16 bytes more behind each tile: the 64 dwords a
// wavefront writes at once are then on 64 banks.  128 experts of 1024 x 4096 bfloat16 in both orientations take 417 us, 5.15 TB/s read and
// written, either order of the blocks; 8 of 512 x 2048 float32 in one 9.1.
constexpr int QW_THREADS = 256;
constexpr int QW_TILE = FP8_TILE + 16;
template <typename L, bool VEC>
__global__ __launch_bounds__(QW_THREADS) void quantize_weights_kernel(const QuantizeWeightsArgs a) {
    __shared__ __attribute__((aligned(16))) char image[8 * QW_TILE];
    __shared__ float wave_max[QW_THREADS / 64];
    const int kb = blockIdx.x, nb = blockIdx.y, e = blockIdx.z;
    const int KB = gridDim.x, NB = gridDim.y;
    const int nq = threadIdx.x & 15, kq = threadIdx.x >> 4;
    const L *w = reinterpret_cast<const L *>(a.w) + (size_t)e * a.n_in * a.n_out;
    float v[8][8];  // [patch * 4 + input][output]
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int in = kb * FP8_BLOCK + (i >> 2) * 64 + kq * 4 + (i & 3);
        load_eight<L, VEC>(w + (size_t)min(in, a.n_in - 1) * a.n_out, nb * FP8_BLOCK + nq * 8, in < a.n_in ? a.n_out : 0, v[i]);
    }
    auto largest = [&](auto of) {
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) l = maximum(l, of(v[i][j]));
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) l = maximum(l, __shfl_xor(l, m));
        if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = l;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < QW_THREADS / 64; ++i) l = maximum(l, wave_max[i]);
        return l;
    };
    float amax = largest([](float x) { return fabsf(x); });
    const bool unusual = fp8_unusual<PGMOE_E4M3>(amax);  // the same in every wavefront
    if (unusual) {
        __syncthreads();
        amax = largest(finite_magnitude);
    }
    const float scale = fp8_scale<PGMOE_E4M3>(amax);
    auto quantise = [&](auto by) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = by(v[i][j]);
    };
    if (unusual) quantise(Fp8CarefulDivisor(scale));
    else quantise(Fp8Divisor(scale));
    if (a.fwd_q) {
        const int o0 = nq * 8;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int o = o0 + j, quad = p * 16 + kq;  // inputs 4 * quad ..
                *reinterpret_cast<uint32_t *>(image + (o >> 4) * QW_TILE + (quad >> 2) * 256 + (o & 15) * 16 + (quad & 3) * 4) =
                    fp8_pack<PGMOE_E4M3>(v[p * 4][j], v[p * 4 + 1][j], v[p * 4 + 2][j], v[p * 4 + 3][j]);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * QW_THREADS + threadIdx.x, tile = at >> 7, in_tile = (at & 127) * 16;
            *reinterpret_cast<uint4 *>(a.fwd_q + ((((size_t)e * NB + nb) * 8 + tile) * KB + kb) * FP8_TILE + in_tile) =
                *reinterpret_cast<const uint4 *>(image + tile * QW_TILE + in_tile);
        }
        if (threadIdx.x == 0) a.fwd_scale[((size_t)e * NB + nb) * KB + kb] = scale;
    }
    if (a.bwd_q) {
        if (a.fwd_q) __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int in = (i >> 2) * 64 + kq * 4 + (i & 3);
            uint2 codes;
            codes.x = fp8_pack<PGMOE_E4M3>(v[i][0], v[i][1], v[i][2], v[i][3]);
            codes.y = fp8_pack<PGMOE_E4M3>(v[i][4], v[i][5], v[i][6], v[i][7]);
            *reinterpret_cast<uint2 *>(image + (in >> 4) * QW_TILE + (nq >> 1) * 256 + (in & 15) * 16 + (nq & 1) * 8) = codes;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * QW_THREADS + threadIdx.x, tile = at >> 7, in_tile = (at & 127) * 16;
            *reinterpret_cast<uint4 *>(a.bwd_q + ((((size_t)e * KB + kb) * 8 + tile) * NB + nb) * FP8_TILE + in_tile) =
                *reinterpret_cast<const uint4 *>(image + tile * QW_TILE + in_tile);
        }
        if (threadIdx.x == 0) a.bwd_scale[((size_t)e * KB + kb) * NB + nb] = scale;
    }
}

static int64_t quantize_rows_grid(int T, int cols) { return ((int64_t)T + 8 * QR_ROWS - 1) / (8 * QR_ROWS) * 8 * fp8_blocks(cols); }
template <typename L, int Q>
static void launch_quantize_rows(const QuantizeRowsArgs &a, hipStream_t s) {
    const dim3 grid(quantize_rows_grid(a.T, a.cols));
    const bool vec = aligned(a.x, 16) && a.cols % 8 == 0 && a.x_stride * sizeof(L) % 16 == 0;
    if (vec) hipLaunchKernelGGL((quantize_rows_kernel<L, Q, true>), grid, dim3(QR_THREADS), 0, s, a);
    else hipLaunchKernelGGL((quantize_rows_kernel<L, Q, false>), grid, dim3(QR_THREADS), 0, s, a);
}
template <typename L>
static void launch_quantize_rows(const QuantizeRowsArgs &a, int dtype, hipStream_t s) {
    if (dtype == PGMOE_E4M3) launch_quantize_rows<L, PGMOE_E4M3>(a, s);
    else launch_quantize_rows<L, PGMOE_E5M2>(a, s);
}
template <typename L>
static void launch_quantize_weights(const QuantizeWeightsArgs &a, int E, hipStream_t s) {
    const dim3 grid(fp8_blocks(a.n_in), fp8_blocks(a.n_out), E);
    const bool vec = aligned(a.w, 16) && a.n_out % 8 == 0;
    if (vec) hipLaunchKernelGGL((quantize_weights_kernel<L, true>), grid, dim3(QW_THREADS), 0, s, a);
    else hipLaunchKernelGGL((quantize_weights_kernel<L, false>), grid, dim3(QW_THREADS), 0, s, a);
}

}  // namespace pgmoe

using namespace pgmoe;

extern "C" {

int pgmoe_quantize_rows(const void *x, int64_t x_stride, int x_dtype, int T, const int32_t *row_of, int copies,
                        const pgmoe_fp8_rows *out, void *stream) {
    const char *fn = "pgmoe_quantize_rows";
    int rc = check_fp8_rows(out, fn, "out");
    if (!rc) rc = check_float_type(x_dtype, fn, "x_dtype");
    if (rc) return rc;
    if (T < 0 || copies < 1) return fail(nullptr, PGMOE_EINVAL, "%s: T=%d, copies=%d: 0 and 1 at least", fn, T, copies);
    if (!row_of && (copies != 1 || T > out->rows))
        return fail(nullptr, PGMOE_EINVAL, "%s: without row_of copies is 1 (got %d) and T at most out->rows (got %d of %d)", fn, copies, T, out->rows);
    if (x_stride < out->cols) return fail(nullptr, PGMOE_EINVAL, "%s: x_stride=%lld is less than out->cols=%d", fn, (long long)x_stride, out->cols);
    if (T == 0 || out->rows == 0) return PGMOE_OK;
    if (quantize_rows_grid(T, out->cols) * QR_THREADS > GRID_THREADS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "%s: T=%d rows of %d columns are more than one launch holds", fn, T, out->cols);
    NEED_PTR(nullptr, fn, x, dtype_bytes(x_dtype));
    OPT_PTR(nullptr, fn, row_of, 4);
    const QuantizeRowsArgs a = {x, (size_t)x_stride, T, out->cols, row_of, copies, (uint8_t *)out->q, (size_t)out->q_stride, out->scale,
                                (size_t)out->scale_stride, out->rows};
    if (x_dtype == PGMOE_F32) launch_quantize_rows<float>(a, out->dtype, (hipStream_t)stream);
    else if (x_dtype == PGMOE_BF16) launch_quantize_rows<__bf16>(a, out->dtype, (hipStream_t)stream);
    else launch_quantize_rows<_Float16>(a, out->dtype, (hipStream_t)stream);
    return launched(fn);
}

int pgmoe_quantize_weights(const void *w, int w_dtype, const pgmoe_fp8_weights *forward, const pgmoe_fp8_weights *backward, void *stream) {
    const char *fn = "pgmoe_quantize_weights";
    int rc = check_float_type(w_dtype, fn, "w_dtype");
    if (!rc && !forward && !backward) rc = fail(nullptr, PGMOE_EINVAL, "%s: both forward and backward are NULL", fn);
    if (!rc && forward) rc = check_fp8_weights(forward, fn, "forward");
    if (!rc && backward) rc = check_fp8_weights(backward, fn, "backward");
    if (rc) return rc;
    const int E = forward ? forward->n_experts : backward->n_experts;
    const int n_in = forward ? forward->n_in : backward->n_out, n_out = forward ? forward->n_out : backward->n_in;
    if (forward && backward && (backward->n_experts != E || backward->n_in != n_out || backward->n_out != n_in))
        return fail(nullptr, PGMOE_EINVAL, "%s: backward is %d x (%d, %d), not the transpose of forward's %d x (%d, %d)", fn, backward->n_experts,
                    backward->n_in, backward->n_out, E, n_in, n_out);
    NEED_PTR(nullptr, fn, w, dtype_bytes(w_dtype));
    const QuantizeWeightsArgs a = {w, n_in, n_out, forward ? (uint8_t *)forward->q : nullptr, backward ? (uint8_t *)backward->q : nullptr,
                                   forward ? forward->scale : nullptr, backward ? backward->scale : nullptr};
    if (w_dtype == PGMOE_F32) launch_quantize_weights<float>(a, E, (hipStream_t)stream);
    else if (w_dtype == PGMOE_BF16) launch_quantize_weights<__bf16>(a, E, (hipStream_t)stream);
    else launch_quantize_weights<_Float16>(a, E, (hipStream_t)stream);
    return launched(fn);
}

}  // extern "C"
