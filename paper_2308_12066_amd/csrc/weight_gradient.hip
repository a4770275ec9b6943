// Gradient of the experts' matrices from rows kept in 8 bits (pgmoe_expert_weight_gradient).
//
//   d_w[e, i, o] = add[e, i, o] + sum over the rows r of expert e of  x[r, i] d_y[r, o],   x[r, i] = code[r, i] * scale[r, i / 128]
//
// The scales of x vary along the sum, so they cannot be taken out of it: the matrix cores' operand is code times scale.  Where scales are
// powers of two that is a bfloat16 as it stands (four bits), and one product a row, input and output is exact.  Otherwise code times scale in 32
// bits is taken apart into three bfloat16 whose sum it is, and so are gradients of 32 bits; those of 16-bit floating point are the sum of two.
#include <atomic>

#include "ffn_common.h"
#include "fp8.h"

namespace pgmoe {

struct GradientArgs {
    const uint8_t *x;
    size_t x_stride;
    const float *x_scale;
    size_t x_scale_stride;
    int rows, n_in, n_out, E;
    const void *d_y;
    size_t d_y_stride;
    const int32_t *offsets;
    const void *add;  // | nullptr
    void *d_w;
    int dtype;  // of d_w and add
    int tiles_in, tiles_out;
};

typedef int intx2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// PIECES bfloat16 whose sum is v but for a part in 2^32 (of two: 16 bits, of three: 24).  All have v's sign and none is zero if v is not, so
// that an infinity times each of them is the infinity that it times v is: pieces are cut off, not rounded, and what is left of v is
// raised by that part.  (Products of pieces that are left out are below 2^-20 of the first, on the mean 2^-23.)
__device__ inline uint32_t high_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }
template <int PIECES>
__device__ inline void take_apart(const float (&v)[8], uint4 (&to)[PIECES]) {
    float rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) rest[j] = __builtin_canonicalizef(v[j]);  // NaN: with a bit that is not cut off
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        to[p] = make_uint4(high_halves(rest[0], rest[1]), high_halves(rest[2], rest[3]), high_halves(rest[4], rest[5]), high_halves(rest[6], rest[7]));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float left = fmaf(v[j], 0x1p-32f, rest[j] - __uint_as_float(__float_as_uint(rest[j]) & 0xffff0000u));
            rest[j] = fabsf(v[j]) < INFINITY ? left : rest[j];
        }
    }
}

// Eight codes times their scale.
template <int Q, int PIECES>
__device__ inline void open_codes(intx2 codes, float scale, uint4 (&to)[PIECES]) {
    if constexpr (PIECES == 1) {  // the conversion takes the scale's exponent
        uint32_t pairs[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x2 pair;
            if constexpr (Q == PGMOE_E4M3)
                pair = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j >> 1], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j >> 1], scale, false);
            else pair = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[j >> 1], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[j >> 1], scale, false);
            pairs[j] = __builtin_bit_cast(uint32_t, pair);
        }
        to[0] = make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]);
    } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            floatx2 pair;
            if constexpr (Q == PGMOE_E4M3) pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(codes[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(codes[j >> 1], false);
            else pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_bf8(codes[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_bf8(codes[j >> 1], false);
            v[2 * j] = pair[0] * scale;
            v[2 * j + 1] = pair[1] * scale;
        }
        take_apart<PIECES>(v, to);
    }
}

// Four rows of 16 neighbouring bfloat16 columns in LDS, one row behind the other's `stride`, as a quarter of a wavefront's operand: lane i of 16 gives the
// address of four columns of row i / 4 and gets column i of all four.
__device__ inline shortx4 read_transposed(const char *at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)at);
}
// The operand of a lane: column lane % 16 and eight of 32 rows.  Which rows a lane takes is free as long as both operands agree: 4 * (lane / 16) ..
// and 16 + 4 * (lane / 16) ..
__device__ inline bf16x8 operand_of(const char *tile, int stride, int lane) {
    const char *at = tile + (size_t)((lane >> 4) * 4 + (lane >> 2 & 3)) * stride + (lane & 3) * 8;
    const shortx4 low = read_transposed(at), high = read_transposed(at + 16 * stride);
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, shortx8{low[0], low[1], low[2], low[3], high[0], high[1], high[2], high[3]});
}

template <typename Y>
constexpr int pieces_of = sizeof(Y) == 4 ? 3 : std::is_same<Y, __bf16>::value ? 1 : 2;

// A workgroup takes 128 inputs by 128 outputs of one expert and goes through its rows 32 at a time: both sides come through registers, where codes are
// converted, into one of two buffers in LDS while the other is multiplied.  Rows in LDS have 32 bytes more behind them than their 128 columns: the eight rows of 32
// bytes that half a wavefront reads at once then lie in different banks.
constexpr int WG_TILE = 128, WG_K = 32, WG_THREADS = 256, WG_STRIDE = 2 * WG_TILE + 32, WG_PLANE = WG_K * WG_STRIDE;
template <int XQ, typename Y, int PX, bool VEC>
__global__ __launch_bounds__(WG_THREADS) void weight_gradient_kernel(const GradientArgs a) {
    constexpr int PY = pieces_of<Y>, BUFFER = (PX + PY) * WG_PLANE, KEPT = PX > PY ? PX : PY;  // KEPT: pieces i and j are multiplied where i + j < KEPT
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e = blockIdx.x / (a.tiles_in * a.tiles_out), tile = blockIdx.x - e * a.tiles_in * a.tiles_out, ti = tile / a.tiles_out, to = tile - ti * a.tiles_out;
    const int lo = max(0, min(a.offsets[e], a.rows)), hi = max(lo, min(a.offsets[e + 1], a.rows)), steps = (hi - lo + WG_K - 1) / WG_K;

    // what a thread brings: eight columns of rows threadIdx.x / 16 and 16 + threadIdx.x / 16 of a step
    const int piece = threadIdx.x & 15, row = threadIdx.x >> 4;
    const uint8_t *x = a.x + (size_t)ti * WG_TILE + piece * 8;
    const float *x_scale = a.x_scale + (size_t)ti * a.x_scale_stride;
    const int col = min(to * WG_TILE + piece * 8, VEC ? a.n_out - 8 : a.n_out - 1);  // columns past the last are there, but nobody's
    const Y *d_y = reinterpret_cast<const Y *>(a.d_y);
    intx2 codes[2];
    float scale[2];
    struct { Y v[8]; } grad[2];
    bool there[2];
    auto request = [&](int step) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = lo + step * WG_K + i * 16 + row;
            there[i] = r < hi;
            const size_t at = there[i] ? r : hi - 1;
            codes[i] = *reinterpret_cast<const intx2 *>(x + at * a.x_stride);
            scale[i] = x_scale[at];
            const Y *g = d_y + at * a.d_y_stride;
            if constexpr (VEC) {
                typedef Y Yx8 __attribute__((ext_vector_type(8), aligned(16)));
                *reinterpret_cast<Yx8 *>(grad[i].v) = *reinterpret_cast<const Yx8 *>(g + col);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) grad[i].v[j] = g[min(col + j, a.n_out - 1)];
            }
        }
    };
    auto keep = [&](char *to) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            char *at = to + (i * 16 + row) * WG_STRIDE + piece * 16;
            const uint4 none = make_uint4(0, 0, 0, 0);
            uint4 px[PX], py[PY];
            open_codes<XQ, PX>(codes[i], scale[i], px);
            if constexpr (PY == 1) {
                py[0] = __builtin_bit_cast(uint4, grad[i]);
            } else {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)grad[i].v[j];
                take_apart<PY>(v, py);
            }
            // rows behind the last are zero on both sides, whatever the last one holds
#pragma unroll
            for (int p = 0; p < PX; ++p) *reinterpret_cast<uint4 *>(at + p * WG_PLANE) = there[i] ? px[p] : none;
#pragma unroll
            for (int p = 0; p < PY; ++p) *reinterpret_cast<uint4 *>(at + (PX + p) * WG_PLANE) = there[i] ? py[p] : none;
        }
    };

    // wavefronts as 2 x 2, each with 64 inputs and 64 outputs.  Gradients are the first operand: a lane's four results of a product are neighbouring outputs of one input.
    const int wi = wave >> 1, wo = wave & 1;
    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 0; o < 4; ++o) acc[i][o] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (steps > 0) {
        request(0);
        keep(lds);
    }
    for (int step = 0; step < steps; ++step) {
        lds_barrier();  // this step's rows are there for everyone, and everyone has read the one before
        const bool more = step + 1 < steps;
        if (more) request(step + 1);
        __builtin_amdgcn_sched_barrier(0);
        const char *now = lds + (step & 1) * BUFFER;
        bf16x8 px[4][PX];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int p = 0; p < PX; ++p) px[i][p] = operand_of(now + p * WG_PLANE + (wi * 64 + i * 16) * 2, WG_STRIDE, lane);
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            bf16x8 py[PY];
#pragma unroll
            for (int p = 0; p < PY; ++p) py[p] = operand_of(now + (PX + p) * WG_PLANE + (wo * 64 + o * 16) * 2, WG_STRIDE, lane);
            // small products first
#pragma unroll
            for (int s = KEPT - 1; s >= 0; --s)
#pragma unroll
                for (int p = 0; p < PY; ++p)
                    if (s - p >= 0 && s - p < PX) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(py[p], px[i][s - p >= 0 && s - p < PX ? s - p : 0], acc[i][o], 0, 0, 0);
                    }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) keep(lds + ((step + 1) & 1) * BUFFER);
    }

    auto finish = [&](auto type) {
        using W = decltype(type);
        typedef W Wx4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int in = ti * WG_TILE + wi * 64 + i * 16 + (lane & 15);
            if (in >= a.n_in) continue;
            const size_t first = ((size_t)e * a.n_in + in) * a.n_out;
#pragma unroll
            for (int o = 0; o < 4; ++o) {
                const int out = to * WG_TILE + wo * 64 + o * 16 + 4 * (lane >> 4);
                W *p = reinterpret_cast<W *>(a.d_w) + first + out;
                const W *q = reinterpret_cast<const W *>(a.add) + first + out;
                floatx4 v = acc[i][o];
                if (VEC) {
                    if (out >= a.n_out) continue;
                    if (a.add) {
                        const Wx4 u = *reinterpret_cast<const Wx4 *>(q);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] += (float)u[j];
                    }
                    *reinterpret_cast<Wx4 *>(p) = Wx4{(W)v[0], (W)v[1], (W)v[2], (W)v[3]};
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (out + j < a.n_out) p[j] = (W)(a.add ? v[j] + (float)q[j] : v[j]);
                }
            }
        }
    };
    if (a.dtype == PGMOE_F32) finish(float());
    else if (a.dtype == PGMOE_BF16) finish(__bf16());
    else finish(_Float16());
}

template <int XQ, typename Y, int PX, bool VEC>
static int launch_gradient(const GradientArgs &a, hipStream_t s) {
    constexpr int LDS = 2 * (PX + pieces_of<Y>) * WG_PLANE;
    if (LDS > 48 * 1024) {  // the kernel's limit is raised once per device
        static std::atomic<uint64_t> raised{0};
        int device = 0;
        if (const hipError_t e = hipGetDevice(&device))
            return e == hipErrorNoDevice ? fail(nullptr, PGMOE_ENODEVICE, "pgmoe_expert_weight_gradient: no HIP device is visible") : hip_fail(nullptr, e, "hipGetDevice");
        if (!(raised.load(std::memory_order_relaxed) >> (device & 63) & 1)) {
            PG_HIP(nullptr, hipFuncSetAttribute(reinterpret_cast<const void *>(&weight_gradient_kernel<XQ, Y, PX, VEC>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
            raised.fetch_or(1ull << (device & 63), std::memory_order_relaxed);
        }
    }
    hipLaunchKernelGGL((weight_gradient_kernel<XQ, Y, PX, VEC>), dim3((unsigned)((int64_t)a.E * a.tiles_in * a.tiles_out)), dim3(WG_THREADS), LDS, s, a);
    return PGMOE_OK;
}
template <int XQ, typename Y>
static int launch_gradient(const GradientArgs &a, bool pow2, hipStream_t s) {
    const bool vec = a.n_out % 8 == 0 && a.d_y_stride * sizeof(Y) % 16 == 0 && aligned(a.d_y, 16) && aligned(a.d_w, 16) && aligned(a.add, 16);
    if (pow2) return vec ? launch_gradient<XQ, Y, 1, true>(a, s) : launch_gradient<XQ, Y, 1, false>(a, s);
    return vec ? launch_gradient<XQ, Y, 3, true>(a, s) : launch_gradient<XQ, Y, 3, false>(a, s);
}
template <int XQ>
static int launch_gradient(const GradientArgs &a, int y_dtype, bool pow2, hipStream_t s) {
    if (y_dtype == PGMOE_F32) return launch_gradient<XQ, float>(a, pow2, s);
    if (y_dtype == PGMOE_BF16) return launch_gradient<XQ, __bf16>(a, pow2, s);
    return launch_gradient<XQ, _Float16>(a, pow2, s);
}

}  // namespace pgmoe

using namespace pgmoe;

extern "C" {

size_t pgmoe_expert_weight_gradient_workspace_bytes(int rows, int n_experts, int n_in, int n_out) { return 0; }

int pgmoe_expert_weight_gradient(const pgmoe_fp8_rows *x, const void *d_y, int64_t d_y_stride, int d_y_dtype, const int32_t *expert_offsets, int n_experts, int n_out,
                                 const void *add, void *d_w, int d_w_dtype, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "pgmoe_expert_weight_gradient";
    int rc = check_fp8_rows(x, fn, "x");
    if (!rc) rc = check_float_type(d_y_dtype, fn, "d_y_dtype");
    if (!rc) rc = check_float_type(d_w_dtype, fn, "d_w_dtype");
    if (rc) return rc;
    if (n_experts < 1 || n_experts > PGMOE_MAX_EXPERTS) return fail(nullptr, PGMOE_EINVAL, "%s: n_experts=%d outside 1..%d", fn, n_experts, PGMOE_MAX_EXPERTS);
    if (n_out < 1 || n_out > FP8_COLS_MAX) return fail(nullptr, PGMOE_EINVAL, "%s: n_out=%d outside 1..%d", fn, n_out, FP8_COLS_MAX);
    if (x->rows > (1 << 24)) return fail(nullptr, PGMOE_EINVAL, "%s: %d rows: at most 2^24", fn, x->rows);
    if (d_y_stride < n_out) return fail(nullptr, PGMOE_EINVAL, "%s: d_y_stride=%lld is less than n_out=%d", fn, (long long)d_y_stride, n_out);
    const int tiles_in = fp8_blocks(x->cols), tiles_out = (n_out + WG_TILE - 1) / WG_TILE;
    if ((int64_t)n_experts * tiles_in * tiles_out * WG_THREADS > GRID_THREADS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "%s: %d matrices of %d x %d are more than one launch holds", fn, n_experts, x->cols, n_out);
    if (x->rows > 0) NEED_PTR(nullptr, fn, d_y, dtype_bytes(d_y_dtype));
    NEED_PTR(nullptr, fn, expert_offsets, 4);
    NEED_PTR(nullptr, fn, d_w, dtype_bytes(d_w_dtype));
    OPT_PTR(nullptr, fn, add, dtype_bytes(d_w_dtype));
    GradientArgs a = {};
    a.x = (const uint8_t *)x->q;
    a.x_stride = (size_t)x->q_stride;
    a.x_scale = x->scale;
    a.x_scale_stride = (size_t)x->scale_stride;
    a.rows = x->rows;
    a.n_in = x->cols;
    a.n_out = n_out;
    a.E = n_experts;
    a.d_y = d_y;
    a.d_y_stride = (size_t)d_y_stride;
    a.offsets = expert_offsets;
    a.add = add;
    a.d_w = d_w;
    a.dtype = d_w_dtype;
    a.tiles_in = tiles_in;
    a.tiles_out = tiles_out;
    const bool pow2 = (x->dtype & PGMOE_SCALE_POW2) != 0;
    rc = fp8_type(x->dtype) == PGMOE_E4M3 ? launch_gradient<PGMOE_E4M3>(a, d_y_dtype, pow2, (hipStream_t)stream) : launch_gradient<PGMOE_E5M2>(a, d_y_dtype, pow2, (hipStream_t)stream);
    return rc ? rc : launched(fn);
}

}  // extern "C"
