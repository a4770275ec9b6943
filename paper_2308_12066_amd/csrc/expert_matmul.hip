// Rows grouped by expert through their experts' 8-bit matrices (pgmoe_expert_matmul).
//
//   y[r, o] = act( sum over blocks b of 128 inputs  sx[r, b] * sw[e, o / 128, b] * sum_{i in b} x[r, i] w[e, i, o] )
//
// The codes become bfloat16, which holds every value of both types, in registers and are multiplied there: four 16x16x32
// products cover the 128 inputs that share both scales, and their sums are taken over into the float32 accumulator with one
// multiply-add each.  Why not the matrix cores' own 8-bit products, at twice the rate: they add up the products of eight
// neighbouring inputs with 14 bits (beside a product of 1, one of 2^-14 is lost).  On normally distributed codes that is
// 1.3e-5 of a result, in every form (16x16x128, 16x16x32) and type, against 1e-8 through bfloat16: more than float32
// results may be off, and more than scales of the next blocks should be.
// The weights are the first operand, so that a lane's four results belong to one row: one product of the two scales serves
// them all, and they are neighbours in y.
#include "ffn_common.h"
#include "fp8.h"

namespace pgmoe {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct MatmulArgs {
    const uint8_t *x;
    size_t x_stride;
    const float *x_scale;
    size_t x_scale_stride;
    int rows, n_out, KB, NB, E;
    const uint8_t *w;
    const float *w_scale;
    const int32_t *offsets;
    int relu;
    void *y;
    size_t y_stride;
    uint8_t *y_q;
    size_t y_q_stride;
    float *y_scale;
    size_t y_scale_stride;
};

// The operand of a lane: 32 of the 128 inputs of row (or output) lane % 16.  Which ones a lane takes is free as long as both
// operands agree: the 16-byte pieces lane / 16 and 4 + lane / 16, the two halves of an operand tile.
struct Operand {
    bf16x8 part[4];
};
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <int Q>
__device__ inline bf16x2 widen(int codes, bool high) {
    return Q == PGMOE_E4M3 ? (high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false))
                           : (high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes, 1.f, false));
}
template <int Q>
__device__ inline bf16x8 widen(int a, int b) {
    const bf16x2 p = widen<Q>(a, false), q = widen<Q>(a, true), r = widen<Q>(b, false), s = widen<Q>(b, true);
    return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
template <int Q>
__device__ inline Operand operand(intx4 a, intx4 b) {
    return {{widen<Q>(a[0], a[1]), widen<Q>(a[2], a[3]), widen<Q>(b[0], b[1]), widen<Q>(b[2], b[3])}};
}

// Weights times rows over one block of inputs, from zero.
__device__ inline floatx4 product(const Operand &w, const Operand &x) {
    floatx4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[i], x.part[i], p, 0, 0, 0);
    return p;
}

// The rows of chunk number `chunk`, clamped to the rows there are whatever the offsets say.
__device__ inline ChunkInfo matmul_chunk(const MatmulArgs &a, int rows_per_chunk, int chunk) {
    ChunkInfo ci = find_chunk(a.offsets, a.E, rows_per_chunk, chunk);
    if (ci.row0 < 0 || ci.row0 >= a.rows) ci.nrows = 0;
    ci.nrows = min(ci.nrows, a.rows - ci.row0);
    return ci;
}

// Four results of row r, outputs o .. o + 3.
template <typename Y, bool VEC>
__device__ inline void store_four(const MatmulArgs &a, int r, int o, floatx4 v) {
    typedef Y Yx4 __attribute__((ext_vector_type(4)));
    Y *p = reinterpret_cast<Y *>(a.y) + (size_t)r * a.y_stride + o;
    if (VEC) {
        if (o < a.n_out) *reinterpret_cast<Yx4 *>(p) = Yx4{(Y)v[0], (Y)v[1], (Y)v[2], (Y)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (o + i < a.n_out) p[i] = (Y)v[i];
    }
}

// Few rows an expert.  A workgroup takes 16 rows and one block of 128 outputs, a wavefront 16 of them, operands straight from
// memory into registers.  Y = void: quantised again, YQ.
constexpr int FEW_THREADS = 512;
template <int XQ, typename Y, int YQ, bool VEC>
__global__ __launch_bounds__(FEW_THREADS) void matmul_few_rows_kernel(const MatmulArgs a) {
    __shared__ float amax_of[8][16];
    const int chunk = blockIdx.x / a.NB, nb = blockIdx.x - chunk * a.NB;
    const ChunkInfo ci = matmul_chunk(a, 16, chunk);
    if (ci.nrows <= 0) return;  // uniform over the workgroup
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = ci.row0 + min(lane & 15, ci.nrows - 1), piece = (lane >> 4) * 16;
    const uint8_t *x = a.x + (size_t)row * a.x_stride + piece;
    const uint8_t *w = a.w + (((size_t)ci.expert * a.NB + nb) * 8 + wave) * a.KB * FP8_TILE + lane * 16;
    const float *sx = a.x_scale + row, *sw = a.w_scale + ((size_t)ci.expert * a.NB + nb) * a.KB;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int kb = 0; kb < a.KB; ++kb) {
        const Operand wf = operand<PGMOE_E4M3>(*reinterpret_cast<const intx4 *>(w), *reinterpret_cast<const intx4 *>(w + 1024));
        const Operand xf = operand<XQ>(*reinterpret_cast<const intx4 *>(x), *reinterpret_cast<const intx4 *>(x + 64));
        const float s = *sx * sw[kb];
        const floatx4 p = product(wf, xf);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(s, p[i], acc[i]);
        w += FP8_TILE;
        x += FP8_BLOCK;
        sx += a.x_scale_stride;
    }
    if (a.relu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = acc[i] > 0.f || acc[i] != acc[i] ? acc[i] : 0.f;
    }
    const bool live = (lane & 15) < ci.nrows;
    const int o = nb * FP8_BLOCK + wave * 16 + 4 * (lane >> 4);
    if constexpr (std::is_void<Y>::value) {
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) amax = fmaxf(amax, finite_magnitude(acc[i]));
        amax = fmaxf(amax, __shfl_xor(amax, 16));
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        if (lane < 16) amax_of[wave][lane] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, amax_of[i][lane & 15]);
        const float scale = fp8_scale<YQ>(amax);
        if (live) {
            *reinterpret_cast<uint32_t *>(a.y_q + (size_t)row * a.y_q_stride + o) = fp8_pack<YQ>(acc[0] / scale, acc[1] / scale, acc[2] / scale, acc[3] / scale);
            if (wave == 0 && lane < 16) a.y_scale[(size_t)nb * a.y_scale_stride + row] = scale;
        }
    } else {
        if (live) store_four<Y, VEC>(a, row, o, acc);
    }
}

template <int XQ, typename Y, int YQ, bool VEC>
static void launch_matmul(const MatmulArgs &a, hipStream_t s) {
    // chunks: sum over the experts of ceil(rows / 16)
    const int64_t chunks = (a.rows + (int64_t)15 * std::min(a.E, a.rows)) / 16;
    hipLaunchKernelGGL((matmul_few_rows_kernel<XQ, Y, YQ, VEC>), dim3((unsigned)(chunks * a.NB)), dim3(FEW_THREADS), 0, s, a);
}
template <int XQ, typename Y>
static void launch_matmul_to(const MatmulArgs &a, hipStream_t s) {
    // whole fours of outputs, each at an address that four results' bytes divide
    if (a.n_out % 4 == 0 && a.y_stride % 4 == 0 && aligned(a.y, 4 * sizeof(Y))) launch_matmul<XQ, Y, 0, true>(a, s);
    else launch_matmul<XQ, Y, 0, false>(a, s);
}
template <int XQ>
static void launch_matmul(const MatmulArgs &a, int y_dtype, hipStream_t s) {
    switch (y_dtype) {
    case PGMOE_F32: return launch_matmul_to<XQ, float>(a, s);
    case PGMOE_BF16: return launch_matmul_to<XQ, __bf16>(a, s);
    case PGMOE_F16: return launch_matmul_to<XQ, _Float16>(a, s);
    case PGMOE_E4M3: return launch_matmul<XQ, void, PGMOE_E4M3, true>(a, s);
    default: return launch_matmul<XQ, void, PGMOE_E5M2, true>(a, s);
    }
}

}  // namespace pgmoe

using namespace pgmoe;

extern "C" int pgmoe_expert_matmul(const pgmoe_fp8_rows *x, const pgmoe_fp8_weights *w, const int32_t *expert_offsets, int relu, void *y,
                                   int64_t y_stride, int y_dtype, const pgmoe_fp8_rows *y_q, void *stream) {
    const char *fn = "pgmoe_expert_matmul";
    int rc = check_fp8_rows(x, fn, "x");
    if (!rc) rc = check_fp8_weights(w, fn, "w");
    if (rc) return rc;
    if (x->cols != w->n_in) return fail(nullptr, PGMOE_EINVAL, "%s: x has %d columns, w n_in=%d", fn, x->cols, w->n_in);
    if (x->rows > (1 << 24)) return fail(nullptr, PGMOE_EINVAL, "%s: %d rows: at most 2^24", fn, x->rows);
    if (relu != 0 && relu != 1) return fail(nullptr, PGMOE_EINVAL, "%s: relu=%d is neither 0 nor 1", fn, relu);
    if ((y != nullptr) == (y_q != nullptr) && !(x->rows == 0 && !y_q)) return fail(nullptr, PGMOE_EINVAL, "%s: exactly one of y and y_q is given", fn);
    if (y_q) {
        if ((rc = check_fp8_rows(y_q, fn, "y_q"))) return rc;
        if (y_q->rows != x->rows || y_q->cols != w->n_out)
            return fail(nullptr, PGMOE_EINVAL, "%s: y_q is %d x %d, the result %d x %d", fn, y_q->rows, y_q->cols, x->rows, w->n_out);
    } else {
        if ((rc = check_float_type(y_dtype, fn, "y_dtype"))) return rc;
        if (y_stride < w->n_out) return fail(nullptr, PGMOE_EINVAL, "%s: y_stride=%lld is less than n_out=%d", fn, (long long)y_stride, w->n_out);
    }
    if (x->rows == 0) return PGMOE_OK;
    // (chunk, block of outputs) items are numbered with 31 bits
    if ((x->rows / 16 + (int64_t)w->n_experts) * fp8_blocks(w->n_out) > 0x7fffffff)
        return fail(nullptr, PGMOE_EINVAL, "%s: %d rows by n_out=%d are more than one launch holds", fn, x->rows, w->n_out);
    if (y) NEED_PTR(nullptr, fn, y, dtype_bytes(y_dtype));
    NEED_PTR(nullptr, fn, expert_offsets, 4);
    MatmulArgs a = {};
    a.x = (const uint8_t *)x->q;
    a.x_stride = (size_t)x->q_stride;
    a.x_scale = x->scale;
    a.x_scale_stride = (size_t)x->scale_stride;
    a.rows = x->rows;
    a.n_out = w->n_out;
    a.KB = fp8_blocks(w->n_in);
    a.NB = fp8_blocks(w->n_out);
    a.E = w->n_experts;
    a.w = (const uint8_t *)w->q;
    a.w_scale = w->scale;
    a.offsets = expert_offsets;
    a.relu = relu;
    a.y = y;
    a.y_stride = (size_t)y_stride;
    if (y_q) {
        a.y_q = (uint8_t *)y_q->q;
        a.y_q_stride = (size_t)y_q->q_stride;
        a.y_scale = y_q->scale;
        a.y_scale_stride = (size_t)y_q->scale_stride;
        y_dtype = y_q->dtype;
    }
    if (x->dtype == PGMOE_E4M3) launch_matmul<PGMOE_E4M3>(a, y_dtype, (hipStream_t)stream);
    else launch_matmul<PGMOE_E5M2>(a, y_dtype, (hipStream_t)stream);
    return launched(fn);
}
