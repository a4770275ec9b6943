// Tokens to the rows of their experts and back, with weights and their gradients, and gradients through the ReLU between an
// expert's two products (pgmoe_dispatch_rows, pgmoe_combine_rows, pgmoe_combine_rows_backward, pgmoe_relu_backward).  All of
// them are bound by memory: every value is read and written once.
#include "fp8.h"

namespace pgmoe {

constexpr int ROWS_COLS = 64 * 8;  // columns a wavefront takes at once, eight a lane

// Where the values of a row go: as a type of their own, as codes, or both.
struct RowsOut {
    void *values;  // [rows, cols] | nullptr
    size_t stride;
    uint8_t *q;  // codes | nullptr
    size_t q_stride;
    float *scale;
    size_t scale_stride;
    int q_dtype;
    bool pow2;
};

// Eight consecutive elements of a row; columns from `cols` on are 0, or not written.  VEC: all eight exist and lie 16-byte aligned.  Otherwise they are still moved at once where
// all eight exist, wherever they lie (8191 tokens of 1217 bfloat16, two rows each, element by element 30.7 us, so 15.6).
template <typename L, bool VEC>
__device__ inline void load_columns(const L *p, int col, int cols, float (&v)[8]) {
    typedef L Lx8 __attribute__((ext_vector_type(8), aligned(sizeof(L))));
    if (!VEC && col + 8 <= cols) {
        const Lx8 x = *reinterpret_cast<const Lx8 *>(p + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
    } else {
        load_eight<L, VEC>(p, col, cols, v);
    }
}
template <typename L, bool VEC>
__device__ inline void store_columns(L *p, int col, int cols, const float (&v)[8]) {
    typedef L Lx8 __attribute__((ext_vector_type(8), aligned(VEC ? 16 : sizeof(L))));
    if (VEC ? col < cols : col + 8 <= cols) {
        Lx8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (L)v[j];
        *reinterpret_cast<Lx8 *>(p + col) = o;
    } else if (!VEC) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < cols) p[col + j] = (L)v[j];
    }
}

// The codes of a block whose 128 values 16 neighbouring lanes have (all lanes of the wavefront are here; v past the last column: 0).
template <int Q>
__device__ inline void store_codes(const RowsOut &out, int64_t r, int col, bool there, float (&v)[8]) {
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
    const float scale = fp8_scale<Q>(amax, out.pow2);
    auto quantise = [&](auto by) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = by(v[j]);
    };
    if (unusual) quantise(Fp8CarefulDivisor(scale));
    else quantise(Fp8Divisor(scale));
    if (!there) return;
    *reinterpret_cast<uint2 *>(out.q + (size_t)r * out.q_stride + col) = make_uint2(fp8_pack<Q>(v[0], v[1], v[2], v[3]), fp8_pack<Q>(v[4], v[5], v[6], v[7]));
    if ((threadIdx.x & 15) == 0) out.scale[(size_t)(col / FP8_BLOCK) * out.scale_stride + r] = scale;
}

template <typename Y, bool VEC, bool QUANT>
__device__ inline void store_row_part(const RowsOut &out, int64_t r, int col, int cols, bool row_there, float (&v)[8]) {
    if (out.values && row_there) store_columns<Y, VEC>(reinterpret_cast<Y *>(out.values) + (size_t)r * out.stride, col, cols, v);
    if constexpr (QUANT) {
        const bool there = row_there && col < fp8_blocks(cols) * FP8_BLOCK;
        if (out.q_dtype == PGMOE_E4M3) store_codes<PGMOE_E4M3>(out, r, col, there, v);
        else store_codes<PGMOE_E5M2>(out, r, col, there, v);
    }
}

struct DealArgs {
    const void *x;  // the tokens, or their gradients
    size_t x_stride;
    const int32_t *row_of;
    const float *weight;  // | nullptr: 1
    int n, copies, d, rows;
    RowsOut out;
    const void *dot;  // rows whose products with the tokens are summed up | nullptr
    size_t dot_stride;
    float *dot_out;  // [n]
};

// rows[row_of[i]] = weight[i] * x[i / copies], and dot_out[i] = <x[i / copies], dot[row_of[i]]>.  PARTS wavefronts an entry i: one, or for
// few entries four, which deal the columns out among themselves; a workgroup has four.
// Bound by memory: 16384 x 2048 float32 to eight bfloat16 rows each with weights and their gradients, 1.21 GB in 244 us, 4.9 TB/s (a copy: 5.2); 16384 x 1024 bfloat16 to two rows
// each as values and codes, 135 MB in 26 to 30 us; one token 2.2.  (More rounds of columns requested together changed nothing.)
template <typename X, typename Y, bool VEC, bool QUANT, int PARTS>
__global__ __launch_bounds__(256) void deal_rows_kernel(const DealArgs a) {
    __shared__ float sums[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, part = PARTS == 4 ? wave : 0;
    const int i = __builtin_amdgcn_readfirstlane(PARTS == 4 ? blockIdx.x : blockIdx.x * 4 + wave);
    if (i >= a.n) return;
    const int r = a.row_of[i];
    if (r < 0 || r >= a.rows) {  // uniform: a copy that was dropped
        if (a.dot_out && part == 0 && lane == 0) a.dot_out[i] = 0.f;
        return;
    }
    const float w = a.weight ? a.weight[i] : 1.f;
    const X *x = reinterpret_cast<const X *>(a.x) + (size_t)(i / a.copies) * a.x_stride;
    const Y *dot = a.dot ? reinterpret_cast<const Y *>(a.dot) + (size_t)r * a.dot_stride : nullptr;
    const int end = QUANT ? fp8_blocks(a.d) * FP8_BLOCK : a.d;
    float sum = 0.f;
    for (int c = part * ROWS_COLS; c < end; c += PARTS * ROWS_COLS) {
        const int col = c + lane * 8;
        float v[8];
        load_columns<X, VEC>(x, col, a.d, v);
        if (dot) {
            float u[8];
            load_columns<Y, VEC>(dot, col, a.d, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(v[j], u[j], sum);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= w;
        if (col + 8 > a.d) {  // weights that are not finite leave the columns past the last zero
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = col + j < a.d ? v[j] : 0.f;
        }
        store_row_part<Y, VEC, QUANT>(a.out, r, col, a.d, true, v);
    }
    if (a.dot_out) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (PARTS == 4) {
            if (lane == 0) sums[wave] = sum;
            __syncthreads();
            sum = sums[0] + sums[1] + sums[2] + sums[3];
        }
        if (part == 0 && lane == 0) a.dot_out[i] = sum;
    }
}

struct GatherArgs {
    const void *rows;
    size_t rows_stride;
    int n_rows;
    const int32_t *row_of;
    int copies;
    const float *weight;  // | nullptr: 1
    const void *add;      // | nullptr
    size_t add_stride;
    int T, d;
    void *y;
    size_t y_stride;
};

// y[t] = add[t] + sum over j of weight[t, j] * rows[row_of[t, j]], in ascending j; one wavefront a token and ROUNDS rounds of columns, which of a row
// are requested together.  Bound by memory: 16384 x 2048 bfloat16 from eight rows each, 605 MB, ROUNDS = 1 154 us, 4 129 (4.7 TB/s).  For up to 1024 tokens the rounds are
// workgroups of their own: 64 x 1024 with a residual 3.3 us.
template <typename R, typename Y, bool VEC, int ROUNDS>
__global__ __launch_bounds__(256) void gather_sum_kernel(const GatherArgs a) {
    const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
    if (t >= a.T) return;
    const int32_t *row_of = a.row_of + (size_t)t * a.copies;
    const float *weight = a.weight ? a.weight + (size_t)t * a.copies : nullptr;
    for (int c = blockIdx.y * ROUNDS * ROWS_COLS; c < a.d; c += gridDim.y * ROUNDS * ROWS_COLS) {
        const int col = c + lane * 8;
        float acc[ROUNDS][8];
#pragma unroll
        for (int q = 0; q < ROUNDS; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[q][i] = 0.f;
        for (int j = 0; j < a.copies; ++j) {
            const int r = row_of[j];
            if (r < 0 || r >= a.n_rows) continue;  // uniform
            const float w = weight ? weight[j] : 1.f;
            const R *row = reinterpret_cast<const R *>(a.rows) + (size_t)r * a.rows_stride;
            float v[ROUNDS][8];
#pragma unroll
            for (int q = 0; q < ROUNDS; ++q) load_columns<R, VEC>(row, col + q * ROWS_COLS, a.d, v[q]);
#pragma unroll
            for (int q = 0; q < ROUNDS; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[q][i] = fmaf(w, v[q][i], acc[q][i]);
        }
#pragma unroll
        for (int q = 0; q < ROUNDS; ++q) {
            const int at = col + q * ROWS_COLS;
            if (a.add) {
                float v[8];
                load_columns<Y, VEC>(reinterpret_cast<const Y *>(a.add) + (size_t)t * a.add_stride, at, a.d, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[q][i] += v[i];
            }
            store_columns<Y, VEC>(reinterpret_cast<Y *>(a.y) + (size_t)t * a.y_stride, at, a.d, acc[q]);
        }
    }
}

struct ReluArgs {
    const void *d_h;
    size_t d_h_stride;
    const uint8_t *h;  // codes of the ReLU's results
    size_t h_stride;
    int h_dtype, rows, cols;
    RowsOut out;
};

// Through the ReLU: zero where its result is (a code's sign bit set, or all others clear), also where the gradient is not finite; NaN among the
// results lets gradients through.  Bound by memory: 32768 x 4096 bfloat16 to bfloat16 and codes, 810 MB in 134 us, 6.0 TB/s; 128 x 4096 3.2 us.  Sixteen lanes a block of 128 columns, 16 rows a workgroup; every eighth workgroup goes through the blocks of the same rows.
constexpr int RELU_ROWS = 16;
template <typename X, typename Y, bool VEC, bool QUANT>
__global__ __launch_bounds__(256) void relu_backward_kernel(const ReluArgs a) {
    const unsigned blocks = fp8_blocks(a.cols), n = blockIdx.x / 8, eighth = n / blocks;
    const int lane = threadIdx.x & 15, col = (n - eighth * blocks) * FP8_BLOCK + lane * 8;
    const int64_t r = (int64_t)(eighth * 8 + blockIdx.x % 8) * RELU_ROWS + (threadIdx.x >> 4);
    if (r >= a.rows) return;  // whole groups of 16 lanes
    float v[8];
    load_columns<X, VEC>(reinterpret_cast<const X *>(a.d_h) + r * a.d_h_stride, col, a.cols, v);
    const uint2 h = *reinterpret_cast<const uint2 *>(a.h + r * a.h_stride + col);
    const uint32_t nan_from = a.h_dtype == PGMOE_E4M3 ? 0x7f : 0x7d;  // e5m2 has an infinity, 0x7c
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t code = (j < 4 ? h.x : h.y) >> (j % 4 * 8) & 0xff;
        const bool through = (code - 1 < 0x7f) || (code & 0x7f) >= nan_from;
        v[j] = through ? v[j] : 0.f;
    }
    store_row_part<Y, VEC, QUANT>(a.out, r, col, a.cols, true, v);
}

// ---- host side
template <typename F>
static void by_type(int dtype, F &&f) {
    if (dtype == PGMOE_F32) f(float());
    else if (dtype == PGMOE_BF16) f(__bf16());
    else f(_Float16());
}
static bool wide(const void *p, int64_t stride, int dtype) { return !p || (aligned(p, 16) && stride * (int64_t)dtype_bytes(dtype) % 16 == 0); }

static int check_matrix(const void *p, int64_t stride, int dtype, int cols, bool optional, const char *fn, const char *what) {
    if (!p && optional) return PGMOE_OK;
    if (!p) return fail(nullptr, PGMOE_EINVAL, "%s: %s is NULL", fn, what);
    if (!aligned(p, dtype_bytes(dtype))) return fail(nullptr, PGMOE_EINVAL, "%s: %s is not %d-byte aligned", fn, what, (int)dtype_bytes(dtype));
    if (stride < cols) return fail(nullptr, PGMOE_EINVAL, "%s: %s has rows %lld elements apart, fewer than the %d of one", fn, what, (long long)stride, cols);
    return PGMOE_OK;
}
static int check_deal(int T, int d, int copies, int n_rows, const char *fn) {
    if (T < 0 || copies < 1) return fail(nullptr, PGMOE_EINVAL, "%s: T=%d, copies=%d: 0 and 1 at least", fn, T, copies);
    if (d < 1 || d > FP8_COLS_MAX) return fail(nullptr, PGMOE_EINVAL, "%s: d=%d outside 1..%d", fn, d, FP8_COLS_MAX);
    if (n_rows < 0) return fail(nullptr, PGMOE_EINVAL, "%s: n_rows=%d is negative", fn, n_rows);
    if ((int64_t)T * copies > (GRID_THREADS_MAX - 255) / 64) return fail(nullptr, PGMOE_EINVAL, "%s: T=%d tokens by copies=%d are more than one launch holds", fn, T, copies);
    return PGMOE_OK;
}
static int check_codes(const pgmoe_fp8_rows *q, int rows, int cols, const char *fn, const char *what) {
    if (!q) return PGMOE_OK;
    const int rc = check_fp8_rows(q, fn, what);
    if (rc) return rc;
    if (q->rows != rows || q->cols != cols) return fail(nullptr, PGMOE_EINVAL, "%s: %s is %d x %d, the rows %d x %d", fn, what, q->rows, q->cols, rows, cols);
    return PGMOE_OK;
}
static RowsOut rows_out(void *values, int64_t stride, const pgmoe_fp8_rows *q) {
    RowsOut o = {values, (size_t)stride, nullptr, 0, nullptr, 0, 0, false};
    if (q) {
        o.q = (uint8_t *)q->q;
        o.q_stride = (size_t)q->q_stride;
        o.scale = q->scale;
        o.scale_stride = (size_t)q->scale_stride;
        o.q_dtype = fp8_type(q->dtype);
        o.pow2 = (q->dtype & PGMOE_SCALE_POW2) != 0;
    }
    return o;
}

static void launch_deal(const DealArgs &a, int x_dtype, int rows_dtype, bool vec, hipStream_t s) {
    by_type(x_dtype, [&](auto x_) {
        by_type(rows_dtype, [&](auto y_) {
            using X = decltype(x_);
            using Y = decltype(y_);
            auto go = [&](auto vec_, auto quant_) {
                constexpr bool VEC = decltype(vec_)::value, QUANT = decltype(quant_)::value;
                if (a.n <= 1024) hipLaunchKernelGGL((deal_rows_kernel<X, Y, VEC, QUANT, 4>), dim3(a.n), dim3(256), 0, s, a);
                else hipLaunchKernelGGL((deal_rows_kernel<X, Y, VEC, QUANT, 1>), dim3((a.n + 3) / 4), dim3(256), 0, s, a);
            };
            if (vec) a.out.q ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
            else a.out.q ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
        });
    });
}

}  // namespace pgmoe

using namespace pgmoe;

extern "C" {

int pgmoe_dispatch_rows(const void *x, int64_t x_stride, int x_dtype, int T, int d, const int32_t *row_of, int copies, const float *weight, void *rows,
                        int64_t rows_stride, int rows_dtype, int n_rows, const pgmoe_fp8_rows *rows_q, void *stream) {
    const char *fn = "pgmoe_dispatch_rows";
    int rc = check_deal(T, d, copies, n_rows, fn);
    if (!rc) rc = check_float_type(x_dtype, fn, "x_dtype");
    if (!rc) rc = check_float_type(rows_dtype, fn, "rows_dtype");
    if (!rc) rc = check_codes(rows_q, n_rows, d, fn, "rows_q");
    if (rc) return rc;
    if (T == 0 || n_rows == 0) return PGMOE_OK;
    if (!rows && !rows_q) return fail(nullptr, PGMOE_EINVAL, "%s: both rows and rows_q are NULL", fn);
    if ((rc = check_matrix(x, x_stride, x_dtype, d, false, fn, "x"))) return rc;
    if ((rc = check_matrix(rows, rows_stride, rows_dtype, d, true, fn, "rows"))) return rc;
    NEED_PTR(nullptr, fn, row_of, 4);
    OPT_PTR(nullptr, fn, weight, 4);
    const DealArgs a = {x, (size_t)x_stride, row_of, weight, T * copies, copies, d, n_rows, rows_out(rows, rows_stride, rows_q), nullptr, 0, nullptr};
    launch_deal(a, x_dtype, rows_dtype, d % 8 == 0 && wide(x, x_stride, x_dtype) && wide(rows, rows_stride, rows_dtype), (hipStream_t)stream);
    return launched(fn);
}

int pgmoe_combine_rows(const void *rows, int64_t rows_stride, int rows_dtype, int n_rows, const int32_t *row_of, int copies, const float *weight, const void *add,
                       int64_t add_stride, int T, int d, void *y, int64_t y_stride, int y_dtype, void *stream) {
    const char *fn = "pgmoe_combine_rows";
    int rc = check_deal(T, d, copies, n_rows, fn);
    if (!rc) rc = check_float_type(rows_dtype, fn, "rows_dtype");
    if (!rc) rc = check_float_type(y_dtype, fn, "y_dtype");
    if (rc) return rc;
    if (T == 0) return PGMOE_OK;
    if ((rc = check_matrix(rows, rows_stride, rows_dtype, d, n_rows == 0, fn, "rows"))) return rc;
    if ((rc = check_matrix(add, add_stride, y_dtype, d, true, fn, "add"))) return rc;
    if ((rc = check_matrix(y, y_stride, y_dtype, d, false, fn, "y"))) return rc;
    NEED_PTR(nullptr, fn, row_of, 4);
    OPT_PTR(nullptr, fn, weight, 4);
    const GatherArgs a = {rows, (size_t)rows_stride, n_rows, row_of, copies, weight, add, (size_t)add_stride, T, d, y, (size_t)y_stride};
    const bool vec = d % 8 == 0 && wide(rows, rows_stride, rows_dtype) && wide(add, add_stride, y_dtype) && wide(y, y_stride, y_dtype);
    const int rounds = (d + ROWS_COLS - 1) / ROWS_COLS, each = T > 1024 ? (rounds > 2 ? 4 : rounds) : 1;  // of a wavefront at once
    const dim3 grid((T + 3) / 4, T <= 1024 ? std::min(rounds, 1024) : 1);
    by_type(rows_dtype, [&](auto r_) {
        by_type(y_dtype, [&](auto y_) {
            using R = decltype(r_);
            using Y = decltype(y_);
            auto go = [&](auto vec_) {
                constexpr bool VEC = decltype(vec_)::value;
                if (each == 1) hipLaunchKernelGGL((gather_sum_kernel<R, Y, VEC, 1>), grid, dim3(256), 0, (hipStream_t)stream, a);
                else if (each == 2) hipLaunchKernelGGL((gather_sum_kernel<R, Y, VEC, 2>), grid, dim3(256), 0, (hipStream_t)stream, a);
                else hipLaunchKernelGGL((gather_sum_kernel<R, Y, VEC, 4>), grid, dim3(256), 0, (hipStream_t)stream, a);
            };
            vec ? go(std::true_type()) : go(std::false_type());
        });
    });
    return launched(fn);
}

int pgmoe_combine_rows_backward(const void *d_y, int64_t d_y_stride, int d_y_dtype, int T, int d, const void *rows, int64_t rows_stride, int rows_dtype, int n_rows,
                                const int32_t *row_of, int copies, const float *weight, void *d_rows, int64_t d_rows_stride, const pgmoe_fp8_rows *d_rows_q,
                                float *d_weight, void *stream) {
    const char *fn = "pgmoe_combine_rows_backward";
    int rc = check_deal(T, d, copies, n_rows, fn);
    if (!rc) rc = check_float_type(d_y_dtype, fn, "d_y_dtype");
    if (!rc) rc = check_float_type(rows_dtype, fn, "rows_dtype");
    if (!rc) rc = check_codes(d_rows_q, n_rows, d, fn, "d_rows_q");
    if (rc) return rc;
    if (T == 0) return PGMOE_OK;
    if (!d_rows && !d_rows_q && !d_weight) return fail(nullptr, PGMOE_EINVAL, "%s: d_rows, d_rows_q and d_weight are NULL", fn);
    if ((rc = check_matrix(d_y, d_y_stride, d_y_dtype, d, false, fn, "d_y"))) return rc;
    if ((rc = check_matrix(rows, rows_stride, rows_dtype, d, !d_weight || n_rows == 0, fn, "rows"))) return rc;
    if ((rc = check_matrix(d_rows, d_rows_stride, rows_dtype, d, true, fn, "d_rows"))) return rc;
    NEED_PTR(nullptr, fn, row_of, 4);
    OPT_PTR(nullptr, fn, weight, 4);
    OPT_PTR(nullptr, fn, d_weight, 4);
    if (!d_weight) rows = nullptr;
    const DealArgs a = {d_y, (size_t)d_y_stride, row_of, weight, T * copies, copies, d, n_rows, rows_out(d_rows, d_rows_stride, d_rows_q), rows, (size_t)rows_stride, d_weight};
    const bool vec = d % 8 == 0 && wide(d_y, d_y_stride, d_y_dtype) && wide(rows, rows_stride, rows_dtype) && wide(d_rows, d_rows_stride, rows_dtype);
    launch_deal(a, d_y_dtype, rows_dtype, vec, (hipStream_t)stream);
    return launched(fn);
}

int pgmoe_relu_backward(const void *d_h, int64_t d_h_stride, int d_h_dtype, int rows, int cols, const void *h_q, int64_t h_q_stride, int h_dtype, void *d_pre,
                        int64_t d_pre_stride, int d_pre_dtype, const pgmoe_fp8_rows *d_pre_q, void *stream) {
    const char *fn = "pgmoe_relu_backward";
    int rc = check_float_type(d_h_dtype, fn, "d_h_dtype");
    if (!rc) rc = check_float_type(d_pre_dtype, fn, "d_pre_dtype");
    if (rc) return rc;
    if (rows < 0 || cols < 1 || cols > FP8_COLS_MAX) return fail(nullptr, PGMOE_EINVAL, "%s: %d rows of %d columns: 0 and more of 1 to %d", fn, rows, cols, FP8_COLS_MAX);
    const pgmoe_fp8_rows h = {const_cast<void *>(h_q), h_q_stride, const_cast<float *>(reinterpret_cast<const float *>(h_q)), rows, rows, cols, h_dtype};
    if ((rc = check_fp8_rows(&h, fn, "h_q"))) return rc;
    if ((rc = check_codes(d_pre_q, rows, cols, fn, "d_pre_q"))) return rc;
    if (rows == 0) return PGMOE_OK;
    if (!d_pre && !d_pre_q) return fail(nullptr, PGMOE_EINVAL, "%s: both d_pre and d_pre_q are NULL", fn);
    if ((rc = check_matrix(d_h, d_h_stride, d_h_dtype, cols, false, fn, "d_h"))) return rc;
    if ((rc = check_matrix(d_pre, d_pre_stride, d_pre_dtype, cols, true, fn, "d_pre"))) return rc;
    const int64_t grid = ((int64_t)rows + 8 * RELU_ROWS - 1) / (8 * RELU_ROWS) * 8 * fp8_blocks(cols);
    if (grid * 256 > GRID_THREADS_MAX) return fail(nullptr, PGMOE_EINVAL, "%s: %d rows of %d columns are more than one launch holds", fn, rows, cols);
    const ReluArgs a = {d_h, (size_t)d_h_stride, (const uint8_t *)h_q, (size_t)h_q_stride, fp8_type(h_dtype), rows, cols, rows_out(d_pre, d_pre_stride, d_pre_q)};
    const bool vec = cols % 8 == 0 && wide(d_h, d_h_stride, d_h_dtype) && wide(d_pre, d_pre_stride, d_pre_dtype);
    by_type(d_h_dtype, [&](auto x_) {
        by_type(d_pre_dtype, [&](auto y_) {
            using X = decltype(x_);
            using Y = decltype(y_);
            auto go = [&](auto vec_, auto quant_) {
                hipLaunchKernelGGL((relu_backward_kernel<X, Y, decltype(vec_)::value, decltype(quant_)::value>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, a);
            };
            if (vec) d_pre_q ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
            else d_pre_q ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
        });
    });
    return launched(fn);
}

}  // extern "C"
