// Blocks of 8-bit floating point with one scale (device code and argument checks shared by quantize.hip and
// expert_matmul.hip).
#ifndef PGMOE_FP8_H
#define PGMOE_FP8_H
#include "pgmoe_internal.h"

namespace pgmoe {

constexpr int FP8_BLOCK = 128;              // values that share a scale
constexpr int FP8_TILE = 16 * FP8_BLOCK;    // bytes of an operand tile of the weights
constexpr int FP8_COLS_MAX = 1 << 22;       // of rows and of one weight matrix's sides
__host__ __device__ inline int fp8_blocks(int n) { return (n + FP8_BLOCK - 1) / FP8_BLOCK; }

// The two types: Q = PGMOE_E4M3 or PGMOE_E5M2.
template <int Q>
constexpr float fp8_largest = Q == PGMOE_E4M3 ? 448.f : 57344.f;

// The larger of both; NaN if one is (one instruction on this chip, with magnitudes taken on the way).
__device__ inline float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float relu_of(float v) { return maximum(v, 0.f); }

// Quotients by the scale of a block.  A block's largest magnitude is first taken with infinities and NaN among its values: it is finite
// nearly always, and then three instructions give the correctly rounded quotient: with the rounded inverse, the remainder
// of the first quotient (exact in one multiply-add) corrects it (Markstein).  The remainder of what does not round to zero is a
// multiple of 2^-63 times the scale's leading bit, exact from scales of 2^-86 on.  Blocks with infinities or NaN, whose largest finite
// magnitude has to be looked for, and scales below 2^-80 take the careful form: both sides raised, what is not finite left alone.
struct Fp8Divisor {
    float scale, inverse;
    __device__ explicit Fp8Divisor(float s) : scale(s), inverse(1.f / s) {}
    __device__ float operator()(float x) const {
        const float q = x * inverse;
        return fmaf(fmaf(q, scale, -x), -inverse, q);  // (the remainder's other sign would lose that of -0)
    }
};
struct Fp8CarefulDivisor {
    float up;
    Fp8Divisor by;
    __device__ explicit Fp8CarefulDivisor(float s) : up(s < 0x1p-80f ? 0x1p64f : 1.f), by(s * up) {}
    __device__ float operator()(float x) const {
        const float q = x * up * by.inverse;
        return fabsf(q) < INFINITY ? by(x * up) : q;
    }
};
template <int Q>
__device__ inline float fp8_scale(float amax) {
    return fmaxf(amax / fp8_largest<Q>, 0x1p-126f);
}
// Is there a block among the wavefront's, of largest magnitude amax, that needs the careful form?
template <int Q>
__device__ inline bool fp8_unusual(float amax) {
    return __any(!(amax < INFINITY && (amax >= 0x1p-79f * fp8_largest<Q> || amax == 0.f)));
}
__device__ inline float finite_magnitude(float x) {  // 0 for infinities and NaN
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}

// Four codes, the first in the low byte.  No clamp: a quotient is at most the largest value times 1 + 2^-23, which rounds to it;
// the conversion turns an infinity into NaN (e4m3) or keeps it (e5m2).
template <int Q>
__device__ inline uint32_t fp8_pack(float a, float b, float c, float d) {
    int v = 0;
    if (Q == PGMOE_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
    }
    return (uint32_t)v;
}

// Eight consecutive elements of a row as floats; columns from `cols` on are 0.  VEC: all eight exist and lie 16-byte aligned.
template <typename L, bool VEC>
__device__ inline void load_eight(const L *p, int col, int cols, float (&v)[8]) {
    typedef L Lx8 __attribute__((ext_vector_type(8), aligned(16)));
    if (VEC) {
        if (col < cols) {
            const Lx8 x = *reinterpret_cast<const Lx8 *>(p + col);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = col + j < cols ? (float)p[min(col + j, cols - 1)] : 0.f;
    }
}

// ---- argument checks
inline int check_float_type(int dtype, const char *fn, const char *what) {
    if (dtype == PGMOE_F32 || dtype == PGMOE_BF16 || dtype == PGMOE_F16) return PGMOE_OK;
    return fail(nullptr, PGMOE_EINVAL, "%s: %s=%d is neither f32 nor bf16 nor f16", fn, what, dtype);
}
inline int check_fp8_rows(const pgmoe_fp8_rows *r, const char *fn, const char *what) {
    if (!r) return fail(nullptr, PGMOE_EINVAL, "%s: %s is NULL", fn, what);
    if (r->dtype != PGMOE_E4M3 && r->dtype != PGMOE_E5M2) return fail(nullptr, PGMOE_EINVAL, "%s: %s has dtype %d, neither e4m3 nor e5m2", fn, what, r->dtype);
    if (r->rows < 0 || r->cols < 1 || r->cols > FP8_COLS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "%s: %s has %d rows of %d columns: 0 and more of 1 to %d", fn, what, r->rows, r->cols, FP8_COLS_MAX);
    if (r->q_stride < (int64_t)FP8_BLOCK * fp8_blocks(r->cols) || r->q_stride % 16)
        return fail(nullptr, PGMOE_EINVAL, "%s: %s has a q_stride of %lld: a multiple of 16 from %d on", fn, what, (long long)r->q_stride, FP8_BLOCK * fp8_blocks(r->cols));
    if (r->scale_stride < r->rows) return fail(nullptr, PGMOE_EINVAL, "%s: %s has a scale_stride of %lld for %d rows", fn, what, (long long)r->scale_stride, r->rows);
    if (r->rows == 0) return PGMOE_OK;
    if (!r->q || !r->scale) return fail(nullptr, PGMOE_EINVAL, "%s: %s has a NULL pointer", fn, what);
    if (!aligned(r->q, 16) || !aligned(r->scale, 4)) return fail(nullptr, PGMOE_EINVAL, "%s: %s has a pointer that is not aligned (q to 16 bytes, scale to 4)", fn, what);
    return PGMOE_OK;
}
inline int check_fp8_weights(const pgmoe_fp8_weights *w, const char *fn, const char *what) {
    if (!w) return fail(nullptr, PGMOE_EINVAL, "%s: %s is NULL", fn, what);
    if (w->n_experts < 1 || w->n_experts > PGMOE_MAX_EXPERTS)
        return fail(nullptr, PGMOE_EINVAL, "%s: %s has n_experts=%d outside 1..%d", fn, what, w->n_experts, PGMOE_MAX_EXPERTS);
    if (w->n_in < 1 || w->n_out < 1 || w->n_in > FP8_COLS_MAX || w->n_out > FP8_COLS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "%s: %s has n_in=%d, n_out=%d outside 1..%d", fn, what, w->n_in, w->n_out, FP8_COLS_MAX);
    if (!w->q || !w->scale) return fail(nullptr, PGMOE_EINVAL, "%s: %s has a NULL pointer", fn, what);
    if (!aligned(w->q, 16) || !aligned(w->scale, 4)) return fail(nullptr, PGMOE_EINVAL, "%s: %s has a pointer that is not aligned (q to 16 bytes, scale to 4)", fn, what);
    return PGMOE_OK;
}

}  // namespace pgmoe
#endif  // PGMOE_FP8_H
