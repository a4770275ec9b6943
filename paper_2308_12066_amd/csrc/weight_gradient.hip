// Gradient of the experts' matrices from rows kept in 8 bits (pgmoe_expert_weight_gradient).
//
//   d_w[e, i, o] = add[e, i, o] + sum over the rows r of expert e of  x[r, i] d_y[r, o],   x[r, i] = code[r, i] * scale[r, i / 128]
//
// The scales of x vary along the sum, so they are in one of its operands; here it is that of the codes, code times scale.  Where scales are
// powers of two that is a bfloat16 as it stands (four bits; scales below 2^-124, e5m2 2^-117, leave some codes less), and one product a row, input and output is exact.  Otherwise code times scale in 32
// bits is taken apart into three bfloat16 whose sum it is, and so are gradients of 32 bits; those of 16-bit floating point are the sum of two.  (A tile of 128 inputs has one scale a row: its mantissa could go
// to the gradients instead, which would take three products whatever their type, where five and six are taken now.  Not built.)
#include <algorithm>
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
    int parts;  // an expert's rows are split into: each writes a float32 plane of its own to d_w, [parts][E][n_in][n_out]
    int tiles_in, tiles_out, group_in, group_out;
    bool sorted;  // items of experts with many rows first, one a workgroup
};

// The steps of part `part` of an expert's `steps`: none for some parts if there are few.
__host__ __device__ inline int first_step(int steps, int part, int parts) { return (int)((int64_t)steps * part / parts); }

typedef int intx2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// PIECES bfloat16 that add up to v's leading 8 * PIECES bits, but for bfloat16's least step, 2^-133, each.  All have v's sign and none is zero if v is not, however small it is, so
// that an infinity times each of them is the infinity that it times v is: pieces are cut off, not rounded, and v and what is left of it each time are first raised by a
// step towards v's side.  v: raised already; of(left, j): raises what is left of v[j].  (Products of pieces that are left out are below 2^-20 of the first, on the mean 2^-23.)
__device__ inline int high_halves(float a, float b) { return (int)__builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }
__device__ inline float between(float v, float limit) { return __builtin_amdgcn_fmed3f(v, -limit, limit); }
constexpr float LEAST_STEP = 0x1p-133f;
template <int PIECES, typename Raised>
__device__ inline void take_apart(float (&v)[8], intx4 (&to)[PIECES], Raised &&raised) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        to[p] = intx4{high_halves(v[0], v[1]), high_halves(v[2], v[3]), high_halves(v[4], v[5]), high_halves(v[6], v[7])};
        if (p + 1 < PIECES) {  // of an infinity the largest bfloat16 is taken off: the infinity is left
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = raised(v[j] - between(__uint_as_float(__float_as_uint(v[j]) & 0xffff0000u), 0x1.fep127f), j);
        }
    }
}
// Gradients: of 16-bit floating point, whose least value is 2^-24, a part in 2^32 is far above a step and does as well.
__device__ inline void take_apart(float (&v)[8], intx4 (&to)[2]) {
    const float whole[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    take_apart<2>(v, to, [&](float left, int j) { return fmaf(whole[j], 0x1p-32f, left); });
}
__device__ inline void take_apart(float (&v)[8], intx4 (&to)[3]) {
    float step[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        step[j] = between(v[j] * 0x1p16f, LEAST_STEP);  // the least float32, 2^-149, has a whole one too, 0 none
        v[j] += step[j];                       // NaN: with a bit that is not cut off
    }
    take_apart<3>(v, to, [&](float left, int j) { return left + step[j]; });
}

// Eight codes times their scale.
template <int Q, int PIECES>
__device__ inline void open_codes(intx2 codes, float scale, intx4 (&to)[PIECES]) {
    if constexpr (PIECES == 1) {  // the conversion takes the scale's exponent
        int pairs[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x2 pair;
            if constexpr (Q == PGMOE_E4M3)
                pair = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j >> 1], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j >> 1], scale, false);
            else pair = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[j >> 1], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[j >> 1], scale, false);
            pairs[j] = __builtin_bit_cast(int, pair);
        }
        to[0] = intx4{pairs[0], pairs[1], pairs[2], pairs[3]};
    } else {
        float v[8], step[8];
        const float least = between(scale, LEAST_STEP);  // the step of a code, which is 2^-16 or more, or 0; rows with a scale of 0 add nothing
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            floatx2 pair;
            if constexpr (Q == PGMOE_E4M3) pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(codes[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(codes[j >> 1], false);
            else pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_bf8(codes[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_bf8(codes[j >> 1], false);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                step[2 * j + i] = between(pair[i], least);
                v[2 * j + i] = fmaf(pair[i], scale, step[2 * j + i]);
            }
        }
        take_apart<PIECES>(v, to, [&](float left, int j) { return left + step[j]; });
    }
}

// Four rows of 16 neighbouring bfloat16 columns in LDS, one row behind the other's `stride`, as a quarter of a wavefront's operand: lane i of 16 gives the
// address of four columns of row i / 4 and gets column i of all four.
__device__ inline shortx4 read_transposed(const char *at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)at);
}
// An operand of 16 columns and 32 rows: of 64 neighbouring columns tile t of four takes 4 t .. 4 t + 3 of each 16.  Which rows a lane takes is free as long as
// both operands agree: quarters of a wavefront start at rows 0, 16, 4 and 20, and go on eight rows further down.  With rows 8 bytes past a multiple
// of 256 apart the 32 pieces of 8 bytes that half a wavefront reads at once lie in different banks.
__device__ inline bf16x8 operand_of(const char *columns, int t, int stride, int lane) {
    const char *at = columns + (size_t)((lane >> 4 & 1) * 16 + (lane >> 5) * 4 + (lane >> 2 & 3)) * stride + (lane & 3) * 32 + t * 8;
    const shortx4 low = read_transposed(at), high = read_transposed(at + 8 * stride);
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, shortx8{low[0], low[1], low[2], low[3], high[0], high[1], high[2], high[3]});
}

template <typename Y>
constexpr int pieces_of = sizeof(Y) == 4 ? 3 : std::is_same<Y, __bf16>::value ? 1 : 2;

// Where a lane's results acc[i][o][r] of a wavefront's NI x 4 tiles are: input 64 (i / 4) + 16 (lane / 16) + 4 (i % 4) + r, output 16 (lane % 16 / 4) + 4 o + lane % 4.
__device__ inline int input_of(int i, int r, int lane) { return (i >> 2) * 64 + (lane >> 4) * 16 + (i & 3) * 4 + r; }

// Lane t of four has v[o], o = 0 .. 3, and gets v[t] of lane o in o.
__device__ inline intx4 transpose_quad(intx4 v, int lane) {
    const bool odd = lane & 1, upper = lane & 2;
    intx4 w, x;
#pragma unroll
    for (int o = 0; o < 4; ++o) {  // with lane t ^ 1
        const int got = __builtin_amdgcn_update_dpp(0, v[o ^ 1], 0xb1, 0xf, 0xf, true);
        w[o] = odd == (o & 1) ? v[o] : got;
    }
#pragma unroll
    for (int o = 0; o < 4; ++o) {  // with lane t ^ 2
        const int got = __builtin_amdgcn_update_dpp(0, w[o ^ 2], 0x4e, 0xf, 0xf, true);
        x[o] = upper == (o >> 1) ? w[o] : got;
    }
    return x;
}
// Four lanes exchange their results of four tiles, so that neighbouring lanes store neighbouring 16 bytes, 256 of each of four inputs at once, past the caches, which then keep
// the rows.  A CU gets 118 GB/s out that way, and 37 if neighbouring lanes store 16 bytes of different inputs, whole lines or not (1024 x 4096 float32 for each of 64 experts
// from 32768 rows: 440, now 415 us).  VEC: 16 bytes of results are all there or none.
template <typename W, bool ADD, int NI>
__device__ __forceinline__ void store_rows(const GradientArgs &a, int e, int in, int out, int lane, const floatx4 (&acc)[NI][4]) {
    typedef W Wx4 __attribute__((ext_vector_type(4)));
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));  // worked out again: what depends on it is not kept in registers across the products
    const int col = out + (lane & 15) * 4;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        Wx4 addend[4];
        if constexpr (ADD) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                addend[r] = *reinterpret_cast<const Wx4 *>(reinterpret_cast<const W *>(a.add) + ((size_t)e * a.n_in + min(in + input_of(i, r, lane), a.n_in - 1)) * a.n_out + min(col, a.n_out - 4));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            floatx4 v = __builtin_bit_cast(floatx4, transpose_quad(__builtin_bit_cast(intx4, floatx4{acc[i][0][r], acc[i][1][r], acc[i][2][r], acc[i][3][r]}), lane));
            if constexpr (ADD) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += (float)addend[r][j];
                asm volatile("" : "+v"(v));  // added up here, not where a store may be left out: the compiler else takes addends for on their way, and waits for results for safety
            }
            const int row = in + input_of(i, r, lane);
            if (row >= a.n_in || col >= a.n_out) continue;
            const Wx4 w = {(W)v[0], (W)v[1], (W)v[2], (W)v[3]};
            Wx4 *to = reinterpret_cast<Wx4 *>(reinterpret_cast<W *>(a.d_w) + ((size_t)e * a.n_in + row) * a.n_out + col);
            if (a.parts == 1) __builtin_nontemporal_store(w, to);
            else *to = w;  // gradient_parts_kernel reads it at once
        }
    }
}
template <typename W, int NI>
__device__ __forceinline__ void store_singly(const GradientArgs &a, int e, int in, int out, int lane, const floatx4 (&acc)[NI][4]) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = in + input_of(i, r, lane);
            if (row >= a.n_in) continue;
#pragma unroll
            for (int o = 0; o < 4; ++o) {
                const int col = out + (lane & 12) * 4 + 4 * o + (lane & 3);
                const size_t at = ((size_t)e * a.n_in + row) * a.n_out + col;
                if (col < a.n_out) reinterpret_cast<W *>(a.d_w)[at] = (W)(a.add ? acc[i][o][r] + (float)reinterpret_cast<const W *>(a.add)[at] : acc[i][o][r]);
            }
        }
}
template <bool VEC, int NI>
__device__ __forceinline__ void store_gradient(const GradientArgs &a, int e, int in, int out, int lane, const floatx4 (&acc)[NI][4]) {
    auto finish = [&](auto type) {
        if constexpr (VEC) a.add ? store_rows<decltype(type), true>(a, e, in, out, lane, acc) : store_rows<decltype(type), false>(a, e, in, out, lane, acc);
        else store_singly<decltype(type)>(a, e, in, out, lane, acc);
    };
    if (a.dtype == PGMOE_F32) finish(float());
    else if (a.dtype == PGMOE_BF16) finish(__bf16());
    else finish(_Float16());
}

// Which tile, of which part of an expert's rows, is item number i.  Workgroups go to the 8 dies in turn: one takes group_in x group_out neighbouring tiles, whose rows
// its L2 then holds.  e >= E: none from here on; ti >= tiles_in or to >= tiles_out: none at this number.
struct GradientItem {
    int e, part, ti, to;
};
__device__ inline GradientItem gradient_item(const GradientArgs &a, int i) {
    const int group_items = a.group_in * a.group_out, turn = i >> 3, group = turn / group_items * 8 + (i & 7), in_group = turn % group_items;
    const int groups_out = (a.tiles_out + a.group_out - 1) / a.group_out, groups_in = (a.tiles_in + a.group_in - 1) / a.group_in;
    const int m = group / (groups_in * groups_out), at = group - m * groups_in * groups_out, e = m / a.parts;
    return {e, m - e * a.parts, at / groups_out * a.group_in + in_group / a.group_out, at % groups_out * a.group_out + in_group % a.group_out};
}

// An item is BI inputs by BO outputs; a workgroup takes every gridDim-th of them and goes through its rows K at a time.  Both sides come through registers, where codes are converted,
// into one of two buffers in LDS while the other is multiplied, also from one item to the next: the first rows of an item arrive under the last products of the one before.
// Bound by the products on many rows, 1.12 PFLOP/s (each further 512 rows for each of 64 experts of 1024 x 4096: 246 us), and by the results on few: their float32 leave at 5.5 TB/s, about
// 160 us of the 411 that 512 rows an expert take, mostly not under the products (workgroups started at different times gained nothing). Without loads the same call takes 340, without stores 270.
template <int WI_, int WO_, int NI_, int K_>
struct GradientShape {
    static constexpr int WI = WI_, WO = WO_, NI = NI_, NO = 4, K = K_;  // wavefronts; 16 x 16 tiles of one
    static constexpr int BI = WI * NI * 16, BO = WO * NO * 16, THREADS = WI * WO * 64;
    // a thread brings XP and YP pieces of eight columns of rows that lie XR and YR apart; bytes from one row to the next in LDS
    static constexpr int XR = THREADS * 8 / BI, YR = THREADS * 8 / BO, XP = K / XR, YP = K / YR, XS = 2 * BI + 8, YS = 2 * BO + 8;
    static_assert(THREADS >= PGMOE_MAX_EXPERTS && BI % 128 == 0 && BO % 128 == 0 && XP * XR == K && YP * YR == K && K % 32 == 0, "whole pieces");
    static constexpr int buffer(int px, int py) { return K * (px * XS + py * YS); }
    // wavefronts a SIMD: of small tiles with few pieces four workgroups fit into a CU
    static constexpr int waves(int px, int py) { return THREADS == 256 && px * py == 1 ? 4 : THREADS == 256 && px * py < 4 ? 3 : 2; }
};
template <int XQ, typename Y, int PX, bool VEC, typename S>
__global__ __launch_bounds__(S::THREADS, S::waves(PX, pieces_of<Y>)) void weight_gradient_kernel(const GradientArgs a) {
    constexpr int XPLANE = S::K * S::XS, YPLANE = S::K * S::YS, PY = pieces_of<Y>, BUFFER = S::buffer(PX, PY), KEPT = PX > PY ? PX : PY;  // KEPT: pieces i and j are multiplied where i + j < KEPT
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / S::WO, wo = wave % S::WO;
    const int x_piece = threadIdx.x % (S::BI / 8), x_row = threadIdx.x / (S::BI / 8), y_piece = threadIdx.x % (S::BO / 8), y_row = threadIdx.x / (S::BO / 8);

    struct Item {
        GradientItem at;
        int first, rows;  // of d_y and x
    };
    // the expert's offsets by scalar loads: a vector load would wait for the results of the item before
    const auto *offsets = (const __attribute__((address_space(4))) int32_t *)a.offsets;
    int expert = 0;
    if (a.sorted) {  // which expert has as many rows that the item's number says?  (uniform)
        const int place = gradient_item(a, blockIdx.x).e;
        int *rows = reinterpret_cast<int *>(lds), t = threadIdx.x;
        if (t < a.E) rows[t] = offsets[t + 1] - offsets[t];
        lds_barrier();
        if (t < a.E) {
            int before = 0;
            for (int j = 0; j < a.E; ++j) before += rows[j] > rows[t] || (rows[j] == rows[t] && j < t);
            if (before == place) rows[a.E] = t;
        }
        lds_barrier();
        expert = __builtin_amdgcn_readfirstlane(place < a.E ? rows[a.E] : 0);
        lds_barrier();
    }
    auto find = [&](int &i, Item &it) {  // the item at number i or the next of this workgroup behind it -> is there one?
        for (;; i += gridDim.x) {
            it.at = gradient_item(a, i);
            if (it.at.e >= a.E) return false;
            if (it.at.ti >= a.tiles_in || it.at.to >= a.tiles_out) continue;
            if (a.sorted) it.at.e = expert;
            const int lo = max(0, min(offsets[it.at.e], a.rows)), n = max(lo, min(offsets[it.at.e + 1], a.rows)) - lo;
            if (a.parts == 1) {
                it.first = lo;
                it.rows = n;
                return true;
            }
            const int steps = (n + S::K - 1) / S::K, from = first_step(steps, it.at.part, a.parts) * S::K, to = min(first_step(steps, it.at.part + 1, a.parts) * S::K, n);
            if (to <= from) continue;  // its plane is not read
            it.first = lo + from;
            it.rows = to - from;
            return true;
        }
    };

    // what a thread brings of an item; columns past the last are others', nobody's result
    const uint8_t *x;
    const float *x_scale;
    const Y *d_y;
    unsigned x_col;
    int col, left;  // rows that are not requested
    auto open = [&](const Item &it) {
        const int block = min(it.at.ti * (S::BI / 128) + x_piece / 16, fp8_blocks(a.n_in) - 1);
        x_col = block * 128 + x_piece % 16 * 8;
        col = min(it.at.to * S::BO + y_piece * 8, VEC ? a.n_out - 8 : a.n_out - 1);
        x = a.x + (size_t)it.first * a.x_stride;
        x_scale = a.x_scale + (size_t)block * a.x_scale_stride + it.first;
        d_y = reinterpret_cast<const Y *>(a.d_y) + (size_t)it.first * a.d_y_stride;
        left = it.rows;
    };
    intx2 codes[S::XP];
    float scale[S::XP];
    struct { Y v[8]; } grad[S::YP];
    int requested;  // rows
    auto request = [&] {  // past the last row the last one, which keep() clears
#pragma unroll
        for (int i = 0; i < S::XP; ++i) {
            const int r = min(x_row + i * S::XR, left - 1);
            scale[i] = x_scale[r];
            if constexpr (VEC) codes[i] = *reinterpret_cast<const intx2 *>(x + ((unsigned)r * (unsigned)a.x_stride + x_col));  // less than 2^32 bytes a step
            else codes[i] = *reinterpret_cast<const intx2 *>(x + (size_t)r * a.x_stride + x_col);
        }
#pragma unroll
        for (int i = 0; i < S::YP; ++i) {
            const int r = min(y_row + i * S::YR, left - 1);
            if constexpr (VEC) {
                typedef Y Yx8 __attribute__((ext_vector_type(8), aligned(16)));
                *reinterpret_cast<Yx8 *>(grad[i].v) =
                    *reinterpret_cast<const Yx8 *>(reinterpret_cast<const char *>(d_y) + ((unsigned)r * ((unsigned)a.d_y_stride * (unsigned)sizeof(Y)) + col * (unsigned)sizeof(Y)));
            } else {
                const Y *g = d_y + (size_t)r * a.d_y_stride;
#pragma unroll
                for (int j = 0; j < 8; ++j) grad[i].v[j] = g[min(col + j, a.n_out - 1)];
            }
        }
        requested = left;
        left -= S::K;
        x += (size_t)S::K * a.x_stride;
        x_scale += S::K;
        d_y += (size_t)S::K * a.d_y_stride;
    };
    int buffer = 0;
    auto keep = [&](int at) {
        char *to = lds + at * BUFFER;
        auto put = [](char *to, intx4 v) {  // 8-byte aligned
            reinterpret_cast<intx2 *>(to)[0] = intx2{v[0], v[1]};
            reinterpret_cast<intx2 *>(to)[1] = intx2{v[2], v[3]};
        };
        const intx4 none = {0, 0, 0, 0};  // rows behind the last are zero on both sides, whatever the last one holds
#pragma unroll
        for (int i = 0; i < S::XP; ++i) {
            const int r = x_row + i * S::XR;
            intx4 px[PX];
            open_codes<XQ, PX>(codes[i], scale[i], px);
#pragma unroll
            for (int p = 0; p < PX; ++p) put(to + p * XPLANE + r * S::XS + x_piece * 16, r < requested ? px[p] : none);
        }
#pragma unroll
        for (int i = 0; i < S::YP; ++i) {
            const int r = y_row + i * S::YR;
            intx4 py[PY];
            if constexpr (PY == 1) {
                py[0] = __builtin_bit_cast(intx4, grad[i]);
            } else {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)grad[i].v[j];
                take_apart(v, py);
            }
#pragma unroll
            for (int p = 0; p < PY; ++p) put(to + PX * XPLANE + p * YPLANE + r * S::YS + y_piece * 16, r < requested ? py[p] : none);
        }
    };
    // Rows are the first operand: a lane's four results of a product are neighbouring inputs of one output (input_of), until store_rows exchanges them.
    floatx4 acc[S::NI][S::NO];
    auto multiply = [&](int at) {
#pragma unroll
        for (int k = 0; k < S::K; k += 32) {
            const char *now = lds + at * BUFFER;
            bf16x8 px[S::NI][PX];
#pragma unroll
            for (int i = 0; i < S::NI; ++i)
#pragma unroll
                for (int p = 0; p < PX; ++p) px[i][p] = operand_of(now + p * XPLANE + k * S::XS + (wi * S::NI + i / 4 * 4) * 32, i % 4, S::XS, lane);
#pragma unroll
            for (int o = 0; o < S::NO; ++o) {
                bf16x8 py[PY];
#pragma unroll
                for (int p = 0; p < PY; ++p) py[p] = operand_of(now + PX * XPLANE + p * YPLANE + k * S::YS + wo * S::NO * 32, o, S::YS, lane);
                // small products first
                static_for<KEPT>([&](auto s_) {
                    static_for<PY>([&](auto p_) {
                        constexpr int s = KEPT - 1 - decltype(s_)::value, p = decltype(p_)::value;
                        if constexpr (s >= p && s - p < PX) {
#pragma unroll
                            for (int i = 0; i < S::NI; ++i) acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(px[i][s - p], py[p], acc[i][o], 0, 0, 0);
                        }
                    });
                });
            }
        }
    };

    int i = blockIdx.x;
    Item it, next;
    if (!find(i, it)) return;  // uniform over the workgroup, as all below
    if (it.rows > 0) {
        open(it);
        request();
        keep(buffer);
    }
    for (;;) {
        i += gridDim.x;
        const bool more = find(i, next);
#pragma unroll
        for (int x = 0; x < S::NI; ++x)
#pragma unroll
            for (int o = 0; o < S::NO; ++o) acc[x][o] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int rows = it.rows; rows > 0; rows -= S::K) {
            lds_barrier();  // these rows are there for everyone, and everyone has read the ones before
            // Requested in any case, behind the last rows the item's own once more: the compiler then knows what is on its way, and does not wait for an item's results for
            // safety (with the offsets by scalar loads 450 to 440 us, 64 experts of 1024 x 4096 from 32768 rows).
            if (rows <= S::K) open(more && next.rows > 0 ? next : it);
            request();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);  // before another wavefront's conversions: 2 to 4 %
            multiply(buffer);
            __builtin_amdgcn_s_setprio(0);
            keep(buffer ^ 1);
            buffer ^= 1;
        }
        if (it.rows == 0 && more && next.rows > 0) {
            open(next);
            request();
            keep(buffer);
        }
        store_gradient<VEC>(a, it.at.part * a.E + it.at.e, it.at.ti * S::BI + wi * S::NI * 16, it.at.to * S::BO + wo * S::NO * 16, lane, acc);
        if (!more) return;
        it = next;
    }
}

// The planes of an expert's parts, added up in their order.
template <typename W, bool VEC>
__global__ __launch_bounds__(256) void gradient_parts_kernel(const float *parts, const GradientArgs a, int K) {
    constexpr int N = VEC ? 4 : 1;
    typedef W WxN __attribute__((ext_vector_type(N)));
    typedef float FxN __attribute__((ext_vector_type(N)));
    const int64_t size = (int64_t)a.n_in * a.n_out, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
    const int e = blockIdx.y;
    if (at >= size) return;
    const int lo = max(0, min(a.offsets[e], a.rows)), steps = (max(lo, min(a.offsets[e + 1], a.rows)) - lo + K - 1) / K;
    FxN sum = {};
#pragma unroll 4
    for (int p = 0; p < a.parts; ++p)
        if (first_step(steps, p + 1, a.parts) > first_step(steps, p, a.parts)) sum += *reinterpret_cast<const FxN *>(parts + ((int64_t)p * a.E + e) * size + at);
    const int64_t to = e * size + at;
    WxN out;
    if (a.add) {
        const WxN add = *reinterpret_cast<const WxN *>(reinterpret_cast<const W *>(a.add) + to);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += (float)add[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = (W)sum[j];
    *reinterpret_cast<WxN *>(reinterpret_cast<W *>(a.d_w) + to) = out;
}

using SmallTile = GradientShape<2, 2, 4, 32>;
using WideTile = GradientShape<2, 4, 4, 32>;
using LargeTile = GradientShape<2, 4, 8, 64>;

// More than 48 KiB of LDS: the kernel's limit is raised once per device.
static int raise_lds(const void *kernel, int bytes, std::atomic<uint64_t> &raised) {
    int device = 0;
    if (const hipError_t e = hipGetDevice(&device))
        return e == hipErrorNoDevice ? fail(nullptr, PGMOE_ENODEVICE, "pgmoe_expert_weight_gradient: no HIP device is visible") : hip_fail(nullptr, e, "hipGetDevice");
    if (!(raised.load(std::memory_order_relaxed) >> (device & 63) & 1)) {
        PG_HIP(nullptr, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        raised.fetch_or(1ull << (device & 63), std::memory_order_relaxed);
    }
    return PGMOE_OK;
}
// Tiles in groups of up to 1024 x 1024, as long as there are two for each die -> item numbers.  With many products for what is read (`spread`) groups are up to 512 x 512 and all alike,
// so that an expert of many rows is all dies'.
static int64_t gradient_items(GradientArgs &a, int tile_in, int tile_out, bool spread) {
    a.tiles_in = (a.n_in + tile_in - 1) / tile_in;
    a.tiles_out = (a.n_out + tile_out - 1) / tile_out;
    a.group_in = std::min(a.tiles_in, (spread ? 512 : 1024) / tile_in);
    a.group_out = std::min(a.tiles_out, (spread ? 512 : 1024) / tile_out);
    if (spread) {
        while (a.tiles_in % a.group_in) --a.group_in;
        while (a.tiles_out % a.group_out) --a.group_out;
    }
    const auto groups = [&] { return (int64_t)a.E * a.parts * ((a.tiles_in + a.group_in - 1) / a.group_in) * ((a.tiles_out + a.group_out - 1) / a.group_out); };
    while (groups() < 16 && a.group_in * a.group_out > 1) (a.group_in > a.group_out ? a.group_in : a.group_out) = (std::max(a.group_in, a.group_out) + 1) / 2;
    return (groups() + 7) / 8 * 8 * a.group_in * a.group_out;
}
template <int XQ, typename Y, int PX, bool VEC, typename S>
static int launch_shape(GradientArgs a, hipStream_t s, int64_t most, bool spread) {  // most: workgroups (0: one an item)
    constexpr int LDS = 2 * S::buffer(PX, pieces_of<Y>);
    static std::atomic<uint64_t> raised{0};
    int64_t grid = gradient_items(a, S::BI, S::BO, spread);
    if (grid * S::THREADS > GRID_THREADS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "pgmoe_expert_weight_gradient: %d matrices of %d x %d are more than one launch holds", a.E, a.n_in, a.n_out);
    if (most) grid = std::min(grid, most);
    if (LDS > 48 * 1024)
        if (const int rc = raise_lds(reinterpret_cast<const void *>(&weight_gradient_kernel<XQ, Y, PX, VEC, S>), LDS, raised)) return rc;
    hipLaunchKernelGGL((weight_gradient_kernel<XQ, Y, PX, VEC, S>), dim3((unsigned)grid), dim3(S::THREADS), LDS, s, a);
    return PGMOE_OK;
}
// Into how many parts the rows of each expert are split where there are fewer tiles than workgroups run at once.  A tile by itself takes 17 to 18.5 ns a row; the rule, fitted to the
// times below, takes the cost of parts, a launch and planes of 64 KiB a tile that are written and read, for 4 us and 0.021 us for each part of each tile.  us without parts / with as many as this says, bfloat16 gradients: one expert of 512 x 1024 from 512 rows 12.7 (2 parts
// would take 14.0), 1024 20.3 / 16.7, 4096 73 / 30, 16384 279 / 42; one of 1024 x 4096 from 1024 rows 25.0 (2: 32.6), 4096 76 / 60; eight of 512 x 512 from 512 rows each
// 13.7 (2: 26.6), 2048 40 / 31; eight of 1024 x 1024 from 4096 each 89 (2: 107).
constexpr int GRADIENT_PARTS = 16, CUS = 256;
static int gradient_parts(int rows, int E, int n_in, int n_out) {
    const int64_t tiles = (int64_t)E * fp8_blocks(n_in) * fp8_blocks(n_out);
    if (tiles > CUS) return 1;
    const int each = rows / E, parts = std::min({512 / (int)tiles, each / 256, GRADIENT_PARTS});
    if (parts < 2) return 1;
    return 0.0185 * each * (parts - 1) / parts > 4 + 0.021 * tiles * parts ? parts : 1;
}
template <int XQ, typename Y, int PX, bool VEC>
static int launch_parts(const GradientArgs &a, float *planes, hipStream_t s) {
    GradientArgs p = a;
    p.d_w = planes;
    p.add = nullptr;
    p.dtype = PGMOE_F32;
    const int rc = launch_shape<XQ, Y, PX, VEC, SmallTile>(p, s, 0, false);
    if (rc) return rc;
    const int64_t size = (int64_t)a.n_in * a.n_out;
    const dim3 grid((unsigned)((size / (VEC ? 4 : 1) + 255) / 256), a.E);
    if (a.dtype == PGMOE_F32) hipLaunchKernelGGL((gradient_parts_kernel<float, VEC>), grid, dim3(256), 0, s, planes, a, SmallTile::K);
    else if (a.dtype == PGMOE_BF16) hipLaunchKernelGGL((gradient_parts_kernel<__bf16, VEC>), grid, dim3(256), 0, s, planes, a, SmallTile::K);
    else hipLaunchKernelGGL((gradient_parts_kernel<_Float16, VEC>), grid, dim3(256), 0, s, planes, a, SmallTile::K);
    return PGMOE_OK;
}
// Which tiles (us, bfloat16 gradients with scales that are powers of two unless said otherwise, float32 results, rows dealt out evenly):
//  * 256 x 256, one workgroup a CU: from 256 rows an expert on the mean on, if the last round of a tile for each CU leaves at most a fifth of them idle (64 experts of 1024 x 4096 from 64 rows each 222, 128 x 128
//    193, 256 rows 282 / 344, 512 399 / 475; 16 of 512 x 2048 from 256 21.3 / 20.1, 2048 76 / 92; 192 tiles: eight of 768 x 2048 from 512 24.8 / 22.7, 2048 64 / 62);
//  * 128 x 256, one workgroup a CU, where pieces of both sides leave room in LDS for no more, if there are more of 128 x 128 than CUs: 16 experts of 2048 x 768 from 512 rows each, three and three pieces
//    149, 128 x 128 217; eight of 1024 x 1024 from 32 rows 13.0 / 17.2; eight of 512 x 512 from 512 rows, three and two pieces 41 / 32.  Against two workgroups a CU, the second when the first ends, and one
//    an item: 16 of 2048 x 1024, three and two pieces, from 512 rows each 156 / 160 / 163, from 32 29.5 / 32.5 / 38.2, with a fifth of 8192 rows in one 218.6 / 218.5 / 223.2;
//  * 128 x 128 otherwise.  (Two or three products with scales that are powers of two have no other: the larger tiles were not built for them.  16 experts
//    of 2048 x 1024 from 512 rows each: 16-bit floating point 84, float32 128; 64 of 1024 x 4096 685 and 1031.)
// And in which order, of the two smaller ones: from 256 rows an expert on the mean on, and if not all items run at once, those of experts with many rows first, one a workgroup, of which the next goes where one has ended
// (`sorted`; in order / sorted, rows dealt out evenly, and with nearly a quarter in one: 8192 rows for 16 experts of 2048 x 1024, three and two pieces, 156 / 167 and 233 / 178; for 32 of 1024 x 1024 86 / 103 and 192 / 143;
// 4096 for 16 of 768 x 2048, one piece, 28.2 / 29.6 and 37 / 33).
template <int XQ, typename Y, int PX, bool VEC>
static int launch_gradient(GradientArgs a, float *planes, hipStream_t s) {
    if (a.parts > 1) return launch_parts<XQ, Y, PX, VEC>(a, planes, s);
    const auto tiles = [&](int in, int out) { return (int64_t)a.E * ((a.n_in + in - 1) / in) * ((a.n_out + out - 1) / out); };
    if constexpr (PX * pieces_of<Y> == 1 && VEC) {
        const int64_t large = tiles(256, 256), rounds = (large + CUS - 1) / CUS;
        if (a.rows / a.E >= 256 && 5 * large >= 4 * CUS * rounds) return launch_shape<XQ, Y, PX, VEC, LargeTile>(a, s, CUS, false);
    }
    const int64_t small = tiles(128, 128);
    a.sorted = a.rows / a.E >= 256 && (PX == 3 && pieces_of<Y> > 1 ? small > CUS : small > 4 * CUS);
    if constexpr (PX == 3 && pieces_of<Y> > 1)
        if (small > CUS) return launch_shape<XQ, Y, PX, VEC, WideTile>(a, s, a.sorted ? 0 : CUS, a.sorted);
    return launch_shape<XQ, Y, PX, VEC, SmallTile>(a, s, 0, a.sorted && PX * pieces_of<Y> > 1);
}
template <int XQ, typename Y>
static int launch_gradient(const GradientArgs &a, bool pow2, float *planes, hipStream_t s) {
    const bool vec = a.n_out % 8 == 0 && a.d_y_stride * sizeof(Y) % 16 == 0 && a.d_y_stride * sizeof(Y) < (1 << 25) && a.x_stride < (1 << 25) && a.x_scale_stride < (1 << 28) && aligned(a.d_y, 16) && aligned(a.d_w, 16) && aligned(a.add, 16);
    if (pow2) return vec ? launch_gradient<XQ, Y, 1, true>(a, planes, s) : launch_gradient<XQ, Y, 1, false>(a, planes, s);
    return vec ? launch_gradient<XQ, Y, 3, true>(a, planes, s) : launch_gradient<XQ, Y, 3, false>(a, planes, s);
}
template <int XQ>
static int launch_gradient(const GradientArgs &a, int y_dtype, bool pow2, float *planes, hipStream_t s) {
    if (y_dtype == PGMOE_F32) return launch_gradient<XQ, float>(a, pow2, planes, s);
    if (y_dtype == PGMOE_BF16) return launch_gradient<XQ, __bf16>(a, pow2, planes, s);
    return launch_gradient<XQ, _Float16>(a, pow2, planes, s);
}

}  // namespace pgmoe

using namespace pgmoe;

extern "C" {

size_t pgmoe_expert_weight_gradient_workspace_bytes(int rows, int n_experts, int n_in, int n_out) {
    if (rows < 1 || n_experts < 1 || n_in < 1 || n_out < 1) return 0;
    const int parts = gradient_parts(rows, n_experts, n_in, n_out);
    return parts > 1 ? (size_t)parts * n_experts * n_in * n_out * sizeof(float) : 0;
}

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
    if (x->rows > 0) NEED_PTR(nullptr, fn, d_y, dtype_bytes(d_y_dtype));
    NEED_PTR(nullptr, fn, expert_offsets, 4);
    NEED_PTR(nullptr, fn, d_w, dtype_bytes(d_w_dtype));
    OPT_PTR(nullptr, fn, add, dtype_bytes(d_w_dtype));
    OPT_PTR(nullptr, fn, workspace, 16);
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
    const size_t need = pgmoe_expert_weight_gradient_workspace_bytes(x->rows, n_experts, x->cols, n_out);
    const bool split = need > 0 && workspace && workspace_bytes >= need;
    a.parts = split ? (int)(need / sizeof(float) / ((size_t)n_experts * x->cols * n_out)) : 1;
    float *planes = (float *)workspace;
    const bool pow2 = (x->dtype & PGMOE_SCALE_POW2) != 0;
    rc = fp8_type(x->dtype) == PGMOE_E4M3 ? launch_gradient<PGMOE_E4M3>(a, d_y_dtype, pow2, planes, (hipStream_t)stream) : launch_gradient<PGMOE_E5M2>(a, d_y_dtype, pow2, planes, (hipStream_t)stream);
    return rc ? rc : launched(fn);
}

}  // extern "C"
