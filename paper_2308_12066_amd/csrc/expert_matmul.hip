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
#include <atomic>

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
    bool once;  // the weights are passed by the caches
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

// Which rows of which expert are chunk number `chunk`, the chunks of an expert being its rows dealt evenly, in whole 16s,
// to as few chunks of at most MOST rows as hold them.  Offsets are clamped to the rows there are, whatever they say.  All
// offsets are loaded at once (four experts a lane).
struct MatmulChunk {
    int expert, row0, nrows;  // nrows == 0: there is no such chunk
};
template <int MOST>
__device__ inline MatmulChunk matmul_chunk(const MatmulArgs &a, int chunk) {
    const int lane = threadIdx.x & 63;
    int lo[4], n[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        lo[q] = n[q] = 0;
        if (q * 64 < a.E) {  // uniform
            const int e = q * 64 + lane;
            lo[q] = a.offsets[min(e, a.E)];
            n[q] = a.offsets[min(e + 1, a.E)];
        }
    }
    MatmulChunk ci = {0, 0, 0};
    int before = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q * 64 >= a.E) break;
        lo[q] = max(0, min(lo[q], a.rows));
        n[q] = max(lo[q], min(n[q], a.rows)) - lo[q];
        const int c = (n[q] + MOST - 1) / MOST, c_incl = before + wave_incl_scan(c);
        const unsigned long long hit = __ballot(chunk >= c_incl - c && chunk < c_incl);
        if (hit) {
            const int src = __ffsll((long long)hit) - 1;  // uniform: read that lane's values directly
            const int rows = __builtin_amdgcn_readlane(n[q], src), chunks = (rows + MOST - 1) / MOST;
            const int each = ((rows + chunks - 1) / chunks + 15) & ~15, k = chunk - __builtin_amdgcn_readlane(c_incl - c, src);
            ci.expert = q * 64 + src;
            ci.row0 = __builtin_amdgcn_readlane(lo[q], src) + k * each;
            ci.nrows = min(each, rows - k * each);
            return ci;
        }
        before = __builtin_amdgcn_readlane(c_incl, 63);
    }
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

// Few rows an expert: the stream of weights.  Operands straight from memory into registers, the next block of inputs requested before the one
// at hand is multiplied.  A workgroup takes 16 rows and 8 / KS tiles of 16 outputs, a wavefront one of them and one KS-th of the inputs; the
// parts are added up in LDS, in order.  One workgroup's stream is bound by its CU: 512 KB in 10.2 us (2 rows, 4096 x 1024, KS = 1), so few
// tiles go to more CUs (KS = 8: 4.1), and long sums to more wavefronts (512 rows over 64 experts of 4096 x 1024 56.1 us with KS = 1, 51.0 with 8;
// with ONCE, weights past the caches, 48.7, of 1024 x 4096 44.7: 5.6 and 6.1 TB/s, a plain read on this chip 6.2).  Two and four blocks requested at once were no faster where KS suits the launch.
// Y = void: quantised again, YQ, which takes a whole block of 128 outputs, KS = 1 (twice the wavefronts for half the inputs each: no faster).
constexpr int FEW_THREADS = 512;
template <int XQ, typename Y, int YQ, bool VEC, int KS, bool ONCE>
__global__ __launch_bounds__(FEW_THREADS) void matmul_few_rows_kernel(const MatmulArgs a) {
    constexpr int TILES = 8 / KS;  // of a workgroup
    __shared__ float amax_of[8][16];
    __shared__ floatx4 parts[KS > 1 ? 8 : 1][64];
    const int part = blockIdx.x % KS, item = blockIdx.x / KS, chunk = item / a.NB, nb = item - chunk * a.NB;
    const MatmulChunk ci = matmul_chunk<16>(a, chunk);
    if (ci.nrows <= 0) return;  // uniform over the workgroup
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tile = part * TILES + wave % TILES, ks = wave / TILES;
    const int row = ci.row0 + min(lane & 15, ci.nrows - 1), first = a.KB * ks / KS, last = a.KB * (ks + 1) / KS;
    const uint8_t *x = a.x + (size_t)row * a.x_stride + (lane >> 4) * 16;
    const uint8_t *w = a.w + (((size_t)ci.expert * a.NB + nb) * 8 + tile) * a.KB * FP8_TILE + lane * 16;
    const float *sx = a.x_scale + row, *sw = a.w_scale + ((size_t)ci.expert * a.NB + nb) * a.KB;
    struct Block {
        intx4 w[2], x[2];
        float s, t;
    };
    auto load = [&](Block &b, int kb) {
        const int k = min(kb, a.KB - 1);  // past the end the last block again, which nobody uses: no conditions in front of loads
        const uint8_t *wk = w + (size_t)k * FP8_TILE, *xk = x + (size_t)k * FP8_BLOCK;
        b.w[0] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const intx4 *>(wk)) : *reinterpret_cast<const intx4 *>(wk);
        b.w[1] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const intx4 *>(wk + 1024)) : *reinterpret_cast<const intx4 *>(wk + 1024);
        b.x[0] = *reinterpret_cast<const intx4 *>(xk);
        b.x[1] = *reinterpret_cast<const intx4 *>(xk + 64);
        b.s = sx[(size_t)k * a.x_scale_stride];
        b.t = sw[k];
    };
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    Block at, next;
    load(at, first);
    for (int kb = first; kb < last; ++kb) {
        load(next, kb + 1);
        const floatx4 p = product(operand<PGMOE_E4M3>(at.w[0], at.w[1]), operand<XQ>(at.x[0], at.x[1]));
        const float s = at.s * at.t;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[v] = fmaf(s, p[v], acc[v]);
        at = next;
    }
    if constexpr (KS > 1) {
        parts[wave][lane] = acc;
        __syncthreads();
        if (ks > 0) return;
#pragma unroll
        for (int i = 1; i < KS; ++i) acc += parts[wave + i * TILES][lane];
    }
    if (a.relu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = relu_of(acc[i]);
    }
    const bool live = (lane & 15) < ci.nrows;
    const int o = nb * FP8_BLOCK + tile * 16 + 4 * (lane >> 4);
    if constexpr (std::is_void<Y>::value) {
        // past the last output are zeros, also where a row or a scale that is not finite made NaN of the weights' zeros
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = o + i < a.n_out ? acc[i] : 0.f;
        auto largest = [&](auto of) {  // of the row's 128 results: four a lane, 16 a wavefront
            float m = maximum(maximum(of(acc[0]), of(acc[1])), maximum(of(acc[2]), of(acc[3])));
            m = maximum(m, __shfl_xor(m, 16));
            m = maximum(m, __shfl_xor(m, 32));
            if (lane < 16) amax_of[wave][lane] = m;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) m = maximum(m, amax_of[i][lane & 15]);
            return m;
        };
        float amax = largest([](float v) { return fabsf(v); });
        if (fp8_unusual<YQ>(amax)) {  // of the same 16 rows in every wavefront
            __syncthreads();
            amax = largest(finite_magnitude);
        }
        const float scale = fp8_scale<YQ>(amax);
        const Fp8CarefulDivisor by(scale);
        if (live) {
            *reinterpret_cast<uint32_t *>(a.y_q + (size_t)row * a.y_q_stride + o) = fp8_pack<YQ>(by(acc[0]), by(acc[1]), by(acc[2]), by(acc[3]));
            if (wave == 0 && lane < 16) a.y_scale[(size_t)nb * a.y_scale_stride + row] = scale;
        }
    } else {
        if (live) store_four<Y, VEC>(a, row, o, acc);
    }
}

// Many rows an expert.  An item is up to TM * 64 rows of one expert and 256 outputs; a workgroup, one per CU, takes every
// gridDim-th of them.  Both operands go straight from memory into a ring of NS stages in LDS, a stage being one block of 128
// inputs, its scales among them; the requests run ahead of the products without regard to where an item ends, so the first
// stages of an item arrive, and the results of the one before leave, under products.  Items of up
// to 256 rows: eight wavefronts as 2 x 4, wavefront (wn, wm) with 128 outputs (one scale) and the row tiles wm, wm + 4, ..; of up to 64 rows:
// 8 x 1, 32 outputs and all row tiles each (4 + 4 of 16 conversions a block of inputs, where 2 x 4 would take 8 + 1).
// 32768 rows over 128 experts of 1024 x 4096 take 318 us with bfloat16 results, 324 to 338 with quantised ones (0.81 to 0.85 PFLOP/s); the products alone
// would take 204.  In trials that left work out, bfloat16 results, 312 us then: without loads 258, without stores 285, without either 236, of which
// 32 are conversions and scales beside the products.  8192 rows of one of 4096 x 4096 1.30 PFLOP/s, 4099 over eight of 2048 x 768 (1.2 us a block, one item for
// 204 of 256 CUs) 25 to 26 us.
//
// LDS, a stage: 16 weight tiles of 2 KiB, 64 bytes more behind each; rows of 128 bytes whose 16-byte pieces are
// exchanged among themselves, piece c of row r at place c ^ (r / 2 % 8); 256 bytes of scales from each wavefront (rows: the
// first four; weights: the fifth's first two).  Both operands are then read without bank conflicts.
//
// The outputs are dealt to the matrix instruction's 16 rows so that what a lane stores at once is 16 bytes, and what the four lanes of
// a row store is 64 bytes side by side: with RUN = 16 / bytes of a result, row i of the a-th product is output
// 4 RUN (4 a / RUN) + RUN (i / 4) + 4 a % RUN + i % 4 of the wavefront's 128 (a lane's four results of a product are rows 4 (lane / 16) ..).
// (Of 32 outputs a lane has 8 codes at most.)
// With 64 bytes a lane in a row, stores of 16 bytes went to 64 places at once: an item ended 5 us later.
constexpr int MATMUL_W_TILE = FP8_TILE + 64;
// The shape of an item: up to TM * 64 rows and 256 outputs; a wavefront has OT tiles of 16 outputs and every WM-th row tile.
template <int TM_, int OT_>
struct MatmulShape {
    static constexpr int TM = TM_, OT = OT_, COLS = 16 / OT, WM = 8 / COLS, MC = TM * 4 / WM;  // MC: most row tiles of a wavefront
    static constexpr int W = 16 * MATMUL_W_TILE, X = TM * 64 * FP8_BLOCK, S = 8 * 256, STAGE = W + X + S;
    static constexpr int TABLE = 3 * PGMOE_MAX_EXPERTS * 4, MAXIMA = OT < 8 ? 8 * 64 * 4 : 0;
    static constexpr int NS = (160 * 1024 - TABLE - MAXIMA) / STAGE, BYTES = NS * STAGE + TABLE + MAXIMA;
    static constexpr int LOADS = 4 + TM + 1;
    static_assert(NS >= 2 && MC <= 4 && (OT == 8 || (OT == 2 && WM == 1)), "a ring; one of the two wavefront shapes below");
};
constexpr int TILE_THREADS = 512, TILE_GROUPS = 256;  // workgroups: one per CU

// The lane's number, worked out where it is asked for: what depends on it is then not kept in registers across the products, where
// every register is in use (one value reloaded from scratch memory is a wait for all requests before it).
__device__ inline int lane_again() {
    int lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    return lane;
}

// The items of a launch, looked up in a table of the experts in LDS: chunks up to and with the expert, its first row, its rows.
// An expert's chunks are full ones of `most` rows and what is left over: of 270 rows 256 and 14, which take 4 + 1 units of work where two of 135
// would take 3 + 3 (4096 rows of one expert of 1024 x 4096 37.9 -> 36.7 us, 32768 over 128 as long either way).  `most` is that of 1 .. MC units (16 WM rows)
// for which the launch should end first: rounds of one item a workgroup, times what a block of inputs costs an item on the mean,
// which is MATMUL_COST + its units.
struct MatmulItem {
    int expert, row0, nrows, nb;  // nrows == 0: there are no more
};
constexpr int MATMUL_COST = 1;
template <typename R>
struct MatmulItems {
    static constexpr int TM = R::TM;
    const int *table;
    int cols, total, most;  // column blocks; chunks; rows of one
    // Offsets are clamped to the rows there are, whatever they say.
    __device__ void build(const MatmulArgs &a, int *to) {
        const int lane = threadIdx.x & 63;
        int lo[4], n[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // all at once
            const int e = q * 64 + lane;
            lo[q] = a.offsets[min(e, a.E)];
            n[q] = a.offsets[min(e + 1, a.E)];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lo[q] = max(0, min(lo[q], a.rows));
            n[q] = max(lo[q], min(n[q], a.rows)) - lo[q];
        }
        cols = (a.NB + 1) / 2;
        most = TM * 64;
        if (R::OT == 8) {
            float best = INFINITY;
            static_for<R::MC>([&](auto u_) {
                constexpr int UNIT = 16 * R::WM, MOST = UNIT * (R::MC - decltype(u_)::value);
                int sum = 0;
                float cost = 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = (n[q] + MOST - 1) / MOST;
                    sum += c;
                    cost += (float)(c * MATMUL_COST + (n[q] + UNIT - 1) / UNIT);
                }
                const int chunks = __builtin_amdgcn_readlane(wave_incl_scan(sum), 63);
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) cost += __shfl_xor(cost, m);
                const float t = (float)((chunks * (int64_t)cols + gridDim.x - 1) / gridDim.x) * cost / (float)max(1, chunks);
                if (t < best) {  // uniform
                    best = t;
                    most = MOST;
                }
            });
        }
        most = __builtin_amdgcn_readfirstlane(most);
        int before = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = (n[q] + most - 1) / most, c_incl = before + wave_incl_scan(c);
            before = __builtin_amdgcn_readlane(c_incl, 63);
            if (threadIdx.x < 64) {
                const int e = q * 64 + lane;
                to[e] = c_incl;
                to[PGMOE_MAX_EXPERTS + e] = lo[q];
                to[2 * PGMOE_MAX_EXPERTS + e] = n[q];
            }
        }
        table = to;
        total = before;
    }
    // Item number i.  Workgroups go to the 8 XCDs in turn: the column blocks of a chunk stay on one and share its rows in its L2.
    __device__ MatmulItem at(int i) const {
        const int turn = i >> 3, group = turn / cols, chunk = group * 8 + (i & 7);
        if (chunk >= total) return {0, 0, 0, 0};
        const intx4 c = *reinterpret_cast<const intx4 *>(table + 4 * lane_again());
        int e = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) e += __popcll(__ballot(c[q] <= chunk));
        const int before = e ? __builtin_amdgcn_readfirstlane(table[e - 1]) : 0, first = __builtin_amdgcn_readfirstlane(table[PGMOE_MAX_EXPERTS + e]);
        const int rows = __builtin_amdgcn_readfirstlane(table[2 * PGMOE_MAX_EXPERTS + e]), from = (chunk - before) * most;
        return {e, first + from, max(1, min(most, rows - from)), (turn - group * cols) * 2};
    }
};

__device__ inline void load_two_tiles_once(const char *src, unsigned lane_off, unsigned lds_tile) {  // load_two_tiles_to_lds, past the caches
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt\n\tglobal_load_lds_dwordx4 %0, %1 offset:1024 nt" ::"v"(lane_off), "s"(src), "s"(lds_tile)
                 : "memory", "m0");
}

// What a wavefront requests: the blocks of its workgroup's items one after the other.
template <typename R>
struct MatmulRequests {
    static constexpr int TM = R::TM;
    const uint8_t *w_src, *x_src;
    const float *s_src;
    unsigned w_second, lds, stage;  // bytes to the wavefront's second weight tile; LDS address of the ring
    int s_last, s_by, x_last;
    size_t s_step;
    int item, left, ahead;  // next item to look up; blocks of the present one that are not requested; requested blocks not yet multiplied
    __device__ void start(char *ring, int first_item) {
        lds = __builtin_amdgcn_readfirstlane(lds_address(ring));
        item = first_item;
        left = ahead = 0;
        stage = 0;
    }
    __device__ void next(const MatmulArgs &a, const MatmulItems<R> &items, int wave) {
        const int lane = lane_again();
        if (left == 0) {  // uniform
            const MatmulItem it = items.at(item);
            if (it.nrows == 0) return;
            item += gridDim.x;
            left = a.KB;
            const size_t block = (size_t)it.expert * a.NB + it.nb;
            const int last = it.nb + 1 < a.NB ? 15 : 7;  // an odd last block of outputs has no neighbour
            w_src = a.w + (block * 8 + min(wave * 2, last)) * a.KB * FP8_TILE;
            w_second = wave * 2 < last ? (unsigned)a.KB * FP8_TILE : 0;
            x_src = a.x + (size_t)it.row0 * a.x_stride;
            x_last = it.nrows - 1;
            // scales: of the rows, 64 from each of the first four wavefronts; of the two blocks of outputs
            s_src = wave < 4 ? a.x_scale + it.row0 : a.w_scale + block * a.KB;
            s_step = wave < 4 ? a.x_scale_stride : 1;
            s_by = wave < 4 ? 4 : 4 * a.KB;
            s_last = wave < 4 ? it.nrows - 1 : (last == 15 ? 1 : 0);
        }
        const unsigned to = lds + stage;
        if (a.once) {  // uniform; as many loads either way
            load_two_tiles_once((const char *)w_src, lane * 16, to + wave * 2 * MATMUL_W_TILE);
            load_two_tiles_once((const char *)w_src + w_second, lane * 16, to + (wave * 2 + 1) * MATMUL_W_TILE);
        } else {
            load_two_tiles_to_lds((const char *)w_src, lane * 16, to + wave * 2 * MATMUL_W_TILE);
            load_two_tiles_to_lds((const char *)w_src + w_second, lane * 16, to + (wave * 2 + 1) * MATMUL_W_TILE);
        }
        w_src += FP8_TILE;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int row = (wave * TM + i) * 8 + (lane >> 3);
            const unsigned off = (unsigned)min(row, x_last) * (unsigned)a.x_stride + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
            load_tile_to_lds((const char *)x_src, off, to + R::W + (wave * TM + i) * 1024);
        }
        x_src += FP8_BLOCK;
        load_dwords_to_lds(s_src, (unsigned)min((wave & 3) * 64 + lane, s_last) * (unsigned)s_by, to + R::W + R::X + wave * 256);
        s_src += s_step;
        stage = stage + R::STAGE == R::NS * R::STAGE ? 0 : stage + R::STAGE;
        --left;
        ++ahead;
    }
};

// Waits until, at most, the loads of `later` more requests and the stores of `tiles` row tiles are outstanding: operations complete in order.
template <int LATER, int LOADS, int STORES>
__device__ inline void wait_for_loads(int later, int tiles) {  // uniform; later 0 .. LATER, tiles 0 .. 4
    static_for<LATER + 1>([&](auto l_) {
        static_for<5>([&](auto t_) {
            constexpr int l = decltype(l_)::value, t = decltype(t_)::value, n = l * LOADS + t * STORES;
            if (later == l && tiles == t) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n < 63 ? n : 63) : "memory");
        });
    });
}

// The products of one item.  stored: row tiles whose results the wavefront stored behind the requests that are outstanding.
template <int XQ, typename R, int MC, int RUN, int STORES>
__device__ inline void matmul_k_loop(const MatmulArgs &a, const MatmulItems<R> &items, MatmulRequests<R> &rq, const char *ring, unsigned &stage, int wave, int stored,
                                     floatx4 (&acc)[R::OT][MC > 0 ? MC : 1]) {
    const int wn = wave % R::COLS, wm = wave / R::COLS;
    constexpr int PER = RUN / 4;  // products of a run
    auto place = [](int t) { return t / PER * PER * MATMUL_W_TILE + t % PER * 64; };
    for (int kb = 0; kb < a.KB; ++kb) {
        // This block's loads have landed: those of the later ones, and stores behind them all, may be outstanding.
        wait_for_loads<R::NS - 2, R::LOADS, STORES>(min(rq.ahead - 1, R::NS - 2), kb <= R::NS - 2 ? stored : 0);
        // Behind the barrier they have for everyone, and everyone has read the block before, whose stage the next request takes.
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (MC == 0 || R::OT == 8) {
            rq.next(a, items, wave);
            --rq.ahead;
        }
        if (MC > 0) {
            const int lane = lane_again(), g = lane >> 4, i16 = lane & 15;
            const int o0 = RUN * (i16 >> 2) + (i16 & 3);  // this lane's output of product 0
            const char *w_at = ring + (wn * R::OT + (o0 >> 4)) * MATMUL_W_TILE + (o0 & 15) * 16 + g * 256;
            const char *x_at = ring + R::W + (wm * 16 + i16) * FP8_BLOCK;
            const int x_low = (g ^ (i16 >> 1)) << 4, x_high = ((4 + g) ^ (i16 >> 1)) << 4;
            const char *s_at = ring + R::W + R::X;
            float s[MC > 0 ? MC : 1];
            const float sw = *reinterpret_cast<const float *>(s_at + stage + 4 * 256 + wn * R::OT / 8 * 4);
#pragma unroll
            for (int m = 0; m < MC; ++m) s[m] = sw * *reinterpret_cast<const float *>(s_at + stage + ((wm + R::WM * m) * 16 + i16) * 4);
            auto row_codes = [&](int m, intx4(&to)[2]) {
                const char *r = x_at + stage + m * 16 * R::WM * FP8_BLOCK;
                to[0] = *reinterpret_cast<const intx4 *>(r + x_low);
                to[1] = *reinterpret_cast<const intx4 *>(r + x_high);
            };
            auto codes = [&](int t, intx4(&to)[2]) {
                to[0] = *reinterpret_cast<const intx4 *>(w_at + stage + place(t));
                to[1] = *reinterpret_cast<const intx4 *>(w_at + stage + place(t) + 1024);
            };
            Operand x[R::OT == 8 && MC > 0 ? MC : 1];
            if constexpr (R::OT == 8) {
#pragma unroll
                for (int m = 0; m < MC; ++m) {
                    intx4 raw[2];
                    row_codes(m, raw);
                    x[m] = operand<XQ>(raw[0], raw[1]);
                }
            }
            // A step is two chains of products.  Beside them run what the step before left to do (its sums into the accumulators) and the
            // conversion of weights that come next, dealt out behind the products one by one: the vector unit's work fits under the
            // matrix cores' then, in a wavefront by itself.
            if constexpr (R::OT == 2) {  // the chains are the two output tiles; rows come one tile after the other
                intx4 raw[2], first[3][2];
                codes(0, first[0]);
                codes(1, first[1]);
                row_codes(0, first[2]);
                if (MC > 1) row_codes(1, raw);
                rq.next(a, items, wave);  // while the first operands are on their way from LDS
                --rq.ahead;
                Operand w[2] = {operand<PGMOE_E4M3>(first[0][0], first[0][1]), operand<PGMOE_E4M3>(first[1][0], first[1][1])}, x_next;
                x[0] = operand<XQ>(first[2][0], first[2][1]);
                floatx4 before[2];
                static_for<MC>([&](auto m_) {
                    constexpr int m = decltype(m_)::value;
                    __builtin_amdgcn_sched_barrier(0);
                    floatx4 p[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j].part[i], x[0].part[i], p[j], 0, 0, 0);
                    if constexpr (m > 0) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[j][m - 1][v] = fmaf(s[m - 1], before[j][v], acc[j][m - 1][v]);
                    }
                    if constexpr (m + 1 < MC) {
                        x_next = operand<XQ>(raw[0], raw[1]);
                        if constexpr (m + 2 < MC) row_codes(m + 2, raw);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) before[j] = p[j];
                    x[0] = x_next;
                });
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[j][MC - 1][v] = fmaf(s[MC - 1], before[j][v], acc[j][MC - 1][v]);
            } else if constexpr (MC == 1) {  // one row tile: the chains are two output tiles
                intx4 next[2][2];
                codes(0, next[0]);
                codes(1, next[1]);
                Operand w[2] = {operand<PGMOE_E4M3>(next[0][0], next[0][1]), operand<PGMOE_E4M3>(next[1][0], next[1][1])}, w_next[2];
                codes(2, next[0]);
                codes(3, next[1]);
                floatx4 before[2];
                static_for<4>([&](auto step_) {
                    constexpr int step = decltype(step_)::value;
                    __builtin_amdgcn_sched_barrier(0);
                    floatx4 p[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j].part[i], x[0].part[i], p[j], 0, 0, 0);
                    if constexpr (step > 0) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[2 * step - 2 + j][0][v] = fmaf(s[0], before[j][v], acc[2 * step - 2 + j][0][v]);
                    }
                    if constexpr (step < 3) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            w_next[j] = operand<PGMOE_E4M3>(next[j][0], next[j][1]);
                            if constexpr (step < 2) codes(2 * step + 4 + j, next[j]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 5, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        before[j] = p[j];
                        w[j] = w_next[j];
                    }
                });
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[6 + j][0][v] = fmaf(s[0], before[j][v], acc[6 + j][0][v]);
            } else {
            constexpr int HALVES = MC > 2 ? 2 : 1, HM = 2;  // row tiles: the chains are two of them
            Operand w = operand<PGMOE_E4M3>(*reinterpret_cast<const intx4 *>(w_at + stage), *reinterpret_cast<const intx4 *>(w_at + stage + 1024)), w_next;
            intx4 low = *reinterpret_cast<const intx4 *>(w_at + stage + place(1)), high;
            floatx4 before[HM];
            static_for<8 * HALVES>([&](auto step_) {
                constexpr int step = decltype(step_)::value, t = step / HALVES, h = step % HALVES;
                __builtin_amdgcn_sched_barrier(0);
                floatx4 p[HM];
#pragma unroll
                for (int j = 0; j < HM; ++j) p[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < HM; ++j)
                        if (2 * h + j < MC) p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[i], x[2 * h + j].part[i], p[j], 0, 0, 0);
                if constexpr (step > 0) {
                    constexpr int tb = (step - 1) / HALVES, hb = (step - 1) % HALVES;
#pragma unroll
                    for (int j = 0; j < HM; ++j)
                        if (2 * hb + j < MC) {
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[tb][2 * hb + j][v] = fmaf(s[2 * hb + j], before[j][v], acc[tb][2 * hb + j][v]);
                        }
                }
                if constexpr (t < 7) {
                    if constexpr (h == 0) {
                        w_next.part[0] = widen<PGMOE_E4M3>(low[0], low[1]);
                        w_next.part[1] = widen<PGMOE_E4M3>(low[2], low[3]);
                        high = *reinterpret_cast<const intx4 *>(w_at + stage + place(t + 1) + 1024);
                    }
                    if constexpr (h == HALVES - 1) {
                        w_next.part[2] = widen<PGMOE_E4M3>(high[0], high[1]);
                        w_next.part[3] = widen<PGMOE_E4M3>(high[2], high[3]);
                        if constexpr (t < 6) low = *reinterpret_cast<const intx4 *>(w_at + stage + place(t + 2));
                    }
                }
#pragma unroll
                for (int i = 0; i < 4 * HM; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);   // a product
                    __builtin_amdgcn_sched_group_barrier(0x2, HALVES == 1 ? 3 : 2, 0);  // what runs beside it
                }
#pragma unroll
                for (int j = 0; j < HM; ++j) before[j] = p[j];
                if constexpr (h == HALVES - 1) w = w_next;
            });
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < HM; ++j)
                if (2 * (HALVES - 1) + j < MC) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[7][2 * (HALVES - 1) + j][v] = fmaf(s[2 * (HALVES - 1) + j], before[j][v], acc[7][2 * (HALVES - 1) + j][v]);
                }
            }
        }
        stage = stage + R::STAGE == R::NS * R::STAGE ? 0 : stage + R::STAGE;
    }
}

// Stores of one row tile of a wavefront whose 128 outputs are all there.
template <typename Y, bool VEC, int OT>
constexpr int tile_stores() {
    if constexpr (std::is_void<Y>::value) return OT == 8 ? 3 : 1;
    else return VEC ? (sizeof(Y) == 4 ? OT : OT / 2) : 4 * OT;
}
template <typename Y, int OT>
constexpr int run_of() {  // results in 16 bytes, as far as a wavefront's outputs go
    if constexpr (std::is_void<Y>::value) return OT == 8 ? 16 : 8;
    else return 16 / sizeof(Y);
}

template <int XQ, typename Y, int YQ, bool VEC, typename R, int MC>
__device__ inline int matmul_item(const MatmulArgs &a, const MatmulItems<R> &items, MatmulRequests<R> &rq, const MatmulItem &it, char *ring, unsigned &stage, int wave,
                                  int stored) {
    constexpr int RUN = run_of<Y, R::OT>(), STORES = tile_stores<Y, VEC, R::OT>(), OT = R::OT;
    floatx4 acc[OT][MC > 0 ? MC : 1];
#pragma unroll
    for (int i = 0; i < OT; ++i)
#pragma unroll
        for (int m = 0; m < MC; ++m) acc[i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
    matmul_k_loop<XQ, R, MC, RUN, STORES>(a, items, rq, ring, stage, wave, stored, acc);
    const int lane = lane_again(), wn = wave % R::COLS, wm = wave / R::COLS;
    const int block = it.nb + wn * OT / 8, o = it.nb * FP8_BLOCK + wn * OT * 16 + RUN * (lane >> 4);  // run r of the lane begins at o + 4 RUN r
    if (OT == 8 && block >= a.NB) return 0;
    if (a.relu) {
#pragma unroll
        for (int m = 0; m < MC; ++m)
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][m][v] = relu_of(acc[i][m][v]);
    }
    float amax[MC > 0 ? MC : 1];  // of a row's block, where that is quantised
    bool unusual = false;
    if constexpr (std::is_void<Y>::value) {
        // past the last output are zeros, also where a row or a scale that is not finite made NaN of the weights' zeros
        if ((block + 1) * FP8_BLOCK > a.n_out) {
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const bool there = o + 4 * RUN * (4 * i / RUN) + 4 * i % RUN + v < a.n_out;
#pragma unroll
                    for (int m = 0; m < MC; ++m) acc[i][m][v] = there ? acc[i][m][v] : 0.f;
                }
        }
        auto largest = [&](auto of) {
#pragma unroll
            for (int m = 0; m < MC; ++m) {
                float l = 0.f;
#pragma unroll
                for (int i = 0; i < OT; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) l = maximum(l, of(acc[i][m][v]));
                l = maximum(l, __shfl_xor(l, 16));
                amax[m] = maximum(l, __shfl_xor(l, 32));
            }
            if constexpr (OT < 8) {  // four wavefronts have a block's outputs.  (No barrier of the compiler's: it would wait for the requests.)
                float *maxima = reinterpret_cast<float *>(ring + R::NS * R::STAGE + R::TABLE);
#pragma unroll
                for (int m = 0; m < MC; ++m)
                    if (lane < 16) maxima[wave * 64 + m * 16 + lane] = amax[m];
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
                for (int m = 0; m < MC; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) amax[m] = maximum(amax[m], maxima[((wave & 4) + i) * 64 + m * 16 + (lane & 15)]);
            }
        };
        largest([](float v) { return fabsf(v); });
#pragma unroll
        for (int m = 0; m < MC; ++m) {
            unusual |= fp8_unusual<YQ>(amax[m]);
            if constexpr (OT < 8) {  // the other block's rows too: if one wavefront looks again all do, they meet at barriers there
                const float *others = reinterpret_cast<const float *>(ring + R::NS * R::STAGE + R::TABLE) + (4 - (wave & 4)) * 64 + m * 16 + (lane & 15);
                unusual |= fp8_unusual<YQ>(maximum(maximum(others[0], others[64]), maximum(others[128], others[192])));
            }
        }
        if (unusual) {
            if (OT < 8) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            largest(finite_magnitude);
        }
    }
    if (block >= a.NB) return 0;
#pragma unroll
    for (int m = 0; m < MC; ++m) {
        const int in_chunk = (wm + R::WM * m) * 16 + (lane & 15), row = it.row0 + in_chunk;
        const bool live = in_chunk < it.nrows;
        if constexpr (std::is_void<Y>::value) {
            const float scale = fp8_scale<YQ>(amax[m]);
            uint32_t codes[OT];
            auto quantise = [&](auto by) {
#pragma unroll
                for (int i = 0; i < OT; ++i) codes[i] = fp8_pack<YQ>(by(acc[i][m][0]), by(acc[i][m][1]), by(acc[i][m][2]), by(acc[i][m][3]));
            };
            if (unusual) quantise(Fp8CarefulDivisor(scale));
            else quantise(Fp8Divisor(scale));
            if (live) {
                uint8_t *q = a.y_q + (size_t)row * a.y_q_stride + o;
                if constexpr (OT == 8) {
                    reinterpret_cast<uint4 *>(q)[0] = make_uint4(codes[0], codes[1], codes[2], codes[3]);
                    reinterpret_cast<uint4 *>(q)[4] = make_uint4(codes[4], codes[5], codes[6], codes[7]);
                } else {
                    *reinterpret_cast<uint2 *>(q) = make_uint2(codes[0], codes[1]);
                }
                if (lane < 16 && (OT == 8 || (wave & 3) == 0)) a.y_scale[(size_t)block * a.y_scale_stride + row] = scale;
            }
        } else if (live) {
            if constexpr (VEC && sizeof(Y) == 2) {
                typedef Y Yx8 __attribute__((ext_vector_type(8), aligned(8)));
#pragma unroll
                for (int i = 0; i < OT; i += 2) {
                    const int at = o + 16 * i;
                    const floatx4 u = acc[i][m], v = acc[i + 1][m];
                    if (at + 4 < a.n_out)
                        *reinterpret_cast<Yx8 *>(reinterpret_cast<Y *>(a.y) + (size_t)row * a.y_stride + at) =
                            Yx8{(Y)u[0], (Y)u[1], (Y)u[2], (Y)u[3], (Y)v[0], (Y)v[1], (Y)v[2], (Y)v[3]};
                    else store_four<Y, true>(a, row, at, u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < OT; ++i) store_four<Y, VEC>(a, row, o + 4 * RUN * (4 * i / RUN) + 4 * i % RUN, acc[i][m]);
            }
        }
    }
    return (block + 1) * FP8_BLOCK <= a.n_out ? MC : 0;  // every row tile has a live row: STORES were issued for each
}

template <int XQ, typename Y, int YQ, bool VEC, typename R>
__global__ __launch_bounds__(TILE_THREADS, 2) void matmul_tiles_kernel(const MatmulArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char ring[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    MatmulItems<R> items;
    items.build(a, reinterpret_cast<int *>(ring + R::NS * R::STAGE));
    __syncthreads();
    MatmulRequests<R> rq;
    rq.start(ring, blockIdx.x);
#pragma unroll
    for (int st = 0; st < R::NS - 1; ++st) rq.next(a, items, wave);
    unsigned stage = 0;
    int stored = 0;
    for (int i = blockIdx.x;; i += gridDim.x) {
        const MatmulItem it = items.at(i);
        if (it.nrows == 0) break;  // uniform over the workgroup; every request has been waited for
        const int rt = (it.nrows + 15) >> 4, own = max(0, (rt - wave / R::COLS + R::WM - 1) / R::WM);
        switch (own) {  // uniform over the wavefront
#define PG_BODY(MC_)                                                                                                                        \
    case MC_:                                                                                                                               \
        if constexpr (MC_ <= R::MC) stored = matmul_item<XQ, Y, YQ, VEC, R, MC_>(a, items, rq, it, ring, stage, wave, stored);               \
        asm volatile("; %0 row tiles" ::"n"(MC_)); /* keeps the bodies' stores apart */                                                      \
        break;
            PG_BODY(0) PG_BODY(1) PG_BODY(2) PG_BODY(3) PG_BODY(4)
#undef PG_BODY
        }
    }
}

constexpr int64_t TILE_STRIDE_MAX = 1 << 23;  // bytes: offsets within a chunk of 256 rows have 31 bits

template <int XQ, typename Y, int YQ, bool VEC, typename R>
static int launch_tiles(const MatmulArgs &a, hipStream_t s) {
    // more than 48 KiB of LDS: the kernel's limit is raised once per device
    static std::atomic<uint64_t> raised{0};
    int device = 0;
    if (const hipError_t e = hipGetDevice(&device)) return e == hipErrorNoDevice ? fail(nullptr, PGMOE_ENODEVICE, "pgmoe_expert_matmul: no HIP device is visible") : hip_fail(nullptr, e, "hipGetDevice");
    if (!(raised.load(std::memory_order_relaxed) >> (device & 63) & 1)) {
        const void *kernel = reinterpret_cast<const void *>(&matmul_tiles_kernel<XQ, Y, YQ, VEC, R>);
        PG_HIP(nullptr, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, R::BYTES));
        raised.fetch_or(1ull << (device & 63), std::memory_order_relaxed);
    }
    // chunks: at most the sum over the experts of ceil(rows / the smallest the kernel may choose), in whole eights
    constexpr int UNIT = R::OT == 8 ? 16 * R::WM : R::TM * 64;
    const int64_t chunks = ((a.rows + (int64_t)(UNIT - 1) * std::min(a.E, a.rows)) / UNIT + 7) & ~(int64_t)7;
    const unsigned groups = (unsigned)std::min<int64_t>(TILE_GROUPS, chunks * ((a.NB + 1) / 2));
    hipLaunchKernelGGL((matmul_tiles_kernel<XQ, Y, YQ, VEC, R>), dim3(groups), dim3(TILE_THREADS), R::BYTES, s, a);
    return PGMOE_OK;
}
// Which kernel, by what there is to deal out; both sides in us a launch, bf16 results, rows dealt to the experts at random,
// weights through the caches:
//  * few rows, to 8 an expert: the tiles would be empty mostly (64 experts of 1024 x 4096, 8 rows each 50.4, in tiles of 64 rows 52.1; 12 rows
//    54.7 / 52.4); also launches of at most two items of 16 rows a CU (64 rows for each of 8 experts of 4096 x 1024 23.3 / 44.2, 128 41.0 / 43.8,
//    256 for one of 1024 x 4096 11.8 / 15.0; not 512 21.3 / 15.1, 48 for each of 8 19.5 / 14.9), and rows too far apart for the tiles;
//  * tiles of 64 rows or of up to 256, by rounds of one item a workgroup, of which the larger take 4 / 3 as long (32 for each of 64 experts of
//    1024 x 4096 55.9 / 63.6, 64 rows 79.7 / 75.8; 512 for each of 8 of 2048 x 768 26.5 / 31.0, 1024 46.3 / 39.4; 96 for each of 8 of
//    1024 x 4096 17.0 / 20.4, 128 27.1 / 24.4).  An expert has half a chunk more than its rows fill, on the mean.
// The inputs of few rows are split so that a wavefront has three blocks at least and there are 24 workgroups a CU at most (experts without rows
// leave empty ones: 128 rows over 46 of 128 experts of 4096 x 1024, room for 1024 items, KS = 1 / 2 / 4 / 8 39.4 / 40.3 / 36.8 / 38.4, of 1024 x 4096 36.9 / 38.6 /
// 45.2 / 64.2), further while workgroups are no more than two a CU: KS = 1 / 2 / 4 / 8
// take 33.9 / 33.2 / 32.3 / 43.0 for one row for each of 64 experts of 1024 x 4096 (eight blocks), 6.8 / 5.0 / 5.1 / 5.0 for 64 rows of one, 6.6 / 4.8 / 3.8 / 3.0
// for 16, 20.5 / 21.1 / 21.6 / 21.6 for 512 rows of one of 4096 x 1024, 38.2 / 31.5 / 25.5 / 23.7 for 64 for each of eight.
struct MatmulPlan {
    int tile;         // rows of an item of the tiled kernel, 64 or 256; 0: few rows
    int ks;           // few rows: wavefronts that share the inputs
    int64_t items16;  // few rows: pieces of 16 rows and 128 outputs, at most
};
static MatmulPlan matmul_plan(int rows, int E, int KB, int NB, int64_t x_stride, bool quantised) {
    const int64_t active = std::min(E, rows), mean = rows / active, cols = (NB + 1) / 2;
    const int64_t chunks16 = (rows + 15 * active) / 16, items16 = chunks16 * NB;
    if (mean > 8 && items16 > 2 * TILE_GROUPS && x_stride < TILE_STRIDE_MAX) {
        const auto rounds = [&](int most) { return (std::max(active, rows / most + active / 2) * cols + TILE_GROUPS - 1) / TILE_GROUPS; };
        return {3 * rounds(64) <= 4 * rounds(256) ? 64 : 256, 0, items16};
    }
    const auto split = [&](int ks) { return ks * items16 <= (3 * ks <= KB ? 24 : ks <= KB ? 2 : 0) * TILE_GROUPS; };
    return {0, quantised ? 1 : split(8) ? 8 : split(4) ? 4 : split(2) ? 2 : 1, items16};
}

template <int XQ, typename Y, int YQ, bool VEC, int KS>
static void launch_few_rows(const MatmulArgs &a, int64_t items16, hipStream_t s) {
    const dim3 grid((unsigned)(items16 * KS));
    if (a.once) hipLaunchKernelGGL((matmul_few_rows_kernel<XQ, Y, YQ, VEC, KS, true>), grid, dim3(FEW_THREADS), 0, s, a);
    else hipLaunchKernelGGL((matmul_few_rows_kernel<XQ, Y, YQ, VEC, KS, false>), grid, dim3(FEW_THREADS), 0, s, a);
}
template <int XQ, typename Y, int YQ, bool VEC>
static int launch_matmul(const MatmulArgs &a, hipStream_t s) {
    const MatmulPlan p = matmul_plan(a.rows, a.E, a.KB, a.NB, (int64_t)a.x_stride, std::is_void<Y>::value);
    if (p.tile == 64) return launch_tiles<XQ, Y, YQ, VEC, MatmulShape<1, 2>>(a, s);
    if (p.tile == 256) return launch_tiles<XQ, Y, YQ, VEC, MatmulShape<4, 8>>(a, s);
    if (p.items16 * p.ks * FEW_THREADS > GRID_THREADS_MAX)
        return fail(nullptr, PGMOE_EINVAL, "pgmoe_expert_matmul: %d rows by n_out=%d are more than one launch holds (%lld items of 16 rows and 128 outputs)", a.rows, a.n_out,
                    (long long)p.items16);
    if constexpr (!std::is_void<Y>::value) {
        if (p.ks == 8) return launch_few_rows<XQ, Y, YQ, VEC, 8>(a, p.items16, s), PGMOE_OK;
        if (p.ks == 4) return launch_few_rows<XQ, Y, YQ, VEC, 4>(a, p.items16, s), PGMOE_OK;
        if (p.ks == 2) return launch_few_rows<XQ, Y, YQ, VEC, 2>(a, p.items16, s), PGMOE_OK;
    }
    return launch_few_rows<XQ, Y, YQ, VEC, 1>(a, p.items16, s), PGMOE_OK;
}
template <int XQ, typename Y>
static int launch_matmul_to(const MatmulArgs &a, hipStream_t s) {
    // whole fours of outputs, each at an address that four results' bytes divide
    if (a.n_out % 4 == 0 && a.y_stride % 4 == 0 && aligned(a.y, 4 * sizeof(Y))) return launch_matmul<XQ, Y, 0, true>(a, s);
    return launch_matmul<XQ, Y, 0, false>(a, s);
}
template <int XQ>
static int launch_matmul(const MatmulArgs &a, int y_dtype, hipStream_t s) {
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
    if ((x->rows / 16 + (int64_t)w->n_experts + 8) * fp8_blocks(w->n_out) > 0x7fffff00)
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
    // Weights that the last-level cache (256 MB) does not hold until the next call, and that an expert's rows read once, pass by the caches: 16 rows for
    // each of 64 experts of 1024 x 4096 52.4 -> 47.4 us, 128 rows over 46 of 128 37.3 -> 35.0, 128 for each of 64 96.6 -> 94.0; not 32 for each of 128 of 1024 x 1024 (134 MB)
    // 27.6 / 30.4, nor 256 for each of 64 of 1024 x 4096, half of which have two chunks, 181 / 187.
    const int64_t active = std::min(a.E, a.rows);
    a.once = active * a.KB * a.NB * (8 * FP8_TILE) >= 256000000 && a.rows / active <= 128;
    a.y = y;
    a.y_stride = (size_t)y_stride;
    if (y_q) {
        a.y_q = (uint8_t *)y_q->q;
        a.y_q_stride = (size_t)y_q->q_stride;
        a.y_scale = y_q->scale;
        a.y_scale_stride = (size_t)y_q->scale_stride;
        y_dtype = y_q->dtype;
    }
    rc = x->dtype == PGMOE_E4M3 ? launch_matmul<PGMOE_E4M3>(a, y_dtype, (hipStream_t)stream) : launch_matmul<PGMOE_E5M2>(a, y_dtype, (hipStream_t)stream);
    return rc ? rc : launched(fn);
}

extern "C" const char *pgmoe_expert_matmul_kernel_name(const pgmoe_fp8_rows *x, const pgmoe_fp8_weights *w, int y_dtype) {
    if (!x || !w || x->rows < 1 || w->n_experts < 1 || w->n_in < 1 || w->n_out < 1) return nullptr;
    const MatmulPlan p = matmul_plan(x->rows, w->n_experts, fp8_blocks(w->n_in), fp8_blocks(w->n_out), x->q_stride, y_dtype == PGMOE_E4M3 || y_dtype == PGMOE_E5M2);
    return p.tile == 64 ? "matmul_tiles_kernel, 64 rows" : p.tile == 256 ? "matmul_tiles_kernel, 256 rows" : "matmul_few_rows_kernel";
}
