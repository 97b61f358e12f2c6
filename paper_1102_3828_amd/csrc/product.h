// Products of 16-bit matrices on the matrix cores: the part that the kernels of softmax.hip and ortho.hip share (not part of the ABI).
//
// D[p][q] = sum_k P(p, k) Q(q, k), fp32 accumulation (v_mfma_f32_16x16x32).  Each operand is held with k innermost ("inner": rows of p,
// contiguous in k) or with its own index innermost ("outer": rows of k, contiguous in p), so no product needs a transposed copy.
// Several 16-bit planes carry one fp32 operand (its leading part, what that leaves, what that leaves again); the product is then the sum
// over pairs of planes, one pair after the other on the same accumulators.
//
// A workgroup owns BM x BN outputs.  Stages of 32 k go straight from memory to LDS, four buffers, so that up to four stages are
// in flight; one barrier a stage.  The fragments of a stage are read from LDS into registers while the products of the stage before
// are formed.  16-byte chunks of a row lie permuted in LDS (by the row, as the source addresses choose), so that the lanes that LDS serves
// together read different banks; outer operands are transposed by the LDS read itself (ds_read_b64_tr_b16).
//
// Lane l of a wavefront holds, of the tile (tm, tn) of 16 x 16 at (p, q), the outputs q + (l & 15) and four consecutive p.
// With P inner the tiles 2 t and 2 t + 1 interleave, so that a lane has eight consecutive p in the pair (one 16-byte store of 16-bit values).
#pragma once

#include "ivfr_internal.h"

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

#define IVFR_PRODUCT_K 32        // k of a stage
#define IVFR_PRODUCT_STAGES 4    // LDS buffers
#define IVFR_PRODUCT_CU 256      // compute units that launches are cut for

struct ProductOperand {
    const uint16_t* base;   // plane 0, 16-byte aligned
    int64_t plane;          // elements between planes
    int64_t ld;             // elements between rows, a multiple of 8
    int extent;             // values of the operand's own index; beyond it the last one (inner), or its last chunk of eight (outer), is read again
    int rows;               // outer: rows of k that may be read; beyond them the last one is read again
};

// Pairs of planes (P, Q), four bits each.  Three planes of bf16 (24 bits of an fp32 value): the six products of which the
// largest neglected one is 2^-24 of the whole; two of fp16 (22 bits and a sign): without the product of the two rests, 2^-22.  Small ones first.
struct ProductPlanes {
    uint32_t p, q;
    int n;
};
inline ProductPlanes product_planes(int planes) {
    if (planes == 3) return {0x001012u, 0x010210u, 6};   // (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    if (planes == 2) return {0x001u, 0x010u, 3};         // (1,0) (0,1) (0,0)
    return {0u, 0u, 1};
}

// What a workgroup computes of a launch's tiles: XCDs take contiguous runs of them (blocks go round the eight XCDs, each with an L2 of its
// own), and a run walks over patches of eight tiles of p.
struct ProductTile {
    int p, q, split;
    bool any;
};
__device__ __forceinline__ ProductTile product_tile(int tiles_p, int tiles_q, int splits) {
    const uint32_t total = (uint32_t)tiles_p * (uint32_t)tiles_q * (uint32_t)splits, per = (total + 7) / 8;
    const uint32_t id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    ProductTile t = {0, 0, 0, (blockIdx.x >> 3) < per && id < total};
    const uint32_t each = (uint32_t)tiles_p * (uint32_t)tiles_q;
    const uint32_t split = id / each;
    const uint32_t in = id - split * each, band = 8u * (uint32_t)tiles_q, b = in / band, first = 8 * b;
    const uint32_t high = (uint32_t)tiles_p - first < 8u ? (uint32_t)tiles_p - first : 8u;
    // (uniform, but divisions are formed in vector registers, and the addresses made of these have to be in scalar ones)
    t.split = __builtin_amdgcn_readfirstlane((int)split);
    t.p = __builtin_amdgcn_readfirstlane((int)(first + (in - b * band) % high));
    t.q = __builtin_amdgcn_readfirstlane((int)((in - b * band) / high));
    return t;
}
inline unsigned product_grid(int64_t tiles) { return (unsigned)((tiles + 7) / 8 * 8); }

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, bool P_OUTER_, bool Q_OUTER_, bool HALF_>
struct Product {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    static constexpr bool P_OUTER = P_OUTER_, Q_OUTER = Q_OUTER_, HALF = HALF_;
    static constexpr int TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;
    static constexpr int KB = 2 * IVFR_PRODUCT_K;                               // bytes of a stage's k
    static constexpr int STAGE = (BM + BN) * KB;                                // bytes of a buffer
    static constexpr int LDS = IVFR_PRODUCT_STAGES * STAGE;
    static constexpr int P_LOADS = BM * KB / 1024, Q_LOADS = BN * KB / 1024;    // of 64 lanes x 16 bytes, a stage
    // Every wavefront issues the same number of loads, so that one count of those in flight holds for all (with fewer loads than
    // wavefronts some are issued twice, the same bytes to the same place).
    static constexpr int P_EACH = (P_LOADS + WAVES - 1) / WAVES, Q_EACH = (Q_LOADS + WAVES - 1) / WAVES, EACH = P_EACH + Q_EACH;
    static_assert(P_LOADS % WAVES == 0 || P_LOADS < WAVES, "");
    static_assert(Q_LOADS % WAVES == 0 || Q_LOADS < WAVES, "");
    static_assert(P_OUTER || TM % 2 == 0, "");
    static_assert(!P_OUTER || BM >= 64, "");
    static_assert(!Q_OUTER || BN >= 64, "");

    // permutation of the chunks of a row in LDS: inner rows have four of them
    static __device__ __forceinline__ int swz_p(int row) { return ((row >> 1) & 1) | ((row >> 2) & 2); }   // rows 0-3, 8-11 together
    static __device__ __forceinline__ int swz_q(int row) { return (row >> 1) & 3; }                        // rows 0-7 together
    static __device__ __forceinline__ int swz_k(int k) { return (k & 3) << 1; }                            // four rows of k together

    static __device__ __forceinline__ void load16(uint32_t lds, uint32_t offset, const uint16_t* base) {
        // (m0 has the LDS address; the compiler uses it for nothing else here.  No register is written, so none can be taken over early.)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
    }
    template <int IN_FLIGHT>
    static __device__ __forceinline__ void wait_and_meet() {   // all but so many loads of this wavefront are in LDS, its LDS reads are done; then the others' too
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(IN_FLIGHT) : "memory");
    }
    static __device__ __forceinline__ floatx4 mfma(short8v a, short8v b, floatx4 c) {
        if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }

    // byte offset, from the operand's first row or column of this tile and the stage's first k, of what lane `lane` of load `i` brings
    template <bool OUTER, int SIZE, bool IS_P>
    static __device__ __forceinline__ uint32_t source(int i, int lane, int64_t ld, int extent, int rows_left) {
        if constexpr (!OUTER) {
            const int row = 16 * i + (lane >> 2);
            const int chunk = (lane & 3) ^ (IS_P ? swz_p(row) : swz_q(row));
            return (uint32_t)(row < extent ? row : extent - 1) * (uint32_t)(2 * ld) + 16u * chunk;
        } else {
            constexpr int PER_ROW = SIZE / 8, ROWS = 64 / PER_ROW;
            const int k = ROWS * i + lane / PER_ROW, last = (extent - 1) >> 3;
            const int chunk = (lane % PER_ROW) ^ swz_k(k);
            return (uint32_t)(k < rows_left ? k : rows_left - 1) * (uint32_t)(2 * ld) + 16u * (chunk < last ? chunk : last);
        }
    }

    // The accumulators of one tile over the stages [first, first + count) of every pair of planes.  p0, q0: the tile's first p and q, below the
    // operands' extents.
    static __device__ __forceinline__ void run(const ProductOperand& P, const ProductOperand& Q, const ProductPlanes& planes, int p0, int q0, int first, int count,
                                               char* smem, floatx4 (&acc)[TM][TN]) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
        const uint16_t* const pb = P.base + (P_OUTER ? (int64_t)p0 : p0 * P.ld) + (int64_t)first * IVFR_PRODUCT_K * (P_OUTER ? P.ld : 1);
        const uint16_t* const qb = Q.base + (Q_OUTER ? (int64_t)q0 : q0 * Q.ld) + (int64_t)first * IVFR_PRODUCT_K * (Q_OUTER ? Q.ld : 1);
        const int64_t pstep = IVFR_PRODUCT_K * (P_OUTER ? P.ld : 1), qstep = IVFR_PRODUCT_K * (Q_OUTER ? Q.ld : 1);
        uint32_t po[P_EACH], qo[Q_EACH];
#pragma unroll
        for (int i = 0; i < P_EACH; ++i) po[i] = source<P_OUTER, BM, true>((wave + i * WAVES) % P_LOADS, lane, P.ld, P.extent - p0, IVFR_PRODUCT_K);
#pragma unroll
        for (int i = 0; i < Q_EACH; ++i) qo[i] = source<Q_OUTER, BN, false>((wave + i * WAVES) % Q_LOADS, lane, Q.ld, Q.extent - q0, IVFR_PRODUCT_K);
        const int total = planes.n * count;
        int pair = 0, at = 0;   // of the next stage to load
        const uint16_t *pn = pb + (planes.p & 15) * P.plane, *qn = qb + (planes.q & 15) * Q.plane;
        auto load = [&](int buf) {
            const uint32_t lp = lds0 + buf * STAGE, lq = lp + BM * KB;
            const int pl = P_OUTER ? P.rows - (first + at) * IVFR_PRODUCT_K : IVFR_PRODUCT_K, ql = Q_OUTER ? Q.rows - (first + at) * IVFR_PRODUCT_K : IVFR_PRODUCT_K;
#pragma unroll
            for (int i = 0; i < P_EACH; ++i) {
                const int f = (wave + i * WAVES) % P_LOADS;
                load16(lp + 1024 * f, P_OUTER && pl < IVFR_PRODUCT_K ? source<P_OUTER, BM, true>(f, lane, P.ld, P.extent - p0, pl) : po[i], pn);
            }
#pragma unroll
            for (int i = 0; i < Q_EACH; ++i) {
                const int f = (wave + i * WAVES) % Q_LOADS;
                load16(lq + 1024 * f, Q_OUTER && ql < IVFR_PRODUCT_K ? source<Q_OUTER, BN, false>(f, lane, Q.ld, Q.extent - q0, ql) : qo[i], qn);
            }
            if (++at < count) {
                pn += pstep;
                qn += qstep;
            } else {
                at = 0;
                ++pair;
                pn = pb + ((planes.p >> (4 * pair)) & 15) * P.plane;
                qn = qb + ((planes.q >> (4 * pair)) & 15) * Q.plane;
            }
        };
        const int wm = wave / WAVES_N * (BM / WAVES_M), wn = wave % WAVES_N * (BN / WAVES_N);
        const int r = lane & 15, g = lane >> 4;
        // where this lane's fragments of the first tile lie; the others at constant distances (the permutations repeat every 16 or 32 rows)
        uint32_t pf[P_OUTER ? 2 : 2], qf[2];
        if constexpr (P_OUTER) {
#pragma unroll
            for (int j = 0; j < 2; ++j) pf[j] = (8 * g + 4 * j + (r >> 2)) * (2 * BM);   // the row of k; the column's chunk comes with the tile
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = wm + 8 * (r >> 2) + 4 * j + (r & 3);
                pf[j] = row * KB + 16 * (g ^ swz_p(row));
            }
        }
        if constexpr (Q_OUTER) {
#pragma unroll
            for (int j = 0; j < 2; ++j) qf[j] = (8 * g + 4 * j + (r >> 2)) * (2 * BN);
        } else {
            const int row = wn + r;
            qf[0] = qf[1] = row * KB + 16 * (g ^ swz_q(row));
        }
        auto outer_read = [&](const char* b, const uint32_t (&rows)[2], int column) {   // eight k of column + (l & 15)
            short8v v;
            const int chunk = ((column >> 3) + ((r & 3) >> 1)) ^ swz_k(r >> 2);   // (8 g + 4 j is a multiple of four)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const short4v h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(b + rows[j] + 16 * chunk + 8 * (r & 1)));
                v[4 * j] = h[0]; v[4 * j + 1] = h[1]; v[4 * j + 2] = h[2]; v[4 * j + 3] = h[3];
            }
            return v;
        };
        auto read = [&](int buf, short8v (&fp)[TM], short8v (&fq)[TN]) {
            const char* bp = smem + buf * STAGE;
            const char* bq = bp + BM * KB;
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                if constexpr (Q_OUTER) fq[t] = outer_read(bq, qf, wn + 16 * t);
                else fq[t] = *reinterpret_cast<const short8v*>(bq + qf[0] + t * 16 * KB);
            }
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                if constexpr (P_OUTER) fp[t] = outer_read(bp, pf, wm + 16 * t);
                else fp[t] = *reinterpret_cast<const short8v*>(bp + pf[t & 1] + (t >> 1) * 32 * KB);
            }
        };
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
        short8v fp[2][TM], fq[2][TN];
#pragma unroll
        for (int s = 0; s < IVFR_PRODUCT_STAGES; ++s)
            if (s < total) load(s);
        if (total >= IVFR_PRODUCT_STAGES) wait_and_meet<3 * EACH>();
        else wait_and_meet<0>();
        if (total > 0) read(0, fp[0], fq[0]);
        auto step = [&](int s, short8v (&cp)[TM], short8v (&cq)[TN], short8v (&np)[TM], short8v (&nq)[TN]) {
            if (s + 1 < total) {
                // in flight: stages up to s + 3; s + 1 is needed, and buffer s & 3 is free once all have read stage s
                if (s + 3 < total) wait_and_meet<2 * EACH>();
                else wait_and_meet<0>();
                if (s + 4 < total) load(s & 3);
                read((s + 1) & 3, np, nq);
            }
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b) acc[a][b] = mfma(cp[a], cq[b], acc[a][b]);
        };
        for (int s = 0; s < total; s += 2) {
            step(s, fp[0], fq[0], fp[1], fq[1]);
            if (s + 1 < total) step(s + 1, fp[1], fq[1], fp[0], fq[0]);
        }
    }

    // first p (of four, or with P inner of eight in the tiles t, t + 1) and q of this lane's outputs in tile (t, u)
    static __device__ __forceinline__ int p_of(int t) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WAVES_N * (BM / WAVES_M);
        return P_OUTER ? wm + 16 * t + 4 * (lane >> 4) : wm + 16 * (t & ~1) + 8 * (lane >> 4) + 4 * (t & 1);
    }
    static __device__ __forceinline__ int q_of(int u) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return wave % WAVES_N * (BN / WAVES_N) + 16 * u + (lane & 15);
    }
};

// rounding to nearest, ties to even
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float from_bf16(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_half(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float from_half(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }

// ---- products that are stored, in fp32 sums over parts of k where there are few tiles (product.hip)

#define IVFR_OUT_F32 0
#define IVFR_OUT_F16 1
#define IVFR_OUT_BF16 2

// out[q][p] = alpha * unit * sum_k P(p, k) Q(q, k) for p < np, q < nq
struct ProductOut {
    ProductOperand P, Q;       // P outer
    bool q_outer, half;
    ProductPlanes planes;
    int stages;                // of 32 k
    int np, nq;
    int type;                  // IVFR_OUT_*
    float alpha;
    const float* unit;         // device factor, or null
    void* out;
    int64_t ld;
    // sums over parts of k: slots slot0 .. slot0 + splits - 1 of partial [slot][nq][np_pad] are written instead of out
    float* partial;
    int slot0;
};
// how such a product is cut
struct ProductPlan {
    int kind, splits;          // tile, parts of k
};
ProductPlan product_plan(int64_t np, int64_t nq, int64_t stages, int pairs, bool q_outer, int n_cu);
inline int64_t product_pad(int64_t np) { return (np + 3) / 4 * 4; }
// partial == null: plan.splits must be 1
int product_launch(const ProductOut& a, const ProductPlan& plan, hipStream_t st);
// out[q][p] = alpha * unit * sum over the slots, in their order
int product_join(const float* partial, int slots, int64_t nq, int np, int type, float alpha, const float* unit, void* out, int64_t ld, hipStream_t st);
