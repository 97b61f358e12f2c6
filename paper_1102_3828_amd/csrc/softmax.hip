// Softmax cross entropy of rows x [n, d] against a set of vectors w [v, d], and its gradient, without keeping the scores.
//
//   z_ij = scale x_i . w_j + offset_j,   L_i = log sum_j exp z_ij,   loss_i = L_i - z_it           (t = target of row i)
//   e_ij = weight_i (exp(z_ij - L_i) - [j = t]),   dx = scale e w,   dw = scale e^T x
//
// Loss: one product w x^T; a workgroup reduces its tile of scores to one (maximum, sum of exponentials) per row, which loss_kernel
// joins over the tiles: 8 bytes per row and tile instead of the scores.
// Gradient: the scores are formed again in pieces of the vectors, e of a piece is written in 16 bits (fp32 calls: three planes of
// 16 bits) and multiplied with w and x.  Statistics and sums are fp32; e is rounded once, to the type of the inputs, in which the matrix cores read it.
#include "product.h"

#include <algorithm>
#include <cmath>

#define GRAD_PIECE_BYTES ((int64_t)1 << 30)   // of e at a time

// ---------------------------------------------------------------- operands

// rows of src in 16-bit planes, padded with zeros to rows_out x ld_out; rows that take no part are zero, whatever they hold:
// left out by an infinite negative offset, or without a target
struct PackArgs {
    const void* src;
    int64_t ld, rows, rows_out, ld_out;
    int d, planes, vec;        // vec: rows start at 16-byte boundaries
    uint16_t* dst;
    const float* offset;       // [rows] or null
    const int64_t* targets;    // [rows] or null
};

template <bool F32>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a) {
    const int64_t chunks = a.ld_out / 8, total = a.rows_out * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int k0 = (int)(i - row * chunks) * 8;
        bool in = row < a.rows;
        if (in && a.offset) in = a.offset[row] != -INFINITY;
        if (in && a.targets) in = a.targets[row] >= 0;
        if constexpr (F32) {
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (in) {
                const float* s = (const float*)a.src + row * a.ld + k0;
                if (a.vec && k0 + 8 <= a.d) {
                    const float4 u = *reinterpret_cast<const float4*>(s), v = *reinterpret_cast<const float4*>(s + 4);
                    f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (k0 + e < a.d) f[e] = s[e];
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                short8v o;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint16_t b = to_bf16(f[e]);
                    o[e] = (short)b;
                    f[e] = f[e] - from_bf16(b);
                    // (an infinity or NaN is whole in the first plane: inf - inf would make the product of an infinite value NaN)
                    if ((b & 0x7f80) == 0x7f80) f[e] = 0.f;
                }
                *reinterpret_cast<short8v*>(a.dst + p * a.rows_out * a.ld_out + row * a.ld_out + k0) = o;
            }
        } else {
            short8v o = {0, 0, 0, 0, 0, 0, 0, 0};
            if (in) {
                const uint16_t* s = (const uint16_t*)a.src + row * a.ld + k0;
                if (a.vec && k0 + 8 <= a.d) o = *reinterpret_cast<const short8v*>(s);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (k0 + e < a.d) o[e] = (short)s[e];
                }
            }
            *reinterpret_cast<short8v*>(a.dst + row * a.ld_out + k0) = o;
        }
    }
}

static int launch_pack(const PackArgs& a, bool f32, hipStream_t st) {
    const int64_t total = a.rows_out * (a.ld_out / 8);
    const unsigned grid = (unsigned)std::min<int64_t>((total + 255) / 256, 8192);
    if (f32) hipLaunchKernelGGL(pack_kernel<true>, dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(pack_kernel<false>, dim3(grid), dim3(256), 0, st, a);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}

// ---------------------------------------------------------------- loss

struct ScoreArgs {
    ProductOperand w, x;       // P, Q
    ProductPlanes planes;
    int stages, tiles_p, tiles_q;
    int v, n;                  // vectors of this piece, rows
    int v0, v_all;             // first vector of this piece; all vectors
    float scale;
    const float* offset;       // of this piece, or null
    const int64_t* targets;
    // loss
    float2* part;              // [n][tiles_p] (maximum, sum of exponentials relative to it)
    float* target_score;       // [n]
    // gradient
    const float* lse;          // [n]
    const float* weight;       // [n]
    const float* unit;         // factor of e, or null
    uint16_t* e;               // [planes][n_pad][e_ld]
    int64_t e_ld;
    int n_pad, v_pad;          // rows and columns of e that are written (zeros beyond n and v)
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// scores of this lane's outputs, in place; vectors that take no part, or do not exist: -inf
template <class C>
__device__ __forceinline__ void scores(const ScoreArgs& a, int p0, floatx4 (&acc)[C::TM][C::TN]) {
    const bool whole = p0 + C::BM <= a.v;
#pragma unroll
    for (int t = 0; t < C::TM; ++t) {
        const int j = p0 + C::p_of(t);
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.offset || !whole) {
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = j + r < a.v ? (a.offset ? a.offset[j + r] : 0.f) : -INFINITY;
        }
#pragma unroll
        for (int u = 0; u < C::TN; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[t][u][r] = o[r] == -INFINITY ? -INFINITY : fmaf(acc[t][u][r], a.scale, o[r]);
    }
}

template <class C>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void score_kernel(ScoreArgs a) {
    __shared__ __align__(1024) char smem[C::LDS];
    const ProductTile tile = product_tile(a.tiles_p, a.tiles_q, 1);
    if (!tile.any) return;   // uniform
    const int p0 = tile.p * C::BM, q0 = tile.q * C::BN;
    floatx4 acc[C::TM][C::TN];
    C::run(a.w, a.x, a.planes, p0, q0, 0, a.stages, smem, acc);
    scores<C>(a, p0, acc);
    __syncthreads();   // the stages are no longer read
    float2* const red = reinterpret_cast<float2*>(smem);   // [WAVES_M][BN]
    const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / C::WAVES_N;
#pragma unroll
    for (int u = 0; u < C::TN; ++u) {
        const int i = q0 + C::q_of(u);
        const int64_t target = i < a.n ? a.targets[i] : -1;
        float m = -INFINITY;
#pragma unroll
        for (int t = 0; t < C::TM; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                m = fmaxf(m, acc[t][u][r]);
                if (target == (int64_t)p0 + C::p_of(t) + r) a.target_score[i] = acc[t][u][r];   // (one lane of the launch; it has i < n)
            }
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float base = m == -INFINITY ? 0.f : m;   // nothing takes part: a sum of zeros, not of NaN
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < C::TM; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) s += exp_of(acc[t][u][r] - base);
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        if (lane < 16) red[wm * C::BN + C::q_of(u)] = make_float2(m, s);
    }
    __syncthreads();
    for (int q = threadIdx.x; q < C::BN; q += C::THREADS) {
        const int i = q0 + q;
        if (i >= a.n) continue;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < C::WAVES_M; ++w) m = fmaxf(m, red[w * C::BN + q].x);
        const float base = m == -INFINITY ? 0.f : m;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < C::WAVES_M; ++w) s += red[w * C::BN + q].y * exp_of(red[w * C::BN + q].x - base);
        a.part[(int64_t)i * a.tiles_p + tile.p] = make_float2(m, s);
    }
}

// A wavefront per row joins its tiles' statistics (in a fixed order).
__global__ __launch_bounds__(256) void loss_kernel(const float2* __restrict__ part, int tiles, const float* __restrict__ target_score,
                                                   const int64_t* __restrict__ targets, int n, int64_t v, float* __restrict__ loss, float* __restrict__ lse) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= n) return;   // uniform over a wavefront
    const float2* p = part + (int64_t)i * tiles;
    float m = -INFINITY, s = 0.f;
    for (int t = lane; t < tiles; t += 64) {
        const float2 x = p[t];
        const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.f : top;
        s = s * exp_of(m - base) + x.y * exp_of(x.x - base);
        m = top;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const float om = __shfl_xor(m, off, 64), os = __shfl_xor(s, off, 64);
        const float top = fmaxf(m, om), base = top == -INFINITY ? 0.f : top;
        s = s * exp_of(m - base) + os * exp_of(om - base);
        m = top;
    }
    if (lane == 0) {
        const float ls = logf(s), L = m == -INFINITY && s == 0.f ? -INFINITY : m + ls;
        if (lse) lse[i] = L;
        if (loss) {
            const int64_t t = targets[i];
            float x;
            if (t < 0) x = 0.f;
            else if (t >= v) x = NAN;
            else {
                const float z = target_score[i];
                x = z == -INFINITY ? INFINITY : (m - z) + ls;
            }
            loss[i] = x;
        }
    }
}

// ---------------------------------------------------------------- gradient

// fp16 calls: e is written in a unit that brings the largest weight to 2^15 (|exp(z - L) - [j = t]| <= 1), so that probabilities down
// to 2^-29 keep all their bits; unit[0] multiplies, unit[1] takes it back.  bf16 has the range of fp32.
__global__ __launch_bounds__(256) void weight_unit_kernel(const float* __restrict__ weight, const int64_t* __restrict__ targets, int n, float* __restrict__ unit) {
    __shared__ float red[4];
    float m = 0.f;
    for (int i = threadIdx.x; i < n; i += 256)
        if (targets[i] >= 0) m = fmaxf(m, fabsf(weight[i]));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        int ex = 0;
        if (m > 0.f && m < INFINITY) (void)frexpf(m, &ex);   // m < 2^ex
        ex = min(max(15 - ex, -110), 110);
        unit[0] = ldexpf(1.f, ex);
        unit[1] = ldexpf(1.f, -ex);
    }
}

template <class C, int PLANES>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void grad_score_kernel(ScoreArgs a) {
    __shared__ __align__(1024) char smem[C::LDS];
    const ProductTile tile = product_tile(a.tiles_p, a.tiles_q, 1);
    if (!tile.any) return;   // uniform
    const int p0 = tile.p * C::BM, q0 = tile.q * C::BN;
    floatx4 acc[C::TM][C::TN];
    C::run(a.w, a.x, a.planes, p0, q0, 0, a.stages, smem, acc);
    scores<C>(a, p0, acc);
    const float unit = a.unit ? a.unit[0] : 1.f;
#pragma unroll
    for (int u = 0; u < C::TN; ++u) {
        const int i = q0 + C::q_of(u);
        if (i >= a.n_pad) continue;
        int64_t target = -1;
        float L = 0.f, g = 0.f;
        if (i < a.n) {
            target = a.targets[i];
            L = a.lse[i];
            g = target < 0 ? 0.f : (a.weight[i] != 0.f && target >= a.v_all ? NAN : a.weight[i] * unit);
        }
        const int at = target >= a.v0 && target - a.v0 < a.v ? (int)(target - a.v0) : -1;
#pragma unroll
        for (int t = 0; t < C::TM; t += 2) {
            const int j = p0 + C::p_of(t);
            if (j >= a.v_pad) continue;   // (a multiple of 8, as j)
            float f[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float z = acc[t + (r >> 2)][u][r & 3];
                const float x = g * (exp_of(z - L) - (j + r == at ? 1.f : 0.f));
                f[r] = z == -INFINITY || g == 0.f ? 0.f : x;
            }
            uint16_t* const o = a.e + (int64_t)i * a.e_ld + j;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                short8v h;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    if constexpr (C::HALF) h[r] = (short)to_half(f[r]);
                    else {
                        const uint16_t b = to_bf16(f[r]);
                        h[r] = (short)b;
                        f[r] -= from_bf16(b);
                    }
                }
                *reinterpret_cast<short8v*>(o + (int64_t)p * a.n_pad * a.e_ld) = h;
            }
        }
    }
}

// ---------------------------------------------------------------- host

// The tile by the sizes: few rows read the vectors once and are bound by that; else 256 x 256 where these give every compute unit a tile.
struct ScoreKind {
    int bm, bn;
};
static const ScoreKind SCORE_KINDS[] = {{256, 256}, {128, 128}, {256, 64}, {256, 16}};

static int score_kind(int64_t n, int64_t v, int n_cu) {
    if (n <= 16) return 3;
    if (n <= 64) return 2;
    return ((n + 255) / 256) * ((v + 255) / 256) >= n_cu ? 0 : 1;
}

template <class C>
static int launch_score(const ScoreArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((score_kernel<C>), dim3(product_grid((int64_t)a.tiles_p * a.tiles_q)), dim3(C::THREADS), 0, st, a);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}
template <class C>
static int launch_grad_score(const ScoreArgs& a, hipStream_t st) {
    if constexpr (!C::HALF)
        if (a.planes.n > 1) {
            hipLaunchKernelGGL((grad_score_kernel<C, 3>), dim3(product_grid((int64_t)a.tiles_p * a.tiles_q)), dim3(C::THREADS), 0, st, a);
            IVFR_HIP(hipGetLastError());
            return IVFR_OK;
        }
    hipLaunchKernelGGL((grad_score_kernel<C, 1>), dim3(product_grid((int64_t)a.tiles_p * a.tiles_q)), dim3(C::THREADS), 0, st, a);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}
template <bool HALF, bool GRAD>
static int launch_scores_of(ScoreArgs& a, int kind, hipStream_t st) {
    a.tiles_p = (int)(((GRAD ? a.v_pad : a.v) + SCORE_KINDS[kind].bm - 1) / SCORE_KINDS[kind].bm);
    a.tiles_q = (int)(((GRAD ? a.n_pad : a.n) + SCORE_KINDS[kind].bn - 1) / SCORE_KINDS[kind].bn);
    typedef Product<256, 256, 2, 4, false, false, HALF> K0;
    typedef Product<128, 128, 2, 2, false, false, HALF> K1;
    typedef Product<256, 64, 8, 1, false, false, HALF> K2;
    typedef Product<256, 16, 8, 1, false, false, HALF> K3;
    if constexpr (GRAD) {
        switch (kind) {
            case 0: return launch_grad_score<K0>(a, st);
            case 1: return launch_grad_score<K1>(a, st);
            case 2: return launch_grad_score<K2>(a, st);
            default: return launch_grad_score<K3>(a, st);
        }
    } else {
        switch (kind) {
            case 0: return launch_score<K0>(a, st);
            case 1: return launch_score<K1>(a, st);
            case 2: return launch_score<K2>(a, st);
            default: return launch_score<K3>(a, st);
        }
    }
}
static int launch_scores(ScoreArgs& a, int kind, bool half, bool grad, hipStream_t st) {
    if (half) return grad ? launch_scores_of<true, true>(a, kind, st) : launch_scores_of<true, false>(a, kind, st);
    return grad ? launch_scores_of<false, true>(a, kind, st) : launch_scores_of<false, false>(a, kind, st);
}

static inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// What a call keeps in its workspace, and where.
struct SoftmaxPlan {
    int planes, stages, kind, n_cu;
    bool half, pack_x, pack_w;
    int64_t kd, n_pad, e_ld, piece;   // columns of packed operands; rows and columns of e, vectors a piece
    int pieces;
    int64_t tiles_p;                  // of the loss
    ProductPlan dx, dw;               // of a whole piece
    int64_t at_x, at_w, at_part, at_target, at_lse, at_unit, at_e, at_dx, at_dw, bytes;
};

static bool rows_aligned(const void* p, int64_t ld, int size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0; }

static int softmax_check(const ivfr_softmax_args* a) {
    IVFR_REQUIRE(a, "softmax: null arguments");
    IVFR_REQUIRE(a->type == IVFR_TYPE_F32 || a->type == IVFR_TYPE_F16 || a->type == IVFR_TYPE_BF16, "softmax: type must be IVFR_TYPE_F32, _F16 or _BF16, got %d", a->type);
    IVFR_REQUIRE(a->n >= 0 && a->n < (1ll << 31) - 256 && a->v >= 1 && a->v < (1ll << 31) - 256, "softmax: n must be in [0, 2^31 - 256) and v in [1, 2^31 - 256), got %lld and %lld",
                 (long long)a->n, (long long)a->v);
    IVFR_REQUIRE(a->d >= 1 && a->d <= 65536, "softmax: d must be in [1, 65536], got %d", a->d);
    IVFR_REQUIRE(a->ldx >= a->d && a->ldw >= a->d && a->ldx < (1 << 22) && a->ldw < (1 << 22), "softmax: ldx and ldw must be in [d, 2^22)");
    IVFR_REQUIRE(((a->n + 127) / 128) * ((a->v + 127) / 128) < (1ll << 30), "softmax: n times v must be below 2^44");
    IVFR_REQUIRE(std::isfinite(a->scale), "softmax: scale must be finite");
    return IVFR_OK;
}

static SoftmaxPlan softmax_plan(const ivfr_softmax_args& a, bool grad) {
    SoftmaxPlan p = {};
    p.n_cu = IVFR_PRODUCT_CU;
    const bool f32 = a.type == IVFR_TYPE_F32;
    p.half = a.type == IVFR_TYPE_F16;
    p.planes = f32 ? 3 : 1;
    p.kd = round_up(a.d, 32);
    p.stages = (int)(p.kd / 32);
    p.n_pad = round_up(a.n, 32);
    const int pairs = product_planes(p.planes).n;
    // gradients read x by rows of k: padded to whole stages; rows that take no part are zeroed in the copy
    p.pack_x = f32 || grad || a.d % 32 || !rows_aligned(a.x, a.ldx, 2);
    p.pack_w = f32 || (grad && a.offset) || a.d % 32 || !rows_aligned(a.w, a.ldw, 2);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    if (p.pack_x) p.at_x = take(p.planes * (grad ? p.n_pad : a.n) * p.kd * 2);
    if (p.pack_w) p.at_w = take(p.planes * a.v * p.kd * 2);
    p.kind = score_kind(a.n, a.v, p.n_cu);
    p.tiles_p = (a.v + SCORE_KINDS[p.kind].bm - 1) / SCORE_KINDS[p.kind].bm;
    p.at_part = take(a.n * p.tiles_p * 8);
    p.at_target = take(a.n * 4);
    if (grad) {
        p.at_lse = take(a.n * 4);
        p.at_unit = take(8);
        // pieces of equal width, a multiple of 256
        const int64_t fit = std::max<int64_t>(256, GRAD_PIECE_BYTES / (2 * p.planes * p.n_pad) / 256 * 256);
        p.pieces = (int)((a.v + fit - 1) / fit);
        p.piece = std::min(round_up((a.v + p.pieces - 1) / p.pieces, 256), round_up(a.v, 32));
        p.pieces = (int)((a.v + p.piece - 1) / p.piece);
        p.e_ld = round_up(p.piece, 64);
        p.at_e = take(p.planes * p.n_pad * p.e_ld * 2);
        p.dx = product_plan(a.d, a.n, (p.piece + 31) / 32, pairs, false, p.n_cu);
        p.dw = product_plan(a.d, p.piece, p.n_pad / 32, pairs, true, p.n_cu);
        if (p.pieces > 1 || p.dx.splits > 1) p.at_dx = take((int64_t)p.pieces * p.dx.splits * a.n * product_pad(a.d) * 4);
        if (p.dw.splits > 1) p.at_dw = take(p.dw.splits * p.piece * product_pad(a.d) * 4);
    }
    p.bytes = at;
    return p;
}

int ivfr_softmax_workspace(const ivfr_softmax_args* args, int32_t grad, int64_t* bytes) {
    IVFR_TRY(softmax_check(args));
    IVFR_REQUIRE(bytes, "softmax: null output");
    *bytes = args->n ? softmax_plan(*args, grad != 0).bytes : 0;
    return IVFR_OK;
}

// The arguments' pointers, for calls with rows.
static int softmax_pointers(const ivfr_softmax_args& a, const SoftmaxPlan& p, const void* workspace, int64_t workspace_bytes) {
    const int size = a.type == IVFR_TYPE_F32 ? 4 : 2;
    IVFR_REQUIRE(a.x && a.w && a.targets, "softmax: null pointer");
    IVFR_REQUIRE(((uintptr_t)a.x % size) == 0 && ((uintptr_t)a.w % size) == 0 && ((uintptr_t)a.targets & 7) == 0 && ((uintptr_t)a.offset & 3) == 0, "softmax: pointers must be aligned to their type");
    IVFR_REQUIRE(workspace || p.bytes == 0, "softmax: null workspace");
    IVFR_REQUIRE(((uintptr_t)workspace & 255) == 0, "softmax: the workspace must be aligned to 256 bytes");
    IVFR_REQUIRE(workspace_bytes >= p.bytes, "softmax: the workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)p.bytes);
    return IVFR_OK;
}

static int pack_operands(const ivfr_softmax_args& a, const SoftmaxPlan& p, bool grad, char* ws, ScoreArgs& s, hipStream_t st) {
    const bool f32 = a.type == IVFR_TYPE_F32;
    s.x = {(const uint16_t*)a.x, 0, a.ldx, (int)a.n, 0};
    s.w = {(const uint16_t*)a.w, 0, a.ldw, (int)a.v, 0};
    if (p.pack_x) {
        PackArgs k = {a.x, a.ldx, a.n, grad ? p.n_pad : a.n, p.kd, a.d, p.planes, rows_aligned(a.x, a.ldx, f32 ? 4 : 2), (uint16_t*)(ws + p.at_x),
                      nullptr, grad ? a.targets : nullptr};
        IVFR_TRY(launch_pack(k, f32, st));
        s.x.base = k.dst;
        s.x.ld = p.kd;
        s.x.plane = k.rows_out * p.kd;
        s.x.extent = (int)k.rows_out;   // (the rows of e reach up to the padding)
    }
    if (p.pack_w) {
        PackArgs k = {a.w, a.ldw, a.v, a.v, p.kd, a.d, p.planes, rows_aligned(a.w, a.ldw, f32 ? 4 : 2), (uint16_t*)(ws + p.at_w), a.offset, nullptr};
        IVFR_TRY(launch_pack(k, f32, st));
        s.w.base = k.dst;
        s.w.ld = p.kd;
        s.w.plane = a.v * p.kd;
    }
    s.planes = product_planes(p.planes);
    s.stages = p.stages;
    s.n = (int)a.n;
    s.v = s.v_all = (int)a.v;
    s.scale = a.scale;
    s.offset = a.offset;
    s.targets = a.targets;
    s.part = (float2*)(ws + p.at_part);
    s.target_score = (float*)(ws + p.at_target);
    return IVFR_OK;
}

static int statistics(const ivfr_softmax_args& a, const SoftmaxPlan& p, ScoreArgs s, float* loss, float* lse, hipStream_t st) {
    IVFR_TRY(launch_scores(s, p.kind, p.half, false, st));
    hipLaunchKernelGGL(loss_kernel, dim3((unsigned)((a.n + 3) / 4)), dim3(256), 0, st, s.part, (int)p.tiles_p, s.target_score, a.targets, (int)a.n, a.v, loss, lse);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}

int ivfr_softmax_loss(const ivfr_softmax_args* args, float* loss, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    IVFR_TRY(softmax_check(args));
    if (args->n == 0) return IVFR_OK;
    const SoftmaxPlan p = softmax_plan(*args, false);
    IVFR_TRY(softmax_pointers(*args, p, workspace, workspace_bytes));
    IVFR_REQUIRE(loss && lse, "softmax: null output");
    IVFR_HIP(hipSetDevice(args->device));
    hipStream_t st = (hipStream_t)stream;
    ScoreArgs s = {};
    IVFR_TRY(pack_operands(*args, p, false, (char*)workspace, s, st));
    return statistics(*args, p, s, loss, lse, st);
}

__global__ __launch_bounds__(256) void zero_kernel(uint4* p, int64_t chunks, uint8_t* tail, int rest) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) p[i] = make_uint4(0, 0, 0, 0);
    if (blockIdx.x == 0 && (int)threadIdx.x < rest) tail[threadIdx.x] = 0;
}

int ivfr_softmax_loss_grad(const ivfr_softmax_args* args, const float* weight, const float* lse, float* loss, void* dx, void* dw,
                           void* workspace, int64_t workspace_bytes, void* stream) {
    IVFR_TRY(softmax_check(args));
    const ivfr_softmax_args& a = *args;
    const int size = a.type == IVFR_TYPE_F32 ? 4 : 2, out_type = a.type;
    hipStream_t st = (hipStream_t)stream;
    IVFR_REQUIRE(dw && ((uintptr_t)dw & 15) == 0, "softmax: dw must be aligned to 16 bytes");
    if (a.n == 0) {   // no rows: no gradient
        IVFR_HIP(hipSetDevice(a.device));
        const int64_t bytes = a.v * a.d * size;
        hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::min<int64_t>(bytes / 4096 + 1, 4096)), dim3(256), 0, st, (uint4*)dw, bytes / 16, (uint8_t*)dw + bytes / 16 * 16, (int)(bytes % 16));
        IVFR_HIP(hipGetLastError());
        return IVFR_OK;
    }
    const SoftmaxPlan p = softmax_plan(a, true);
    IVFR_TRY(softmax_pointers(a, p, workspace, workspace_bytes));
    IVFR_REQUIRE(weight && dx, "softmax: null pointer");
    IVFR_REQUIRE(((uintptr_t)dx & 15) == 0, "softmax: dx must be aligned to 16 bytes");
    IVFR_HIP(hipSetDevice(a.device));
    char* const ws = (char*)workspace;
    ScoreArgs s = {};
    IVFR_TRY(pack_operands(a, p, true, ws, s, st));
    float* const unit = p.half ? (float*)(ws + p.at_unit) : nullptr;
    if (unit) {
        hipLaunchKernelGGL(weight_unit_kernel, dim3(1), dim3(256), 0, st, weight, a.targets, (int)a.n, unit);
        IVFR_HIP(hipGetLastError());
    }
    if (!lse || loss) {
        float* const own_lse = (float*)(ws + p.at_lse);
        IVFR_TRY(statistics(a, p, s, loss, own_lse, st));
        if (!lse) lse = own_lse;
    }
    s.lse = lse;
    s.weight = weight;
    s.unit = unit;
    s.e = (uint16_t*)(ws + p.at_e);
    s.e_ld = p.e_ld;
    s.n_pad = (int)p.n_pad;
    const bool parts = p.pieces > 1 || p.dx.splits > 1;
    const ProductOperand x = s.x, w = s.w;
    for (int i = 0; i < p.pieces; ++i) {
        const int64_t v0 = (int64_t)i * p.piece, here = std::min(p.piece, a.v - v0);
        s.v0 = (int)v0;
        s.v = (int)here;
        s.v_pad = (int)round_up(here, 32);
        s.w = w;
        s.w.base = w.base + v0 * w.ld;
        s.w.extent = (int)here;
        s.offset = a.offset ? a.offset + v0 : nullptr;
        IVFR_TRY(launch_scores(s, score_kind(a.n, here, p.n_cu), p.half, true, st));
        ProductOut o = {};
        o.half = p.half;
        o.planes = s.planes;
        o.type = out_type;
        o.alpha = a.scale;
        o.unit = unit;
        o.np = a.d;
        o.ld = a.d;
        // dx [n, d]: over the vectors of the piece
        o.P = s.w;
        o.P.extent = a.d;
        o.P.rows = (int)here;
        o.Q = {s.e, p.n_pad * p.e_ld, p.e_ld, (int)a.n, 0};
        o.q_outer = false;
        o.stages = s.v_pad / 32;
        o.nq = (int)a.n;
        o.out = dx;
        o.partial = parts ? (float*)(ws + p.at_dx) : nullptr;
        o.slot0 = i * p.dx.splits;
        IVFR_TRY(product_launch(o, p.dx, st));
        // dw [here, d]: over the rows
        o.P = x;
        o.P.extent = a.d;
        o.P.rows = (int)p.n_pad;
        o.Q = {s.e, p.n_pad * p.e_ld, p.e_ld, (int)here, (int)p.n_pad};
        o.q_outer = true;
        o.stages = (int)(p.n_pad / 32);
        o.nq = (int)here;
        o.out = (char*)dw + v0 * a.d * size;
        o.partial = p.dw.splits > 1 ? (float*)(ws + p.at_dw) : nullptr;
        o.slot0 = 0;
        IVFR_TRY(product_launch(o, p.dw, st));
        if (p.dw.splits > 1) IVFR_TRY(product_join(o.partial, p.dw.splits, here, a.d, out_type, a.scale, unit, o.out, a.d, st));
    }
    if (parts) IVFR_TRY(product_join((float*)(ws + p.at_dx), p.pieces * p.dx.splits, a.n, a.d, out_type, a.scale, unit, dx, a.d, st));
    return IVFR_OK;
}
