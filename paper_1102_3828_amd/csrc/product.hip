// Products that are stored (product.h): gradients of softmax.hip.
#include "product.h"

#include <algorithm>

struct OutArgs {
    ProductOut o;
    int tiles_p, tiles_q, splits, per;   // stages of a part
};

__device__ __forceinline__ void store_value(void* out, int64_t at, int type, float x) {
    if (type == IVFR_OUT_F32) ((float*)out)[at] = x;
    else ((uint16_t*)out)[at] = type == IVFR_OUT_F16 ? to_half(x) : to_bf16(x);
}

// four consecutive values, the first `some` of them in range
__device__ __forceinline__ void store_four(void* out, int64_t at, int type, const floatx4 x, int some, bool whole) {
    if (whole && some >= 4) {
        if (type == IVFR_OUT_F32) *reinterpret_cast<floatx4*>((float*)out + at) = x;
        else {
            short4v h;
#pragma unroll
            for (int r = 0; r < 4; ++r) h[r] = (short)(type == IVFR_OUT_F16 ? to_half(x[r]) : to_bf16(x[r]));
            *reinterpret_cast<short4v*>((uint16_t*)out + at) = h;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < some) store_value(out, at + r, type, x[r]);
    }
}

template <class C>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void out_kernel(OutArgs a) {
    __shared__ __align__(1024) char smem[C::LDS];
    const ProductTile tile = product_tile(a.tiles_p, a.tiles_q, a.splits);
    if (!tile.any) return;   // uniform
    const ProductOut& o = a.o;
    const int p0 = tile.p * C::BM, q0 = tile.q * C::BN, first = tile.split * a.per;
    const int count = o.stages - first < a.per ? o.stages - first : a.per;
    floatx4 acc[C::TM][C::TN];
    C::run(o.P, o.Q, o.planes, p0, q0, first, count, smem, acc);
    const float alpha = o.partial ? 1.f : o.alpha * (o.unit ? o.unit[1] : 1.f);
    const int64_t ld = o.partial ? (o.np + 3) / 4 * 4 : o.ld;
    const int type = o.partial ? IVFR_OUT_F32 : o.type, limit = o.partial ? (int)ld : o.np;
    void* const out = o.partial ? (void*)(o.partial + (int64_t)(o.slot0 + tile.split) * o.nq * ld) : o.out;
    const bool whole = ld % 4 == 0 && ((uintptr_t)out & 15) == 0;   // uniform
#pragma unroll
    for (int u = 0; u < C::TN; ++u) {
        const int q = q0 + C::q_of(u);
        if (q >= o.nq) continue;
#pragma unroll
        for (int t = 0; t < C::TM; ++t) {
            const int p = p0 + C::p_of(t);
            if (p < limit) store_four(out, q * ld + p, type, acc[t][u] * alpha, limit - p, whole);
        }
    }
}

// A thread takes four neighbouring values through all slots.
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ partial, int slots, int64_t nq, int np, int type, float alpha,
                                                   const float* __restrict__ unit, void* __restrict__ out, int64_t ld) {
    const int pad = (np + 3) / 4 * 4, quads = pad / 4;
    const int64_t total = nq * quads, slot = nq * pad;
    const float f = alpha * (unit ? unit[1] : 1.f);
    const bool whole = ld % 4 == 0 && ((uintptr_t)out & 15) == 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / quads;
        const int p = (int)(i - q * quads) * 4;
        const float* s = partial + 4 * i;
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = 0; k < slots; ++k) sum += *reinterpret_cast<const floatx4*>(s + k * slot);
        store_four(out, q * ld + p, type, sum * f, np - p, whole);
    }
}

int product_join(const float* partial, int slots, int64_t nq, int np, int type, float alpha, const float* unit, void* out, int64_t ld, hipStream_t st) {
    const int64_t total = nq * (product_pad(np) / 4);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)std::min<int64_t>((total + 255) / 256, 8192)), dim3(256), 0, st, partial, slots, nq, np, type, alpha, unit, out, ld);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}

// Tiles of p x q; workgroups that a compute unit holds (by LDS); cycles of a stage on a compute unit that holds that many, by what was measured
struct Kind {
    int bm, bn, resident;
    double stage;
};
static const Kind KINDS[] = {{256, 256, 1, 1300}, {128, 128, 2, 900}, {64, 64, 5, 900}, {256, 16, 2, 420}};

ProductPlan product_plan(int64_t np, int64_t nq, int64_t stages, int pairs, bool q_outer, int n_cu) {
    ProductPlan best = {0, 1};
    double least = 1e300;
    for (int k = 0; k < 4; ++k) {
        if (k == 3 && (q_outer || nq > 64)) continue;
        const int64_t tiles = ((np + KINDS[k].bm - 1) / KINDS[k].bm) * ((nq + KINDS[k].bn - 1) / KINDS[k].bn);
        for (int s = 1; s <= 128 && s <= stages; s *= 2) {
            const int64_t per = (stages + s - 1) / s, parts = (stages + per - 1) / per, slots = (int64_t)n_cu * KINDS[k].resident;
            const double rounds = (double)((tiles * parts + slots - 1) / slots);
            double cost = rounds * ((double)per * pairs * KINDS[k].stage + 4000.0);
            if (s > 1) cost += 6000.0 + (double)parts * np * nq * 8.0 / 1900.0;   // partial sums written and read, a launch
            if (cost < least) {
                least = cost;
                best = {k, (int)parts};
            }
        }
    }
    return best;
}

template <class C>
static int launch(const ProductOut& o, int splits, hipStream_t st) {
    OutArgs a = {o, (o.np + C::BM - 1) / C::BM, (o.nq + C::BN - 1) / C::BN, splits, (o.stages + splits - 1) / splits};
    hipLaunchKernelGGL((out_kernel<C>), dim3(product_grid((int64_t)a.tiles_p * a.tiles_q * splits)), dim3(C::THREADS), 0, st, a);
    IVFR_HIP(hipGetLastError());
    return IVFR_OK;
}

template <bool HALF>
static int launch_kind(const ProductOut& o, const ProductPlan& plan, hipStream_t st) {
    if (o.q_outer) {
        if (plan.kind == 0) return launch<Product<256, 256, 2, 4, true, true, HALF>>(o, plan.splits, st);
        if (plan.kind == 1) return launch<Product<128, 128, 2, 2, true, true, HALF>>(o, plan.splits, st);
        return launch<Product<64, 64, 2, 2, true, true, HALF>>(o, plan.splits, st);
    }
    if (plan.kind == 0) return launch<Product<256, 256, 2, 4, true, false, HALF>>(o, plan.splits, st);
    if (plan.kind == 1) return launch<Product<128, 128, 2, 2, true, false, HALF>>(o, plan.splits, st);
    if (plan.kind == 2) return launch<Product<64, 64, 2, 2, true, false, HALF>>(o, plan.splits, st);
    return launch<Product<256, 16, 8, 1, true, false, HALF>>(o, plan.splits, st);
}

int product_launch(const ProductOut& o, const ProductPlan& plan, hipStream_t st) {
    return o.half ? launch_kind<true>(o, plan, st) : launch_kind<false>(o, plan, st);
}
