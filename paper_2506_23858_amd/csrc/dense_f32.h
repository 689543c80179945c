// Shared by the float32 kernels of dense attention, on the float32 and (split operands) on the bfloat16 matrix instruction.
#pragma once
#include "dense_common.h"

#include <cmath>

// A wavefront's 32 x D result from accumulators (column l32 = row of the result) to rows: 16-byte stores.
template <int D>
__device__ __forceinline__ void store_row(char* row, const f32x16_t (&acc)[D / 32], float f, int hf) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4_t x = {acc[dt][4 * i] * f, acc[dt][4 * i + 1] * f, acc[dt][4 * i + 2] * f, acc[dt][4 * i + 3] * f};
            *reinterpret_cast<f32x4_t*>(row + (32 * dt + 8 * i + 4 * hf) * 4) = x;
        }
}
// Base-2 score of x = <q, k> before the bias (scl: signed scale * log2 e); t: tanh of the capped score.
template <bool CAP>
__device__ __forceinline__ float score32(const DenseArgs& a, float x, float scl, float& t) {
    if constexpr (CAP) {
        t = tanhf((a.negate ? -x : x) * a.cap_arg);
        return a.cap2 * t;
    } else {
        return x * scl;
    }
}
// Weight of x = <q, k> from c2 = -(log-sum-exp + bias), base 2; f: the cap's derivative 1 - tanh^2.
template <bool CAP>
__device__ __forceinline__ float weight32(const DenseArgs& a, float x, float scl, float c2, float& f) {
    float t = 0.f;
    const float s2 = score32<CAP>(a, x, scl, t);
    f = CAP ? 1.f - t * t : 1.f;
    return exp2_raw(CAP ? s2 + c2 : fmaf(x, scl, c2));
}
__device__ __forceinline__ f32x16_t zeros16() { return f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

struct Keys { int any_lo, any_hi, all_lo, all_hi, own_lo, own_hi; };
// Keys that any row of the workgroup reads (any), that all rows of the wavefront read (all: no row without keys among them) and that any of them reads (own); w: 2 * NW
// words of LDS.
template <int NW>
__device__ __forceinline__ Keys tile_keys(int lo, int hi, int wave, int lane, int* w) {
    const bool some = lo < hi;
    Keys k = {some ? lo : INT32_MAX, some ? hi : 0, some ? lo : INT32_MAX, some ? hi : 0, 0, 0};
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        k.any_lo = min(k.any_lo, __shfl_xor(k.any_lo, o, 64));
        k.any_hi = max(k.any_hi, __shfl_xor(k.any_hi, o, 64));
        k.all_lo = max(k.all_lo, __shfl_xor(k.all_lo, o, 64));
        k.all_hi = min(k.all_hi, __shfl_xor(k.all_hi, o, 64));
    }
    k.own_lo = __builtin_amdgcn_readfirstlane(k.any_lo);
    k.own_hi = __builtin_amdgcn_readfirstlane(k.any_hi);
    if constexpr (NW > 1) {
        if (lane == 0) {
            w[wave] = k.any_lo;
            w[NW + wave] = k.any_hi;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            k.any_lo = min(k.any_lo, w[i]);
            k.any_hi = max(k.any_hi, w[NW + i]);
        }
    }
    k.any_lo = __builtin_amdgcn_readfirstlane(k.any_lo);
    k.any_hi = __builtin_amdgcn_readfirstlane(k.any_hi);
    k.all_lo = __builtin_amdgcn_readfirstlane(k.all_lo);
    k.all_hi = __builtin_amdgcn_readfirstlane(k.all_hi);
    if (k.any_lo >= k.any_hi) k.any_lo = k.any_hi = 0;
    return k;
}

#define BY_SCORES(LAUNCH)                   \
    do {                                    \
        if (cap && a.slopes) LAUNCH(true, true);   \
        else if (cap) LAUNCH(true, false);         \
        else if (a.slopes) LAUNCH(false, true);    \
        else LAUNCH(false, false);                 \
    } while (0)
