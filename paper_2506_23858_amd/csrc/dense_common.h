// Shared by the kernels of dense attention (vmoba_dense_fwd, vmoba_dense_bwd).
//
// Packed rows.  The query heads that share a key head are rows of one matrix: row m = q * G + g (G = Hq / Hkv) is query q of head
// hkv * G + g.  So a tile of rows reads a key head once for all its query heads, one query of many heads still fills a tile, and the sums
// of dK and dV over shared heads are sums over rows like any other.
//
// Scores in base 2: s2 = log2(e) * s.  x = <q, k> is multiplied by |softmax_scale| * log2(e) (a negative scale turns the sign of an
// operand instead, so that the order of scores is that of x), or goes through the cap:
//   cap tanh(z / cap) = cap (1 - 2 r),  r = 1 / (1 + e^(2 z / cap)),  1 - tanh^2 = 4 r (1 - r).
#pragma once
#include "attn_common.h"

constexpr float DENSE_LOG2E = 1.4426950408889634f;
constexpr float DENSE_LN2 = 0.6931471805599453f;

struct DenseArgs {
    TensorView Q, K, V, O, dO, dQ, dK, dV;
    const float* slopes;
    const int *key_lo, *key_hi, *q_pos;
    long long q_first;
    float* LSE;
    float *part_o, *part_lse;      // forward, more than one split: [splits][B * Hkv][M][D] and [splits][B * Hkv][M] (base 2)
    char* row_info;                // backward: ROW_INFO bytes per 32 rows, see RowInfo
    int4* row_bounds;              // backward: {lowest lo, highest hi, highest lo, lowest hi} of every 32 rows with keys
    int B, Hq, Hkv, G, Sq, Sk, M;
    int splits;
    float scale, scale_log2;       // softmax_scale; max(|softmax_scale| log2 e, FLT_MIN)
    float cap2, cap_in, cap_arg;   // cap log2(e); 2 scale_log2 / cap; |softmax_scale| / cap
    unsigned negate;               // 0x80008000 for a negative scale (bfloat16 pairs)
};

// What the dK/dV kernel needs to know of 32 consecutive rows, one 1 KB request: arrays of 32 words.
struct RowInfo {
    float lse2[32];        // log-sum-exp of the row, base 2; +inf for a row without keys (all its weights are then 0)
    float ndelta[32];      // -rowsum(dO * O)
    int lo[32], hi[32];    // its keys
    float slope2[32];      // slope * log2(e)
    int pos[32];           // its position
    int pad[64];
};
static_assert(sizeof(RowInfo) == 1024, "one request of 64 lanes x 16 bytes");

// Key range of row m's query, within 0 .. Sk; {0, 0} if it has none.
__device__ __forceinline__ int2 dense_range(const DenseArgs& a, int b, int q) {
    if (!a.key_lo) return make_int2(0, a.Sk);
    const long long i = (long long)b * a.Sq + q;
    const int lo = max(a.key_lo[i], 0), hi = min(a.key_hi[i], a.Sk);
    return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
}
__device__ __forceinline__ int dense_position(const DenseArgs& a, int b, int q) {
    return a.q_pos ? a.q_pos[(long long)b * a.Sq + q] : (int)(a.q_first + q);
}
__device__ __forceinline__ const char* row_ptr(const TensorView& t, int b, long long s, int h, int es) {
    return t.ptr + (b * t.stride_b + s * t.stride_s + h * t.stride_h) * es;
}
// Base-2 score of x = <q, k> before the bias; r: what the cap's derivative is formed from.
template <bool CAP>
__device__ __forceinline__ float dense_score(const DenseArgs& a, float x, float& r) {
    if constexpr (CAP) {
        r = __builtin_amdgcn_rcpf(1.f + exp2_raw(x * a.cap_in));
        return fmaf(-2.f * a.cap2, r, a.cap2);
    } else {
        return x * a.scale_log2;
    }
}
// bfloat16 pairs with the values that are not finite replaced by 0; `found` collects whether there were any.
__device__ __forceinline__ bf16x8_t finite_only(bf16x8_t x, unsigned& found) {
    u32x4_t w = __builtin_bit_cast(u32x4_t, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned lo = (w[i] & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u, hi = (w[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
        found |= lo | hi;
        w[i] &= ~(lo | hi);
    }
    return __builtin_bit_cast(bf16x8_t, w);
}
// The forward kernels' last step for a wavefront that met values of V that are not finite in groups of 32 keys with masked pairs, where they were
// taken out of the product: the rows that do read such a key get weight times value added.  A rare path, one key at a time.  lo_a, hi_a, lse_a
// (base 2) are those of row m0 + lane % 16, _b of row m0 + 16 + lane % 16; part0: place of the split's first row.
template <class T, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void dense_repair(const DenseArgs& a, int b, int hk, int m0, int lane, long long part0, int k_first, int k_end, int all_lo,
                                             int all_hi, int lo_a, int lo_b, int hi_a, int hi_b, float lse_a, float lse_b) {
    __threadfence();
    constexpr int CPL = D / 64, ES = sizeof(T);              // channels per lane
    for (int kb = k_first; kb < k_end; kb += 32) {
        if (kb >= all_lo && kb + 32 <= all_hi && kb + 32 <= k_end) continue;
        for (int key = kb; key < min(kb + 32, k_end); ++key) {
            const T *vrow = (const T*)row_ptr(a.V, b, key, hk, ES) + lane * CPL, *krow = (const T*)row_ptr(a.K, b, key, hk, ES) + lane * CPL;
            float v[CPL];
            bool bad = false;
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
                v[c] = (float)vrow[c];
                bad = bad || !(fabsf(v[c]) < INFINITY);
            }
            if (__builtin_amdgcn_ballot_w64(bad) == 0) continue;
            for (int r = 0; r < 32; ++r) {
                const int m = m0 + r;
                const int rl = __shfl(r < 16 ? lo_a : lo_b, r & 15, 64), rh = __shfl(r < 16 ? hi_a : hi_b, r & 15, 64);
                const float lse2 = __shfl(r < 16 ? lse_a : lse_b, r & 15, 64);
                if (m >= a.M || key < rl || key >= rh) continue;
                const int q = m / a.G, h = hk * a.G + (m - q * a.G);
                const T* qrow = (const T*)row_ptr(a.Q, b, q, h, ES) + lane * CPL;
                float x = 0.f;
#pragma unroll
                for (int c = 0; c < CPL; ++c) x = fmaf((float)qrow[c], (float)krow[c], x);
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
                float unused;
                float s2 = dense_score<CAP>(a, a.negate ? -x : x, unused);
                if constexpr (BIAS) s2 -= a.slopes[h] * DENSE_LOG2E * fabsf((float)(dense_position(a, b, q) - key));
                const float p = exp2_raw(s2 - lse2);
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    if (fabsf(v[c]) < INFINITY) continue;
                    if (a.splits > 1) {
                        float* o = a.part_o + (part0 + m) * D + lane * CPL + c;
                        *o += p * v[c];
                    } else {
                        T* o = (T*)row_ptr(a.O, b, q, h, ES) + lane * CPL + c;
                        *o = (T)((float)*o + p * v[c]);
                    }
                }
            }
        }
    }
}
// Workgroup ids go round the 8 XCDs: XCD x = id % 8 takes the x-th eighth of `total` items, so that the tiles of one key head share
// an L2.  -1: this workgroup has none.
__device__ __forceinline__ int dense_item(int total) {
    const int per = (total + 7) >> 3, slot = (int)(blockIdx.x >> 3), f = (int)(blockIdx.x & 7) * per + slot;
    return slot < per && f < total ? f : -1;
}
static inline unsigned dense_grid(int64_t total) { return (unsigned)(ceil_div64(total, 8) * 8); }

// Most rows of a tile that one wavefront takes alone, and the rows of the tile of four.
constexpr int DENSE_FEW_ROWS = 32, DENSE_TILE_ROWS = 128;

void launch_dense_fwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_fwd_f32(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_bwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_bwd_f32(int D, bool cap, hipStream_t st, const DenseArgs& a);
