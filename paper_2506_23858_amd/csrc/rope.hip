// vmoba_rope: rotary positions of queries and keys.
//
// Bound by HBM: every row is read once and written once.  A thread owns VEC pairs of a token (VEC = 8 bfloat16 or 4 float32 values:
// 16-byte accesses) and walks heads of the call's tensors with them, so an angle's sine and cosine are computed once per token and head group, not
// once per head.  The angle in turns, position * frequency / 2 pi, is reduced to [-1/2, 1/2] in float64: the error of
// a float32 angle, position * 2^-24, would reach whole radians at positions of some millions.
#include "common.h"

#include <cmath>

namespace {

constexpr int MAX_TENSORS = 8;
struct RopeTensor { TensorView in, out; int heads; };
struct RopeArgs {
    RopeTensor t[MAX_TENSORS];
    const double* freqs;
    const int* positions;
    long long pos_stride_b, first;
    long long tokens;          // B * S
    int n_tensors, total_heads, S, D, P, axes, dims0, dims01;      // P: rotated pairs; pairs below dims0 / dims01 belong to axis 0 / to axis 0 or 1
    int gh, gw;                // grid extents H and W (no positions, three axes)
    int chunks, tail_chunks;   // groups of VEC pairs and, behind them, of VEC copied channels
    int heads_per_part;
    float mscale;
    int negative;
};

template <class T, int N> struct VecOf { T v[N]; };

template <class T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }

// HALF: pairs (p, p + P), else (2p, 2p + 1).  ALIGNED: every 16-byte access is aligned and every group is whole.
template <class T, bool HALF, bool ALIGNED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    constexpr int VEC = 16 / sizeof(T);
    using Vec = VecOf<T, VEC>;
    const int per_token = a.chunks + a.tail_chunks;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long token = id / per_token;
    const int c = (int)(id - token * per_token);
    if (token >= a.tokens) return;
    const int b = (int)(token / a.S), s = (int)(token - (long long)b * a.S);
    const int h0 = blockIdx.y * a.heads_per_part, h1 = min(h0 + a.heads_per_part, a.total_heads);

    auto load = [](const T* p) {
        Vec v;
        if constexpr (ALIGNED) v = *reinterpret_cast<const Vec*>(__builtin_assume_aligned(p, 16));
        else __builtin_memcpy(&v, p, sizeof(v));
        return v;
    };
    auto store = [](T* p, const Vec& v) {
        if constexpr (ALIGNED) *reinterpret_cast<Vec*>(__builtin_assume_aligned(p, 16)) = v;
        else __builtin_memcpy(p, &v, sizeof(v));
    };
    // f(input row, output row) for the heads of this part, tensor by tensor
    auto rows = [&](auto f) {
        int base = 0;
        for (int i = 0; i < a.n_tensors; ++i) {
            const RopeTensor& t = a.t[i];
            const int e0 = max(h0 - base, 0), e1 = min(h1 - base, t.heads);
            const T* src = (const T*)t.in.ptr + b * t.in.stride_b + s * t.in.stride_s;
            T* dst = (T*)t.out.ptr + b * t.out.stride_b + s * t.out.stride_s;
#pragma unroll 4
            for (int h = e0; h < e1; ++h) f(src + h * t.in.stride_h, dst + h * t.out.stride_h);
            base += t.heads;
        }
    };

    if (c >= a.chunks) {                       // channels that are not rotated
        const int d0 = 2 * a.P + (c - a.chunks) * VEC, n = min(VEC, a.D - d0);
        rows([&](const T* src, T* dst) {
            if (ALIGNED || n == VEC) store(dst + d0, load(src + d0));
            else
                for (int j = 0; j < n; ++j) dst[d0 + j] = src[d0 + j];
        });
        return;
    }
    const int p0 = c * VEC, n = min(VEC, a.P - p0);
    float cs[VEC], sn[VEC];
    {
        long long at[3] = {a.first, 0, 0};
        if (a.positions) {
            const int* q = a.positions + b * a.pos_stride_b + (long long)s * a.axes;
            for (int x = 0; x < a.axes; ++x) at[x] += q[x];
        } else if (a.axes == 3) {
            const int hw = a.gh * a.gw, t = s / hw, r = s - t * hw;
            at[0] += t;
            at[1] = r / a.gw;
            at[2] = r - (int)at[1] * a.gw;
        } else {
            at[0] += s;
        }
        const double p_t = (double)at[0], p_h = (double)at[1], p_w = (double)at[2];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int p = min(p0 + j, a.P - 1);
            const double turns = (p < a.dims0 ? p_t : p < a.dims01 ? p_h : p_w) * (a.freqs[p] * 0.15915494309189533577);
            float si, co;
            sincospif(2.f * (float)(turns - rint(turns)), &si, &co);
            cs[j] = co * a.mscale;
            sn[j] = (a.negative ? -si : si) * a.mscale;
        }
    }
    rows([&](const T* src, T* dst) {
        if (ALIGNED || n == VEC) {
            const int i0 = HALF ? p0 : 2 * p0, i1 = HALF ? p0 + a.P : 2 * p0 + VEC;
            const Vec x = load(src + i0), y = load(src + i1);
            Vec u, v;
            if constexpr (HALF) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float p = (float)x.v[j], q = (float)y.v[j];
                    u.v[j] = (T)(p * cs[j] - q * sn[j]);
                    v.v[j] = (T)(p * sn[j] + q * cs[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float p = (float)(j < VEC / 2 ? x.v[2 * j % VEC] : y.v[2 * j % VEC]);
                    const float q = (float)(j < VEC / 2 ? x.v[(2 * j + 1) % VEC] : y.v[(2 * j + 1) % VEC]);
                    const T r = (T)(p * cs[j] - q * sn[j]), w = (T)(p * sn[j] + q * cs[j]);
                    if (j < VEC / 2) { u.v[2 * j % VEC] = r; u.v[(2 * j + 1) % VEC] = w; }
                    else { v.v[2 * j % VEC] = r; v.v[(2 * j + 1) % VEC] = w; }
                }
            }
            store(dst + i0, u);
            store(dst + i1, v);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j < n) {
                    const int i0 = HALF ? p0 + j : 2 * (p0 + j), i1 = HALF ? p0 + j + a.P : i0 + 1;
                    const float p = (float)src[i0], q = (float)src[i1];
                    dst[i0] = (T)(p * cs[j] - q * sn[j]);
                    dst[i1] = (T)(p * sn[j] + q * cs[j]);
                }
        }
    });
}

bool dims_ok(int n_axes, const int32_t* dims) {
    if (n_axes < 1 || n_axes > 3 || !dims) return false;
    for (int i = 0; i < n_axes; ++i)
        if (dims[i] <= 0 || dims[i] % 2 || dims[i] > 1024) return false;
    return true;
}

}  // namespace

extern "C" int vmoba_rope_freqs(int n_axes, const int32_t* dims, double base, int scaling, double factor, int64_t train_len, double* freqs,
                                float* mscale) {
    if (!dims_ok(n_axes, dims) || !freqs || !mscale) return VMOBA_ERR_INVALID_ARG;
    if (!std::isfinite(base) || base <= 0.0 || !std::isfinite(factor) || factor < 1.0) return VMOBA_ERR_INVALID_ARG;
    if (scaling < VMOBA_ROPE_PLAIN || scaling > VMOBA_ROPE_YARN) return VMOBA_ERR_UNSUPPORTED;
    if (scaling == VMOBA_ROPE_YARN && train_len <= 0) return VMOBA_ERR_INVALID_ARG;
    for (int a = 0; a < n_axes; ++a)
        if (scaling == VMOBA_ROPE_NTK && dims[a] <= 2) return VMOBA_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586477;
    int n = 0;
    for (int a = 0; a < n_axes; ++a) {
        const double d = dims[a], b = scaling == VMOBA_ROPE_NTK ? base * std::pow(factor, d / (d - 2.0)) : base;
        for (int i = 0; i < dims[a] / 2; ++i) {
            const double w = std::pow(b, -2.0 * i / d);
            double f = w;
            if (scaling == VMOBA_ROPE_LINEAR) f = w / factor;
            if (scaling == VMOBA_ROPE_YARN) {
                const double g = std::fmin(1.0, std::fmax(0.0, ((double)train_len * w / two_pi - 1.0) / 31.0));
                f = (1.0 - g) * w / factor + g * w;
            }
            freqs[n++] = f;
        }
    }
    *mscale = scaling == VMOBA_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return VMOBA_OK;
}

extern "C" int vmoba_rope(int B, int64_t S, int D, int n_tensors, const int32_t* Hh, const vmoba_tensor* in, const vmoba_tensor* out,
                          const double* freqs, int n_axes, const int32_t* dims, int layout, int inverse, float mscale, const vmoba_grid* grid,
                          int64_t first, const int32_t* positions, int64_t pos_stride_b, void* stream) {
    if (B < 0 || S < 0 || n_tensors < 1 || n_tensors > MAX_TENSORS || !Hh || !in || !out || !freqs) return VMOBA_ERR_INVALID_ARG;
    if (!dims_ok(n_axes, dims) || !std::isfinite(mscale) || (inverse != 0 && inverse != 1)) return VMOBA_ERR_INVALID_ARG;
    if (layout != VMOBA_ROPE_HALF && layout != VMOBA_ROPE_INTERLEAVED) return VMOBA_ERR_UNSUPPORTED;
    if (D < 2 || D > 1024 || D % 2) return VMOBA_ERR_UNSUPPORTED;
    int R = 0;
    for (int i = 0; i < n_axes; ++i) R += dims[i];
    if (R > D) return VMOBA_ERR_INVALID_ARG;
    if (S > INT32_MAX || (int64_t)B * S > ((int64_t)1 << 40)) return VMOBA_ERR_UNSUPPORTED;
    RopeArgs a{};
    const bool bf16 = in[0].dtype == VMOBA_BF16;
    const int vec = bf16 ? 8 : 4;
    bool copies = false;                       // a tensor that does not stay in place
    for (int i = 0; i < n_tensors; ++i) {
        if (Hh[i] < 1 || !tensor_ok(&in[i]) || !tensor_ok(&out[i])) return VMOBA_ERR_INVALID_ARG;
        if (in[i].dtype != in[0].dtype || out[i].dtype != in[0].dtype) return VMOBA_ERR_UNSUPPORTED;
        const bool same = in[i].ptr == out[i].ptr;
        if (same && (in[i].stride_b != out[i].stride_b || in[i].stride_s != out[i].stride_s || in[i].stride_h != out[i].stride_h)) return VMOBA_ERR_INVALID_ARG;
        copies = copies || !same;
        a.t[i] = {make_view(&in[i]), make_view(&out[i]), Hh[i]};
        if (a.total_heads > (1 << 20) - Hh[i]) return VMOBA_ERR_UNSUPPORTED;
        a.total_heads += Hh[i];
    }
    if (!positions) {
        if (n_axes == 2) return VMOBA_ERR_INVALID_ARG;
        if (n_axes == 3) {
            if (!grid || grid->T <= 0 || grid->H <= 0 || grid->W <= 0) return VMOBA_ERR_INVALID_ARG;
            if ((int64_t)grid->T * grid->H > INT32_MAX || (int64_t)grid->T * grid->H * grid->W != S) return VMOBA_ERR_INVALID_ARG;
            a.gh = grid->H;
            a.gw = grid->W;
        }
    }
    if (B == 0 || S == 0) return VMOBA_OK;
    a.freqs = freqs;
    a.positions = positions;
    a.pos_stride_b = pos_stride_b;
    a.first = first;
    a.tokens = (int64_t)B * S;
    a.n_tensors = n_tensors;
    a.S = (int)S;
    a.D = D;
    a.P = R / 2;
    a.axes = n_axes;
    a.dims0 = n_axes > 1 ? dims[0] / 2 : R / 2;
    a.dims01 = n_axes > 2 ? a.dims0 + dims[1] / 2 : R / 2;
    a.chunks = (int)ceil_div64(a.P, vec);
    a.tail_chunks = copies ? (int)ceil_div64(D - R, vec) : 0;
    a.mscale = mscale;
    a.negative = inverse;
    const bool aligned = a.P % vec == 0 && (D - R) % vec == 0;
    const int64_t blocks = ceil_div64(a.tokens * (a.chunks + a.tail_chunks), 256);
    if (blocks > INT32_MAX) return VMOBA_ERR_UNSUPPORTED;
    // The heads are dealt to more threads, down to one each, until there are eight workgroups per compute unit.
    const int64_t parts = blocks >= 2048 ? 1 : ceil_div64(2048, blocks);
    a.heads_per_part = (int)ceil_div64(a.total_heads, parts < a.total_heads ? parts : a.total_heads);
    const dim3 g((unsigned)blocks, (unsigned)ceil_div64(a.total_heads, a.heads_per_part));
    hipStream_t st = (hipStream_t)stream;
#define LAUNCH(T, HALF)                                                             \
    do {                                                                            \
        if (aligned) rope_kernel<T, HALF, true><<<g, dim3(256), 0, st>>>(a);        \
        else rope_kernel<T, HALF, false><<<g, dim3(256), 0, st>>>(a);               \
    } while (0)
    if (bf16 && layout == VMOBA_ROPE_HALF) LAUNCH(__bf16, true);
    else if (bf16) LAUNCH(__bf16, false);
    else if (layout == VMOBA_ROPE_HALF) LAUNCH(float, true);
    else LAUNCH(float, false);
#undef LAUNCH
    VMOBA_CHECK_LAUNCH();
    return VMOBA_OK;
}
