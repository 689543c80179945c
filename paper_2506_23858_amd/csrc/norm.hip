// vmoba_rmsnorm_fwd / vmoba_rmsnorm_bwd: root-mean-square norm with the residual's addition, an 8-bit output with scales, and the gradient.
//
// Bound by HBM: every row is read once and written once, and held in registers between.  A row belongs to a group of L lanes of one
// wavefront (short rows: several rows per wavefront), or to the four wavefronts of a workgroup (rows that would not fit one
// wavefront's registers); a lane owns NC pieces of 16 bytes, L pieces apart.  Groups walk rows with a stride, so the weight is loaded once
// per group and not once per row, and the weight's gradient is summed in registers: one partial row per workgroup, added
// up in a fixed order by a second, small launch.
#include "attn_common.h"

#include <cfloat>
#include <cmath>

namespace {

constexpr int MAX_D = 16384;

struct NormArgs {
    TensorView x, residual, total, y, dy, dtotal, dx;
    const void* weight;
    float *y_scale, *inv_rms, *partial;
    long long rows;
    int S, Hh, D, weight_bf16;
    float eps;
};

template <class T, int N> struct VecOf { T v[N]; };

// A row's pieces: 16 bytes of T at a time where the row is aligned and whole, element by element at its end.  Every one is touched once: non-temporal
// (forward with residual, 32 760 x 1536 bfloat16: 113 -> 107 us).
template <class T, bool ALIGNED, int VEC>
__device__ __forceinline__ void load_piece(const T* row, int d0, int D, float (&f)[VEC]) {
    VecOf<T, VEC> v;
    if (ALIGNED || d0 + VEC <= D) {
        if constexpr (ALIGNED) {
            const u32x4_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + d0));
            __builtin_memcpy(&v, &x, sizeof(v));
        } else {
            __builtin_memcpy(&v, row + d0, sizeof(v));
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = (float)v.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = d0 + j < D ? (float)row[d0 + j] : 0.f;
    }
}
template <class T, bool ALIGNED, int VEC>
__device__ __forceinline__ void store_piece(T* row, int d0, int D, const float (&f)[VEC]) {
    if (ALIGNED || d0 + VEC <= D) {
        VecOf<T, VEC> v;
#pragma unroll
        for (int j = 0; j < VEC; ++j) v.v[j] = (T)f[j];
        if constexpr (ALIGNED) {
            u32x4_t x;
            __builtin_memcpy(&x, &v, sizeof(v));
            __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t*>(row + d0));
        } else {
            __builtin_memcpy(row + d0, &v, sizeof(v));
        }
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (d0 + j < D) row[d0 + j] = (T)f[j];
    }
}
template <bool ALIGNED, int VEC>
__device__ __forceinline__ void store_piece8(uint8_t* row, int d0, int D, const float (&f)[VEC]) {
    uint32_t w[VEC / 4];
#pragma unroll
    for (int j = 0; j < VEC / 4; ++j) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
        w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], p, true);
    }
    if (ALIGNED || d0 + VEC <= D) {
        if constexpr (ALIGNED) __builtin_memcpy(__builtin_assume_aligned(row + d0, VEC), w, VEC);
        else __builtin_memcpy(row + d0, w, VEC);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (d0 + j < D) row[d0 + j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
}

// Sum or maximum over the L lanes of a group (L <= 64: within the wavefront; 256: through `lds`, one word per wavefront and call).
template <int L, bool MAX>
__device__ __forceinline__ float reduce(float x, float* lds) {
#pragma unroll
    for (int o = (L < 64 ? L : 64) / 2; o >= 1; o >>= 1) {
        const float y = __shfl_xor(x, o, 64);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    if constexpr (L == 256) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = MAX ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3])) : (lds[0] + lds[1]) + (lds[2] + lds[3]);
        __syncthreads();
    }
    return x;
}

template <int NC, int VEC, int L>
__device__ __forceinline__ void load_weight(const NormArgs& a, int lane, float (&w)[NC][VEC]) {
    auto load = [&](auto type) {
        using W = decltype(type);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d0 = (c * L + lane) * VEC;
            const W* p = (const W*)a.weight + d0;
            if (d0 + VEC <= a.D) {
                VecOf<W, VEC> v;
                __builtin_memcpy(&v, p, sizeof(v));
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[c][j] = (float)v.v[j];
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[c][j] = d0 + j < a.D ? (float)p[j] : 0.f;
            }
        }
    };
    if (a.weight && a.weight_bf16) load(__bf16{});
    else if (a.weight) load(float{});
    else
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) w[c][j] = (c * L + lane) * VEC + j < a.D ? 1.f : 0.f;
}
struct RowAt { int b, h, s; };
__device__ __forceinline__ RowAt row_at(long long r, const NormArgs& a) {      // rows in the order (b, s, h)
    RowAt q;
    if (a.rows < (1LL << 31)) {                              // (a 64-bit division is some hundred instructions)
        const unsigned u = (unsigned)r, bs = a.Hh == 1 ? u : u / (unsigned)a.Hh;
        q.h = (int)(u - bs * (unsigned)a.Hh);
        q.b = bs < (unsigned)a.S ? 0 : (int)(bs / (unsigned)a.S);
        q.s = (int)(bs - (unsigned)q.b * (unsigned)a.S);
    } else {
        const long long bs = r / a.Hh;
        q.h = (int)(r - bs * a.Hh);
        q.b = (int)(bs / a.S);
        q.s = (int)(bs - (long long)q.b * a.S);
    }
    return q;
}
template <class T>
__device__ __forceinline__ T* row_of(const TensorView& t, const RowAt& q) { return (T*)t.ptr + q.b * t.stride_b + q.s * t.stride_s + q.h * t.stride_h; }

template <class T, bool ALIGNED, bool OUT8, int L, int NC>
__global__ __launch_bounds__(256) void rmsnorm_fwd_kernel(NormArgs a) {
    constexpr int VEC = 16 / sizeof(T), GROUPS = 256 / L;
    __shared__ float lds[4];
    const int lane = threadIdx.x % L;
    float w[NC][VEC];
    load_weight<NC, VEC, L>(a, lane, w);
    for (long long r = (long long)blockIdx.x * GROUPS + threadIdx.x / L; r < a.rows; r += (long long)gridDim.x * GROUPS) {
        const RowAt q = row_at(r, a);
        const T* x = row_of<T>(a.x, q);
        float t[NC][VEC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d0 = (c * L + lane) * VEC;
            if (d0 < a.D) load_piece<T, ALIGNED, VEC>(x, d0, a.D, t[c]);
            else
#pragma unroll
                for (int j = 0; j < VEC; ++j) t[c][j] = 0.f;
        }
        if (a.residual.ptr) {
            const T* res = row_of<T>(a.residual, q);
            float e[NC][VEC];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d0 = (c * L + lane) * VEC;
                if (d0 < a.D) load_piece<T, ALIGNED, VEC>(res, d0, a.D, e[c]);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) e[c][j] = 0.f;
            }
            T* total = row_of<T>(a.total, q);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d0 = (c * L + lane) * VEC;
#pragma unroll
                for (int j = 0; j < VEC; ++j) t[c][j] = (float)(T)(t[c][j] + e[c][j]);      // what is stored is normalised
                if (d0 < a.D) store_piece<T, ALIGNED, VEC>(total, d0, a.D, t[c]);
            }
        }
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) ss = fmaf(t[c][j], t[c][j], ss);
        ss = reduce<L, false>(ss, lds);
        const float inv = 1.f / sqrtf(ss / (float)a.D + a.eps);
        if (a.inv_rms && lane == 0) a.inv_rms[r] = inv;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) t[c][j] = t[c][j] * inv * w[c][j];
        if constexpr (OUT8) {
            float top = 0.f;
            bool nan = false;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    top = fmaxf(top, fabsf(t[c][j]));
                    nan = nan || t[c][j] != t[c][j];
                }
            // (a NaN that the maximum passes over makes the whole row's scale one)
            top = reduce<L, true>(nan ? INFINITY : top, lds);
            const bool some = top / 448.f > 0.f;
            const float scale = top == INFINITY ? NAN : some ? top / 448.f : 1.f, up = top == INFINITY ? NAN : some ? fminf(448.f / top, FLT_MAX) : 1.f;
            if (lane == 0) a.y_scale[r] = scale;
            uint8_t* y = (uint8_t*)a.y.ptr + q.b * a.y.stride_b + q.s * a.y.stride_s + q.h * a.y.stride_h;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d0 = (c * L + lane) * VEC;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float v = t[c][j] * up;
                    t[c][j] = v > 448.f ? 448.f : v < -448.f ? -448.f : v;      // the roundings can pass the largest value
                }
                if (d0 < a.D) store_piece8<ALIGNED, VEC>(y, d0, a.D, t[c]);
            }
        } else {
            T* y = row_of<T>(a.y, q);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d0 = (c * L + lane) * VEC;
                if (d0 < a.D) store_piece<T, ALIGNED, VEC>(y, d0, a.D, t[c]);
            }
        }
    }
}

template <class T, bool ALIGNED, int L, int NC>
__global__ __launch_bounds__(256) void rmsnorm_bwd_kernel(NormArgs a) {
    constexpr int VEC = 16 / sizeof(T), GROUPS = 256 / L;
    __shared__ float lds[4];
    const int lane = threadIdx.x % L;
    float w[NC][VEC], dw[NC][VEC];
    load_weight<NC, VEC, L>(a, lane, w);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) dw[c][j] = 0.f;
    for (long long r = (long long)blockIdx.x * GROUPS + threadIdx.x / L; r < a.rows; r += (long long)gridDim.x * GROUPS) {
        const RowAt q = row_at(r, a);
        const T *x = row_of<T>(a.x, q), *dy = row_of<T>(a.dy, q), *more = a.dtotal.ptr ? row_of<T>(a.dtotal, q) : nullptr;
        float n[NC][VEC], g[NC][VEC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d0 = (c * L + lane) * VEC;
            if (d0 < a.D) {
                load_piece<T, ALIGNED, VEC>(x, d0, a.D, n[c]);
                load_piece<T, ALIGNED, VEC>(dy, d0, a.D, g[c]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) n[c][j] = g[c][j] = 0.f;
            }
        }
        const float inv = a.inv_rms[r];
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                n[c][j] *= inv;
                dw[c][j] = fmaf(g[c][j], n[c][j], dw[c][j]);
                g[c][j] *= w[c][j];
                dot = fmaf(g[c][j], n[c][j], dot);
            }
        const float mean = reduce<L, false>(dot, lds) / (float)a.D;
        T* dx = row_of<T>(a.dx, q);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d0 = (c * L + lane) * VEC;
            if (d0 >= a.D) continue;
            float e[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) e[j] = 0.f;
            if (more) load_piece<T, ALIGNED, VEC>(more, d0, a.D, e);
#pragma unroll
            for (int j = 0; j < VEC; ++j) e[j] = fmaf(g[c][j] - n[c][j] * mean, inv, e[j]);
            store_piece<T, ALIGNED, VEC>(dx, d0, a.D, e);
        }
    }
    if (!a.partial) return;
    // one row of sums per workgroup: groups of the same lanes are added in their order
    float* out = a.partial + (long long)blockIdx.x * a.D;
    if constexpr (GROUPS == 1) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int d = (c * L + lane) * VEC + j;
                if (d < a.D) out[d] = dw[c][j];
            }
    } else {
        __shared__ float sums[GROUPS * L * VEC];
        for (int c = 0; c < NC; ++c) {
            __syncthreads();
#pragma unroll
            for (int cc = 0; cc < NC; ++cc)
                if (cc == c)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sums[threadIdx.x * VEC + j] = dw[cc][j];
            __syncthreads();
            for (int i = threadIdx.x; i < L * VEC; i += 256) {
                float s = 0.f;
                for (int gI = 0; gI < GROUPS; ++gI) s += sums[gI * L * VEC + i];
                if (c * L * VEC + i < a.D) out[c * L * VEC + i] = s;
            }
        }
    }
}

// dweight[d] = sum of the workgroups' rows, in a fixed order: 16 channels x 64 interleaved shares of the rows per workgroup
__global__ __launch_bounds__(1024) void rmsnorm_dweight_kernel(const float* __restrict__ partial, float* __restrict__ dweight, int n, int D) {
    __shared__ float sums[64][17];
    const int d = blockIdx.x * 16 + threadIdx.x % 16, part = threadIdx.x / 16;
    float s = 0.f;
    if (d < D) {
#pragma unroll 8
        for (int i = part; i < n; i += 64) s += partial[(long long)i * D + d];
    }
    sums[part][threadIdx.x % 16] = s;
    __syncthreads();
    if (part == 0 && d < D) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) t += sums[i][threadIdx.x % 16];
        dweight[d] = t;
    }
}

// Lanes and pieces per lane of a row of D channels, VEC channels a piece.
struct Shape { int L, NC; };
Shape shape_for(int D, int vec) {
    const int pieces = (D + vec - 1) / vec;
    if (pieces <= 16) return {16, 1};
    if (pieces <= 32) return {32, 1};
    if (pieces <= 64) return {64, 1};
    if (pieces <= 128) return {64, 2};
    if (pieces <= 192) return {64, 3};
    if (pieces <= 256) return {64, 4};
    if (pieces <= 512) return {256, 2};
    if (pieces <= 1024) return {256, 4};
    if (pieces <= 2048) return {256, 8};
    return {256, 16};
}
// Most workgroups of a backward call, which is also the most partial rows of dweight.
constexpr int64_t BWD_WORKGROUPS = 1024;
// Workgroups that share `need` workgroups' worth of rows equally, no more of them than run at a time.  (Forward calls: 32 760 x 1536 bfloat16,
// where 1024 run, 82 us with as many, 92 with twice as many, 113 with 1280; 168 480 x 128 float32, one piece per lane, 42 us with as many, 33 with twice.)
int64_t even_grid(int64_t need, int64_t running) { return ceil_div64(need, ceil_div64(need, running)); }
template <class F>
int64_t running_workgroups(F kernel) {
    int per_cu = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, 256, 0) != hipSuccess || per_cu < 1) per_cu = 2;
    return (int64_t)per_cu * vmoba_num_cus();
}

bool norm_tensor_ok(const vmoba_tensor* t, int dtype) {
    const int es = dtype == VMOBA_F8E4M3 ? 1 : dtype_size(dtype);
    return t && t->ptr && t->dtype == dtype && ((uintptr_t)t->ptr) % es == 0;
}
bool aligned16(const vmoba_tensor* t, int es, int bytes) {     // rows start at multiples of `bytes`
    const int64_t per = bytes / es;
    return ((uintptr_t)t->ptr) % bytes == 0 && t->stride_b % per == 0 && t->stride_s % per == 0 && t->stride_h % per == 0;
}
int check_sizes(int B, int Hh, int64_t S, int D) {
    if (B < 0 || S < 0 || Hh <= 0 || D <= 0) return VMOBA_ERR_INVALID_ARG;
    if (D > MAX_D || S > INT32_MAX || (double)B * (double)S * Hh > 1e12) return VMOBA_ERR_UNSUPPORTED;
    return VMOBA_OK;
}
bool weight_ok(const void* weight, int dtype) {
    return !weight || ((dtype == VMOBA_F32 || dtype == VMOBA_BF16) && ((uintptr_t)weight) % dtype_size(dtype) == 0);
}

#define DISPATCH_SHAPE(CALL)                                        \
    switch (shape.L * 100 + shape.NC) {                             \
        case 1601: CALL(16, 1); break;                              \
        case 3201: CALL(32, 1); break;                              \
        case 6401: CALL(64, 1); break;                              \
        case 6402: CALL(64, 2); break;                              \
        case 6403: CALL(64, 3); break;                              \
        case 6404: CALL(64, 4); break;                              \
        case 25602: CALL(256, 2); break;                            \
        case 25604: CALL(256, 4); break;                            \
        case 25608: CALL(256, 8); break;                            \
        default: if constexpr (sizeof(T) == 4) CALL(256, 16); break; \
    }

template <class T, bool ALIGNED, bool OUT8>
void launch_fwd(const Shape& shape, hipStream_t st, const NormArgs& a) {
#define CALL(L, NC)                                                                                                        \
    do {                                                                                                                   \
        static const int64_t running = running_workgroups(rmsnorm_fwd_kernel<T, ALIGNED, OUT8, L, NC>);                    \
        const unsigned grid = (unsigned)even_grid(ceil_div64(a.rows, 256 / L), (NC == 1 ? 2 : 1) * running);                                  \
        rmsnorm_fwd_kernel<T, ALIGNED, OUT8, L, NC><<<dim3(grid), dim3(256), 0, st>>>(a);                                  \
    } while (0)
    DISPATCH_SHAPE(CALL)
#undef CALL
}
// Returns the number of partial rows of dweight still to be added.  Up to ONE_WORKGROUP steps of rows are left to a single workgroup, whose row of sums is dweight:
// a step costs 1.5 us, the second launch 2.2 and the host another 3 (1536 bfloat16 channels, in a graph: 4 rows 6.8 -> 4.6 us, 8 rows 6.9 -> 6.1; 12 rows would go to 7.7).
constexpr int64_t ONE_WORKGROUP = 2;
template <class T, bool ALIGNED>
unsigned launch_bwd(const Shape& shape, hipStream_t st, NormArgs a, float* dweight) {
    unsigned grid = 0;
#define CALL(L, NC)                                                                                                        \
    do {                                                                                                                   \
        static const int64_t running = running_workgroups(rmsnorm_bwd_kernel<T, ALIGNED, L, NC>);                          \
        const int64_t need = ceil_div64(a.rows, 256 / L);                                                                  \
        const bool one = dweight && need <= ONE_WORKGROUP;                                                                 \
        if (one) a.partial = dweight;                                                                                      \
        grid = one ? 1 : (unsigned)even_grid(need, running < BWD_WORKGROUPS ? running : BWD_WORKGROUPS);                   \
        rmsnorm_bwd_kernel<T, ALIGNED, L, NC><<<dim3(grid), dim3(256), 0, st>>>(a);                                        \
        if (one) grid = 0;                                                                                                 \
    } while (0)
    DISPATCH_SHAPE(CALL)
#undef CALL
    return grid;
}

}  // namespace

extern "C" size_t vmoba_rmsnorm_workspace_bytes(int B, int Hh, int64_t S, int D) {
    if (check_sizes(B, Hh, S, D) != VMOBA_OK) return 0;
    // a workgroup holds at least one row, so there are never more partial rows than rows
    const int64_t rows = (int64_t)B * Hh * S;
    return align_up((size_t)(rows < BWD_WORKGROUPS ? rows : BWD_WORKGROUPS) * D * 4, 256);
}

extern "C" int vmoba_rmsnorm_fwd(int B, int Hh, int64_t S, int D, const vmoba_tensor* x, const vmoba_tensor* residual, const void* weight,
                                 int weight_dtype, float eps, const vmoba_tensor* total, const vmoba_tensor* y, float* y_scale, float* inv_rms,
                                 void* stream) {
    if (const int rc = check_sizes(B, Hh, S, D)) return rc;
    if (!x || !y || (x->dtype != VMOBA_F32 && x->dtype != VMOBA_BF16)) return VMOBA_ERR_INVALID_ARG;
    const int dt = x->dtype, es = dtype_size(dt);
    if (y->dtype != dt && y->dtype != VMOBA_F8E4M3) return VMOBA_ERR_UNSUPPORTED;
    const bool out8 = y->dtype == VMOBA_F8E4M3;
    if (!norm_tensor_ok(x, dt) || !norm_tensor_ok(y, y->dtype) || (residual && !norm_tensor_ok(residual, dt)) || (total && !norm_tensor_ok(total, dt)))
        return VMOBA_ERR_INVALID_ARG;
    if ((residual != nullptr) != (total != nullptr) || out8 != (y_scale != nullptr)) return VMOBA_ERR_INVALID_ARG;
    if (!weight_ok(weight, weight_dtype) || !std::isfinite(eps) || eps < 0.f) return VMOBA_ERR_INVALID_ARG;
    if (B == 0 || S == 0) return VMOBA_OK;
    NormArgs a{};
    a.x = make_view(x);
    a.y = make_view(y);
    if (residual) { a.residual = make_view(residual); a.total = make_view(total); }
    a.weight = weight;
    a.weight_bf16 = weight_dtype == VMOBA_BF16;
    a.y_scale = y_scale;
    a.inv_rms = inv_rms;
    a.rows = (long long)B * Hh * S;
    a.S = (int)S;
    a.Hh = Hh;
    a.D = D;
    a.eps = eps;
    const int vec = 16 / es;
    const bool aligned = D % vec == 0 && aligned16(x, es, 16) && (out8 ? aligned16(y, 1, vec) : aligned16(y, es, 16)) &&
                         (!residual || (aligned16(residual, es, 16) && aligned16(total, es, 16)));
    const Shape shape = shape_for(D, vec);
    hipStream_t st = (hipStream_t)stream;
#define BY_ALIGNMENT(T, OUT8)                                        \
    do {                                                             \
        if (aligned) launch_fwd<T, true, OUT8>(shape, st, a);  \
        else launch_fwd<T, false, OUT8>(shape, st, a);         \
    } while (0)
    if (dt == VMOBA_BF16 && out8) BY_ALIGNMENT(__bf16, true);
    else if (dt == VMOBA_BF16) BY_ALIGNMENT(__bf16, false);
    else if (out8) BY_ALIGNMENT(float, true);
    else BY_ALIGNMENT(float, false);
#undef BY_ALIGNMENT
    VMOBA_CHECK_LAUNCH();
    return VMOBA_OK;
}

extern "C" int vmoba_rmsnorm_bwd(int B, int Hh, int64_t S, int D, const vmoba_tensor* x, const void* weight, int weight_dtype, const float* inv_rms,
                                 const vmoba_tensor* dy, const vmoba_tensor* dtotal, const vmoba_tensor* dx, float* dweight, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (const int rc = check_sizes(B, Hh, S, D)) return rc;
    if (!x || (x->dtype != VMOBA_F32 && x->dtype != VMOBA_BF16)) return VMOBA_ERR_INVALID_ARG;
    const int dt = x->dtype, es = dtype_size(dt);
    if (!norm_tensor_ok(x, dt) || !norm_tensor_ok(dy, dt) || !norm_tensor_ok(dx, dt) || (dtotal && !norm_tensor_ok(dtotal, dt)) || !inv_rms)
        return VMOBA_ERR_INVALID_ARG;
    if (!weight_ok(weight, weight_dtype) || (dweight && B > 0 && S > 0 && (!workspace || (uintptr_t)workspace % 16)))
        return VMOBA_ERR_INVALID_ARG;
    if (dweight && workspace_bytes < vmoba_rmsnorm_workspace_bytes(B, Hh, S, D)) return VMOBA_ERR_WORKSPACE;
    NormArgs a{};
    a.x = make_view(x);
    a.dy = make_view(dy);
    a.dx = make_view(dx);
    if (dtotal) a.dtotal = make_view(dtotal);
    a.weight = weight;
    a.weight_bf16 = weight_dtype == VMOBA_BF16;
    a.inv_rms = const_cast<float*>(inv_rms);
    a.partial = dweight ? (float*)workspace : nullptr;
    a.rows = (long long)B * Hh * S;
    a.S = (int)S;
    a.Hh = Hh;
    a.D = D;
    const int vec = 16 / es;
    const bool aligned = D % vec == 0 && aligned16(x, es, 16) && aligned16(dy, es, 16) && aligned16(dx, es, 16) && (!dtotal || aligned16(dtotal, es, 16));
    const Shape shape = shape_for(D, vec);
    unsigned grid = 0;
    hipStream_t st = (hipStream_t)stream;
    if (a.rows > 0) {
        if (dt == VMOBA_BF16 && aligned) grid = launch_bwd<__bf16, true>(shape, st, a, dweight);
        else if (dt == VMOBA_BF16) grid = launch_bwd<__bf16, false>(shape, st, a, dweight);
        else if (aligned) grid = launch_bwd<float, true>(shape, st, a, dweight);
        else grid = launch_bwd<float, false>(shape, st, a, dweight);
        VMOBA_CHECK_LAUNCH();
    }
    if (dweight && (grid > 0 || a.rows == 0)) {
        rmsnorm_dweight_kernel<<<dim3((unsigned)ceil_div64(D, 16)), dim3(1024), 0, st>>>((const float*)workspace, dweight, (int)grid, D);
        VMOBA_CHECK_LAUNCH();
    }
    return VMOBA_OK;
}
