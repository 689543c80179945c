// vmoba_rope: rotary positions of queries and keys.
//
// Bound by HBM: every row is read once and written once.  A thread owns VEC pairs of a token (VEC = 8 bfloat16 or 4 float32 values: two accesses of 16
// bytes a row, each of which its neighbours continue) and walks heads of the call's tensors with them, so an angle's sine and cosine are
// computed once per token and head group, not once per head.  The angle in turns, position * frequency / 2 pi, is reduced to [-1/2, 1/2] in float64: the error of
// a float32 angle, position * 2^-24, would reach whole radians at positions of some millions.
// 32 760 tokens x 24 heads x 128 bfloat16: 77 us (5.2 TB/s, the rate of a large copy; with cached accesses, and angles computed before the first request, 85 to 93).
// Where pairs do not fall into whole groups of VEC (58 of 64 channels, say), rows go through LDS and pairs are turned one by one there: 29 pairs of
// 32 760 x 20 heads x 64 take 60 us so, and took 146 with accesses of 2 bytes.
#include "common.h"

#include <cmath>

namespace {

constexpr int MAX_TENSORS = 8;
struct RopeTensor { TensorView in, out; int heads; };
struct RopeArgs {
    RopeTensor t[MAX_TENSORS];
    const double* freqs;
    const int* positions;
    double first;
    long long pos_stride_b, tokens;      // tokens: B * S
    int n_tensors, total_heads, S, D, P, axes, dims0, dims01;      // P: rotated pairs; pairs below dims0 / dims01 belong to axis 0 / to axis 0 or 1
    int gh, gw;                // grid extents H and W (no positions, three axes)
    int chunks, tail_chunks;   // threads per token: groups of VEC pairs and, behind them, of twice VEC copied channels
    int heads_per_part;
    float mscale;
    int negative;
};

template <class T, int N> struct VecOf { T v[N]; };

// Position of a token along the axes, float64 (exact below 2^53).
struct TokenPosition { double t, h, w; };
__device__ __forceinline__ TokenPosition position_of(const RopeArgs& a, int b, int s) {
    if (a.positions) {
        const int* q = a.positions + b * a.pos_stride_b + (long long)s * a.axes;
        return {a.first + (double)q[0], a.axes > 1 ? (double)q[1] : 0.0, a.axes > 2 ? (double)q[2] : 0.0};
    }
    if (a.axes == 3) {
        const int hw = a.gh * a.gw, t = s / hw, r = s - t * hw, h = r / a.gw;
        return {a.first + (double)t, (double)h, (double)(r - h * a.gw)};
    }
    return {a.first + (double)s, 0.0, 0.0};
}
// Sine and cosine of pair p there, with the call's sign and factor.  The angle in turns is reduced to a quarter turn around 0 (float64, then float32: 2^-27 of
// a turn), where the Taylor polynomials of degree 9 and 10 are off by less than 2^-28.
__device__ __forceinline__ void sine_cosine(const RopeArgs& a, const TokenPosition& at, int p, float& sn, float& cs) {
    const double quarters = (p < a.dims0 ? at.t : p < a.dims01 ? at.h : at.w) * (a.freqs[p] * 0.63661977236758134308);      // 2 / pi
    const double whole = rint(quarters);
    const int k = (int)(fabs(quarters) > 1e9 ? whole - 4.0 * rint(whole * 0.25) : whole) & 3;
    const float x = (float)(quarters - whole) * 1.57079632679489661923f, y = x * x;
    const float si = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float co = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float s = k & 1 ? co : si, c = k & 1 ? si : co;                // sin(x + k pi/2), cos(x + k pi/2) up to their signs
    cs = (((k + 1) & 2) != 0 ? -c : c) * a.mscale;
    sn = (((k & 2) != 0) != (a.negative != 0) ? -s : s) * a.mscale;
}

// HALF: pairs (p, p + P), else (2p, 2p + 1).  Rotated pairs and copied channels come in whole groups of VEC.
template <class T, bool HALF>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    constexpr int VEC = 16 / sizeof(T);
    using Vec = VecOf<T, VEC>;
    const int per_token = a.chunks + a.tail_chunks;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    int c, b, s;
    if (a.tokens * per_token < (1LL << 31)) {  // (a 64-bit division is some hundred instructions)
        const unsigned token = (unsigned)id / (unsigned)per_token;
        if (token >= (unsigned)a.tokens) return;
        c = (int)((unsigned)id - token * (unsigned)per_token);
        b = (int)(token / (unsigned)a.S);
        s = (int)(token - (unsigned)b * (unsigned)a.S);
    } else {
        const long long token = id / per_token;
        if (token >= a.tokens) return;
        c = (int)(id - token * per_token);
        b = (int)(token / a.S);
        s = (int)(token - (long long)b * a.S);
    }
    const int h0 = blockIdx.y * a.heads_per_part, h1 = min(h0 + a.heads_per_part, a.total_heads);

    // (each row is touched once: non-temporal)
    auto load = [](const T* p) {
        const u32x4_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
        return __builtin_bit_cast(Vec, x);
    };
    auto store = [](T* p, const Vec& v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(p)); };
    // The thread's two pieces of a row: channels i0 and i1 onwards.  HALF: the pairs' first and second channels.  Otherwise pairs i0/2 .. and i1/2 ..
    // Threads behind the pairs copy two pieces each (the last one perhaps the same piece twice), in the same loop: as a branch of their own they would
    // make their wavefronts walk the heads twice.
    const bool copies = c >= a.chunks;
    const int k = c - a.chunks, pieces = (a.D - 2 * a.P) / VEC;
    const int i0 = copies ? 2 * a.P + k * VEC : c * VEC, i1 = copies ? 2 * a.P + min(k + a.tail_chunks, pieces - 1) * VEC : HALF ? i0 + a.P : i0 + a.chunks * VEC;
    // The first rows are on their way while sines and cosines are computed.
    constexpr int AHEAD = 4;
    auto src_of = [&](const RopeTensor& t) { return (const T*)t.in.ptr + b * t.in.stride_b + s * t.in.stride_s; };
    int i = 0, base = 0;
    while (h0 >= base + a.t[i].heads) base += a.t[i++].heads;
    int e = h0 - base, e1 = min(h1 - base, a.t[i].heads);
    Vec x0[AHEAD], y0[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        const T* src = src_of(a.t[i]) + min(e + u, e1 - 1) * a.t[i].in.stride_h;
        x0[u] = load(src + i0);
        y0[u] = load(src + i1);
    }
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) cs[j] = sn[j] = 0.f;
    if (!copies) {
        const TokenPosition at = position_of(a, b, s);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sine_cosine(a, at, HALF ? i0 + j : j < VEC / 2 ? i0 / 2 + j : i1 / 2 + j - VEC / 2, sn[j], cs[j]);
    }
    auto turn = [&](const Vec& x, const Vec& y, T* dst) {
        Vec u, v;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if constexpr (HALF) {
                const float p = (float)x.v[j], q = (float)y.v[j];
                u.v[j] = (T)(p * cs[j] - q * sn[j]);
                v.v[j] = (T)(p * sn[j] + q * cs[j]);
            } else {
                const Vec& from = j < VEC / 2 ? x : y;
                Vec& to = j < VEC / 2 ? u : v;
                const float p = (float)from.v[2 * j % VEC], q = (float)from.v[(2 * j + 1) % VEC];
                to.v[2 * j % VEC] = (T)(p * cs[j] - q * sn[j]);
                to.v[(2 * j + 1) % VEC] = (T)(p * sn[j] + q * cs[j]);
            }
        }
        store(dst + i0, copies ? x : u);
        store(dst + i1, copies ? y : v);
    };
    for (bool first = true;; first = false) {
        const RopeTensor& t = a.t[i];
        T* dst = (T*)t.out.ptr + b * t.out.stride_b + s * t.out.stride_s;
        if (first) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (e + u < e1) turn(x0[u], y0[u], dst + (e + u) * t.out.stride_h);
            e += AHEAD;
        }
        const T* src = src_of(t);
#pragma unroll 4
        for (int h = e; h < e1; ++h) turn(load(src + h * t.in.stride_h + i0), load(src + h * t.in.stride_h + i1), dst + h * t.out.stride_h);
        base += t.heads;
        if (h1 <= base) return;
        ++i;
        e = 0;
        e1 = min(h1 - base, a.t[i].heads);
    }
}

// Any number of pairs: rows of up to TOKENS tokens and `block_heads` heads go through LDS in whole pieces of 16 bytes, and pairs are turned there one by one.
constexpr int TOKENS = 8, ROW_BYTES = 16384;
template <class T, bool HALF>
__global__ __launch_bounds__(256) void rope_lds_kernel(RopeArgs a, int tokens, int block_heads) {
    constexpr int VEC = 16 / sizeof(T);
    extern __shared__ __align__(16) char smem[];
    f32x2_t* const table = reinterpret_cast<f32x2_t*>(smem);                       // [tokens][P] cosine, sine
    const int pitch = (a.D + VEC - 1) / VEC * VEC, pieces = pitch / VEC;            // of a row in LDS
    T* const buf = reinterpret_cast<T*>(smem + ((tokens * a.P * 8 + 15) & ~15));
    const long long token0 = (long long)blockIdx.x * tokens;
    const int n = (int)min((long long)tokens, a.tokens - token0), t = threadIdx.x;
    for (int i = t; i < n * a.P; i += 256) {
        const long long token = token0 + i / a.P;
        const int b = (int)(token / a.S), s = (int)(token - (long long)b * a.S);
        float sn, cs;
        sine_cosine(a, position_of(a, b, s), i % a.P, sn, cs);
        table[i] = f32x2_t{cs, sn};
    }
    const int h0 = blockIdx.y * a.heads_per_part, h1 = min(h0 + a.heads_per_part, a.total_heads);
    int base = 0;
    for (int k = 0; k < a.n_tensors; ++k) {
        const RopeTensor& x = a.t[k];
        const int e0 = max(h0 - base, 0), e1 = min(h1 - base, x.heads);
        base += x.heads;
        for (int hb = e0; hb < e1; hb += block_heads) {
            const int heads = min(block_heads, e1 - hb), rows = n * heads;          // row r: token r / heads, head hb + r % heads
            auto row = [&](const TensorView& v, int r) {
                const long long token = token0 + r / heads;
                const int b = (int)(token / a.S), s = (int)(token - (long long)b * a.S);
                return (T*)v.ptr + b * v.stride_b + s * v.stride_s + (hb + r % heads) * v.stride_h;
            };
            __syncthreads();
            for (int i = t; i < rows * pieces; i += 256) {
                const int r = i / pieces, d0 = i % pieces * VEC;
                const T* src = row(x.in, r) + d0;
                if (d0 + VEC <= a.D) *reinterpret_cast<u32x4_t*>(buf + r * pitch + d0) = *reinterpret_cast<const u32x4_t*>(src);
                else
                    for (int j = 0; d0 + j < a.D; ++j) buf[r * pitch + d0 + j] = src[j];
            }
            __syncthreads();
            for (int i = t; i < rows * a.P; i += 256) {
                const int r = i / a.P, p = i % a.P;
                T* const q = buf + r * pitch;
                const int c0 = HALF ? p : 2 * p, c1 = HALF ? p + a.P : 2 * p + 1;
                const f32x2_t cs = table[r / heads * a.P + p];
                const float u = (float)q[c0], v = (float)q[c1];
                q[c0] = (T)(u * cs.x - v * cs.y);
                q[c1] = (T)(u * cs.y + v * cs.x);
            }
            __syncthreads();
            for (int i = t; i < rows * pieces; i += 256) {
                const int r = i / pieces, d0 = i % pieces * VEC;
                T* dst = row(x.out, r) + d0;
                if (d0 + VEC <= a.D) *reinterpret_cast<u32x4_t*>(dst) = *reinterpret_cast<const u32x4_t*>(buf + r * pitch + d0);
                else
                    for (int j = 0; d0 + j < a.D; ++j) dst[j] = buf[r * pitch + d0 + j];
            }
        }
    }
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
    a.first = (double)first;
    a.tokens = (int64_t)B * S;
    a.n_tensors = n_tensors;
    a.S = (int)S;
    a.D = D;
    a.P = R / 2;
    a.axes = n_axes;
    a.dims0 = n_axes > 1 ? dims[0] / 2 : R / 2;
    a.dims01 = n_axes > 2 ? a.dims0 + dims[1] / 2 : R / 2;
    a.chunks = (int)ceil_div64(a.P, vec);
    a.tail_chunks = copies ? (int)ceil_div64(D - R, 2 * vec) : 0;
    a.mscale = mscale;
    a.negative = inverse;
    hipStream_t st = (hipStream_t)stream;
    const bool half = layout == VMOBA_ROPE_HALF;
    // The heads are dealt to more threads, down to one each, until there are `enough` workgroups.
    auto deal = [&](int64_t blocks, int64_t enough) {
        const int64_t parts = blocks >= enough ? 1 : ceil_div64(enough, blocks);
        a.heads_per_part = (int)ceil_div64(a.total_heads, parts < a.total_heads ? parts : a.total_heads);
        return dim3((unsigned)blocks, (unsigned)ceil_div64(a.total_heads, a.heads_per_part));
    };
    if (a.P % vec == 0 && (D - R) % vec == 0) {
        const int64_t blocks = ceil_div64(a.tokens * (a.chunks + a.tail_chunks), 256);
        if (blocks > INT32_MAX) return VMOBA_ERR_UNSUPPORTED;
        const dim3 g = deal(blocks, 1024);
        if (bf16 && half) rope_kernel<__bf16, true><<<g, dim3(256), 0, st>>>(a);
        else if (bf16) rope_kernel<__bf16, false><<<g, dim3(256), 0, st>>>(a);
        else if (half) rope_kernel<float, true><<<g, dim3(256), 0, st>>>(a);
        else rope_kernel<float, false><<<g, dim3(256), 0, st>>>(a);
    } else {
        const int row = (int)ceil_div64(D, vec) * 16;
        const int tokens = (int)(a.tokens < TOKENS ? a.tokens : ROW_BYTES / row < TOKENS ? ROW_BYTES / row : TOKENS);
        const int heads = ROW_BYTES / (row * tokens) < a.total_heads ? ROW_BYTES / (row * tokens) : a.total_heads;
        const int64_t blocks = ceil_div64(a.tokens, tokens);
        if (blocks > INT32_MAX) return VMOBA_ERR_UNSUPPORTED;
        const dim3 g = deal(blocks, 1024);
        const size_t lds = align_up((size_t)tokens * a.P * 8, 16) + (size_t)tokens * heads * row;
        if (bf16 && half) rope_lds_kernel<__bf16, true><<<g, dim3(256), lds, st>>>(a, tokens, heads);
        else if (bf16) rope_lds_kernel<__bf16, false><<<g, dim3(256), lds, st>>>(a, tokens, heads);
        else if (half) rope_lds_kernel<float, true><<<g, dim3(256), lds, st>>>(a, tokens, heads);
        else rope_lds_kernel<float, false><<<g, dim3(256), lds, st>>>(a, tokens, heads);
    }
    VMOBA_CHECK_LAUNCH();
    return VMOBA_OK;
}
