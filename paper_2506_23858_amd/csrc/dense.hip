// vmoba_key_ranges, vmoba_dense_fwd, vmoba_dense_bwd: arguments, workspaces and the small kernels around the products.
#include "dense_common.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace {

__global__ __launch_bounds__(256) void key_ranges_kernel(int B, int Sq, int Sk, const int* __restrict__ doc_off, long long doc_stride, int n_docs,
                                                         const int* __restrict__ prefix, long long prefix_stride, int causal,
                                                         const int* __restrict__ q_pos, long long q_first, int* __restrict__ lo, int* __restrict__ hi) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)B * Sq) return;
    const int b = (int)(i / Sq), r = (int)(i - (long long)b * Sq);
    const long long p = q_pos ? q_pos[i] : q_first + r;
    long long first = 0, end = Sk;
    int d = 0;
    if (doc_off) {                                           // the last document that begins at or before p
        const int* off = doc_off + b * doc_stride;
        int a = -1, z = n_docs;
        while (z - a > 1) {
            const int mid = (a + z) >> 1;
            if (off[mid] <= p) a = mid; else z = mid;
        }
        d = a;
        first = a < 0 ? 0 : off[a];
        end = a < 0 ? 0 : off[a + 1];
        if (p < first || p >= end) first = end = 0;          // between or outside the documents
    }
    if (causal && first < end) {
        const long long seen = prefix ? first + prefix[b * prefix_stride + d] : first;
        end = min(end, max(p + 1, seen));
    }
    first = min(max(first, 0LL), (long long)Sk);
    end = min(max(end, first), (long long)Sk);
    const bool none = first >= end;
    lo[i] = none ? 0 : (int)first;
    hi[i] = none ? 0 : (int)end;
}

// Joins the splits of a forward call: rows and log-sum-exps (base 2) of every split, whose weights are 2^(lse - max).
template <class T, int D>
__global__ __launch_bounds__(256) void dense_merge_kernel(DenseArgs a) {
    constexpr int LPR = D / 4;
    const long long n = (long long)a.B * a.Hkv * a.M, i = ((long long)blockIdx.x * 256 + threadIdx.x) / LPR;
    const int part = threadIdx.x % LPR;
    if (i >= n) return;
    float top = -INFINITY;
    for (int s = 0; s < a.splits; ++s) {
        const float l = a.part_lse[s * n + i];
        top = l > top || l != l ? l : top;                   // (a NaN stays)
    }
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    if (top != -INFINITY)
        for (int s = 0; s < a.splits; ++s) {
            const float w = exp2_raw(a.part_lse[s * n + i] - top);
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a.part_o + (s * n + i) * D + part * 4);
            if (w == 0.f) continue;                          // a split without keys of this row
            sum += w;
            acc += x * w;
        }
    const float inv = top == -INFINITY ? 0.f : 1.f / sum;
    const int bh = (int)(i / a.M), m = (int)(i - (long long)bh * a.M), b = bh / a.Hkv, hk = bh - b * a.Hkv, q = m / a.G, h = hk * a.G + (m - q * a.G);
    char* dst = const_cast<char*>(row_ptr(a.O, b, q, h, sizeof(T)));
    if constexpr (sizeof(T) == 2) {
        const u32x2_t v = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
        *reinterpret_cast<u32x2_t*>(dst + part * 8) = v;
    } else {
        *reinterpret_cast<f32x4_t*>(dst + part * 16) = acc * inv;
    }
    if (part == 0) a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = top == -INFINITY ? -INFINITY : (top + log2f(sum)) * DENSE_LN2;
}

// What the backward kernels read of every packed row, 32 rows per workgroup, 8 lanes a row.
template <class T, int D>
__global__ __launch_bounds__(256) void dense_rows_kernel(DenseArgs a) {
    constexpr int CPL = D / 8, VEC = 16 / sizeof(T);
    __shared__ int4 bounds[32];
    const int n_chunks = (a.M + 31) / 32, bh = blockIdx.x / n_chunks, c = blockIdx.x - bh * n_chunks, b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int r = threadIdx.x >> 3, part = threadIdx.x & 7, m = c * 32 + r, mc = min(m, a.M - 1), q = mc / a.G, h = hk * a.G + (mc - q * a.G);
    const char *o = row_ptr(a.O, b, q, h, sizeof(T)) + part * CPL * sizeof(T), *g = row_ptr(a.dO, b, q, h, sizeof(T)) + part * CPL * sizeof(T);
    float d = 0.f;
#pragma unroll
    for (int i = 0; i < CPL / VEC; ++i) {
        struct alignas(16) Vec { T v[VEC]; };
        const Vec x = *reinterpret_cast<const Vec*>(o + i * 16), y = *reinterpret_cast<const Vec*>(g + i * 16);
#pragma unroll
        for (int j = 0; j < VEC; ++j) d = fmaf((float)x.v[j], (float)y.v[j], d);
    }
    d += __shfl_xor(d, 4, 64);
    d += __shfl_xor(d, 2, 64);
    d += __shfl_xor(d, 1, 64);
    RowInfo* info = reinterpret_cast<RowInfo*>(a.row_info) + blockIdx.x;
    if (part == 0) {
        int2 k = dense_range(a, b, q);
        float lse2 = a.LSE[((long long)b * a.Hq + h) * a.Sq + q] * DENSE_LOG2E;
        if (m >= a.M) k = make_int2(0, 0);
        if (k.x >= k.y || lse2 == -INFINITY) lse2 = INFINITY;
        info->lse2[r] = lse2;
        info->ndelta[r] = m < a.M ? -d : 0.f;
        info->lo[r] = k.x;
        info->hi[r] = k.y;
        info->slope2[r] = a.slopes ? a.slopes[h] * DENSE_LOG2E : 0.f;
        info->pos[r] = dense_position(a, b, q);
        const bool some = k.x < k.y;
        bounds[r] = some ? make_int4(k.x, k.y, k.x, k.y) : make_int4(INT32_MAX, 0, INT32_MAX, 0);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int4 t = bounds[0];
        for (int i = 1; i < 32; ++i) {
            const int4 x = bounds[i];
            t = make_int4(min(t.x, x.x), max(t.y, x.y), max(t.z, x.z), min(t.w, x.w));
        }
        a.row_bounds[blockIdx.x] = t;
    }
}

// Key splits of a forward call: as many workgroups as run at a time (two per compute unit), at least 128 keys each.  One query
// of 16 heads on 4 key heads, 8 sequences of 32 760 keys: 32 tiles on 512 places.
int splits_for(int64_t tiles, int64_t Sk) {
    const int64_t places = 512, by_places = places / std::max<int64_t>(tiles, 1), by_keys = ceil_div64(Sk, 128);
    return (int)std::max<int64_t>(1, std::min(by_places, by_keys));
}

struct Sizes { int G, splits; int64_t M, fwd, bwd; };
// false: not a supported geometry
bool sizes_of(int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, Sizes& z) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv || (D != 64 && D != 128)) return false;
    z.G = Hq / Hkv;
    if (Sq >= (1 << 24) || Sk >= (1 << 24) || Sq * z.G >= (1 << 24)) return false;
    z.M = Sq * z.G;
    const int rows = z.M <= DENSE_FEW_ROWS ? 32 : DENSE_TILE_ROWS;
    const int64_t tiles = (int64_t)B * Hkv * ceil_div64(z.M, rows);
    if (tiles > (1 << 22) || (int64_t)B * Hkv * ceil_div64(Sk, 128) > (1 << 24) || (int64_t)B * Hkv * ceil_div64(z.M, 32) > (1 << 26)) return false;
    z.splits = splits_for(tiles, Sk);
    z.fwd = z.splits > 1 ? (int64_t)align_up((size_t)z.splits * B * Hkv * z.M * 4, 256) + (int64_t)z.splits * B * Hkv * z.M * D * 4 : 0;
    z.bwd = (int64_t)B * Hkv * ceil_div64(z.M, 32) * (int64_t)(sizeof(RowInfo) + sizeof(int4));
    return true;
}

bool reach_ok(const vmoba_tensor* t, int64_t S) {      // rows by 24-bit numbers and strides, 32-bit offsets
    const int es = dtype_size(t->dtype);
    return t->stride_s >= 0 && t->stride_s * es < (1 << 23) && (uint64_t)S * (uint64_t)t->stride_s * es < ((uint64_t)1 << 32);
}

// Arguments both directions share; fills what the kernels read of them.
int check(int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, const vmoba_tensor* Q, const vmoba_tensor* K, const vmoba_tensor* V,
          const vmoba_scores* how, const vmoba_tensor* O, const float* LSE, Sizes& z, DenseArgs& a) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv || !how || !LSE) return VMOBA_ERR_INVALID_ARG;
    if (!tensor_ok(Q) || !tensor_ok(K) || !tensor_ok(V) || !tensor_ok(O)) return VMOBA_ERR_INVALID_ARG;
    if (!std::isfinite(how->softmax_scale) || !std::isfinite(how->cap) || how->cap < 0.f) return VMOBA_ERR_INVALID_ARG;
    if ((how->key_lo != nullptr) != (how->key_hi != nullptr)) return VMOBA_ERR_INVALID_ARG;
    if (how->q_first < INT32_MIN || how->q_first + Sq > INT32_MAX) return VMOBA_ERR_INVALID_ARG;
    if (K->dtype != Q->dtype || V->dtype != Q->dtype || O->dtype != Q->dtype) return VMOBA_ERR_UNSUPPORTED;
    if (!sizes_of(B, Hq, Hkv, Sq, Sk, D, z)) return VMOBA_ERR_UNSUPPORTED;
    if (!reach_ok(K, Sk) || !reach_ok(V, Sk)) return VMOBA_ERR_UNSUPPORTED;
    a.Q = make_view(Q);
    a.K = make_view(K);
    a.V = make_view(V);
    a.O = make_view(O);
    a.slopes = how->slopes;
    a.key_lo = how->key_lo;
    a.key_hi = how->key_hi;
    a.q_pos = how->q_pos;
    a.q_first = how->q_first;
    a.LSE = const_cast<float*>(LSE);
    a.B = B;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = z.G;
    a.Sq = (int)Sq;
    a.Sk = (int)Sk;
    a.M = (int)z.M;
    a.splits = 1;
    const float magnitude = std::fabs(how->softmax_scale);
    a.scale = how->softmax_scale;
    a.scale_log2 = std::max(magnitude * DENSE_LOG2E, FLT_MIN);
    a.negate = how->softmax_scale < 0.f ? 0x80008000u : 0u;
    if (how->cap > 0.f) {
        a.cap2 = how->cap * DENSE_LOG2E;
        a.cap_in = 2.f * a.scale_log2 / how->cap;
        a.cap_arg = magnitude / how->cap;
    }
    return VMOBA_OK;
}

}  // namespace

extern "C" size_t vmoba_dense_workspace_bytes(int op, int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, int dtype) {
    Sizes z;
    if ((dtype != VMOBA_F32 && dtype != VMOBA_BF16) || !sizes_of(B, Hq, Hkv, Sq, Sk, D, z)) return 0;
    const int64_t n = op == VMOBA_OP_ATTN_FWD ? z.fwd : op == VMOBA_OP_ATTN_BWD ? z.bwd : 0;
    return op == VMOBA_OP_ATTN_FWD || op == VMOBA_OP_ATTN_BWD ? align_up((size_t)std::max<int64_t>(n, 256), 256) : 0;
}

extern "C" int vmoba_key_ranges(int B, int64_t Sq, int64_t Sk, const int32_t* doc_off, int64_t doc_stride_b, int32_t n_docs, const int32_t* prefix,
                                int64_t prefix_stride_b, int causal, const int32_t* q_pos, int64_t q_first, int32_t* lo, int32_t* hi, void* stream) {
    if (B <= 0 || Sq <= 0 || Sk <= 0 || !lo || !hi || lo == hi || (causal != 0 && causal != 1)) return VMOBA_ERR_INVALID_ARG;
    if (n_docs < 1 || (!doc_off && n_docs != 1) || doc_stride_b < 0 || prefix_stride_b < 0 || (prefix && !causal)) return VMOBA_ERR_INVALID_ARG;
    if (Sq > INT32_MAX || Sk > INT32_MAX || (int64_t)B * Sq > ((int64_t)1 << 38)) return VMOBA_ERR_UNSUPPORTED;
    if (q_first < INT32_MIN || q_first > INT32_MAX) return VMOBA_ERR_INVALID_ARG;
    key_ranges_kernel<<<dim3((unsigned)ceil_div64((int64_t)B * Sq, 256)), dim3(256), 0, (hipStream_t)stream>>>(
        B, (int)Sq, (int)Sk, doc_off, doc_stride_b, n_docs, prefix, prefix_stride_b, causal, q_pos, q_first, lo, hi);
    VMOBA_CHECK_LAUNCH();
    return VMOBA_OK;
}

extern "C" int vmoba_dense_fwd(int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, const vmoba_tensor* Q, const vmoba_tensor* K,
                               const vmoba_tensor* V, const vmoba_scores* how, const vmoba_tensor* O, float* LSE, void* workspace,
                               size_t workspace_bytes, void* stream) {
    Sizes z;
    DenseArgs a{};
    if (const int rc = check(B, Hq, Hkv, Sq, Sk, D, Q, K, V, how, O, LSE, z, a)) return rc;
    if (!workspace || (uintptr_t)workspace & 255) return VMOBA_ERR_INVALID_ARG;
    if (workspace_bytes < vmoba_dense_workspace_bytes(VMOBA_OP_ATTN_FWD, B, Hq, Hkv, Sq, Sk, D, Q->dtype)) return VMOBA_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const bool bf16 = Q->dtype == VMOBA_BF16, cap = how->cap > 0.f;
    a.splits = z.splits;
    a.part_lse = (float*)workspace;
    a.part_o = (float*)((char*)workspace + align_up((size_t)z.splits * B * Hkv * z.M * 4, 256));
    if (bf16) launch_dense_fwd_bf16(D, cap, st, a);
    else launch_dense_fwd_f32(D, cap, st, a);
    VMOBA_CHECK_LAUNCH();
    if (a.splits > 1) {
        const dim3 grid((unsigned)ceil_div64((int64_t)B * Hkv * z.M * (D / 4), 256));
        if (bf16 && D == 128) dense_merge_kernel<__bf16, 128><<<grid, dim3(256), 0, st>>>(a);
        else if (bf16) dense_merge_kernel<__bf16, 64><<<grid, dim3(256), 0, st>>>(a);
        else if (D == 128) dense_merge_kernel<float, 128><<<grid, dim3(256), 0, st>>>(a);
        else dense_merge_kernel<float, 64><<<grid, dim3(256), 0, st>>>(a);
        VMOBA_CHECK_LAUNCH();
    }
    return VMOBA_OK;
}

extern "C" int vmoba_dense_bwd(int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, const vmoba_tensor* Q, const vmoba_tensor* K,
                               const vmoba_tensor* V, const vmoba_scores* how, const vmoba_tensor* O, const float* LSE, const vmoba_tensor* dO,
                               const vmoba_tensor* dQ, const vmoba_tensor* dK, const vmoba_tensor* dV, void* workspace, size_t workspace_bytes,
                               void* stream) {
    Sizes z;
    DenseArgs a{};
    if (const int rc = check(B, Hq, Hkv, Sq, Sk, D, Q, K, V, how, O, LSE, z, a)) return rc;
    if (!tensor_ok(dO) || !tensor_ok(dQ) || !tensor_ok(dK) || !tensor_ok(dV) || !workspace || (uintptr_t)workspace & 255) return VMOBA_ERR_INVALID_ARG;
    if (dO->dtype != Q->dtype || dQ->dtype != Q->dtype || dK->dtype != Q->dtype || dV->dtype != Q->dtype) return VMOBA_ERR_UNSUPPORTED;
    if (workspace_bytes < vmoba_dense_workspace_bytes(VMOBA_OP_ATTN_BWD, B, Hq, Hkv, Sq, Sk, D, Q->dtype)) return VMOBA_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const bool bf16 = Q->dtype == VMOBA_BF16, cap = how->cap > 0.f;
    a.dO = make_view(dO);
    a.dQ = make_view(dQ);
    a.dK = make_view(dK);
    a.dV = make_view(dV);
    const int64_t chunks = (int64_t)B * Hkv * ceil_div64(z.M, 32);
    a.row_info = (char*)workspace;
    a.row_bounds = (int4*)((char*)workspace + chunks * (int64_t)sizeof(RowInfo));
    const dim3 grid((unsigned)chunks);
    if (bf16 && D == 128) dense_rows_kernel<__bf16, 128><<<grid, dim3(256), 0, st>>>(a);
    else if (bf16) dense_rows_kernel<__bf16, 64><<<grid, dim3(256), 0, st>>>(a);
    else if (D == 128) dense_rows_kernel<float, 128><<<grid, dim3(256), 0, st>>>(a);
    else dense_rows_kernel<float, 64><<<grid, dim3(256), 0, st>>>(a);
    VMOBA_CHECK_LAUNCH();
    if (bf16) launch_dense_bwd_bf16(D, cap, st, a);
    else launch_dense_bwd_f32(D, cap, st, a);
    VMOBA_CHECK_LAUNCH();
    return VMOBA_OK;
}
