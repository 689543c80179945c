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
    // one pass with a running maximum, MB splits in flight
    constexpr int MB = 16;
    float top = -INFINITY, sum = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < a.splits; s0 += MB) {
        float l[MB], before = top;
        f32x4_t x[MB];
#pragma unroll
        for (int u = 0; u < MB; ++u) {
            const long long at = min(s0 + u, a.splits - 1) * n + i;
            l[u] = s0 + u < a.splits ? a.part_lse[at] : -INFINITY;
            x[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + at * D + part * 4);
        }
#pragma unroll
        for (int u = 0; u < MB; ++u) top = l[u] > top || l[u] != l[u] ? l[u] : top;      // (a NaN stays)
        if (top == -INFINITY) continue;
        const float alpha = exp2_raw(before - top);
        sum *= alpha;
        acc *= alpha;
#pragma unroll
        for (int u = 0; u < MB; ++u) {
            const float w = exp2_raw(l[u] - top);
            if (w == 0.f) continue;                          // a split without keys of this row
            sum += w;
            acc += x[u] * w;
        }
    }
    const float inv = top == -INFINITY ? 0.f : 1.f / sum;
    const int bh = (int)(i / a.M), m = (int)(i - (long long)bh * a.M), b = bh / a.Hkv, hk = bh - b * a.Hkv, q = query_of(a, m), h = hk * a.G + (m - q * a.G);
    char* dst = const_cast<char*>(row_ptr(a.O, b, q, h, sizeof(T)));
    if constexpr (sizeof(T) == 2) {
        const u32x2_t v = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
        *reinterpret_cast<u32x2_t*>(dst + part * 8) = v;
    } else {
        *reinterpret_cast<f32x4_t*>(dst + part * 16) = acc * inv;
    }
    if (part == 0) a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = top == -INFINITY ? -INFINITY : (top + log2f(sum)) * DENSE_LN2;
}

// Joins the splits of a backward call's dQ (ROWS) or dK and dV: sums in the order of the splits.
template <class T, int D, bool ROWS>
__global__ __launch_bounds__(256) void dense_sum_kernel(DenseArgs a) {
    constexpr int LPR = D / 4;
    const long long n = (long long)a.B * a.Hkv * (ROWS ? a.M : a.Sk), all = ROWS ? n : 2 * n, i = ((long long)blockIdx.x * 256 + threadIdx.x) / LPR;
    const int part = threadIdx.x % LPR;
    if (i >= all) return;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) acc += *reinterpret_cast<const f32x4_t*>(a.part_o + (s * all + i) * D + part * 4);
    const int per = ROWS ? a.M : a.Sk;
    const long long row = i < n ? i : i - n;
    const int bh = (int)(row / per), r = (int)(row - (long long)bh * per), b = bh / a.Hkv, hk = bh - b * a.Hkv, q = ROWS ? query_of(a, r) : r;
    char* dst = const_cast<char*>(row_ptr(ROWS ? a.dQ : i < n ? a.dK : a.dV, b, q, ROWS ? hk * a.G + (r - q * a.G) : hk, sizeof(T)));
    if constexpr (sizeof(T) == 2) {
        const u32x2_t v = {pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        *reinterpret_cast<u32x2_t*>(dst + part * 8) = v;
    } else {
        *reinterpret_cast<f32x4_t*>(dst + part * 16) = acc;
    }
}

// Tiles in order of falling cost, so that the long ones do not begin when the others are done.  One workgroup for the row tiles (cost: keys between the first and the
// last that its rows read; forward: that its first, middle and last row read, an estimate that costs three look-ups) and, in a
// backward call, a second one for the key tiles (cost: chunks of 32 rows that read one of its keys).  Tiles with masks count more.  Costs are sorted into 64 classes.
struct OrderArgs { int *order_q, *cost_q, *order_k, *cost_k; int rows_per_tile; };
__global__ __launch_bounds__(1024) void dense_order_kernel(DenseArgs a, OrderArgs o) {
    __shared__ int classes[64], top;
    const bool keys = blockIdx.x == 1;
    const int tiles = keys ? (a.Sk + DENSE_TILE_ROWS - 1) / DENSE_TILE_ROWS : (a.M + o.rows_per_tile - 1) / o.rows_per_tile, n = a.B * tiles, t = threadIdx.x;
    const int n_chunks = (a.M + 31) / 32;
    __shared__ int near[8192];                               // costs of as many tiles
    int *cost = n <= 8192 ? near : keys ? o.cost_k : o.cost_q, *order = keys ? o.order_k : o.order_q;
    if (t < 64) classes[t] = 0;
    if (t == 0) top = 1;
    if (keys) {                                              // +1 where a chunk's keys begin, -1 behind their end; then running sums
        for (int i = t; i < n; i += 1024) cost[i] = 0;
        __syncthreads();
        for (int i = t; i < a.B * n_chunks; i += 1024) {
            const int b = i / n_chunks;
            const int4 r = a.row_bounds[(long long)b * a.Hkv * n_chunks + (i - b * n_chunks)];
            if (r.x >= r.y) continue;
            const int first = r.x / DENSE_TILE_ROWS, last = (r.y - 1) / DENSE_TILE_ROWS;
            auto add = [&](int from, int to) {
                atomicAdd(cost + b * tiles + from, 1);
                if (to + 1 < tiles) atomicSub(cost + b * tiles + to + 1, 1);
            };
            add(first, last);
            if (r.x % DENSE_TILE_ROWS) add(first, first);    // (a tile that is read in part counts twice: masks)
            if (r.y % DENSE_TILE_ROWS) add(last, last);
        }
        __syncthreads();
        for (int b = t >> 6; b < a.B; b += 16) {             // a wavefront per batch element
            int carry = 0;
            for (int i0 = 0; i0 < tiles; i0 += 64) {
                const int i = i0 + (t & 63);
                int x = i < tiles ? __hip_atomic_load(cost + b * tiles + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int y = __shfl_up(x, off, 64);
                    if ((t & 63) >= off) x += y;
                }
                x += carry;
                carry = __shfl(x, 63, 64);
                if (i < tiles) cost[b * tiles + i] = x;
            }
        }
    } else {
        for (int i = t; i < n; i += 1024) {
            const int b = i / tiles, m0 = (i - b * tiles) * o.rows_per_tile, m1 = min(m0 + o.rows_per_tile, a.M) - 1;
            int first = INT32_MAX, end = 0, all_first = 0, all_end = INT32_MAX;
            if (o.cost_k) {
                for (int c = m0 >> 5; c <= m1 >> 5; ++c) {
                    const int4 r = a.row_bounds[(long long)b * a.Hkv * n_chunks + c];
                    first = min(first, r.x);
                    end = max(end, r.y);
                    all_first = max(all_first, r.z);
                    all_end = min(all_end, r.w);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const int2 r = dense_range(a, b, query_of(a, k == 0 ? m0 : k == 1 ? (m0 + m1) >> 1 : m1));
                    if (r.x < r.y) {
                        first = min(first, r.x);
                        end = max(end, r.y);
                        all_first = max(all_first, r.x);
                        all_end = min(all_end, r.y);
                    }
                }
            }
            const int keys_read = max(end - first, 0);
            cost[i] = (keys_read + (first != all_first || end != all_end ? keys_read / 2 : 0)) / 32;      // (rows of several ranges: masks)
        }
    }
    __syncthreads();
    for (int i = t; i < n; i += 1024) atomicMax(&top, cost[i]);
    __syncthreads();
    auto class_of = [&](int i) { return 63 - (int)((long long)min(max(cost[i], 0), top) * 63 / top); };
    for (int i = t; i < n; i += 1024) atomicAdd(classes + class_of(i), 1);
    __syncthreads();
    if (t == 0) {
        int sum = 0;
        for (int k = 0; k < 64; ++k) {
            const int x = classes[k];
            classes[k] = sum;
            sum += x;
        }
    }
    __syncthreads();
    for (int i = t; i < n; i += 1024) order[atomicAdd(classes + class_of(i), 1)] = i;
}

// What the backward kernels read of every packed row, 32 rows per workgroup, 8 lanes a row.
template <class T, int D>
__global__ __launch_bounds__(256) void dense_rows_kernel(DenseArgs a) {
    constexpr int CPL = D / 8, VEC = 16 / sizeof(T);
    __shared__ int4 bounds[32];
    const int n_chunks = (a.M + 31) / 32, bh = blockIdx.x / n_chunks, c = blockIdx.x - bh * n_chunks, b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int r = threadIdx.x >> 3, part = threadIdx.x & 7, m = c * 32 + r, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
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
        else if (!(fabsf(d) < INFINITY)) lse2 = NAN;
        info->c2[r] = (sizeof(T) == 2 && a.cap2 > 0.f ? a.cap2 : 0.f) - lse2;
        info->ndelta[r] = m < a.M && fabsf(d) < INFINITY ? -d : 0.f;
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

// Splits of a row tile's keys and, dK/dV, of a key tile's rows: as many pieces as run at a time (two per compute unit), of at least 256 keys or rows each; float32 without
// ranges, whose keys take four times as long, and single queries (one of 16 heads on 4 key heads, 8 sequences of 32 760 keys: 32 tiles on 512 places): 128.  (bfloat16 with 128:
// 256 tokens x 12 heads 19 us, 17 with 256; 600 x 12, causal, 32 and 29; 512 x 12 alike; 512 x 2 18 and 20.)  With ranges tiles cost different amounts, and
// the longest of a few that all run at once decides: for float32 four times as many pieces (backward with split operands twice as many), unless there are so many tiles that
// their order evens them out (2 x 2001 tokens, 16 heads on 4, 64 channels, causal, on the float32 instruction, forward and backward: 1450 -> 900 us; with split operands
// forward 183 -> 149, backward 499 -> 446, 468 with four times as many).  bfloat16 keeps to one round: its groups of keys take a quarter of the time, and pieces' ends
// cost as much (1637 tokens x 12 heads, causal: 49 us, 74 with four times the pieces).
constexpr int64_t PLACES = 512, MANY_TILES = 640;
int splits_for(int64_t tiles, int64_t pieces, int64_t most) { return (int)std::max<int64_t>(1, std::min(pieces / std::max<int64_t>(tiles, 1), most)); }
// Forward, bfloat16, equal tiles of many rows: one piece per compute unit.  A second one there hides less than its rows cost on their way to the merge
// (2 x 1024 tokens, 16 heads on 4: 53 us, now 38; 700 x 12: 34 and 29; 3000 x 1: 35 and 28; 1664 x 12: 49 and 50); with ranges it
// shortens the longest piece (1664 x 12, causal: 46 us, 53 with one).
int64_t forward_places(bool ranges, bool f32) { return ranges || f32 ? PLACES : PLACES / 2; }
// More pieces of work than run at a time: their order matters.
bool order_matters(int64_t pieces) { return pieces > PLACES; }

// float32 calls with enough work -- multiply-adds of one product over all pairs, masked ones too: the host does not know the ranges -- split their operands
// (dense_split.hip).  What that costs is two launches and a pass over the inputs in either direction, and the launches of the kernels that take over where three terms
// do not hold an input.  Without / with it, forward and backward, us, 12 heads: 512 tokens x 64 (2.0e8) 24 + 87 / 29 + 74; 512 x 128 (4.0e8) 39 + 151 / 39 + 103; 700 x 64 (3.8e8)
// 40 + 131 / 39 + 101; 1024 x 128 88 + 330 / 66 + 218; 8 heads, 8192 x 128: 2278 + 8725 / 1259 + 4379.
bool use_split(int64_t BH, int64_t M, int64_t Sk, int D) {
    return M > DENSE_FEW_ROWS && (double)BH * (double)M * (double)Sk * D >= 3e8 && (uint64_t)std::max(M, Sk) * 12 * D < ((uint64_t)1 << 32) &&
           BH * std::max(M, Sk) < ((int64_t)1 << 31);
}

struct Sizes {
    int G, rows_per_tile;
    int splits, dq_splits, row_splits;         // forward and dQ: of a row tile's keys; dK/dV: of a key tile's rows
    int64_t M, q_tiles, k_tiles, chunks;       // tiles and chunks of all batch elements and key heads
    size_t part_lse, part_o, order, fwd;       // forward workspace: offsets, bytes
    size_t info, bounds, order_b, part_b, bwd; // backward
    bool split;                                // operands of float32 calls are split: planes of Q (and dO), of K and V, and the flag
    size_t flag, split_q, split_kv, flag_b, split_qd, split_kv_b;
};
// false: not a supported geometry
bool sizes_of(int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, bool ranges, bool f32, Sizes& z) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv || (D != 64 && D != 128)) return false;
    z.G = Hq / Hkv;
    if (Sq >= (1 << 24) || Sk >= (1 << 24) || Sq * z.G >= (1 << 24)) return false;
    z.M = Sq * z.G;
    z.rows_per_tile = z.M <= 16 ? 16 : z.M <= DENSE_FEW_ROWS ? DENSE_FEW_ROWS : DENSE_TILE_ROWS;
    const int64_t BH = (int64_t)B * Hkv;
    z.q_tiles = BH * ceil_div64(z.M, z.rows_per_tile);
    z.k_tiles = BH * ceil_div64(Sk, DENSE_TILE_ROWS);
    z.chunks = BH * ceil_div64(z.M, 32);
    if (z.q_tiles > (1 << 22) || z.k_tiles > (1 << 22) || z.chunks > (1 << 24)) return false;
    const bool few = z.M <= DENSE_FEW_ROWS;    // (single queries: bytes are what counts, and a piece's share of them is even enough)
    z.split = f32 && use_split(BH, z.M, Sk, D);
    const bool uneven = ranges && f32;
    auto pieces = [&](int64_t tiles, int64_t equal, int64_t unequal) { return uneven && tiles <= MANY_TILES ? unequal : equal; };
    const int64_t least = f32 && !ranges ? 128 : 256;
    const int64_t dq_tiles = BH * ceil_div64(z.M, DENSE_TILE_ROWS), backward = (z.split ? 2 : 4) * PLACES;
    z.splits = few ? splits_for(z.q_tiles, PLACES, ceil_div64(Sk, 128))
                   : splits_for(z.q_tiles, pieces(z.q_tiles, forward_places(ranges, f32), 4 * PLACES), ceil_div64(Sk, least));
    z.dq_splits = splits_for(dq_tiles, pieces(dq_tiles, PLACES, backward), ceil_div64(Sk, least));
    z.row_splits = splits_for(z.k_tiles, pieces(z.k_tiles, PLACES, backward), z.M / 256);
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        const size_t at = off;
        off += align_up((size_t)bytes, 256);
        return at;
    };
    z.part_lse = take(z.splits > 1 ? z.splits * BH * z.M * 4 : 0);
    z.part_o = take(z.splits > 1 ? z.splits * BH * z.M * D * 4 : 0);
    z.order = take(order_matters(z.q_tiles * z.splits) ? 2 * (z.q_tiles / Hkv) * 4 : 0);
    z.flag = take(z.split ? 4 : 0);
    z.split_q = take(z.split ? BH * z.M * 6 * D : 0);
    z.split_kv = take(z.split ? BH * Sk * 12 * D : 0);
    z.fwd = std::max<size_t>(off, 256);
    off = 0;
    z.info = take(z.chunks * (int64_t)sizeof(RowInfo));
    z.bounds = take(z.chunks * (int64_t)sizeof(int4));
    z.order_b = take(2 * (B * ceil_div64(z.M, DENSE_TILE_ROWS) + z.k_tiles / Hkv) * 4);
    z.part_b = take(std::max<int64_t>(z.row_splits > 1 ? 2 * z.row_splits * BH * Sk : 0, z.dq_splits > 1 ? z.dq_splits * BH * z.M : 0) * D * 4);
    z.flag_b = take(z.split ? 4 : 0);
    z.split_qd = take(z.split ? BH * z.M * 12 * D : 0);
    z.split_kv_b = take(z.split ? BH * Sk * 12 * D : 0);
    z.bwd = off;
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
    if (how->cap > (Q->dtype == VMOBA_BF16 ? 4096.f : 1e30f)) return VMOBA_ERR_UNSUPPORTED;
    if (!sizes_of(B, Hq, Hkv, Sq, Sk, D, how->key_lo != nullptr, Q->dtype == VMOBA_F32, z)) return VMOBA_ERR_UNSUPPORTED;
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
    a.G_magic = z.G > 1 && z.G < 256 ? (unsigned)((((uint64_t)1 << 32) + z.G - 1) / z.G) : 0u;
    a.splits = 1;
    const float magnitude = std::fabs(how->softmax_scale);
    a.scale = how->softmax_scale;
    a.scale_log2 = std::max(magnitude * DENSE_LOG2E, FLT_MIN);
    a.negate = how->softmax_scale < 0.f ? 0x80008000u : 0u;
    if (how->cap > 0.f) {
        a.cap2 = how->cap * DENSE_LOG2E;
        a.cap_in = std::min(2.f * a.scale_log2 / how->cap, FLT_MAX);      // (finite, so that a score of 0 stays 0)
        a.cap_arg = std::min(magnitude / how->cap, FLT_MAX);
    }
    return VMOBA_OK;
}

}  // namespace

extern "C" size_t vmoba_dense_workspace_bytes(int op, int B, int Hq, int Hkv, int64_t Sq, int64_t Sk, int D, int dtype) {
    Sizes y, z;      // whether there are key ranges is not known here
    if ((dtype != VMOBA_F32 && dtype != VMOBA_BF16) || !sizes_of(B, Hq, Hkv, Sq, Sk, D, false, dtype == VMOBA_F32, y) ||
        !sizes_of(B, Hq, Hkv, Sq, Sk, D, true, dtype == VMOBA_F32, z))
        return 0;
    return op == VMOBA_OP_ATTN_FWD ? std::max(y.fwd, z.fwd) : op == VMOBA_OP_ATTN_BWD ? std::max(y.bwd, z.bwd) : 0;
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
    char* const ws = (char*)workspace;
    a.part_lse = (float*)(ws + z.part_lse);
    a.part_o = (float*)(ws + z.part_o);
    if (a.key_lo && order_matters(z.q_tiles * z.splits)) {
        int* order = (int*)(ws + z.order);
        dense_order_kernel<<<dim3(1), dim3(1024), 0, st>>>(a, OrderArgs{order, order + z.q_tiles / Hkv, nullptr, nullptr, z.rows_per_tile});
        VMOBA_CHECK_LAUNCH();
        a.order_q = order;
    }
    if (bf16) launch_dense_fwd_bf16(D, cap, st, a);
    else {
        if (z.split) {
            const SplitOperands x = {ws + z.split_q, ws + z.split_kv, (const int*)(ws + z.flag)};
            launch_dense_split(D, false, st, a, x);
            launch_dense_fwd_split(D, cap, st, a, x);
            VMOBA_CHECK_LAUNCH();
            a.run_if = x.flag;
        }
        launch_dense_fwd_f32(D, cap, st, a);
    }
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
    // packed rows of Q and dO by 32-bit offsets
    for (const vmoba_tensor* t : {Q, dO})
        if (!reach_ok(t, Sq) || (z.G > 1 && (t->stride_h < 0 || (uint64_t)(z.G - 1) * (uint64_t)t->stride_h * dtype_size(t->dtype) +
                                                                      (uint64_t)Sq * (uint64_t)t->stride_s * dtype_size(t->dtype) >= ((uint64_t)1 << 32))))
            return VMOBA_ERR_UNSUPPORTED;
    a.dO = make_view(dO);
    a.dQ = make_view(dQ);
    a.dK = make_view(dK);
    a.dV = make_view(dV);
    char* const ws = (char*)workspace;
    a.row_info = ws + z.info;
    a.row_bounds = (int4*)(ws + z.bounds);
    a.part_o = (float*)(ws + z.part_b);
    const dim3 grid((unsigned)z.chunks);
    if (bf16 && D == 128) dense_rows_kernel<__bf16, 128><<<grid, dim3(256), 0, st>>>(a);
    else if (bf16) dense_rows_kernel<__bf16, 64><<<grid, dim3(256), 0, st>>>(a);
    else if (D == 128) dense_rows_kernel<float, 128><<<grid, dim3(256), 0, st>>>(a);
    else dense_rows_kernel<float, 64><<<grid, dim3(256), 0, st>>>(a);
    VMOBA_CHECK_LAUNCH();
    const int64_t nq = B * ceil_div64(z.M, DENSE_TILE_ROWS), nk = z.k_tiles / Hkv;
    if (a.key_lo && order_matters(std::max(nq * z.dq_splits, nk * z.row_splits) * Hkv)) {
        int* order = (int*)(ws + z.order_b);
        dense_order_kernel<<<dim3(2), dim3(1024), 0, st>>>(a, OrderArgs{order, order + nq, order + 2 * nq, order + 2 * nq + nk, DENSE_TILE_ROWS});
        VMOBA_CHECK_LAUNCH();
        a.order_q = order;
        a.order_k = order + 2 * nq;
    }
    a.splits = z.dq_splits;
    const SplitOperands x = {ws + z.split_qd, ws + z.split_kv_b, (const int*)(ws + z.flag_b)};
    if (z.split) {
        launch_dense_split(D, true, st, a, x);
        launch_dense_dq_split(D, cap, st, a, x);
        VMOBA_CHECK_LAUNCH();
        a.run_if = x.flag;
    }
    if (bf16) launch_dense_dq_bf16(D, cap, st, a);
    else launch_dense_dq_f32(D, cap, st, a);
    VMOBA_CHECK_LAUNCH();
#define SUM(ROWS, COUNT)                                                                                             \
    do {                                                                                                             \
        const dim3 sums((unsigned)ceil_div64((COUNT) * (D / 4), 256));                                               \
        if (bf16 && D == 128) dense_sum_kernel<__bf16, 128, ROWS><<<sums, dim3(256), 0, st>>>(a);                    \
        else if (bf16) dense_sum_kernel<__bf16, 64, ROWS><<<sums, dim3(256), 0, st>>>(a);                            \
        else if (D == 128) dense_sum_kernel<float, 128, ROWS><<<sums, dim3(256), 0, st>>>(a);                        \
        else dense_sum_kernel<float, 64, ROWS><<<sums, dim3(256), 0, st>>>(a);                                       \
        VMOBA_CHECK_LAUNCH();                                                                                        \
    } while (0)
    if (a.splits > 1) SUM(true, (int64_t)B * Hkv * z.M);
    a.splits = z.row_splits;
    if (z.split) launch_dense_dkv_split(D, cap, st, a, x);
    if (bf16) launch_dense_dkv_bf16(D, cap, st, a);
    else launch_dense_dkv_f32(D, cap, st, a);
    VMOBA_CHECK_LAUNCH();
    if (a.splits > 1) SUM(false, 2 * (int64_t)B * Hkv * Sk);
#undef SUM
    return VMOBA_OK;
}
