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
    const int* run_if;             // float32 kernels: null, or a flag on the device without which they leave at once
    float *part_o, *part_lse;      // more than one split: forward [splits][B * Hkv][M][D] and [splits][B * Hkv][M] (base 2); dQ [splits][B * Hkv][M][D];
                                   // dK and dV [splits][2][B * Hkv][Sk][D]
    const int *order_q, *order_k;  // places by falling cost: [B * row tiles] and, backward, [B * key tiles]; null: as they come
    char* row_info;                // backward: ROW_INFO bytes per 32 rows, see RowInfo
    int4* row_bounds;              // backward: {lowest lo, highest hi, highest lo, lowest hi} of every 32 rows with keys
    int B, Hq, Hkv, G, Sq, Sk, M;
    int splits;                    // of a row tile's keys (forward, dQ), of a key tile's rows (dK/dV)
    float scale, scale_log2;       // softmax_scale; max(|softmax_scale| log2 e, FLT_MIN)
    float cap2, cap_in, cap_arg;   // cap log2(e); 2 scale_log2 / cap; |softmax_scale| / cap
    unsigned G_magic;              // see query_of; 0: divide
    unsigned negate;               // 0x80008000 for a negative scale (bfloat16 pairs)
};

// What the dK/dV kernel needs to know of 32 consecutive rows, one 1 KB request: arrays of 32 words.
struct RowInfo {
    float c2[32];          // -(log-sum-exp of the row, base 2), bfloat16 calls with a cap: + cap2; -inf for a row without keys (all its weights are then
                           // 0), NaN for a row whose delta is not finite (its weights are then NaN)
    float ndelta[32];      // -rowsum(dO * O), finite
    int lo[32], hi[32];    // its keys
    float slope2[32];      // slope * log2(e)
    int pos[32];           // its position
    int pad[64];
};
static_assert(sizeof(RowInfo) == 1024, "one request of 64 lanes x 16 bytes");

// Operands of a RowTile16 from one address per lane and tile: k-step ks and channel tile ct only turn bits of the piece position, and a tile lies at a multiple
// of 256 bytes, so they are an exclusive-or with lane address + tile place (twelve addresses of their own would take twelve registers).
template <int D>
struct DenseTile : RowTile16<D> {
    using Base = RowTile16<D>;
    __device__ static __forceinline__ bf16x8_t rows(const char* base, uint32_t at, int kt, int ks) {
        return *reinterpret_cast<const bf16x8_t*>(base + (at ^ (uint32_t)(ks * 64)) + kt * 16 * Base::RB);
    }
    __device__ static __forceinline__ bf16x8_t transposed(const char* base, uint32_t at, int ct) {
        const char* p = base + (at ^ (uint32_t)(ct * 32));
        const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(p + 16 * Base::RB));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};
// A value the compiler may not take out of the loop (it would keep all addresses that follow from it in registers).
__device__ __forceinline__ uint32_t pinned(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}
// m / G for a packed row m < 2^24 (magic = ceil(2^32 / G) for 1 < G < 256: the error of the product stays below 1 / G)
__device__ __forceinline__ int query_of(const DenseArgs& a, int m) {
    return a.G == 1 ? m : a.G_magic ? (int)__umulhi((unsigned)m, a.G_magic) : m / a.G;
}

// Byte offset of packed row m of Q or dO from its first one (the host has checked that 32 bits reach): q * ss + g * sh = m * sh + q * (ss - G * sh).
__device__ __forceinline__ uint32_t packed_row(const DenseArgs& a, int m, uint32_t ss, uint32_t sh) {
    return a.G == 1 ? (uint32_t)m * ss : (uint32_t)m * sh + (uint32_t)query_of(a, m) * (ss - (uint32_t)a.G * sh);
}

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
// The forward kernels' last step for a wavefront that met values of V that are not finite in groups of 32 keys where they were taken out of the product: those not
// inside all_lo .. all_hi.  The rows that do read such a key get weight times value added.  A rare path, one key at a time.  lo_a, hi_a, lse_a
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
                const int q = query_of(a, m), h = hk * a.G + (m - q * a.G);
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
// The chunks of 32 packed rows that read any key of first .. end - 1, in order (the same for all wavefronts of a workgroup).  A wavefront looks at the bounds of 64 of
// them at a time and keeps those of the chunk it returned, so that the walk's loop holds no load of its own.  Split s of several takes every splits-th chunk.
struct ChunkWalk {
    const int4* bounds;
    int n, first, end, lane, split, splits, window = -64;
    unsigned long long pending = 0;
    int4 mine;
    int any_lo, any_hi, all_lo, all_hi;      // of the chunk that next() returned: keys that any of its rows, that all of them read
    __device__ __forceinline__ ChunkWalk(const int4* b, int chunks, int k0, int k1, int l, int s, int ss)
        : bounds(b), n(chunks), first(k0), end(k1), lane(l), split(s), splits(ss) {}
    __device__ __forceinline__ int next() {
        while (pending == 0) {
            window += 64;
            if (window >= n) return -1;
            const int c = window + lane;
            mine = c < n ? bounds[c] : make_int4(INT32_MAX, 0, 0, 0);
            pending = __builtin_amdgcn_ballot_w64(mine.x < end && mine.y > first && (splits == 1 || c % splits == split));
        }
        const int i = __builtin_ctzll(pending);
        pending &= pending - 1;
        any_lo = __builtin_amdgcn_readlane(mine.x, i);
        any_hi = __builtin_amdgcn_readlane(mine.y, i);
        all_lo = __builtin_amdgcn_readlane(mine.z, i);
        all_hi = __builtin_amdgcn_readlane(mine.w, i);
        return window + i;
    }
};
// A tile in LDS loses its values that are not finite (bfloat16, `bytes` of it, by `threads` threads); whether this thread met any.
__device__ __forceinline__ bool clean_tile(char* tile, int bytes, int threads) {
    unsigned found = 0;
    for (int i = (int)threadIdx.x * 16; i < bytes; i += threads * 16) {
        bf16x8_t* p = reinterpret_cast<bf16x8_t*>(tile + i);
        *p = finite_only(*p, found);
    }
    return found != 0;
}
// Which work a workgroup does.  There are `ranks` pieces for each of `heads` key heads, the costliest first where it matters (see dense_order_kernel).  Workgroup
// ids go round the 8 XCDs and each XCD has an L2 of its own, so XCD x = id % 8 takes heads / 8 heads as a whole, rank by rank; of the rem = heads % 8 heads left
// over, rank r's go to XCDs (r rem + 0 .. rem - 1) % 8, which gives every XCD the same number in P = 8 / gcd(rem, 8) ranks.
__host__ __device__ constexpr int dense_period(int rem) { return rem == 0 ? 1 : rem & 1 ? 8 : rem & 2 ? 4 : 2; }
static inline unsigned dense_grid(int64_t ranks, int heads) {
    const int P = dense_period(heads & 7);
    return (unsigned)(8 * ceil_div64(ranks, P) * ((heads >> 3) * P + (heads & 7) * P / 8));
}
struct DensePiece { int rank, head; };      // rank -1: none
__device__ __forceinline__ DensePiece dense_piece(int ranks, int heads) {
    const int x = (int)(blockIdx.x & 7), s = (int)(blockIdx.x >> 3), full = heads >> 3, rem = heads & 7, P = dense_period(rem), C = full * P + rem * P / 8;
    int r = s / C * P, w = s % C;
    for (;; ++r) {
        const int j = (x - r * rem) & 7;             // the head left over that this XCD would take of rank r
        const int n = full + (j < rem ? 1 : 0);
        if (w < n) return r < ranks ? DensePiece{r, w < full ? x * full + w : 8 * full + j} : DensePiece{-1, 0};
        w -= n;
    }
}

// The (batch element, tile) of a rank, and its split.
struct DenseTask { int b, tile, split; };
__device__ __forceinline__ DenseTask dense_task(int rank, int splits, int tiles, const int* order) {
    const int place = rank / splits, bt = order ? order[place] : place, b = bt / tiles;
    return {b, bt - b * tiles, rank - place * splits};
}

// A split's share of keys first .. end - 1, in whole steps of STEP keys.
template <int STEP>
__device__ __forceinline__ void split_keys(int split, int splits, int& first, int& end) {
    if (splits == 1) return;
    const int steps = (end - first + STEP - 1) / STEP, per = (steps + splits - 1) / splits, s0 = min(split * per, steps), s1 = min(s0 + per, steps);
    end = min(end, first + s1 * STEP);
    first += s0 * STEP;
}

// Most rows of a tile that one wavefront takes alone, and the rows of the tile of four.
constexpr int DENSE_FEW_ROWS = 32, DENSE_TILE_ROWS = 128;

void launch_dense_fwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_fwd_f32(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_dq_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_dq_f32(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_dkv_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a);
void launch_dense_dkv_f32(int D, bool cap, hipStream_t st, const DenseArgs& a);
// The same from operands split into bfloat16 terms (dense_split.hip): rows of planes [B * Hkv][M][Q's three, backward dO's three][D] and
// [B * Hkv][Sk][K's three, V's three][D]; flag: set where three terms do not hold an input, and then the kernels leave at once.
struct SplitOperands { const char *q, *kv; const int* flag; };
void launch_dense_split(int D, bool backward, hipStream_t st, const DenseArgs& a, const SplitOperands& x);
void launch_dense_fwd_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x);
void launch_dense_dq_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x);
void launch_dense_dkv_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x);
