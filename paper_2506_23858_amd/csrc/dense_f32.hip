// Dense attention, float32, for small calls and for inputs that dense_split.hip cannot split: the same decomposition as the bfloat16 kernels on v_mfma_f32_32x32x2_f32.
//
// Operand plumbing (lane = 32 * hf + l32): A: row l32, k = hf; B: column l32, k = hf; C/D: column l32, rows 8 * i + 4 * hf + r as value
// 4 * i + r.  The order of a contraction is free, so
//   * over channels, lane half hf takes channels hf * D/2 + t at step t: both operands are runs of a row, 16 bytes at a time;
//   * over 32 keys (or rows), step 4 * i + r takes keys 8 * i + 4 * hf + r: the accumulator value itself is the B operand, and A is a
//     column of the tile, 32 consecutive floats of two rows.
// Tiles of 32 rows go through registers to LDS, requested one tile ahead, in rows padded by 16 bytes and in two buffers, so that a tile is one barrier.  One such instruction is 64 cycles of the
// matrix pipe for one LDS read of 4 or a quarter of one of 16 bytes: the pipe is what bounds these kernels.
#include "dense_f32.h"

namespace {

template <int D> constexpr int PITCH = D + 4;                // floats per tile row

// 32 rows of a tensor through registers to LDS, by NT threads.
template <int D, int NT>
struct Stage {
    static constexpr int PPR = D / 4, N = 32 * PPR / NT;
    f32x4_t x[N];
    template <class F>
    __device__ __forceinline__ void load(F row) {            // row(r): pointer to row r of the tile
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = i * NT + (int)threadIdx.x;
            x[i] = *reinterpret_cast<const f32x4_t*>(row(p / PPR) + p % PPR * 16);
        }
    }
    __device__ __forceinline__ void store(float* tile) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = i * NT + (int)threadIdx.x;
            *reinterpret_cast<f32x4_t*>(tile + p / PPR * PITCH<D> + p % PPR * 4) = x[i];
        }
    }
};
// acc += A . B over the channels: A rows l32 of an LDS tile, B the lane's fragment (channels hf * D/2 ...).
template <int D>
__device__ __forceinline__ f32x16_t over_channels(const float* tile, const float (&frag)[D / 2], f32x16_t acc, int l32, int hf) {
    const float* row = tile + l32 * PITCH<D> + hf * (D / 2);
#pragma unroll
    for (int t = 0; t < D / 2; t += 4) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(row + t);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], frag[t + j], acc, 0, 0, 0);
    }
    return acc;
}
// acc[dt] += (tile columns 32 * dt + l32)^T . p over the tile's 32 rows.  Values of the classes `special` count as 0: NOT_FINITE where a
// mask cuts the tile (their weight of 0 would make them NaNs), none elsewhere.  A test and a selection in the shadow of the matrix
// instruction: with a branch at each value instead, and one tile buffer, 8192 tokens x 8 heads x 128 channels took 2.68 ms (now 2.27)
// forward and 10.0 (8.7) backward.
constexpr int NOT_FINITE = 0x207;                            // classes of a float: NaNs, -inf, +inf
template <int D>
__device__ __forceinline__ void over_rows(const float* tile, const f32x16_t& p, f32x16_t (&acc)[D / 32], int l32, int hf, int special) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const float* row = tile + (8 * (v >> 2) + 4 * hf + (v & 3)) * PITCH<D> + l32;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const float x = row[32 * dt];
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_amdgcn_classf(x, special) ? 0.f : x, p[v], acc[dt], 0, 0, 0);
        }
    }
}
template <int D>
__device__ __forceinline__ void load_fragment(float (&f)[D / 2], const char* row, int hf) {
#pragma unroll
    for (int t = 0; t < D / 2; t += 4) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(row + (hf * (D / 2) + t) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[t + j] = x[j];
    }
}
template <int D, int NW, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * NW, 1) void dense_fwd_f32_kernel(DenseArgs a) {
    constexpr int NT = 64 * NW, TILE = 32 * PITCH<D>;
    __shared__ __align__(16) float smem[2][2 * TILE];
    __shared__ int words[2 * NW];
    if (a.run_if && !*a.run_if) return;
    const int tiles = (a.M + 32 * NW - 1) / (32 * NW);
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int split = task.split, tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int m0 = tile * 32 * NW + wave * 32, m = m0 + l32, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const int2 range = dense_range(a, b, q);
    const int lo = m < a.M ? range.x : 0, hi = m < a.M ? range.y : 0;
    const float slope2 = BIAS ? a.slopes[h] * DENSE_LOG2E : 0.f;
    const int pos = BIAS ? dense_position(a, b, q) : 0;
    const Keys keys = tile_keys<NW>(lo, hi, wave, lane, words);
    int k_first = keys.any_lo, k_end = keys.any_hi;
    split_keys<32>(split, a.splits, k_first, k_end);
    float qf[D / 2];
    load_fragment<D>(qf, row_ptr(a.Q, b, q, h, 4), hf);
    f32x16_t acc[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zeros16();
    const float none = CAP || BIAS || scl > 0.f ? -INFINITY : INFINITY;      // stands for a masked score
    float m_run = -3e38f, l_run = 0.f;
    bool found = false;                                      // values of V that over_rows took out
    const char *kbase = row_ptr(a.K, b, 0, hk, 4), *vbase = row_ptr(a.V, b, 0, hk, 4);
    const long long kss = a.K.stride_s * 4, vss = a.V.stride_s * 4;
    Stage<D, NT> sk, sv;
    auto fetch = [&](int kb) {
        sk.load([&](int r) { return kbase + min(kb + r, a.Sk - 1) * kss; });
        sv.load([&](int r) { return vbase + min(kb + r, a.Sk - 1) * vss; });
    };
    auto place = [&](int buf) {
        sk.store(smem[buf]);
        sv.store(smem[buf] + TILE);
    };
    if (k_first < k_end) {
        fetch(k_first);
        place(0);
    }
    int buf = 0;
    for (int kb = k_first; kb < k_end; kb += 32, buf ^= 1) {
        __syncthreads();
        const float* tk = smem[buf];
        if (kb + 32 < k_end) fetch(kb + 32);
        const bool masked = kb < keys.all_lo || kb + 32 > keys.all_hi || kb + 32 > k_end;
        f32x16_t s = over_channels<D>(tk, qf, zeros16(), l32, hf);
        const float rel = BIAS ? (float)(pos - kb - 4 * hf) : 0.f;
        const int first_key = lo - kb - 4 * hf, end = min(hi, k_end) - kb - 4 * hf;
        float mx = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = 8 * (v >> 2) + (v & 3);
            float t, s2 = score32<CAP>(a, s[v], scl, t);
            if constexpr (BIAS) s2 = fmaf(-slope2, fabsf(rel - (float)key), s2);
            if constexpr (CAP || BIAS) s[v] = s2;
            mx = fmaxf(mx, s2);
        }
        if (masked) {
            mx = -INFINITY;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = 8 * (v >> 2) + (v & 3);
                s[v] = key >= first_key && key < end ? s[v] : none;
                mx = fmaxf(mx, CAP || BIAS ? s[v] : s[v] * scl);
            }
            const float* half = tk + TILE + l32 * PITCH<D> + hf * (D / 2);
#pragma unroll
            for (int t = 0; t < D / 2; t += 4) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(half + t);
#pragma unroll
                for (int j = 0; j < 4; ++j) found |= __builtin_amdgcn_classf(x[j], NOT_FINITE);
            }
        }
        mx = swap_halves_max(mx);
        const float m_new = fmaxf(m_run, mx), alpha = exp2_raw(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const float p = exp2_raw(CAP || BIAS ? s[v] - m_run : fmaf(s[v], scl, -m_run));
            l_run += p;
            s[v] = p;
        }
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[dt][v] *= alpha;
        }
        over_rows<D>(tk + TILE, s, acc, l32, hf, masked ? NOT_FINITE : 0);
        if (kb + 32 < k_end) place(buf ^ 1);
    }
    const float l = swap_halves_sum(l_run), inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m_run + log2f(l);
    const long long part0 = ((long long)split * a.B * a.Hkv + bh) * a.M;
    if (m < a.M) {
        if (a.splits > 1) {
            store_row<D>((char*)(a.part_o + (part0 + m) * D), acc, inv, hf);
            if (hf == 0) a.part_lse[part0 + m] = lse2;
        } else {
            store_row<D>(const_cast<char*>(row_ptr(a.O, b, q, h, 4)), acc, inv, hf);
            if (hf == 0) a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = lse2 * DENSE_LN2;
        }
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(found) == 0, 1)) return;
    // (rows m0 + 16 + lane % 16 are lanes 16 .. 31)
    dense_repair<float, D, CAP, BIAS>(a, b, hk, m0, lane, part0, k_first, k_end, keys.all_lo, keys.all_hi, lo, __shfl(lo, 16 + (lane & 15), 64), hi,
                                      __shfl(hi, 16 + (lane & 15), 64), lse2, __shfl(lse2, 16 + (lane & 15), 64));
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void dense_dq_f32_kernel(DenseArgs a) {
    constexpr int TILE = 32 * PITCH<D>;
    __shared__ __align__(16) float smem[2][2 * TILE];
    __shared__ int words[8];
    if (a.run_if && !*a.run_if) return;
    const int tiles = (a.M + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int m = tile * 128 + wave * 32 + l32, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const RowInfo& info = (reinterpret_cast<const RowInfo*>(a.row_info) + (long long)bh * ((a.M + 31) / 32))[mc >> 5];
    const int lo = m < a.M ? info.lo[mc & 31] : 0, hi = m < a.M ? info.hi[mc & 31] : 0;
    const float c2 = info.c2[mc & 31], nd = info.ndelta[mc & 31], slope2 = BIAS ? info.slope2[mc & 31] : 0.f;
    const int pos = BIAS ? info.pos[mc & 31] : 0;
    const Keys keys = tile_keys<4>(lo, hi, wave, lane, words);
    int k_first = keys.any_lo, k_end = keys.any_hi;
    split_keys<32>(task.split, a.splits, k_first, k_end);
    float qf[D / 2], dof[D / 2];
    load_fragment<D>(qf, row_ptr(a.Q, b, q, h, 4), hf);
    load_fragment<D>(dof, row_ptr(a.dO, b, q, h, 4), hf);
    f32x16_t acc[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zeros16();
    const char *kbase = row_ptr(a.K, b, 0, hk, 4), *vbase = row_ptr(a.V, b, 0, hk, 4);
    const long long kss = a.K.stride_s * 4, vss = a.V.stride_s * 4;
    Stage<D, 256> sk, sv;
    auto fetch = [&](int kb) {
        sk.load([&](int r) { return kbase + min(kb + r, a.Sk - 1) * kss; });
        sv.load([&](int r) { return vbase + min(kb + r, a.Sk - 1) * vss; });
    };
    auto place = [&](int buf) {
        sk.store(smem[buf]);
        sv.store(smem[buf] + TILE);
    };
    if (k_first < k_end) {
        fetch(k_first);
        place(0);
    }
    int buf = 0;
    for (int kb = k_first; kb < k_end; kb += 32, buf ^= 1) {
        __syncthreads();
        const float* tk = smem[buf];
        if (kb + 32 < k_end) fetch(kb + 32);
        const bool masked = kb < keys.all_lo || kb + 32 > keys.all_hi || kb + 32 > k_end;
        f32x16_t s = over_channels<D>(tk, qf, zeros16(), l32, hf), dp;
#pragma unroll
        for (int v = 0; v < 16; ++v) dp[v] = nd;
        dp = over_channels<D>(tk + TILE, dof, dp, l32, hf);
        const float rel = BIAS ? (float)(pos - kb - 4 * hf) : 0.f;
        const int first_key = lo - kb - 4 * hf, end = min(hi, k_end) - kb - 4 * hf;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = 8 * (v >> 2) + (v & 3);
            float f;
            const float p = weight32<CAP>(a, s[v], scl, BIAS ? c2 - slope2 * fabsf(rel - (float)key) : c2, f);
            s[v] = p * dp[v] * f;
        }
        if (masked) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = 8 * (v >> 2) + (v & 3);
                s[v] = key >= first_key && key < end ? s[v] : 0.f;
            }
        }
        over_rows<D>(tk, s, acc, l32, hf, masked ? NOT_FINITE : 0);
        if (kb + 32 < k_end) place(buf ^ 1);
    }
    if (m < a.M)
        store_row<D>(a.splits > 1 ? (char*)(a.part_o + (((long long)task.split * a.B * a.Hkv + bh) * a.M + m) * D) : const_cast<char*>(row_ptr(a.dQ, b, q, h, 4)),
                     acc, a.scale, hf);
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void dense_dkv_f32_kernel(DenseArgs a) {
    constexpr int TILE = 32 * PITCH<D>;
    __shared__ __align__(16) float smem[2][2 * TILE];
    __shared__ RowInfo infos[2];
    if (a.run_if && !*a.run_if) return;
    const int tiles = (a.Sk + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_k);
    const int tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int k0 = tile * 128, kw = k0 + wave * 32, key = kw + l32;
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const int n_chunks = (a.M + 31) / 32;
    const RowInfo* info = reinterpret_cast<const RowInfo*>(a.row_info) + (long long)bh * n_chunks;
    const int4* bounds = a.row_bounds + (long long)bh * n_chunks;
    float kf[D / 2], vf[D / 2];
    load_fragment<D>(kf, row_ptr(a.K, b, min(key, a.Sk - 1), hk, 4), hf);
    load_fragment<D>(vf, row_ptr(a.V, b, min(key, a.Sk - 1), hk, 4), hf);
    f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dk[dt] = dv[dt] = zeros16();
    Stage<D, 256> sq, so;
    uint32_t si = 0;                                         // the thread's word of the row information
    ChunkWalk walk(bounds, n_chunks, k0, k0 + 128, lane, task.split, a.splits);
    auto fetch = [&](int c) {
        auto row = [&](const TensorView& t) {
            return [&, c](int r) {
                const int m = min(c * 32 + r, a.M - 1), q = query_of(a, m);
                return row_ptr(t, b, q, hk * a.G + (m - q * a.G), 4);
            };
        };
        sq.load(row(a.Q));
        so.load(row(a.dO));
        si = reinterpret_cast<const uint32_t*>(info + c)[tid];
    };
    auto place = [&](int buf) {
        sq.store(smem[buf]);
        so.store(smem[buf] + TILE);
        reinterpret_cast<uint32_t*>(&infos[buf])[tid] = si;
    };
    int c = walk.next();
    if (c >= 0) {
        fetch(c);
        place(0);
    }
    for (int buf = 0; c >= 0; buf ^= 1) {
        const int all_lo = walk.all_lo, all_hi = walk.all_hi;
        __syncthreads();
        const float* tq = smem[buf];
        const RowInfo& ri = infos[buf];
        c = walk.next();
        if (c >= 0) fetch(c);
        const bool masked = kw < all_lo || kw + 32 > all_hi;
        f32x16_t s = over_channels<D>(tq, kf, zeros16(), l32, hf), dp;
#pragma unroll
        for (int v = 0; v < 16; ++v) dp[v] = ri.ndelta[8 * (v >> 2) + 4 * hf + (v & 3)];
        dp = over_channels<D>(tq + TILE, vf, dp, l32, hf);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int r = 8 * (v >> 2) + 4 * hf + (v & 3);
            float f;
            s[v] = weight32<CAP>(a, s[v], scl, BIAS ? ri.c2[r] - ri.slope2[r] * fabsf((float)(ri.pos[r] - key)) : ri.c2[r], f);
            dp[v] *= s[v] * f;
        }
        if (masked) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = 8 * (v >> 2) + 4 * hf + (v & 3);
                const bool reads = key >= ri.lo[r] && key < ri.hi[r];
                s[v] = reads ? s[v] : 0.f;
                dp[v] = reads ? dp[v] : 0.f;
            }
        }
        over_rows<D>(tq + TILE, s, dv, l32, hf, masked ? NOT_FINITE : 0);
        over_rows<D>(tq, dp, dk, l32, hf, masked ? NOT_FINITE : 0);
        if (c >= 0) place(buf ^ 1);
    }
    if (key < a.Sk && a.splits > 1) {                        // this split's sums, added up by dense_sum_kernel
        const long long n = (long long)a.B * a.Hkv * a.Sk;
        float* dst = a.part_o + (2 * task.split * n + (long long)bh * a.Sk + key) * D;
        store_row<D>((char*)dst, dk, a.scale, hf);
        store_row<D>((char*)(dst + n * D), dv, 1.f, hf);
    } else if (key < a.Sk) {
        store_row<D>(const_cast<char*>(row_ptr(a.dK, b, key, hk, 4)), dk, a.scale, hf);
        store_row<D>(const_cast<char*>(row_ptr(a.dV, b, key, hk, 4)), dv, 1.f, hf);
    }
}

template <int D, int NW>
void launch_fwd(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 32 * NW) * a.splits, a.Hkv)), block(64 * NW);
#define LAUNCH(CAP, BIAS) dense_fwd_f32_kernel<D, NW, CAP, BIAS><<<grid, block, 0, st>>>(a)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}
template <int D>
void launch_dq(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 128) * a.splits, a.Hkv)), block(256);
#define LAUNCH(CAP, BIAS) dense_dq_f32_kernel<D, CAP, BIAS><<<grid, block, 0, st>>>(a)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}
template <int D>
void launch_dkv(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.Sk, 128) * a.splits, a.Hkv)), block(256);
#define LAUNCH(CAP, BIAS) dense_dkv_f32_kernel<D, CAP, BIAS><<<grid, block, 0, st>>>(a)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}

}  // namespace

void launch_dense_fwd_f32(int D, bool cap, hipStream_t st, const DenseArgs& a) {
    const bool few = a.M <= DENSE_FEW_ROWS;
    if (D == 128) few ? launch_fwd<128, 1>(cap, st, a) : launch_fwd<128, 4>(cap, st, a);
    else few ? launch_fwd<64, 1>(cap, st, a) : launch_fwd<64, 4>(cap, st, a);
}
void launch_dense_dq_f32(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_dq<128>(cap, st, a) : launch_dq<64>(cap, st, a); }
void launch_dense_dkv_f32(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_dkv<128>(cap, st, a) : launch_dkv<64>(cap, st, a); }
