// Dense attention, float32, for calls large enough to be bound by the matrix pipe: the decomposition of dense_f32.hip with every operand
// split into three bfloat16 terms and six products of terms for one (attn_split.hip derives why that is as good as the float32
// instruction: what is left out is below 2^-25 |a b|).  Six 32-cycle instructions do the work of eight 64-cycle ones.
//
// Inputs are split once per call into rows of planes in the workspace, packed rows in their order, so that tiles travel from global memory straight to LDS.
// Where an input holds a value that three terms do not hold (NaN, infinity, above 2^26, below 2^-100 and not 0), the splitting pass
// raises a flag, these kernels leave at once and those of dense_f32.hip, launched behind them, do the work.  So nothing here meets
// a value that is not finite, and masked pairs need no more than a weight of 0.
//
// Soft-max weights and dz are split in registers after a multiplication by 2^16 (attn_split.hip), taken back where sums are written.
//
// 8192 tokens x 8 heads x 128, float32 instruction -> these: forward 2.28 -> 1.26 ms (218 TFLOP/s of float32 work; that instruction alone holds 153), backward 8.73 ->
// 4.38 ms; 64 channels 1.33 -> 0.71 and 3.97 -> 2.30.  What bounds them: the matrix pipe, beside the splitting of weights, 6 vector instructions a value and term.
#include "dense_f32.h"
#include "split_common.h"

namespace {

struct SplitSource { TensorView x; char* dst; int rows, heads, G, planes, plane0; };      // rows per head, key heads, query heads that share one
struct SplitSources { SplitSource s[4]; };
// Rows of tensor blockIdx.y -> planes plane0 .. plane0 + 2 of its rows [B * heads][rows][planes][D]; one thread per eight channels.
// Bound by HBM: 4 bytes in, 6 out a value.
template <int D>
__global__ __launch_bounds__(256) void dense_split_kernel(SplitSources all, int B, int* __restrict__ flag) {
    constexpr int PPR = D / 8;
    const SplitSource& s = all.s[blockIdx.y];
    const unsigned id = blockIdx.x * (256 / PPR) + threadIdx.x / PPR, piece = threadIdx.x % PPR;
    if (id >= (unsigned)B * s.heads * s.rows) return;
    const unsigned bh = id / (unsigned)s.rows, r = id - bh * s.rows, b = bh / (unsigned)s.heads, hk = bh - b * s.heads;
    const unsigned q = s.G == 1 ? r : r / (unsigned)s.G, h = hk * s.G + (r - q * s.G);
    const f32x4_t* x = reinterpret_cast<const f32x4_t*>(row_ptr(s.x, (int)b, q, (int)h, 4)) + piece * 2;
    const f32x4_t v[2] = {x[0], x[1]};
    u32x4_t t[3];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = v[i >> 1][(i & 1) * 2], c = v[i >> 1][(i & 1) * 2 + 1];
        uint32_t th, tm, tl;
        split2(a, c, th, tm, tl);
        t[0][i] = th; t[1][i] = tm; t[2][i] = tl;
        bad |= outside_terms(a) || outside_terms(c);
    }
    char* d = s.dst + ((unsigned long long)id * s.planes + s.plane0) * (D * 2) + piece * 16;
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4_t*>(d + p * D * 2) = t[p];
    if (bad) *flag = 1;                                      // (any number of threads, the same value)
}
__global__ void dense_clear_flag_kernel(int* flag) { *flag = 0; }

// Forward: 4 wavefronts x 32 packed rows, 32 keys at a time.  One buffer for K and one for V: the next keys are requested as soon as S^T of these is
// complete, the next values after O^T; two workgroups per compute unit fill each other's waits.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void dense_fwd_split_kernel(DenseArgs a, SplitOperands x) {
    using ST = SplitTile<D>;
    constexpr int DT = ST::DT, IPW = ST::IPW, RB6 = 12 * D;
    __shared__ __align__(1024) char smem[2 * ST::TILE];
    __shared__ int words[8];
    if (*x.flag) return;
    const int tiles = (a.M + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int m = task.tile * 128 + wave * 32 + l32, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const int2 range = dense_range(a, b, q);
    const int lo = m < a.M ? range.x : 0, hi = m < a.M ? range.y : 0;
    const float slope2 = BIAS ? a.slopes[h] * DENSE_LOG2E : 0.f;
    const int pos = BIAS ? dense_position(a, b, q) : 0;
    const Keys keys = tile_keys<4>(lo, hi, wave, lane, words);
    int k_first = keys.any_lo, k_end = keys.any_hi;
    split_keys<32>(task.split, a.splits, k_first, k_end);
    const char* kv = x.kv + (long long)bh * a.Sk * RB6;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const uint32_t pc16 = ST::request_piece(lane);
    auto request = [&](int kb, int tensor) {
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const uint32_t row = (uint32_t)min(kb + ST::req_row(wave, i, lane), a.Sk - 1);
            dma_row16<0>(kv, row, RB6, pc16 + (uint32_t)(tensor * 3 + ST::req_plane(wave, i)) * (2 * D), lds0 + (uint32_t)(tensor * ST::TILE) + ST::req_lds(wave, i));
        }
    };
    f32x16_t acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = zeros16();
    float m_run = -3e38f, l_run = 0.f;                       // l_run: this lane half's share of the row's sum
    if (k_first < k_end) {
        bf16x8_t qf[3][ST::KSTEPS];
        load_terms<D>(x.q + ((long long)bh * a.M + mc) * (6 * D), hf, qf);
        const ST st(lane);
        request(k_first, 0);
        request(k_first, 1);
        for (int kb = k_first; kb < k_end; kb += 32) {
            VMOBA_WAIT_VMCNT(IPW);                           // the keys have landed, the values (younger) may be on their way
            __syncthreads();
            f32x16_t s = st.over_channels(smem, qf, [](int) {});
            __syncthreads();                                 // everybody is done with the keys
            const int next = kb + 32 < k_end ? kb + 32 : kb; // (after the last group: its own keys again, so that the waits count alike)
            request(next, 0);
            const float rel = BIAS ? (float)(pos - kb - hf) : 0.f;      // value v is key kb + hf + acc_row(v, 0)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float t;
                s[v] = score32<CAP>(a, s[v], scl, t);
                if constexpr (BIAS) s[v] = fmaf(-slope2, fabsf(rel - (float)acc_row(v, 0)), s[v]);
            }
            if (kb < keys.all_lo || kb + 32 > keys.all_hi || kb + 32 > k_end) {
                const int first_key = lo - kb - hf, end = min(hi, k_end) - kb - hf;
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = acc_row(v, 0) >= first_key && acc_row(v, 0) < end ? s[v] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
            const float m_new = fmaxf(m_run, swap_halves_max(mx));
            if (__builtin_amdgcn_ballot_w64(m_new > m_run)) {
                const float alpha = exp2_raw(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[dt][v] *= alpha;
                m_run = m_new;
            }
            Terms w;
            auto weights = [&](int j) __attribute__((always_inline)) {
                const float p0 = exp2_raw(s[2 * j] - m_run), p1 = exp2_raw(s[2 * j + 1] - m_run);
                l_run += p0 + p1;
                w.pair(j, p0 * LIFT, p1 * LIFT);
            };
#pragma unroll
            for (int j = 0; j < 4; ++j) weights(j);
            VMOBA_WAIT_VMCNT(IPW);                           // the values have landed
            __syncthreads();
            st.template over_rows<true>(smem + ST::TILE, w, acc, weights);
            __syncthreads();                                 // everybody is done with the values
            request(next, 1);
        }
    }
    const float l = swap_halves_sum(l_run), inv = l == 0.f ? 0.f : UNLIFT / l, lse2 = l == 0.f ? -INFINITY : m_run + log2f(l);
    const long long part0 = ((long long)task.split * a.B * a.Hkv + bh) * a.M;
    if (m < a.M) {
        if (a.splits > 1) {
            store_row<D>((char*)(a.part_o + (part0 + m) * D), acc, inv, hf);
            if (hf == 0) a.part_lse[part0 + m] = lse2;
        } else {
            store_row<D>(const_cast<char*>(row_ptr(a.O, b, q, h, 4)), acc, inv, hf);
            if (hf == 0) a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = lse2 * DENSE_LN2;
        }
    }
    VMOBA_WAIT_VMCNT(0);                                     // no request may reach LDS that belongs to another workgroup by then
}

// dQ: the terms of Q and dO take 3 * D / 2 registers: one wavefront per SIMD (D = 128), and a second buffer for the next keys and values.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void dense_dq_split_kernel(DenseArgs a, SplitOperands x) {
    using ST = SplitTile<D>;
    constexpr int DT = ST::DT, IPW = ST::IPW, RB6 = 12 * D;
    __shared__ __align__(1024) char smem[2][2 * ST::TILE];
    __shared__ int words[8];
    if (*x.flag) return;
    const int tiles = (a.M + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int m = task.tile * 128 + wave * 32 + l32, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const RowInfo& info = (reinterpret_cast<const RowInfo*>(a.row_info) + (long long)bh * ((a.M + 31) / 32))[mc >> 5];
    const int lo = m < a.M ? info.lo[mc & 31] : 0, hi = m < a.M ? info.hi[mc & 31] : 0;
    const float c2 = info.c2[mc & 31], nd = info.ndelta[mc & 31], slope2 = BIAS ? info.slope2[mc & 31] : 0.f;
    const int pos = BIAS ? info.pos[mc & 31] : 0;
    const Keys keys = tile_keys<4>(lo, hi, wave, lane, words);
    int k_first = keys.any_lo, k_end = keys.any_hi;
    split_keys<32>(task.split, a.splits, k_first, k_end);
    const char* kv = x.kv + (long long)bh * a.Sk * RB6;
    const uint32_t pc16 = ST::request_piece(lane);
    auto request = [&](int kb, int buf) {
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem[buf];
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const uint32_t row = (uint32_t)min(kb + ST::req_row(wave, i, lane), a.Sk - 1);
            const uint32_t off = pc16 + (uint32_t)ST::req_plane(wave, i) * (2 * D), l = lds + ST::req_lds(wave, i);
            dma_row16<0>(kv, row, RB6, off, l);
            dma_row16<ST::TILE>(kv, row, RB6, off + 6 * D, l);
        }
    };
    f32x16_t acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = zeros16();
    if (k_first < k_end) {
        bf16x8_t qf[3][ST::KSTEPS], dof[3][ST::KSTEPS];
        load_terms<D>(x.q + ((long long)bh * a.M + mc) * RB6, hf, qf);
        load_terms<D>(x.q + ((long long)bh * a.M + mc) * RB6 + 6 * D, hf, dof);
        const ST st(lane);
        request(k_first, 0);
        int buf = 0;
        for (int kb = k_first; kb < k_end; kb += 32, buf ^= 1) {
            VMOBA_WAIT_VMCNT(0);
            __syncthreads();                                 // this group has landed; everybody is done with the one before
            if (kb + 32 < k_end) request(kb + 32, buf ^ 1);
            if (kb >= keys.own_hi || kb + 32 <= keys.own_lo) continue;      // (no row of the wavefront reads it)
            const char *sK = smem[buf], *sV = smem[buf] + ST::TILE;
            const f32x16_t s = st.over_channels(sK, qf, [](int) {});
            const float rel = BIAS ? (float)(pos - kb - hf) : 0.f;
            float p[16];                                     // 2^16 times weight and cap's derivative
            const f32x16_t dp = st.over_channels(sV, dof, [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int v = 2 * j; v < 2 * j + 2; ++v) {
                    const float bias2 = BIAS ? slope2 * fabsf(rel - (float)acc_row(v, 0)) : 0.f;
                    float f;
                    p[v] = weight32<CAP>(a, s[v], scl, c2 - bias2, f) * LIFT * f;
                    asm volatile("" : "+v"(p[v]));
                }
            });
            if (kb < keys.all_lo || kb + 32 > keys.all_hi || kb + 32 > k_end) {
                const int first_key = lo - kb - hf, end = min(hi, k_end) - kb - hf;
#pragma unroll
                for (int v = 0; v < 16; ++v) p[v] = acc_row(v, 0) >= first_key && acc_row(v, 0) < end ? p[v] : 0.f;
            }
            Terms w;
            auto dz_pair = [&](int j) __attribute__((always_inline)) { w.pair(j, p[2 * j] * (dp[2 * j] + nd), p[2 * j + 1] * (dp[2 * j + 1] + nd)); };
#pragma unroll
            for (int j = 0; j < 4; ++j) dz_pair(j);
            st.template over_rows<true>(sK, w, acc, dz_pair);
        }
    }
    if (m < a.M)
        store_row<D>(a.splits > 1 ? (char*)(a.part_o + (((long long)task.split * a.B * a.Hkv + bh) * a.M + m) * D) : const_cast<char*>(row_ptr(a.dQ, b, q, h, 4)),
                     acc, a.scale * UNLIFT, hf);
}

// dK/dV: 128 keys own (32 per wavefront), chunks of 32 packed rows walked through two buffers: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dz.
// D = 64: two wavefronts per SIMD although 24 registers spill (2 x 2001 tokens, 16 heads on 4, causal, backward: 475 -> 446 us; 5000 x 12, causal: 868 -> 775;
// the reloads wait for the requests in flight, but requesting behind them gains nothing).
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void dense_dkv_split_kernel(DenseArgs a, SplitOperands x) {
    using ST = SplitTile<D>;
    constexpr int DT = ST::DT, IPW = ST::IPW, RB6 = 12 * D;
    __shared__ __align__(1024) char smem[2][2 * ST::TILE];   // [buffer][Q, dO]
    __shared__ __align__(1024) RowInfo infos[2];
    if (*x.flag) return;
    const int tiles = (a.Sk + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_k);
    const int tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int k0 = tile * 128, kw = k0 + wave * 32, key = kw + l32;
    const float scl = a.negate ? -a.scale_log2 : a.scale_log2;
    const int n_chunks = (a.M + 31) / 32;
    const char* info = a.row_info + (long long)bh * n_chunks * sizeof(RowInfo);
    const char* qd = x.q + (long long)bh * a.M * RB6;
    const uint32_t pc16 = ST::request_piece(lane);
    auto request = [&](int c, int buf) {
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem[buf];
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const uint32_t row = (uint32_t)min(c * 32 + ST::req_row(wave, i, lane), a.M - 1);
            const uint32_t off = pc16 + (uint32_t)ST::req_plane(wave, i) * (2 * D), l = lds + ST::req_lds(wave, i);
            dma_row16<0>(qd, row, RB6, off, l);
            dma_row16<ST::TILE>(qd, row, RB6, off + 6 * D, l);
        }
        if (wave == 0) dma16(info, (uint32_t)c * (uint32_t)sizeof(RowInfo) + lane * 16, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(char*)&infos[buf]);
    };
    f32x16_t acc[2][DT];                                     // dV^T, dK^T
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[i][dt] = zeros16();
    ChunkWalk walk(a.row_bounds + (long long)bh * n_chunks, n_chunks, k0, k0 + 128, lane, task.split, a.splits);
    int c = walk.next();
    if (c >= 0) {
        bf16x8_t kf[3][ST::KSTEPS], vf[3][ST::KSTEPS];
        const char* krow = x.kv + ((long long)bh * a.Sk + min(key, a.Sk - 1)) * RB6;
        load_terms<D>(krow, hf, kf);
        load_terms<D>(krow + 6 * D, hf, vf);
        const ST st(lane);
        request(c, 0);
        for (int buf = 0; c >= 0; buf ^= 1) {
            const int any_lo = walk.any_lo, any_hi = walk.any_hi, all_lo = walk.all_lo, all_hi = walk.all_hi;
            VMOBA_WAIT_VMCNT(0);
            __syncthreads();
            c = walk.next();
            if (c >= 0) request(c, buf ^ 1);
            if (kw >= any_hi || kw + 32 <= any_lo) continue; // (no row of the chunk reads a key of the wavefront)
            const char *tQ = smem[buf], *tdO = smem[buf] + ST::TILE;
            const RowInfo& ri = infos[buf];
            const f32x16_t s = st.template over_channels<true>(tQ, kf, [](int) {});
            const bool masked = kw < all_lo || kw + 32 > all_hi;
            float p[16], g[CAP ? 16 : 1];                    // 2^16 times the weight; that times the cap's derivative
            Terms pw, dw;
            const f32x16_t dp = st.template over_channels<true>(tdO, vf, [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int v = 2 * j; v < 2 * j + 2; ++v) {
                    const int r = acc_row(v, 0) + hf;
                    const float bias2 = BIAS ? ri.slope2[r] * fabsf((float)(ri.pos[r] - key)) : 0.f;
                    float f;
                    p[v] = weight32<CAP>(a, s[v], scl, ri.c2[r] - bias2, f) * LIFT;
                    if (masked) p[v] = key >= ri.lo[r] && key < ri.hi[r] ? p[v] : 0.f;
                    if constexpr (CAP) g[v] = p[v] * f;
                }
                pw.pair(j, p[2 * j], p[2 * j + 1]);
            });
            st.template over_rows<false>(tdO, pw, acc[0], [&](int j) __attribute__((always_inline)) {
                const int r0 = acc_row(2 * j, 0) + hf, r1 = acc_row(2 * j + 1, 0) + hf;
                dw.pair(j, (CAP ? g[2 * j] : p[2 * j]) * (dp[2 * j] + ri.ndelta[r0]), (CAP ? g[2 * j + 1] : p[2 * j + 1]) * (dp[2 * j + 1] + ri.ndelta[r1]));
            });
            st.template over_rows<false>(tQ, dw, acc[1], [](int) {});
        }
    }
    if (key < a.Sk && a.splits > 1) {                        // this split's sums, added up by dense_sum_kernel
        const long long n = (long long)a.B * a.Hkv * a.Sk;
        float* dst = a.part_o + (2 * task.split * n + (long long)bh * a.Sk + key) * D;
        store_row<D>((char*)dst, acc[1], a.scale * UNLIFT, hf);
        store_row<D>((char*)(dst + n * D), acc[0], UNLIFT, hf);
    } else if (key < a.Sk) {
        store_row<D>(const_cast<char*>(row_ptr(a.dK, b, key, hk, 4)), acc[1], a.scale * UNLIFT, hf);
        store_row<D>(const_cast<char*>(row_ptr(a.dV, b, key, hk, 4)), acc[0], UNLIFT, hf);
    }
}

template <int D>
void launch_fwd(bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 128) * a.splits, a.Hkv)), block(256);
#define LAUNCH(CAP, BIAS) dense_fwd_split_kernel<D, CAP, BIAS><<<grid, block, 0, st>>>(a, x)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}
template <int D>
void launch_dq(bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 128) * a.splits, a.Hkv)), block(256);
#define LAUNCH(CAP, BIAS) dense_dq_split_kernel<D, CAP, BIAS><<<grid, block, 0, st>>>(a, x)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}
template <int D>
void launch_dkv(bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.Sk, 128) * a.splits, a.Hkv)), block(256);
#define LAUNCH(CAP, BIAS) dense_dkv_split_kernel<D, CAP, BIAS><<<grid, block, 0, st>>>(a, x)
    BY_SCORES(LAUNCH);
#undef LAUNCH
}

}  // namespace

void launch_dense_split(int D, bool backward, hipStream_t st, const DenseArgs& a, const SplitOperands& x) {
    const int planes = backward ? 6 : 3;
    SplitSources s{};
    s.s[0] = {a.K, (char*)x.kv, a.Sk, a.Hkv, 1, 6, 0};
    s.s[1] = {a.V, (char*)x.kv, a.Sk, a.Hkv, 1, 6, 3};
    s.s[2] = {a.Q, (char*)x.q, a.M, a.Hkv, a.G, planes, 0};
    s.s[3] = {a.dO, (char*)x.q, a.M, a.Hkv, a.G, planes, 3};
    dense_clear_flag_kernel<<<dim3(1), dim3(1), 0, st>>>((int*)x.flag);
    const dim3 grid((unsigned)ceil_div64((int64_t)a.B * a.Hkv * (a.M > a.Sk ? a.M : a.Sk), 256 / (D / 8)), backward ? 4 : 3);
    if (D == 128) dense_split_kernel<128><<<grid, dim3(256), 0, st>>>(s, a.B, (int*)x.flag);
    else dense_split_kernel<64><<<grid, dim3(256), 0, st>>>(s, a.B, (int*)x.flag);
}
void launch_dense_fwd_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) { D == 128 ? launch_fwd<128>(cap, st, a, x) : launch_fwd<64>(cap, st, a, x); }
void launch_dense_dq_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) { D == 128 ? launch_dq<128>(cap, st, a, x) : launch_dq<64>(cap, st, a, x); }
void launch_dense_dkv_split(int D, bool cap, hipStream_t st, const DenseArgs& a, const SplitOperands& x) { D == 128 ? launch_dkv<128>(cap, st, a, x) : launch_dkv<64>(cap, st, a, x); }
