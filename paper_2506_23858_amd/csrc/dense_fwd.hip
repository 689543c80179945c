// Forward kernel of dense attention, bfloat16: one pass over a tile's keys with a running maximum and sum.
//
// A workgroup of NW wavefronts owns 32 * NW packed rows and walks the keys that any of them reads in groups of 32.  Products are
// transposed, so that a row is a column of the matrix instruction (lane % 16):
//   S^T[key, row] = K[key, :] . Q[row, :]       A = K rows from LDS, B = Q^T in registers
//   O^T[d, row]  += V^T[d, key] . P^T[key, row] A = V^T by transpose reads, B = P^T packed from S^T's accumulators
// on v_mfma_f32_16x16x32_bf16 (see RowTile16).  Step n of a wavefront issues, unit by unit,
//     S^T(n+1) (matrix)      P(n) from S^T(n) (vector)      O^T += V(n-1)^T . P(n-1)^T (matrix)
// with the LDS operands of a unit fetched two units ahead.  Rows of K and V go straight from global memory to rings of four groups each;
// step n requests K(n+4) and V(n+2) into the places of K(n) and V(n-2), which were last read in step n-1, after a wait for what was
// requested two steps before and a barrier.
//
// The running maximum is raised only when a score passes it by 2^8 (weights stay below 2^8), so a step mostly compares and does not rescale.
// Weights are rounded to bfloat16 for the second product (relative error 2^-9 each, as the inputs'); their sum is that of the float32 values.
//
// Masks.  A row reads keys lo .. hi - 1.  A group that all of the wavefront's rows read whole takes no test.  In the others scores outside the range
// are replaced by -inf, and values that are not finite by 0 -- weight 0 times infinity is no number --; if there were any, the rows
// that do read them get weight times value added at the end (`repair`).
//
// NW = 4: 128 rows, two workgroups per compute unit.  NW = 1: up to 32 rows (single queries), where the keys' bytes are what counts.  With
// few tiles the keys are split over `splits` workgroups, whose normalised rows and sums a second launch joins.
#include "dense_common.h"

#include <cfloat>
#include <cmath>

namespace {

template <int D, int NW, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * NW, NW == 1 ? 1 : 2) void dense_fwd_kernel(DenseArgs a) {
    using TL = RowTile16<D>;
    constexpr int GK = 32;                                   // keys per group
    constexpr int KSTEPS = D / 32, CT = D / 16, UNITS = CT;
    constexpr int RB = TL::RB, PPR = TL::PPR, RPI = TL::RPI, SLOT = TL::HB, NR = 4;
    constexpr int IPW = GK / RPI / NW;                       // requests per wavefront, tensor and group
    constexpr int V0 = NR * SLOT;
    constexpr int OPITCH = D * 2 + 16;
    constexpr bool RAW = !CAP && !BIAS;                      // scores stay products; scale_log2 is applied with the subtraction of the maximum
    static_assert(UNITS == 2 * KSTEPS && IPW >= 1 && IPW % TL::NPC == 0, "units, requests");
    __shared__ __align__(1024) char smem[2 * NR * SLOT + 64];
    static_assert(NW * 32 * OPITCH <= 2 * NR * SLOT, "the tile's rows on their way out");

    const int tiles = (a.M + 32 * NW - 1) / (32 * NW);
    const int item = dense_item(a.B * a.Hkv * tiles * a.splits);
    if (item < 0) return;
    const int split = item % a.splits, tile = item / a.splits % tiles, bh = item / a.splits / tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int m0 = tile * 32 * NW + wave * 32;               // the wavefront's first row
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const float scale = RAW ? a.scale_log2 : 1.f, lazy = 8.f / scale;

    // ---- the lane's two rows (m0 + l16 and m0 + 16 + l16): their keys, Q^T fragments
    int lo[2], hi[2], head[2], query[2];
    float slope2[2], pos[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int m = m0 + 16 * t + l16, mc = min(m, a.M - 1), q = mc / a.G;
        query[t] = q;
        head[t] = hk * a.G + (mc - q * a.G);
        const int2 r = dense_range(a, b, q);
        lo[t] = m < a.M ? r.x : 0;
        hi[t] = m < a.M ? r.y : 0;
        slope2[t] = 0.f;
        pos[t] = 0.f;
        if constexpr (BIAS) {
            slope2[t] = a.slopes[head[t]] * DENSE_LOG2E;
            pos[t] = (float)dense_position(a, b, q);
        }
    }
    int row_pos[2] = {0, 0};
    if constexpr (BIAS) {
        row_pos[0] = dense_position(a, b, query[0]);
        row_pos[1] = dense_position(a, b, query[1]);
    }
    // keys of the wavefront (any row) and of all its rows; a row without keys makes every group a masked one
    int any_lo = INT32_MAX, any_hi = 0, all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const bool some = lo[t] < hi[t];
        any_lo = min(any_lo, some ? lo[t] : INT32_MAX);
        any_hi = max(any_hi, some ? hi[t] : 0);
        all_lo = max(all_lo, some ? lo[t] : INT32_MAX);
        all_hi = min(all_hi, some ? hi[t] : 0);
    }
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) {
        any_lo = min(any_lo, __shfl_xor(any_lo, o, 64));
        any_hi = max(any_hi, __shfl_xor(any_hi, o, 64));
        all_lo = max(all_lo, __shfl_xor(all_lo, o, 64));
        all_hi = min(all_hi, __shfl_xor(all_hi, o, 64));
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    if constexpr (NW > 1) {
        int* w = reinterpret_cast<int*>(smem + 2 * NR * SLOT);
        if (lane == 0) {
            w[wave] = any_lo;
            w[NW + wave] = any_hi;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            any_lo = min(any_lo, w[i]);
            any_hi = max(any_hi, w[NW + i]);
        }
    }
    int k_first = __builtin_amdgcn_readfirstlane(any_lo), k_end = __builtin_amdgcn_readfirstlane(any_hi);
    if (k_first >= k_end) k_first = k_end = 0;
    if (a.splits > 1) {                                      // this split's share of the tile's groups
        const int groups = (k_end - k_first + GK - 1) / GK, per = (groups + a.splits - 1) / a.splits;
        const int s0 = min(split * per, groups), s1 = min(s0 + per, groups);
        k_end = min(k_end, k_first + s1 * GK);
        k_first += s0 * GK;
    }
    const int n_groups = (k_end - k_first + GK - 1) / GK;

    bf16x8_t qf[2][KSTEPS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const char* p = row_ptr(a.Q, b, query[t], head[t], 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + ks * 64);
            qf[t][ks] = __builtin_bit_cast(bf16x8_t, x ^ a.negate);
        }
    }

    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4_t oacc[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) oacc[ct][0] = oacc[ct][1] = zero4;
    // m: what is subtracted from base-2 scores; limit: the score that raises it.  l: this lane's share of the row's sum
    float m_run[2] = {-3e38f, -3e38f}, limit[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
    unsigned found = 0;

    if (n_groups > 0) {
        const char *kbase = row_ptr(a.K, b, 0, hk, 2), *vbase = row_ptr(a.V, b, 0, hk, 2);
        const uint32_t kss = (uint32_t)(a.K.stride_s * 2), vss = (uint32_t)(a.V.stride_s * 2);
        uint32_t pc16[TL::NPC];
#pragma unroll
        for (int i = 0; i < TL::NPC; ++i) pc16[i] = TL::request_piece(lane, i);
        const int dr = wave * IPW * RPI + lane / PPR;        // row of a group that the lane's first request asks for
        auto request = [&](int tensor, int n, uint32_t slot) {
#pragma unroll
            for (int i = 0; i < IPW; ++i) {
                const uint32_t row = (uint32_t)min(k_first + n * GK + dr + i * RPI, a.Sk - 1);
                const uint32_t l = lds0 + slot + (uint32_t)(wave * IPW + i) * 1024;
                if (tensor == 0) dma_row16<0>(kbase, row, kss, pc16[i % TL::NPC], l);
                else dma_row16<V0>(vbase, row, vss, pc16[i % TL::NPC], l);
            }
        };
        uint32_t rlane[TL::NRB], tlane[TL::NTB];
#pragma unroll
        for (int i = 0; i < TL::NRB; ++i) rlane[i] = TL::row_lane(lane, i);
#pragma unroll
        for (int i = 0; i < TL::NTB; ++i) tlane[i] = V0 + TL::tr_lane(lane, i);
        // unit u of S^T: keys 16 * (u / KSTEPS), k-step u % KSTEPS; of the second product: channel tile u
        auto readK = [&](uint32_t slot, int u) { return TL::rows(smem, rlane, slot, u / KSTEPS, u % KSTEPS); };
        auto readV = [&](uint32_t slot, int u) { return TL::transposed(smem, tlane, slot, u); };

        uint32_t r0 = 0, r1 = SLOT, r2 = 2 * SLOT, r3 = 3 * SLOT;      // ring places of groups n .. n + 3
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            request(0, n, n * SLOT);
            if (n < 2) request(1, n, n * SLOT);
        }
        VMOBA_WAIT_VMCNT(0);
        asm volatile("s_barrier" ::: "memory");
        f32x4_t sA[2][2], sB[2][2];                          // [16 keys][16 rows]: value i is key 16 * kt + 4 * g + i
        bf16x8_t pA[2], pB[2];
        bf16x8_t opK[4], opV[4];
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t) sA[u / KSTEPS][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(readK(0, u), qf[t][u % KSTEPS], u % KSTEPS == 0 ? zero4 : sA[u / KSTEPS][t], 0, 0, 0);
        opK[0] = readK(SLOT, 0);
        opK[1] = readK(SLOT, 1);
        opV[0] = opV[1] = opK[0];                            // (there is no group -1)
        bool masked_before = false;

        auto step = [&](auto first, int n, f32x4_t(&s)[2][2], f32x4_t(&s_next)[2][2], bf16x8_t(&p_new)[2], const bf16x8_t(&p_prev)[2]) __attribute__((always_inline)) {
            constexpr bool FIRST = decltype(first)::value;
            VMOBA_WAIT_VMCNT(2 * IPW);
            asm volatile("s_barrier" ::: "memory");
            const int kb = k_first + n * GK;
            const bool masked = kb < all_lo || kb + GK > all_hi || kb + GK > k_end;
            if constexpr (!RAW) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float rel = BIAS ? (float)(row_pos[t] - kb - 4 * g) : 0.f;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float r;
                            float v = dense_score<CAP>(a, s[kt][t][i], r);
                            if constexpr (BIAS) v = fmaf(-slope2[t], fabsf(rel - (float)(16 * kt + i)), v);
                            s[kt][t][i] = v;
                        }
                }
            }
            if (masked) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int first_key = lo[t] - kb - 4 * g, end = min(hi[t], k_end) - kb - 4 * g;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * kt + i < first_key || 16 * kt + i >= end) s[kt][t][i] = -INFINITY;
                }
            }
            float alpha[2] = {1.f, 1.f};
            bool raised = false;
            unsigned w[2][4];                                // P(n) as packed pairs
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int u2 = u + 2;
                const bf16x8_t nk = u2 < UNITS ? readK(r1, u2) : readK(r2, u2 - UNITS);
                const bf16x8_t nv = u2 < UNITS ? readV(r3, u2) : readV(r0, u2 - UNITS);
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    s_next[u / KSTEPS][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(opK[u & 3], qf[t][u % KSTEPS], u % KSTEPS == 0 ? zero4 : s_next[u / KSTEPS][t], 0, 0, 0);
                if constexpr (!FIRST) {
                    if (__builtin_expect(masked_before, 0)) opV[u & 3] = finite_only(opV[u & 3], found);
#pragma unroll
                    for (int t = 0; t < 2; ++t) oacc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(opV[u & 3], p_prev[t], oacc[u][t], 0, 0, 0);
                }
                if (u == 0) {
                    float mx[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        mx[t] = fmaxf(s[0][t][0], s[0][t][1]);
                        mx[t] = fmaxf(fmaxf(mx[t], s[0][t][2]), s[0][t][3]);
                        mx[t] = fmaxf(fmaxf(mx[t], s[1][t][0]), s[1][t][1]);
                        mx[t] = fmaxf(fmaxf(mx[t], s[1][t][2]), s[1][t][3]);
                    }
                    if (__builtin_expect(__builtin_amdgcn_ballot_w64(mx[0] > limit[0] || mx[1] > limit[1]) != 0, 0)) {
                        raised = true;
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            float x = mx[t];
                            x = fmaxf(x, __shfl_xor(x, 16, 64));
                            x = fmaxf(x, __shfl_xor(x, 32, 64));
                            const float m_new = x > limit[t] ? x * scale : m_run[t];
                            alpha[t] = exp2_raw(m_run[t] - m_new);
                            limit[t] = x > limit[t] ? x + lazy : limit[t];
                            m_run[t] = m_new;
                            l_run[t] *= alpha[t];
                        }
                    }
                }
                // 8 pairs of values over the other units
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (1 + j * (UNITS - 1) / 8 == u) {
                        const int t = j >> 2, kt = (j >> 1) & 1, i = (j & 1) * 2;
                        const float p0 = exp2_raw(RAW ? fmaf(s[kt][t][i], scale, -m_run[t]) : s[kt][t][i] - m_run[t]);
                        const float p1 = exp2_raw(RAW ? fmaf(s[kt][t][i + 1], scale, -m_run[t]) : s[kt][t][i + 1] - m_run[t]);
                        l_run[t] += p0 + p1;
                        w[t][j & 3] = pack_bf16x2(p0, p1);
                        asm volatile("" : "+v"(w[t][j & 3]));
                    }
                }
                if (u == 1) {
                    request(0, n + 4, r0);
                    request(1, n + 2, r2);
                }
                opK[u2 & 3] = nk;
                opV[u2 & 3] = nv;
                __builtin_amdgcn_sched_barrier(0);
            }
            if (__builtin_expect(raised, 0)) {               // the accumulators hold groups up to n - 1, relative to the old maximum
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) oacc[ct][t][i] *= alpha[t];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) p_new[t] = __builtin_bit_cast(bf16x8_t, u32x4_t{w[t][0], w[t][1], w[t][2], w[t][3]});
            masked_before = masked;
            const uint32_t r = r0;
            r0 = r1;
            r1 = r2;
            r2 = r3;
            r3 = r;
        };
        step(std::true_type{}, 0, sA, sB, pA, pB);
        int n = 1;
        for (; n + 1 < n_groups; n += 2) {
            step(std::false_type{}, n, sB, sA, pB, pA);
            step(std::false_type{}, n + 1, sA, sB, pA, pB);
        }
        if (n < n_groups) {
            step(std::false_type{}, n, sB, sA, pB, pA);
            pA[0] = pB[0];
            pA[1] = pB[1];
        }
        // the last group's second product; no request may be on its way to LDS when the tile's rows go there
        VMOBA_WAIT_VMCNT(0);
        asm volatile("s_barrier" ::: "memory");
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            bf16x8_t v = readV(r3, u);
            if (masked_before) v = finite_only(v, found);
#pragma unroll
            for (int t = 0; t < 2; ++t) oacc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pA[t], oacc[u][t], 0, 0, 0);
        }
    }

    // ---- rows out
    float lse2[2], inv[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float l = l_run[t];
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        inv[t] = l == 0.f ? 0.f : 1.f / l;                   // (a NaN stays one)
        lse2[t] = l == 0.f ? -INFINITY : m_run[t] + log2f(l);
    }
    const long long part0 = ((long long)split * a.B * a.Hkv + bh) * a.M;
    if (a.splits > 1) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int m = m0 + 16 * t + l16;
            if (m < a.M) {
                float* dst = a.part_o + (part0 + m) * D + 4 * g;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) *reinterpret_cast<f32x4_t*>(dst + 16 * ct) = oacc[ct][t] * inv[t];
                if (g == 0) a.part_lse[part0 + m] = lse2[t];
            }
        }
    } else {
        __syncthreads();                                     // everybody has read the last values
        char* mine = smem + wave * 32 * OPITCH;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                u32x2_t v;
                v.x = pack_bf16x2(oacc[ct][t][0] * inv[t], oacc[ct][t][1] * inv[t]);
                v.y = pack_bf16x2(oacc[ct][t][2] * inv[t], oacc[ct][t][3] * inv[t]);
                *reinterpret_cast<u32x2_t*>(mine + (t * 16 + l16) * OPITCH + (ct * 16 + g * 4) * 2) = v;
            }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < 32 * PPR / 64; ++k) {
            const int row = k * (64 / PPR) + lane / PPR, m = m0 + row;
            if (m < a.M) {
                const int q = m / a.G, h = hk * a.G + (m - q * a.G);
                *reinterpret_cast<u32x4_t*>(const_cast<char*>(row_ptr(a.O, b, q, h, 2)) + lane % PPR * 16) =
                    *reinterpret_cast<const u32x4_t*>(mine + row * OPITCH + lane % PPR * 16);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (g == 0 && m0 + 16 * t + l16 < a.M) a.LSE[((long long)b * a.Hq + head[t]) * a.Sq + query[t]] = lse2[t] * DENSE_LN2;
    }

    if (__builtin_expect(__builtin_amdgcn_ballot_w64(found != 0) == 0, 1)) return;
    dense_repair<__bf16, D, CAP, BIAS>(a, b, hk, m0, lane, part0, k_first, k_end, all_lo, all_hi, lo[0], lo[1], hi[0], hi[1], lse2[0], lse2[1]);
}

template <int D, int NW>
void launch_fwd(bool cap, hipStream_t st, const DenseArgs& a) {
    const int64_t items = (int64_t)a.B * a.Hkv * ceil_div64(a.M, 32 * NW) * a.splits;
    const dim3 grid(dense_grid(items)), block(64 * NW);
    if (cap && a.slopes) dense_fwd_kernel<D, NW, true, true><<<grid, block, 0, st>>>(a);
    else if (cap) dense_fwd_kernel<D, NW, true, false><<<grid, block, 0, st>>>(a);
    else if (a.slopes) dense_fwd_kernel<D, NW, false, true><<<grid, block, 0, st>>>(a);
    else dense_fwd_kernel<D, NW, false, false><<<grid, block, 0, st>>>(a);
}

}  // namespace

void launch_dense_fwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a) {
    const bool few = a.M <= DENSE_FEW_ROWS;
    if (D == 128) few ? launch_fwd<128, 1>(cap, st, a) : launch_fwd<128, 4>(cap, st, a);
    else few ? launch_fwd<64, 1>(cap, st, a) : launch_fwd<64, 4>(cap, st, a);
}
