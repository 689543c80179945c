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
// Masks.  A row reads keys lo .. hi - 1.  A group that all of the wavefront's rows read whole takes no test; in the others scores outside the range
// are replaced by -inf.  A masked value that is not finite would still spoil its row -- weight 0 times infinity is no number --, so the group that passes the
// last key loses such values in LDS before it is multiplied, and a tile whose sums end up not finite is computed again with all groups
// cleaned so; the rows that do read such values then get weight times value added (dense_repair).  Rows without keys take part with a query of zeros; their sums are dropped.
//
// NW = 4: 128 rows, two workgroups per compute unit.  NW = 1: up to 32 rows (single queries), where the keys' bytes are what counts.  With
// few tiles the keys are split over `splits` workgroups, whose normalised rows and sums a second launch joins.
#include "dense_common.h"

#include <cfloat>
#include <cmath>

namespace {

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;      // (fmaxf makes two more instructions of it, to quiet NaNs)
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// QT: 16-row tiles of a wavefront.
template <int D, int NW, int QT, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * NW, 2) void dense_fwd_kernel(DenseArgs a) {
    using TL = RowTile16<D>;
    constexpr int GK = 32;                                   // keys per group
    constexpr int ROWS = 16 * QT;                            // rows per wavefront
    constexpr int KSTEPS = D / 32, CT = D / 16, UNITS = CT;
    constexpr int PPR = TL::PPR, RPI = TL::RPI, SLOT = TL::HB, NR = 4;
    constexpr int IPW = GK / RPI / NW;                       // requests per wavefront, tensor and group
    constexpr int V0 = NR * SLOT;
    constexpr int OPITCH = D * 2 + 16;
    static_assert(UNITS == 2 * KSTEPS && IPW >= 1 && IPW % TL::NPC == 0, "units, requests");
    __shared__ __align__(1024) char smem[2 * NR * SLOT + 32];
    static_assert(NW * ROWS * OPITCH <= 2 * NR * SLOT, "the tile's rows on their way out");

    const int tiles = (a.M + ROWS * NW - 1) / (ROWS * NW);
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int split = task.split, tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int m0 = tile * ROWS * NW + wave * ROWS;           // the wavefront's first row
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    // What is kept of a score, and the factor it has still to be multiplied by: x itself; with the cap -r (base-2 score cap2 - 2 cap2 r, the constant
    // goes to the log-sum-exp at the end); with a bias the base-2 score
    const float scale = BIAS ? 1.f : CAP ? 2.f * a.cap2 : a.scale_log2, shift = CAP && !BIAS ? a.cap2 : 0.f, lazy = 8.f / scale;

    // ---- the lane's rows (m0 + 16 t + l16): their keys, Q^T fragments
    int lo[QT], hi[QT], row_pos[QT];
    float slope2[QT];
    bf16x8_t qf[QT][KSTEPS];
    int any_lo = INT32_MAX, any_hi = 0, all_lo = 0, all_hi = INT32_MAX;      // keys of any row and of all (that have any)
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int m = m0 + 16 * t + l16, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
        const int2 r = dense_range(a, b, q);
        lo[t] = m < a.M ? r.x : 0;
        hi[t] = m < a.M ? r.y : 0;
        slope2[t] = BIAS ? a.slopes[h] * DENSE_LOG2E : 0.f;
        row_pos[t] = BIAS ? dense_position(a, b, q) : 0;
        const bool some = lo[t] < hi[t];
        const char* p = row_ptr(a.Q, b, q, h, 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + ks * 64) ^ a.negate;
            qf[t][ks] = __builtin_bit_cast(bf16x8_t, some ? x : u32x4_t{0u, 0u, 0u, 0u});
        }
        any_lo = min(any_lo, some ? lo[t] : INT32_MAX);
        any_hi = max(any_hi, some ? hi[t] : 0);
        all_lo = max(all_lo, some ? lo[t] : 0);
        all_hi = min(all_hi, some ? hi[t] : INT32_MAX);
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
    int* const words = reinterpret_cast<int*>(smem + 2 * NR * SLOT);
    if constexpr (NW > 1) {
        if (lane == 0) {
            words[wave] = any_lo;
            words[NW + wave] = any_hi;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            any_lo = min(any_lo, words[i]);
            any_hi = max(any_hi, words[NW + i]);
        }
        __syncthreads();
    }
    // from here on: whether a value that was cleaned away was not finite, whether a sum is not
    if (tid < 2) words[tid] = 0;
    int k_first = __builtin_amdgcn_readfirstlane(any_lo), k_end = __builtin_amdgcn_readfirstlane(any_hi);
    if (k_first >= k_end) k_first = k_end = 0;
    split_keys<GK>(split, a.splits, k_first, k_end);
    all_hi = min(all_hi, k_end);
    const int n_groups = (k_end - k_first + GK - 1) / GK;

    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4_t oacc[CT][QT];
    // m: what is subtracted from base-2 scores; limit: the (kept) score that raises it.  l: this lane's share of the row's sum
    float m_run[QT], limit[QT], l_run[QT];
    bool careful = false;                                    // every group is cleaned and masked
again:
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < QT; ++t) oacc[ct][t] = zero4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m_run[t] = -3e38f;
        limit[t] = -INFINITY;
        l_run[t] = 0.f;
    }
    if (n_groups > 0) {
        const char *kbase = row_ptr(a.K, b, 0, hk, 2), *vbase = row_ptr(a.V, b, 0, hk, 2);
        const uint32_t kss = (uint32_t)(a.K.stride_s * 2), vss = (uint32_t)(a.V.stride_s * 2);
        const int dr = wave * IPW * RPI + lane / PPR;        // row of a group that the lane's first request asks for
        uint32_t k_off[IPW], v_off[IPW];                     // byte offsets inside a group
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            k_off[i] = (uint32_t)(dr + i * RPI) * kss + TL::request_piece(lane, i % TL::NPC);
            v_off[i] = (uint32_t)(dr + i * RPI) * vss + TL::request_piece(lane, i % TL::NPC);
        }
        // The next group of K (n) or V to ring place `slot`.  Rows behind the last key repeat it.
        const int n_whole = max(0, a.Sk - k_first) / GK;      // groups whose rows all exist
        const char *k_next = kbase + (long long)k_first * kss, *v_next = vbase + (long long)k_first * vss;
        auto request = [&](auto values, int n, int slot) {
            constexpr bool VALUES = decltype(values)::value;
            const uint32_t l = lds0 + (uint32_t)((VALUES ? V0 : 0) + slot * SLOT) + (uint32_t)(wave * IPW) * 1024;
            if (__builtin_expect(n < n_whole, 1)) {
#pragma unroll
                for (int i = 0; i < IPW; ++i) dma16(VALUES ? v_next : k_next, VALUES ? v_off[i] : k_off[i], l + i * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < IPW; ++i) {
                    const uint32_t row = (uint32_t)min(k_first + n * GK + dr + i * RPI, a.Sk - 1);
                    dma16(VALUES ? vbase : kbase, row * (VALUES ? vss : kss) + TL::request_piece(lane, i % TL::NPC), l + i * 1024);
                }
            }
            if (VALUES) v_next += (unsigned long long)(GK * vss);
            else k_next += (unsigned long long)(GK * kss);
        };
        using Keys = std::false_type;
        using Values = std::true_type;
        uint32_t rlane[TL::NRB], tlane[TL::NTB];
#pragma unroll
        for (int i = 0; i < TL::NRB; ++i) rlane[i] = TL::row_lane(lane, i);
#pragma unroll
        for (int i = 0; i < TL::NTB; ++i) tlane[i] = TL::tr_lane(lane, i);
        // unit u of S^T: keys 16 * (u / KSTEPS), k-step u % KSTEPS; of the second product: channel tile u.  Ring places are constants in the steps
        auto readK = [&](int slot, int u) { return TL::rows(smem + slot * SLOT, rlane, 0, u / KSTEPS, u % KSTEPS); };
        auto readV = [&](int slot, int u) { return TL::transposed(smem + V0 + slot * SLOT, tlane, 0, u); };
        // A group's values that are not finite become 0 before anybody reads them
        auto clean_values = [&](int slot) {
            if (clean_tile(smem + V0 + slot * SLOT, SLOT, 64 * NW)) words[0] = 1;
            __builtin_amdgcn_s_waitcnt(0xC07F);
            asm volatile("s_barrier" ::: "memory");
        };
        // product x -> kept score, of 16 keys kt of the group at kb
        auto keep_score = [&](f32x4_t(&s)[2][QT], int kt, int t, int i, int kb) {
            if constexpr (CAP || BIAS) {
                if constexpr (BIAS) {
                    float r;
                    const float v = dense_score<CAP>(a, s[kt][t][i], r);
                    s[kt][t][i] = fmaf(-slope2[t], fabsf((float)(row_pos[t] - kb - 4 * g) - (float)(16 * kt + i)), v);
                } else {
                    s[kt][t][i] = __builtin_amdgcn_rcpf(-1.f - exp2_raw(s[kt][t][i] * a.cap_in));
                }
            }
        };

#pragma unroll
        for (int n = 0; n < 4; ++n) {
            request(Keys{}, n, n);
            if (n < 2) request(Values{}, n, n);
        }
        VMOBA_WAIT_VMCNT(0);
        asm volatile("s_barrier" ::: "memory");
        f32x4_t sA[2][QT], sB[2][QT];                        // [16 keys][16 rows]: value i is key 16 * kt + 4 * g + i
        bf16x8_t pA[QT], pB[QT];
        bf16x8_t opK[4], opV[4];
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int t = 0; t < QT; ++t) sA[u / KSTEPS][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(readK(0, u), qf[t][u % KSTEPS], u % KSTEPS == 0 ? zero4 : sA[u / KSTEPS][t], 0, 0, 0);
#pragma unroll
        for (int v = 0; v < 4 * QT; ++v) keep_score(sA, 0, v >> 2, v & 3, k_first);
        opK[0] = readK(1, 0);
        opK[1] = readK(1, 1);
        opV[0] = opV[1] = opK[0];                            // (there is no group -1)

        // Step n, n % 4 = R
        auto step = [&](auto first, auto place, int n, f32x4_t(&s)[2][QT], f32x4_t(&s_next)[2][QT], bf16x8_t(&p_new)[QT], const bf16x8_t(&p_prev)[QT]) __attribute__((always_inline)) {
            constexpr bool FIRST = decltype(first)::value;
            constexpr int R = decltype(place)::value, R1 = (R + 1) & 3, R2 = (R + 2) & 3, R3 = (R + 3) & 3;
            VMOBA_WAIT_VMCNT(2 * IPW);
            asm volatile("s_barrier" ::: "memory");
            const int kb = k_first + n * GK;
            if (__builtin_expect(careful || kb + GK > k_end, 0)) clean_values(R);
#pragma unroll
            for (int v = 0; v < 4 * QT; ++v) keep_score(s, 1, v >> 2, v & 3, kb);
            if (__builtin_expect(careful || kb < all_lo || kb + GK > all_hi, 0)) {
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const int first_key = lo[t] - kb - 4 * g, end = min(hi[t], k_end) - kb - 4 * g;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * kt + i < first_key || 16 * kt + i >= end) s[kt][t][i] = -INFINITY;
                }
            }
            float alpha[QT];
            bool raised = false;
            unsigned w[QT][4];                               // P(n) as packed pairs
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int u2 = u + 2;
                const bf16x8_t nk = u2 < UNITS ? readK(R1, u2) : readK(R2, u2 - UNITS);
                const bf16x8_t nv = u2 < UNITS ? readV(R3, u2) : readV(R, u2 - UNITS);
#pragma unroll
                for (int t = 0; t < QT; ++t)
                    s_next[u / KSTEPS][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(opK[u & 3], qf[t][u % KSTEPS], u % KSTEPS == 0 ? zero4 : s_next[u / KSTEPS][t], 0, 0, 0);
                if constexpr (!FIRST) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) oacc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(opV[u & 3], p_prev[t], oacc[u][t], 0, 0, 0);
                }
                if (u == 0) {
                    float mx[QT];
                    unsigned long long over = 0;
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        mx[t] = max3(max3(s[0][t][0], s[0][t][1], s[0][t][2]), s[0][t][3], s[1][t][0]);
                        mx[t] = max3(mx[t], max3(s[1][t][1], s[1][t][2], s[1][t][3]), mx[t]);
                        over |= __builtin_amdgcn_ballot_w64(mx[t] > limit[t]);
                    }
                    if (__builtin_expect(over != 0, 0)) {
                        raised = true;
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
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
                // pairs of values over the other units
#pragma unroll
                for (int j = 0; j < 4 * QT; ++j) {
                    if (1 + j * (UNITS - 1) / (4 * QT) == u) {
                        const int t = j >> 2, kt = (j >> 1) & 1, i = (j & 1) * 2;
                        const float p0 = exp2_raw(BIAS ? s[kt][t][i] - m_run[t] : fmaf(s[kt][t][i], scale, -m_run[t]));
                        const float p1 = exp2_raw(BIAS ? s[kt][t][i + 1] - m_run[t] : fmaf(s[kt][t][i + 1], scale, -m_run[t]));
                        l_run[t] += p0 + p1;
                        w[t][j & 3] = pack_bf16x2(p0, p1);
                        asm volatile("" : "+v"(w[t][j & 3]));
                    }
                }
                // scores of the next group's first 16 keys
                if (u >= KSTEPS) {
#pragma unroll
                    for (int v = 0; v < 4 * QT; ++v)
                        if (KSTEPS + v * KSTEPS / (4 * QT) == u) keep_score(s_next, 0, v >> 2, v & 3, kb + GK);
                }
                if (u == 1) request(Keys{}, n + 4, R);
                if (u == 2) request(Values{}, n + 2, R2);
                opK[u2 & 3] = nk;
                opV[u2 & 3] = nv;
                __builtin_amdgcn_sched_barrier(0);
            }
            if (__builtin_expect(raised, 0)) {               // the accumulators hold groups up to n - 1, relative to the old maximum
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) oacc[ct][t][i] *= alpha[t];
            }
#pragma unroll
            for (int t = 0; t < QT; ++t) p_new[t] = __builtin_bit_cast(bf16x8_t, u32x4_t{w[t][0], w[t][1], w[t][2], w[t][3]});
        };
        using P0 = std::integral_constant<int, 0>;
        using P1 = std::integral_constant<int, 1>;
        using P2 = std::integral_constant<int, 2>;
        using P3 = std::integral_constant<int, 3>;
        const std::false_type later{};
        step(std::true_type{}, P0{}, 0, sA, sB, pA, pB);
        int n = 1;
        for (; n + 3 < n_groups; n += 4) {
            step(later, P1{}, n, sB, sA, pB, pA);
            step(later, P2{}, n + 1, sA, sB, pA, pB);
            step(later, P3{}, n + 2, sB, sA, pB, pA);
            step(later, P0{}, n + 3, sA, sB, pA, pB);
        }
        if (n < n_groups) {
            step(later, P1{}, n, sB, sA, pB, pA);
            if (n + 1 < n_groups) {
                step(later, P2{}, n + 1, sA, sB, pA, pB);
                if (n + 2 < n_groups) {
                    step(later, P3{}, n + 2, sB, sA, pB, pA);
#pragma unroll
                    for (int t = 0; t < QT; ++t) pA[t] = pB[t];
                }
            } else {
#pragma unroll
                for (int t = 0; t < QT; ++t) pA[t] = pB[t];
            }
        }
        // the last group's second product; no request may be on its way to LDS when the tile's rows go there
        VMOBA_WAIT_VMCNT(0);
        asm volatile("s_barrier" ::: "memory");
        const char* last = smem + V0 + ((n_groups - 1) & 3) * SLOT;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const bf16x8_t v = TL::transposed(last, tlane, 0, u);
#pragma unroll
            for (int t = 0; t < QT; ++t) oacc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pA[t], oacc[u][t], 0, 0, 0);
        }
        if (!careful) {
            float z = 0.f;                                   // NaN if a sum is not finite
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z = fmaf(oacc[ct][t][i], 0.f, z);
            if (__builtin_expect(z != 0.f, 0)) words[1] = 1;
            __syncthreads();
            if (__builtin_expect(__builtin_amdgcn_readfirstlane(words[1]) != 0, 0)) {
                careful = true;
                goto again;
            }
        }
    }

    // ---- rows out
    float lse2[QT], inv[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        float l = l_run[t];
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (lo[t] >= hi[t]) {                                // a row without keys
            l = 0.f;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) oacc[ct][t] = zero4;
        }
        inv[t] = l == 0.f ? 0.f : 1.f / l;                   // (a NaN stays one)
        lse2[t] = l == 0.f ? -INFINITY : m_run[t] + log2f(l) + shift;
    }
    const long long part0 = ((long long)split * a.B * a.Hkv + bh) * a.M;
    if (a.splits > 1) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
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
        char* mine = smem + wave * ROWS * OPITCH;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                u32x2_t v;
                v.x = pack_bf16x2(oacc[ct][t][0] * inv[t], oacc[ct][t][1] * inv[t]);
                v.y = pack_bf16x2(oacc[ct][t][2] * inv[t], oacc[ct][t][3] * inv[t]);
                *reinterpret_cast<u32x2_t*>(mine + (t * 16 + l16) * OPITCH + (ct * 16 + g * 4) * 2) = v;
            }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < ROWS * PPR / 64; ++k) {
            const int row = k * (64 / PPR) + lane / PPR, m = m0 + row;
            if (m < a.M) {
                const int q = query_of(a, m), h = hk * a.G + (m - q * a.G);
                *reinterpret_cast<u32x4_t*>(const_cast<char*>(row_ptr(a.O, b, q, h, 2)) + lane % PPR * 16) =
                    *reinterpret_cast<const u32x4_t*>(mine + row * OPITCH + lane % PPR * 16);
            }
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int m = m0 + 16 * t + l16;
            if (g == 0 && m < a.M) {
                const int q = query_of(a, m), h = hk * a.G + (m - q * a.G);
                a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = lse2[t] * DENSE_LN2;
            }
        }
    }

    if (__builtin_expect(__builtin_amdgcn_readfirstlane(words[0]) == 0, 1)) return;
    constexpr int T1 = QT - 1;                               // (a wavefront of one tile: its second one has no keys)
    dense_repair<__bf16, D, CAP, BIAS>(a, b, hk, m0, lane, part0, k_first, k_end, careful ? INT32_MAX : 0, k_end, lo[0], QT == 2 ? lo[T1] : 0, hi[0],
                                       QT == 2 ? hi[T1] : 0, lse2[0], lse2[T1]);
}

template <int D, int NW, int QT>
void launch_fwd(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 16 * QT * NW) * a.splits, a.Hkv)), block(64 * NW);
    if (cap && a.slopes) dense_fwd_kernel<D, NW, QT, true, true><<<grid, block, 0, st>>>(a);
    else if (cap) dense_fwd_kernel<D, NW, QT, true, false><<<grid, block, 0, st>>>(a);
    else if (a.slopes) dense_fwd_kernel<D, NW, QT, false, true><<<grid, block, 0, st>>>(a);
    else dense_fwd_kernel<D, NW, QT, false, false><<<grid, block, 0, st>>>(a);
}
template <int D>
void launch_rows(bool cap, hipStream_t st, const DenseArgs& a) {
    if (a.M <= 16) launch_fwd<D, 1, 1>(cap, st, a);
    else if (a.M <= DENSE_FEW_ROWS) launch_fwd<D, 1, 2>(cap, st, a);
    else launch_fwd<D, 4, 2>(cap, st, a);
}

}  // namespace

void launch_dense_fwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_rows<128>(cap, st, a) : launch_rows<64>(cap, st, a); }
