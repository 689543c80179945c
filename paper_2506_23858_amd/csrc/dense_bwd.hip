// Backward kernels of dense attention, bfloat16.  Two passes over the pairs and no atomics, so the same call gives the same bits: the dQ
// kernel owns rows and walks their keys (S, dP, dQ: three products), the dK/dV kernel owns keys and walks the rows that read
// them (S, dP, dV, dK: four).  Seven products for the five that a single pass with dQ in atomics would need.
//
// dz = P (dP - delta) (1 - tanh^2), rounded to bfloat16 for the products that follow (relative error 2^-9 a value, like P's).
// Masked pairs: P and dz are replaced by 0, whatever the scores are; operands that the last products contract over (K rows for dQ, Q and dO rows
// for dK and dV) lose their values that are not finite in groups with masked pairs.  A pair that does read such a value has P or delta not finite
// and gives NaN.
#include "dense_common.h"

namespace {

// s: x = <q, k> -> weight P; f: what P * (dP - delta) is multiplied by.
template <bool CAP>
__device__ __forceinline__ float weight_of(const DenseArgs& a, float x, float bias2, float lse2, float& f) {
    float r = 0.f;
    const float s2 = dense_score<CAP>(a, x, r);
    f = CAP ? 4.f * r * (1.f - r) : 1.f;
    return exp2_raw(s2 - bias2 - lse2);
}

// ---------------------------------------------------------------------------------------------
// dQ: the forward kernel's decomposition; 4 wavefronts x 32 rows, chunks of 64 keys through two LDS buffers, requested one chunk ahead.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void dense_dq_kernel(DenseArgs a) {
    using TL = RowTile16<D>;
    constexpr int KC = 64;
    constexpr int KSTEPS = D / 32, CT = D / 16;
    constexpr int HB = TL::HB, PPR = TL::PPR, RPI = TL::RPI;
    constexpr int BUF = 4 * HB;                 // 64 rows of K, then 64 rows of V
    constexpr int IPW = KC / RPI / 4;
    constexpr int OPITCH = D * 2 + 16;
    static_assert(IPW % TL::NPC == 0 && 4 * 32 * OPITCH <= 2 * BUF, "requests, rows on their way out");
    __shared__ __align__(1024) char smem[2 * BUF + 64];

    const int tiles = (a.M + 127) / 128;
    const int item = dense_item(a.B * a.Hkv * tiles);
    if (item < 0) return;
    const int tile = item % tiles, bh = item / tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int m0 = tile * 128 + wave * 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const RowInfo* info = reinterpret_cast<const RowInfo*>(a.row_info) + (long long)bh * ((a.M + 31) / 32);

    int lo[2], hi[2], row_pos[2];
    float lse2[2], slope2[2];
    f32x4_t ndl[2];
    bf16x8_t qf[2][KSTEPS], dof[2][KSTEPS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int m = m0 + 16 * t + l16, mc = min(m, a.M - 1), q = mc / a.G, h = hk * a.G + (mc - q * a.G);
        const RowInfo& r = info[mc >> 5];
        lo[t] = m < a.M ? r.lo[mc & 31] : 0;
        hi[t] = m < a.M ? r.hi[mc & 31] : 0;
        lse2[t] = r.lse2[mc & 31];
        const float d = r.ndelta[mc & 31];
        ndl[t] = f32x4_t{d, d, d, d};
        slope2[t] = BIAS ? r.slope2[mc & 31] : 0.f;
        row_pos[t] = BIAS ? r.pos[mc & 31] : 0;
        const char *p = row_ptr(a.Q, b, q, h, 2) + g * 16, *p2 = row_ptr(a.dO, b, q, h, 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            qf[t][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p + ks * 64) ^ a.negate);
            dof[t][ks] = *reinterpret_cast<const bf16x8_t*>(p2 + ks * 64);
        }
    }
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
    {
        int* w = reinterpret_cast<int*>(smem + 2 * BUF);
        if (lane == 0) {
            w[wave] = any_lo;
            w[4 + wave] = any_hi;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            any_lo = min(any_lo, w[i]);
            any_hi = max(any_hi, w[4 + i]);
        }
    }
    int k_first = __builtin_amdgcn_readfirstlane(any_lo), k_end = __builtin_amdgcn_readfirstlane(any_hi);
    if (k_first >= k_end) k_first = k_end = 0;
    const int n_chunks = (k_end - k_first + KC - 1) / KC;

    const char *kbase = row_ptr(a.K, b, 0, hk, 2), *vbase = row_ptr(a.V, b, 0, hk, 2);
    const uint32_t kss = (uint32_t)(a.K.stride_s * 2), vss = (uint32_t)(a.V.stride_s * 2);
    uint32_t pc16[TL::NPC];
#pragma unroll
    for (int i = 0; i < TL::NPC; ++i) pc16[i] = TL::request_piece(lane, i);
    auto request = [&](int c) {
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const uint32_t row = (uint32_t)min(k_first + c * KC + (wave * IPW + i) * RPI + lane / PPR, a.Sk - 1);
            const uint32_t l = lds0 + (uint32_t)(c & 1) * BUF + (uint32_t)(wave * IPW + i) * 1024;
            dma_row16<0>(kbase, row, kss, pc16[i % TL::NPC], l);
            dma_row16<2 * HB>(vbase, row, vss, pc16[i % TL::NPC], l);
        }
    };
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4_t acc[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct][0] = acc[ct][1] = zero4;
    uint32_t rlane[TL::NRB], tlane[TL::NTB];
#pragma unroll
    for (int i = 0; i < TL::NRB; ++i) rlane[i] = TL::row_lane(lane, i);
#pragma unroll
    for (int i = 0; i < TL::NTB; ++i) tlane[i] = TL::tr_lane(lane, i);

    if (n_chunks > 0) request(0);
    VMOBA_WAIT_VMCNT(0);
    __syncthreads();
    unsigned found = 0;
    for (int c = 0; c < n_chunks; ++c) {
        const uint32_t buf = (uint32_t)(c & 1) * BUF;
        if (c + 1 < n_chunks) request(c + 1);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int kb = k_first + c * KC + mt * 32;
            if (kb >= k_end) break;
            const bool masked = kb < all_lo || kb + 32 > all_hi;
            f32x4_t s[2][2], dp[2][2];            // [16 keys][16 rows]: value i is key 16 * kt + 4 * g + i
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) {
                    const bf16x8_t x = TL::rows(smem, rlane, buf + mt * HB, kt, ks);
#pragma unroll
                    for (int t = 0; t < 2; ++t) s[kt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, qf[t][ks], ks == 0 ? zero4 : s[kt][t], 0, 0, 0);
                }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) {
                    const bf16x8_t x = TL::rows(smem, rlane, buf + (2 + mt) * HB, kt, ks);
#pragma unroll
                    for (int t = 0; t < 2; ++t) dp[kt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, dof[t][ks], ks == 0 ? ndl[t] : dp[kt][t], 0, 0, 0);
                }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float rel = BIAS ? (float)(row_pos[t] - kb - 4 * g) : 0.f;
                const int first_key = lo[t] - kb - 4 * g, end = hi[t] - kb - 4 * g;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float f;
                        const float p = weight_of<CAP>(a, s[kt][t][i], BIAS ? slope2[t] * fabsf(rel - (float)(16 * kt + i)) : 0.f, lse2[t], f);
                        float d = p * f * dp[kt][t][i];
                        if (masked && (16 * kt + i < first_key || 16 * kt + i >= end)) d = 0.f;
                        s[kt][t][i] = d;
                    }
            }
            bf16x8_t ds[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float d8[8] = {s[0][t][0], s[0][t][1], s[0][t][2], s[0][t][3], s[1][t][0], s[1][t][1], s[1][t][2], s[1][t][3]};
                ds[t] = pack8(d8);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                bf16x8_t x = TL::transposed(smem, tlane, buf + mt * HB, ct);
                if (masked) x = finite_only(x, found);
#pragma unroll
                for (int t = 0; t < 2; ++t) acc[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, ds[t], acc[ct][t], 0, 0, 0);
            }
        }
        VMOBA_WAIT_VMCNT(0);
        __syncthreads();
    }
    char* mine = smem + wave * 32 * OPITCH;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x2_t v;
            v.x = pack_bf16x2(acc[ct][t][0] * a.scale, acc[ct][t][1] * a.scale);
            v.y = pack_bf16x2(acc[ct][t][2] * a.scale, acc[ct][t][3] * a.scale);
            *reinterpret_cast<u32x2_t*>(mine + (t * 16 + l16) * OPITCH + (ct * 16 + g * 4) * 2) = v;
        }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < 32 * PPR / 64; ++k) {
        const int row = k * (64 / PPR) + lane / PPR, m = m0 + row;
        if (m < a.M) {
            const int q = m / a.G, h = hk * a.G + (m - q * a.G);
            *reinterpret_cast<u32x4_t*>(const_cast<char*>(row_ptr(a.dQ, b, q, h, 2)) + lane % PPR * 16) =
                *reinterpret_cast<const u32x4_t*>(mine + row * OPITCH + lane % PPR * 16);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// dK/dV: a workgroup owns 128 keys, a wavefront 32 of them (key = column = lane % 16), and walks the packed rows that read any of them in
// chunks of 32:
//   S   = Q . K^T      A = Q rows (LDS),   B = K^T (registers)
//   dP  = dO . V^T     A = dO rows (LDS),  B = V^T (LDS: its 32 registers are what two wavefronts per SIMD have not got)
//   dV^T += dO^T . P   A = dO^T by transpose reads, B = P packed from S
//   dK^T += Q^T . dz   A = Q^T by transpose reads,  B = dz
// Which chunks those are stands in row_bounds: a wavefront looks at 64 of them at a time.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void dense_dkv_kernel(DenseArgs a) {
    using TL = RowTile16<D>;
    constexpr int KSTEPS = D / 32, CT = D / 16;
    constexpr int HB = TL::HB, PPR = TL::PPR, RPI = TL::RPI;
    constexpr int BUF = 2 * HB + (int)sizeof(RowInfo);   // 32 rows of Q, of dO, and what is known of them
    constexpr int B0 = 4 * HB;                           // V: 128 rows, first
    constexpr int IPW = 32 / RPI / 4;
    constexpr int OPITCH = D * 2 + 16;
    static_assert(IPW >= 1 && IPW % TL::NPC == 0 && 4 * 32 * OPITCH <= B0 + 2 * BUF, "requests, rows on their way out");
    __shared__ __align__(1024) char smem[B0 + 2 * BUF];

    const int tiles = (a.Sk + 127) / 128;
    const int item = dense_item(a.B * a.Hkv * tiles);
    if (item < 0) return;
    const int tile = item % tiles, bh = item / tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int k0 = tile * 128, kw = k0 + wave * 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int n_chunks = (a.M + 31) / 32;
    const char* info = a.row_info + (long long)bh * n_chunks * (long long)sizeof(RowInfo);
    const int4* bounds = a.row_bounds + (long long)bh * n_chunks;

    // K fragments of the wavefront's keys (column l16 of 16-key half kt), V rows of the workgroup's
    bf16x8_t kf[2][KSTEPS];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const char* p = row_ptr(a.K, b, min(kw + 16 * kt + l16, a.Sk - 1), hk, 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kf[kt][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p + ks * 64) ^ a.negate);
    }
    uint32_t pc16[TL::NPC];
#pragma unroll
    for (int i = 0; i < TL::NPC; ++i) pc16[i] = TL::request_piece(lane, i);
    const char* vbase = row_ptr(a.V, b, 0, hk, 2);
#pragma unroll
    for (int i = 0; i < 4 * IPW; ++i)
        dma_row16<0>(vbase, (uint32_t)min(kw + i * RPI + lane / PPR, a.Sk - 1), (uint32_t)(a.V.stride_s * 2), pc16[i % TL::NPC], lds0 + (uint32_t)(wave * 4 * IPW + i) * 1024);

    auto request = [&](int c, int par) {
        const uint32_t l = lds0 + B0 + (uint32_t)par * BUF;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int m = min(c * 32 + (wave * IPW + i) * RPI + lane / PPR, a.M - 1), q = m / a.G, h = hk * a.G + (m - q * a.G);
            dma16_at(row_ptr(a.Q, b, q, h, 2) + pc16[i % TL::NPC], l + (uint32_t)(wave * IPW + i) * 1024);
            dma16_at(row_ptr(a.dO, b, q, h, 2) + pc16[i % TL::NPC], l + HB + (uint32_t)(wave * IPW + i) * 1024);
        }
        if (wave == 3) dma16_at(info + (long long)c * (long long)sizeof(RowInfo) + lane * 16, l + 2 * HB);
    };
    // chunks whose rows read one of the 128 keys, in order; the same for all wavefronts
    int window = 0;
    unsigned long long pending = 0;
    auto look = [&]() {
        const int c = window + lane;
        const int4 r = c < n_chunks ? bounds[c] : make_int4(INT32_MAX, 0, 0, 0);
        pending = __builtin_amdgcn_ballot_w64(r.x < k0 + 128 && r.y > k0);
    };
    auto next_chunk = [&]() {
        while (pending == 0) {
            window += 64;
            if (window >= n_chunks) return -1;
            look();
        }
        const int i = __builtin_ctzll(pending);
        pending &= pending - 1;
        return window + i;
    };
    look();

    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4_t dv[CT][2], dk[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) dv[ct][0] = dv[ct][1] = dk[ct][0] = dk[ct][1] = zero4;
    uint32_t rlane[TL::NRB], tlane[TL::NTB];
#pragma unroll
    for (int i = 0; i < TL::NRB; ++i) rlane[i] = TL::row_lane(lane, i);
#pragma unroll
    for (int i = 0; i < TL::NTB; ++i) tlane[i] = TL::tr_lane(lane, i);
    const uint32_t vrows = (uint32_t)wave * HB;

    int c = next_chunk(), par = 0;
    if (c >= 0) request(c, 0);
    VMOBA_WAIT_VMCNT(0);
    __syncthreads();
    unsigned found = 0;
    while (c >= 0) {
        const int c_next = next_chunk();
        if (c_next >= 0) request(c_next, par ^ 1);
        const uint32_t buf = B0 + (uint32_t)par * BUF;
        const RowInfo* ri = reinterpret_cast<const RowInfo*>(smem + buf + 2 * HB);
        const int4 bd = bounds[c];
        const int all_lo = __builtin_amdgcn_readfirstlane(bd.z), all_hi = __builtin_amdgcn_readfirstlane(bd.w);
        const bool masked = kw < all_lo || kw + 32 > all_hi;
        f32x4_t s[2][2], dp[2][2];                        // [16 rows][16 keys]: value i is row 16 * t + 4 * g + i
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                const bf16x8_t x = TL::rows(smem, rlane, buf, t, ks);
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) s[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, kf[kt][ks], ks == 0 ? zero4 : s[t][kt], 0, 0, 0);
            }
        f32x4_t nd[2], lse2[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            nd[t] = *reinterpret_cast<const f32x4_t*>(ri->ndelta + 16 * t + 4 * g);
            lse2[t] = *reinterpret_cast<const f32x4_t*>(ri->lse2 + 16 * t + 4 * g);
        }
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const bf16x8_t v0 = TL::rows(smem, rlane, vrows, 0, ks), v1 = TL::rows(smem, rlane, vrows, 1, ks);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8_t x = TL::rows(smem, rlane, buf + HB, t, ks);
                dp[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, v0, ks == 0 ? nd[t] : dp[t][0], 0, 0, 0);
                dp[t][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, v1, ks == 0 ? nd[t] : dp[t][1], 0, 0, 0);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4_t slope2 = zero4;
            u32x4_t pos = {0u, 0u, 0u, 0u}, lo = pos, hi = pos;
            if constexpr (BIAS) {
                slope2 = *reinterpret_cast<const f32x4_t*>(ri->slope2 + 16 * t + 4 * g);
                pos = *reinterpret_cast<const u32x4_t*>(ri->pos + 16 * t + 4 * g);
            }
            if (masked) {
                lo = *reinterpret_cast<const u32x4_t*>(ri->lo + 16 * t + 4 * g);
                hi = *reinterpret_cast<const u32x4_t*>(ri->hi + 16 * t + 4 * g);
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const int key = kw + 16 * kt + l16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f;
                    float p = weight_of<CAP>(a, s[t][kt][i], BIAS ? slope2[i] * fabsf((float)((int)pos[i] - key)) : 0.f, lse2[t][i], f);
                    float d = p * f * dp[t][kt][i];
                    if (masked) {
                        const bool reads = key >= (int)lo[i] && key < (int)hi[i];
                        // (a row of dO that is not finite shows in delta; its values are taken out of the product below)
                        p = !reads ? 0.f : fabsf(nd[t][i]) < INFINITY ? p : NAN;
                        d = reads ? d : 0.f;
                    }
                    s[t][kt][i] = p;
                    dp[t][kt][i] = d;
                }
            }
        }
        bf16x8_t pf[2], df[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const float p8[8] = {s[0][kt][0], s[0][kt][1], s[0][kt][2], s[0][kt][3], s[1][kt][0], s[1][kt][1], s[1][kt][2], s[1][kt][3]};
            const float d8[8] = {dp[0][kt][0], dp[0][kt][1], dp[0][kt][2], dp[0][kt][3], dp[1][kt][0], dp[1][kt][1], dp[1][kt][2], dp[1][kt][3]};
            pf[kt] = pack8(p8);
            df[kt] = pack8(d8);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            bf16x8_t x = TL::transposed(smem, tlane, buf + HB, ct), y = TL::transposed(smem, tlane, buf, ct);
            if (masked) {
                x = finite_only(x, found);
                y = finite_only(y, found);
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                dv[ct][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pf[kt], dv[ct][kt], 0, 0, 0);
                dk[ct][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, df[kt], dk[ct][kt], 0, 0, 0);
            }
        }
        VMOBA_WAIT_VMCNT(0);
        __syncthreads();
        c = c_next;
        par ^= 1;
    }
    char* mine = smem + wave * 32 * OPITCH;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const TensorView& out = which == 0 ? a.dV : a.dK;
        const float f = which == 0 ? 1.f : a.scale;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const f32x4_t x = which == 0 ? dv[ct][kt] : dk[ct][kt];
                u32x2_t v;
                v.x = pack_bf16x2(x[0] * f, x[1] * f);
                v.y = pack_bf16x2(x[2] * f, x[3] * f);
                *reinterpret_cast<u32x2_t*>(mine + (kt * 16 + l16) * OPITCH + (ct * 16 + g * 4) * 2) = v;
            }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < 32 * PPR / 64; ++k) {
            const int row = k * (64 / PPR) + lane / PPR, key = kw + row;
            if (key < a.Sk)
                *reinterpret_cast<u32x4_t*>(const_cast<char*>(row_ptr(out, b, key, hk, 2)) + lane % PPR * 16) =
                    *reinterpret_cast<const u32x4_t*>(mine + row * OPITCH + lane % PPR * 16);
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
    }
}

template <int D>
void launch_bwd(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 gq(dense_grid((int64_t)a.B * a.Hkv * ceil_div64(a.M, 128))), gk(dense_grid((int64_t)a.B * a.Hkv * ceil_div64(a.Sk, 128))), block(256);
#define BOTH(CAP, BIAS)                                     \
    do {                                                    \
        dense_dq_kernel<D, CAP, BIAS><<<gq, block, 0, st>>>(a);   \
        dense_dkv_kernel<D, CAP, BIAS><<<gk, block, 0, st>>>(a);  \
    } while (0)
    if (cap && a.slopes) BOTH(true, true);
    else if (cap) BOTH(true, false);
    else if (a.slopes) BOTH(false, true);
    else BOTH(false, false);
#undef BOTH
}

}  // namespace

void launch_dense_bwd_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_bwd<128>(cap, st, a) : launch_bwd<64>(cap, st, a); }
