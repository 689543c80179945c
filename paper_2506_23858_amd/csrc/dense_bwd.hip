// Backward kernels of dense attention, bfloat16.  Two passes over the pairs and no atomics, so the same call gives the same bits: the dQ
// kernel owns rows and walks their keys (S, dP, dQ: three products), the dK/dV kernel owns keys and walks the rows that read
// them (S, dP, dV, dK: four).  Seven products for the five that a single pass with dQ in atomics would need.
//
// dz = P (dP - delta) (1 - tanh^2), 1 - tanh^2 = 4 (r - r^2), rounded to bfloat16 for the products that follow (relative error 2^-9 a value, like P's).
// Masked pairs: their scores are replaced (-inf, or 0 with an infinite log-sum-exp), so P and dz are 0.  A masked value that is not finite would still spoil a sum -- 0 times
// infinity is no number --, so tiles that pass the last key or hold rows without keys lose such values in LDS before they are multiplied, and a
// workgroup whose sums end up not finite starts again with all tiles cleaned so.  A pair that does read such a value has a log-sum-exp or a delta that is not
// finite, and gives NaN.
#include "dense_common.h"

namespace {

// x = <q, k> -> weight P, from c2 = -(log-sum-exp + bias), base 2, with the cap + cap2 (see RowInfo); f (cap alone): a quarter of what P (dP - delta) is multiplied
// by, r - r^2; the 4 is in the factor that the sums end with.
template <bool CAP>
__device__ __forceinline__ float weight_of(const DenseArgs& a, float x, float c2, float& f) {
    if constexpr (CAP) {
        const float r = __builtin_amdgcn_rcpf(1.f + exp2_raw(x * a.cap_in));
        f = fmaf(-r, r, r);
        return exp2_raw(fmaf(-2.f * a.cap2, r, c2));
    } else {
        return exp2_raw(fmaf(x, a.scale_log2, c2));
    }
}

// ---------------------------------------------------------------------------------------------
// dQ: the forward kernel's decomposition; 4 wavefronts x 32 rows, chunks of 64 keys through two LDS buffers, requested one chunk ahead.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void dense_dq_kernel(DenseArgs a) {
    using TL = DenseTile<D>;
    constexpr int KC = 64;
    constexpr int KSTEPS = D / 32, CT = D / 16;
    constexpr int HB = TL::HB, PPR = TL::PPR, RPI = TL::RPI;
    constexpr int BUF = 4 * HB;                 // 64 rows of K, then 64 rows of V
    constexpr int IPW = KC / RPI / 4;
    constexpr int OPITCH = D * 2 + 16;
    static_assert(IPW % TL::NPC == 0 && 4 * 32 * OPITCH <= 2 * BUF, "requests, rows on their way out");
    __shared__ __align__(1024) char smem[2 * BUF + 64];

    const int tiles = (a.M + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_q);
    const int tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int m0 = tile * 128 + wave * 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const RowInfo* info = reinterpret_cast<const RowInfo*>(a.row_info) + (long long)bh * ((a.M + 31) / 32);

    int lo[2], hi[2], row_pos[2];
    float c2[2], slope2[2];
    f32x4_t ndl[2];
    bf16x8_t qf[2][KSTEPS], dof[2][KSTEPS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int m = m0 + 16 * t + l16, mc = min(m, a.M - 1), q = query_of(a, mc), h = hk * a.G + (mc - q * a.G);
        const RowInfo& r = info[mc >> 5];
        lo[t] = m < a.M ? r.lo[mc & 31] : 0;
        hi[t] = m < a.M ? r.hi[mc & 31] : 0;
        c2[t] = r.c2[mc & 31];
        const float d = r.ndelta[mc & 31];
        ndl[t] = f32x4_t{d, d, d, d};
        slope2[t] = BIAS ? r.slope2[mc & 31] : 0.f;
        row_pos[t] = BIAS ? r.pos[mc & 31] : 0;
        const bool some = lo[t] < hi[t];            // (a row without keys: a query of zeros, weights of 0 by its log-sum-exp)
        const char *p = row_ptr(a.Q, b, q, h, 2) + g * 16, *p2 = row_ptr(a.dO, b, q, h, 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + ks * 64) ^ a.negate;
            qf[t][ks] = __builtin_bit_cast(bf16x8_t, some ? x : u32x4_t{0u, 0u, 0u, 0u});
            unsigned unused = 0;      // (what was not finite shows in the row's log-sum-exp, see dense_rows_kernel)
            dof[t][ks] = finite_only(*reinterpret_cast<const bf16x8_t*>(p2 + ks * 64), unused);
        }
    }
    int any_lo = INT32_MAX, any_hi = 0, all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const bool some = lo[t] < hi[t];
        any_lo = min(any_lo, some ? lo[t] : INT32_MAX);
        any_hi = max(any_hi, some ? hi[t] : 0);
        all_lo = max(all_lo, some ? lo[t] : 0);
        all_hi = min(all_hi, some ? hi[t] : INT32_MAX);
        if (m0 + 16 * t + l16 >= a.M) c2[t] = -INFINITY;
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
    const int wave_lo = __builtin_amdgcn_readfirstlane(any_lo), wave_hi = __builtin_amdgcn_readfirstlane(any_hi);
    int* const words = reinterpret_cast<int*>(smem + 2 * BUF);
    if (lane == 0) {
        words[wave] = any_lo;
        words[4 + wave] = any_hi;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        any_lo = min(any_lo, words[i]);
        any_hi = max(any_hi, words[4 + i]);
    }
    __syncthreads();
    if (tid == 0) words[0] = 0;                 // from here on: whether a sum is not finite
    int k_first = __builtin_amdgcn_readfirstlane(any_lo), k_end = __builtin_amdgcn_readfirstlane(any_hi);
    if (k_first >= k_end) k_first = k_end = 0;
    split_keys<KC>(task.split, a.splits, k_first, k_end);
    all_hi = min(all_hi, k_end);
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
    bool careful = false;                       // every chunk is cleaned and masked
    const uint32_t rlane = TL::row_lane(lane, 0), tlane = TL::tr_lane(lane, 0);
    uint32_t rows0 = 0, cols0 = 0;              // lane addresses in the current chunk's buffer

    // A 32-key group is a sequence of units of one LDS operand and two matrix instructions (one per 16 rows): S^T over (16 keys, k-step), dP^T over
    // the same, the third product over the channel tiles.  Operands pass through a ring, fetched AHEAD units before use; weights are computed
    // between the matrix instructions, those of the first 16 keys from the middle of the first phase on.  Fences keep that order.
    constexpr int NP = 2 * KSTEPS, NSEQ = 3 * NP, AHEAD = 3, RING = AHEAD + 1;
    static_assert(NP == CT, "as many units in each phase");
    auto fetch = [&](int mt, int n) -> bf16x8_t {      // operand of unit n of group mt
        if (n < NP) return TL::rows(smem + mt * HB, rows0, n / KSTEPS, n % KSTEPS);
        if (n < 2 * NP) return TL::rows(smem + (2 + mt) * HB, rows0, (n - NP) / KSTEPS, n % KSTEPS);
        return TL::transposed(smem + mt * HB, cols0, n - 2 * NP);
    };
again:
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct][0] = acc[ct][1] = zero4;
    if (n_chunks > 0) request(0);
    VMOBA_WAIT_VMCNT(0);
    __syncthreads();
    for (int c = 0; c < n_chunks; ++c) {
        const uint32_t buf = (uint32_t)(c & 1) * BUF;
        const int kc = k_first + c * KC;
        if (__builtin_expect(careful || kc + KC > k_end, 0)) {
            clean_tile(smem + buf, BUF, 256);
            __syncthreads();
        }
        if (c + 1 < n_chunks) request(c + 1);
        rows0 = rlane + buf;
        cols0 = tlane + buf;
        bf16x8_t op[RING];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int kb = kc + mt * 32;
            if (kb + 32 > wave_lo && kb < min(wave_hi, k_end)) {      // (keys that one of the wavefront's rows reads)
                const bool masked = careful || kb < all_lo || kb + 32 > all_hi;
                f32x4_t s[2][2], dp[2][2];            // [16 keys][16 rows]: value i is key 16 * kt + 4 * g + i
                bf16x8_t ds[2];
                float rel[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) rel[t] = BIAS ? (float)(row_pos[t] - kb - 4 * g) : 0.f;
                auto p_value = [&](int v) {           // S^T -> P^T (1 - tanh^2), in place
                    const int kt = v >> 3, t = (v >> 2) & 1, i = v & 3;
                    float f = 1.f;
                    float p = weight_of<CAP>(a, s[kt][t][i], BIAS ? fmaf(-slope2[t], fabsf(rel[t] - (float)(16 * kt + i)), c2[t]) : c2[t], f);
                    if constexpr (CAP) p *= f;
                    s[kt][t][i] = p;
                };
                auto ds_value = [&](int v) {
                    const int kt = v >> 3, t = (v >> 2) & 1, i = v & 3;
                    float d = s[kt][t][i] * dp[kt][t][i];
                    asm volatile("" : "+v"(d));
                    s[kt][t][i] = d;
                };
#pragma unroll
                for (int n = 0; n < RING; ++n) op[n] = fetch(mt, n < AHEAD ? n : 0);
#pragma unroll
                for (int n = 0; n < NSEQ; ++n) {
                    if (n + AHEAD < NSEQ) op[(n + AHEAD) % RING] = fetch(mt, n + AHEAD);
                    const int m = n % NP, kt = m / KSTEPS, ks = m % KSTEPS;
                    if ((n == KSTEPS + 1 || n == NP) && __builtin_expect(masked, 0)) {      // the scores of the first, of the second 16 keys are complete
                        const int half = n == NP ? 1 : 0;
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const int first_key = lo[t] - kb - 4 * g - 16 * half, end = min(hi[t], k_end) - kb - 4 * g - 16 * half;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (i < first_key || i >= end) s[half][t][i] = -INFINITY;      // (with the cap: r = 1, so f = 0)
                        }
                    }
                    if (n == 2 * NP) {
#pragma unroll
                        for (int v = 8; v < 16; ++v) ds_value(v);
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const float d8[8] = {s[0][t][0], s[0][t][1], s[0][t][2], s[0][t][3], s[1][t][0], s[1][t][1], s[1][t][2], s[1][t][3]};
                            ds[t] = pack8(d8);
                        }
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (n < NP)
                            s[kt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n % RING], qf[t][ks], ks == 0 ? zero4 : s[kt][t], 0, 0, 0);
                        else if (n < 2 * NP)
                            dp[kt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n % RING], dof[t][ks], ks == 0 ? ndl[t] : dp[kt][t], 0, 0, 0);
                        else
                            acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n % RING], ds[t], acc[m][t], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    constexpr int E0 = KSTEPS + 1, E1 = NP;             // units of the first 8 weights
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        if (E0 + v * (E1 - E0) / 8 == n) p_value(v);
                        if (NP + v * NP / 8 == n) p_value(8 + v);
                        if (NP + KSTEPS + v * KSTEPS / 8 == n) ds_value(v);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        VMOBA_WAIT_VMCNT(0);
        __syncthreads();
    }
    if (!careful) {
        float z = 0.f;                          // NaN if a sum is not finite
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = fmaf(acc[ct][t][i], 0.f, z);
        if (__builtin_expect(z != 0.f, 0)) words[0] = 1;
        __syncthreads();
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(words[0]) != 0, 0)) {
            careful = true;
            goto again;
        }
    }
    const float out = CAP ? 4.f * a.scale : a.scale;
    if (a.splits > 1) {                         // this split's sums, added up by dense_sum_kernel
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int m = m0 + 16 * t + l16;
            if (m < a.M) {
                float* dst = a.part_o + (((long long)task.split * a.B * a.Hkv + bh) * a.M + m) * D + 4 * g;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) *reinterpret_cast<f32x4_t*>(dst + 16 * ct) = acc[ct][t] * out;
            }
        }
        return;
    }
    char* mine = smem + wave * 32 * OPITCH;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x2_t v;
            v.x = pack_bf16x2(acc[ct][t][0] * out, acc[ct][t][1] * out);
            v.y = pack_bf16x2(acc[ct][t][2] * out, acc[ct][t][3] * out);
            *reinterpret_cast<u32x2_t*>(mine + (t * 16 + l16) * OPITCH + (ct * 16 + g * 4) * 2) = v;
        }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < 32 * PPR / 64; ++k) {
        const int row = k * (64 / PPR) + lane / PPR, m = m0 + row;
        if (m < a.M) {
            const int q = query_of(a, m), h = hk * a.G + (m - q * a.G);
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
    using TL = DenseTile<D>;
    constexpr int KSTEPS = D / 32, CT = D / 16;
    constexpr int HB = TL::HB, PPR = TL::PPR, RPI = TL::RPI;
    constexpr int BUF = 2 * HB + (int)sizeof(RowInfo);   // 32 rows of Q, of dO, and what is known of them
    constexpr int B0 = 4 * HB;                           // V: 128 rows, first
    constexpr int IPW = 32 / RPI / 4;
    constexpr int OPITCH = D * 2 + 16;
    static_assert(IPW >= 1 && IPW % TL::NPC == 0 && 4 * 32 * OPITCH <= B0 + 2 * BUF, "requests, rows on their way out");
    __shared__ __align__(1024) char smem[B0 + 2 * BUF + 16];

    const int tiles = (a.Sk + 127) / 128;
    const DensePiece piece = dense_piece(a.B * tiles * a.splits, a.Hkv);
    if (piece.rank < 0) return;
    const DenseTask task = dense_task(piece.rank, a.splits, tiles, a.order_k);
    const int tile = task.tile, b = task.b, hk = piece.head, bh = b * a.Hkv + hk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int k0 = tile * 128, kw = k0 + wave * 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int n_chunks = (a.M + 31) / 32;
    const char* info = a.row_info + (long long)bh * n_chunks * (long long)sizeof(RowInfo);
    ChunkWalk walk(a.row_bounds + (long long)bh * n_chunks, n_chunks, k0, k0 + 128, lane, task.split, a.splits);

    // K fragments of the wavefront's keys (column l16 of 16-key half kt), V rows of the workgroup's
    bf16x8_t kf[2][KSTEPS];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const char* p = row_ptr(a.K, b, min(kw + 16 * kt + l16, a.Sk - 1), hk, 2) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kf[kt][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p + ks * 64) ^ a.negate);
    }
    const char* vbase = row_ptr(a.V, b, 0, hk, 2);
#pragma unroll
    for (int i = 0; i < 4 * IPW; ++i)
        dma_row16<0>(vbase, (uint32_t)min(kw + i * RPI + lane / PPR, a.Sk - 1), (uint32_t)(a.V.stride_s * 2), TL::request_piece(lane, i % TL::NPC), lds0 + (uint32_t)(wave * 4 * IPW + i) * 1024);

    const char *qbase = row_ptr(a.Q, b, 0, hk * a.G, 2), *obase = row_ptr(a.dO, b, 0, hk * a.G, 2);
    const uint32_t qss = (uint32_t)(a.Q.stride_s * 2), qsh = (uint32_t)(a.Q.stride_h * 2), oss = (uint32_t)(a.dO.stride_s * 2), osh = (uint32_t)(a.dO.stride_h * 2);
    auto request = [&](int c, int par) {
        const uint32_t l = lds0 + B0 + (uint32_t)par * BUF;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int m = min(c * 32 + (wave * IPW + i) * RPI + lane / PPR, a.M - 1);
            const uint32_t piece = TL::request_piece(lane, i);
            dma16(qbase, packed_row(a, m, qss, qsh) + piece, l + (uint32_t)(wave * IPW + i) * 1024);
            dma16(obase, packed_row(a, m, oss, osh) + piece, l + HB + (uint32_t)(wave * IPW + i) * 1024);
        }
        if (wave == 3) dma16(info + (long long)c * (long long)sizeof(RowInfo), (uint32_t)lane * 16, l + 2 * HB);
    };

    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4_t dv[CT][2], dk[CT][2];
    bool careful = false;                                // every chunk is cleaned and masked
    int* const words = reinterpret_cast<int*>(smem + B0 + 2 * BUF);
    if (tid == 0) words[0] = 0;                          // whether a sum is not finite
    const uint32_t rlane = TL::row_lane(lane, 0), tlane = TL::tr_lane(lane, 0);

    // A chunk is a sequence of units: S over (16 rows, k-step), one operand and two matrix instructions (one per 16 keys) each; dP over the k-steps, four operands (V of both key
    // halves, dO of both row halves) and four; dV over the channel tiles, dK over the channel tiles, one and two.  Weights are computed in the second half of the
    // first phase and in the second one, dz in the third.
    constexpr int NP = 2 * KSTEPS;
    static_assert(NP == CT, "as many units in the first phase as in the last two");
again:
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) dv[ct][0] = dv[ct][1] = dk[ct][0] = dk[ct][1] = zero4;
    int c = walk.next(), par = 0;
    if (c >= 0) request(c, 0);
    VMOBA_WAIT_VMCNT(0);
    __syncthreads();
    clean_tile(smem, 4 * HB, 256);             // V: a value that is not finite shows in the log-sum-exp or delta of the rows that read it
    __syncthreads();
    while (c >= 0) {
        const int all_lo = walk.all_lo, all_hi = walk.all_hi;
        const bool one_range = walk.any_lo == all_lo && walk.any_hi == all_hi;      // of all the chunk's rows
        const bool none = kw >= walk.any_hi || kw + 32 <= walk.any_lo;              // of the wavefront's keys is read
        const uint32_t buf = B0 + (uint32_t)par * BUF;
        const RowInfo* ri = reinterpret_cast<const RowInfo*>(smem + buf + 2 * HB);
        const bool masked = careful || kw < all_lo || kw + 32 > all_hi;
        if (__builtin_expect(careful || all_lo == INT32_MAX, 0)) {      // (a chunk with rows that read no key)
            clean_tile(smem + buf, 2 * HB, 256);
            __syncthreads();
        }
        const int c_next = walk.next();
        if (c_next >= 0) request(c_next, par ^ 1);
        if (__builtin_expect(!none, 1)) {
        bool reads[2];                                    // one range: whether the chunk's rows read the lane's keys
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) reads[kt] = kw + 16 * kt + l16 >= all_lo && kw + 16 * kt + l16 < all_hi;
        const uint32_t rows0 = rlane + buf, cols0 = tlane + buf, vrows0 = pinned(rlane) + (uint32_t)wave * HB;
        f32x4_t s[2][2], dp[2][2];                        // [16 rows][16 keys]: value i is row 16 * t + 4 * g + i
        unsigned pw[2][4];                                // P as packed pairs
        auto p_pair = [&](int j) {                        // values 2 j and 2 j + 1: S -> P (packed), P (1 - tanh^2) in its place
            const int t = j >> 2, kt = (j >> 1) & 1, i0 = (j & 1) * 2, r0 = 16 * t + 4 * g + i0, key = kw + 16 * kt + l16;
            f32x2_t c2 = *reinterpret_cast<const f32x2_t*>(ri->c2 + r0);
            float p[2];
            if (__builtin_expect(masked, 0)) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (one_range ? !reads[kt] : key < ri->lo[r0 + e] || key >= ri->hi[r0 + e]) {
                        s[t][kt][i0 + e] = 0.f;
                        c2[e] = -INFINITY;
                    }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float f = 1.f;
                if constexpr (BIAS) c2[e] = fmaf(-ri->slope2[r0 + e], fabsf((float)(ri->pos[r0 + e] - key)), c2[e]);
                p[e] = weight_of<CAP>(a, s[t][kt][i0 + e], c2[e], f);
                s[t][kt][i0 + e] = CAP ? p[e] * f : p[e];
            }
            pw[kt][2 * t + (j & 1)] = pack_bf16x2(p[0], p[1]);
        };
        auto ds_value = [&](int v) {
            const int t = v >> 3, kt = (v >> 2) & 1, i = v & 3;
            dp[t][kt][i] *= s[t][kt][i];
        };
        bf16x8_t op[4];
#pragma unroll
        for (int n = 0; n < 3; ++n) op[n] = TL::rows(smem, rows0, n / KSTEPS, n % KSTEPS);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int t = n / KSTEPS, ks = n % KSTEPS;
            if (n + 3 < NP) op[(n + 3) & 3] = TL::rows(smem, rows0, (n + 3) / KSTEPS, (n + 3) % KSTEPS);
            else if (n + 3 < NP + 2) op[(n + 3) & 3] = TL::rows(smem, vrows0, n + 3 - NP, 0);
            else op[(n + 3) & 3] = TL::rows(smem + HB, rows0, 0, 0);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n & 3], kf[kt][ks], ks == 0 ? zero4 : s[t][kt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int E0 = KSTEPS + 1;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (E0 + j * (NP - E0) / 4 == n) p_pair(j);
            __builtin_amdgcn_sched_barrier(0);
        }
        // V of the first and of the second 16 keys, dO of the first 16 rows; dO of the others is fetched in the unit
        bf16x8_t v0 = op[NP & 3], v1 = op[(NP + 1) & 3], x0 = op[(NP + 2) & 3];
        f32x4_t nd[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) nd[t] = *reinterpret_cast<const f32x4_t*>(ri->ndelta + 16 * t + 4 * g);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const bf16x8_t x1 = TL::rows(smem + HB, rows0, 1, ks);
            dp[0][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0, v0, ks == 0 ? nd[0] : dp[0][0], 0, 0, 0);
            dp[0][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0, v1, ks == 0 ? nd[0] : dp[0][1], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (ks + 1 < KSTEPS) x0 = TL::rows(smem + HB, rows0, 0, ks + 1);
            else x0 = TL::transposed(smem + HB, cols0, 0);
            if (KSTEPS == 4 || ks == 0) p_pair(KSTEPS == 4 ? 4 + ks : 4);
            if (KSTEPS == 2 && ks == 1) p_pair(6);
            __builtin_amdgcn_sched_barrier(0);
            dp[1][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1, v0, ks == 0 ? nd[1] : dp[1][0], 0, 0, 0);
            dp[1][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1, v1, ks == 0 ? nd[1] : dp[1][1], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (ks + 1 < KSTEPS) {
                v0 = TL::rows(smem, vrows0, 0, ks + 1);
                v1 = TL::rows(smem, vrows0, 1, ks + 1);
            } else {
                v0 = TL::transposed(smem + HB, cols0, 1);
            }
            if (KSTEPS == 2) p_pair(ks == 0 ? 5 : 7);
            __builtin_amdgcn_sched_barrier(0);
        }
        bf16x8_t pf[2], df[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) pf[kt] = __builtin_bit_cast(bf16x8_t, u32x4_t{pw[kt][0], pw[kt][1], pw[kt][2], pw[kt][3]});
        op[0] = x0;
        op[1] = v0;
#pragma unroll
        for (int n = 0; n < 2 * CT; ++n) {
            const int ct = n % CT, n2 = n + 2;
            if (n2 < 2 * CT) op[n2 & 3] = TL::transposed(n2 < CT ? smem + HB : smem, cols0, n2 % CT);
            if (n == CT) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const float d8[8] = {dp[0][kt][0], dp[0][kt][1], dp[0][kt][2], dp[0][kt][3], dp[1][kt][0], dp[1][kt][1], dp[1][kt][2], dp[1][kt][3]};
                    df[kt] = pack8(d8);
                }
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                if (n < CT) dv[ct][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n & 3], pf[kt], dv[ct][kt], 0, 0, 0);
                else dk[ct][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[n & 3], df[kt], dk[ct][kt], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (n < CT) {
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (v * CT / 16 == n) ds_value(v);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        }
        VMOBA_WAIT_VMCNT(0);
        __syncthreads();
        c = c_next;
        par ^= 1;
    }
    if (!careful) {
        float z = 0.f;                                    // NaN if a sum is not finite
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = fmaf(dk[ct][kt][i], 0.f, fmaf(dv[ct][kt][i], 0.f, z));
        if (__builtin_expect(z != 0.f, 0)) words[0] = 1;
        __syncthreads();
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(words[0]) != 0, 0)) {
            careful = true;
            walk.window = -64;
            goto again;
        }
    }
    const float scale_k = CAP ? 4.f * a.scale : a.scale;
    if (a.splits > 1) {                                   // this split's sums, added up by dense_sum_kernel
        const long long n = (long long)a.B * a.Hkv * a.Sk;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int key = kw + 16 * kt + l16;
            if (key < a.Sk) {
                float* dst = a.part_o + (2 * task.split * n + (long long)bh * a.Sk + key) * D + 4 * g;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    *reinterpret_cast<f32x4_t*>(dst + 16 * ct) = dk[ct][kt] * scale_k;
                    *reinterpret_cast<f32x4_t*>(dst + n * D + 16 * ct) = dv[ct][kt];
                }
            }
        }
        return;
    }
    char* mine = smem + wave * 32 * OPITCH;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const TensorView& out = which == 0 ? a.dV : a.dK;
        const float f = which == 0 ? 1.f : scale_k;
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

#define BY_SCORES(KERNEL)                                                              \
    do {                                                                               \
        if (cap && a.slopes) KERNEL<D, true, true><<<grid, block, 0, st>>>(a);         \
        else if (cap) KERNEL<D, true, false><<<grid, block, 0, st>>>(a);               \
        else if (a.slopes) KERNEL<D, false, true><<<grid, block, 0, st>>>(a);          \
        else KERNEL<D, false, false><<<grid, block, 0, st>>>(a);                       \
    } while (0)
template <int D>
void launch_dq(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.M, 128) * a.splits, a.Hkv)), block(256);
    BY_SCORES(dense_dq_kernel);
}
template <int D>
void launch_dkv(bool cap, hipStream_t st, const DenseArgs& a) {
    const dim3 grid(dense_grid((int64_t)a.B * ceil_div64(a.Sk, 128) * a.splits, a.Hkv)), block(256);
    BY_SCORES(dense_dkv_kernel);
}

}  // namespace

void launch_dense_dq_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_dq<128>(cap, st, a) : launch_dq<64>(cap, st, a); }
void launch_dense_dkv_bf16(int D, bool cap, hipStream_t st, const DenseArgs& a) { D == 128 ? launch_dkv<128>(cap, st, a) : launch_dkv<64>(cap, st, a); }
