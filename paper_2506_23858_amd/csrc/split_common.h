// Float32 operands as three bfloat16 terms each: pieces shared by the block-sparse (attn_split.hip, which derives them) and the dense
// (dense_split.hip) kernels on the bfloat16 matrix instruction.
#pragma once
#include "attn_common.h"

constexpr float LIFT = 0x1p16f, UNLIFT = 0x1p-16f;                                // of weights and dS
constexpr uint32_t SMALLEST = 27u << 23, TOO_LARGE = 153u << 23;                  // 2^-100 and 2^26 as float bits

// A value that three terms do not hold: neither 0 nor of a magnitude from 2^-100 up to 2^26
__device__ __forceinline__ bool outside_terms(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u && u - SMALLEST >= TOO_LARGE - SMALLEST;
}
// two floats -> their bfloat16 pairs h, m, l (low half = a)
__device__ __forceinline__ void split2(float a, float b, uint32_t& h, uint32_t& m, uint32_t& l) {
    h = pack_bf16x2(a, b);
    const float ra = a - bf16lo_to_f32(h), rb = b - bf16hi_to_f32(h);
    m = pack_bf16x2(ra, rb);
    l = pack_bf16x2(ra - bf16lo_to_f32(m), rb - bf16hi_to_f32(m));
}

// The terms of 16 values per lane in accumulator order, as the B operand of a product over the tile's rows: filled pair by pair.
struct Terms {
    uint32_t t[3][8];
    __device__ __forceinline__ void pair(int j, float a, float b) {
        split2(a, b, t[0][j], t[1][j], t[2][j]);
        asm volatile("" : "+v"(t[0][j]), "+v"(t[1][j]), "+v"(t[2][j]));       // here, not where it is used
    }
    __device__ __forceinline__ void operand(int s, bf16x8_t (&b)[3]) const {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const u32x4_t u = {t[p][4 * s], t[p][4 * s + 1], t[p][4 * s + 2], t[p][4 * s + 3]};
            b[p] = __builtin_bit_cast(bf16x8_t, u);
        }
    }
};
// c += a . b by terms, small products first.  SWAP: in the order of c += b . a, so that a product computed with its operands the other
// way round has the same rounding errors (the weights that dK/dV recomputes then match the LSE they are normalised by).
template <bool SWAP>
__device__ __forceinline__ f32x16_t mfma6(const bf16x8_t (&a)[3], const bf16x8_t (&b)[3], f32x16_t c) {
    constexpr int X = SWAP ? 0 : 2, Y = SWAP ? 0 : 1;
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[X], b[2 - X], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2 - X], b[X], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[Y], b[1 - Y], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1 - Y], b[Y], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], c, 0, 0, 0);
}

// Tiles of 32 rows x 3 planes in LDS (plane p of a tile HB bytes after plane p - 1) and the requests that fill them.
template <int D>
struct SplitTile : RowTile<D> {
    using TL = RowTile<D>;
    static constexpr int KSTEPS = D / 16, DT = D / 32;
    static constexpr int TILE = 3 * TL::HB;
    static constexpr int REQ = 3 * 32 / TL::RPI;         // requests per tile, shared by four wavefronts
    static constexpr int IPW = REQ / 4;
    static_assert(IPW * 4 == REQ, "equal shares");
    uint32_t rl[TL::NRB], tl[2][TL::NTB];
    __device__ __forceinline__ SplitTile(int lane) {
#pragma unroll
        for (int k = 0; k < TL::NRB; ++k) rl[k] = TL::row_lane(lane, k);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int dt = 0; dt < TL::NTB; ++dt) tl[t][dt] = TL::tr_lane(lane, t, dt);
    }
    __device__ __forceinline__ void rows3(const char* tile, int ks, bf16x8_t (&a)[3]) const {
#pragma unroll
        for (int p = 0; p < 3; ++p) a[p] = TL::rows(tile + p * TL::HB, rl, 0, ks);
    }
    __device__ __forceinline__ void transposed3(const char* tile, int u, bf16x8_t (&a)[3]) const {
#pragma unroll
        for (int p = 0; p < 3; ++p) a[p] = TL::transposed(tile + p * TL::HB, tl, 0, u / DT, u % DT);
    }
    // request i of wavefront `wave` for a tile at LDS address lds: row (of 32) this lane's lanes fetch, and the plane
    __device__ static __forceinline__ int req_row(int wave, int i, int lane) { return (wave * IPW + i) % (32 / TL::RPI) * TL::RPI + lane / TL::PPR; }
    __device__ static __forceinline__ int req_plane(int wave, int i) { return (wave * IPW + i) / (32 / TL::RPI); }
    __device__ static __forceinline__ uint32_t req_lds(int wave, int i) {
        return (uint32_t)(req_plane(wave, i) * TL::HB + (wave * IPW + i) % (32 / TL::RPI) * TL::GP);
    }
    // Vector work of eight value pairs goes between the matrix instructions of a product, PAIRS pairs after every group of six
    // (a wavefront alone on its SIMD would leave the matrix pipe idle for it).
    static constexpr int PAIRS = 8 / KSTEPS;
    static_assert(KSTEPS == 2 * DT, "as many groups in a product over channels as over rows");
    // product over channels: [row rho, column] = tile . f; side(pair) as above
    template <bool SWAP = false, class F>
    __device__ __forceinline__ f32x16_t over_channels(const char* tile, const bf16x8_t (&f)[3][KSTEPS], F&& side) const {
        f32x16_t acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bf16x8_t a[2][3];
        rows3(tile, 0, a[0]);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            if (ks + 1 < KSTEPS) rows3(tile, ks + 1, a[(ks + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
            const bf16x8_t b[3] = {f[0][ks], f[1][ks], f[2][ks]};
            acc = mfma6<SWAP>(a[ks & 1], b, acc);
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) side(ks * PAIRS + j);
            __builtin_amdgcn_sched_barrier(0);
        }
        return acc;
    }
    // product over the tile's rows: acc[dt] += tile^T . w.  With LATE the second half of w's pairs is filled by `side` on the way
    // (side(pair) for pairs 4 .. 7), otherwise w is complete and side runs over all eight pairs of something else.
    template <bool LATE, class F>
    __device__ __forceinline__ void over_rows(const char* tile, const Terms& w, f32x16_t (&acc)[DT], F&& side) const {
        bf16x8_t b[3], a[2][3];
        transposed3(tile, 0, a[0]);
#pragma unroll
        for (int u = 0; u < 2 * DT; ++u) {
            if (u + 1 < 2 * DT) transposed3(tile, u + 1, a[(u + 1) & 1]);
            if (u % DT == 0) w.operand(u / DT, b);
            __builtin_amdgcn_sched_barrier(0);
            acc[u % DT] = mfma6<false>(a[u & 1], b, acc[u % DT]);
            if constexpr (LATE) {
                if (u < DT)
#pragma unroll
                    for (int j = 0; j < 4 / DT; ++j) side(4 + u * (4 / DT) + j);
            } else {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) side(u * PAIRS + j);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

template <int D>
__device__ __forceinline__ void load_terms(const char* row, int hf, bf16x8_t (&f)[3][D / 16]) {
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) f[p][ks] = *reinterpret_cast<const bf16x8_t*>(row + (p * D + ks * 16 + hf * 8) * 2);
}
