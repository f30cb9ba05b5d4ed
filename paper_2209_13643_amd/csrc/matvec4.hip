// Products of shares with public 4-bit weights: z[m][n] = sum over k of x[m][k] w[n][k], w[n][k] = q[n][k] s[n][k / group]
// with q in [-8, 7] and s a fixed-point integer.  Linear in the shares with public factors: every party multiplies its own
// words, with no triple and no exchange, and rescales by the scale's fraction bits.
//
// On the matrix cores the weights are the left operand, 16 rows, and a row of x is the right one: its 16 columns are the eight
// digits of both parties' words, so one 16 x 16 x 64 product serves a whole row.  The digit sums of a group are exact in 32
// bits, times the group's scale they are added up in 64, and the eight digits join at the end.  Bound by reading the weights
// (25088 x 4096: 51 MB) where there are many, by latency and the scales' 64-bit products where there are few.
#include "attention.h"
#include "digits.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

struct MatvecArgs {
    const u64* x[2]; u64* z[2];
    const u8* w; const int32_t* scales;
    int M, K, N, group, groups, row_bytes, shift;
};

constexpr int kBlock = 256;                   // columns that a wave takes at a time
constexpr int most_waves(int mt) { return mt <= 2 ? 16 : 8; }

// The digits of a block of x in LDS, as the lanes of a product read them: for every set of G columns (kg: a quarter of them) and
// column c = 8 party + digit, the words' bytes in the order in which a lane's weights come out of their halves, even columns
// first.  Rows are padded so that the stores of 64 lanes spread over the banks.
template <int G> struct Digits {
    static constexpr int sets = kBlock / G;
    static constexpr int dwords = G == 32 ? 2 : 4;                      // of a lane and a product
    static constexpr int row = 16 * dwords + (G == 32 ? 2 : 4);         // dwords of a quarter
    static constexpr int set = G == 128 ? 8 * row + 16 : G == 64 ? 4 * row + 64 - 4 * row % 64 + 16 : 4 * row;
    static constexpr int total = sets * set;
    // place of digit q of eight words from column 8 g8, even (0) or odd (1) ones
    __device__ static __forceinline__ int at(int party, int g8, int odd)
    {
        if (G == 128) return g8 / 16 * set + (odd * 4 + g8 % 16 / 4) * row + party * 32 + g8 % 4;
        if (G == 64) return g8 / 8 * set + g8 % 8 / 2 * row + party * 32 + odd * 2 + g8 % 2;
        return g8 / 4 * set + g8 % 4 * row + party * 16 + odd;
    }
};

// A workgroup has 16 rows of the weights and MT rows of x; its waves share the columns, a block at a time.
template <int G, int MT>
__global__ __launch_bounds__(64 * most_waves(MT)) void k_matvec4(MatvecArgs q)
{
    typedef Digits<G> D;
    constexpr int kBytes = G / 8;                                       // of weights of a lane and a set
    __shared__ uint32_t digits[most_waves(MT)][D::total];
    __shared__ u64 sums[most_waves(MT)][MT][16][2];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), waves = blockDim.x / 64, lane = threadIdx.x % 64;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * MT, kg = lane / 16;
    const u8* const w_row = q.w + (size_t)min(n0 + lane % 16, q.N - 1) * q.row_bytes;
    const int party = lane / 32, g8 = lane % 32;
    const u64* const x = q.x[party];
    uint32_t* const mine = digits[wave];
    int64_t z[MT][4] = {};
    for (int k0 = wave * kBlock; k0 < q.K; k0 += waves * kBlock) {
        uint32_t w[8];                                                  // [set][kBytes / 4]
        int scale[D::sets][4];
#pragma unroll
        for (int s = 0; s < D::sets; ++s) {
            const int at = min(k0 / 2 + s * (G / 2) + kg * kBytes, q.row_bytes - kBytes);      // beyond the row the digits are zero
            if (G == 128) *reinterpret_cast<i32x4*>(w + s * 4) = *reinterpret_cast<const i32x4*>(w_row + at);
            else if (G == 64) *reinterpret_cast<i32x2*>(w + s * 2) = *reinterpret_cast<const i32x2*>(w_row + at);
            else w[s] = *reinterpret_cast<const uint32_t*>(w_row + at);
            const int g = min((k0 + s * G) / q.group, q.groups - 1);
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[s][r] = q.scales[(size_t)min(n0 + kg * 4 + r, q.N - 1) * q.groups + g];
        }
        struct Eight { u64 w[8]; };
        const auto words = [&](int m) {
            const int k = k0 + g8 * 8;
            const u64* const row = x + (size_t)min(m0 + m, q.M - 1) * q.K;
            Eight v;
            if (k0 + kBlock <= q.K)
#pragma unroll
                for (int j = 0; j < 8; j += 2) { const u64x2u t = *reinterpret_cast<const u64x2u*>(row + k + j); v.w[j] = t.x; v.w[j + 1] = t.y; }
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) { const u64 t = row[min(k + j, q.K - 1)]; v.w[j] = k + j < q.K ? t : 0; }
            return v;
        };
        Eight next = words(0);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const Eight v = next;
            if (m + 1 < MT) next = words(m + 1);                        // one row ahead, and no further: registers
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const u64 four[4] = { v.w[odd], v.w[2 + odd], v.w[4 + odd], v.w[6 + odd] };
                uint32_t d[8];
                digits_of_4(four, d);
#pragma unroll
                for (int p = 0; p < 8; ++p) mine[D::at(party, g8, odd) + p * D::dwords] = d[p];
            }
            __builtin_amdgcn_wave_barrier();                            // one wave: its LDS accesses are in order
#pragma unroll
            for (int s = 0; s < D::sets; ++s) {
                const uint32_t* const at = mine + s * D::set + kg * D::row + lane % 16 * D::dwords;
                i32x4 acc = { 0, 0, 0, 0 };
                const auto low = [&](int i) { return (int)((w[i] << 4) & 0xf0f0f0f0u); };      // 16 q of the even columns, of the odd ones
                const auto high = [&](int i) { return (int)(w[i] & 0xf0f0f0f0u); };
                if constexpr (G == 128) {
                    const i32x4 even = *reinterpret_cast<const i32x4*>(at), odd = *reinterpret_cast<const i32x4*>(at + 4 * D::row);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ low(s * 4), low(s * 4 + 1), low(s * 4 + 2), low(s * 4 + 3) }, even, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ high(s * 4), high(s * 4 + 1), high(s * 4 + 2), high(s * 4 + 3) }, odd, acc, 0, 0, 0);
                } else if constexpr (G == 64) {
                    const i32x4 b = *reinterpret_cast<const i32x4*>(at);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ low(s * 2), low(s * 2 + 1), high(s * 2), high(s * 2 + 1) }, b, acc, 0, 0, 0);
                } else {
                    const long b = *reinterpret_cast<const long*>(at);
                    const long a = (long)((u64)(uint32_t)high(s) << 32 | (uint32_t)low(s));
                    acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, acc, 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) z[m][r] += (int64_t)(acc[r] >> 4) * scale[s][r];   // the sixteenth is exact
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // lane: column c = 8 party + digit of the product, rows 4 kg + r
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            u64 v = (u64)z[m][r] << (lane % 8 * 8);
#pragma unroll
            for (int d = 1; d < 8; d *= 2) v += (u64)__shfl_xor((unsigned long long)v, d);
            if (lane % 8 == 0) sums[wave][m][kg * 4 + r][lane % 16 / 8] = v;
        }
    __syncthreads();
    for (int t = threadIdx.x; t < MT * 32; t += blockDim.x) {
        const int m = t / 32, n = t % 16, p = t / 16 % 2;
        u64 v = 0;
        for (int i = 0; i < waves; ++i) v += sums[i][m][n][p];
        if (m0 + m < q.M && n0 + n < q.N) q.z[p][(size_t)(m0 + m) * q.N + n0 + n] = rescaled(p, v, q.shift);
    }
}

template <int G, int MT> void launch(const MatvecArgs& q, hipStream_t st)
{
    const int blocks = (q.K + kBlock - 1) / kBlock, waves = blocks < most_waves(MT) ? blocks : most_waves(MT);
    k_matvec4<G, MT><<<dim3((q.N + 15) / 16, (q.M + MT - 1) / MT), 64 * waves, 0, st>>>(q);
}
template <int G> void launch(const MatvecArgs& q, hipStream_t st)
{
    if (q.M == 1) launch<G, 1>(q, st);
    else if (q.M == 2) launch<G, 2>(q, st);
    else if (q.M <= 4) launch<G, 4>(q, st);
    else launch<G, 8>(q, st);
}

}  // namespace

extern "C" {

int mpc_matvec4(mpc_ctx* c, mpc_cshare x, const uint8_t* w, const int32_t* scales, mpc_share z,
                int M, int K, int N, int group, int scale_bits)
{
    if (!c || !w || !scales || M <= 0 || K <= 0 || N <= 0 || scale_bits < 0 || scale_bits > 31) return MPC_EINVAL;
    if (group <= 0 || (group != 32 && group != 64 && group % 128)) return MPC_EINVAL;
    if (((uintptr_t)w & 15) || ((uintptr_t)scales & 3)) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) if (!x.p[i] || !z.p[i]) return MPC_EINVAL;
    if (K > MPC_MAX_K_TOTAL || M > 65535) return MPC_ERANGE;
    MatvecArgs q{};
    q.groups = (K + group - 1) / group; q.row_bytes = (K + 31) / 32 * 16;
    const size_t out = (size_t)M * N * 8;
    if (!outputs_apart(z, out, x, (size_t)M * K * 8, false)) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) {
        q.x[i] = x.p[i]; q.z[i] = z.p[i];
        if (overlap(z.p[i], out, w, (size_t)N * q.row_bytes) || overlap(z.p[i], out, scales, (size_t)N * q.groups * 4)) return MPC_EINVAL;
    }
    q.w = w; q.scales = scales; q.M = M; q.K = K; q.N = N; q.group = group; q.shift = scale_bits;
    MPC_TRY(lane_first(c));
    if (group == 32) launch<32>(q, c->s[0]);
    else if (group == 64) launch<64>(q, c->s[0]);
    else launch<128>(q, c->s[0]);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
