// Products of shares with public 4-bit weights: z[m][n] = sum over k of x[m][k] w[n][k], w[n][k] = q[n][k] s[n][k / group]
// with q in [-8, 7] and s a fixed-point integer.  Linear in the shares with public factors: every party multiplies its own
// words, with no triple and no exchange, and rescales by the scale's fraction bits.
//
// On the matrix cores the weights are the left operand, 16 rows, and a row of x is the right one: its 16 columns are the eight
// digits of both parties' words, so one 16 x 16 x 64 product serves a whole row.  The digit sums of a group are exact in 32
// bits, times the group's scale they are added up in 64, and the eight digits join at the end.  One row of 25088 x 4096 takes
// 16 to 18 us (51 MB of weights, 2.9 to 3.2 TB/s): every workgroup also reads x, twice the bytes of its weights out of the L2, and without either
// of the two it takes 12.  Several rows are bound by the digits' and the scales' vector instructions, few weights by latency.  Many
// rows (a prompt's) are far from their bytes: every 16 rows of the weights read all digits of x again, 4096 x 768 x 2304 694 us for
// 202 MB, 4096 x 768 x 768 280.
#include "attention.h"
#include "digits.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

struct MatvecArgs {
    const u64* x[2]; u64* z[2];
    const u8* w; const int32_t* scales;
    uint32_t* digits;                     // digits in memory, or none
    u64* partial;                         // [split][row][party][N], where the columns are split over workgroups
    int M, K, N, group, groups, row_bytes, shift, blocks, splits;
};

constexpr int kBlock = 256;                   // columns that a wave takes at a time
constexpr int kUnits = 256, kLong = 4;
constexpr int kMostN = 1 << 25;               // 2^21 workgroups of up to 1024 threads
constexpr int most_waves(int mt) { return mt == 1 ? 16 : 8; }

// Whether the digits of x are made once, by a launch of their own, instead of by every workgroup for itself.  us with and without:
// 8 x 25088 x 4096 50 / 76, 16 x 4096 x 4096 30 / 44; but 4 x 4096 x 4096 12 / 12, 8 x 1024 x 4096 13 / 11, 1 x 768 x 2304 7 / 4.
bool small(int M, int K, int N) { return (long long)M * K * N < 1ll << 27; }
bool digits_in_memory(int M, int K, int N) { return M > 4 && !small(M, K, N); }

// Rows of x to a workgroup; launch() takes two of four where that is faster, us with four and two: 16 x 768 x 2304 12 / 10,
// 4 x 768 x 768 6.7 / 4.8, but for larger products 4 x 25088 x 4096 40 / 43 and for groups of 32 4 x 4096 x 4096 15 / 20.
int rows_at_once(int M, int K, int N) { return digits_in_memory(M, K, N) ? 8 : M < 3 ? M : 4; }
// Into how many workgroups the columns are split: few rows of the weights that are long leave most units idle, and a workgroup's
// waves go through several blocks one after the other.  The sums are added by a launch of their own.  us without and with, groups of
// 128: 1 x 25088 x 10 14 / 8, 1 x 25088 x 1000 17 / 13, 8 x 25088 x 200 22 / 17; but for more than kUnits workgroups 1 x 25088 x 4096
// 18 / 21, and for fewer than kLong blocks to a wave 16 x 4096 x 1000 12 / 18.
int splits_of(int M, int K, int N)
{
    const int mt = rows_at_once(M, K, N), blocks = (K + kBlock - 1) / kBlock, waves = most_waves(mt);
    const long long workgroups = (N + 15ll) / 16 * ((M + mt - 1) / mt);
    if (blocks < kLong * waves || workgroups >= kUnits) return 1;
    const int splits = (int)((kUnits + workgroups - 1) / workgroups), most = blocks / waves;
    return splits < most ? splits : most;
}

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

// The same digits in memory, made once for all workgroups: what a lane needs of a block, 16 dwords, as four pieces of 16 bytes,
// [row][block][piece][lane].
template <int G> __global__ __launch_bounds__(256) void k_digits4(MatvecArgs q)
{
    const int g8 = threadIdx.x % 32, party = threadIdx.x / 32 % 2, block = blockIdx.x * 4 + threadIdx.x / 64, m = blockIdx.y;
    if (block >= q.blocks) return;
    u64 v[8];
    const u64* const row = q.x[party] + (size_t)m * q.K;
#pragma unroll
    for (int j = 0; j < 8; ++j) { const int k = block * kBlock + g8 * 8 + j; const u64 t = row[min(k, q.K - 1)]; v[j] = k < q.K ? t : 0; }
    uint32_t* const to = q.digits + ((size_t)m * q.blocks + block) * 1024;
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
        const u64 four[4] = { v[odd], v[2 + odd], v[4 + odd], v[6 + odd] };
        uint32_t d[8];
        digits_of_4(four, d);
        const int i = G == 128 ? g8 / 16 * 8 + odd * 4 + g8 % 4 : G == 64 ? g8 / 8 * 4 + odd * 2 + g8 % 2 : g8 / 4 * 2 + odd;
        const int kg = G == 128 ? g8 % 16 / 4 : G == 64 ? g8 % 8 / 2 : g8 % 4;
#pragma unroll
        for (int p = 0; p < 8; ++p) to[i / 4 * 256 + (kg * 16 + party * 8 + p) * 4 + i % 4] = d[p];
    }
}

// What lanes of a wave hand to one another through LDS: the hardware has a wave's accesses in order, and the compiler keeps them so.
__device__ __forceinline__ void wave_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// A workgroup has 16 rows of the weights and MT rows of x; its waves share the columns, a block at a time.  MADE: the digits are
// in memory, else a wave makes those of its blocks.
template <int G, int MT, bool MADE>
__global__ __launch_bounds__(64 * most_waves(MT)) void k_matvec4(MatvecArgs q)
{
    typedef Digits<G> D;
    constexpr int kBytes = G / 8;                                       // of weights of a lane and a set
    __shared__ uint32_t digits[MADE ? 1 : most_waves(MT)][MADE ? 1 : D::total];
    __shared__ u64 sums[most_waves(MT)][MT][16][2];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), waves = blockDim.x / 64, lane = threadIdx.x % 64;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * MT, kg = lane / 16;
    const u8* const w_row = q.w + (size_t)min(n0 + lane % 16, q.N - 1) * q.row_bytes;
    const int party = lane / 32, g8 = lane % 32;
    const u64* const x = q.x[party];
    uint32_t* const mine = digits[MADE ? 0 : wave];
    int64_t z[MT][4] = {};
    union Right { u64 words[8]; uint32_t d[16]; };                      // eight words to be made into digits, or a lane's digits
    const auto right = [&](int block, int m) {
        const int at_m = min(m0 + m, q.M - 1);
        Right v;
        if constexpr (MADE) {
            const uint32_t* const from = q.digits + ((size_t)at_m * q.blocks + block) * 1024 + lane * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<i32x4*>(v.d + i * 4) = *reinterpret_cast<const i32x4*>(from + i * 256);
        } else {
            const int k = block * kBlock + g8 * 8;
            const u64* const row = x + (size_t)at_m * q.K;
            if (block * kBlock + kBlock <= q.K)
#pragma unroll
                for (int j = 0; j < 8; j += 2) { const u64x2u t = *reinterpret_cast<const u64x2u*>(row + k + j); v.words[j] = t.x; v.words[j + 1] = t.y; }
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) { const u64 t = row[min(k + j, q.K - 1)]; v.words[j] = k + j < q.K ? t : 0; }
        }
        return v;
    };
    const int per = (q.blocks + q.splits - 1) / q.splits, first = blockIdx.z * per, last = min(first + per, q.blocks);
    for (int block = first + wave; block < last; block += waves) {
        const int k0 = block * kBlock;
        Right next = right(block, 0);
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
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const Right v = next;
            if (m + 1 < MT) next = right(block, m + 1);                 // one row ahead, and no further: registers
            if constexpr (!MADE) {
#pragma unroll
                for (int odd = 0; odd < 2; ++odd) {
                    const u64 four[4] = { v.words[odd], v.words[2 + odd], v.words[4 + odd], v.words[6 + odd] };
                    uint32_t d[8];
                    digits_of_4(four, d);
#pragma unroll
                    for (int p = 0; p < 8; ++p) mine[D::at(party, g8, odd) + p * D::dwords] = d[p];
                }
                wave_in_order();
            }
#pragma unroll
            for (int s = 0; s < D::sets; ++s) {
                uint32_t b[G == 128 ? 8 : D::dwords];
                if constexpr (MADE) {
#pragma unroll
                    for (int i = 0; i < (int)(sizeof(b) / 4); ++i) b[i] = v.d[s * (sizeof(b) / 4) + i];
                } else {
                    const uint32_t* const at = mine + s * D::set + kg * D::row + lane % 16 * D::dwords;
#pragma unroll
                    for (int i = 0; i < (int)(sizeof(b) / 4); ++i) b[i] = at[i / 4 * 4 * D::row + i % 4];
                }
                i32x4 acc = { 0, 0, 0, 0 };
                const auto low = [&](int i) { return (int)((w[i] << 4) & 0xf0f0f0f0u); };      // 16 q of the even columns, of the odd ones
                const auto high = [&](int i) { return (int)(w[i] & 0xf0f0f0f0u); };
                const auto four = [&](int i) { return i32x4{ (int)b[i], (int)b[i + 1], (int)b[i + 2], (int)b[i + 3] }; };
                if constexpr (G == 128) {
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ low(s * 4), low(s * 4 + 1), low(s * 4 + 2), low(s * 4 + 3) }, four(0), acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ high(s * 4), high(s * 4 + 1), high(s * 4 + 2), high(s * 4 + 3) }, four(4), acc, 0, 0, 0);
                } else if constexpr (G == 64)
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{ low(s * 2), low(s * 2 + 1), high(s * 2), high(s * 2 + 1) }, four(0), acc, 0, 0, 0);
                else
                    acc = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)((u64)(uint32_t)high(s) << 32 | (uint32_t)low(s)), (long)((u64)b[1] << 32 | b[0]), acc, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) z[m][r] += (int64_t)(acc[r] >> 4) * scale[s][r];   // the sixteenth is exact
            }
            if constexpr (!MADE) wave_in_order();                       // read, before the next row's or block's are written
            if (MT > 1) __builtin_amdgcn_sched_barrier(0);
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
        if (m0 + m >= q.M || n0 + n >= q.N) continue;
        if (q.splits > 1) q.partial[(((size_t)blockIdx.z * q.M + m0 + m) * 2 + p) * q.N + n0 + n] = v;
        else q.z[p][(size_t)(m0 + m) * q.N + n0 + n] = rescaled(p, v, q.shift);
    }
}

// the splits' sums
__global__ __launch_bounds__(256) void k_matvec4_join(MatvecArgs q)
{
    const size_t n = 2 * (size_t)q.M * q.N, at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= n) return;
    const size_t m = at / q.N / 2, p = at / q.N % 2;
    u64 v = 0;
    for (int i = 0; i < q.splits; ++i) v += q.partial[(size_t)i * n + at];
    q.z[p][m * q.N + at % q.N] = rescaled((int)p, v, q.shift);
}

template <int G, int MT, bool MADE> void launch(const MatvecArgs& q, hipStream_t st)
{
    const int waves = q.blocks < most_waves(MT) ? q.blocks : most_waves(MT);
    k_matvec4<G, MT, MADE><<<dim3((q.N + 15) / 16, (q.M + MT - 1) / MT, q.splits), 64 * waves, 0, st>>>(q);
    if (q.splits > 1) k_matvec4_join<<<dim3((unsigned)((2 * (size_t)q.M * q.N + 255) / 256)), 256, 0, st>>>(q);
}
template <int G> void launch(const MatvecArgs& q, hipStream_t st)
{
    if (digits_in_memory(q.M, q.K, q.N)) {
        k_digits4<G><<<dim3((q.blocks + 3) / 4, q.M), 256, 0, st>>>(q);
        launch<G, 8, true>(q, st);
    }
    else if (q.M == 1) launch<G, 1, false>(q, st);
    else if (q.M == 2 || (G > 32 && small(q.M, q.K, q.N))) launch<G, 2, false>(q, st);
    else launch<G, 4, false>(q, st);
}

}  // namespace

extern "C" {

size_t mpc_matvec4_workspace_bytes(int M, int K, int N)
{
    if (M <= 0 || K <= 0 || N <= 0 || K > MPC_MAX_K_TOTAL || M > 65535 || N > kMostN) return 0;
    const int splits = splits_of(M, K, N);
    return (digits_in_memory(M, K, N) ? (size_t)M * ((K + kBlock - 1) / kBlock) * 4096 : 0) + (splits > 1 ? 16 * (size_t)splits * M * N : 0);
}

int mpc_matvec4(mpc_ctx* c, mpc_cshare x, const uint8_t* w, const int32_t* scales, mpc_share z,
                int M, int K, int N, int group, int scale_bits)
{
    if (!c || !w || !scales || M <= 0 || K <= 0 || N <= 0 || scale_bits < 0 || scale_bits > 31) return MPC_EINVAL;
    if (group <= 0 || (group != 32 && group != 64 && group % 128)) return MPC_EINVAL;
    if (((uintptr_t)w & 15) || ((uintptr_t)scales & 3)) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) if (!x.p[i] || !z.p[i]) return MPC_EINVAL;
    if (K > MPC_MAX_K_TOTAL || M > 65535 || N > kMostN) return MPC_ERANGE;
    MatvecArgs q{};
    q.groups = K / group + (K % group != 0); q.row_bytes = (K + 31) / 32 * 16;
    const size_t out = (size_t)M * N * 8;
    if (!outputs_apart(z, out, x, (size_t)M * K * 8, false)) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) {
        q.x[i] = x.p[i]; q.z[i] = z.p[i];
    }
    if (!apart(z, out, w, (size_t)N * q.row_bytes) || !apart(z, out, scales, (size_t)N * q.groups * 4)) return MPC_EINVAL;
    q.w = w; q.scales = scales; q.M = M; q.K = K; q.N = N; q.group = group; q.shift = scale_bits;
    q.blocks = (K + kBlock - 1) / kBlock;
    q.splits = splits_of(M, K, N);
    const size_t need = mpc_matvec4_workspace_bytes(M, K, N), partial = q.splits > 1 ? 16 * (size_t)q.splits * M * N : 0;
    if (need) {
        if (!c->ws || c->ws_bytes < need) return MPC_ENOMEM;
        q.digits = reinterpret_cast<uint32_t*>(c->ws);                 // a multiple of 4 KB, if any
        q.partial = reinterpret_cast<u64*>(reinterpret_cast<u8*>(c->ws) + (need - partial));
    }
    MPC_TRY(lane_first(c));
    if (group == 32) launch<32>(q, c->s[0]);
    else if (group == 64) launch<64>(q, c->s[0]);
    else launch<128>(q, c->s[0]);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
