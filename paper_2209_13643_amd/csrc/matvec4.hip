// Products of shares with public 4-bit weights: z[m][n] = sum over k of x[m][k] w[n][k], w[n][k] = q[n][k] s[n][k / group]
// with q in [-8, 7] and s a fixed-point integer.  Linear in the shares with public factors: every party multiplies its own
// words, with no triple and no exchange, and rescales by the scale's fraction bits.
#include "attention.h"

namespace {

constexpr int kWaves = 4;

struct MatvecArgs {
    const u64* x[2]; u64* z[2];
    const u8* w; const int32_t* scales;
    int M, K, N, group, groups, row_bytes, shift;
};

__global__ __launch_bounds__(64 * kWaves) void k_matvec4(MatvecArgs q)
{
    const int n = blockIdx.x * kWaves + threadIdx.x / 64, m = blockIdx.y, lane = threadIdx.x % 64;
    if (n >= q.N) return;
    u64 z[2] = { 0, 0 };
    for (int k0 = lane * 8; k0 < q.K; k0 += 64 * 8) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(q.w + (size_t)n * q.row_bytes + k0 / 2);
        const u64 s = (u64)(int64_t)q.scales[(size_t)n * q.groups + k0 / q.group];
        for (int t = 0; t < 8 && k0 + t < q.K; ++t) {
            const u64 f = s * (u64)(int64_t)((int32_t)(w << (28 - 4 * t)) >> 28);
            for (int p = 0; p < 2; ++p) z[p] += f * q.x[p][(size_t)m * q.K + k0 + t];
        }
    }
    for (int p = 0; p < 2; ++p)
        for (int d = 32; d; d >>= 1) z[p] += __shfl_xor((unsigned long long)z[p], d);
    if (lane < 2) q.z[lane][(size_t)m * q.N + n] = rescaled(lane, lane ? z[1] : z[0], q.shift);
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
    k_matvec4<<<dim3((N + kWaves - 1) / kWaves, M), 64 * kWaves, 0, c->s[0]>>>(q);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
