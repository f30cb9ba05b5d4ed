// Learned relative position bias on shares, and its gradient.  Both are linear in the shares, so every party works on its
// own words: no triple, no exchange, no rescale.
//   y[b,h,i,j] = x[b,h,i,j] + table[m(j-i)][h]         m: public bucket of a distance; none: y = 0
//   table_grad[u][h] = sum over b and all (i,j) with m(j-i) = u of g[b,h,i,j],   x_grad = g where there is a bucket, else 0
// Sums are exact mod 2^64, whatever their order.  Bound by HBM: one read and one write of every pair (the table's gradient
// alone: one read).
#include "attention.h"

namespace {

constexpr int kThreads = 256;
constexpr int kCols = 1024;              // columns of a tile, at most
constexpr int kRows = 512;               // rows of a tile, at most
constexpr int kTilePairs = 8192;         // (i, j) pairs of a tile, at most

struct BiasArgs {
    const u64* x[2]; const u64* table[2]; const int32_t* buckets; u64* out[2];
    u64* grad[2];                        // gradient only
    unsigned BH, H, Tq, Tk; int n_buckets;
    unsigned rows, cols, row_tiles, col_tiles;      // a tile is rows x cols
    unsigned B, batches;                            // gradient: matrices of one head, and how many of them a workgroup sums
};

// What the distances of a tile add, and where nothing is kept: entry k is distance j - i = j0 - i0 - (rows - 1) + k.
__global__ __launch_bounds__(kThreads) void k_position_bias(BiasArgs q)
{
    // (word, kept mask); rows + cols is largest at either end of cols: kCols + kTilePairs / kCols, kRows + kTilePairs / kRows
    __shared__ ulonglong2 by_distance[kCols + kTilePairs / kCols];
    unsigned t = blockIdx.x;
    const unsigned jt = t % q.col_tiles; t /= q.col_tiles;
    const unsigned it = t % q.row_tiles; t /= q.row_tiles;
    const unsigned bh = t % q.BH, party = t / q.BH, h = bh % q.H;
    const unsigned i0 = it * q.rows, j0 = jt * q.cols;
    const unsigned rows = q.Tq - i0 < q.rows ? q.Tq - i0 : q.rows, cols = q.Tk - j0 < q.cols ? q.Tk - j0 : q.cols;
    const u64* const table = q.table[party];
    for (unsigned k = threadIdx.x; k < rows + cols - 1; k += kThreads) {
        const int u = q.buckets[(size_t)j0 + k + (q.Tq - i0 - rows)];      // j - i + Tq - 1
        const bool kept = u >= 0 && u < q.n_buckets;
        by_distance[k] = kept ? ulonglong2{ table[(size_t)u * q.H + h], ~0ull } : ulonglong2{ 0, 0 };
    }
    __syncthreads();
    const size_t at = ((size_t)bh * q.Tq + i0) * q.Tk + j0;
    const u64* const x = q.x[party] + at;
    u64* const out = q.out[party] + at;
    const unsigned pairs = (cols + 1) / 2, dr = kThreads / pairs, dc = kThreads % pairs;
    unsigned r = threadIdx.x / pairs, c = threadIdx.x % pairs;
    while (r < rows) {
        const size_t o = (size_t)r * q.Tk + 2 * c;
        const unsigned k = rows - 1 - r + 2 * c;
        const ulonglong2 d0 = by_distance[k];
        if (2 * c + 1 < cols) {
            const ulonglong2 d1 = by_distance[k + 1];
            u64x2u w = { 0, 0 };
            if (d0.y | d1.y) w = *reinterpret_cast<const u64x2u*>(x + o);
            *reinterpret_cast<u64x2u*>(out + o) = u64x2u{ (w.x + d0.x) & d0.y, (w.y + d1.x) & d1.y };
        } else out[o] = d0.y ? x[o] + d0.x : 0;
        r += dr; c += dc;
        if (c >= pairs) { c -= pairs; ++r; }
    }
}

__global__ __launch_bounds__(kThreads) void k_zero_pair(u64* a, u64* b, size_t n)
{
    const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (i < n) { a[i] = 0; b[i] = 0; }
}

// A thread walks one diagonal of the tile after another, through all rows and matrices of the workgroup, and keeps the sum in
// a register: neighbouring threads read neighbouring words, and one sum a diagonal goes to its bucket.
template <bool SCORES>
__global__ __launch_bounds__(kThreads) void k_position_bias_grad(BiasArgs q)
{
    extern __shared__ u64 sums[];
    unsigned t = blockIdx.x;
    const unsigned jt = t % q.col_tiles; t /= q.col_tiles;
    const unsigned it = t % q.row_tiles; t /= q.row_tiles;
    const unsigned h = t % q.H; t /= q.H;
    const unsigned party = t & 1, b0 = (t >> 1) * q.batches;
    const unsigned i0 = it * q.rows, j0 = jt * q.cols;
    const int rows = q.Tq - i0 < q.rows ? q.Tq - i0 : q.rows, cols = q.Tk - j0 < q.cols ? q.Tk - j0 : q.cols;
    const unsigned nb = q.B - b0 < q.batches ? q.B - b0 : q.batches;
    for (int u = threadIdx.x; u < q.n_buckets; u += kThreads) sums[u] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < rows + cols - 1; k += kThreads) {
        const int u = q.buckets[(size_t)j0 + k + (q.Tq - i0 - rows)];
        const bool kept = u >= 0 && u < q.n_buckets;
        if (!kept && !SCORES) continue;
        const int first = rows - 1 - k > 0 ? rows - 1 - k : 0, last = rows + cols - 1 - k < rows ? rows + cols - 1 - k : rows;   // rows of the diagonal
        u64 sum = 0;
        for (unsigned b = 0; b < nb; ++b) {
            const size_t at = (((size_t)(b0 + b) * q.H + h) * q.Tq + i0) * q.Tk + j0;
            for (int r = first; r < last; ++r) {
                const size_t o = at + (size_t)r * q.Tk + (k + r - (rows - 1));
                const u64 w = kept ? q.x[party][o] : 0;
                sum += w;
                if (SCORES) q.out[party][o] = w;
            }
        }
        if (kept) atomicAdd((unsigned long long*)&sums[u], (unsigned long long)sum);
    }
    __syncthreads();
    for (int u = threadIdx.x; u < q.n_buckets; u += kThreads)
        if (sums[u]) atomicAdd((unsigned long long*)&q.grad[party][(size_t)u * q.H + h], (unsigned long long)sums[u]);
}

int bias_shape(BiasArgs& q, int B, int H, int Tq, int Tk, int n_buckets)
{
    if (B <= 0 || H <= 0 || Tq <= 0 || Tk <= 0 || n_buckets <= 0) return MPC_EINVAL;
    if (n_buckets > MPC_MAX_BUCKETS || (long long)Tq + Tk - 1 > INT32_MAX || (long long)B * H > INT32_MAX) return MPC_ERANGE;
    q.B = B; q.H = H; q.BH = (unsigned)B * H; q.Tq = Tq; q.Tk = Tk; q.n_buckets = n_buckets;
    return MPC_OK;
}

}  // namespace

extern "C" {

int mpc_position_bias(mpc_ctx* c, mpc_cshare x, mpc_cshare table, const int32_t* buckets, mpc_share out,
                      int B, int H, int Tq, int Tk, int n_buckets)
{
    BiasArgs q{};
    if (!c || !buckets) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) if (!x.p[i] || !table.p[i] || !out.p[i]) return MPC_EINVAL;
    MPC_TRY(bias_shape(q, B, H, Tq, Tk, n_buckets));
    const size_t bytes = (size_t)q.BH * Tq * Tk * 8;
    if (!outputs_apart(out, bytes, x, bytes, true) || !outputs_apart(out, bytes, table, (size_t)n_buckets * H * 8, false)) return MPC_EINVAL;
    q.cols = Tk < kCols ? Tk : kCols;
    q.rows = kTilePairs / q.cols; if (q.rows > kRows) q.rows = kRows; if (q.rows > q.Tq) q.rows = q.Tq;
    q.row_tiles = (q.Tq + q.rows - 1) / q.rows; q.col_tiles = (q.Tk + q.cols - 1) / q.cols;
    const size_t grid = 2 * (size_t)q.BH * q.row_tiles * q.col_tiles;
    if (grid > INT32_MAX) return MPC_ERANGE;
    for (int i = 0; i < 2; ++i) { q.x[i] = x.p[i]; q.table[i] = table.p[i]; q.out[i] = out.p[i]; }
    q.buckets = buckets;
    MPC_TRY(lane_first(c));
    k_position_bias<<<dim3((unsigned)grid), kThreads, 0, c->s[0]>>>(q);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

int mpc_position_bias_grad(mpc_ctx* c, mpc_cshare g, const int32_t* buckets, mpc_share table_grad, mpc_share scores_grad,
                           int B, int H, int Tq, int Tk, int n_buckets)
{
    BiasArgs q{};
    if (!c || !buckets || !scores_grad.p[0] != !scores_grad.p[1]) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) if (!g.p[i] || !table_grad.p[i]) return MPC_EINVAL;
    MPC_TRY(bias_shape(q, B, H, Tq, Tk, n_buckets));
    const size_t bytes = (size_t)q.BH * Tq * Tk * 8, table_bytes = (size_t)n_buckets * H * 8;
    const bool scores = scores_grad.p[0] != nullptr;
    if (!outputs_apart(table_grad, table_bytes, g, bytes, false)) return MPC_EINVAL;
    if (scores && (!outputs_apart(scores_grad, bytes, g, bytes, true) ||
                   !outputs_apart(table_grad, table_bytes, mpc_cshare{ { scores_grad.p[0], scores_grad.p[1] } }, bytes, false))) return MPC_EINVAL;
    q.cols = Tk < kCols ? Tk : kCols;
    q.rows = Tq < 32 ? Tq : 32;
    q.row_tiles = (q.Tq + q.rows - 1) / q.rows; q.col_tiles = (q.Tk + q.cols - 1) / q.cols;
    const size_t one = 2 * (size_t)H * q.row_tiles * q.col_tiles;
    size_t splits = (2048 + one - 1) / one; if (splits > q.B) splits = q.B;
    q.batches = (unsigned)((q.B + splits - 1) / splits);
    const size_t grid = one * ((q.B + q.batches - 1) / q.batches);
    if (grid > INT32_MAX) return MPC_ERANGE;
    for (int i = 0; i < 2; ++i) { q.x[i] = g.p[i]; q.grad[i] = table_grad.p[i]; q.out[i] = scores_grad.p[i]; }
    q.buckets = buckets;
    MPC_TRY(lane_first(c));
    const size_t words = (size_t)n_buckets * H;
    k_zero_pair<<<dim3((unsigned)((words + kThreads - 1) / kThreads)), kThreads, 0, c->s[0]>>>(table_grad.p[0], table_grad.p[1], words);
    const size_t lds = (size_t)n_buckets * 8;
    if (scores) k_position_bias_grad<true><<<dim3((unsigned)grid), kThreads, lds, c->s[0]>>>(q);
    else k_position_bias_grad<false><<<dim3((unsigned)grid), kThreads, lds, c->s[0]>>>(q);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
