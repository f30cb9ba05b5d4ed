// Learned relative position bias on shares, and its gradient.  Both are linear in the shares, so every party works on its
// own words: no triple, no exchange, no rescale.
//   y[b,h,i,j] = x[b,h,i,j] + table[m(j-i)][h]         m: public bucket of a distance; none: y = 0
//   table_grad[u][h] = sum over b and all (i,j) with m(j-i) = u of g[b,h,i,j],   x_grad = g where there is a bucket, else 0
// Sums are exact mod 2^64, whatever their order.  Bound by HBM: one read and one write of every pair (the table's gradient
// alone: one read).
#include "attention.h"

#include <algorithm>

namespace {

constexpr int kThreads = 512;
constexpr int kSumThreads = 256;
constexpr int kCols = 1024;              // columns of a tile, at most
constexpr int kRows = 512;               // rows of a tile, at most
constexpr int kTilePairs = 4096;         // (i, j) pairs of a tile, at most

constexpr int kAtOnce = 8;               // rows of the gradient on their way at a time
constexpr size_t kEnough = 2048;         // workgroups; of the gradient up to four times as many
constexpr size_t kFewRounds = 8;
constexpr int kFewBuckets = 256;         // with more, a workgroup's partial sums cost too much for that
constexpr unsigned kMostWaves = 8;       // of them

struct BiasArgs {
    const u64* x[2]; const u64* table[2]; const int32_t* buckets; u64* out[2];
    u64* grad[2];                        // gradient only
    unsigned BH, H, Tq, Tk; int n_buckets;
    unsigned rows, cols, row_tiles, col_tiles;      // a tile is rows x cols; gradient: rows, and col_tiles of 512 diagonals
    unsigned B, batches, splits, parts, waves;      // gradient: matrices of one head, and how many of them an item has
    u64* partial;                                   // gradient: [party][H][bucket][part]
};

// A workgroup's tile: what its distances add, and where nothing is kept, is made once in LDS (entry k is distance j - i =
// j0 - i0 - (rows - 1) + k), then a thread moves two pairs at a time.  96 x 512 x 512: 130 us, 6.2 TB/s; with 256 threads 134 (and
// with ordinary accesses 10 % more), with 1024 and tiles of twice the size 136.  The tiles of a column follow one another: a matrix
// of two columns had its left tiles, all of a causal mask's reads, on every other die (24 x 1500 x 1500: 317 us, so 255, and 241
// with 512 threads).
__global__ __launch_bounds__(kThreads) void k_position_bias(BiasArgs q)
{
    // (word, kept mask); rows + cols is largest at either end of cols: kCols + kTilePairs / kCols, kRows + kTilePairs / kRows
    __shared__ ulonglong2 by_distance[kCols + kTilePairs / kCols];
    unsigned t = blockIdx.x;
    const unsigned it = t % q.row_tiles; t /= q.row_tiles;
    const unsigned jt = t % q.col_tiles; t /= q.col_tiles;
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
            if (d0.y | d1.y) w = __builtin_nontemporal_load(reinterpret_cast<const u64x2u*>(x + o));
            __builtin_nontemporal_store(u64x2u{ (w.x + d0.x) & d0.y, (w.y + d1.x) & d1.y }, reinterpret_cast<u64x2u*>(out + o));
        } else out[o] = d0.y ? x[o] + d0.x : 0;
        r += dr; c += dc;
        if (c >= pairs) { c -= pairs; ++r; }
    }
}

// A wave takes 128 diagonals of a block of rows, two to a lane, through all matrices of its workgroup, and keeps their sums in
// registers: a row's words are read side by side, and one sum a diagonal goes to its bucket in LDS; the workgroups' buckets are added
// up by a second launch unless there is one to a head (atomics on the table would need a launch ahead to clear it).  Diagonal k of a block of `rows` rows
// from i0 on holds the pairs (i0 + r, r + k - (rows - 1)).  Row blocks follow one another: shares of diagonals that do not read
// (masked ones) and those that do would otherwise go to different dies (18 x 1121 x 1121, causal: 162 us, so 135).
// 96 x 512 x 512: 77 us with the sums' launch, 5.2 TB/s.
template <bool SCORES>
__global__ __launch_bounds__(64 * kMostWaves) void k_position_bias_grad(BiasArgs q)
{
    extern __shared__ u64 sums[];
    const unsigned part = blockIdx.x % q.parts, h = blockIdx.x / q.parts % q.H, party = blockIdx.x / q.parts / q.H;
    for (int u = threadIdx.x; u < q.n_buckets; u += blockDim.x) sums[u] = 0;
    __syncthreads();
    const unsigned items = q.row_tiles * q.col_tiles * q.splits;
    for (unsigned item = part; item < items; item += q.parts) {
        const unsigned it = item % q.row_tiles, dt = item / q.row_tiles % q.col_tiles, b0 = item / q.row_tiles / q.col_tiles * q.batches;
        const unsigned i0 = it * q.rows;
        const int rows = min(q.Tq - i0, q.rows), cols = q.Tk;
        const unsigned nb = min(q.B - b0, q.batches);
        const int k = (dt * blockDim.x + threadIdx.x) * 2, last = rows + cols - 2;
        if (k <= last) {
            const int32_t* const m = q.buckets + (q.Tq - i0 - rows);
            const int u0 = m[k], u1 = k < last ? m[k + 1] : -1;
            const bool kept0 = u0 >= 0 && u0 < q.n_buckets, kept1 = u1 >= 0 && u1 < q.n_buckets;
            const int j0 = k - (rows - 1);                                 // column of the first diagonal in row 0
            const int from = max(-j0, 0), to = min(cols - 1 - j0, rows);   // rows that have both diagonals
            u64 s0 = 0, s1 = 0;
            const size_t stride = (size_t)q.H * q.Tq * cols;
            if (SCORES || kept0 || kept1)
                for (unsigned b = 0; b < nb; ++b) {
                    const size_t at = (b0 + b) * stride + ((size_t)h * q.Tq + i0) * cols;
                    const u64* const x = q.x[party] + at;
                    u64* const out = SCORES ? q.out[party] + at : nullptr;
                    const auto one = [&](int r, int j, bool kept, u64& s) {
                        const size_t o = (size_t)r * cols + j;
                        const u64 w = kept ? x[o] : 0;
                        s += w;
                        if (SCORES) out[o] = w;
                    };
                    if (j0 < 0 && from - 1 < rows && k < last) one(from - 1, 0, kept1, s1);    // the row before them has the second
                    if (to < rows && to >= 0) one(to, cols - 1, kept0, s0);                    // the row behind them the first
                    size_t o = (size_t)from * cols + (from + j0);
                    int r = from;
                    for (; r + kAtOnce <= to; r += kAtOnce) {
                        u64x2u w[kAtOnce];
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            const u64x2u* const from = reinterpret_cast<const u64x2u*>(x + o + (size_t)i * (cols + 1));
                            // read for good without the scores' gradient (96 x 512 x 512: 80 -> 77 us); with it 11 -> 13 us for 24 x 197 x 197
                            if (SCORES) w[i] = kept0 || kept1 ? *from : u64x2u{ 0, 0 }; else w[i] = __builtin_nontemporal_load(from);
                        }
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            s0 += w[i].x; s1 += w[i].y;
                            if (SCORES) *reinterpret_cast<u64x2u*>(out + o + (size_t)i * (cols + 1)) = u64x2u{ kept0 ? w[i].x : 0, kept1 ? w[i].y : 0 };
                        }
                        o += (size_t)kAtOnce * (cols + 1);
                    }
                    for (; r < to; ++r, o += cols + 1) {
                        const u64x2u w = !SCORES || kept0 || kept1 ? *reinterpret_cast<const u64x2u*>(x + o) : u64x2u{ 0, 0 };
                        s0 += w.x; s1 += w.y;
                        if (SCORES) *reinterpret_cast<u64x2u*>(out + o) = u64x2u{ kept0 ? w.x : 0, kept1 ? w.y : 0 };
                    }
                }
            if (kept0) atomicAdd((unsigned long long*)&sums[u0], (unsigned long long)s0);
            if (kept1) atomicAdd((unsigned long long*)&sums[u1], (unsigned long long)s1);
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < q.n_buckets; u += blockDim.x)
        if (q.parts == 1) q.grad[party][(size_t)u * q.H + h] = sums[u];
        else q.partial[((size_t)(party * q.H + h) * q.n_buckets + u) * q.parts + part] = sums[u];
}

// the workgroups' sums of a bucket and head, a wave each
__global__ __launch_bounds__(kSumThreads) void k_position_bias_sums(BiasArgs q)
{
    const unsigned n = 2 * q.H * (unsigned)q.n_buckets, at = blockIdx.x * (kSumThreads / 64) + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (at >= n) return;
    u64 s = 0;
    for (unsigned i = lane; i < q.parts; i += 64) s += q.partial[(size_t)at * q.parts + i];
#pragma unroll
    for (int d = 32; d; d /= 2) s += (u64)__shfl_xor((unsigned long long)s, d);
    const unsigned u = at % q.n_buckets, ph = at / q.n_buckets;
    if (lane == 0) q.grad[ph / q.H][(size_t)u * q.H + ph % q.H] = s;
}

// How the gradient is shared out: blocks of 32 rows, of fewer where that makes too few items, and even shares of their diagonals; as
// many matrices to an item as leave enough; and workgroups (parts) for each party and head, one to an item up to four times
// enough.  With a fixed number, some of two items, and a second share of few diagonals, 16 x 1175 x 1175 with the scores' gradient
// took 206 us instead of 129, 24 x 1500 x 1500 without it 183 instead of 154.
void share_out(BiasArgs& q)
{
    size_t one = 0;
    for (q.rows = 32; ; q.rows /= 2) {
        if (q.rows > q.Tq) q.rows = q.Tq;
        const size_t diagonals = (size_t)q.rows + q.Tk - 1;
        const unsigned waves = (unsigned)((diagonals + 127) / 128);
        q.row_tiles = (q.Tq + q.rows - 1) / q.rows; q.col_tiles = (waves + kMostWaves - 1) / kMostWaves;
        q.waves = (waves + q.col_tiles - 1) / q.col_tiles;
        // A party's head that is a few rounds of loads is one workgroup's, which then needs no second launch: 12 x 64 x 64 11.5 us a call
        // with two, 9.8 with one (of the device 6.5 and 7.2), 24 x 1 x 115 11.7 and 10.4 (5.2 and 4.4).
        if ((size_t)q.B * q.row_tiles * q.col_tiles * ((q.rows + kAtOnce - 1) / kAtOnce) <= kFewRounds) { q.batches = q.B; q.splits = q.parts = 1; return; }
        one = 2 * (size_t)q.H * q.row_tiles * q.col_tiles;
        if (one * q.B >= kEnough || q.rows <= 8) break;
    }
    const size_t splits = std::min<size_t>((kEnough + one - 1) / one, q.B);
    q.batches = (unsigned)((q.B + splits - 1) / splits);
    q.splits = (q.B + q.batches - 1) / q.batches;
    const size_t items = (size_t)q.row_tiles * q.col_tiles * q.splits;
    const size_t most = ((q.n_buckets > kFewBuckets ? kEnough : 4 * kEnough) + 2 * q.H - 1) / (2 * q.H), each = (items + most - 1) / most;
    q.parts = (unsigned)((items + each - 1) / each);
}

int bias_shape(BiasArgs& q, int B, int H, int Tq, int Tk, int n_buckets)
{
    if (B <= 0 || H <= 0 || Tq <= 0 || Tk <= 0 || n_buckets <= 0) return MPC_EINVAL;
    if (n_buckets > MPC_MAX_BUCKETS || (long long)Tq + Tk > INT32_MAX - 2048 ||      // diagonals are counted in int, up to 1024 of a workgroup at a time
        (long long)B * H > INT32_MAX || 2ll * H * n_buckets > INT32_MAX) return MPC_ERANGE;
    if ((long long)Tq * Tk > MPC_MAX_PAIRS / ((long long)B * H)) return MPC_ERANGE;      // by division: bytes and tiles are counted in 64 bits
    q.B = B; q.H = H; q.BH = (unsigned)B * H; q.Tq = Tq; q.Tk = Tk; q.n_buckets = n_buckets;
    return MPC_OK;
}

}  // namespace

extern "C" {

size_t mpc_position_bias_grad_workspace_bytes(int B, int H, int Tq, int Tk, int n_buckets)
{
    BiasArgs q{};
    if (bias_shape(q, B, H, Tq, Tk, n_buckets) != MPC_OK) return 0;
    share_out(q);
    return align_up(2 * (size_t)H * n_buckets * q.parts * 8);
}

int mpc_position_bias(mpc_ctx* c, mpc_cshare x, mpc_cshare table, const int32_t* buckets, mpc_share out,
                      int B, int H, int Tq, int Tk, int n_buckets)
{
    BiasArgs q{};
    if (!c || !buckets) return MPC_EINVAL;
    for (int i = 0; i < 2; ++i) if (!x.p[i] || !table.p[i] || !out.p[i]) return MPC_EINVAL;
    MPC_TRY(bias_shape(q, B, H, Tq, Tk, n_buckets));
    q.cols = Tk < kCols ? Tk : kCols;
    q.rows = kTilePairs / q.cols; if (q.rows > kRows) q.rows = kRows; if (q.rows > q.Tq) q.rows = q.Tq;
    q.row_tiles = (q.Tq + q.rows - 1) / q.rows; q.col_tiles = (q.Tk + q.cols - 1) / q.cols;
    const size_t grid = 2 * (size_t)q.BH * q.row_tiles * q.col_tiles, bytes = (size_t)q.BH * Tq * Tk * 8;
    if (!launchable(grid, kThreads)) return MPC_ERANGE;
    if (!apart(out, bytes, buckets, ((size_t)Tq + Tk - 1) * 4)) return MPC_EINVAL;
    if (!outputs_apart(out, bytes, x, bytes, true) || !outputs_apart(out, bytes, table, (size_t)n_buckets * H * 8, false)) return MPC_EINVAL;
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
    share_out(q);
    const size_t items = (size_t)q.row_tiles * q.col_tiles * q.splits, sums = (2 * (size_t)H * n_buckets + kSumThreads / 64 - 1) / (kSumThreads / 64);
    if (items > INT32_MAX || !launchable(2 * (size_t)H * q.parts, 64 * q.waves) || !launchable(sums, kSumThreads)) return MPC_ERANGE;
    const size_t bytes = (size_t)q.BH * Tq * Tk * 8, table_bytes = (size_t)n_buckets * H * 8, public_bytes = ((size_t)Tq + Tk - 1) * 4;
    const bool scores = scores_grad.p[0] != nullptr;
    if (!outputs_apart(table_grad, table_bytes, g, bytes, false) || !apart(table_grad, table_bytes, buckets, public_bytes)) return MPC_EINVAL;
    if (scores && (!apart(scores_grad, bytes, buckets, public_bytes) || !outputs_apart(scores_grad, bytes, g, bytes, true) ||
                   !outputs_apart(table_grad, table_bytes, mpc_cshare{ { scores_grad.p[0], scores_grad.p[1] } }, bytes, false))) return MPC_EINVAL;
    WsAlloc ws(c->ws, c->ws_bytes);
    q.partial = ws.take<u64>(2 * (size_t)H * n_buckets * q.parts);
    if (!ws.ok) return MPC_ENOMEM;
    for (int i = 0; i < 2; ++i) { q.x[i] = g.p[i]; q.grad[i] = table_grad.p[i]; q.out[i] = scores_grad.p[i]; }
    q.buckets = buckets;
    MPC_TRY(lane_first(c));
    const dim3 grid(2 * (unsigned)H * q.parts), block(64 * q.waves);
    const size_t lds = (size_t)n_buckets * 8;
    if (scores) k_position_bias_grad<true><<<grid, block, lds, c->s[0]>>>(q);
    else k_position_bias_grad<false><<<grid, block, lds, c->s[0]>>>(q);
    if (q.parts > 1) k_position_bias_sums<<<dim3((unsigned)sums), kSumThreads, 0, c->s[0]>>>(q);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
