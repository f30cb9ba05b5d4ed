// Linear attention with a public decay for each head, on shares: S_t = g S_{t-1} + k_t v_t^T, o_t = q_t S_t.
//
// One token (mpc_linear_attention_step): U = k v^T and q S are Beaver products, the decay is a public factor that joins U at
// scale 2^2f so that one rescale serves both: S' = trunc(g S + U), o = trunc(q S').
//
// Prompts (mpc_linear_attention), in chunks of 64 tokens, pow[n] = g^n, L tokens in the chunk:
//   P = trunc(Q K^T), W[i][j] = trunc(P[i][j] pow[i-j]) for j <= i, else zero    Qd[i] = trunc(Q[i] pow[i+1])
//   Kd[j] = trunc(K[j] pow[L-1-j]), U = Kd^T V                                   S' = trunc(pow[L] S + U)
//   O = trunc([W | Qd] [V ; S])
// Three launches: everything that one chunk has for itself (P, W and W V, U, and their openings), the states from chunk to chunk
// (element by element), and the states' part of O.
//
// All products are Alg. 1 with party 0's local product folded into its addend (the folded calls of the linear layers):
// party 0 has c_0 + (x_0 + e_1)(y_0 + f_1), party 1 has c_1 + e b_1 + a_1 f.  A thread has both
// parties' shares and forms the opened words from them, in every job that needs them; no job waits for another's.  So there is no
// receiver.  A masked word is stored once in a call, by the job named at the store, where the peer's receive buffer would be: the
// traffic of sending it.  Nothing reads these buffers.
#include "attention.h"
#include "digits.h"

namespace {

constexpr int kChunk = MPC_ATTENTION_CHUNK;   // 64
constexpr int kThreads = 512;
constexpr int kBoxes = 256;                   // workgroups of a launch, one to a compute unit, each with send buffers of its own
constexpr int kStateBoxes = 2048;             // workgroups of the states' launch, eight to a compute unit: 512 words each
constexpr long long kMaxStride = MPC_ATTENTION_MAX_TOKEN_STRIDE;   // 64 tokens stay below 2^31 bytes
constexpr size_t kBoxWords = (size_t)kThreads * 4;   // per direction

struct Rows { const u64* p[2]; long long b, t, h; };     // words of (batch, token, head) at p + b*b + t*t + h*h

struct ChunkArgs {
    Rows q, k, v;
    const u64 *a_q[2], *a_k[2], *a_qd[2], *a_kd[2], *a_v[2], *a_w[2], *a_s[2], *c_p[2], *c_u[2], *c_o[2], *state[2];
    u64 *o[2]; long long ob, ot, oh;
    u64* state_out[2];
    const int32_t* decay;                     // [H][65]
    u64* part[2];                             // c_o + W V, not yet rescaled: [BH][T][dv]
    u64* u[2];                                // U; then the states: party 0's operand (u[0]) and opened words (u[1]): [BH][chunks][dk][dv]
    u64* box;
    int B, H, T, dk, dv, chunks, bits;
    int mt, nt;                               // tiles of 64 along dk and dv
    int rows_jobs;                            // jobs that form P and W: one for all of W V, or one for each tile of dv
    unsigned cells;                           // chunks of all heads
};

// Products of 64 x 64 x 64 words run on the matrix cores, from eight digit planes of each operand tile in LDS,
// [digit][k/16][row][16]; five operand tiles fill the 160 KB of a compute unit.
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kPlane = 64 * 64, kOperand = 8 * kPlane;      // bytes
enum { kOwnLeft, kOwnRight, kOpenLeft, kMaskRight, kOpenRight, kOperands, kMaskLeft = kOwnLeft };

// The first four waves bring the left operand, the others the right one: 16 words a thread, as four quads of rows 16 apart.
// Wave w of the four has words 16w..16w+15 of the contraction.  Where a row's words are adjacent in memory (ADJACENT), four lanes
// read 64 bytes of a row at once, and quad kq is words {2kq, 2kq+1, 8+2kq, 9+2kq} (PAIRS): a product does not care about the order
// if both operands have the same.  Elsewhere sixteen lanes read 128 bytes across the rows.  Stores to LDS meet every bank once
// either way.
struct Place { int wave, lane; };             // wave: the same for all lanes, read once (a scalar)
__device__ __forceinline__ Place place() { return Place{ __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), (int)threadIdx.x % 64 }; }
// The same place again: offsets and conditions that follow from the lane are made anew, instead of being kept (and spilled) across
// jobs and steps.
__device__ __forceinline__ Place anew(Place p) { asm volatile("" : "+v"(p.lane)); return p; }

struct Quad { u64 w[4]; };

// a quad's digits, from the place of its first one
__device__ __forceinline__ void stage_at(u8* at, const Quad& q)
{
    uint32_t d[8];
    digits_of_4(q.w, d);
#pragma unroll
    for (int p = 0; p < 8; ++p) *reinterpret_cast<uint32_t*>(at + p * kPlane) = d[p];
}

// A tile of `rows` rows and `cols` words along the contraction, at most 64 each of what is there; word (row, k) lies at
// p + row*rs + k*ks words, one of the strides being 1 (ADJACENT: ks).  Rows and columns that are not there repeat the last one.
// Offsets within a tile are below 2^31 bytes (kMaxStride).
template <bool ADJACENT, bool PAIRS = true> struct Tile {
    int rows, cols, row0, k0, quad;
    __device__ __forceinline__ Tile(const Place& p, int rows_, int cols_)
        : rows(rows_), cols(cols_), row0(ADJACENT ? p.lane / 4 : p.lane % 16), quad(ADJACENT ? p.lane % 4 : p.lane / 16) { k0 = p.wave % 4 * 16 + quad * (PAIRS ? 2 : 4); }
    __device__ __forceinline__ int row(int i) const { return row0 + i * 16; }
    __device__ __forceinline__ int k(int j) const { return PAIRS ? k0 + j % 2 + j / 2 * 8 : k0 + j; }
    __device__ __forceinline__ Quad load(const u64* p, long long stride, int i) const
    {
        const u8* const base = reinterpret_cast<const u8*>(p);
        const unsigned r = min(row(i), rows - 1), s = (unsigned)stride * 8;
        Quad q;
        if (ADJACENT && cols % 2 == 0) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const u64x2u w = *reinterpret_cast<const u64x2u*>(base + (r * s + min(k(j), cols - 2) * 8u));
                q.w[j] = w.x; q.w[j + 1] = w.y;
            }
        } else
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned c = min(k(j), cols - 1);
                q.w[j] = *reinterpret_cast<const u64*>(base + (ADJACENT ? r * s + c * 8 : c * s + r * 8));
            }
        return q;
    }
    __device__ __forceinline__ bool has(int i, int j) const { return row(i) < rows && k(j) < cols; }
    __device__ __forceinline__ void clear(int i, Quad& q) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) q.w[j] = has(i, j) ? q.w[j] : 0;
    }
    __device__ __forceinline__ void stage(u8* lds, int operand, int i, const Quad& q) const
    {
        stage_at(lds + operand * kOperand + k0 / 16 * 1024 + (row(i) * 16 + quad * 4), q);
    }
};

// A thread's four quads of an operand.  Their words are asked for together, ahead of the barrier behind which the last products'
// operands may be written over: one after the other their latency was most of a job's time.  The barrier stands outside of what
// only one half of the waves does.
//
// Words of a sharing and of its mask.
struct Masked { Quad x0, x1, a0, a1; };
struct Words { const u64 *x0, *x1; long long stride; const u64 *a0, *a1; long long a_stride; };
template <class T> __device__ __forceinline__ Masked masked(const T& t, const Words& w, int i)
{
    return Masked{ t.load(w.x0, w.stride, i), t.load(w.x1, w.stride, i), t.load(w.a0, w.a_stride, i), t.load(w.a1, w.a_stride, i) };
}
// party 0's operand x_0 + e_1 and the opened words; DECAY: of words times public factors f(j), rescaled
struct NoPower { __device__ uint32_t operator()(int) const { return 1; } };
template <bool DECAY, class Power> __device__ __forceinline__ void open_quad(const Masked& r, Power f, int bits, Quad& own, Quad& open, Quad& e0, Quad& e1)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        u64 w0 = r.x0.w[j], w1 = r.x1.w[j];
        if (DECAY) { w0 = rescaled<0>(w0 * f(j), bits); w1 = rescaled<1>(w1 * f(j), bits); }
        e0.w[j] = w0 - r.a0.w[j]; e1.w[j] = w1 - r.a1.w[j];
        own.w[j] = w0 + e1.w[j]; open.w[j] = e0.w[j] + e1.w[j];
    }
}
// party 0's operand, the opened words and, of a right operand, party 1's mask
template <bool LEFT, class T> __device__ __forceinline__ void stage_operand(u8* lds, const T& t, int i, Quad own, Quad open, Quad mask)
{
    t.clear(i, own); t.clear(i, open);
    t.stage(lds, LEFT ? kOwnLeft : kOwnRight, i, own);
    t.stage(lds, LEFT ? kOpenLeft : kOpenRight, i, open);
    if (!LEFT) { t.clear(i, mask); t.stage(lds, kMaskRight, i, mask); }
}
// power(i, j): the public factor of word j of quad i; sent(to party 0, to party 1)
template <bool LEFT, bool DECAY, class T, class Power, class Sent>
__device__ __forceinline__ void stage_masked(u8* lds, const T& t, const Masked (&w)[4], Power power, int bits, Sent sent)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Quad own, open, e0, e1;
        open_quad<DECAY>(w[i], [&](int j) { return power(i, j); }, bits, own, open, e0, e1);
        sent(e1, e0);
        stage_operand<LEFT>(lds, t, i, own, open, w[i].a1);
    }
}
struct NoPowers { __device__ uint32_t operator()(int, int) const { return 1; } };

// The send buffers of a workgroup (sent is sent: nothing reads them) hold what a thread sends at a time, a quad in either direction:
// they stay in the L2 (with room for a whole tile, 128 KB a workgroup, they were written back to memory, 160 MB a launch of 8 x 512 tokens of 12 heads).
struct Box {
    u64 *to0, *to1;
    __device__ __forceinline__ Box(u64* box) : to0(box + blockIdx.x * 2 * kBoxWords + threadIdx.x * 2), to1(to0 + kBoxWords) {}
    __device__ __forceinline__ void put(const Quad& e1, const Quad& e0) const
    {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            *reinterpret_cast<u64x2u*>(to0 + j * kThreads) = u64x2u{ e1.w[j], e1.w[j + 1] };
            *reinterpret_cast<u64x2u*>(to1 + j * kThreads) = u64x2u{ e0.w[j], e0.w[j + 1] };
        }
    }
};

// A wave has 16 rows and two tiles of 16 columns; acc[tile][s] sums the products of digits i + j = s.  One K step of 64 adds at
// most (s + 1) 2^20 to it.
struct Sums { i32x4 s[2][8]; };
__device__ __forceinline__ void clear(Sums& z)
{
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < 8; ++s) z.s[t][s] = i32x4{ 0, 0, 0, 0 };
}
__device__ __forceinline__ void multiply(const u8* lds, const Place& p, int left, int right, Sums& z)
{
    const int wave = p.wave, lane = p.lane;
    const u8* const l = lds + left * kOperand + (lane / 16 * 64 + wave % 4 * 16 + lane % 16) * 16;
    const u8* const r = lds + right * kOperand + (lane / 16 * 64 + wave / 4 * 32 + lane % 16) * 16;
    i32x4 a[8];
#pragma unroll
    for (int d = 0; d < 8; ++d) a[d] = *reinterpret_cast<const i32x4*>(l + d * kPlane);
    i32x4 b0 = *reinterpret_cast<const i32x4*>(r), b1 = *reinterpret_cast<const i32x4*>(r + 256);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        // the next digit's operands are on their way under this one's products, and no further ones: registers
        const i32x4 c0 = b0, c1 = b1;
        if (j < 7) { b0 = *reinterpret_cast<const i32x4*>(r + (j + 1) * kPlane); b1 = *reinterpret_cast<const i32x4*>(r + (j + 1) * kPlane + 256); }
#pragma unroll
        for (int i = 0; i < 8 - j; ++i) {
            z.s[0][i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], c0, z.s[0][i + j], 0, 0, 0);
            z.s[1][i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], c1, z.s[1][i + j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}
// z += sum of the digit sums, of one or two K steps: below 2^31 up to acc[1] 2^8
__device__ __forceinline__ void join(const Sums& a, u64 (&z)[8])
{
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int low = a.s[t][0][r] + a.s[t][1][r] * 256;
            const uint32_t high = (uint32_t)a.s[t][4][r] + ((uint32_t)a.s[t][5][r] << 8) + ((uint32_t)a.s[t][6][r] << 16) + ((uint32_t)a.s[t][7][r] << 24);
            const int64_t w = (int64_t)low + (int64_t)a.s[t][2][r] * 65536 + (int64_t)a.s[t][3][r] * 16777216;
            z[t * 4 + r] += (u64)w + ((u64)high << 32);
        }
}

// z0 += own0 own0', z1 += open mask1' + mask1 open' once both operands are in LDS.  ask() is for what third() needs, which puts
// party 1's mask of the left operand in the place of party 0's operand, under the first two products.
template <class Ask, class Third> __device__ __forceinline__ void multiply_all(u8* lds, const Place& p, Ask ask, Third third, u64 (&z0)[8], u64 (&z1)[8])
{
    Sums a;
    clear(a);
    ask();
    __syncthreads();
    multiply(lds, p, kOwnLeft, kOwnRight, a);
    join(a, z0);
    clear(a);
    multiply(lds, p, kOpenLeft, kMaskRight, a);
    __syncthreads();
    third();
    __syncthreads();
    multiply(lds, p, kMaskLeft, kOpenRight, a);
    join(a, z1);
}
// the same with the mask of a left operand that lies in memory: all waves bring it, two quads each
template <class T> __device__ __forceinline__ void multiply_all(u8* lds, const Place& p, const T& t, const u64* a1, long long stride, u64 (&z0)[8], u64 (&z1)[8])
{
    const int first = p.wave / 4 * 2;
    Quad m[2];
    multiply_all(lds, p, [&] { m[0] = t.load(a1, stride, first); m[1] = t.load(a1, stride, first + 1); },
        [&] {
#pragma unroll
            for (int i = 0; i < 2; ++i) { t.clear(first + i, m[i]); t.stage(lds, kMaskLeft, first + i, m[i]); }
        }, z0, z1);
}
// each(index, row, column) of a thread's words of the product
template <class Each> __device__ __forceinline__ void each_word(const Place& p, Each each)
{
#pragma unroll
    for (int r = 0; r < 8; ++r) each(r, p.wave % 4 * 16 + p.lane / 16 * 4 + r % 4, p.wave / 4 * 32 + r / 4 * 16 + p.lane % 16);
}

// The jobs of a launch: `kinds` for each of `cells` chunks.  A chunk's jobs follow one another on one of the eight dies (workgroups
// go round the dies), so that what they share is in its L2.  Where a workgroup would come to the same kind every time, the kinds
// take turns from round to round: they differ in length (8 x 512 tokens of 12 heads, this launch 269 -> 218 us).
struct Jobs {
    unsigned cells, kinds, step, n;
    bool turns;
    __device__ __forceinline__ Jobs(unsigned cells_, unsigned kinds_) : cells(cells_), kinds(kinds_), step(gridDim.x / 8), n(blockIdx.x / 8) { turns = step % kinds == 0; }
    __device__ __forceinline__ unsigned cell() const { return n / kinds * 8 + blockIdx.x % 8; }
    __device__ __forceinline__ unsigned kind() const { return (n + (turns ? n / step : 0)) % kinds; }
    __device__ __forceinline__ void next() { n += step; }
};

// P, W and W V of a chunk, or one tile of its U.  8 x 512 tokens of 12 heads of 64 x 64: 214 us of the call's 291, 0.71 GB.  Bound by
// what follows one another in a product: its loads (3.3 TB/s over all), the digits (vector instructions fill 23 % of the cycles)
// and the matrix instructions (14 %), since five operand tiles leave room for one workgroup to a compute unit.  All 256 registers
// are used, and 19 words are spilled (80 bytes a lane): nine offsets, read again in every job, and ten words of U's jobs between
// their loads and their digits.
__global__ __launch_bounds__(kThreads) void k_chunk_open(ChunkArgs q)
{
    extern __shared__ __attribute__((aligned(16))) u8 lds[];          // kOperands kOperand
    const Place at_start = place();
    const bool left = at_start.wave < 4;
    const Box box(q.box);
    for (Jobs job(q.cells, q.rows_jobs + q.mt * q.nt); job.cell() < q.cells; job.next()) {
        const Place p = anew(at_start);
        const int kind = job.kind(), bh = job.cell() / q.chunks, chunk = job.cell() - bh * q.chunks;
        const int b = bh / q.H, h = bh - b * q.H, t0 = chunk * kChunk, L = min(q.T - t0, kChunk);
        const int32_t* const pow = q.decay + h * (kChunk + 1);
        const long long at = (long long)bh * q.T + t0;            // the chunk's first token in the dense arrays
        const long long ok = b * q.k.b + h * q.k.h + t0 * q.k.t, ov = b * q.v.b + h * q.v.h + t0 * q.v.t;
        u64 z0[8], z1[8];                                         // start from the addends, asked for first
        if (kind < q.rows_jobs) {
            const int n_first = kind * 64, n_end = q.rows_jobs > 1 ? min(q.dv, n_first + 64) : q.dv;
            const auto to_box = [&](const Quad& e1, const Quad& e0) { if (n_first == 0) box.put(e1, e0); };     // sent once
            // P turned round, K Q^T: a thread's four words of a column are neighbours in a row of W, a quad of the next product
            const int turned = p.wave % 4 * 16 + p.lane / 16 * 4, i0 = p.wave / 4 * 32 + p.lane % 16;    // j of its first word, i of tile 0
            const auto quad_at = [&](const u64* w, int t) {       // of [token][64]; above the diagonal the row's last one again
                const int i = min(i0 + t * 16, L - 1);
                const u64* const from = w + at * kChunk + (unsigned)(i * kChunk + min(turned, i & ~3));
                const u64x2u lo = *reinterpret_cast<const u64x2u*>(from), hi = *reinterpret_cast<const u64x2u*>(from + 2);
                return Quad{ { lo.x, lo.y, hi.x, hi.y } };
            };
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const Quad c0 = quad_at(q.c_p[0], t), c1 = quad_at(q.c_p[1], t);
#pragma unroll
                for (int j = 0; j < 4; ++j) { z0[t * 4 + j] = c0.w[j]; z1[t * 4 + j] = c1.w[j]; }
            }
            const long long oq = b * q.q.b + h * q.q.h + t0 * q.q.t;
            for (int k0 = 0; k0 < q.dk; k0 += 64) {
                const Place ps = anew(p);
                const Tile<true> t(ps, L, q.dk - k0);
                const long long oa = at * q.dk + k0;
                const Words from = left ? Words{ q.k.p[0] + ok + k0, q.k.p[1] + ok + k0, q.k.t, q.a_k[0] + oa, q.a_k[1] + oa, q.dk }
                                        : Words{ q.q.p[0] + oq + k0, q.q.p[1] + oq + k0, q.q.t, q.a_q[0] + oa, q.a_q[1] + oa, q.dk };
                const Masked w[4] = { masked(t, from, 0), masked(t, from, 1), masked(t, from, 2), masked(t, from, 3) };
                __syncthreads();
                if (left) stage_masked<true, false>(lds, t, w, NoPowers{}, 0, to_box);
                else stage_masked<false, false>(lds, t, w, NoPowers{}, 0, to_box);
                multiply_all(lds, ps, t, q.a_k[1] + oa, q.dk, z0, z1);
            }
            Quad own[2], open[2], mask[2];                        // W
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const Quad a0 = quad_at(q.a_w[0], t), a1 = quad_at(q.a_w[1], t);
                const int i = i0 + t * 16;
                Quad e0, e1;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t f = pow[max(i - turned - j, 0)];
                    const u64 w0 = rescaled<0>(rescaled<0>(z0[t * 4 + j], q.bits) * f, q.bits), w1 = rescaled<1>(rescaled<1>(z1[t * 4 + j], q.bits) * f, q.bits);
                    const bool below = i < L && turned + j <= i;  // nothing above the diagonal
                    e0.w[j] = below ? w0 - a0.w[j] : 0; e1.w[j] = below ? w1 - a1.w[j] : 0;
                    own[t].w[j] = below ? w0 + e1.w[j] : 0; open[t].w[j] = e0.w[j] + e1.w[j]; mask[t].w[j] = below ? a1.w[j] : 0;
                }
                to_box(e1, e0);
            }
            for (int n0 = n_first; n0 < n_end; n0 += 64) {
                const Place ps = anew(p);
                const Tile<false, false> tv(ps, q.dv - n0, L);
                const long long oa = at * q.dv + n0, o = ov + n0;
                const int first = ps.wave / 4 * 2;                // all waves bring V, two quads each
                Masked v[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) v[i] = masked(tv, Words{ q.v.p[0] + o, q.v.p[1] + o, q.v.t, q.a_v[0] + oa, q.a_v[1] + oa, q.dv }, first + i);
                each_word(ps, [&](int r, int i, int j) {
                    const unsigned at_o = min(i, L - 1) * q.dv + min(j, q.dv - n0 - 1);
                    z0[r] = (q.c_o[0] + oa)[at_o]; z1[r] = (q.c_o[1] + oa)[at_o];
                });
                u8* const w_at = lds + ps.wave % 4 * 1024 + ((ps.wave / 4 * 32 + ps.lane % 16) * 16 + ps.lane / 16 * 4);
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    Quad vo, vp, e0, e1;
                    open_quad<false>(v[i], NoPower{}, 0, vo, vp, e0, e1);    // sent with U's tiles
                    tv.clear(first + i, vo); tv.clear(first + i, vp); tv.clear(first + i, v[i].a1);
                    tv.stage(lds, kOwnRight, first + i, vo); tv.stage(lds, kOpenRight, first + i, vp); tv.stage(lds, kMaskRight, first + i, v[i].a1);
                    stage_at(w_at + kOwnLeft * kOperand + i * 256, own[i]);
                    stage_at(w_at + kOpenLeft * kOperand + i * 256, open[i]);
                }
                multiply_all(lds, ps, [] {}, [&] { stage_at(w_at + kMaskLeft * kOperand, mask[0]); stage_at(w_at + kMaskLeft * kOperand + 256, mask[1]); }, z0, z1);
                each_word(anew(p), [&](int r, int i, int j) {
                    if (i >= L || n0 + j >= q.dv) return;
                    (q.part[0] + oa)[(unsigned)(i * q.dv + j)] = z0[r]; (q.part[1] + oa)[(unsigned)(i * q.dv + j)] = z1[r];
                });
            }
        } else {
            const int tile = kind - q.rows_jobs, m0 = tile / q.nt * 64, n0 = tile % q.nt * 64;      // contraction over the chunk's tokens
            const long long cell = (long long)job.cell() * q.dk * q.dv;
            each_word(p, [&](int r, int i, int j) {
                const unsigned o = min(m0 + i, q.dk - 1) * q.dv + min(n0 + j, q.dv - 1);
                z0[r] = (q.c_u[0] + cell)[o]; z1[r] = (q.c_u[1] + cell)[o];
            });
            const Tile<false, false> tk(p, q.dk - m0, L);
            const long long oa = at * q.dk + m0, oav = at * q.dv + n0;
            const Words from = left ? Words{ q.k.p[0] + ok + m0, q.k.p[1] + ok + m0, q.k.t, q.a_kd[0] + oa, q.a_kd[1] + oa, q.dk }
                                    : Words{ q.v.p[0] + ov + n0, q.v.p[1] + ov + n0, q.v.t, q.a_v[0] + oav, q.a_v[1] + oav, q.dv };
            const Tile<false, false> t(p, left ? q.dk - m0 : q.dv - n0, L);
            const Masked w[4] = { masked(t, from, 0), masked(t, from, 1), masked(t, from, 2), masked(t, from, 3) };
            uint32_t f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = pow[max(L - 1 - t.k(j), 0)];
            __syncthreads();
            if (left) stage_masked<true, true>(lds, t, w, [&](int, int j) { return f[j]; }, q.bits, [&](const Quad& e1, const Quad& e0) { if (n0 == 0) box.put(e1, e0); });
            else stage_masked<false, false>(lds, t, w, NoPowers{}, 0, [&](const Quad& e1, const Quad& e0) { if (m0 == 0) box.put(e1, e0); });
            multiply_all(lds, p, tk, q.a_kd[1] + oa, q.dk, z0, z1);
            each_word(anew(p), [&](int r, int i, int j) {
                const int d = m0 + i, e = n0 + j;
                if (d >= q.dk || e >= q.dv) return;
                const unsigned o = d * q.dv + e;
                (q.u[0] + cell)[o] = z0[r]; (q.u[1] + cell)[o] = z1[r];
            });
        }
    }
}

// From chunk to chunk, a state element to a thread: what the chunk's O needs of S takes the place of its U.  Bound by HBM, 48 bytes an
// element and chunk: 33 us for the same 768 chunks, 4.6 TB/s.  Few heads with many chunks are bound by latency: a chunk's words are
// asked for only behind the stores of the one before.
__global__ __launch_bounds__(256) void k_chunk_states(ChunkArgs q)
{
    const long long per = (long long)q.dk * q.dv, n = (long long)q.B * q.H * per;
    u64* const box0 = q.box + (size_t)blockIdx.x * 512 + threadIdx.x;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < n; e += (long long)gridDim.x * 256) {
        const long long bh = e / per, first = bh * q.chunks * per + e % per;
        const int32_t* const pow = q.decay + bh % q.H * (kChunk + 1);
        u64 s0 = q.state[0] ? q.state[0][e] : 0, s1 = q.state[0] ? q.state[1][e] : 0;
        for (int c = 0; c < q.chunks; ++c) {
            const long long o = first + c * per;
            const u64 u0 = q.u[0][o], u1 = q.u[1][o], e0 = s0 - q.a_s[0][o], e1 = s1 - q.a_s[1][o];
            box0[0] = e1; box0[256] = e0;
            q.u[0][o] = s0 + e1; q.u[1][o] = e0 + e1;
            const int L = q.T - c * kChunk < kChunk ? q.T - c * kChunk : kChunk;
            const u64 f = (uint32_t)pow[L];
            s0 = rescaled<0>(s0 * f + u0, q.bits); s1 = rescaled<1>(s1 * f + u1, q.bits);
        }
        if (q.state_out[0]) { q.state_out[0][e] = s0; q.state_out[1][e] = s1; }
    }
}

// O of a chunk, 64 columns of dv: the states' part joins what the chunk has for itself.  71 us there, 3.9 TB/s, bound as k_chunk_open;
// what is read and written for good passes by the caches (the call 301 -> 296).
__global__ __launch_bounds__(kThreads) void k_chunk_out(ChunkArgs q)
{
    extern __shared__ __attribute__((aligned(16))) u8 lds[];          // kOperands kOperand
    const Place at_start = place();
    const bool left = at_start.wave < 4;
    const Box box(q.box);
    for (Jobs job(q.cells, q.nt); job.cell() < q.cells; job.next()) {
        const Place p = anew(at_start);
        const int n0 = job.kind() * 64, bh = job.cell() / q.chunks, chunk = job.cell() - bh * q.chunks;
        const int b = bh / q.H, h = bh - b * q.H, t0 = chunk * kChunk, L = min(q.T - t0, kChunk);
        const int32_t* const pow = q.decay + h * (kChunk + 1);
        const long long at = (long long)bh * q.T + t0;
        u64 z0[8], z1[8];
        each_word(p, [&](int r, int i, int j) {
            const unsigned o = min(i, L - 1) * q.dv + min(n0 + j, q.dv - 1);
            z0[r] = __builtin_nontemporal_load(q.part[0] + at * q.dv + o); z1[r] = __builtin_nontemporal_load(q.part[1] + at * q.dv + o);
        });
        for (int k0 = 0; k0 < q.dk; k0 += 64) {
            const Place ps = anew(p);
            const Tile<true> tq(ps, L, q.dk - k0);
            const long long oa = at * q.dk + k0;
            const Tile<false> ts(ps, q.dv - n0, q.dk - k0);
            Masked w[4];                                              // of the state: party 0's operand, the opened words and party 1's mask
            uint32_t f[4];
            if (left) {
                const long long o = b * q.q.b + h * q.q.h + t0 * q.q.t + k0;
                const Words from{ q.q.p[0] + o, q.q.p[1] + o, q.q.t, q.a_qd[0] + oa, q.a_qd[1] + oa, q.dk };
#pragma unroll
                for (int i = 0; i < 4; ++i) { w[i] = masked(tq, from, i); f[i] = pow[min(tq.row(i), L - 1) + 1]; }
            } else {
                const long long o = ((long long)job.cell() * q.dk + k0) * q.dv + n0;
#pragma unroll
                for (int i = 0; i < 4; ++i) { w[i].x0 = ts.load(q.u[0] + o, q.dv, i); w[i].x1 = ts.load(q.u[1] + o, q.dv, i); w[i].a1 = ts.load(q.a_s[1] + o, q.dv, i); }
            }
            __syncthreads();
            if (left) stage_masked<true, true>(lds, tq, w, [&](int i, int) { return f[i]; }, q.bits, [&](const Quad& e1, const Quad& e0) { if (n0 == 0) box.put(e1, e0); });
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) stage_operand<false>(lds, ts, i, w[i].x0, w[i].x1, w[i].a1);
            multiply_all(lds, ps, tq, q.a_qd[1] + oa, q.dk, z0, z1);
        }
        const long long to = b * q.ob + h * q.oh + t0 * q.ot + n0;
        each_word(anew(p), [&](int r, int i, int j) {
            if (i >= L || n0 + j >= q.dv) return;
            const long long o = i * q.ot;
            __builtin_nontemporal_store(rescaled<0>(z0[r], q.bits), q.o[0] + to + o + j);
            __builtin_nontemporal_store(rescaled<1>(z1[r], q.bits), q.o[1] + to + o + j);
        });
    }
}

// ---- one token
struct StepArgs {
    Rows q, k, v;
    const u64 *a_q[2], *a_k[2], *a_v[2], *a_s[2], *c_u[2], *c_o[2], *state[2];
    u64 *o[2]; long long ob, oh;
    u64* state_out[2];
    const int32_t* decay;
    u64* box;
    int B, H, dk, dv, bits, slices;
};
constexpr int kSlice = 32;                    // columns of the state in a workgroup: sixteen lanes, two columns each
constexpr int kGroups = 256 / (kSlice / 2);   // rows at a time
constexpr int kStepBoxes = 1024;              // four workgroups to a compute unit
constexpr int kMaxD = MPC_ATTENTION_MAX_D;
// send buffers of a workgroup, per direction: k and q, v, and the two rows of the state that a thread sends at a time; they stay in
// the L2
constexpr size_t kStepBoxWords = 2 * kMaxD + kSlice + 2 * 256 * 2;

struct StepShared {
    u64 part[2][kGroups][kSlice];
    u64 kq[2][3][kMaxD];                      // k, q: party 0's operand, opened words, party 1's mask
};

// One slice of one head's state; WHOLE: all of its columns are there.
template <bool WHOLE> __device__ __forceinline__ void step_slice(const StepArgs& q, StepShared& lds, u64* box, unsigned bh, unsigned slice)
{
    const int pair = threadIdx.x % (kSlice / 2), group = threadIdx.x / (kSlice / 2);
    const unsigned b = bh / q.H, h = bh - b * q.H;
    const int e = slice * kSlice + pair * 2, n = q.dv - e;                     // columns from this thread's first one on
    const u64 f = (uint32_t)q.decay[h * (kChunk + 1) + 1];
    const auto two = [&](const u64* p) {                                       // a thread's words of a row, read for good
        if (WHOLE) return __builtin_nontemporal_load(reinterpret_cast<const u64x2u*>(p));
        return u64x2u{ n > 0 ? p[0] : 0, n > 1 ? p[1] : 0 };
    };
    const auto put = [&](u64* p, u64x2u w) {
        if (WHOLE) __builtin_nontemporal_store(w, reinterpret_cast<u64x2u*>(p));
        else { if (n > 0) p[0] = w.x; if (n > 1) p[1] = w.y; }
    };
    struct Row { u64x2u s0, s1, c0, c1, a0, a1; };
    const long long first = (long long)bh * q.dk * q.dv + e;
    const auto row = [&](int d) {
        const long long o = first + (long long)min(d, q.dk - 1) * q.dv;
        return Row{ two(q.state[0] + o), two(q.state[1] + o), two(q.c_u[0] + o), two(q.c_u[1] + o), two(q.a_s[0] + o), two(q.a_s[1] + o) };
    };
    const long long ov = b * q.v.b + h * q.v.h + e, oav = (long long)bh * q.dv + e;
    const u64x2u v0 = two(q.v.p[0] + ov), v1 = two(q.v.p[1] + ov), av0 = two(q.a_v[0] + oav), av1 = two(q.a_v[1] + oav);
    {
        const int which = threadIdx.x / kMaxD, d = threadIdx.x % kMaxD;
        const Rows& x = which ? q.q : q.k;
        const u64* const* a = which ? q.a_q : q.a_k;
        if (d < q.dk) {
            const long long o = b * x.b + h * x.h + d, oa = (long long)bh * q.dk + d;
            const u64 x0 = x.p[0][o], m1 = a[1][oa], e1 = x.p[1][o] - m1, e0 = x0 - a[0][oa];
            if (slice == 0) { box[threadIdx.x] = e1; box[kStepBoxWords + threadIdx.x] = e0; }
            lds.kq[which][0][d] = x0 + e1; lds.kq[which][1][d] = e0 + e1; lds.kq[which][2][d] = m1;
        }
    }
    const u64x2u f0 = v0 - av0, f1 = v1 - av1, y0 = v0 + f1, fv = f0 + f1;
    if (group == 0) {
        u64* const to = box + 2 * kMaxD + pair * 2;
        *reinterpret_cast<u64x2u*>(to) = f1; *reinterpret_cast<u64x2u*>(to + kStepBoxWords) = f0;
    }
    u64x2u z0 = { 0, 0 }, z1 = { 0, 0 };
    const auto use = [&](const Row& r, int d, int slot) {
        if (d >= q.dk) return;
        const u64x2u w0 = r.s0 * f + r.c0 + lds.kq[0][0][d] * y0, w1 = r.s1 * f + r.c1 + lds.kq[0][1][d] * av1 + lds.kq[0][2][d] * fv;
        const u64x2u s0 = { rescaled<0>(w0.x, q.bits), rescaled<0>(w0.y, q.bits) }, s1 = { rescaled<1>(w1.x, q.bits), rescaled<1>(w1.y, q.bits) };
        const long long o = first + (long long)d * q.dv;
        put(q.state_out[0] + o, s0); put(q.state_out[1] + o, s1);
        const u64x2u e1 = s1 - r.a1, e0 = s0 - r.a0;
        u64* const to = box + 2 * kMaxD + kSlice + (slot * 256 + threadIdx.x) * 2;
        *reinterpret_cast<u64x2u*>(to) = e1; *reinterpret_cast<u64x2u*>(to + kStepBoxWords) = e0;
        z0 += lds.kq[1][0][d] * (s0 + e1);
        z1 += lds.kq[1][1][d] * r.a1 + lds.kq[1][2][d] * (e0 + e1);
    };
    for (int d0 = 0; d0 < q.dk; d0 += 2 * kGroups) {
        const int d = d0 + group;
        const Row r0 = row(d), r1 = row(d + kGroups);
        if (d0 == 0) __syncthreads();                                          // k and q are there
        use(r0, d, 0);
        use(r1, d + kGroups, 1);
    }
    lds.part[0][group][pair * 2] = z0.x; lds.part[0][group][pair * 2 + 1] = z0.y;
    lds.part[1][group][pair * 2] = z1.x; lds.part[1][group][pair * 2 + 1] = z1.y;
    __syncthreads();
    if (threadIdx.x < 2 * kSlice) {
        const int party = threadIdx.x / kSlice, c = threadIdx.x % kSlice, at = slice * kSlice + c;
        if (at < q.dv) {
            u64 z = q.c_o[party][(long long)bh * q.dv + at];
            for (int g = 0; g < kGroups; ++g) z += lds.part[party][g][c];
            q.o[party][b * q.ob + h * q.oh + at] = rescaled(party, z, q.bits);
        }
    }
    __syncthreads();
}

// A state element moves 64 bytes (the state, its mask and the outer product's addend of both parties in, the new state out): bound
// by HBM.  2048 heads of 64 x 64: 110 us, 5.1 TB/s; with slices of 16 columns 124, with ordinary stores 118, with send buffers
// for a whole slice, which leave the L2, 139.  96 heads of 64 x 64 are 192 workgroups, not enough for the chip's memory: 10 us, 2.6
// TB/s.  Columns that fill no slice are moved word by word: 640 heads of 97 x 99 131 us, of 96 x 96 79.  Four workgroups to a
// unit leave a thread 128 registers: three addresses are spilled (28 bytes a lane) and read again once a slice, none for a row.
__global__ __launch_bounds__(256, 4) void k_step(StepArgs q)
{
    __shared__ StepShared lds;
    u64* const box = q.box + (size_t)blockIdx.x * 2 * kStepBoxWords;
    const unsigned jobs = (unsigned)q.B * q.H * q.slices;
    for (unsigned job = blockIdx.x; job < jobs; job += gridDim.x) {
        const unsigned bh = job / q.slices, slice = job - bh * q.slices;
        if ((int)(slice + 1) * kSlice <= q.dv) step_slice<true>(q, lds, box, bh, slice);
        else step_slice<false>(q, lds, box, bh, slice);
    }
}

bool strides_in(const mpc_strides& s) { return s.batch >= 0 && s.token >= 0 && s.head >= 0; }
bool far_tokens(const mpc_strides& s, int T) { return T > 1 && s.token > kMaxStride; }
// beyond MPC_ATTENTION_MAX_EXTENT words from the first entry of an axis to its last one: offsets are counted in 64 bits
bool far_apart(const mpc_strides& s, int B, int T, int H)
{
    const auto far = [](long long stride, int n) { return n > 1 && stride > MPC_ATTENTION_MAX_EXTENT / (n - 1); };
    return far(s.batch, B) || far(s.token, T) || far(s.head, H);
}

// words from the first to the last one of [B][T][H][d] with these strides
size_t extent(const mpc_strides& s, int B, int T, int H, int d)
{
    return (size_t)s.batch * (B - 1) + (size_t)s.token * (T - 1) + (size_t)s.head * (H - 1) + d;
}

// no two of the output's words share a place: in the order of their strides, every axis steps over the ones within it
bool strides_out(const mpc_strides& s, int B, int T, int H, int d)
{
    long long st[3] = { s.batch, s.token, s.head }; int n[3] = { B, T, H };
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (st[j] > st[j + 1]) { std::swap(st[j], st[j + 1]); std::swap(n[j], n[j + 1]); }
    long long within = d;
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) continue;
        if (st[i] < within) return false;
        within = st[i] * (n[i] - 1) + within;
    }
    return true;
}

Rows rows_of(const mpc_cshare& s, const mpc_strides& st) { return Rows{ { s.p[0], s.p[1] }, st.batch, st.token, st.head }; }

bool both(const mpc_cshare& s) { return s.p[0] && s.p[1]; }
mpc_cshare seen(const mpc_share& s) { return mpc_cshare{ { s.p[0], s.p[1] } }; }

int shape_ok(mpc_ctx* c, int B, int T, int H, int dk, int dv)
{
    if (B <= 0 || T <= 0 || H <= 0 || dk <= 0 || dv <= 0) return MPC_EINVAL;
    if (dk > MPC_ATTENTION_MAX_D || dv > MPC_ATTENTION_MAX_D || H > INT32_MAX / (kChunk + 1) || T > INT32_MAX - kChunk) return MPC_ERANGE;
    const long long chunks = (T + kChunk - 1) / kChunk, heads = (long long)B * H;
    if (heads > INT32_MAX / 5 || chunks > INT32_MAX / 5 / heads) return MPC_ERANGE;           // jobs of a launch; no product past 64 bits
    return c && c->frac_bits > 30 ? MPC_ERANGE : MPC_OK;       // a decay of one has to fit 31 bits
}

struct ChunkPlan { size_t part, u, box, total; long long chunks; };
ChunkPlan plan(int B, int T, int H, int dk, int dv)
{
    ChunkPlan p{};
    const size_t BH = (size_t)B * H;
    p.chunks = (T + kChunk - 1) / kChunk;
    p.part = BH * T * dv; p.u = BH * p.chunks * dk * dv; p.box = kStateBoxes * 512 > kBoxes * 2 * kBoxWords ? kStateBoxes * 512 : kBoxes * 2 * kBoxWords;
    p.total = 2 * align_up(p.part * 8) + 2 * align_up(p.u * 8) + align_up(p.box * 8);
    return p;
}

}  // namespace

extern "C" {

size_t mpc_linear_attention_workspace_bytes(int B, int T, int H, int dk, int dv)
{
    return shape_ok(nullptr, B, T, H, dk, dv) == MPC_OK ? plan(B, T, H, dk, dv).total : 0;
}

size_t mpc_linear_attention_step_workspace_bytes(int B, int H, int dk, int dv)
{
    return shape_ok(nullptr, B, 1, H, dk, dv) == MPC_OK ? (size_t)kStepBoxes * 2 * kStepBoxWords * 8 : 0;
}

int mpc_linear_attention(mpc_ctx* c, const mpc_attention_operands* x, const mpc_attention_material* m, int B, int T, int H, int dk, int dv)
{
    if (!c || !x || !m) return MPC_EINVAL;
    const auto [q, k, v, sq, sk, sv, decay, state, o, so, state_out] = *x;
    if (!decay || !both(q) || !both(k) || !both(v) || !both(seen(o))) return MPC_EINVAL;
    if (!state.p[0] != !state.p[1] || !state_out.p[0] != !state_out.p[1]) return MPC_EINVAL;
    const mpc_cshare* const mats[] = { &m->a_q, &m->a_k, &m->a_qd, &m->a_kd, &m->a_v, &m->a_w, &m->a_s, &m->c_p, &m->c_u, &m->c_o };
    for (const mpc_cshare* w : mats) if (!both(*w)) return MPC_EINVAL;
    MPC_TRY(shape_ok(c, B, T, H, dk, dv));
    if (!strides_in(sq) || !strides_in(sk) || !strides_in(sv) || !strides_in(so)) return MPC_EINVAL;
    if (far_apart(sq, B, T, H) || far_apart(sk, B, T, H) || far_apart(sv, B, T, H) || far_apart(so, B, T, H)) return MPC_ERANGE;
    if (!strides_out(so, B, T, H, dv)) return MPC_EINVAL;
    if (far_tokens(sq, T) || far_tokens(sk, T) || far_tokens(sv, T)) return MPC_ERANGE;
    const ChunkPlan p = plan(B, T, H, dk, dv);
    const size_t n_o = extent(so, B, T, H, dv) * 8, n_s = (size_t)B * H * dk * dv * 8;
    const size_t BHT = (size_t)B * H * T * 8;
    const size_t sizes[] = { BHT * dk, BHT * dk, BHT * dk, BHT * dk, BHT * dv, BHT * kChunk, p.u * 8, BHT * kChunk, p.u * 8, BHT * dv };
    const mpc_cshare* const in[] = { &q, &k, &v };
    const size_t n_in[] = { extent(sq, B, T, H, dk) * 8, extent(sk, B, T, H, dk) * 8, extent(sv, B, T, H, dv) * 8 };
    for (int pass = 0; pass < 2; ++pass) {
        const mpc_share& out = pass ? state_out : o;
        const size_t n = pass ? n_s : n_o;
        if (!out.p[0]) continue;
        for (int i = 0; i < 3; ++i) if (!outputs_apart(out, n, *in[i], n_in[i], false)) return MPC_EINVAL;
        for (int i = 0; i < 10; ++i) if (!outputs_apart(out, n, *mats[i], sizes[i], false)) return MPC_EINVAL;
        if (state.p[0] && !outputs_apart(out, n, state, n_s, pass == 1)) return MPC_EINVAL;
    }
    const size_t n_decay = (size_t)H * (kChunk + 1) * 4;
    if (!apart(o, n_o, decay, n_decay)) return MPC_EINVAL;
    if (state_out.p[0] && (!outputs_apart(o, n_o, seen(state_out), n_s, false) || !apart(state_out, n_s, decay, n_decay))) return MPC_EINVAL;

    ChunkArgs a{};
    a.q = rows_of(q, sq); a.k = rows_of(k, sk); a.v = rows_of(v, sv);
    a.decay = decay; a.ob = so.batch; a.ot = so.token; a.oh = so.head;
    WsAlloc ws(c->ws, c->ws_bytes);
    for (int i = 0; i < 2; ++i) {
        a.a_q[i] = m->a_q.p[i]; a.a_k[i] = m->a_k.p[i]; a.a_qd[i] = m->a_qd.p[i]; a.a_kd[i] = m->a_kd.p[i]; a.a_v[i] = m->a_v.p[i];
        a.a_w[i] = m->a_w.p[i]; a.a_s[i] = m->a_s.p[i]; a.c_p[i] = m->c_p.p[i]; a.c_u[i] = m->c_u.p[i]; a.c_o[i] = m->c_o.p[i];
        a.state[i] = state.p[i]; a.o[i] = o.p[i]; a.state_out[i] = state_out.p[i];
        a.part[i] = ws.take<u64>(p.part); a.u[i] = ws.take<u64>(p.u);
    }
    a.box = ws.take<u64>(p.box);
    if (!ws.ok) return MPC_ENOMEM;
    a.B = B; a.H = H; a.T = T; a.dk = dk; a.dv = dv; a.chunks = (int)p.chunks; a.bits = c->frac_bits;
    a.mt = (dk + 63) / 64; a.nt = (dv + 63) / 64; a.cells = (unsigned)((long long)B * H * p.chunks);
    const auto grid = [](long long jobs, long long most) { return dim3((unsigned)(jobs < most ? jobs : most)); };
    const long long rounds = (a.cells + 7) / 8 * 8;               // the same for every die
    // With units to spare, P is formed again for each tile of W V: 8 heads of 128 x 128 over 200 tokens 83 -> 74 us.  In more than one round
    // of workgroups that is work for nothing.
    a.rows_jobs = rounds * (a.nt + a.mt * a.nt) <= kBoxes ? a.nt : 1;
    MPC_TRY(lane_first(c));
    k_chunk_open<<<grid(rounds * (a.rows_jobs + a.mt * a.nt), kBoxes), kThreads, kOperands * kOperand, c->s[0]>>>(a);
    k_chunk_states<<<grid(((long long)n_s / 8 + 255) / 256, kStateBoxes), 256, 0, c->s[0]>>>(a);
    k_chunk_out<<<grid(rounds * a.nt, kBoxes), kThreads, kOperands * kOperand, c->s[0]>>>(a);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

int mpc_linear_attention_step(mpc_ctx* c, const mpc_attention_operands* x, const mpc_attention_step_material* m, int B, int H, int dk, int dv)
{
    if (!c || !x || !m) return MPC_EINVAL;
    auto [q, k, v, sq, sk, sv, decay, state, o, so, state_out] = *x;
    if (!decay || !both(q) || !both(k) || !both(v) || !both(state) || !both(seen(o)) || !both(seen(state_out))) return MPC_EINVAL;
    const mpc_cshare* const mats[] = { &m->a_q, &m->a_k, &m->a_v, &m->a_s, &m->c_u, &m->c_o };
    for (const mpc_cshare* w : mats) if (!both(*w)) return MPC_EINVAL;
    MPC_TRY(shape_ok(c, B, 1, H, dk, dv));
    sq.token = sk.token = sv.token = so.token = 0;
    if (!strides_in(sq) || !strides_in(sk) || !strides_in(sv) || !strides_in(so)) return MPC_EINVAL;
    if (far_apart(sq, B, 1, H) || far_apart(sk, B, 1, H) || far_apart(sv, B, 1, H) || far_apart(so, B, 1, H)) return MPC_ERANGE;
    if (!strides_out(so, B, 1, H, dv)) return MPC_EINVAL;
    const size_t BH = (size_t)B * H * 8, n_s = BH * dk * dv, n_o = extent(so, B, 1, H, dv) * 8;
    const size_t sizes[] = { BH * dk, BH * dk, BH * dv, n_s, n_s, BH * dv };
    const mpc_cshare* const in[] = { &q, &k, &v };
    const size_t n_in[] = { extent(sq, B, 1, H, dk) * 8, extent(sk, B, 1, H, dk) * 8, extent(sv, B, 1, H, dv) * 8 };
    for (int pass = 0; pass < 2; ++pass) {
        const mpc_share& out = pass ? state_out : o;
        const size_t n = pass ? n_s : n_o;
        for (int i = 0; i < 3; ++i) if (!outputs_apart(out, n, *in[i], n_in[i], false)) return MPC_EINVAL;
        for (int i = 0; i < 6; ++i) if (!outputs_apart(out, n, *mats[i], sizes[i], false)) return MPC_EINVAL;
        if (!outputs_apart(out, n, state, n_s, pass == 1)) return MPC_EINVAL;
    }
    const size_t n_decay = (size_t)H * (kChunk + 1) * 4;
    if (!outputs_apart(o, n_o, seen(state_out), n_s, false) || !apart(o, n_o, decay, n_decay) || !apart(state_out, n_s, decay, n_decay)) return MPC_EINVAL;
    if (!c->ws || c->ws_bytes < mpc_linear_attention_step_workspace_bytes(B, H, dk, dv)) return MPC_ENOMEM;
    StepArgs a{};
    a.q = rows_of(q, sq); a.k = rows_of(k, sk); a.v = rows_of(v, sv);
    for (int i = 0; i < 2; ++i) {
        a.a_q[i] = m->a_q.p[i]; a.a_k[i] = m->a_k.p[i]; a.a_v[i] = m->a_v.p[i]; a.a_s[i] = m->a_s.p[i];
        a.c_u[i] = m->c_u.p[i]; a.c_o[i] = m->c_o.p[i]; a.state[i] = state.p[i]; a.o[i] = o.p[i]; a.state_out[i] = state_out.p[i];
    }
    a.ob = so.batch; a.oh = so.head; a.decay = decay; a.box = reinterpret_cast<u64*>(c->ws);
    a.B = B; a.H = H; a.dk = dk; a.dv = dv; a.bits = c->frac_bits; a.slices = (dv + kSlice - 1) / kSlice;
    const long long jobs = (long long)B * H * a.slices;           // at most four slices to a head
    MPC_TRY(lane_first(c));
    k_step<<<dim3((unsigned)(jobs < kStepBoxes ? jobs : kStepBoxes)), 256, 0, c->s[0]>>>(a);
    MPC_HIP(c, hipGetLastError());
    return lane_fanout(c);
}

}  // extern "C"
