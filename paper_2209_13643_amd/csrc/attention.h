// Shared by the attention and public-weight kernels: vector access, the local rescale, overlap checks of the entry points.
#pragma once
#include "common.h"

typedef u64 u64x2u __attribute__((ext_vector_type(2), aligned(8)));   // two words at any word's address

// z >> bits for bits in [0, 31], in two single-width instructions
__device__ __forceinline__ u64 shifted(u64 z, int bits)
{
    const uint32_t lo = (uint32_t)z, hi = (uint32_t)(z >> 32);
    return (u64)(hi >> bits) << 32 | __builtin_amdgcn_alignbit(hi, lo, bits);
}
// one party's side of the local rescale by 0 to 31 bits; none leaves the word as it is
template <int PARTY> __device__ __forceinline__ u64 rescaled(u64 z, int bits)
{
    return PARTY == 0 ? shifted(z, bits) : (u64)0 - shifted((u64)0 - z, bits);
}
__device__ __forceinline__ u64 rescaled(int party, u64 z, int bits) { return party == 0 ? rescaled<0>(z, bits) : rescaled<1>(z, bits); }

static inline bool overlap(const void* p, size_t np, const void* q, size_t nq)
{
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + nq && b < a + np;
}
// a launch has fewer than 2^32 threads
static inline bool launchable(size_t blocks, size_t threads) { return blocks <= UINT32_MAX / threads; }
// an output apart from a public array
static inline bool apart(const mpc_share& out, size_t n_out, const void* p, size_t n)
{
    return !overlap(out.p[0], n_out, p, n) && !overlap(out.p[1], n_out, p, n);
}
// every output apart from every input, other than an output that is the very array of its own party's input
static inline bool outputs_apart(const mpc_share& out, size_t n_out, const mpc_cshare& in, size_t n_in, bool may_be_same)
{
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            if (may_be_same && i == j && (const uint64_t*)out.p[i] == in.p[j]) continue;
            if (overlap(out.p[i], n_out, in.p[j], n_in)) return false;
        }
    return !overlap(out.p[0], n_out, out.p[1], n_out);
}
