// embed.hip -- the token embedding with scaling as a layer's product: row i of
// C is scale times row tok[i] of the table E (zero for tok[i] = -1), i.e. C = S
// E with S the n x vocab matrix that holds scale at (i, tok[i]).  S is never
// formed: bound at r1 its columns are
//     W(v) = scale sum over the i with tok[i] = v of eq(r1, i),
// the lookup's transpose applied to eq(r1, .) (what a gradient of the table
// is to the rows' gradients), and
//     C~(r1, r2) = sum_v W(v) e(v),   e(v) = sum_j E[v, j] eq(r2, j),
// is the matrix layer's sum-check (Eq. (4)) over the vocabulary's variables,
// which ends in W~(rho), computable from the public tokens, and E~(rho, r2).
// Rows past the vocabulary and columns past the table's width are zero.
#include <algorithm>

#include "common.hpp"
#include "m61.hpp"
#include "ra.h"

namespace ra {

// W's sums: W(v) mod p is acc[v] + 2^32 acc[rows + v] (tail.hpp), each word a
// sum of values below 2^32, so no add wraps and their order does not matter.
// A token outside [-1, vocab) is not followed: it sets *bad.
__global__ __launch_bounds__(256) void k_embed_scatter(const int32_t *__restrict__ tok, uint32_t n, uint32_t vocab,
                                                       uint64_t rows, const uint64_t *__restrict__ E1, uint64_t scale,
                                                       unsigned long long *__restrict__ acc, uint32_t *__restrict__ bad)
{
    for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) {
        const int32_t v = tok[i];
        if (v < -1 || (v >= 0 && (uint32_t)v >= vocab)) {
            atomicOr(bad, 1u);
            continue;
        }
        if (v < 0) continue;
        const uint64_t e = m61::mul(E1[i], scale);
        atomicAdd(acc + v, (unsigned long long)(e & 0xFFFFFFFFull));
        atomicAdd(acc + rows + v, (unsigned long long)(e >> 32));
    }
}

// e(v) for v < rows, one wave per row: eq(r2, j) = hi 2^31 + lo, the two sums
// exact in int64 (|limb E| < 2^46, at most d / 64 + 1 <= 2^15 terms a lane).
__global__ __launch_bounds__(256) void k_embed_bind(const int16_t *__restrict__ E, uint64_t ld, uint32_t vocab, uint32_t d,
                                                    uint64_t rows, const uint64_t *__restrict__ E2,
                                                    uint64_t *__restrict__ b)
{
    const uint64_t v = ((uint64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;  // wave-uniform
    const int lane = threadIdx.x & 63;
    if (v >= rows) return;
    int64_t lo = 0, hi = 0;
    if (v < vocab)
        for (uint32_t j = lane; j < d; j += 64) {
            const uint64_t e = E2[j];
            const int32_t z = E[v * ld + j];
            lo += (int64_t)(int32_t)(e & 0x7FFFFFFFull) * z;
            hi += (int64_t)(int32_t)(e >> 31) * z;
        }
    const uint64_t s = m61::wave_sum(m61::add(m61::from_i64(lo), m61::rotl(m61::from_i64(hi), 31)));
    if (lane == 0) b[v] = s;
}

// C, n x 2^lk, and the tokens' status to *status (after the scatter, so *bad
// is final).
__global__ __launch_bounds__(256) void k_embed_product(const int32_t *__restrict__ tok, const int16_t *__restrict__ E,
                                                       uint64_t ld, uint32_t vocab, uint32_t d, int32_t scale, uint64_t N,
                                                       int lk, int64_t *__restrict__ C, const uint32_t *__restrict__ bad,
                                                       uint64_t *__restrict__ status)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = *bad;
    for (uint64_t x = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; x < N; x += (uint64_t)gridDim.x * blockDim.x) {
        const int32_t v = tok[x >> lk];
        const uint32_t j = (uint32_t)(x & ((1ull << lk) - 1));
        C[x] = v >= 0 && (uint32_t)v < vocab && j < d ? (int64_t)scale * E[(uint64_t)v * ld + j] : 0;
    }
}

void launch_embed_sides(const EmbedArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(k_embed_scatter, dim3((unsigned)std::min<uint64_t>((a.n + 255) / 256, 1024)), dim3(256), 0, st,
                       a.tok, a.n, a.vocab, a.rows, a.E1, a.scale < 0 ? m61::P - (uint64_t)(-(int64_t)a.scale) : (uint64_t)a.scale,
                       (unsigned long long *)a.acc, a.bad);
    hipLaunchKernelGGL(k_embed_bind, dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, st, a.E, a.ld, a.vocab, a.d,
                       a.rows, a.E2, a.b);
}

void launch_embed_product(const EmbedArgs &a, int64_t *C, hipStream_t st)
{
    const uint64_t N = (uint64_t)a.n << a.lk;
    hipLaunchKernelGGL(k_embed_product, dim3((unsigned)std::min<uint64_t>((N + 255) / 256, 4096)), dim3(256), 0, st,
                       a.tok, a.E, a.ld, a.vocab, a.d, a.scale, N, a.lk, C, a.bad, a.status);
}

}  // namespace ra
