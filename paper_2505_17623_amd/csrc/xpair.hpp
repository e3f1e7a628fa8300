// xpair.hpp -- pieces of a sum-check round over the Boolean cube with the
// factor EQ(x) = eq(r, x) split off (xrounds.hip): the weights eq(r_>j, i) from
// suffix eq tables, and the sums of a pair of a product of two tables.  Shared
// by the ReLU zero-check (xrounds.hip) and the gated product (gate.hip).
#pragma once
#include "common.hpp"
#include "m61.hpp"

namespace ra {

// Terms of one pair with weight w of sum_x EQ(x) d(x) s(x), added to the
// folded acc[0..3) = Z_0, Z_1, U.  Inputs are folded or canonical.
__device__ __forceinline__ void relu_pair(uint64_t w, uint64_t d0, uint64_t d1, uint64_t s0, uint64_t s1,
                                          uint64_t *acc)
{
    const uint64_t ed0 = m61::lmul(w, d0), ed1 = m61::lmul(w, d1);
    acc[0] = m61::lmacc(acc[0], ed0, s0);
    acc[1] = m61::lmacc(acc[1], ed1, s1);
    acc[2] = m61::lmacc(acc[2], ed0 + ed1, s0 + s1);  // sums of two folded values are loose
}

template <int NV>
__device__ __forceinline__ void fold_all(uint64_t *acc)
{
#pragma unroll
    for (int q = 0; q < NV; q++) acc[q] = m61::fold(acc[q]);
}

// lo + z (hi - lo), folded.
__device__ __forceinline__ uint64_t fold(uint64_t lo, uint64_t hi, uint64_t z)
{
    return m61::lmacc(lo, z, m61::lsub(hi, lo));
}

// Field value of a small signed integer (|v| < 2^62), folded.
__device__ __forceinline__ uint64_t small_to_field(int64_t v) { return m61::fold((uint64_t)v + 4 * m61::P); }

// The weights eq(r_{j+c+1 .. j+C-1}, u) e of the pairs of C fused rounds in a
// sub-cube of weight e; rr = r_j .. r_{j+C-1}.
template <int C>
__device__ __forceinline__ void x_weights(uint64_t e, const uint64_t *rr, uint64_t (&w)[1 << C])
{
    // round c uses w[(1 << (C-1-c)) - 1 + u] (indices 0 .. 2^C - 2)
    w[0] = e;  // round C - 1 (u empty)
#pragma unroll
    for (int c = C - 2; c >= 0; c--) {
        const int hn = 1 << (C - 1 - c), base = hn - 1, pb = (hn >> 1) - 1;
        // u = (msb, rest): eq1(r_{j+c+1}, msb) times the weight of `rest` one round later
#pragma unroll
        for (int u = 0; u < hn / 2; u++) {
            const uint64_t hi = m61::lmul(rr[c + 1], w[pb + u]);
            w[base + hn / 2 + u] = hi;
            w[base + u] = m61::lsub(w[pb + u], hi);
        }
    }
}

// eq(r_{lN-nvar .. lN-1}, k) from the suffix heaps (folded or canonical).
__device__ __forceinline__ uint64_t suffix_weight(const uint64_t *HS, const uint64_t *LS, int nvar, int L, uint64_t k)
{
    if (nvar <= L) return LS[(1ull << nvar) + k];
    return m61::lmul(HS[(1ull << (nvar - L)) + (k >> L)], LS[(1ull << L) + (k & ((1ull << L) - 1))]);
}

}  // namespace ra
