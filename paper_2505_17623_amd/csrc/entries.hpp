// entries.hpp -- a layer's product that is computed entry by entry (the gated
// product, the token embedding), with the rescale / ReLU witness of Sec. II-A
// and III-B in the same pass when the caller has announced it (WitEpi): each
// entry of C gives R, Rm, Y, Z and the bit word while it is in registers, and
// the workgroup's partial claims at (r1, r2) and range flag.
//
// A thread keeps its V columns over all its rows, so a claim is sum_col E2[col]
// (sum_row E1[row] z): E1 in limbs (21 bits against the 31-bit R and Y, 31
// bits against the 16-bit Rm), the inner sums exact in int64 (at most 2^12
// rows a thread: N <= 2^31 over 2^18 threads of two columns), one product in F_p a
// column at the end; Z~ follows from R~ and Y~.
#pragma once
#include <type_traits>

#include "claims.hpp"
#include "common.hpp"
#include "m61.hpp"

namespace ra {

constexpr int entries_lds_words(int nt) { return m61::block_sum_words(3, nt); }

// Columns a thread takes: 2 where rows allow it and the outputs are aligned for
// stores of pairs.
inline int entries_width(uint64_t k, const int64_t *C, const WitEpi *we)
{
    uintptr_t a = (uintptr_t)C;
    if (we)
        a |= (uintptr_t)we->bits | ((uintptr_t)we->R | (uintptr_t)we->Y | (uintptr_t)we->Z) << 1 | (uintptr_t)we->Rm << 2;
    return k >= 2 && (a & 15) == 0 ? 2 : 1;
}
// Workgroups of nt threads (a power of two, one witness partial each; N = n k).
inline int entries_blocks(uint64_t N, int V, int nt)
{
    uint64_t b = 1;
    while (b < (uint64_t)kMaxBlocks && b * nt * V < N) b <<= 1;
    return (int)b;
}

// f(integral constants V and WIT) for the variant that k columns and e's buffers take.
template <typename F> inline void entries_variant(uint64_t k, const EntriesArgs &e, F f)
{
    using std::integral_constant;
    const bool two = entries_width(k, e.C, e.wit ? &e.we : nullptr) == 2;
    if (two && e.wit) f(integral_constant<int, 2>{}, integral_constant<bool, true>{});
    else if (two) f(integral_constant<int, 2>{}, integral_constant<bool, false>{});
    else if (e.wit) f(integral_constant<int, 1>{}, integral_constant<bool, true>{});
    else f(integral_constant<int, 1>{}, integral_constant<bool, false>{});
}

// Workgroup blk of nblk (NT threads each): load(row, col, c) gives V entries
// of C from (row, col) on, e1(row) and e2(col) eq(r1, row) and eq(r2, col)
// (canonical).  Without WIT C is written and the workgroup's smallest and
// largest entry, to mm[2 blk ..].  red: entries_lds_words(NT) words.
template <int V, bool WIT, int NT, typename Load, typename E1, typename E2>
__device__ __forceinline__ void entries_block(const Load &load, const E1 &eq1v, const E2 &eq2v, uint64_t n, int lk,
                                              int64_t *__restrict__ C, const WitEpi &we, int64_t *__restrict__ mm,
                                              int blk, int nblk, uint64_t *red)
{
    typedef long long v2l __attribute__((ext_vector_type(2)));
    typedef int v2i __attribute__((ext_vector_type(2)));
    typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
    const uint64_t G = (uint64_t)nblk * NT, g = (uint64_t)blk * NT + threadIdx.x;  // powers of two
    const uint64_t q = (1ull << lk) / V, rstep = G > q ? G / q : 1;
    uint64_t acc[3] = {0, 0, 0};
    int64_t lo = INT64_MAX, hi = INT64_MIN;
    int oor = 0;
    for (uint64_t cq = g & (q - 1); cq < q; cq += G) {
        const uint64_t col = cq * V;
        uint64_t sr[V][3] = {}, sm[V][2] = {}, sy[V][3] = {};
        for (uint64_t row = G > q ? g / q : 0; row < n; row += rstep) {
            int64_t c[V];
            load(row, col, c);
            const uint64_t x = (row << lk) + col;
            if constexpr (V == 2) {
                *(v2l *)&C[x] = v2l{c[0], c[1]};
            } else {
                C[x] = c[0];
            }
            if constexpr (!WIT) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    lo = c[i] < lo ? c[i] : lo;
                    hi = c[i] > hi ? c[i] : hi;
                }
                continue;
            }
            const uint64_t e = eq1v(row);
            const int32_t e0 = (int32_t)(e & 0x1FFFFF), e1 = (int32_t)((e >> 21) & 0x1FFFFF), e2 = (int32_t)(e >> 42);
            const int32_t el = (int32_t)(e & 0x7FFFFFFF), eh = (int32_t)(e >> 31);
            WitOut o[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
                o[i] = witness_entry(c[i], we.s, we.t, we.relu, we.half, oor);
                sr[i][0] += (uint64_t)((int64_t)e0 * o[i].r);
                sr[i][1] += (uint64_t)((int64_t)e1 * o[i].r);
                sr[i][2] += (uint64_t)((int64_t)e2 * o[i].r);
                sm[i][0] += (uint64_t)((int64_t)el * o[i].rm);
                sm[i][1] += (uint64_t)((int64_t)eh * o[i].rm);
                sy[i][0] += (uint64_t)((int64_t)e0 * o[i].y);
                sy[i][1] += (uint64_t)((int64_t)e1 * o[i].y);
                sy[i][2] += (uint64_t)((int64_t)e2 * o[i].y);
            }
            if constexpr (V == 2) {
                *(v2i *)&we.R[x] = v2i{o[0].r, o[1].r};
                *(v2i *)&we.Y[x] = v2i{o[0].y, o[1].y};
                *(v2i *)&we.Z[x] = v2i{o[0].z, o[1].z};
                *(v2u16 *)&we.Rm[x] = v2u16{(unsigned short)o[0].rm, (unsigned short)o[1].rm};
                *(v2l *)&we.bits[x] = v2l{(long long)o[0].w, (long long)o[1].w};
            } else {
                we.R[x] = o[0].r;
                we.Y[x] = o[0].y;
                we.Z[x] = o[0].z;
                we.Rm[x] = (uint16_t)o[0].rm;
                we.bits[x] = o[0].w;
            }
        }
        if constexpr (WIT) {
            auto value3 = [](const uint64_t *s) {
                return m61::fold(m61::from_i64((int64_t)s[0]) + m61::rotl(m61::from_i64((int64_t)s[1]), 21) +
                                 m61::rotl(m61::from_i64((int64_t)s[2]), 42));
            };
#pragma unroll
            for (int i = 0; i < V; i++) {
                const uint64_t e2 = eq2v(col + i);
                acc[0] = m61::lmacc(acc[0], value3(sr[i]), e2);
                acc[1] = m61::lmacc(acc[1],
                                    m61::fold(m61::from_i64((int64_t)sm[i][0]) +
                                              m61::rotl(m61::from_i64((int64_t)sm[i][1]), 31)),
                                    e2);
                acc[2] = m61::lmacc(acc[2], value3(sy[i]), e2);
            }
        }
    }
    if constexpr (!WIT) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const int64_t a = __shfl_xor(lo, off, 64), b = __shfl_xor(hi, off, 64);
            lo = a < lo ? a : lo;
            hi = b > hi ? b : hi;
        }
        int64_t *w = (int64_t *)red;
        if ((threadIdx.x & 63) == 0) {
            w[2 * (threadIdx.x >> 6)] = lo;
            w[2 * (threadIdx.x >> 6) + 1] = hi;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int v = 1; v < NT / 64; v++) {
                lo = w[2 * v] < lo ? w[2 * v] : lo;
                hi = w[2 * v + 1] > hi ? w[2 * v + 1] : hi;
            }
            mm[2 * blk] = lo;
            mm[2 * blk + 1] = hi;
        }
    } else {
        const int any = __syncthreads_or(oor);
        const uint64_t *t = m61::block_sum_lds<3>(acc, red);
        if (threadIdx.x == 0) {
            const uint64_t z = we.relu ? m61::rotl(m61::add(t[0], t[2]), 60) : t[0];  // 2^60 = 1/2
            for (int i = 0; i < 3; i++) we.claim_part[4 * (size_t)blk + i] = t[i];
            we.claim_part[4 * (size_t)blk + 3] = z;
            we.flags[blk] = (uint32_t)any;
        }
    }
}

}  // namespace ra
