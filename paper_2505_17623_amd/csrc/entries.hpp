// entries.hpp -- a layer's product that is computed entry by entry (the gated
// product, the token embedding), with the rescale / ReLU witness of Sec. II-A
// and III-B in the same pass when the caller has announced it (WitEpi): each
// entry of C gives R, Rm, Y, Z and the bit word while it is in registers, and
// the workgroup's partial claims at (r1, r2) and range flag.
//
// A thread keeps its V columns over all its rows, so a claim is sum_col E2[col]
// (sum_row E1[row] z), E1 in limbs of 31 bits, the inner sums exact in int64 (at
// most 2^12 rows a thread: N <= 2^31 over 2^19 threads of a column or two), one
// product in F_p a column at the end.  Only Rm~ and Y~ are summed: C = 2^s R +
// Rm - half entry by entry, so R~ follows from C~, which is the sum that the
// product's sum-check claims, and Z~ from R~ and Y~ (claims.hpp).
#pragma once
#include <type_traits>

#include "claims.hpp"
#include "common.hpp"
#include "m61.hpp"

namespace ra {

constexpr int entries_lds_words(int nt) { return m61::block_sum_words(2, nt); }

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

// witness_entry (claims.hpp) with R in 32 bits from the shift on: the same for
// an entry within the range; *oor is set for every other.
__device__ __forceinline__ WitOut witness_entry32(int64_t c, int s, int t, int relu, int64_t half, int &oor)
{
    WitOut o;
    const int64_t cc = c + half, q = cc >> s;
    o.r = (int32_t)q;
    const int32_t sign = o.r >> 31;
    oor |= (int32_t)(q >> 32) != sign || ((uint32_t)(o.r ^ sign) >> (t + 1)) != 0;
    o.rm = (int32_t)((uint32_t)cc & ((1u << s) - 1u));
    o.y = (o.r ^ sign) - sign;
    o.z = relu ? o.r & ~sign : o.r;
    o.w = (uint64_t)(uint32_t)o.rm | ((uint64_t)((uint32_t)o.r + (2u << t)) << s);
    if (relu) o.w |= (uint64_t)(uint32_t)o.y << (s + t + 2);
    return o;
}

// The workgroup's witness partial: its sums of Rm~ and Y~ and its range flag.
template <int NT>
__device__ __forceinline__ void entries_claims(const uint64_t (&acc)[2], int oor, const WitEpi &we, int blk, uint64_t *red)
{
    const int any = __syncthreads_or(oor);
    const uint64_t *t = m61::block_sum_lds<2>(acc, red);
    if (threadIdx.x < 4)
        we.claim_part[4 * (size_t)blk + threadIdx.x] = threadIdx.x == 1 || threadIdx.x == 2 ? t[threadIdx.x - 1] : 0;
    if (threadIdx.x == 0) we.flags[blk] = (uint32_t)any;
}
// The workgroup's smallest and largest entry, to mm[2 blk ..].
template <int NT>
__device__ __forceinline__ void entries_extremes(int64_t lo, int64_t hi, int64_t *mm, int blk, uint64_t *red)
{
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
    if (threadIdx.x != 0) return;
    for (int v = 1; v < NT / 64; v++) {
        lo = w[2 * v] < lo ? w[2 * v] : lo;
        hi = w[2 * v + 1] > hi ? w[2 * v + 1] : hi;
    }
    mm[2 * blk] = lo;
    mm[2 * blk + 1] = hi;
}

// Workgroup blk of nblk (NT threads each): load.fetch<M>(row, step, col, raw)
// asks for V entries of M rows from (row, col) on, load.value(raw[u], c) gives
// row u's; e1(row) and e2(col) are eq(r1, row) and eq(r2, col) (canonical).  A
// thread has the loads of U of its rows in flight.  Without WIT C is written
// and the workgroup's smallest and largest entry, to mm[2 blk ..].  red:
// entries_lds_words(NT) words.
template <int V, bool WIT, int NT, int U, typename Load, typename E1, typename E2>
__device__ __forceinline__ void entries_block(const Load &load, const E1 &eq1v, const E2 &eq2v, uint64_t n, int lk,
                                              int64_t *__restrict__ C, const WitEpi &we, int64_t *__restrict__ mm,
                                              int blk, int nblk, uint64_t *red)
{
    typedef long long v2l __attribute__((ext_vector_type(2)));
    typedef int v2i __attribute__((ext_vector_type(2)));
    typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
    const uint64_t G = (uint64_t)nblk * NT, g = (uint64_t)blk * NT + threadIdx.x;  // powers of two
    const uint64_t q = (1ull << lk) / V, rstep = G > q ? G / q : 1;
    auto limbs = [](const uint64_t *s) {  // s[0] + 2^31 s[1]
        return m61::fold(m61::from_i64((int64_t)s[0]) + m61::rotl(m61::from_i64((int64_t)s[1]), 31));
    };
    uint64_t acc[2] = {0, 0};
    int64_t lo = INT64_MAX, hi = INT64_MIN;
    int oor = 0;
    for (uint64_t cq = g & (q - 1); cq < q; cq += G) {
        const uint64_t col = cq * V;
        uint64_t sm[V][2] = {}, sy[V][2] = {}, fy[V] = {};
        auto rows = [&](auto count, uint64_t row0) {
            constexpr int M = decltype(count)::value;
            typename Load::Raw raw[M];
            uint64_t e[M];
            load.template fetch<M>(row0, rstep, col, raw);
            if constexpr (WIT)
#pragma unroll
                for (int u = 0; u < M; u++) e[u] = eq1v(row0 + u * rstep);
#pragma unroll
            for (int u = 0; u < M; u++) {
                int64_t c[V];
                load.value(raw[u], c);
                const uint64_t x = ((row0 + u * rstep) << lk) + col;
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
                const int32_t el = (int32_t)(e[u] & 0x7FFFFFFF), eh = (int32_t)(e[u] >> 31);
                WitOut o[V];
#pragma unroll
                for (int i = 0; i < V; i++) {
                    o[i] = witness_entry32(c[i], we.s, we.t, we.relu, we.half, oor);
                    sm[i][0] += (uint64_t)((int64_t)el * o[i].rm);
                    sm[i][1] += (uint64_t)((int64_t)eh * o[i].rm);
                    sy[i][0] += (uint64_t)((int64_t)el * o[i].y);
                    sy[i][1] += (uint64_t)((int64_t)eh * o[i].y);
                    if (we.t > 17) {  // |Y| <= 2^(t+1): past 2^18 a row's terms are reduced at once
                        fy[i] = m61::fold(fy[i] + limbs(sy[i]));
                        sy[i][0] = sy[i][1] = 0;
                    }
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
        };
        uint64_t row = G > q ? g / q : 0;  // the same number of rows for every thread that has any
        if constexpr (U > 1)
            for (; row + (U - 1) * rstep < n; row += U * rstep) rows(std::integral_constant<int, U>{}, row);
        for (; row < n; row += rstep) rows(std::integral_constant<int, 1>{}, row);
        if constexpr (WIT) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const uint64_t e2 = eq2v(col + i);
                acc[0] = m61::lmacc(acc[0], limbs(sm[i]), e2);
                acc[1] = m61::lmacc(acc[1], m61::fold(fy[i] + limbs(sy[i])), e2);
            }
        }
    }
    if constexpr (WIT) entries_claims<NT>(acc, oor, we, blk, red);
    else entries_extremes<NT>(lo, hi, mm, blk, red);
}

}  // namespace ra
