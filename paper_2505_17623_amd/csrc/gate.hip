// gate.hip -- the gated product as a layer's product: C = A B entry by entry
// (the two factors are activations, e.g. the two projections of a gated
// feed-forward block), and its sum-check
//     C~(r1, r2) = sum_x eq(r, x) A(x) B(x),   r = (r1, r2), x over {0,1}^(log n k),
// of degree 3 (Sec. II-D), which ends in A~(rho) and B~(rho).  The witness and
// the range check of C are those of every layer.
//
// EQ(x) = eq(r, x) is split off as in xrounds.hip: round j's polynomial is
// K_j eq1(r_j, X) s_j(X) with K_j = prod_{l<j} eq1(r_l, rho_l) and
//     s_j(X) = sum_i eq(r_>j, i) a_X b_X,   a_X = a_lo + X (a_hi - a_lo),
// a quadratic known from three sums over the pairs (relu_pair): Z_0, Z_1 at X
// = 0, 1 and U = sum w (a_lo + a_hi)(b_lo + b_hi), with s_j(2) = 3 Z_0 + 6 Z_1
// - 2 U.
#include <algorithm>

#include "assemble.hpp"
#include "common.hpp"
#include "entries.hpp"
#include "m61.hpp"
#include "xpair.hpp"
#include "xsetup.hpp"

namespace ra {

// Entries i + t q (i < q, q a power of two), t < cnt <= NL, of a factor (int16
// or int32, rows `ld` entries apart, 0: one row for all).  An entry's place
// (x >> lk) ld + (x mod 2^lk) is additive over disjoint bits of x, so those of
// t q are the same for every thread.  All loads go out before any is waited
// for: the type is looked at once, and a load gives the extended value.
template <int NL>
__device__ __forceinline__ void gate_fetch(const GateSrc &s, uint64_t i, uint64_t q, int cnt, int lk, int32_t (&out)[NL])
{
    const uint64_t mask = (1ull << lk) - 1, at = (i >> lk) * s.ld + (i & mask);
    if (s.i16) {
        const int16_t *p = (const int16_t *)s.p + at;
#pragma unroll
        for (int t = 0; t < NL; t++)
            if (t < cnt) out[t] = p[((t * q) >> lk) * s.ld + ((t * q) & mask)];
    } else {
        const int32_t *p = (const int32_t *)s.p + at;
#pragma unroll
        for (int t = 0; t < NL; t++)
            if (t < cnt) out[t] = p[((t * q) >> lk) * s.ld + ((t * q) & mask)];
    }
}

// An int32 as a loose residue (m61.hpp): p + v, within 2^32 of 2^61.
__device__ __forceinline__ uint64_t int_to_loose(int64_t v) { return (uint64_t)v + m61::P; }

// V entries of C = A B, exact in int64 (|C| <= 2^62).
template <int V> struct GateProduct {
    GateSrc A, B;
    struct Raw {
        int32_t a[V], b[V];
    };
    template <int U>
    __device__ __forceinline__ void fetch(uint64_t row, uint64_t step, uint64_t col, Raw (&raw)[U]) const
    {
        // no more alignment than the entries have
        if (A.i16) {
#pragma unroll
            for (int u = 0; u < U; u++) pair16(A, row + u * step, col, raw[u].a);
        } else {
#pragma unroll
            for (int u = 0; u < U; u++)
                __builtin_memcpy(raw[u].a, (const int32_t *)A.p + (row + u * step) * A.ld + col, sizeof raw[u].a);
        }
        if (B.i16) {
#pragma unroll
            for (int u = 0; u < U; u++) pair16(B, row + u * step, col, raw[u].b);
        } else {
#pragma unroll
            for (int u = 0; u < U; u++)
                __builtin_memcpy(raw[u].b, (const int32_t *)B.p + (row + u * step) * B.ld + col, sizeof raw[u].b);
        }
    }
    __device__ __forceinline__ static void pair16(const GateSrc &s, uint64_t row, uint64_t col, int32_t (&v)[V])
    {
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = ((const int16_t *)s.p)[row * s.ld + col + i];
    }
    __device__ __forceinline__ void value(const Raw &r, int64_t (&c)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; i++) c[i] = (int64_t)r.a[i] * r.b[i];
    }
};

// The suffix eq tables of r (xsetup.hpp; the prefix products K_j the tails make
// for themselves) by the first nx threads, the eq tables E1 (r1) and E2 (r2) by
// the others.
__global__ __launch_bounds__(256) void k_gate_setup(XSetupArgs a, int nx, int ln, uint64_t *E1, uint64_t *E2)
{
    __shared__ uint64_t rl[64];
    if ((int)threadIdx.x < a.lN) rl[threadIdx.x] = a.r[threadIdx.x];
    __syncthreads();
    const uint64_t g = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (g < (uint64_t)nx) {
        x_tables_body(a, (int)g, rl);
        return;
    }
    const uint64_t i = g - nx, n = 1ull << ln;
    if (i < n) E1[i] = eq_suffix(rl, 0, ln, i);
    else if (i - n < 1ull << (a.lN - ln)) E2[i - n] = eq_suffix(rl, ln, a.lN - ln, i - n);
}

// C rounds of one sub-cube held in registers (u, v folded or loose), weights w
// (x_weights): round c's sums added to acc[3 c ..], folded every fourth pair.
template <int R>
__device__ __forceinline__ void gate_rounds(uint64_t (&u)[1 << R], uint64_t (&v)[1 << R], const uint64_t (&w)[1 << R],
                                            const uint64_t (&rho)[R], uint64_t (&acc)[3 * R])
{
#pragma unroll
    for (int c = 0; c < R; c++) {
        const int h = (1 << R) >> (c + 1), base = h - 1;
#pragma unroll
        for (int p = 0; p < h; p++) {
            // the terms summed before a fold, not folded into the sum one by
            // one: that order takes 50 more registers (140 against 94)
            const uint64_t e0 = m61::lmul(w[base + p], u[p]), e1 = m61::lmul(w[base + p], u[p + h]);
            acc[3 * c] += m61::lmul(e0, v[p]);
            acc[3 * c + 1] += m61::lmul(e1, v[p + h]);
            acc[3 * c + 2] += m61::lmul(e0 + e1, v[p] + v[p + h]);
            u[p] = fold(u[p], u[p + h], rho[c]);
            v[p] = fold(v[p], v[p + h], rho[c]);
            if ((p & 3) == 3 || p == h - 1) fold_all<3>(acc + 3 * c);
        }
    }
}

// R rounds j .. j + R - 1 over tables of 2^R q entries in one pass: a thread
// holds the 2^R entries i + t q that end in entry i of the folded tables.
template <int R>
__global__ __launch_bounds__(256) void k_gate_pass(GateArgs a, int j, uint64_t q)
{
    constexpr int NL = 1 << R;
    __shared__ uint64_t red[m61::block_sum_words(3 * R, kThreads)];
    uint64_t rho[R], rr[R], acc[3 * R] = {};
#pragma unroll
    for (int c = 0; c < R; c++) {
        rho[c] = a.rho[j + c];
        rr[c] = a.r[j + c];
    }
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < q; i += (uint64_t)gridDim.x * kThreads) {
        uint64_t u[NL], v[NL], w[NL];
#pragma unroll
        for (int t = 0; t < NL; t++) {
            u[t] = a.T0[i + t * q];
            v[t] = a.T1[i + t * q];
        }
        x_weights<R>(suffix_weight(a.HS, a.LS, a.lN - j - R, a.L, i), rr, w);
        gate_rounds<R>(u, v, w, rho, acc);
        a.T0[i] = m61::canon(u[0]);
        a.T1[i] = m61::canon(v[0]);
    }
    const uint64_t *t = m61::block_sum_lds<3 * R>(acc, red);
    if (threadIdx.x < 3 * R) a.part[(size_t)(3 * j + threadIdx.x) * kEntryMaxBlocks + blockIdx.x] = t[threadIdx.x];
}

// The first R rounds, from the factors, and the product C of the same entries:
// a thread's 2^R entries of C go out, with the witness where it is announced
// (WIT; else the workgroup's extremes, as entries.hpp), while it works on its
// field products, so that the stores (30 bytes an entry) and the products
// overlap.  (Workgroups of their own for C beside those of the rounds did not:
// 512 x 16384 entries took 92 us, 56 and 44 apart; so, 78.)
// The claims' weights are eq(r, i + t q) = eq(r_0 .. r_{R-1}, t) eq(r_R .., i):
// the 2^R first factors are the same for all threads, so sum_t of them times the
// integers is exact in int64 by limbs (31 bits against Rm's 16, 21 against
// Y's 31), and the second factor, the rounds' own, multiplies once.
template <int R, bool WIT>
__global__ __launch_bounds__(256, 3) void k_gate_first(GateArgs a, uint64_t q, EntriesArgs e)
{
    constexpr int NL = 1 << R;
    __shared__ uint64_t red[m61::block_sum_words(3 * R, kThreads)];
    uint64_t rho[R], rr[R], acc[3 * R] = {}, claims[2] = {};
    int64_t lo = INT64_MAX, hi = INT64_MIN;
    int oor = 0;
#pragma unroll
    for (int c = 0; c < R; c++) {
        rho[c] = a.rho[c];
        rr[c] = a.r[c];
    }
    int32_t km[NL][2], ky[NL][3];
    if constexpr (WIT)
#pragma unroll
        for (int t = 0; t < NL; t++) {
            uint64_t k = 1;
#pragma unroll
            for (int c = 0; c < R; c++) k = m61::lmul(k, (t >> (R - 1 - c)) & 1 ? rr[c] : m61::lsub(1, rr[c]));
            k = m61::canon(k);
            km[t][0] = __builtin_amdgcn_readfirstlane((int32_t)(k & 0x7FFFFFFF));
            km[t][1] = __builtin_amdgcn_readfirstlane((int32_t)(k >> 31));
#pragma unroll
            for (int l = 0; l < 3; l++) ky[t][l] = __builtin_amdgcn_readfirstlane((int32_t)((k >> (21 * l)) & 0x1FFFFF));
        }
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < q; i += (uint64_t)gridDim.x * kThreads) {
        int32_t ai[NL], bi[NL];
        gate_fetch<NL>(a.A, i, q, NL, a.lk, ai);
        gate_fetch<NL>(a.B, i, q, NL, a.lk, bi);
        const uint64_t ei = suffix_weight(a.HS, a.LS, a.lN - R, a.L, i);
        uint64_t sm[2] = {}, sy[3] = {};
#pragma unroll
        for (int t = 0; t < NL; t++) {
            const int64_t c = (int64_t)ai[t] * bi[t];
            const uint64_t x = i + t * q;
            e.C[x] = c;
            if constexpr (WIT) {
                const WitOut o = witness_entry32(c, e.we.s, e.we.t, e.we.relu, e.we.half, oor);
                e.we.R[x] = o.r;
                e.we.Rm[x] = (uint16_t)o.rm;
                e.we.Y[x] = o.y;
                e.we.Z[x] = o.z;
                e.we.bits[x] = o.w;
#pragma unroll
                for (int l = 0; l < 2; l++) sm[l] += (uint64_t)((int64_t)km[t][l] * o.rm);
#pragma unroll
                for (int l = 0; l < 3; l++) sy[l] += (uint64_t)((int64_t)ky[t][l] * o.y);
            } else {
                lo = c < lo ? c : lo;
                hi = c > hi ? c : hi;
            }
        }
        if constexpr (WIT) {
            claims[0] = m61::lmacc(claims[0], m61::fold(m61::from_i64((int64_t)sm[0]) +
                                                        m61::rotl(m61::from_i64((int64_t)sm[1]), 31)), ei);
            claims[1] = m61::lmacc(claims[1], m61::fold(m61::from_i64((int64_t)sy[0]) +
                                                        m61::rotl(m61::from_i64((int64_t)sy[1]), 21) +
                                                        m61::rotl(m61::from_i64((int64_t)sy[2]), 42)), ei);
        }
        uint64_t u[NL], v[NL], w[NL];
#pragma unroll
        for (int t = 0; t < NL; t++) {
            u[t] = int_to_loose(ai[t]);
            v[t] = int_to_loose(bi[t]);
        }
        x_weights<R>(ei, rr, w);
        gate_rounds<R>(u, v, w, rho, acc);
        a.T0[i] = m61::canon(u[0]);
        a.T1[i] = m61::canon(v[0]);
    }
    const uint64_t *t = m61::block_sum_lds<3 * R>(acc, red);
    if (threadIdx.x < 3 * R) a.part[(size_t)threadIdx.x * kEntryMaxBlocks + blockIdx.x] = t[threadIdx.x];
    __syncthreads();
    if constexpr (WIT) entries_claims<kThreads>(claims, oor, e.we, blockIdx.x, red);
    else entries_extremes<kThreads>(lo, hi, e.mm, blockIdx.x, red);
}

// Round j's value at X from its sums g = (Z_0, Z_1, U), lin = K_j eq1(r_j, X).
__device__ __forceinline__ uint64_t gate_round_eval(const uint64_t *g, uint64_t lin, int X)
{
    const uint64_t f2 = m61::lsub(m61::fold(m61::fold(3 * g[0] + 4 * g[1]) + 2 * g[1]), 2 * g[2]);
    const uint64_t f = X < 2 ? g[X] : X == 2 ? f2 : m61::lmacc(g[0], 3, m61::lsub(f2, g[1]));
    return m61::canon(m61::lmul(lin, f));
}

// One workgroup per round and one for the end, blockIdx.x = lN.  A round below
// j0 sums its pass's partials; a later one folds the tables the passes left (the
// factors themselves when j0 = 0) up to its round, the first rounds in
// registers while more than 2^kEntryTailLog entries are left, then in LDS, and takes
// its sums.  What it needs besides, the weights eq(r_>j, .) as the products of
// two small tables and K_j, it makes itself.  Without passes (ALONE) the further
// workgroups compute the product, with eq values from the point, and the
// tables E1, E2 (nx workgroups): the call is one launch.
template <bool ALONE, int V, bool WIT>
__global__ __launch_bounds__(kEntryTailThreads) void k_gate_tails(GateArgs a, int j0, EntriesArgs e)
{
    constexpr int NT = kEntryTailThreads, S = 1 << kEntryTailLog, EM = 1 << (kEntryTailMax - kEntryTailLog), FH = 64;
    constexpr int IT = S / NT;
    __shared__ uint64_t t0[S], t1[S];
    __shared__ uint64_t red[m61::block_sum_words(3, NT)];
    __shared__ uint64_t rl[32], rhol[32], H[FH], Lw[FH], Kj;
    const int j = blockIdx.x, tid = threadIdx.x, ln = a.lN - a.lk;
    if (j > a.lN) {  // workgroup-uniform
        const int b = j - a.lN - 1;
        const GateProduct<V> load{a.A, a.B};
        if constexpr (ALONE) {
            if (tid < a.lN) rl[tid] = a.r[tid];
            __syncthreads();
            if (b >= e.total) {
                const uint64_t n = 1ull << ln, k = 1ull << a.lk, step = (uint64_t)(gridDim.x - a.lN - 1 - e.total) * NT;
                for (uint64_t i = (uint64_t)(b - e.total) * NT + tid; i < n + k; i += step) {
                    if (i < n) a.E1[i] = eq_suffix(rl, 0, ln, i);
                    else a.E2[i - n] = eq_suffix(rl, ln, a.lk, i - n);
                }
                return;
            }
            entries_block<V, WIT, NT, 1>(load, [&](uint64_t row) { return eq_suffix(rl, 0, ln, row); },
                                      [&](uint64_t col) { return eq_suffix(rl, ln, a.lk, col); }, 1ull << ln, a.lk,
                                      e.C, e.we, e.mm, b, e.total, red);
        }
        return;
    }
    uint64_t g[3] = {0, 0, 0};
    const int m = a.lN - j0, base = m < kEntryTailLog ? m : kEntryTailLog, C = m - base;  // C <= 2 rounds in registers
    const int nvar = a.lN - j - 1, lo = nvar / 2, hi = nvar - lo;  // of the weights (j >= j0: at most 12)
    // the tables' entries (or a pass's partials) are asked for first, and land
    // while the point, the weights and K_j are made
    uint64_t u[IT][EM], v[IT][EM];
    int32_t ai[IT][EM] = {}, bi[IT][EM] = {};
    if (j >= j0)
#pragma unroll
        for (int it = 0; it < IT; it++) {
            const int i = it * NT + tid < 1 << base ? it * NT + tid : 0;  // past the end: entry 0's, unused
            if (j0 == 0) {
                gate_fetch<EM>(a.A, i, 1ull << base, 1 << C, a.lk, ai[it]);
                gate_fetch<EM>(a.B, i, 1ull << base, 1 << C, a.lk, bi[it]);
            } else {
#pragma unroll
                for (int t = 0; t < EM; t++)
                    if (t < 1 << C) {
                        u[it][t] = a.T0[i + (t << base)];
                        v[it][t] = a.T1[i + (t << base)];
                    }
            }
        }
    if (tid < a.lN) {
        rl[tid] = a.r[tid];
        rhol[tid] = a.rho[tid];
    }
    __syncthreads();
    if (tid < 64) {  // K_j: a prefix product over the first wave (lN < 64)
        uint64_t k = 1;
        if (tid < j && j < a.lN) k = m61::mul(eq1_at(rl[tid], 0), m61::sub(1, rhol[tid]));
        if (tid < j && j < a.lN) k = m61::add(m61::canon(k), m61::mul(rl[tid], rhol[tid]));
        k = m61::wave_prefix_mul(k);
        if (tid == 63) Kj = k;
    }
    if (j >= j0 && j < a.lN) {
        if (tid >= 64 && tid - 64 < 1 << hi) H[tid - 64] = eq_suffix(rl, j + 1, hi, tid - 64);
        if (tid >= 128 && tid - 128 < 1 << lo) Lw[tid - 128] = eq_suffix(rl, j + 1 + hi, lo, tid - 128);
    }
    __syncthreads();
    if (j < j0) {
        const int s = j - j % kEntryPass, r = j0 - s < kEntryPass ? j0 - s : kEntryPass;
        const int nb = entry_blocks(1ull << (a.lN - s - r));
        const uint64_t *p = a.part + 3 * (size_t)j * kEntryMaxBlocks;
        for (int b = tid; b < nb; b += NT)
            for (int q = 0; q < 3; q++) g[q] = m61::fold(g[q] + p[(size_t)q * kEntryMaxBlocks + b]);
    } else {
        const int jj = j - j0, n0 = 1 << base;
        auto weight = [&](int i) { return m61::lmul(H[i >> lo], Lw[i & ((1 << lo) - 1)]); };
#pragma unroll
        for (int it = 0; it < IT; it++) {
            const int i = it * NT + tid;
            if (i >= n0) continue;
            if (j0 == 0)
#pragma unroll
                for (int t = 0; t < EM; t++) {
                    u[it][t] = small_to_field(ai[it][t]);
                    v[it][t] = small_to_field(bi[it][t]);
                }
#pragma unroll
            for (int c = 0; c < kEntryTailMax - kEntryTailLog; c++) {
                const int h = (1 << C) >> (c + 1);
                if (c > jj || h == 0) continue;
#pragma unroll
                for (int p = 0; p < EM / 2; p++) {
                    if (p >= h) continue;
                    const uint64_t u1 = h == 2 ? u[it][p + 2] : u[it][1], v1 = h == 2 ? v[it][p + 2] : v[it][1];
                    if (c == jj) {
                        relu_pair(weight(p * n0 + i), u[it][p], u1, v[it][p], v1, g);
                    } else {
                        u[it][p] = fold(u[it][p], u1, rhol[j0 + c]);
                        v[it][p] = fold(v[it][p], v1, rhol[j0 + c]);
                    }
                }
            }
            t0[i] = u[it][0];
            t1[i] = v[it][0];
        }
        __syncthreads();
        if (jj >= C) {
            int n = n0;
            for (int b = j0 + C; b < j; b++) {  // an entry's two sources are read by its own thread only
                const uint64_t z = rhol[b];
                n >>= 1;
                for (int i = tid; i < n; i += NT) {
                    t0[i] = fold(t0[i], t0[i + n], z);
                    t1[i] = fold(t1[i], t1[i + n], z);
                }
                __syncthreads();
            }
            if (j == a.lN) {
                if (tid != 0) return;
                const uint64_t u = m61::canon(t0[0]), v = m61::canon(t1[0]);
                if (a.lN == 0) a.tr[0] = *e.c0 = m61::mul(u, v);
                a.tr[1 + 4 * (size_t)a.lN] = u;
                a.tr[2 + 4 * (size_t)a.lN] = v;
                return;
            }
            const int h = n >> 1;
            for (int i = tid; i < h; i += NT) {
                relu_pair(weight(i), t0[i], t0[i + h], t1[i], t1[i + h], g);
            }
        }
    }
    const uint64_t lin = m61::lmul(Kj, eq1_at(rl[j], tid & 3));
    const uint64_t *t = m61::block_sum_lds<3>(g, red);
    if (tid >= 4) return;
    const uint64_t val = gate_round_eval(t, lin, tid), next = __shfl_down(val, 1, 64);
    a.tr[1 + 4 * (size_t)j + tid] = val;
    if (j == 0 && tid == 0) a.tr[0] = *e.c0 = m61::add(val, next);  // the claimed sum g_1(0) + g_1(1)
}

int gate_entries(const GateArgs &a, const EntriesArgs &e)
{
    if (entry_passes(a.lN)) return entry_blocks(1ull << (a.lN - std::min(entry_pass_rounds(a.lN), kEntryPass)));
    return entries_blocks(1ull << a.lN, entries_width(1ull << a.lk, e.C, e.wit ? &e.we : nullptr), kEntryTailThreads);
}

void launch_gate(const GateArgs &a, const EntriesArgs &e, hipStream_t st)
{
    const int np = entry_passes(a.lN), j0 = entry_pass_rounds(a.lN);
    const uint64_t tables = (1ull << (a.lN - a.lk)) + (1ull << a.lk);  // entries of E1 and E2
    const dim3 tail(kEntryTailThreads);
    if (np == 0) {
        const unsigned nx = (unsigned)((tables + kEntryTailThreads - 1) / kEntryTailThreads);
        entries_variant(1ull << a.lk, e, [&](auto V, auto W) {
            hipLaunchKernelGGL((k_gate_tails<true, decltype(V)::value, decltype(W)::value>),
                               dim3(a.lN + 1 + e.total + nx), tail, 0, st, a, 0, e);
        });
        return;
    }
    const XSetupArgs xs{a.r, nullptr, nullptr, a.lN, a.L, a.nhs, a.HS, a.LS, nullptr, nullptr, nullptr, 0, 0};
    const int nx = (x_setup_count(xs) + kThreads - 1) / kThreads;
    const unsigned ne = (unsigned)((tables + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(k_gate_setup, dim3(nx + ne), dim3(kThreads), 0, st, xs, nx * kThreads, a.lN - a.lk, a.E1, a.E2);
    for (int p = 0, j = 0; p < np; p++) {
        const int r = j0 - j < kEntryPass ? j0 - j : kEntryPass;
        const uint64_t q = 1ull << (a.lN - j - r);
        const int nb = entry_blocks(q);
        const dim3 blk(kThreads);
        if (p == 0) {
#define RA_GATE_FIRST(R)                                                                                    \
    do {                                                                                                    \
        if (e.wit) hipLaunchKernelGGL((k_gate_first<R, true>), dim3(nb), blk, 0, st, a, q, e);              \
        else hipLaunchKernelGGL((k_gate_first<R, false>), dim3(nb), blk, 0, st, a, q, e);                   \
    } while (0)
            if (r == 3) RA_GATE_FIRST(3);
            else if (r == 2) RA_GATE_FIRST(2);
            else RA_GATE_FIRST(1);
#undef RA_GATE_FIRST
        } else if (r == 3) hipLaunchKernelGGL(k_gate_pass<3>, dim3(nb), blk, 0, st, a, j, q);
        else if (r == 2) hipLaunchKernelGGL(k_gate_pass<2>, dim3(nb), blk, 0, st, a, j, q);
        else hipLaunchKernelGGL(k_gate_pass<1>, dim3(nb), blk, 0, st, a, j, q);
        j += r;
    }
    hipLaunchKernelGGL((k_gate_tails<false, 1, false>), dim3(a.lN + 1), tail, 0, st, a, j0, e);
}

}  // namespace ra
