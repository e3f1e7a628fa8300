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

// Entry (row, col) of a factor: int16 or int32, rows `ld` entries apart (0:
// one row for all).
__device__ __forceinline__ int32_t gate_load(const GateSrc &s, uint64_t x, int lk)
{
    const uint64_t at = (x >> lk) * s.ld + (x & ((1ull << lk) - 1));
    return s.i16 ? (int32_t)((const int16_t *)s.p)[at] : ((const int32_t *)s.p)[at];
}

// V entries of C = A B, exact in int64 (|C| <= 2^62).
template <int V> struct GateProduct {
    GateSrc A, B;
    __device__ __forceinline__ void factor(const GateSrc &s, uint64_t at, int32_t (&v)[V]) const
    {
        if (s.i16) {  // uniform; the loads need no more alignment than the entries have
            int16_t h[V];
            __builtin_memcpy(h, (const int16_t *)s.p + at, sizeof h);
#pragma unroll
            for (int i = 0; i < V; i++) v[i] = h[i];
        } else {
            __builtin_memcpy(v, (const int32_t *)s.p + at, sizeof v);
        }
    }
    __device__ __forceinline__ void operator()(uint64_t row, uint64_t col, int64_t (&c)[V]) const
    {
        int32_t a[V], b[V];
        factor(A, row * A.ld + col, a);
        factor(B, row * B.ld + col, b);
#pragma unroll
        for (int i = 0; i < V; i++) c[i] = (int64_t)a[i] * b[i];
    }
};

// The suffix eq tables of r and the prefix products K_j (xsetup.hpp) by the
// first nx threads, the eq tables E1 (r1) and E2 (r2) by the others.
__global__ __launch_bounds__(256) void k_gate_setup(XSetupArgs a, int nx, int ln, uint64_t *E1, uint64_t *E2)
{
    __shared__ uint64_t rl[64], sl[64];
    if ((int)threadIdx.x < a.lN) {
        rl[threadIdx.x] = a.r[threadIdx.x];
        sl[threadIdx.x] = a.sigx[threadIdx.x];
    }
    __syncthreads();
    const uint64_t g = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (g < (uint64_t)nx) {  // nx a multiple of the workgroup
        x_setup_body(a, (int)g, rl, sl, sl);
        return;
    }
    const uint64_t i = g - nx, n = 1ull << ln;
    if (i < n) E1[i] = eq_suffix(rl, 0, ln, i);
    else if (i - n < 1ull << (a.lN - ln)) E2[i - n] = eq_suffix(rl, ln, a.lN - ln, i - n);
}

// R rounds j .. j + R - 1 over tables of 2^R q entries in one pass: a thread
// holds the 2^R entries i + t q that end in entry i of the folded tables.  The
// first pass reads the factors themselves.
template <int R, bool FIRST>
__device__ __forceinline__ void gate_pass_block(const GateArgs &a, int j, uint64_t q, int blk, int nblk, uint64_t *red)
{
    constexpr int NL = 1 << R;
    uint64_t rho[R], rr[R], acc[3 * R];
#pragma unroll
    for (int c = 0; c < R; c++) {
        rho[c] = a.rho[j + c];
        rr[c] = a.r[j + c];
    }
#pragma unroll
    for (int c = 0; c < 3 * R; c++) acc[c] = 0;
    const int nvar = a.lN - j - R;
    for (uint64_t i = (uint64_t)blk * kThreads + threadIdx.x; i < q; i += (uint64_t)nblk * kThreads) {
        uint64_t u[NL], v[NL], w[NL];
#pragma unroll
        for (int t = 0; t < NL; t++) {
            u[t] = FIRST ? small_to_field(gate_load(a.A, i + t * q, a.lk)) : a.T0[i + t * q];
            v[t] = FIRST ? small_to_field(gate_load(a.B, i + t * q, a.lk)) : a.T1[i + t * q];
        }
        x_weights<R>(suffix_weight(a.HS, a.LS, nvar, a.L, i), rr, w);
#pragma unroll
        for (int c = 0; c < R; c++) {
            const int h = NL >> (c + 1), base = h - 1;
#pragma unroll
            for (int p = 0; p < h; p++) {
                relu_pair(w[base + p], u[p], u[p + h], v[p], v[p + h], acc + 3 * c);
                u[p] = fold(u[p], u[p + h], rho[c]);
                v[p] = fold(v[p], v[p + h], rho[c]);
                if ((p & 3) == 3 || p == h - 1) fold_all<3>(acc + 3 * c);
            }
        }
        a.T0[i] = m61::canon(u[0]);
        a.T1[i] = m61::canon(v[0]);
    }
    const uint64_t *t = m61::block_sum_lds<3 * R>(acc, red);
    if (threadIdx.x < 3 * R)
        a.part[(size_t)(3 * j + threadIdx.x) * kGateMaxBlocks + blk] = t[threadIdx.x];
}

template <int R>
__global__ __launch_bounds__(256) void k_gate_pass(GateArgs a, int j, uint64_t q)
{
    __shared__ uint64_t red[m61::block_sum_words(3 * R, kThreads)];
    gate_pass_block<R, false>(a, j, q, blockIdx.x, gridDim.x, red);
}

// The first pass and the product (with the witness) side by side: the one
// works on its field products, the other waits on memory.
template <int R, int V, bool WIT>
__global__ __launch_bounds__(256) void k_gate_main(GateArgs a, uint64_t q, int npass, int64_t *C, WitEpi we, int nent)
{
    constexpr int W = m61::block_sum_words(3 * R, kThreads);
    __shared__ uint64_t red[W > entries_lds_words(kThreads) ? W : entries_lds_words(kThreads)];
    const int b = blockIdx.x, both = 2 * (npass < nent ? npass : nent);
    const bool pass = b < both ? (b & 1) == 0 : npass > nent;  // workgroup-uniform
    const int idx = b < both ? b >> 1 : b - both / 2;
    if (pass) gate_pass_block<R, true>(a, 0, q, idx, npass, red);
    else entries_block<V, WIT, kThreads>(GateProduct<V>{a.A, a.B}, 1ull << (a.lN - a.lk), a.lk, C, we, idx, nent, red);
}

// Round j's value at X from its sums g = (Z_0, Z_1, U).
__device__ __forceinline__ uint64_t gate_round_eval(const uint64_t *g, uint64_t K, uint64_t r, int X)
{
    const uint64_t f2 = m61::lsub(m61::fold(m61::fold(3 * g[0] + 4 * g[1]) + 2 * g[1]), 2 * g[2]);
    const uint64_t f = X < 2 ? g[X] : X == 2 ? f2 : m61::lmacc(g[0], 3, m61::lsub(f2, g[1]));
    return m61::canon(m61::lmul(m61::lmul(K, eq1_at(r, X)), f));
}

// One workgroup per round and one for the end, blockIdx.x = lN.  A round below
// j0 sums its pass's partials; a later one folds the tables the passes left (the
// factors themselves when j0 = 0; at most 2^kGateTailLog entries) in LDS up to
// its round and takes its sums.
// Without passes (j0 = 0) further workgroups compute the product (ENT).
template <bool ENT, int V, bool WIT>
__global__ __launch_bounds__(kGateTailThreads) void k_gate_tails(GateArgs a, int j0, int64_t *C, WitEpi we)
{
    __shared__ uint64_t t0[1 << kGateTailLog], t1[1 << kGateTailLog];
    __shared__ uint64_t red[m61::block_sum_words(3, kGateTailThreads)];
    const int j = blockIdx.x, tid = threadIdx.x;
    if (ENT && j > a.lN) {  // workgroup-uniform
        entries_block<V, WIT, kGateTailThreads>(GateProduct<V>{a.A, a.B}, 1ull << (a.lN - a.lk), a.lk, C, we,
                                                j - a.lN - 1, (int)gridDim.x - a.lN - 1, red);
        return;
    }
    uint64_t g[3] = {0, 0, 0};
    if (j < j0) {
        const int s = j - j % kGatePass, nb = gate_blocks(1ull << (a.lN - s - gate_pass_rounds(j0 - s)));
        const uint64_t *p = a.part + 3 * (size_t)j * kGateMaxBlocks;
        for (int b = tid; b < nb; b += blockDim.x)
            for (int q = 0; q < 3; q++) g[q] = m61::fold(g[q] + p[(size_t)q * kGateMaxBlocks + b]);
    } else {
        int n = 1 << (a.lN - j0);
        for (int i = tid; i < n; i += blockDim.x) {
            t0[i] = j0 == 0 ? small_to_field(gate_load(a.A, i, a.lk)) : a.T0[i];
            t1[i] = j0 == 0 ? small_to_field(gate_load(a.B, i, a.lk)) : a.T1[i];
        }
        __syncthreads();
        for (int b = j0; b < j; b++) {  // an entry's two sources are read by its own thread only
            const uint64_t z = a.rho[b];
            n >>= 1;
            for (int i = tid; i < n; i += blockDim.x) {
                t0[i] = fold(t0[i], t0[i + n], z);
                t1[i] = fold(t1[i], t1[i + n], z);
            }
            __syncthreads();
        }
        if (j == a.lN) {
            if (tid != 0) return;
            const uint64_t u = m61::canon(t0[0]), v = m61::canon(t1[0]);
            if (a.lN == 0) a.tr[0] = m61::mul(u, v);
            a.tr[1 + 4 * (size_t)a.lN] = u;
            a.tr[2 + 4 * (size_t)a.lN] = v;
            return;
        }
        const int h = n >> 1;
        for (int i = tid; i < h; i += blockDim.x) {
            relu_pair(a.LS[h + i], t0[i], t0[i + h], t1[i], t1[i + h], g);
            fold_all<3>(g);
        }
    }
    const uint64_t *t = m61::block_sum_lds<3>(g, red);
    if (tid >= 4) return;
    a.tr[1 + 4 * (size_t)j + tid] = gate_round_eval(t, a.K[j], a.r[j], tid);
    if (j == 0 && tid == 0)
        a.tr[0] = m61::add(gate_round_eval(t, a.K[0], a.r[0], 0), gate_round_eval(t, a.K[0], a.r[0], 1));
}

int gate_entries(uint64_t N, uint64_t k, const int64_t *C, const WitEpi *we)
{
    return entries_blocks(N, entries_width(k, C, we), N > 1ull << kGateTailLog ? kThreads : kGateTailThreads);
}

void launch_gate(const GateArgs &a, uint64_t *E1, uint64_t *E2, int64_t *C, const WitEpi *we, hipStream_t st)
{
    const uint64_t N = 1ull << a.lN, k = 1ull << a.lk;
    const XSetupArgs xs{a.r, a.rho, nullptr, a.lN, a.L, a.nhs, a.HS, a.LS, a.K, nullptr, nullptr, 0, 0};
    const int nx = (x_setup_count(xs) + kThreads - 1) / kThreads;
    const unsigned ne = (unsigned)((N / k + k + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(k_gate_setup, dim3(nx + ne), dim3(kThreads), 0, st, xs, nx * kThreads, a.lN - a.lk, E1, E2);
    const int V = entries_width(k, C, we), nent = gate_entries(N, k, C, we);
    const WitEpi w = we ? *we : WitEpi{};
    const int j0 = a.lN > kGateTailLog ? a.lN - kGateTailLog : 0;  // rounds over the global tables
    if (j0 == 0) {
        const dim3 grid(a.lN + 1 + nent), blk(kGateTailThreads);
        if (V == 2 && we) hipLaunchKernelGGL((k_gate_tails<true, 2, true>), grid, blk, 0, st, a, 0, C, w);
        else if (V == 2) hipLaunchKernelGGL((k_gate_tails<true, 2, false>), grid, blk, 0, st, a, 0, C, w);
        else if (we) hipLaunchKernelGGL((k_gate_tails<true, 1, true>), grid, blk, 0, st, a, 0, C, w);
        else hipLaunchKernelGGL((k_gate_tails<true, 1, false>), grid, blk, 0, st, a, 0, C, w);
        return;
    }
    for (int j = 0; j < j0; j += kGatePass) {
        const int r = gate_pass_rounds(j0 - j);
        const uint64_t q = 1ull << (a.lN - j - r);
        const int nb = gate_blocks(q);
        if (j > 0) {
            const dim3 grid(nb), blk(kThreads);
            if (r == 3) hipLaunchKernelGGL(k_gate_pass<3>, grid, blk, 0, st, a, j, q);
            else if (r == 2) hipLaunchKernelGGL(k_gate_pass<2>, grid, blk, 0, st, a, j, q);
            else hipLaunchKernelGGL(k_gate_pass<1>, grid, blk, 0, st, a, j, q);
            continue;
        }
        const dim3 grid(nb + nent), blk(kThreads);
#define RA_GATE_MAIN(R)                                                                                              \
    do {                                                                                                             \
        if (V == 2 && we) hipLaunchKernelGGL((k_gate_main<R, 2, true>), grid, blk, 0, st, a, q, nb, C, w, nent);      \
        else if (V == 2) hipLaunchKernelGGL((k_gate_main<R, 2, false>), grid, blk, 0, st, a, q, nb, C, w, nent);      \
        else if (we) hipLaunchKernelGGL((k_gate_main<R, 1, true>), grid, blk, 0, st, a, q, nb, C, w, nent);           \
        else hipLaunchKernelGGL((k_gate_main<R, 1, false>), grid, blk, 0, st, a, q, nb, C, w, nent);                  \
    } while (0)
        if (r == 3) RA_GATE_MAIN(3);
        else if (r == 2) RA_GATE_MAIN(2);
        else RA_GATE_MAIN(1);
#undef RA_GATE_MAIN
    }
    hipLaunchKernelGGL((k_gate_tails<false, 1, false>), dim3(a.lN + 1), dim3(kGateTailThreads), 0, st, a, j0, nullptr, w);
}

}  // namespace ra
