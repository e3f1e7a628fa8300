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

// C = A B, exact in int64 (|C| <= 2^62).
__global__ __launch_bounds__(256) void k_gate_product(GateSrc A, GateSrc B, uint64_t N, int lk, int64_t *__restrict__ C)
{
    for (uint64_t x = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; x < N; x += (uint64_t)gridDim.x * blockDim.x)
        C[x] = (int64_t)gate_load(A, x, lk) * gate_load(B, x, lk);
}

// The suffix eq tables of r and the prefix products K_j (xsetup.hpp).
__global__ __launch_bounds__(256) void k_gate_setup(XSetupArgs a)
{
    __shared__ uint64_t rl[64], sl[64];
    if ((int)threadIdx.x < a.lN) {
        rl[threadIdx.x] = a.r[threadIdx.x];
        sl[threadIdx.x] = a.sigx[threadIdx.x];
    }
    __syncthreads();
    x_setup_body(a, blockIdx.x * blockDim.x + threadIdx.x, rl, sl, sl);
}

// R rounds j .. j + R - 1 over tables of 2^R q entries in one pass: a thread
// holds the 2^R entries i + t q that end in entry i of the folded tables.  The
// first pass reads the factors themselves.
template <int R, bool FIRST>
__global__ __launch_bounds__(256) void k_gate_pass(GateArgs a, int j, uint64_t q)
{
    constexpr int NL = 1 << R;
    __shared__ uint64_t red[m61::block_sum_words(3 * R, kThreads)];
    uint64_t rho[R], rr[R], acc[3 * R];
#pragma unroll
    for (int c = 0; c < R; c++) {
        rho[c] = a.rho[j + c];
        rr[c] = a.r[j + c];
    }
#pragma unroll
    for (int c = 0; c < 3 * R; c++) acc[c] = 0;
    const int nvar = a.lN - j - R;
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < q; i += (uint64_t)gridDim.x * blockDim.x) {
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
        a.part[(size_t)(3 * j + threadIdx.x) * kGateMaxBlocks + blockIdx.x] = t[threadIdx.x];
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
__global__ __launch_bounds__(kGateTailThreads) void k_gate_tails(GateArgs a, int j0)
{
    __shared__ uint64_t t0[1 << kGateTailLog], t1[1 << kGateTailLog];
    __shared__ uint64_t red[m61::block_sum_words(3, kGateTailThreads)];
    const int j = blockIdx.x, tid = threadIdx.x;
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

template <int R> static void gate_pass(const GateArgs &a, int j, hipStream_t st)
{
    const uint64_t q = 1ull << (a.lN - j - R);
    const dim3 grid(gate_blocks(q)), blk(kThreads);
    if (j == 0) hipLaunchKernelGGL((k_gate_pass<R, true>), grid, blk, 0, st, a, j, q);
    else hipLaunchKernelGGL((k_gate_pass<R, false>), grid, blk, 0, st, a, j, q);
}

void launch_gate(const GateArgs &a, int64_t *C, hipStream_t st)
{
    const uint64_t N = 1ull << a.lN;
    const XSetupArgs xs{a.r, a.rho, nullptr, a.lN, a.L, a.nhs, a.HS, a.LS, a.K, nullptr, nullptr, 0, 0};
    hipLaunchKernelGGL(k_gate_setup, dim3((x_setup_count(xs) + kThreads - 1) / kThreads), dim3(kThreads), 0, st, xs);
    hipLaunchKernelGGL(k_gate_product, dim3((unsigned)std::min<uint64_t>((N + kThreads - 1) / kThreads, 4096)),
                       dim3(kThreads), 0, st, a.A, a.B, N, a.lk, C);
    const int j0 = a.lN > kGateTailLog ? a.lN - kGateTailLog : 0;  // rounds over the global tables
    for (int j = 0; j < j0; j += kGatePass) {
        const int r = gate_pass_rounds(j0 - j);
        if (r == 3) gate_pass<3>(a, j, st);
        else if (r == 2) gate_pass<2>(a, j, st);
        else gate_pass<1>(a, j, st);
    }
    hipLaunchKernelGGL(k_gate_tails, dim3(a.lN + 1), dim3(kGateTailThreads), 0, st, a, j0);
}

}  // namespace ra
