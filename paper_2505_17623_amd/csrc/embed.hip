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
#include "entries.hpp"
#include "m61.hpp"
#include "tail.hpp"
#include "xsetup.hpp"

namespace ra {

typedef int v4i __attribute__((ext_vector_type(4)));

// e(v) = sum_j E[v, j] e_j (e_j = eq(r2, j), zero past d) on the matrix cores.
// A row of the table is taken as 2 d bytes, as it lies in memory: with E = 256
// hi + lo, lo read as lo - 128 (a xor of its top bit),
//   e(v) = sum_j (lo - 128) e_j + hi (256 e_j) + 128 sum_{j < d} e_j,
// and e_j and 256 e_j mod p are cut into eight signed bytes (x + C) ^ C with C =
// 0x80..80, so the sum is an int8 product of the rows with eight columns
// (v_mfma_i32_16x16x64_i8; columns 8 to 15 zero) that needs nothing of an
// entry but that xor: the pass runs at the rate the table is read.  A sum of
// byte products over a wave's quarter of a row stays below 2^31 for d <= 2^17.
// The columns as fragments: chunk q of 32 entries, lane group g, limb c: 16
// bytes at ((4 q + g) 8 + c) 16, entries 32 q + 8 g .. + 8, each e_j's limb c
// and then 256 e_j's.
__device__ __forceinline__ uint32_t limb_byte(uint64_t e, int c)
{
    constexpr uint64_t C = 0x8080808080808080ull;
    return (uint32_t)(((e + C) ^ C) >> (8 * c)) & 0xFFu;
}

__device__ __forceinline__ void embed_limbs(const uint64_t *r2, int lk, uint32_t d, uint32_t t, v4i *__restrict__ limbs)
{
    const uint32_t j0 = t & ~7u;  // t = (4 q + g) 8 + c
    const int c = t & 7, low = lk < 3 ? lk : 3;
    // eq(r2, j0 + u): the coordinates above the last three once, then those
    uint64_t e[8];
    e[0] = j0 < d ? eq_suffix(r2, 0, lk - low, j0 >> low) : 0;
    for (int i = 0; i < low; i++) {
        const uint64_t z = r2[lk - low + i];
#pragma unroll
        for (int u = 3; u >= 0; u--)
            if (u < 1 << i) {
                e[2 * u + 1] = m61::lmul(e[u], z);
                e[2 * u] = m61::lsub(e[u], e[2 * u + 1]);
            }
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < 8; u++) {
        const uint64_t x = u < 1 << low && j0 + u < d ? m61::canon(e[u]) : 0;
        w[u >> 1] |= (limb_byte(x, c) | limb_byte(m61::rotl(x, 8), c) << 8) << (16 * (u & 1));
    }
    limbs[t] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

// All that depends on the challenges alone, and W's sums: nl threads write the
// columns' fragments, the next n and 2^lk the eq tables E1 and E2, the last n
// (one a token) add eq(r1, i) scale to W(tok[i]).  W(v) mod p is acc[v] + 2^32
// acc[rows + v] (tail.hpp), each word a sum of values below 2^32, so no add
// wraps and their order does not matter.  A token outside [-1, vocab) is not
// followed; it sets *status.
__global__ __launch_bounds__(256) void k_embed_front(EmbedArgs a, uint32_t nl, uint64_t scale)
{
    __shared__ uint64_t rl[64];
    const int ln = a.ln, lk = a.lk, tid = threadIdx.x;
    if (tid < ln + lk) rl[tid] = a.r[tid];
    __syncthreads();
    uint64_t i = (uint64_t)blockIdx.x * blockDim.x + tid;
    if (i < nl) {
        embed_limbs(rl + ln, lk, a.d, (uint32_t)i, (v4i *)a.limbs);
        return;
    }
    i -= nl;
    if (i < a.n) {
        a.E1[i] = eq_suffix(rl, 0, ln, i);
        return;
    }
    i -= a.n;
    if (i < 1ull << lk) {
        a.E2[i] = eq_suffix(rl, ln, lk, i);
        return;
    }
    i -= 1ull << lk;
    if (i >= a.n) return;
    const int32_t v = a.tok[i];
    if (v < 0 || (uint32_t)v >= a.vocab) {
        if (v != -1) *a.status = 1;
        return;
    }
    const uint64_t e = m61::mul(eq_suffix(rl, 0, ln, i), scale);
    atomicAdd((unsigned long long *)a.acc + v, (unsigned long long)(e & 0xFFFFFFFFull));
    atomicAdd((unsigned long long *)a.acc + a.rows + v, (unsigned long long)(e >> 32));
}

// sum_{j < d} eq(r2, j) from the coordinates of r2 (lk of them): for every set
// bit of d, the prefix of d above it fixed, that bit zero, the rest free.
__device__ __forceinline__ uint64_t eq_prefix_sum(const uint64_t *r2, int lk, uint32_t d)
{
    if (d >> lk) return 1;
    uint64_t pre = 1, sum = 0;
    for (int i = 0; i < lk; i++) {
        const uint64_t z = r2[i], one = m61::lsub(1, z);
        const int bit = (d >> (lk - 1 - i)) & 1;
        if (bit) sum = m61::lmacc(sum, pre, one);
        pre = m61::lmul(pre, bit ? z : one);
    }
    return m61::canon(sum);
}

// A workgroup takes 16 RT rows, each of its four waves every fourth chunk of
// them; U chunks' loads are issued before the first is used.  Rows may start
// at any even address; the last chunk of a width that is no multiple of 32 is
// read entry by entry.
template <int RT, int U>
__global__ __launch_bounds__(256) void k_embed_bind(const int16_t *__restrict__ E, uint64_t ld, uint32_t vocab, uint32_t d,
                                                    uint64_t rows, const v4i *__restrict__ limbs,
                                                    const uint64_t *__restrict__ r2, int lk, uint64_t *__restrict__ b)
{
    __shared__ int32_t part[4][16 * RT][9];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, g = lane >> 4, c = lane & 15;
    const uint64_t v0 = (uint64_t)blockIdx.x * (16 * RT);
    const uint32_t nq = d / 32;  // whole chunks
    const v4i flip{0x00800080, 0x00800080, 0x00800080, 0x00800080}, none{0, 0, 0, 0};
    const int16_t *row[RT];
    v4i acc[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const uint64_t v = v0 + 16 * t + c;
        row[t] = E + (v < vocab ? v : vocab - 1) * ld + 8 * g;
        acc[t] = none;
    }
    const v4i *col = limbs + 8 * g + (c & 7);
    for (uint32_t q0 = wv; q0 < nq; q0 += 4 * U) {
        v4i a[U][RT], w[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const uint32_t q = q0 + 4 * u < nq ? q0 + 4 * u : q0;  // wave-uniform
#pragma unroll
            for (int t = 0; t < RT; t++) __builtin_memcpy(&a[u][t], row[t] + 32 * q, 16);
            w[u] = col[32 * q];
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const v4i y = c < 8 && q0 + 4 * u < nq ? w[u] : none;
#pragma unroll
            for (int t = 0; t < RT; t++)
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][t] ^ flip, y, acc[t], 0, 0, 0);
        }
    }
    if ((d & 31) && wv == (int)(nq & 3)) {  // wave-uniform
        const v4i y = c < 8 ? col[32 * nq] : none;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            v4i x = none;
#pragma unroll
            for (int u = 0; u < 8; u++)
                if (32 * nq + 8 * g + u < d) x[u >> 1] |= (int)((uint32_t)(uint16_t)row[t][32 * nq + u] << (16 * (u & 1)));
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x ^ flip, y, acc[t], 0, 0, 0);
        }
    }
    // lane l, register r: row 4 (l / 16) + r, limb l % 16
#pragma unroll
    for (int t = 0; t < RT; t++)
#pragma unroll
        for (int r = 0; r < 4; r++)
            if (c < 8) part[wv][16 * t + 4 * g + r][c] = acc[t][r];
    __syncthreads();
    if (tid >= 16 * RT || v0 + tid >= rows) return;
    uint64_t s = 0;
    if (v0 + tid < vocab) {
        s = m61::rotl(eq_prefix_sum(r2, lk, d), 7);
#pragma unroll
        for (int l = 0; l < 8; l++) {
            const int64_t x = (int64_t)part[0][tid][l] + part[1][tid][l] + part[2][tid][l] + part[3][tid][l];
            s = m61::fold(s + m61::rotl(m61::from_i64(x), 8 * l));
        }
    }
    b[v0 + tid] = m61::canon(s);
}

// V entries of C: scale times the token's row, zero past d, for token -1 and
// for one outside the vocabulary.
template <int V> struct EmbedRows {
    const int32_t *tok;
    const int16_t *E;
    uint64_t ld;
    uint32_t vocab, d;
    int32_t scale;
    __device__ __forceinline__ void operator()(uint64_t row, uint64_t col, int64_t (&c)[V]) const
    {
        const int32_t v = tok[row];
        int16_t h[V] = {};
        if (v >= 0 && (uint32_t)v < vocab && col < d) {
            const int16_t *p = E + (uint64_t)v * ld + col;
            if (col + V <= d) {
                __builtin_memcpy(h, p, sizeof h);
            } else {
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (col + i < d) h[i] = p[i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) c[i] = (int64_t)scale * h[i];
    }
};

// The product (with the witness), and the sum-check's last rounds as its first
// workgroups.
template <int V, bool WIT>
__global__ __launch_bounds__(256) void k_embed_product(EmbedArgs a, int64_t *C, WitEpi we, TailArgs ta, XJobs jobs,
                                                       int ntail)
{
    __shared__ uint64_t smem[kTailSmem];
    static_assert(kTailSmem >= entries_lds_words(kThreads), "the tail's LDS serves the product");
    if ((int)blockIdx.x < ntail) {  // workgroup-uniform
        tail_block<KIND_MATMUL>(ta, jobs, blockIdx.x, smem);
        return;
    }
    entries_block<V, WIT, kThreads>(EmbedRows<V>{a.tok, a.E, a.ld, a.vocab, a.d, a.scale}, a.n, a.lk, C, we,
                                    (int)blockIdx.x - ntail, (int)gridDim.x - ntail, smem);
}

void launch_embed_front(const EmbedArgs &a, hipStream_t st)
{
    const uint64_t scale = a.scale < 0 ? m61::P - (uint64_t)(-(int64_t)a.scale) : (uint64_t)a.scale;
    const uint32_t nl = embed_limb_words(a.d) / 2;
    const uint64_t threads = nl + 2 * (uint64_t)a.n + (1ull << a.lk);
    hipLaunchKernelGGL(k_embed_front, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, nl, scale);
}

void launch_embed_bind(const EmbedArgs &a, hipStream_t st)
{
    const uint64_t *r2 = a.r + a.ln;
    // 64 rows a workgroup use each fragment of the columns four times; 16 rows
    // where 64 would leave CUs without a workgroup
    if (a.rows >= 64 * 256)
        hipLaunchKernelGGL((k_embed_bind<4, 4>), dim3((unsigned)(a.rows / 64)), dim3(256), 0, st, a.E, a.ld, a.vocab,
                           a.d, a.rows, (const v4i *)a.limbs, r2, a.lk, a.b);
    else
        hipLaunchKernelGGL((k_embed_bind<1, 8>), dim3((unsigned)((a.rows + 15) / 16)), dim3(256), 0, st, a.E, a.ld,
                           a.vocab, a.d, a.rows, (const v4i *)a.limbs, r2, a.lk, a.b);
}

int embed_entries(uint64_t N, uint64_t k, const int64_t *C, const WitEpi *we)
{
    return entries_blocks(N, entries_width(k, C, we), kThreads);
}

void launch_embed_product(const EmbedArgs &a, int64_t *C, const WitEpi *we, const TailArgs &ta, const XJobs &jobs,
                          hipStream_t st)
{
    const uint64_t k = 1ull << a.lk;
    const int V = entries_width(k, C, we), ntail = 1 + jobs.nslot;
    const dim3 grid(ntail + embed_entries(a.n * k, k, C, we)), blk(kThreads);
    const WitEpi w = we ? *we : WitEpi{};
    if (V == 2 && we) hipLaunchKernelGGL((k_embed_product<2, true>), grid, blk, 0, st, a, C, w, ta, jobs, ntail);
    else if (V == 2) hipLaunchKernelGGL((k_embed_product<2, false>), grid, blk, 0, st, a, C, w, ta, jobs, ntail);
    else if (we) hipLaunchKernelGGL((k_embed_product<1, true>), grid, blk, 0, st, a, C, w, ta, jobs, ntail);
    else hipLaunchKernelGGL((k_embed_product<1, false>), grid, blk, 0, st, a, C, w, ta, jobs, ntail);
}

}  // namespace ra
