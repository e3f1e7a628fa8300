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

typedef int v4i __attribute__((ext_vector_type(4)));

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

__global__ __launch_bounds__(256) void k_embed_limbs(const uint64_t *__restrict__ E2, uint32_t d, uint32_t count,
                                                     v4i *__restrict__ limbs)
{
    const uint32_t t = blockIdx.x * blockDim.x + threadIdx.x;  // (4 q + g) 8 + c
    if (t >= count) return;
    const uint32_t j0 = t & ~7u;
    const int c = t & 7;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < 8; u++) {
        const uint64_t e = j0 + u < d ? E2[j0 + u] : 0;
        w[u >> 1] |= (limb_byte(e, c) | limb_byte(m61::rotl(e, 8), c) << 8) << (16 * (u & 1));
    }
    limbs[t] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
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
    const uint32_t count = embed_limb_words(a.d) / 2;
    hipLaunchKernelGGL(k_embed_limbs, dim3((count + 255) / 256), dim3(256), 0, st, a.E2, a.d, count, (v4i *)a.limbs);
    // 64 rows a workgroup use each fragment of the columns four times; 16 rows
    // where 64 would leave CUs without a workgroup
    if (a.rows >= 64 * 256)
        hipLaunchKernelGGL((k_embed_bind<4, 4>), dim3((unsigned)(a.rows / 64)), dim3(256), 0, st, a.E, a.ld, a.vocab,
                           a.d, a.rows, (const v4i *)a.limbs, a.r2, a.lk, a.b);
    else
        hipLaunchKernelGGL((k_embed_bind<1, 8>), dim3((unsigned)((a.rows + 15) / 16)), dim3(256), 0, st, a.E, a.ld,
                           a.vocab, a.d, a.rows, (const v4i *)a.limbs, a.r2, a.lk, a.b);
}

void launch_embed_product(const EmbedArgs &a, int64_t *C, hipStream_t st)
{
    const uint64_t N = (uint64_t)a.n << a.lk;
    hipLaunchKernelGGL(k_embed_product, dim3((unsigned)std::min<uint64_t>((N + 255) / 256, 4096)), dim3(256), 0, st,
                       a.tok, a.E, a.ld, a.vocab, a.d, a.scale, N, a.lk, C, a.bad, a.status);
}

}  // namespace ra
