// embed.hip -- the token embedding with scaling as a layer's product: row i of
// C is scale times row tok[i] of the table E (zero for tok[i] = -1), i.e. C = S
// E with S the n x vocab matrix that holds scale at (i, tok[i]).  S is never
// formed: bound at r1 its columns are
//     W(v) = scale sum over the i with tok[i] = v of eq(r1, i),
// the lookup's transpose applied to eq(r1, .) (what a gradient of the table
// is to the rows' gradients), and
//     C~(r1, r2) = sum_v W(v) e(v),   e(v) = sum_j E[v, j] eq(r2, j),
// is the matrix layer's sum-check (Eq. (4)) over the vocabulary's variables. It
// ends in W~(rho), computable from the public tokens, and E~(rho, r2).
// Rows past the vocabulary and columns past the table's width are zero.
#include <algorithm>

#include "common.hpp"
#include "entries.hpp"
#include "m61.hpp"
#include "xpair.hpp"
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

// All that depends on the challenges alone: nl threads write the columns'
// fragments, the next n and 2^lk the eq tables E1 and E2; W's 2 rows words are
// cleared by all of them.
__global__ __launch_bounds__(256) void k_embed_front(EmbedArgs a, uint32_t nl)
{
    __shared__ uint64_t rl[64];
    const int ln = a.ln, lk = a.lk, tid = threadIdx.x;
    if (tid < ln + lk) rl[tid] = a.r[tid];
    const uint64_t g = (uint64_t)blockIdx.x * blockDim.x + tid;
    for (uint64_t i = g; i < 2 * a.rows; i += (uint64_t)gridDim.x * blockDim.x) a.W[i] = 0;
    __syncthreads();
    uint64_t i = g;
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
    if (i < 1ull << lk) a.E2[i] = eq_suffix(rl, ln, lk, i);
}

// W's sums, one thread a token: W(v) = acc[v] + 2^32 acc[rows + v] mod p, each
// word a sum of values below 2^32, so no add wraps (n <= 2^31) and their order
// does not matter.  A token outside [-1, vocab) is not followed; it sets
// *status.
__device__ __forceinline__ void embed_scatter(const EmbedArgs &a, uint64_t *status, uint64_t scale, uint64_t i)
{
    if (i >= a.n) return;
    const int32_t v = a.tok[i];
    if (v < 0 || (uint32_t)v >= a.vocab) {
        if (v != -1) *status = 1;
        return;
    }
    const uint64_t e = m61::mul(a.E1[i], scale);
    atomicAdd((unsigned long long *)a.W + v, (unsigned long long)(e & 0xFFFFFFFFull));
    atomicAdd((unsigned long long *)a.W + a.rows + v, (unsigned long long)(e >> 32));
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

// A workgroup takes 16 RT rows, each of its four waves a quarter of their
// chunks; U chunks' loads are issued before the first is used.  Rows may start
// at any even address; the last chunk of a width that is no multiple of 32 is
// read entry by entry.  What bounds it is the order in which memory is asked:
// with the waves' chunks interleaved and a chunk's rows one after the other the
// same loads took 204 us at 128000 x 4096 (1.05 GB), so 167 (6.3 TB/s, the same
// table again and again for one token; 185, 5.7 TB/s, where a call for 1024
// tokens has written its outputs between).
// The first ns workgroups scatter the tokens' weights.
template <int RT, int U>
__global__ __launch_bounds__(256) void k_embed_bind(EmbedArgs args, int ns, uint64_t scale)
{
    __shared__ int32_t part[4][16 * RT][9];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, g = lane >> 4, c = lane & 15;
    if ((int)blockIdx.x < ns) {  // workgroup-uniform
        embed_scatter(args, args.tr + 3 + 3 * (size_t)args.lv, scale, (uint64_t)blockIdx.x * 256 + tid);
        return;
    }
    const int16_t *__restrict__ E = args.E;
    const v4i *__restrict__ limbs = (const v4i *)args.limbs;
    const uint64_t ld = args.ld, rows = args.rows, *r2 = args.r + args.ln;
    const uint32_t vocab = args.vocab, d = args.d;
    const int lk = args.lk;
    const uint64_t v0 = (uint64_t)(blockIdx.x - ns) * (16 * RT);
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
    // a wave's chunks are a quarter of the row in one piece, and a row's are asked
    // for one after the other, so that memory sees 64 U bytes of a row at a time
    const uint32_t per = (nq + 3) / 4, qe = (wv + 1) * per < nq ? (wv + 1) * per : nq;
    for (uint32_t q0 = wv * per; q0 < qe; q0 += U) {
        v4i a[U][RT], w[U];
#pragma unroll
        for (int u = 0; u < U; u++) w[u] = col[32 * (q0 + u < qe ? q0 + u : q0)];
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int u = 0; u < U; u++)
                __builtin_memcpy(&a[u][t], row[t] + 32 * (q0 + u < qe ? q0 + u : q0), 16);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const v4i y = c < 8 && q0 + u < qe ? w[u] : none;
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
    args.b[v0 + tid] = m61::canon(s);
}

// V entries of C: scale times the token's row, zero past d, for token -1 and
// for one outside the vocabulary.
template <int V> struct EmbedRows {
    const int32_t *tok;
    const int16_t *E;
    uint64_t ld;
    uint32_t vocab, d;
    int32_t scale;
    struct Raw {
        int16_t h[V];
    };
    template <int U>
    __device__ __forceinline__ void fetch(uint64_t row, uint64_t step, uint64_t col, Raw (&raw)[U]) const
    {
        int32_t v[U];
#pragma unroll
        for (int u = 0; u < U; u++) v[u] = tok[row + u * step];
        const bool whole = V == 1 || !(d & 1);  // a pair of columns lies within the table's or past them
        const uint64_t c0 = col < d ? col : 0;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int16_t *p = E + (uint64_t)((uint32_t)v[u] < vocab ? v[u] : 0) * ld + c0;  // row 0 for those outside
            if (whole) {
                __builtin_memcpy(raw[u].h, p, sizeof raw[u].h);
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) raw[u].h[i] = p[c0 + i < d ? i : 0];
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < V; i++)
                if ((uint32_t)v[u] >= vocab || col + i >= d) raw[u].h[i] = 0;
    }
    __device__ __forceinline__ void value(const Raw &r, int64_t (&c)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; i++) c[i] = (int64_t)scale * r.h[i];
    }
};

// One pair of a round of sum_v W(v) e(v), added to folded sums: at X = 0 and
// 1, and the differences' products.
__device__ __forceinline__ void embed_pair(uint64_t u0, uint64_t u1, uint64_t v0, uint64_t v1, uint64_t *g)
{
    g[0] = m61::lmacc(g[0], u0, v0);
    g[1] = m61::lmacc(g[1], u1, v1);
    g[2] = m61::lmacc(g[2], m61::lsub(u1, u0), m61::lsub(v1, v0));
}

// W's value from its two sums.
__device__ __forceinline__ uint64_t embed_weight(uint64_t lo, uint64_t hi)
{
    return m61::fold(m61::canon(lo) + m61::rotl(m61::canon(hi), 32));
}

// R rounds j .. j + R - 1 over tables of 2^R q entries (the first pass: W and
// e themselves): a thread holds the 2^R entries that end in entry i of the
// folded tables.
template <int R, bool FIRST>
__device__ __forceinline__ void embed_pass_block(const EmbedArgs &a, int j, uint64_t q, int blk, int nblk, uint64_t *red)
{
    constexpr int NL = 1 << R;
    uint64_t rho[R], acc[3 * R];
#pragma unroll
    for (int c = 0; c < R; c++) rho[c] = a.rho[j + c];
#pragma unroll
    for (int c = 0; c < 3 * R; c++) acc[c] = 0;
    for (uint64_t i = (uint64_t)blk * kThreads + threadIdx.x; i < q; i += (uint64_t)nblk * kThreads) {
        uint64_t u[NL], v[NL], hi[NL];
#pragma unroll
        for (int t = 0; t < NL; t++) {  // loads first
            u[t] = FIRST ? a.W[i + t * q] : a.T0[i + t * q];
            hi[t] = FIRST ? a.W[a.rows + i + t * q] : 0;
            v[t] = FIRST ? a.b[i + t * q] : a.T1[i + t * q];
        }
        if (FIRST)
#pragma unroll
            for (int t = 0; t < NL; t++) u[t] = embed_weight(u[t], hi[t]);
#pragma unroll
        for (int c = 0; c < R; c++) {
            const int h = NL >> (c + 1);
#pragma unroll
            for (int p = 0; p < h; p++) {
                embed_pair(u[p], u[p + h], v[p], v[p + h], acc + 3 * c);
                u[p] = fold(u[p], u[p + h], rho[c]);
                v[p] = fold(v[p], v[p + h], rho[c]);
            }
        }
        a.T0[i] = m61::canon(u[0]);
        a.T1[i] = m61::canon(v[0]);
    }
    const uint64_t *t = m61::block_sum_lds<3 * R>(acc, red);
    if (threadIdx.x < 3 * R)
        a.part[(size_t)(3 * j + threadIdx.x) * kEntryMaxBlocks + blk] = t[threadIdx.x];
}

template <int V, bool WIT, int NT>
__device__ __forceinline__ void embed_product_block(const EmbedArgs &a, const EntriesArgs &e, int idx, uint64_t *red)
{
    entries_block<V, WIT, NT, 4>(EmbedRows<V>{a.tok, a.E, a.ld, a.vocab, a.d, a.scale},
                              [&](uint64_t row) { return a.E1[row]; }, [&](uint64_t col) { return a.E2[col]; }, a.n,
                              a.lk, e.C, e.we, e.mm, idx, e.total, red);
}

template <int R, bool FIRST>
__global__ __launch_bounds__(256) void k_embed_pass(EmbedArgs a, int j, uint64_t q)
{
    __shared__ uint64_t red[m61::block_sum_words(3 * R, kThreads)];
    embed_pass_block<R, FIRST>(a, j, q, blockIdx.x, gridDim.x, red);
}

// One workgroup per round and one for the end, blockIdx.x = lv, as
// k_gate_tails; the further workgroups compute the product (the passes, short of
// workgroups and waiting on memory, were no faster beside it).
template <int V, bool WIT>
__global__ __launch_bounds__(kEntryTailThreads) void k_embed_tails(EmbedArgs a, int j0, EntriesArgs e)
{
    constexpr int NT = kEntryTailThreads, S = 1 << kEntryTailLog, EM = 1 << (kEntryTailMax - kEntryTailLog);
    constexpr int IT = S / NT;
    __shared__ uint64_t t0[S], t1[S];
    __shared__ uint64_t red[m61::block_sum_words(3, NT)];
    __shared__ uint64_t rhol[32];
    const int j = blockIdx.x, tid = threadIdx.x;
    if (j > a.lv) {  // workgroup-uniform
        embed_product_block<V, WIT, NT>(a, e, j - a.lv - 1, red);
        return;
    }
    uint64_t g[3] = {0, 0, 0};
    const int m = a.lv - j0, base = m < kEntryTailLog ? m : kEntryTailLog, C = m - base;  // C <= 2 rounds in registers
    uint64_t u[IT][EM] = {}, v[IT][EM] = {}, hi[IT][EM] = {};
    if (j >= j0) {  // asked for first, as in k_gate_tails
        const uint64_t *p0 = j0 == 0 ? a.W : a.T0, *p1 = j0 == 0 ? a.b : a.T1;
#pragma unroll
        for (int it = 0; it < IT; it++) {
            const int i = it * NT + tid < 1 << base ? it * NT + tid : 0;  // past the end: entry 0's, unused
#pragma unroll
            for (int t = 0; t < EM; t++)
                if (t < 1 << C) {
                    u[it][t] = p0[i + (t << base)];
                    v[it][t] = p1[i + (t << base)];
                    if (j0 == 0) hi[it][t] = a.W[a.rows + i + (t << base)];
                }
        }
    }
    if (tid < a.lv) rhol[tid] = a.rho[tid];
    if (j < j0) {
        const int s = j - j % kEntryPass, r = j0 - s < kEntryPass ? j0 - s : kEntryPass;
        const int nb = entry_blocks(1ull << (a.lv - s - r));
        const uint64_t *p = a.part + 3 * (size_t)j * kEntryMaxBlocks;
        for (int b = tid; b < nb; b += NT)
            for (int q = 0; q < 3; q++) g[q] = m61::fold(g[q] + p[(size_t)q * kEntryMaxBlocks + b]);
    } else {
        const int jj = j - j0, n0 = 1 << base;
        __syncthreads();
#pragma unroll
        for (int it = 0; it < IT; it++) {
            const int i = it * NT + tid;
            if (i >= n0) continue;
            if (j0 == 0)
#pragma unroll
                for (int t = 0; t < EM; t++) u[it][t] = embed_weight(u[it][t], hi[it][t]);
#pragma unroll
            for (int c = 0; c < kEntryTailMax - kEntryTailLog; c++) {
                const int h = (1 << C) >> (c + 1);
                if (c > jj || h == 0) continue;
#pragma unroll
                for (int p = 0; p < EM / 2; p++) {
                    if (p >= h) continue;
                    const uint64_t u1 = h == 2 ? u[it][p + 2] : u[it][1], v1 = h == 2 ? v[it][p + 2] : v[it][1];
                    if (c == jj) {
                        embed_pair(u[it][p], u1, v[it][p], v1, g);
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
            if (j == a.lv) {
                if (tid != 0) return;
                const uint64_t u = m61::canon(t0[0]), v = m61::canon(t1[0]);
                if (a.lv == 0) a.tr[0] = *e.c0 = m61::mul(u, v);
                a.tr[1 + 3 * (size_t)a.lv] = u;
                a.tr[2 + 3 * (size_t)a.lv] = v;
                return;
            }
            const int h = n >> 1;
            for (int i = tid; i < h; i += NT) {
                embed_pair(t0[i], t0[i + h], t1[i], t1[i + h], g);
            }
        }
    }
    const uint64_t *t = m61::block_sum_lds<3>(g, red);
    if (tid != 0) return;
    a.tr[1 + 3 * (size_t)j] = t[0];
    a.tr[2 + 3 * (size_t)j] = t[1];
    // at 2: g_0 + 2 (g_1 - g_0) + 2 (differences' products)
    a.tr[3 + 3 * (size_t)j] = m61::sub(m61::add(m61::add(t[1], t[1]), m61::add(t[2], t[2])), t[0]);
    if (j == 0) a.tr[0] = *e.c0 = m61::add(t[0], t[1]);
}

int embed_entries(const EmbedArgs &a, const EntriesArgs &e)
{
    const int V = entries_width(1ull << a.lk, e.C, e.wit ? &e.we : nullptr);
    return entries_blocks((uint64_t)a.n << a.lk, V, kEntryTailThreads);
}

void launch_embed(const EmbedArgs &a, const EntriesArgs &e, hipStream_t st)
{
    const uint64_t scale = a.scale < 0 ? m61::P - (uint64_t)(-(int64_t)a.scale) : (uint64_t)a.scale;
    const uint32_t nl = embed_limb_words(a.d) / 2;
    const uint64_t threads = nl + (uint64_t)a.n + (1ull << a.lk);
    hipLaunchKernelGGL(k_embed_front, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, nl);
    const int ns = (int)((a.n + 255) / 256);
    // 32 rows a workgroup use each fragment of the columns twice (128000 x 4096:
    // 167 us, with 16 rows 171); 16 rows where 32 would leave a CU fewer than two
    // workgroups
    if (a.rows >= 32 * 512)
        hipLaunchKernelGGL((k_embed_bind<2, 8>), dim3(ns + (unsigned)(a.rows / 32)), dim3(256), 0, st, a, ns, scale);
    else
        hipLaunchKernelGGL((k_embed_bind<1, 8>), dim3(ns + (unsigned)((a.rows + 15) / 16)), dim3(256), 0, st, a, ns, scale);
    const int j0 = entry_pass_rounds(a.lv);
    for (int j = 0; j < j0; j += kEntryPass) {
        const int r = j0 - j < kEntryPass ? j0 - j : kEntryPass;
        const uint64_t q = 1ull << (a.lv - j - r);
        const dim3 grid(entry_blocks(q)), blk(kThreads);
#define RA_EMBED_PASS(R)                                                                       \
    do {                                                                                       \
        if (j == 0) hipLaunchKernelGGL((k_embed_pass<R, true>), grid, blk, 0, st, a, j, q);    \
        else hipLaunchKernelGGL((k_embed_pass<R, false>), grid, blk, 0, st, a, j, q);          \
    } while (0)
        if (r == 3) RA_EMBED_PASS(3);
        else if (r == 2) RA_EMBED_PASS(2);
        else RA_EMBED_PASS(1);
#undef RA_EMBED_PASS
    }
    entries_variant(1ull << a.lk, e, [&](auto V, auto W) {
        hipLaunchKernelGGL((k_embed_tails<decltype(V)::value, decltype(W)::value>), dim3(a.lv + 1 + e.total),
                           dim3(kEntryTailThreads), 0, st, a, j0, e);
    });
}

}  // namespace ra
