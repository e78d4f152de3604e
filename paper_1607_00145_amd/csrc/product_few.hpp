// product_few.hpp -- products of few rows (device code) that no tile suits: C[i, j] = sum
// over K of M(i, k) N(j, k) with rows of N at any address, for up to 32 rows i or up to
// 64 of all experts together, and of one to four rows (product_is_few says when).
//
// The first kernel is for N off the 16-byte grid, which tiles would copy first.  Bound by
// N's bytes, and where these are few by the launch and two memory latencies.  A
// workgroup takes 32 rows of N (columns of C) and its eight wavefronts every eighth
// panel of 128 bytes of K; N goes from memory straight into the registers that the
// MFMA reads, 64 bytes of one row a lane, so that no byte waits for a barrier, and
// the eight partial results are summed in wavefront order through LDS.  5 to 32 rows
// with 8192 x 4096 in bf16 take 18 to 22 us (67 MB: 3.1 to 3.7 TB/s; blocks of 32 x 32 take
// 12, and where N is copied before 30 more).
#pragma once
#include "product.hpp"

namespace gett {

constexpr int kFewCols = 32, kFewWaves = 8;   // columns of C of a workgroup, its wavefronts

template <typename T> struct Few {
    static constexpr int EP = 16 / sizeof(T), KP = 8 * EP;
    // four pieces of a row from k on
    static __device__ __forceinline__ void load(const T *row, int k, i4 v[4])
    {
#pragma unroll
        for (int s = 0; s < 4; ++s)
            v[s] = load16(row + k + s * EP);
    }
    // the same with zeros behind K
    static __device__ __forceinline__ void load_last(const T *row, int k, int extent, i4 v[4])
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Run<T, EP> r;
#pragma unroll
            for (int x = 0; x < EP; ++x)
                r.v[x] = k + s * EP + x < extent ? row[k + s * EP + x] : from_float<T>(0.0f);
            v[s] = __builtin_bit_cast(i4, r);
        }
    }
};

template <typename T>
__global__ __launch_bounds__(64 * kFewWaves) void product_few_kernel(ProductArgs g, int groups)
{
    typedef Few<T> F;
    constexpr int NW = kFewWaves;
    constexpr int ROW = 36;   // floats of a row of partial results: whole vectors, few conflicts
    __shared__ __attribute__((aligned(16))) float sums[NW][32][ROW];
    const int lane = (int)threadIdx.x & 63, q = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int slot = (int)quotient(blockIdx.x, g.tilesN, g.bandInv);
    const int col0 = ((int)blockIdx.x - slot * g.tilesN) * kFewCols;
    int begin = 0, end = g.m, e = 0;
    if (groups == kByRows) {
        // a workgroup for each row of the list; that of an expert's first row takes the
        // expert (or all rows of none)
        e = 0;
        for (int e0 = 0; e0 < g.experts; e0 += 64) {
            const int x = e0 + lane;
            const int n = __popcll(__ballot(x < g.experts && expert_offset(g.offsets, x + 1, g.m) <= slot));
            e += n;
            if (n < 64) break;
        }
        e = __builtin_amdgcn_readfirstlane(e);
        begin = expert_offset(g.offsets, e, g.m);
        if (slot != begin) return;
        end = e == g.experts ? g.m : expert_offset(g.offsets, e + 1, g.m);
    }
    const bool empty = groups == kByRows && e == g.experts;
    Epilogue o = g.out;
    if (groups == kByRows && o.bias && !empty) o.bias += (int64_t)e * g.n * sizeof(T);
    if (empty) {
        o.bias = nullptr;
        o.activation = GETT_ACTIVATION_NONE;
    }
    const uint64_t key = o.drop.cut ? o.drop.key() : 0;
    const int col = col0 + q < g.n ? col0 + q : g.n - 1;   // (the last again: not stored)
    const T *N = reinterpret_cast<const T *>(g.N + (groups == kByRows && !empty ? (int64_t)e * g.stepN : 0) +
                                             (int64_t)col * g.ldn);
    const int panels = empty ? 0 : g.k / F::KP;    // whole ones
    const bool rest = !empty && g.k % F::KP;
    // Rows are often a power of two apart: workgroups begin at different panels, so
    // that together they ask all memory channels and not a few (one row of 4096 with
    // 8192 x 4096: 22.8 -> 19.6 us).
    const int turn = panels > 0 ? (int)(blockIdx.x * NW % (unsigned)panels) : 0;
    for (int row0 = begin; row0 < end; row0 += 32) {
        // rows that are not there are the last one again: not stored
        int64_t from = min(row0 + q, end - 1);
        if (g.order && !empty)
            from = quotient(min((uint32_t)g.order[from], (uint32_t)g.m - 1), g.choices, g.choicesInv);
        const T *M = reinterpret_cast<const T *>(g.M + (empty ? 0 : from * g.ldm));
        f16v acc;
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[x] = 0.0f;
        auto multiply = [&](const i4 w[4], const i4 x[4]) {
#pragma unroll
            for (int s = 0; s < 4; ++s) acc = product_mfma<T>(w[s], x[s], acc);
        };
        // U panels on their way
        auto some = [&](auto count, int t) {
            constexpr int U = decltype(count)::value;
            i4 w[U][4], x[U][4];
            int k[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                int p = t + u * NW + turn;
                if (p >= panels) p -= panels;
                k[u] = p * F::KP + 4 * h * F::EP;
                F::load(N, k[u], w[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) F::load(M, k[u], x[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) multiply(w[u], x[u]);
        };
        constexpr int U = 4;
        int t = wave;
        for (; t + (U - 1) * NW < panels; t += U * NW) some(std::integral_constant<int, U>{}, t);
        for (; t < panels; t += NW) some(std::integral_constant<int, 1>{}, t);
        if (rest && wave == NW - 1) {
            i4 w[4], x[4];
            const int k = panels * F::KP + 4 * h * F::EP;
            F::load_last(N, k, g.k, w);
            F::load_last(M, k, g.k, x);
            multiply(w, x);
        }
        __syncthreads();   // the rows before are read
        if (row0 + q < end) {
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f4 *>(&sums[wave][q][8 * a + 4 * h]) =
                    f4{acc[4 * a], acc[4 * a + 1], acc[4 * a + 2], acc[4 * a + 3]};
        }
        __syncthreads();
        const int count = min(32, end - row0) * 4;   // runs of eight columns
        if ((int)threadIdx.x < count) {
            const int r = (int)threadIdx.x >> 2, c = ((int)threadIdx.x & 3) * 8;
            float v[8] = {};
#pragma unroll
            for (int s = 0; s < NW; ++s) {
                const f4 lo = *reinterpret_cast<const f4 *>(&sums[s][r][c]);
                const f4 hi = *reinterpret_cast<const f4 *>(&sums[s][r][c + 4]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] += lo[i];
                    v[4 + i] += hi[i];
                }
            }
            product_store<T>(o, key, row0 + r, col0 + c, g.n - col0 - c, v);
        }
    }
}

// One to four rows, or rows of experts that are nearly all different: no matrix unit,
// of whose 32 rows it would fill one.  A wavefront takes two rows of N whole, 1 KB of one
// after the other, so that every load is a run of whole lines; its lanes multiply
// their 16 bytes with x's, and sum up across the wavefront at the end.  The sixteen
// wavefronts of a workgroup have up to 128 KB on their way.  Bound by the weights' bytes:
// eight experts of 1024 x 2048 for a token in bf16 take 9 us (33 MB, and the launch), one
// row with 2048 x 2048 4.7.  (Where the blocks of 32 columns fill the card they are
// faster: 8192 x 4096 takes 14 us here, 20 in the kernel above, 12 in those.)
constexpr int kRowWaves = 16;

template <typename T, int R>
__global__ __launch_bounds__(64 * kRowWaves) void product_row_kernel(ProductArgs g, int groups)
{
    constexpr int EP = 16 / sizeof(T), STEP = 64 * EP, CPW = kFewCols / kRowWaves, U = R == 1 ? 8 : R == 2 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float sums[R][kFewCols];
    const int lane = (int)threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int slot = (int)quotient(blockIdx.x, g.tilesN, g.bandInv);
    const int col0 = ((int)blockIdx.x - slot * g.tilesN) * kFewCols;
    const int row0 = groups == kByRows ? slot : 0;
    int e = 0;
    Epilogue o = g.out;
    bool empty = false;
    int64_t from = row0;
    if (groups == kByRows) {
        if (g.order)
            from = quotient(min((uint32_t)g.order[row0], (uint32_t)g.m - 1), g.choices, g.choicesInv);
        for (int e0 = 0; e0 < g.experts; e0 += 64) {
            const int x = e0 + lane;
            const int n = __popcll(__ballot(x < g.experts && expert_offset(g.offsets, x + 1, g.m) <= slot));
            e += n;
            if (n < 64) break;
        }
        e = __builtin_amdgcn_readfirstlane(e);
        empty = e == g.experts;
        if (o.bias) o.bias += (int64_t)e * g.n * sizeof(T);
        if (empty) {
            o.bias = nullptr;
            o.activation = GETT_ACTIVATION_NONE;
            from = 0;
        }
    }
    const T *N[CPW], *M[R];
#pragma unroll
    for (int c = 0; c < CPW; ++c) {
        const int col = min(col0 + wave * CPW + c, g.n - 1);   // (the last again: not stored)
        N[c] = reinterpret_cast<const T *>(g.N + (empty ? 0 : (int64_t)e * g.stepN) + (int64_t)col * g.ldn);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        M[r] = reinterpret_cast<const T *>(g.M + (groups == kByRows ? from : (int64_t)min(r, g.m - 1)) * g.ldm);
    float acc[CPW][R];
#pragma unroll
    for (int c = 0; c < CPW; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[c][r] = 0.0f;
    auto add = [&](const Run<T, EP> &w, const Run<T, EP> x[R], int c) {
#pragma unroll
        for (int i = 0; i < EP; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[c][r] = fmaf(to_float(w.v[i]), to_float(x[r].v[i]), acc[c][r]);
    };
    auto some = [&](auto count, int k) {
        constexpr int N_ = decltype(count)::value;
        typedef Run<T, EP> V;
        V w[N_][CPW], x[N_][R];
#pragma unroll
        for (int u = 0; u < N_; ++u)
#pragma unroll
            for (int c = 0; c < CPW; ++c)
                w[u][c] = *reinterpret_cast<const V *>(N[c] + k + u * STEP);
#pragma unroll
        for (int u = 0; u < N_; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r)
                x[u][r] = *reinterpret_cast<const V *>(M[r] + k + u * STEP);
#pragma unroll
        for (int u = 0; u < N_; ++u)
#pragma unroll
            for (int c = 0; c < CPW; ++c) add(w[u][c], x[u], c);
    };
    if (!empty) {
        int k = lane * EP;
        const int whole = g.k / STEP * STEP;
        for (; k + (U - 1) * STEP < whole; k += U * STEP) some(std::integral_constant<int, U>{}, k);
        for (; k < whole; k += STEP) some(std::integral_constant<int, 1>{}, k);
        if (k + EP <= g.k) {
            some(std::integral_constant<int, 1>{}, k);
        } else if (k < g.k) {
            for (int i = 0; k + i < g.k; ++i)
#pragma unroll
                for (int c = 0; c < CPW; ++c)
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        acc[c][r] = fmaf(to_float(N[c][k + i]), to_float(M[r][k + i]), acc[c][r]);
        }
    }
#pragma unroll
    for (int c = 0; c < CPW; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int d = 32; d; d >>= 1) acc[c][r] += __shfl_xor(acc[c][r], d);
            if (lane == 0) sums[r][wave * CPW + c] = acc[c][r];
        }
    __syncthreads();
    const int r = (int)threadIdx.x >> 2, c = ((int)threadIdx.x & 3) * 8;
    if (r >= R || row0 + r >= g.m) return;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sums[r][c + i];
    product_store<T>(o, o.drop.cut ? o.drop.key() : 0, row0 + r, col0 + c, g.n - col0 - c, v);
}

}  // namespace gett
