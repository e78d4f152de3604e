// orth.hip -- Newton-Schulz orthogonalisation of a stack of matrices.
//
//     X_0 = G / (|G| + eps);   S = X X^T;   B = b S + c S^2;   X <- a X + B X
//
// X is held with its shorter side as rows (m <= n), so S and B are m x m.
// Bound: matrix instructions.  S and S^2 are symmetric, so only the tiles on
// and below the diagonal are computed and the others mirrored: m^2 n + m^3 +
// 2 m^2 n operations per step instead of 2 m^2 n + 2 m^3 + 2 m^2 n, each three
// MFMA operations, since numbers are held in two parts.
//
// 4096 x 4096, five steps: 3.64-3.81 ms by card, in every type; a step's three
// products 193-214, 195-215 and 346-394 us (1.0 to 1.2 PFLOP/s of MFMA operations;
// the update's panels alone, without reading the addend and writing both
// orientations, 1.2), the norm 13.5 and the start 41-47.
// Mid-sized matrices are chains of 17 launches, each a load latency, a short K and
// the stores, waiting for the one before: 517 x 1000 129 us, products of 5 to 12;
// 1024 x 1024 189, 2048 x 2048 800-890.
//
// Numbers.  |X| <= 1 at the start and every singular value stays below 3
// (gett_orthogonalize refuses other polynomials), so all entries of X, S and
// B are below 15 and fit a half after multiplication by 2^12, which keeps
// entries down to 2^-26 normal.  A matrix is held as two halves, hi + lo (22
// bits; products in panel.hpp, sums in 32 bits), for every type: the result is
// as close to the 64-bit one as that of products in 32 bits (1.5e-6 of its norm
// for both at 512 x 517).  The low part's grid ends at 2^-36, which the steps
// magnify by a^steps in the directions of small numbers: beside one element 1e6
// times the others the error is 1.5e-6 where 32 bits leave 2e-7 (512 x 512).  A
// third part would cost three more products.  One half would not do for bf16
// either: 4096 x 4096 would take 1.6 ms, but its fifteen roundings leave 1.1e-3 to
// 2.9e-3 of the norm beside the 1.7e-3 that rounding the result costs.
//
// Every product has K along the rows of both operands: S from X, S^2 from S
// (symmetric), B X from B and X^T.  So X is kept in both orientations, and
// the update's epilogue, whose lanes hold runs of neighbours along rows and
// columns alike, writes both in vectors.  Rows are padded with zeros to whole
// panels.
#include <math.h>

#include "launch.hpp"
#include "matrix.hpp"
#include "panel.hpp"

namespace gett {
namespace {

constexpr float kUp = 4096.0f, kDown = 1.0f / 4096.0f;   // halves hold 2^12 x
constexpr int kNormThreads = 256;
constexpr int kNormBlocks = 1024;   // at most, per matrix; one partial sum each

// ----------------------------------------------------------------- storage ---

// Numbers of one panel: the high parts of eight and then their low parts (slab
// 0 takes the even pieces of a panel, slab 1 the odd ones).
constexpr int kNumbers = 32;
__host__ __device__ inline int64_t panel_count(int64_t k) { return (k + kNumbers - 1) / kNumbers; }
// columns of a row, padding included
__host__ __device__ inline int padded(int k) { return (int)panel_count(k) * kNumbers; }
// the byte of number k in its panel
__host__ __device__ constexpr int in_panel(int k) { return (k >> 3) * 32 + (k & 7) * 2; }
// the byte of column k of a row in a matrix of `rows` rows
__device__ __forceinline__ int64_t at(int rows, int row, int k)
{
    return ((int64_t)(k / kNumbers) * rows + row) * 128 + in_panel(k % kNumbers);
}

// N neighbours (N divides 8 and the column): held values are 2^12 x
template <int N> __device__ __forceinline__ void store_run(char *p, const float *v)
{
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    vec hi, lo;
#pragma unroll
    for (int i = 0; i < N; ++i) hi[i] = (_Float16)v[i];
#pragma unroll
    for (int i = 0; i < N; ++i) lo[i] = (_Float16)(v[i] - (float)hi[i]);
    *reinterpret_cast<vec *>(p) = hi;
    *reinterpret_cast<vec *>(p + 16) = lo;
}
template <int N> __device__ __forceinline__ void load_run(const char *p, float *v)
{
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    const vec hi = *reinterpret_cast<const vec *>(p);
    const vec lo = *reinterpret_cast<const vec *>(p + 16);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

// ------------------------------------------------------------ norm and start ---

// A stack of matrices: element [i, k] of matrix z at z sb + i si + k sk
template <typename T> struct Stack {
    T *p;
    int64_t sb, si, sk;
};

// the sum over a workgroup, in a fixed order; `lds` holds one value a wavefront
__device__ __forceinline__ double block_sum(double v, double *lds)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kNormThreads / 64; ++w) sum += lds[w];
    return sum;
}

// partial[z][block] = sum of squares of rows block, block + blocks, ... where
// `rows` is the direction of the larger stride; bound by reading G
template <typename T>
__global__ __launch_bounds__(kNormThreads) void orth_norm_kernel(Stack<const T> G, int rows,
                                                                 int cols, int blocks,
                                                                 Recip blocksInv, double *partial)
{
    __shared__ double lds[kNormThreads / 64];
    const int z = (int)quotient(blockIdx.x, blocks, blocksInv), b = (int)blockIdx.x - z * blocks;
    const T *p = G.p + z * G.sb;
    constexpr int N = 16 / (int)sizeof(T);   // values of 16 bytes
    double s = 0.0;
    for (int i = b; i < rows; i += blocks) {
        const T *row = p + i * G.si;
        const int whole = G.sk == 1 ? cols / N : 0;
#pragma unroll 4
        for (int k = (int)threadIdx.x; k < whole; k += kNormThreads) {
            const Run<T, N> v = *reinterpret_cast<const Run<T, N> *>(row + k * N);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const double x = (double)to_float(v.v[j]);
                s += x * x;
            }
        }
        for (int k = whole * N + (int)threadIdx.x; k < cols; k += kNormThreads) {
            const double x = (double)to_float(row[k * G.sk]);
            s += x * x;
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partial[(int64_t)z * blocks + b] = s;
}

// X_0 in both orientations, a 64 x 64 tile a workgroup
constexpr int kStart = 64;
template <typename T>
__global__ __launch_bounds__(kNormThreads) void orth_start_kernel(
    Stack<const T> G, int m, int n, int tiles, Recip tilesInv, int tilesN, Recip tilesNInv,
    const double *partial, int blocks, double eps, char *X, char *XT, int64_t stackX, int64_t stackXT)
{
    __shared__ double lds[kNormThreads / 64];
    __shared__ float tile[kStart][kStart + 1];
    const int tid = (int)threadIdx.x;
    const int z = (int)quotient(blockIdx.x, tiles, tilesInv), t = (int)blockIdx.x - z * tiles;
    const int tm = (int)quotient((uint32_t)t, tilesN, tilesNInv);
    const int i0 = tm * kStart, k0 = (t - tm * tilesN) * kStart;
    // the tile's loads are on their way while the norm is summed
    const T *g = G.p + z * G.sb;
    const bool along = G.sk <= G.si;   // neighbouring lanes take neighbours in memory
    constexpr int U = kStart * kStart / kNormThreads;
    T x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = u * kNormThreads + tid, a = e / kStart, b = e % kStart;
        const int i = i0 + (along ? a : b), k = k0 + (along ? b : a);
        x[u] = g[(i < m ? i : m - 1) * G.si + (k < n ? k : n - 1) * G.sk];
    }
    double sum = 0.0;
    for (int b = tid; b < blocks; b += kNormThreads) sum += partial[(int64_t)z * blocks + b];
    sum = block_sum(sum, lds);
    // an infinity or a NaN anywhere makes the whole matrix NaN
    const double scale =
        sum < (double)INFINITY ? (double)kUp / (sqrt(sum) + eps) : (double)NAN;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = u * kNormThreads + tid, a = e / kStart, b = e % kStart;
        const int i = along ? a : b, k = along ? b : a;
        tile[i][k] = i0 + i < m && k0 + k < n ? (float)((double)to_float(x[u]) * scale) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kStart * kStart / 8 / kNormThreads; ++u) {
        const int e = u * kNormThreads + tid;
        const int a = e / (kStart / 8), c = e % (kStart / 8) * 8;
        float v[8];
        if (i0 + a < m && k0 + c < padded(n)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[a][c + i];
            store_run<8>(X + z * stackX + at(m, i0 + a, k0 + c), v);
        }
        if (k0 + a < n && i0 + c < padded(m)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[c + i][a];
            store_run<8>(XT + z * stackXT + at(n, k0 + a, i0 + c), v);
        }
    }
}

// O = X_0 (no steps)
template <typename T>
__global__ __launch_bounds__(256) void orth_copy_kernel(const char *X, int64_t stackX, int m, int n,
                                                        Stack<T> O, int64_t total)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= total) return;
    const int64_t z = e / ((int64_t)m * n), rest = e % ((int64_t)m * n);
    const int i = (int)(rest / n), k = (int)(rest % n);
    float v;
    load_run<1>(X + z * stackX + at(m, i, k), &v);
    O.p[z * O.sb + i * O.si + k * O.sk] = from_float<T>(v * kDown);
}

// ---------------------------------------------------------------- products ---

enum Step { kGram, kPoly, kUpdate, kLast };

struct ProductArgs {
    const char *P, *Q;          // the operands, K along their rows
    int64_t stackP, stackQ;
    int m, n, panels;           // rows of P, rows of Q, panels of a row
    const char *addend;         // Poly: S; Update, Last: X; [row][col] as `out`
    char *out, *outT;           // [row][col], and its transpose
    int64_t stackOut, stackOutT;
    float factor, scale;        // out = factor * product + scale * addend
};

// Passes in which a tile's panels, [panel][row][128 bytes], go through LDS.
template <typename S, bool ACROSS> constexpr int image_passes()
{
    constexpr int ROWS = ACROSS ? S::BN : S::BM, COLS = ACROSS ? S::BM : S::BN;
    constexpr int FIT = S::lds(kPanelSplit) / (ROWS * 128), ALL = COLS / kNumbers;
    return FIT < ALL ? ALL / FIT : 1;
}

// Small tiles have LDS to spare for the addend, which then arrives with the
// first panels; large ones load it after the sums, where panels were.
template <typename S> constexpr bool kAddendEarly = S::BM == 64;

// Starts the loads of a tile's panels of a matrix of `rows` rows and `panels`
// panels, as the LDS image of pass `pass`.  Outside the matrix any of its
// values will do: what becomes of them is replaced by zeros.
template <typename S>
__device__ __forceinline__ void load_panels(const Panel<kPanelSplit, S> &p, char *image,
                                            const char *from, int rows, int panels, int row0,
                                            int col0, int pass)
{
    constexpr int E = kNumbers;
    constexpr int PP = S::BN / E / (kAddendEarly<S> ? 1 : image_passes<S, false>());
    const int lane = (int)threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
    for (int u = 0; u < PP * S::BM / 8 / (S::THREADS / 64); ++u) {
        const int k = u * (S::THREADS / 64) + wave;   // eight rows of a panel
        const int panel = k / (S::BM / 8), row = row0 + k % (S::BM / 8) * 8 + (lane >> 3);
        int to = col0 / E + pass * PP + panel;
        to = to < panels ? to : panels - 1;
        const char *src = from + ((int64_t)to * rows + (row < rows ? row : rows - 1)) * 128 +
                          (lane & 7) * 16;
        __builtin_amdgcn_global_load_lds((matrix_global *)src, (matrix_lds *)(image + k * 1024), 16, 0,
                                         0);
    }
}

// Writes a tile's accumulators (held values) to panels at `out`, a matrix of
// `rows` rows and `panels` panels, as [row][col] or ACROSS as its transpose,
// `row0` / `col0` being the tile's first row and column there.  The lanes'
// runs are a few elements of many rows, so they are put in order in LDS, the
// panels' image: every store of a wavefront then covers 1 KB.
template <typename S, bool ACROSS>
__device__ __forceinline__ void store_panels(Panel<kPanelSplit, S> &p, char *lds, char *out,
                                             int rows, int panels, int row0, int col0)
{
    constexpr int E = kNumbers;
    constexpr int ROWS = ACROSS ? S::BN : S::BM, COLS = ACROSS ? S::BM : S::BN;
    constexpr int FR = ACROSS ? S::FN : S::FM, FC = ACROSS ? S::FM : S::FN;   // runs of a lane
    constexpr int ALL = COLS / E, PP = ALL / image_passes<S, ACROSS>();
    static_assert(ALL % PP == 0 && (PP * E) % (32 * FC) == 0, "a wavefront's columns in one pass");
    const int tid = (int)threadIdx.x;
    const int mine = (ACROSS ? p.wm : p.wn) * 32 * FC;   // this wavefront's first column
#pragma unroll
    for (int pass = 0; pass < ALL / PP; ++pass) {
        __syncthreads();
        if (mine / (PP * E) == pass) {
            // each pass rounds anew: the compiler would round all values once
            // and keep the parts, twice the registers, in scratch memory
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) asm volatile("" : "+v"(p.acc[i][j]));
#pragma unroll
            for (int e = 0; e < 16; ++e) {
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    const int row = ACROSS ? p.col(f) : p.row(f, e);
                    const int col = (ACROSS ? p.row(0, e) : p.col(0)) - pass * PP * E;
                    const int in = col % E;
                    const int byte = in_panel(in);
                    // pieces of a row lie by an exclusive or, so that the lanes'
                    // rows, a power of two apart, fall on different banks
                    const int x = row / FR & 7;
                    char *at = lds + (col / E * ROWS + row) * 128 + ((byte >> 4 ^ x) << 4) + (byte & 15);
                    typedef _Float16 vec __attribute__((ext_vector_type(FC)));
                    vec hi, lo;
#pragma unroll
                    for (int c = 0; c < FC; ++c) {
                        const float v = ACROSS ? p.acc[c][f][e] : p.acc[f][c][e];
                        hi[c] = (_Float16)v;
                        lo[c] = (_Float16)(v - (float)hi[c]);
                    }
                    *reinterpret_cast<vec *>(at) = hi;
                    *reinterpret_cast<vec *>(lds + (col / E * ROWS + row) * 128 +
                                             (((byte >> 4) + 1 ^ x) << 4) + (byte & 15)) = lo;
                }
                __builtin_amdgcn_sched_barrier(0);   // no registers for many addresses
            }
        }
        __syncthreads();
        for (int u = tid; u < PP * ROWS * 8; u += S::THREADS) {
            const int piece = u & 7, row = u / 8 % ROWS, panel = u / 8 / ROWS;
            const i4 v = *reinterpret_cast<const i4 *>(lds + (panel * ROWS + row) * 128 +
                                                       ((piece ^ (row / FR & 7)) << 4));
            const int to = (col0 + pass * PP * E) / E + panel;
            if (row0 + row < rows && to < panels)
                *reinterpret_cast<i4 *>(out + ((int64_t)to * rows + row0 + row) * 128 + piece * 16) = v;
        }
    }
}

template <int STEP, typename S, typename T>
__global__ __launch_bounds__(S::THREADS) void orth_product_kernel(ProductArgs d, PanelGrid grid,
                                                                  Stack<T> O)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    constexpr int FM = S::FM, FN = S::FN;
    constexpr bool kSymmetric = STEP == kGram || STEP == kPoly;
    int tm, tn;
    const PanelItem w = panel_item(grid, (int)blockIdx.x);
    const int z = w.z;
    if constexpr (kSymmetric) panel_triangle(w.tile, tm, tn);
    else panel_tile(grid, w.tile, tm, tn);
    const PanelOperand A = {reinterpret_cast<const uint8_t *>(d.P) + z * d.stackP, nullptr, d.m,
                            tm * S::BM};
    const PanelOperand B = {reinterpret_cast<const uint8_t *>(d.Q) + z * d.stackQ, nullptr, d.n,
                            tn * S::BN};
    Panel<kPanelSplit, S> p;
    p.init();
    const int col = B.row0 + p.col(0), padN = padded(d.n);
    const char *addend = STEP == kGram ? nullptr : d.addend + z * d.stackOut;
    const int panelsN = padN / kNumbers;
    if constexpr (STEP != kGram && kAddendEarly<S>)
        load_panels<S>(p, dyn_lds + S::lds(kPanelSplit), addend, d.m, panelsN, A.row0, B.row0, 0);
    p.run(dyn_lds, A, B, w.t0, w.t1);
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);   // vmcnt 0 (the addend, if no panel came)
    __syncthreads();
    if (!panel_join<kPanelSplit, S>(p, grid, w, dyn_lds)) return;

    // rows and columns of the padding become zeros
    constexpr int PASSES = STEP == kGram || kAddendEarly<S> ? 1 : image_passes<S, false>();
#pragma unroll 1
    for (int pass = 0; pass < PASSES; ++pass) {
        const char *image = dyn_lds + (kAddendEarly<S> ? S::lds(kPanelSplit) : 0);
        if constexpr (STEP != kGram && !kAddendEarly<S>) {
            __syncthreads();
            load_panels<S>(p, dyn_lds, addend, d.m, panelsN, A.row0, B.row0, pass);
            __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);   // vmcnt 0
            __syncthreads();
        }
        constexpr int SPAN = S::BN / PASSES;   // columns of a pass
        if (PASSES > 1 && p.wn * 32 * FN / SPAN != pass) continue;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                float x[FN] = {};
                if constexpr (STEP != kGram) {
                    const int c = p.col(0) - pass * SPAN;
                    load_run<FN>(image + at(S::BM, p.row(i, e), c), x);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    float v = d.factor * p.acc[i][j][e];
                    if constexpr (STEP != kGram) v += d.scale * x[j];
                    p.acc[i][j][e] = A.row0 + p.row(i, e) < d.m && col + j < d.n ? v : 0.0f;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(p.acc[i][j]));   // computed here
    if constexpr (STEP != kLast) {
        store_panels<S, false>(p, dyn_lds, d.out + z * d.stackOut, d.m, panelsN, A.row0, B.row0);
        // the other orientation: X^T, or the mirrored tile
        if (!kSymmetric || tm != tn)
            store_panels<S, true>(p, dyn_lds, d.outT + z * d.stackOutT, d.n, padded(d.m) / kNumbers,
                                  B.row0, A.row0);
    } else if (O.si != 1 || O.sk == 1) {
        // a lane's rows: four times FM in a row, then as many are another's
        T *o = O.p + z * O.sb + (A.row0 + p.row(0, 0)) * O.si + col * O.sk;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if (A.row0 + p.row(i, e) < d.m) {
                    if (O.sk == 1 && col + FN <= d.n) {
                        Run<T, FN> v;
#pragma unroll
                        for (int j = 0; j < FN; ++j) v.v[j] = from_float<T>(p.acc[i][j][e] * kDown);
                        *reinterpret_cast<Run<T, FN> *>(o) = v;
                    } else {
#pragma unroll
                        for (int j = 0; j < FN; ++j)
                            if (col + j < d.n) o[j * O.sk] = from_float<T>(p.acc[i][j][e] * kDown);
                    }
                }
                o += O.si;
                asm volatile("" : "+v"(o));   // one pointer, not one per row
            }
            if (e % 4 == 3) o += 4 * FM * O.si;
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {   // neighbours in memory run along the rows, FM of which a lane holds
        T *own = O.p + z * O.sb + (A.row0 + p.row(0, 0)) + col * O.sk;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int down = p.row(0, e) - p.row(0, 0), left = d.m - (A.row0 + p.row(0, e));
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if (col + j >= d.n) continue;
                T *o = own + down + j * O.sk;
                if (left >= FM) {
                    Run<T, FM> v;
#pragma unroll
                    for (int i = 0; i < FM; ++i) v.v[i] = from_float<T>(p.acc[i][j][e] * kDown);
                    *reinterpret_cast<Run<T, FM> *>(o) = v;
                } else {
#pragma unroll
                    for (int i = 0; i < FM; ++i)
                        if (i < left) o[i] = from_float<T>(p.acc[i][j][e] * kDown);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ------------------------------------------------------------ short products ---
//
// A product of few tiles is a chain of latencies, not of work.  Here a
// workgroup takes a block of 32 x 32 results and each of its eight wavefronts
// every eighth panel, through LDS of its own: eight panels' loads are in flight
// together, and no barrier comes before the eight partial results are summed,
// in wavefront order, through LDS.  (Two panels a wavefront in flight leave
// room for one workgroup on a CU instead of two: 256 x 2048, S 9.9 us for 8.4.)

constexpr int kShortWaves = 8;
constexpr int kShortE = 32, kShortThreads = 64 * kShortWaves;
constexpr int kShortOwn = 2 * kShortE * 128;   // LDS of a wavefront
constexpr int kShortPitch = kShortE + 2, kShortAcross = kShortE + 1;
constexpr int kShortLds = kShortWaves * kShortOwn + kShortE * kShortAcross * 4;

template <int STEP, typename T>
__global__ __launch_bounds__(kShortThreads) void orth_short_kernel(ProductArgs d, PanelGrid grid,
                                                                   Stack<T> O)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    constexpr int E = kShortE, W = kShortWaves, N = E * E / kShortThreads;
    constexpr bool kSymmetric = STEP == kGram || STEP == kPoly;
    const int tid = (int)threadIdx.x, lane = tid & 63, r = tid & 31, h = (tid >> 5) & 1;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char *const own = dyn_lds + wave * kShortOwn;
    float *const turned = reinterpret_cast<float *>(dyn_lds + W * kShortOwn);
    int tm, tn;
    const PanelItem w = panel_item(grid, (int)blockIdx.x);
    const int z = w.z;
    if constexpr (kSymmetric) panel_triangle(w.tile, tm, tn);
    else panel_tile(grid, w.tile, tm, tn);
    const int row0 = tm * E, col0 = tn * E, padM = padded(d.m), padN = padded(d.n);

    // a lane's 16 bytes of each load of eight rows: piece p of row r lies at
    // place p ^ (r / 2 mod 8) of its row; rows past the last read it again, and
    // their results are not stored
    const char *from[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int lr = u % 4 * 8 + (lane >> 3), piece = (lane & 7) ^ (lr >> 1 & 7);
        const int row = (u < 4 ? row0 : col0) + lr, rows = u < 4 ? d.m : d.n;
        from[u] = (u < 4 ? d.P + z * d.stackP : d.Q + z * d.stackQ) +
                  (int64_t)(row < rows ? row : rows - 1) * 128 + piece * 16;
    }
    // the results that this lane sums, and the addend's numbers there
    const int lr = tid / (E / N), lc = tid % (E / N) * N, row = row0 + lr, col = col0 + lc;
    float x[N] = {};
    if constexpr (STEP != kGram)
        if (row < d.m && col < padN)
            load_run<N>(d.addend + z * d.stackOut + at(d.m, row, col), x);

    f16v acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    for (int t = wave; t < d.panels; t += W) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            __builtin_amdgcn_global_load_lds(
                (matrix_global *)(from[u] + (int64_t)t * (u < 4 ? d.m : d.n) * 128),
                (matrix_lds *)(own + u * 1024), 16, 0, 0);
        __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);   // vmcnt 0
        asm volatile("" ::: "memory");
        i4 a[4], b[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int place = (4 * h + s) ^ (r >> 1 & 7);
            a[s] = *reinterpret_cast<const i4 *>(own + r * 128 + place * 16);
            b[s] = *reinterpret_cast<const i4 *>(own + 4096 + r * 128 + place * 16);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s % 2 == 0) {
                acc = mfma_half(a[s], b[s], acc);
                acc = mfma_half(a[s], b[s + 1], acc);
                acc = mfma_half(a[s + 1], b[s], acc);
            }
        }
        __builtin_amdgcn_s_waitcnt(0);   // own LDS has been read
        asm volatile("" ::: "memory");
    }
    float *const mine = reinterpret_cast<float *>(own);
#pragma unroll
    for (int e = 0; e < 16; ++e) mine[(8 * (e >> 2) + 4 * h + (e & 3)) * kShortPitch + r] = acc[e];
    __syncthreads();

    // rows and columns of the padding become zeros
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
#pragma unroll
    for (int p = 0; p < W; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += reinterpret_cast<const float *>(dyn_lds + p * kShortOwn)[lr * kShortPitch + lc + i];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = d.factor * v[i];
        if constexpr (STEP != kGram) v[i] += d.scale * x[i];
        if (row >= d.m || col + i >= d.n) v[i] = 0.0f;
    }
    // the other orientation: X^T or the mirrored block; for a result whose
    // neighbours in memory lie along its rows, the only one
    const bool turn = STEP == kLast ? O.si == 1 && O.sk != 1 : !kSymmetric || tm != tn;
    if (turn) {
#pragma unroll
        for (int i = 0; i < N; ++i) turned[lr * kShortAcross + lc + i] = v[i];
        __syncthreads();
    }
    const int trow = row0 + lc, tcol = col0 + lr;   // of N neighbours of a column
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = turn ? turned[(lc + i) * kShortAcross + lr] : 0.0f;
    if constexpr (STEP != kLast) {
        if (row < d.m && col < padN)
            store_run<N>(d.out + z * d.stackOut + at(d.m, row, col), v);
        if (turn && tcol < d.n && trow < padM)
            store_run<N>(d.outT + z * d.stackOutT + at(d.n, tcol, trow), y);
    } else {
        const int er = turn ? trow : row, ec = turn ? tcol : col;   // first of the N
        const int left = turn ? (ec < d.n ? d.m - er : 0) : (er < d.m ? d.n - ec : 0);
        T *const o = O.p + z * O.sb + er * O.si + ec * O.sk;
        Run<T, N> out;
#pragma unroll
        for (int i = 0; i < N; ++i) out.v[i] = from_float<T>((turn ? y[i] : v[i]) * kDown);
        if (left >= N && (turn || O.sk == 1)) {
            *reinterpret_cast<Run<T, N> *>(o) = out;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) o[i * (turn ? O.si : O.sk)] = out.v[i];
        }
    }
}

// Square tiles (the symmetric products mirror them).
typedef PanelShape<2, 4, 4, 2, 2> Big;
typedef PanelShape<2, 2, 2, 2, 2> Mid;
typedef PanelShape<1, 1, 2, 2, 4> Small;

template <int STEP> int64_t tile_count(int64_t edge, int64_t m, int64_t n)
{
    const int64_t tm = (m + edge - 1) / edge, tn = (n + edge - 1) / edge;
    return STEP == kGram || STEP == kPoly ? tm * (tm + 1) / 2 : tm * tn;
}

// The tiles of one product: 0 Big, 1 Mid, 2 Small, 3 a short product's blocks,
// and how they are shared.
struct Choice {
    int shape;
    PanelCut cut;
    int64_t slotBytes;
    bool launchable;   // not too many tiles for a launch
};
// A short product's price beside panel_cut's, which leave out a launch's fixed
// time: that is 1.3 us shorter here, and a wavefront's panel takes 0.65, with two
// workgroups on a CU 1.6.  us as tiles of 64 x 64 and here: 160 x 160, S 5.8 /
// 4.2, update 6.9 / 4.2; 517 x 1000, S 11.4 / 7.1, S^2 9.5 / 5.2; 256 x 2048, S
// 11.3 / 8.4, update 8.7 / 8.1; 768 x 768, S 10.2 / 8.5.  With more blocks than
// are resident the tiles' fewer loads win: S of 1024 x 1024 11.2 / 12.1, the
// update of 517 x 1000 11.6 / 12.0.
PanelCut short_cut(int64_t blocks, int64_t panels)
{
    PanelCut c;
    c.full = c.blocks = blocks;
    const double each = (double)((panels + kShortWaves - 1) / kShortWaves);
    if (blocks <= 2 * kPanelCus) c.us = (blocks <= kPanelCus ? 0.65 : 1.6) * each - 1.3;
    return c;
}
template <int STEP> Choice choose(int64_t batch, int64_t m, int64_t n, int64_t panels)
{
    const PanelCut c[4] = {
        panel_cut<Big>(kPanelSplit, batch * tile_count<STEP>(Big::BM, m, n), panels),
        panel_cut<Mid>(kPanelSplit, batch * tile_count<STEP>(Mid::BM, m, n), panels),
        panel_cut<Small>(kPanelSplit, batch * tile_count<STEP>(Small::BM, m, n), panels),
        short_cut(batch * tile_count<STEP>(kShortE, m, n), panels)};
    int s = 0;
    for (int i = 1; i < 4; ++i)
        if (c[i].us < c[s].us) s = i;
    const int64_t tile[4] = {Big::TILE, Mid::TILE, Small::TILE, 0};
    const int64_t edge[4] = {Big::BM, Mid::BM, Small::BM, kShortE};
    const int64_t threads[4] = {Big::THREADS, Mid::THREADS, Small::THREADS, kShortThreads};
    PanelGrid g;
    const bool ok = panel_grid(g, batch, (m + edge[s] - 1) / edge[s], (n + edge[s] - 1) / edge[s],
                               tile_count<STEP>(edge[s], m, n), c[s], (int)panels, nullptr, nullptr);
    return {s, c[s], c[s].shared() * c[s].slices * tile[s] * 4,
            ok && fits_launch(c[s].blocks, threads[s])};
}

struct Workspace {
    float *slots;
    int *counters;
};

template <int STEP, typename S, typename T>
hipError_t product_launch(const ProductArgs &d, const PanelCut &c, const Workspace &w,
                          const Stack<T> &O, int64_t batch, hipStream_t stream)
{
    constexpr auto k = orth_product_kernel<STEP, S, T>;
    constexpr int lds = S::lds(kPanelSplit) + (STEP != kGram && kAddendEarly<S> ? S::TILE * 4 : 0);
    const hipError_t e = allow_dynamic_lds<k>(lds);
    if (e != hipSuccess) return e;
    PanelGrid g;
    if (!panel_grid(g, batch, (d.m + S::BM - 1) / S::BM, (d.n + S::BN - 1) / S::BN,
                    tile_count<STEP>(S::BM, d.m, d.n), c, d.panels, w.slots, w.counters))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3((unsigned)c.blocks), dim3(S::THREADS), lds, stream, d, g, O);
    return hipGetLastError();
}

template <int STEP, typename T>
hipError_t short_launch(const ProductArgs &d, const PanelCut &c, const Stack<T> &O, int64_t batch,
                        hipStream_t stream)
{
    constexpr auto k = orth_short_kernel<STEP, T>;
    const hipError_t e = allow_dynamic_lds<k>(kShortLds);
    if (e != hipSuccess) return e;
    PanelGrid g;
    if (!panel_grid(g, batch, (d.m + kShortE - 1) / kShortE, (d.n + kShortE - 1) / kShortE,
                    tile_count<STEP>(kShortE, d.m, d.n), c, d.panels, nullptr, nullptr))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3((unsigned)c.blocks), dim3(kShortThreads), kShortLds, stream, d, g, O);
    return hipGetLastError();
}

template <int STEP, typename T>
hipError_t product(const ProductArgs &d, const Choice &c, const Workspace &w, const Stack<T> &O,
                   int64_t batch, hipStream_t stream)
{
    if (c.shape == 0) return product_launch<STEP, Big, T>(d, c.cut, w, O, batch, stream);
    if (c.shape == 1) return product_launch<STEP, Mid, T>(d, c.cut, w, O, batch, stream);
    if (c.shape == 2) return product_launch<STEP, Small, T>(d, c.cut, w, O, batch, stream);
    return short_launch<STEP, T>(d, c.cut, O, batch, stream);
}

struct Problem {
    int64_t batch;
    int m, n;
    double a, b, c, eps;
    int steps;
    hipStream_t stream;
};

// ------------------------------------------------------------ small matrices ---
//
// A matrix whose X, X^T and S fit the 160 KB of a CU goes through all steps in
// one workgroup: no launch and no memory between them.  That wins up to the edge of
// what fits, for one matrix and for many; us so and by launches (in a graph,
// without the host's time for 17 launches), floats, bf16 the same within 6 %:
// 64 x 64 24 / 51, 12 x 64 x 128 30 / 55, and at the edge 32 x 576 49 / 54, 64 x 256
// 41 / 55, 96 x 128 47 / 55; 12 of these 50 / 58, 41 / 58, 49 / 57; 200 of them 55 /
// 156, 46 / 146, 54 / 188; 600 of them 169 / 384, 135 / 312, 154 / 396.  Bound: the
// latency of each step's three products, of the LDS accesses between them and of
// their barriers.
//
// Rows are padded to 32 (zeros, which stay zeros) and lie 16 bytes more than
// their length apart, so that sixteen rows' pieces fall on different banks.  A
// wavefront takes blocks of 32 x 32 of a product in turn; a lane then holds
// column r and four times four neighbouring rows: the transpose is written in
// vectors, X itself value by value.  B takes S's place: the blocks wait in
// registers until all have read S (kSmallBlocks a wavefront at most).

constexpr int kSmallWaves = 8;
constexpr int kSmallBlocks = 2;
constexpr int kSmallLds = 160 * 1024 - 256;

__host__ __device__ inline int small_pitch(int k) { return k * 4 + 16; }
inline int64_t small_lds(int64_t m, int64_t n)
{
    const int64_t mp = (m + 31) / 32 * 32, np = (n + 31) / 32 * 32;
    return mp * small_pitch((int)np) + (np + mp) * small_pitch((int)mp);
}
inline bool small_fits(int64_t m, int64_t n)
{
    const int64_t mb = (m + 31) / 32;
    return m <= 1024 && n <= 4096 && mb * mb <= kSmallWaves * kSmallBlocks &&
           small_lds(m, n) <= kSmallLds;
}

__device__ __forceinline__ f16v small_block(const char *a, const char *b, int k)
{
    f16v acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    constexpr int GROUP = 32;   // bytes of eight numbers, their high parts first
#pragma unroll 2
    for (int t = 0; t < k / 16; ++t) {
        const i4 ah = *reinterpret_cast<const i4 *>(a + 2 * t * GROUP);
        const i4 bh = *reinterpret_cast<const i4 *>(b + 2 * t * GROUP);
        acc = mfma_half(ah, bh, acc);
        const i4 al = *reinterpret_cast<const i4 *>(a + 2 * t * GROUP + 16);
        const i4 bl = *reinterpret_cast<const i4 *>(b + 2 * t * GROUP + 16);
        acc = mfma_half(ah, bl, acc);
        acc = mfma_half(al, bh, acc);
    }
    return acc;
}

template <typename T>
__global__ __launch_bounds__(kSmallWaves * 64) void orth_small_kernel(Stack<const T> G, Stack<T> O,
                                                                      int m, int n, double eps,
                                                                      int steps, float ca, float cb,
                                                                      float cc)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    __shared__ double sums[kSmallWaves];
    constexpr int THREADS = kSmallWaves * 64;
    const int tid = (int)threadIdx.x, lane = tid & 63, r = tid & 31, h = (tid >> 5) & 1;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int mp = (m + 31) & ~31, np = (n + 31) & ~31, mb = mp / 32, nb = np / 32;
    const int pX = small_pitch(np), pS = small_pitch(mp);
    char *const X = dyn_lds, *const XT = X + mp * pX, *const S = XT + np * pS;
    constexpr int GROUP = 32;
    const T *g = G.p + (int64_t)blockIdx.x * G.sb;

    // the norm, and all of the matrices zero
    const bool along = G.sk <= G.si;
    const int inner = along ? n : m, outer = along ? m : n;
    const int64_t so = along ? G.si : G.sk, si = along ? G.sk : G.si;
    double sum = 0.0;
    for (int o = wave; o < outer; o += kSmallWaves)
        for (int i = lane; i < inner; i += 64) {
            const double v = (double)to_float(g[o * so + i * si]);
            sum += v * v;
        }
    const i4 zero = {0, 0, 0, 0};
    for (int i = tid; i < (mp * pX + (np + mp) * pS) / 16; i += THREADS)
        reinterpret_cast<i4 *>(dyn_lds)[i] = zero;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) sum += sums[w];
    const double scale =
        sum < (double)INFINITY ? (double)kUp / (sqrt(sum) + eps) : (double)NAN;
    for (int o = wave; o < outer; o += kSmallWaves)
        for (int i = lane; i < inner; i += 64) {
            const float v = (float)((double)to_float(g[o * so + i * si]) * scale);
            const int row = along ? o : i, col = along ? i : o;
            store_run<1>(X + row * pX + in_panel(col), &v);
            store_run<1>(XT + col * pS + in_panel(row), &v);
        }
    __syncthreads();

    const auto writes = [&](char *M, int pitch, int row0, int col0, const f16v &v) {
        // the transpose: four times four neighbours of a row
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float x[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            store_run<4>(M + (col0 + r) * pitch + in_panel(row0 + 8 * q + 4 * h), x);
        }
    };
    for (int step = 0; step < steps; ++step) {
        const bool last = step + 1 == steps;
        for (int b = wave; b < mb * mb; b += kSmallWaves) {   // S = X X^T
            const int bi = b / mb, bj = b - bi * mb;
            f16v v = small_block(X + (bi * 32 + r) * pX + h * GROUP,
                                       X + (bj * 32 + r) * pX + h * GROUP, np);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] *= kDown;
            writes(S, pS, bi * 32, bj * 32, v);
        }
        __syncthreads();
        f16v poly[kSmallBlocks];   // B = b S + c S^2
#pragma unroll
        for (int u = 0; u < kSmallBlocks; ++u) {
            const int b = wave + u * kSmallWaves;
            if (b >= mb * mb) break;
            const int bi = b / mb, bj = b - bi * mb;
            poly[u] = small_block(S + (bi * 32 + r) * pS + h * GROUP,
                                        S + (bj * 32 + r) * pS + h * GROUP, mp);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float x[4];   // S is symmetric: its column r
                load_run<4>(S + (bj * 32 + r) * pS + in_panel(bi * 32 + 8 * q + 4 * h), x);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    poly[u][4 * q + e] = cb * x[e] + cc * kDown * poly[u][4 * q + e];
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kSmallBlocks; ++u) {
            const int b = wave + u * kSmallWaves;
            if (b >= mb * mb) break;
            const int bi = b / mb, bj = b - bi * mb;
            writes(S, pS, bi * 32, bj * 32, poly[u]);
        }
        __syncthreads();
        // X <- a X + B X, a block of columns (all of its rows) at a time: the
        // wavefront that reads these rows of X^T, into registers, writes them
        constexpr int KS = 8;   // steps of 16 numbers: m <= 128
        for (int bj = wave; bj < nb; bj += kSmallWaves) {
            char *const column = XT + (bj * 32 + r) * pS;
            i4 bh[KS], bl[KS];
#pragma unroll
            for (int t = 0; t < KS; ++t)
                if (t < mp / 16) {
                    bh[t] = *reinterpret_cast<const i4 *>(column + (2 * t + h) * GROUP);
                    bl[t] = *reinterpret_cast<const i4 *>(column + (2 * t + h) * GROUP + 16);
                }
            const int col = bj * 32 + r;
            T *const o = O.p + (int64_t)blockIdx.x * O.sb + col * O.sk;
#pragma unroll 1
            for (int bi = 0; bi < mb; ++bi) {
                // the rows' offsets are made here, not kept through the steps
                int px = pX;
                int64_t down = O.si;
                asm volatile("" : "+s"(px), "+s"(down));
                const char *const a = S + (bi * 32 + r) * pS + h * GROUP;
                f16v v;
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    if (t < mp / 16) {
                        const i4 ah = *reinterpret_cast<const i4 *>(a + 2 * t * GROUP);
                        v = mfma_half(ah, bh[t], v);
                        const i4 al = *reinterpret_cast<const i4 *>(a + 2 * t * GROUP + 16);
                        v = mfma_half(ah, bl[t], v);
                        v = mfma_half(al, bh[t], v);
                    }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x[4];
                    load_run<4>(column + in_panel(bi * 32 + 8 * q + 4 * h), x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[4 * q + e] = ca * x[e] + kDown * v[4 * q + e];
                }
                const int row0 = bi * 32 + 4 * h;
                if (!last) {
                    writes(XT, pS, bi * 32, bj * 32, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = v[e];
                        store_run<1>(X + (row0 + 8 * (e >> 2) + (e & 3)) * px + in_panel(col), &x);
                    }
                } else if (col < n) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int row = row0 + 8 * (e >> 2) + (e & 3);
                        if (row < m) o[row * down] = from_float<T>(v[e] * kDown);
                    }
                }
            }
        }
        __syncthreads();
    }
    if (steps == 0)
        for (int o = wave; o < m; o += kSmallWaves)
            for (int i = lane; i < n; i += 64) {
                float v;
                load_run<1>(X + o * pX + in_panel(i), &v);
                O.p[(int64_t)blockIdx.x * O.sb + o * O.si + i * O.sk] = from_float<T>(v * kDown);
            }
}

template <typename T>
gett_status_t small_launch(const Problem &P, const Stack<const T> &G, const Stack<T> &O)
{
    constexpr auto k = orth_small_kernel<T>;
    if (!fits_launch(P.batch, kSmallWaves * 64)) return GETT_ERROR_NOT_SUPPORTED;
    if (allow_dynamic_lds<k>(kSmallLds) != hipSuccess) return GETT_ERROR_HIP;
    hipLaunchKernelGGL(k, dim3((unsigned)P.batch), dim3(kSmallWaves * 64),
                       (size_t)small_lds(P.m, P.n), P.stream, G, O, P.m, P.n, P.eps, P.steps,
                       (float)P.a, (float)P.b, (float)P.c);
    return hipGetLastError() == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
}


template <typename T>
gett_status_t orthogonalize_typed(const Problem &P, Stack<const T> G, Stack<T> O)
{
    const int m = P.m, n = P.n;
    if (small_fits(m, n)) return small_launch<T>(P, G, O);
    const int64_t panelsX = panel_count(n), panelsS = panel_count(m);
    const int64_t X = m * panelsX * 128, XT = n * panelsS * 128, SS = m * panelsS * 128;
    // the norm reads along the smaller stride
    const bool along = G.sk <= G.si;
    const int outer = along ? m : n, inner = along ? n : m;
    const int blocks = outer < kNormBlocks ? outer : kNormBlocks;
    const int64_t head = (P.batch * blocks * 8 + 255) / 256 * 256;
    const int64_t startM = (m + kStart - 1) / kStart, startN = (n + kStart - 1) / kStart;
    const int64_t copies = ((int64_t)m * n * P.batch + 255) / 256;
    if (!fits_launch(P.batch * startM * startN, kNormThreads) ||
        !fits_launch(P.batch * blocks, kNormThreads) || !fits_launch(copies, 256))
        return GETT_ERROR_NOT_SUPPORTED;
    // without a quintic term to speak of S^2 is not needed
    const bool quintic = fabs(P.c) * 0x1p40 > fabs(P.b);
    const Choice gram = choose<kGram>(P.batch, m, m, panelsX);
    const Choice quad = choose<kPoly>(P.batch, m, m, quintic ? panelsS : 0);
    const Choice update = choose<kUpdate>(P.batch, m, n, panelsS);
    int64_t slotBytes = 0, counters = 0;
    for (const Choice *c : {&gram, &quad, &update}) {
        if (P.steps > 0 && !c->launchable) return GETT_ERROR_NOT_SUPPORTED;
        slotBytes = slotBytes > c->slotBytes ? slotBytes : c->slotBytes;
        counters = counters > c->cut.shared() ? counters : c->cut.shared();
    }
    Partials w;
    const int64_t matrices = head + P.batch * (X + 2 * XT + 2 * SS);
    const gett_status_t ws = stream_workspace(P.stream, (uint64_t)counters,
                                              (uint64_t)(matrices + slotBytes), w);
    if (ws != GETT_SUCCESS) return ws;
    const Workspace slots = {reinterpret_cast<float *>(static_cast<char *>(w.tiles) + matrices),
                             w.counters};
    double *partial = static_cast<double *>(w.tiles);
    char *x = static_cast<char *>(w.tiles) + head, *xt = x + P.batch * X;
    char *xt2 = xt + P.batch * XT, *s = xt2 + P.batch * XT, *poly = s + P.batch * SS;

    Stack<const T> g = G;
    if (!along) std::swap(g.si, g.sk);
    hipLaunchKernelGGL((orth_norm_kernel<T>), dim3((unsigned)(P.batch * blocks)),
                       dim3(kNormThreads), 0, P.stream, g, outer, inner, blocks, recip(blocks),
                       partial);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return GETT_ERROR_HIP;
    hipLaunchKernelGGL((orth_start_kernel<T>), dim3((unsigned)(P.batch * startM * startN)),
                       dim3(kNormThreads), 0, P.stream, G, m, n, (int)(startM * startN),
                       recip(startM * startN), (int)startN, recip(startN), partial, blocks, P.eps, x, xt, X, XT);
    e = hipGetLastError();
    if (e != hipSuccess) return GETT_ERROR_HIP;
    if (P.steps == 0) {
        hipLaunchKernelGGL((orth_copy_kernel<T>), dim3((unsigned)copies), dim3(256), 0,
                           P.stream, x, X, m, n, O, (int64_t)m * n * P.batch);
        return hipGetLastError() == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
    }
    const Stack<T> none = {nullptr, 0, 0, 0};
    for (int i = 0; i < P.steps; ++i) {
        ProductArgs d = {};
        d.P = d.Q = x;
        d.stackP = d.stackQ = X;
        d.m = d.n = m;
        d.panels = (int)panelsX;
        d.out = d.outT = s;
        d.stackOut = d.stackOutT = SS;
        d.factor = kDown;
        e = product<kGram, T>(d, gram, slots, none, P.batch, P.stream);
        if (e != hipSuccess) return GETT_ERROR_HIP;
        d.P = d.Q = d.addend = s;
        d.stackP = d.stackQ = SS;
        d.panels = quintic ? (int)panelsS : 0;
        d.out = d.outT = poly;
        d.factor = (float)(P.c * kDown);
        d.scale = (float)P.b;
        e = product<kPoly, T>(d, quad, slots, none, P.batch, P.stream);
        if (e != hipSuccess) return GETT_ERROR_HIP;
        d.P = poly;
        d.Q = xt;
        d.stackQ = XT;
        d.n = n;
        d.addend = d.out = x;
        d.outT = xt2;
        d.stackOut = X;
        d.stackOutT = XT;
        d.panels = (int)panelsS;
        d.factor = kDown;
        d.scale = (float)P.a;
        e = i + 1 < P.steps ? product<kUpdate, T>(d, update, slots, none, P.batch, P.stream)
                            : product<kLast, T>(d, update, slots, O, P.batch, P.stream);
        if (e != hipSuccess) return GETT_ERROR_HIP;
        std::swap(xt, xt2);
    }
    return GETT_SUCCESS;
}

// The largest |f| of f(x) = sum of the powers on [0, x1], from the ends and
// the points where the derivative vanishes.
double largest_step(double a, double b, double c, double s1)
{
    // s -> a s + b s^3 + c s^5; derivative a + 3 b x + 5 c x^2 with x = s^2
    auto f = [&](double s) { return fabs(a * s + b * s * s * s + c * s * s * s * s * s); };
    double best = f(s1);
    const double A = 5 * c, B = 3 * b, C = a;
    double roots[2];
    int n = 0;
    if (A != 0) {
        const double disc = B * B - 4 * A * C;
        if (disc >= 0) {
            roots[n++] = (-B + sqrt(disc)) / (2 * A);
            roots[n++] = (-B - sqrt(disc)) / (2 * A);
        }
    } else if (B != 0) {
        roots[n++] = -C / B;
    }
    for (int i = 0; i < n; ++i)
        if (roots[i] > 0 && sqrt(roots[i]) < s1) best = fmax(best, f(sqrt(roots[i])));
    return best;
}
double largest_poly(double b, double c, double x1)
{
    auto f = [&](double x) { return fabs(b * x + c * x * x); };
    double best = f(x1);
    if (c != 0) {
        const double x = -b / (2 * c);
        if (x > 0 && x < x1) best = fmax(best, f(x));
    }
    return best;
}

}  // namespace

// Singular values stay within the halves' range (Numbers, above); 1 % for
// the products' rounding.
bool orth_in_range(double a, double b, double c, int steps)
{
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        s *= 1.01;
        if (!(largest_poly(b, c, s * s) <= 15.0)) return false;
        const double next = largest_step(a, b, c, s);
        if (!(next <= 3.0)) return false;
        s = next;
    }
    return true;
}

}  // namespace gett

extern "C" {

void gett_orthogonalize_tiles(int64_t batch, int64_t rows, int64_t cols, struct gett_tiles out[3])
{
    using namespace gett;
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (small_fits(m, n)) {
        out[0] = out[1] = out[2] = {0, 1, 0, batch};
        return;
    }
    const auto put = [](const auto &c) -> gett_tiles {
        const int64_t edge[4] = {Big::BM, Mid::BM, Small::BM, kShortE};
        return {edge[c.shape], c.cut.slices, c.cut.shared(), c.cut.blocks};
    };
    out[0] = put(choose<kGram>(batch, m, m, panel_count(n)));
    out[1] = put(choose<kPoly>(batch, m, m, panel_count(m)));
    out[2] = put(choose<kUpdate>(batch, m, n, panel_count(m)));
}

gett_status_t gett_orthogonalize(gett_dtype_t dtype, int64_t batch, int64_t rows, int64_t cols,
                                 const void *G, int64_t stride_batch, int64_t stride_row,
                                 int64_t stride_col, double a, double b, double c, double eps,
                                 int steps, void *O, int64_t ostride_batch, int64_t ostride_row,
                                 int64_t ostride_col, void *stream)
{
    using namespace gett;
    if (!float_type(dtype) || batch < 0 || rows < 0 || cols < 0 || steps < 0 ||
        !(eps >= 0.0) || !(fabs(a) < INFINITY) || !(fabs(b) < INFINITY) ||
        !(fabs(c) < INFINITY) || stride_row < 1 || stride_col < 1 || ostride_row < 1 ||
        ostride_col < 1 || (batch > 1 && (stride_batch < 1 || ostride_batch < 1)))
        return GETT_ERROR_INVALID_VALUE;
    if (rows >= (1 << 20) || cols >= (1 << 20) || steps > 1000 || !orth_in_range(a, b, c, steps))
        return GETT_ERROR_NOT_SUPPORTED;
    if (batch == 0 || rows == 0 || cols == 0) return GETT_SUCCESS;
    if (batch >= INT32_MAX) return GETT_ERROR_NOT_SUPPORTED;
    const int64_t item = type_size(dtype);
    if (!G || !O || (uintptr_t)G % item || (uintptr_t)O % item) return GETT_ERROR_INVALID_VALUE;
    if (batch == 1) stride_batch = ostride_batch = 1;
    const int64_t oneG = span_bytes(rows, cols, stride_row, stride_col, item);
    const int64_t oneO = span_bytes(rows, cols, ostride_row, ostride_col, item);
    if (oneG < 0 || oneO < 0) return GETT_ERROR_NOT_SUPPORTED;
    // matrices of the stack as one more direction
    const int64_t spanG = span_bytes(batch, oneG / item, stride_batch, 1, item);
    const int64_t spanO = span_bytes(batch, oneO / item, ostride_batch, 1, item);
    if (spanG < 0 || spanO < 0) return GETT_ERROR_NOT_SUPPORTED;
    // (matrices may interleave, as the column slices of a weight's heads do)
    const int64_t extents[3] = {batch, rows, cols};
    const int64_t strides[3] = {ostride_batch, ostride_row, ostride_col};
    try {   // (it takes a little host memory)
        if (!strides_injective(3, extents, strides)) return GETT_ERROR_NOT_SUPPORTED;
    } catch (...) {
        return GETT_ERROR_ALLOC;
    }
    const bool same = G == O && stride_row == ostride_row && stride_col == ostride_col &&
                      stride_batch == ostride_batch;
    if (!same && overlaps(G, spanG, O, spanO)) return GETT_ERROR_INVALID_VALUE;

    Problem P = {batch, (int)rows, (int)cols, a, b, c, eps, steps, static_cast<hipStream_t>(stream)};
    if (rows > cols) {   // the shorter side as rows
        std::swap(P.m, P.n);
        std::swap(stride_row, stride_col);
        std::swap(ostride_row, ostride_col);
    }
    if (dtype == GETT_FLOAT32)
        return orthogonalize_typed<float>(
            P, {static_cast<const float *>(G), stride_batch, stride_row, stride_col},
            {static_cast<float *>(O), ostride_batch, ostride_row, ostride_col});
    if (dtype == GETT_FLOAT16)
        return orthogonalize_typed<_Float16>(
            P, {static_cast<const _Float16 *>(G), stride_batch, stride_row, stride_col},
            {static_cast<_Float16 *>(O), ostride_batch, ostride_row, ostride_col});
    return orthogonalize_typed<bf16>(
        P, {static_cast<const bf16 *>(G), stride_batch, stride_row, stride_col},
        {static_cast<bf16 *>(O), ostride_batch, ostride_row, ostride_col});
}

}  // extern "C"
