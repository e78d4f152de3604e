// orth.hip -- Newton-Schulz orthogonalisation of a stack of matrices.
//
//     X_0 = G / (|G| + eps);   S = X X^T;   B = b S + c S^2;   X <- a X + B X
//
// X is held with its shorter side as rows (m <= n), so S and B are m x m.
// Bound: matrix instructions, 2 m n + 4 m (m + n) ... per step; S and S^2 are
// symmetric, so only the tiles on and below the diagonal are computed and the
// others mirrored: m^2 n + m^3 + 2 m^2 n multiplications' flops per step
// instead of 2 m^2 n + 2 m^3 + 2 m^2 n.
//
// Numbers.  |X| <= 1 at the start and every singular value stays below 3
// (gett_orthogonalize refuses other polynomials), so all entries of X, S and
// B are below 15 and fit a half after multiplication by 2^12, which keeps
// entries down to 2^-26 normal.  A float matrix is held as two halves, hi +
// lo (22 bits; products in panel.hpp, sums in 32 bits): the result is as close
// to the 64-bit one as that of products in 32 bits (1.5e-6 of its norm for
// both at 512 x 517) at a fifth of their price.  For bf16 one half is held:
// 1.3e-3 of the norm, below the 1.7e-3 that rounding the result to bf16
// costs anyway.
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
constexpr int kNormBlocks = 256;   // at most, per matrix; one partial sum each

// ----------------------------------------------------------------- storage ---

// Numbers of one panel: Half 64 halves; Split 32, the high parts of eight
// numbers and then their low parts (slab 0 takes the even pieces of a panel,
// slab 1 the odd ones).
template <int KIND> __host__ __device__ inline int panel_elements() { return KIND == kPanelSplit ? 32 : 64; }
template <int KIND> inline int64_t panel_count(int64_t k)
{
    const int e = panel_elements<KIND>();
    return (k + e - 1) / e;
}
// columns of a row, padding included
template <int KIND> __host__ __device__ inline int padded(int k)
{
    const int e = panel_elements<KIND>();
    return (k + e - 1) / e * e;
}
// the byte of column k of a row in a matrix of `rows` rows
template <int KIND> __device__ __forceinline__ int64_t at(int rows, int row, int k)
{
    const int e = panel_elements<KIND>(), in = k % e;
    return ((int64_t)(k / e) * rows + row) * 128 +
           (KIND == kPanelSplit ? (in >> 3) * 32 + (in & 7) * 2 : in * 2);
}

// N neighbours (N divides 8 and the column): held values are 2^12 x
template <int KIND, int N> __device__ __forceinline__ void store_run(char *p, const float *v)
{
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    vec hi;
#pragma unroll
    for (int i = 0; i < N; ++i) hi[i] = (_Float16)v[i];
    *reinterpret_cast<vec *>(p) = hi;
    if constexpr (KIND == kPanelSplit) {
        vec lo;
#pragma unroll
        for (int i = 0; i < N; ++i) lo[i] = (_Float16)(v[i] - (float)hi[i]);
        *reinterpret_cast<vec *>(p + 16) = lo;
    }
}
template <int KIND, int N> __device__ __forceinline__ void load_run(const char *p, float *v)
{
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    const vec hi = *reinterpret_cast<const vec *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)hi[i];
    if constexpr (KIND == kPanelSplit) {
        const vec lo = *reinterpret_cast<const vec *>(p + 16);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += (float)lo[i];
    }
}

// ------------------------------------------------------------ norm and start ---

// A stack of matrices: element [i, k] of matrix z at z sb + i si + k sk
template <typename T> struct Stack {
    T *p;
    int64_t sb, si, sk;
};

__device__ __forceinline__ double block_sum(double v, double *lds)
{
    const int tid = (int)threadIdx.x;
    lds[tid] = v;
    __syncthreads();
#pragma unroll
    for (int n = kNormThreads / 2; n > 0; n >>= 1) {
        if (tid < n) lds[tid] += lds[tid + n];
        __syncthreads();
    }
    return lds[0];
}

// partial[z][block] = sum of squares of rows block, block + blocks, ... where
// `rows` is the direction of the larger stride
template <typename T>
__global__ __launch_bounds__(kNormThreads) void orth_norm_kernel(Stack<const T> G, int rows,
                                                                 int cols, int blocks,
                                                                 double *partial)
{
    __shared__ double lds[kNormThreads];
    const int z = (int)blockIdx.x / blocks, b = (int)blockIdx.x % blocks;
    const T *p = G.p + z * G.sb;
    double s = 0.0;
    for (int i = b; i < rows; i += blocks)
#pragma unroll 4
        for (int k = (int)threadIdx.x; k < cols; k += kNormThreads) {
            const double v = (double)to_float(p[i * G.si + k * G.sk]);
            s += v * v;
        }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partial[(int64_t)z * blocks + b] = s;
}

// X_0 in both orientations, a 64 x 64 tile a workgroup
constexpr int kStart = 64;
template <typename T, int KIND>
__global__ __launch_bounds__(kNormThreads) void orth_start_kernel(
    Stack<const T> G, int m, int n, int tilesM, int tilesN, const double *partial, int blocks,
    double eps, char *X, char *XT, int64_t stackX, int64_t stackXT)
{
    __shared__ double lds[kNormThreads];
    __shared__ float tile[kStart][kStart + 1];
    const int tid = (int)threadIdx.x;
    const int tiles = tilesM * tilesN, z = (int)blockIdx.x / tiles, t = (int)blockIdx.x % tiles;
    const int i0 = t / tilesN * kStart, k0 = t % tilesN * kStart;
    const double sum = block_sum(tid < blocks ? partial[(int64_t)z * blocks + tid] : 0.0, lds);
    // an infinity or a NaN anywhere makes the whole matrix NaN
    const double scale =
        sum < (double)INFINITY ? (double)kUp / (sqrt(sum) + eps) : (double)NAN;
    const T *g = G.p + z * G.sb;
    const bool along = G.sk <= G.si;   // neighbouring lanes take neighbours in memory
#pragma unroll 4
    for (int u = 0; u < kStart * kStart / kNormThreads; ++u) {
        const int e = u * kNormThreads + tid;
        const int a = e / kStart, b = e % kStart;
        const int i = along ? a : b, k = along ? b : a;
        float v = 0.0f;
        if (i0 + i < m && k0 + k < n)
            v = (float)((double)to_float(g[(i0 + i) * G.si + (k0 + k) * G.sk]) * scale);
        tile[i][k] = v;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kStart * kStart / 8 / kNormThreads; ++u) {
        const int e = u * kNormThreads + tid;
        const int a = e / (kStart / 8), c = e % (kStart / 8) * 8;
        float v[8];
        if (i0 + a < m && k0 + c < padded<KIND>(n)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[a][c + i];
            store_run<KIND, 8>(X + z * stackX + at<KIND>(m, i0 + a, k0 + c), v);
        }
        if (k0 + a < n && i0 + c < padded<KIND>(m)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[c + i][a];
            store_run<KIND, 8>(XT + z * stackXT + at<KIND>(n, k0 + a, i0 + c), v);
        }
    }
}

// O = X_0 (no steps)
template <typename T, int KIND>
__global__ __launch_bounds__(256) void orth_copy_kernel(const char *X, int64_t stackX, int m, int n,
                                                        Stack<T> O, int64_t total)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= total) return;
    const int64_t z = e / ((int64_t)m * n), rest = e % ((int64_t)m * n);
    const int i = (int)(rest / n), k = (int)(rest % n);
    float v;
    load_run<KIND, 1>(X + z * stackX + at<KIND>(m, i, k), &v);
    O.p[z * O.sb + i * O.si + k * O.sk] = from_float<T>(v * kDown);
}

// ---------------------------------------------------------------- products ---

enum Step { kGram, kPoly, kUpdate, kLast };

struct ProductArgs {
    const char *P, *Q;          // the operands, K along their rows
    int64_t stackP, stackQ;
    int m, n, panels;           // rows of P, rows of Q, panels of a row
    int tilesM, tilesN, tiles;  // tiles of one matrix
    const char *addend;         // Poly: S; Update, Last: X; [row][col] as `out`
    char *out, *outT;           // [row][col], and its transpose
    int64_t stackOut, stackOutT;
    float scale, factor;        // addend's and the product's factor
};

// The t-th tile on or below the diagonal, row by row.
__device__ __forceinline__ void triangle_tile(int t, int &tm, int &tn)
{
    tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
    while (tm * (tm + 1) / 2 > t) --tm;
    tn = t - tm * (tm + 1) / 2;
}

template <int KIND, int STEP, typename S, typename T>
__global__ __launch_bounds__(S::THREADS) void orth_product_kernel(ProductArgs d, Stack<T> O)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    constexpr int FM = S::FM, FN = S::FN;
    const int z = (int)blockIdx.x / d.tiles, t = (int)blockIdx.x % d.tiles;
    int tm, tn;
    constexpr bool kSymmetric = STEP == kGram || STEP == kPoly;
    if constexpr (kSymmetric) triangle_tile(t, tm, tn);
    else panel_tile(t, d.tilesM, d.tilesN, 4, tm, tn);
    const PanelOperand A = {reinterpret_cast<const uint8_t *>(d.P) + z * d.stackP, nullptr, d.m,
                            tm * S::BM};
    const PanelOperand B = {reinterpret_cast<const uint8_t *>(d.Q) + z * d.stackQ, nullptr, d.n,
                            tn * S::BN};
    Panel<KIND, S> p;
    p.init();
    p.run(dyn_lds, A, B, 0, d.panels);

    const int padN = padded<KIND>(d.n), padM = padded<KIND>(d.m);
    const int col = B.row0 + p.col(0);
    char *out = d.out + z * d.stackOut;
    const char *addend = STEP == kGram ? nullptr : d.addend + z * d.stackOut;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int row0 = A.row0 + p.row(0, e);   // FM neighbouring rows
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row = row0 + i;
            float x[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) x[j] = 0.0f;
            if constexpr (STEP != kGram)
                if (row < d.m && col < padN)
                    load_run<KIND, FN>(addend + at<KIND>(d.m, row, col), x);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                // rows and columns of the padding are zeros
                float v = d.factor * p.acc[i][j][e];
                if constexpr (STEP != kGram) v += d.scale * x[j];
                p.acc[i][j][e] = row < d.m && col + j < d.n ? v : 0.0f;
            }
            if constexpr (STEP != kLast) {
                float v[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) v[j] = p.acc[i][j][e];
                if (row < d.m && col < padN)
                    store_run<KIND, FN>(out + at<KIND>(d.m, row, col), v);
            } else if (O.si != 1 || O.sk == 1) {
                T *o = O.p + z * O.sb + row * O.si + col * O.sk;
                if (row < d.m && O.sk == 1 && col + FN <= d.n) {
                    Run<T, FN> v;
#pragma unroll
                    for (int j = 0; j < FN; ++j) v.v[j] = from_float<T>(p.acc[i][j][e] * kDown);
                    *reinterpret_cast<Run<T, FN> *>(o) = v;
                } else if (row < d.m) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        if (col + j < d.n) o[j * O.sk] = from_float<T>(p.acc[i][j][e] * kDown);
                }
            }
        }
        // the other orientation: X^T, or the mirrored tile
        if constexpr (STEP != kLast) {
            if (!kSymmetric || tm != tn) {
                char *outT = d.outT + z * d.stackOutT;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    float v[FM];
#pragma unroll
                    for (int i = 0; i < FM; ++i) v[i] = p.acc[i][j][e];
                    if (col + j < d.n && row0 < padM)
                        store_run<KIND, FM>(outT + at<KIND>(d.n, col + j, row0), v);
                }
            }
        } else if (O.si == 1 && O.sk != 1) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if (col + j >= d.n) continue;
                T *o = O.p + z * O.sb + row0 + (int64_t)(col + j) * O.sk;
                if (row0 + FM <= d.m) {
                    Run<T, FM> v;
#pragma unroll
                    for (int i = 0; i < FM; ++i) v.v[i] = from_float<T>(p.acc[i][j][e] * kDown);
                    *reinterpret_cast<Run<T, FM> *>(o) = v;
                } else {
#pragma unroll
                    for (int i = 0; i < FM; ++i)
                        if (row0 + i < d.m) o[i] = from_float<T>(p.acc[i][j][e] * kDown);
                }
            }
        }
    }
}

template <int KIND, int STEP, typename S, typename T>
hipError_t product_launch(ProductArgs d, const Stack<T> &O, int64_t batch, hipStream_t stream)
{
    constexpr auto k = orth_product_kernel<KIND, STEP, S, T>;
    const hipError_t e = allow_dynamic_lds<k>(S::LDS);
    if (e != hipSuccess) return e;
    d.tilesM = (d.m + S::BM - 1) / S::BM;
    d.tilesN = (d.n + S::BN - 1) / S::BN;
    const int64_t tiles = STEP == kGram || STEP == kPoly ? (int64_t)d.tilesM * (d.tilesM + 1) / 2
                                                         : (int64_t)d.tilesM * d.tilesN;
    if (tiles * batch >= INT32_MAX) return hipErrorInvalidValue;
    d.tiles = (int)tiles;
    hipLaunchKernelGGL(k, dim3((unsigned)(tiles * batch)), dim3(S::THREADS), S::LDS, stream, d, O);
    return hipGetLastError();
}

// Square tiles (the symmetric products mirror them).
typedef PanelShape<2, 4, 4, 2> Big;
typedef PanelShape<2, 2, 2, 2> Mid;
typedef PanelShape<1, 1, 2, 2> Small;

template <int KIND, int STEP, typename T>
hipError_t product(const ProductArgs &d, const Stack<T> &O, int64_t batch, hipStream_t stream)
{
    auto tiles = [&](int64_t edge) {
        const int64_t tm = (d.m + edge - 1) / edge, tn = (d.n + edge - 1) / edge;
        return batch * (STEP == kGram || STEP == kPoly ? tm * (tm + 1) / 2 : tm * tn);
    };
    if (tiles(256) >= 256) return product_launch<KIND, STEP, Big, T>(d, O, batch, stream);
    if (tiles(128) >= 256) return product_launch<KIND, STEP, Mid, T>(d, O, batch, stream);
    return product_launch<KIND, STEP, Small, T>(d, O, batch, stream);
}

struct Problem {
    int64_t batch;
    int m, n;
    double a, b, c, eps;
    int steps;
    hipStream_t stream;
};

template <typename T, int KIND>
gett_status_t orthogonalize_typed(const Problem &P, Stack<const T> G, Stack<T> O)
{
    const int m = P.m, n = P.n;
    const int64_t panelsX = panel_count<KIND>(n), panelsS = panel_count<KIND>(m);
    const int64_t X = m * panelsX * 128, XT = n * panelsS * 128, SS = m * panelsS * 128;
    // the norm reads along the smaller stride
    const bool along = G.sk <= G.si;
    const int outer = along ? m : n, inner = along ? n : m;
    const int blocks = outer < kNormBlocks ? outer : kNormBlocks;
    const int64_t head = (P.batch * blocks * 8 + 255) / 256 * 256;
    const int64_t startM = (m + kStart - 1) / kStart, startN = (n + kStart - 1) / kStart;
    const int64_t copies = ((int64_t)m * n * P.batch + 255) / 256;
    if (P.batch * startM * startN >= INT32_MAX || P.batch * blocks >= INT32_MAX ||
        copies >= INT32_MAX)
        return GETT_ERROR_NOT_SUPPORTED;
    Partials w;
    const gett_status_t ws = stream_workspace(
        P.stream, 0, (uint64_t)(head + P.batch * (X + 2 * XT + 2 * SS)), w);
    if (ws != GETT_SUCCESS) return ws;
    double *partial = static_cast<double *>(w.tiles);
    char *x = static_cast<char *>(w.tiles) + head, *xt = x + P.batch * X;
    char *xt2 = xt + P.batch * XT, *s = xt2 + P.batch * XT, *poly = s + P.batch * SS;

    Stack<const T> g = G;
    if (!along) std::swap(g.si, g.sk);
    hipLaunchKernelGGL((orth_norm_kernel<T>), dim3((unsigned)(P.batch * blocks)),
                       dim3(kNormThreads), 0, P.stream, g, outer, inner, blocks, partial);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return GETT_ERROR_HIP;
    hipLaunchKernelGGL((orth_start_kernel<T, KIND>), dim3((unsigned)(P.batch * startM * startN)),
                       dim3(kNormThreads), 0, P.stream, G, m, n, (int)startM, (int)startN, partial,
                       blocks, P.eps, x, xt, X, XT);
    e = hipGetLastError();
    if (e != hipSuccess) return GETT_ERROR_HIP;
    if (P.steps == 0) {
        hipLaunchKernelGGL((orth_copy_kernel<T, KIND>), dim3((unsigned)copies), dim3(256), 0,
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
        e = product<KIND, kGram, T>(d, none, P.batch, P.stream);
        if (e != hipSuccess) return GETT_ERROR_HIP;
        d.P = d.Q = d.addend = s;
        d.stackP = d.stackQ = SS;
        d.panels = (int)panelsS;
        d.out = d.outT = poly;
        d.scale = (float)P.b;
        d.factor = (float)(P.c * kDown);
        e = product<KIND, kPoly, T>(d, none, P.batch, P.stream);
        if (e != hipSuccess) return GETT_ERROR_HIP;
        d.P = poly;
        d.Q = xt;
        d.stackQ = XT;
        d.n = n;
        d.addend = d.out = x;
        d.outT = xt2;
        d.stackOut = X;
        d.stackOutT = XT;
        d.scale = (float)P.a;
        d.factor = kDown;
        e = i + 1 < P.steps ? product<KIND, kUpdate, T>(d, none, P.batch, P.stream)
                            : product<KIND, kLast, T>(d, O, P.batch, P.stream);
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

// Singular values stay within the halves' range (orth.hip, Numbers); 1 % for
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
    if (!matrix_injective(rows, cols, ostride_row, ostride_col) ||
        (batch > 1 && (__int128)ostride_batch * item < oneO))
        return GETT_ERROR_NOT_SUPPORTED;
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
        return orthogonalize_typed<float, kPanelSplit>(
            P, {static_cast<const float *>(G), stride_batch, stride_row, stride_col},
            {static_cast<float *>(O), ostride_batch, ostride_row, ostride_col});
    if (dtype == GETT_FLOAT16)
        return orthogonalize_typed<_Float16, kPanelSplit>(
            P, {static_cast<const _Float16 *>(G), stride_batch, stride_row, stride_col},
            {static_cast<_Float16 *>(O), ostride_batch, ostride_row, ostride_col});
    return orthogonalize_typed<bf16, kPanelHalf>(
        P, {static_cast<const bf16 *>(G), stride_batch, stride_row, stride_col},
        {static_cast<bf16 *>(O), ostride_batch, ostride_row, ostride_col});
}

}  // extern "C"
