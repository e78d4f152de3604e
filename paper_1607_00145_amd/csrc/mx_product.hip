// mx_product.hip -- products of packed 4-bit matrices,
//     C[m, n] <- alpha * sum_k A[m, k] B[n, k] + beta * C[m, n],
// and of float rows, quantised on the way, with a packed matrix.
//
// Many rows: tiles of C, the operands' panels through LDS (panel.hpp).  Bound:
// the matrix units, busy for 54 % of the cycles of a clock that falls to 1.74 GHz;
// 8192 x 8192 x 8192 into bf16 takes 253-263 us by card (4.2-4.3 PFLOP/s; the
// instructions alone, on random operands in registers, reach 6.2).  Between few
// rows and large tiles, tiles of 64 x 64 take their panels one after the other, on
// few CUs: 48 x 1024 x 8192 12.9 us, 64 x 8192 x 4096 8.9.  A tile's results go out as they lie, FN neighbours
// a lane.
// Few rows (up to 32): bound by B's bytes, and below some 16 MB of them by the
// launch and two memory latencies.  A workgroup takes 32 rows of B (32 columns
// of C) and its wavefronts every eighth panel; B goes from memory straight
// into the registers that the MFMA reads (a lane's two pieces of a panel are
// 32 bytes of one row), so no byte waits for a barrier, and the eight partial
// results are summed in wavefront order through LDS.  8192 x 4096 (17.8 MB)
// with 16 packed rows takes 5.4 us (as tiles 7.6), with 32 rows 6.6 (8.0),
// with one bf16 row packed on its way 6.6.
#include "launch.hpp"
#include "matrix.hpp"
#include "mx.hpp"
#include "panel.hpp"

namespace gett {

namespace {

template <typename T> struct Result {
    T *C;
    int64_t sm, sn;
    int m, n;
    float alpha, beta;
};

// N neighbouring columns of one row: alpha * sum + beta * C, rounded once
template <typename T, int N>
__device__ __forceinline__ void store_row(const Result<T> &o, int row, int col, const float *sum)
{
    if (row >= o.m || col >= o.n) return;
    T *p = o.C + (int64_t)row * o.sm + (int64_t)col * o.sn;
    if (o.sn == 1 && col + N <= o.n) {
        Run<T, N> v;
        if (o.beta != 0.0f) {
            const Run<T, N> c = *reinterpret_cast<const Run<T, N> *>(p);
#pragma unroll
            for (int i = 0; i < N; ++i)
                v.v[i] = from_float<T>(o.alpha * sum[i] + o.beta * to_float(c.v[i]));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v.v[i] = from_float<T>(o.alpha * sum[i]);
        }
        *reinterpret_cast<Run<T, N> *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i < o.n) {
                float v = o.alpha * sum[i];
                if (o.beta != 0.0f) v += o.beta * to_float(p[i * o.sn]);
                p[i * o.sn] = from_float<T>(v);
            }
    }
}

// ------------------------------------------------------------------- tiles ---

// One product: its operands, its share of the launch and its result.
template <typename T> struct TileJob {
    PanelOperand A, B;
    PanelGrid grid;
    Result<T> o;
    int blocks;
};

// Workgroups of the first product, then those of the second (if there is one).
template <typename T, typename S>
__global__ __launch_bounds__(S::THREADS) void mx_tile_kernel(TileJob<T> first, TileJob<T> second)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    const bool is2 = (int)blockIdx.x >= first.blocks;
    PanelOperand A = is2 ? second.A : first.A, B = is2 ? second.B : first.B;
    const PanelGrid grid = is2 ? second.grid : first.grid;
    const Result<T> o = is2 ? second.o : first.o;
    int tm, tn;
    const PanelItem w = panel_item(grid, (int)blockIdx.x - (is2 ? first.blocks : 0));
    panel_tile(grid, w.tile, tm, tn);
    A.row0 = tm * S::BM;
    B.row0 = tn * S::BN;
    Panel<kPanelMx, S> p;
    p.init();
    p.run(dyn_lds, A, B, w.t0, w.t1);
    __syncthreads();
    if (!panel_join<kPanelMx, S>(p, grid, w, dyn_lds)) return;
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            float v[S::FN];
#pragma unroll
            for (int j = 0; j < S::FN; ++j) v[j] = p.acc[i][j][e];
            store_row<T, S::FN>(o, A.row0 + p.row(i, e), B.row0 + p.col(0), v);
        }
}

typedef PanelShape<2, 4, 4, 2, 2> Big;
typedef PanelShape<2, 2, 2, 2, 2> Mid;
typedef PanelShape<1, 1, 2, 2, 4> Small;

struct TilePlan {
    int shape;   // 0 Big, 1 Mid, 2 Small
    PanelCut cut;
    int64_t slotBytes, counters;
};

template <typename S>
void consider(TilePlan &best, int shape, int64_t m, int64_t n, int64_t panels)
{
    const int64_t tiles = ((m + S::BM - 1) / S::BM) * ((n + S::BN - 1) / S::BN);
    const PanelCut c = panel_cut<S>(kPanelMx, tiles, panels);
    if (shape == 0 || c.us < best.cut.us)
        best = {shape, c, c.shared() * c.slices * S::TILE * 4, c.shared()};
}

TilePlan tile_plan(int64_t m, int64_t n, int64_t panels)
{
    TilePlan p;
    consider<Big>(p, 0, m, n, panels);
    consider<Mid>(p, 1, m, n, panels);
    consider<Small>(p, 2, m, n, panels);
    return p;
}

template <typename T, typename S> hipError_t tile_launch(const TileJob<T> *j, int n, hipStream_t stream)
{
    constexpr auto k = mx_tile_kernel<T, S>;
    const hipError_t e = allow_dynamic_lds<k>(S::lds(kPanelMx));
    if (e != hipSuccess) return e;
    TileJob<T> none = {};
    const int64_t blocks = (int64_t)j[0].blocks + (n == 2 ? j[1].blocks : 0);
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(S::THREADS), S::lds(kPanelMx), stream, j[0],
                       n == 2 ? j[1] : none);
    return hipGetLastError();
}

// ---------------------------------------------------------------- few rows ---

constexpr int kFewWaves = 8;
constexpr int kFewCols = 32;

// A's side of one panel: FM fragments of two pieces, and their scales
template <int FM> struct FewPacked {
    const uint8_t *codes, *scales;
    int m;
    struct Frag {
        i4 v[FM][2];
        int s[FM];   // the scales of both pieces in the low 16 bits
    };
    __device__ __forceinline__ void load(Frag &f, int t, int r, int q) const
    {
        const int64_t R = mx_scale_rows(m);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row = FM * r + i < m ? FM * r + i : m - 1;
            const i4 *p =
                reinterpret_cast<const i4 *>(codes + ((int64_t)t * m + row) * kTileBytes + q * 32);
            f.v[i][0] = p[0];
            f.v[i][1] = p[1];
            f.s[i] = *reinterpret_cast<const uint16_t *>(
                scales + ((t * 2 + (q >> 1)) * R + row) * 4 + (q & 1) * 2);
        }
    }
};

// the same from float rows, one per lane r (FM is 1): each lane packs two
// blocks of 32 neighbours of its row
template <typename TA> struct FewFloat {
    const TA *A;
    int64_t sm, sk;
    int m, k;
    struct Frag {
        i4 v[1][2];
        int s[1];
    };
    __device__ __forceinline__ void load(Frag &f, int t, int r, int q) const
    {
        f.s[0] = 0;
        f.v[0][0] = f.v[0][1] = i4{0, 0, 0, 0};
        if (r >= m) return;
        const int k0 = t * kTileK + q * 64;
        const TA *p = A + (int64_t)r * sm + (int64_t)k0 * sk;
        if (sk == 1 && (t + 1) * kTileK <= k) {   // the same for all lanes
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float x[32];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const Run<TA, 8> v = *reinterpret_cast<const Run<TA, 8> *>(p + 32 * b + 8 * c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[8 * c + i] = to_float(v.v[i]);
                }
                pack(f, b, x);
            }
        } else {
            // element by element, columns past the last read as the last and
            // replaced: no branches, so that a block's loads go out together
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
                const int left = k - (k0 + 32 * b) - 1;   // the last column's place
                if (left < 0) break;                      // (zeros)
                const TA *q = p + 32 * b * sk;
                TA v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = q[(i < left ? i : left) * sk];
                float x[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = i <= left ? to_float(v[i]) : 0.0f;
                if (b == 0) pack(f, 0, x);
                else pack(f, 1, x);
            }
        }
    }
    static __device__ __forceinline__ void pack(Frag &f, int b, const float *x)
    {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        const uint32_t sb = scale_byte(top);
        const float s = scale_value(sb);
#pragma unroll
        for (int c = 0; c < 4; ++c) f.v[0][b][c] = (int)codes8(x + 8 * c, s);
        f.s[0] |= (int)(sb << (8 * b));
    }
};

// DEEP: panels of a wavefront whose loads are in flight together
template <typename T, typename LA, int FM, int DEEP>
__global__ __launch_bounds__(kFewWaves * 64) void mx_few_kernel(LA A, const uint8_t *codesB,
                                                               const uint8_t *scalesB, int panels,
                                                               Result<T> o)
{
    constexpr int FN = 2;
    __shared__ f4 part[kFewWaves][FM * FN][64];
    const int tid = (int)threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col0 = (int)blockIdx.x * kFewCols;
    const int64_t R = mx_scale_rows(o.n);
    const uint8_t *pb[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int row = col0 + FN * r + j < o.n ? col0 + FN * r + j : o.n - 1;
        pb[j] = codesB + (int64_t)row * kTileBytes + q * 32;
    }
    const int64_t rs = col0 + FN * r < R ? col0 + FN * r : R - FN;
    f4 acc[FM][FN] = {};
    for (int t0 = wave; t0 < panels; t0 += kFewWaves * DEEP) {
        i4 b[DEEP][FN][2];
        f2 sb[DEEP];   // a word of four scales per row
        typename LA::Frag a[DEEP];
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
            const int t = t0 + u * kFewWaves;
            if (t < panels) {
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const i4 *p = reinterpret_cast<const i4 *>(pb[j] + (int64_t)t * o.n * kTileBytes);
                    b[u][j][0] = p[0];
                    b[u][j][1] = p[1];
                }
                sb[u] = *reinterpret_cast<const f2 *>(scalesB + ((t * 2 + (q >> 1)) * R + rs) * 4);
            }
        }
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
            const int t = t0 + u * kFewWaves;
            if (t < panels) A.load(a[u], t, r, q);
        }
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
            if (t0 + u * kFewWaves >= panels) break;
            // this lane group's two scales of the word
            const int s0 = (int)(__float_as_uint(sb[u][0]) >> ((q & 1) * 16));
            const int s1 = (int)(__float_as_uint(sb[u][1]) >> ((q & 1) * 16));
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                acc[i][0] = mfma_mx16<0, 0>(a[u].v[i][0], b[u][0][0], acc[i][0], a[u].s[i], s0);
                acc[i][0] = mfma_mx16<1, 1>(a[u].v[i][1], b[u][0][1], acc[i][0], a[u].s[i], s0);
                acc[i][1] = mfma_mx16<0, 0>(a[u].v[i][0], b[u][1][0], acc[i][1], a[u].s[i], s1);
                acc[i][1] = mfma_mx16<1, 1>(a[u].v[i][1], b[u][1][1], acc[i][1], a[u].s[i], s1);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) part[wave][i * FN + j][lane] = acc[i][j];
    __syncthreads();
    // wavefront w sums fragment rows w, w + 8, ...
    for (int i = wave; i < FM; i += kFewWaves) {
        f4 s[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            s[j] = part[0][i * FN + j][lane];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) s[j] += part[w][i * FN + j][lane];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v[FN] = {s[0][e], s[1][e]};
            store_row<T, FN>(o, FM * (4 * q + e) + i, col0 + FN * r, v);
        }
    }
}

template <typename T, typename LA, int FM>
hipError_t few_launch(const LA &A, const void *codesB, const void *scalesB, int panels,
                      const Result<T> &o, hipStream_t stream)
{
    const unsigned blocks = (unsigned)((o.n + kFewCols - 1) / kFewCols);
    const uint8_t *cb = static_cast<const uint8_t *>(codesB);
    const uint8_t *sb = static_cast<const uint8_t *>(scalesB);
    hipLaunchKernelGGL((mx_few_kernel<T, LA, FM, 2>), dim3(blocks), dim3(kFewWaves * 64), 0,
                       stream, A, cb, sb, panels, o);
    return hipGetLastError();
}

struct Packed {
    const void *codes, *scales;
    int64_t rows;
};

// A product of m x k by n x k: operands (exchanged where C's neighbours lie
// along m: C^T = B A^T), result and plan; few rows need no tiles.  The plan
// depends on sizes and strides alone: a call whose operands go to the workspace
// makes its products without pointers, to size it, and then again with them.
struct Product {
    Packed A, B;
    int64_t k;
    void *C;
    int64_t sm, sn;
    bool few;
    TilePlan plan;
};
Product product_of(Packed A, Packed B, int64_t k, void *C, int64_t sm, int64_t sn)
{
    Product p = {A, B, k, C, sm, sn, false, {}};
    if (sm == 1 && sn != 1) {
        std::swap(p.A, p.B);
        std::swap(p.sm, p.sn);
    }
    p.few = k > 0 && p.A.rows <= 32;
    if (!p.few) p.plan = tile_plan(p.A.rows, p.B.rows, mx_tiles(k));
    return p;
}

template <typename T> Result<T> result(const Product &p, double alpha, double beta)
{
    return {static_cast<T *>(p.C), p.sm, p.sn, (int)p.A.rows, (int)p.B.rows, (float)alpha,
            (float)beta};
}

template <typename T>
hipError_t few_packed(const Product &p, double alpha, double beta, hipStream_t stream)
{
    const int panels = (int)mx_tiles(p.k), m = (int)p.A.rows;
    const uint8_t *ca = static_cast<const uint8_t *>(p.A.codes);
    const uint8_t *sa = static_cast<const uint8_t *>(p.A.scales);
    const Result<T> o = result<T>(p, alpha, beta);
    return m <= 16 ? few_launch<T, FewPacked<1>, 1>({ca, sa, m}, p.B.codes, p.B.scales, panels, o, stream)
                   : few_launch<T, FewPacked<2>, 2>({ca, sa, m}, p.B.codes, p.B.scales, panels, o, stream);
}

// One or two products of one result type; slots for shared sums lie at `slots`
// (the second product's behind the first's), counters likewise.
template <typename T>
hipError_t contract_typed(const Product *p, int n, float *slots, int *counters, double alpha,
                          double beta, hipStream_t stream)
{
    TileJob<T> jobs[2];
    for (int i = 0; i < n; ++i) {
        if (p[i].few) {
            const hipError_t e = few_packed<T>(p[i], alpha, beta, stream);
            if (e != hipSuccess) return e;
            continue;
        }
        const TilePlan &plan = p[i].plan;
        const int64_t edge = plan.shape == 0 ? Big::BM : plan.shape == 1 ? Mid::BM : Small::BM;
        const int64_t tm = (p[i].A.rows + edge - 1) / edge, tn = (p[i].B.rows + edge - 1) / edge;
        TileJob<T> &j = jobs[i];
        j.A = {static_cast<const uint8_t *>(p[i].A.codes),
               static_cast<const uint8_t *>(p[i].A.scales), (int)p[i].A.rows, 0};
        j.B = {static_cast<const uint8_t *>(p[i].B.codes),
               static_cast<const uint8_t *>(p[i].B.scales), (int)p[i].B.rows, 0};
        j.o = result<T>(p[i], alpha, beta);
        j.blocks = (int)plan.cut.blocks;
        if (!panel_grid(j.grid, 1, tm, tn, tm * tn, plan.cut, (int)mx_tiles(p[i].k), slots, counters))
            return hipErrorInvalidValue;
        slots += plan.slotBytes / 4;
        counters += plan.counters;
    }
    auto launch = [&](const TileJob<T> *j, int count, int shape) {
        return shape == 0   ? tile_launch<T, Big>(j, count, stream)
               : shape == 1 ? tile_launch<T, Mid>(j, count, stream)
                            : tile_launch<T, Small>(j, count, stream);
    };
    if (n == 2 && !p[0].few && !p[1].few && p[0].plan.shape == p[1].plan.shape &&
        fits_launch((int64_t)jobs[0].blocks + jobs[1].blocks, Big::THREADS))
        return launch(jobs, 2, p[0].plan.shape);
    for (int i = 0; i < n; ++i)
        if (!p[i].few) {
            const hipError_t e = launch(jobs + i, 1, p[i].plan.shape);
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

gett_status_t contract_launch(const Product *p, int n, float *slots, int *counters, double alpha,
                              double beta, gett_dtype_t dtype, hipStream_t stream)
{
    const hipError_t e =
        dtype == GETT_FLOAT32    ? contract_typed<float>(p, n, slots, counters, alpha, beta, stream)
        : dtype == GETT_BFLOAT16 ? contract_typed<bf16>(p, n, slots, counters, alpha, beta, stream)
                                 : contract_typed<_Float16>(p, n, slots, counters, alpha, beta, stream);
    return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
}

// Whether a product goes into one launch.
bool launchable(const Product &p)
{
    if (p.few) return fits_launch((p.B.rows + kFewCols - 1) / kFewCols, kFewWaves * 64);
    const int64_t edge = p.plan.shape == 0 ? Big::BM : p.plan.shape == 1 ? Mid::BM : Small::BM;
    const int64_t tm = (p.A.rows + edge - 1) / edge, tn = (p.B.rows + edge - 1) / edge;
    PanelGrid g;
    return panel_grid(g, 1, tm, tn, tm * tn, p.plan.cut, (int)mx_tiles(p.k), nullptr, nullptr) &&
           fits_launch(p.plan.cut.blocks, p.plan.shape == 0 ? Big::THREADS : Mid::THREADS);
}

// The stream's workspace for a call: `before` bytes of its own, then the slots
// of its products; refused, before anything is enqueued, where a product has too
// many tiles for a launch.
gett_status_t product_workspace(const Product *p, int n, int64_t before, hipStream_t stream,
                                Partials &w)
{
    int64_t bytes = before, counters = 0;
    for (int i = 0; i < n; ++i) {
        if (!launchable(p[i])) return GETT_ERROR_NOT_SUPPORTED;
        bytes += p[i].plan.slotBytes;
        counters += p[i].plan.counters;
    }
    return bytes == 0 ? GETT_SUCCESS
                      : stream_workspace(stream, (uint64_t)counters, (uint64_t)bytes, w);
}
float *slots_of(const Partials &w, int64_t before)
{
    return reinterpret_cast<float *>(static_cast<char *>(w.tiles) + before);
}

// the whole call: one product of packed operands
gett_status_t contract(const Packed &A, const Packed &B, int64_t k, double alpha, double beta,
                       gett_dtype_t dtype, void *C, int64_t sm, int64_t sn, hipStream_t stream)
{
    const Product p = product_of(A, B, k, C, sm, sn);
    Partials w;
    const gett_status_t ws = product_workspace(&p, 1, 0, stream, w);
    if (ws != GETT_SUCCESS) return ws;
    return contract_launch(&p, 1, slots_of(w, 0), w.counters, alpha, beta, dtype, stream);
}

template <typename TA, typename T>
hipError_t few_float(const void *A, int64_t sam, int64_t sak, int64_t k, Packed B,
                     const Result<T> &o, hipStream_t stream)
{
    const FewFloat<TA> a = {static_cast<const TA *>(A), sam, sak, o.m, (int)k};
    return few_launch<T, FewFloat<TA>, 1>(a, B.codes, B.scales, (int)mx_tiles(k), o, stream);
}
template <typename T>
hipError_t few_float_of(gett_dtype_t dtypeA, const void *A, int64_t sam, int64_t sak, int64_t k,
                        Packed B, const Result<T> &o, hipStream_t stream)
{
    if (dtypeA == GETT_FLOAT32) return few_float<float, T>(A, sam, sak, k, B, o, stream);
    if (dtypeA == GETT_BFLOAT16) return few_float<bf16, T>(A, sam, sak, k, B, o, stream);
    return few_float<_Float16, T>(A, sam, sak, k, B, o, stream);
}

// Whether a float A of m rows is packed inside its product with an n x k B:
// every workgroup then packs all of A again, but a launch is saved.  us in
// one launch and in two, bf16: 8192 x 4096, 1 row 6.6 / 7.4, 16 rows 8.2 /
// 8.6; 515 x 1000, 1 row 5.5 / 6.8; 2048 x 2048, 16 rows 5.2 / 6.9; 8192 x
// 8192, 8 rows 11.9 / 12.4, 12 rows 13.3 / 12.7, 16 rows 14.6 / 13.0.
bool packs_inside(int64_t m, int64_t n, int64_t k)
{
    return m <= 8 || (m <= 16 && n * k <= (int64_t)1 << 25);
}

template <typename T>
Result<T> few_result(void *C, int64_t sm, int64_t sn, int64_t m, int64_t n, double alpha, double beta)
{
    return {static_cast<T *>(C), sm, sn, (int)m, (int)n, (float)alpha, (float)beta};
}

// C's arguments; `C` may be null where C is empty
gett_status_t result_ok(int64_t m, int64_t n, int64_t k, gett_dtype_t dtype, const void *C,
                        int64_t sm, int64_t sn)
{
    if (!float_type(dtype) || m < 0 || n < 0 || k < 0 || sm < 1 || sn < 1)
        return GETT_ERROR_INVALID_VALUE;
    if (m >= kMaxRows || n >= kMaxRows || k >= kMaxCols) return GETT_ERROR_NOT_SUPPORTED;
    if (m == 0 || n == 0) return GETT_SUCCESS;
    if (!C || (uintptr_t)C % type_size(dtype)) return GETT_ERROR_INVALID_VALUE;
    if (span_bytes(m, n, sm, sn, type_size(dtype)) < 0 || !matrix_injective(m, n, sm, sn))
        return GETT_ERROR_NOT_SUPPORTED;
    return GETT_SUCCESS;
}

bool clear_of(const void *C, int64_t bytesC, const void *codes, const void *scales, int64_t rows,
              int64_t k)
{
    return !overlaps(C, bytesC, codes, mx_code_bytes(rows, k)) &&
           !overlaps(C, bytesC, scales, mx_scale_bytes(rows, k));
}

}  // namespace
}  // namespace gett

extern "C" {

void gett_mx_tiles(int64_t m, int64_t n, int64_t k, struct gett_tiles *out)
{
    using namespace gett;
    const Product p = product_of({nullptr, nullptr, m}, {nullptr, nullptr, n}, k, nullptr, n, 1);
    const PanelCut &c = p.plan.cut;
    if (p.few) *out = {0, 1, 0, (n + kFewCols - 1) / kFewCols};
    else *out = {p.plan.shape == 0 ? Big::BM : p.plan.shape == 1 ? Mid::BM : Small::BM, c.slices,
                 c.shared(), c.blocks};
}

gett_status_t gett_mx_contract(int64_t m, int64_t n, int64_t k, double alpha,
                               const void *codes_A, const void *scales_A, const void *codes_B,
                               const void *scales_B, double beta, gett_dtype_t dtype, void *C,
                               int64_t stride_m, int64_t stride_n, void *stream)
{
    using namespace gett;
    const gett_status_t st = result_ok(m, n, k, dtype, C, stride_m, stride_n);
    if (st != GETT_SUCCESS || m == 0 || n == 0) return st;
    if (alpha == 0.0) k = 0;
    if (k > 0) {
        if (!packed_ok(codes_A, scales_A) || !packed_ok(codes_B, scales_B))
            return GETT_ERROR_INVALID_VALUE;
        const int64_t bytes = span_bytes(m, n, stride_m, stride_n, type_size(dtype));
        if (!clear_of(C, bytes, codes_A, scales_A, m, k) ||
            !clear_of(C, bytes, codes_B, scales_B, n, k))
            return GETT_ERROR_INVALID_VALUE;
    }
    return contract({codes_A, scales_A, m}, {codes_B, scales_B, n}, k, alpha, beta, dtype, C,
                    stride_m, stride_n, static_cast<hipStream_t>(stream));
}

gett_status_t gett_mx_apply(int64_t m, int64_t n, int64_t k, double alpha, gett_dtype_t dtype_A,
                            const void *A, int64_t stride_am, int64_t stride_ak,
                            const void *codes_B, const void *scales_B, double beta,
                            gett_dtype_t dtype, void *C, int64_t stride_m, int64_t stride_n,
                            void *stream)
{
    using namespace gett;
    if (!float_type(dtype_A) || stride_am < 1 || stride_ak < 1) return GETT_ERROR_INVALID_VALUE;
    const gett_status_t st = result_ok(m, n, k, dtype, C, stride_m, stride_n);
    if (st != GETT_SUCCESS || m == 0 || n == 0) return st;
    if (alpha == 0.0) k = 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (k == 0)
        return contract({nullptr, nullptr, m}, {nullptr, nullptr, n}, 0, 0.0, beta, dtype, C, stride_m,
                        stride_n, s);
    if (!A || (uintptr_t)A % type_size(dtype_A) || !packed_ok(codes_B, scales_B))
        return GETT_ERROR_INVALID_VALUE;
    const int64_t bytesA = span_bytes(m, k, stride_am, stride_ak, type_size(dtype_A));
    const int64_t bytesC = span_bytes(m, n, stride_m, stride_n, type_size(dtype));
    if (bytesA < 0) return GETT_ERROR_NOT_SUPPORTED;
    if (overlaps(C, bytesC, A, bytesA) || !clear_of(C, bytesC, codes_B, scales_B, n, k))
        return GETT_ERROR_INVALID_VALUE;
    if (packs_inside(m, n, k)) {
        if (!fits_launch((n + kFewCols - 1) / kFewCols, kFewWaves * 64)) return GETT_ERROR_NOT_SUPPORTED;
        const Packed W = {codes_B, scales_B, n};
        hipError_t e;
        if (dtype == GETT_FLOAT32)
            e = few_float_of<float>(dtype_A, A, stride_am, stride_ak, k, W,
                                    few_result<float>(C, stride_m, stride_n, m, n, alpha, beta), s);
        else if (dtype == GETT_BFLOAT16)
            e = few_float_of<bf16>(dtype_A, A, stride_am, stride_ak, k, W,
                                   few_result<bf16>(C, stride_m, stride_n, m, n, alpha, beta), s);
        else
            e = few_float_of<_Float16>(dtype_A, A, stride_am, stride_ak, k, W,
                                       few_result<_Float16>(C, stride_m, stride_n, m, n, alpha, beta),
                                       s);
        return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
    }
    // A's packed copy and the slots of shared sums, in the stream's workspace.
    // The hold lasts until both launches are enqueued.
    const int64_t codeBytes = mx_code_bytes(m, k), packed = codeBytes + mx_scale_bytes(m, k);
    const Packed B = {codes_B, scales_B, n};
    Product p = product_of({nullptr, nullptr, m}, B, k, C, stride_m, stride_n);
    Partials w;
    gett_status_t ws = product_workspace(&p, 1, packed, s, w);
    if (ws != GETT_SUCCESS) return ws;
    char *codes = static_cast<char *>(w.tiles), *scales = codes + codeBytes;
    p = product_of({codes, scales, m}, B, k, C, stride_m, stride_n);
    const QuantizeJob q = {m, k, A, stride_am, stride_ak, codes, scales, nullptr, nullptr};
    ws = quantize_launch(dtype_A, &q, 1, s);
    if (ws != GETT_SUCCESS) return ws;
    return contract_launch(&p, 1, slots_of(w, packed), w.counters, alpha, beta, dtype, s);
}

gett_status_t gett_mx_linear(int64_t m, int64_t n, int64_t k, gett_dtype_t dtype_X, const void *X,
                             int64_t stride_xm, int64_t stride_xk, gett_dtype_t dtype_W,
                             const void *W, int64_t stride_wn, int64_t stride_wk, void *Y,
                             int64_t stride_ym, int64_t stride_yn, void *codes_xt,
                             void *scales_xt, void *codes_wt, void *scales_wt, void *stream)
{
    using namespace gett;
    gett_status_t st = matrix_ok(dtype_X, m, k, X, stride_xm, stride_xk);
    if (st == GETT_SUCCESS) st = matrix_ok(dtype_W, n, k, W, stride_wn, stride_wk);
    if (st == GETT_SUCCESS) st = result_ok(m, n, k, dtype_X, Y, stride_ym, stride_yn);
    if (st != GETT_SUCCESS) return st;
    const bool xt = codes_xt || scales_xt, wt = codes_wt || scales_wt;
    if ((xt && !packed_ok(codes_xt, scales_xt)) || (wt && !packed_ok(codes_wt, scales_wt)))
        return GETT_ERROR_INVALID_VALUE;
    if ((xt && m >= kMaxCols) || (wt && n >= kMaxCols)) return GETT_ERROR_NOT_SUPPORTED;
    // every output clear of the inputs and of the other outputs
    struct Range {
        const void *p;
        int64_t n;
    };
    auto whole = [](gett_dtype_t t, int64_t r, int64_t c, const void *p, int64_t sr, int64_t sc) {
        return Range{r > 0 && c > 0 ? p : nullptr, r > 0 && c > 0 ? span_bytes(r, c, sr, sc, type_size(t)) : 0};
    };
    const Range out[5] = {whole(dtype_X, m, n, Y, stride_ym, stride_yn),
                          {codes_xt, mx_code_bytes(k, m)}, {scales_xt, mx_scale_bytes(k, m)},
                          {codes_wt, mx_code_bytes(k, n)}, {scales_wt, mx_scale_bytes(k, n)}};
    const Range in[2] = {whole(dtype_X, m, k, X, stride_xm, stride_xk),
                         whole(dtype_W, n, k, W, stride_wn, stride_wk)};
    if (in[0].n < 0 || in[1].n < 0) return GETT_ERROR_NOT_SUPPORTED;
    for (int i = 0; i < 5; ++i) {
        for (int j = i + 1; j < 5; ++j)
            if (out[i].p && out[j].p && overlaps(out[i].p, out[i].n, out[j].p, out[j].n))
                return GETT_ERROR_INVALID_VALUE;
        for (const Range &x : in)
            if (out[i].p && x.p && overlaps(out[i].p, out[i].n, x.p, x.n))
                return GETT_ERROR_INVALID_VALUE;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t cx = mx_code_bytes(m, k), px = cx + mx_scale_bytes(m, k);
    const int64_t cw = mx_code_bytes(n, k), pw = cw + mx_scale_bytes(n, k);
    Product p = product_of({nullptr, nullptr, m}, {nullptr, nullptr, n}, k, Y, stride_ym, stride_yn);
    Partials w;
    gett_status_t ws = product_workspace(&p, 1, px + pw, s, w);
    if (ws != GETT_SUCCESS) return ws;
    char *x = static_cast<char *>(w.tiles), *y = x + px;
    p = product_of({x, x + cx, m}, {y, y + cw, n}, k, Y, stride_ym, stride_yn);
    const QuantizeJob q[2] = {
        {m, k, X, stride_xm, stride_xk, x, x + cx, codes_xt, scales_xt},
        {n, k, W, stride_wn, stride_wk, y, y + cw, codes_wt, scales_wt}};
    if (dtype_X == dtype_W) {
        ws = quantize_launch(dtype_X, q, 2, s);
    } else {
        ws = quantize_launch(dtype_X, q, 1, s);
        if (ws == GETT_SUCCESS) ws = quantize_launch(dtype_W, q + 1, 1, s);
    }
    if (ws != GETT_SUCCESS || m == 0 || n == 0) return ws;
    return contract_launch(&p, 1, slots_of(w, px + pw), w.counters, k > 0 ? 1.0 : 0.0, 0.0, dtype_X, s);
}

gett_status_t gett_mx_linear_grad(int64_t m, int64_t n, int64_t k, gett_dtype_t dtype_Y,
                                  const void *dY, int64_t stride_ym, int64_t stride_yn,
                                  const void *codes_xt, const void *scales_xt,
                                  const void *codes_wt, const void *scales_wt, void *dX,
                                  int64_t stride_xm, int64_t stride_xk, gett_dtype_t dtype_W,
                                  void *dW, int64_t stride_wn, int64_t stride_wk, void *stream)
{
    using namespace gett;
    gett_status_t st = matrix_ok(dtype_Y, m, n, dY, stride_ym, stride_yn);
    if (st != GETT_SUCCESS) return st;
    if (!float_type(dtype_W) || k < 0) return GETT_ERROR_INVALID_VALUE;
    if (!dX && !dW) return m > 0 && n > 0 && k > 0 ? GETT_ERROR_INVALID_VALUE : GETT_SUCCESS;
    if (dX) st = result_ok(m, k, n, dtype_Y, dX, stride_xm, stride_xk);
    if (dW && st == GETT_SUCCESS) st = result_ok(n, k, m, dtype_W, dW, stride_wn, stride_wk);
    if (st != GETT_SUCCESS) return st;
    const bool sum = m > 0 && n > 0 && k > 0;
    if (sum && ((dX && !packed_ok(codes_wt, scales_wt)) || (dW && !packed_ok(codes_xt, scales_xt))))
        return GETT_ERROR_INVALID_VALUE;
    const int64_t bytesY = sum ? span_bytes(m, n, stride_ym, stride_yn, type_size(dtype_Y)) : 0;
    const int64_t bytesX = m > 0 && k > 0 && dX ? span_bytes(m, k, stride_xm, stride_xk, type_size(dtype_Y)) : 0;
    const int64_t bytesW = n > 0 && k > 0 && dW ? span_bytes(n, k, stride_wn, stride_wk, type_size(dtype_W)) : 0;
    if (bytesY < 0) return GETT_ERROR_NOT_SUPPORTED;
    if (bytesX && bytesW && overlaps(dX, bytesX, dW, bytesW)) return GETT_ERROR_INVALID_VALUE;
    for (int i = 0; i < 2 && sum; ++i) {
        const void *o = i ? dW : dX;
        const int64_t bytes = i ? bytesW : bytesX;
        if (!o) continue;
        if (overlaps(o, bytes, dY, bytesY) || (dX && !clear_of(o, bytes, codes_wt, scales_wt, k, n)) ||
            (dW && !clear_of(o, bytes, codes_xt, scales_xt, k, m)))
            return GETT_ERROR_INVALID_VALUE;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    // dX = dY W: sums over n;  dW = dY^T X: sums over m
    const int64_t cd = mx_code_bytes(m, n), pd = dX ? cd + mx_scale_bytes(m, n) : 0;
    const int64_t ct = mx_code_bytes(n, m), pt = dW ? ct + mx_scale_bytes(n, m) : 0;
    const bool wantX = dX && m > 0 && k > 0, wantW = dW && n > 0 && k > 0;
    if (!wantX && !wantW) return GETT_SUCCESS;
    const int count = wantX && wantW ? 2 : 1;
    Product p[2];
    auto make = [&](const char *d, const char *t) {
        int i = 0;
        if (wantX)
            p[i++] = product_of({d, d + cd, m}, {codes_wt, scales_wt, k}, n, dX, stride_xm, stride_xk);
        if (wantW)
            p[i] = product_of({t, t + ct, n}, {codes_xt, scales_xt, k}, m, dW, stride_wn, stride_wk);
    };
    make(nullptr, nullptr);
    Partials w;
    gett_status_t ws = product_workspace(p, count, pd + pt, s, w);
    if (ws != GETT_SUCCESS) return ws;
    char *d = static_cast<char *>(w.tiles), *t = d + pd;
    make(d, t);
    if (sum) {
        const QuantizeJob q = {m, n, dY, stride_ym, stride_yn, wantX ? d : nullptr, wantX ? d + cd : nullptr,
                               wantW ? t : nullptr, wantW ? t + ct : nullptr};
        ws = quantize_launch(dtype_Y, &q, 1, s);
        if (ws != GETT_SUCCESS) return ws;
    }
    if (dtype_W == dtype_Y || count == 1)
        return contract_launch(p, count, slots_of(w, pd + pt), w.counters, 1.0, 0.0,
                               wantX ? dtype_Y : dtype_W, s);
    ws = contract_launch(p, 1, slots_of(w, pd + pt), w.counters, 1.0, 0.0, dtype_Y, s);
    if (ws != GETT_SUCCESS) return ws;
    return contract_launch(p + 1, 1, slots_of(w, pd + pt + p[0].plan.slotBytes),
                           w.counters + p[0].plan.counters, 1.0, 0.0, dtype_W, s);
}

}  // extern "C"
