// mx_product.hip -- products of packed 4-bit matrices,
//     C[m, n] <- alpha * sum_k A[m, k] B[n, k] + beta * C[m, n],
// and of float rows, quantised on the way, with a packed matrix.
//
// Many rows: tiles of C, the operands' panels through LDS (panel.hpp).
// Few rows: bound by B's bytes.  A workgroup takes 32 rows of B (32 columns
// of C) and its wavefronts every eighth panel; B goes from memory straight
// into the registers that the MFMA reads (a lane's two pieces of a panel are
// 32 bytes of one row), so no byte waits for a barrier, and the eight partial
// results are summed in wavefront order through LDS.
#include "matrix.hpp"
#include "launch.hpp"
#include "panel.hpp"

namespace gett {

bool packed_ok(const void *codes, const void *scales);
gett_status_t quantize_launch(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                              int64_t sr, int64_t sc, void *codes, void *scales, void *codesT,
                              void *scalesT, hipStream_t stream);

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

template <typename T, typename S>
__global__ __launch_bounds__(S::THREADS) void mx_tile_kernel(PanelOperand A, PanelOperand B,
                                                            PanelGrid grid, Result<T> o)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    int tm, tn;
    const PanelItem w = panel_item(grid, (int)blockIdx.x);
    panel_tile(grid, w.tile, tm, tn);
    A.row0 = tm * S::BM;
    B.row0 = tn * S::BN;
    Panel<kPanelMx, S> p;
    p.init();
    p.run(dyn_lds, A, B, w.t0, w.t1);
    __syncthreads();
    if (!panel_join<kPanelMx, S>(p, grid, w, dyn_lds) || p.group > 0) return;
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

template <typename T, typename S>
hipError_t tile_launch(const PanelOperand &A, const PanelOperand &B, int panels, const TilePlan &p,
                       float *slots, int *counters, const Result<T> &o, hipStream_t stream)
{
    constexpr auto k = mx_tile_kernel<T, S>;
    const hipError_t e = allow_dynamic_lds<k>(S::lds(kPanelMx));
    if (e != hipSuccess) return e;
    const int64_t tilesM = (o.m + S::BM - 1) / S::BM, tilesN = (o.n + S::BN - 1) / S::BN;
    PanelGrid g;
    if (!panel_grid(g, 1, tilesM, tilesN, tilesM * tilesN, p.cut, panels, slots, counters))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3((unsigned)p.cut.blocks), dim3(S::THREADS), S::lds(kPanelMx), stream,
                       A, B, g, o);
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
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float x[32];
            const int k0 = t * kTileK + q * 64 + b * 32, left = r < m ? k - k0 : 0;
            const TA *p = A + (int64_t)r * sm + (int64_t)k0 * sk;
            if (sk == 1 && left >= 32) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const Run<TA, 8> v = *reinterpret_cast<const Run<TA, 8> *>(p + 8 * c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[8 * c + i] = to_float(v.v[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = i < left ? to_float(p[i * sk]) : 0.0f;
            }
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
            const uint32_t sb = scale_byte(top);
            const float s = scale_value(sb);
#pragma unroll
            for (int c = 0; c < 4; ++c) f.v[0][b][c] = (int)codes8(x + 8 * c, s);
            f.s[0] |= (int)(sb << (8 * b));
        }
    }
};

// `deep`: panels whose loads are in flight together
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

// Few rows go their own way; tiles get slots for shared sums behind the
// `before` bytes of the stream's workspace that the caller has in use.
bool few_rows(int64_t m, int64_t k) { return k > 0 && m <= 32; }

template <typename T>
hipError_t contract_typed(const Packed &A, const Packed &B, int64_t k, const TilePlan &plan,
                          float *slots, int *counters, const Result<T> &o, hipStream_t stream)
{
    const int panels = (int)mx_tiles(k);
    const uint8_t *ca = static_cast<const uint8_t *>(A.codes);
    const uint8_t *sa = static_cast<const uint8_t *>(A.scales);
    const uint8_t *cb = static_cast<const uint8_t *>(B.codes);
    const uint8_t *sb = static_cast<const uint8_t *>(B.scales);
    if (few_rows(o.m, k))
        return o.m <= 16 ? few_launch<T, FewPacked<1>, 1>({ca, sa, o.m}, cb, sb, panels, o, stream)
                         : few_launch<T, FewPacked<2>, 2>({ca, sa, o.m}, cb, sb, panels, o, stream);
    const PanelOperand pa = {ca, sa, o.m, 0}, pb = {cb, sb, o.n, 0};
    if (plan.shape == 0)
        return tile_launch<T, Big>(pa, pb, panels, plan, slots, counters, o, stream);
    if (plan.shape == 1)
        return tile_launch<T, Mid>(pa, pb, panels, plan, slots, counters, o, stream);
    return tile_launch<T, Small>(pa, pb, panels, plan, slots, counters, o, stream);
}

template <typename T>
Result<T> result(void *C, int64_t sm, int64_t sn, int64_t m, int64_t n, double alpha, double beta)
{
    return Result<T>{static_cast<T *>(C), sm, sn, (int)m, (int)n, (float)alpha, (float)beta};
}

// What a product of m x k by n x k needs of the workspace, with C's neighbours
// along n (or exchanged).
struct Need {
    bool swapped;
    TilePlan plan;
};
Need need_of(int64_t m, int64_t n, int64_t k, int64_t sm, int64_t sn)
{
    Need w = {};
    w.swapped = sm == 1 && sn != 1;   // C's neighbours lie along m: C^T = B A^T
    if (w.swapped) std::swap(m, n);
    if (!few_rows(m, k)) w.plan = tile_plan(m, n, mx_tiles(k));
    return w;
}

gett_status_t contract_launch(Packed A, Packed B, int64_t k, const Need &need, float *slots,
                              int *counters, double alpha, double beta, gett_dtype_t dtype, void *C,
                              int64_t sm, int64_t sn, hipStream_t stream)
{
    if (need.swapped) {
        std::swap(A, B);
        std::swap(sm, sn);
    }
    const int64_t m = A.rows, n = B.rows;
    hipError_t e;
    if (dtype == GETT_FLOAT32)
        e = contract_typed<float>(A, B, k, need.plan, slots, counters,
                                  result<float>(C, sm, sn, m, n, alpha, beta), stream);
    else if (dtype == GETT_BFLOAT16)
        e = contract_typed<bf16>(A, B, k, need.plan, slots, counters,
                                 result<bf16>(C, sm, sn, m, n, alpha, beta), stream);
    else
        e = contract_typed<_Float16>(A, B, k, need.plan, slots, counters,
                                     result<_Float16>(C, sm, sn, m, n, alpha, beta), stream);
    return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
}

// the whole call: the product alone
gett_status_t contract(const Packed &A, const Packed &B, int64_t k, double alpha, double beta,
                       gett_dtype_t dtype, void *C, int64_t sm, int64_t sn, hipStream_t stream)
{
    const Need need = need_of(A.rows, B.rows, k, sm, sn);
    Partials w;
    if (need.plan.slotBytes > 0) {
        const gett_status_t ws = stream_workspace(stream, (uint64_t)need.plan.counters,
                                                  (uint64_t)need.plan.slotBytes, w);
        if (ws != GETT_SUCCESS) return ws;
    }
    return contract_launch(A, B, k, need, static_cast<float *>(w.tiles), w.counters, alpha, beta,
                           dtype, C, sm, sn, stream);
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
    if (m <= 16) {
        const Packed B = {codes_B, scales_B, n};
        hipError_t e;
        if (dtype == GETT_FLOAT32)
            e = few_float_of<float>(dtype_A, A, stride_am, stride_ak, k, B,
                                    result<float>(C, stride_m, stride_n, m, n, alpha, beta), s);
        else if (dtype == GETT_BFLOAT16)
            e = few_float_of<bf16>(dtype_A, A, stride_am, stride_ak, k, B,
                                   result<bf16>(C, stride_m, stride_n, m, n, alpha, beta), s);
        else
            e = few_float_of<_Float16>(dtype_A, A, stride_am, stride_ak, k, B,
                                       result<_Float16>(C, stride_m, stride_n, m, n, alpha, beta),
                                       s);
        return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
    }
    // A's packed copy and the slots of shared sums, in the stream's workspace.
    // The hold lasts until both launches are enqueued.
    const int64_t codeBytes = mx_code_bytes(m, k), packed = codeBytes + mx_scale_bytes(m, k);
    const Need need = need_of(m, n, k, stride_m, stride_n);
    Partials w;
    gett_status_t ws = stream_workspace(s, (uint64_t)need.plan.counters,
                                        (uint64_t)(packed + need.plan.slotBytes), w);
    if (ws != GETT_SUCCESS) return ws;
    char *codes = static_cast<char *>(w.tiles), *scales = codes + codeBytes;
    ws = quantize_launch(dtype_A, m, k, A, stride_am, stride_ak, codes, scales, nullptr, nullptr, s);
    if (ws != GETT_SUCCESS) return ws;
    return contract_launch({codes, scales, m}, {codes_B, scales_B, n}, k, need,
                           reinterpret_cast<float *>(codes + packed), w.counters, alpha, beta, dtype,
                           C, stride_m, stride_n, s);
}

}  // extern "C"
