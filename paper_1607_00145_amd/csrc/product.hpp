// product.hpp -- products of plain matrices in 16 and 32 bits for the layers of
// gett_layers.h (device code): one tile of
//     C[i, j] = sum over K of M(i, k) N(j, k)
// for a workgroup, whose M and N lie as rows (k fastest) or as columns (the row of C
// fastest), all three products of a linear layer being of one of these forms:
//     y = x w^T    M = x  rows,           N = w  rows
//     dx = dz w    M = dz rows,           N = w  columns
//     dw = dz^T x  M = dz columns,        N = x  columns
// so that no operand is transposed in memory.
//
// Panels.  K is cut into panels of 128 bytes (64 numbers of 16 bits, 32 of 32).  A
// panel goes from memory straight into LDS, 16 bytes a lane.  One MFMA 32 x 32
// takes 16 bytes a lane of either operand: lane l the piece 4 (l / 32) + s of row
// l % 32, for the slabs s = 0..3 of a panel; in 16 bits that is one instruction of
// K = 16, in 32 bits four of K = 2 (which two numbers of K meet in an instruction
// does not matter as long as both operands say the same).
//
// Rows lie in LDS as they are, 128 bytes each, piece p of row r at place p ^ f(r):
// sixteen lanes that read together then fall on all sixteen places of 256 bytes.
// Columns lie with k slowest.  In 16 bits ds_read_tr16 hands each lane four k of
// its row: sixteen lanes read four neighbouring rows of C at four k each and
// exchange them.  Piece p of k lies at p ^ 4 (k % 4), for the same reason.  In 32
// bits a lane reads its four numbers by themselves (the instructions take
// sixteen times as long as the ones in 16 bits, and LDS has the time).
//
// N comes first in the instruction, so that a lane's results are of one row i
// and of columns j that follow one another; which row of N is which row of an
// instruction's operand is chosen so that the results of two instructions make
// runs of eight columns: 16 bytes of a 16-bit C, and one block of random bits.
#pragma once
#include <type_traits>

#include "layers.hpp"
#include "panel.hpp"

namespace gett {

// One operand, its tile's rows from the first on.
struct Side {
    const char *p;        // k = 0 of the tile's first row
    int64_t ld;           // bytes from a row (Rows) or a k (Columns) to the next
    int count;            // rows of the tile that are there
    int extent;           // numbers along K
};

// How a product's result is written.
struct Epilogue {
    const char *bias;       // n numbers of the type, or nullptr
    const char *residual;
    char *Z, *Y;
    int64_t ldr, ldz, ldy;  // elements
    int activation;
    int wide;               // Y is in 32 bits whatever the type
    Drop drop;
};

// A product, or the products of a list of experts.
struct ProductArgs {
    const char *M, *N;
    int64_t ldm, ldn;       // bytes
    int64_t stepN;          // bytes between the experts' N (kByRows), of Y (kByK: elements)
    int m, n;               // rows and columns of C (of one expert's: kByK)
    int k;                  // of the sum (kByK: of all experts together)
    int fullM, fullN;       // rows of a column operand that may be read (m, n rounded up where
                            // they are zeros)
    int kM, kN;             // K of the operands that may be read
    int tilesM, tilesN;
    Recip tilesMInv, tilesNInv;
    int experts;
    const int32_t *offsets; // device, experts + 1
    const int32_t *order;   // device: M's rows are those of order[.] / choices, or nullptr
    int choices;
    Recip choicesInv;
    Epilogue out;
};

enum ProductForm { kRowsRows, kRowsColumns, kColumnsColumns };
enum ProductGroups { kWhole, kByRows, kByK };

template <int FM_, int FN_, int WM_, int WN_, int NS_> struct ProductShape {
    static constexpr int FM = FM_, FN = FN_, WM = WM_, WN = WN_, NS = NS_;
    static constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int STAGE = (BM + BN) * 128;
    static constexpr int JA = BM / 8 / NW, JB = BN / 8 / NW, J = JA + JB;   // loads a lane
    static constexpr int LDS = NS * STAGE;
    static_assert(FN % 2 == 0 && (FM & (FM - 1)) == 0 && (FN & (FN - 1)) == 0, "runs of eight");
    static_assert(JA * 8 * NW == BM && JB * 8 * NW == BN, "whole instructions");
    static_assert((NS - 1) * J < 64, "vmcnt");
    static_assert(LDS >= NW * 32 * 32 * FN * 4, "results");
};

constexpr uint32_t kNowhere = 0xfffffff0u;   // behind every buffer: such a load gives zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t whole_buffer(const char *p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), 0, (int)kNowhere, 0x00027000);
}

typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s4 lds_s4;

template <typename T> __device__ __forceinline__ f16v product_mfma(i4 a, i4 b, f16v c);
template <> __device__ __forceinline__ f16v product_mfma<bf16>(i4 a, i4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f16v product_mfma<_Float16>(i4 a, i4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f16v product_mfma<float>(i4 a, i4 b, f16v c)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(a[j]), __int_as_float(b[j]), c, 0, 0, 0);
    return c;
}

template <typename T, bool MCOL, bool NCOL, typename S> struct Product {
    static constexpr int FM = S::FM, FN = S::FN, NS = S::NS;
    static constexpr int EP = 16 / sizeof(T);      // numbers of a piece
    static constexpr int KP = 8 * EP;              // of a panel
    f16v acc[FM][FN];
    int q, h, wm, wn;

    __device__ __forceinline__ void init()
    {
        const int tid = (int)threadIdx.x;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        q = tid & 31;
        h = (tid >> 5) & 1;
        wm = wave / S::WN;
        wn = wave % S::WN;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    }
    // acc[i][2 u + x][4 a + y] is that of row 32 i + q and column 64 u + 16 a + 8 h +
    // 4 x + y of the wavefront's part.

    // Where a lane's 16 bytes of load j lie: k or piece that decides whether they
    // are within K (`at`), and the offset from the panel's first byte.
    template <bool COL, int B, bool ISN, typename Row>
    __device__ __forceinline__ static void place(const Side &x, int j, int wave, int lane, Row rowOffset,
                                                 uint32_t &off, int &at)
    {
        const int L = (j * S::NW + wave) * 64 + lane;
        if constexpr (COL) {
            constexpr int PR = B / EP;             // pieces of one k
            const int k = L / PR, pl = L % PR;
            const int piece = sizeof(T) == 2 ? pl ^ (4 * (k & 3) & (PR - 1)) : pl;
            at = k;
            off = piece * EP < x.count ? (uint32_t)(k * x.ld) + piece * 16 : kNowhere;
        } else {
            const int r = L >> 3, pl = L & 7;
            const int piece = pl ^ (ISN ? ((r >> 1) & 1) | ((r >> 3) & 3) << 1 : (r >> 1) & 7);
            at = piece * EP;
            off = r < x.count ? rowOffset(r) + piece * 16 : kNowhere;
        }
    }

    // The panels of K = [0, extent) of both sides; `lds` holds S::LDS bytes.
    template <typename RowM>
    __device__ __forceinline__ void run(char *lds, const Side &M, const Side &N, RowM rowM, int panels)
    {
        constexpr int NW = S::NW, J = S::J, JA = S::JA;
        const int lane = (int)threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        uint32_t off[J];
        int at[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j < JA)
                place<MCOL, S::BM, false>(M, j, wave, lane, rowM, off[j], at[j]);
            else
                place<NCOL, S::BN, true>(N, j - JA, wave, lane,
                                         [&](int r) { return (uint32_t)(r * N.ld); }, off[j], at[j]);
        }
        const int64_t stepM = MCOL ? KP * M.ld : 128, stepN = NCOL ? KP * N.ld : 128;
        const char *pm = M.p, *pn = N.p;
        int leftM = M.extent, leftN = N.extent;
        auto issue = [&](int stage) {
            const __amdgpu_buffer_rsrc_t rm = whole_buffer(pm), rn = whole_buffer(pn);
            char *base = lds + stage * S::STAGE;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool isM = j < JA;
                char *dst = base + (isM ? 0 : S::BM * 128) + ((isM ? j : j - JA) * NW + wave) * 1024;
                const uint32_t o = at[j] < (isM ? leftM : leftN) ? off[j] : kNowhere;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(isM ? rm : rn, (matrix_lds *)dst, 16, (int)o,
                                                         0, 0, 0);
            }
            pm += stepM;
            pn += stepN;
            leftM -= KP;
            leftN -= KP;
        };

        // A lane's own address in a stage for fragment 0 and slab 0; the others are
        // that, exclusive or (and plus) constants.
        const int j4 = lane & 3, k4 = (lane >> 2) & 3, g2 = (lane >> 4) & 1;
        int ownM, ownN;
        if constexpr (!MCOL) {
            ownM = (wm * 32 * FM + q) * 128 + ((4 * h) ^ ((q >> 1) & 7)) * 16;
        } else if constexpr (sizeof(T) == 2) {
            constexpr int PR = S::BM / EP;
            const int piece = wm * 4 * FM + 2 * g2 + (j4 >> 1);
            ownM = (32 * h + k4) * PR * 16 + (piece ^ (4 * k4 & (PR - 1))) * 16 + (j4 & 1) * 8;
        } else {
            ownM = 16 * h * S::BM * 4 + (wm * 32 * FM + q) * 4;
        }
        const int nq = 16 * (q >> 3) + 8 * ((q >> 2) & 1) + (q & 3);   // row of N of fragment 0
        if constexpr (!NCOL) {
            ownN = (wn * 32 * FN + nq) * 128 +
                   ((4 * h) ^ (((q >> 1) & 1) | ((q >> 2) & 1) << 1 | ((q >> 3) & 1) << 2)) * 16;
        } else if constexpr (sizeof(T) == 2) {
            constexpr int PR = S::BN / EP;
            const int piece = wn * 4 * FN + 4 * g2 + j4;
            ownN = (32 * h + k4) * PR * 16 + (piece ^ (4 * k4 & (PR - 1))) * 16;
        } else {
            ownN = 16 * h * S::BN * 4 + (wn * 32 * FN + nq) * 4;
        }
        ownN += S::BM * 128;
        int atM = ownM, atN = ownN;
        auto at_stage = [&](int stage) {
            atM = ownM + stage * S::STAGE;
            atN = ownN + stage * S::STAGE;
            asm volatile("" : "+v"(atM), "+v"(atN));
        };
        auto quad = [&](int address) {
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s4 *)((__attribute__((address_space(3))) char *)lds + address));
        };
        auto join = [](s4 a, s4 b) {
            return __builtin_bit_cast(i4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        i4 a[2][FM], b[2][FN];
        auto read = [&](int set, int s) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if constexpr (!MCOL) {
                    a[set][i] = *reinterpret_cast<const i4 *>(lds + (atM ^ (s * 16)) + i * 4096);
                } else if constexpr (sizeof(T) == 2) {
                    constexpr int KB = S::BM * 2;      // bytes of one k
                    const int x = (atM ^ (i * 64)) + 8 * s * KB;
                    a[set][i] = join(quad(x), quad(x + 4 * KB));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        a[set][i][j] = *reinterpret_cast<const int *>(
                            lds + atM + (4 * s + j) * S::BM * 4 + i * 128);
                }
            }
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                if constexpr (!NCOL) {
                    b[set][f] = *reinterpret_cast<const i4 *>(lds + (atN ^ (s * 16)) +
                                                             (64 * (f >> 1) + 4 * (f & 1)) * 128);
                } else if constexpr (sizeof(T) == 2) {
                    constexpr int KB = S::BN * 2;
                    const int x = (atN ^ (128 * (f >> 1))) + 8 * (f & 1) + 8 * s * KB;
                    b[set][f] = join(quad(x), quad(x + 4 * KB));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        b[set][f][j] = *reinterpret_cast<const int *>(
                            lds + atN + (4 * s + j) * S::BN * 4 + (64 * (f >> 1) + 4 * (f & 1)) * 4);
                }
            }
        };
        auto mma = [&](int set) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int f = 0; f < FN; ++f)
                    acc[i][f] = product_mfma<T>(b[set][f], a[set][i], acc[i][f]);
        };
        // no fence: a release would wait for the loads in flight as well
        auto barrier = []() { asm volatile("s_barrier" ::: "memory"); };
        // s_waitcnt operands: lgkmcnt 0 and that many loads left on their way
        auto wait_for = [](int left) constexpr { return (left & 15) | (left >> 4) << 14 | 7 << 4; };
        constexpr int kAll = wait_for(0), kFirst = wait_for((NS - 1) * J);
        constexpr int kNext = wait_for((NS - 2) * J);

        if (panels <= 0) return;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < panels) issue(i);
        if (panels >= NS) __builtin_amdgcn_s_waitcnt(kFirst);
        else __builtin_amdgcn_s_waitcnt(kAll);
        barrier();
        at_stage(0);
        read(0, 0);
        int stage = 0;
        // While a panel is multiplied the next NS - 1 are on their way; one barrier a
        // panel, after its last LDS read and before its last MFMAs.
        auto panel = [&](auto more, auto load) {
            static_for<4>([&](auto step) {
                constexpr int s = decltype(step)::value, set = s & 1;
                if constexpr (s < 3) {
                    read(set ^ 1, s + 1);
                } else if constexpr (more) {
                    __builtin_amdgcn_s_waitcnt(load ? kNext : kAll);   // the next is there
                    barrier();
                    if constexpr (load) issue(stage);
                    stage = stage + 1 == NS ? 0 : stage + 1;
                    at_stage(stage);
                    read(set ^ 1, 0);
                }
                mma(set);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        const std::true_type yes;
        const std::false_type no;
        int t = 0;
        for (; t + NS < panels; ++t) panel(yes, yes);
        for (; t + 1 < panels; ++t) panel(yes, no);
        panel(no, no);
    }
};

// ------------------------------------------------------------------- kernel ---

template <typename T>
__device__ __forceinline__ void product_store(const Epilogue &o, uint64_t key, int64_t row, int col,
                                              int left, float v[8])
{
    if (left <= 0) return;
    if (o.bias) {
        float x[8];
        load8(reinterpret_cast<const T *>(o.bias) + col, left, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += x[i];
    }
    if (o.Z) store8(reinterpret_cast<T *>(o.Z) + row * o.ldz + col, left, v);
    if (o.activation != GETT_ACTIVATION_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate(o.activation, v[i]);
    }
    if (o.drop.cut) drop8(v, o.drop, key, (uint32_t)row, (uint32_t)col);
    if (o.residual) {
        float x[8];
        load8(reinterpret_cast<const T *>(o.residual) + row * o.ldr + col, left, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += x[i];
    }
    if (o.wide) store8(reinterpret_cast<float *>(o.Y) + row * o.ldy + col, left, v);
    else store8(reinterpret_cast<T *>(o.Y) + row * o.ldy + col, left, v);
}

// offsets[e], brought into [0, rows]
__device__ __forceinline__ int expert_offset(const int32_t *offsets, int e, int rows)
{
    const int v = offsets[e];
    return v < 0 ? 0 : v > rows ? rows : v;
}

// Tiles of BM rows of a list of experts.  Expert e's begin with number
// offsets[e] / BM + e, which leaves each as many as it needs and needs no table:
// the last e whose first is not behind `slot`.  What lies behind the last expert's
// rows counts as one more expert.
template <int BM>
__device__ __forceinline__ int expert_of_slot(const int32_t *offsets, int experts, int rows, int slot)
{
    const int lane = (int)threadIdx.x & 63;
    int found = 0;
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int e = e0 + lane;
        const bool before = e <= experts && expert_offset(offsets, e < experts ? e : experts, rows) / BM + e <= slot;
        const int n = __popcll(__ballot(before));
        found += n;
        if (n < 64) break;
    }
    return found - 1;   // expert 0's first is 0
}

template <typename T, ProductForm FORM, typename S>
__global__ __launch_bounds__(S::THREADS) void product_kernel(ProductArgs g, int groups)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    constexpr bool MCOL = FORM == kColumnsColumns, NCOL = FORM != kRowsRows;
    constexpr int KP = 128 / (int)sizeof(T);
    const int bid = (int)blockIdx.x;
    int tm = (int)quotient((uint32_t)bid, g.tilesN, g.tilesNInv);
    const int tn = bid - tm * g.tilesN;
    // rows of M and of C, K, and the expert's share of them
    int row0 = 0, rows = g.m, first = 0, sum = g.k, e = 0;
    bool empty = false;
    if (groups == kByRows) {
        e = expert_of_slot<S::BM>(g.offsets, g.experts, g.m, tm);
        e = __builtin_amdgcn_readfirstlane(e);
        const int begin = expert_offset(g.offsets, e, g.m);
        rows = e == g.experts ? g.m : expert_offset(g.offsets, e + 1, g.m);
        row0 = begin + (tm - (begin / S::BM + e)) * S::BM;
        empty = e == g.experts;
    } else if (groups == kByK) {
        e = (int)quotient((uint32_t)tm, g.tilesM, g.tilesMInv);
        tm -= e * g.tilesM;
        first = expert_offset(g.offsets, e, g.k);
        sum = expert_offset(g.offsets, e + 1, g.k) - first;
        row0 = tm * S::BM;
    } else {
        row0 = tm * S::BM;
    }
    if (row0 >= rows) return;
    const int col0 = tn * S::BN;
    Product<T, MCOL, NCOL, S> p;
    p.init();
    if (!empty) {
        const bool gathered = FORM == kRowsRows && g.order;
        Side M, N;
        M.ld = g.ldm;
        N.ld = g.ldn;
        N.p = g.N + (groups == kByRows ? (int64_t)e * g.stepN : 0);
        if constexpr (MCOL) {
            M.p = g.M + (int64_t)first * g.ldm + (int64_t)row0 * sizeof(T);
            M.count = g.fullM - row0;
            M.extent = sum;
        } else {
            M.p = g.M + (gathered ? 0 : (int64_t)row0 * g.ldm);
            M.count = rows - row0;
            M.extent = g.kM;
        }
        if constexpr (NCOL) {
            N.p += (int64_t)first * g.ldn + (int64_t)col0 * sizeof(T);
            N.count = g.fullN - col0;
            N.extent = sum;
        } else {
            N.p += (int64_t)col0 * g.ldn;
            N.count = g.n - col0;
            N.extent = g.kN;
        }
        const int32_t *order = g.order + (gathered ? row0 : 0);
        auto rowM = [&](int r) {
            if (FORM == kRowsRows && gathered) {
                const uint32_t id = min((uint32_t)order[r], (uint32_t)g.m - 1);
                r = (int)quotient(id, g.choices, g.choicesInv);
            }
            return (uint32_t)(r * g.ldm);
        };
        p.run(dyn_lds, M, N, rowM, (sum + KP - 1) / KP);
    }
    Epilogue o = g.out;
    if (groups == kByRows && o.bias) o.bias += (int64_t)e * g.n * sizeof(T);
    if (groups == kByK) o.Y += (int64_t)e * g.stepN * (o.wide ? 4 : sizeof(T));
    if (empty) {
        o.bias = nullptr;
        o.activation = GETT_ACTIVATION_NONE;
    }
    const uint64_t key = o.drop.cut ? o.drop.key() : 0;
    // The results go through LDS, 32 rows of a wavefront at a time, so that one
    // loop (and not one copy of the epilogue for each register) takes them, whole
    // lines of C each time.  Piece x of row r lies at x ^ (r % 16).
    constexpr int W = 32 * S::FN;                 // columns of a wavefront
    const int lane = (int)threadIdx.x & 63;
    char *mine = dyn_lds + (p.wm * S::WN + p.wn) * 32 * W * 4;
    __syncthreads();
    static_for<S::FM>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
#pragma unroll
        for (int u = 0; u < S::FN / 2; ++u)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int piece = 16 * u + 4 * a + 2 * p.h + x;
                    const f16v &c = p.acc[i][2 * u + x];
                    *reinterpret_cast<f4 *>(mine + p.q * W * 4 + (piece ^ (p.q & 15)) * 16) =
                        f4{c[4 * a], c[4 * a + 1], c[4 * a + 2], c[4 * a + 3]};
                }
        constexpr int PER = W / 8, ROWS = 64 / PER;   // runs of a row, rows a pass
        const int run = lane % PER, first = lane / PER;
        const int c = col0 + p.wn * W + 8 * run;
#pragma unroll 1
        for (int r = first; r < 32; r += ROWS) {
            const int row = row0 + p.wm * 32 * S::FM + 32 * i + r;
            if (row >= rows) break;
            const f4 lo = *reinterpret_cast<const f4 *>(mine + r * W * 4 + ((2 * run) ^ (r & 15)) * 16);
            const f4 hi = *reinterpret_cast<const f4 *>(mine + r * W * 4 + ((2 * run + 1) ^ (r & 15)) * 16);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            product_store<T>(o, key, row, c, g.n - c, v);
        }
    });
}

}  // namespace gett
