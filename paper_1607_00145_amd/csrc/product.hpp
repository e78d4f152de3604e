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
// Bound by the matrix unit in large tiles: 8192 x 8192 x 4096 in bf16 takes 440 us for
// y, 400 for dx and for dw (1.25 and 1.37 PFLOP/s; a large library product reaches
// 1.59 on the card), with two MFMA operands read for each 256 x 256 x 64 panel
// from LDS while the next panel's come.  What was tried beside it: tiles of 256 x
// 128 with panels of 64 bytes, which halve the work between two barriers, 480; the
// instructions of 32 bits in another order, the same.
//
// N comes first in the instruction, so that a lane's results are of one row i
// and of four columns j that follow one another: they go to LDS in vectors, and from
// there to the epilogue in runs of eight columns, which are 16 bytes of a 16-bit C
// and one block of random bits.
#pragma once
#include <type_traits>

#include "layers.hpp"
#include "panel.hpp"
#include "product_plan.hpp"

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
    int tiles, tilesM, tilesN, bandRows;   // bandRows: of tiles, all experts' together
    Recip tilesMInv, bandInv;
    int full, slices;       // tiles from `full` on are shared by `slices` workgroups each,
    Recip slicesInv;        // units: full + the others' slices
    int units;
    float *slots;
    int *counters;
    int experts;
    const int32_t *offsets; // device, experts + 1
    const int32_t *order;   // device: M's rows are those of order[.] / choices, or nullptr
    int choices;
    Recip choicesInv;
    Epilogue out;
};

// FM x FN blocks of 32 x 32 for each of WM x WN wavefronts, NS stages of P panels.
template <int FM_, int FN_, int WM_, int WN_, int NS_, int P_ = 1> struct ProductShape {
    static constexpr int FM = FM_, FN = FN_, WM = WM_, WN = WN_, NS = NS_, P = P_;
    static constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr bool SLABS = false;
    static constexpr int PANEL = (BM + BN) * 128, STAGE = P * PANEL;
    static constexpr int JA = BM / 8 / NW, JB = BN / 8 / NW, JP = JA + JB, J = P * JP;   // loads a lane
    static constexpr int W = 32 * FN;                   // columns of a wavefront
    static constexpr int RESULTS = 16 * W * 4;          // of LDS a wavefront, for its results
    static constexpr int LDS = NS * STAGE + NW * RESULTS;
    static_assert((FM & (FM - 1)) == 0 && (FN & (FN - 1)) == 0, "addresses by exclusive or");
    static_assert(JA * 8 * NW == BM && JB * 8 * NW == BN, "whole instructions");
    static_assert((NS - 1) * J < 64, "vmcnt");
};

// One block of 32 x 32 for four wavefronts, each of which takes one slab of every panel,
// three workgroups a CU: for products that have too few larger tiles to fill the card.
// Bound by a barrier and the LDS latency behind it, 0.13 us a stage of two panels (fp32
// 0.33, of which the MFMAs have 0.25), until several are on a CU.  (Stages of one panel,
// four of them: 512 x 512 x 4096 in bf16 10.4 us, where this takes 8.5; eight of them, or
// the epilogue's operands fetched before the panels, were not better.)
struct ProductSlabs {
    static constexpr int FM = 1, FN = 1, NS = 3, P = 2, BM = 32, BN = 32, NW = 4, THREADS = 256;
    static constexpr bool SLABS = true;
    static constexpr int PANEL = (BM + BN) * 128, STAGE = P * PANEL, JA = 1, JB = 1, JP = 2, J = P * JP;
    static constexpr int ROW = 36;   // floats of a row of partial sums: whole vectors, few conflicts
    static constexpr int LDS = NS * STAGE;
    static_assert(LDS >= 4 * 32 * ROW * 4, "the partial sums come where the stages were");
};

constexpr uint32_t kNowhere = 0xfffffff0u;   // behind every buffer: such a load gives zeros

// A buffer from p on, as the instruction takes it; p is the same in all lanes.
__device__ __forceinline__ i4 whole_buffer(const char *p)
{
    const uint64_t a = (uint64_t)p;
    return i4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
              __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)), (int)kNowhere, 0x00027000};
}
// 16 bytes a lane straight into LDS, 1 KB from `at` on.  Written out, and not by the
// builtin: after that the compiler lets the first ds_read_tr16 wait for every load on
// its way, since it cannot tell their addresses apart (8192 x 8192 x 4096 in bf16, dw:
// 600 us by the builtin, 422 so).  It has no result in registers; the compiler's own
// waits count it as younger than what they wait for, or wait longer.  (m0 cannot be
// named as overwritten; nothing else in these kernels takes it.)
__device__ __forceinline__ void load_to_lds(i4 buffer, uint32_t offset, uint32_t at)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :: "v"(offset), "s"(buffer), "s"(at) : "memory");
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
    int q, h, wm, wn;       // wm, wn: the wavefront's part of the tile (of slabs: 0, its slab)

    __device__ __forceinline__ void locate()
    {
        const int tid = (int)threadIdx.x;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        q = tid & 31;
        h = (tid >> 5) & 1;
        if constexpr (S::SLABS) {
            wm = 0;
            wn = wave;
        } else {
            wm = wave / S::WN;
            wn = wave % S::WN;
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    }
    // acc[i][f][4 a + y] is that of row 32 i + q and column 32 f + 8 a + 4 h + y of the
    // wavefront's part.

    // A lane's 16 bytes of load j: the number along K that decides whether they are
    // within it is `first` and j times `step` ...
    template <bool COL, int B> struct Along {
        static constexpr int PR = B / EP;          // pieces of one k of columns
        static constexpr int step = COL ? S::NW * 64 / PR : 0;
        static_assert(COL ? S::NW * 64 % PR == 0 : S::NW % 2 == 0, "the same for every load");
        static __device__ __forceinline__ int first(int wave, int lane)
        {
            return COL ? (wave * 64 + lane) / PR : ((lane & 7) ^ ((wave * 8 + (lane >> 3)) >> 1 & 7)) * EP;
        }
    };
    // ... and this their offset from the panel's first byte.
    template <bool COL, int B, typename Row>
    __device__ __forceinline__ static uint32_t place(const Side &x, int j, int wave, int lane, Row rowOffset)
    {
        const int L = (j * S::NW + wave) * 64 + lane;
        if constexpr (COL) {
            constexpr int PR = B / EP;
            const int k = L / PR, pl = L % PR;
            const int piece = sizeof(T) == 2 ? pl ^ (4 * (k & 3) & (PR - 1)) : pl;
            return piece * EP < x.count ? (uint32_t)(k * x.ld) + piece * 16 : kNowhere;
        } else {
            const int r = L >> 3, piece = (L & 7) ^ ((r >> 1) & 7);
            return r < x.count ? rowOffset(r) + piece * 16 : kNowhere;
        }
    }

    // Loads on their way to LDS: what a lane fetches of each panel, and the next
    // panel.  In the order of issue a stage's J loads follow one another.
    uint32_t off[S::JP], panelM, panelN;
    int alongM, alongN;
    const char *pm, *pn;
    int64_t stepM, stepN;
    int leftM, leftN, panels;
    uint32_t ldsAt;

    i4 rm, rn;
    uint32_t to;
    __device__ __forceinline__ void issue_begin(int stage)
    {
        rm = whole_buffer(pm);
        rn = whole_buffer(pn);
        to = ldsAt + stage * S::STAGE;
    }
    __device__ __forceinline__ void issue_one(int j)
    {
        const int panel = j / S::JP;
        j -= panel * S::JP;
        const bool isM = j < S::JA;
        const int at = panel * KP + (isM ? alongM + j * Along<MCOL, S::BM>::step
                                         : alongN + (j - S::JA) * Along<NCOL, S::BN>::step);
        uint32_t o = off[j];
        if (panel) o = o == kNowhere ? o : o + panel * (isM ? panelM : panelN);
        o = at < (isM ? leftM : leftN) ? o : kNowhere;
        load_to_lds(isM ? rm : rn, o, to + panel * S::PANEL + (isM ? 0 : S::BM * 128) +
                                          (isM ? j : j - S::JA) * S::NW * 1024);
    }
    __device__ __forceinline__ void issue_end()
    {
        pm += stepM;
        pn += stepN;
        leftM -= S::P * KP;
        leftN -= S::P * KP;
    }
    // Takes a tile and sends the loads of its first panels; nobody reads LDS any more.
    template <typename RowM>
    __device__ __forceinline__ void begin(char *lds, const Side &M, const Side &N, RowM rowM, int count)
    {
        const int lane = (int)threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int j = 0; j < S::JP; ++j) {
            off[j] = j < S::JA ? place<MCOL, S::BM>(M, j, wave, lane, rowM)
                               : place<NCOL, S::BN>(N, j - S::JA, wave, lane,
                                                    [&](int r) { return (uint32_t)(r * N.ld); });
        }
        alongM = Along<MCOL, S::BM>::first(wave, lane);
        alongN = Along<NCOL, S::BN>::first(wave, lane);
        stepM = MCOL ? S::P * KP * M.ld : S::P * 128;
        stepN = NCOL ? S::P * KP * N.ld : S::P * 128;
        panelM = (uint32_t)(stepM / S::P);
        panelN = (uint32_t)(stepN / S::P);
        pm = M.p;
        pn = N.p;
        ldsAt = (uint32_t)(uintptr_t)(matrix_lds *)lds + wave * 1024;
        leftM = M.extent;
        leftN = N.extent;
        panels = count;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < panels) {
                issue_begin(i);
#pragma unroll
                for (int j = 0; j < S::J; ++j) issue_one(j);
                issue_end();
            }
    }

    // The sums over the panels of the tile that was begun; at least `after` stores
    // were issued since.
    template <int AFTER> __device__ __forceinline__ void run(char *lds, bool after)
    {
        constexpr int J = S::J;
        const int lane = (int)threadIdx.x & 63;
        // A lane's own address in a stage for fragment 0 and slab 0; the others are
        // that, exclusive or (and plus) constants.
        const int j4 = lane & 3, k4 = (lane >> 2) & 3, g2 = (lane >> 4) & 1;
        auto own = [&](auto column, auto size, int first) {
            constexpr int B = decltype(size)::value;
            if constexpr (!decltype(column)::value) {
                return (first + q) * 128 + ((4 * h) ^ ((q >> 1) & 7)) * 16;
            } else if constexpr (sizeof(T) == 2) {
                constexpr int PR = B / EP;
                const int piece = first / EP + 2 * g2 + (j4 >> 1);
                return (32 * h + k4) * PR * 16 + (piece ^ (4 * k4 & (PR - 1))) * 16 + (j4 & 1) * 8;
            } else {
                return 16 * h * B * 4 + (first + q) * 4;
            }
        };
        int ownM = own(std::bool_constant<MCOL>{}, std::integral_constant<int, S::BM>{}, wm * 32 * FM);
        int ownN = S::BM * 128 + own(std::bool_constant<NCOL>{}, std::integral_constant<int, S::BN>{},
                                     S::SLABS ? 0 : wn * 32 * FN);
        if constexpr (S::SLABS) {   // (columns: four k of 32 bits, eight of 16)
            ownM = MCOL ? ownM + wn * S::BM * 16 : ownM ^ wn * 16;
            ownN = NCOL ? ownN + wn * S::BN * 16 : ownN ^ wn * 16;
        }
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
        // Slabs read together.  One block of 32 x 32 a wavefront has too few MFMAs in a
        // slab to cover the reads of the next: it reads whole stages where it is alone on
        // its CU.
        constexpr int G = S::SLABS ? S::P : S::P > 1 ? 4 * S::P : 1, STEPS = S::SLABS ? 1 : 4 * S::P / G;
        i4 a[2][G][FM], b[2][G][FN];
        auto fragment = [&](auto column, auto size, int own, int s, int i) {
            constexpr int B = decltype(size)::value;
            own += (S::SLABS ? s : s / 4) * S::PANEL;
            s = S::SLABS ? 0 : s % 4;
            if constexpr (!decltype(column)::value) {
                return *reinterpret_cast<const i4 *>(lds + (own ^ (s * 16)) + i * 4096);
            } else if constexpr (sizeof(T) == 2) {
                constexpr int KB = B * 2;      // bytes of one k
                const int x = (own ^ (i * 64)) + 8 * s * KB;
                return join(quad(x), quad(x + 4 * KB));
            } else {
                i4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = *reinterpret_cast<const int *>(lds + own + (4 * s + j) * B * 4 + i * 128);
                return v;
            }
        };
        auto read_m = [&](int set, int g, int s, int i) {
            a[set][g][i] = fragment(std::bool_constant<MCOL>{}, std::integral_constant<int, S::BM>{}, atM, s + g, i);
        };
        auto read_n = [&](int set, int g, int s, int f) {
            b[set][g][f] = fragment(std::bool_constant<NCOL>{}, std::integral_constant<int, S::BN>{}, atN, s + g, f);
        };
        // the x-th fragment of a group of slabs, in the order that the MFMAs want them
        auto read_one = [&](int set, int s, int x) {
            const int g = x / (FM + FN), y = x - g * (FM + FN);
            if (y == 0) read_m(set, g, s, 0);
            else if (y <= FN) read_n(set, g, s, y - 1);
            else read_m(set, g, s, y - FN);
        };
        // no fence: a release would wait for the loads in flight as well
        auto barrier = []() { asm volatile("s_barrier" ::: "memory"); };
        // s_waitcnt operands: lgkmcnt 0 and that many loads left on their way
        auto wait_for = [](int left) constexpr { return (left & 15) | (left >> 4) << 14 | 7 << 4; };
        constexpr int kAll = wait_for(0), kFirst = wait_for((NS - 1) * J);
        constexpr int kNext = wait_for((NS - 2) * J);

        if (panels <= 0) return;
        constexpr int kFirst2 = wait_for((NS - 1) * J + AFTER);
        if (panels < NS) __builtin_amdgcn_s_waitcnt(kAll);
        else if (after) __builtin_amdgcn_s_waitcnt(kFirst2);
        else __builtin_amdgcn_s_waitcnt(kFirst);
        barrier();
        at_stage(0);
        constexpr int READS = G * (FM + FN), MFMAS = G * FM * FN;
#pragma unroll
        for (int x = 0; x < READS; ++x) read_one(0, 0, x);
        int stage = 0;
        // While a panel is multiplied the next NS - 1 are on their way; one barrier a
        // panel, after its last LDS read and before its last MFMAs.  The order is
        // written out: between two MFMAs a fragment of the next slab is read, and in
        // the last slab the loads go out as well, so that the matrix unit waits for
        // neither to be issued.
        auto panel = [&](auto more, auto load, auto set0) {
            static_for<STEPS>([&](auto step) {
                constexpr int s = decltype(step)::value, set = (decltype(set0)::value + s) & 1;
                constexpr bool last = s == STEPS - 1, reads = !last || more, loads = last && load;
                if constexpr (last && more) {
                    __builtin_amdgcn_s_waitcnt(load ? kNext : kAll);   // the next is there
                    barrier();
                    if constexpr (loads) issue_begin(stage);
                    stage = stage + 1 == NS ? 0 : stage + 1;
                    at_stage(stage);
                }
                static_for<MFMAS>([&](auto xc) {
                    constexpr int x = decltype(xc)::value, y = x / (FM * FN);
                    constexpr int i = x % (FM * FN) / FN, f = x % FN;
                    constexpr int r0 = x * READS / MFMAS, r1 = (x + 1) * READS / MFMAS;
                    constexpr int l0 = x * J / MFMAS, l1 = (x + 1) * J / MFMAS;
                    if constexpr (reads)
                        static_for<r1 - r0>([&](auto z) {
                            read_one(set ^ 1, last ? 0 : (s + 1) * G, r0 + decltype(z)::value);
                        });
                    acc[i][f] = product_mfma<T>(b[set][y][f], a[set][y][i], acc[i][f]);
                    if constexpr (loads)
                        static_for<l1 - l0>([&](auto z) { issue_one(l0 + decltype(z)::value); });
                    __builtin_amdgcn_sched_barrier(0);
                });
                if constexpr (loads) issue_end();
            });
        };
        const std::true_type yes;
        const std::false_type no;
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, 1> odd;
        const int n = panels;
        int t = 0;
        if constexpr (STEPS % 2 == 0) {
            for (; t + NS < n; ++t) panel(yes, yes, even);
            for (; t + 1 < n; ++t) panel(yes, no, even);
            panel(no, no, even);
        } else {
            // (the next panel is in the other set)
            for (; t + NS + 1 < n; t += 2) {
                panel(yes, yes, even);
                panel(yes, yes, odd);
            }
            if (t + NS < n) {
                panel(yes, yes, even);
                ++t;
                for (; t + 2 < n; t += 2) {
                    panel(yes, no, odd);
                    panel(yes, no, even);
                }
                if (t + 1 < n) {
                    panel(yes, no, odd);
                    panel(no, no, even);
                } else {
                    panel(no, no, odd);
                }
            } else {
                for (; t + 2 < n; t += 2) {
                    panel(yes, no, even);
                    panel(yes, no, odd);
                }
                if (t + 1 < n) {
                    panel(yes, no, even);
                    panel(no, no, odd);
                } else {
                    panel(no, no, even);
                }
            }
        }
    }
};

// ------------------------------------------------------------------- kernel ---

// Eight sums of a row -> the result: v += bias; Z; activation; dropout (its bits in w);
// v += residual; Y.
template <typename T>
__device__ __forceinline__ void product_finish(const Epilogue &o, int64_t row, int col, int left, float v[8],
                                               const Run<T, 8> &bias, const Run<T, 8> &residual,
                                               const uint32_t w[4])
{
    if (o.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += to_float(bias.v[i]);
    }
    if (o.Z) store8(reinterpret_cast<T *>(o.Z) + row * o.ldz + col, left, v);
    activate8(o.activation, v);
    if (o.drop.cut) drop8(v, o.drop, w);
    if (o.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += to_float(residual.v[i]);
    }
    if (o.wide) store8(reinterpret_cast<float *>(o.Y) + row * o.ldy + col, left, v);
    else store8(reinterpret_cast<T *>(o.Y) + row * o.ldy + col, left, v);
}
// The same where rows come one by one.
template <typename T>
__device__ __forceinline__ void product_store(const Epilogue &o, uint64_t key, int64_t row, int col,
                                              int left, float v[8])
{
    if (left <= 0) return;
    Run<T, 8> bias = {}, residual = {};
    uint32_t w[4] = {};
    if (o.bias) bias = raw8(reinterpret_cast<const T *>(o.bias) + col, left);
    if (o.residual) residual = raw8(reinterpret_cast<const T *>(o.residual) + row * o.ldr + col, left);
    if (o.drop.cut) philox((uint32_t)col >> 3, (uint32_t)row, o.drop.offset, key, w);
    product_finish<T>(o, row, col, left, v, bias, residual, w);
}

// offsets[e], brought into [0, rows]
__device__ __forceinline__ int expert_offset(const int32_t *offsets, int e, int rows)
{
    const int v = offsets[e];
    return v < 0 ? 0 : v > rows ? rows : v;
}

// Tiles of 1 << shift rows of a list of experts.  Expert e's begin with number
// (offsets[e] >> shift) + e, which leaves each as many as it needs and needs no table:
// the last e whose first is not behind `slot`.  What lies behind the last expert's
// rows counts as one more expert.
__device__ __forceinline__ int expert_of_slot(const int32_t *offsets, int experts, int rows, int slot,
                                              int shift)
{
    const int lane = (int)threadIdx.x & 63;
    int found = 0;
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int e = e0 + lane;
        const bool before = e <= experts && (expert_offset(offsets, e < experts ? e : experts, rows) >> shift) + e <= slot;
        const int n = __popcll(__ballot(before));
        found += n;
        if (n < 64) break;
    }
    return max(found - 1, 0);   // (expert 0's first is 0, or what lies before it is its own)
}

// A workgroup's tile: rows and columns of C, the expert, and its share of K.
struct TileAt {
    int row0, rows, col0, e, first, sum;
    bool empty;          // rows of no expert
    int shared, slice;   // number among the shared tiles (-1: whole), slice
};

// Unit `id` of the launch; false where nothing is to be done.  Workgroups go round
// the eight XCDs, each with an L2 of its own: the ids of one XCD are made neighbours,
// and neighbours walk bands of four tile rows, so that the tiles that are on an XCD
// together share operands.
template <typename S>
__device__ __forceinline__ bool product_tile(const ProductArgs &g, int groups, int id, TileAt &t)
{
    t.shared = -1;
    t.slice = 0;
    if (id >= g.full) {
        const int u = id - g.full;
        t.shared = (int)quotient((uint32_t)u, g.slices, g.slicesInv);
        t.slice = u - t.shared * g.slices;
        id = g.full + t.shared;
    } else if (id < (g.full & ~7)) {
        id = (id & 7) * (g.full >> 3) + (id >> 3);
    }
    const int inBand = 4 * g.tilesN;
    const int band = (int)quotient((uint32_t)id, inBand, g.bandInv), rest = id - band * inBand;
    const int height = min(g.bandRows - 4 * band, 4);
    const int tn = height == 4 ? rest >> 2 : height == 3 ? (int)__umulhi((uint32_t)rest, 0x55555556u)
                                                         : rest >> (height - 1);
    int tm = 4 * band + rest - tn * height;
    t.col0 = tn * S::BN;
    t.rows = g.m;
    t.first = 0;
    t.sum = g.k;
    t.e = 0;
    t.empty = false;
    if (groups == kByRows) {
        const int e = __builtin_amdgcn_readfirstlane(
            expert_of_slot(g.offsets, g.experts, g.m, tm, __builtin_ctz(S::BM)));
        const int begin = expert_offset(g.offsets, e, g.m);
        t.e = e;
        t.empty = e == g.experts;
        t.rows = t.empty ? g.m : expert_offset(g.offsets, e + 1, g.m);
        t.row0 = begin + (tm - (begin / S::BM + e)) * S::BM;
        return t.row0 < t.rows;
    }
    if (groups == kByK) {
        t.e = (int)quotient((uint32_t)tm, g.tilesM, g.tilesMInv);
        tm -= t.e * g.tilesM;
        t.first = expert_offset(g.offsets, t.e, g.k);
        t.sum = expert_offset(g.offsets, t.e + 1, g.k) - t.first;
    }
    t.row0 = tm * S::BM;
    return true;
}

// Adds up a shared tile; true for the workgroup that holds the sum.  The slices' sums
// go to slots in device memory in lane order (device-scope accesses, which pass by
// the XCD's own L2), and the last to arrive adds them in slice order: results do not
// depend on who that is.  Counters are zero between launches.
template <typename T, bool MCOL, bool NCOL, typename S>
__device__ __forceinline__ bool product_join(Product<T, MCOL, NCOL, S> &p, const ProductArgs &g,
                                             const TileAt &t, char *lds)
{
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid));   // (addresses made here, and not kept through all tiles)
    constexpr int N = S::THREADS, TILE = S::BM * S::BN;
    float *first = g.slots + (int64_t)t.shared * g.slices * TILE + tid;
    float *own = first + (int64_t)t.slice * TILE;
    static_for<S::FM * S::FN>([&](auto xc) {
        constexpr int x = decltype(xc)::value;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            __hip_atomic_store(own + (x * 16 + e) * N, p.acc[x / S::FN][x % S::FN][e], __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    });
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);   // vmcnt 0: the stores are done
    __syncthreads();
    int *last = reinterpret_cast<int *>(lds);
    if (tid == 0)
        *last = __hip_atomic_fetch_add(g.counters + t.shared, 1, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT) == g.slices - 1;
    __syncthreads();
    const bool mine = *last;
    __syncthreads();   // everyone has read it
    if (!mine) return false;
    if (tid == 0)
        __hip_atomic_store(g.counters + t.shared, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    static_for<S::FM * S::FN>([&](auto xc) {
        constexpr int x = decltype(xc)::value;
        f16v &acc = p.acc[x / S::FN][x % S::FN];
        for (int s0 = 0; s0 < g.slices; s0 += 2) {   // two slices' loads together
            float v[2][16];
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s0 + s < g.slices)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        v[s][e] = __hip_atomic_load(first + (int64_t)(s0 + s) * TILE + (x * 16 + e) * N,
                                                    __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s0 + s < g.slices)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[e] = s0 + s == 0 ? v[s][e] : acc[e] + v[s][e];
        }
        __builtin_amdgcn_sched_barrier(0);
    });
    return true;
}

// Sends the loads of a tile's first panels.
template <typename T, ProductForm FORM, typename S>
__device__ __forceinline__ void product_begin(Product<T, FORM == kColumnsColumns, FORM != kRowsRows, S> &p,
                                              const ProductArgs &g, int groups, const TileAt &t,
                                              char *dyn_lds)
{
    constexpr bool MCOL = FORM == kColumnsColumns, NCOL = FORM != kRowsRows;
    constexpr int KP = S::P * 128 / (int)sizeof(T);   // of a stage
    const bool gathered = FORM == kRowsRows && g.order;
    Side M, N;
    M.ld = g.ldm;
    N.ld = g.ldn;
    N.p = g.N + (groups == kByRows ? (int64_t)t.e * g.stepN : 0);
    if constexpr (MCOL) {
        M.p = g.M + (int64_t)t.first * g.ldm + (int64_t)t.row0 * sizeof(T);
        M.count = g.fullM - t.row0;
        M.extent = t.sum;
    } else {
        M.p = g.M + (gathered ? 0 : (int64_t)t.row0 * g.ldm);
        M.count = t.rows - t.row0;
        M.extent = g.kM;
    }
    if constexpr (NCOL) {
        N.p += (int64_t)t.first * g.ldn + (int64_t)t.col0 * sizeof(T);
        N.count = g.fullN - t.col0;
        N.extent = t.sum;
    } else {
        N.p += (int64_t)t.col0 * g.ldn;
        N.count = g.n - t.col0;
        N.extent = g.kN;
    }
    const int32_t *order = g.order + (gathered ? t.row0 : 0);
    auto rowM = [&](int r) {
        if (FORM == kRowsRows && gathered) {
            const uint32_t id = min((uint32_t)order[r], (uint32_t)g.m - 1);
            r = (int)quotient(id, g.choices, g.choicesInv);
        }
        return (uint32_t)(r * g.ldm);
    };
    int panels = t.empty ? 0 : (t.sum + KP - 1) / KP;
    if (t.shared >= 0) {
        // A gradient in tiles of 64 has stages of one panel or two by how many workgroups
        // its launch has, the other gradient's among them.  Its slices are whole pairs of
        // panels in both, so that its sums do not depend on what else is wanted.
        constexpr int CUT = FORM != kRowsRows && S::BM == 64 ? 2 / S::P : 1;
        const int cuts = (panels + CUT - 1) / CUT;
        const int t0 = CUT * (int)quotient((uint32_t)(cuts * t.slice), g.slices, g.slicesInv);
        const int t1 = CUT * (int)quotient((uint32_t)(cuts * (t.slice + 1)), g.slices, g.slicesInv);
        panels = min(t1, panels) - t0;
        M.p += t0 * (MCOL ? KP * M.ld : S::P * 128);
        N.p += t0 * (NCOL ? KP * N.ld : S::P * 128);
        M.extent -= t0 * KP;
        N.extent -= t0 * KP;
    }
    p.begin(dyn_lds, M, N, rowM, panels);
}

// A tile's epilogue.
template <typename T, ProductForm FORM>
__device__ __forceinline__ Epilogue product_epilogue(const ProductArgs &g, int groups, const TileAt &t)
{
    Epilogue o = g.out;
    if constexpr (FORM != kRowsRows) {   // gradients are the sums themselves
        o.bias = o.residual = nullptr;
        o.Z = nullptr;
        o.activation = GETT_ACTIVATION_NONE;
        o.drop.cut = 0;
    }
    if (groups == kByRows && o.bias) o.bias += (int64_t)t.e * g.n * sizeof(T);
    if (groups == kByK) o.Y += (int64_t)t.e * g.stepN * (o.wide ? 4 : sizeof(T));
    if (t.empty) {
        o.bias = nullptr;
        o.activation = GETT_ACTIVATION_NONE;
    }
    return o;
}

// Workgroups take tile after tile.  A tile's loads begin before the results of the
// one before are written: its first panels arrive while those leave.
template <typename T, ProductForm FORM, typename S>
__device__ __forceinline__ void product_work(const ProductArgs &g, int groups, int id, int stride,
                                             char *dyn_lds)
{
    Product<T, FORM == kColumnsColumns, FORM != kRowsRows, S> p;
    p.locate();
    auto begin = [&](const TileAt &t) { product_begin<T, FORM, S>(p, g, groups, t, dyn_lds); };
    const uint64_t key = g.out.drop.cut ? g.out.drop.key() : 0;
    const int lane = (int)threadIdx.x & 63;
    char *mine = dyn_lds + S::NS * S::STAGE + (p.wm * S::WN + p.wn) * S::RESULTS;
    TileAt t;
    bool there = false;
    for (; id < g.units && !there; id += stride) there = product_tile<S>(g, groups, id, t);
    if (!there) return;
    begin(t);
    bool after = false;   // a whole tile's stores came after the loads
    while (true) {
        constexpr int STORES = S::FM * S::FN * (sizeof(T) == 2 ? 2 : 4);
        p.clear();
        p.template run<(S::NS - 1) * S::J + STORES < 64 ? STORES : 0>(dyn_lds, after);
        __syncthreads();
        TileAt now = t;
        there = false;
        for (; id < g.units && !there; id += stride) there = product_tile<S>(g, groups, id, t);
        if (there) begin(t);
        after = false;
        if (now.shared >= 0 &&
            !product_join(p, g, now, dyn_lds + S::NS * S::STAGE)) {
            if (!there) return;
            continue;
        }
        const Epilogue o = product_epilogue<T, FORM>(g, groups, now);
        after = now.row0 + S::BM <= now.rows && now.col0 + S::BN <= g.n;
        // The results go through LDS, 16 rows of a wavefront at a time, so that one
        // loop (and not one copy of the epilogue for each register) takes them, whole
        // lines of C each time.  Piece x of row r lies at x ^ r.  A step's rows of
        // the residual are on their way a step before (8192 x 8192 x 4096 in bf16 with
        // bias, Z, GELU, dropout and residual: 625 us with each waiting for its own, 589
        // so).  Such a product takes 556 us, one without any of it 440: the residual's
        // and Z's bytes and the random bits (about 25 us) are not hidden under the
        // MFMAs, of which the same wavefronts have no more to do by then.
        constexpr int W = S::W, PER = W / 8, ROWS = 64 / PER;   // runs of a row, rows a pass
        constexpr int PASSES = 16 / ROWS, STEPS = 2 * S::FM;
        constexpr int SWAP = W / 4 < 16 ? W / 4 - 1 : 15;
        const int run = lane % PER, rowIn = lane / PER;
        const int c = now.col0 + p.wn * W + 8 * run, left = g.n - c;
        const int row0 = now.row0 + p.wm * 32 * S::FM + rowIn;
        Run<T, 8> bias = {}, ahead[PASSES] = {};
        PhiloxColumn column = {};
        if (o.bias && left > 0) bias = raw8(reinterpret_cast<const T *>(o.bias) + c, left);
        if (o.drop.cut) column = philox_column((uint32_t)c >> 3, o.drop.offset, key);
        auto fetch = [&](int step) {
#pragma unroll
            for (int y = 0; y < PASSES; ++y) {
                const int64_t row = row0 + 16 * step + ROWS * y;
                if (o.residual && left > 0 && row < now.rows)
                    ahead[y] = raw8(reinterpret_cast<const T *>(o.residual) + row * o.ldr + c, left);
            }
        };
        fetch(0);
#pragma unroll 1
        for (int step = 0; step < STEPS; ++step) {
            static_for<S::FM>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                if (step >> 1 != i || p.q >> 4 != (step & 1)) return;
#pragma unroll
                for (int f = 0; f < S::FN; ++f)
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const int piece = 8 * f + 2 * a + p.h;
                        const f16v &v = p.acc[i][f];
                        *reinterpret_cast<f4 *>(mine + (p.q & 15) * W * 4 +
                                                (piece ^ (p.q & SWAP)) * 16) =
                            f4{v[4 * a], v[4 * a + 1], v[4 * a + 2], v[4 * a + 3]};
                    }
            });
            wave_exchange();
            Run<T, 8> residual[PASSES];
            float v[PASSES][8];
#pragma unroll
            for (int y = 0; y < PASSES; ++y) {
                const int r = rowIn + ROWS * y;
                const f4 lo = *reinterpret_cast<const f4 *>(mine + r * W * 4 + ((2 * run) ^ (r & SWAP)) * 16);
                const f4 hi = *reinterpret_cast<const f4 *>(mine + r * W * 4 + ((2 * run + 1) ^ (r & SWAP)) * 16);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    v[y][x] = lo[x];
                    v[y][4 + x] = hi[x];
                }
                residual[y] = ahead[y];
            }
            wave_exchange();   // (all are read)
            if (step + 1 < STEPS) fetch(step + 1);
#pragma unroll
            for (int y = 0; y < PASSES; ++y) {
                const int row = row0 + 16 * step + ROWS * y;
                if (row >= now.rows || left <= 0) continue;
                uint32_t w[4] = {};
                if (o.drop.cut) philox_row(column, (uint32_t)row, w);
                product_finish<T>(o, row, c, left, v[y], bias, residual[y], w);
            }
        }
        if (!there) return;
    }
}

// A block of 32 x 32 whose wavefronts share K: their four sums are added in the order of
// the slabs, and a row's runs of eight columns leave from four lanes.
template <typename T, ProductForm FORM, typename S>
__device__ __forceinline__ void product_slabs(const ProductArgs &g, int groups, int id, char *dyn_lds)
{
    TileAt t;
    if (!product_tile<S>(g, groups, id, t)) return;
    Product<T, FORM == kColumnsColumns, FORM != kRowsRows, S> p;
    p.locate();
    product_begin<T, FORM, S>(p, g, groups, t, dyn_lds);
    p.clear();
    p.template run<0>(dyn_lds, false);
    __syncthreads();
    float *sums = reinterpret_cast<float *>(dyn_lds);
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const f16v &v = p.acc[0][0];
        *reinterpret_cast<f4 *>(sums + (p.wn * 32 + p.q) * S::ROW + 8 * a + 4 * p.h) =
            f4{v[4 * a], v[4 * a + 1], v[4 * a + 2], v[4 * a + 3]};
    }
    __syncthreads();
    const int r = (int)threadIdx.x >> 2, c = ((int)threadIdx.x & 3) * 8;
    if (r >= 32 || t.row0 + r >= t.rows) return;
    float v[8] = {};
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const f4 lo = *reinterpret_cast<const f4 *>(sums + (y * 32 + r) * S::ROW + c);
        const f4 hi = *reinterpret_cast<const f4 *>(sums + (y * 32 + r) * S::ROW + c + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] += lo[i];
            v[4 + i] += hi[i];
        }
    }
    const Epilogue o = product_epilogue<T, FORM>(g, groups, t);
    product_store<T>(o, o.drop.cut ? o.drop.key() : 0, t.row0 + r, t.col0 + c, g.n - t.col0 - c, v);
}

template <typename T, ProductForm FORM, typename S>
__global__ __launch_bounds__(S::THREADS) void product_slabs_kernel(ProductArgs g, int groups)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    product_slabs<T, FORM, S>(g, groups, (int)blockIdx.x, dyn_lds);
}
template <typename T, typename S>
__global__ __launch_bounds__(S::THREADS) void product_slabs_pair_kernel(ProductArgs x, int groupsX, int blocks,
                                                                        ProductArgs w, int groupsW)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    const int id = (int)blockIdx.x;
    if (id < blocks) product_slabs<T, kRowsColumns, S>(x, groupsX, id, dyn_lds);
    else product_slabs<T, kColumnsColumns, S>(w, groupsW, id - blocks, dyn_lds);
}

template <typename T, ProductForm FORM, typename S>
__global__ __launch_bounds__(S::THREADS) void product_kernel(ProductArgs g, int groups)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    product_work<T, FORM, S>(g, groups, (int)blockIdx.x, (int)gridDim.x, dyn_lds);
}

// The two products of a backward pass in one launch: `blocks` workgroups for dz w, the
// others for dz^T x.  Those of the second begin where those of the first leave off
// (two launches, one: 12 experts' 903 rows of 500 x 333 in fp32 28, 21 us; 32 experts'
// 32768 rows of 2048 x 1536 in bf16 576, 548).
template <typename T, typename S>
__global__ __launch_bounds__(S::THREADS) void product_pair_kernel(ProductArgs x, int groupsX, int blocks,
                                                                  ProductArgs w, int groupsW)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    const int id = (int)blockIdx.x;
    if (id < blocks) product_work<T, kRowsColumns, S>(x, groupsX, id, blocks, dyn_lds);
    else product_work<T, kColumnsColumns, S>(w, groupsW, id - blocks, (int)gridDim.x - blocks, dyn_lds);
}

}  // namespace gett
