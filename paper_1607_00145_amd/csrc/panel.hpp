// panel.hpp -- the product core of the matrix operators (device code):
// acc[i][j] = sum over K of row i of one operand times row j of another.
//
// Both operands are cut along K into panels of 128 bytes a row; a panel's rows
// follow one another in memory, panel after panel (row after row, the rows of
// a panel would lie a power of two apart and share few L2 channels: 181 us for
// the half-precision product 4096^3 that takes XXX this way).  A row's 128 bytes
// are eight 16-byte pieces, taken as four slabs of two pieces, slab s the
// pieces s and s + 4.  One MFMA 32 x 32 takes a slab of 32 rows of each operand
// (16 bytes a lane: lane l gives row l % 32, piece 4 (l / 32) + s), whatever
// the bytes stand for:
//   Mx     64 4-bit numbers a slab, and a scale per piece (32 numbers):
//          v_mfma_scale 32x32x64;
//   Half   16 halves a slab: v_mfma 32x32x16 f16;
//   Split  numbers in two parts (x = hi + lo, 22 bits), eight high parts in an
//          even piece and their low parts in the odd piece after it: slabs 2 j
//          and 2 j + 1 give hi hi' + hi lo' + lo hi', three MFMAs; lo lo' is
//          below the sums' own rounding.
// All of them take as long for 32 bytes of their rows, so one tile geometry
// serves them.  (32 x 32 and not 16 x 16: from one wavefront per SIMD the
// instructions alone reach 9.3 PFLOP/s in 4 bits and 2.4 in halves, the 16 x 16
// ones 5.5 and 1.5.)
//
// Rows of a lane.  Lane r = l % 32 of an operand with F fragments holds rows
// F r .. F r + F - 1, one per fragment.  So a lane's F scales are neighbours
// (one load), and the results of a lane are F neighbours along both
// directions: C is stored in vectors along either of its dimensions.
//
// LDS.  Panels go from memory straight into LDS (16 bytes a lane, 1 KB an
// instruction: eight whole rows, each a full line of 128 bytes).  A pair of
// rows takes 256 bytes, sixteen places; piece p of the pair's second row counts
// as piece 8 + p, and piece p lies at place p ^ (row / F mod 16) (F = 1:
// p ^ (row / 2 mod 8)).  Sixteen neighbouring lanes read one piece of sixteen
// different row / F, so they fall on sixteen different places: 210 bytes a
// clock and CU, the rate of reads that follow one another being 227.
//
// Pipeline, two stages of LDS.  While panel t is multiplied, panel t + 1 is
// on its way; one barrier per panel, after the last LDS read of t and before
// its last MFMAs:
//   read slabs g of t | MFMAs of slabs g - 1         (for each group of slabs)
//   wait for t + 1; barrier; loads of t + 2 into t's stage
//   read the first group of t + 1 | MFMAs of the last group of t
#pragma once
#include <type_traits>

#include "matrix.hpp"

namespace gett {

typedef __attribute__((address_space(1))) void matrix_global;
typedef __attribute__((address_space(3))) void matrix_lds;

enum PanelKind { kPanelMx, kPanelHalf, kPanelSplit };

template <int N, int I = 0, typename F> __device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, I + 1>(f);
    }
}

template <int FM_, int FN_, int WM_, int WN_> struct PanelShape {
    static constexpr int FM = FM_, FN = FN_, WM = WM_, WN = WN_;   // fragments, wavefronts
    static constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int STAGE = (BM + BN) * 128;
    static constexpr int LDS = 2 * STAGE;
    static constexpr int J = (BM + BN) / 8 / NW;   // load instructions a wavefront per panel
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "whole instructions per operand");
};

// One operand of a tile: rows [row0, row0 + tile rows) of a matrix of `rows`
// rows.  Rows past the last read the last one again; their results are not
// stored.
struct PanelOperand {
    const uint8_t *data;     // panel 0, row 0
    const uint8_t *scales;   // Mx: the packed scales
    int rows, row0;
    // rows row0 ... of panel t, and nothing behind the panel's last row
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t panel(int t) const
    {
        const uint8_t *p = data + ((int64_t)t * rows + row0) * 128;
        const int64_t bytes = (int64_t)(rows - row0) * 128;
        return __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t *>(p), 0, (int)(uint32_t)(bytes < 0xffffffffll ? bytes : 0xffffffffll),
            0x00027000);
    }
};

typedef float f16v __attribute__((ext_vector_type(16)));

template <int OA, int OB>
__device__ __forceinline__ f4 mfma_mx16(i4 a, i4 b, f4 c, int sa, int sb)
{
    const i8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, OA, sa, OB, sb);
}
template <int O>
__device__ __forceinline__ f16v mfma_mx32(i4 a, i4 b, f16v c, int sa, int sb)
{
    const i8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, O, sa, O, sb);
}
__device__ __forceinline__ f16v mfma_half(i4 a, i4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// The scales of a lane's F rows and four slabs, a word per row.
template <int F> struct PanelScales {
    int v[F];
    __device__ __forceinline__ void load(const uint8_t *p)
    {
        if constexpr (F == 1) {
            v[0] = *reinterpret_cast<const int *>(p);
        } else {
            typedef int vec __attribute__((ext_vector_type(F)));
            const vec x = *reinterpret_cast<const vec *>(p);
#pragma unroll
            for (int i = 0; i < F; ++i) v[i] = x[i];
        }
    }
};

// place of piece p (8 + p in the second row of its pair) of a row of lane r
template <int F> __device__ __forceinline__ int panel_place(int p, int r)
{
    return p ^ (F > 1 ? r & 15 : (r >> 1) & 7);
}

template <int KIND, typename S> struct Panel {
    static constexpr int FM = S::FM, FN = S::FN;
    static constexpr int G = KIND == kPanelSplit ? 2 : 1;   // slabs read together
    f16v acc[FM][FN];
    int r, h, wm, wn;

    __device__ __forceinline__ void init()
    {
        const int tid = (int)threadIdx.x;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        r = tid & 31;
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
    // row (column) of the tile that accumulator element acc[i][j][e] stands for
    __device__ __forceinline__ int row(int i, int e) const
    {
        return wm * 32 * FM + FM * (8 * (e >> 2) + 4 * h + (e & 3)) + i;
    }
    __device__ __forceinline__ int col(int j) const { return wn * 32 * FN + FN * r + j; }

    // panels [t0, t1) of both operands; `lds` holds S::LDS bytes
    __device__ __forceinline__ void run(char *lds, const PanelOperand &A, const PanelOperand &B,
                                        int t0, int t1)
    {
        constexpr int NW = S::NW, J = S::J, JA = S::BM / 8 / NW;
        const int lane = (int)threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        // this lane's piece of each load: 16 places of a pair of rows
        uint32_t off[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const bool isA = j < JA;
            const int F = isA ? FM : FN;
            const int pair = ((isA ? j : j - JA) * NW + wave) * 4 + (lane >> 4);
            const int x = 2 * pair / F;   // the lane r of the pair's rows (F = 1: of the first)
            const int p = (lane & 15) ^ (F > 1 ? x & 15 : (x >> 1) & 7);
            const int row = 2 * pair + (p >> 3), last = (isA ? A.rows - A.row0 : B.rows - B.row0) - 1;
            off[j] = (uint32_t)(row < last ? row : last) * 128 + (uint32_t)(p & 7) * 16;
        }
        // buffer loads: a lane's offset stays, the panel's base is a scalar
        int at = t0;
        auto issue = [&](int stage) {
            const __amdgpu_buffer_rsrc_t ra = A.panel(at), rb = B.panel(at);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                char *dst = lds + stage * S::STAGE + (j < JA ? 0 : S::BM * 128) +
                            ((j < JA ? j : j - JA) * NW + wave) * 1024;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(j < JA ? ra : rb, (matrix_lds *)dst, 16,
                                                         (int)off[j], 0, 0, 0);
            }
            ++at;
        };
        // scales of panel t: a lane's are neighbours (gett_matrix.h)
        PanelScales<FM> sa, nextA;
        PanelScales<FN> sb, nextB;
        const uint8_t *pa = nullptr, *pb = nullptr;
        int64_t stepA = 0, stepB = 0;
        if constexpr (KIND == kPanelMx) {
            const int64_t RA = mx_scale_rows(A.rows), RB = mx_scale_rows(B.rows);
            int64_t rowA = A.row0 + wm * 32 * FM + FM * r, rowB = B.row0 + wn * 32 * FN + FN * r;
            rowA = rowA < RA - FM ? rowA : RA - FM;
            rowB = rowB < RB - FN ? rowB : RB - FN;
            stepA = RA * kTileBlocks;
            stepB = RB * kTileBlocks;
            pa = A.scales + t0 * stepA + (h * RA + rowA) * 4;
            pb = B.scales + t0 * stepB + (h * RB + rowB) * 4;
        }
        auto scales = [&](PanelScales<FM> &x, PanelScales<FN> &y) {
            if constexpr (KIND == kPanelMx) {
                x.load(pa);
                y.load(pb);
                pa += stepA;
                pb += stepB;
            }
        };

        // LDS reads: rows F r + i of the wavefront's part, piece 4 h + s.  The
        // place is an exclusive or, so an address is the lane's own for piece
        // 4 h of an even row, exclusive or a constant.  It is made anew per
        // panel (the compiler would keep all of them in registers).
        const int ownA = (wm * 32 * FM + FM * r) / 2 * 256 +
                         panel_place<FM>(4 * h + (FM == 1 ? 8 * (r & 1) : 0), r) * 16;
        const int ownB = S::BM * 128 + (wn * 32 * FN + FN * r) / 2 * 256 +
                         panel_place<FN>(4 * h + (FN == 1 ? 8 * (r & 1) : 0), r) * 16;
        i4 a[2][G][FM], b[2][G][FN];
        int atA = ownA, atB = ownB;
        auto at_stage = [&](int stage) {
            atA = ownA + stage * S::STAGE;
            atB = ownB + stage * S::STAGE;
            asm volatile("" : "+v"(atA), "+v"(atB));
        };
        auto read = [&](int set, int s) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    a[set][g][i] = *reinterpret_cast<const i4 *>(
                        lds + (atA ^ ((8 * (i & 1) + s + g) * 16)) + (i >> 1) * 256);
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    b[set][g][j] = *reinterpret_cast<const i4 *>(
                        lds + (atB ^ ((8 * (j & 1) + s + g) * 16)) + (j >> 1) * 256);
            }
        };
        auto mma = [&](int set, auto slab) {
            constexpr int s = decltype(slab)::value;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    if constexpr (KIND == kPanelMx)
                        acc[i][j] = mfma_mx32<s>(a[set][0][i], b[set][0][j], acc[i][j], sa.v[i],
                                                 sb.v[j]);
                    else
                        acc[i][j] = mfma_half(a[set][0][i], b[set][0][j], acc[i][j]);
                }
            if constexpr (KIND == kPanelSplit) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = mfma_half(a[set][0][i], b[set][1][j], acc[i][j]);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = mfma_half(a[set][1][i], b[set][0][j], acc[i][j]);
            }
        };
        // no fence: a release would wait for the loads in flight as well
        auto barrier = []() { asm volatile("s_barrier" ::: "memory"); };
        constexpr int kAllLoads = 7 << 4;   // vmcnt 0, lgkmcnt 0
        constexpr int STEPS = 4 / G;        // groups of slabs per panel

        const int n = t1 - t0;
        if (n <= 0) return;
        issue(0);
        scales(sa, sb);
        __builtin_amdgcn_s_waitcnt(kAllLoads);
        barrier();
        if (n > 1) issue(1);
        at_stage(0);
        read(0, 0);
        // one panel; `more`: another follows, `load`: and one after that
        auto panel = [&](int stage, auto more, auto load) {
            if constexpr (more) scales(nextA, nextB);
            static_for<STEPS>([&](auto step) {
                constexpr int s = decltype(step)::value;
                if constexpr (s + 1 < STEPS) {
                    read((s + 1) & 1, (s + 1) * G);
                } else if constexpr (more) {
                    __builtin_amdgcn_s_waitcnt(kAllLoads);   // t + 1 loaded, t read
                    barrier();
                    if constexpr (load) issue(stage);
                    at_stage(stage ^ 1);
                    read((s + 1) & 1, 0);
                }
                mma(s & 1, std::integral_constant<int, s * G>{});
                // the reads of one group lie among the first MFMAs of the one
                // before, and stay there
                constexpr int READS = G * (FM + FN);
                constexpr int MFMAS = FM * FN * (KIND == kPanelSplit ? 3 : 1);
                if constexpr (s + 1 < STEPS || more) {
                    static_for<(READS < MFMAS ? READS : MFMAS)>([](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        __builtin_amdgcn_sched_group_barrier(0x100, i + 1 < MFMAS ? 1 : READS - i, 0);
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (KIND == kPanelMx && more) {
                sa = nextA;
                sb = nextB;
            }
        };
        const std::true_type yes;
        const std::false_type no;
        int t = 0;
        for (; t + 2 < n; ++t) panel(t & 1, yes, yes);
        if (t + 1 < n) {
            panel(t & 1, yes, no);
            ++t;
        }
        panel(t & 1, no, no);
    }
};

// The tile of workgroup `bid` of `tilesM` x `tilesN`.  Workgroups go round
// the eight XCDs, each with an L2 of its own: the ids of one XCD are made
// neighbours, and they walk bands of `band` tile rows, column by column, so
// that the tiles resident on an XCD share operand rows.
__device__ __forceinline__ void panel_tile(int bid, int tilesM, int tilesN, int band, int &tm,
                                           int &tn)
{
    const int total = tilesM * tilesN, per = total >> 3;
    int id = bid;
    if (bid < per * 8) id = (bid & 7) * per + (bid >> 3);
    const int inBand = band * tilesN, b = id / inBand, rest = id % inBand;
    const int height = tilesM - b * band < band ? tilesM - b * band : band;
    tm = b * band + rest % height;
    tn = rest / height;
}

}  // namespace gett
