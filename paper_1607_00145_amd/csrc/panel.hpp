// panel.hpp -- the product core of the matrix operators (device code):
// acc[i][j] = sum over K of row i of one operand times row j of another.
//
// Both operands lie row after row with K along the row, cut into panels of
// 128 bytes, and a panel holds two slabs of 64 bytes.  One MFMA 16 x 16 takes
// a slab of 16 rows of each operand (16 bytes a lane: lane l gives row l % 16,
// piece 2 (l / 16) + s), whatever the bytes stand for:
//   Mx     128 4-bit numbers a slab, and a scale per 16-byte piece (32
//          numbers): v_mfma_scale 16x16x128;
//   Half   32 halves a slab: v_mfma 16x16x32 f16;
//   Split  32 numbers in two parts each (x = hi + lo, 22 bits), the high parts
//          in slab 0 and the low ones in slab 1: hi hi' + hi lo' + lo hi', three
//          MFMAs; lo lo' is below the sums' own rounding.
// All of them take 16 cycles for 64 bytes of two rows, so one tile geometry
// serves them.
//
// Rows of a lane.  Lane r = l % 16 of an operand with F fragments holds rows
// F r .. F r + F - 1, one per fragment.  So a lane's F scales are neighbours
// (one load), and the results of a lane are F neighbours along both
// directions: C is stored in vectors along either of its dimensions.
// A sum may take K in any order that both operands share; with this one a
// lane's two scales are neighbours too.
//
// LDS.  Panels go from memory straight into LDS (16 bytes a lane, 1 KB an
// instruction: eight whole rows, each a full line of 128 bytes).  A pair of
// rows takes 256 bytes, sixteen pieces; piece p of the pair lies at
// p ^ (row / F mod 16).  The sixteen lanes of a read take one piece of
// sixteen different row / F, so they fall on sixteen different places, and
// any eight neighbours of them on different ones mod 8: no conflicts with 32
// or 64 banks.
//
// Pipeline, two stages of LDS.  While panel t is multiplied, panel t + 1 is
// on its way; per panel one barrier, placed after the last LDS read of t:
//   read slab 1 of t | MFMAs of slab 0
//   wait for t + 1; barrier; loads of t + 2 into t's stage
//   read slab 0 of t + 1 | MFMAs of slab 1
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
    static constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int STAGE = (BM + BN) * 128;
    static constexpr int LDS = 2 * STAGE;
    static constexpr int J = (BM + BN) / 8 / NW;   // load instructions a wavefront per panel
    static_assert(FM % 2 == 0 && FN % 2 == 0, "a pair of rows belongs to one lane");
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "whole instructions per operand");
};

// One operand of a tile: rows [row0, row0 + tile rows) of a matrix of `rows`
// rows, `pitch` bytes apart (a multiple of 128).  Rows past the last read the
// last one again; their results are not stored.
struct PanelOperand {
    const uint8_t *data;     // row 0
    const uint8_t *scales;   // Mx: the packed scales
    int64_t pitch;
    int rows, row0;
    __device__ __forceinline__ const uint8_t *tile() const { return data + (int64_t)row0 * pitch; }
};

template <int OA, int OB>
__device__ __forceinline__ f4 mfma_mx(i4 a, i4 b, f4 c, int sa, int sb)
{
    const i8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, OA, sa, OB, sb);
}
__device__ __forceinline__ f4 mfma_half(i4 a, i4 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// The scales of a lane's F rows and two blocks: 2 F bytes, fragment by
// fragment.
template <int F> struct PanelScales {
    static constexpr int N = F / 2;
    int v[N];
    __device__ __forceinline__ void load(const uint8_t *p)
    {
        typedef int vec __attribute__((ext_vector_type(N)));
        if constexpr (N == 1) {
            v[0] = *reinterpret_cast<const int *>(p);
        } else {
            const vec x = *reinterpret_cast<const vec *>(p);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = x[i];
        }
    }
};

template <int KIND, typename S> struct Panel {
    static constexpr int FM = S::FM, FN = S::FN;
    f4 acc[FM][FN];
    int lane, r, q, wm, wn;

    __device__ __forceinline__ void init()
    {
        const int tid = (int)threadIdx.x;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        lane = tid & 63;
        r = lane & 15;
        q = lane >> 4;
        wm = wave / S::WN;
        wn = wave % S::WN;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // row (column) of the tile that accumulator element acc[i][j][e] stands for
    __device__ __forceinline__ int row(int i, int e) const
    {
        return wm * 16 * FM + FM * (4 * q + e) + i;
    }
    __device__ __forceinline__ int col(int j) const { return wn * 16 * FN + FN * r + j; }

    // panels [t0, t1) of both operands; `lds` holds S::LDS bytes
    __device__ __forceinline__ void run(char *lds, const PanelOperand &A, const PanelOperand &B,
                                        int t0, int t1)
    {
        constexpr int NW = S::NW, J = S::J, JA = S::BM / 8 / NW;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        // this lane's piece of each load: 16 pieces of a pair of rows
        uint32_t off[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const bool isA = j < JA;
            const int F = isA ? FM : FN;
            const int pair = ((isA ? j : j - JA) * NW + wave) * 4 + (lane >> 4);
            const int p = (lane & 15) ^ ((2 * pair / F) & 15);
            const int row = 2 * pair + (p >> 3), last = (isA ? A.rows - A.row0 : B.rows - B.row0) - 1;
            off[j] = (uint32_t)((row < last ? row : last) * (uint32_t)(isA ? A.pitch : B.pitch) +
                                (uint32_t)(p & 7) * 16);
        }
        const uint8_t *ga = A.tile() + (int64_t)t0 * 128, *gb = B.tile() + (int64_t)t0 * 128;
        auto issue = [&](int stage) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const uint8_t *src = (j < JA ? ga : gb) + off[j];
                char *dst = lds + stage * S::STAGE + (j < JA ? 0 : S::BM * 128) +
                            ((j < JA ? j : j - JA) * NW + wave) * 1024;
                __builtin_amdgcn_global_load_lds((matrix_global *)src, (matrix_lds *)dst, 16, 0, 0);
            }
            ga += 128;
            gb += 128;
        };
        // scales of panel t: a lane's are neighbours (gett_matrix.h)
        PanelScales<FM> sa, sa1, sa2;
        PanelScales<FN> sb, sb1, sb2;
        const uint8_t *pa = nullptr, *pb = nullptr;
        int64_t stepA = 0, stepB = 0;
        if constexpr (KIND == kPanelMx) {
            const int64_t RA = mx_scale_rows(A.rows), RB = mx_scale_rows(B.rows);
            int64_t ra = A.row0 + wm * 16 * FM + FM * r, rb = B.row0 + wn * 16 * FN + FN * r;
            ra = ra < RA - FM ? ra : RA - FM;
            rb = rb < RB - FN ? rb : RB - FN;
            stepA = RA * kTileBlocks;
            stepB = RB * kTileBlocks;
            pa = A.scales + t0 * stepA + (q * RA + ra) * 2;
            pb = B.scales + t0 * stepB + (q * RB + rb) * 2;
        }
        auto scales = [&](PanelScales<FM> &x, PanelScales<FN> &y) {
            if constexpr (KIND == kPanelMx) {
                x.load(pa);
                y.load(pb);
                pa += stepA;
                pb += stepB;
            }
        };

        // LDS addresses: piece 2 q + s of a lane's even and odd rows
        const int baseA = (wm * 8 * FM + FM / 2 * r) * 256;
        const int baseB = S::BM * 128 + (wn * 8 * FN + FN / 2 * r) * 256;
        int at[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < 2; ++s) at[h][s] = ((8 * h + 2 * q + s) ^ r) * 16;
        auto readA = [&](i4 (&f)[FM], int stage, int s) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
                f[i] = *reinterpret_cast<const i4 *>(lds + stage * S::STAGE + baseA +
                                                     at[i & 1][s] + (i >> 1) * 256);
        };
        auto readB = [&](i4 (&f)[FN], int stage, int s) {
#pragma unroll
            for (int i = 0; i < FN; ++i)
                f[i] = *reinterpret_cast<const i4 *>(lds + stage * S::STAGE + baseB +
                                                     at[i & 1][s] + (i >> 1) * 256);
        };
        auto mma = [&](const i4 (&a)[FM], const i4 (&b)[FN], auto slab) {
            constexpr int s = decltype(slab)::value;
            static_for<FM>([&](auto ic) {
                static_for<FN>([&](auto jc) {
                    constexpr int i = decltype(ic)::value, j = decltype(jc)::value;
                    if constexpr (KIND == kPanelMx)
                        acc[i][j] = mfma_mx<2 * (i & 1) + s, 2 * (j & 1) + s>(
                            a[i], b[j], acc[i][j], sa.v[i >> 1], sb.v[j >> 1]);
                    else
                        acc[i][j] = mfma_half(a[i], b[j], acc[i][j]);
                });
            });
        };
        // no fence: a release would wait for the loads in flight as well
        auto barrier = []() { asm volatile("s_barrier" ::: "memory"); };
        constexpr int kAllLoads = 7 << 4;   // vmcnt 0, lgkmcnt 0

        const std::integral_constant<int, 0> s0;
        const std::integral_constant<int, 1> s1;
        const int n = t1 - t0;
        if (n <= 0) return;
        i4 a0[FM], b0[FN], a1[FM], b1[FN];
        issue(0);
        scales(sa, sb);
        __builtin_amdgcn_s_waitcnt(kAllLoads);
        barrier();
        if (n > 1) {
            issue(1);
            scales(sa1, sb1);
        }
        readA(a0, 0, 0);
        readB(b0, 0, 0);
        for (int t = 0; t < n; ++t) {
            const int stage = t & 1;
            readA(a1, stage, 1);
            readB(b1, stage, 1);
            mma(a0, b0, s0);
            if constexpr (KIND == kPanelSplit) mma(a0, b1, s0);
            if (t + 1 < n) {
                __builtin_amdgcn_s_waitcnt(kAllLoads);   // t + 1 loaded, t read
                barrier();
                if (t + 2 < n) {
                    issue(stage);
                    scales(sa2, sb2);
                }
                readA(a0, stage ^ 1, 0);
                if constexpr (KIND != kPanelSplit) readB(b0, stage ^ 1, 0);
            }
            if constexpr (KIND == kPanelSplit) {
                mma(a1, b0, s0);
                if (t + 1 < n) readB(b0, stage ^ 1, 0);
            } else {
                mma(a1, b1, s1);
            }
            if constexpr (KIND == kPanelMx) {
                sa = sa1;
                sb = sb1;
                sa1 = sa2;
                sb1 = sb2;
            }
        }
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
