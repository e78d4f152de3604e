// panel.hpp -- the product core of the matrix operators (device code):
// acc[i][j] = sum over K of row i of one operand times row j of another.
//
// Both operands are cut along K into panels of 128 bytes a row; a panel's rows
// follow one another in memory, panel after panel, so that an instruction's loads
// are one run of 1 KB (row after row, the rows of a panel lie a power of two
// apart: 2 to 5 % more for a 4096 x 4096 update).  A row's 128 bytes
// are eight 16-byte pieces, taken as four slabs of two pieces, slab s the
// pieces s and s + 4.  One MFMA 32 x 32 takes a slab of 32 rows of each operand
// (16 bytes a lane: lane l gives row l % 32, piece 4 (l / 32) + s), whatever
// the bytes stand for:
//   Mx     64 4-bit numbers a slab, and a scale per piece (32 numbers):
//          v_mfma_scale 32x32x64;
//   Split  numbers in two parts (x = hi + lo, 22 bits), eight high parts in an
//          even piece and their low parts in the odd piece after it: slabs 2 j
//          and 2 j + 1 give hi hi' + hi lo' + lo hi', three MFMAs; lo lo' is
//          below the sums' own rounding.
// Both take as long for 32 bytes of their rows, so one tile geometry
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
// Pipeline, NS stages of LDS.  While panel t is multiplied, the next NS - 1 are
// on their way; one barrier per panel, after the last LDS read of t and before
// its last MFMAs:
//   read slabs g of t | MFMAs of slabs g - 1         (for each group of slabs)
//   wait for t + 1; barrier; loads of t + NS into t's stage
//   read the first group of t + 1 | MFMAs of the last group of t
// Two stages do for the large tiles (three or four: the same time within 2 %);
// small tiles, whose panels take less than a load's latency, have four.
//
// Two things keep the large tiles from the instructions' peak, 10 PFLOP/s in 4 bits
// and 2.5 in halves: the clock, 1.67-1.89 GHz under them where 2.4 is the highest (the
// card's power; the instructions alone, on operands of random bits, make 6.2 and 1.6),
// and the matrix units, which are busy for 50-54 % (4 bits) and 58-64 % (two parts) of
// the cycles: eight wavefronts read LDS and wait at one barrier together.
#pragma once
#include <type_traits>

#include "kernel.hpp"
#include "matrix.hpp"

namespace gett {

typedef __attribute__((address_space(1))) void matrix_global;
typedef __attribute__((address_space(3))) void matrix_lds;

enum PanelKind { kPanelMx, kPanelSplit };

template <int N, int I = 0, typename F> __device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, I + 1>(f);
    }
}

template <int FM_, int FN_, int WM_, int WN_, int NS_> struct PanelShape {
    static constexpr int FM = FM_, FN = FN_, WM = WM_, WN = WN_;   // fragments, wavefronts
    static constexpr int NS = NS_;                                 // stages
    static constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int DATA = (BM + BN) * 128;      // bytes of a stage without scales
    static constexpr int SCALES = (BM + BN) * 8;      // of its scales
    static constexpr int J = DATA / 1024 / NW;        // load instructions a wavefront per panel
    static constexpr int JS = SCALES / 256 / NW;      // and for scales
    static constexpr int TILE = BM * BN;              // elements
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "whole instructions per operand");
    static_assert(SCALES % (256 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0, "64 scale words each");
    static constexpr int lds(int kind) { return NS * (DATA + (kind == kPanelMx ? SCALES : 0)); }
};

// One operand of a tile: rows [row0, row0 + tile rows) of a matrix of `rows`
// rows.  Rows past the last read the last one again; their results are not
// stored.
struct PanelOperand {
    const uint8_t *data;     // panel 0, row 0
    const uint8_t *scales;   // Mx: the packed scales
    int rows, row0;
    // rows row0 ... of panel t, and nothing behind the panel's last row; the
    // scale words of half h likewise
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t panel(int t) const
    {
        const uint8_t *p = data + ((int64_t)t * rows + row0) * 128;
        const int64_t bytes = (int64_t)(rows - row0) * 128;
        return __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t *>(p), 0, (int)(uint32_t)(bytes < 0xffffffffll ? bytes : 0xffffffffll),
            0x00027000);
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t words(int t, int half, int64_t R) const
    {
        const uint8_t *p = scales + (((int64_t)t * 2 + half) * R + row0) * 4;
        const int64_t bytes = (R - row0) * 4;
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

// place of piece p (8 + p in the second row of its pair) of a row of lane r
template <int F> __device__ __forceinline__ int panel_place(int p, int r)
{
    return p ^ (F > 1 ? r & 15 : (r >> 1) & 7);
}

template <int KIND, typename S> struct Panel {
    static constexpr int FM = S::FM, FN = S::FN, NS = S::NS;
    static constexpr int STAGE = S::DATA + (KIND == kPanelMx ? S::SCALES : 0);
    // Slabs read together.  One block of 32 x 32 a wavefront has too few MFMAs
    // in a slab to cover the reads of the next: it reads whole panels.
    static constexpr int G = FM * FN == 1 ? 4 : KIND == kPanelSplit ? 2 : 1;
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

    // panels [t0, t1) of both operands; `lds` holds S::lds(KIND) bytes.
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
            char *base = lds + stage * STAGE;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                char *dst = base + (j < JA ? 0 : S::BM * 128) + ((j < JA ? j : j - JA) * NW + wave) * 1024;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(j < JA ? ra : rb, (matrix_lds *)dst, 16,
                                                         (int)off[j], 0, 0, 0);
            }
            if constexpr (KIND == kPanelMx) {
                // [A's rows, half 0][half 1][B's rows, half 0][half 1], 64 words
                // an instruction; words past the last row come as zeros
                const int64_t RA = mx_scale_rows(A.rows), RB = mx_scale_rows(B.rows);
#pragma unroll
                for (int j = 0; j < S::JS; ++j) {
                    const int u = wave * S::JS + j;   // which 64 words
                    const bool isA = u < S::BM / 32;
                    const int v = isA ? u : u - S::BM / 32, per = (isA ? S::BM : S::BN) / 64;
                    const int half = v / per, first = (v - half * per) * 64;
                    const __amdgpu_buffer_rsrc_t rs =
                        isA ? A.words(at, half, RA) : B.words(at, half, RB);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (matrix_lds *)(base + S::DATA + u * 256),
                                                             4, (first + lane) * 4, 0, 0, 0);
                }
            }
            ++at;
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
            atA = ownA + stage * STAGE;
            atB = ownB + stage * STAGE;
            asm volatile("" : "+v"(atA), "+v"(atB));
        };
        // the scale words of this lane's rows in stage `stage`
        int sa[FM], sb[FN];
        auto scales = [&](int stage) {
            if constexpr (KIND == kPanelMx) {
                const char *w = lds + stage * STAGE + S::DATA;
                const int *pa = reinterpret_cast<const int *>(w) + h * S::BM + wm * 32 * FM + FM * r;
                const int *pb = reinterpret_cast<const int *>(w) + 2 * S::BM + h * S::BN +
                                wn * 32 * FN + FN * r;
#pragma unroll
                for (int i = 0; i < FM; ++i) sa[i] = pa[i];
#pragma unroll
                for (int j = 0; j < FN; ++j) sb[j] = pb[j];
            }
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
        auto mma = [&](int set, auto slab) {   // slabs [slab, slab + G)
            static_for<G>([&](auto gc) {
                constexpr int g = decltype(gc)::value, s = decltype(slab)::value + g;
                auto each = [&](int ga, int gb) {
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) {
                            if constexpr (KIND == kPanelMx)
                                acc[i][j] = mfma_mx32<s>(a[set][ga][i], b[set][gb][j], acc[i][j],
                                                         sa[i], sb[j]);
                            else
                                acc[i][j] = mfma_half(a[set][ga][i], b[set][gb][j], acc[i][j]);
                        }
                };
                if constexpr (KIND == kPanelMx) {
                    each(g, g);
                } else if constexpr (g % 2 == 0) {
                    each(g, g);
                    each(g, g + 1);
                    each(g + 1, g);
                }
            });
        };
        // no fence: a release would wait for the loads in flight as well
        auto barrier = []() { asm volatile("s_barrier" ::: "memory"); };
        constexpr int STEPS = 4 / G;        // groups of slabs per panel
        // s_waitcnt operands (gfx9 encoding): lgkmcnt 0 and that many loads left
        // on their way
        constexpr int LOADS = J + (KIND == kPanelMx ? S::JS : 0);
        static_assert((NS - 1) * LOADS < 64, "vmcnt range");
        auto wait_for = [](int left) constexpr { return (left & 15) | (left >> 4) << 14 | 7 << 4; };
        constexpr int kAll = wait_for(0), kFirst = wait_for((NS - 1) * LOADS);
        constexpr int kNext = wait_for((NS - 2) * LOADS);

        const int n = t1 - t0;
        if (n <= 0) return;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < n) issue(i);
        if (n >= NS) __builtin_amdgcn_s_waitcnt(kFirst);
        else __builtin_amdgcn_s_waitcnt(kAll);
        barrier();
        at_stage(0);
        read(0, 0);
        int stage = 0;
        // one panel, whose first slabs are in set `set0`; `more`: another follows,
        // `load`: one is loaded (a bool: perhaps)
        auto panel = [&](auto more, auto load, auto set0) {
            constexpr bool steady = std::is_same<decltype(load), std::true_type>::value;
            constexpr bool perhaps = std::is_same<decltype(load), bool>::value;
            scales(stage);
            static_for<STEPS>([&](auto step) {
                constexpr int s = decltype(step)::value, set = (decltype(set0)::value + s) & 1;
                if constexpr (s + 1 < STEPS) {
                    read(set ^ 1, (s + 1) * G);
                } else if constexpr (more) {
                    __builtin_amdgcn_s_waitcnt(steady ? kNext : kAll);   // t + 1 loaded, t read
                    barrier();
                    if constexpr (steady) {
                        issue(stage);
                    } else if constexpr (perhaps) {
                        if (load) issue(stage);
                    }
                    stage = stage + 1 == NS ? 0 : stage + 1;
                    at_stage(stage);
                    read(set ^ 1, 0);
                }
                mma(set, std::integral_constant<int, s * G>{});
                // the reads of one group lie among the first MFMAs of the one
                // before, and stay there
                constexpr int READS = G * (FM + FN);
                constexpr int MFMAS = FM * FN * (KIND == kPanelSplit ? 3 * G / 2 : G);
                if constexpr (s + 1 < STEPS || more) {
                    static_for<(READS < MFMAS ? READS : MFMAS)>([](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        __builtin_amdgcn_sched_group_barrier(0x100, i + 1 < MFMAS ? 1 : READS - i, 0);
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        const std::true_type yes;
        const std::false_type no;
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, STEPS % 2> odd;   // the next panel's set
        int t = 0;
        if constexpr (STEPS % 2 == 0) {
            // (no branch inside a panel: across one, the sums would be copied)
            for (; t + NS < n; ++t) panel(yes, yes, even);
            for (; t + 1 < n; ++t) panel(yes, no, even);
            panel(no, no, even);
        } else {
            for (; t + NS + 1 < n; t += 2) {
                panel(yes, yes, even);
                panel(yes, yes, odd);
            }
            for (; t + 2 < n; t += 2) {
                panel(yes, t + NS < n, even);
                panel(yes, t + 1 + NS < n, odd);
            }
            if (t + 1 < n) {
                panel(yes, t + NS < n, even);
                panel(no, no, odd);
            } else {
                panel(no, no, even);
            }
        }
    }
};

// The work of a launch: the tiles of one or several matrices of results.
//
// Slices.  The tiles from `full` on are each shared among `slices` workgroups, a
// run of panels each.  Their sums go to slots in device memory in lane order
// (device-scope accesses, which pass by the XCD's own L2, so no fence writes
// caches back), and the last to arrive adds them in slice order: results do not
// depend on who that is.  Counters are zero between launches.
//
// Order.  Workgroups go round the eight XCDs, each with an L2 of its own: the
// ids of one XCD are made neighbours, and neighbours walk bands of four tile
// rows, column by column, so that the tiles resident on an XCD share operand
// rows.
//
// Divisions are multiplications by the host's reciprocals: with the compiler's
// own a launch began with 900 scalar instructions, a microsecond.
struct PanelGrid {
    int tilesM, tilesN, tiles;   // of one matrix
    int full, slices, panels;
    Recip tilesInv, bandInv, slicesInv;
    float *slots;
    int *counters;
};

struct PanelItem {
    int z, tile;          // matrix, tile in it
    int shared, slice;    // index among the shared tiles (-1: whole), slice
    int t0, t1;           // panels
};

__device__ __forceinline__ PanelItem panel_item(const PanelGrid &g, int bid)
{
    PanelItem w = {0, 0, -1, 0, 0, g.panels};
    int tile = bid;
    if (bid >= g.full) {
        const int u = bid - g.full;
        w.shared = (int)quotient((uint32_t)u, g.slices, g.slicesInv);
        w.slice = u - w.shared * g.slices;
        tile = g.full + w.shared;
        w.t0 = (int)quotient((uint32_t)(g.panels * w.slice), g.slices, g.slicesInv);
        w.t1 = (int)quotient((uint32_t)(g.panels * (w.slice + 1)), g.slices, g.slicesInv);
        if (g.slices == 1) w.shared = -1;
    } else if (bid < (g.full & ~7)) {
        tile = (bid & 7) * (g.full >> 3) + (bid >> 3);
    }
    w.z = (int)quotient((uint32_t)tile, g.tiles, g.tilesInv);
    w.tile = tile - w.z * g.tiles;
    return w;
}

constexpr int kPanelBand = 4;
__device__ __forceinline__ void panel_tile(const PanelGrid &g, int id, int &tm, int &tn)
{
    const int inBand = kPanelBand * g.tilesN;
    const int b = (int)quotient((uint32_t)id, inBand, g.bandInv), rest = id - b * inBand;
    const int height = g.tilesM - b * kPanelBand;
    if (height >= kPanelBand) tn = rest >> 2;
    else if (height == 3) tn = (int)__umulhi((uint32_t)rest, 0x55555556u);
    else tn = rest >> (height - 1);
    tm = b * kPanelBand + rest - tn * (height < kPanelBand ? height : kPanelBand);
}
// the t-th tile on or below the diagonal, row by row
__device__ __forceinline__ void panel_triangle(int t, int &tm, int &tn)
{
    tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
    while (tm * (tm + 1) / 2 > t) --tm;
    tn = t - tm * (tm + 1) / 2;
}

// Adds up a shared tile; true for the workgroup that holds the sum (and for a
// tile that is not shared).  `lds` may be any LDS but is overwritten.
template <int KIND, typename S>
__device__ __forceinline__ bool panel_join(Panel<KIND, S> &p, const PanelGrid &d,
                                           const PanelItem &w, char *lds)
{
    if (w.shared < 0) return true;
    const int tid = (int)threadIdx.x;
    constexpr int N = S::THREADS;
    float *first = d.slots + (int64_t)w.shared * d.slices * S::TILE + tid;
    float *own = first + (int64_t)w.slice * S::TILE;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                __hip_atomic_store(own + ((i * S::FN + j) * 16 + e) * N, p.acc[i][j][e],
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);   // vmcnt 0: the stores are done
    __syncthreads();
    int *last = reinterpret_cast<int *>(lds);
    if (tid == 0)
        *last = __hip_atomic_fetch_add(d.counters + w.shared, 1, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT) == d.slices - 1;
    __syncthreads();
    if (!*last) return false;
    if (tid == 0)
        __hip_atomic_store(d.counters + w.shared, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const float *at = first + (i * S::FN + j) * 16 * N;
            for (int s0 = 0; s0 < d.slices; s0 += 2) {   // two slices' loads together
                float v[2][16];
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (s0 + s < d.slices)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            v[s][e] = __hip_atomic_load(at + (int64_t)(s0 + s) * S::TILE + e * N,
                                                        __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (s0 + s < d.slices)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            p.acc[i][j][e] = s0 + s == 0 ? v[s][e] : p.acc[i][j][e] + v[s][e];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    __syncthreads();   // everyone has read `last`
    return true;
}

// Host: how the tiles of a launch are shared.  Whole rounds of tiles (as many as
// are resident at once) stay whole; the tiles of a last, incomplete round may
// be cut so that their slices fill it.  us per panel and round, with the CUs
// full and with one workgroup each, and for the join of s slices, measured: the
// products of 4096 x 4096 (Big, Mid) and 517 x 1000 (Small).
struct PanelCut {
    int64_t full = 0, slices = 1, blocks = 0;
    double us = 1e300;
    int64_t shared() const { return slices > 1 ? (blocks - full) / slices : 0; }
};
constexpr int64_t kPanelCus = 256;
template <typename S> PanelCut panel_cut(int kind, int64_t tiles, int64_t panels)
{
    constexpr bool big = S::BM == 256, mid = S::BM == 128;
    constexpr int64_t slots = (big ? 1 : 2) * kPanelCus;
    const double full = big ? (kind == kPanelSplit ? 2.3 : 2.1) : mid ? 1.2 : 0.45;
    const double alone = big ? full : kind == kPanelSplit ? (mid ? 1.0 : 0.30) : (mid ? 0.75 : 0.25);
    const double join = big ? 15 : mid ? 8 : 6, joinEach = big ? 6 : mid ? 1.5 : 0.3;
    const int64_t rounds = tiles / slots, rest = tiles % slots;
    PanelCut best;
    for (int64_t s = 1; s <= 16; ++s) {
        if (s > 1 && (rest * s > slots || panels < 2 * s)) break;
        double t = rounds * panels * full;
        if (rest) t += (double)((panels + s - 1) / s) * (rest * s <= kPanelCus ? alone : full);
        if (s > 1) t += join + joinEach * s;
        if (t < best.us) {
            best.full = s > 1 ? tiles - rest : tiles;
            best.slices = s;
            best.blocks = best.full + (s > 1 ? rest * s : 0);
            best.us = t;
        }
    }
    return best;
}

// Fills in a grid; false where it has too many workgroups for a launch.
inline bool panel_grid(PanelGrid &g, int64_t batch, int64_t tilesM, int64_t tilesN, int64_t tiles,
                       const PanelCut &cut, int panels, float *slots, int *counters)
{
    if (cut.blocks >= INT32_MAX || tiles * batch >= INT32_MAX ||
        kPanelBand * tilesN >= INT32_MAX || (int64_t)panels * cut.slices >= INT32_MAX)
        return false;
    g = {(int)tilesM, (int)tilesN, (int)tiles, (int)cut.full, (int)cut.slices, panels,
         recip(tiles), recip(kPanelBand * tilesN), recip(cut.slices), slots, counters};
    return true;
}

}  // namespace gett
