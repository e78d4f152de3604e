// route.hip -- the choice of experts and the order of the chosen rows.
//
// A wavefront takes a token; the k largest are taken one by one (k is small), each the
// largest of the lanes' largest, of equal ones the lowest.  What is compared is held
// in 64 bits, as whole numbers of the same order whose halves go through the
// wavefront one after the other (DPP: no trip through LDS).  (Choosing in 32 bits, and
// again in 64 where a bound of the error does not decide, was no faster: one token in
// a hundred is enough for every workgroup to wait for one.)  16384 tokens of 256
// experts in 8 groups take 40 us, bound by instructions: four sigmoids a lane in 64 bits
// and twelve picks one after the other; the bytes (17 MB) would take 3.4.  A single
// token takes 5.5 us, all latency.
//
// That is choose_quickly, for finite logits and biases of up to 512 experts, whose
// groups are a power of two of lanes where there are any.  Everything else is chosen by
// choose_exactly, from LDS: 16384 tokens of 160 experts in 8 groups take 107 us, of
// 1024 experts 158.
//
// The order of the rows by expert is a stable counting sort: chunks of whole tokens,
// up to 512 rows, are chosen and counted in one launch, the counts summed over the
// chunks, and each chunk writes its rows, with no atomics whose order could show.  Up
// to 512 rows it is one launch of one workgroup in all.  A chunk is a workgroup, so that
// few choices a token leave CUs without one: 16384 tokens of 256 experts take 26 us
// with eight choices (256 workgroups), 46 with two and 76 with one (32).
#include "launch.hpp"
#include "layer_util.hpp"

namespace gett {

namespace {

constexpr int kChunk = 512;       // rows (token, choice) of a workgroup, at most
constexpr int kThreads = 1024;

struct RouteJob {
    const void *logits;
    int64_t ld;
    const float *bias;
    int tokens, experts, k, scoring, groups, topGroups, renormalize;
    double scale;
    float *weights;
    int32_t *index, *order, *offsets, *place;
    int32_t *counts;   // experts x chunks, then the experts' totals
    int chunks, chunkTokens;
};

// A larger one first, of equal ones the lower index; -inf is nothing.
struct Best {
    double key;
    int at;
    __device__ __forceinline__ void take(double k, int i)
    {
        if (k > key || (k == key && i < at)) {
            key = k;
            at = i;
        }
    }
};
__device__ __forceinline__ Best wave_best(Best b)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) b.take(__shfl_xor(b.key, d), __shfl_xor(b.at, d));
    return b;
}
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// One token in 64 bits, of any logits and any groups: lane l sees to the experts l, l +
// 64, ... and the groups l, l + 64, ...  `keys` holds `experts` doubles of LDS of the
// wavefront's own.  Small, not fast: a group's keys are read by one lane, once for each
// group that opens, and every pick is a chain of 18 exchanges (see the figures above).
template <typename T>
__device__ __forceinline__ void choose_exactly(const RouteJob &j, int64_t token, double *keys)
{
    const int lane = (int)threadIdx.x & 63;
    const double none = -__builtin_huge_val();
    const float least = -__builtin_huge_valf();
    const bool soft = j.scoring == GETT_SCORE_SOFTMAX, plain = !j.bias && j.groups == 1;
    const T *row = reinterpret_cast<const T *>(j.logits) + token * j.ld;
    bool nan = false;
    float most = least;
    for (int e = lane; e < j.experts; e += 64) {
        const float x = to_float(row[e]);
        nan |= x != x;
        most = fmaxf(most, x);   // (a NaN is passed over)
    }
    nan = __any(nan);
    most = wave_max(most);
    double total = 1.0;
    if (soft) {
        total = 0.0;
        for (int e = lane; e < j.experts; e += 64) {
            const float x = to_float(row[e]);
            if (x > least) total += exp((double)x - (double)most);
        }
        total = wave_sum(total);
    }
    float top = most;
    auto score_of = [&](float x) {
        return soft ? exp((double)x - (double)top) / total : 1.0 / (1.0 + exp(-(double)x));
    };
    for (int e = lane; e < j.experts; e += 64) {
        const float x = to_float(row[e]);
        double c = none;
        if (x > least) c = plain ? (double)x : j.bias ? score_of(x) + (double)j.bias[e] : score_of(x);
        keys[e] = c != c ? none : c;
    }
    if (j.groups > 1) {
        wave_exchange();   // a group's keys are other lanes' than the group
        const int size = j.experts / j.groups;
        uint32_t open = 0;   // of this lane's groups
        for (int r = 0; r < j.topGroups; ++r) {
            Best best = {none, INT32_MAX};
            for (int g = lane; g < j.groups; g += 64) {
                if (open >> (g >> 6) & 1) continue;
                double a = none, b = none;
                for (int e = g * size; e < (g + 1) * size; ++e) {
                    const double v = keys[e];
                    b = v > a ? a : v > b ? v : b;
                    a = v > a ? v : a;
                }
                best.take(b > none ? a + b : a, g);
            }
            best = wave_best(best);
            if (best.key == none) break;
            if ((best.at & 63) == lane) open |= 1u << (best.at >> 6);
        }
        wave_exchange();   // (all are read)
        for (int e0 = 0; e0 < j.experts; e0 += 64) {
            const int e = e0 + lane, g = e < j.experts ? e / size : 0;
            const uint32_t bits = __shfl(open, g & 63);
            if (e < j.experts && !(bits >> (g >> 6) & 1)) keys[e] = none;
        }
    }
    // the k largest: lane r keeps the r-th
    int mine = -1;
    for (int r = 0; r < j.k; ++r) {
        Best best = {none, INT32_MAX};
        for (int e = lane; e < j.experts; e += 64) best.take(keys[e], e);
        best = wave_best(best);
        if (best.key == none) break;
        if ((best.at & 63) == lane) keys[best.at] = none;
        if (lane == r) mine = best.at;
    }
    const float chosen = mine >= 0 ? to_float(row[mine]) : least;
    if (soft && j.renormalize) top = wave_max(chosen);   // (as in choose_quickly)
    const double score = mine >= 0 ? score_of(chosen) : 0.0;
    double w = score;
    if (j.renormalize) {
        const double sum = wave_sum(score);
        w = sum > 0.0 || sum != sum ? score / sum : 0.0;
    }
    if (lane < j.k) {
        float out = mine < 0 ? 0.0f : (float)(w * j.scale);
        if (nan || (soft && most == __builtin_huge_valf())) out = __builtin_nanf("");
        j.weights[token * j.k + lane] = out;
        j.index[token * j.k + lane] = mine;
    }
}

// The largest of the lanes' values.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    auto step = [&](auto ctrl) {
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    step(std::integral_constant<int, 0x111>{});   // from the lane 1, 2, 4, 8 before in the row
    step(std::integral_constant<int, 0x112>{});
    step(std::integral_constant<int, 0x114>{});
    step(std::integral_constant<int, 0x118>{});
    step(std::integral_constant<int, 0x142>{});   // from the last lane of the row before,
    step(std::integral_constant<int, 0x143>{});   // and of the half before
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// Numbers as whole numbers of the same order (no NaN, -0 made 0); 0 is less than all.
__device__ __forceinline__ uint64_t ordered(double d)
{
    const uint64_t b = (uint64_t)__double_as_longlong(d + 0.0);
    return b ^ (b >> 63 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double from_ordered(uint64_t u)
{
    return __longlong_as_double((long long)(u ^ (u >> 63 ? 1ull << 63 : ~0ull)));
}
// The largest of the lanes' N values each, in halves: which lane has it, and where; of
// equal ones the lowest lane's lowest.  False where all are 0.  The low halves are only
// looked at where the high ones do not decide.
template <int N>
__device__ __forceinline__ bool pick(const uint32_t (&high)[N], const uint32_t (&low)[N], int &lane, int &at)
{
    uint32_t local = high[0];
#pragma unroll
    for (int i = 1; i < N; ++i) local = max(local, high[i]);
    const uint32_t most = wave_max_u32(local);
    if (most == 0) return false;
    uint64_t has[N], any = 0;
    int count = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        has[i] = __ballot(high[i] == most);
        any |= has[i];
        count += __popcll(has[i]);
    }
    if (count > 1) {
        uint32_t l = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) l = max(l, high[i] == most ? low[i] : 0);
        l = wave_max_u32(l);
        any = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            has[i] = __ballot(high[i] == most && low[i] == l);
            any |= has[i];
        }
    }
    lane = __ffsll((unsigned long long)any) - 1;
    at = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
        if (has[i] >> lane & 1) at = i;
    return true;
}

// One token whose logits and biases are numbers: lane l holds the experts PER l ... PER l
// + PER - 1, a group has a power of two of lanes.  False where that is not so (nothing
// is written then).
template <typename T, int PER>
__device__ __forceinline__ bool choose_quickly(const RouteJob &j, int64_t token)
{
    const int lane = (int)threadIdx.x & 63;
    const float none = -__builtin_huge_valf();
    const bool soft = j.scoring == GETT_SCORE_SOFTMAX, plain = !j.bias && j.groups == 1;
    const int size = j.experts / j.groups, lanes = size / PER;   // lanes of a group
    if (j.groups > 1 && (size % PER || (lanes & (lanes - 1)))) return false;
    const T *row = reinterpret_cast<const T *>(j.logits) + token * j.ld + lane * PER;
    float x[PER], most = none;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool there = lane * PER + i < j.experts;
        x[i] = there ? to_float(row[i]) : none;
        odd |= x[i] != x[i] || x[i] == __builtin_huge_valf();
        most = fmaxf(most, x[i]);
    }
    uint64_t key[PER];
    double total = 1.0;
    if (soft) most = wave_max(most);
    if (plain) {
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = x[i] == none ? 0 : ordered((double)x[i]);
    }
    if (!plain || (soft && !j.renormalize)) {   // scores, or their sum
        double s[PER];
        if (soft) {
            total = 0.0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                s[i] = x[i] == none ? 0.0 : exp((double)x[i] - (double)most);
                total += s[i];
            }
            total = wave_sum(total);
        }
        if (!plain) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                double c = soft ? s[i] / total : 1.0 / (1.0 + exp(-(double)x[i]));
                if (j.bias) {
                    const float bias = lane * PER + i < j.experts ? j.bias[lane * PER + i] : 0.0f;
                    odd |= !(fabsf(bias) < __builtin_huge_valf());
                    c += (double)bias;
                }
                key[i] = x[i] == none ? 0 : ordered(c);
            }
        }
    }
    if (__any(odd)) return false;
    if (j.groups > 1) {
        // the two largest of each group
        uint64_t a = 0, b = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            b = max(b, min(a, key[i]));
            a = max(a, key[i]);
        }
        for (int d = 1; d < lanes; d <<= 1) {
            const uint64_t a2 = __shfl_xor(a, d), b2 = __shfl_xor(b, d);
            b = max(min(a, a2), max(b, b2));
            a = max(a, a2);
        }
        uint64_t sum = a == 0 ? 0 : ordered(b ? from_ordered(a) + from_ordered(b) : from_ordered(a));
        if (lane * PER >= j.experts || lane & (lanes - 1)) sum = 0;   // a group's first lane has it
        uint32_t high[1] = {(uint32_t)(sum >> 32)}, low[1] = {(uint32_t)sum};
        bool open = false;
        for (int r = 0; r < j.topGroups; ++r) {
            int first, at;
            if (!pick<1>(high, low, first, at)) break;
            open |= lane >= first && lane < first + lanes;
            if (lane == first) high[0] = 0;
        }
        if (!open) {
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = 0;
        }
    }
    uint32_t high[PER], low[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        high[i] = (uint32_t)(key[i] >> 32);
        low[i] = (uint32_t)key[i];
    }
    int mine = -1;
    float chosen = 0.0f;
    for (int r = 0; r < j.k; ++r) {
        int from, at;
        if (!pick<PER>(high, low, from, at)) break;
        float v = x[0];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i == at) v = x[i];
            if (i == at && lane == from) high[i] = 0;
        }
        v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), from));
        if (lane == r) {
            mine = from * PER + at;
            chosen = v;
        }
    }
    // Of renormalised weights the scores' own sum is no matter: relative to the largest
    // of the chosen they do not all vanish, as far below the token's largest as a bias
    // or the groups may have them.  (Without these the two are the same.)
    if (soft && j.renormalize && !plain) most = wave_max(mine >= 0 ? chosen : none);
    double score = 0.0;
    if (mine >= 0)
        score = soft ? exp((double)chosen - (double)most) / total : 1.0 / (1.0 + exp(-(double)chosen));
    double w = score;
    if (j.renormalize) {
        const double sum = wave_sum(score);
        w = sum > 0.0 ? score / sum : 0.0;
    }
    if (lane < j.k) {
        j.weights[token * j.k + lane] = mine < 0 ? 0.0f : (float)(w * j.scale);
        j.index[token * j.k + lane] = mine;
    }
    return true;
}

template <typename T, int PER>
__device__ __forceinline__ void choose(const RouteJob &j, int64_t token, double *keys)
{
    if constexpr (PER <= 8) {   // (of 1024 experts a lane's sixteen do not fit the registers)
        if (choose_quickly<T, PER>(j, token)) return;
    }
    choose_exactly<T>(j, token, keys);
}

// The lanes of a wavefront that have the same e, 0 <= e < 1024.
__device__ __forceinline__ uint64_t same_lanes(int e)
{
    uint64_t m = ~0ull;
#pragma unroll
    for (int b = 0; b < 10; ++b) {
        const uint64_t set = __ballot(e >> b & 1);
        m &= e >> b & 1 ? set : ~set;
    }
    return m;
}

// Writes a chunk's rows, those from row0 on.  `waves` holds 8 x experts counts; base[e]
// is where the chunk's rows of expert e begin.
__device__ __forceinline__ void place_rows(const RouteJob &j, int row0, int rows, int32_t *waves,
                                           const int32_t *base)
{
    const int tid = (int)threadIdx.x, r = row0 + tid, lane = tid & 63, wave = tid >> 6;
    const bool there = tid < kChunk && tid < rows;
    const int e = there ? j.index[r] : -1;
    for (int i = tid; i < kChunk / 64 * j.experts; i += kThreads) waves[i] = 0;
    __syncthreads();
    const uint64_t alike = same_lanes(e < 0 ? 0 : e) & __ballot(e >= 0);
    const int rank = __popcll(alike & ((1ull << lane) - 1));
    if (e >= 0 && rank == 0) waves[wave * j.experts + e] = __popcll(alike);
    __syncthreads();
    if (e >= 0) {
        int at = base[e] + rank;
        for (int w = 0; w < wave; ++w) at += waves[w * j.experts + e];
        j.order[at] = r;
        j.place[r] = at;
    } else if (there) {
        j.place[r] = -1;
    }
}

// Chooses for a chunk's tokens and counts their rows per expert.
template <typename T, int PER>
__device__ __forceinline__ void choose_rows(const RouteJob &j, int token0, int tokens, double *keys,
                                            int32_t *counts)
{
    const int tid = (int)threadIdx.x, wave = tid >> 6;
    for (int i = tid; i < j.experts; i += kThreads) counts[i] = 0;
    for (int t = wave; t < tokens; t += kThreads / 64)
        choose<T, PER>(j, token0 + t, keys + wave * j.experts);
    __syncthreads();   // (drains the stores, which this workgroup reads back)
    const int e = tid < tokens * j.k ? j.index[(int64_t)token0 * j.k + tid] : -1;
    if (e >= 0) atomicAdd(&counts[e], 1);   // (whole numbers: in any order the same)
    __syncthreads();
}

// Where the rows of this thread's expert begin, from the number of each; 1024 threads.
__device__ __forceinline__ int scan_experts(int count, int32_t *lds)
{
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    int v = count;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += lds[w];
    __syncthreads();
    return before + v - count;
}

template <typename T, int PER>
__global__ __launch_bounds__(kThreads) void route_choose_kernel(RouteJob j)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    __shared__ int32_t counts[kMostExperts];
    const int token0 = (int)blockIdx.x * j.chunkTokens, tokens = min(j.tokens - token0, j.chunkTokens);
    choose_rows<T, PER>(j, token0, tokens, reinterpret_cast<double *>(dyn_lds), counts);
    for (int i = (int)threadIdx.x; i < j.experts; i += kThreads)
        j.counts[(int64_t)i * j.chunks + blockIdx.x] = counts[i];
}

// A wavefront for an expert: its rows before each chunk, and in all.
__global__ __launch_bounds__(256) void route_scan_kernel(RouteJob j)
{
    const int lane = (int)threadIdx.x & 63, e = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    if (e >= j.experts) return;
    int32_t *counts = j.counts + (int64_t)e * j.chunks;
    int before = 0;
    for (int c0 = 0; c0 < j.chunks; c0 += 64) {
        const int n = c0 + lane < j.chunks ? counts[c0 + lane] : 0;
        int v = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        if (c0 + lane < j.chunks) counts[c0 + lane] = before + v - n;
        before += __shfl(v, 63);
    }
    if (lane == 0) j.counts[(int64_t)j.experts * j.chunks + e] = before;
}

__global__ __launch_bounds__(kThreads) void route_place_kernel(RouteJob j)
{
    extern __shared__ int32_t waves[];
    __shared__ int32_t base[kMostExperts];
    __shared__ int32_t lds[16];
    __shared__ int live;
    const int e = (int)threadIdx.x;
    const int n = e < j.experts ? j.counts[(int64_t)j.experts * j.chunks + e] : 0;
    const int at = scan_experts(n, lds);
    if (e < j.experts) {
        base[e] = at + j.counts[(int64_t)e * j.chunks + blockIdx.x];
        if (blockIdx.x == 0) j.offsets[e] = at;
    }
    if (e == j.experts - 1) {
        live = at + n;
        if (blockIdx.x == 0) j.offsets[j.experts] = at + n;
    }
    __syncthreads();
    const int token0 = (int)blockIdx.x * j.chunkTokens, tokens = min(j.tokens - token0, j.chunkTokens);
    place_rows(j, token0 * j.k, tokens * j.k, waves, base);
    const int r = token0 * j.k + (int)threadIdx.x;
    if ((int)threadIdx.x < tokens * j.k && r >= live) j.order[r] = -1;
}

// Everything, for up to 512 rows.
template <typename T, int PER>
__global__ __launch_bounds__(kThreads) void route_small_kernel(RouteJob j)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    __shared__ int32_t counts[kMostExperts];
    __shared__ int32_t lds[16];
    __shared__ int live;
    choose_rows<T, PER>(j, 0, j.tokens, reinterpret_cast<double *>(dyn_lds), counts);
    const int e = (int)threadIdx.x;
    const int n = e < j.experts ? counts[e] : 0;
    const int at = scan_experts(n, lds);
    if (e < j.experts) {
        counts[e] = at;
        j.offsets[e] = at;
    }
    if (e == j.experts - 1) {
        j.offsets[j.experts] = at + n;
        live = at + n;
    }
    __syncthreads();
    place_rows(j, 0, j.tokens * j.k, reinterpret_cast<int32_t *>(dyn_lds), counts);
    const int r = (int)threadIdx.x;
    if (r < j.tokens * j.k && r >= live) j.order[r] = -1;
}

// ----------------------------------------------------------------- gradient ---

struct RouteGradJob {
    const void *logits;
    void *dlogits;
    int64_t ld, ldd;
    int tokens, experts, k, scoring, renormalize;
    double scale;
    const int32_t *index;
    const float *dweights;
};

// With c the chosen scores, w = scale c / sum c (or scale c) and g = scale dweights:
//     renormalised  dc = (g - sum(g c) / sum c) / sum c, otherwise g
//     softmax       dx = s (ds - sum(ds s)),  sigmoid  dx = ds s (1 - s)
// where ds is dc at the chosen experts and 0 elsewhere.  The sum over ds s is zero
// where the weights are renormalised: only a softmax that is not has a gradient
// outside the chosen, and needs their scores.  All logits are read all the same: a NaN
// among them, or a +inf under a softmax, has made the token's weights NaN wherever it
// is, and so its gradient is.  16384 tokens of 256 experts in 32 bits take 12 us (34 MB,
// and the launch), of 1024 23 (134 MB: 5.8 TB/s).
template <typename T, int PER>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteGradJob j)
{
    __shared__ float spread[4][64 * PER];
    const int lane = (int)threadIdx.x & 63;
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= j.tokens) return;
    float *ds = spread[threadIdx.x >> 6];
    const T *row = reinterpret_cast<const T *>(j.logits) + token * j.ld;
    const bool soft = j.scoring == GETT_SCORE_SOFTMAX, dense = soft && !j.renormalize;
    // lane r: the r-th choice, its logit and its gradient
    int at = lane < j.k ? j.index[token * j.k + lane] : -1;
    if (at >= j.experts) at = -1;
    const float chosen = at >= 0 ? to_float(row[at]) : -__builtin_huge_valf();
    double g = at >= 0 ? j.scale * (double)j.dweights[token * j.k + lane] : 0.0;
    float x[PER];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        x[i] = e < j.experts ? to_float(row[e]) : -__builtin_huge_valf();
        odd |= x[i] != x[i] || (soft && x[i] == __builtin_huge_valf());
    }
    const bool nan = __any(odd);
    double s[PER], total = 1.0, rest = 0.0;
    float most = soft ? wave_max(chosen) : 0.0f;
    if (dense) {
#pragma unroll
        for (int i = 0; i < PER; ++i) most = fmaxf(most, x[i]);
        most = wave_max(most);
        total = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = x[i] == -__builtin_huge_valf() ? 0.0 : exp((double)x[i] - (double)most);
            total += s[i];
        }
        total = wave_sum(total);
    }
    double c = 0.0;
    if (at >= 0) c = soft ? exp((double)chosen - (double)most) / total : 1.0 / (1.0 + exp(-(double)chosen));
    double mine;
    if (j.renormalize) {
        const double sum = wave_sum(c), dot = wave_sum(g * c);
        mine = sum > 0.0 || sum != sum ? (g - dot / sum) / sum * c : 0.0;
        if (!soft) mine *= 1.0 - c;
    } else if (soft) {
        rest = wave_sum(g * c);
        mine = c * (g - rest);
    } else {
        mine = g * c * (1.0 - c);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < j.experts)   // (a total of 0: every logit is -inf)
            ds[i * 64 + lane] = dense && total != 0.0 ? (float)(-s[i] / total * rest) : 0.0f;
    wave_exchange();
    if (at >= 0) ds[at] = (float)mine;
    wave_exchange();
    T *out = reinterpret_cast<T *>(j.dlogits) + token * j.ldd;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < j.experts)
            out[i * 64 + lane] = from_float<T>(nan ? __builtin_nanf("") : ds[i * 64 + lane]);
}

// f(an integral constant of the experts a lane holds)
template <typename F> gett_status_t with_experts(int experts, F &&f)
{
    if (experts <= 64) return f(std::integral_constant<int, 1>{});
    if (experts <= 128) return f(std::integral_constant<int, 2>{});
    if (experts <= 256) return f(std::integral_constant<int, 4>{});
    if (experts <= 512) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

gett_status_t route_ok(gett_dtype_t dtype, int64_t tokens, int experts, int k, int scoring)
{
    if (!float_type(dtype) || tokens < 0 || experts < 1 || k < 1 || k > experts ||
        (scoring != GETT_SCORE_SOFTMAX && scoring != GETT_SCORE_SIGMOID))
        return GETT_ERROR_INVALID_VALUE;
    if (experts > kMostExperts || k > kMostChoices || tokens >= kLayerRows || tokens * k >= kLayerRows)
        return GETT_ERROR_NOT_SUPPORTED;
    return GETT_SUCCESS;
}

}  // namespace

}  // namespace gett

extern "C" {

gett_status_t gett_route(gett_dtype_t dtype, int64_t tokens, int experts, int k,
                         const void *logits, int64_t stride, int scoring, const float *bias,
                         int groups, int top_groups, int renormalize, double scale, float *weights,
                         int32_t *index, int32_t *order, int32_t *offsets, int32_t *place,
                         void *stream)
{
    using namespace gett;
    gett_status_t st = route_ok(dtype, tokens, experts, k, scoring);
    if (st != GETT_SUCCESS) return st;
    if (groups < 1 || experts % groups || top_groups < 1 || top_groups > groups ||
        (int64_t)experts / groups * top_groups < k || scale != scale)
        return GETT_ERROR_INVALID_VALUE;
    const int64_t rows = tokens * k;
    Extent x, b = {}, out[5];
    st = layer_matrix(dtype, tokens, experts, logits, stride, x);
    if (st == GETT_SUCCESS && bias) st = layer_list(experts, 4, bias, b);
    const void *outputs[5] = {weights, index, order, place, offsets};
    for (int i = 0; i < 5 && st == GETT_SUCCESS; ++i)
        st = layer_list(i < 4 ? rows : experts + 1, 4, outputs[i], out[i]);
    if (st != GETT_SUCCESS) return st;
    for (int i = 0; i < 5; ++i) {
        if (!apart(out[i], x) || !apart(out[i], b)) return GETT_ERROR_INVALID_VALUE;
        for (int j = i + 1; j < 5; ++j)
            if (!apart(out[i], out[j])) return GETT_ERROR_INVALID_VALUE;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t chunkTokens = kChunk / k, chunks = (tokens + chunkTokens - 1) / chunkTokens;
    RouteJob j = {logits, stride, bias, (int)tokens, experts, k, scoring, groups, top_groups, renormalize,
                  scale, weights, index, order, offsets, place, nullptr, (int)chunks, (int)chunkTokens};
    // a double an expert for each wavefront, and counts
    const size_t lds = kThreads / 64 * (size_t)experts * 8, countBytes = kChunk / 64 * (size_t)experts * 4;
    const bool small = chunks <= 1;
    Partials hold;
    if (!small) {
        if (!fits_launch(chunks, kThreads)) return GETT_ERROR_NOT_SUPPORTED;
        st = stream_workspace(s, 0, ((uint64_t)chunks + 1) * experts * 4, hold);
        if (st != GETT_SUCCESS) return st;
        j.counts = static_cast<int32_t *>(hold.tiles);
    }
    st = with_experts(experts, [&](auto per) {
        return with_type(dtype, [&](auto v) {
            constexpr int PER = decltype(per)::value;
            constexpr size_t most = kThreads / 64 * 64 * PER * 8;
            if (small) {
                constexpr auto kernel = route_small_kernel<decltype(v), PER>;
                if (allow_dynamic_lds<kernel>(most) != hipSuccess) return GETT_ERROR_HIP;
                hipLaunchKernelGGL(kernel, dim3(1), dim3(kThreads), lds, s, j);
            } else {
                constexpr auto kernel = route_choose_kernel<decltype(v), PER>;
                if (allow_dynamic_lds<kernel>(most) != hipSuccess) return GETT_ERROR_HIP;
                hipLaunchKernelGGL(kernel, dim3((unsigned)chunks), dim3(kThreads), lds, s, j);
            }
            return launched(hipGetLastError());
        });
    });
    if (st != GETT_SUCCESS || small) return st;
    hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)((experts + 3) / 4)), dim3(256), 0, s, j);
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)chunks), dim3(kThreads), countBytes, s, j);
    return launched(hipGetLastError());
}

gett_status_t gett_route_grad(gett_dtype_t dtype, int64_t tokens, int experts, int k,
                              const void *logits, int64_t stride, int scoring, int renormalize,
                              double scale, const int32_t *index, const float *dweights,
                              void *dlogits, int64_t stride_d, void *stream)
{
    using namespace gett;
    gett_status_t st = route_ok(dtype, tokens, experts, k, scoring);
    if (st != GETT_SUCCESS) return st;
    if (scale != scale) return GETT_ERROR_INVALID_VALUE;
    Extent x, d, ei, ew;
    st = layer_matrix(dtype, tokens, experts, logits, stride, x);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, tokens, experts, dlogits, stride_d, d);
    if (st == GETT_SUCCESS) st = layer_list(tokens * k, 4, index, ei);
    if (st == GETT_SUCCESS) st = layer_list(tokens * k, 4, dweights, ew);
    if (st != GETT_SUCCESS || tokens == 0) return st;
    if (!apart(d, x) || !apart(d, ei) || !apart(d, ew)) return GETT_ERROR_INVALID_VALUE;
    if (!fits_launch((tokens + 3) / 4, 256)) return GETT_ERROR_NOT_SUPPORTED;
    const RouteGradJob j = {logits, dlogits, stride, stride_d, (int)tokens, experts, k, scoring,
                            renormalize, scale, index, dweights};
    return with_experts(experts, [&](auto per) {
        return with_type(dtype, [&](auto v) {
            hipLaunchKernelGGL((route_grad_kernel<decltype(v), decltype(per)::value>),
                               dim3((unsigned)((tokens + 3) / 4)), dim3(256), 0,
                               static_cast<hipStream_t>(stream), j);
            return launched(hipGetLastError());
        });
    });
}

}  // extern "C"
