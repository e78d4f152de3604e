// route.hip -- the choice of experts and the order of the chosen rows.
//
// A wavefront takes a token: lane l holds the experts l, l + 64, ...; the k largest
// are taken one by one (k is small), each the largest of the lanes' largest.  The
// order of the rows by expert is a stable counting sort: chunks of 1024 rows are
// counted, the counts summed over the chunks, and each chunk writes its rows, with no
// atomics whose order could show.  Up to 1024 rows it is one launch of one
// workgroup in all.
#include "launch.hpp"
#include "layer_util.hpp"

namespace gett {

namespace {

constexpr int kChunk = 1024;   // rows (token, choice) that a workgroup orders

struct RouteJob {
    const void *logits;
    int64_t ld;
    const float *bias;
    int tokens, experts, k, scoring, groups, topGroups, renormalize;
    double scale;
    float *weights;
    int32_t *index, *order, *offsets, *place;
    int32_t *counts;   // chunks x experts
    int chunks;
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

// One token; `keys` holds `experts` doubles of LDS of the wavefront's own.
template <typename T, int PER>
__device__ __forceinline__ void choose(const RouteJob &j, int64_t token, double *keys)
{
    const int lane = (int)threadIdx.x & 63;
    const double none = -__builtin_huge_val();
    const T *row = reinterpret_cast<const T *>(j.logits) + token * j.ld;
    float x[PER];
    bool nan = false;
    float most = -__builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        x[i] = e < j.experts ? to_float(row[e]) : -__builtin_huge_valf();
        if (x[i] != x[i]) {
            nan = true;
            x[i] = -__builtin_huge_valf();
        }
        most = fmaxf(most, x[i]);
    }
    nan = __any(nan);
    most = wave_max(most);
    // scores in 64 bits
    double s[PER], total = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (j.scoring == GETT_SCORE_SOFTMAX) {
            s[i] = x[i] == -__builtin_huge_valf() ? 0.0 : exp((double)x[i] - (double)most);
            total += s[i];
        } else {
            s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
        }
    }
    if (j.scoring == GETT_SCORE_SOFTMAX) {
        total = wave_sum(total);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] /= total;
    }
    // choices
    const bool plain = !j.bias && j.groups == 1;
    double key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        double c = none;
        if (e < j.experts && x[i] != -__builtin_huge_valf()) {
            c = plain ? (double)x[i] : j.bias ? s[i] + (double)j.bias[e] : s[i];
            if (c != c) c = none;
        }
        key[i] = c;
    }
    if (j.groups > 1) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i * 64 + lane < j.experts) keys[i * 64 + lane] = key[i];
        const int size = j.experts / j.groups;
        // lane g holds the groups g, g + 64, ...
        double score[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int g = i * 64 + lane;
            double a = none, b = none;
            if (g < j.groups)
                for (int e = g * size; e < (g + 1) * size; ++e) {
                    const double v = keys[e];
                    if (v > a) {
                        b = a;
                        a = v;
                    } else if (v > b) {
                        b = v;
                    }
                }
            score[i] = b > none ? a + b : a;
        }
        uint32_t open = 0;   // of this lane's groups
        for (int r = 0; r < j.topGroups; ++r) {
            Best b = {none, INT32_MAX};
#pragma unroll
            for (int i = 0; i < PER; ++i) b.take(score[i], i * 64 + lane);
            b = wave_best(b);
            if (b.key == none) break;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (b.at == i * 64 + lane) {
                    open |= 1u << i;
                    score[i] = none;
                }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = i * 64 + lane, g = e < j.experts ? e / size : 0;
            const uint32_t bits = __shfl(open, g & 63);
            if (!(bits >> (g >> 6) & 1)) key[i] = none;
        }
    }
    // the k largest: lane r keeps the r-th
    int mine = -1;
    double score = 0.0, sum = 0.0;
    for (int r = 0; r < j.k; ++r) {
        Best b = {none, INT32_MAX};
#pragma unroll
        for (int i = 0; i < PER; ++i) b.take(key[i], i * 64 + lane);
        b = wave_best(b);
        if (b.key == none) break;
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (b.at == i * 64 + lane) {
                v = s[i];
                key[i] = none;
            }
        v = __shfl(v, b.at & 63);
        sum += v;
        if (lane == r) {
            mine = b.at;
            score = v;
        }
    }
    if (lane < j.k) {
        double w = score;
        if (j.renormalize) w = sum > 0.0 || sum != sum ? score / sum : 0.0;
        float out = mine < 0 ? 0.0f : (float)(w * j.scale);
        if (nan || (j.scoring == GETT_SCORE_SOFTMAX && most == __builtin_huge_valf()))
            out = __builtin_nanf("");
        j.weights[token * j.k + lane] = out;
        j.index[token * j.k + lane] = mine;
    }
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

// Writes a chunk's rows.  `waves` holds 16 x experts counts; base[e] is where the
// chunk's rows of expert e begin.
__device__ __forceinline__ void place_chunk(const RouteJob &j, int chunk, int32_t *waves,
                                            const int32_t *base)
{
    const int rows = j.tokens * j.k;
    const int r = chunk * kChunk + (int)threadIdx.x, lane = (int)threadIdx.x & 63;
    const int wave = (int)threadIdx.x >> 6;
    const int e = r < rows ? j.index[r] : -1;
    for (int i = (int)threadIdx.x; i < 16 * j.experts; i += kChunk) waves[i] = 0;
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
    } else if (r < rows) {
        j.place[r] = -1;
    }
}

// Rows of a chunk per expert.
__device__ __forceinline__ void count_chunk(const RouteJob &j, int chunk, int32_t *counts)
{
    for (int i = (int)threadIdx.x; i < j.experts; i += kChunk) counts[i] = 0;
    __syncthreads();
    const int r = chunk * kChunk + (int)threadIdx.x;
    const int e = r < j.tokens * j.k ? j.index[r] : -1;
    if (e >= 0) atomicAdd(&counts[e], 1);   // (whole numbers: in any order the same)
    __syncthreads();
}

// counts[experts] -> where each begins, and offsets[experts] last; 1024 threads.
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
__global__ __launch_bounds__(256) void route_choose_kernel(RouteJob j)
{
    __shared__ double keys[4][64 * PER];
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token < j.tokens) choose<T, PER>(j, token, keys[threadIdx.x >> 6]);
}

__global__ __launch_bounds__(kChunk) void route_count_kernel(RouteJob j)
{
    __shared__ int32_t counts[kMostExperts];
    count_chunk(j, (int)blockIdx.x, counts);
    for (int i = (int)threadIdx.x; i < j.experts; i += kChunk)
        j.counts[(int64_t)blockIdx.x * j.experts + i] = counts[i];
}

// Counts of the chunks -> where each chunk's rows of each expert begin.
__global__ __launch_bounds__(kChunk) void route_scan_kernel(RouteJob j)
{
    __shared__ int32_t lds[16];
    const int e = (int)threadIdx.x;
    int total = 0;
    if (e < j.experts)
        for (int c = 0; c < j.chunks; ++c) total += j.counts[(int64_t)c * j.experts + e];
    int at = scan_experts(total, lds);
    if (e >= j.experts) return;
    j.offsets[e] = at;
    if (e == j.experts - 1) j.offsets[j.experts] = at + total;
    for (int c = 0; c < j.chunks; ++c) {
        const int n = j.counts[(int64_t)c * j.experts + e];
        j.counts[(int64_t)c * j.experts + e] = at;
        at += n;
    }
}

__global__ __launch_bounds__(kChunk) void route_place_kernel(RouteJob j)
{
    extern __shared__ int32_t waves[];
    place_chunk(j, (int)blockIdx.x, waves, j.counts + (int64_t)blockIdx.x * j.experts);
    const int r = (int)blockIdx.x * kChunk + (int)threadIdx.x;
    if (r < j.tokens * j.k && r >= j.offsets[j.experts]) j.order[r] = -1;
}

// Everything, for up to 1024 rows.
template <typename T, int PER>
__global__ __launch_bounds__(kChunk) void route_small_kernel(RouteJob j)
{
    extern __shared__ __attribute__((aligned(256))) char dyn_lds[];
    __shared__ int32_t counts[kMostExperts];
    __shared__ int32_t lds[16];
    __shared__ int total;
    const int wave = (int)threadIdx.x >> 6;
    double *keys = reinterpret_cast<double *>(dyn_lds) + wave * j.experts;
    for (int t = wave; t < j.tokens; t += 16) choose<T, PER>(j, t, keys);
    __syncthreads();   // (drains the stores, which this workgroup reads back)
    count_chunk(j, 0, counts);
    const int e = (int)threadIdx.x;
    const int n = e < j.experts ? counts[e] : 0;
    const int at = scan_experts(n, lds);
    if (e < j.experts) {
        counts[e] = at;
        j.offsets[e] = at;
    }
    if (e == j.experts - 1) {
        j.offsets[j.experts] = at + n;
        total = at + n;
    }
    __syncthreads();
    place_chunk(j, 0, reinterpret_cast<int32_t *>(dyn_lds), counts);
    const int r = (int)threadIdx.x;
    if (r < j.tokens * j.k && r >= total) j.order[r] = -1;
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

// With c the chosen scores and w = scale c / sum c (or scale c), g = scale dweights:
//     renormalised  dc = (g - sum(g c) / sum c) / sum c
//     softmax       dx = s (ds - sum(ds s)),  sigmoid  dx = ds s (1 - s)
// where ds is dc at the chosen experts and 0 elsewhere.
template <typename T, int PER>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteGradJob j)
{
    __shared__ float spread[4][64 * PER];
    const int lane = (int)threadIdx.x & 63;
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= j.tokens) return;
    float *ds = spread[threadIdx.x >> 6];
    const T *row = reinterpret_cast<const T *>(j.logits) + token * j.ld;
    float x[PER], most = -__builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        x[i] = e < j.experts ? to_float(row[e]) : -__builtin_huge_valf();
        most = fmaxf(most, x[i]);
        if (e < j.experts) ds[e] = 0.0f;
    }
    most = wave_max(most);
    double s[PER], total = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (j.scoring == GETT_SCORE_SOFTMAX) {
            s[i] = x[i] == -__builtin_huge_valf() ? 0.0 : exp((double)x[i] - (double)most);
            total += s[i];
        } else {
            s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
        }
    }
    if (j.scoring == GETT_SCORE_SOFTMAX) {
        total = wave_sum(total);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = total > 0.0 || total != total ? s[i] / total : 0.0;
    }
    // lane r: the r-th choice and its score
    int at = lane < j.k ? j.index[token * j.k + lane] : -1;
    if (at >= j.experts) at = -1;
    double c = 0.0;
    for (int r = 0; r < j.k; ++r) {
        const int e = __shfl(at, r);
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e >= 0 && i == e >> 6) v = s[i];
        v = __shfl(v, e & 63);
        if (lane == r && e >= 0) c = v;
    }
    double g = at >= 0 ? j.scale * (double)j.dweights[token * j.k + lane] : 0.0;
    if (j.renormalize) {
        const double sum = wave_sum(c), dot = wave_sum(g * c);
        g = at >= 0 && (sum > 0.0 || sum != sum) ? (g - dot / sum) / sum : 0.0;
    }
    // sum(ds s), which the renormalised gradient has at zero
    const double dot = j.scoring == GETT_SCORE_SOFTMAX ? wave_sum(at >= 0 ? g * c : 0.0) : 0.0;
    // the chosen experts' own values, in 64 bits until here
    T *out = reinterpret_cast<T *>(j.dlogits) + token * j.ldd;
    if (at >= 0)
        ds[at] = (float)(j.scoring == GETT_SCORE_SOFTMAX ? c * (g - dot) : g * c * (1.0 - c));
    uint32_t chosen = 0;
    for (int r = 0; r < j.k; ++r) {
        const int e = __shfl(at, r);
        if (e >= 0 && (e & 63) == lane) chosen |= 1u << (e >> 6);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        if (e >= j.experts) continue;
        const float rest = j.scoring == GETT_SCORE_SOFTMAX ? (float)(-s[i] * dot) : 0.0f;
        out[e] = from_float<T>(chosen >> i & 1 ? ds[e] : rest);
    }
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
    if (experts > kMostExperts || k > kMostChoices || tokens >= kLayerRows ||
        tokens * k >= INT32_MAX - kChunk)
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
    const int64_t chunks = (rows + kChunk - 1) / kChunk;
    RouteJob j = {logits, stride, bias, (int)tokens, experts, k, scoring, groups, top_groups, renormalize,
                  scale, weights, index, order, offsets, place, nullptr, (int)chunks};
    // 16 counts, or doubles, an expert
    const size_t countBytes = 16 * (size_t)experts * 4, keyBytes = 16 * (size_t)experts * 8;
    if (chunks <= 1)
        return with_experts(experts, [&](auto per) {
            return with_type(dtype, [&](auto v) {
                constexpr auto kernel = route_small_kernel<decltype(v), decltype(per)::value>;
                if (allow_dynamic_lds<kernel>(16 * 64 * decltype(per)::value * 8) != hipSuccess)
                    return GETT_ERROR_HIP;
                hipLaunchKernelGGL(kernel, dim3(1), dim3(kChunk), keyBytes, s, j);
                return launched(hipGetLastError());
            });
        });
    if (!fits_launch(chunks, kChunk)) return GETT_ERROR_NOT_SUPPORTED;
    Partials hold;
    st = stream_workspace(s, 0, (uint64_t)chunks * experts * 4, hold);
    if (st != GETT_SUCCESS) return st;
    j.counts = static_cast<int32_t *>(hold.tiles);
    st = with_experts(experts, [&](auto per) {
        return with_type(dtype, [&](auto v) {
            hipLaunchKernelGGL((route_choose_kernel<decltype(v), decltype(per)::value>),
                               dim3((unsigned)((tokens + 3) / 4)), dim3(256), 0, s, j);
            return launched(hipGetLastError());
        });
    });
    if (st != GETT_SUCCESS) return st;
    hipLaunchKernelGGL(route_count_kernel, dim3((unsigned)chunks), dim3(kChunk), 0, s, j);
    hipLaunchKernelGGL(route_scan_kernel, dim3(1), dim3(kChunk), 0, s, j);
    if (allow_dynamic_lds<route_place_kernel>(16 * kMostExperts * 4) != hipSuccess) return GETT_ERROR_HIP;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)chunks), dim3(kChunk), countBytes, s, j);
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
