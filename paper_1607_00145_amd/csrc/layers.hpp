// layers.hpp -- what the operators of gett_layers.h share: their random numbers,
// activations, argument checks and vectors.
#pragma once
#include "gett_layers.h"
#include "kernel.hpp"
#include "matrix.hpp"

namespace gett {

// ------------------------------------------------------------------ dropout ---

// A call's dropout as its kernels take it; cut 0: none.
struct Drop {
    uint32_t cut;
    float scale;
    uint64_t seed, offset;
    const int64_t *seedAt;   // device, or nullptr
    __device__ __forceinline__ uint64_t key() const { return seedAt ? (uint64_t)*seedAt : seed; }
};

inline bool drop_ok(const gett_dropout_t *d)
{
    return !d || (d->p >= 0.0 && d->p <= 1.0 && (uintptr_t)d->seed_device % 8 == 0);
}
inline Drop drop_of(const gett_dropout_t *d)
{
    if (!d) return {0, 1.0f, 0, 0, nullptr};
    const double t = __builtin_nearbyint(d->p * 65536.0);
    return {(uint32_t)t, t < 65536.0 ? (float)(65536.0 / (65536.0 - t)) : 0.0f, d->seed, d->offset,
            d->seed_device};
}

// The block of counter {c0, c1, offset}: 10 rounds, of which each multiplies two
// words by constants and exchanges the halves of the products, and a key that
// moves by its Weyl constants.
__device__ __forceinline__ void philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t key,
                                       uint32_t out[4])
{
    uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)q;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// philox for one c0 and many c1: what of the first three rounds does not depend on c1
// (four of twenty products) is kept.
struct PhiloxColumn {
    uint32_t a, b, c, d, e;
    uint32_t k0, k1;
};
__device__ __forceinline__ PhiloxColumn philox_column(uint32_t c0, uint64_t offset, uint64_t key)
{
    constexpr uint32_t W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
    constexpr uint64_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u;
    const uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
    const uint64_t p1 = M0 * c0, q1 = M1 * (uint32_t)offset;
    const uint32_t c2 = (uint32_t)(p1 >> 32) ^ (uint32_t)(offset >> 32) ^ k1;
    const uint64_t q2 = M1 * c2;
    const uint64_t p3 = M0 * ((uint32_t)(q2 >> 32) ^ (uint32_t)q1 ^ (k0 + W0));
    return {(uint32_t)(q1 >> 32) ^ k0, (uint32_t)p1 ^ (k1 + W1), (uint32_t)q2 ^ (k0 + 2 * W0),
            (uint32_t)(p3 >> 32) ^ (k1 + 2 * W1), (uint32_t)p3, k0 + 3 * W0, k1 + 3 * W1};
}
__device__ __forceinline__ void philox_row(const PhiloxColumn &s, uint32_t c1, uint32_t out[4])
{
    constexpr uint64_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u;
    const uint64_t p2 = M0 * (c1 ^ s.a);
    const uint64_t q3 = M1 * ((uint32_t)(p2 >> 32) ^ s.b);
    uint32_t c0 = (uint32_t)(q3 >> 32) ^ s.c, c2 = s.d ^ (uint32_t)p2;
    uint32_t c1_ = (uint32_t)q3, c3 = s.e, k0 = s.k0, k1 = s.k1;
#pragma unroll
    for (int i = 3; i < 10; ++i) {
        const uint64_t p = M0 * c0, q = M1 * c2;
        c0 = (uint32_t)(q >> 32) ^ c1_ ^ k0;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c1_ = (uint32_t)q;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1_;
    out[2] = c2;
    out[3] = c3;
}

// Eight neighbours of one row, from a column that is a multiple of 8.  A block
// of random bits serves the eight of them (16 bits each: with 32 the generator, and
// not memory, would be what bounds a 16-bit dropout).
__device__ __forceinline__ void drop8(float v[8], const Drop &d, const uint32_t w[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (w[i] & 0xffff) >= d.cut ? v[2 * i] * d.scale : 0.0f;
        v[2 * i + 1] = (w[i] >> 16) >= d.cut ? v[2 * i + 1] * d.scale : 0.0f;
    }
}
__device__ __forceinline__ void drop8(float v[8], const Drop &d, uint64_t key, uint32_t row, uint32_t col)
{
    uint32_t w[4];
    philox(col >> 3, row, d.offset, key, w);
    drop8(v, d, w);
}

// -------------------------------------------------------------- activations ---

// e^x, within two steps for |x| < 100 or so
__device__ __forceinline__ float quick_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// The tail 1 - cdf(|z|) of the normal distribution and e^(-z^2/2), within 0.8e-7:
// Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26,
//     erfc(x) = (a1 t + ... + a5 t^5) e^(-x^2), t = 1 / (1 + p x), x = |z| / sqrt 2,
// with halved coefficients.  (The library's erff and expf take three times as long,
// and an epilogue of 8192 x 8192 results 170 us.)
__device__ __forceinline__ float normal_tail(float z, float &e)
{
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.23164189f * fabsf(z));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    return t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f +
               t * (-0.7265760135f + t * 0.5307027145f)))) * e;
}
// z, or the number next to an infinity: times 0 it is 0, as the limits are (z of 16 bits
// is infinite beyond 65504 and its slope 0 or 1).  What NaN becomes does not matter:
// the other factor is one.
__device__ __forceinline__ float finite(float z) { return fmaxf(fminf(z, 3e38f), -3e38f); }
__device__ __forceinline__ float gelu(float z)
{
    // z cdf(z), as max(z, 0) less |z| times the tail; |z| finite: of infinity it is 0
    float e;
    const float tail = normal_tail(z, e);
    const float positive = z < 0.0f ? 0.0f : z;   // (a NaN stays one)
    return positive - fminf(fabsf(z), 3e38f) * tail;
}
__device__ __forceinline__ float gelu_slope(float z)
{
    float e;
    const float tail = normal_tail(z, e);
    return (z < 0.0f ? tail : 1.0f - tail) + finite(z) * 0.39894228f * e;
}
__device__ __forceinline__ float silu(float z)
{
    return fmaxf(z, -3e38f) * __builtin_amdgcn_rcpf(1.0f + quick_exp(-z));
}
__device__ __forceinline__ float silu_slope(float z)
{
    const float s = __builtin_amdgcn_rcpf(1.0f + quick_exp(-z));
    return s * (1.0f + finite(z) * (1.0f - s));
}
__device__ __forceinline__ float relu(float z) { return z < 0.0f ? 0.0f : z; }
__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : z != z ? z : 0.0f; }

// Eight numbers through one activation: which one is asked once, and the eight chains
// of dependent instructions run side by side.
template <typename F> __device__ __forceinline__ void each8(float v[8], const float z[8], F f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f(v[i], z[i]);
}
__device__ __forceinline__ void activate8(int kind, float v[8])
{
    if (kind == GETT_ACTIVATION_GELU) each8(v, v, [](float, float z) { return gelu(z); });
    else if (kind == GETT_ACTIVATION_SILU) each8(v, v, [](float, float z) { return silu(z); });
    else if (kind == GETT_ACTIVATION_RELU) each8(v, v, [](float, float z) { return relu(z); });
}
// v times the slope at z
__device__ __forceinline__ void slope8(int kind, float v[8], const float z[8])
{
    if (kind == GETT_ACTIVATION_GELU) each8(v, z, [](float g, float z) { return g * gelu_slope(z); });
    else if (kind == GETT_ACTIVATION_SILU) each8(v, z, [](float g, float z) { return g * silu_slope(z); });
    else if (kind == GETT_ACTIVATION_RELU) each8(v, z, [](float g, float z) { return g * relu_slope(z); });
}

// Between one lane's store to LDS and another's load of it, in one wavefront: the
// hardware does its LDS accesses in order, and this keeps the compiler from moving
// them or from taking a lane's own earlier value.  No instruction of its own.
__device__ __forceinline__ void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------------ vectors ---

// Whole vectors at any element address.  (Stored element by element, eight numbers
// of 16 bits become a store of 12 bytes between two of two.)
typedef int any16 __attribute__((ext_vector_type(4), aligned(2)));
typedef float any16f __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ i4 load16(const void *p)
{
    const any16 w = *reinterpret_cast<const any16 *>(p);
    return i4{w[0], w[1], w[2], w[3]};
}

__device__ __forceinline__ int pack2(float a, float b, bf16)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(int, b2{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ int pack2(float a, float b, _Float16)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(int, h2{(_Float16)a, (_Float16)b});
}

// the same as they lie in memory
template <typename T> __device__ __forceinline__ Run<T, 8> raw8(const T *p, int left)
{
    Run<T, 8> r;
    if (left >= 8) {
        struct {
            i4 v[sizeof(T) / 2];
        } w;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w.v[i] = load16(p + i * (16 / sizeof(T)));
        r = __builtin_bit_cast(Run<T, 8>, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = i < left ? p[i] : from_float<T>(0.0f);
    }
    return r;
}
// `left` of eight neighbours (0 for the others), and back
template <typename T> __device__ __forceinline__ void load8(const T *p, int left, float v[8])
{
    const Run<T, 8> r = raw8(p, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(r.v[i]);
}
template <typename T> __device__ __forceinline__ void store8(T *p, int left, const float v[8])
{
    if (left >= 8) {
        if constexpr (sizeof(T) == 4) {
            any16f *q = reinterpret_cast<any16f *>(p);
            q[0] = any16f{v[0], v[1], v[2], v[3]};
            q[1] = any16f{v[4], v[5], v[6], v[7]};
        } else {
            any16 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], T());
            *reinterpret_cast<any16 *>(p) = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = from_float<T>(v[i]);
    }
}

// ------------------------------------------------------------- host checks ---

constexpr int64_t kLayerRows = (int64_t)1 << 30;   // rows of a matrix, exclusive
constexpr int64_t kLayerCols = (int64_t)1 << 21;   // columns, exclusive
constexpr int kMostExperts = 1024, kMostChoices = 32;

// One matrix argument of a call: what it may overlap, and whether it is there.
struct Extent {
    const char *p;
    int64_t bytes;
};
inline gett_status_t layer_matrix(gett_dtype_t t, int64_t rows, int64_t cols, const void *p,
                                  int64_t stride, Extent &e)
{
    e = {nullptr, 0};
    if (rows < 0 || cols < 0) return GETT_ERROR_INVALID_VALUE;
    if (rows >= kLayerRows || cols >= kLayerCols) return GETT_ERROR_NOT_SUPPORTED;
    if (rows == 0 || cols == 0) return GETT_SUCCESS;
    if (rows > 1 && stride < cols) return GETT_ERROR_INVALID_VALUE;
    if (!p || (uintptr_t)p % type_size(t)) return GETT_ERROR_INVALID_VALUE;
    const int64_t n = span_bytes(rows, cols, rows > 1 ? stride : cols, 1, type_size(t));
    if (n < 0) return GETT_ERROR_NOT_SUPPORTED;
    e = {static_cast<const char *>(p), n};
    return GETT_SUCCESS;
}
// a list of `n` items of `item` bytes
inline gett_status_t layer_list(int64_t n, int64_t item, const void *p, Extent &e)
{
    e = {nullptr, 0};
    if (n <= 0) return GETT_SUCCESS;
    if (!p || (uintptr_t)p % item) return GETT_ERROR_INVALID_VALUE;
    e = {static_cast<const char *>(p), n * item};
    return GETT_SUCCESS;
}
inline bool apart(const Extent &a, const Extent &b)
{
    return !a.bytes || !b.bytes || a.p + a.bytes <= b.p || b.p + b.bytes <= a.p;
}
inline bool activation_ok(int a) { return a >= GETT_ACTIVATION_NONE && a <= GETT_ACTIVATION_SILU; }

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline gett_status_t launched(hipError_t e) { return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP; }

// Calls f with a value of the element type.
template <typename F> auto with_type(gett_dtype_t t, F &&f)
{
    if (t == GETT_FLOAT32) return f(float());
    if (t == GETT_BFLOAT16) return f(bf16());
    return f(_Float16());
}

}  // namespace gett
