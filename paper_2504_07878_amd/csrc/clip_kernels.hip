// The length of many gradients together, and its clipping (clip.h). Squares are exact in 64 bits (fp32 ones rounded once) and summed there, in an order that only the list decides: fp32
// squares would lose gradients below 1e-23 and overflow from 1e19 on.
#include "clip.h"

#include <float.h>

namespace tr {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, LOADS = CLIP_TILE / 16 / THREADS;

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float &to, float v) { to = v; }
__device__ __forceinline__ void put(bf16_t &to, float v)
{
    const __bf16 b = (__bf16)v;
    __builtin_memcpy(&to, &b, 2);
}

template <class T> struct Vector { T v[16 / sizeof(T)]; };
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any;
template <class T> __device__ __forceinline__ void store_past(T *p, const Vector<T> &x)
{
    u32x4_any v;
    __builtin_memcpy(&v, &x, 16);
    __builtin_nontemporal_store(v, (u32x4_any *)p);
}

template <class T> __device__ __forceinline__ Vector<T> load_past(const T *p)
{
    const u32x4_any v = __builtin_nontemporal_load((const u32x4_any *)p);
    Vector<T> x;
    __builtin_memcpy(&x, &v, 16);
    return x;
}

// a whole tile, all its loads at once
template <bool PAST, class T> __device__ __forceinline__ void load_tile(Vector<T> (&x)[LOADS], const T *p)
{
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        if constexpr (PAST) x[i] = load_past(p + (i * THREADS + threadIdx.x) * N);
        else __builtin_memcpy(&x[i], p + (i * THREADS + threadIdx.x) * N, 16);
    }
}

// f(gradient, first element, elements, whether to read past the caches) for the tiles of a list that are this workgroup's
template <bool BACK, class F> __device__ __forceinline__ void each_tile(const ClipList &l, F f)
{
    const uint32_t tiles = l.tile[l.n];
    int i = 0;
    for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        while (l.tile[i + 1] <= t) ++i;
        const int size = l.half[i] ? 2 : 4;
        const long long at = (long long)(BACK ? l.tile[i + 1] - 1 - t : t - l.tile[i]) * (CLIP_TILE / size), left = l.count[i] - at;
        f(i, at, (int)(left < CLIP_TILE / size ? left : CLIP_TILE / size), BACK ? t >= l.past : t < l.past);
    }
}

template <bool PAST, class T> __device__ __forceinline__ double squares_of(const T *p, int len)
{
    constexpr int N = 16 / sizeof(T);
    double sum = 0;
    const auto add = [&](const Vector<T> &x) {
#pragma unroll
        for (int e = 0; e < N; ++e) { const double y = wide(x.v[e]); sum = fma(y, y, sum); }
    };
    if (len == CLIP_TILE / (int)sizeof(T)) {
        Vector<T> x[LOADS];
        load_tile<PAST>(x, p);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) add(x[i]);
        return sum;
    }
    for (int i = threadIdx.x * N; i < len; i += THREADS * N) {
        Vector<T> x{};
        if (i + N <= len) __builtin_memcpy(&x, p + i, 16);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) if (i + e < len) x.v[e] = p[i + e];
        }
        add(x);
    }
    return sum;
}

__device__ __forceinline__ double sum_of_all(double v, double *s)
{
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < WAVES; ++w) v += s[w];
    return v;
}

__device__ __forceinline__ double sum_of_sums(const double *sums, int n, double *s)
{
    double v = 0;
    for (int i = threadIdx.x; i < n; i += THREADS) v += sums[i];
    return sum_of_all(v, s);
}

// Bound by memory: 494 million bf16 elements at 6.3 TB/s, 5.6 where none of them is in the last-level cache.
__global__ __launch_bounds__(THREADS) void squares_kernel(ClipList l, double *sums)
{
    __shared__ double s[WAVES];
    double sum = 0;
    each_tile<false>(l, [&](int i, long long at, int len, bool past) {
        if (l.half[i]) sum += past ? squares_of<true>((const bf16_t *)l.in[i] + at, len) : squares_of<false>((const bf16_t *)l.in[i] + at, len);
        else sum += past ? squares_of<true>((const float *)l.in[i] + at, len) : squares_of<false>((const float *)l.in[i] + at, len);
    });
    sum = sum_of_all(sum, s);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__global__ __launch_bounds__(THREADS) void join_kernel(const double *sums, int n, double *to, float *norm)
{
    __shared__ double s[WAVES];
    const double sum = sum_of_sums(sums, n, s);      // (behind a barrier: `to` may be one of them)
    if (threadIdx.x == 0) {
        if (to) *to = sum;
        if (norm) *norm = (float)sqrt(sum);
    }
}

// by * 2^shift: a scale below 2^-126 keeps all its bits. (One more instruction an element, beside the memory: 494 million fp32 elements 1004 us with it and without.)
struct Scale {
    float by;
    int shift;
    __device__ __forceinline__ float operator()(float v) const { return ldexpf(v * by, shift); }
    __device__ __forceinline__ bool none() const { return by == 1.f && shift == 0; }
};

template <bool PAST, class T> __device__ __forceinline__ void scale_tile(const T *p, T *q, int len, Scale by)
{
    constexpr int N = 16 / sizeof(T);
    const auto scale = [&](Vector<T> &x) {
#pragma unroll
        for (int e = 0; e < N; ++e) put(x.v[e], by(wide(x.v[e])));
    };
    if (len == CLIP_TILE / (int)sizeof(T)) {
        Vector<T> x[LOADS];
        load_tile<PAST>(x, p);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            scale(x[i]);
            store_past(q + (i * THREADS + threadIdx.x) * N, x[i]);
        }
        return;
    }
    for (int i = threadIdx.x * N; i < len; i += THREADS * N) {
        if (i + N <= len) {
            Vector<T> x;
            __builtin_memcpy(&x, p + i, 16);
            scale(x);
            __builtin_memcpy(q + i, &x, 16);
        } else {
            for (int e = i; e < len; ++e) put(q[e], by(wide(p[e])));
        }
    }
}

// Bound by memory: what was squared last is scaled first, as it may still be in the last-level cache, and stores go past it. (136 million bf16 elements into a buffer, squares included: 165 us
// forwards, 153 backwards, 127 with such stores, 124 with loads as clip.h has them.)
__global__ __launch_bounds__(THREADS) void scale_kernel(ClipList l, const double *sums, int n, double max_norm, float *norm)
{
    __shared__ double s[WAVES];
    const double length = sqrt(sum_of_sums(sums, n, s));
    const float said = (float)length;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = said;
    double ratio = length > max_norm && said < INFINITY ? max_norm / length : 1.0;      // (infinity, lengths that 32 bits do not hold, NaN: 1)
    int shift = 0;
    if (ratio < FLT_MIN) ratio = frexp(ratio, &shift);
    const Scale by{(float)ratio, shift};
    each_tile<true>(l, [&](int i, long long at, int len, bool past) {
        if (by.none() && l.in[i] == l.out[i]) return;      // as they are
        const auto scale = [&](const auto *p, auto *q) {
            if (past) scale_tile<true>(p + at, q + at, len, by);
            else scale_tile<false>(p + at, q + at, len, by);
        };
        if (l.half[i]) scale((const bf16_t *)l.in[i], (bf16_t *)l.out[i]);
        else scale((const float *)l.in[i], (float *)l.out[i]);
    });
}

}  // namespace

void launch_clip_squares(hipStream_t s, const ClipList &l, double *sums) { hipLaunchKernelGGL(squares_kernel, dim3(clip_groups(l)), dim3(THREADS), 0, s, l, sums); }

void launch_clip_join(hipStream_t s, const double *sums, int n, double *to, float *norm) { hipLaunchKernelGGL(join_kernel, dim3(1), dim3(THREADS), 0, s, sums, n, to, norm); }

void launch_clip_scale(hipStream_t s, const ClipList &l, const double *sums, int n, double max_norm, float *norm)
{
    hipLaunchKernelGGL(scale_kernel, dim3(clip_groups(l)), dim3(THREADS), 0, s, l, sums, n, max_norm, norm);
}

}  // namespace tr
