// The length of many gradients together, and its clipping (clip.h). Squares are exact in 64 bits (fp32 ones rounded once) and summed there, in an order that only the list decides: fp32
// squares would lose gradients below 1e-23 and overflow from 1e19 on.
#include "clip.h"

#include <algorithm>

namespace tr {

namespace {

constexpr int THREADS = 256;

struct Tile { int of; long long at; int len; };

__device__ __forceinline__ Tile tile_at(const ClipList &l, uint32_t t)
{
    int lo = 0, hi = l.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (l.tile[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const long long at = (long long)(t - l.tile[lo]) * CLIP_TILE, left = l.count[lo] - at;
    return Tile{lo, at, (int)(left < CLIP_TILE ? left : CLIP_TILE)};
}

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float &to, float v) { to = v; }
__device__ __forceinline__ void put(bf16_t &to, float v)
{
    const __bf16 b = (__bf16)v;
    __builtin_memcpy(&to, &b, 2);
}

template <class T> __device__ __forceinline__ double squares_of(const T *p, int len)
{
    constexpr int N = 16 / sizeof(T);
    double sum = 0;
    for (int i = threadIdx.x * N; i < len; i += THREADS * N) {
        T v[N];
        if (i + N <= len) __builtin_memcpy(v, p + i, 16);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = i + e < len ? p[i + e] : T(0);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) { const double x = wide(v[e]); sum = fma(x, x, sum); }
    }
    return sum;
}

__device__ __forceinline__ double sum_of_all(double v, double *s)
{
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    return s[0] + s[1] + s[2] + s[3];
}

// bound by memory
__global__ __launch_bounds__(THREADS) void squares_kernel(ClipList l, ClipState *state, bool first, bool last, double max_norm, float *norm)
{
    __shared__ double s_sum[THREADS / 64];
    __shared__ bool s_last;
    double sum = 0;
    const uint32_t tiles = l.tile[l.n];
    for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const Tile x = tile_at(l, t);
        sum += l.half[x.of] ? squares_of((const bf16_t *)l.in[x.of] + x.at, x.len) : squares_of((const float *)l.in[x.of] + x.at, x.len);
    }
    sum = sum_of_all(sum, s_sum);
    if (threadIdx.x == 0) {
        // past the L2, and there before it is counted: the last to arrive finds them all
        __hip_atomic_store(&state->part[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_s_waitcnt(0);
        s_last = __hip_atomic_fetch_add(&state->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    sum = 0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += THREADS) sum += __hip_atomic_load(&state->part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = sum_of_all(sum, s_sum);
    if (threadIdx.x == 0) {
        state->arrived = 0;
        if (!first) sum += state->squares;
        state->squares = sum;
        if (last) {
            const double length = sqrt(sum);
            *norm = (float)length;
            state->scale = length > max_norm && length < INFINITY ? (float)(max_norm / length) : 1.f;     // (infinity, NaN: 1)
        }
    }
}

template <class T> __device__ __forceinline__ void scale_tile(const T *p, T *q, int len, float by)
{
    constexpr int N = 16 / sizeof(T);
    for (int i = threadIdx.x * N; i < len; i += THREADS * N) {
        T v[N];
        if (i + N <= len) {
            __builtin_memcpy(v, p + i, 16);
#pragma unroll
            for (int e = 0; e < N; ++e) put(v[e], wide(v[e]) * by);
            __builtin_memcpy(q + i, v, 16);
        } else {
            for (int e = i; e < len; ++e) put(q[e], wide(p[e]) * by);
        }
    }
}

__global__ __launch_bounds__(THREADS) void scale_kernel(ClipList l, const ClipState *state)
{
    const float by = state->scale;
    const uint32_t tiles = l.tile[l.n];
    for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const Tile x = tile_at(l, t);
        if (by == 1.f && l.in[x.of] == l.out[x.of]) continue;      // as they are
        if (l.half[x.of]) scale_tile((const bf16_t *)l.in[x.of] + x.at, (bf16_t *)l.out[x.of] + x.at, x.len, by);
        else scale_tile((const float *)l.in[x.of] + x.at, (float *)l.out[x.of] + x.at, x.len, by);
    }
}

int groups(const ClipList &l) { return (int)std::max(1u, std::min<uint32_t>(CLIP_GROUPS, l.tile[l.n])); }

}  // namespace

void launch_clip_squares(hipStream_t s, const ClipList &l, ClipState *state, bool first, bool last, double max_norm, float *norm)
{
    hipLaunchKernelGGL(squares_kernel, dim3(groups(l)), dim3(THREADS), 0, s, l, state, first, last, max_norm, norm);
}

void launch_clip_scale(hipStream_t s, const ClipList &l, const ClipState *state)
{
    if (l.n) hipLaunchKernelGGL(scale_kernel, dim3(groups(l)), dim3(THREADS), 0, s, l, state);
}

}  // namespace tr
