// What becomes of a block of products in the losses over the vocabulary. All products are computed transposed: the accumulator registers of a lane run
// along the output's contiguous dimension (runs of 8: tile_feature) and the lanes along its rows, so that a row's softmax needs one exchange between
// lanes, and stores are whole runs.
#pragma once
#include "mfma_common.h"
#include "vocab_loss.h"

namespace tr {

__device__ __forceinline__ void run_of(const f32x16 &c, int h, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c[8 * h + e];
}

// (stores of 8 and 16 bytes need no alignment in global memory: rows of odd length)
template <class U, class T> __device__ __forceinline__ void store_bits(T *p, const U &u) { __builtin_memcpy(p, &u, sizeof(U)); }
__device__ __forceinline__ void store_run(float *p, const float (&v)[8])
{
    store_bits(p, make_float4(v[0], v[1], v[2], v[3]));
    store_bits(p + 4, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b)
{
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}
__device__ __forceinline__ void store_run(bf16_t *p, const float (&v)[8])
{
    store_bits(p, make_uint4(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])));
}
__device__ __forceinline__ void store_one(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_one(bf16_t *p, float v) { *p = (bf16_t)two_bf16(v, 0.f); }
__device__ __forceinline__ float load_one(const float *p) { return *p; }
__device__ __forceinline__ float load_one(const bf16_t *p) { return __uint_as_float((uint32_t)*p << 16); }

// elements k .. k + 7 of a bf16 row of d that may begin anywhere; zeros past its end
__device__ __forceinline__ uint4 load8(const bf16_t *row, int k, int d)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k + 8 <= d) __builtin_memcpy(&v, row + k, 16);
    else {
        uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) if (k + e < d) q[e >> 1] |= (uint32_t)row[k + e] << (16 * (e & 1));
        v = make_uint4(q[0], q[1], q[2], q[3]);
    }
    return v;
}

// A running softmax is (m, s): s = sum of 2^(k c - m) over the products c seen, k = log2(e) / T, m a whole number at least the largest k c (-inf: none seen).
// Since m is whole, moving a sum to another m is exact, and k c - m is rounded once (fma), relative to itself: what is near the top keeps all its bits.
__device__ __forceinline__ float whole_above(float top) { return ceilf(top); }
__device__ __forceinline__ float term(float c, float k, float m) { return __builtin_amdgcn_exp2f(fmaf(c, k, -m)); }
__device__ __forceinline__ float2 join(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), at = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - at) + b.y * __builtin_amdgcn_exp2f(b.x - at));
}

// The running softmax of a lane's N products of one row, value(i) at vocabulary entry first + offset(i), joined with those of the lanes `apart`, 2 apart, ... from it; entries at
// or past `left` from first on do not exist.
template <int N, class Value, class Offset> __device__ __forceinline__ float2 column_softmax(Value value, Offset offset, int left, float k2, int apart)
{
    float top = -INFINITY, sum = 0.f;
    if (left >= offset(N - 1) + 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, value(i));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) top = offset(i) < left ? fmaxf(top, value(i)) : top;
    }
    for (int o = apart; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    top = whole_above(top * k2);
    const float at = top == -INFINITY ? 0.f : top;
    if (left >= offset(N - 1) + 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum += term(value(i), k2, at);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) sum += offset(i) < left ? term(value(i), k2, at) : 0.f;
    }
    for (int o = apart; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    return make_float2(top, sum);
}

// p - 1 of cross entropy's own entry, at place `at` of a run of products c(0) .. c(7), weighed
template <class Product> __device__ __forceinline__ float less_one(Product c, unsigned at, float weight, float lse)
{
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) z = at == e ? c(e) : z;
    return weight * (expf(z - lse) - 1.f);
}

}  // namespace tr
