// The part of HIP that kernels of this library without matrix instructions use, on the CPU: lanes.cpp runs a workgroup's lanes one at a time, in an order that the test sets, so that
// a wait that is missing between wavefronts gives wrong results every time instead of hardly ever. For tests only; the kernels are compiled from their own sources.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <functional>
#include <new>
#include <type_traits>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)

struct dim3 { unsigned x, y, z; dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {} };
struct uint2 { uint32_t x, y; };
struct uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
struct alignas(16) float4 { float x, y, z, w; };
inline uint2 make_uint2(uint32_t x, uint32_t y) { return uint2{x, y}; }
inline float4 make_float4(float x, float y, float z, float w) { return float4{x, y, z, w}; }

typedef void *hipStream_t;
enum hipError_t { hipSuccess = 0, hipErrorLaunchFailure = 719 };
hipError_t hipGetLastError();      // of a launch whose lanes were not together where they have to be

namespace lanes {

extern dim3 thread, block, threads, blocks;      // of the lane that runs

enum Op { NONE, ANY, BALLOT, MOVE, READ, FENCE, BARRIER, DONE };
// What a lane says at a place where lanes meet, and what it hears there. `with`: MOVE's control, READ's lane, BARRIER's line
uint64_t meet(Op op, uint64_t say, int with = 0, int rows = 0xf);
void launch(const char *name, dim3 grid, dim3 size, std::function<void()> kernel);

struct bf16 {      // rounded to the nearest, ties to even
    uint16_t bits;
    explicit bf16(float v)
    {
        uint32_t b;
        memcpy(&b, &v, 4);
        bits = v != v ? (uint16_t)(b >> 16 | 0x40) : (uint16_t)((b + 0x7fff + (b >> 16 & 1)) >> 16);
    }
};

template <class To, class From> inline To bits(From v)
{
    static_assert(sizeof(To) == sizeof(From));
    To to;
    memcpy(&to, &v, sizeof(to));
    return to;
}

}  // namespace lanes

#define __bf16 lanes::bf16
#define threadIdx lanes::thread
#define blockIdx lanes::block
#define blockDim lanes::threads
#define gridDim lanes::blocks
#define hipLaunchKernelGGL(kernel, grid, size, lds, stream, ...) lanes::launch(#kernel, grid, size, [=] { (kernel)(__VA_ARGS__); })
#define asm(...)      // (constants that are to be kept in scalar registers)

#define __syncthreads() (void)lanes::meet(lanes::BARRIER, 0, __LINE__)
#define __builtin_amdgcn_fence(...) (void)lanes::meet(lanes::FENCE, 0)
#define __builtin_amdgcn_wave_barrier() (void)lanes::meet(lanes::FENCE, 0)
#define __builtin_amdgcn_update_dpp(old, v, control, rows, banks, zero) (int)lanes::meet(lanes::MOVE, (uint32_t)(v), control, rows)      // (old is 0, banks all, in these kernels)
#define __builtin_amdgcn_readlane(v, lane) (int)lanes::meet(lanes::READ, (uint32_t)(v), lane)
#define __shfl_xor(v, o) lanes::bits<double>(lanes::meet(lanes::MOVE, lanes::bits<uint64_t>(v), 0x1000 + (o)))      // (of doubles)

inline bool __any(bool v) { return lanes::meet(lanes::ANY, v); }
inline uint64_t __ballot(bool v) { return lanes::meet(lanes::BALLOT, v); }
inline int __popc(uint32_t v) { return __builtin_popcount(v); }
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline int __ffs(uint32_t v) { return __builtin_ffs((int)v); }
inline int __clz(uint32_t v) { return v ? __builtin_clz(v) : 32; }
inline uint32_t __float_as_uint(float v) { return lanes::bits<uint32_t>(v); }
inline float __uint_as_float(uint32_t v) { return lanes::bits<float>(v); }
inline long long __double_as_longlong(double v) { return lanes::bits<long long>(v); }
inline double __longlong_as_double(long long v) { return lanes::bits<double>(v); }
inline double __hiloint2double(int hi, int lo) { return lanes::bits<double>((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo); }
template <class A, class B> inline std::common_type_t<A, B> min(A a, B b) { return b < a ? b : a; }
template <class A, class B> inline std::common_type_t<A, B> max(A a, B b) { return a < b ? b : a; }
// (one lane runs at a time)
template <class T, class V> inline T atomicAdd(T *p, V v) { const T was = *p; *p += (T)v; return was; }
template <class T, class V> inline T atomicMax(T *p, V v) { const T was = *p; *p = std::max(was, (T)v); return was; }
template <class T, class V> inline T atomicMin(T *p, V v) { const T was = *p; *p = std::min(was, (T)v); return was; }
