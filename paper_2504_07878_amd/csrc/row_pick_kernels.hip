// Tokens drawn from rows of logits, and a row's largest logits (row_pick.h).
#include "row_pick.h"

#include <float.h>

namespace tr {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BIN_BITS = 11, BINS = 1 << BIN_BITS;

// Logits as whole numbers in their order. -inf and NaN are no tokens: key 0. (-0 is 0.)
__device__ __forceinline__ uint32_t key_of(float z)
{
    if (!(z > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// f(key, id) for the tokens of a row, 16 bytes at a time; a row may begin at any element
template <class T, class F> __device__ __forceinline__ void each_token(const T *row, int vocab, F f)
{
    constexpr int N = 16 / sizeof(T);
    for (int i = threadIdx.x * N; i < vocab; i += THREADS * N) {
        T v[N];
        if (i + N <= vocab) __builtin_memcpy(v, row + i, 16);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = row[min(i + e, vocab - 1)];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float z;
            if constexpr (sizeof(T) == 4) z = v[e];
            else z = __uint_as_float((uint32_t)v[e] << 16);
            const uint32_t key = i + e < vocab ? key_of(z) : 0;
            if (key) f(key, (uint32_t)(i + e));
        }
    }
}

struct Shared {
    u64 bin[BINS];
    u64 part[WAVES];
    u64 before, at;
    uint32_t place;
    int found;
    u64 entry[PICK_MAX_ENTRIES];
    int entries;
};

__device__ __forceinline__ u64 sum_of_all(u64 v, Shared &s)
{
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % 64 == 0) s.part[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < WAVES; ++w) v += s.part[w];
    return v;
}
__device__ __forceinline__ u64 max_of_all(u64 v, Shared &s)
{
    for (int o = 1; o < 64; o *= 2) v = max(v, __shfl_xor(v, o));
    __syncthreads();
    if (threadIdx.x % 64 == 0) s.part[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < WAVES; ++w) v = max(v, s.part[w]);
    return v;
}

struct Border { bool found; uint32_t place; u64 before, at; };

// The first place up to which the amounts come to `want` (> 0) or more, what lies before it and what at it. each(add) calls add(place, amount) for everything; places are below
// 2^bits. Eleven bits of the place at a time, by a histogram of amounts. All threads get the answer.
template <class Each> __device__ __forceinline__ Border find_border(Each each, int bits, u64 want, Shared &s)
{
    uint32_t base = 0;
    u64 before = 0, at = 0;
    do {
        const int shift = max(0, bits - BIN_BITS);
        const bool whole = bits >= 32;
        const uint32_t span = whole ? 0 : 1u << bits;
        __syncthreads();
        for (int i = threadIdx.x; i < BINS; i += THREADS) s.bin[i] = 0;
        if (threadIdx.x == 0) s.found = 0;
        __syncthreads();
        each([&](uint32_t place, u64 amount) {
            const uint32_t d = place - base;
            if (whole || d < span) atomicAdd(&s.bin[d >> shift], amount);
        });
        __syncthreads();
        constexpr int N = BINS / THREADS;
        u64 mine[N], sum = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) sum += mine[e] = s.bin[threadIdx.x * N + e];
        u64 upto = sum;
        for (int o = 1; o < 64; o *= 2) {
            const u64 v = __shfl_up(upto, o);
            if (threadIdx.x % 64 >= o) upto += v;
        }
        if (threadIdx.x % 64 == 63) s.part[threadIdx.x / 64] = upto;
        __syncthreads();
        u64 run = before + upto - sum;
        for (int w = 0; w < (int)threadIdx.x / 64; ++w) run += s.part[w];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (run < want && want <= run + mine[e]) {      // (for one thread and one bin at most)
                s.found = 1; s.before = run; s.at = mine[e]; s.place = base + ((uint32_t)(threadIdx.x * N + e) << shift);
            }
            run += mine[e];
        }
        __syncthreads();
        if (!s.found) return Border{false, 0, 0, 0};
        base = s.place; before = s.before; at = s.at;
        bits = shift;
    } while (bits > 0);
    return Border{true, base, before, at};
}

// What is kept of a row: all keys above `key`, and of those equal to it ids up to `last`
struct Kept {
    uint32_t key, last;
    __device__ __forceinline__ bool has(uint32_t k, uint32_t id) const { return k > key || (k == key && id <= last); }
};
constexpr uint32_t ANY = 0xffffffffu;

template <class T> __device__ __forceinline__ uint32_t id_of_tie(const T *row, int vocab, int id_bits, uint32_t key, u64 nth, Shared &s)
{
    return find_border([&](auto add) { each_token(row, vocab, [&](uint32_t k, uint32_t id) { if (k == key) add(id, 1); }); }, id_bits, nth, s).place;
}

template <class T> __global__ __launch_bounds__(THREADS) void sample_kernel(PickArgs a, int id_bits)
{
    __shared__ Shared s;
    const int r = blockIdx.x, vocab = a.vocab;
    const T *row = (const T *)a.logits + (long long)r * a.stride;
    const float t = a.temperatures ? a.temperatures[r] : a.temperature, top_p = a.top_ps ? a.top_ps[r] : a.top_p, min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const int top_k = a.top_ks ? a.top_ks[r] : a.top_k;

    u64 first = 0;
    each_token(row, vocab, [&](uint32_t key, uint32_t id) { first = max(first, (u64)key << 32 | (ANY - id)); });
    first = max_of_all(first, s);
    if (!first || !(t > 0.f)) {
        if (threadIdx.x == 0) { a.token[r] = first ? (int)(ANY - (uint32_t)first) : -1; a.logprob[r] = 0.f; }
        return;
    }
    const uint32_t top_key = (uint32_t)(first >> 32);
    const double top = logit_of(top_key), per = 1.4426950408889634 / (double)fminf(t, FLT_MAX), unit = ldexp(1.0, a.unit);
    const auto mass = [&](uint32_t key) { return key == top_key ? (u64)unit : (u64)(exp2(((double)logit_of(key) - top) * per) * unit + 0.5); };

    Kept kept{1, ANY};
    u64 ties = 0;       // 0: all of them
    if (top_k > 0 && top_k < vocab) {
        const Border b = find_border([&](auto add) { each_token(row, vocab, [&](uint32_t key, uint32_t) { add(~key, 1); }); }, 32, top_k, s);
        if (b.found) { kept.key = ~b.place; ties = top_k - b.before < b.at ? top_k - b.before : 0; }
    }
    if (top_p < 1.f) {
        u64 sum = 0, equal = 0;
        each_token(row, vocab, [&](uint32_t key, uint32_t) { sum += key > kept.key || (key == kept.key && !ties) ? mass(key) : 0; });
        if (ties) equal = ties * mass(kept.key);
        sum = sum_of_all(sum, s) + equal;
        const u64 want = min(max((u64)ceil(fmax((double)top_p, 0.0) * (double)sum), 1ull), sum);
        const Border b = find_border([&](auto add) { each_token(row, vocab, [&](uint32_t key, uint32_t) { if (key >= kept.key) add(~key, mass(key)); }); }, 32, want, s);
        const uint32_t key = ~b.place;
        const u64 one = mass(key), need = (want - b.before + one - 1) / one;
        if (key != kept.key || !ties || need < ties) ties = need < b.at / one ? need : 0;
        kept.key = key;
    }
    if (min_p > 0.f) {
        uint32_t least = top_key;
        if (min_p < 1.f) {
            const double at = top + (double)fminf(t, FLT_MAX) * log((double)min_p);
            float f = (float)at;
            if ((double)f < at) f = nextafterf(f, INFINITY);
            least = max(key_of(f), 1u);
        }
        if (least > kept.key) { kept.key = least; ties = 0; }
        if (min_p > 1.f) ties = 1;
    }
    if (ties) kept.last = id_of_tie(row, vocab, id_bits, kept.key, ties, s);

    u64 sum = 0;
    each_token(row, vocab, [&](uint32_t key, uint32_t id) { sum += kept.has(key, id) ? mass(key) : 0; });
    sum = sum_of_all(sum, s);
    const double u = fmin(fmax((double)a.u[r], 0.0), 1.0);
    const u64 below = min((u64)(u * (double)sum), sum - 1);
    const Border b = find_border([&](auto add) { each_token(row, vocab, [&](uint32_t key, uint32_t id) { if (kept.has(key, id)) add(id, mass(key)); }); }, id_bits, below + 1, s);
    if (threadIdx.x == 0) {
        float z;
        if constexpr (sizeof(T) == 4) z = row[b.place];
        else z = __uint_as_float((uint32_t)row[b.place] << 16);
        a.token[r] = (int)b.place;
        a.logprob[r] = (float)((z == top ? 0.0 : ((double)z - top) * per * 0.6931471805599453) - log((double)sum / unit));
    }
}

template <class T> __global__ __launch_bounds__(THREADS) void top_kernel(PickArgs a, int id_bits)
{
    __shared__ Shared s;
    const int r = blockIdx.x, vocab = a.vocab;
    const T *row = (const T *)a.logits + (long long)r * a.stride;
    Kept kept{1, ANY};
    const Border b = find_border([&](auto add) { each_token(row, vocab, [&](uint32_t key, uint32_t) { add(~key, 1); }); }, 32, a.entries, s);
    if (b.found) {
        kept.key = ~b.place;
        const u64 ties = a.entries - b.before;
        if (ties < b.at) kept.last = id_of_tie(row, vocab, id_bits, kept.key, ties, s);
    }
    __syncthreads();
    s.entry[threadIdx.x] = ~0ull;
    if (threadIdx.x == 0) s.entries = 0;
    __syncthreads();
    each_token(row, vocab, [&](uint32_t key, uint32_t id) { if (kept.has(key, id)) s.entry[atomicAdd(&s.entries, 1)] = (u64)~key << 32 | id; });
    for (int size = 2; size <= PICK_MAX_ENTRIES; size *= 2)
        for (int step = size / 2; step; step /= 2) {
            __syncthreads();
            const int i = threadIdx.x, j = i ^ step;
            if (j > i) {
                const u64 x = s.entry[i], y = s.entry[j];
                if ((x > y) == !(i & size)) { s.entry[i] = y; s.entry[j] = x; }
            }
        }
    __syncthreads();
    if ((int)threadIdx.x < a.entries) {
        const u64 e = s.entry[threadIdx.x];
        a.ids[(long long)r * a.entries + threadIdx.x] = e == ~0ull ? -1 : (int)(uint32_t)e;
        a.values[(long long)r * a.entries + threadIdx.x] = e == ~0ull ? -INFINITY : logit_of(~(uint32_t)(e >> 32));
    }
}

int bits_of(int vocab)
{
    int bits = 1;
    while ((1 << bits) < vocab) ++bits;
    return bits;
}

}  // namespace

void launch_sample(hipStream_t s, const PickArgs &a)
{
    if (a.dtype == DT_BF16) hipLaunchKernelGGL(sample_kernel<bf16_t>, dim3(a.rows), dim3(THREADS), 0, s, a, bits_of(a.vocab));
    else hipLaunchKernelGGL(sample_kernel<float>, dim3(a.rows), dim3(THREADS), 0, s, a, bits_of(a.vocab));
}

void launch_top(hipStream_t s, const PickArgs &a)
{
    static_assert(PICK_MAX_ENTRIES == THREADS);
    if (a.dtype == DT_BF16) hipLaunchKernelGGL(top_kernel<bf16_t>, dim3(a.rows), dim3(THREADS), 0, s, a, bits_of(a.vocab));
    else hipLaunchKernelGGL(top_kernel<float>, dim3(a.rows), dim3(THREADS), 0, s, a, bits_of(a.vocab));
}

}  // namespace tr
