// Tokens drawn from rows of logits, and a row's largest logits (row_pick.h).
//
// Every wavefront reads a part of a row once and leaves its largest tokens (up to `listed` of 1024, whatever their logits: it looks for a threshold that few enough
// lanes reach) and, where they are asked for, its sum of weights (parts_kernel). A workgroup a row takes the parts' tokens: down to the largest of the parts' thresholds it
// has them all (decide_kernel). As long as top-k, top-p and min-p end above that, they and the draw are searches among these. A row so flat that top-p or min-p do not is read twice more:
// for the step of a histogram of masses in which top-p ends (steps_kernel), and for the tokens in that step and the sums of what is above it, part by part (place_kernel, finish_kernel).
// Rows of up to 8192 tokens are one workgroup's from the start.
//
// What runs once a workgroup is kept short: loops over tokens are not unrolled, and tokens lie in LDS for it. Instructions that are fetched for the first time cost more here than
// executing them (the same in registers, unrolled: 88 KB of code for decide_kernel, 12.8 us for one row with top-k and top-p).
#include "row_pick.h"

#include <algorithm>
#include <float.h>

namespace tr {

namespace {

typedef unsigned long long u64;
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any;

constexpr int THREADS = PICK_THREADS, WAVES = PICK_WAVES, EACH = PICK_PART / 64;
constexpr int DECIDERS = 512;      // threads of a workgroup that decides on a row (1024: 9.6 instead of 7.8 us for one row)
constexpr int BIN_BITS = 9, BINS = 1 << BIN_BITS;
static_assert(BINS == DECIDERS);
constexpr int MAX_PARTS = PICK_MAX_VOCAB / PICK_PART;
constexpr int FEW = 256, FEW_PLACES = 128;      // tokens that are compared with each other, all with all, instead of all that is left to do, or of a step (5 us among 250)
constexpr int LESS = 2048;    // tokens that are put together once a search has left so few
constexpr uint32_t LOWEST = 0x00800000u, ANY = 0xffffffffu;      // key of the lowest finite logit
constexpr int PER = PICK_PART / DECIDERS;      // tokens of a part, or parts of a row, a thread
static_assert(MAX_PARTS == PICK_PART);

// Logits as whole numbers in their order. -inf and NaN are no tokens: key 0. (-0 is 0.)
__device__ __forceinline__ uint32_t key_of(float z)
{
    if (!(z > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }

// ------------------------------------------------------------------ across lanes

// v of a lane before this one (row_shr, row_bcast), or zeros
template <int C, int ROWS, class V> __device__ __forceinline__ V lanes_before(V v)
{
    if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), C, ROWS, 0xf, false));
    else {
        const u64 x = __builtin_bit_cast(u64, v);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, C, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), C, ROWS, 0xf, false);
        return __builtin_bit_cast(V, (u64)hi << 32 | lo);
    }
}
// v of another lane (quad_perm, row_half_mirror, row_mirror)
template <int C> __device__ __forceinline__ u64 lanes_from(u64 v)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, C, 0xf, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), C, 0xf, 0xf, false);
    return (u64)hi << 32 | lo;
}
// join of the values of all lanes up to this one; zero is the join's neutral value
template <class V, class Join> __device__ __forceinline__ V wave_upto(V v, Join join)
{
    v = join(v, lanes_before<0x111, 0xf>(v));
    v = join(v, lanes_before<0x112, 0xf>(v));
    v = join(v, lanes_before<0x114, 0xf>(v));
    v = join(v, lanes_before<0x118, 0xf>(v));
    v = join(v, lanes_before<0x142, 0xa>(v));
    return join(v, lanes_before<0x143, 0xc>(v));
}
template <class V> __device__ __forceinline__ V last_lane(V v)
{
    if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    else {
        const u64 x = __builtin_bit_cast(u64, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, 63), hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), 63);
        return __builtin_bit_cast(V, (u64)hi << 32 | lo);
    }
}
struct Plus { template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct Larger { template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; } };
template <class V> __device__ __forceinline__ V wave_sum(V v) { return last_lane(wave_upto(v, Plus{})); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { return last_lane(wave_upto(v, Larger{})); }

// ------------------------------------------------------------------ weights

// The exponential by a table and a short polynomial is P. T. P. Tang's method (Table-driven implementation of the exponential function in IEEE floating-point arithmetic, ACM Transactions on
// Mathematical Software 15, 1989), with values of its own: 2^(j / 32) as 64-bit words, less j << 47, so that with k << 47 added, k = 32 e + j, it is the word of 2^(k / 32)
__device__ const uint2 POWERS[32] = {
    {0x00000000, 0x3ff00000}, {0xd3158574, 0x3fefd9b0}, {0x6cf9890f, 0x3fefb558}, {0xd0125b51, 0x3fef9301}, {0x3c7d517b, 0x3fef72b8}, {0x3168b9aa, 0x3fef5487},
    {0x6e756238, 0x3fef387a}, {0xf51fdee1, 0x3fef1e9d}, {0x0a31b715, 0x3fef06fe}, {0x373aa9cb, 0x3feef1a7}, {0x4c123422, 0x3feedea6}, {0x6061892d, 0x3feece08},
    {0xd5362a27, 0x3feebfda}, {0x569d4f82, 0x3feeb42b}, {0xdd485429, 0x3feeab07}, {0xb03a5585, 0x3feea47e}, {0x667f3bcd, 0x3feea09e}, {0xe8ec5f74, 0x3fee9f75},
    {0x73eb0187, 0x3feea114}, {0x994cce13, 0x3feea589}, {0x422aa0db, 0x3feeace5}, {0xb0cdc5e5, 0x3feeb737}, {0x82a3f090, 0x3feec491}, {0xb23e255d, 0x3feed503},
    {0x995ad3ad, 0x3feee89f}, {0xf2fb5e47, 0x3feeff76}, {0xdd85529c, 0x3fef199b}, {0xdcef9069, 0x3fef3720}, {0xdcfba487, 0x3fef5818}, {0x337b9b5f, 0x3fef7c97},
    {0xa2a490da, 0x3fefa4af}, {0x5b6e4540, 0x3fefd076}};

// a constant in scalar registers: an operand of a multiply-add there, where the compiler would copy it to vector registers every time
__device__ __forceinline__ double uniform(double v)
{
    asm("" : "+s"(v));
    return v;
}

// What a row's user set, and what weights are relative to
struct Row {
    float t, p, m;
    int k;                    // 0: all
    bool cut, summed;         // some filter is set; the parts' sums are wanted
    double top, per, unit;    // largest logit, 32 log2(e) / T, 2^a.unit
    uint32_t top_key;
    const uint2 *powers;      // in LDS: 32 entries are one to each pair of banks
    // exp((z - top) / T) = 2^(x / 32), x = k + f, |f| <= 1/2: 2^(k / 32) from the table, 2^(f / 32) - 1 = f q(f), q interpolated at four Chebyshev nodes (1.6e-13 off at most). 64 bits
    // are for the borders: a share that top-p ends at, or a draw, that is off by 1e-8 of all takes another token once in a hundred rows of a hundred thousand even tokens.
    __device__ __forceinline__ double weight(float z) const { return top == INFINITY ? infinite_weight(z) : finite_weight(z); }
    __device__ __forceinline__ double infinite_weight(float z) const { return z == INFINITY ? 1.0 : 0.0; }
    __device__ __forceinline__ double finite_weight(float z) const
    {
        constexpr double WHOLE = 6755399441055744.0;      // 3 2^51: what is added to it is rounded to a whole number
        const double x = fmax(((double)z - top) * per, -32000.0), n = x + WHOLE, f = x - (n - WHOLE);
        const uint32_t k = (uint32_t)__double_as_longlong(n);
        const double q = fma(fma(fma(fma(uniform(9.172598566029335e-09), f, uniform(1.6938609067364198e-06)), f, uniform(0.00023459619820112603)), f, uniform(0.021660849392187844)), f, 1.0);
        const uint2 word = powers[k & 31];
        return __hiloint2double((int)(word.y + (k << 15)), (int)word.x) * q;
    }
    // in units (2^51 of them at most: rounded by adding 2^52)
    __device__ __forceinline__ u64 in_units(double w) const { return (u64)__double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull; }
    __device__ __forceinline__ u64 mass(float z) const { return in_units(weight(z)); }
    __device__ __forceinline__ u64 mass(uint32_t key) const { return mass(logit_of(key)); }
    __device__ __forceinline__ void relative_to(uint32_t key) { top_key = key; top = logit_of(key); }
};

__device__ __forceinline__ void load_powers(uint2 *powers) { if (threadIdx.x % 64 < 32) powers[threadIdx.x % 64] = POWERS[threadIdx.x % 64]; }      // (every wavefront all of them)

template <bool TOP> __device__ __forceinline__ Row row_of(const PickArgs &a, int r, const uint2 *powers)
{
    Row row{};
    row.t = 1.f; row.p = 1.f;
    if constexpr (TOP) row.k = a.entries;
    else {
        const float t = a.temperatures ? a.temperatures[r] : a.temperature;
        if (t > 0.f) {
            row.t = fminf(t, FLT_MAX);
            row.p = a.top_ps ? a.top_ps[r] : a.top_p;
            row.m = a.min_ps ? a.min_ps[r] : a.min_p;
            row.k = max(a.top_ks ? a.top_ks[r] : a.top_k, 0);
        } else row.k = 1;          // the first of the order
    }
    if (row.k >= a.vocab) row.k = 0;
    row.cut = row.k > 0 || row.p < 1.f || row.m > 0.f;
    row.summed = !TOP && row.k == 0 && (row.p < 1.f || !row.cut);
    row.per = 46.16624130844683 / (double)row.t;
    row.unit = __longlong_as_double((long long)(1023 + a.unit) << 52);
    row.powers = powers;
    return row;
}

// The smallest key that min_p (> 0) keeps: weight >= min_p where the logit is at least max + T log min_p
__device__ __forceinline__ uint32_t least_key(const Row &r)
{
    if (!(r.m < 1.f)) return r.top_key;
    const double at = r.top + (double)r.t * log((double)r.m);
    float f = (float)at;
    if ((double)f < at) f = nextafterf(f, INFINITY);
    return max(key_of(f), LOWEST);
}

__device__ __forceinline__ double evenly(float u) { return fmin(fmax((double)u, 0.0), 1.0); }      // (NaN: 0)

// ------------------------------------------------------------------ a workgroup's searches

template <int HELD, bool WHOLE = false> struct Shared {
    static constexpr bool by_place = WHOLE;      // a token's id is its place
    u64 bin[BINS];
    u64 part[DECIDERS / 64];
    u64 before, at;
    double run;
    uint2 powers[32];
    uint32_t place, top, from, n, most, least;
    uint32_t first, last;
    int found, entries;
    u64 few[FEW], few_mass[FEW];
    union {
        u64 entry[PICK_MAX_ENTRIES];
        u64 mass[MAX_PARTS];
    };
    uint32_t key[HELD + LESS], id[(WHOLE ? 0 : HELD) + LESS];      // tokens, key 0: none; behind them those that a first step has left
    static constexpr int held = HELD, ids = WHOLE ? 0 : HELD;
};

// sum of the values of all threads up to this one, and of all
template <class V, class S> __device__ __forceinline__ V sum_upto(V v, V &total, S &s)
{
    static_assert(sizeof(V) == 8);
    v = wave_upto(v, Plus{});
    __syncthreads();
    if (threadIdx.x % 64 == 63) s.part[threadIdx.x / 64] = __builtin_bit_cast(u64, v);
    __syncthreads();
    V run = 0, before = 0;
#pragma unroll
    for (int w = 0; w < DECIDERS / 64; ++w) {
        if (w == (int)threadIdx.x / 64) before = run;
        run += __builtin_bit_cast(V, s.part[w]);
    }
    total = run;
    return before + v;
}
template <class V, class S> __device__ __forceinline__ V sum_of_all(V v, S &s)
{
    V total;
    sum_upto(v, total, s);
    return total;
}

struct Border { bool found; uint32_t place; u64 before, at; };

// One step of find_border: places from `base` on, below base + 2^bits, in steps of 2^shift; what lies before base comes to `before`. place: where the step begins; at: what it holds.
template <class Each, class S> __device__ __forceinline__ Border border_step(Each each, uint32_t base, int bits, int shift, u64 before, u64 want, S &s)
{
    const uint32_t most = bits >= 32 ? ANY : (1u << bits) - 1;
    __syncthreads();
    s.bin[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.found = 0;
    __syncthreads();
    each([&](uint32_t place) { return place - base <= most; }, [&](uint32_t place, u64 amount) { atomicAdd(&s.bin[(place - base) >> shift], amount); });
    __syncthreads();
    u64 total;
    const u64 mine = s.bin[threadIdx.x], upto = before + sum_upto(mine, total, s);
    if (upto - mine < want && want <= upto) {      // (for one thread at most)
        s.found = 1; s.before = upto - mine; s.at = mine; s.place = base + (threadIdx.x << shift);
    }
    __syncthreads();
    return s.found ? Border{true, s.place, s.before, s.at} : Border{false, 0, 0, 0};
}

// Few tokens compared with each other, all with all: a team of 2 to 16 neighbouring lanes for each, as many as there are lanes for
struct Team {
    int lanes, token, lane;
    __device__ __forceinline__ explicit Team(int n) : lanes(n <= DECIDERS / 16 ? 16 : n <= DECIDERS / 8 ? 8 : n <= DECIDERS / 4 ? 4 : 2), token((int)threadIdx.x / lanes), lane((int)threadIdx.x % lanes) {}
    // f(j) for the lane's share of the tokens to compare with
    template <class F> __device__ __forceinline__ void each(int n, F f) const
    {
        if (token < n)
#pragma unroll 4
            for (int j = lane; j < n; j += lanes) f(j);
    }
    __device__ __forceinline__ u64 sum(u64 v) const
    {
        v += lanes_from<0xb1>(v);                      // lane ^ 1
        if (lanes >= 4) v += lanes_from<0x4e>(v);      // lane ^ 2
        if (lanes >= 8) v += lanes_from<0x141>(v);     // the other four of eight
        if (lanes >= 16) v += lanes_from<0x140>(v);    // the other eight of sixteen
        return v;
    }
    __device__ __forceinline__ int sum(int v) const { return (int)sum((u64)v); }
};

// The first place up to which the amounts come to `want` (> 0) or more, what lies before it and what at it. each(in, put) calls put(place, amount) for everything whose place in(place) names; places are below
// 2^bits. Nine bits of the place at a time, by a histogram of amounts, until the step that holds the place has so few of everything that they can be compared all with all. All threads
// get the answer. b: of a step before, which bits are left of.
template <class Each, class S> __device__ __forceinline__ Border find_border(Each each, int bits, u64 want, S &s, Border b = Border{true, 0, 0, 0}, bool stepped = false)
{
#pragma unroll 1
    for (;;) {
        if (!stepped) {
            const int shift = max(0, bits - BIN_BITS);
            b = border_step(each, b.place, bits, shift, b.before, want, s);
            bits = shift;
        } else __syncthreads();      // (others may still read what the caller counted in s.entries)
        if (!b.found || bits == 0) return b;
        stepped = false;
        const uint32_t most = bits >= 32 ? ANY : (1u << bits) - 1;
        if (threadIdx.x == 0) s.entries = 0;
        __syncthreads();
        each([&](uint32_t place) { return place - b.place <= most; }, [&](uint32_t place, u64 amount) {
            const int i = atomicAdd(&s.entries, 1);
            if (i < FEW_PLACES) { s.few[i] = place; s.few_mass[i] = amount; }
        });
        __syncthreads();
        const int n = s.entries;
        if (n > FEW_PLACES) continue;
        const Team team(n);
        const int i = team.token;
        const uint32_t place = i < n ? (uint32_t)s.few[i] : 0;
        u64 before = 0, at = 0;
        team.each(n, [&](int j) {
            const uint32_t other = (uint32_t)s.few[j];
            const u64 amount = s.few_mass[j];
            before += other < place ? amount : 0;
            at += other == place ? amount : 0;
        });
        before = b.before + team.sum(before);
        at = team.sum(at);
        if (i < n && before < want && want <= before + at) { s.place = place; s.before = before; s.at = at; }      // (the same from all that are equal)
        __syncthreads();
        return Border{true, s.place, s.before, s.at};
    }
}

// Where a row's tokens come from. tally(in, amount, put) calls put(key, id, amount(key)) for the tokens that in(key, id) names.
// What a workgroup holds, all tokens of keys `from` and above: four at a time, so that their amounts are computed side by side
template <class S> struct Pool {
    S &s;
    uint32_t from, n;
    bool less = false;      // those behind the others
    __device__ __forceinline__ bool all() const { return from <= LOWEST; }
    template <class In, class Amount, class Put> __device__ __forceinline__ void tally(In in, Amount amount, Put put) const
    {
        constexpr int N = 4;
        const uint32_t *const keys = s.key + (less ? S::held : 0), *const ids = s.id + (less ? S::ids : 0);
#pragma unroll 1
        for (uint32_t first = threadIdx.x; first < n; first += N * DECIDERS) {
            uint32_t key[N], id[N];
            u64 v[N];
            bool ok[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t i = first + e * DECIDERS, at = i < n ? i : first;
                key[e] = i < n ? keys[at] : 0;
                id[e] = S::by_place && !less ? at : ids[at];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) ok[e] = (key[e] != 0) & in(key[e], id[e]);
            if (__any(ok[0] | ok[1] | ok[2] | ok[3])) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = amount(key[e]);
#pragma unroll
                for (int e = 0; e < N; ++e) if (ok[e]) put(key[e], id[e], v[e]);
            }
        }
    }
    // Only the tokens that in(key, id) names from here on, where they are few enough
    template <class In> __device__ __forceinline__ void lessen(In in)
    {
        if (less) return;
        __syncthreads();
        if (threadIdx.x == 0) s.entries = 0;
        __syncthreads();
        tally(in, [](uint32_t) { return 0; }, [&](uint32_t key, uint32_t id, u64) {
            const int i = atomicAdd(&s.entries, 1);
            if (i < LESS) { s.key[S::held + i] = key; s.id[S::ids + i] = id; }
        });
        __syncthreads();
        if (s.entries <= LESS) { less = true; n = s.entries; }
    }
};

// The row itself, 16 bytes at a time; it may begin at any element
template <class T> struct Streamed {
    const T *row;
    int vocab;
    static constexpr uint32_t from = LOWEST;
    __device__ __forceinline__ bool all() const { return true; }
    template <class In> __device__ __forceinline__ void lessen(In) {}
    template <class In, class Amount, class Put> __device__ __forceinline__ void tally(In in, Amount amount, Put put) const
    {
        constexpr int N = 16 / sizeof(T);
#pragma unroll 1
        for (int i = threadIdx.x * N; i < vocab; i += DECIDERS * N) {
            T v[N];
            if (i + N <= vocab) __builtin_memcpy(v, row + i, 16);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = row[min(i + e, vocab - 1)];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t key = i + e < vocab ? key_of(wide(v[e])) : 0;
                if (key && in(key, (uint32_t)(i + e))) put(key, (uint32_t)(i + e), (u64)amount(key));
            }
        }
    }
};

// What is kept of a row: all keys above `key`, and of those equal to it ids up to `last`
struct Kept {
    uint32_t key, last;
    u64 mass;             // 0: not known
    __device__ __forceinline__ bool has(uint32_t k, uint32_t id) const { return (k > key) | ((k == key) & (id <= last)); }
};

__device__ __forceinline__ int bits_of(uint32_t v) { return v ? 32 - __clz(v) : 1; }

// a share of `sum`, one unit at least
__device__ __forceinline__ u64 share_of(float p, u64 sum) { return max(min((u64)ceil(fmax((double)p, 0.0) * (double)sum), sum), 1ull); }
__device__ __forceinline__ u64 share_of(float p, double weight, double unit) { return max((u64)ceil(fmax((double)p, 0.0) * weight * unit), 1ull); }

__device__ __forceinline__ void put_draw(const PickArgs &a, int r, const Row &row, uint32_t id, float z, double total)
{
    a.token[r] = (int)id;
    a.logprob[r] = (float)((z == row.top ? 0.0 : ((double)z - row.top) * row.per * 0.021660849392497955) - log(total));      // (ln 2 / 32)
}
__device__ __forceinline__ void put_nothing(const PickArgs &a, int r, bool top)
{
    if (top) for (int i = threadIdx.x; i < a.entries; i += DECIDERS) { a.ids[(long long)r * a.entries + i] = -1; a.values[(long long)r * a.entries + i] = -INFINITY; }
    else if (threadIdx.x == 0) { a.token[r] = -1; a.logprob[r] = 0.f; }
}

// A first step towards the border of top-k or top-p, where one was taken: key places from b.place on, less than 2^shift of them; top-p's share, where it was computed (0: not); whether it
// was found that the filters end beyond what the source knows
struct First { Border b; int shift; u64 want; bool beyond; };

// What the filters keep, listed in order (TOP) or drawn from; false: more than the source knows of. `weight`: of the whole row, for a source that does not hold it all.
// Searches follow each other: where top-k ends, where top-p does, which of equal tokens are kept, which token is drawn. One piece of code is all of them.
template <bool TOP, class Source, class S> __device__ __forceinline__ bool search(Source &src, const PickArgs &a, int r, const Row &row, double weight, const First &first, S &s)
{
    enum { BY_COUNT, BY_MASS, KEPT, BY_TIE, BY_DRAW };
    Kept kept{LOWEST, ANY, 0};
    bool cut = false, stepped = first.b.found;
    u64 ties = 0, equal = 0, want = 0, sum = 0;      // ties 0: all of them, of `equal` ones
    int mode = row.k > 0 ? BY_COUNT : row.p < 1.f ? BY_MASS : KEPT;
    const bool ended = row.m > 0.f && least_key(row) >= src.from;      // by min-p, if by nothing else before
#pragma unroll 1
    for (;;) {
        if (mode == KEPT) {
            if (row.m > 0.f) {
                const uint32_t least = least_key(row);
                if (!cut && least < src.from) return false;
                if (least > kept.key) { kept.key = least; ties = 0; kept.mass = 0; }
                if (row.m > 1.f) { ties = 1; equal = ANY; kept.mass = 0; }
                cut = true;
            }
            if (!cut && !src.all()) return false;
            mode = ties ? BY_TIE : BY_DRAW;
        }
        if (TOP && mode == BY_DRAW) break;
        const uint32_t least = max(kept.key, src.from);
        const bool by_key = mode == BY_COUNT || mode == BY_MASS, by_mass = mode == BY_MASS || mode == BY_DRAW;
        if (mode == BY_COUNT) want = row.k;
        if (mode == BY_TIE) want = ties;
        if (by_mass) {
            if (mode == BY_MASS && !cut && first.want) want = first.want;
            else if (mode == BY_MASS && !cut && !src.all()) want = share_of(row.p, weight, row.unit);
            else {
                sum = kept.mass;
                if (!sum) {
                    const bool some = mode == BY_MASS && ties;      // of the equal ones: which is not known yet
                    src.tally([&](uint32_t key, uint32_t id) { return kept.has(key, id) & !(some & (key == kept.key)); }, [&](uint32_t key) { return row.mass(key); },
                              [&](uint32_t, uint32_t, u64 m) { sum += m; });
                    sum = sum_of_all(sum, s) + (mode == BY_MASS && ties ? ties * row.mass(kept.key) : 0);
                }
                want = mode == BY_MASS ? share_of(row.p, sum) : min((u64)(evenly(a.u[r]) * (double)sum), sum - 1) + 1;
            }
        }
        const bool few = mode == BY_TIE && equal <= FEW_PLACES;      // no step is needed to get to them
        const int bits = stepped ? first.shift : bits_of(by_key ? row.top_key - least : (uint32_t)a.vocab - 1);
        // what is looked through: keys above `over` and ids of it up to `last`, no keys above `most`
        const uint32_t over = by_key ? least : kept.key, last = mode == BY_DRAW ? kept.last : ANY, most = mode == BY_TIE ? kept.key : ANY, key_bits = by_key ? ANY : 0;
        const auto place = [&](uint32_t key, uint32_t id) { return (key_bits & (row.top_key - key)) | (~key_bits & id); };
        const Border b = find_border([&](auto in, auto put) {
            src.tally([&](uint32_t key, uint32_t id) { return ((key > over) | ((key == over) & (id <= last))) & (key <= most) & in(place(key, id)); },
                      [&](uint32_t key) { return by_mass ? row.mass(key) : 1; }, [&](uint32_t key, uint32_t id, u64 m) { put(place(key, id), m); });
        }, bits, want, s, stepped ? first.b : Border{true, 0, 0, 0}, stepped | few);
        stepped = false;
        if (mode == BY_COUNT) {
            if (!b.found && !src.all() && !(ended && !(row.p < 1.f))) return false;
            if (b.found) {
                kept.key = row.top_key - b.place; equal = b.at; ties = want - b.before < b.at ? want - b.before : 0; cut = true;
                if (!TOP) src.lessen([&](uint32_t key, uint32_t) { return key >= kept.key; });
            }
            mode = row.p < 1.f ? BY_MASS : KEPT;
        } else if (mode == BY_MASS) {
            if (!b.found) {
                if (!ended) return false;
                mode = KEPT;
                continue;
            }
            const uint32_t key = row.top_key - b.place;
            const u64 one = row.mass(key), need = (want - b.before + one - 1) / one;
            equal = b.at / one;
            if (key != kept.key || !ties || need < ties) ties = need < equal ? need : 0;
            kept.key = key;
            kept.mass = ties ? b.before + ties * one : b.before + b.at;
            cut = true;
            mode = KEPT;
        } else if (mode == BY_TIE) {
            kept.last = b.place;
            mode = BY_DRAW;
        } else {
            // (its logit: what the draw was from)
            src.tally([&](uint32_t, uint32_t id) { return id == b.place; }, [](uint32_t) { return 0; },
                      [&](uint32_t key, uint32_t id, u64) { put_draw(a, r, row, id, logit_of(key), (double)sum / row.unit); });
            return true;
        }
    }
    if constexpr (TOP) {
        __syncthreads();
        for (int i = threadIdx.x; i < PICK_MAX_ENTRIES; i += DECIDERS) s.entry[i] = ~0ull;
        if (threadIdx.x == 0) s.entries = 0;
        __syncthreads();
        src.tally([&](uint32_t key, uint32_t id) { return kept.has(key, id); }, [](uint32_t) { return 0; },
                  [&](uint32_t key, uint32_t id, u64) { s.entry[atomicAdd(&s.entries, 1)] = (u64)~key << 32 | id; });
        __syncthreads();
        const int n = s.entries;
#pragma unroll 1
        for (int size = 2; size < 2 * n; size *= 2)
#pragma unroll 1
            for (int step = size / 2; step; step /= 2) {
                __syncthreads();
                if (threadIdx.x >= PICK_MAX_ENTRIES / 2) continue;
                const int x = (threadIdx.x / step) * 2 * step + threadIdx.x % step, y = x + step;
                const u64 v = s.entry[x], w = s.entry[y];
                if ((v > w) == !(x & size)) { s.entry[x] = w; s.entry[y] = v; }
            }
        __syncthreads();
        for (int i = threadIdx.x; i < a.entries; i += DECIDERS) {
            const u64 e = s.entry[i];
            a.ids[(long long)r * a.entries + i] = e == ~0ull ? -1 : (int)(uint32_t)e;
            a.values[(long long)r * a.entries + i] = e == ~0ull ? -INFINITY : logit_of(~(uint32_t)(e >> 32));
        }
    }
    return true;
}

// One workgroup looks through a row in memory, as often as it takes.
template <class T, bool TOP, class S> __device__ __forceinline__ void whole_row(const PickArgs &a, int r, const Row &row, S &s)
{
    Streamed<T> all{(const T *)a.logits + (long long)r * a.stride, a.vocab};
    search<TOP>(all, a, r, row, 0.0, First{}, s);
}

// Tokens that a workgroup can compare all with all: those from where top-k or top-p end on, or min-p. A team of lanes a token adds up what comes before it in the order, and then, of what is kept,
// what comes before it by id. false: more than FEW, or more than the source knows of.
template <bool TOP, class S> __device__ __forceinline__ bool among_few(Pool<S> &src, const PickArgs &a, int r, const Row &row, double weight, uint32_t low, First &first, S &s)
{
    if (row.k > FEW) return false;
    uint32_t floor = max(src.from, low);
    bool closed = floor <= LOWEST;
    const uint32_t least = row.m > 0.f ? least_key(row) : 0;
    if (row.m > 0.f && least >= floor && !(row.p < 1.f && row.k > 0)) { floor = least; closed = true; }      // (top-p's is a share of all that top-k keeps)
    u64 want = 0;
    if (row.p < 1.f && row.k == 0) {
        if (!src.all()) want = share_of(row.p, weight, row.unit);
        else {
            u64 sum = 0;
            src.tally([](uint32_t, uint32_t) { return true; }, [&](uint32_t key) { return row.mass(key); }, [&](uint32_t, uint32_t, u64 m) { sum += m; });
            want = share_of(row.p, sum_of_all(sum, s));
        }
    }
    // steps of equal width down to the floor (keys are denser the nearer logits are to zero)
    const bool by_step = (row.k > 0 || row.p < 1.f) && row.top < INFINITY;
    const float high = logit_of(row.top_key), scale = (BINS - 1) / fmaxf(high - logit_of(floor), FLT_MIN);
    const auto step = [&](uint32_t key) { return (uint32_t)fminf((high - logit_of(key)) * scale, (float)BINS); };
    uint32_t last = ANY;
    if (by_step) {
        const bool by_count = row.k > 0;
        const Border b = border_step([&](auto in, auto put) {
            src.tally([&](uint32_t key, uint32_t) { return (key >= floor) & in(step(key)); }, [&](uint32_t key) { return by_count ? 1 : row.mass(key); },
                      [&](uint32_t key, uint32_t, u64 m) { put(step(key), m); });
        }, 0, BIN_BITS, 0, 0, by_count ? (u64)row.k : want, s);
        first.want = want;
        if (b.found) { last = b.place; closed = true; first.b = b; }
    }
    first.beyond = by_step && !closed && floor == src.from && scale > 0;
    if (!closed) return false;
    __syncthreads();
    if (threadIdx.x == 0) { s.entries = 0; s.most = 0; s.least = ANY; }
    __syncthreads();
    src.tally([&](uint32_t key, uint32_t) { return (key >= floor) & (!by_step | (step(key) <= last)); }, [](uint32_t) { return 0; }, [&](uint32_t key, uint32_t id, u64) {
        const int i = atomicAdd(&s.entries, 1);
        if (i < FEW) s.few[i] = (u64)~key << 32 | id;
        if (i < LESS) { s.key[S::held + i] = key; s.id[S::ids + i] = id; }
        if (by_step && step(key) == last) { atomicMax(&s.most, key); atomicMin(&s.least, key); }
    });
    __syncthreads();
    const int n = s.entries;
    if (n > FEW) {
        // the border is in the step's keys
        if (first.b.found) { first.shift = bits_of(s.most - s.least); first.b.place = row.top_key - s.most; }
        if (n <= LESS) { src.less = true; src.n = n; }
        return false;
    }
    const Team team(n);
    const int i = team.token;
    const bool speaks = i < n && team.lane == 0;
    const u64 mine = i < n ? s.few[i] : ~0ull;
    const uint32_t key = ~(uint32_t)(mine >> 32), id = (uint32_t)mine;
    if constexpr (TOP) {
        int rank = 0;
        team.each(n, [&](int j) { rank += s.few[j] < mine; });
        rank = team.sum(rank);
        if (speaks && rank < a.entries) {
            a.ids[(long long)r * a.entries + rank] = (int)id;
            a.values[(long long)r * a.entries + rank] = logit_of(key);
        }
        for (int e = n + threadIdx.x; e < a.entries; e += DECIDERS) { a.ids[(long long)r * a.entries + e] = -1; a.values[(long long)r * a.entries + e] = -INFINITY; }
        return true;
    }
    const u64 own = i < n ? row.mass(key) : 0;
    if (speaks) s.few_mass[i] = own;
    __syncthreads();
    int rank = 0;
    u64 before = 0;
    team.each(n, [&](int j) {
        const bool less = s.few[j] < mine;
        rank += less;
        before += less ? s.few_mass[j] : 0;
    });
    rank = team.sum(rank);
    before = team.sum(before);
    bool kept = i < n && (row.k == 0 || rank < row.k);
    if (row.p < 1.f) {
        if (row.k > 0) want = share_of(row.p, sum_of_all(kept && speaks ? own : (u64)0, s));
        kept = kept && before < want;
    }
    if (row.m > 0.f) kept = kept && (rank == 0 || (key >= least && !(row.m > 1.f)));
    const u64 sum = sum_of_all(kept && speaks ? own : (u64)0, s);
    if (speaks) s.few_mass[i] = kept ? own : 0;
    __syncthreads();
    const u64 below = min((u64)(evenly(a.u[r]) * (double)sum), sum - 1);
    before = 0;
    team.each(n, [&](int j) { before += (uint32_t)s.few[j] < id ? s.few_mass[j] : 0; });
    before = team.sum(before);
    if (kept && speaks && before <= below && below < before + own) put_draw(a, r, row, id, logit_of(key), (double)sum / row.unit);
    return true;
}

struct Found { int at; double before; };

// The first of the values (PER a thread, in the threads' order) up to which they add up to more than `want`; where rounding leaves none the last that is no zero. `before`: sum of the
// threads' before this one. Sums in 64 bits in a fixed order.
template <class S> __device__ __forceinline__ Found first_over(const double (&v)[PER], double before, double want, S &s)
{
    double run = before, found_at = before;
    uint32_t first = ANY, last = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const double from = run;
        run += v[e];
        if (!(v[e] > 0)) continue;
        const uint32_t i = threadIdx.x * PER + e;
        last = i + 1;
        if (first != ANY) continue;
        found_at = from;                                  // (of the first that is over, or of the last)
        if (run > want) first = i;
    }
    if (threadIdx.x == 0) { s.first = ANY; s.last = 0; }
    const uint32_t wave_first = ~wave_max(~first), wave_last = wave_max(last);
    __syncthreads();
    if (threadIdx.x % 64 == 0) { atomicMin(&s.first, wave_first); atomicMax(&s.last, wave_last); }
    __syncthreads();
    const uint32_t at = s.first != ANY ? s.first : s.last - 1;
    if (at / PER == threadIdx.x) s.run = found_at;
    __syncthreads();
    return Found{(int)at, s.run};
}

// A draw from a row that nothing is cut from, which more than one workgroup has read in parts that are one piece each: the part by the parts' weights, then the token in it
template <class T, class S> __device__ __forceinline__ void draw_freely(const PickArgs &a, int r, const T *logits, const Row &row, const double (&parts)[PER], S &s)
{
    double total, rest, sum = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += parts[e];
    double before = sum_upto(sum, total, s) - sum;
    // (the first and the last tokens may weigh nothing beside the others, where weights in units are 0)
    constexpr double END = 0x1p-45;
    const double want = fmin(fmax(evenly(a.u[r]), END), 1 - END) * total;
    const Found part = first_over(parts, before, want, s);
    float z[PER];
    double v[PER];
    const int first = part.at * PICK_PART + threadIdx.x * PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) z[e] = first + e < a.vocab ? wide(logits[first + e]) : -INFINITY;
    sum = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += v[e] = z[e] > -INFINITY ? row.weight(z[e]) : 0;
    before = sum_upto(sum, rest, s) - sum;
    const Found token = first_over(v, before, want - part.before, s);
#pragma unroll
    for (int e = 0; e < PER; ++e) if (token.at == (int)threadIdx.x * PER + e) put_draw(a, r, row, first + e, z[e], total);
}

// ------------------------------------------------------------------ the kernels

// A part of a row: blocks of a load each, `step` apart, in LDS as 32 bits, EACH a lane (-inf, NaN: no token). A load past the row's end is moved back, and what it has twice is dropped.
template <class T> struct Part {
    static constexpr int N = 16 / sizeof(T), BLOCKS = EACH / N, BLOCK = 64 * N;
    float (*z)[64][4];           // [EACH / 4][lane][4]
    uint32_t first, step;        // of the lane
    int vocab;
    __device__ __forceinline__ uint32_t at(int block) const
    {
        return min(first + block * step, (uint32_t)(vocab - N));
    }
    __device__ __forceinline__ uint32_t id(int e) const { return at(e / N) + e % N; }
    __device__ __forceinline__ float &logit(int e) const { return z[e / 4][threadIdx.x % 64][e % 4]; }
    // returns the largest of the lane's
    template <bool PAST = false> __device__ __forceinline__ float load(const T *logits)
    {
        T raw[BLOCKS][N];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const char *const p = (const char *)logits + at(i) * (uint32_t)sizeof(T);
            u32x4_any v;
            if constexpr (PAST) v = __builtin_nontemporal_load((const u32x4_any *)p);
            else __builtin_memcpy(&v, p, 16);
            __builtin_memcpy(raw[i], &v, 16);
        }
        // (the last lane's last load ends within the row: so do all)
        const bool whole = __builtin_amdgcn_readlane((int)(first + (BLOCKS - 1) * step), 63) + N <= vocab;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = wide(raw[i][e]);
            if (!whole) {
#pragma unroll
                for (int e = 0; e < N; ++e) if (at(i) + e < first + i * step) v[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, v[e]);
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4 *>(&z[(i * N + e) / 4][threadIdx.x % 64][0]) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        return most;
    }
    // f(logit, place) for the lane's
    template <class F> __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (int i = 0; i < EACH / 4; ++i) {
            const float4 v = *reinterpret_cast<const float4 *>(&z[i][threadIdx.x % 64][0]);
            f(v.x, 4 * i); f(v.y, 4 * i + 1); f(v.z, 4 * i + 2); f(v.w, 4 * i + 3);
        }
    }
    // Leaves the tokens of a mask of the lane's in a list, lanes one after the other, and nothing in the rest of it
    __device__ __forceinline__ void list(uint32_t mask, int upto, int sum, int listed, uint2 *to) const
    {
        const int lane = threadIdx.x % 64;
        int i = upto - __popc(mask);
#pragma unroll 1
        for (; mask; mask &= mask - 1) {
            const int e = __ffs(mask) - 1;
            to[i++] = make_uint2(key_of(logit(e)), id(e));
        }
        for (int l = lane; l < listed; l += 64) if (l >= sum) to[l] = make_uint2(0, 0);
    }
};

// Bound by its instructions where sums are wanted: 35 a token and lane with the list, 22 without, half of them 64-bit ones for the weight (256 rows of 152064 bf16 logits 44 us, 64 free fp32 rows 12).
// Without sums 13, bound by memory (1024 rows of 151936 fp32 logits 104 us, 6 TB/s). 16 tokens a lane: with 32 fewer wavefronts wait for the loads at once.
template <class T, bool TOP, bool PAST> __global__ __launch_bounds__(THREADS, 8) void parts_kernel(PickArgs a)
{
    __shared__ float s_z[WAVES][EACH / 4][64][4];
    __shared__ uint2 s_powers[32];
    const int r = blockIdx.x / a.groups, lane = threadIdx.x % 64, wave = threadIdx.x / 64, parts = a.groups * WAVES, part = (blockIdx.x % a.groups) * WAVES + wave;
    Row row = row_of<TOP>(a, r, s_powers);
    // Of a row that is cut from, blocks of all parts take turns, so that large logits that lie together are spread over the parts; of one that is drawn from freely a part is one
    // piece, so that its sum is a step of the sums by id.
    using P = Part<T>;
    if (a.queue && blockIdx.x == 0 && threadIdx.x == 0) a.queue[0] = 0;
    P p{s_z[wave], (uint32_t)part * (row.cut ? P::BLOCK : PICK_PART) + lane * P::N, (uint32_t)(row.cut ? parts * P::BLOCK : P::BLOCK), a.vocab};
    const uint32_t lane_top = key_of(p.template load<PAST>((const T *)a.logits + (long long)r * a.stride));
    if (row.summed) load_powers(s_powers);
    PickHead head{};
    head.top = wave_max(lane_top);
    if (row.summed && head.top) {
        row.relative_to(head.top);
        double sum = 0;
        if (row.top < INFINITY) p.each([&](float z, int) { sum += row.finite_weight(z); });
        else p.each([&](float z, int) { sum += row.infinite_weight(z); });
        head.sum = wave_sum(sum);
    }
    if (row.cut) {
        // a threshold that few enough tokens reach: one that listed_lanes lanes or somewhat fewer reach with their largest, then fewer until the tokens fit
        uint32_t from = LOWEST, mask = 0;
        const uint32_t least_top = ~wave_max(~lane_top);
        int lanes = a.listed_lanes, upto = 0, sum = 0;
        bool look = __popcll(__ballot(lane_top != 0)) <= a.listed;      // there may be so few tokens
#pragma unroll 1
        for (;; look = true) {
            if (look) {
                const float least = logit_of(from);
                mask = 0;
                p.each([&](float z, int e) { mask |= (uint32_t)(z >= least) << e; });
                upto = wave_upto(__popc(mask), Plus{});
                sum = last_lane(upto);
                if (sum <= a.listed) break;
                mask = sum = 0;
            }
            uint32_t below = max(from, least_top), above = head.top + 1;              // no lane reaches it
            from = above;
#pragma unroll 1
            while (above - below > 1) {
                const uint32_t mid = below + (above - below) / 2;
                const int c = __popcll(__ballot(lane_top >= mid));
                if (c > lanes) below = mid;
                else {
                    above = from = mid;
                    if (c > lanes * 3 / 4) break;
                }
            }
            lanes = lanes * 3 / 4;
            if (from > head.top) break;                               // nothing is listed
        }
        head.from = from;
        p.list(mask, upto, sum, a.listed, a.list + ((long long)r * parts + part) * a.listed);
    }
    if (lane == 0) a.head[(long long)r * parts + part] = head;
}

// the parts' lists, `listed` a part, into a workgroup's pool: those of keys `least` and above
template <int HELD> struct Lists {
    uint2 v[HELD / DECIDERS];
    __device__ __forceinline__ void load(const PickArgs &a, int r, int parts)
    {
        const uint2 *const list = a.list + (long long)r * parts * a.listed;
        const uint32_t all = parts * a.listed;
#pragma unroll
        for (int e = 0; e < HELD / DECIDERS; ++e) {
            const uint32_t i = e * DECIDERS + threadIdx.x;
            v[e] = i < all ? list[i] : make_uint2(0, 0);
        }
    }
    template <class S> __device__ __forceinline__ uint32_t hold(uint32_t least, S &s, uint32_t *lowest = nullptr) const      // (s.n is zero, behind a barrier)
    {
        int n = 0;
#pragma unroll
        for (int e = 0; e < HELD / DECIDERS; ++e) n += v[e].x && v[e].x >= least;
        const int upto = wave_upto(n, Plus{});
        uint32_t at = 0;
        if (threadIdx.x % 64 == 63) at = atomicAdd(&s.n, (uint32_t)upto);
        at = last_lane(at) + upto - n;
        if (lowest) {
            uint32_t low = ANY;
#pragma unroll
            for (int e = 0; e < HELD / DECIDERS; ++e) low = v[e].x ? min(low, v[e].x) : low;
            low = ~wave_max(~low);
            if (threadIdx.x % 64 == 0) atomicMin(lowest, low);
        }
#pragma unroll
        for (int e = 0; e < HELD / DECIDERS; ++e) if (v[e].x && v[e].x >= least) { s.key[at] = v[e].x; s.id[at++] = v[e].y; }
        __syncthreads();
        return s.n;
    }
};

// Where large logits lie together, or by chance, a part has so many of them that its threshold is far above the others': what is known of the row then ends there. The parts of the largest
// thresholds, one a wavefront, are read again, down to the next part's (37 us for 64 rows of 151936 whose largest 300 are neighbours, top-k 50; with whole_row instead 620). false: nothing to gain, or no room.
template <class T, int HELD, class S> __device__ __forceinline__ bool mend(const PickArgs &a, int r, const T *logits, int parts, Pool<S> &pool, Lists<HELD> &lists, S &s)
{
    const PickHead *const head = a.head + (long long)r * parts;
    const uint32_t from = ANY - find_border([&](auto in, auto put) {
        for (int i = threadIdx.x; i < parts; i += DECIDERS) if (in(ANY - head[i].from)) put(ANY - head[i].from, 1);
    }, 32, WAVES + 1, s).place;      // (a row has more parts)
    if (from >= pool.from) return false;
    __syncthreads();
    if (threadIdx.x == 0) { s.n = 0; s.entries = 0; }
    __syncthreads();
    for (int i = threadIdx.x; i < parts; i += DECIDERS) if (head[i].from > from) s.few[atomicAdd(&s.entries, 1)] = i;
    lists.load(a, r, parts);
    lists.hold(from, s);
    if ((int)threadIdx.x / 64 < s.entries) {
        using P = Part<T>;
        const uint32_t part = (uint32_t)s.few[threadIdx.x / 64], listed = head[part].from, first = part * P::BLOCK + threadIdx.x % 64 * P::N;
#pragma unroll 1
        for (uint32_t begin = first; begin < (uint32_t)a.vocab; begin += parts * P::BLOCK) {
            const uint32_t at = min(begin, (uint32_t)(a.vocab - P::N));
            T v[P::N];
            __builtin_memcpy(v, logits + at, 16);
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                const uint32_t key = key_of(wide(v[e]));
                if (at + e < begin || key < from || key >= listed) continue;
                const uint32_t i = atomicAdd(&s.n, 1);
                if (i < HELD) { s.key[i] = key; s.id[i] = at + e; }
            }
        }
    }
    __syncthreads();
    if (s.n > HELD) return false;
    pool.from = from;
    pool.n = s.n;
    pool.less = false;
    return true;
}

// One workgroup a row. Bound by the latency of a few loads and of some twenty barriers: one row of 151936 8.3 us, the largest 16 of 64 rows 6, 256 rows with top-p, which ends among thousands, 32.
template <class T, bool TOP, bool WHOLE, int HELD> __global__ __launch_bounds__(DECIDERS) void decide_kernel(PickArgs a)
{
    using S = Shared<HELD, WHOLE>;
    __shared__ S s;
    const int r = blockIdx.x, vocab = a.vocab, parts = a.groups * WAVES;
    const T *const logits = (const T *)a.logits + (long long)r * a.stride;
    Row row = row_of<TOP>(a, r, s.powers);
    if (threadIdx.x == 0) { s.top = 0; s.from = LOWEST; s.n = 0; s.least = ANY; }
    load_powers(s.powers);
    Pool<S> pool{s, LOWEST, (uint32_t)vocab};
    double weight = 0;
    uint32_t low = LOWEST;
    if constexpr (WHOLE) {
        constexpr int N = 16 / sizeof(T);
        __syncthreads();
        uint32_t top = 0;
        if (vocab >= N) {
#pragma unroll
            for (int i = 0; i < (HELD + DECIDERS * N - 1) / (DECIDERS * N); ++i) {
                const int at = min((i * DECIDERS + (int)threadIdx.x) * N, vocab - N);      // (some twice, the same)
                T v[N];
                __builtin_memcpy(v, logits + at, 16);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint32_t key = key_of(wide(v[e]));
                    s.key[at + e] = key;
                    top = max(top, key);
                }
            }
        } else if ((int)threadIdx.x < vocab) {
            top = key_of(wide(logits[threadIdx.x]));
            s.key[threadIdx.x] = top;
        }
        // as many tokens as there are threads with tokens are not below the least of the threads' largest: few filters end below that
        const uint32_t least = ~wave_max(top ? ~top : 0);
        top = wave_max(top);
        if (threadIdx.x % 64 == 0) { atomicMax(&s.top, top); atomicMin(&s.least, least); }
        __syncthreads();
        if (!s.top) { put_nothing(a, r, TOP); return; }
        row.relative_to(s.top);
        if (vocab > FEW) low = s.least;
    } else {
        PickHead head[PER]{};
#pragma unroll
        for (int e = 0; e < PER; ++e) if ((int)threadIdx.x * PER + e < parts) head[e] = a.head[(long long)r * parts + threadIdx.x * PER + e];
        Lists<HELD> lists;
        if (row.cut) lists.load(a, r, parts);
        __syncthreads();
        uint32_t top = 0, from = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) { top = max(top, head[e].top); from = max(from, head[e].from); }
        top = wave_max(top); from = wave_max(from);
        if (threadIdx.x % 64 == 0) { atomicMax(&s.top, top); atomicMax(&s.from, from); }
        __syncthreads();
        if (!s.top) { put_nothing(a, r, TOP); return; }
        row.relative_to(s.top);
        pool.from = s.from;
        if constexpr (!TOP) {
            if (row.summed) {
                double v[PER], sum = 0;
#pragma unroll
                for (int e = 0; e < PER; ++e) sum += v[e] = head[e].top ? head[e].sum * row.weight(logit_of(head[e].top)) : 0;
                if (!row.cut) {
                    draw_freely(a, r, logits, row, v, s);
                    return;
                }
                weight = sum_of_all(sum, s);
            }
        }
        pool.n = lists.hold(pool.from, s);
    }
    First first{};
    if (among_few<TOP>(pool, a, r, row, weight, low, first, s)) return;
#pragma unroll 1
    for (bool last = WHOLE || row.k == 0;; last = true) {
        if (!first.beyond && search<TOP>(pool, a, r, row, weight, first, s)) return;
        if constexpr (WHOLE) break;
        else {
            Lists<HELD> lists;
            if (last || !mend(a, r, logits, parts, pool, lists, s)) break;
            first = First{};
        }
    }
    if constexpr (!TOP) {
        if (!WHOLE && a.queue && row.k == 0 && row.top < INFINITY && pool.from <= row.top_key) {
            if (threadIdx.x == 0) {
                PickSearch q{};
                q.stage = row.p < 1.f ? PICK_STEP : PICK_LEAST;
                q.top_key = row.top_key;
                q.least = row.m > 0.f ? least_key(row) : 0;
                q.from = logit_of(pool.from);
                // what top-p leaves out, and the border with it, weighs (1 - p) of all or more, and none of it more than the border: that weighs (1 - p) / vocab of all or more
                const double share = fmax((double)row.p, 0.0), least = row.top + (double)row.t * log(0.5 * (1 - share) * weight / vocab);
                q.scale = (float)((PICK_STEPS - 2) / fmax((double)q.from - least, 1e-30));
                q.want = share_of(row.p, weight, row.unit);
                a.search[r] = q;
                a.queue[1 + atomicAdd(a.queue, 1u)] = r;
            }
            return;
        }
    }
    if constexpr (!WHOLE) whole_row<T, TOP>(a, r, row, s);
}

// ------------------------------------------------------------------ rows that are searched

// The step of a logit below `from`; larger logits are in no later step, and what is no token is in none
__device__ __forceinline__ int step_of(float z, const PickSearch &q) { return (int)fminf((q.from - z) * q.scale, (float)PICK_STEPS); }

constexpr int STEP_COPIES = THREADS / PICK_STEPS;      // of the histogram, for neighbouring lanes: even tokens meet in few steps

// Bound by the 64-bit LDS atomics (32 rows of 151936 11 us; a third to half of the LDS cycles are conflicts).
// Masses by steps below `from`, in the last place that of everything from it on; what is below all steps is left out
template <class T> __global__ __launch_bounds__(THREADS, 8) void steps_kernel(PickArgs a)
{
    __shared__ float s_z[WAVES][EACH / 4][64][4];
    __shared__ uint2 s_powers[32];
    __shared__ u64 step[STEP_COPIES][PICK_STEPS + 1];
    static_assert(STEP_COPIES * PICK_STEPS == THREADS);
    load_powers(s_powers);
    const uint32_t items = a.queue[0] * a.groups;
#pragma unroll 1
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int r = a.queue[1 + item / a.groups], group = item % a.groups;
        const PickSearch q = a.search[r];
        if (q.stage != PICK_STEP) continue;
        step[threadIdx.x / PICK_STEPS][threadIdx.x % PICK_STEPS] = 0;
        Row row = row_of<false>(a, r, s_powers);
        row.relative_to(q.top_key);
        using P = Part<T>;
        P p{s_z[threadIdx.x / 64], (uint32_t)(group * WAVES + threadIdx.x / 64) * PICK_PART + threadIdx.x % 64 * P::N, P::BLOCK, a.vocab};
        p.load((const T *)a.logits + (long long)r * a.stride);
        __syncthreads();
        u64 above = 0;
        p.each([&](float z, int) {
            const int at = z >= q.from ? -1 : step_of(z, q);
            if (at >= PICK_STEPS - 1) return;                        // (-inf and NaN too)
            const u64 m = row.in_units(row.finite_weight(z));
            if (at < 0) above += m;
            else atomicAdd(&step[threadIdx.x % STEP_COPIES][at], m);
        });
        above = wave_sum(above);
        if (threadIdx.x % 64 == 0) atomicAdd(&step[0][PICK_STEPS - 1], above);
        __syncthreads();
        if (threadIdx.x < PICK_STEPS) {
            u64 sum = 0;
#pragma unroll
            for (int c = 0; c < STEP_COPIES; ++c) sum += step[c][threadIdx.x];
            a.steps[((long long)r * a.groups + group) * PICK_STEPS + threadIdx.x] = sum;
        }
        __syncthreads();
    }
}

// Bound by its instructions and by the latency before them (32 rows of 151936 14 us).
// The step that top-p ends in; of each part the mass of what is above it and its tokens in it. Where min-p alone decides, the mass of what it keeps.
template <class T> __global__ __launch_bounds__(THREADS, 8) void place_kernel(PickArgs a)
{
    __shared__ float s_z[WAVES][EACH / 4][64][4];
    __shared__ uint2 s_powers[32];
    __shared__ u64 s_sum[STEP_COPIES][PICK_STEPS];
    __shared__ int s_step;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, parts = a.groups * WAVES;
    load_powers(s_powers);
    const uint32_t items = a.queue[0] * a.groups;
#pragma unroll 1
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int r = a.queue[1 + item / a.groups], group = item % a.groups, part = group * WAVES + wave;
        const PickSearch q = a.search[r];
        Row row = row_of<false>(a, r, s_powers);
        row.relative_to(q.top_key);
        using P = Part<T>;
        P p{s_z[wave], (uint32_t)part * PICK_PART + lane * P::N, P::BLOCK, a.vocab};
        p.load((const T *)a.logits + (long long)r * a.stride);
        int step = PICK_STEPS;                    // none
        uint32_t stage = q.stage;
        if (stage == PICK_STEP) {
            const int at = threadIdx.x % PICK_STEPS, quarter = threadIdx.x / PICK_STEPS;
            const u64 *const steps = a.steps + (long long)r * a.groups * PICK_STEPS + at;
            u64 sum = 0;
#pragma unroll 4
            for (int g = quarter; g < a.groups; g += STEP_COPIES) sum += steps[g * PICK_STEPS];
            __syncthreads();
            s_sum[quarter][at] = sum;
            if (threadIdx.x == 0) s_step = PICK_STEPS;
            __syncthreads();
            if (wave == 0) {
                // (what is above all steps, which the last place holds, comes before them)
                u64 v[PICK_STEPS / 64];
#pragma unroll
                for (int e = 0; e < PICK_STEPS / 64; ++e) {
                    v[e] = 0;
#pragma unroll
                    for (int c = 0; c < STEP_COPIES; ++c) v[e] += s_sum[c][lane * (PICK_STEPS / 64) + e];
                }
                u64 run = last_lane(v[PICK_STEPS / 64 - 1]), mine = 0;
                if (lane == 63) v[PICK_STEPS / 64 - 1] = 0;
#pragma unroll
                for (int e = 0; e < PICK_STEPS / 64; ++e) mine += v[e];
                run += wave_upto(mine, Plus{}) - mine;
#pragma unroll
                for (int e = 0; e < PICK_STEPS / 64; ++e) {
                    if (run < q.want && q.want <= run + v[e]) s_step = lane * (PICK_STEPS / 64) + e;
                    run += v[e];
                }
            }
            __syncthreads();
            step = s_step;
            if (step == PICK_STEPS) stage = PICK_WHOLE;
            else if (q.least && step_of(logit_of(q.least), q) < step) stage = PICK_LEAST;
        }
        if (group == 0 && threadIdx.x == 0) a.search[r].found = stage;
        if (stage == PICK_WHOLE) continue;
        PickHead head{};
        const float least = stage == PICK_LEAST ? logit_of(q.least) : q.from;
        u64 mass = 0;
        uint32_t mask = 0;
        p.each([&](float z, int e) {
            const int at = stage == PICK_STEP ? step_of(z, q) : PICK_STEPS;      // (-inf, NaN: PICK_STEPS)
            if (z >= least || at < step) mass += row.in_units(row.finite_weight(z));
            else mask |= (uint32_t)(at == step) << e;
        });
        head.mass = wave_sum(mass);
        if (stage == PICK_STEP) {
            const int upto = wave_upto(__popc(mask), Plus{}), sum = last_lane(upto);
            head.count = sum;
            if (sum <= a.listed) p.list(mask, upto, sum, a.listed, a.list + ((long long)r * parts + part) * a.listed);
        }
        if (lane == 0) a.head[(long long)r * parts + part] = head;
    }
}

// The place in the step, and the draw: the part by the parts' masses, then the token in it. One workgroup a row, bound by latency (32 rows 16 us).
template <class T> __global__ __launch_bounds__(DECIDERS) void finish_kernel(PickArgs a)
{
    constexpr int HELD = PICK_LISTED;
    __shared__ Shared<HELD> s;
    const int vocab = a.vocab, parts = a.groups * WAVES;
    load_powers(s.powers);
    const uint32_t rows = a.queue[0];
#pragma unroll 1
    for (uint32_t item = blockIdx.x; item < rows; item += gridDim.x) {
        const int r = a.queue[1 + item];
        const PickSearch q = a.search[r];
        const T *const logits = (const T *)a.logits + (long long)r * a.stride;
        Row row = row_of<false>(a, r, s.powers);
        row.relative_to(q.top_key);
        __syncthreads();
        if (threadIdx.x == 0) { s.n = 0; s.from = ANY; }
        bool whole = q.found == PICK_WHOLE;
        Lists<HELD> lists;
        if (q.found == PICK_STEP) lists.load(a, r, parts);
        u64 above = 0;
        if (!whole) {
            u64 over = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int w = threadIdx.x * PER + e;
                PickHead head{};
                if (w < parts) head = a.head[(long long)r * parts + w];
                s.mass[w] = head.mass;
                above += head.mass;
                over += head.count > (uint32_t)a.listed;
            }
            whole = sum_of_all(over, s) != 0;
            above = sum_of_all(above, s);
        }
        if (whole) {
            whole_row<T, false>(a, r, row, s);
            continue;
        }
        Kept kept{q.least, ANY, 0};
        if (q.found == PICK_STEP) {
            const Pool<Shared<HELD>> pool{s, LOWEST, lists.hold(LOWEST, s, &s.from)};      // (and the smallest of them)
            const uint32_t high = key_of(q.from);
            const auto mass = [&](uint32_t key) { return row.in_units(row.finite_weight(logit_of(key))); };
            const Border b = find_border([&](auto in, auto put) {
                pool.tally([&](uint32_t key, uint32_t) { return in(high - key); }, mass, [&](uint32_t key, uint32_t, u64 m) { put(high - key, m); });
            }, bits_of(high - s.from), q.want - above, s);
            kept.key = high - b.place;
            const u64 one = row.mass(kept.key), need = (q.want - above - b.before + one - 1) / one;
            const u64 equal = b.at / one;
            u64 ties = need < equal ? need : 0;
            if (q.least > kept.key) { kept.key = q.least; ties = 0; }
            if (ties) kept.last = find_border([&](auto in, auto put) {
                pool.tally([&](uint32_t key, uint32_t id) { return (key == kept.key) & in(id); }, [](uint32_t) { return 1; }, [&](uint32_t, uint32_t id, u64 m) { put(id, m); });
            }, bits_of(vocab - 1), ties, s, Border{true, 0, 0, 0}, equal <= FEW_PLACES).place;
            __syncthreads();
            pool.tally([&](uint32_t key, uint32_t id) { return kept.has(key, id); }, mass, [&](uint32_t, uint32_t id, u64 m) { atomicAdd(&s.mass[id / PICK_PART], m); });
            __syncthreads();
        }
        // the part, then the token in it
        u64 total, sum = 0, part[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) sum += part[e] = s.mass[threadIdx.x * PER + e];
        u64 run = sum_upto(sum, total, s) - sum;
        const u64 below = min((u64)(evenly(a.u[r]) * (double)total), total - 1);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (run <= below && below < run + part[e]) { s.place = threadIdx.x * PER + e; s.before = run; }
            run += part[e];
        }
        __syncthreads();
        const int first = s.place * PICK_PART + threadIdx.x * PER;
        const u64 left = below - s.before;
        float z[PER];
        u64 v[PER], rest;
#pragma unroll
        for (int e = 0; e < PER; ++e) z[e] = first + e < vocab ? wide(logits[first + e]) : -INFINITY;
        sum = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const uint32_t key = key_of(z[e]);
            sum += v[e] = key && kept.has(key, first + e) ? row.in_units(row.finite_weight(z[e])) : 0;
        }
        run = sum_upto(sum, rest, s) - sum;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (run <= left && left < run + v[e]) put_draw(a, r, row, first + e, z[e], (double)total / row.unit);
            run += v[e];
        }
    }
}

template <class T, bool TOP> void launch_parts(hipStream_t s, const PickArgs &a)
{
    const unsigned all = (unsigned)a.rows * a.groups;
    if (a.past) hipLaunchKernelGGL((parts_kernel<T, TOP, true>), dim3(all), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((parts_kernel<T, TOP, false>), dim3(all), dim3(THREADS), 0, s, a);
    if (a.groups * WAVES * a.listed <= 4096) hipLaunchKernelGGL((decide_kernel<T, TOP, false, 4096>), dim3(a.rows), dim3(DECIDERS), 0, s, a);
    else hipLaunchKernelGGL((decide_kernel<T, TOP, false, PICK_LISTED>), dim3(a.rows), dim3(DECIDERS), 0, s, a);
    if constexpr (!TOP) {
        if (!a.queue) return;
        // rows of the queue, which the host does not know: as many workgroups as run at once, which are soon gone where it is empty
        hipLaunchKernelGGL(steps_kernel<T>, dim3(std::min(all, 1024u)), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(place_kernel<T>, dim3(std::min(all, 1024u)), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(finish_kernel<T>, dim3(std::min(a.rows, 256)), dim3(DECIDERS), 0, s, a);
    }
}

template <class T, bool TOP> void launch(hipStream_t s, const PickArgs &a)
{
    const dim3 rows(a.rows), threads(DECIDERS);
    if (!a.head) {
        if (a.vocab <= 4096) hipLaunchKernelGGL((decide_kernel<T, TOP, true, 4096>), rows, threads, 0, s, a);
        else hipLaunchKernelGGL((decide_kernel<T, TOP, true, 8192>), rows, threads, 0, s, a);
        return;
    }
    launch_parts<T, TOP>(s, a);
}

}  // namespace

void launch_sample(hipStream_t s, const PickArgs &a)
{
    if (a.dtype == DT_BF16) launch<bf16_t, false>(s, a);
    else launch<float, false>(s, a);
}

void launch_top(hipStream_t s, const PickArgs &a)
{
    if (a.dtype == DT_BF16) launch<bf16_t, true>(s, a);
    else launch<float, true>(s, a);
}

}  // namespace tr
