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

constexpr int THREADS = PICK_THREADS, WAVES = PICK_WAVES, EACH = PICK_PART / 64;
constexpr int BIN_BITS = 11, BINS = 1 << BIN_BITS;
constexpr int MAX_PARTS = PICK_MAX_VOCAB / PICK_PART;
constexpr int PART_STEPS = PICK_PART / THREADS;      // tokens a thread where a workgroup looks through a part
constexpr int FEW = 256;      // tokens that are compared with each other, all with all
constexpr uint32_t LOWEST = 0x00800000u, ANY = 0xffffffffu;      // key of the lowest finite logit
static_assert(MAX_PARTS == 2 * THREADS && PART_STEPS == 2 && THREADS == 2 * FEW);

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

// 2^(j / 32) as 64-bit words, less j << 47: with k << 47 added, k = 32 e + j, the word of 2^(k / 32)
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
        const double q = fma(fma(fma(uniform(9.172598566029335e-09), f, uniform(1.6938609067364198e-06)), f, uniform(0.00023459619820112603)), f, uniform(0.021660849392187844));
        const uint2 word = powers[k & 31];
        const double power = __hiloint2double((int)(word.y + (k << 15)), (int)word.x);
        return fma(power, q * f, power);
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
    u64 part[WAVES];
    u64 before, at;
    double run;
    uint2 powers[32];
    uint32_t place, top, from, n;
    uint32_t first, last;
    int found, entries;
    union {
        struct { u64 few[FEW], few_mass[FEW]; };
        u64 entry[PICK_MAX_ENTRIES];
        u64 mass[MAX_PARTS];
    };
    uint32_t key[HELD], id[WHOLE ? 1 : HELD];      // tokens, key 0: none
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
    for (int w = 0; w < WAVES; ++w) {
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
    constexpr int N = BINS / THREADS;
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += THREADS) s.bin[i] = 0;
    if (threadIdx.x == 0) s.found = 0;
    __syncthreads();
    each([&](uint32_t place, auto amount) {
        const uint32_t d = place - base;
        if (d <= most) atomicAdd(&s.bin[d >> shift], (u64)amount());
    });
    __syncthreads();
    u64 mine[N], sum = 0, total;
#pragma unroll
    for (int e = 0; e < N; ++e) sum += mine[e] = s.bin[threadIdx.x * N + e];
    u64 run = before + sum_upto(sum, total, s) - sum;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (run < want && want <= run + mine[e]) {      // (for one thread and one bin at most)
            s.found = 1; s.before = run; s.at = mine[e]; s.place = base + ((uint32_t)(threadIdx.x * N + e) << shift);
        }
        run += mine[e];
    }
    __syncthreads();
    return s.found ? Border{true, s.place, s.before, s.at} : Border{false, 0, 0, 0};
}

// The first place up to which the amounts come to `want` (> 0) or more, what lies before it and what at it. each(add) calls add(place, amount) for everything, amount() being what it is; places are below
// 2^bits. Eleven bits of the place at a time, by a histogram of amounts. All threads get the answer. b: of a step before, which bits are left of.
template <class Each, class S> __device__ __forceinline__ Border find_border(Each each, int bits, u64 want, S &s, Border b = Border{true, 0, 0, 0})
{
#pragma unroll 1
    do {
        const int shift = max(0, bits - BIN_BITS);
        b = border_step(each, b.place, bits, shift, b.before, want, s);
        bits = shift;
    } while (bits > 0 && b.found);
    return b;
}

// Where a row's tokens come from: what a workgroup holds, all tokens of keys `from` and above
template <class S> struct Pool {
    const S &s;
    uint32_t from, n;
    __device__ __forceinline__ bool all() const { return from <= LOWEST; }
    template <class F> __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) if (const uint32_t key = s.key[i]) f(key, S::by_place ? i : s.id[i]);
    }
};

// The row itself, 16 bytes at a time; it may begin at any element
template <class T> struct Streamed {
    const T *row;
    int vocab;
    static constexpr uint32_t from = LOWEST;
    __device__ __forceinline__ bool all() const { return true; }
    template <class F> __device__ __forceinline__ void each(F f) const
    {
        constexpr int N = 16 / sizeof(T);
#pragma unroll 1
        for (int i = threadIdx.x * N; i < vocab; i += THREADS * N) {
            T v[N];
            if (i + N <= vocab) __builtin_memcpy(v, row + i, 16);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = row[min(i + e, vocab - 1)];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t key = i + e < vocab ? key_of(wide(v[e])) : 0;
                if (key) f(key, (uint32_t)(i + e));
            }
        }
    }
};

// What is kept of a row: all keys above `key`, and of those equal to it ids up to `last`
struct Kept {
    uint32_t key, last;
    __device__ __forceinline__ bool has(uint32_t k, uint32_t id) const { return k > key || (k == key && id <= last); }
};

__device__ __forceinline__ int bits_of(uint32_t v) { return v ? 32 - __clz(v) : 1; }

// a share of `sum`, one unit at least
__device__ __forceinline__ u64 share_of(float p, u64 sum) { return max(min((u64)ceil(fmax((double)p, 0.0) * (double)sum), sum), 1ull); }
__device__ __forceinline__ u64 share_of(float p, double weight, double unit) { return max((u64)ceil(fmax((double)p, 0.0) * weight * unit), 1ull); }

// A first step towards the border of top-k or top-p (key places, 2^shift of them), where one was taken
struct First { Border b; int shift; };

// What the filters keep; false: more than the source knows of. `weight`: of the whole row, for a source that does not hold it all.
template <class Source, class S> __device__ __forceinline__ bool keep(const Source &src, const Row &r, double weight, int vocab, const First &first, Kept &kept, S &s)
{
    const int key_bits = first.b.found ? first.shift : bits_of(r.top_key - src.from);
    const Border from = first.b.found ? first.b : Border{true, 0, 0, 0};
    bool cut = false;
    u64 ties = 0;                     // 0: all of them
    kept = Kept{LOWEST, ANY};
    if (r.k > 0) {
        const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t) { add(r.top_key - key, [] { return 1; }); }); }, key_bits, r.k, s, from);
        if (!b.found && !src.all()) return false;
        if (b.found) { kept.key = r.top_key - b.place; ties = r.k - b.before < b.at ? r.k - b.before : 0; cut = true; }
    }
    if (r.p < 1.f) {
        const uint32_t least = max(kept.key, src.from);
        u64 want;
        if (cut || src.all()) {
            u64 sum = 0;
            src.each([&](uint32_t key, uint32_t) { sum += key > kept.key || (key == kept.key && !ties) ? r.mass(key) : 0; });
            want = share_of(r.p, sum_of_all(sum, s) + (ties ? ties * r.mass(kept.key) : 0));
        } else want = share_of(r.p, weight, r.unit);
        const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t) { if (key >= least) add(r.top_key - key, [&] { return r.mass(key); }); }); },
                                     cut ? bits_of(r.top_key - least) : key_bits, want, s, cut ? Border{true, 0, 0, 0} : from);
        if (!b.found) return false;
        const uint32_t key = r.top_key - b.place;
        const u64 one = r.mass(key), need = (want - b.before + one - 1) / one;
        if (key != kept.key || !ties || need < ties) ties = need < b.at / one ? need : 0;
        kept.key = key;
        cut = true;
    }
    if (r.m > 0.f) {
        const uint32_t least = least_key(r);
        if (!cut && least < src.from) return false;
        if (least > kept.key) { kept.key = least; ties = 0; }
        if (r.m > 1.f) ties = 1;
        cut = true;
    }
    if (!cut && !src.all()) return false;
    if (ties) kept.last = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t id) { if (key == kept.key) add(id, [] { return 1; }); }); }, bits_of(vocab - 1), ties, s).place;
    return true;
}

__device__ __forceinline__ void put_draw(const PickArgs &a, int r, const Row &row, uint32_t id, float z, double total)
{
    a.token[r] = (int)id;
    a.logprob[r] = (float)((z == row.top ? 0.0 : ((double)z - row.top) * row.per * 0.021660849392497955) - log(total));      // (ln 2 / 32)
}
__device__ __forceinline__ void put_nothing(const PickArgs &a, int r, bool top)
{
    if (top) for (int i = threadIdx.x; i < a.entries; i += THREADS) { a.ids[(long long)r * a.entries + i] = -1; a.values[(long long)r * a.entries + i] = -INFINITY; }
    else if (threadIdx.x == 0) { a.token[r] = -1; a.logprob[r] = 0.f; }
}

template <class T, class Source, class S> __device__ __forceinline__ bool draw(const Source &src, const PickArgs &a, int r, const T *logits, const Row &row, double weight, const First &first, S &s)
{
    Kept kept;
    if (!keep(src, row, weight, a.vocab, first, kept, s)) return false;
    u64 sum = 0;
    src.each([&](uint32_t key, uint32_t id) { sum += kept.has(key, id) ? row.mass(key) : 0; });
    sum = sum_of_all(sum, s);
    const u64 below = min((u64)(evenly(a.u[r]) * (double)sum), sum - 1);
    const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t id) { if (kept.has(key, id)) add(id, [&] { return row.mass(key); }); }); }, bits_of(a.vocab - 1), below + 1, s);
    if (threadIdx.x == 0) put_draw(a, r, row, b.place, wide(logits[b.place]), (double)sum / row.unit);
    return true;
}

template <class Source, class S> __device__ __forceinline__ bool list_top(const Source &src, const PickArgs &a, int r, const Row &row, const First &first, S &s)
{
    Kept kept;
    if (!keep(src, row, 0.0, a.vocab, first, kept, s)) return false;
    __syncthreads();
    for (int i = threadIdx.x; i < PICK_MAX_ENTRIES; i += THREADS) s.entry[i] = ~0ull;
    if (threadIdx.x == 0) s.entries = 0;
    __syncthreads();
    src.each([&](uint32_t key, uint32_t id) { if (kept.has(key, id)) s.entry[atomicAdd(&s.entries, 1)] = (u64)~key << 32 | id; });
    __syncthreads();
    const int n = s.entries;
#pragma unroll 1
    for (int size = 2; size < 2 * n; size *= 2)
#pragma unroll 1
        for (int step = size / 2; step; step /= 2) {
            __syncthreads();
            const int x = (threadIdx.x / step) * 2 * step + threadIdx.x % step, y = x + step;
            const u64 v = s.entry[x], w = s.entry[y];
            if ((v > w) == !(x & size)) { s.entry[x] = w; s.entry[y] = v; }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < a.entries; i += THREADS) {
        const u64 e = s.entry[i];
        a.ids[(long long)r * a.entries + i] = e == ~0ull ? -1 : (int)(uint32_t)e;
        a.values[(long long)r * a.entries + i] = e == ~0ull ? -INFINITY : logit_of(~(uint32_t)(e >> 32));
    }
    return true;
}

// Tokens that a workgroup can compare all with all: those from where top-k or top-p end on, or min-p. Two threads a token add up what comes before it in the order, and then, of what is kept,
// what comes before it by id. false: more than FEW, or more than the source knows of.
template <bool TOP, class S> __device__ __forceinline__ bool among_few(const Pool<S> &src, const PickArgs &a, int r, const Row &row, double weight, First &first, S &s)
{
    if (row.k > FEW) return false;
    uint32_t floor = src.from;
    bool closed = src.all();
    const uint32_t least = row.m > 0.f ? least_key(row) : 0;
    if (row.m > 0.f && least >= floor && !(row.p < 1.f && row.k > 0)) { floor = least; closed = true; }      // (top-p's is a share of all that top-k keeps)
    u64 want = 0;
    if (row.p < 1.f && row.k == 0) {
        if (!src.all()) want = share_of(row.p, weight, row.unit);
        else {
            u64 sum = 0;
            src.each([&](uint32_t key, uint32_t) { sum += row.mass(key); });
            want = share_of(row.p, sum_of_all(sum, s));
        }
    }
    if (row.k > 0 || row.p < 1.f) {
        const int bits = bits_of(row.top_key - floor), shift = max(0, bits - BIN_BITS);
        const bool by_count = row.k > 0;
        const Border b = border_step([&](auto add) { src.each([&](uint32_t key, uint32_t) { if (key >= floor) add(row.top_key - key, [&] { return by_count ? 1 : row.mass(key); }); }); }, 0, bits, shift, 0,
                                     by_count ? (u64)row.k : want, s);
        first = First{b, shift};
        if (b.found) { floor = row.top_key - min(row.top_key - floor, b.place + ((1u << shift) - 1)); closed = true; }
    }
    if (!closed) return false;
    __syncthreads();
    if (threadIdx.x == 0) s.entries = 0;
    __syncthreads();
    src.each([&](uint32_t key, uint32_t id) {
        if (key < floor) return;
        const int i = atomicAdd(&s.entries, 1);
        if (i < FEW) s.few[i] = (u64)~key << 32 | id;
    });
    __syncthreads();
    const int n = s.entries;
    if (n > FEW) return false;
    const int i = threadIdx.x / 2, half = threadIdx.x % 2;
    const u64 mine = i < n ? s.few[i] : ~0ull;
    const uint32_t key = ~(uint32_t)(mine >> 32), id = (uint32_t)mine;
    if constexpr (TOP) {
        int rank = 0;
        if (i < n)
#pragma unroll 4
            for (int j = half; j < n; j += 2) rank += s.few[j] < mine;
        rank += __shfl_xor(rank, 1);
        if (i < n && half == 0 && rank < a.entries) {
            a.ids[(long long)r * a.entries + rank] = (int)id;
            a.values[(long long)r * a.entries + rank] = logit_of(key);
        }
        for (int e = n + threadIdx.x; e < a.entries; e += THREADS) { a.ids[(long long)r * a.entries + e] = -1; a.values[(long long)r * a.entries + e] = -INFINITY; }
        return true;
    }
    const u64 own = i < n ? row.mass(key) : 0;
    if (i < n && half == 0) s.few_mass[i] = own;
    __syncthreads();
    int rank = 0;
    u64 before = 0;
    if (i < n)
#pragma unroll 4
        for (int j = half; j < n; j += 2) {
            const bool less = s.few[j] < mine;
            rank += less;
            before += less ? s.few_mass[j] : 0;
        }
    rank += __shfl_xor(rank, 1);
    before += __shfl_xor(before, 1);
    bool kept = i < n && (row.k == 0 || rank < row.k);
    if (row.p < 1.f) {
        if (row.k > 0) want = share_of(row.p, sum_of_all(kept && half == 0 ? own : (u64)0, s));
        kept = kept && before < want;
    }
    if (row.m > 0.f) kept = kept && (rank == 0 || (key >= least && !(row.m > 1.f)));
    const u64 sum = sum_of_all(kept && half == 0 ? own : (u64)0, s);
    if (i < n && half == 0) s.few_mass[i] = kept ? own : 0;
    __syncthreads();
    const u64 below = min((u64)(evenly(a.u[r]) * (double)sum), sum - 1);
    before = 0;
    if (kept)
#pragma unroll 4
        for (int j = half; j < n; j += 2) before += (uint32_t)s.few[j] < id ? s.few_mass[j] : 0;
    before += __shfl_xor(before, 1);
    if (kept && half == 0 && before <= below && below < before + own) put_draw(a, r, row, id, logit_of(key), (double)sum / row.unit);
    return true;
}

struct Found { int at; double before; };

// The first of the values (N a thread, in the threads' order) up to which they add up to more than `want`; where rounding leaves none the last that is no zero. `before`: sum of the
// threads' before this one. Sums in 64 bits in a fixed order.
template <int N, class S> __device__ __forceinline__ Found first_over(const double (&v)[N], double before, double want, S &s)
{
    double run = before, found_at = before;
    uint32_t first = ANY, last = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const double from = run;
        run += v[e];
        if (!(v[e] > 0)) continue;
        const uint32_t i = threadIdx.x * N + e;
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
    if (at / N == threadIdx.x) s.run = found_at;
    __syncthreads();
    return Found{(int)at, s.run};
}

// A draw from a row that nothing is cut from, which more than one workgroup has read in parts that are one piece each: the part by the parts' weights (two a thread), then the token in it
template <class T, class S> __device__ __forceinline__ void draw_freely(const PickArgs &a, int r, const T *logits, const Row &row, const double (&parts)[2], S &s)
{
    double total, rest;
    double before = sum_upto(parts[0] + parts[1], total, s) - (parts[0] + parts[1]);
    const double want = evenly(a.u[r]) * total;
    const Found part = first_over(parts, before, want, s);
    float z[PART_STEPS];
    double v[PART_STEPS], sum = 0;
    const int first = part.at * PICK_PART + threadIdx.x * PART_STEPS;
#pragma unroll
    for (int e = 0; e < PART_STEPS; ++e) z[e] = first + e < a.vocab ? wide(logits[first + e]) : -INFINITY;
#pragma unroll
    for (int e = 0; e < PART_STEPS; ++e) sum += v[e] = z[e] > -INFINITY ? row.weight(z[e]) : 0;
    before = sum_upto(sum, rest, s) - sum;
    const Found token = first_over(v, before, want - part.before, s);
#pragma unroll
    for (int e = 0; e < PART_STEPS; ++e) if (token.at == (int)threadIdx.x * PART_STEPS + e) put_draw(a, r, row, first + e, z[e], total);
}

// ------------------------------------------------------------------ the kernels

// A part of a row: blocks of a load each, `step` apart, in LDS as 32 bits, EACH a lane (-inf: no token). A load past the row's end is moved back, and what it has twice is dropped.
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
    __device__ __forceinline__ float load(const T *logits)
    {
        T raw[BLOCKS][N];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) __builtin_memcpy(raw[i], (const char *)logits + at(i) * (uint32_t)sizeof(T), 16);
        // (the last lane's last load ends within the row: so do all)
        const bool whole = __builtin_amdgcn_readlane((int)(first + (BLOCKS - 1) * step), 63) + N <= vocab;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[e] = wide(raw[i][e]);
                v[e] = v[e] > -INFINITY ? v[e] : -INFINITY;
            }
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

// Bound by its instructions: some 40 a token and lane where sums are wanted, half of them 64-bit ones for the weight.
template <class T, bool TOP> __global__ __launch_bounds__(THREADS, 8) void parts_kernel(PickArgs a)
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
    const uint32_t lane_top = key_of(p.load((const T *)a.logits + (long long)r * a.stride));
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
            lanes /= 2;
            if (from > head.top) break;                               // nothing is listed
        }
        head.from = from;
        p.list(mask, upto, sum, a.listed, a.list + ((long long)r * parts + part) * a.listed);
    }
    if (lane == 0) a.head[(long long)r * parts + part] = head;
}

// the parts' lists, `listed` a part, into a workgroup's pool: those of keys `least` and above
template <int HELD> struct Lists {
    uint2 v[HELD / THREADS];
    __device__ __forceinline__ void load(const PickArgs &a, int r, int parts)
    {
        const uint2 *const list = a.list + (long long)r * parts * a.listed;
        const uint32_t all = parts * a.listed;
#pragma unroll
        for (int e = 0; e < HELD / THREADS; ++e) {
            const uint32_t i = e * THREADS + threadIdx.x;
            v[e] = i < all ? list[i] : make_uint2(0, 0);
        }
    }
    template <class S> __device__ __forceinline__ uint32_t hold(uint32_t least, S &s) const      // (s.n is zero, behind a barrier)
    {
        int n = 0;
#pragma unroll
        for (int e = 0; e < HELD / THREADS; ++e) n += v[e].x && v[e].x >= least;
        const int upto = wave_upto(n, Plus{});
        uint32_t at = 0;
        if (threadIdx.x % 64 == 63) at = atomicAdd(&s.n, (uint32_t)upto);
        at = last_lane(at) + upto - n;
#pragma unroll
        for (int e = 0; e < HELD / THREADS; ++e) if (v[e].x && v[e].x >= least) { s.key[at] = v[e].x; s.id[at++] = v[e].y; }
        __syncthreads();
        return s.n;
    }
};

// One workgroup a row. Bound by the latency of a few loads and of some twenty barriers.
template <class T, bool TOP, bool WHOLE, int HELD> __global__ __launch_bounds__(THREADS) void decide_kernel(PickArgs a)
{
    using S = Shared<HELD, WHOLE>;
    __shared__ S s;
    const int r = blockIdx.x, vocab = a.vocab, parts = a.groups * WAVES;
    const T *const logits = (const T *)a.logits + (long long)r * a.stride;
    Row row = row_of<TOP>(a, r, s.powers);
    if (threadIdx.x == 0) { s.top = 0; s.from = LOWEST; s.n = 0; }
    load_powers(s.powers);
    Pool<S> pool{s, LOWEST, (uint32_t)vocab};
    double weight = 0;
    if constexpr (WHOLE) {
        constexpr int N = 16 / sizeof(T);
        __syncthreads();
        uint32_t top = 0;
        if (vocab >= N) {
#pragma unroll
            for (int i = 0; i < HELD / THREADS / N; ++i) {
                const int at = min((i * THREADS + (int)threadIdx.x) * N, vocab - N);      // (some twice, the same)
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
        top = wave_max(top);
        if (threadIdx.x % 64 == 0) atomicMax(&s.top, top);
        __syncthreads();
        if (!s.top) { put_nothing(a, r, TOP); return; }
        row.relative_to(s.top);
    } else {
        PickHead head[2]{};
#pragma unroll
        for (int e = 0; e < 2; ++e) if ((int)threadIdx.x * 2 + e < parts) head[e] = a.head[(long long)r * parts + threadIdx.x * 2 + e];
        Lists<HELD> lists;
        if (row.cut) lists.load(a, r, parts);
        __syncthreads();
        const uint32_t top = wave_max(max(head[0].top, head[1].top)), from = wave_max(max(head[0].from, head[1].from));
        if (threadIdx.x % 64 == 0) { atomicMax(&s.top, top); atomicMax(&s.from, from); }
        __syncthreads();
        if (!s.top) { put_nothing(a, r, TOP); return; }
        row.relative_to(s.top);
        pool.from = s.from;
        if constexpr (!TOP) {
            if (row.summed) {
                double v[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) v[e] = head[e].top ? head[e].sum * row.weight(logit_of(head[e].top)) : 0;
                if (!row.cut) {
                    draw_freely(a, r, logits, row, v, s);
                    return;
                }
                weight = sum_of_all(v[0] + v[1], s);
            }
        }
        pool.n = lists.hold(pool.from, s);
    }
    First first{};
    if (among_few<TOP>(pool, a, r, row, weight, first, s)) return;
    if constexpr (TOP) {
        if (list_top(pool, a, r, row, first, s)) return;
    } else {
        if (draw(pool, a, r, logits, row, weight, first, s)) return;
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
    if constexpr (!WHOLE) {
        const Streamed<T> whole{logits, vocab};
        if constexpr (TOP) list_top(whole, a, r, row, First{}, s);
        else draw(whole, a, r, logits, row, weight, First{}, s);
    }
}

// ------------------------------------------------------------------ rows that are searched

// The step of a logit below `from`; larger logits are in no later step
__device__ __forceinline__ int step_of(float z, const PickSearch &q) { return (int)fminf((q.from - z) * q.scale, (float)PICK_STEPS); }

// Masses by steps below `from`, in the last place that of everything from it on; what is below all steps is left out
template <class T> __global__ __launch_bounds__(THREADS, 8) void steps_kernel(PickArgs a)
{
    __shared__ float s_z[WAVES][EACH / 4][64][4];
    __shared__ uint2 s_powers[32];
    __shared__ u64 step[PICK_STEPS];
    static_assert(PICK_STEPS == THREADS);
    load_powers(s_powers);
    const uint32_t items = a.queue[0] * a.groups;
#pragma unroll 1
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int r = a.queue[1 + item / a.groups], group = item % a.groups;
        const PickSearch q = a.search[r];
        if (q.stage != PICK_STEP) continue;
        step[threadIdx.x] = 0;
        Row row = row_of<false>(a, r, s_powers);
        row.relative_to(q.top_key);
        using P = Part<T>;
        P p{s_z[threadIdx.x / 64], (uint32_t)(group * WAVES + threadIdx.x / 64) * PICK_PART + threadIdx.x % 64 * P::N, P::BLOCK, a.vocab};
        p.load((const T *)a.logits + (long long)r * a.stride);
        __syncthreads();
        u64 above = 0;
        p.each([&](float z, int) {
            const int at = z >= q.from ? -1 : step_of(z, q);
            if (z == -INFINITY || at >= PICK_STEPS - 1) return;
            const u64 m = row.in_units(row.finite_weight(z));
            if (at < 0) above += m;
            else atomicAdd(&step[at], m);
        });
        above = wave_sum(above);
        if (threadIdx.x % 64 == 0) atomicAdd(&step[PICK_STEPS - 1], above);
        __syncthreads();
        a.steps[((long long)r * a.groups + group) * PICK_STEPS + threadIdx.x] = step[threadIdx.x];
    }
}

// The step that top-p ends in; of each part the mass of what is above it and its tokens in it. Where min-p alone decides, the mass of what it keeps.
template <class T> __global__ __launch_bounds__(THREADS, 8) void place_kernel(PickArgs a)
{
    __shared__ float s_z[WAVES][EACH / 4][64][4];
    __shared__ uint2 s_powers[32];
    __shared__ u64 s_part[WAVES];
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
            u64 sum = 0;
            const u64 *const steps = a.steps + (long long)r * a.groups * PICK_STEPS + threadIdx.x;
#pragma unroll 4
            for (int g = 0; g < a.groups; ++g) sum += steps[g * PICK_STEPS];
            // (what is above all steps, which the last place holds, comes before them)
            u64 upto = wave_upto(threadIdx.x == PICK_STEPS - 1 ? 0 : sum, Plus{});
            __syncthreads();
            if (threadIdx.x == 0) s_step = PICK_STEPS;
            if (lane == 63) s_part[wave] = wave == WAVES - 1 ? sum : upto;
            __syncthreads();
            upto += s_part[WAVES - 1];
#pragma unroll
            for (int w = 0; w < WAVES - 1; ++w) upto += w < wave ? s_part[w] : 0;
            if (threadIdx.x < PICK_STEPS - 1 && upto - sum < q.want && q.want <= upto) s_step = threadIdx.x;
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
            if (z == -INFINITY) return;
            const int at = stage == PICK_STEP ? step_of(z, q) : PICK_STEPS;
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

// The place in the step, and the draw: the part by the parts' masses, then the token in it
template <class T> __global__ __launch_bounds__(THREADS) void finish_kernel(PickArgs a)
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
        if (threadIdx.x == 0) s.n = 0;
        bool whole = q.found == PICK_WHOLE;
        u64 above = 0;
        if (!whole) {
            u64 over = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int w = threadIdx.x * 2 + e;
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
            const Streamed<T> all{logits, vocab};
            draw(all, a, r, logits, row, 0.0, First{}, s);
            continue;
        }
        Kept kept{q.least, ANY};
        if (q.found == PICK_STEP) {
            Lists<HELD> lists;
            lists.load(a, r, parts);
            const Pool<Shared<HELD>> pool{s, LOWEST, lists.hold(LOWEST, s)};
            const Border b = find_border([&](auto add) { pool.each([&](uint32_t key, uint32_t) { add(q.top_key - key, [&] { return row.mass(key); }); }); }, bits_of(q.top_key - LOWEST),
                                         q.want - above, s);
            kept.key = q.top_key - b.place;
            const u64 one = row.mass(kept.key), need = (q.want - above - b.before + one - 1) / one;
            u64 ties = need < b.at / one ? need : 0;
            if (q.least > kept.key) { kept.key = q.least; ties = 0; }
            if (ties) kept.last = find_border([&](auto add) { pool.each([&](uint32_t key, uint32_t id) { if (key == kept.key) add(id, [] { return 1; }); }); }, bits_of(vocab - 1), ties, s).place;
            __syncthreads();
            pool.each([&](uint32_t key, uint32_t id) { if (kept.has(key, id)) atomicAdd(&s.mass[id / PICK_PART], row.mass(key)); });
            __syncthreads();
        }
        u64 total, rest;
        const u64 m[2] = {s.mass[threadIdx.x * 2], s.mass[threadIdx.x * 2 + 1]};
        u64 run = sum_upto(m[0] + m[1], total, s) - m[0] - m[1];
        const u64 below = min((u64)(evenly(a.u[r]) * (double)total), total - 1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (run <= below && below < run + m[e]) { s.place = threadIdx.x * 2 + e; s.before = run; }
            run += m[e];
        }
        __syncthreads();
        const int first = s.place * PICK_PART + threadIdx.x * PART_STEPS;
        const u64 left = below - s.before;
        float z[PART_STEPS];
        u64 v[PART_STEPS], sum = 0;
#pragma unroll
        for (int e = 0; e < PART_STEPS; ++e) z[e] = first + e < vocab ? wide(logits[first + e]) : -INFINITY;
#pragma unroll
        for (int e = 0; e < PART_STEPS; ++e) {
            const uint32_t key = key_of(z[e]);
            sum += v[e] = key && kept.has(key, first + e) ? row.mass(key) : 0;
        }
        run = sum_upto(sum, rest, s) - sum;
#pragma unroll
        for (int e = 0; e < PART_STEPS; ++e) {
            if (run <= left && left < run + v[e]) put_draw(a, r, row, first + e, z[e], (double)total / row.unit);
            run += v[e];
        }
    }
}

template <class T, bool TOP> void launch_parts(hipStream_t s, const PickArgs &a)
{
    const unsigned all = (unsigned)a.rows * a.groups;
    hipLaunchKernelGGL((parts_kernel<T, TOP>), dim3(all), dim3(THREADS), 0, s, a);
    if (a.groups * WAVES * a.listed <= 4096) hipLaunchKernelGGL((decide_kernel<T, TOP, false, 4096>), dim3(a.rows), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((decide_kernel<T, TOP, false, PICK_LISTED>), dim3(a.rows), dim3(THREADS), 0, s, a);
    if constexpr (!TOP) {
        if (!a.queue) return;
        // rows of the queue, which the host does not know: as many workgroups as run at once, which are soon gone where it is empty
        hipLaunchKernelGGL(steps_kernel<T>, dim3(std::min(all, 1024u)), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(place_kernel<T>, dim3(std::min(all, 1024u)), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(finish_kernel<T>, dim3(std::min(a.rows, 256)), dim3(THREADS), 0, s, a);
    }
}

template <class T, bool TOP> void launch(hipStream_t s, const PickArgs &a)
{
    const dim3 rows(a.rows), threads(THREADS);
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
