// Tokens drawn from rows of logits, and a row's largest logits (row_pick.h).
//
// Every wavefront reads a part of a row once, into registers, and leaves its largest tokens (about `listed` of 1024, whatever their logits: it looks for a threshold that few enough
// lanes reach) and, where they are asked for, its sum of weights (parts_kernel). A workgroup a row takes the parts' tokens into registers: down to the largest of the parts' thresholds it
// has them all (decide_kernel). As long as top-k, top-p and min-p end above that, they and the draw are searches in its registers. A row so flat that top-p or min-p do not is read twice more:
// for the step of a histogram of masses in which top-p ends (steps_kernel), and for the tokens in that step and the sums of what is above it, part by part (place_kernel, finish_kernel).
// Rows of up to 8192 tokens are one workgroup's from the start.
#include "row_pick.h"

#include <float.h>
#include <type_traits>

namespace tr {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = PICK_THREADS, WAVES = PICK_WAVES, EACH = PICK_EACH;
constexpr int BIN_BITS = 11, BINS = 1 << BIN_BITS;
constexpr int MAX_PARTS = (PICK_MAX_VOCAB + PICK_PART - 1) / PICK_PART;
constexpr uint32_t LOWEST = 0x00800000u, ANY = 0xffffffffu;      // key of the lowest finite logit

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

// 2^x, x <= 0: Taylor's series of e^(f ln 2), |f| <= 1/2, whose next term is below 2^-52
__device__ __forceinline__ double pow2(double x)
{
    x = fmax(x, -1200.0);
    const double n = rint(x), f = x - n;
    double p = 2.5678435993488196e-11;
    p = fma(p, f, 4.44553827187081e-10);
    p = fma(p, f, 7.054911620801121e-09);
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 0.00015403530393381606);
    p = fma(p, f, 0.0013333558146428441);
    p = fma(p, f, 0.009618129107628477);
    p = fma(p, f, 0.055504108664821576);
    p = fma(p, f, 0.2402265069591007);
    p = fma(p, f, 0.6931471805599453);
    return ldexp(fma(p, f, 1.0), (int)n);
}

// What a row's user set, and what weights are relative to
struct Row {
    float t, p, m;
    int k;                  // 0: all
    bool cut, summed;       // some filter is set; the parts' sums are wanted
    double top, per, unit;  // largest logit, log2(e) / T, 2^unit
    uint32_t top_key;
    __device__ __forceinline__ double power(float z) const { return z == top ? 0.0 : ((double)z - top) * per; }     // (an infinite one is there by itself)
    __device__ __forceinline__ u64 mass(uint32_t key) const { return (u64)(pow2(power(logit_of(key))) * unit + 0.5); }
};

constexpr int FEW = 256;      // tokens that are compared with each other, all with all

struct Shared {
    u64 bin[BINS];
    u64 part[WAVES];
    u64 before, at;
    uint32_t place;
    int found, first, last;
    double run;
    int entries;
    union {
        struct { double sum[MAX_PARTS]; uint32_t top[MAX_PARTS]; uint16_t count[MAX_PARTS]; };
        struct { u64 few[FEW], few_mass[FEW]; };
        struct { u64 mass[MAX_PARTS]; uint16_t listed[MAX_PARTS]; };
        u64 entry[PICK_MAX_ENTRIES];
    };
};

template <class T, class Join> __device__ __forceinline__ T wave_all(T v, Join join)
{
    for (int o = 1; o < 64; o *= 2) v = join(v, __shfl_xor(v, o));
    return v;
}
template <class T, class Join> __device__ __forceinline__ T all_of(T v, Join join, Shared &s)
{
    static_assert(sizeof(T) == 8);
    v = wave_all(v, join);
    __syncthreads();
    if (threadIdx.x % 64 == 0) __builtin_memcpy(&s.part[threadIdx.x / 64], &v, 8);
    __syncthreads();
    __builtin_memcpy(&v, &s.part[0], 8);
    for (int w = 1; w < WAVES; ++w) {
        T x;
        __builtin_memcpy(&x, &s.part[w], 8);
        v = join(v, x);
    }
    return v;
}
__device__ __forceinline__ u64 sum_of_all(u64 v, Shared &s) { return all_of(v, [](u64 a, u64 b) { return a + b; }, s); }
// sum of the values of all threads up to this one, and of all
template <class V> __device__ __forceinline__ V sum_upto(V v, V &total, Shared &s)
{
    static_assert(sizeof(V) == 8);
    for (int o = 1; o < 64; o *= 2) {
        const V x = __shfl_up(v, o);
        if ((int)threadIdx.x % 64 >= o) v += x;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 63) __builtin_memcpy(&s.part[threadIdx.x / 64], &v, 8);
    __syncthreads();
    V run = 0, before = 0;
    for (int w = 0; w < WAVES; ++w) {
        V x;
        __builtin_memcpy(&x, &s.part[w], 8);
        if (w == (int)threadIdx.x / 64) before = run;
        run += x;
    }
    total = run;
    return before + v;
}

struct Border { bool found; uint32_t place; u64 before, at; };

// One step of find_border: places from `base` on, below base + 2^bits, in steps of 2^shift; what lies before base comes to `before`. place: where the step begins; at: what it holds.
template <class Each> __device__ __forceinline__ Border border_step(Each each, uint32_t base, int bits, int shift, u64 before, u64 want, Shared &s)
{
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

// The first place up to which the amounts come to `want` (> 0) or more, what lies before it and what at it. each(add) calls add(place, amount) for everything; places are below
// 2^bits. Eleven bits of the place at a time, by a histogram of amounts. All threads get the answer.
template <class Each> __device__ __forceinline__ Border find_border(Each each, int bits, u64 want, Shared &s)
{
    Border b{true, 0, 0, 0};
    do {
        const int shift = max(0, bits - BIN_BITS);
        b = border_step(each, b.place, bits, shift, b.before, want, s);
        bits = shift;
    } while (bits > 0 && b.found);
    return b;
}

// ------------------------------------------------------------------ where a row's tokens come from

// The deciding workgroup's registers: all tokens of keys `from` and above
struct Held {
    uint32_t key[EACH], id[EACH], from;
    u64 m[EACH];
    __device__ __forceinline__ bool all() const { return from <= LOWEST; }
    template <class F> __device__ __forceinline__ void each(F f) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) if (key[e] >= from) f(key[e], id[e], [&] { return m[e]; });
    }
    __device__ __forceinline__ void weigh(const Row &r, uint32_t least)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) m[e] = key[e] >= least ? r.mass(key[e]) : 0;
    }
};

// The row itself, 16 bytes at a time; it may begin at any element
template <class T> struct Streamed {
    const T *row;
    int vocab;
    const Row &r;
    static constexpr uint32_t from = LOWEST;
    __device__ __forceinline__ bool all() const { return true; }
    __device__ __forceinline__ void weigh(const Row &, uint32_t) {}
    template <class F> __device__ __forceinline__ void each(F f) const
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
                const uint32_t key = i + e < vocab ? key_of(wide(v[e])) : 0;
                if (key) f(key, (uint32_t)(i + e), [&] { return r.mass(key); });
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

// The smallest key that min_p (> 0) keeps: weight >= min_p where the logit is at least max + T log min_p
__device__ __forceinline__ uint32_t least_key(const Row &r)
{
    if (!(r.m < 1.f)) return r.top_key;
    const double at = r.top + (double)r.t * log((double)r.m);
    float f = (float)at;
    if ((double)f < at) f = nextafterf(f, INFINITY);
    return max(key_of(f), LOWEST);
}

// What the filters keep; false: more than the source knows of. `mass`: of the whole row, for a source that does not hold it all.
template <class Source> __device__ __forceinline__ bool keep(Source &src, const Row &r, double mass, int vocab, Kept &kept, Shared &s)
{
    const int key_bits = bits_of(r.top_key - src.from);
    bool cut = false;
    u64 ties = 0;                     // 0: all of them
    kept = Kept{LOWEST, ANY};
    if (r.k > 0 && r.k < vocab) {
        const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t, auto) { add(r.top_key - key, 1); }); }, key_bits, r.k, s);
        if (!b.found && !src.all()) return false;
        if (b.found) { kept.key = r.top_key - b.place; ties = r.k - b.before < b.at ? r.k - b.before : 0; cut = true; }
    }
    if (r.p < 1.f) {
        const uint32_t least = max(kept.key, src.from);
        src.weigh(r, least);
        u64 want;
        if (cut || src.all()) {
            u64 sum = 0;
            src.each([&](uint32_t key, uint32_t, auto m) { sum += key > kept.key || (key == kept.key && !ties) ? m() : 0; });
            sum = sum_of_all(sum, s) + (ties ? ties * r.mass(kept.key) : 0);
            want = min((u64)ceil(fmax((double)r.p, 0.0) * (double)sum), sum);
        } else {
            want = (u64)ceil(fmax((double)r.p, 0.0) * mass * r.unit);
        }
        want = max(want, 1ull);
        const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t, auto m) { if (key >= least) add(r.top_key - key, m()); }); }, key_bits, want, s);
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
    if (ties) kept.last = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t id, auto) { if (key == kept.key) add(id, 1); }); }, bits_of(vocab - 1), ties, s).place;
    return true;
}

__device__ __forceinline__ double evenly(float u) { return fmin(fmax((double)u, 0.0), 1.0); }      // (NaN: 0)

__device__ __forceinline__ void put_draw(const PickArgs &a, int r, const Row &row, uint32_t id, float z, double total)
{
    a.token[r] = (int)id;
    a.logprob[r] = (float)(row.power(z) * 0.6931471805599453 - log(total));
}

template <class T, class Source> __device__ __forceinline__ bool draw(Source &src, const PickArgs &a, int r, const T *logits, const Row &row, double mass, Shared &s)
{
    Kept kept;
    if (!keep(src, row, mass, a.vocab, kept, s)) return false;
    src.weigh(row, kept.key);
    u64 sum = 0;
    src.each([&](uint32_t key, uint32_t id, auto m) { sum += kept.has(key, id) ? m() : 0; });
    sum = sum_of_all(sum, s);
    const u64 below = min((u64)(evenly(a.u[r]) * (double)sum), sum - 1);
    const Border b = find_border([&](auto add) { src.each([&](uint32_t key, uint32_t id, auto m) { if (kept.has(key, id)) add(id, m()); }); }, bits_of(a.vocab - 1), below + 1, s);
    if (threadIdx.x == 0) put_draw(a, r, row, b.place, wide(logits[b.place]), (double)sum / row.unit);
    return true;
}

template <class Source> __device__ __forceinline__ bool list_top(Source &src, const PickArgs &a, int r, const Row &row, Shared &s)
{
    Kept kept;
    if (!keep(src, row, 0.0, a.vocab, kept, s)) return false;
    __syncthreads();
    for (int i = threadIdx.x; i < PICK_MAX_ENTRIES; i += THREADS) s.entry[i] = ~0ull;
    if (threadIdx.x == 0) s.entries = 0;
    __syncthreads();
    src.each([&](uint32_t key, uint32_t id, auto) { if (kept.has(key, id)) s.entry[atomicAdd(&s.entries, 1)] = (u64)~key << 32 | id; });
    __syncthreads();
    const int n = s.entries;
    for (int size = 2; size < 2 * n; size *= 2)
        for (int step = size / 2; step; step /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < PICK_MAX_ENTRIES / 2; i += THREADS) {
                const int x = (i / step) * 2 * step + i % step, y = x + step;
                const u64 v = s.entry[x], w = s.entry[y];
                if ((v > w) == !(x & size)) { s.entry[x] = w; s.entry[y] = v; }
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < a.entries; i += THREADS) {
        const u64 e = i < PICK_MAX_ENTRIES ? s.entry[i] : ~0ull;
        a.ids[(long long)r * a.entries + i] = e == ~0ull ? -1 : (int)(uint32_t)e;
        a.values[(long long)r * a.entries + i] = e == ~0ull ? -INFINITY : logit_of(~(uint32_t)(e >> 32));
    }
    return true;
}

// Tokens that a workgroup can compare all with all: those from where top-k or top-p end on, or min-p. Two threads a token add up what comes before it in the order, and then, of what is kept,
// what comes before it by id. false: more than FEW, or more than the source knows of.
template <bool TOP, class T> __device__ __forceinline__ bool among_few(Held &src, const PickArgs &a, int r, const T *logits, const Row &row, double mass, Shared &s)
{
    if (row.k > FEW) return false;
    uint32_t floor = src.from;
    bool closed = src.all();
    const uint32_t least = row.m > 0.f ? least_key(row) : 0;
    if (row.m > 0.f && least >= floor && !(row.p < 1.f && row.k > 0)) { floor = least; closed = true; }      // (top-p's is a share of all that top-k keeps)
    u64 want = 0;
    if (row.k > 0 || row.p < 1.f) {
        const int bits = bits_of(row.top_key - floor), shift = max(0, bits - BIN_BITS);
        Border b;
        if (row.k > 0) b = border_step([&](auto add) { src.each([&](uint32_t key, uint32_t, auto) { if (key >= floor) add(row.top_key - key, 1); }); }, 0, bits, shift, 0, row.k, s);
        else {
            src.weigh(row, floor);
            if (!src.all()) want = max((u64)ceil(fmax((double)row.p, 0.0) * mass * row.unit), 1ull);
            else {
                u64 sum = 0;      // (min-p has no part in what top-p is a share of)
                src.each([&](uint32_t key, uint32_t, auto m) { sum += key >= floor ? m() : row.mass(key); });
                sum = sum_of_all(sum, s);
                want = max(min((u64)ceil(fmax((double)row.p, 0.0) * (double)sum), sum), 1ull);
            }
            b = border_step([&](auto add) { src.each([&](uint32_t key, uint32_t, auto m) { if (key >= floor) add(row.top_key - key, m()); }); }, 0, bits, shift, 0, want, s);
        }
        if (b.found) { floor = row.top_key - min(row.top_key - floor, b.place + ((1u << shift) - 1)); closed = true; }
    }
    if (!closed) return false;
    __syncthreads();
    if (threadIdx.x == 0) s.entries = 0;
    __syncthreads();
    src.each([&](uint32_t key, uint32_t id, auto) {
        if (key < floor) return;
        const int i = atomicAdd(&s.entries, 1);
        if (i < FEW) s.few[i] = (u64)~key << 32 | id;
    });
    __syncthreads();
    const int n = s.entries;
    if (n > FEW) return false;
    static_assert(THREADS == 2 * FEW);
    const int i = threadIdx.x / 2, half = threadIdx.x % 2;
    const u64 mine = i < n ? s.few[i] : ~0ull;
    const uint32_t key = ~(uint32_t)(mine >> 32), id = (uint32_t)mine;
    if constexpr (TOP) {
        int rank = 0;
        if (i < n) for (int j = half; j < n; j += 2) rank += s.few[j] < mine;
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
    if (i < n) for (int j = half; j < n; j += 2) {
        const bool less = s.few[j] < mine;
        rank += less;
        before += less ? s.few_mass[j] : 0;
    }
    rank += __shfl_xor(rank, 1);
    before += __shfl_xor(before, 1);
    bool kept = i < n && (row.k == 0 || rank < row.k);
    if (row.p < 1.f && row.k > 0) {
        const u64 sum = sum_of_all(kept && half == 0 ? own : 0, s);
        want = max(min((u64)ceil(fmax((double)row.p, 0.0) * (double)sum), sum), 1ull);
    }
    if (row.p < 1.f) kept = kept && before < want;
    if (row.m > 0.f) kept = kept && (rank == 0 || (key >= least && !(row.m > 1.f)));
    const u64 sum = sum_of_all(kept && half == 0 ? own : 0, s);
    if (i < n && half == 0) s.few_mass[i] = kept ? own : 0;
    __syncthreads();
    const u64 below = min((u64)(evenly(a.u[r]) * (double)sum), sum - 1);
    before = 0;
    if (kept) for (int j = half; j < n; j += 2) before += (uint32_t)s.few[j] < id ? s.few_mass[j] : 0;
    before += __shfl_xor(before, 1);
    if (kept && half == 0 && before <= below && below < before + own) put_draw(a, r, row, id, logit_of(key), (double)sum / row.unit);
    return true;
}

struct Found { int at; double before; };

// The first of the values (two a thread, in the threads' order) up to which they add up to more than `want`; where rounding leaves none the last that is no zero. `upto`: sum_upto of a
// thread's two. Sums in 64 bits in a fixed order.
__device__ __forceinline__ Found first_over(const double (&v)[2], double upto, double want, Shared &s)
{
    const double run[3] = {upto - (v[0] + v[1]), upto - v[1], upto};
    if (threadIdx.x == 0) { s.first = 0x7fffffff; s.last = 0; }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (!(v[e] > 0)) continue;
        atomicMax(&s.last, (int)threadIdx.x * 2 + e);
        if (run[e + 1] > want) atomicMin(&s.first, (int)threadIdx.x * 2 + e);
    }
    __syncthreads();
    const int at = min(s.first, s.last);
    if (at / 2 == (int)threadIdx.x) s.run = run[at % 2];
    __syncthreads();
    return Found{at, s.run};
}

// A draw from a row that nothing is cut from, which more than one workgroup has read in pieces of PICK_PART tokens: the piece by the pieces' sums, then the token in it
template <class T> __device__ __forceinline__ void draw_freely(const PickArgs &a, int r, const T *logits, const Row &row, int parts, Shared &s)
{
    static_assert(MAX_PARTS == 2 * THREADS && PICK_PART == 2 * THREADS);
    double v[2], total, rest;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int w = threadIdx.x * 2 + e;
        v[e] = w < parts && s.top[w] ? s.sum[w] * pow2(row.power(logit_of(s.top[w]))) : 0;
    }
    double upto = sum_upto(v[0] + v[1], total, s);
    const double want = evenly(a.u[r]) * total;
    const Found part = first_over(v, upto, want, s);
    float z[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int id = part.at * PICK_PART + threadIdx.x * 2 + e;
        z[e] = id < a.vocab ? wide(logits[id]) : -INFINITY;
        v[e] = z[e] > -INFINITY ? pow2(row.power(z[e])) : 0;
    }
    upto = sum_upto(v[0] + v[1], rest, s);
    const Found token = first_over(v, upto, want - part.before, s);
    if (token.at / 2 == (int)threadIdx.x) put_draw(a, r, row, part.at * PICK_PART + token.at, z[token.at % 2], total);
}

// ------------------------------------------------------------------ the kernels

template <bool TOP> __device__ __forceinline__ Row row_of(const PickArgs &a, int r)
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
    row.per = 1.4426950408889634 / (double)row.t;
    row.unit = __longlong_as_double((long long)(1023 + a.unit) << 52);
    return row;
}

// A part of a row in registers: blocks of a load each, `step` apart. A load past the end is moved back, and what it has twice is dropped (-inf, as NaN is).
template <class T> struct Part {
    static constexpr int N = 16 / sizeof(T), BLOCKS = EACH / N, BLOCK = 64 * N;
    float z[EACH];
    uint32_t at[BLOCKS];
    __device__ __forceinline__ uint32_t id(int e) const { return at[e / N] + e % N; }
    __device__ __forceinline__ void load(const T *logits, int vocab, long long first, long long step)
    {
        first += threadIdx.x % 64 * N;
        if (vocab >= N) {
            T raw[BLOCKS][N];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                at[i] = (uint32_t)min(first + i * step, (long long)(vocab - N));
                __builtin_memcpy(raw[i], logits + at[i], 16);
            }
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float v = wide(raw[i][e]);
                    z[i * N + e] = v > -INFINITY && (long long)at[i] + e >= first + i * step ? v : -INFINITY;
                }
        } else {
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                at[i] = (uint32_t)min(first + i * step, (long long)vocab);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    z[i * N + e] = -INFINITY;
                    if ((int)at[i] + e < vocab) {
                        const float v = wide(logits[at[i] + e]);
                        if (v > -INFINITY) z[i * N + e] = v;
                    }
                }
            }
        }
    }
    // Leaves the tokens that want(e) names in a list, lanes one after the other; nothing where they are more than `most`. Returns how many there are.
    template <class Want> __device__ __forceinline__ int list(Want want, int most, uint2 *to) const
    {
        const int lane = threadIdx.x % 64;
        int n = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) n += want(e);
        int upto = n;
        for (int o = 1; o < 64; o *= 2) {
            const int x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        const int sum = __shfl(upto, 63);
        if (sum <= most) {
            int i = upto - n;
#pragma unroll
            for (int e = 0; e < EACH; ++e) if (want(e)) to[i++] = make_uint2(key_of(z[e]), id(e));
        }
        return sum;
    }
};

// Bound by memory and, where sums are asked for, by as many 64-bit instructions.
template <class T, bool TOP> __global__ __launch_bounds__(THREADS) void parts_kernel(PickArgs a)
{
    using P = Part<T>;
    const int r = blockIdx.x / a.groups, lane = threadIdx.x % 64, parts = a.groups * WAVES, part = (blockIdx.x % a.groups) * WAVES + threadIdx.x / 64;
    Row row = row_of<TOP>(a, r);
    // Of a row that is cut from, blocks of all parts take turns, so that large logits that lie together are spread over the parts; of one that is drawn from freely a part is one
    // piece, so that its sum is a step of the sums by id.
    P p;
    p.load((const T *)a.logits + (long long)r * a.stride, a.vocab, row.cut ? (long long)part * P::BLOCK : (long long)part * PICK_PART, row.cut ? (long long)parts * P::BLOCK : P::BLOCK);
    float most = p.z[0];
#pragma unroll
    for (int e = 1; e < EACH; ++e) most = fmaxf(most, p.z[e]);
    const uint32_t lane_top = key_of(most);
    PickHead head{};
    head.top = wave_all(lane_top, [](auto x, auto y) { return x > y ? x : y; });
    if (row.summed && head.top) {
        row.top = logit_of(head.top);
#pragma unroll
        for (int e = 0; e < EACH; ++e) head.sum += p.z[e] > -INFINITY ? pow2(row.power(p.z[e])) : 0;
        head.sum = wave_all(head.sum, [](double x, double y) { return x + y; });
    }
    if (row.cut) {
        // a threshold that few enough tokens reach: one that listed_lanes lanes or somewhat fewer reach with their largest, then fewer until the tokens fit
        uint2 *const list = a.list + ((long long)r * parts + part) * a.listed;
        uint32_t from = LOWEST;
        int lanes = 64;
        for (;;) {
            const float least = logit_of(from);
            const int n = p.list([&](int e) { return p.z[e] >= least; }, a.listed, list);
            if (n <= a.listed) { head.count = n; break; }
            lanes = lanes == 64 ? a.listed_lanes : lanes / 2;
            uint32_t below = from, above = head.top + 1;              // no lane reaches it
            from = above;
            while (above - below > 1) {
                const uint32_t mid = below + (above - below) / 2;
                const int c = __popcll(__ballot(lane_top >= mid));
                if (c > lanes) below = mid;
                else {
                    above = from = mid;
                    if (c > lanes * 3 / 4) break;
                }
            }
            if (from > head.top) break;                               // nothing is listed
        }
        head.from = from;
    }
    if (lane == 0) a.head[(long long)r * parts + part] = head;
}

// One workgroup a row. Bound by the latency of a few loads and of some twenty barriers.
template <class T, bool TOP, bool WHOLE> __global__ __launch_bounds__(THREADS) void decide_kernel(PickArgs a)
{
    __shared__ Shared s;
    const int r = blockIdx.x, vocab = a.vocab, parts = a.groups * WAVES;
    const T *const logits = (const T *)a.logits + (long long)r * a.stride;
    Row row = row_of<TOP>(a, r);
    const auto larger = [](auto x, auto y) { return x > y ? x : y; };
    Held held;
    uint32_t top = 0;
    if constexpr (WHOLE) {
        using P = Part<T>;
        P p;
        p.load(logits, vocab, (long long)(threadIdx.x / 64) * P::BLOCK, (long long)WAVES * P::BLOCK);
#pragma unroll
        for (int e = 0; e < EACH; ++e) { held.key[e] = key_of(p.z[e]); held.id[e] = p.id(e); top = max(top, held.key[e]); }
        held.from = LOWEST;
        top = (uint32_t)all_of((u64)top, larger, s);
    } else {
        uint32_t from = LOWEST;
        for (int w = threadIdx.x; w < parts; w += THREADS) {
            const PickHead head = a.head[(long long)r * parts + w];
            s.sum[w] = head.sum; s.top[w] = head.top; s.count[w] = (uint16_t)head.count;
            top = max(top, head.top); from = max(from, head.from);
        }
        top = (uint32_t)all_of((u64)top, larger, s);
        held.from = (uint32_t)all_of((u64)from, larger, s);
        if (row.cut) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const uint32_t q = e * THREADS + threadIdx.x, w = __umulhi(q, a.listed_inverse), j = q - w * a.listed;
                uint2 v = make_uint2(0, 0);
                if (w < (uint32_t)parts && j < s.count[w]) v = a.list[((long long)r * parts + w) * a.listed + j];
                held.key[e] = v.x; held.id[e] = v.y;
            }
        }
        if (a.searched && threadIdx.x == 0) a.search[r].stage = PICK_DONE;
    }
    if (!top) {
        if constexpr (TOP) {
            for (int i = threadIdx.x; i < a.entries; i += THREADS) { a.ids[(long long)r * a.entries + i] = -1; a.values[(long long)r * a.entries + i] = -INFINITY; }
        } else if (threadIdx.x == 0) { a.token[r] = -1; a.logprob[r] = 0.f; }
        return;
    }
    row.top_key = top;
    row.top = logit_of(top);
    double mass = 0;
    if constexpr (!TOP && !WHOLE) {
        if (!row.cut) {
            draw_freely(a, r, logits, row, parts, s);
            return;
        }
        if (row.summed) {
            double mine = 0;
            for (int w = threadIdx.x; w < parts; w += THREADS) mine += s.top[w] ? s.sum[w] * pow2(row.power(logit_of(s.top[w]))) : 0;
            mass = all_of(mine, [](double x, double y) { return x + y; }, s);
        }
    }
    if (among_few<TOP>(held, a, r, logits, row, mass, s)) return;
    if constexpr (TOP) {
        if (list_top(held, a, r, row, s)) return;
    } else {
        if (draw(held, a, r, logits, row, mass, s)) return;
        if (!WHOLE && a.searched && row.k == 0 && row.top < INFINITY && held.from <= top) {
            if (threadIdx.x == 0) {
                PickSearch q{};
                q.stage = row.p < 1.f ? PICK_STEP : PICK_LEAST;
                q.top_key = top;
                q.least = row.m > 0.f ? least_key(row) : 0;
                q.from = logit_of(held.from);
                // what top-p leaves out, and the border with it, weighs (1 - p) of all or more, and none of it more than the border: that weighs (1 - p) / vocab of all or more
                const double share = fmax((double)row.p, 0.0), least = row.top + (double)row.t * log(0.5 * (1 - share) * mass / vocab);
                q.scale = (float)((PICK_STEPS - 2) / fmax((double)q.from - least, 1e-30));
                q.want = max((u64)ceil(share * mass * row.unit), 1ull);
                a.search[r] = q;
            }
            return;
        }
    }
    if constexpr (!WHOLE) {
        Streamed<T> whole{logits, vocab, row};
        if constexpr (TOP) list_top(whole, a, r, row, s);
        else draw(whole, a, r, logits, row, mass, s);
    }
}

// ------------------------------------------------------------------ rows that are searched

// The step of a logit below `from`; larger logits are in no later step
__device__ __forceinline__ int step_of(float z, const PickSearch &q) { return (int)fminf((q.from - z) * q.scale, (float)PICK_STEPS); }

__device__ __forceinline__ Row searched_row(const PickArgs &a, int r, const PickSearch &q)
{
    Row row = row_of<false>(a, r);
    row.top_key = q.top_key;
    row.top = logit_of(q.top_key);
    return row;
}

// Masses by steps below `from`, in the last place that of everything from it on; what is below all steps is left out
template <class T> __global__ __launch_bounds__(THREADS) void steps_kernel(PickArgs a)
{
    const int r = blockIdx.x / a.groups, group = blockIdx.x % a.groups;
    const PickSearch q = a.search[r];
    if (q.stage != PICK_STEP) return;
    __shared__ u64 step[PICK_STEPS];
    static_assert(PICK_STEPS == THREADS);
    step[threadIdx.x] = 0;
    const Row row = searched_row(a, r, q);
    using P = Part<T>;
    P p;
    p.load((const T *)a.logits + (long long)r * a.stride, a.vocab, ((long long)group * WAVES + threadIdx.x / 64) * PICK_PART, P::BLOCK);
    __syncthreads();
    u64 above = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const float z = p.z[e];
        const int at = z >= q.from ? -1 : step_of(z, q);
        if (z == -INFINITY || at >= PICK_STEPS - 1) continue;
        const u64 m = row.mass(key_of(z));
        if (at < 0) above += m;
        else atomicAdd(&step[at], m);
    }
    above = wave_all(above, [](u64 x, u64 y) { return x + y; });
    if (threadIdx.x % 64 == 0) atomicAdd(&step[PICK_STEPS - 1], above);
    __syncthreads();
    a.steps[((long long)r * a.groups + group) * PICK_STEPS + threadIdx.x] = step[threadIdx.x];
}

// The step that top-p ends in; of each part the mass of what is above it and its tokens in it. Where min-p alone decides, the mass of what it keeps.
template <class T> __global__ __launch_bounds__(THREADS) void place_kernel(PickArgs a)
{
    __shared__ u64 s_part[WAVES];
    __shared__ int s_step;
    const int r = blockIdx.x / a.groups, group = blockIdx.x % a.groups, lane = threadIdx.x % 64, wave = threadIdx.x / 64, parts = a.groups * WAVES, part = group * WAVES + wave;
    const PickSearch q = a.search[r];
    if (q.stage == PICK_DONE) return;
    const Row row = searched_row(a, r, q);
    using P = Part<T>;
    P p;
    p.load((const T *)a.logits + (long long)r * a.stride, a.vocab, (long long)part * PICK_PART, P::BLOCK);
    int step = PICK_STEPS;                    // none
    uint32_t stage = q.stage;
    if (stage == PICK_STEP) {
        u64 sum = 0;
        for (int g = 0; g < a.groups; ++g) sum += a.steps[((long long)r * a.groups + g) * PICK_STEPS + threadIdx.x];
        // (what is above all steps, which the last place holds, comes before them)
        u64 upto = threadIdx.x == PICK_STEPS - 1 ? 0 : sum;
        for (int o = 1; o < 64; o *= 2) {
            const u64 v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        if (threadIdx.x == 0) s_step = PICK_STEPS;
        if (lane == 63) s_part[wave] = wave == WAVES - 1 ? sum : upto;
        __syncthreads();
        u64 before = s_part[WAVES - 1];
        for (int w = 0; w < wave; ++w) before += s_part[w];
        upto += before;
        if (threadIdx.x < PICK_STEPS - 1 && upto - sum < q.want && q.want <= upto) s_step = threadIdx.x;
        __syncthreads();
        step = s_step;
        if (step == PICK_STEPS) stage = PICK_WHOLE;
        else if (q.least && step_of(logit_of(q.least), q) < step) stage = PICK_LEAST;
    }
    if (group == 0 && threadIdx.x == 0) { a.search[r].found = stage; }
    if (stage == PICK_WHOLE) return;
    PickHead head{};
    const float least = stage == PICK_LEAST ? logit_of(q.least) : q.from;
    u64 mass = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const float z = p.z[e];
        if (z >= least || (stage == PICK_STEP && z > -INFINITY && step_of(z, q) < step)) mass += row.mass(key_of(z));
    }
    head.mass = wave_all(mass, [](u64 x, u64 y) { return x + y; });
    if (stage == PICK_STEP) head.count = p.list([&](int e) { return p.z[e] > -INFINITY && p.z[e] < q.from && step_of(p.z[e], q) == step; }, a.listed, a.list + ((long long)r * parts + part) * a.listed);
    if (lane == 0) a.head[(long long)r * parts + part] = head;
}

// The place in the step, and the draw: the part by the parts' masses, then the token in it
template <class T> __global__ __launch_bounds__(THREADS) void finish_kernel(PickArgs a)
{
    __shared__ Shared s;
    const int r = blockIdx.x, vocab = a.vocab, parts = a.groups * WAVES;
    const PickSearch q = a.search[r];
    if (q.stage == PICK_DONE) return;
    const T *const logits = (const T *)a.logits + (long long)r * a.stride;
    const Row row = searched_row(a, r, q);
    const auto plus = [](u64 x, u64 y) { return x + y; };
    bool whole = q.found == PICK_WHOLE;
    u64 above = 0;
    if (!whole) {
        u64 over = 0;
        for (int w = threadIdx.x; w < MAX_PARTS; w += THREADS) {
            PickHead head{};
            if (w < parts) head = a.head[(long long)r * parts + w];
            s.mass[w] = head.mass;
            s.listed[w] = (uint16_t)head.count;
            above += head.mass;
            over += head.count > (uint32_t)a.listed;
        }
        whole = all_of(over, plus, s) != 0;
        above = all_of(above, plus, s);
    }
    if (whole) {
        Streamed<T> all{logits, vocab, row};
        draw(all, a, r, logits, row, 0.0, s);
        return;
    }
    Kept kept{q.least, ANY};
    if (q.found == PICK_STEP) {
        Held held;
        held.from = LOWEST;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const uint32_t i = e * THREADS + threadIdx.x, w = __umulhi(i, a.listed_inverse), j = i - w * a.listed;
            uint2 v = make_uint2(0, 0);
            if (w < (uint32_t)parts && j < s.listed[w]) v = a.list[((long long)r * parts + w) * a.listed + j];
            held.key[e] = v.x; held.id[e] = v.y;
        }
        held.weigh(row, LOWEST);
        const Border b = find_border([&](auto add) { held.each([&](uint32_t key, uint32_t, auto m) { add(q.top_key - key, m()); }); }, bits_of(q.top_key - LOWEST), q.want - above, s);
        kept.key = q.top_key - b.place;
        const u64 one = row.mass(kept.key), need = (q.want - above - b.before + one - 1) / one;
        u64 ties = need < b.at / one ? need : 0;
        if (q.least > kept.key) { kept.key = q.least; ties = 0; }
        if (ties) kept.last = find_border([&](auto add) { held.each([&](uint32_t key, uint32_t id, auto) { if (key == kept.key) add(id, 1); }); }, bits_of(vocab - 1), ties, s).place;
        __syncthreads();
        held.each([&](uint32_t key, uint32_t id, auto m) { if (kept.has(key, id)) atomicAdd(&s.mass[id / PICK_PART], m()); });
        __syncthreads();
    }
    static_assert(MAX_PARTS == 2 * THREADS && PICK_PART == 2 * THREADS);
    u64 v[2] = {s.mass[threadIdx.x * 2], s.mass[threadIdx.x * 2 + 1]}, total, rest;
    u64 upto = sum_upto(v[0] + v[1], total, s), run = upto - v[0] - v[1];
    const u64 below = min((u64)(evenly(a.u[r]) * (double)total), total - 1);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (run <= below && below < run + v[e]) { s.place = threadIdx.x * 2 + e; s.before = run; }
        run += v[e];
    }
    __syncthreads();
    const uint32_t first = s.place * PICK_PART;
    const u64 left = below - s.before;
    float z[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t id = first + threadIdx.x * 2 + e;
        z[e] = id < (uint32_t)vocab ? wide(logits[id]) : -INFINITY;
        const uint32_t key = key_of(z[e]);
        v[e] = key && kept.has(key, id) ? row.mass(key) : 0;
    }
    run = sum_upto(v[0] + v[1], rest, s) - v[0] - v[1];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (run <= left && left < run + v[e]) put_draw(a, r, row, first + threadIdx.x * 2 + e, z[e], (double)total / row.unit);
        run += v[e];
    }
}

template <class T, bool TOP> void launch(hipStream_t s, const PickArgs &a)
{
    const dim3 rows(a.rows), all((unsigned)a.rows * a.groups), threads(THREADS);
    if (a.groups == 1) {
        hipLaunchKernelGGL((decide_kernel<T, TOP, true>), rows, threads, 0, s, a);
        return;
    }
    hipLaunchKernelGGL((parts_kernel<T, TOP>), all, threads, 0, s, a);
    hipLaunchKernelGGL((decide_kernel<T, TOP, false>), rows, threads, 0, s, a);
    if constexpr (!TOP) {
        if (!a.searched) return;
        hipLaunchKernelGGL(steps_kernel<T>, all, threads, 0, s, a);
        hipLaunchKernelGGL(place_kernel<T>, all, threads, 0, s, a);
        hipLaunchKernelGGL(finish_kernel<T>, rows, threads, 0, s, a);
    }
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
