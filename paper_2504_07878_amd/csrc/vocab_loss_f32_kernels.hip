// Products of the losses over the vocabulary on 32-bit matrix instructions: fp32 rows and head, and the gradients of fp32 rows over a bf16 head, widened where it is read; any stride and
// alignment. (The softmax and the probabilities of fp32 rows over a bf16 head have faster ones, on three bf16 rows for each.)
//
// A workgroup of 4 wavefronts (2 x 2, an accumulator of 32 x 32 each) computes a 64 x 64 block of C[n][m] = sum_k A[m][k] B[n][k] in steps of 32 k: both operands
// go through registers into LDS as [row][k], two steps ahead, in two buffers. A lane reads four k at a time: k = 8 g + 4 (lane / 32) + j for the j-th product of group g.
// Small blocks, since models of this type are small: they have to fill the chip. Bound by latency there: 133 of 190 rows x 4096 x 256 take 11 us for the softmax, 16 us for
// both gradients (5 us for a single step; blocks of 128 x 128, 16 k a step, in one buffer, the gradients apart: 52, 40 and 33; one step ahead, and loads that waited for each
// other: 21, 13 and 11, 19 of the first for the listed entries). 1024 rows x 32768 x 896: 97 TFLOP/s (a library product 112 to 141). Three products:
//   softmax, probabilities: m = vocabulary entry, n = row that counts, k = feature
//   gradient to the hidden rows: m = feature, n = row, k = vocabulary entry of the piece; summed over the pieces in `acc`, one sum per split of k
//   gradient to the head: m = feature, n = vocabulary entry, k = row
#include "vocab_loss_epilogues.h"
#include <algorithm>
#include <type_traits>

namespace tr {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
constexpr int BK = 32, PITCH = BK + 4;       // 16-byte reads of 16 rows meet 16 different places of the 64 banks

// Loads of 16 bytes from any element on (global loads need no alignment here): lines of odd length need them (probabilities and gradients of 58 rows x 10911 x 1397 over a bf16 head,
// both on these instructions: element by element, under conditions, 252 us, so 121, 67 of it the gradients; with 1400 features 97).
typedef f32x4 __attribute__((aligned(2))) loose16;

// four elements of a line from p on, as fp32
__device__ __forceinline__ void four_of(const float *p, float (&v)[4])
{
    const f32x4 x = *reinterpret_cast<const loose16 *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
}
// N from j on, zeros at or past `limit`: elements one by one, under no condition, which would have each load wait for the one before
template <int N, class T> __device__ __forceinline__ void some_of(const T *line, int j, int limit, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = load_one(line + min(j + e, limit - 1));
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = j + e < limit ? v[e] : 0.f;
}

// An operand is lines of memory: line o, o < lines, has elements 0 .. limit - 1 from p + o * ld on, with a list from p + list[o] * ld. ALONG_K: a line is a row of the
// operand (k runs along it); otherwise it is one k.
template <class T, bool LISTED = false> struct Lines {
    const T *p; long long ld; int lines, limit; const int *list;
    __device__ __forceinline__ Lines(const void *p_, long long ld_, int lines_, int limit_, const int *list_ = nullptr) : p((const T *)p_), ld(ld_), lines(lines_), limit(limit_), list(list_) {}
    __device__ __forceinline__ int place(int o) const { return LISTED ? list[min(o, lines - 1)] : min(o, lines - 1); }    // of line o, or of the last
};

struct alignas(16) Tiles { float a[2][F32_BLOCK * PITCH], b[2][F32_BLOCK * PITCH]; };

// How an operand's eight elements in a run are read: where lines are multiples of eight long, they are there or not together; otherwise the last ones of a line are read from where
// eight are left, and moved down; lines shorter than eight element by element.
enum { EIGHTS, MOVED, SINGLES };

// A thread's eight elements of the tiles (64 x 32) from row0 on, step after step from k0 on: of a row, or of a k (whose place is read a step ahead); zeros where there
// is nothing. Read as they are, under no condition, from the nearest place that is there, and widened when they are used: until then nothing waits for them.
template <bool ALONG_K, int HOW, class Op> struct Steps {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(Op::p)>>;
    static constexpr bool RAW = sizeof(T) == 2 && HOW != SINGLES;
    struct Read { f32x4 u[RAW ? 1 : 2]; int down; };     // down: places to move by, 8: nothing is there
    const Op &op;
    int place, line, along;
    __device__ __forceinline__ Steps(const Op &op_, int row0, int k0) : op(op_)
    {
        const int t = threadIdx.x;
        line = ALONG_K ? row0 + (t >> 2) : k0 + (t >> 3);
        along = ALONG_K ? k0 + (t & 3) * 8 : row0 + (t & 7) * 8;
        place = op.place(line);
    }
    __device__ __forceinline__ void next(Read &r)
    {
        const T *at = op.p + place * op.ld;
        if constexpr (HOW == SINGLES) {
            float v[8];
            some_of(at, along, op.limit, v);
            r.u[0] = f32x4{v[0], v[1], v[2], v[3]};
            r.u[1] = f32x4{v[4], v[5], v[6], v[7]};
            r.down = line < op.lines ? 0 : 8;
        } else {
            const int from = min(along, op.limit - 8);
            r.u[0] = *reinterpret_cast<const loose16 *>(at + from);
            if constexpr (!RAW) r.u[1] = *reinterpret_cast<const loose16 *>(at + from + 4);
            r.down = line < op.lines ? along - from : 8;
        }
        if (ALONG_K) along += BK;
        else { line += BK; place = op.place(line); }
    }
    static __device__ __forceinline__ void values(const Read &r, float (&v)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (!RAW) v[e] = r.u[e >> 2][e & 3];
            else v[e] = __uint_as_float(e & 1 ? __float_as_uint(r.u[0][e >> 1]) & 0xffff0000u : __float_as_uint(r.u[0][e >> 1]) << 16);
            v[e] = r.down < 8 ? v[e] : 0.f;
        }
        if constexpr (HOW == MOVED) {
#pragma unroll
            for (int by = 4; by; by >>= 1)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = !(r.down & by) ? v[e] : e + by < 8 ? v[e + by < 8 ? e + by : e] : 0.f;
        }
    }
    static __device__ __forceinline__ void write(float *lds, const Read &r)
    {
        float v[8];
        values(r, v);
        const int t = threadIdx.x;
        if (ALONG_K) {
            f32x4 *to = reinterpret_cast<f32x4 *>(lds + (t >> 2) * PITCH + (t & 3) * 8);
            to[0] = f32x4{v[0], v[1], v[2], v[3]};
            to[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[((t & 7) * 8 + e) * PITCH + (t >> 3)] = v[e];
        }
    }
};
// own LDS accesses are done, then the workgroup's barrier; loads may be under way
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));   // lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
template <bool A_ALONG, bool B_ALONG, int HOW, class A, class B>
__device__ __forceinline__ void products_of(const A &a, const B &b, int m0, int n0, int k_lo, int k_hi, Tiles &sm, f32x16 (&c)[1][1])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int arow = (w >> 1) * 32 + tile_feature(lane & 31), brow = (w & 1) * 32 + (lane & 31), at = (lane >> 5) * 4;
    Steps<A_ALONG, HOW, A> from_a(a, m0, k_lo);
    Steps<B_ALONG, HOW, B> from_b(b, n0, k_lo);
    typename Steps<A_ALONG, HOW, A>::Read ra[2];
    typename Steps<B_ALONG, HOW, B>::Read rb[2];
    from_a.next(ra[0]); from_b.next(rb[0]);
    from_a.next(ra[1]); from_b.next(rb[1]);
    const auto step = [&](auto buffer) {
        constexpr int buf = decltype(buffer)::value;
        from_a.write(sm.a[buf], ra[buf]);
        from_b.write(sm.b[buf], rb[buf]);
        lds_barrier();          // (the other buffer's readers are past it when it is written again)
        from_a.next(ra[buf]); from_b.next(rb[buf]);     // (past the end: for nobody)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < BK; g += 8) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(sm.a[buf] + arow * PITCH + g + at), y = *reinterpret_cast<const f32x4 *>(sm.b[buf] + brow * PITCH + g + at);
#pragma unroll
            for (int q = 0; q < 4; ++q) c[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[q], y[q], c[0][0], 0, 0, 0);
        }
    };
    for (int k = k_lo;; k += 2 * BK) {
        step(std::integral_constant<int, 0>{});
        if (k + BK >= k_hi) break;
        step(std::integral_constant<int, 1>{});
        if (k + 2 * BK >= k_hi) break;
    }
}

// c = this wavefront's products of the block at (m0, n0) over k in [k_lo, k_hi), whole steps unless k_hi is the operands' end
template <bool A_ALONG, bool B_ALONG, class A, class B>
__device__ __forceinline__ void products(const A &a, const B &b, int m0, int n0, int k_lo, int k_hi, Tiles &sm, f32x16 (&c)[1][1])
{
#pragma unroll
    for (int r = 0; r < 16; ++r) c[0][0][r] = 0.f;
    if (k_lo >= k_hi) return;
    if (((a.limit | b.limit) & 7) == 0) products_of<A_ALONG, B_ALONG, EIGHTS>(a, b, m0, n0, k_lo, k_hi, sm, c);
    else if (min(a.limit, b.limit) >= 8) products_of<A_ALONG, B_ALONG, MOVED>(a, b, m0, n0, k_lo, k_hi, sm, c);
    else products_of<A_ALONG, B_ALONG, SINGLES>(a, b, m0, n0, k_lo, k_hi, sm, c);
}

// f(n, first m of a run of 8, the run) for every run of the block
template <class F> __device__ __forceinline__ void each_run(const f32x16 (&c)[1][1], F f)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float v[8];
        run_of(c[0][0], h, v);
        f((w & 1) * 32 + (lane & 31), (w >> 1) * 32 + 16 * h + 8 * (lane >> 5), v);
    }
}

// Products of listed entries: a wavefront takes 32 of them, its rows of the head against its hidden rows, of which only the diagonal is kept (the matrix unit
// is all but idle in a product this small, and it gives the bits that the same pair has in a block: the same instructions over the same steps of k).
__device__ __forceinline__ void entries_group(const LossArgs &a, int group)
{
    const int lane = threadIdx.x & 63, e = group * 32 + (lane & 31), hf = lane >> 5, count = a.head->count;
    if ((long long)group * 32 >= (long long)count * a.entries) return;
    const int i = e / a.entries, j = e - i * a.entries;
    bool on = i < count;
    const float *h = (const float *)a.hidden;         // (a lane without an entry reads what is there, for nobody)
    const float *w = (const float *)a.weight;
    if (on) {
        const int r = a.idx[i], id = a.ids[(long long)r * a.entries + j];
        h += r * a.hs;
        on = id >= 0 && id < a.vocab;
        if (on) w += id * a.ws;
    }
    f32x16 c;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
    constexpr int AT_ONCE = 16;      // groups of 8 k whose loads are requested together
    float x[AT_ONCE][4], y[AT_ONCE][4];
    const auto multiply = [&](int g) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[g][q], y[g][q], c, 0, 0, 0);
    };
    int k0 = 0;
    for (; k0 + 8 * AT_ONCE <= a.dim; k0 += 8 * AT_ONCE) {
#pragma unroll
        for (int g = 0; g < AT_ONCE; ++g) { four_of(w + k0 + 8 * g + 4 * hf, x[g]); four_of(h + k0 + 8 * g + 4 * hf, y[g]); }
#pragma unroll
        for (int g = 0; g < AT_ONCE; ++g) multiply(g);
    }
    for (; k0 + 8 <= a.dim; k0 += 8) {
        four_of(w + k0 + 4 * hf, x[0]);
        four_of(h + k0 + 4 * hf, y[0]);
        multiply(0);
    }
    if (k0 < a.dim) {
        some_of(w, k0 + 4 * hf, a.dim, x[0]);
        some_of(h, k0 + 4 * hf, a.dim, y[0]);
        multiply(0);
    }
    // row m of column n lies in register (m / 8) * 4 + m % 4 of lane n + 32 * (m / 4 % 2)
    const int n = lane & 31;
    float d = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d = (n >> 3) * 4 + (n & 3) == r ? c[r] : d;
    if (on && ((n >> 2) & 1) == hf) a.value[e] = d;
}

// The first `extra` workgroups of the grid's rows take listed entries, as long as there are any.
__device__ __forceinline__ void entries_of(const LossArgs &a, int extra) { entries_group(a, (blockIdx.y * extra + blockIdx.x) * 4 + (threadIdx.x >> 6)); }

__global__ __launch_bounds__(256) void f32_softmax_kernel(LossArgs a, int extra)
{
    __shared__ Tiles sm;
    const int m0 = ((int)blockIdx.x - extra) * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count, w = threadIdx.x >> 6;
    if (m0 < 0) {
        entries_of(a, extra);
        return;
    }
    if (n0 >= count) return;
    const Lines<float> A(a.weight, a.ws, a.vocab, a.dim);
    const Lines<float, true> B(a.hidden, a.hs, count, a.dim, a.idx);
    f32x16 c[1][1];
    products<true, true>(A, B, m0, n0, 0, a.dim, sm, c);
    const int lane = threadIdx.x & 63, m = m0 + (w >> 1) * 32 + 8 * (lane >> 5);
    const float2 t = column_softmax<16>([&](int i) { return c[0][0][i]; }, [](int i) { return 16 * (i >> 3) + (i & 7); }, a.vocab - m, LOG2E / a.temperature, 32);
    if (lane < 32) a.part[((size_t)(m0 / F32_BLOCK) * 2 + (w >> 1)) * a.part_ld + n0 + (w & 1) * 32 + lane] = t;
}

__global__ __launch_bounds__(256) void f32_probabilities_kernel(LossArgs a, int v0, int vn, int extra)
{
    __shared__ Tiles sm;
    const int m0 = ((int)blockIdx.x - extra) * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    if (m0 < 0) {
        entries_of(a, extra);
        return;
    }
    if (n0 >= count) return;
    const Lines<float> A((const float *)a.weight + (long long)v0 * a.ws, a.ws, vn, a.dim);
    const Lines<float, true> B(a.hidden, a.hs, count, a.dim, a.idx);
    f32x16 c[1][1];
    products<true, true>(A, B, m0, n0, 0, a.dim, sm, c);
    const float k = 1.0f / a.temperature;
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (n >= count) return;
        const float lse = a.lse[a.idx[n]], weight = a.grad[a.idx[n]] / a.head->scale;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = m + e < vn ? weight * expf(fmaf(v[e], k, -lse)) : 0.f;
        const unsigned own = a.teacher ? ~0u : (unsigned)(a.ids[a.idx[n]] - v0 - m);
        if (own < 8) {
            const float own_x = less_one([&](int e) { return v[e]; }, own, weight, lse);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = own == e ? own_x : x[e];
        }
        store_run((float *)a.G + (size_t)n * a.g_ld + m, x);
    });
}

// split: of the piece's vocabulary, its sums in acc[split]
template <class WT> __device__ __forceinline__ void hidden_grad(const LossArgs &a, int v0, int vn, int per, int first, int m0, int n0, int split, Tiles &sm)
{
    const int count = a.head->count;
    if (n0 >= count) return;
    const Lines<WT> A((const WT *)a.weight + (long long)v0 * a.ws, a.ws, vn, a.dim);
    const Lines<float> B(a.G, a.g_ld, count, (vn + 7) & ~7);      // (G is zero from vn on to the end of a block)
    f32x16 c[1][1];
    products<false, true>(A, B, m0, n0, min(vn, split * per), min(vn, (split + 1) * per), sm, c);
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (m >= a.d_pad) return;
        float *to = a.acc + ((size_t)split * a.n_pad + n) * a.d_pad + m;
        if (!first) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += to[e];
        }
        store_run(to, v);
    });
}

template <class WT> __device__ __forceinline__ void weight_grad(const LossArgs &a, int v0, int vn, int m0, int n0, Tiles &sm)
{
    const int count = a.head->count;
    const Lines<float, true> A(a.hidden, a.hs, count, a.dim, a.idx);
    const Lines<float> B(a.G, a.g_ld, count, (vn + 7) & ~7);      // (G is zero from vn on to the end of a block)
    f32x16 c[1][1];
    products<false, false>(A, B, m0, n0, 0, count, sm, c);
    const float k = a.head->scale * a.temperature;
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (n >= vn) return;
        WT *to = (WT *)a.d_weight + (long long)(v0 + n) * a.dws + m;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= k;
        if (m + 8 <= a.dim) store_run(to, v);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (m + e < a.dim) store_one(to + e, v[e]);
        }
    });
}

// Both gradients of a piece in one launch: the first `hidden` workgroups (mb x nb blocks of every split) take the rows', the others the head's. Small models' launches are short
// and wait for each other (133 of 190 rows x 4096 x 256: 12 and 10 us apart, 16 together).
template <class WT> __global__ __launch_bounds__(256) void f32_gradients_kernel(LossArgs a, int v0, int vn, int per, int first, int hidden, int mb, int nb)
{
    __shared__ Tiles sm;
    const int b = blockIdx.x;
    if (b < hidden) hidden_grad<WT>(a, v0, vn, per, first, b % mb * F32_BLOCK, b / mb % nb * F32_BLOCK, b / (mb * nb), sm);
    else weight_grad<WT>(a, v0, vn, (b - hidden) % mb * F32_BLOCK, (b - hidden) / mb * F32_BLOCK, sm);
}

int blocks(int n) { return (n + F32_BLOCK - 1) / F32_BLOCK; }
// Workgroups for listed entries in each row of a grid `across` blocks wide. The first rows' take them, those of the others end at once: no more than blocks, or 64, unless it takes more.
int entry_blocks(const LossArgs &a, int across)
{
    const int all = (int)(((long long)a.rows * a.entries + 127) / 128), rows = blocks(a.rows);
    return std::max((all + rows - 1) / rows, std::min(all, std::max(64, across)));
}

template <class Go> void by_head(const LossArgs &a, Go go)
{
    if (a.wdt == DT_BF16) go(bf16_t{});
    else go(float{});
}

}  // namespace

void launch_f32_softmax(hipStream_t s, const LossArgs &a)
{
    const int extra = entry_blocks(a, blocks(a.vocab));
    hipLaunchKernelGGL(f32_softmax_kernel, dim3(extra + blocks(a.vocab), blocks(a.rows)), dim3(256), 0, s, a, extra);
}

int f32_softmax_parts(const LossArgs &a) { return blocks(a.vocab) * 2; }

void launch_f32_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    const int extra = v0 == 0 && a.teacher ? entry_blocks(a, blocks(vn)) : 0;
    hipLaunchKernelGGL(f32_probabilities_kernel, dim3(extra + blocks(vn), blocks(a.rows)), dim3(256), 0, s, a, v0, vn, extra);
}

void launch_f32_gradients(hipStream_t s, const LossArgs &a, int v0, int vn, bool first)
{
    by_head(a, [&](auto wt) {
        const int per = ((vn + a.splits - 1) / a.splits + BK - 1) / BK * BK;   // whole steps
        const int mb = blocks(a.dim), nb = blocks(a.rows), hidden = a.d_hidden && a.rows ? mb * nb * a.splits : 0;
        const int all = hidden + (a.d_weight ? mb * blocks(vn) : 0);
        if (all) hipLaunchKernelGGL((f32_gradients_kernel<decltype(wt)>), dim3(all), dim3(256), 0, s, a, v0, vn, per, (int)first, hidden, mb, nb);
    });
}

}  // namespace tr
