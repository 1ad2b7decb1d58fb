// Products of the losses over the vocabulary on 32-bit matrix instructions: fp32 rows and a head of either type, any stride and alignment, widened where they
// are read. (The softmax of fp32 rows over a bf16 head has faster ones, on three bf16 rows for each.)
//
// A workgroup of 4 wavefronts (2 x 2, an accumulator of 32 x 32 each) computes a 64 x 64 block of C[n][m] = sum_k A[m][k] B[n][k] in steps of 32 k: both operands
// go through registers into LDS as [row][k], one step ahead, in two buffers. A lane reads four k at a time: k = 8 g + 4 (lane / 32) + j for the j-th product of group g.
// Small blocks, since models of this type are small: they have to fill the chip. Bound by latency there: 133 of 190 rows x 4096 x 256 take 21 us for the softmax, 13 and 11 us for
// the gradients (blocks of 128 x 128, 16 k a step, in one buffer: 52, 40 and 33). Three products:
//   softmax, probabilities: m = vocabulary entry, n = row that counts, k = feature
//   gradient to the hidden rows: m = feature, n = row, k = vocabulary entry of the piece; summed over the pieces in `acc`, one sum per split of k
//   gradient to the head: m = feature, n = vocabulary entry, k = row
#include "vocab_loss_epilogues.h"

namespace tr {

namespace {

constexpr int BK = 32, PITCH = BK + 4;       // 16-byte reads of 16 rows meet 16 different places of the 64 banks

// eight elements of a line from j on, as fp32; zeros at or past `limit` and where there is no line. `wide`: the line lies on 16 bytes
__device__ __forceinline__ void eight_of(const float *line, int j, int limit, bool wide, float (&v)[8])
{
    if (line && wide && j + 8 <= limit) {
        const float4 x = *reinterpret_cast<const float4 *>(line + j), y = *reinterpret_cast<const float4 *>(line + j + 4);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = line && j + e < limit ? line[j + e] : 0.f;
    }
}
__device__ __forceinline__ void eight_of(const bf16_t *line, int j, int limit, bool, float (&v)[8])
{
    const uint4 u = line ? load8(line, j, limit) : make_uint4(0, 0, 0, 0);
    const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(q[e] << 16); v[2 * e + 1] = __uint_as_float(q[e] & 0xffff0000u); }
}

template <class T> __device__ __forceinline__ void four_of(const T *line, int j, int limit, bool wide, float (&v)[4])
{
    if (line && wide && j + 4 <= limit) {
        if constexpr (sizeof(T) == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(line + j);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2 *>(line + j);
            v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u); v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = line && j + e < limit ? load_one(line + j + e) : 0.f;
    }
}

// An operand is lines of memory: line o has elements 0 .. limit - 1. ALONG_K: a line is a row of the operand (k runs along it); otherwise it is one k.
template <class T> struct Lines {              // line o at p + o * ld, o < lines
    const T *p; long long ld; int lines, limit; bool wide;
    __device__ __forceinline__ Lines(const void *p_, long long ld_, int lines_, int limit_) : p((const T *)p_), ld(ld_), lines(lines_), limit(limit_)
    {
        wide = ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * sizeof(T))) & 15) == 0;
    }
    __device__ __forceinline__ void read(int o, int j, float (&v)[8]) const { eight_of(o < lines ? p + o * ld : nullptr, j, limit, wide, v); }
};
template <class T> struct ListedLines {        // line o at p + list[o] * ld
    Lines<T> l; const int *list;
    __device__ __forceinline__ void read(int o, int j, float (&v)[8]) const { eight_of(o < l.lines ? l.p + list[o] * l.ld : nullptr, j, l.limit, l.wide, v); }
};

struct Tiles { float a[2][F32_BLOCK * PITCH], b[2][F32_BLOCK * PITCH]; };

// a thread's eight elements of a tile (64 x 32): of a row, or of a k
template <bool ALONG_K, class Op> __device__ __forceinline__ void read_tile(const Op &op, int row0, int k0, float (&v)[8])
{
    const int t = threadIdx.x;
    if (ALONG_K) op.read(row0 + (t >> 2), k0 + (t & 3) * 8, v);
    else op.read(k0 + (t >> 3), row0 + (t & 7) * 8, v);
}
template <bool ALONG_K> __device__ __forceinline__ void write_tile(float *lds, const float (&v)[8])
{
    const int t = threadIdx.x;
    if (ALONG_K) store_run(lds + (t >> 2) * PITCH + (t & 3) * 8, v);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) lds[((t & 7) * 8 + e) * PITCH + (t >> 3)] = v[e];
    }
}

// c = this wavefront's products of the block at (m0, n0) over k in [k_lo, k_hi), whole steps unless k_hi is the operands' end
template <bool A_ALONG, bool B_ALONG, class A, class B>
__device__ __forceinline__ void products(const A &a, const B &b, int m0, int n0, int k_lo, int k_hi, Tiles &sm, f32x16 (&c)[1][1])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int arow = (w >> 1) * 32 + tile_feature(lane & 31), brow = (w & 1) * 32 + (lane & 31), at = (lane >> 5) * 4;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[0][0][r] = 0.f;
    if (k_lo >= k_hi) return;
    float va[8], vb[8];
    read_tile<A_ALONG>(a, m0, k_lo, va);
    read_tile<B_ALONG>(b, n0, k_lo, vb);
    int buf = 0;
    for (int k = k_lo; k < k_hi; k += BK, buf ^= 1) {
        write_tile<A_ALONG>(sm.a[buf], va);
        write_tile<B_ALONG>(sm.b[buf], vb);
        __syncthreads();        // (the other buffer's readers are past it when it is written again)
        if (k + BK < k_hi) { read_tile<A_ALONG>(a, m0, k + BK, va); read_tile<B_ALONG>(b, n0, k + BK, vb); }
#pragma unroll
        for (int g = 0; g < BK; g += 8) {
            const float4 x = *reinterpret_cast<const float4 *>(sm.a[buf] + arow * PITCH + g + at), y = *reinterpret_cast<const float4 *>(sm.b[buf] + brow * PITCH + g + at);
            c[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, y.x, c[0][0], 0, 0, 0);
            c[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, y.y, c[0][0], 0, 0, 0);
            c[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, y.z, c[0][0], 0, 0, 0);
            c[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, y.w, c[0][0], 0, 0, 0);
        }
    }
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
template <class WT> __device__ __forceinline__ void entries_group(const LossArgs &a, int group)
{
    const int lane = threadIdx.x & 63, e = group * 32 + (lane & 31), hf = lane >> 5, count = a.head->count;
    if ((long long)group * 32 >= (long long)count * a.entries) return;
    const int i = e / a.entries, j = e - i * a.entries;
    const float *h = nullptr;
    const WT *w = nullptr;
    if (i < count) {
        const int r = a.idx[i], id = a.ids[(long long)r * a.entries + j];
        if (id >= 0 && id < a.vocab) { h = (const float *)a.hidden + r * a.hs; w = (const WT *)a.weight + id * a.ws; }
    }
    const bool hw = ((reinterpret_cast<uintptr_t>(a.hidden) | (uintptr_t)(a.hs * 4)) & 15) == 0, ww = ((reinterpret_cast<uintptr_t>(a.weight) | (uintptr_t)(a.ws * sizeof(WT))) & 15) == 0;
    f32x16 c;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
    constexpr int AT_ONCE = 8;       // groups of 8 k whose loads are requested together
    for (int k0 = 0; k0 < a.dim; k0 += 8 * AT_ONCE) {
        float x[AT_ONCE][4], y[AT_ONCE][4];
#pragma unroll
        for (int g = 0; g < AT_ONCE; ++g) { four_of(w, k0 + 8 * g + 4 * hf, a.dim, ww, x[g]); four_of(h, k0 + 8 * g + 4 * hf, a.dim, hw, y[g]); }
#pragma unroll
        for (int g = 0; g < AT_ONCE; ++g)
            if (k0 + 8 * g < a.dim) {
#pragma unroll
                for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[g][q], y[g][q], c, 0, 0, 0);
            }
    }
    // row m of column n lies in register (m / 8) * 4 + m % 4 of lane n + 32 * (m / 4 % 2)
    const int n = lane & 31;
    float d = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d = (n >> 3) * 4 + (n & 3) == r ? c[r] : d;
    if (w && ((n >> 2) & 1) == hf) a.value[e] = d;
}

// The first `extra` workgroups along x, of the first row of them, take listed entries.
__global__ __launch_bounds__(256) void f32_softmax_kernel(LossArgs a, int extra)
{
    __shared__ Tiles sm;
    const int m0 = ((int)blockIdx.x - extra) * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count, w = threadIdx.x >> 6;
    if (m0 < 0) {
        if (n0 == 0) entries_group<float>(a, blockIdx.x * 4 + w);
        return;
    }
    if (n0 >= count) return;
    const Lines<float> A(a.weight, a.ws, a.vocab, a.dim);
    const ListedLines<float> B{Lines<float>(a.hidden, a.hs, count, a.dim), a.idx};
    f32x16 c[1][1];
    products<true, true>(A, B, m0, n0, 0, a.dim, sm, c);
    const int lane = threadIdx.x & 63, m = m0 + (w >> 1) * 32 + 8 * (lane >> 5);
    const float2 t = column_softmax<16>([&](int i) { return c[0][0][i]; }, [](int i) { return 16 * (i >> 3) + (i & 7); }, a.vocab - m, LOG2E / a.temperature, 32);
    if (lane < 32) a.part[((size_t)(m0 / F32_BLOCK) * 2 + (w >> 1)) * a.part_ld + n0 + (w & 1) * 32 + lane] = t;
}

template <class WT> __global__ __launch_bounds__(256) void f32_probabilities_kernel(LossArgs a, int v0, int vn, int extra)
{
    __shared__ Tiles sm;
    const int m0 = ((int)blockIdx.x - extra) * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    if (m0 < 0) {
        if (n0 == 0) entries_group<WT>(a, blockIdx.x * 4 + (threadIdx.x >> 6));
        return;
    }
    if (n0 >= count) return;
    const Lines<WT> A((const WT *)a.weight + (long long)v0 * a.ws, a.ws, vn, a.dim);
    const ListedLines<float> B{Lines<float>(a.hidden, a.hs, count, a.dim), a.idx};
    f32x16 c[1][1];
    products<true, true>(A, B, m0, n0, 0, a.dim, sm, c);
    const float k = 1.0f / a.temperature;
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (n >= count) return;
        const float lse = a.lse[a.idx[n]], weight = a.grad[a.idx[n]] / a.head->scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = m + e < vn ? weight * expf(fmaf(v[e], k, -lse)) : 0.f;
        store_run((float *)a.G + (size_t)n * a.g_ld + m, v);
    });
}

// blockIdx.z: split of the piece's vocabulary, its sums in acc[split]
template <class WT> __global__ __launch_bounds__(256) void f32_hidden_grad_kernel(LossArgs a, int v0, int vn, int per, int first)
{
    __shared__ Tiles sm;
    const int m0 = blockIdx.x * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    if (n0 >= count) return;
    const Lines<WT> A((const WT *)a.weight + (long long)v0 * a.ws, a.ws, vn, a.dim);
    const Lines<float> B(a.G, a.g_ld, count, vn);
    f32x16 c[1][1];
    products<false, true>(A, B, m0, n0, min(vn, (int)blockIdx.z * per), min(vn, ((int)blockIdx.z + 1) * per), sm, c);
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (m >= a.d_pad) return;
        float *to = a.acc + ((size_t)blockIdx.z * a.n_pad + n) * a.d_pad + m;
        if (!first) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += to[e];
        }
        store_run(to, v);
    });
}

template <class WT> __global__ __launch_bounds__(256) void f32_weight_grad_kernel(LossArgs a, int v0, int vn)
{
    __shared__ Tiles sm;
    const int m0 = blockIdx.x * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    const ListedLines<float> A{Lines<float>(a.hidden, a.hs, count, a.dim), a.idx};
    const Lines<float> B(a.G, a.g_ld, count, vn);
    f32x16 c[1][1];
    products<false, false>(A, B, m0, n0, 0, count, sm, c);
    const float k = a.head->scale * a.temperature;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.d_weight) | (uintptr_t)(a.dws * sizeof(WT))) & 15) == 0;
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (n >= vn) return;
        WT *to = (WT *)a.d_weight + (long long)(v0 + n) * a.dws + m;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= k;
        if (wide && m + 8 <= a.dim) store_run(to, v);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (m + e < a.dim) store_one(to + e, v[e]);
        }
    });
}

int blocks(int n) { return (n + F32_BLOCK - 1) / F32_BLOCK; }
int entry_blocks(const LossArgs &a) { return (int)(((long long)a.rows * a.entries + 127) / 128); }

template <class Go> void by_head(const LossArgs &a, Go go)
{
    if (a.wdt == DT_BF16) go(bf16_t{});
    else go(float{});
}

}  // namespace

void launch_f32_softmax(hipStream_t s, const LossArgs &a)
{
    const int extra = entry_blocks(a);
    hipLaunchKernelGGL(f32_softmax_kernel, dim3(extra + blocks(a.vocab), blocks(a.rows)), dim3(256), 0, s, a, extra);
}

int f32_softmax_parts(const LossArgs &a) { return blocks(a.vocab) * 2; }

void launch_f32_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    by_head(a, [&](auto wt) {
        const int extra = v0 == 0 ? entry_blocks(a) : 0;
        hipLaunchKernelGGL((f32_probabilities_kernel<decltype(wt)>), dim3(extra + blocks(vn), blocks(a.rows)), dim3(256), 0, s, a, v0, vn, extra);
    });
}

void launch_f32_hidden_grad(hipStream_t s, const LossArgs &a, int v0, int vn, bool first)
{
    by_head(a, [&](auto wt) {
        const int per = ((vn + a.splits - 1) / a.splits + BK - 1) / BK * BK;   // whole steps
        hipLaunchKernelGGL((f32_hidden_grad_kernel<decltype(wt)>), dim3(blocks(a.dim), blocks(a.rows), a.splits), dim3(256), 0, s, a, v0, vn, per, (int)first);
    });
}

void launch_f32_weight_grad(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    by_head(a, [&](auto wt) { hipLaunchKernelGGL((f32_weight_grad_kernel<decltype(wt)>), dim3(blocks(a.dim), blocks(vn)), dim3(256), 0, s, a, v0, vn); });
}

}  // namespace tr
