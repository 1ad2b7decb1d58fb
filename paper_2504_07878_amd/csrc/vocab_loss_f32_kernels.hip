// Products of the losses over the vocabulary on 32-bit matrix instructions: operands of either storage type, any stride and alignment, widened where they
// are read; used wherever an operand is fp32.
//
// A workgroup of 4 wavefronts (2 x 2, each 2 x 2 accumulators of 32 x 32) computes a 128 x 128 block of C[n][m] = sum_k A[m][k] B[n][k], 16 k at a time:
// both operands go through registers into LDS as [k][row], the next step's are requested before this step's products. Three products:
//   softmax, probabilities: m = vocabulary entry, n = row that counts, k = feature
//   gradient to the hidden rows: m = feature, n = row, k = vocabulary entry of the piece; summed over the pieces in `acc`, one sum per split of k
//   gradient to the head: m = feature, n = vocabulary entry, k = row
#include "vocab_loss_epilogues.h"

namespace tr {

namespace {

constexpr int BK = 16, PITCH = F32_BLOCK + 4;

// operands: at(row of the block's dimension, k) or 0 beyond either. CONTIGUOUS_K: how threads are laid over a tile, so that neighbours read neighbours.
template <class WT> struct HeadRows {          // weight[v][k]
    static constexpr bool contiguous_k = true;
    const WT *w; long long ws; int v0, vn, d;
    __device__ __forceinline__ float at(int m, int k) const { return m < vn && k < d ? load_one(w + (v0 + m) * ws + k) : 0.f; }
};
template <class HT> struct HiddenRows {        // hidden[idx[n]][k]
    static constexpr bool contiguous_k = true;
    const HT *h; long long hs; const int *idx; int count, d;
    __device__ __forceinline__ float at(int n, int k) const { return n < count && k < d ? load_one(h + idx[n] * hs + k) : 0.f; }
};
template <class WT> struct HeadColumns {       // weight[k][m]
    static constexpr bool contiguous_k = false;
    const WT *w; long long ws; int v0, vn, d;
    __device__ __forceinline__ float at(int m, int k) const { return m < d && k < vn ? load_one(w + (v0 + k) * ws + m) : 0.f; }
};
struct PieceRows {                             // G[n][k]
    static constexpr bool contiguous_k = true;
    const float *g; int ld, count, vn;
    __device__ __forceinline__ float at(int n, int k) const { return n < count && k < vn ? g[(size_t)n * ld + k] : 0.f; }
};
template <class HT> struct HiddenColumns {     // hidden[idx[k]][m]
    static constexpr bool contiguous_k = false;
    const HT *h; long long hs; const int *idx; int count, d;
    __device__ __forceinline__ float at(int m, int k) const { return m < d && k < count ? load_one(h + idx[k] * hs + m) : 0.f; }
};
struct PieceColumns {                          // G[k][n]
    static constexpr bool contiguous_k = false;
    const float *g; int ld, count, vn;
    __device__ __forceinline__ float at(int n, int k) const { return n < vn && k < count ? g[(size_t)k * ld + n] : 0.f; }
};

struct Tiles { float a[BK * PITCH], b[BK * PITCH]; };

template <class Op> __device__ __forceinline__ void read8(const Op &op, int row0, int k0, float (&v)[8])
{
    const int t = threadIdx.x;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = Op::contiguous_k ? op.at(row0 + (t >> 1), k0 + (t & 1) * 8 + e) : op.at(row0 + (t & 15) * 8 + e, k0 + (t >> 4));
}
template <class Op> __device__ __forceinline__ void write8(float *lds, const float (&v)[8])
{
    const int t = threadIdx.x;
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[Op::contiguous_k ? ((t & 1) * 8 + e) * PITCH + (t >> 1) : (t >> 4) * PITCH + (t & 15) * 8 + e] = v[e];
}

// c = products of the block at (m0, n0) over k in [k_lo, k_hi), whole steps unless k_hi is the operands' end
template <class A, class B> __device__ __forceinline__ void products(const A &a, const B &b, int m0, int n0, int k_lo, int k_hi, Tiles &sm, f32x16 (&c)[2][2])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
    const int arow = wm * 64 + tile_feature(lane & 31), brow = wn * 64 + (lane & 31), kk = lane >> 5;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) c[i][j][r] = 0.f;
    float va[8], vb[8];
    if (k_lo < k_hi) { read8(a, m0, k_lo, va); read8(b, n0, k_lo, vb); }
    for (int k = k_lo; k < k_hi; k += BK) {
        __syncthreads();
        write8<A>(sm.a, va); write8<B>(sm.b, vb);
        __syncthreads();
        if (k + BK < k_hi) { read8(a, m0, k + BK, va); read8(b, n0, k + BK, vb); }
#pragma unroll
        for (int s = 0; s < BK; s += 2) {
            float x[2], y[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) { x[i] = sm.a[(s + kk) * PITCH + arow + 32 * i]; y[i] = sm.b[(s + kk) * PITCH + brow + 32 * i]; }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[j], c[i][j], 0, 0, 0);
        }
    }
}

// f(n, first m of a run of 8, the run) for every run of the block
template <class F> __device__ __forceinline__ void each_run(const f32x16 (&c)[2][2], F f)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                run_of(c[i][j], h, v);
                f(wn * 64 + j * 32 + (lane & 31), wm * 64 + i * 32 + 16 * h + 8 * (lane >> 5), v);
            }
}

template <class HT, class WT> __global__ __launch_bounds__(256) void f32_softmax_kernel(LossArgs a)
{
    __shared__ Tiles sm;
    const int m0 = blockIdx.x * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    if (n0 >= count) return;
    const HeadRows<WT> A{(const WT *)a.weight, a.ws, 0, a.vocab, a.dim};
    const HiddenRows<HT> B{(const HT *)a.hidden, a.hs, a.idx, count, a.dim};
    f32x16 c[2][2];
    products(A, B, m0, n0, 0, a.dim, sm, c);
    const int w = threadIdx.x >> 6;
    softmax_part(c, a.part + ((size_t)blockIdx.x * 2 + (w >> 1)) * a.part_ld + n0 + (w & 1) * 64, m0 + (w >> 1) * 64, a.vocab, LOG2E / a.temperature);
}

template <class HT, class WT> __global__ __launch_bounds__(256) void f32_probabilities_kernel(LossArgs a, int v0, int vn)
{
    __shared__ Tiles sm;
    const int m0 = blockIdx.x * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    if (n0 >= count) return;
    const HeadRows<WT> A{(const WT *)a.weight, a.ws, v0, vn, a.dim};
    const HiddenRows<HT> B{(const HT *)a.hidden, a.hs, a.idx, count, a.dim};
    f32x16 c[2][2];
    products(A, B, m0, n0, 0, a.dim, sm, c);
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
    const HeadColumns<WT> A{(const WT *)a.weight, a.ws, v0, vn, a.dim};
    const PieceRows B{(const float *)a.G, a.g_ld, count, vn};
    f32x16 c[2][2];
    products(A, B, m0, n0, min(vn, (int)blockIdx.z * per), min(vn, ((int)blockIdx.z + 1) * per), sm, c);
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

template <class HT, class WT> __global__ __launch_bounds__(256) void f32_weight_grad_kernel(LossArgs a, int v0, int vn)
{
    __shared__ Tiles sm;
    const int m0 = blockIdx.x * F32_BLOCK, n0 = blockIdx.y * F32_BLOCK, count = a.head->count;
    const HiddenColumns<HT> A{(const HT *)a.hidden, a.hs, a.idx, count, a.dim};
    const PieceColumns B{(const float *)a.G, a.g_ld, count, vn};
    f32x16 c[2][2];
    products(A, B, m0, n0, 0, count, sm, c);
    const float k = a.head->scale * a.temperature;
    each_run(c, [&](int n, int m, float (&v)[8]) {
        n += n0; m += m0;
        if (n >= vn) return;
        WT *to = (WT *)a.d_weight + (long long)(v0 + n) * a.dws + m;
#pragma unroll
        for (int e = 0; e < 8; ++e) if (m + e < a.dim) store_one(to + e, k * v[e]);
    });
}

// Products of listed entries: a wavefront takes 32 of them, its rows of the head against its hidden rows, of which only the diagonal is kept (the matrix unit
// is all but idle in a product this small, and it gives the bits that the same pair has in a block: the same instruction over the same steps of k).
template <class HT, class WT> __global__ __launch_bounds__(64) void f32_entries_kernel(LossArgs a)
{
    const int lane = threadIdx.x, e = blockIdx.x * 32 + (lane & 31), kk = lane >> 5, count = a.head->count;
    if ((long long)blockIdx.x * 32 >= (long long)count * a.entries) return;
    const int i = e / a.entries, j = e - i * a.entries;
    const HT *h = (const HT *)a.hidden;
    const WT *w = (const WT *)a.weight;
    bool on = i < count;
    if (on) {
        const int r = a.idx[i], id = a.ids[(long long)r * a.entries + j];
        on = id >= 0 && id < a.vocab;
        h += r * a.hs;
        if (on) w += id * a.ws;
    }
    f32x16 c;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
    for (int k = 0; k < a.dim; k += BK) {
        float x[BK / 2], y[BK / 2];
#pragma unroll
        for (int s = 0; s < BK / 2; ++s) {
            const int at = k + 2 * s + kk;
            const bool in = on && at < a.dim;
            x[s] = in ? load_one(w + at) : 0.f;
            y[s] = in ? load_one(h + at) : 0.f;
        }
#pragma unroll
        for (int s = 0; s < BK / 2; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[s], y[s], c, 0, 0, 0);
    }
    // row m of column n lies in register (m / 8) * 4 + m % 4 of lane n + 32 * (m / 4 % 2)
    const int n = lane & 31;
    float d = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d = (n >> 3) * 4 + (n & 3) == r ? c[r] : d;
    if (on && ((n >> 2) & 1) == kk) a.value[e] = d;
}

int blocks(int n) { return (n + F32_BLOCK - 1) / F32_BLOCK; }

template <class Go> void by_types(const LossArgs &a, Go go)
{
    if (a.wdt == DT_BF16) go(float{}, bf16_t{});
    else go(float{}, float{});
}

}  // namespace

void launch_f32_softmax(hipStream_t s, const LossArgs &a)
{
    if (!a.rows) return;
    by_types(a, [&](auto ht, auto wt) {
        hipLaunchKernelGGL((f32_softmax_kernel<decltype(ht), decltype(wt)>), dim3(blocks(a.vocab), blocks(a.rows)), dim3(256), 0, s, a);
    });
}

void launch_f32_entries(hipStream_t s, const LossArgs &a)
{
    if (!a.rows) return;
    by_types(a, [&](auto ht, auto wt) {
        hipLaunchKernelGGL((f32_entries_kernel<decltype(ht), decltype(wt)>), dim3((unsigned)(((long long)a.rows * a.entries + 31) / 32)), dim3(64), 0, s, a);
    });
}

void launch_f32_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    if (!a.rows) return;
    by_types(a, [&](auto ht, auto wt) {
        hipLaunchKernelGGL((f32_probabilities_kernel<decltype(ht), decltype(wt)>), dim3(blocks(vn), blocks(a.rows)), dim3(256), 0, s, a, v0, vn);
    });
}

void launch_f32_hidden_grad(hipStream_t s, const LossArgs &a, int v0, int vn, bool first)
{
    if (!a.rows) return;
    const int per = ((vn + a.splits - 1) / a.splits + BK - 1) / BK * BK;   // whole steps
    const dim3 grid(blocks(a.dim), blocks(a.rows), a.splits);
    if (a.wdt == DT_BF16) hipLaunchKernelGGL((f32_hidden_grad_kernel<bf16_t>), grid, dim3(256), 0, s, a, v0, vn, per, first);
    else hipLaunchKernelGGL((f32_hidden_grad_kernel<float>), grid, dim3(256), 0, s, a, v0, vn, per, first);
}

void launch_f32_weight_grad(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    by_types(a, [&](auto ht, auto wt) {
        hipLaunchKernelGGL((f32_weight_grad_kernel<decltype(ht), decltype(wt)>), dim3(blocks(a.dim), blocks(vn)), dim3(256), 0, s, a, v0, vn);
    });
}

}  // namespace tr
