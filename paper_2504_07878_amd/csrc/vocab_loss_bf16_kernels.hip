// Products of the losses over the vocabulary on bf16 matrix instructions: both operands bf16, sums in fp32.
//
// Four products, all computed transposed (see vocab_loss_epilogues.h), C[n][m] = sum_k A[m][k] B[n][k]:
//   softmax, probabilities     m = vocabulary entry, n = row that counts, k = feature: both operands lie with k contiguous
//   gradient to the rows       m = feature, n = row, k = vocabulary entry of the piece: A is the head, whose k runs from row to row; B = G, k contiguous
//   gradient to the head       m = feature, n = vocabulary entry, k = row: both operands have k from row to row
// A workgroup computes a block of 256 (m) x 256, 128 or 64 (n) in steps of 64 k. Both operands of a step are copied to LDS by direct loads, as they lie in
// memory, one step ahead; an operand with k from row to row is turned where it is read (the transposing LDS read). Within a tile the 16-byte pieces of a row (or
// the 32-byte pieces, where k runs from row to row) are permuted by the row, on the way in through the lanes' addresses, so that reads meet no bank conflicts.
// The matrix operands of 16 k are read into registers one such step ahead, across the steps' barriers too.
#include "vocab_loss_epilogues.h"
#include <algorithm>
#include <type_traits>

namespace tr {

namespace {

constexpr int BK = 64;                 // k per step
typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t lane_off, const char *base)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds), "v"(lane_off), "s"(base) : "memory");
}
// own loads have landed, own LDS reads are done, then the workgroup's barrier
__device__ __forceinline__ void landed_and_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((0 & 15) | (7 << 4) | (0 << 8));   // vmcnt 0, expcnt 7 (no wait), lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One operand's tile of T rows of its dimension x 64 k in LDS. KC: k contiguous in memory, LDS [row][64 k]; otherwise [64 k][T]. FEAT: rows are read in
// the order of the matrix instruction's output runs (tile_feature). WAVES share the copying.
template <int T, bool KC, bool FEAT, int WAVES> struct Tile {
    static constexpr int BYTES = T * BK * 2, COPIES = BYTES / 1024 / WAVES;
    static_assert(BYTES % (1024 * WAVES) == 0, "whole copies");
    static constexpr int MASK = T >= 256 ? 7 : T / 16 - 1;   // 32-byte pieces of a row of T elements that are permuted

    static __device__ __forceinline__ int key(int row) { return FEAT ? (row & 3) | ((row >> 1) & 4) : row & 7; }

    uint32_t off[COPIES], krow[COPIES];
    const char *base;
    uint32_t ld, advance;

    // p: element (first row, first k) of the operand; ld: elements from one line of memory to the next; limit: rows (KC) or columns that exist from p on
    __device__ __forceinline__ void init(const bf16_t *p, long long ld_elems, int limit)
    {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        base = (const char *)p;
        ld = (uint32_t)ld_elems * 2;
        advance = KC ? BK * 2 : BK * ld;
#pragma unroll
        for (int q = 0; q < COPIES; ++q) {
            const int g = w * COPIES + q;
            if (KC) {
                const int row = g * 8 + (lane >> 3), piece = (lane & 7) ^ key(row);
                off[q] = (uint32_t)min(row, limit - 1) * ld + piece * 16;
                krow[q] = 0;
            } else {
                const int at = g * 1024 + lane * 16, k = at / (T * 2), in = at % (T * 2), piece = (in >> 5) ^ (k & MASK), col = piece * 16 + ((in >> 4) & 1) * 8;
                krow[q] = k;
                off[q] = (uint32_t)min(col, limit - 8) * 2;
            }
        }
    }
    // copies of the next step into LDS at byte `lds`; kleft: lines that are left (read only where k runs from row to row)
    __device__ __forceinline__ void issue(uint32_t lds, int kleft)
    {
        const int w = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < COPIES; ++q) {
            uint32_t o = off[q];
            if (!KC) o += min(krow[q], (uint32_t)(kleft - 1)) * ld;
            load_to_lds(__builtin_amdgcn_readfirstlane(lds + (w * COPIES + q) * 1024), o, base);
        }
        base += advance;
    }
};

// Reads matrix operands from a tile: N of them, of 32 rows each, from row r0 on; step kk of 16 k.
template <int T, bool KC, bool FEAT, int N> struct Reader {
    static constexpr int MASK = T >= 256 ? 7 : T / 16 - 1;
    uint32_t at[KC ? 4 : 2 * N];
    __device__ __forceinline__ void init(int r0)
    {
        const int lane = threadIdx.x & 63, hf = lane >> 5;
        if (KC) {
            const int in = lane & 31, row = r0 + (FEAT ? tile_feature(in) : in), key = FEAT ? (row & 3) | ((row >> 1) & 4) : row & 7;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) at[kk] = row * (BK * 2) + (((kk * 2 + hf) ^ key) << 4);
        } else {
            // groups of 16 lanes turn 4 (k) x 16 elements; lane 4 r + c brings k = r, columns of quad c, and gets its own column's four k
            const int g = (lane >> 4) & 1, r = (lane >> 2) & 3, c = lane & 3, quad = FEAT ? 2 * (c & 1) + (c >> 1) : c;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int k = 4 * t + r, piece = (r0 >> 4) + 2 * n + g;
                    at[t * N + n] = (8 * hf + k) * (T * 2) + ((piece ^ (k & MASK)) << 5) + quad * 8;
                }
        }
    }
    template <int KK> __device__ __forceinline__ void read(uint32_t lds, bf16x8 (&o)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (KC) {
                o[n] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8 *>(lds + at[KK] + n * 32 * BK * 2);
            } else {
                typedef __attribute__((address_space(3))) s16x4 *lp;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lp>(lds + at[n] + KK * 16 * T * 2));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lp>(lds + at[N + n] + KK * 16 * T * 2));
                o[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    }
};

// Block of WM x WN wavefronts, each MI x NI accumulators; A_KC, B_KC: where the operands have k contiguous.
template <int WM_, int WN_, int MI_, int NI_, bool A_KC, bool B_KC> struct Block {
    static constexpr int WM = WM_, WN = WN_, MI = MI_, NI = NI_, WAVES = WM * WN, TM = WM * MI * 32, TN = WN * NI * 32;
    using TA = Tile<TM, A_KC, true, WAVES>;
    using TB = Tile<TN, B_KC, false, WAVES>;
    static constexpr int STAGE = TA::BYTES + TB::BYTES, LDS = 2 * STAGE;

    TA a;
    TB b;
    f32x16 c[MI][NI];

    // K: k in all; whole steps are copied, and what lies past K in the last has to be zero in one operand and finite in the other
    __device__ __forceinline__ void run(uint32_t lds, int K)
    {
        const int w = threadIdx.x >> 6, wm = w / WN, wn = w % WN, steps = (K + BK - 1) / BK;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) c[i][j][r] = 0.f;
        if (!steps) return;
        Reader<TM, A_KC, true, MI> ra;
        Reader<TN, B_KC, false, NI> rb;
        ra.init(wm * MI * 32);
        rb.init(wn * NI * 32);
        int left = K;
        auto issue = [&](int stage) {
            a.issue(lds + stage * STAGE, left);
            b.issue(lds + stage * STAGE + TA::BYTES, left);
            left -= BK;
        };
        bf16x8 xa[2][MI], xb[2][NI];
        auto multiply = [&](int p) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xa[p][i], xb[p][j], c[i][j], 0, 0, 0);
        };
        issue(0);
        landed_and_barrier();
        if (steps > 1) issue(1);
        uint32_t at = lds;
        ra.template read<0>(at, xa[0]);
        rb.template read<0>(at + TA::BYTES, xb[0]);
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
            ra.template read<1>(at, xa[1]); rb.template read<1>(at + TA::BYTES, xb[1]);
            multiply(0);
            ra.template read<2>(at, xa[0]); rb.template read<2>(at + TA::BYTES, xb[0]);
            multiply(1);
            ra.template read<3>(at, xa[1]); rb.template read<3>(at + TA::BYTES, xb[1]);
            multiply(0);
            // every wavefront holds the step's last operands: its buffer is free, and the next step's has landed
            landed_and_barrier();
            if (s + 2 < steps) issue(s & 1);
            at = lds + ((s + 1) & 1) * STAGE;
            if (s + 1 < steps) { ra.template read<0>(at, xa[0]); rb.template read<0>(at + TA::BYTES, xb[0]); }
            multiply(1);
        }
    }

    // f(accumulator along n, n, first m of a run of 8, the run)
    template <class F> __device__ __forceinline__ void each_run(F f) const
    {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w / WN, wn = w % WN;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float v[8];
                    run_of(c[i][j], h, v);
                    f(j, (wn * NI + j) * 32 + (lane & 31), (wm * MI + i) * 32 + 16 * h + 8 * (lane >> 5), v);
                }
    }
};

extern __shared__ char dynamic_lds[];
__device__ __forceinline__ uint32_t lds_start() { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)dynamic_lds; }

// Which block a workgroup computes. Workgroup b runs on XCD b mod 8, whose workgroups take a contiguous piece of an order that walks groups of GN blocks along n and, in
// a group, along m: those that run at a time share GN tiles of one operand and a few of the other in the XCD's L2. false: none.
constexpr int GN = 8;
__device__ __forceinline__ bool block_of(int mb, int nb, int &m, int &n)
{
    const int items = mb * nb, per = (items + 7) >> 3, at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= items) return false;
    const int group = at / (GN * mb), in = at - group * GN * mb, width = min(GN, nb - group * GN);
    m = in / width;
    n = group * GN + in % width;
    return true;
}
dim3 grid_of(int mb, int nb) { return dim3((mb * nb + 7) / 8 * 8); }

__device__ __forceinline__ const bf16_t *head_rows(const LossArgs &a, int v0, long long &ld)
{
    ld = a.direct ? a.ws : a.d_pad;
    return a.direct ? (const bf16_t *)a.weight + (long long)v0 * a.ws : (const bf16_t *)a.wp;
}

template <int TN> struct ByRows;    // blocks along the rows: 256 x TN
template <> struct ByRows<256> { template <bool A, bool B> using of = Block<2, 4, 4, 2, A, B>; };
template <> struct ByRows<128> { template <bool A, bool B> using of = Block<4, 2, 2, 2, A, B>; };
template <> struct ByRows<64> { template <bool A, bool B> using of = Block<8, 1, 1, 2, A, B>; };

template <int TN> __global__ __launch_bounds__(512) void bf16_softmax_kernel(LossArgs a, int v0, int vn)
{
    using Bl = typename ByRows<TN>::template of<true, true>;
    __shared__ float2 red[Bl::WAVES * Bl::NI * 32];
    const int count = a.head->count;
    int m, n;
    if (!block_of((vn + Bl::TM - 1) / Bl::TM, (count + TN - 1) / TN, m, n)) return;
    Bl bl;
    long long ld;
    const bf16_t *w = head_rows(a, v0, ld);
    bl.a.init(w + m * Bl::TM * ld, ld, vn - m * Bl::TM);
    bl.b.init((const bf16_t *)a.hp + (size_t)n * TN * a.d_pad, a.d_pad, TN);
    bl.run(lds_start(), a.d_pad);
    const int wv = threadIdx.x >> 6;
    softmax_part<Bl::WM, Bl::WN, Bl::MI, Bl::NI>(bl.c, red, a.part + (size_t)(v0 / Bl::TM + m) * a.n_pad + n * TN, m * Bl::TM, vn, LOG2E / a.temperature, wv / Bl::WN, wv % Bl::WN);
}

template <int TN> __global__ __launch_bounds__(512) void bf16_probabilities_kernel(LossArgs a, int v0, int vn)
{
    using Bl = typename ByRows<TN>::template of<true, true>;
    const int count = a.head->count;
    int m, n;
    if (!block_of((vn + Bl::TM - 1) / Bl::TM, (count + TN - 1) / TN, m, n)) return;
    Bl bl;
    long long ld;
    const bf16_t *w = head_rows(a, v0, ld);
    bl.a.init(w + m * Bl::TM * ld, ld, vn - m * Bl::TM);
    bl.b.init((const bf16_t *)a.hp + (size_t)n * TN * a.d_pad, a.d_pad, TN);
    bl.run(lds_start(), a.d_pad);
    const float k2 = LOG2E / a.temperature;
    const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) % Bl::WN;
    float lse2[Bl::NI], weight[Bl::NI];
#pragma unroll
    for (int j = 0; j < Bl::NI; ++j) {
        const int row = n * TN + (wn * Bl::NI + j) * 32 + (lane & 31);
        lse2[j] = row < count ? a.lse[a.idx[row]] * LOG2E : 0.f;
        weight[j] = row < count ? a.grad[a.idx[row]] / a.head->scale : 0.f;
    }
    bl.each_run([&](int j, int i, int v, float (&x)[8]) {   // rows that do not count and entries that do not exist: zeros, which the next products read
        const int row = n * TN + i;
        v += m * Bl::TM;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = row < count && v + e < vn ? weight[j] * term(x[e], k2, lse2[j]) : 0.f;
        store_run((bf16_t *)a.G + (size_t)row * a.piece + v, x);
    });
}

template <int TN> __global__ __launch_bounds__(512) void bf16_hidden_grad_kernel(LossArgs a, int v0, int vn, int first)
{
    using Bl = typename ByRows<TN>::template of<false, true>;
    const int count = a.head->count, nb = (count + TN - 1) / TN, mb = (a.d_pad + Bl::TM - 1) / Bl::TM, splits = bf16_splits(a, count);
    int m, n;
    if (!block_of(mb * splits, nb, m, n)) return;
    const int split = m / mb, per = ((vn + splits - 1) / splits + BK - 1) / BK * BK, k0 = min(vn, split * per), k1 = min(vn, k0 + per);
    m -= split * mb;
    Bl bl;
    long long ld;
    const bf16_t *w = head_rows(a, v0, ld);
    bl.a.init(w + k0 * ld + m * Bl::TM, ld, a.d_pad - m * Bl::TM);
    bl.b.init((const bf16_t *)a.G + (size_t)n * TN * a.piece + k0, a.piece, TN);
    bl.run(lds_start(), k1 - k0);
    bl.each_run([&](int, int i, int d, float (&x)[8]) {
        d += m * Bl::TM;
        if (d >= a.d_pad) return;
        float *to = a.acc + ((size_t)split * bf16_rows(a, count) + n * TN + i) * a.d_pad + d;
        if (!first) {
            const float4 p = reinterpret_cast<const float4 *>(to)[0], q = reinterpret_cast<const float4 *>(to)[1];
            x[0] += p.x; x[1] += p.y; x[2] += p.z; x[3] += p.w; x[4] += q.x; x[5] += q.y; x[6] += q.z; x[7] += q.w;
        }
        store_run(to, x);
    });
}

__global__ __launch_bounds__(512) void bf16_weight_grad_kernel(LossArgs a, int v0, int vn)
{
    using Bl = Block<2, 4, 4, 2, false, false>;
    int m, n;
    if (!block_of((a.d_pad + Bl::TM - 1) / Bl::TM, (vn + Bl::TN - 1) / Bl::TN, m, n)) return;
    Bl bl;
    bl.a.init((const bf16_t *)a.hp + m * Bl::TM, a.d_pad, a.d_pad - m * Bl::TM);
    bl.b.init((const bf16_t *)a.G + n * Bl::TN, a.piece, a.piece - n * Bl::TN);
    bl.run(lds_start(), (a.head->count + BK - 1) / BK * BK);
    const float k = a.head->scale * a.temperature;
    const bool whole = ((reinterpret_cast<uintptr_t>(a.d_weight) | (uintptr_t)(a.dws * 2)) & 15) == 0;
    bl.each_run([&](int, int i, int d, float (&x)[8]) {
        const int v = n * Bl::TN + i;
        d += m * Bl::TM;
        if (v >= vn || d >= a.dim) return;
        bf16_t *to = (bf16_t *)a.d_weight + (long long)(v0 + v) * a.dws + d;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= k;
        if (whole && d + 8 <= a.dim) store_run(to, x);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (d + e < a.dim) store_one(to + e, x[e]);
        }
    });
}

// Rows that count, one after the other, whole steps long; zeros up to the end of the last block.
__global__ __launch_bounds__(256) void bf16_pack_rows_kernel(LossArgs a)
{
    const int i = blockIdx.x, count = a.head->count;
    if (i >= (count + BF16_BLOCK - 1) / BF16_BLOCK * BF16_BLOCK) return;
    const bf16_t *h = (const bf16_t *)a.hidden + (i < count ? a.idx[i] : 0) * a.hs;
    for (int k = threadIdx.x; k < a.d_pad; k += 256) ((bf16_t *)a.hp)[(size_t)i * a.d_pad + k] = i < count && k < a.dim ? h[k] : (bf16_t)0;
}

__global__ __launch_bounds__(256) void bf16_pack_head_kernel(LossArgs a, int v0)
{
    const bf16_t *w = (const bf16_t *)a.weight + (long long)(v0 + blockIdx.x) * a.ws;
    for (int k = threadIdx.x; k < a.d_pad; k += 256) ((bf16_t *)a.wp)[(size_t)blockIdx.x * a.d_pad + k] = k < a.dim ? w[k] : (bf16_t)0;
}

// Products of listed entries: a wavefront takes 32 of them, its rows of the head against its hidden rows, of which only the diagonal is kept.
__global__ __launch_bounds__(64) void bf16_entries_kernel(LossArgs a)
{
    const int lane = threadIdx.x, e = blockIdx.x * 32 + (lane & 31), hf = lane >> 5, count = a.head->count;
    if ((long long)blockIdx.x * 32 >= (long long)count * a.entries) return;
    const int i = e / a.entries, j = e - i * a.entries;
    bool on = i < count;
    const bf16_t *h = (const bf16_t *)a.hp, *w = (const bf16_t *)a.weight;
    if (on) {
        const int id = a.ids[(long long)a.idx[i] * a.entries + j];
        on = id >= 0 && id < a.vocab;
        h += (size_t)i * a.d_pad;
        if (on) w += id * a.ws;
    }
    f32x16 c;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
    if (a.direct) {
#pragma unroll 8
        for (int k = 0; k < a.d_pad; k += 16) {
            const bf16x8 x = *reinterpret_cast<const bf16x8 *>(w + k + 8 * hf), y = *reinterpret_cast<const bf16x8 *>(h + k + 8 * hf);
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
        }
    } else {
        for (int k = 0; k < a.d_pad; k += 16) {
            uint32_t q[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int at = k + 8 * hf + 2 * p;
                q[p] = (at < a.dim ? (uint32_t)w[at] : 0u) | (at + 1 < a.dim ? (uint32_t)w[at + 1] << 16 : 0u);
            }
            const bf16x8 x = __builtin_bit_cast(bf16x8, make_uint4(q[0], q[1], q[2], q[3])), y = *reinterpret_cast<const bf16x8 *>(h + k + 8 * hf);
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
        }
    }
    const int n = lane & 31;   // row m of column n lies in register (m / 8) * 4 + m % 4 of lane n + 32 * (m / 4 % 2)
    float d = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d = (n >> 3) * 4 + (n & 3) == r ? c[r] : d;
    if (on && ((n >> 2) & 1) == hf) a.value[e] = d;
}

int up_div(int n, int by) { return (n + by - 1) / by; }

// a kernel's dynamic LDS beyond 64 KiB has to be allowed once per kernel and device; asking again costs nothing that counts beside a launch
template <class... P, class... A> void launch(void (*kernel)(P...), dim3 grid, int lds, hipStream_t s, A... args)
{
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    hipLaunchKernelGGL(kernel, grid, dim3(512), lds, s, args...);
}

template <class Go> void by_block(const LossArgs &a, Go go)
{
    if (a.n_block == 64) go(std::integral_constant<int, 64>{});
    else if (a.n_block == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 256>{});
}

}  // namespace

void launch_bf16_pack_rows(hipStream_t s, const LossArgs &a)
{
    hipLaunchKernelGGL(bf16_pack_rows_kernel, dim3(up_div(a.rows, BF16_BLOCK) * BF16_BLOCK), dim3(256), 0, s, a);
}

void launch_bf16_pack_head(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    hipLaunchKernelGGL(bf16_pack_head_kernel, dim3(vn), dim3(256), 0, s, a, v0);
}

void launch_bf16_entries(hipStream_t s, const LossArgs &a)
{
    hipLaunchKernelGGL(bf16_entries_kernel, dim3((unsigned)(((long long)a.rows * a.entries + 31) / 32)), dim3(64), 0, s, a);
}

void launch_bf16_softmax(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    by_block(a, [&](auto t) {
        constexpr int TN = decltype(t)::value;
        launch(bf16_softmax_kernel<TN>, grid_of(up_div(vn, BF16_BLOCK), up_div(a.rows, TN)), ByRows<TN>::template of<true, true>::LDS, s, a, v0, vn);
    });
}

void launch_bf16_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    by_block(a, [&](auto t) {
        constexpr int TN = decltype(t)::value;
        launch(bf16_probabilities_kernel<TN>, grid_of(up_div(vn, BF16_BLOCK), up_div(a.rows, TN)), ByRows<TN>::template of<true, true>::LDS, s, a, v0, vn);
    });
}

void launch_bf16_hidden_grad(hipStream_t s, const LossArgs &a, int v0, int vn, bool first)
{
    by_block(a, [&](auto t) {
        constexpr int TN = decltype(t)::value;
        // the rows that count, and with them the splits, are known on the device: the largest product of the two over any count
        const int mb = up_div(a.d_pad, BF16_BLOCK), most = std::max(mb * up_div(a.rows, TN), std::min(256, mb * up_div(a.rows, TN) * a.splits));
        launch(bf16_hidden_grad_kernel<TN>, grid_of(most, 1), ByRows<TN>::template of<false, true>::LDS, s, a, v0, vn, (int)first);
    });
}

void launch_bf16_weight_grad(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    using Bl = Block<2, 4, 4, 2, false, false>;
    launch(bf16_weight_grad_kernel, grid_of(up_div(a.d_pad, Bl::TM), up_div(vn, Bl::TN)), Bl::LDS, s, a, v0, vn);
}

}  // namespace tr
