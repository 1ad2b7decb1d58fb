// Losses over the vocabulary: rows, listed entries and sums. Small kernels beside the products; what they compute is in vocab_loss.h.
#include "vocab_loss_epilogues.h"
#include <algorithm>
#include <type_traits>

namespace tr {

// ------------------------------------------------------------------ rows that count

template <bool TEACHER>
__device__ __forceinline__ bool entry_counts(const LossArgs &a, long long at)
{
    const int id = a.ids[at];
    const float t = TEACHER ? a.teacher[at] : 0.f;         // (read at the same time)
    return (id >= 0) & (id < a.vocab) & (t != -INFINITY);
}

// A row counts if it has an entry (and, for gradients, a weight).
template <bool TEACHER>
__device__ __forceinline__ int row_state(const LossArgs &a, int r)
{
    int st = ROW_SKIP;
    const long long at = (long long)r * a.entries;
    if (!TEACHER) {
        const int id = a.ids[r];
        st = id < 0 ? ROW_SKIP : id < a.vocab ? ROW_COUNTS : ROW_BAD;
    } else {
        for (int j = 0; j < a.entries && st == ROW_SKIP; j += 8) {     // most rows have one among their first
            bool any = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) any |= entry_counts<TEACHER>(a, at + min(j + e, a.entries - 1));
            if (any) st = ROW_COUNTS;
        }
    }
    if (a.grad && a.grad[r] == 0.f) st = ROW_SKIP;
    return st;
}

// weights that cannot be divided by (none, infinite, too small for a reciprocal share) are taken as they are
__device__ __forceinline__ float usable(float top) { return top > 1e-30f && top < INFINITY ? top : 1.f; }
__device__ __forceinline__ int half_of(const LossArgs &a, int count) { return !a.pairs || count == 0 || count > PAIR_ROWS ? 0 : PAIR_ROWS; }

__device__ __forceinline__ void skipped(const LossArgs &a, int r, int st)
{
    const float v = st == ROW_BAD ? __uint_as_float(0x7fc00000u) : 0.f;
    a.loss[r] = v;
    a.lse[r] = v;
}

// Row `to` of the packed rows: row `from` that counts (-1: zeros), whole steps long. fp32 rows: blocks of 64 rows x 3 planes, a plane being what the ones
// before it leave, rounded to bf16.
template <class HT> __device__ __forceinline__ void pack_row(const LossArgs &a, int to, int from)
{
    const HT *h = (const HT *)a.hidden + (long long)max(from, 0) * a.hs;
    if constexpr (sizeof(HT) == 2) {
        bf16_t *p = (bf16_t *)a.hp + (size_t)to * a.d_pad;
        for (int k = threadIdx.x * 8; k < a.d_pad; k += blockDim.x * 8) *reinterpret_cast<uint4 *>(p + k) = from < 0 ? make_uint4(0, 0, 0, 0) : load8(h, k, a.dim);
    } else {
        bf16_t *p = (bf16_t *)a.hp + (size_t)((to >> 6) * 192 + (to & 63)) * a.d_pad;
        for (int k = threadIdx.x; k < a.d_pad; k += blockDim.x) {
            float v = from >= 0 && k < a.dim ? h[k] : 0.f;
#pragma unroll
            for (int l = 0; l < 3; ++l) {
                const bf16_t b = (bf16_t)two_bf16(v, 0.f);
                p[(size_t)l * 64 * a.d_pad + k] = b;
                v -= load_one(&b);
            }
        }
    }
}

__device__ __forceinline__ void describe_row(const LossArgs &a, int to, int from, float scale)
{
    LossRow x{0.f, 0.f, -1, 0};
    if (from >= 0) x = LossRow{a.lse[from], a.grad[from] / scale, a.teacher ? -1 : a.ids[from], 0};
    a.row[to] = x;
}

// Everything at once for few rows: workgroup j finds row j's place by going over the states of all rows, and packs it; the packed rows past the last are cleared, and
// with pairs the second halves written, by the workgroups from the end.
template <bool TEACHER, class HT>
__global__ __launch_bounds__(256) void loss_prepare_kernel(LossArgs a, int packed)
{
    __shared__ int before_s[4], count_s[4], own_s;
    __shared__ float top_s[4];
    const int j = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
    int before = 0, count = 0;
    float top = 0.f;
    for (int r = t; r < a.rows; r += 256) {
        const int st = row_state<TEACHER>(a, r);
        if (r == j) own_s = st;
        if (st == ROW_COUNTS) {
            ++count;
            before += r < j;
            if (a.grad) { const float g = fabsf(a.grad[r]); top = g > top ? g : top; }
        }
    }
    for (int o = 32; o; o >>= 1) { before += __shfl_xor(before, o); count += __shfl_xor(count, o); top = fmaxf(top, __shfl_xor(top, o)); }
    if (lane == 0) { before_s[w] = before; count_s[w] = count; top_s[w] = top; }
    __syncthreads();
    before = (before_s[0] + before_s[1]) + (before_s[2] + before_s[3]);
    count = (count_s[0] + count_s[1]) + (count_s[2] + count_s[3]);
    const int half = half_of(a, count), own = j < a.rows ? own_s : (int)ROW_SKIP;
    const float scale = usable(fmaxf(fmaxf(top_s[0], top_s[1]), fmaxf(top_s[2], top_s[3])));
    const bool describes = a.grad && t == 0;
    if (j == 0 && t == 0) {
        a.head->count = count; a.head->half = half;
        a.head->scale = scale;
    }
    if (j < a.rows && t == 0) {
        a.state[j] = (unsigned char)own;
        if (own == ROW_COUNTS) a.idx[before] = j;
        else if (!a.grad) skipped(a, j, own);
    }
    if (!packed) return;
    if (own == ROW_COUNTS) {
        for (int at = before; at <= before + half; at += half ? half : 1) {
            pack_row<HT>(a, at, j);
            if (describes) describe_row(a, at, j, scale);
        }
    }
    // rows without anything: [count, half or the end), and with pairs [half + count, the end)
    const int firsts = half ? half : packed, gap = firsts - count, all = half ? gap + packed - half - count : gap;
    for (int i = j; i < all; i += gridDim.x) {
        const int at = i < gap ? count + i : half + count + (i - gap);
        pack_row<HT>(a, at, -1);
        if (describes) describe_row(a, at, -1, scale);
    }
}

// For many rows: their states, one thread a row, ...
template <bool TEACHER>
__global__ __launch_bounds__(256) void loss_state_kernel(LossArgs a)
{
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r < a.rows) a.state[r] = (unsigned char)row_state<TEACHER>(a, r);
}

// ... their list by one workgroup, in order, 1024 rows at a time; the rows that do not count get their loss here. The rows' weights in the
// gradients are taken relative to the largest |weight|, by which the gradients are multiplied at the end: with equal weights G then holds p - q itself, whose
// 0 - 1 has no rounding.
__global__ __launch_bounds__(1024) void loss_list_kernel(LossArgs a)
{
    __shared__ int sums[16];
    __shared__ float tops[16];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    int before = 0;
    float top = 0.f;
    for (int r0 = 0; r0 < a.rows; r0 += 1024) {
        const int r = r0 + t;
        const int st = r < a.rows ? a.state[r] : (int)ROW_SKIP;
        const bool on = st == ROW_COUNTS;
        const unsigned long long m = __ballot(on);
        if (lane == 0) sums[w] = __popcll(m);
        __syncthreads();
        int at = before + __popcll(m & ((1ull << lane) - 1));
        for (int i = 0; i < 16; ++i) { at += i < w ? sums[i] : 0; before += sums[i]; }
        __syncthreads();
        if (on) {
            a.idx[at] = r;
            if (a.grad) {
                const float g = fabsf(a.grad[r]);
                top = g > top ? g : top;
            }
        } else if (r < a.rows && !a.grad) skipped(a, r, st);
    }
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) tops[w] = top;
    __syncthreads();
    if (t == 0) {
        for (int i = 0; i < 16; ++i) top = fmaxf(top, tops[i]);
        a.head->count = before; a.head->half = half_of(a, before); a.head->scale = usable(top);
    }
}

// ... and the packed rows, one after the other, zeros up to the end of the last block.
template <class HT>
__global__ __launch_bounds__(256) void loss_pack_kernel(LossArgs a)
{
    const int i = blockIdx.x, count = a.head->count, half = a.head->half;
    if (i >= (bf16_products_rows(count, half) + BF16_BLOCK - 1) / BF16_BLOCK * BF16_BLOCK) return;
    const int row = half && i >= half ? i - half : i;
    const int from = row < count ? a.idx[row] : -1;
    pack_row<HT>(a, i, from);
    if (a.grad && threadIdx.x == 0) describe_row(a, i, from, a.head->scale);
}

template <bool TEACHER, class HT> static void rows_of(hipStream_t s, const LossArgs &a)
{
    const int packed = a.hp ? (a.rows + BF16_BLOCK - 1) / BF16_BLOCK * BF16_BLOCK : 0;
    if (a.rows <= 1024 && (long long)a.rows * a.entries <= 16384) {
        const int used = !a.hp ? 0 : a.n_block < 256 ? (a.rows + a.n_block - 1) / a.n_block * a.n_block : packed;   // what the products' blocks read
        hipLaunchKernelGGL((loss_prepare_kernel<TEACHER, HT>), dim3(std::max(a.rows, used)), dim3(256), 0, s, a, used);
        return;
    }
    hipLaunchKernelGGL((loss_state_kernel<TEACHER>), dim3((a.rows + 255) / 256), dim3(256), 0, s, a);
    hipLaunchKernelGGL(loss_list_kernel, dim3(1), dim3(1024), 0, s, a);
    if (packed) hipLaunchKernelGGL((loss_pack_kernel<HT>), dim3(packed), dim3(256), 0, s, a);
}

void launch_loss_rows(hipStream_t s, const LossArgs &a)
{
    if (!a.rows) { hipLaunchKernelGGL(loss_list_kernel, dim3(1), dim3(1024), 0, s, a); return; }
    if (a.teacher) { if (a.hdt == DT_BF16) rows_of<true, bf16_t>(s, a); else rows_of<true, float>(s, a); }
    else { if (a.hdt == DT_BF16) rows_of<false, bf16_t>(s, a); else rows_of<false, float>(s, a); }
}

// ------------------------------------------------------------------ listed entries

__device__ __forceinline__ float sum64(float v)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

struct Shares { float top, total; };   // of a row's entries: q_j = exp((t_j - top) / T) / total

template <bool TEACHER>
__device__ __forceinline__ Shares shares_of(const LossArgs &a, int r)
{
    if constexpr (!TEACHER) return Shares{0.f, 1.f};
    else {
        const int lane = threadIdx.x & 63;
        const long long at = (long long)r * a.entries;
        float top = -INFINITY, total = 0.f;
        for (int j = lane; j < a.entries; j += 64) if (entry_counts<TEACHER>(a, at + j)) top = fmaxf(top, a.teacher[at + j]);
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        for (int j = lane; j < a.entries; j += 64) if (entry_counts<TEACHER>(a, at + j)) total += expf((a.teacher[at + j] - top) / a.temperature);
        return Shares{top, sum64(total)};
    }
}

// A workgroup takes ROWS rows that count: 256 / ROWS threads join a row's running softmaxes, then a wavefront takes the row's entries. Sums in a fixed order.
// lse - z_j = ln 2 (m - k c_j) + log s: no rounding of lse in it.
template <bool TEACHER, int ROWS>
__global__ __launch_bounds__(256) void loss_finish_kernel(LossArgs a, int parts)
{
    __shared__ float2 joined[4][ROWS];
    const int i0 = blockIdx.x * ROWS, t = threadIdx.x, lane = t & 63, w = t >> 6, mine = min(i0 + t % ROWS, a.rows - 1);
    float2 x = make_float2(-INFINITY, 0.f);
#pragma unroll 4
    for (int p = t / ROWS; p < parts; p += 256 / ROWS) x = join(x, a.part[(size_t)p * a.part_ld + mine]);    // (of a row that does not count: for nobody)
    const int count = a.head->count;
    if (i0 >= count) return;
    for (int o = ROWS; o < 64; o *= 2) x = join(x, make_float2(__shfl_xor(x.x, o), __shfl_xor(x.y, o)));
    if (lane < ROWS) joined[w][lane] = x;
    __syncthreads();
    for (int q = w; q < ROWS && i0 + q < count; q += 4) {
        const int i = i0 + q, r = a.idx[i];
        const float2 st = join(join(joined[0][q], joined[1][q]), join(joined[2][q], joined[3][q]));
        const float ls = logf(st.y), k2 = LOG2E / a.temperature, at = st.x == -INFINITY ? 0.f : st.x;
        const Shares sh = shares_of<TEACHER>(a, r);
        const float ltot = TEACHER ? logf(sh.total) : 0.f;
        float s = 0.f;
        for (int j = lane; j < a.entries; j += 64) {
            const long long from = (long long)r * a.entries + j;
            if (!entry_counts<TEACHER>(a, from)) continue;
            const float rel = TEACHER ? (a.teacher[from] - sh.top) / a.temperature : 0.f, e = TEACHER ? expf(rel) / sh.total : 1.f;
            const float left = LN2 * -fmaf(a.value[(size_t)i * a.entries + j], k2, -at) + ls;
            if (e != 0.f) s += e * ((rel - ltot) + left);
        }
        s = sum64(s);
        if (lane == 0) {
            a.lse[r] = LN2 * st.x + ls;
            a.loss[r] = a.temperature * a.temperature * s;
        }
    }
}

// What G holds for an entry v of row i.
template <bool BF16> __device__ __forceinline__ void place_entry(const LossArgs &a, int i, int v, float x)
{
    if constexpr (BF16) {
        bf16_t *to = (bf16_t *)a.G + (size_t)i * a.g_ld + v;
        store_one(to, x);
        const int half = a.head->half;
        if (half) { const bf16_t hi = (bf16_t)two_bf16(x, 0.f); store_one(to + (size_t)half * a.g_ld, x - load_one(&hi)); }
    } else ((float *)a.G)[(size_t)i * a.g_ld + v] = x;
}

// p - q of every listed entry of a teacher's from its product (an id listed twice: p less both shares, in both places), by the row's weight. PLACE: into G right away.
template <bool PLACE, bool BF16>
__global__ __launch_bounds__(256) void loss_values_kernel(LossArgs a)
{
    const int i = blockIdx.x, lane = threadIdx.x & 63;
    if (i >= a.head->count) return;
    const int r = a.idx[i];
    const float lse = a.lse[r], k = 1.0f / a.temperature, weight = a.grad[r] / a.head->scale;
    const Shares sh = shares_of<true>(a, r);
    const long long at0 = (long long)r * a.entries;
    for (int j0 = threadIdx.x - lane; j0 < a.entries; j0 += 256) {
        const int j = j0 + lane;
        const bool on = j < a.entries && entry_counts<true>(a, at0 + j);
        const int id = on ? a.ids[at0 + j] : -1;
        float q = 0.f;
        for (int o0 = 0; o0 < a.entries; o0 += 64) {       // a wavefront's 64 shares at a time, each handed to all its lanes
            const int o = o0 + lane;
            const bool other = o < a.entries && entry_counts<true>(a, at0 + o);
            const int others = other ? a.ids[at0 + o] : -1;
            const float share = other ? expf((a.teacher[at0 + o] - sh.top) / a.temperature) / sh.total : 0.f;
            for (int n = 0; n < min(64, a.entries - o0); ++n) {
                const int same = __shfl(others, n);
                const float its = __shfl(share, n);
                q += same == id ? its : 0.f;
            }
        }
        if (!on) continue;
        float &v = a.value[(size_t)i * a.entries + j];
        const float x = weight * (expf(fmaf(v, k, -lse)) - q);
        if (PLACE) place_entry<BF16>(a, i, id, x);
        else v = x;
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void loss_scatter_kernel(LossArgs a, int v0, int vn)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int i = (int)(at / a.entries), j = (int)(at % a.entries);
    if (i >= a.head->count) return;
    const long long from = (long long)a.idx[i] * a.entries + j;
    const int v = a.ids[from] - v0;
    if (v < 0 || v >= vn || !entry_counts<true>(a, from)) return;
    place_entry<BF16>(a, i, v, a.value[at]);
}

// Few rows take a workgroup each, so that their parts are read at once; many take eight, whose parts lie together.
void launch_loss_finish(hipStream_t s, const LossArgs &a, int parts)
{
    if (!a.rows) return;
    const auto go = [&](auto teacher) {
        if (a.rows <= 256) hipLaunchKernelGGL((loss_finish_kernel<decltype(teacher)::value, 1>), dim3(a.rows), dim3(256), 0, s, a, parts);
        else hipLaunchKernelGGL((loss_finish_kernel<decltype(teacher)::value, 8>), dim3((a.rows + 7) / 8), dim3(256), 0, s, a, parts);
    };
    if (a.teacher) go(std::true_type{});
    else go(std::false_type{});
}

void launch_loss_values(hipStream_t s, const LossArgs &a, bool place)
{
    if (!a.rows) return;
    const auto go = [&](auto bf16) {
        if (place) hipLaunchKernelGGL((loss_values_kernel<true, decltype(bf16)::value>), dim3(a.rows), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((loss_values_kernel<false, decltype(bf16)::value>), dim3(a.rows), dim3(256), 0, s, a);
    };
    if (a.hdt == DT_BF16) go(std::true_type{});
    else go(std::false_type{});
}

void launch_loss_scatter(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    if (!a.rows) return;
    const dim3 grid((unsigned)(((long long)a.rows * a.entries + 255) / 256));
    if (a.hdt == DT_BF16) hipLaunchKernelGGL(loss_scatter_kernel<true>, grid, dim3(256), 0, s, a, v0, vn);
    else hipLaunchKernelGGL(loss_scatter_kernel<false>, grid, dim3(256), 0, s, a, v0, vn);
}

// ------------------------------------------------------------------ gradient to the hidden rows

// A workgroup takes ROWS rows that count, 256 columns of each: 4 / ROWS wavefronts a row take every such split each, in order, joined in a fixed order. It also clears those
// of the rows of the same numbers that do not count.
template <class HT, bool BF16, int ROWS>
__global__ __launch_bounds__(256) void hidden_grad_kernel(LossArgs a)
{
    __shared__ float4 sums[4][64];
    constexpr int SHARE = 4 / ROWS;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * ROWS + w / SHARE, part = w % SHARE, count = a.head->count, j = blockIdx.y * 256 + lane * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float4 &to, const float4 u) { to.x += u.x; to.y += u.y; to.z += u.z; to.w += u.w; };
    auto store = [&](int r, const float (&x)[4]) {
        HT *out = (HT *)a.d_hidden + (long long)r * a.dhs + j;
        if (j + 4 <= a.dim) {
            if constexpr (sizeof(HT) == 2) store_bits(out, make_uint2(two_bf16(x[0], x[1]), two_bf16(x[2], x[3])));
            else store_bits(out, make_float4(x[0], x[1], x[2], x[3]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (j + e < a.dim) store_one(out + e, x[e]);
        }
    };
    if (i < count) {
        const int half = BF16 ? a.head->half : 0, rows = BF16 ? bf16_products_rows(count, half) : a.n_pad, splits = BF16 ? bf16_splits(a, rows) : a.splits;
        const size_t apart = (size_t)(BF16 ? bf16_rows(a, rows) : rows) * a.d_pad;
        const float *at = a.acc + (size_t)i * a.d_pad + j;
        if (j < a.d_pad) {
#pragma unroll 8
            for (int p = part; p < splits; p += SHARE) add(v, *reinterpret_cast<const float4 *>(at + p * apart));
            if (half) {
                at += (size_t)half * a.d_pad;
#pragma unroll 8
                for (int p = part; p < splits; p += SHARE) add(v, *reinterpret_cast<const float4 *>(at + p * apart));
            }
        }
    }
    if constexpr (SHARE > 1) {
        sums[w][lane] = v;
        __syncthreads();
#pragma unroll
        for (int q = 1; q < SHARE; ++q) if (part == 0) add(v, sums[w + q][lane]);
    }
    if (part == 0) {
        const float k = a.head->scale * a.temperature, x[4] = {k * v.x, k * v.y, k * v.z, k * v.w}, none[4] = {0.f, 0.f, 0.f, 0.f};
        if (i < count) store(a.idx[i], x);
        if (i < a.rows && a.state[i] != ROW_COUNTS) store(i, none);
    }
}

void launch_loss_hidden_grad(hipStream_t s, const LossArgs &a)
{
    if (!a.rows) return;
    const int ny = (a.dim + 255) / 256;
    if (a.hdt == DT_BF16) {
        if (a.rows <= 512) hipLaunchKernelGGL((hidden_grad_kernel<bf16_t, true, 1>), dim3(a.rows, ny), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((hidden_grad_kernel<bf16_t, true, 4>), dim3((a.rows + 3) / 4, ny), dim3(256), 0, s, a);
    } else hipLaunchKernelGGL((hidden_grad_kernel<float, false, 1>), dim3(a.rows, ny), dim3(256), 0, s, a);
}

}  // namespace tr
