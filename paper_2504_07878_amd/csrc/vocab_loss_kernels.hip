// Losses over the vocabulary: rows, listed entries and sums. Small kernels beside the products; what they compute is in vocab_loss.h.
#include "vocab_loss_epilogues.h"

namespace tr {

// ------------------------------------------------------------------ rows that count

template <bool TEACHER>
__device__ __forceinline__ bool entry_counts(const LossArgs &a, long long at)
{
    const int id = a.ids[at];
    return id >= 0 && id < a.vocab && (!TEACHER || a.teacher[at] != -INFINITY);
}

// A row counts if it has an entry (and, for gradients, a weight). One thread a row: the entries of a row lie together, and the first that counts ends the search.
template <bool TEACHER>
__global__ __launch_bounds__(256) void loss_state_kernel(LossArgs a)
{
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r >= a.rows) return;
    int st = ROW_SKIP;
    for (int j = 0; j < a.entries && st == ROW_SKIP; ++j) {
        const long long at = (long long)r * a.entries + j;
        if (entry_counts<TEACHER>(a, at)) st = ROW_COUNTS;
        else if (!TEACHER && a.ids[at] >= a.vocab) st = ROW_BAD;
    }
    if (a.grad && a.grad[r] == 0.f) st = ROW_SKIP;
    a.state[r] = (unsigned char)st;
}

// One workgroup lists the rows that count, in order, 1024 rows at a time; the rows that do not get their loss here. The rows' weights in the
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
        } else if (r < a.rows && !a.grad) {
            const float v = st == ROW_BAD ? __uint_as_float(0x7fc00000u) : 0.f;
            a.loss[r] = v;
            a.lse[r] = v;
        }
    }
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) tops[w] = top;
    __syncthreads();
    if (t == 0) {
        for (int i = 0; i < 16; ++i) top = fmaxf(top, tops[i]);
        // weights that cannot be divided by (none, infinite, too small for a reciprocal share) are taken as they are
        a.head->count = before; a.head->rows = a.rows; a.head->scale = top > 1e-30f && top < INFINITY ? top : 1.f;
    }
}

void launch_loss_rows(hipStream_t s, const LossArgs &a)
{
    if (a.rows > 0) {
        if (a.teacher) hipLaunchKernelGGL((loss_state_kernel<true>), dim3((a.rows + 255) / 256), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((loss_state_kernel<false>), dim3((a.rows + 255) / 256), dim3(256), 0, s, a);
    }
    hipLaunchKernelGGL(loss_list_kernel, dim3(1), dim3(1024), 0, s, a);
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

// A workgroup takes a row: it joins the blocks' running softmaxes, then takes the row's entries. Sums in a fixed order.
// lse - z_j = ln 2 (m - k c_j) + log s: no rounding of lse in it.
template <bool TEACHER>
__global__ __launch_bounds__(256) void loss_finish_kernel(LossArgs a, int parts)
{
    __shared__ float2 joined[4];
    __shared__ float sums[4];
    const int i = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (i >= a.head->count) return;
    const int r = a.idx[i];
    float2 t = make_float2(-INFINITY, 0.f);
    for (int p = threadIdx.x; p < parts; p += 256) t = join(t, a.part[(size_t)p * a.part_ld + i]);
    for (int o = 32; o; o >>= 1) {
        const float2 u = make_float2(__shfl_xor(t.x, o), __shfl_xor(t.y, o));
        t = lane & o ? join(u, t) : join(t, u);
    }
    if (lane == 0) joined[w] = t;
    __syncthreads();
    t = join(join(joined[0], joined[1]), join(joined[2], joined[3]));
    const float ls = logf(t.y), k2 = LOG2E / a.temperature, at = t.x == -INFINITY ? 0.f : t.x;
    const Shares sh = shares_of<TEACHER>(a, r);
    const float ltot = TEACHER ? logf(sh.total) : 0.f;
    float s = 0.f;
    for (int j = threadIdx.x; j < a.entries; j += 256) {
        const long long from = (long long)r * a.entries + j;
        if (!entry_counts<TEACHER>(a, from)) continue;
        const float rel = TEACHER ? (a.teacher[from] - sh.top) / a.temperature : 0.f, q = TEACHER ? expf(rel) / sh.total : 1.f;
        const float left = LN2 * -fmaf(a.value[(size_t)i * a.entries + j], k2, -at) + ls;
        if (q != 0.f) s += q * ((rel - ltot) + left);
    }
    s = sum64(s);
    if (lane == 0) sums[w] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        a.lse[r] = LN2 * t.x + ls;
        a.loss[r] = a.temperature * a.temperature * ((sums[0] + sums[1]) + (sums[2] + sums[3]));
    }
}

// p - q of every listed entry of a row from its product (an id listed twice: p less both shares, in both places), by the row's weight
template <bool TEACHER>
__global__ __launch_bounds__(256) void loss_values_kernel(LossArgs a)
{
    const int i = blockIdx.x;
    if (i >= a.head->count) return;
    const int r = a.idx[i];
    const float lse = a.lse[r], k = 1.0f / a.temperature, weight = a.grad[r] / a.head->scale;
    const Shares sh = shares_of<TEACHER>(a, r);
    const long long at0 = (long long)r * a.entries;
    for (int j = threadIdx.x; j < a.entries; j += 256) {
        if (!entry_counts<TEACHER>(a, at0 + j)) continue;
        const int id = a.ids[at0 + j];
        float q = 1.f;
        if (TEACHER) {
            q = 0.f;
            for (int o = 0; o < a.entries; ++o)
                if (a.ids[at0 + o] == id && entry_counts<TEACHER>(a, at0 + o)) q += expf((a.teacher[at0 + o] - sh.top) / a.temperature) / sh.total;
        }
        float &v = a.value[(size_t)i * a.entries + j];
        v = weight * (expf(fmaf(v, k, -lse)) - q);
    }
}

template <bool TEACHER, class GT>
__global__ __launch_bounds__(256) void loss_scatter_kernel(LossArgs a, int v0, int vn)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int i = (int)(at / a.entries), j = (int)(at % a.entries);
    if (i >= a.head->count) return;
    const long long from = (long long)a.idx[i] * a.entries + j;
    const int v = a.ids[from] - v0;
    if (v < 0 || v >= vn || !entry_counts<TEACHER>(a, from)) return;
    store_one((GT *)a.G + (size_t)i * a.piece + v, a.value[at]);
}

void launch_loss_finish(hipStream_t s, const LossArgs &a, int parts)
{
    if (!a.rows) return;
    if (a.teacher) hipLaunchKernelGGL((loss_finish_kernel<true>), dim3(a.rows), dim3(256), 0, s, a, parts);
    else hipLaunchKernelGGL((loss_finish_kernel<false>), dim3(a.rows), dim3(256), 0, s, a, parts);
}

void launch_loss_values(hipStream_t s, const LossArgs &a)
{
    if (!a.rows) return;
    if (a.teacher) hipLaunchKernelGGL((loss_values_kernel<true>), dim3(a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((loss_values_kernel<false>), dim3(a.rows), dim3(256), 0, s, a);
}

void launch_loss_scatter(hipStream_t s, const LossArgs &a, int v0, int vn, bool g_bf16)
{
    if (!a.rows) return;
    const dim3 grid((unsigned)(((long long)a.rows * a.entries + 255) / 256));
    if (a.teacher) {
        if (g_bf16) hipLaunchKernelGGL((loss_scatter_kernel<true, bf16_t>), grid, dim3(256), 0, s, a, v0, vn);
        else hipLaunchKernelGGL((loss_scatter_kernel<true, float>), grid, dim3(256), 0, s, a, v0, vn);
    } else {
        if (g_bf16) hipLaunchKernelGGL((loss_scatter_kernel<false, bf16_t>), grid, dim3(256), 0, s, a, v0, vn);
        else hipLaunchKernelGGL((loss_scatter_kernel<false, float>), grid, dim3(256), 0, s, a, v0, vn);
    }
}

// ------------------------------------------------------------------ gradient to the hidden rows

// a workgroup writes the i-th row that counts from its sums, in order of the splits, and clears row i if that does not count
template <class HT, bool BF16>
__global__ __launch_bounds__(256) void hidden_grad_kernel(LossArgs a)
{
    const int i = blockIdx.x, count = a.head->count;
    if (i < count) {
        const int r = a.idx[i], splits = BF16 ? bf16_splits(a, count) : a.splits;
        const size_t apart = (size_t)(BF16 ? bf16_rows(a, count) : a.n_pad) * a.d_pad;
        const float c = a.head->scale * a.temperature;
        HT *out = (HT *)a.d_hidden + (long long)r * a.dhs;
        for (int j = threadIdx.x; j < a.dim; j += 256) {
            float v = 0.f;
            for (int p = 0; p < splits; ++p) v += a.acc[p * apart + (size_t)i * a.d_pad + j];
            store_one(out + j, c * v);
        }
    }
    if (a.state[i] != ROW_COUNTS) {
        HT *out = (HT *)a.d_hidden + (long long)i * a.dhs;
        for (int j = threadIdx.x; j < a.dim; j += 256) store_one(out + j, 0.f);
    }
}

void launch_loss_hidden_grad(hipStream_t s, const LossArgs &a, bool bf16)
{
    if (!a.rows) return;
    if (bf16) hipLaunchKernelGGL((hidden_grad_kernel<bf16_t, true>), dim3(a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((hidden_grad_kernel<float, false>), dim3(a.rows), dim3(256), 0, s, a);
}

}  // namespace tr
