// Products of the losses over the vocabulary on bf16 matrix instructions: both operands bf16, sums in fp32. The softmax and the probabilities also take fp32 rows over a bf16 head: a row
// is then the sum of three bf16 rows (planes), each what the ones before leave, rounded: 24 bits, and every product with the head is exact.
//
// Four products, all computed transposed (see vocab_loss_epilogues.h), C[n][m] = sum_k A[m][k] B[n][k]:
//   softmax, probabilities     m = vocabulary entry, n = row that counts, k = feature: both operands lie with k contiguous
//   gradient to the rows       m = feature, n = row, k = vocabulary entry of the piece: A is the head, whose k runs from row to row; B = G, k contiguous
//   gradient to the head       m = feature, n = vocabulary entry, k = row: both operands have k from row to row
// All in steps of 64 k. Both operands of a step are copied to LDS by direct loads, as they lie in memory; an operand with k from row to row is turned where it is read
// (the transposing LDS read). Within a tile the 16-byte pieces of a line (or the 32-byte pieces, where k runs from row to row) are permuted by the line, on the way in through
// the lanes' addresses, so that reads meet no bank conflicts. Three schedules:
//   turns_kernel    blocks of 256 x 256, for more than 256 rows. 6144 rows x 151936 x 896 (8192, three quarters of them counting) take 1510 us for the softmax, 1.11 PFLOP/s with
//                   the matrix pipes 52 % busy at 2.0 GHz; 2048 rows x 152064 x 3584 1790 us, 1.25 PFLOP/s, 61 % at 1.9 GHz (a library product of 8192^3: 1.30, of
//                   4096 x 151936 x 896: 0.98). Bound by power and copies together, 1.6 us a step, and by what lies between two blocks, 5 us: the exponentials.
//   stream_kernel   blocks of 256 x 64 or 128, for fewer rows. Bound by the head's bytes: 272 MB in 50 us, 5.4 TB/s, what copies reach here. Rows in planes, however many (300 of 500 rows x
//                   151936 x 896: softmax 250 us, probabilities 268, 0.98 and 0.91 PFLOP/s; on 32-bit instructions, 64 x 64, the probabilities took 872).
//   block_kernel    blocks of 128 x 128, where there are few blocks, and for the gradient to the head of few rows.
#include "vocab_loss_epilogues.h"
#include <algorithm>
#include <atomic>
#include <type_traits>

namespace tr {

namespace {

constexpr int BK = 64;                 // k per step
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ int wavefront() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t lane_off, const char *base)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds), "v"(lane_off), "s"(base) : "memory");
}
// own loads but the youngest N have landed, own LDS reads are done, then the workgroup's barrier
template <int N> __device__ __forceinline__ void landed_and_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (0 << 8) | ((N >> 4) << 14));   // vmcnt N, expcnt 7 (no wait), lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Matrix instructions of 16 x 16 x 32: in registers alone they sustain 1.97 PFLOP/s on random data where those of 32 x 32 x 16 sustain 1.74 (the chip's power bounds both), since
// they move half as much of the accumulators (softmax of 2048 rows x 152064 x 3584: 1867 -> 1780 us). An operand is 16 rows x 32 k, lane l holding k = 8 (l / 16) .. + 7 of row
// l mod 16; lane l of the result holds rows 4 (l / 16) .. + 3 of column l mod 16. Where m lies along memory in the result and k contiguous in A, A's rows are taken in pairs of
// operands over 32 rows, row 4 a + e of the first being 8 a + e and of the second 8 a + 4 + e, so that a lane's results of a pair are 8 in a run.

// How the pieces of a line of a tile are permuted (exclusive or). LDS has 64 banks of 4 bytes: the 16 lanes that a 16-byte read serves at a time have to meet 16
// different pieces of 256 bytes, two lines of 64 k; the 32 lanes of an 8-byte read 8 different pieces of 32 bytes, from 8 lines of one column. (Keyed by the
// lowest bits of the line instead, half of all LDS cycles were conflicts.)
template <bool PAIRED> __device__ __forceinline__ int row_key(int row) { return PAIRED ? ((row >> 1) & 1) | ((row >> 2) & 6) : (row >> 1) & 7; }
__device__ __forceinline__ int k_key(int k) { return ((k & 3) << 1) ^ ((k >> 3) & 1); }

__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14)); }   // lgkmcnt 0
template <int N> __device__ __forceinline__ void wait_all_but() { __builtin_amdgcn_s_waitcnt(N | (7 << 4) | (0 << 8)); }   // vmcnt N < 16 and lgkmcnt 0

// One operand's tile of T rows of its dimension x 64 k in LDS. KC: k contiguous in memory, LDS [row][64 k]; otherwise [64 k][T]. PAIRED: rows are read
// in pairs of operands. WAVES share the copying.
template <int T, bool KC, bool PAIRED, int WAVES> struct Tile {
    static constexpr bool K_CONTIGUOUS = KC;
    static constexpr int BYTES = T * BK * 2, COPIES = BYTES / 1024 / WAVES;
    static_assert(BYTES % (1024 * WAVES) == 0, "whole copies");
    static_assert(KC || T >= 128, "eight pieces of 32 bytes a line");

    uint32_t off[COPIES], krow[COPIES];
    const char *base;
    uint32_t ld, advance;

    // p: element (first row, first k) of the operand; ld: elements from one line of memory to the next; limit: rows (KC) or columns that exist from p on
    __device__ __forceinline__ void init(const bf16_t *p, long long ld_elems, int limit)
    {
        const int lane = threadIdx.x & 63, w = wavefront();
        base = (const char *)p;
        ld = (uint32_t)ld_elems * 2;
        advance = KC ? BK * 2 : BK * ld;
#pragma unroll
        for (int q = 0; q < COPIES; ++q) {
            const int g = w * COPIES + q;
            if (KC) {
                const int row = g * 8 + (lane >> 3), piece = (lane & 7) ^ row_key<PAIRED>(row);
                off[q] = (uint32_t)min(row, limit - 1) * ld + piece * 16;
                krow[q] = 0;
            } else {
                const int at = g * 1024 + lane * 16, k = at / (T * 2), in = at % (T * 2), piece = (in >> 5) ^ k_key(k), col = piece * 16 + ((in >> 4) & 1) * 8;
                krow[q] = k;
                off[q] = (uint32_t)min(col, limit - 8) * 2;
            }
        }
    }
    // copies of the next step into LDS at byte `lds`; kleft: lines that are left (read only where k runs from row to row)
    __device__ __forceinline__ void issue(uint32_t lds, int kleft)
    {
        const int w = wavefront();
#pragma unroll
        for (int q = 0; q < COPIES; ++q) {
            uint32_t o = off[q];
            if (!KC) o += min(krow[q], (uint32_t)(kleft - 1)) * ld;
            load_to_lds(lds + (w * COPIES + q) * 1024, o, base);
        }
        base += advance;
    }
};

// Reads matrix operands from a tile: N of them, of 16 rows each, from row r0 on (a multiple of 16 N); step KK of 32 k.
template <int T, bool KC, bool PAIRED, int N> struct Reader {
    uint32_t at[2];
    __device__ __forceinline__ void init(int r0)
    {
        const int lane = threadIdx.x & 63, in = lane & 15, g = lane >> 4;
        if (KC) {
            const int row = r0 + (PAIRED ? 8 * (in >> 2) + (in & 3) : in);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = row * (BK * 2) + (((kk * 4 + g) ^ row_key<PAIRED>(row)) << 4);
        } else {
            // groups of 16 lanes turn 4 (k) x 16 elements; lane 4 r + c brings k = r, columns of quad c, and gets its own column's four k
            const int r = in >> 2, c = in & 3;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = 8 * g + 4 * t + r;
                at[t] = k * (T * 2) + (((r0 >> 4) ^ k_key(k)) << 5) + c * 8;
            }
        }
    }
    template <int KK> __device__ __forceinline__ void read(uint32_t lds, bf16x8 (&o)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (KC) {
                const int rows = PAIRED ? (n >> 1) * 32 + (n & 1) * 4 : n * 16;      // (the key is the same there)
                o[n] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8 *>(lds + at[KK] + rows * BK * 2);
            } else {
                typedef __attribute__((address_space(3))) s16x4 *lp;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lp>(lds + (at[0] ^ (n << 5)) + KK * 32 * T * 2));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lp>(lds + (at[1] ^ (n << 5)) + KK * 32 * T * 2));
                o[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    }
};

template <int MI, int NI> __device__ __forceinline__ void clear(f32x4 (&c)[MI][NI])
{
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) c[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// c += a b, `PLANES` operands of b for every column in turn
template <int MI, int NI, int PLANES> __device__ __forceinline__ void multiply(f32x4 (&c)[MI][NI], const bf16x8 (&a)[MI], const bf16x8 (&b)[NI * PLANES])
{
#pragma unroll
    for (int l = 0; l < PLANES; ++l)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[l * NI + j], c[i][j], 0, 0, 0);
}

// WM x WN wavefronts, each MI x NI accumulators; A_KC, B_KC: where the operands have k contiguous. PLANES rows of B for every column.
template <int WM_, int WN_, int MI_, int NI_, bool A_KC, bool B_KC, int PLANES = 1> struct Shape {
    static constexpr int WM = WM_, WN = WN_, MI = MI_, NI = NI_, WAVES = WM * WN, TM = WM * MI * 16, TN = WN * NI * 16, PL = PLANES;
    using TA = Tile<TM, A_KC, A_KC, WAVES>;
    using TB = Tile<TN * PL, B_KC, false, WAVES>;
    using RA = Reader<TM, A_KC, A_KC, MI>;
    using RB = Reader<TN * PL, B_KC, false, NI * PL>;
};

// One block: STAGES steps in LDS, one barrier a step; the matrix operands of 32 k are read one such step ahead, across the barriers too (STAGES > 1).
template <int STAGES, class S> struct Block : S {
    using S::WM; using S::WN; using S::MI; using S::NI; using S::TM; using S::TN;
    using TA = typename S::TA;
    using TB = typename S::TB;
    static constexpr int STAGE = TA::BYTES + TB::BYTES, LDS = STAGES * STAGE, AT_ONCE = STAGES == 1 ? 4 : 3;   // (workgroups a compute unit)

    TA a;
    TB b;
    f32x4 c[MI][NI];

    // c += the products over K k; whole steps are copied, and what lies past K in the last has to be zero in one operand and finite in the other
    __device__ __forceinline__ void run(uint32_t lds, int K)
    {
        const int w = wavefront(), wm = w / WN, wn = w % WN, steps = (K + BK - 1) / BK;
        if (!steps) return;
        typename S::RA ra;
        typename S::RB rb;
        ra.init(wm * MI * 16);
        rb.init(wn * NI * 16);
        int left = K;
        auto issue = [&](int stage) {
            a.issue(lds + stage * STAGE, left);
            b.issue(lds + stage * STAGE + TA::BYTES, left);
            left -= BK;
        };
        bf16x8 xa[2][MI], xb[2][NI];
        if constexpr (STAGES == 1) {
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                issue(0);
                landed_and_barrier<0>();
                ra.template read<0>(lds, xa[0]); rb.template read<0>(lds + TA::BYTES, xb[0]);
                multiply<MI, NI, 1>(c, xa[0], xb[0]);
                ra.template read<1>(lds, xa[0]); rb.template read<1>(lds + TA::BYTES, xb[0]);
                landed_and_barrier<0>();
                multiply<MI, NI, 1>(c, xa[0], xb[0]);
            }
        } else {
            constexpr int COPIES = TA::COPIES + TB::COPIES;
#pragma unroll
            for (int p = 0; p < STAGES; ++p)
                if (p < steps) issue(p);
            if (steps >= STAGES) landed_and_barrier<(STAGES - 1) * COPIES>();
            else landed_and_barrier<0>();
            uint32_t at = lds;
            ra.template read<0>(at, xa[0]);
            rb.template read<0>(at + TA::BYTES, xb[0]);
            int stage = 0;
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                ra.template read<1>(at, xa[1]); rb.template read<1>(at + TA::BYTES, xb[1]);
                multiply<MI, NI, 1>(c, xa[0], xb[0]);
                // every wavefront holds the step's last operands: its place is free, and the next step's has landed
                if (s + STAGES <= steps) landed_and_barrier<(STAGES - 2) * COPIES>();
                else landed_and_barrier<0>();
                if (s + STAGES < steps) issue(stage);
                stage = stage + 1 < STAGES ? stage + 1 : 0;
                at = lds + stage * STAGE;
                if (s + 1 < steps) { ra.template read<0>(at, xa[0]); rb.template read<0>(at + TA::BYTES, xb[0]); }
                multiply<MI, NI, 1>(c, xa[1], xb[1]);
            }
        }
    }
};

extern __shared__ char dynamic_lds[];
__device__ __forceinline__ uint32_t lds_start() { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)dynamic_lds; }

// The order in which blocks are taken. Workgroup b runs on XCD b mod 8, whose workgroups take a contiguous piece of an order that walks groups of GN blocks along n
// and, in a group, along m: those that run at a time share GN tiles of one operand and a few of the other in the XCD's L2.
constexpr int GN = 8;        // (4 and 6: the same within 2 %)
struct Order {
    int mb, nb, first, end;      // first of this workgroup (of an XCD's first few), end of its XCD's
    __device__ __forceinline__ Order(int mb_, int nb_, int b) : mb(mb_), nb(nb_)
    {
        const int items = mb * nb, per = (items + 7) >> 3;
        first = (b & 7) * per + (b >> 3);
        end = min(items, ((b & 7) + 1) * per);
    }
    __device__ __forceinline__ Order() {}
    __device__ __forceinline__ void at(int i, int &m, int &n) const
    {
        const int group = i / (GN * mb), in = i - group * GN * mb, width = min(GN, nb - group * GN);
        m = in / width;
        n = group * GN + in - m * width;
    }
};

// Where a block's operands lie.
struct Place {
    const bf16_t *a, *b;
    long long lda, ldb;
    int a_limit, b_limit, n_limit, K, m, n, split;   // n_limit: rows of the product that exist from n's block on
};

__device__ __forceinline__ const bf16_t *head_rows(const LossArgs &a, int v0, long long &ld)
{
    ld = a.direct ? a.ws : a.d_pad;
    return a.direct ? (const bf16_t *)a.weight + (long long)v0 * a.ws : (const bf16_t *)a.wp;
}

// What a kernel does: its blocks of TM x TN and their order, the place of block i, and what becomes of a wavefront's accumulators.
template <int TM, int TN> struct Logits {
    static constexpr bool A_KC = true, B_KC = true;
    const LossArgs &a;
    int v0, vn, count, half, rows;
    Order o;
    __device__ __forceinline__ Logits(const LossArgs &a_, int v0_, int vn_, int, int b)
        : a(a_), v0(v0_), vn(vn_), count(a_.head->count), half(a_.grad ? a_.head->half : 0), rows(bf16_products_rows(count, half)), o((vn + TM - 1) / TM, (rows + TN - 1) / TN, b) {}
    __device__ __forceinline__ Place place(int i) const
    {
        Place p;
        o.at(i, p.m, p.n);
        p.a = head_rows(a, v0, p.lda);
        p.a += (long long)p.m * TM * p.lda;
        const int planes = a.hdt == DT_F32 ? 3 : 1;
        p.b = (const bf16_t *)a.hp + (size_t)p.n * TN * planes * a.d_pad;
        p.ldb = a.d_pad; p.a_limit = vn - p.m * TM; p.b_limit = TN * planes; p.n_limit = rows - p.n * TN; p.K = a.d_pad;
        return p;
    }
    template <int WN, int MI, int NI> __device__ __forceinline__ void start(const Place &, f32x4 (&c)[MI][NI]) const { clear(c); }
};

constexpr int LDS_OF_RING = 144 << 10;      // of stream_kernel at most; behind it what a block's wavefronts exchange

template <int TM, int TN> struct Softmax : Logits<TM, TN> {
    using Logits<TM, TN>::Logits;
    template <int WM, int WN, int MI, int NI> __device__ __forceinline__ void done(const Place &p, const f32x4 (&c)[MI][NI])
    {
        const LossArgs &a = this->a;
        const int lane = threadIdx.x & 63, w = wavefront(), wm = w / WN, wn = w % WN, m = p.m * TM + wm * MI * 16 + 8 * (lane >> 4);
        float2 *red = reinterpret_cast<float2 *>(dynamic_lds + (TM == 128 ? 0 : LDS_OF_RING)) + wm * TN + wn * NI * 16;   // (block_kernel: its LDS is free by then)
        constexpr bool JOIN = WM > 2 || TM == 128;       // few rows or small blocks: the wavefronts join their parts in LDS
        float2 *to = JOIN ? red : a.part + ((size_t)(this->v0 / TM + p.m) * WM + wm) * a.part_ld + p.n * TN + wn * NI * 16;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const float2 t = column_softmax<MI * 4>([&](int i) { return c[(i >> 3) * 2 + ((i >> 2) & 1)][j][i & 3]; }, [](int i) { return (i >> 3) * 32 + (i & 7); }, this->vn - m,
                                                    LOG2E / a.temperature, 16);
            if (lane < 16) to[j * 16 + lane] = t;
        }
        if constexpr (JOIN) {
            red -= wm * TN + wn * NI * 16;
            __syncthreads();
            for (int i = threadIdx.x; i < TN; i += WM * WN * 64) {
                float2 t = red[i];
#pragma unroll
                for (int q = 1; q < WM; ++q) t = join(t, red[q * TN + i]);
                a.part[(size_t)(this->v0 / TM + p.m) * a.part_ld + p.n * TN + i] = t;
            }
        }
    }
};

// GT: type of G. With fp32 rows (in planes) it is fp32, and a probability is the exponential that the listed entries have too, from lse as it is: no rounding of lse in units of ln 2.
template <int TM, int TN, class GT> struct ProbabilitiesIn : Logits<TM, TN> {
    using Logits<TM, TN>::Logits;
    static constexpr bool PLANES = sizeof(GT) == 4;
    LossRow row[4];
    // the rows' numbers, asked for before the products that they wait for
    template <int WN, int MI, int NI> __device__ __forceinline__ void start(const Place &p, f32x4 (&c)[MI][NI])
    {
        static_assert(NI <= 4, "rows held");
        clear(c);
#pragma unroll
        for (int j = 0; j < NI; ++j) row[j] = this->a.row[p.n * TN + (wavefront() % WN * NI + j) * 16 + (threadIdx.x & 15)];
    }
    template <int WM, int WN, int MI, int NI> __device__ __forceinline__ void done(const Place &p, const f32x4 (&c)[MI][NI])
    {
        const LossArgs &a = this->a;
        const int lane = threadIdx.x & 63, w = wavefront(), first = p.n * TN + w % WN * NI * 16, half = this->half;
        const float k2 = LOG2E / a.temperature, k = 1.0f / a.temperature;
        const int v0 = p.m * TM + w / WN * MI * 16 + 8 * (lane >> 4), there = this->vn - v0;   // entries that exist from this lane's first on
        const int needed = (this->rows + 63) / 64 * 64;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int at = first + j * 16;
            if (at >= needed) continue;               // (the products read whole steps of 64 rows)
            const bool second = half && at >= half;   // of a pair: what rounding leaves
            GT *to = (GT *)a.G + (size_t)(at + (lane & 15)) * a.g_ld + v0;
            const float lse2 = row[j].lse * LOG2E, weight = row[j].weight;
#pragma unroll
            for (int i = 0; i < MI; i += 2) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float product = c[i + (e >> 2)][j][e & 3];
                    x[e] = weight * (PLANES ? expf(fmaf(product, k, -row[j].lse)) : term(product, k2, lse2));
                }
                // rows that do not count and entries that do not exist: zeros, which the next products read
                if (this->vn < p.m * TM + TM || this->rows < p.n * TN + TN || half) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = weight != 0.f && i * 16 + e < there ? x[e] : 0.f;
                }
                if (second) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const uint32_t hi = two_bf16(x[e], x[e + 1]);
                        x[e] -= __uint_as_float(hi << 16);
                        x[e + 1] -= __uint_as_float(hi & 0xffff0000u);
                    }
                }
                store_run(to + i * 16, x);
            }
            const unsigned own = (unsigned)(row[j].target - this->v0 - v0);
            if (!__any(own < MI * 16)) continue;
            // cross entropy's few places of p - 1, once more (in the runs' own loop: 6144 rows x 151936 x 896 1815 us instead of 1730)
#pragma unroll
            for (int i = 0; i < MI; i += 2) {
                if (own - i * 16 >= 8) continue;
                const float x = less_one([&](int e) { return c[i + (e >> 2)][j][e & 3]; }, own - i * 16, weight, row[j].lse);
                if constexpr (PLANES) to[own] = x;
                else {
                    const bf16_t hi = (bf16_t)two_bf16(x, 0.f);
                    to[own] = second ? (bf16_t)two_bf16(x - load_one(&hi), 0.f) : hi;
                }
            }
        }
    }
};
template <int TM, int TN> struct Probabilities : ProbabilitiesIn<TM, TN, bf16_t> { using ProbabilitiesIn<TM, TN, bf16_t>::ProbabilitiesIn; };
template <int TM, int TN> struct PlaneProbabilities : ProbabilitiesIn<TM, TN, float> { using ProbabilitiesIn<TM, TN, float>::ProbabilitiesIn; };

// Every sum over the piece's vocabulary in `splits` parts (a power of two). A part belongs to 8 / splits XCDs, which share its blocks, or an XCD has splits / 8 whole parts: what an
// XCD reads of the head and of G, it reads alone, or with few.
template <int TM, int TN> struct HiddenGrad {
    static constexpr bool A_KC = false, B_KC = true;
    const LossArgs &a;
    int v0, vn, first, mb, nb, rows, splits, per, tiles;
    Order o;
    __device__ __forceinline__ HiddenGrad(const LossArgs &a_, int v0_, int vn_, int first_, int b) : a(a_), v0(v0_), vn(vn_), first(first_)
    {
        rows = bf16_products_rows(a.head->count, a.head->half);
        mb = (a.d_pad + TM - 1) / TM;
        nb = (rows + TN - 1) / TN;
        tiles = mb * nb;
        splits = bf16_splits(a, rows);
        per = ((vn + splits - 1) / splits + 63) / 64 * 64;
        o.mb = mb; o.nb = nb;
        const int x = b & 7, j = b >> 3;
        if (splits >= 8) {
            const int own = tiles * (splits >> 3);
            o.first = x * own + j;
            o.end = (x + 1) * own;
        } else {
            const int sharing = 8 / splits, own = (tiles + sharing - 1) / sharing, of = x / sharing * tiles;
            o.first = of + x % sharing * own + j;
            o.end = of + min(tiles, (x % sharing + 1) * own);
        }
    }
    __device__ __forceinline__ Place place(int i) const
    {
        Place p;
        p.split = i / tiles;
        o.at(i - p.split * tiles, p.m, p.n);
        const int k0 = min(vn, p.split * per);
        p.K = min(vn, k0 + per) - k0;
        p.a = head_rows(a, v0, p.lda);
        p.a += k0 * p.lda + p.m * TM; p.a_limit = a.d_pad - p.m * TM;
        p.b = (const bf16_t *)a.G + (size_t)p.n * TN * a.g_ld + k0; p.ldb = a.g_ld; p.b_limit = TN; p.n_limit = rows - p.n * TN;
        return p;
    }
    // where a wavefront's sums lie: f(accumulator, their place)
    template <int WN, int MI, int NI, class F> __device__ __forceinline__ void each(const Place &p, f32x4 (&c)[MI][NI], F f) const
    {
        const int lane = threadIdx.x & 63, w = wavefront(), d0 = p.m * TM + w / WN * MI * 16;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            float *at = a.acc + ((size_t)p.split * bf16_rows(a, rows) + p.n * TN + (w % WN * NI + j) * 16 + (lane & 15)) * a.d_pad + d0 + 4 * (lane >> 4);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (d0 + i * 16 >= a.d_pad) break;       // (d_pad: a multiple of 64)
                f(c[i][j], reinterpret_cast<f32x4 *>(at + i * 16));
            }
        }
    }
    // what the products are added to: the sums of the pieces before, all read at once (added at the end instead, a few at a time, as
    // registers allow: 6144 rows x 151936 x 896 in five pieces 2005 us, so 1890)
    template <int WN, int MI, int NI> __device__ __forceinline__ void start(const Place &p, f32x4 (&c)[MI][NI]) const
    {
        clear(c);
        if (first || p.K == 0) return;
        each<WN>(p, c, [](f32x4 &x, const f32x4 *at) { x = *at; });
        __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));       // vmcnt 0: here, not in the loop
    }
    template <int WM, int WN, int MI, int NI> __device__ __forceinline__ void done(const Place &p, f32x4 (&c)[MI][NI])
    {
        if (!first && p.K == 0) return;
        each<WN>(p, c, [](const f32x4 &x, f32x4 *at) { *at = x; });
    }
};

template <int TM, int TN> struct WeightGrad {
    static constexpr bool A_KC = false, B_KC = false;
    const LossArgs &a;
    int v0, vn, rows;
    Order o;
    __device__ __forceinline__ WeightGrad(const LossArgs &a_, int v0_, int vn_, int, int b)
        : a(a_), v0(v0_), vn(vn_), rows(bf16_products_rows(a_.head->count, a_.head->half)), o((a_.d_pad + TM - 1) / TM, (vn_ + TN - 1) / TN, b) {}
    __device__ __forceinline__ Place place(int i) const
    {
        Place p;
        p.n = i / o.mb;                   // all blocks of some rows of the head before the next rows: whole rows are written at a time
        p.m = i - p.n * o.mb;
        p.K = (rows + 63) / 64 * 64;      // G and the packed rows are zero from the last row that counts to there
        p.a = (const bf16_t *)a.hp + p.m * TM; p.lda = a.d_pad; p.a_limit = a.d_pad - p.m * TM;
        p.b = (const bf16_t *)a.G + p.n * TN; p.ldb = a.g_ld; p.b_limit = a.piece - p.n * TN; p.n_limit = vn - p.n * TN;
        return p;
    }
    template <int WN, int MI, int NI> __device__ __forceinline__ void start(const Place &, f32x4 (&c)[MI][NI]) const { clear(c); }
    template <int WM, int WN, int MI, int NI> __device__ __forceinline__ void done(const Place &p, const f32x4 (&c)[MI][NI])
    {
        const float k = a.head->scale * a.temperature;
        bf16_t *const out = (bf16_t *)a.d_weight + (long long)(v0 + p.n * TN) * a.dws + p.m * TM;
        const int vs = vn - p.n * TN, ds = a.dim - p.m * TM;      // what exists of the block
        const int lane = threadIdx.x & 63, w = wavefront(), d0 = w / WN * MI * 16 + 4 * (lane >> 4);
        auto rounded = [&](int i, int j) { return make_uint2(two_bf16(k * c[i][j][0], k * c[i][j][1]), two_bf16(k * c[i][j][2], k * c[i][j][3])); };
        if constexpr (TM == 128) {
            // through LDS, which is free by then, so that a row's stores are whole lines of memory: 16-byte pieces, permuted by the row
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int v = (w % WN * NI + j) * 16 + (lane & 15);
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const int d = d0 + i * 16;
                    *reinterpret_cast<uint2 *>(dynamic_lds + v * (TM * 2) + (((d >> 3) ^ (v & 15)) << 4) + (d & 4) * 2) = rounded(i, j);
                }
            }
            __syncthreads();
#pragma unroll 4
            for (int at = threadIdx.x; at < TN * 16; at += WM * WN * 64) {
                const int v = at >> 4, d = (at & 15) * 8;
                if (v >= vs || d >= ds) continue;
                const uint4 u = *reinterpret_cast<const uint4 *>(dynamic_lds + v * (TM * 2) + (((at & 15) ^ (v & 15)) << 4));
                bf16_t *to = out + (long long)v * a.dws + d;
                if (d + 8 <= ds) store_bits(to, u);
                else {
                    const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (d + e < ds) to[e] = (bf16_t)(q[e >> 1] >> (16 * (e & 1)));
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int v = (w % WN * NI + j) * 16 + (lane & 15);
                if (v >= vs) continue;
                bf16_t *to = out + (long long)v * a.dws + d0;
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const uint2 u = rounded(i, j);
                    if (d0 + i * 16 + 4 <= ds) store_bits(to + i * 16, u);
                    else {
                        const uint32_t q[2] = {u.x, u.y};
#pragma unroll
                        for (int e = 0; e < 4; ++e) if (d0 + i * 16 + e < ds) to[i * 16 + e] = (bf16_t)(q[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
        }
    }
};

// Products of listed entries: a wavefront takes 16 of them, its rows of the head against its packed rows, of which only the diagonal is kept: the matrix unit is
// all but idle in a product this small, and it gives the bits that the same pair has in a block (the same instruction over the same steps of k).
template <int PLANES> __device__ __forceinline__ void entries_group(const LossArgs &a, int group, bool packed)   // packed: the whole head is
{
    const int lane = threadIdx.x & 63, e = group * 16 + (lane & 15), g = lane >> 4, count = a.head->count;
    const int i = e / a.entries, j = e - i * a.entries;
    bool on = i < count;
    const bf16_t *h = (const bf16_t *)a.hp, *w = packed ? (const bf16_t *)a.wp : (const bf16_t *)a.weight;
    if (on) {
        const int id = a.ids[(long long)a.idx[i] * a.entries + j];
        on = id >= 0 && id < a.vocab;
        h += (size_t)(PLANES == 1 ? i : (i >> 6) * 64 * PLANES + (i & 63)) * a.d_pad;
        if (on) w = packed ? (const bf16_t *)a.wp + (size_t)id * a.d_pad : w + id * a.ws;
    }
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
    // N steps of 32 k, their loads requested together; ANYWHERE: the head's row may begin anywhere, PART: and end within the steps
    auto steps = [&](auto n, auto anywhere, auto part, int k0) {
        constexpr int N = decltype(n)::value;
        bf16x8 x[N], y[N][PLANES];
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int k = k0 + 32 * q + 8 * g;
            if constexpr (decltype(part)::value) x[q] = __builtin_bit_cast(bf16x8, load8(w, k, on ? a.dim : 0));
            else if constexpr (decltype(anywhere)::value) __builtin_memcpy(&x[q], w + k, 16);
            else x[q] = *reinterpret_cast<const bf16x8 *>(w + k);
#pragma unroll
            for (int l = 0; l < PLANES; ++l) y[q][l] = *reinterpret_cast<const bf16x8 *>(h + (size_t)l * 64 * a.d_pad + k);
        }
#pragma unroll
        for (int q = 0; q < N; ++q)
#pragma unroll
            for (int l = 0; l < PLANES; ++l) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[q], y[q][l], c, 0, 0, 0);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    constexpr int MOST = PLANES == 1 ? 14 : 8;
    using Many = std::integral_constant<int, MOST>;
    using One = std::integral_constant<int, 1>;
    int k = 0;
    if (a.direct || packed) {
        for (; k + 32 * MOST <= a.d_pad; k += 32 * MOST) steps(Many{}, No{}, No{}, k);
        for (; k < a.d_pad; k += 32) steps(One{}, No{}, No{}, k);
    } else {
        for (; k + 32 * MOST <= a.dim; k += 32 * MOST) steps(Many{}, Yes{}, No{}, k);
        for (; k < a.d_pad; k += 32) steps(One{}, Yes{}, Yes{}, k);
    }
    const int n = lane & 15;
    const float d = n & 2 ? (n & 1 ? c[3] : c[2]) : (n & 1 ? c[1] : c[0]);
    if (on && n >> 2 == g) a.value[e] = d;
}

// every `apart`-th group from `first` on
template <int PLANES> __device__ __forceinline__ void entries_from(const LossArgs &a, int first, int apart, bool packed)
{
    const long long all = (long long)a.head->count * a.entries;
    for (int group = first; (long long)group * 16 < all; group += apart) entries_group<PLANES>(a, group, packed);
}

__global__ __launch_bounds__(64) void bf16_entries_kernel(LossArgs a, bool packed) { entries_from<1>(a, blockIdx.x, gridDim.x, packed); }

// Few rows, bound by the head's bytes: one workgroup a compute unit takes block after block, the copies running on across blocks (a workgroup a block: 78 us for one row over
// 151936 x 896, so 63): rings of both operands' steps in LDS, one barrier a step. The first `extra` (a multiple of 8) workgroups take listed entries instead.
template <template <int, int> class Job_, class Sh> __global__ __launch_bounds__(Sh::WAVES * 64) void stream_kernel(LossArgs a, int v0, int vn, int flag, int extra)
{
    using Job = Job_<Sh::TM, Sh::TN>;
    if constexpr (Job::A_KC)
        if ((int)blockIdx.x < extra) {
            entries_from<Sh::PL>(a, blockIdx.x * Sh::WAVES + wavefront(), extra * Sh::WAVES, !a.direct && vn == a.vocab);
            return;
        }
    constexpr int MI = Sh::MI, NI = Sh::NI;
    constexpr int A_TILES = 3, B_TILES = Sh::PL > 1 ? 2 : 3;     // rings of both operands; B's (the rows, in L2) may be shorter
    constexpr int UNDER_WAY = A_TILES == B_TILES ? Sh::TA::COPIES + Sh::TB::COPIES : Sh::TA::COPIES;   // copies that may be, when a step's last have landed
    static_assert(A_TILES * Sh::TA::BYTES + B_TILES * Sh::TB::BYTES <= LDS_OF_RING, "LDS");
    Job job(a, v0, vn, flag, blockIdx.x - extra);
    const int begin = job.o.first, end = job.o.end, stride = (gridDim.x - extra) >> 3, w = wavefront();
    if (begin >= end) return;
    const uint32_t lds_a = lds_start(), lds_b = lds_a + A_TILES * Sh::TA::BYTES;
    typename Sh::TA ta;
    typename Sh::TB tb;
    int item_a = begin, item_b = begin, steps_a, steps_b, left_a, left_b, to_a = 0, to_b = 0;      // of the copies
    auto open_a = [&] {
        for (steps_a = 0; item_a < end; item_a += stride) {
            const Place p = job.place(item_a);
            if (p.K > 0) { steps_a = (p.K + BK - 1) / BK; left_a = p.K; ta.init(p.a, p.lda, p.a_limit); break; }
        }
    };
    auto open_b = [&] {
        for (steps_b = 0; item_b < end; item_b += stride) {
            const Place p = job.place(item_b);
            if (p.K > 0) { steps_b = (p.K + BK - 1) / BK; left_b = p.K; tb.init(p.b, p.ldb, p.b_limit); break; }
        }
    };
    auto copy_a = [&] {       // whether there was one
        if (!steps_a) return false;
        ta.issue(lds_a + to_a * Sh::TA::BYTES, left_a);
        to_a = to_a + 1 < A_TILES ? to_a + 1 : 0;
        left_a -= BK;
        if (--steps_a == 0) { item_a += stride; open_a(); }
        return true;
    };
    auto copy_b = [&] {
        if (!steps_b) return;
        tb.issue(lds_b + to_b * Sh::TB::BYTES, left_b);
        to_b = to_b + 1 < B_TILES ? to_b + 1 : 0;
        left_b -= BK;
        if (--steps_b == 0) { item_b += stride; open_b(); }
    };
    open_a();
    open_b();
    bool full = false;        // the copies that may be under way are
#pragma unroll
    for (int q = 0; q < A_TILES - 1; ++q) {
        if (q >= A_TILES - B_TILES) copy_b();
        full = copy_a();
    }
    static_assert(Sh::PL == 1 || Sh::WN == 1, "a row's planes belong to one wavefront");
    typename Sh::RA ra;
    typename Sh::RB rb;
    ra.init(w / Sh::WN * MI * 16);
    rb.init(w % Sh::WN * NI * 16);
    f32x4 c[MI][NI];
    int from_a = 0, from_b = 0;
#pragma unroll 1
    for (int it = begin; it < end; it += stride) {
        const Place p = job.place(it);
        job.template start<Sh::WN>(p, c);
#pragma unroll 1
        for (int s = (p.K + BK - 1) / BK; s; --s) {
            // this step has landed, and everyone has read the one before, whose places are the next copies'
            if (full) landed_and_barrier<UNDER_WAY>();
            else landed_and_barrier<0>();
            copy_b();
            full = copy_a();
            const uint32_t at_a = lds_a + from_a * Sh::TA::BYTES, at_b = lds_b + from_b * Sh::TB::BYTES;
            bf16x8 xa[2][MI], xb[2][NI * Sh::PL];
            ra.template read<0>(at_a, xa[0]); rb.template read<0>(at_b, xb[0]);
            ra.template read<1>(at_a, xa[1]); rb.template read<1>(at_b, xb[1]);
            multiply<MI, NI, Sh::PL>(c, xa[0], xb[0]);
            multiply<MI, NI, Sh::PL>(c, xa[1], xb[1]);
            from_a = from_a + 1 < A_TILES ? from_a + 1 : 0;
            from_b = from_b + 1 < B_TILES ? from_b + 1 : 0;
        }
        job.template done<Sh::WM, Sh::WN, MI, NI>(p, c);
    }
}

// One block a workgroup, the first `extra` (a multiple of 8) take listed entries. As many of them a compute unit as LDS has room for hide each other's copies: their registers
// are bounded for that (gradient to the head of 300 of 500 rows, 151936 x 896: 198 us where the compiler's choice left room for two, 138 with four).
template <template <int, int> class Job_, class Bl> __global__ __launch_bounds__(Bl::WAVES * 64, Bl::AT_ONCE) void block_kernel(LossArgs a, int v0, int vn, int flag, int extra)
{
    using Job = Job_<Bl::TM, Bl::TN>;
    if constexpr (Job::A_KC)
        if ((int)blockIdx.x < extra) {
            entries_from<1>(a, blockIdx.x * Bl::WAVES + wavefront(), extra * Bl::WAVES, !a.direct && vn == a.vocab);
            return;
        }
    Job job(a, v0, vn, flag, blockIdx.x - extra);
    if (job.o.first >= job.o.end) return;
    const Place p = job.place(job.o.first);
    Bl bl;
    bl.a.init(p.a, p.lda, p.a_limit);
    bl.b.init(p.b, p.ldb, p.b_limit);
    job.template start<Bl::WN>(p, bl.c);
    bl.run(lds_start(), p.K);
    job.template done<Bl::WM, Bl::WN, Bl::MI, Bl::NI>(p, bl.c);
}

// Blocks of 256 x 256, one workgroup a compute unit, block after block, the copies never stopping (softmax of 2048 rows x 152064 x 3584, a workgroup a block: 1977 us; in turns:
// 1881; copies running on: 1835; 1780 with the present instructions). 8 wavefronts of 128 x 64; the first four and the last four (one of each
// on every SIMD) take turns: while one reads its matrix operands of 32 k from LDS, the other's matrix instructions run. LDS holds five tiles, a step's two, A's of the next
// two steps and B's of the next: A (the operand that comes from beyond L2 more often) has two steps of time to arrive, B one.
template <template <int, int> class Job_> __global__ __launch_bounds__(512) void turns_kernel(LossArgs a, int v0, int vn, int flag)
{
    constexpr int WM = 2, WN = 4, MI = 8, NI = 4, T = 256, TILES = 5;
    using Job = Job_<T, T>;
    using Sh = Shape<WM, WN, MI, NI, Job::A_KC, Job::B_KC>;
    using TA = typename Sh::TA;
    using TB = typename Sh::TB;
    Job job(a, v0, vn, flag, blockIdx.x);
    const int begin = job.o.first, end = job.o.end, stride = gridDim.x >> 3, w = wavefront();
    if (begin >= end) return;
    const bool second = w >= 4;
    const uint32_t lds = lds_start();

    // the copies: an operand's next step, of this block or of the next that has any
    TA ta;
    TB tb;
    int ia = begin, ib = begin, steps_a, steps_b, left_a, left_b;
    auto open_a = [&] {
        for (steps_a = 0; ia < end; ia += stride) {
            const Place p = job.place(ia);
            if (p.K > 0) { steps_a = (p.K + BK - 1) / BK; left_a = p.K; ta.init(p.a, p.lda, p.a_limit); break; }
        }
    };
    auto open_b = [&] {
        for (steps_b = 0; ib < end; ib += stride) {
            const Place p = job.place(ib);
            if (p.K > 0) { steps_b = (p.K + BK - 1) / BK; left_b = p.K; tb.init(p.b, p.ldb, p.b_limit); break; }
        }
    };
    uint32_t to = lds;            // the next free tile
    auto turn = [&](uint32_t &t, int by) { t += by * TA::BYTES; t = t >= lds + TILES * TA::BYTES ? t - TILES * TA::BYTES : t; };
    auto copy_a = [&] {
        ta.issue(to, left_a);
        turn(to, 1);
        left_a -= BK;
        if (--steps_a == 0) { ia += stride; open_a(); }
    };
    auto copy_b = [&] {
        tb.issue(to, left_b);
        turn(to, 1);
        left_b -= BK;
        if (--steps_b == 0) { ib += stride; open_b(); }
    };
    auto barrier = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };

    open_a();
    open_b();
    if (steps_a) {
        copy_a();
        copy_b();
        if (steps_a) copy_a();    // two steps ahead of B from here on, as far as there are steps
        else turn(to, 1);
    }
    landed_and_barrier<0>();
    if (second) barrier();

    typename Sh::RA ra;
    typename Sh::RB rb;
    ra.init(w / WN * MI * 16);
    rb.init(w % WN * NI * 16);
    f32x4 c[MI][NI];
    bf16x8 xa[MI], xb[NI];
    auto products = [&] {
        __builtin_amdgcn_s_setprio(1);
        multiply<MI, NI, 1>(c, xa, xb);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    };
    uint32_t at_a = lds, at_b = lds + TA::BYTES;
#pragma unroll 1
    for (int item = begin; item < end; item += stride) {
        const Place p = job.place(item);
        const bool works = w / WN * MI * 16 < p.a_limit && w % WN * NI * 16 < p.n_limit;   // the last blocks: nothing is multiplied that does not exist
        job.template start<WN>(p, c);
#pragma unroll 1
        for (int s = (p.K + BK - 1) / BK; s; --s) {
            if (works) {
                ra.template read<0>(at_a, xa);
                rb.template read<0>(at_b, xb);
            }
            // the tiles of the step before are free: everyone has read them
            if (steps_b) copy_b();
            const bool ahead = steps_a > 0;
            if (ahead) copy_a();
            wait_lds();
            barrier();
            if (works) products();
            barrier();
            if (works) {
                ra.template read<1>(at_a, xa);
                rb.template read<1>(at_b, xb);
            }
            // before the barrier after which the next step is read: both its tiles are there, A's of the step after may be under way
            if (second) {
                if (ahead) wait_all_but<TA::COPIES>();
                else wait_all_but<0>();
            } else wait_lds();
            barrier();
            if (works) products();
            if (!second) {
                if (ahead) wait_all_but<TA::COPIES>();
                else wait_all_but<0>();
            }
            barrier();
            turn(at_a, 2);
            turn(at_b, 2);
        }
        job.template done<WM, WN, MI, NI>(p, c);
    }
    if (!second) barrier();
}

// (a thread takes eight elements, wherever rows begin: 28958 rows of 126 18 us with a workgroup a row, so 6)
__global__ __launch_bounds__(256) void bf16_pack_head_kernel(LossArgs a, int v0, int vn)
{
    const int eights = a.d_pad / 8;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int v = (int)(at / eights), k = (int)(at - (long long)v * eights) * 8;
    if (v < vn) *reinterpret_cast<uint4 *>((bf16_t *)a.wp + (size_t)v * a.d_pad + k) = load8((const bf16_t *)a.weight + (v0 + v) * a.ws, k, a.dim);
}

int up_div(int n, int by) { return (n + by - 1) / by; }

// (A kernel's dynamic LDS beyond 64 KiB has to be allowed once per device.)
template <auto KERNEL, class... A> void launch(dim3 grid, int threads, int lds, hipStream_t s, A... args)
{
    static std::atomic<uint64_t> allowed{0};
    int device = 0;
    (void)hipGetDevice(&device);
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit) && hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess)
        allowed.fetch_or(bit, std::memory_order_relaxed);
    hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, s, args...);
}

// Groups of listed entries; 2^20 rows of 1024 are 2^26, more than wavefronts that one launch may have (2^32 threads): beyond MOST_GROUPS a wavefront takes several.
int entry_groups(const LossArgs &a) { return (int)(((long long)a.rows * a.entries + 15) / 16); }
constexpr int MOST_GROUPS = 1 << 18;

// Where blocks of 256 x 256 would leave half of the chip without one, those of 128 x 128 (three a compute unit) are four times as many: 817 of 1021 rows x 5003 x 1001, softmax
// 30 -> 20 us. With more blocks the large ones are faster: 6144 x 151936 x 896 1545 us against 1793, 2048 x 152064 x 3584
// 1796 against 2106 (300 of 500 rows x 151936 x 896, softmax and probabilities: 291 both ways).
int product_rows(const LossArgs &a) { return a.pairs ? std::max(a.rows, 2 * PAIR_ROWS) : a.rows; }     // at most
bool small_blocks(int m, int n) { return up_div(m, 256) * up_div(n, 256) <= 128; }

// entries: listed entries too
template <template <int, int> class Job> void launch_job(hipStream_t s, const LossArgs &a, int v0, int vn, int flag, bool entries)
{
    constexpr bool A = Job<256, 64>::A_KC, B = Job<256, 64>::B_KC;
    const auto stream = [&](auto shape) {
        using Sh = decltype(shape);
        const int extra = entries ? up_div(std::min(entry_groups(a), MOST_GROUPS), 64) * 8 : 0;
        // a workgroup a compute unit: a few of them take entries only, since the head's bytes come as fast without them
        const dim3 persistent(extra <= 64 ? 256 : 256 + extra);
        launch<stream_kernel<Job, Sh>>(persistent, 512, LDS_OF_RING + Sh::WM * Sh::TN * (int)sizeof(float2), s, a, v0, vn, flag, extra);
    };
    constexpr bool PLANES = std::is_same_v<Job<256, 64>, PlaneProbabilities<256, 64>>;      // a job of fp32 rows alone
    if constexpr (PLANES || std::is_same_v<Job<256, 64>, Softmax<256, 64>>)
        if (a.hdt == DT_F32) { stream(Shape<8, 1, 2, 4, A, B, 3>{}); return; }
    if constexpr (!PLANES) {
        if (a.n_block == 64) stream(Shape<8, 1, 2, 4, A, B>{});
        else if (a.n_block == 128) stream(Shape<4, 2, 4, 4, A, B>{});
        else if (A && small_blocks(vn, product_rows(a))) {
            if constexpr (A) {
                using Bl = Block<2, Shape<2, 2, 4, 4, A, B>>;
                const int own = entries ? up_div(std::min(entry_groups(a), MOST_GROUPS), 32) * 8 : 0;
                launch<block_kernel<Job, Bl>>(dim3(own + up_div(up_div(vn, Bl::TM) * up_div(product_rows(a), Bl::TN), 8) * 8), 256, Bl::LDS, s, a, v0, vn, flag, own);
            }
        } else launch<turns_kernel<Job>>(dim3(256), 512, 5 * 256 * BK * 2, s, a, v0, vn, flag);
    }
}

}  // namespace

void launch_bf16_pack_head(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    hipLaunchKernelGGL(bf16_pack_head_kernel, dim3((unsigned)(((long long)vn * (a.d_pad / 8) + 255) / 256)), dim3(256), 0, s, a, v0, vn);
}

void launch_bf16_entries(hipStream_t s, const LossArgs &a, bool packed)
{
    hipLaunchKernelGGL(bf16_entries_kernel, dim3(std::min(entry_groups(a), MOST_GROUPS)), dim3(64), 0, s, a, packed);
}

void launch_bf16_softmax(hipStream_t s, const LossArgs &a, int v0, int vn, bool entries) { launch_job<Softmax>(s, a, v0, vn, 0, entries); }

// Which launches take the listed entries along: those of few rows, or of small blocks (two launches less of 6 us each, 817 of 1021 rows x 5003 x 1001). Beside many large blocks
// a launch of their own costs nothing, and would keep the persistent workgroups waiting.
bool bf16_takes_entries(const LossArgs &a, int vn) { return a.n_block < 256 || small_blocks(vn, product_rows(a)); }

// (blocks of 256 x 256 leave two parts each, those of 128 x 128 one, in the same places)
int bf16_softmax_parts(const LossArgs &a) { return up_div(a.vocab, a.n_block < 256 ? BF16_BLOCK : BF16_BLOCK / 2); }

void launch_bf16_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn, bool entries)
{
    if (a.hdt == DT_F32) launch_job<PlaneProbabilities>(s, a, v0, vn, 0, entries);
    else launch_job<Probabilities>(s, a, v0, vn, 0, entries);
}

void launch_bf16_hidden_grad(hipStream_t s, const LossArgs &a, int v0, int vn, bool first)
{
    launch_job<HiddenGrad>(s, a, v0, vn, first, false);
}

// Blocks of 256 x 256 or, several a compute unit, of 128 x 128 in one step's LDS: while one loads or stores another multiplies. Small ones
//   where there are few (small_blocks: 1280 rows x 275 x 1366 38 -> 24 us);
//   for few rows, where it is a matter of writing (300 of 500 rows x 151936 x 896: 139 us against 189; 1200 rows x 64000 x 3584 would be 1160 against 1073);
//   up to more rows for narrow heads whose last large blocks would be half empty (896 features, 4096 rows, three quarters of them counting: 850 against 960 us, 2048 rows x 64000 x 640
//   383 against 392; but 8192 rows x 64000 x 896 1930 against 1840, 2048 x 64000 x 1024 610 against 602, 8192 x 64000 x 1344 3040 against 2610).
void launch_bf16_weight_grad(hipStream_t s, const LossArgs &a, int v0, int vn)
{
    using Bl = Block<1, Shape<2, 2, 4, 4, false, false>>;
    const bool half_empty = a.d_pad < 1024 && a.d_pad % 256 && a.d_pad % 256 <= 128;
    const int blocks = up_div(a.d_pad, Bl::TM) * up_div(vn, Bl::TN);
    if (a.rows <= (half_empty ? 4096 : 1024) || small_blocks(a.d_pad, vn)) launch<block_kernel<WeightGrad, Bl>>(dim3(up_div(blocks, 8) * 8), 256, Bl::LDS, s, a, v0, vn, 0, 0);
    else launch<turns_kernel<WeightGrad>>(dim3(256), 512, 5 * 256 * BK * 2, s, a, v0, vn, 0);
}

}  // namespace tr
