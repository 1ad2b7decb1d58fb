// Losses over the vocabulary: what the host side (vocab_loss_api.hip) and the kernels share.
//
// z[r][v] = k * hidden[r] . weight[v] (k = 1 / temperature), lse[r] = log sum_v exp z[r][v]. A row's loss compares softmax(z) with shares q over a few
// listed entries of the vocabulary: one entry of share 1 (cross entropy), or the softmax of a teacher's logits (distillation). The gradient to the
// products hidden . weight is T g (p - q), p = exp(z - lse), g the row's weight; it exists only in pieces of the vocabulary, as a matrix G of the piece's
// g / max |g| (p - q).
//
// Only rows that count take part: they are listed once per call (`idx`) and everything behind works on that list, so that masked rows cost nothing and
// whatever their hidden rows hold reaches neither gradient.
#pragma once
#include "tr_internal.h"

namespace tr {

struct LossHead {
    int count;      // rows that count
    int half;       // > 0: rows of G in pairs, see below
    float scale;    // largest |weight| of a row that counts
    int pad;
};
// Pairs: with 32 rows or fewer (bf16 products) G has a second row for every row, `half` (32) rows further on, with what rounding the first to bf16 left, and the packed rows are
// there twice. The products are bound by the head's bytes then and take 64 rows at no more cost, and few rows average few roundings. (Up to 64 rows: gradients of 50 rows x 151936 x
// 896 250 us against 212; up to 128: 100 rows 340 against 248.)
constexpr int PAIR_ROWS = 32;

// What the probabilities of a row of products need (gradients, bf16 products); rows that are none have weight 0.
struct alignas(16) LossRow { float lse, weight; int target, none; };    // target: cross entropy's entry

struct LossArgs {
    const void *hidden, *weight;
    long long hs, ws;             // elements from row to row
    int hdt, wdt;                 // DT_*
    int rows, dim, vocab, entries;
    const int *ids;               // [rows][entries]
    const float *teacher;         // [rows][entries], NULL: every row's one entry has share 1
    float temperature;
    const float *grad;            // [rows] weights of the rows' losses (gradients only)
    float *loss, *lse;            // [rows]; gradients read lse
    void *d_hidden, *d_weight;    // either may be NULL
    long long dhs, dws;
    // workspace
    LossHead *head;
    int *idx;                     // [n_pad] rows that count, in order
    unsigned char *state;         // [rows] ROW_*
    float2 *part;                 // [parts of the vocabulary][part_ld] running softmaxes
    float *value;                 // [n_pad][entries] products of the listed entries, then what G has there
    void *G;                      // [n_pad][g_ld], a piece's columns; lines are not a power of two apart, so that a column's do not meet in one memory channel
    float *acc;                   // [splits][n_pad, or the blocks that count (bf16)][d_pad] sums of the gradient to the hidden rows
    void *hp;                     // [n_pad][d_pad] rows that count (bf16 products), fp32 rows in three planes
    LossRow *row;                 // [n_pad] theirs
    void *wp;                     // [piece][d_pad] rows of the head where they cannot be read as they lie
    int n_pad, d_pad, piece, g_ld, splits, part_ld;
    int pairs;                    // rows may be in pairs (gradients, bf16 products)
    int n_block;                  // rows per block (bf16 products)
    bool direct;                  // the head is read as it lies (bf16 products): rows on 16 bytes, whole steps of 64 features
};

enum { ROW_SKIP = 0, ROW_COUNTS = 1, ROW_BAD = 2 };

constexpr int LOSS_MAX_ENTRIES = 1024;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Rows that count, their list, zeros (NaN for an id at or past the vocabulary) for the others; the rows packed for bf16 products.
void launch_loss_rows(hipStream_t s, const LossArgs &a);
// lse and loss of the rows that count from `parts` running softmaxes each.
void launch_loss_finish(hipStream_t s, const LossArgs &a, int parts);
// From the products of the listed entries: what G has for them, and their places in G for one piece of the vocabulary (place: both at once, for a vocabulary of one piece).
void launch_loss_values(hipStream_t s, const LossArgs &a, bool place);
void launch_loss_scatter(hipStream_t s, const LossArgs &a, int v0, int vn);
// The gradient to the hidden rows from the splits' sums (as the bf16 or the f32 products leave them), weighed and rounded; zeros for rows that do not count.
void launch_loss_hidden_grad(hipStream_t s, const LossArgs &a);

// Products of the listed entries, each the bits that the softmax's and the probabilities' own products have, for every pair of types: the products' roundings are the same in z and in lse,
// so that nothing of them is left in lse - z and 1 - p where p is near 1. A loss has no rounding of lse in it either; a gradient is given lse as fp32, and 1 - p keeps that rounding, 2^-24 |lse|.
void launch_bf16_entries(hipStream_t s, const LossArgs &a, bool packed);   // packed: a.wp holds the whole head

// Products on 32-bit matrix instructions, any stride (vocab_loss_f32_kernels.hip): fp32 rows and head, the gradients over a bf16 head too. Blocks of 64 x 64. The
// softmax and the first piece's probabilities bring the products of the listed entries.
constexpr int F32_BLOCK = 64;
void launch_f32_softmax(hipStream_t s, const LossArgs &a);
int f32_softmax_parts(const LossArgs &a);
void launch_f32_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn);
void launch_f32_gradients(hipStream_t s, const LossArgs &a, int v0, int vn, bool first);     // those asked for

// bf16 rows and head (vocab_loss_bf16_kernels.hip): blocks of 256 vocabulary entries or features. Softmax and probabilities of fp32 rows over a bf16 head too.
constexpr int BF16_BLOCK = 256;
void launch_bf16_pack_head(hipStream_t s, const LossArgs &a, int v0, int vn);
// entries: the listed entries' products too, in the same launch (blocks of fewer than 256 rows only)
void launch_bf16_softmax(hipStream_t s, const LossArgs &a, int v0, int vn, bool entries);
int bf16_softmax_parts(const LossArgs &a);
bool bf16_takes_entries(const LossArgs &a, int vn);      // the softmax and the probabilities of a piece of vn entries take the listed ones along
void launch_bf16_probabilities(hipStream_t s, const LossArgs &a, int v0, int vn, bool entries);
void launch_bf16_hidden_grad(hipStream_t s, const LossArgs &a, int v0, int vn, bool first);
void launch_bf16_weight_grad(hipStream_t s, const LossArgs &a, int v0, int vn);
#ifdef __HIPCC__
__host__ __device__ inline int bf16_products_rows(int count, int half) { return half ? 2 * half : count; }
__host__ __device__ inline int bf16_rows(const LossArgs &a, int rows) { return (rows + a.n_block - 1) / a.n_block * a.n_block; }   // whole blocks
// Splits of the sums of the gradient to `rows` rows (of products), a power of two, at most a.splits: those for which a workgroup a compute unit is done first, when it takes
// `tiles` * n blocks, 256 at a time, of (steps / n + SPLIT_COST) steps of 64 k each; the sums' reading and writing costs a block about as much as that many steps.
// (6144 rows x 151936 x 896, 8 splits instead of 2: 2060 -> 1890 us; 2048 x 152064 x 3584: 2114 -> 2347 us, so 2.)
constexpr int SPLIT_COST = 16;
__host__ __device__ inline int bf16_splits(const LossArgs &a, int rows)
{
    const int tiles = (rows + a.n_block - 1) / a.n_block * ((a.d_pad + BF16_BLOCK - 1) / BF16_BLOCK), steps = (a.piece + 63) / 64;
    int best = 1, least = 0x7fffffff;
    for (int n = 1; n <= a.splits && (n <= 8 || tiles * n <= 256) && (n == 1 || tiles < 1024); n *= 2) {
        const int time = (tiles * n + 255) / 256 * ((steps + n - 1) / n + SPLIT_COST);
        if (time < least) { least = time; best = n; }
    }
    return best;
}
#endif

}  // namespace tr
