// Declarations shared by the kernels of a reader's training step around its attention: embedding, dropout, layer norm, cross entropy
// over a vocabulary (gfx950 only).
#pragma once
#include "reader.h"

struct EmbedArgs {
    const char *table, *d_out;
    char *out, *d_table;
    const int64_t *ids;
    int64_t n, vocabulary, table_stride, d_out_stride;  // strides in bytes
    int32_t width, add;
    float scale;
    // gradient's workspace
    int32_t *keys[2], *places[2];      // tokens in ascending order, and where each stood; two of each where several launches sort
    int32_t *counts, *totals;          // [bins][blocks] of a pass, [bins]
    int32_t *shared, *begins;          // how many tokens several chunks share, and the chunks in which they begin
    int32_t sorted;                    // which of the two holds the result
    int32_t bits, passes, digit;       // bits of a key, passes, bits a pass
    int32_t chunk;                     // sorted places that a team of threads adds up
    float *part;                       // [chunks][2][columns()] sums of tokens that several chunks share
    __host__ __device__ int columns() const { return (width + 7) & ~7; }
};
// Up to this many tokens are sorted by one workgroup in one launch.
#define SORT_ONE 8192
#define SORT_TILE 1024
void plaid_launch_embedding(hipStream_t st, const EmbedArgs &e, int dtype);
void plaid_launch_embedding_backward(hipStream_t st, const EmbedArgs &e, int dtype);

void plaid_launch_dropout(hipStream_t st, const char *x, const char *residual, int64_t n, uint32_t threshold, const int64_t *rng, char *out, int dtype);

struct NormArgs {
    const char *x, *weight, *bias, *d_out;
    char *out, *dx, *dweight, *dbias;
    float *statistics;                 // [rows][2] mean, 1 / sqrt(variance + eps)
    int64_t rows, x_stride, d_out_stride;  // strides in bytes
    int32_t width, workers;
    float eps;
    float *part;                       // [workers][2][width] sums of dweight and dbias
};
#define NORM_WIDEST 16384
#define NORM_MANY 2048
void plaid_launch_layer_norm(hipStream_t st, const NormArgs &a, int dtype);
void plaid_launch_layer_norm_backward(hipStream_t st, const NormArgs &a, int dtype);

// Cross entropy.  Rows that have a target are packed first; what follows sees only those.
struct LossRow {
    int32_t target, exponent;          // d_loss = fraction 2^exponent
    float fraction, top, log_total;    // lse = top + log_total
};
struct LossArgs {
    const char *hidden, *weight;
    const int64_t *targets;
    const float *d_loss;
    float *loss, *lse;
    char *d_hidden, *d_weight;
    int64_t rows, vocabulary, hidden_stride, weight_stride, d_loss_stride;  // strides in bytes
    int32_t width;
    float scale;
    // workspace
    int32_t padded_rows, pitch;        // rows rounded up to LOSS_TILE, width to LOSS_STEP
    int32_t *state;                    // [0] rows that have a target, [1] the exponent that `scaled` is relative to
    int32_t *reach;                    // [rows] what each of them wants there, null where that is its exponent (bf16) or nothing is scaled
    int32_t *list;                     // [rows] which these are
    LossRow *row;                      // [padded_rows]
    char *packed;                      // [rows / 256][pitch / 64][256][64] states, with the sign of the scale
    char *scaled;                      // [rows / 64][columns / 256][64][256] the same times 2^(exponent - state[1])
    float2 *part;                      // [parts][padded_rows] largest product and sum of exponentials beside it over parts of the
                                       // vocabulary, without the target
    float2 *running;                   // [padded_rows] over all parts before
    float *own;                        // [padded_rows] product of the target
    char *gradient;                    // [rows / 256][piece / 256][256][256] of the scores, over a piece of the vocabulary
    float *d_part;                     // [parts][tiles of rows that have a target][columns / 256][256 x 256] sums of d_hidden, in the
                                       // order of the products' registers
    float *w_part;                     // [parts][piece / 256][columns / 256][256 x 256] the same of d_weight, null where its axis is never cut
    int32_t *target;                   // [padded_rows] LossRow::target alone
    float *rest;                       // [padded_rows] what the rounding of the target's entry of `gradient` left out
    int32_t columns;                   // width rounded up to LOSS_TILE
    int32_t hidden_steps;              // steps of a whole piece along d_hidden's axis
    int64_t first;                     // the piece's first entry, and how many there are
    int32_t piece, last;               // last: no piece comes after this one
};
#define LOSS_TILE 256
#define LOSS_STEP 64
#define LOSS_PART 128
#define LOSS_PART_STEPS 6
#define LOSS_PARTS 512  // tiles of all parts of d_hidden, where there are several
#define LOSS_FEW 128
#define LOSS_PREPARE_ONE 1536
// Tiles that the parts of d_hidden have at most, and those of d_weight where its axis may be cut, else 0.
constexpr int64_t loss_most_parts(int64_t tiles, int64_t steps)
{
    const int64_t most = steps < 4 ? 1 : steps / 4;
    return tiles > LOSS_PARTS ? tiles : tiles * most < LOSS_PARTS ? tiles * most : LOSS_PARTS;
}
constexpr int64_t loss_hidden_parts(int64_t padded_rows, int64_t columns, int64_t steps) { return loss_most_parts(padded_rows / LOSS_TILE * (columns / LOSS_TILE), steps); }
constexpr int64_t loss_weight_parts(int64_t padded_rows, int64_t columns, int64_t steps)
{
    const int64_t tiles = (steps + 3) / 4 * (columns / LOSS_TILE);
    return tiles < 256 ? loss_most_parts(tiles, padded_rows / LOSS_STEP) : 0;
}
void plaid_launch_loss_pack(hipStream_t st, const LossArgs &a, int dtype, bool backward);
void plaid_launch_loss_few(hipStream_t st, const LossArgs &a, int dtype, int entries, bool gradient);
void plaid_launch_loss_join(hipStream_t st, const LossArgs &a, int parts, bool packed);
void plaid_launch_loss_scores(hipStream_t st, const LossArgs &a, int dtype, bool backward);
void plaid_launch_loss_gradients(hipStream_t st, const LossArgs &a, int dtype);
void plaid_launch_loss_gradients_join(hipStream_t st, const LossArgs &a, int dtype);

#ifdef __HIP__
// An axis of a grid has fewer than 2^32 threads: more workgroups than WIDE_GRID, of up to 1024, take a second one, whose last row goes past the end.
#define WIDE_GRID (1 << 21)
inline dim3 wide_grid(int64_t blocks) { return blocks <= WIDE_GRID ? dim3((unsigned)blocks) : dim3(WIDE_GRID, (unsigned)((blocks + WIDE_GRID - 1) / WIDE_GRID)); }
__device__ __forceinline__ int64_t wide_block() { return (int64_t)blockIdx.y * WIDE_GRID + blockIdx.x; }

// Parts that the gradients' axes are cut into: the vocabulary's for d_hidden, the rows' for d_weight (where it has fewer tiles than the chip units).
// Both share a launch and fill up what the other leaves: so many that none takes longer than all together take on average (7296 rows of
// 2048 on 128000 entries, 160 tiles of d_hidden: one part, 4820 us for both gradients in place of 4960 with three at the time; 8000 rows of 256 on 5000
// entries, 20 tiles of d_weight: 64 us in place of 164 with one).  d_hidden alone: as few as leave least of the chip idle in the last round.  A
// part costs what LOSS_PART_STEPS steps of it cost, as its sums are written and read.
struct LossParts {
    int hidden, weight;
};
__device__ __forceinline__ LossParts loss_parts(const LossArgs &a, int live)
{
    const int widths = a.columns / LOSS_TILE, tiles = (live + LOSS_TILE - 1) / LOSS_TILE * widths, steps = a.hidden_steps;
    LossParts p = {1, 1};
    if (tiles == 0) return p;
    if (a.d_weight) {
        const int w_tiles = (steps + 3) / 4 * widths, w_steps = (live + LOSS_STEP - 1) / LOSS_STEP;
        const int64_t all = (a.d_hidden ? (int64_t)tiles * steps : 0) + (int64_t)w_tiles * w_steps;
        const int share = max((int)(all / 256), LOSS_PART_STEPS);
        p.hidden = max(1, min(min((steps + share - 1) / share, LOSS_PARTS / tiles), steps / 4));
        if (a.w_part) p.weight = max(1, min(min(w_steps / share, LOSS_PARTS / w_tiles), w_steps / 4));  // not for less than twice as long
        return p;
    }
    float least = 0.0f;
    for (int s = 1; s == 1 || (s * tiles <= LOSS_PARTS && 4 * s <= steps); ++s) {
        const float cost = (float)((tiles * s + 255) / 256) * ((float)steps / (float)s + LOSS_PART_STEPS);
        if (s == 1 || cost < 0.98f * least) p.hidden = s, least = cost;
    }
    return p;
}

// Scores s = scale h . W are formed from products u = h . W whose sign is that of the scale (the packed states carry it), so that the largest product
// has the largest score: statistics are those of products, and a score costs one multiply-add on its way into an exponential.
__device__ __forceinline__ float score_factor(const LossArgs &a) { return fabsf(a.scale); }
// The same for exponentials of base two.  A factor of zero would meet the infinities of entries that are left out; beside this one every
// product that is not huge is nothing as well.
#define LEAST_FACTOR 1e-30f
__device__ __forceinline__ float exponent_factor(const LossArgs &a) { return fmaxf(fabsf(a.scale), LEAST_FACTOR) * LOG2E; }

// G of a row, in units of its d_loss's power of two, times 2^15 in fp16: of a product, by the score it is.  The target's is the probability less
// one, formed so that it keeps its digits where the probability is almost one: its score is then `top`, rounded as the forward pass rounded it, so that
// the difference is exactly nothing and what is left is the logarithm beside it.  (Fused into the subtraction the product would keep what `top` lost, 2^-24 of
// the score, which is more than all the others' probabilities.)
//
// The others' differences from `top` are formed first, in one fused operation: the rounding of `top`, 2^-24 of the largest score, is what a probability is
// off by beside the products' own.  (Exponent and shift each scaled to base two before, for one operation less, cost 2^-22: scores of 2^20 that differ by a
// few units had probabilities off by a tenth.  Both directions of 7296 rows of 2048 on 128000 entries: 9280 to 9310 us in place of 9280.)
struct ScoreGradient {
    float scale, top, log_total, shift, factor;
    __device__ __forceinline__ ScoreGradient(const LossRow &x, const LossArgs &a, int dtype)
        : scale(fmaxf(score_factor(a), LEAST_FACTOR)), top(x.top), log_total(x.log_total), shift(x.log_total * LOG2E),
          factor(x.fraction * (dtype == PLAID_FP16 ? 0x1p15f : 1.0f))
    {
    }
    __device__ __forceinline__ float other(float product) const
    {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(__builtin_fmaf(product, scale, -top), LOG2E, -shift)) * factor;
    }
    __device__ __forceinline__ float target(float product) const
    {
#pragma clang fp contract(off)
        const float score = product * scale;
        return expm1f((score - top) - log_total) * factor;
    }
};
// The target's entry of G rounds like the others, but a row has nothing larger, so that its rounding alone would be as much of a gradient's error as the
// result's own: what it left out is kept in 32 bits, and both gradients add its product.  (Where it is no number, they need no digits.)
template <int DT>
__device__ __forceinline__ float left_out(float g)
{
    const float rest = g - unpack<DT>(pack2<DT>(g, 0.0f), 0);
    return fabsf(rest) < INFINITY ? rest : 0.0f;
}

// Sixteen bytes of a row that starts at any element: the memory system takes such addresses.
typedef i32x4 __attribute__((aligned(2))) i32x4_any;

struct Eight {
    float x[8];
};
template <int DT>
__device__ __forceinline__ Eight unpack8(i32x4 w)
{
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.x[2 * i] = unpack<DT>(w[i], 0), r.x[2 * i + 1] = unpack<DT>(w[i], 1);
    return r;
}
template <int DT>
__device__ __forceinline__ i32x4 pack8(const Eight &r)
{
    return i32x4{pack2<DT>(r.x[0], r.x[1]), pack2<DT>(r.x[2], r.x[3]), pack2<DT>(r.x[4], r.x[5]), pack2<DT>(r.x[6], r.x[7])};
}
// Elements at .. at + 7 of a row of `width`; those past its end are zero, and not read.
__device__ __forceinline__ i32x4 load_piece(const char *row, int at, int width)
{
    if (at + 8 <= width) return *(const i32x4_any *)(row + 2 * at);
    i32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (at + i < width) w[i / 2] |= (int)((uint32_t) * (const uint16_t *)(row + 2 * (at + i)) << (16 * (i & 1)));
    return w;
}
__device__ __forceinline__ void store_piece(char *row, int at, int width, i32x4 w)
{
    if (at + 8 <= width) {
        *(i32x4_any *)(row + 2 * at) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (at + i < width) *(uint16_t *)(row + 2 * (at + i)) = (uint16_t)((uint32_t)w[i / 2] >> (16 * (i & 1)));
}
#endif
