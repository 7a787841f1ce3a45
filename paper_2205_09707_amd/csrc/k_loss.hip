// Cross entropy over a vocabulary: what goes before and after its products, and the scores of a few rows.
#include "train.h"

// With s_tv = scale h_t . W_v:  lse_t = log sum_v exp s_tv, loss_t = lse_t - s_t,target, and for gradients
//   G_tv = d_loss_t (exp(s_tv - lse_t) - [v = target_t]),  dh_t = scale sum_v G_tv W_v,  dW_v = scale sum_t G_tv h_t.
// Scores are never kept: the products' kernels (k_loss_mm.hip) leave a maximum and a sum of exponentials for each part of the vocabulary,
// joined here.  lse is kept as two numbers, the maximum and the logarithm of the sum beside it, so that a probability near one keeps its
// distance from one.

// --- rows that have a target ----------------------------------------------------------------------------------------------------
// One workgroup numbers them; the others have a loss of zero.  A row's place goes by those before it, so the order is the caller's.
// Backward, d_loss = fraction 2^exponent: the fraction goes into G, which rounds to the type before it is multiplied, the power of two
// into what G is multiplied with, where it is exact, so that G in fp16 stays in its range however small the gradient of a mean is.
#define NO_EXPONENT (-100000)
__global__ __launch_bounds__(1024) void loss_list_kernel(LossArgs a, int backward)
{
    __shared__ int wave_sum[16], wave_top[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0, top = NO_EXPONENT;
    for (int64_t first = 0; first < a.rows; first += 1024) {
        const int64_t t = first + threadIdx.x;
        const int64_t target = t < a.rows ? a.targets[t] : -1;
        const bool live = target >= 0 && target < a.vocabulary;
        const uint64_t votes = __ballot(live);
        if (lane == 0) wave_sum[wave] = __popcll(votes);
        __syncthreads();
        int at = before + __popcll(votes & ((1ull << lane) - 1)), all = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += wave_sum[w];
            all += wave_sum[w];
        }
        before += all;
        if (live) {
            a.list[at] = (int)t;
            LossRow r = {(int)target, 0, 0.0f, 0.0f, 0.0f};
            if (backward) {
                const float d = *(const float *)((const char *)a.d_loss + t * a.d_loss_stride);
                if (fabsf(d) < INFINITY) r.fraction = frexpf(d, &r.exponent);
                else r.fraction = d;
                if (d == 0.0f) r.exponent = NO_EXPONENT;
                top = max(top, r.exponent);
                r.top = a.lse[2 * t], r.log_total = a.lse[2 * t + 1];
            }
            a.row[at] = r;
        } else if (!backward && t < a.rows) {
            a.loss[t] = 0.0f;
            if (a.lse) *(float2 *)(a.lse + 2 * t) = {0.0f, 0.0f};
        }
        __syncthreads();
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
    if (lane == 0) wave_top[wave] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < 16; ++w) top = max(top, wave_top[w]);
        a.state[0] = before, a.state[1] = top == NO_EXPONENT ? 0 : top;
    }
}

// Their states, packed; zeros up to a whole tile of rows and a whole step of columns.  A workgroup has a row.
template <int DT, bool BACKWARD>
__global__ __launch_bounds__(128) void loss_pack_kernel(LossArgs a)
{
    const int live = uniform_load(a.state), top = uniform_load(a.state + 1), i = blockIdx.x;
    if (i >= (live + LOSS_TILE - 1) / LOSS_TILE * LOSS_TILE) return;
    const bool there = i < live;
    const char *from = a.hidden + (there ? (int64_t)uniform_load(a.list + i) : 0) * a.hidden_stride;
    char *to = a.packed + (int64_t)i * a.pitch * 2, *scaled = BACKWARD ? a.scaled + (int64_t)i * a.pitch * 2 : nullptr;
    float power = 1.0f;
    if (BACKWARD && there) {
        const int e = uniform_load(&a.row[i].exponent);
        if (e != NO_EXPONENT) power = ldexpf(1.0f, e - top);
    }
    for (int at = threadIdx.x * 8; at < a.pitch; at += 1024) {
        const i32x4 w = there && at < a.width ? *(const i32x4 *)(from + 2 * at) : i32x4{0, 0, 0, 0};
        *(i32x4 *)(to + 2 * at) = w;
        if (BACKWARD) {
            Eight v = unpack8<DT>(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v.x[j] *= power;
            *(i32x4 *)(scaled + 2 * at) = pack8<DT>(v);
        }
    }
}

// A row without a target has no gradient.
__global__ __launch_bounds__(128) void loss_zero_kernel(LossArgs a)
{
    const int64_t t = blockIdx.x, target = uniform_load(a.targets + t);
    if (target >= 0 && target < a.vocabulary) return;
    for (int at = threadIdx.x * 8; at < a.width; at += 1024) *(i32x4 *)(a.d_hidden + (t * a.width + at) * 2) = i32x4{0, 0, 0, 0};
}

void plaid_launch_loss_pack(hipStream_t st, const LossArgs &a, int dtype, bool backward)
{
    loss_list_kernel<<<1, 1024, 0, st>>>(a, backward);
    const unsigned grid = (unsigned)a.padded_rows;
    if (!backward) loss_pack_kernel<PLAID_BF16, false><<<grid, 128, 0, st>>>(a);
    else if (dtype == PLAID_BF16) loss_pack_kernel<PLAID_BF16, true><<<grid, 128, 0, st>>>(a);
    else loss_pack_kernel<PLAID_FP16, true><<<grid, 128, 0, st>>>(a);
    if (backward && a.d_hidden) loss_zero_kernel<<<(unsigned)a.rows, 128, 0, st>>>(a);
}

// --- few rows -------------------------------------------------------------------------------------------------------------------
// The vocabulary's rows go straight from memory into registers, the operand of the matrix instruction, and are read once; the states come
// out of the caches.  A wave has 16 BLOCKS entries and up to 16 GROUPS rows.
template <int DT, int BLOCKS, int GROUPS>
__global__ __launch_bounds__(256) void loss_few_kernel(LossArgs a)
{
    constexpr int STEP = 32;
    const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), v0 = wave * (16 * BLOCKS);
    if (v0 >= a.vocabulary) return;
    const char *w[BLOCKS], *h[GROUPS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) w[i] = a.weight + min(v0 + 16 * i + l, a.vocabulary - 1) * a.weight_stride + 16 * q;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) h[i] = a.hidden + min((int64_t)16 * i + l, a.rows - 1) * a.hidden_stride + 16 * q;
    f32x4 acc[BLOCKS][GROUPS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const int whole = a.width / STEP;
#pragma unroll 4
    for (int s = 0; s < whole; ++s) {
        i32x4 x[BLOCKS], y[GROUPS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) x[i] = *(const i32x4 *)(w[i] + s * (2 * STEP));
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) y[j] = *(const i32x4 *)(h[j] + s * (2 * STEP));
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) acc[i][j] = mfma16<DT>(x[i], y[j], acc[i][j]);
    }
    if (whole * STEP < a.width) {
        const bool there = whole * STEP + 8 * q < a.width;
        const i32x4 zero = {0, 0, 0, 0};
        i32x4 x[BLOCKS], y[GROUPS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) x[i] = there ? *(const i32x4 *)(w[i] + whole * (2 * STEP)) : zero;
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) y[j] = there ? *(const i32x4 *)(h[j] + whole * (2 * STEP)) : zero;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) acc[i][j] = mfma16<DT>(x[i], y[j], acc[i][j]);
    }
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        const int64_t t = 16 * j + l;
        const int64_t target = t < a.rows ? a.targets[t] - v0 : -1;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int v = 16 * i + 4 * q + r;
                float s = acc[i][j][r] * a.scale;
                if (v0 + v >= a.vocabulary) s = -INFINITY;
                else if (v == target) a.own[t] = s;
                acc[i][j][r] = s;
                most = fmaxf(most, s);
            }
        most = max_halves(max_rows(most));
        const float base = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * LOG2E);
        sum = sum_halves(sum_rows(sum));
        if (lane < 16 && t < a.rows) a.part[wave * a.padded_rows + t] = {most, sum};
    }
}

void plaid_launch_loss_few(hipStream_t st, const LossArgs &a, int dtype, int blocks)
{
    const int groups = (int)((a.rows + 15) / 16);
    const unsigned grid = (unsigned)((a.vocabulary + 64 * blocks - 1) / (64 * blocks));
#define GO(DT, B, G) loss_few_kernel<DT, B, G><<<grid, 256, 0, st>>>(a)
#define GROUPS(DT, B) (groups == 1 ? GO(DT, B, 1) : groups == 2 ? GO(DT, B, 2) : groups == 3 ? GO(DT, B, 3) : GO(DT, B, 4))
    if (dtype == PLAID_BF16) blocks == 1 ? GROUPS(PLAID_BF16, 1) : GROUPS(PLAID_BF16, 4);
    else blocks == 1 ? GROUPS(PLAID_FP16, 1) : GROUPS(PLAID_FP16, 4);
#undef GROUPS
#undef GO
}

// --- parts joined ---------------------------------------------------------------------------------------------------------------
// ROWS rows a workgroup; its threads of one row take the parts in turn.  With the last piece come the loss and lse.
__device__ __forceinline__ float2 join_parts(float2 x, float2 y)
{
    const float m = fmaxf(x.x, y.x), base = m == -INFINITY ? 0.0f : m;
    return {m, x.y * __builtin_amdgcn_exp2f((x.x - base) * LOG2E) + y.y * __builtin_amdgcn_exp2f((y.x - base) * LOG2E)};
}
template <int ROWS>
__global__ __launch_bounds__(256) void loss_join_kernel(LossArgs a, int parts, int packed)
{
    constexpr int SHARES = 256 / ROWS;
    __shared__ float2 lds[SHARES][ROWS];
    const int r = threadIdx.x % ROWS, share = threadIdx.x / ROWS, live = packed ? uniform_load(a.state) : (int)a.rows;
    const int i = blockIdx.x * ROWS + r;
    float2 x = {-INFINITY, 0.0f};
    if (i < live) {
#pragma unroll 4
        for (int p = share; p < parts; p += SHARES) x = join_parts(x, a.part[(int64_t)p * a.padded_rows + i]);
    }
    lds[share][r] = x;
    __syncthreads();
    if (share != 0 || i >= live) return;
    for (int s = 1; s < SHARES; ++s) x = join_parts(x, lds[s][r]);
    if (a.first > 0) x = join_parts(a.running[i], x);
    if (!a.last) {
        a.running[i] = x;
        return;
    }
    const int64_t t = packed ? (int64_t)a.list[i] : i;
    const bool there = packed || (a.targets[t] >= 0 && a.targets[t] < a.vocabulary);
    const float rest = logf(x.y);
    a.loss[t] = there ? (x.x - a.own[i]) + rest : 0.0f;
    if (a.lse) *(float2 *)(a.lse + 2 * t) = there ? float2{x.x, rest} : float2{0.0f, 0.0f};
}

void plaid_launch_loss_join(hipStream_t st, const LossArgs &a, int parts, bool packed)
{
    if (a.rows >= 4096) loss_join_kernel<32><<<(unsigned)((a.rows + 31) / 32), 256, 0, st>>>(a, parts, packed);
    else if (a.rows >= 512) loss_join_kernel<8><<<(unsigned)((a.rows + 7) / 8), 256, 0, st>>>(a, parts, packed);
    else loss_join_kernel<1><<<(unsigned)a.rows, 256, 0, st>>>(a, parts, packed);
}

// --- gradient of the states: the splits' sums added up, in order ------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(128) void loss_d_hidden_join_kernel(LossArgs a)
{
    const int i = blockIdx.x;
    if (i >= uniform_load(a.state)) return;
    const int64_t t = uniform_load(a.list + i);
    const int e = uniform_load(&a.row[i].exponent);
    // the power of two last, where the result may leave the normal range
    const float factor = a.scale * (DT == PLAID_FP16 ? 0x1p-15f : 1.0f);
    for (int at = threadIdx.x * 8; at < a.width; at += 1024) {
        Eight v = {};
        for (int s = 0; s < a.splits; ++s) {
            const float *p = a.d_part + ((int64_t)s * a.padded_rows + i) * a.columns + at;
            const f32x4 x = *(const f32x4 *)p, y = *(const f32x4 *)(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v.x[j] += x[j], v.x[4 + j] += y[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v.x[j] = ldexpf(v.x[j] * factor, e == NO_EXPONENT ? 0 : e);
        *(i32x4 *)(a.d_hidden + (t * a.width + at) * 2) = pack8<DT>(v);
    }
}
void plaid_launch_loss_d_hidden_join(hipStream_t st, const LossArgs &a, int dtype)
{
    if (dtype == PLAID_BF16) loss_d_hidden_join_kernel<PLAID_BF16><<<(unsigned)a.rows, 128, 0, st>>>(a);
    else loss_d_hidden_join_kernel<PLAID_FP16><<<(unsigned)a.rows, 128, 0, st>>>(a);
}
