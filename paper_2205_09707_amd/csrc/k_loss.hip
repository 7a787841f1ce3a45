// Cross entropy over a vocabulary: what goes before and after its products, and the scores of a few rows.
#include "train.h"

#define NO_EXPONENT (-100000)  // of a d_loss of zero

// With s_tv = scale h_t . W_v:  lse_t = log sum_v exp s_tv, loss_t = lse_t - s_t,target, and for gradients
//   G_tv = d_loss_t (exp(s_tv - lse_t) - [v = target_t]),  dh_t = scale sum_v G_tv W_v,  dW_v = scale sum_t G_tv h_t.
// Scores are never kept: the products' kernels (k_loss_mm.hip) leave a maximum and a sum of exponentials for each part of the vocabulary,
// joined here.  lse is kept as two numbers, the maximum and the logarithm of the sum beside it, so that a probability near one keeps its
// distance from one.

// --- rows that have a target ----------------------------------------------------------------------------------------------------
// They are numbered in the caller's order, and their states packed in the order in which the products' tiles take them, with zeros up to a whole
// tile of rows and a whole step of columns; a row without a target has a loss of zero and no gradient.  Backward, d_loss = fraction 2^exponent:
// the fraction goes into G, which rounds to the type before it is multiplied, the power of two into what G is multiplied with, so that G in fp16
// stays in its range however small the gradient of a mean is.  d_hidden takes it from the sums, in 32 bits, d_weight, whose sums go over the rows, in the
// states, relative to state[1].  In bf16 that is the largest exponent.  fp16 would lose the digits of rows with a small d_loss below its normal range while the range
// above is empty, so there the largest state of all rows, with its row's power, takes the type's last binade: the states of a row 2^-r of that one are exact down to
// 2^(r - 29) of the row's own largest, and what rounds there rounds by 2^-40 of the largest of all.  (Finding it is a launch of its own, 2.5 to 5 us.)
__device__ __forceinline__ bool has_target(const LossArgs &a, int64_t t, int &target)
{
    const int64_t v = a.targets[t];
    target = (int)v;
    return v >= 0 && v < a.vocabulary;
}
__device__ __forceinline__ LossRow loss_row(const LossArgs &a, int64_t t, int target, bool backward)
{
    LossRow r = {target, 0, 0.0f, 0.0f, 0.0f};
    if (backward) {
        const float d = *(const float *)((const char *)a.d_loss + t * a.d_loss_stride);
        if (fabsf(d) < INFINITY) r.fraction = frexpf(d, &r.exponent);
        else r.fraction = d;
        if (d == 0.0f) r.exponent = NO_EXPONENT;
        r.top = a.lse[2 * t], r.log_total = a.lse[2 * t + 1];
    }
    return r;
}
// A row's exponent beside state[1]; above 40 only where all states are zero or not finite.
__device__ __forceinline__ int state_shift(int exponent, int top) { return exponent == NO_EXPONENT ? 0 : min(exponent - top, 40); }

// fp16: what state[1] has to be for a row's largest finite state to take the last binade, a wave a row.
__global__ __launch_bounds__(256) void loss_reach_kernel(LossArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    int target = 0, reach = NO_EXPONENT;
    if (t >= a.rows) return;
    if (has_target(a, t, target)) {
        const char *row = a.hidden + t * a.hidden_stride;
        int most = 0;  // bits of a magnitude; they ascend as it does
        for (int at = lane * 8; at < a.width; at += 512) {
            const i32x4 w = *(const i32x4 *)(row + 2 * at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int bits = (w[i / 2] >> (16 * (i & 1))) & 0x7fff;
                most = max(most, bits < 0x7c00 ? bits : 0);
            }
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) most = max(most, __shfl_xor(most, o));
        const int exponent = loss_row(a, t, target, true).exponent;
        int e;
        (void)frexpf(unpack<PLAID_FP16>(most, 0), &e);
        if (most > 0 && exponent != NO_EXPONENT) reach = exponent + e - 16;
    }
    if (lane == 0) a.reach[t] = reach;
}
// 128 threads; t < 0: zeros.
template <int DT, bool BACKWARD>
__device__ __forceinline__ void pack_row(const LossArgs &a, int place, int64_t t, int shift)
{
    constexpr int BLOCK = LOSS_TILE * LOSS_STEP * 2;
    const char *from = a.hidden + (t < 0 ? 0 : t) * a.hidden_stride;
    char *to = a.packed + (int64_t)(place / LOSS_TILE) * (a.pitch / LOSS_STEP) * BLOCK + place % LOSS_TILE * (2 * LOSS_STEP);
    char *scaled = BACKWARD ? a.scaled + (int64_t)(place / LOSS_STEP) * (a.columns / LOSS_TILE) * BLOCK + place % LOSS_STEP * (2 * LOSS_TILE) : nullptr;
    const float power = ldexpf(1.0f, shift);
    const int sign = a.scale < 0.0f ? (int)0x80008000u : 0;
    for (int at = threadIdx.x * 8; at < (BACKWARD ? a.columns : a.pitch); at += 1024) {
        i32x4 w = t >= 0 && at < a.width ? *(const i32x4 *)(from + 2 * at) : i32x4{0, 0, 0, 0};
        w ^= i32x4{sign, sign, sign, sign};
        if (at < a.pitch) *(i32x4 *)(to + (int64_t)(at / LOSS_STEP) * BLOCK + at % LOSS_STEP * 2) = w;
        if (BACKWARD) {
            Eight v = unpack8<DT>(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v.x[j] *= power;
            *(i32x4 *)(scaled + (int64_t)(at / LOSS_TILE) * BLOCK + at % LOSS_TILE * 2) = pack8<DT>(v);
        }
    }
}
template <bool BACKWARD>
__device__ __forceinline__ void no_target(const LossArgs &a, int64_t t)
{
    if (!BACKWARD) {
        if (threadIdx.x == 0) {
            a.loss[t] = 0.0f;
            if (a.lse) *(float2 *)(a.lse + 2 * t) = {0.0f, 0.0f};
        }
    } else if (a.d_hidden)
        for (int at = threadIdx.x * 8; at < a.width; at += 1024) *(i32x4 *)(a.d_hidden + (t * a.width + at) * 2) = i32x4{0, 0, 0, 0};
}

// Up to LOSS_PREPARE_ONE rows: one launch, in which each row's workgroup looks at all targets itself.  (A forward call of width 512 on 30000 entries, with
// it and with the two launches below: 300 rows 29 and 32 us, 1000 47 and 48, 1500 63.7 and 64.1, 2000 80.5 and 79.4.)
template <int DT, bool BACKWARD>
__global__ __launch_bounds__(128) void loss_prepare_kernel(LossArgs a)
{
    __shared__ int found[2][3];
    const int rows = (int)a.rows, t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int live = 0, before = 0, top = NO_EXPONENT;
    for (int first = 0; first < rows; first += 128) {
        const int i = first + threadIdx.x;
        int target = 0;
        const bool mine = i < rows && has_target(a, i, target);
        live += __popcll(__ballot(mine)), before += __popcll(__ballot(mine && i < t));
        if (BACKWARD && mine) top = max(top, a.reach ? a.reach[i] : loss_row(a, i, target, true).exponent);
    }
    if (BACKWARD)
#pragma unroll
        for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
    if (lane == 0) found[wave][0] = live, found[wave][1] = before, found[wave][2] = top;
    __syncthreads();
    live = found[0][0] + found[1][0], before = found[0][1] + found[1][1], top = max(found[0][2], found[1][2]);
    if (top == NO_EXPONENT) top = 0;
    if (t == 0 && threadIdx.x == 0) a.state[0] = live, a.state[1] = top;
    int target = 0;
    const bool mine = t < rows && has_target(a, t, target);
    if (mine) {
        const LossRow r = loss_row(a, t, target, BACKWARD);
        if (threadIdx.x == 0) {
            a.list[before] = t, a.row[before] = r;
            if (BACKWARD) a.target[before] = target;
        }
        pack_row<DT, BACKWARD>(a, before, t, state_shift(r.exponent, top));
        return;
    }
    // the others, and those past the end, are as many as there are places up to the last tile's end
    const int place = live + (t < rows ? t - before : t - live);
    if (place < (live + LOSS_TILE - 1) / LOSS_TILE * LOSS_TILE) pack_row<DT, BACKWARD>(a, place, -1, 0);
    if (t < rows) no_target<BACKWARD>(a, t);
}

// More rows: one workgroup numbers them.
__global__ __launch_bounds__(1024) void loss_list_kernel(LossArgs a, int backward)
{
    __shared__ int wave_sum[16], wave_top[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0, top = NO_EXPONENT;
    for (int64_t first = 0; first < a.rows; first += 1024) {
        const int64_t t = first + threadIdx.x;
        int target = 0;
        const bool live = t < a.rows && has_target(a, t, target);
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
            const LossRow r = loss_row(a, t, target, backward);
            if (backward) top = max(top, a.reach ? a.reach[t] : r.exponent);
            a.list[at] = (int)t;
            a.row[at] = r;
            if (backward) a.target[at] = target;
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
// Workgroup i has place i, and row i if that has no target.
template <int DT, bool BACKWARD>
__global__ __launch_bounds__(128) void loss_pack_kernel(LossArgs a)
{
    const int live = uniform_load(a.state), top = uniform_load(a.state + 1), i = blockIdx.x;
    int target = 0;
    if (i < a.rows && !has_target(a, i, target)) no_target<BACKWARD>(a, i);
    if (i >= (live + LOSS_TILE - 1) / LOSS_TILE * LOSS_TILE) return;
    const int e = BACKWARD && i < live ? uniform_load(&a.row[i].exponent) : NO_EXPONENT;
    pack_row<DT, BACKWARD>(a, i, i < live ? uniform_load(a.list + i) : -1, state_shift(e, top));
}

void plaid_launch_loss_pack(hipStream_t st, const LossArgs &a, int dtype, bool backward)
{
    const unsigned grid = (unsigned)a.padded_rows;
    if (a.reach && a.rows > 0) loss_reach_kernel<<<(unsigned)((a.rows + 3) / 4), 256, 0, st>>>(a);
    if (a.rows <= LOSS_PREPARE_ONE) {
        if (!backward) loss_prepare_kernel<PLAID_BF16, false><<<grid, 128, 0, st>>>(a);
        else if (dtype == PLAID_BF16) loss_prepare_kernel<PLAID_BF16, true><<<grid, 128, 0, st>>>(a);
        else loss_prepare_kernel<PLAID_FP16, true><<<grid, 128, 0, st>>>(a);
        return;
    }
    loss_list_kernel<<<1, 1024, 0, st>>>(a, backward);
    if (!backward) loss_pack_kernel<PLAID_BF16, false><<<grid, 128, 0, st>>>(a);
    else if (dtype == PLAID_BF16) loss_pack_kernel<PLAID_BF16, true><<<grid, 128, 0, st>>>(a);
    else loss_pack_kernel<PLAID_FP16, true><<<grid, 128, 0, st>>>(a);
}

// Largest products and sums of exponentials beside them, of two parts; f: exponent_factor.
__device__ __forceinline__ float2 join_parts(float2 x, float2 y, float f)
{
    const float m = fmaxf(x.x, y.x), base = m == -INFINITY ? 0.0f : m;
    return {m, x.y * __builtin_amdgcn_exp2f((x.x - base) * f) + y.y * __builtin_amdgcn_exp2f((y.x - base) * f)};
}

// --- few rows -------------------------------------------------------------------------------------------------------------------
// The vocabulary is read at the rate of memory if enough of it is under way: a workgroup has 64 BLOCKS entries, a quarter for each of its four
// waves, and up to 16 GROUPS rows (more than 128: those of 128 after those); 64 columns of both go straight into LDS, some steps ahead of the
// products.  Forward it takes the caller's rows, all of them (a row without a target has its own column of the result, and is left out when parts are joined); backward (GRADIENT) the
// packed ones, and leaves G over the piece as the products take it, with zeros up to whole steps of 64 rows and entries.
template <int DT, int WAVES, int BLOCKS, int GROUPS, bool GRADIENT>
__global__ __launch_bounds__(WAVES * 64) void loss_few_kernel(LossArgs a)
{
    constexpr int ENTRIES = 16 * WAVES * BLOCKS, W_LOADS = 2 * BLOCKS, H_PIECES = 2 * GROUPS, H_LOADS = (H_PIECES + WAVES - 1) / WAVES, LOADS = W_LOADS + H_LOADS;
    constexpr int STAGES = 3;
    __shared__ __align__(16) char lds_w[STAGES][ENTRIES * 128], lds_h[STAGES][GROUPS * 16 * 128];
    __shared__ float2 joined[WAVES][16 * GROUPS];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), l = lane & 15, q = lane >> 4;
    const int rows = GRADIENT ? uniform_load(a.state) : (int)a.rows, row0 = blockIdx.y * (16 * GROUPS);
    if (GRADIENT && row0 >= (rows + LOSS_STEP - 1) / LOSS_STEP * LOSS_STEP && row0 > 0) return;  // no one reads what would be here
    const int64_t first = GRADIENT ? a.first : 0, end = GRADIENT ? a.first + a.piece : a.vocabulary, v0 = first + (int64_t)blockIdx.x * ENTRIES;
    // a load has eight rows of 128 bytes, whose chunks change places as lds_chunk says; with fewer pieces of states than waves some are brought twice
    const char *from[LOADS];
    int to[LOADS], chunk[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const bool w = i < W_LOADS;
        const int piece = w ? wave * W_LOADS + i : (wave + WAVES * (i - W_LOADS)) % H_PIECES, row = piece * 8 + (lane >> 3);
        chunk[i] = (lane & 7) ^ swizzle<64>(row);
        to[i] = piece * 1024;
        if (w) from[i] = a.weight + min(v0 + row, a.vocabulary - 1) * a.weight_stride;
        else if (GRADIENT) from[i] = a.packed + (int64_t)(row0 / LOSS_TILE) * (a.pitch / LOSS_STEP) * (LOSS_TILE * 128) + (row0 % LOSS_TILE + row) * 128;
        else from[i] = a.hidden + min((int64_t)row0 + row, a.rows - 1) * a.hidden_stride;
        from[i] += chunk[i] * 16;
    }
    const int steps = (a.width + 63) / 64, left = a.width - (steps - 1) * 64;
    // Wide rows lie a power of two apart more often than not, and all workgroups at the same columns would ask the same few channels of memory: so
    // each begins at other columns, by its entries (90 rows on 128000 x 2048: 128 us in place of 172; on 50000 x 1024 24 in place of 23).
    const int begin = steps > 16 ? (int)(v0 / ENTRIES % steps) : 0;
    const auto bring = [&](int turn, int stage) {
        const int s = turn + begin < steps ? turn + begin : turn + begin - steps;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const bool packed = GRADIENT && i >= W_LOADS;
            const char *p = from[i] + (int64_t)s * (packed ? LOSS_TILE * 128 : 128);
            if (!packed && s == steps - 1 && chunk[i] * 8 >= left) p = (const char *)zero_row;  // zeros past the end of the rows
            load_to_lds(p, (i < W_LOADS ? lds_w[stage] : lds_h[stage]) + to[i]);
        }
    };
    f32x4 acc[BLOCKS][GROUPS], odd[BLOCKS][GROUPS];  // two sums, of every other 32 columns: each has half as many roundings, of half the size
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) acc[i][j] = odd[i][j] = f32x4{0, 0, 0, 0};
    int place[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) place[k] = l * 128 + (((4 * k + q) ^ swizzle<64>(l)) << 4);  // rows 16 on: 2048 bytes
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (s < steps) bring(s, s);
    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + STAGES - 1 <= steps) wait_loads<LOADS * (STAGES - 2)>();
        else wait_loads<0>();
        lds_barrier();  // this step's tiles have come, and all waves are done with those of the step before
        if (s + STAGES - 1 < steps) bring(s + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        const char *w = lds_w[stage] + wave * (BLOCKS * 2048), *h = lds_h[stage];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            i32x4 x[BLOCKS], y[GROUPS];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) x[i] = *(const i32x4 *)(w + i * 2048 + place[k]);
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) y[j] = *(const i32x4 *)(h + j * 2048 + place[k]);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                for (int j = 0; j < GROUPS; ++j) {
                    f32x4 &sum = k ? odd[i][j] : acc[i][j];
                    sum = mfma16<DT>(x[i], y[j], sum);
                }
        }
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) acc[i][j] += odd[i][j];
    // a lane's results: row 16 j + l, entries 16 i + 4 q .. + 3 from the wave's first
    const int64_t mine = v0 + wave * (16 * BLOCKS) + 4 * q;
    if constexpr (GRADIENT) {
        const int pieces = (a.piece + LOSS_TILE - 1) / LOSS_TILE;
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
            const int t = row0 + 16 * j + l;
            const bool there = t < rows;
            const LossRow x = there ? a.row[t] : LossRow{-1, 0, 0.0f, 0.0f, 0.0f};
            const ScoreGradient gradient(x, a, DT);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                float g[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t v = mine + 16 * i + r;
                    g[r] = gradient.other(acc[i][j][r]);
                    if (v == x.target) {
                        g[r] = gradient.target(acc[i][j][r]);
                        if (there && v < end) a.rest[t] = left_out<DT>(g[r]);
                    }
                    if (!there || v >= end) g[r] = 0.0f;
                }
                const int at = (int)(mine - first) + 16 * i;
                char *out = a.gradient + ((int64_t)(t / LOSS_TILE) * pieces + at / LOSS_TILE) * (LOSS_TILE * LOSS_TILE * 2) + (t % LOSS_TILE * LOSS_TILE + at % LOSS_TILE) * 2;
                *(i32x2 *)out = i32x2{pack2<DT>(g[0], g[1]), pack2<DT>(g[2], g[3])};
            }
        }
        return;
    }
    const float sign = a.scale < 0.0f ? -1.0f : 1.0f, f = exponent_factor(a);
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        const int64_t t = row0 + 16 * j + l;
        const int64_t target = t < rows ? a.targets[t] : -1;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t v = mine + 16 * i + r;
                float s = acc[i][j][r] * sign;
                if (v == target && v < end) a.own[t] = s;
                if (v == target || v >= end) s = -INFINITY;
                acc[i][j][r] = s;
                most = fmaxf(most, s);
            }
        most = max_halves(max_rows(most));
        const float base = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * f);
        sum = sum_halves(sum_rows(sum));
        if (lane < 16) joined[wave][16 * j + l] = {most, sum};
    }
    __syncthreads();
    if (threadIdx.x < 16 * GROUPS && row0 + (int)threadIdx.x < rows) {
        const int t = threadIdx.x;
        float2 x = join_parts(join_parts(joined[0][t], joined[1][t], f), join_parts(joined[2][t], joined[3][t], f), f);
        if constexpr (WAVES == 8) x = join_parts(x, join_parts(join_parts(joined[4][t], joined[5][t], f), join_parts(joined[6][t], joined[7][t], f), f), f);
        a.part[(int64_t)blockIdx.x * a.padded_rows + row0 + t] = x;
    }
}

template <int DT, int WAVES, int BLOCKS>
static void launch_few(hipStream_t st, const LossArgs &a, bool gradient)
{
    const int groups = (int)((a.rows + 15) / 16);
    const int64_t entries = gradient ? a.piece : a.vocabulary;
    const dim3 grid((unsigned)((entries + 16 * WAVES * BLOCKS - 1) / (16 * WAVES * BLOCKS)), (unsigned)((a.rows + 127) / 128 < 1 ? 1 : (a.rows + 127) / 128));
#define GO(G, GRADIENT) loss_few_kernel<DT, WAVES, BLOCKS, G, GRADIENT><<<grid, WAVES * 64, 0, st>>>(a)
    if constexpr (WAVES == 8) {
        if (gradient) GO(8, true);
        else if (groups <= 6) GO(6, false);
        else GO(8, false);
    } else if constexpr (BLOCKS == 2) {
        if (gradient) GO(4, true);
        else if (groups == 1) GO(1, false);
        else if (groups == 2) GO(2, false);
        else if (groups == 3) GO(3, false);
        else GO(4, false);
    } else {
        if (gradient) groups <= 4 ? GO(4, true) : GO(8, true);
        else if (groups == 1) GO(1, false);
        else if (groups == 2) GO(2, false);
        else if (groups == 3) GO(3, false);
        else if (groups == 4) GO(4, false);
        else if (groups <= 6) GO(6, false);
        else GO(8, false);
    }
#undef GO
}
// entries: of a workgroup, 64, 128 (up to 64 rows) or 256 (more rows)
void plaid_launch_loss_few(hipStream_t st, const LossArgs &a, int dtype, int entries, bool gradient)
{
#define GO(DT) entries == 64 ? launch_few<DT, 4, 1>(st, a, gradient) : entries == 128 ? launch_few<DT, 4, 2>(st, a, gradient) : launch_few<DT, 8, 2>(st, a, gradient)
    if (dtype == PLAID_BF16) GO(PLAID_BF16);
    else GO(PLAID_FP16);
#undef GO
}

// --- parts joined ---------------------------------------------------------------------------------------------------------------
// ROWS rows a workgroup, so that lanes read neighbours where there are many rows, and all threads have work where there are few (a forward call on
// 32000 entries of 512 with 1, 8 and 32 rows: 16 rows 10.2, 11.4, 15.6 us; 500 30.9, 30.7, 32.5; 8000 296, 285, 281); its threads of one row take the
// parts in turn.  With the last piece come the loss and lse: the target's score is not among the parts, so that where it is the largest the sum beside it is what the others have, and a loss near nothing keeps its digits.
template <int ROWS>
__global__ __launch_bounds__(256) void loss_join_kernel(LossArgs a, int parts, int packed)
{
    constexpr int SHARES = 256 / ROWS;
    __shared__ float2 lds[4][ROWS];
    const int r = threadIdx.x % ROWS, share = threadIdx.x / ROWS, live = packed ? uniform_load(a.state) : (int)a.rows;
    const int i = blockIdx.x * ROWS + r;
    const float f = exponent_factor(a);
    float2 x = {-INFINITY, 0.0f};
    if (i < live) {
#pragma unroll 4
        for (int p = share; p < parts; p += SHARES) x = join_parts(x, a.part[(int64_t)p * a.padded_rows + i], f);
    }
#pragma unroll
    for (int o = ROWS; o < 64; o <<= 1) x = join_parts(x, {__shfl_xor(x.x, o), __shfl_xor(x.y, o)}, f);
    if ((threadIdx.x & 63) < ROWS) lds[threadIdx.x >> 6][r] = x;
    __syncthreads();
    if (share != 0 || i >= live) return;
    x = join_parts(join_parts(lds[0][r], lds[1][r], f), join_parts(lds[2][r], lds[3][r], f), f);
    if (a.first > 0) x = join_parts(a.running[i], x, f);
    if (!a.last) {
        a.running[i] = x;
        return;
    }
    const int64_t t = packed ? (int64_t)a.list[i] : i;
    const bool there = packed || (a.targets[t] >= 0 && a.targets[t] < a.vocabulary);
    const float own = there ? a.own[i] : 0.0f;
    // log(exp(own) + sum), beside the larger of the two; where both are infinite or not a number, so is the result
    const float top = x.x > own ? x.x : own;
    const float rest = x.x > own ? logf(x.y + __builtin_amdgcn_exp2f((own - top) * f))
                                 : x.x == -INFINITY && x.y == 0.0f ? 0.0f : log1pf(x.y * __builtin_amdgcn_exp2f((x.x - top) * f));
    a.loss[t] = there ? (top - own) * score_factor(a) + rest : 0.0f;
    if (a.lse) *(float2 *)(a.lse + 2 * t) = there ? float2{top * score_factor(a), rest} : float2{0.0f, 0.0f};
}

void plaid_launch_loss_join(hipStream_t st, const LossArgs &a, int parts, bool packed)
{
    if (a.rows >= 4096) loss_join_kernel<32><<<(unsigned)((a.rows + 31) / 32), 256, 0, st>>>(a, parts, packed);
    else if (a.rows > LOSS_FEW) loss_join_kernel<8><<<(unsigned)((a.rows + 7) / 8), 256, 0, st>>>(a, parts, packed);
    else loss_join_kernel<1><<<(unsigned)a.rows, 256, 0, st>>>(a, parts, packed);
}

// --- gradients: the parts' sums added up, in order -----------------------------------------------------------------------------------
// The sums lie in tiles of 256 rows (of states, or entries) and columns, in the order in which the products' registers hold them: for a wave of 128
// columns and 64 rows [32 rows' half][32 columns' quarter][8 columns' quarter][lane][4 columns], a lane being a row and a half of the 8
// columns.  A workgroup has 32 rows of a tile, each of its waves 8 columns.
template <int DT, bool WEIGHT>
__device__ __forceinline__ void join_gradients(const LossArgs &a, int id)
{
    const int live = uniform_load(a.state), widths = a.columns / LOSS_TILE, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = WEIGHT ? a.piece : live, row_tiles = (rows + LOSS_TILE - 1) / LOSS_TILE;
    const int block = id & 7, k = id >> 3 & 7, tile = id >> 6, row = tile / widths * LOSS_TILE + block * 32 + (lane & 31);
    if (tile / widths * LOSS_TILE + block * 32 >= rows) return;
    const LossParts parts = loss_parts(a, live);
    const int splits = WEIGHT ? parts.weight : parts.hidden;
    if (WEIGHT && splits == 1) return;  // written by the products
    const int64_t part = (int64_t)row_tiles * widths * (LOSS_TILE * LOSS_TILE);
    const bool there = row < rows;
    int64_t to = 0;
    int e = 0;
    if constexpr (WEIGHT) to = a.first + row, e = uniform_load(a.state + 1);
    else if (there) to = a.list[row], e = a.row[row].exponent;
    // the power of two last, where the result may leave the normal range
    const float factor = (WEIGHT ? score_factor(a) : a.scale) * (DT == PLAID_FP16 ? 0x1p-15f : 1.0f);
    // wave w of these four: eight of columns 64 w .. 64 w + 63, two quarters of 32
    const int i = (wave & 1) * 2 + k / 4, c = k % 4, column = tile % widths * LOSS_TILE + wave * 64 + k * 8 + 4 * (lane >> 5);
    const float *p = (WEIGHT ? a.w_part : a.d_part) + (int64_t)tile * (LOSS_TILE * LOSS_TILE) + ((wave >> 1) * 4 + block / 2) * 8192 + (((block & 1) * 4 + i) * 4 + c) * 256 + lane * 4;
    f32x4 v = {0, 0, 0, 0};
    i32x2 w = {0, 0};  // the target's, and what its entry of G left out
    float rest = 0.0f;
    if (!WEIGHT && there && column < a.width) w = *(const i32x2 *)(a.weight + a.row[row].target * a.weight_stride + column * 2), rest = a.rest[row];
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v += *(const f32x4 *)(p + s * part);
    if (!WEIGHT)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float more = rest * unpack<DT>(w[j / 2], j & 1);
            if (fabsf(more) < INFINITY) v[j] += more;
        }
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = ldexpf(v[j] * factor, e == NO_EXPONENT ? 0 : e);
    char *out = WEIGHT ? a.d_weight : a.d_hidden;
    if (there && column < a.width) *(i32x2 *)(out + (to * a.width + column) * 2) = i32x2{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
}
template <int DT>
__global__ __launch_bounds__(256) void loss_gradients_join_kernel(LossArgs a, int hidden)
{
    const int id = (int)wide_block();
    if (id < hidden) join_gradients<DT, false>(a, id);
    else join_gradients<DT, true>(a, id - hidden);
}
// After each piece for d_weight, if its axis may be cut, after the last one for d_hidden.
void plaid_launch_loss_gradients_join(hipStream_t st, const LossArgs &a, int dtype)
{
    const int widths = a.columns / LOSS_TILE, hidden = a.d_hidden && a.last ? a.padded_rows / LOSS_TILE * widths * 64 : 0;
    const int weight = a.d_weight && a.w_part ? (a.piece + LOSS_TILE - 1) / LOSS_TILE * widths * 64 : 0;
    if (hidden + weight == 0) return;
    if (dtype == PLAID_BF16) loss_gradients_join_kernel<PLAID_BF16><<<wide_grid(hidden + weight), 256, 0, st>>>(a, hidden);
    else loss_gradients_join_kernel<PLAID_FP16><<<wide_grid(hidden + weight), 256, 0, st>>>(a, hidden);
}
