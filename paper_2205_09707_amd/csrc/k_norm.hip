// Layer norm and its gradients.
#include "train.h"

// With m the mean of a row, r = 1 / sqrt(variance + eps) and x^ = (x - m) r:  y = x^ w + b, and with g = dy w
//   dx = r (g - mean(g) - x^ mean(g x^)),   dw = sum over rows of dy x^,   db = sum over rows of dy.
// A row's threads keep it in registers, so that the variance is that of x - m (no difference of large numbers) and the row is read once.
// LANES threads have a row, each up to C pieces of eight neighbouring elements, LANES * 8 elements apart.  Rows may start at any element.
//
// Memory bounds them: 100000 rows of 2048 in bf16 take 157 us forward (819 MB, 5.2 TB/s) and 241 backward (1.23 GB, 5.1 TB/s), and 6 to add up the
// workers' sums.  4001 rows of 765 out of rows of 784, in the caches, 8, 12 and 5 us: a chain of loads, sums across lanes and stores.
// How many threads have a row: as few as hold it in registers, so that no barrier is needed and narrow rows leave no lanes idle (200000 x 64,
// forward and backward: 38 us with eight lanes, 147 with 64).  Forward, us with a wave and with 256 threads: 100000 x 2048 146 and 171, 100000 x 1500
// 130 and 241, 3000 x 2048 7.7 and 8.4, but 512 x 2048 5.4 and 4.8, 64 x 4096 9.1 and 4.9, 50000 x 4096 160 and 147.  Backward, where a thread also holds
// two sums for each of its columns: 60000 x 1500 240 and 323 in all, 100000 x 2048 234 and 240.

// Sums of a row's threads; all of them get both.
template <int LANES>
__device__ __forceinline__ float2 row_sum(float2 s, float2 *lds)
{
#pragma unroll
    for (int o = (LANES < 64 ? LANES : 64) / 2; o; o >>= 1) s.x += __shfl_xor(s.x, o), s.y += __shfl_xor(s.y, o);
    if constexpr (LANES > 64) {
        __syncthreads();  // the sums before have been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = {0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) s.x += lds[w].x, s.y += lds[w].y;
    }
    return s;
}

template <int DT, int LANES, int C>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(NormArgs a)
{
    constexpr int THREADS = LANES < 256 ? 256 : LANES;
    __shared__ float2 lds[THREADS / 64];
    const int lane = threadIdx.x % LANES;
    const int64_t row = wide_block() * (THREADS / LANES) + threadIdx.x / LANES;
    if (row >= a.rows) return;  // whole teams
    const char *x = a.x + row * a.x_stride;
    Eight v[C];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * LANES + lane) * 8;
        v[c] = unpack8<DT>(load_piece(x, at, a.width));
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[c].x[i];
    }
    const float mean = row_sum<LANES>({sum, 0.0f}, lds).x / (float)a.width;
    float square = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c].x[i] -= mean;
            if ((c * LANES + lane) * 8 + i < a.width) square += v[c].x[i] * v[c].x[i];
        }
    const float inverse = 1.0f / sqrtf(row_sum<LANES>({square, 0.0f}, lds).x / (float)a.width + a.eps);
    if (a.statistics && lane == 0) *(float2 *)(a.statistics + 2 * row) = {mean, inverse};
    char *out = a.out + row * a.width * 2;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * LANES + lane) * 8;
        if (at >= a.width) break;
        const Eight w = unpack8<DT>(a.weight ? load_piece(a.weight, at, a.width) : i32x4{}), b = unpack8<DT>(a.bias ? load_piece(a.bias, at, a.width) : i32x4{});
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c].x[i] = v[c].x[i] * inverse * (a.weight ? w.x[i] : 1.0f) + b.x[i];
        store_piece(out, at, a.width, pack8<DT>(v[c]));
    }
}

// Workers go over the rows in turn and keep the sums of dw and db of their columns in registers; the last launch adds up the workers', in order.
template <int DT, int LANES, int C>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_grad_kernel(NormArgs a)
{
    constexpr int THREADS = LANES < 256 ? 256 : LANES, TEAMS = THREADS / LANES;
    __shared__ float2 lds[THREADS / 64];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    i32x4 w[C];
    Eight dw[C] = {}, db[C] = {};
#pragma unroll
    for (int c = 0; c < C; ++c) w[c] = a.weight ? load_piece(a.weight, (c * LANES + lane) * 8, a.width) : i32x4{};
    const float per = 1.0f / (float)a.width;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS) {
        const char *x = a.x + row * a.x_stride, *d = a.d_out + row * a.d_out_stride;
        i32x4 xr[C], dr[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            xr[c] = load_piece(x, (c * LANES + lane) * 8, a.width);
            dr[c] = load_piece(d, (c * LANES + lane) * 8, a.width);
        }
        const float2 st = {uniform_load(a.statistics + 2 * row), uniform_load(a.statistics + 2 * row + 1)};
        float2 sum = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Eight xv = unpack8<DT>(xr[c]), dv = unpack8<DT>(dr[c]), wv = unpack8<DT>(w[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float n = (xv.x[i] - st.x) * st.y, g = a.weight ? dv.x[i] * wv.x[i] : dv.x[i];
                sum.x += g, sum.y += g * n;  // past the end d_out is zero
                dw[c].x[i] += dv.x[i] * n, db[c].x[i] += dv.x[i];
            }
        }
        sum = row_sum<LANES>(sum, lds);
        const float m0 = sum.x * per, m1 = sum.y * per;
        if (a.dx) {
            char *dx = a.dx + row * a.width * 2;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * LANES + lane) * 8;
                if (at >= a.width) break;
                const Eight xv = unpack8<DT>(xr[c]), dv = unpack8<DT>(dr[c]), wv = unpack8<DT>(w[c]);
                Eight r;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float n = (xv.x[i] - st.x) * st.y, g = a.weight ? dv.x[i] * wv.x[i] : dv.x[i];
                    r.x[i] = st.y * (g - m0 - n * m1);
                }
                store_piece(dx, at, a.width, pack8<DT>(r));
            }
        }
    }
    if (!a.part) return;
    // the teams of a workgroup, in order
    constexpr int COLUMNS = LANES * 8;
    __shared__ float both[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? COLUMNS : 1];
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Eight &s = k ? db[c] : dw[c];
            if constexpr (TEAMS > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) both[team][i * LANES + lane] = s.x[i];
                __syncthreads();
                for (int at = threadIdx.x; at < COLUMNS; at += THREADS) {
                    const int column = c * COLUMNS + at % LANES * 8 + at / LANES;
                    float t = 0.0f;
#pragma unroll
                    for (int j = 0; j < TEAMS; ++j) t += both[j][at];
                    if (column < a.width) part[k * a.width + column] = t;
                }
            } else {
                const int at = (c * LANES + lane) * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at + i < a.width) part[k * a.width + at + i] = s.x[i];
            }
        }
}

// A workgroup has NORM_JOIN columns of dw or of db; its shares take the workers in turn.  (us with 64, 32 and 16 columns: 1024 workers of 2048 columns 7.4,
// 5.5, 8.4; 501 of 765 5.5, 4.8, 5.4; 750 of 4096 4.4, 4.6, 6.7; 1024 of 64 5.1, 3.9, 3.8.)
#define NORM_JOIN 32
template <int DT>
__global__ __launch_bounds__(1024) void norm_join_kernel(NormArgs a)
{
    constexpr int SHARES = 1024 / NORM_JOIN;
    __shared__ float lds[SHARES][NORM_JOIN];
    const int mine = threadIdx.x % NORM_JOIN, share = threadIdx.x / NORM_JOIN, column = blockIdx.x * NORM_JOIN + mine, k = blockIdx.y;
    char *out = k ? a.dbias : a.dweight;
    if (!out) return;
    float sum = 0.0f;
    if (column < a.width) {
        const float *p = a.part + k * a.width + column;
#pragma unroll 8
        for (int i = share; i < a.workers; i += SHARES) sum += p[(int64_t)i * 2 * a.width];
    }
    lds[share][mine] = sum;
    __syncthreads();
    if (share == 0 && column < a.width) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < SHARES; ++i) sum += lds[i][mine];
        store16<DT>(out + 2 * column, sum);
    }
}

template <int DT>
static void launch_norm(hipStream_t st, const NormArgs &a)
{
    const int pieces = (a.width + 7) / 8;
    const bool many = a.rows >= NORM_MANY;
#define GO(LANES, C) norm_kernel<DT, LANES, C><<<wide_grid((a.rows * LANES + 255) / (LANES < 256 ? 256 : LANES)), LANES < 256 ? 256 : LANES, 0, st>>>(a)
    if (pieces == 1) GO(1, 1);
    else if (pieces <= 8) GO(8, 1);
    else if (pieces <= 16) GO(16, 1);
    else if (pieces <= 32) GO(32, 1);
    else if (pieces <= 64) GO(64, 1);
    else if (pieces <= 128) GO(64, 2);
    else if (pieces <= 192 && many) GO(64, 3);
    else if (pieces <= 256) many ? GO(64, 4) : GO(256, 1);
    else if (pieces <= 320 && many) GO(64, 5);
    else if (pieces <= 384 && many) GO(64, 6);
    else if (pieces <= 512) GO(256, 2);
    else if (pieces <= 1024) GO(256, 4);
    else GO(1024, 2);
#undef GO
}
template <int DT>
static void launch_norm_backward(hipStream_t st, const NormArgs &a)
{
    const int pieces = (a.width + 7) / 8;
#define GO(LANES, C) norm_grad_kernel<DT, LANES, C><<<a.workers, LANES < 256 ? 256 : LANES, 0, st>>>(a)
    if (pieces == 1) GO(1, 1);
    else if (pieces <= 8) GO(8, 1);
    else if (pieces <= 16) GO(16, 1);
    else if (pieces <= 32) GO(32, 1);
    else if (pieces <= 64) GO(64, 1);
    else if (pieces <= 128) GO(64, 2);
    else if (pieces <= 192) GO(64, 3);
    else if (pieces <= 256) GO(256, 1);
    else if (pieces <= 512) GO(256, 2);
    else if (pieces <= 1024) GO(256, 4);
    else GO(1024, 2);
#undef GO
    if (a.part) norm_join_kernel<DT><<<dim3((a.width + NORM_JOIN - 1) / NORM_JOIN, 2), 1024, 0, st>>>(a);
}
void plaid_launch_layer_norm(hipStream_t st, const NormArgs &a, int dtype) { dtype == PLAID_BF16 ? launch_norm<PLAID_BF16>(st, a) : launch_norm<PLAID_FP16>(st, a); }
void plaid_launch_layer_norm_backward(hipStream_t st, const NormArgs &a, int dtype)
{
    dtype == PLAID_BF16 ? launch_norm_backward<PLAID_BF16>(st, a) : launch_norm_backward<PLAID_FP16>(st, a);
}
