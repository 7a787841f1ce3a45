// Gradients of attention to states of another length.
#include "reader.h"

// With P = exp(s - lse), dP = dO v^T and dS = P (dP - delta), delta_i = dO_i . out_i:
//   dv = P^T dO,   dk = scale dS^T q,   dq = scale dS k,   dbias_j = sum_i dS_ij.
// P is formed again from the statistics of the forward pass.  Two kernels, each with its own sums in registers and nothing
// added up in memory, so that every sum has one order: grad_k_kernel owns keys (a wave 32 of them, the keys and values in
// registers) and passes over the rows of all heads that share them; grad_q_kernel owns rows and passes over the keys.  Forming
// s and dP twice costs 7 products in place of 5.  What the other side brings goes through LDS once and is read both along its
// rows (for s and dP) and transposed (for the sums); the products s and dP leave their registers as the operands that the sums
// need, as in the forward kernel.

template <int DT, int D>
__global__ __launch_bounds__(256) void delta_kernel(GradArgs g)
{
    constexpr int LANES = D / 8;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    float sum = 0.0f;
    if (at < g.a.num_queries * g.a.heads) {
        const int c = threadIdx.x % LANES;
        const i32x4 x = *(const i32x4 *)(g.a.out + (at * D + c * 8) * 2), y = *(const i32x4 *)(g.d_out + (at * D + c * 8) * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += unpack<DT>(x[e], 0) * unpack<DT>(y[e], 0) + unpack<DT>(x[e], 1) * unpack<DT>(y[e], 1);
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) sum += __shfl_xor(sum, o);
        if (c == 0) g.delta[at] = sum;
    }
}

#define GRAD_ROWS 32  // rows of a step of grad_k_kernel
#define GRAD_KEYS 64  // keys of a step of grad_q_kernel

template <int DT, int D, int NW, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void grad_k_kernel(GradArgs g, int64_t tiles, int splits)
{
    constexpr int THREADS = NW * 64, KEYS = NW * 32, SHIFT = NW == 8 ? 8 : 7, CHUNKS = D / 8;
    constexpr int N = GRAD_ROWS * CHUNKS / THREADS > 0 ? GRAD_ROWS * CHUNKS / THREADS : 1;
    const AttendArgs &a = g.a;
    __shared__ __align__(16) char s_q[2][GRAD_ROWS * D * 2], s_o[2][GRAD_ROWS * D * 2];
    __shared__ __align__(16) float s_m[2][GRAD_ROWS], s_l[2][GRAD_ROWS], s_delta[2][GRAD_ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const WorkPlace w = work_place(a, tiles);
    const int head = w.head, split = w.split;
    const TilePlace tp = find_tile(a.k_offsets, a.n, a.num_keys, 1, SHIFT, w.place);
    if (tp.r < 0) return;
    const int len = (int)(tp.end - tp.begin);
    const int64_t row0 = clamp64(a.q_offsets[tp.r], 0, a.num_queries);
    const int tokens = (int)(clamp64(a.q_offsets[tp.r + 1], row0, a.num_queries) - row0), rows = tokens * a.group;
    const int steps = (rows + GRAD_ROWS - 1) / GRAD_ROWS, share = (steps + splits - 1) / splits;
    const int begin = split * share, end = min(steps, begin + share);

    const int key = tp.tile * KEYS + wave * 32 + (lane & 31);
    const bool there = key < len;
    i32x4 k[D / 16], v[D / 16];
    {
        const char *pk = a.k + (tp.begin + key) * a.k_token + head * a.k_head + h * 16;
        const char *pv = a.v + (tp.begin + key) * a.v_token + head * a.v_head + h * 16;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            k[s] = v[s] = i32x4{0, 0, 0, 0};
            if (there) k[s] = *(const i32x4 *)(pk + s * 32), v[s] = *(const i32x4 *)(pv + s * 32);
        }
    }
    float bias = 0.0f;
    if (BIAS && there) bias = load16<DT>(a.bias + 2 * (tp.begin + key));
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dk[t] = zero16(), dv[t] = zero16();
    float dbias = 0.0f;

    i32x4 xq[N], xo[N];
    float xm = 0.0f, xl = INFINITY, xd = 0.0f;
    auto load = [&](int step) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, row = step * GRAD_ROWS + u / CHUNKS;
            xq[i] = xo[i] = i32x4{0, 0, 0, 0};
            if (u < GRAD_ROWS * CHUNKS && row < rows) {
                const int token = row_token(a, row), hd = head * a.group + row - token * a.group;
                xq[i] = *(const i32x4 *)(a.q + (row0 + token) * a.q_token + hd * a.q_head + u % CHUNKS * 16);
                xo[i] = *(const i32x4 *)(g.d_out + (((row0 + token) * a.heads + hd) * D + u % CHUNKS * 8) * 2);
            }
        }
        if (threadIdx.x < GRAD_ROWS) {
            const int row = step * GRAD_ROWS + threadIdx.x;
            xm = 0.0f, xl = INFINITY, xd = 0.0f;  // no row, or one that no key was left for: its weights are 0
            if (row < rows) {
                const int token = row_token(a, row), hd = head * a.group + row - token * a.group;
                const int64_t at = (row0 + token) * a.heads + hd;
                const float m = a.lse[2 * at], l = a.lse[2 * at + 1];
                if (m != -INFINITY) xm = m, xl = l * LOG2E, xd = g.delta[at];
            }
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS;
            if (u < GRAD_ROWS * CHUNKS) {
                *(i32x4 *)(s_q[buf] + lds_chunk<D>(u / CHUNKS, u % CHUNKS)) = xq[i];
                *(i32x4 *)(s_o[buf] + lds_chunk<D>(u / CHUNKS, u % CHUNKS)) = xo[i];
            }
        }
        if (threadIdx.x < GRAD_ROWS) s_m[buf][threadIdx.x] = xm, s_l[buf][threadIdx.x] = xl, s_delta[buf][threadIdx.x] = xd;
    };
    if (begin < end) {
        load(begin);
        store(0);
    }
    __syncthreads();
    for (int step = begin; step < end; ++step) {
        const int buf = (step - begin) & 1;
        if (step + 1 < end) load(step + 1);
        f32x16 p = zero16(), ds = zero16();
#pragma unroll
        for (int s = 0; s < D / 16; ++s) p = mfma32<DT>(lds_rows<D>(s_q[buf], 0, s), k[s], p);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) ds = mfma32<DT>(lds_rows<D>(s_o[buf], 0, s), v[s], ds);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 m = *(const f32x4 *)&s_m[buf][8 * i + 4 * h], l = *(const f32x4 *)&s_l[buf][8 * i + 4 * h],
                        delta = *(const f32x4 *)&s_delta[buf][8 * i + 4 * h];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // the difference to the maximum first: a bias may be the type's lowest value
                const float x = (fmaf(p[4 * i + e], a.scale, bias) - m[e]) * LOG2E - l[e];
                p[4 * i + e] = __builtin_amdgcn_exp2f(x);
                ds[4 * i + e] = p[4 * i + e] * (ds[4 * i + e] - delta[e]);
                dbias += ds[4 * i + e];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const i32x4 pr = round8<DT>(p, i), dr = round8<DT>(ds, i);
#pragma unroll
            for (int t = 0; t < D / 32; ++t) {
                dv[t] = mfma32<DT>(lds_columns<D>(s_o[buf], 16 * i, t), pr, dv[t]);
                dk[t] = mfma32<DT>(lds_columns<D>(s_q[buf], 16 * i, t), dr, dk[t]);
            }
        }
        if (step + 1 < end) store(buf ^ 1);
        __syncthreads();
    }

    dbias = sum_halves(dbias);
    if (!there) return;
    // a masked key's column may hold anything and is zero
    const bool masked = BIAS && bias == -INFINITY;
    const int64_t at = (tp.begin + key) * a.kv_heads + head;
    if (BIAS && h == 0 && g.dbias_part) g.dbias_part[((int64_t)split * a.kv_heads + head) * a.num_keys + tp.begin + key] = masked ? 0.0f : dbias;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = masked ? 0.0f : dk[t][4 * i + e] * a.scale, y[e] = masked ? 0.0f : dv[t][4 * i + e];
            const int d = 32 * t + 8 * i + 4 * h;
            if (splits > 1) {
                const int64_t to = ((int64_t)split * a.num_keys * a.kv_heads + at) * D + d;
                *(f32x4 *)(g.dk_part + to) = x;
                *(f32x4 *)(g.dv_part + to) = y;
            } else {
                if (g.dk) *(i32x2 *)(g.dk + (at * D + d) * 2) = i32x2{pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])};
                if (g.dv) *(i32x2 *)(g.dv + (at * D + d) * 2) = i32x2{pack2<DT>(y[0], y[1]), pack2<DT>(y[2], y[3])};
            }
        }
}

template <int DT, int D, int NW, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void grad_q_kernel(GradArgs g, int64_t tiles, int splits)
{
    constexpr int THREADS = NW * 64, ROWS = NW * 32, SHIFT = NW == 8 ? 8 : 7, CHUNKS = D / 8;
    constexpr int N = (GRAD_KEYS * CHUNKS + THREADS - 1) / THREADS;
    const AttendArgs &a = g.a;
    __shared__ __align__(16) char s_k[2][GRAD_KEYS * D * 2], s_v[2][GRAD_KEYS * D * 2];
    __shared__ __align__(16) float s_bias[2][BIAS ? GRAD_KEYS : 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const WorkPlace w = work_place(a, tiles);
    const int head_kv = w.head, split = w.split;
    const TilePlace tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, w.place);
    if (tp.r < 0) return;
    const int tokens = (int)(tp.end - tp.begin), rows = tokens * a.group;
    const int64_t key0 = clamp64(a.k_offsets[tp.r], 0, a.num_keys);
    const int len = (int)(clamp64(a.k_offsets[tp.r + 1], key0, a.num_keys) - key0);
    const int steps = (len + GRAD_KEYS - 1) / GRAD_KEYS, share = (steps + splits - 1) / splits;
    const int begin = split * share, end = min(steps, begin + share);

    const int row = tp.tile * ROWS + wave * 32 + (lane & 31);
    const bool there = row < rows;
    const int token = row_token(a, there ? row : 0), head = head_kv * a.group + (there ? row : 0) - token * a.group;
    const int64_t at = (tp.begin + token) * a.heads + head;
    i32x4 q[D / 16], d_out[D / 16];
    {
        const char *pq = a.q + (tp.begin + token) * a.q_token + head * a.q_head + h * 16, *po = g.d_out + at * D * 2 + h * 16;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            q[s] = d_out[s] = i32x4{0, 0, 0, 0};
            if (there) q[s] = *(const i32x4 *)(pq + s * 32), d_out[s] = *(const i32x4 *)(po + s * 32);
        }
    }
    float m = 0.0f, l = INFINITY, delta = 0.0f;
    if (there && a.lse[2 * at] != -INFINITY) m = a.lse[2 * at], l = a.lse[2 * at + 1] * LOG2E, delta = g.delta[at];
    f32x16 dq[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dq[t] = zero16();

    i32x4 xk[N], xv[N];
    float xb = -INFINITY;
    auto load = [&](int step) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, key = step * GRAD_KEYS + u / CHUNKS;
            xk[i] = xv[i] = i32x4{0, 0, 0, 0};
            bool in = u < GRAD_KEYS * CHUNKS && key < len;
            if constexpr (BIAS) in = in && load16<DT>(a.bias + 2 * (key0 + key)) != -INFINITY;
            if (in) {
                xk[i] = *(const i32x4 *)(a.k + (key0 + key) * a.k_token + head_kv * a.k_head + u % CHUNKS * 16);
                xv[i] = *(const i32x4 *)(a.v + (key0 + key) * a.v_token + head_kv * a.v_head + u % CHUNKS * 16);
            }
        }
        if constexpr (BIAS) {
            const int key = step * GRAD_KEYS + threadIdx.x;
            if (threadIdx.x < GRAD_KEYS) xb = key < len ? load16<DT>(a.bias + 2 * (key0 + key)) : -INFINITY;
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS;
            if (u < GRAD_KEYS * CHUNKS) {
                *(i32x4 *)(s_k[buf] + lds_chunk<D>(u / CHUNKS, u % CHUNKS)) = xk[i];
                *(i32x4 *)(s_v[buf] + lds_chunk<D>(u / CHUNKS, u % CHUNKS)) = xv[i];
            }
        }
        if constexpr (BIAS)
            if (threadIdx.x < GRAD_KEYS) s_bias[buf][threadIdx.x] = xb;
    };
    if (begin < end) {
        load(begin);
        store(0);
    }
    __syncthreads();
    for (int step = begin; step < end; ++step) {
        const int buf = (step - begin) & 1;
        if (step + 1 < end) load(step + 1);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            f32x16 s = zero16(), ds = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) s = mfma32<DT>(lds_rows<D>(s_k[buf], 32 * mt, d), q[d], s);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) ds = mfma32<DT>(lds_rows<D>(s_v[buf], 32 * mt, d), d_out[d], ds);
            const bool whole = (step + 1) * GRAD_KEYS <= len;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 b{0, 0, 0, 0};
                if constexpr (BIAS) b = *(const f32x4 *)&s_bias[buf][32 * mt + 8 * i + 4 * h];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p = __builtin_amdgcn_exp2f((fmaf(s[4 * i + e], a.scale, b[e]) - m) * LOG2E - l);
                    if constexpr (BIAS) p = b[e] == -INFINITY ? 0.0f : p;
                    else if (!whole) p = step * GRAD_KEYS + 32 * mt + 8 * i + 4 * h + e < len ? p : 0.0f;
                    ds[4 * i + e] = p * (ds[4 * i + e] - delta);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const i32x4 dr = round8<DT>(ds, i);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) dq[t] = mfma32<DT>(lds_columns<D>(s_k[buf], 32 * mt + 16 * i, t), dr, dq[t]);
            }
        }
        if (step + 1 < end) store(buf ^ 1);
        __syncthreads();
    }
    if (!there) return;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = dq[t][4 * i + e] * a.scale;
            const int d = 32 * t + 8 * i + 4 * h;
            if (splits > 1) *(f32x4 *)(g.dq_part + ((int64_t)split * a.num_queries * a.heads + at) * D + d) = x;
            else *(i32x2 *)(g.dq + (at * D + d) * 2) = i32x2{pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])};
        }
}

// out[i] = sum over the splits of part[s][i], in their order, for the rows that a request owns.
template <int DT>
__global__ __launch_bounds__(256) void add_splits_kernel(const float *part, char *out, int64_t count, int splits, const int64_t *offsets, int n,
                                                         int64_t per_row)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= count) return;
    const int64_t row = i / per_row;
    if (row < offsets[0] || row >= offsets[n]) return;
    f32x4 sum{0, 0, 0, 0};
    for (int s = 0; s < splits; ++s) {
        const f32x4 x = *(const f32x4 *)(part + s * count + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    *(i32x2 *)(out + 2 * i) = i32x2{pack2<DT>(sum[0], sum[1]), pack2<DT>(sum[2], sum[3])};
}
// dbias[j] = sum over splits and key heads.
template <int DT>
__global__ __launch_bounds__(256) void add_bias_kernel(const float *part, char *out, int64_t keys, int parts, const int64_t *offsets, int n)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= keys || i < offsets[0] || i >= offsets[n]) return;
    float sum = 0.0f;
    for (int s = 0; s < parts; ++s) sum += part[s * keys + i];
    store16<DT>(out + 2 * i, sum);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int DT, int D, int NW>
static void launch_k(hipStream_t st, const GradArgs &g, int splits)
{
    const int64_t tiles = g.a.num_keys / (NW * 32) + g.a.n;
    const dim3 grid((unsigned)(tiles * g.a.kv_heads * splits)), block(NW * 64);
    if (g.a.bias) grad_k_kernel<DT, D, NW, true><<<grid, block, 0, st>>>(g, tiles, splits);
    else grad_k_kernel<DT, D, NW, false><<<grid, block, 0, st>>>(g, tiles, splits);
}
template <int DT, int D, int NW>
static void launch_q(hipStream_t st, const GradArgs &g, int splits)
{
    const int64_t tiles = g.a.num_queries * g.a.group / (NW * 32) + g.a.n;
    const dim3 grid((unsigned)(tiles * g.a.kv_heads * splits)), block(NW * 64);
    if (g.a.bias) grad_q_kernel<DT, D, NW, true><<<grid, block, 0, st>>>(g, tiles, splits);
    else grad_q_kernel<DT, D, NW, false><<<grid, block, 0, st>>>(g, tiles, splits);
}
template <int DT, int D>
static void launch(hipStream_t st, const GradArgs &g, int q_waves, int q_splits, int k_waves, int k_splits)
{
    const AttendArgs &a = g.a;
    const int64_t q_values = a.num_queries * a.heads * D, k_values = a.num_keys * a.kv_heads * D;
    if (a.num_queries > 0) delta_kernel<DT, D><<<dim3((unsigned)ceil_div(q_values / 8, 256)), dim3(256), 0, st>>>(g);
    if ((g.dk || g.dv || g.dbias) && a.num_keys > 0) {
        if (k_waves == 8) launch_k<DT, D, 8>(st, g, k_splits);
        else launch_k<DT, D, 4>(st, g, k_splits);
        if (k_splits > 1) {
            const dim3 grid((unsigned)ceil_div(k_values / 4, 256));
            if (g.dk) add_splits_kernel<DT><<<grid, dim3(256), 0, st>>>(g.dk_part, g.dk, k_values, k_splits, a.k_offsets, a.n, (int64_t)a.kv_heads * D);
            if (g.dv) add_splits_kernel<DT><<<grid, dim3(256), 0, st>>>(g.dv_part, g.dv, k_values, k_splits, a.k_offsets, a.n, (int64_t)a.kv_heads * D);
        }
        if (g.dbias)
            add_bias_kernel<DT><<<dim3((unsigned)ceil_div(a.num_keys, 256)), dim3(256), 0, st>>>(g.dbias_part, g.dbias, a.num_keys, k_splits * a.kv_heads,
                                                                                                a.k_offsets, a.n);
    }
    if (g.dq && a.num_queries > 0) {
        if (q_waves == 8) launch_q<DT, D, 8>(st, g, q_splits);
        else launch_q<DT, D, 4>(st, g, q_splits);
        if (q_splits > 1)
            add_splits_kernel<DT><<<dim3((unsigned)ceil_div(q_values / 4, 256)), dim3(256), 0, st>>>(g.dq_part, g.dq, q_values, q_splits, a.q_offsets, a.n,
                                                                                                    (int64_t)a.heads * D);
    }
}
void plaid_launch_attend_grad(hipStream_t st, const GradArgs &g, int dtype, int head_dim, int q_waves, int q_splits, int k_waves, int k_splits)
{
    if (dtype == PLAID_BF16) head_dim == 64 ? launch<PLAID_BF16, 64>(st, g, q_waves, q_splits, k_waves, k_splits) : launch<PLAID_BF16, 128>(st, g, q_waves, q_splits, k_waves, k_splits);
    else head_dim == 64 ? launch<PLAID_FP16, 64>(st, g, q_waves, q_splits, k_waves, k_splits) : launch<PLAID_FP16, 128>(st, g, q_waves, q_splits, k_waves, k_splits);
}
