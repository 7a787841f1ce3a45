// Gradients of attention to states of another length.
#include <stddef.h>

#include "reader.h"

// With P = exp(s - lse), dP = dO v^T and dS = P (dP - delta), delta_i = dO_i . out_i:
//   dv = P^T dO,   dk = scale dS^T q,   dq = scale dS k,   dbias_j = sum_i dS_ij.
// P is formed again from the statistics of the forward pass.  Two kernels, each with its own sums in registers and nothing
// added up in memory, so that every sum has one order: grad_k_kernel owns keys and passes over the rows of all heads that share
// them; grad_q_kernel owns rows and passes over the keys.  Forming s and dP twice costs 7 products in place of 5; sums of dq in
// memory, one for each tile of keys, would cost more: at 6250 keys 49 times dq in 32 bits, written and read.  What the other side
// brings goes into LDS once and is read both along its rows (for s and dP) and transposed (for the sums); the results leave their
// registers as the operands that the sums need, as in the forward kernel.

// Whether any weight is left in a row.
__device__ __forceinline__ bool row_counts(float2 lse) { return lse.x != -INFINITY && lse.y != -INFINITY; }

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
        if (c == 0) {
            const float2 lse = *(const float2 *)(g.a.lse + 2 * at);
            g.delta[at] = row_counts(lse) ? -sum : 0.0f;
            g.exponent[at] = (row_counts(lse) ? -lse.y : -INFINITY) * g.a.inv_scale;
        }
    }
}

// The shift of a request's biases (see Shift): all of its rows have the same, -infinity where every key is masked.
__device__ __forceinline__ float request_shift(const AttendArgs &a, int64_t row0, int rows)
{
    const float c = rows ? uniform_load(a.lse + 2 * row0 * a.heads) : -INFINITY;
    return c == -INFINITY ? 0.0f : c;
}

// Whether a key can have a weight beside the shift c: not with a bias of -infinity, nor with one so low that no score makes up for it.
__device__ __forceinline__ bool weighs(float bias, float c) { return !(bias - c <= -0x1p100f); }

// Whether a request has one such key.  Then P = 1 and dP = delta by definition, and dq, dk and dbias are zero: what is left of dP - delta in
// 32 bits is rounding.  The loop ends where a second one is found, mostly in its first round.
template <int DT, bool BIAS>
__device__ __forceinline__ bool one_key(const AttendArgs &a, int64_t key0, int len, float c)
{
    if (!BIAS || len < 2) return len == 1;
    int live = 0;
    for (int at = threadIdx.x & 63; live < 2; at += 256) {
#pragma unroll
        for (int i = 0; i < 4; ++i) live += __popcll(__ballot(at + 64 * i < len && weighs(load16<DT>(a.bias + 2 * (key0 + min(at + 64 * i, len - 1))), c)));
        if (uniform(at) + 256 >= len) break;
    }
    return live == 1;
}

// What the rows bring (-lse / scale, -delta) and the keys' biases over the scale are what the matrix instruction adds the products to;
// a weight then takes one multiply-add and an exponential.  P and dS round to the type before they are multiplied again; P, which is at most 1
// and with many keys far below what fp16 holds in full (2^-14), times 2^WEIGHT there, which dv is freed of in the end.
// Measured on 16 requests of 456 tokens x 16 heads, 6250 keys of 4 heads, D = 128, biases: grad_k 843 us (746 GFLOP, 0.89 PFLOP/s),
// grad_q 598 (560 GFLOP, 0.94 PFLOP/s; its sums of dS and |dS| take 50 of them), delta 12 (180 MB, 4.6 TB/s with the statistics), the last
// launch 6.  Bound by products and what feeds them: before those sums, without exponentials both together took 1454 in place of 1522, without
// loads 1298.  Both in one launch are no faster (the same for short answers, 1684 in place of 1565 for these).

// --- gradients of keys and values ---------------------------------------------------------------------------------------------
// A wave of 32 keys would hold their keys, values and both sums, 192 registers, before it multiplies anything.  So two waves of
// one SIMD share 32 keys: the first forms P (keys and the sum dv in registers), the second, a phase behind, takes P from LDS and
// forms dS (values and the sum dk in registers).  Each does half of the products; P, in 32 bits, costs a fifth of the traffic in LDS.
// The two kinds run in phases like the forward kernel's groups (k_attend_many.hip), products on one side, exponentials on the other;
// the first kind asks for q, the second for dO, two steps ahead.
#define WEIGHT 15
constexpr __device__ float powf2(int e) { return __builtin_bit_cast(float, (e + 127) << 23); }
template <int NW>
struct GradK {
    static constexpr int PAIRS = NW / 2, KEYS = PAIRS * 32, SHIFT = NW == 8 ? 7 : 6, ROWS = NW == 8 ? 64 : 32;  // rows of a step
    static constexpr int AHEAD = 2, Q_TILES = AHEAD + 2, O_TILES = AHEAD + 1;  // q is read in four phases, dO in two
};

template <int D, int NW>
struct GradKLds {
    using K = GradK<NW>;
    char q[K::Q_TILES][K::ROWS * D * 2], o[K::O_TILES][K::ROWS * D * 2];
    float p[K::PAIRS][K::ROWS / 32][4][64][4];   // as the first wave's registers hold it
    float row[NW][4][64];                        // each wave's own: the rows' exponents, or their deltas
};

template <int DT, int D, int NW, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void grad_k_kernel(GradArgs g, int64_t tiles, int splits)
{
    using K = GradK<NW>;
    constexpr int ROWS = K::ROWS, BLOCKS = ROWS / 32, CHUNKS = D / 8, AT_ONCE = 512 / D, N = ROWS / AT_ONCE / K::PAIRS;
    const AttendArgs &a = g.a;
    __shared__ __align__(16) GradKLds<D, NW> lds;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    const int second = wave >= K::PAIRS, pair = second ? wave - K::PAIRS : wave;
    const WorkPlace w = work_place(a, tiles, splits, blockIdx.x);
    const int head = w.head, split = w.split;
    const int of = min(lane, a.n - 1);
    const int work = (int)(a.q_offsets[of + 1] - a.q_offsets[of]);
    const TilePlace tp = a.n <= SORTED_REQUESTS ? find_sorted_tile(a.k_offsets, a.n, a.num_keys, 1, K::SHIFT, w.place, work)
                                                : find_tile(a.k_offsets, a.n, a.num_keys, 1, K::SHIFT, w.place);
    if (tp.r < 0) return;
    const int len = (int)(tp.end - tp.begin);
    const int64_t row0 = clamp64(uniform_load(a.q_offsets + tp.r), 0, a.num_queries);
    const int tokens = (int)(clamp64(uniform_load(a.q_offsets + tp.r + 1), row0, a.num_queries) - row0), rows = tokens * a.group;
    const int steps = (rows + ROWS - 1) / ROWS, share = (steps + splits - 1) / splits;
    const int begin = split * share, end = min(steps, begin + share);

    const int key = tp.tile * K::KEYS + pair * 32 + (lane & 31);
    const bool there = key < len;
    i32x4 kv[D / 16];  // the first wave's keys, the second one's values
    {
        const char *x = second ? a.v : a.k;
        const int64_t token = second ? a.v_token : a.k_token, hd = second ? a.v_head : a.k_head;
        const char *at = x + (tp.begin + (there ? key : len - 1)) * token + head * hd + h * 16;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) kv[s] = *(const i32x4 *)(at + s * 32);
    }
    float bias = 0.0f;
    if (BIAS) bias = there ? load16<DT>(a.bias + 2 * (tp.begin + key)) : 0.0f;
    const float c = BIAS ? request_shift(a, row0, rows) : 0.0f, cs = a.scale * LOG2E, bias_e = (bias - c) * LOG2E + (DT == PLAID_FP16 ? WEIGHT : 0);
    const bool alone = BIAS && beside(c);
    f32x16 sum[D / 32];  // the first wave's dv, the second one's dk
#pragma unroll
    for (int t = 0; t < D / 32; ++t) sum[t] = zero16();
    float dbias = 0.0f;

    // Rows past the end repeat the last one, which the last step leaves out; tiles past the last repeat that.  Where a step is a whole number of tokens a lane's rows
    // lie at the same distances from the step's first token in every step.
    const bool aligned = ROWS % a.group == 0;
    // The first waves bring q, the second ones dO.
    const char *mine = second ? g.d_out : a.q;
    const int64_t token_bytes = second ? (int64_t)a.heads * (D * 2) : a.q_token, head_bytes = second ? D * 2 : a.q_head;
    uint32_t off[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int in = (pair * N + i) * AT_ONCE + lane / CHUNKS, chunk = (lane % CHUNKS) ^ swizzle<D>(in), token = row_token(a, in), hd = in - token * a.group;
        off[i] = (uint32_t)token * (uint32_t)token_bytes + (uint32_t)hd * (uint32_t)head_bytes + chunk * 16;
    }
    // the tiles' places in the rings; nothing below branches on the kind of wave but the weights
    auto q_tile = [&](int step) { return (uint32_t)step % K::Q_TILES * (uint32_t)sizeof(lds.q[0]); };
    auto o_tile = [&](int step) { return (uint32_t)step % K::O_TILES * (uint32_t)sizeof(lds.o[0]); };
    constexpr uint32_t O_AT = K::Q_TILES * sizeof(lds.q[0]);
    using Lds = GradKLds<D, NW>;
    static_assert(offsetof(Lds, o) == O_AT, "dO's ring lies behind q's");
    const char *ring = lds.q[0];
    auto load = [&](int step) {
        const int t = min(step, end - 1);
        const uint32_t to = lds_address(ring) + (second ? O_AT + o_tile(step) : q_tile(step)) + pair * N * 1024;
        if (aligned && (t + 1) * ROWS <= rows) {
            const char *base = mine + (row0 + row_token(a, t * ROWS)) * token_bytes + (int64_t)head * a.group * head_bytes;
#pragma unroll
            for (int i = 0; i < N; ++i) load_to_lds(base, off[i], to + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int in = (pair * N + i) * AT_ONCE + lane / CHUNKS, row = min(t * ROWS + in, rows - 1), chunk = (lane % CHUNKS) ^ swizzle<D>(in);
                const int token = row_token(a, row), hd = head * a.group + row - token * a.group;
                load_to_lds(mine + (row0 + token) * token_bytes + hd * head_bytes + chunk * 16, to + i * 1024);
            }
        }
    };
    auto load_row = [&](int step) {
        const int row = min(min(step, end - 1) * ROWS + lane % ROWS, rows - 1), token = row_token(a, row);
        load4_to_lds((second ? g.delta : g.exponent) + (row0 + token) * a.heads + head * a.group + row - token * a.group, lds.row[wave][step & 3]);
    };
    f32x16 s[BLOCKS];
    i32x4 p[2 * BLOCKS];
    // s = q k^T, or dP = dO v^T; the products are added to what the rows bring, -lse / scale or -delta
    constexpr int EARLY = 4, READS = BLOCKS * D / 16;  // operands that are read before the products of add end
    i32x4 early[EARLY];
    auto operand = [&](int step, int i) { return lds_rows<D>(ring + (second ? O_AT + o_tile(step) : q_tile(step)), 32 * (i % BLOCKS), i / BLOCKS); };
    auto before_form = [&](int step) {
        typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
        const lds_f32x4 *x = (const lds_f32x4 *)&lds.row[wave][step & 3][4 * h];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) s[b] = join16(x[8 * b], x[8 * b + 2], x[8 * b + 4], x[8 * b + 6]);
#pragma unroll
        for (int i = 0; i < EARLY; ++i) early[i] = operand(step, i);
    };
    auto form = [&](int step) {
#pragma unroll
        for (int i = 0; i < READS; ++i) s[i % BLOCKS] = mfma32<DT>(i < EARLY ? early[i] : operand(step, i), kv[i / BLOCKS], s[i % BLOCKS]);
    };
    auto add_operand = [&](int step, int i, int t) { return lds_columns<D>(ring + (second ? q_tile(step) : O_AT + o_tile(step)), 16 * i, t); };
    auto add = [&](int step, int from) {  // dv += dO^T P, or dk += q^T dS
#pragma unroll
        for (int i = from; i < 2 * BLOCKS; ++i)
#pragma unroll
            for (int t = 0; t < D / 32; ++t) sum[t] = mfma32<DT>(add_operand(step, i, t), p[i], sum[t]);
    };
    auto add_dbias = [&]() {
        if (!BIAS || !second) return;
        float sums[4] = {dbias, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[i & 3] += s[b][i];
        dbias = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    };
    auto weights = [&](int step) {
        load_row(step + 2);
        load(step + K::AHEAD);
        if (!second) {
            if (alone) {
                const float *of_row = lds.row[wave][step & 3];
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = vanish(s[b][i], of_row[32 * b + 8 * (i >> 2) + 4 * h + (i & 3)]);
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = BIAS || DT == PLAID_FP16 ? fmaf(s[b][i], cs, bias_e) : s[b][i] * cs;
            if ((step + 1) * ROWS > rows) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (step * ROWS + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3) >= rows) s[b][i] = -INFINITY;  // no row: its weights are 0
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = s[b][4 * i + e] = __builtin_amdgcn_exp2f(s[b][4 * i + e]);
                    *(f32x4 *)lds.p[pair][b][i][lane] = x;
                }
        } else {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 x = *(const f32x4 *)lds.p[pair][b][i][lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][4 * i + e] *= DT == PLAID_FP16 ? x[e] * powf2(-WEIGHT) : x[e];
                }
        }
#pragma unroll
        for (int i = 0; i < 2 * BLOCKS; ++i) p[i] = round8<DT>(s[i >> 1], i & 1);
    };
    constexpr int STEP = N + 1;  // loads of a step: q or dO, and the rows' numbers
    if (begin < end) {
        load_row(begin);
        load(begin);
        load_row(begin + 1);
        load(begin + 1);
        wait_all_loads();  // the keys or values too
        lds_barrier();
        if (second) lds_barrier();
        before_form(begin);
        form(begin);
        lds_barrier();
        for (int step = begin; step + 1 < end; ++step) {
            weights(step);
            wait_loads<STEP *(K::AHEAD - 1)>();  // the next step's have arrived
            lds_barrier();
            __builtin_amdgcn_s_setprio(1);
            i32x4 first[D / 32];
#pragma unroll
            for (int t = 0; t < D / 32; ++t) first[t] = add_operand(step, 0, t);
            __builtin_amdgcn_sched_barrier(0);
            add_dbias();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < D / 32; ++t) sum[t] = mfma32<DT>(first[t], p[0], sum[t]);
            add(step, 1);
            before_form(step + 1);
            constexpr int OTHERS = (2 * BLOCKS - 1) * (D / 32) * 2 + BLOCKS * 4 + EARLY - 6, PAIRS = BLOCKS * (D / 32) - 1;
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (OTHERS + PAIRS - 1) / PAIRS, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            form(step + 1);
#pragma unroll
            for (int i = 0; i < (READS - EARLY) / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, EARLY, 0);
            lds_barrier();
            __builtin_amdgcn_s_setprio(0);
        }
        weights(end - 1);
        lds_barrier();
        add_dbias();
        if (end * ROWS > rows) {
            // what stands in for rows past the end may not be finite and must not meet their weights of zero
#pragma unroll
            for (int i = 0; i < 2 * BLOCKS; ++i) {
                i32x4 keep;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int left = rows - ((end - 1) * ROWS + 16 * i + 8 * (x >> 1) + 4 * h + 2 * (x & 1));
                    keep[x] = left >= 2 ? -1 : left == 1 ? 0xffff : 0;
                }
#pragma unroll
                for (int t = 0; t < D / 32; ++t) sum[t] = mfma32<DT>(add_operand(end - 1, i, t) & keep, p[i], sum[t]);
            }
        } else {
            add(end - 1, 0);
        }
        if (!second) lds_barrier();
        wait_loads<0>();  // nothing may arrive in LDS that is no longer the workgroup's
    }

    dbias = sum_halves(dbias);
    const int own = __popc((uint32_t)__ballot(there && (!BIAS || weighs(bias, c))));  // of the wave's keys
    const bool one = second && own == 1 && one_key<DT, BIAS>(a, tp.begin, len, c);
    if (!there) return;
    // a masked key's column may hold anything and is zero
    const bool masked = BIAS && bias == -INFINITY;
    const int64_t at = (tp.begin + key) * a.kv_heads + head;
    if (BIAS && second && h == 0 && g.dbias_part) g.dbias_part[((int64_t)split * a.kv_heads + head) * a.num_keys + tp.begin + key] = masked || one ? 0.0f : dbias;
    const float factor = second ? g.factor : DT == PLAID_FP16 ? powf2(-WEIGHT) : 1.0f;
    char *out = second ? g.dk : g.dv;
    float *part = second ? g.dk_part : g.dv_part;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = masked || one ? 0.0f : sum[t][4 * i + e] * factor;
            const int d = 32 * t + 8 * i + 4 * h;
            if (splits > 1) *(f32x4 *)(part + ((int64_t)split * a.num_keys * a.kv_heads + at) * D + d) = x;
            else if (out) *(i32x2 *)(out + (at * D + d) * 2) = i32x2{pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])};
        }
}

// --- gradients of queries -----------------------------------------------------------------------------------------------------
// A wave owns 32 rows: q, dO and the sum dq in registers, 32 keys a step.  Workgroups of four waves, two on a compute unit, so that one
// multiplies while the other forms exponentials: a sixth less time than eight waves in phases at D = 128 (545 in place of 650 us), 934 in place
// of 1010 for both gradients at 64.  For a request of at most 32 keys one step sees all of a row, and delta is the sum of P dP over that of P.
//
// Other requests begin with delta = dO . out, whose error, that of an out rounded to the type, grows with |dO| |out| and not with dS: in bf16
// 3.6 of 1000 off in dq where two keys share the weight, 85 where one has 0.99 of it.  But the sum of dS over a row's keys is zero, so what
// it comes to is that error.  It is added to delta, for grad_k_kernel as well, and where it is more than DELTA_OFF of the sum of |dS|, half of
// what rounding dS costs, finish_kernel makes the rows' pass over the keys again: 2.3 of 1000 then, as everywhere.  Weights spread over some
// hundred keys do not come near that; 16 short answers on up to 900 keys, the shortest on 70, pay 5 us for second passes and 5 for joining the sums.
#define GRAD_KEYS 32
#define DELTA_OFF(DT) ((DT) == PLAID_BF16 ? 0x1p-9f : 0x1p-12f)
template <int D, bool BIAS>
struct GradQLds {
    static constexpr int AHEAD = 3, K_TILES = AHEAD + 1, V_TILES = AHEAD;  // keys are read in two phases, values in one
    char k[K_TILES][GRAD_KEYS * D * 2], v[V_TILES][GRAD_KEYS * D * 2];
    float bias[BIAS ? 4 : 1][4][BIAS ? GRAD_KEYS : 4];  // each wave's own
    uint32_t raw[BIAS ? 4 : 1][4][64];                   // as they are loaded
    float2 sums[256];                                    // of dS and |dS| over a lane's keys: there are no registers for them
    int far[4];                                          // whether a wave has a row whose delta was too far off
};

// Workgroup id of a launch's first or second pass.
template <int DT, int D, bool BIAS, bool AGAIN>
__device__ __forceinline__ void grad_q_pass(const GradArgs &g, int64_t tiles, int splits, int id, GradQLds<D, BIAS> &lds)
{
    using L = GradQLds<D, BIAS>;
    constexpr uint32_t TILE = GRAD_KEYS * D * 2;
    constexpr int ROWS = 128, SHIFT = 7, CHUNKS = D / 8, AT_ONCE = 512 / D, N = GRAD_KEYS / AT_ONCE / 4;
    constexpr uint16_t NONE = DT == PLAID_BF16 ? 0xff80 : 0xfc00;  // -infinity
    const AttendArgs &a = g.a;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    if constexpr (AGAIN) {
        if (splits == 1) {
            const i32x4 far = uniform_load((const i32x4 *)g.far + id);
            if (!(far[0] | far[1] | far[2] | far[3])) return;
        }
    }
    const WorkPlace w = work_place(a, tiles, splits, id);
    const int head_kv = w.head, split = w.split;
    const int of = min(lane, a.n - 1);
    const int work = (int)(a.k_offsets[of + 1] - a.k_offsets[of]);
    const TilePlace tp = a.n <= SORTED_REQUESTS ? find_sorted_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, w.place, work)
                                                : find_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, w.place);
    if (tp.r < 0) return;
    const int tokens = (int)(tp.end - tp.begin), rows = tokens * a.group;
    const int row = tp.tile * ROWS + wave * 32 + (lane & 31);
    const bool there = row < rows;
    const int token = row_token(a, there ? row : 0), head = head_kv * a.group + (there ? row : 0) - token * a.group;
    const int64_t at = (tp.begin + token) * a.heads + head;
    float minus_delta;
    if constexpr (AGAIN) {
        minus_delta = g.delta[at];
        if (splits > 1) {  // the parts' sums
            float off = 0.0f, size = 0.0f;
#pragma unroll 4
            for (int i = 0; i < splits; ++i) {
                const float2 x = *(const float2 *)(g.row_part + 2 * ((int64_t)i * a.num_queries * a.heads + at));
                off += x.x, size += x.y;
            }
            minus_delta -= off;
            if (split == 0 && there && h == 0) g.delta_sum[at] = minus_delta;
            const int far = uniform(__any(there && fabsf(off) > DELTA_OFF(DT) * size) ? 1 : 0);
            if (lane == 0) lds.far[wave] = far;
            lds_barrier();
            if (!g.dq || !(lds.far[0] | lds.far[1] | lds.far[2] | lds.far[3])) return;
        }
    }
    const int64_t key0 = clamp64(uniform_load(a.k_offsets + tp.r), 0, a.num_keys);
    const int len = (int)(clamp64(uniform_load(a.k_offsets + tp.r + 1), key0, a.num_keys) - key0);
    const int steps = (len + GRAD_KEYS - 1) / GRAD_KEYS, share = (steps + splits - 1) / splits;
    const int begin = split * share, end = min(steps, begin + share);
    i32x4 q[D / 16], d_out[D / 16];
    {
        const char *pq = a.q + (tp.begin + token) * a.q_token + head * a.q_head + h * 16, *po = g.d_out + at * D * 2 + h * 16;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[s] = *(const i32x4 *)(pq + s * 32), d_out[s] = *(const i32x4 *)(po + s * 32);
    }
    const float2 lse = *(const float2 *)(a.lse + 2 * at);
    const bool counts = row_counts(lse);
    const float c = BIAS ? request_shift(a, tp.begin, rows) : 0.0f, ex = counts ? lse.y * LOG2E : INFINITY, cs = a.scale * LOG2E;
    const bool alone = BIAS && beside(c);
    if constexpr (!AGAIN) {
        minus_delta = counts && steps > 1 ? g.delta[at] : 0.0f;
        lds.sums[threadIdx.x] = float2{0.0f, 0.0f};
    }
    f32x16 dq[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dq[t] = zero16();

    // keys past the end repeat the last one; tiles past the last repeat that
    uint32_t masked = 0;  // keys of bias -infinity, and places past the end, in the tile that is asked for next
    const char *keys = a.k + key0 * a.k_token + head_kv * a.k_head, *values = a.v + key0 * a.v_token + head_kv * a.v_head;
    uint32_t key_row[N], value_row[N], chunk[N];  // bytes of a lane's row in a tile, and within the row
    const uint32_t to_k = lds_address(lds.k[0]) + wave * N * 1024, to_v = lds_address(lds.v[0]) + wave * N * 1024;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int in = (wave * N + i) * AT_ONCE + lane / CHUNKS;
        key_row[i] = (uint32_t)in * (uint32_t)a.k_token, value_row[i] = (uint32_t)in * (uint32_t)a.v_token, chunk[i] = ((lane % CHUNKS) ^ swizzle<D>(in)) * 16;
    }
    auto load = [&](int step) {
        const int t = min(step, end - 1), last = min(len - 1 - t * GRAD_KEYS, GRAD_KEYS - 1);
        const uint64_t first = (uint32_t)t * GRAD_KEYS;
        const char *bk = keys + first * (uint32_t)a.k_token, *bv = values + first * (uint32_t)a.v_token;
        const uint32_t last_k = (uint32_t)last * (uint32_t)a.k_token, last_v = (uint32_t)last * (uint32_t)a.v_token;
        const uint32_t k_at = to_k + (uint32_t)step % L::K_TILES * TILE, v_at = to_v + (uint32_t)step % L::V_TILES * TILE;
        const uint32_t none = masked >> (wave * N * AT_ONCE) >> (lane / CHUNKS);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t off_k = min(key_row[i], last_k) + chunk[i], off_v = min(value_row[i], last_v) + chunk[i];
            if constexpr (BIAS) {
                const bool hidden = none >> (i * AT_ONCE) & 1;
                load_to_lds(hidden ? (const char *)zero_row : bk + off_k, k_at + i * 1024);
                load_to_lds(hidden ? (const char *)zero_row : bv + off_v, v_at + i * 1024);
            } else {
                load_to_lds(bk, off_k, k_at + i * 1024);
                load_to_lds(bv, off_v, v_at + i * 1024);
            }
        }
    };
    const char *biases = a.bias + 2 * key0;
    auto load_bias = [&](int step) {
        const int t = min(step, end - 1), last = len - 1 - t * GRAD_KEYS;
        load2_to_lds(biases + (uint64_t)(uint32_t)t * (2 * GRAD_KEYS), 2 * min(lane & 31, last), lds.raw[wave][step & 3]);
    };
    uint32_t raw = 0;  // read some time before it is used
    auto read_bias = [&](int step) { raw = lds.raw[wave][step & 3][lane]; };
    auto store_bias = [&](int step) {
        const uint16_t x = min(step, end - 1) * GRAD_KEYS + (lane & 31) < len ? (uint16_t)raw : NONE;
        lds.bias[wave][step & 3][lane & 31] = (unpack<DT>(x, 0) - c) * a.inv_scale;
        masked = (uint32_t)__ballot(x == NONE);
    };
    f32x16 s, ds;  // q k^T + b / scale, dO v^T - delta
    i32x4 r[2];
    constexpr int EARLY = 4, READS = 2 * (D / 16);  // operands that are read before the products of add end
    i32x4 early[EARLY];
    auto operand = [&](int step, int i) {
        return lds_rows<D>(i % 2 ? lds.v[(uint32_t)step % L::V_TILES] : lds.k[(uint32_t)step % L::K_TILES], 0, i / 2);
    };
    auto before_form = [&](int step) {
        if constexpr (BIAS) {
            typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
            const lds_f32x4 *b = (const lds_f32x4 *)&lds.bias[wave][step & 3][4 * h];
            s = join16(b[0], b[2], b[4], b[6]);
        } else {
            s = zero16();
        }
#pragma unroll
        for (int i = 0; i < EARLY; ++i) early[i] = operand(step, i);
    };
    auto form = [&](int step) {
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = minus_delta;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            const i32x4 x = i < EARLY ? early[i] : operand(step, i);
            if (i % 2) ds = mfma32<DT>(x, d_out[i / 2], ds);
            else s = mfma32<DT>(x, q[i / 2], s);
        }
    };
    auto add = [&](int step) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < D / 32; ++t) dq[t] = mfma32<DT>(lds_columns<D>(lds.k[(uint32_t)step % L::K_TILES], 16 * i, t), r[i], dq[t]);
    };
    auto weights = [&](int step) {
        if constexpr (BIAS) {
            // the biases that the step before asked for first
            wait_loads<2 * N>();
            read_bias(step + L::AHEAD);
            if (alone) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float b = lds.bias[wave][step & 3][8 * (i >> 2) + 4 * h + (i & 3)];
                    s[i] = b == -INFINITY ? b : vanish(s[i], b);
                }
            }
        } else {
            load(step + L::AHEAD);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], cs, -ex);
        if (!BIAS && (step + 1) * GRAD_KEYS > len) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = step * GRAD_KEYS + 8 * (i >> 2) + 4 * h + (i & 3) < len ? s[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i]);
        if (!AGAIN && steps == 1) {
            float delta = 0.0f, total = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) delta = fmaf(s[i], ds[i], delta), total += s[i];
            delta = sum_halves(delta), total = sum_halves(total);
            delta = total == 0.0f ? 0.0f : delta / total;
            if (there && h == 0) g.delta[at] = -delta;
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] -= delta;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= s[i];
        if constexpr (!AGAIN) {
            float2 &sums = lds.sums[threadIdx.x];
            const float2 former = sums;
            float off[2] = {0.0f, 0.0f}, size[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 16; ++i) off[i & 1] += ds[i], size[i & 1] += fabsf(ds[i]);
            sums = float2{former.x + (off[0] + off[1]), former.y + (size[0] + size[1])};
        }
        r[0] = round8<DT>(ds, 0), r[1] = round8<DT>(ds, 1);
        if constexpr (BIAS) {
            store_bias(step + L::AHEAD);
            load_bias(step + L::AHEAD + 1);
            load(step + L::AHEAD);
        }
    };
    constexpr int STEP = 2 * N + BIAS;  // loads of a step
    if (begin < end) {
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i <= L::AHEAD; ++i) load_bias(begin + i);
            wait_loads<0>();
        }
#pragma unroll
        for (int i = 0; i < L::AHEAD; ++i) {
            if constexpr (BIAS) {
                read_bias(begin + i);
                store_bias(begin + i);
            }
            load(begin + i);
        }
        wait_all_loads();  // the rows too
        lds_barrier();
        before_form(begin);
        form(begin);
        lds_barrier();
        for (int step = begin; step + 1 < end; ++step) {
            weights(step);
            wait_loads<STEP *(L::AHEAD - 1)>();  // the next step's keys and values
            lds_barrier();
            __builtin_amdgcn_s_setprio(1);
            add(step);
            before_form(step + 1);
            constexpr int FIRST = 12, OTHERS = 2 * (D / 32) * 2 + (BIAS ? 4 : 0) + EARLY - FIRST, PAIRS = D / 32 - 1;
            __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (OTHERS + PAIRS - 1) / PAIRS, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            form(step + 1);
#pragma unroll
            for (int i = 0; i < (READS - EARLY) / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, EARLY, 0);
            lds_barrier();
            __builtin_amdgcn_s_setprio(0);
        }
        weights(end - 1);
        lds_barrier();
        add(end - 1);
        wait_loads<0>();  // nothing may arrive in LDS that is no longer the workgroup's
    }
    bool one = AGAIN && one_key<DT, BIAS>(a, key0, len, c);
    if constexpr (!AGAIN) {
        float off = lds.sums[threadIdx.x].x, size = lds.sums[threadIdx.x].y;
        // with one key the two are one number: otherwise there is nothing to look for
        one = !__any(there && fabsf(off) != size) && one_key<DT, BIAS>(a, key0, len, c);
        if (steps <= 1 || !counts || one) off = size = 0.0f;
        off = sum_halves(off), size = sum_halves(size);
        if (splits > 1) {
            if (there && h == 0) *(float2 *)(g.row_part + 2 * ((int64_t)split * a.num_queries * a.heads + at)) = float2{off, size};
        } else {
            if (steps > 1 && there && h == 0) g.delta[at] = minus_delta - off;
            const int far = uniform(__any(there && fabsf(off) > DELTA_OFF(DT) * size) ? 1 : 0);
            if (lane == 0) g.far[4 * (int64_t)id + wave] = far;
        }
    }
    if (!there) return;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = counts && !one ? dq[t][4 * i + e] * g.factor : 0.0f;  // without a key: whatever q holds
            const int d = 32 * t + 8 * i + 4 * h;
            if (splits > 1) *(f32x4 *)(g.dq_part + ((int64_t)split * a.num_queries * a.heads + at) * D + d) = x;
            else if (g.dq) *(i32x2 *)(g.dq + (at * D + d) * 2) = i32x2{pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])};
        }
}
template <int DT, int D, bool BIAS>
__global__ __launch_bounds__(256, 2) void grad_q_kernel(GradArgs g, int64_t tiles, int splits)
{
    __shared__ __align__(16) GradQLds<D, BIAS> lds;
    grad_q_pass<DT, D, BIAS, false>(g, tiles, splits, blockIdx.x, lds);
}

// What the kernels above left in parts, in one launch: out[i] = sum over the parts of part[s][i], in their order, for the rows that a
// request owns.  dbias is a sum over splits and key heads.
struct Sums {
    const float *part;
    char *out;
    int64_t count, per_row;  // values, values of a row: 1 a thread or a multiple of 4
    const int64_t *offsets;
    int32_t parts, n;
    uint32_t groups;         // workgroups up to this sum's last one
};
struct AllSums {
    Sums of[4];
};
template <int DT>
__device__ __forceinline__ void add_parts(const AllSums &all, uint32_t id)
{
    int which = 0;
    while (id >= all.of[which].groups) ++which;
    const Sums &x = all.of[which];
    const int64_t at = (int64_t)(id - (which ? all.of[which - 1].groups : 0)) * 256 + threadIdx.x;
    if (x.per_row == 1) {
        if (at >= x.count || at < x.offsets[0] || at >= x.offsets[x.n]) return;
        float sum = 0.0f;
#pragma unroll 4
        for (int s = 0; s < x.parts; ++s) sum += x.part[s * x.count + at];
        store16<DT>(x.out + 2 * at, sum);
        return;
    }
    const int64_t i = at * 4;
    if (i >= x.count) return;
    const int64_t row = i / x.per_row;
    if (row < x.offsets[0] || row >= x.offsets[x.n]) return;
    f32x4 sum{0, 0, 0, 0};
    for (int s = 0; s < x.parts; ++s) {
        const f32x4 y = *(const f32x4 *)(x.part + s * x.count + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += y[e];
    }
    *(i32x2 *)(x.out + 2 * i) = i32x2{pack2<DT>(sum[0], sum[1]), pack2<DT>(sum[2], sum[3])};
}

template <int DT>
__global__ __launch_bounds__(256) void add_parts_kernel(AllSums all)
{
    add_parts<DT>(all, blockIdx.x);
}
// The second pass of the rows that need one, by `again` workgroups, and sums.  With q's keys in one part it is the last launch, in which
// the sums are those of dbias alone; else it comes before grad_k_kernel and joins the parts' sums of dS.
template <int DT, int D, bool BIAS>
__global__ __launch_bounds__(256, 2) void finish_kernel(GradArgs g, int64_t tiles, int splits, uint32_t again, AllSums all)
{
    __shared__ __align__(16) GradQLds<D, BIAS> lds;
    if (blockIdx.x < again) grad_q_pass<DT, D, BIAS, true>(g, tiles, splits, blockIdx.x, lds);
    else add_parts<DT>(all, blockIdx.x - again);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int DT, int D, int NW>
static void launch_k(hipStream_t st, const GradArgs &g, int splits)
{
    const int64_t tiles = g.a.num_keys / GradK<NW>::KEYS + g.a.n;
    const dim3 grid((unsigned)(tiles * g.a.kv_heads * splits)), block(NW * 64);
    if (g.a.bias) grad_k_kernel<DT, D, NW, true><<<grid, block, 0, st>>>(g, tiles, splits);
    else grad_k_kernel<DT, D, NW, false><<<grid, block, 0, st>>>(g, tiles, splits);
}
template <int DT, int D>
static void launch_q(hipStream_t st, const GradArgs &g, int splits)
{
    const int64_t tiles = g.a.num_queries * g.a.group / 128 + g.a.n;
    const dim3 grid((unsigned)(tiles * g.a.kv_heads * splits)), block(256);
    if (g.a.bias) grad_q_kernel<DT, D, true><<<grid, block, 0, st>>>(g, tiles, splits);
    else grad_q_kernel<DT, D, false><<<grid, block, 0, st>>>(g, tiles, splits);
}
template <int DT, int D>
static void launch_finish(hipStream_t st, const GradArgs &g, int splits, const AllSums &all, uint32_t groups)
{
    const int64_t tiles = g.a.num_queries * g.a.group / 128 + g.a.n;
    const uint32_t again = (uint32_t)(tiles * g.a.kv_heads * splits);
    const dim3 grid(again + groups), block(256);
    if (g.a.bias) finish_kernel<DT, D, true><<<grid, block, 0, st>>>(g, tiles, splits, again, all);
    else finish_kernel<DT, D, false><<<grid, block, 0, st>>>(g, tiles, splits, again, all);
}
template <int DT, int D>
static void launch(hipStream_t st, GradArgs g, int q_splits, int k_waves, int k_splits)
{
    const AttendArgs &a = g.a;
    const int64_t q_values = a.num_queries * a.heads * D, k_values = a.num_keys * a.kv_heads * D;
    AllSums all = {};
    uint32_t groups = 0;
    int sums = 0;
    auto add = [&](const float *part, char *out, int64_t count, int64_t per_row, int parts, const int64_t *offsets) {
        if (!out) return;
        groups += (uint32_t)ceil_div(count, per_row == 1 ? 256 : 1024);
        all.of[sums++] = {part, out, count, per_row, offsets, parts, a.n, groups};
    };
    if (a.num_queries > 0) delta_kernel<DT, D><<<dim3((unsigned)ceil_div(q_values / 8, 256)), dim3(256), 0, st>>>(g);
    // also without dq: what it finds out about delta is dk's and dbias's as well, which are the same whatever is asked for
    const bool rows = (g.dq || g.dk || g.dbias) && a.num_queries > 0;
    if (rows) {
        launch_q<DT, D>(st, g, q_splits);
        if (q_splits > 1) {
            launch_finish<DT, D>(st, g, q_splits, all, 0);
            g.delta = g.delta_sum;  // for dk and dbias
            add(g.dq_part, g.dq, q_values, (int64_t)a.heads * D, q_splits, a.q_offsets);
        } else if (g.dq && k_splits > 1) {
            launch_finish<DT, D>(st, g, 1, all, 0);
        }
    }
    if ((g.dk || g.dv || g.dbias) && a.num_keys > 0) {
        if constexpr (D == 128) {
            if (k_waves == 8) launch_k<DT, D, 8>(st, g, k_splits);
            else launch_k<DT, D, 4>(st, g, k_splits);
        } else {
            launch_k<DT, D, 4>(st, g, k_splits);
        }
        if (k_splits > 1) {
            add(g.dk_part, g.dk, k_values, (int64_t)a.kv_heads * D, k_splits, a.k_offsets);
            add(g.dv_part, g.dv, k_values, (int64_t)a.kv_heads * D, k_splits, a.k_offsets);
        }
        add(g.dbias_part, g.dbias, a.num_keys, 1, k_splits * a.kv_heads, a.k_offsets);
    }
    if (rows && g.dq && q_splits == 1 && k_splits == 1) launch_finish<DT, D>(st, g, 1, all, groups);
    else if (groups > 0) add_parts_kernel<DT><<<dim3(groups), dim3(256), 0, st>>>(all);
}
void plaid_launch_attend_grad(hipStream_t st, const GradArgs &g, int dtype, int head_dim, int q_splits, int k_waves, int k_splits)
{
    if (dtype == PLAID_BF16)
        head_dim == 64 ? launch<PLAID_BF16, 64>(st, g, q_splits, k_waves, k_splits) : launch<PLAID_BF16, 128>(st, g, q_splits, k_waves, k_splits);
    else head_dim == 64 ? launch<PLAID_FP16, 64>(st, g, q_splits, k_waves, k_splits) : launch<PLAID_FP16, 128>(st, g, q_splits, k_waves, k_splits);
}
