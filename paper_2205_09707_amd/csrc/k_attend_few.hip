// Attention where a request has few rows, single tokens above all: keys and values pass through the chip once, and the work
// is cut along the keys.
#include "reader.h"

// The recurrence of the softmax is that of k_attend_many.hip.  Rows come in tiles of 16; a wave takes 32 keys at a time, as
// s^T = k q^T in two 16 x 16 products, whose registers are the operand of o^T = v^T p^T in the 16 x 16 x 32 product.
// A step of the workgroup is 128 keys, one piece a wave; the waves' sums are joined in LDS at a segment's end.
// The order of the dimensions inside a product is free, so a lane takes D / 4 neighbours of its key: from the cache that is
// one load of 16 bytes (8 at D = 64) under one scale, from a dense tensor D / 32 loads of 16 bytes.  The cache's value codes
// lie as the operand wants them; dense values go through the wave's own LDS and the transposing read.
//
// All tiles' steps, request after request, form one line that the workers (workgroups of a key head) share evenly, however
// uneven the requests are.  A worker's stretch is a tail of a tile, whole tiles and a head of one: whole tiles it finishes,
// the two others leave their sums in its two places, and join_workers_kernel adds them up in the order of the line.

template <int SRC>
__device__ __forceinline__ int64_t key_count(const AttendArgs &a, int r, int64_t &base)
{
    base = 0;
    if constexpr (SRC == PLAID_SOURCE_PAGED) return clamp64(a.lengths[r], 0, (int64_t)a.max_blocks << a.block_shift);
    base = clamp64(a.k_offsets[r], 0, a.num_keys);
    return clamp64(a.k_offsets[r + 1], base, a.num_keys) - base;
}

struct Request {
    int64_t row0, key0, len;
    int tokens, tiles, steps;  // a request without keys has one step, which writes its zeros
};
template <int SRC>
__device__ __forceinline__ Request request(const AttendArgs &a, int r)
{
    Request q;
    q.row0 = clamp64(a.q_offsets[r], 0, a.num_queries);
    q.tokens = (int)(clamp64(a.q_offsets[r + 1], q.row0, a.num_queries) - q.row0);
    q.tiles = (int)(((int64_t)q.tokens * a.group + FEW_ROWS - 1) / FEW_ROWS);
    q.len = key_count<SRC>(a, r, q.key0);
    q.steps = (int)((q.len + FEW_KEYS - 1) / FEW_KEYS);
    if (q.steps < 1) q.steps = 1;
    return q;
}
__device__ __forceinline__ int64_t wave_sum(int64_t x)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ int64_t wave_prefix(int64_t x)  // sum over lower lanes and this one
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// Steps of all requests and of those before r (r = n: of all).
template <int SRC>
__device__ __forceinline__ int64_t all_work(const AttendArgs &a, int r, int64_t &before)
{
    int64_t all = 0, some = 0;
    for (int i = threadIdx.x & 63; i < a.n; i += 64) {
        const Request q = request<SRC>(a, i);
        const int64_t w = (int64_t)q.tiles * q.steps;
        all += w;
        if (i < r) some += w;
    }
    before = wave_sum(some);
    return wave_sum(all);
}
// The request that holds place `at` of the line, and the place where it begins.
template <int SRC>
__device__ __forceinline__ int find_work(const AttendArgs &a, int64_t share_of, int64_t worker, int64_t &total, int64_t &at, int64_t &end, int64_t &first)
{
    const int lane = threadIdx.x & 63, per = (a.n + 63) >> 6;
    int64_t mine = 0;
    for (int i = lane * per; i < min(a.n, (lane + 1) * per); ++i) {
        const Request q = request<SRC>(a, i);
        mine += (int64_t)q.tiles * q.steps;
    }
    const int64_t upto = wave_prefix(mine);
    total = __shfl(upto, 63);
    const int64_t share = (total + share_of - 1) / share_of;
    at = worker * share;
    end = min(total, at + share);
    if (at >= end) return -1;
    const int block = __popcll(__ballot(upto <= at));  // lanes whose requests all end before
    int64_t left = __shfl(upto - mine, block);
    for (int i = block * per;; i += 64) {
        int64_t w = 0;
        if (i + lane < a.n) {
            const Request q = request<SRC>(a, i + lane);
            w = (int64_t)q.tiles * q.steps;
        }
        const int64_t to = left + wave_prefix(w);
        const int k = __popcll(__ballot(to <= at));
        if (k < 64) {
            first = __shfl(to - w, k);
            return i + k;
        }
        left = __shfl(to, 63);
    }
}

template <int DT, int D, int SRC>
struct Piece {  // 32 keys' data of a wave, as loaded
    i32x4 k[2][D / 32], v[D / 16];
    int bias[4];
};
template <int DT, int D>
struct Piece<DT, D, PLAID_SOURCE_PAGED> {
    i32x4 k[2], v[2], vs[2];
    int ks[2], ok[2];
};

template <int D, int SRC>
struct FewLds {
    union {
        char v[SRC == PLAID_SOURCE_PAGED ? 16 : 4 * 32 * D * 2];  // dense values, a part for each wave
        float o[4][FEW_ROWS][D + 4];
    };
    float ml[4][FEW_ROWS][2];
};

template <int DT, int D, int SRC>
__global__ __launch_bounds__(256, 2) void attend_few_kernel(AttendArgs a, int workers)
{
    constexpr int KS = D / 32, OT = D / 16;  // steps of the score product, tiles of the output
    __shared__ __align__(16) FewLds<D, SRC> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = lane >> 4, m16 = lane & 15;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head_kv = (int)(id / workers), worker = (int)(id % workers);
    int64_t total, at, end, first;
    int r = find_work<SRC>(a, workers, worker, total, at, end, first);
    if (r < 0) return;
    const float cs = SRC == PLAID_SOURCE_BIAS ? LOG2E : a.scale * LOG2E;

    while (at < end) {
        Request rq = request<SRC>(a, r);
        while (at >= first + (int64_t)rq.tiles * rq.steps) {  // to the request that owns the place
            first += (int64_t)rq.tiles * rq.steps;
            rq = request<SRC>(a, ++r);
        }
        const int tile = (int)((at - first) / rq.steps), begin = (int)((at - first) % rq.steps);
        const int stop = (int)min((int64_t)rq.steps, begin + (end - at));
        const int rows = rq.tokens * a.group, row = tile * FEW_ROWS + m16;
        const bool there = row < rows;
        const int token = row_token(a, there ? row : 0), head = head_kv * a.group + (there ? row : 0) - token * a.group;
        const int len = (int)rq.len;
        int limit = len;
        if constexpr (SRC == PLAID_SOURCE_PAGED)
            if (a.causal) limit = there ? (int)clamp64((int64_t)a.lengths[r] - rq.tokens + token + 1, 0, len) : len;
        int least = limit;
        if constexpr (SRC == PLAID_SOURCE_PAGED) {
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
        }

        i32x4 q[KS];
        {
            const char *p = a.q + (rq.row0 + token) * a.q_token + head * a.q_head + kg * (D / 2);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                q[s] = i32x4{0, 0, 0, 0};
                if (there) q[s] = *(const i32x4 *)(p + 16 * s);
#pragma unroll
                for (int e = 0; e < 4; ++e) q[s][e] ^= (int)a.negate_q;
            }
        }
        f32x4 o[OT];
#pragma unroll
        for (int t = 0; t < OT; ++t) o[t] = f32x4{0, 0, 0, 0};
        float m = -INFINITY, l = 0.0f;

        // --- loads of a piece
        int ids[2] = {-1, -1};  // paged: the blocks of the piece to be loaded next
        auto find = [&](int step) {
            if constexpr (SRC == PLAID_SOURCE_PAGED) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int key = step * FEW_KEYS + wave * 32 + 16 * c;
                    ids[c] = step < stop && key < len ? a.table[r * a.table_stride + (key >> a.block_shift)] : -1;
                }
            }
        };
        auto load = [&](int step, Piece<DT, D, SRC> &x) {
            const int key0 = step * FEW_KEYS + wave * 32;
            if constexpr (SRC == PLAID_SOURCE_PAGED) {
                const int64_t bs = 1ll << a.block_shift;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int in = (key0 + 16 * c) & (int)(bs - 1);
                    x.ok[c] = (uint32_t)ids[c] < (uint64_t)a.num_blocks;
                    x.k[c] = x.v[c] = x.vs[c] = i32x4{0, 0, 0, 0};
                    x.ks[c] = 0;
                    if (x.ok[c]) {
                        const uint8_t *p = a.cache + ((int64_t)ids[c] * a.kv_heads + head_kv) * (bs * D * 17 / 16);
                        const uint8_t *k = p + (in + m16) * (D / 2) + kg * (D / 8), *v = p + bs * (D / 2) + in * (D / 2) + lane * (D / 8);
                        const uint8_t *ks = p + bs * D + (in + m16) * KS + (kg * KS) / 4, *vs = p + bs * D + bs * KS + (in + 4 * kg) * KS;
                        if constexpr (D == 128) {
                            x.k[c] = *(const i32x4 *)k, x.v[c] = *(const i32x4 *)v, x.vs[c] = *(const i32x4 *)vs;
                        } else {
                            const i32x2 k2 = *(const i32x2 *)k, v2 = *(const i32x2 *)v, s2 = *(const i32x2 *)vs;
                            x.k[c] = i32x4{k2[0], k2[1], 0, 0}, x.v[c] = i32x4{v2[0], v2[1], 0, 0}, x.vs[c] = i32x4{s2[0], s2[1], 0, 0};
                        }
                        x.ks[c] = *ks;
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int key = key0 + 16 * c + m16;
                    const char *p = a.k + (rq.key0 + key) * a.k_token + head_kv * a.k_head + kg * (D / 2);
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        x.k[c][s] = i32x4{0, 0, 0, 0};
                        if (key < len) x.k[c][s] = *(const i32x4 *)(p + 16 * s);
                    }
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const int unit = i * 64 + lane, key = key0 + unit / (D / 8);
                    x.v[i] = i32x4{0, 0, 0, 0};
                    if (key < len) x.v[i] = *(const i32x4 *)(a.v + (rq.key0 + key) * a.v_token + head_kv * a.v_head + unit % (D / 8) * 16);
                }
                if constexpr (SRC == PLAID_SOURCE_BIAS) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int key = key0 + 16 * c + 4 * kg;
                        const uint16_t *p = (const uint16_t *)a.bias + rq.key0 + key;
                        uint16_t b[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) b[e] = key + e < len ? p[e] : (DT == PLAID_BF16 ? 0xff80 : 0xfc00);
                        x.bias[2 * c] = b[0] | (b[1] << 16), x.bias[2 * c + 1] = b[2] | (b[3] << 16);
                    }
                }
            }
        };

        Piece<DT, D, SRC> now, next;
        find(begin);
        load(begin, now);
        find(begin + 1);
        for (int step = begin; step < stop; ++step) {
            if (step + 1 < stop) {
                load(step + 1, next);
                find(step + 2);
            }
            const int key0 = step * FEW_KEYS + wave * 32;
            if (key0 < len) {
                char *mine = nullptr;
                if constexpr (SRC != PLAID_SOURCE_PAGED) {
                    mine = lds.v + wave * (32 * D * 2);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const int unit = i * 64 + lane;
                        *(i32x4 *)(mine + lds_chunk<D>(unit / (D / 8), unit % (D / 8))) = now.v[i];
                    }
                }
                f32x4 s[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    s[c] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int d = 0; d < KS; ++d) {
                        i32x4 k;
                        if constexpr (SRC == PLAID_SOURCE_PAGED) {
                            const float power = scale_power(now.ks[c]);
                            const int w = now.k[c][d];
                            k = i32x4{codes2<DT, 0>(w, power), codes2<DT, 1>(w, power), codes2<DT, 2>(w, power), codes2<DT, 3>(w, power)};
                        } else {
                            k = now.k[c][d];
                        }
                        s[c] = mfma16<DT>(k, q[d], s[c]);
                    }
                }
                bool hide = false;  // whether some key of the piece may be masked for some row
                if constexpr (SRC == PLAID_SOURCE_BIAS) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float b = unpack<DT>(now.bias[2 * c + (e >> 1)], e & 1);
                            s[c][e] = b == -INFINITY ? -INFINITY : fmaf(s[c][e], a.scale, b);
                        }
                } else {
                    hide = key0 + 32 > least;
                    if constexpr (SRC == PLAID_SOURCE_PAGED) hide = hide || !(now.ok[0] & now.ok[1]);
                    if (hide) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                bool seen = key0 + 16 * c + 4 * kg + e < limit;
                                if constexpr (SRC == PLAID_SOURCE_PAGED) seen = seen && now.ok[c];
                                s[c][e] = seen ? s[c][e] : -INFINITY;
                            }
                    }
                }
                float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any((top - m) * cs > 8.0f)) {
                    const float to = fmaxf(m, top);
                    const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - to) * cs);
                    m = to;
                    l *= alpha;
#pragma unroll
                    for (int t = 0; t < OT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][e] *= alpha;
                }
                const float ref = m == -INFINITY ? 0.0f : m, ref_cs = ref * cs;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = SRC == PLAID_SOURCE_BIAS ? (s[c][e] - ref) * cs : fmaf(s[c][e], cs, -ref_cs);
                        s[c][e] = __builtin_amdgcn_exp2f(x);
                        l += s[c][e];
                    }
                const i32x4 p{pack2<DT>(s[0][0], s[0][1]), pack2<DT>(s[0][2], s[0][3]), pack2<DT>(s[1][0], s[1][1]), pack2<DT>(s[1][2], s[1][3])};
                if constexpr (SRC == PLAID_SOURCE_PAGED) {
#pragma unroll
                    for (int g = 0; g < KS; ++g) {
                        i32x4 lo, hi;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int w = now.v[c][g];
                            float power[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                const int byte = t * KS + g;
                                power[t] = scale_power((now.vs[c][byte >> 2] >> ((byte & 3) * 8)) & 255);
                                // a token past the end may hold anything: the smallest power keeps its products with 0 zero
                                if (hide) power[t] = key0 + 16 * c + 4 * kg + t < len ? power[t] : 0.0f;
                            }
                            const int t0 = codes2<DT, 0>(w, power[0]), t1 = codes2<DT, 1>(w, power[1]), t2 = codes2<DT, 2>(w, power[2]),
                                      t3 = codes2<DT, 3>(w, power[3]);
                            lo[2 * c] = (int)__builtin_amdgcn_perm(t1, t0, 0x05040100), lo[2 * c + 1] = (int)__builtin_amdgcn_perm(t3, t2, 0x05040100);
                            hi[2 * c] = (int)__builtin_amdgcn_perm(t1, t0, 0x07060302), hi[2 * c + 1] = (int)__builtin_amdgcn_perm(t3, t2, 0x07060302);
                        }
                        o[2 * g] = mfma16<DT>(lo, p, o[2 * g]);
                        o[2 * g + 1] = mfma16<DT>(hi, p, o[2 * g + 1]);
                    }
                } else {
                    i32x4 keep{-1, -1, -1, -1};  // what masked keys hold must not meet their zero weights
                    if constexpr (SRC == PLAID_SOURCE_BIAS) {
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            keep[w] = (unpack<DT>(now.bias[w], 0) == -INFINITY ? 0 : 0xffff) | (unpack<DT>(now.bias[w], 1) == -INFINITY ? 0 : (int)0xffff0000);
                    }
                    const int rr = m16 >> 2, cc = (m16 & 3) >> 1, swz = (rr << 1) | (kg & 1);
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
                    for (int t = 0; t < OT; ++t) {
                        const char *x = mine + (4 * kg + rr) * (D * 2) + (((2 * t + cc) ^ swz) << 4) + (m16 & 1) * 8;
                        const i32x2 u = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)x));
                        const i32x2 w = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(x + 16 * (D * 2))));
                        o[t] = mfma16<DT>(i32x4{u[0] & keep[0], u[1] & keep[1], w[0] & keep[2], w[1] & keep[3]}, p, o[t]);
                    }
                }
            }
            if (step + 1 < stop) now = next;
        }

        // --- the waves' sums joined
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const float natural = SRC == PLAID_SOURCE_BIAS ? m : (m == -INFINITY ? m : m * a.scale);
        __syncthreads();  // the values of all waves have been read, and a former tile's sums
#pragma unroll
        for (int t = 0; t < OT; ++t) *(f32x4 *)&lds.o[wave][m16][16 * t + 4 * kg] = o[t];
        if (kg == 0) lds.ml[wave][m16][0] = natural, lds.ml[wave][m16][1] = l;
        __syncthreads();
        {
            const int y = threadIdx.x >> 4, x = threadIdx.x & 15;  // a row and D / 16 of its dimensions
            float top = -INFINITY, w[4], sum = 0.0f, acc[D / 16];
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, lds.ml[i][y][0]);
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = __builtin_amdgcn_exp2f((lds.ml[i][y][0] - ref) * LOG2E);
                sum += w[i] * lds.ml[i][y][1];
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                acc[d] = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[d] += w[i] * lds.o[i][y][x * (D / 16) + d];
            }
            const int row_out = tile * FEW_ROWS + y;
            if (begin == 0 && stop == rq.steps) {
                if (row_out < rows) {
                    const int tk = row_token(a, row_out);
                    const int64_t to = (rq.row0 + tk) * a.heads + head_kv * a.group + row_out - tk * a.group;
                    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
                    for (int d = 0; d < D / 16; d += 4)
                        *(i32x2 *)(a.out + (to * D + x * (D / 16) + d) * 2) =
                            i32x2{pack2<DT>(acc[d] * inv, acc[d + 1] * inv), pack2<DT>(acc[d + 2] * inv, acc[d + 3] * inv)};
                    if (a.lse && x == 0) a.lse[2 * to] = sum == 0.0f ? -INFINITY : top, a.lse[2 * to + 1] = sum == 0.0f ? 0.0f : logf(sum);
                }
            } else {
                const int64_t slot = ((int64_t)worker * 2 + (begin == 0)) * a.kv_heads + head_kv;
#pragma unroll
                for (int d = 0; d < D / 16; d += 4)
                    *(f32x4 *)(a.part_o + (slot * FEW_ROWS + y) * D + x * (D / 16) + d) = f32x4{acc[d], acc[d + 1], acc[d + 2], acc[d + 3]};
                if (x == 0) a.part_ml[(slot * FEW_ROWS + y) * 2] = top, a.part_ml[(slot * FEW_ROWS + y) * 2 + 1] = sum;
            }
        }
        __syncthreads();  // before the next tile's values and sums
        at += stop - begin;
    }
}

// Tiles that several workers have parts of, joined in the order of the line.
template <int DT, int D, int SRC>
__global__ __launch_bounds__(256) void join_workers_kernel(AttendArgs a, int workers)
{
    const TilePlace tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, 4, blockIdx.x);
    if (tp.r < 0) return;
    const int head_kv = blockIdx.y;
    int64_t before;
    const int64_t total = all_work<SRC>(a, tp.r, before), share = (total + workers - 1) / workers;
    const Request rq = request<SRC>(a, tp.r);
    const int64_t begin = before + (int64_t)tp.tile * rq.steps, end = begin + rq.steps;
    const int64_t w0 = begin / share, w1 = (end - 1) / share;
    if (w0 == w1) return;
    const int y = threadIdx.x >> 4, x = threadIdx.x & 15, row = tp.tile * FEW_ROWS + y;
    if (row >= rq.tokens * a.group) return;
    auto place = [&](int64_t w) { return ((w * 2 + (w == w0)) * a.kv_heads + head_kv) * FEW_ROWS + y; };
    float top = -INFINITY, sum = 0.0f, acc[D / 16];
    for (int64_t w = w0; w <= w1; ++w) top = fmaxf(top, a.part_ml[2 * place(w)]);
    const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) acc[d] = 0.0f;
#pragma unroll 4
    for (int64_t w = w0; w <= w1; ++w) {
        const int64_t p = place(w);
        const float f = __builtin_amdgcn_exp2f((a.part_ml[2 * p] - ref) * LOG2E);
        sum += f * a.part_ml[2 * p + 1];
#pragma unroll
        for (int d = 0; d < D / 16; d += 4) {
            const f32x4 v = *(const f32x4 *)(a.part_o + p * D + x * (D / 16) + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[d + e] += f * v[e];
        }
    }
    const int tk = row_token(a, row);
    const int64_t to = (rq.row0 + tk) * a.heads + head_kv * a.group + row - tk * a.group;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int d = 0; d < D / 16; d += 4)
        *(i32x2 *)(a.out + (to * D + x * (D / 16) + d) * 2) = i32x2{pack2<DT>(acc[d] * inv, acc[d + 1] * inv), pack2<DT>(acc[d + 2] * inv, acc[d + 3] * inv)};
    if (a.lse && x == 0) a.lse[2 * to] = sum == 0.0f ? -INFINITY : top, a.lse[2 * to + 1] = sum == 0.0f ? 0.0f : logf(sum);
}

template <int DT, int D, int SRC>
static void launch(hipStream_t st, const AttendArgs &a, int workers, int64_t tiles)
{
    attend_few_kernel<DT, D, SRC><<<dim3((unsigned)(workers * a.kv_heads)), dim3(256), 0, st>>>(a, workers);
    if (workers > 1) join_workers_kernel<DT, D, SRC><<<dim3((unsigned)tiles, (unsigned)a.kv_heads), dim3(256), 0, st>>>(a, workers);
}
template <int DT, int D>
static void launch_source(hipStream_t st, const AttendArgs &a, int source, int workers, int64_t tiles)
{
    if (source == PLAID_SOURCE_DENSE) launch<DT, D, PLAID_SOURCE_DENSE>(st, a, workers, tiles);
    else if (source == PLAID_SOURCE_BIAS) launch<DT, D, PLAID_SOURCE_BIAS>(st, a, workers, tiles);
    else launch<DT, D, PLAID_SOURCE_PAGED>(st, a, workers, tiles);
}
void plaid_launch_attend_few(hipStream_t st, const AttendArgs &a, int dtype, int head_dim, int source, int workers, int64_t tiles)
{
    if (dtype == PLAID_BF16) head_dim == 64 ? launch_source<PLAID_BF16, 64>(st, a, source, workers, tiles) : launch_source<PLAID_BF16, 128>(st, a, source, workers, tiles);
    else head_dim == 64 ? launch_source<PLAID_FP16, 64>(st, a, source, workers, tiles) : launch_source<PLAID_FP16, 128>(st, a, source, workers, tiles);
}
