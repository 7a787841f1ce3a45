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
// uneven the requests are.  (Where no request has many keys a workgroup of twice the waves takes a tile, and there is nothing to
// join: one launch in place of two.)  A worker's stretch is a tail of a tile, whole tiles and a head of one: whole tiles it finishes,
// the two others leave their sums in its two places, and join_workers_kernel adds them up in the order of the line.
//
// Bound by reading: 64 contexts of 1 to 8192 tokens in the cache, 8 key heads of 128 (279 MB): 58 us = 4.8 TB/s and 8 of joining, which is
// a chain of loads by 64 x 8 workgroups; 4 of 115 000 (523 MB): 101 = 5.2 TB/s and 11; 4 x 65 000 dense keys with biases (1.07 GB): 195 = 5.5
// TB/s and 9.5.  Twice the workers: 65.5 in place of 63.4, and 29 in place of 21 for one context of 20 000.

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
template <int SRC, int NW>
__device__ __forceinline__ Request request(const AttendArgs &a, int r)
{
    Request q;
    q.row0 = clamp64(a.q_offsets[r], 0, a.num_queries);
    q.tokens = (int)(clamp64(a.q_offsets[r + 1], q.row0, a.num_queries) - q.row0);
    q.tiles = (int)(((int64_t)q.tokens * a.group + FEW_ROWS - 1) / FEW_ROWS);
    q.len = key_count<SRC>(a, r, q.key0);
    q.steps = (int)((q.len + NW * 32 - 1) / (NW * 32));
    if (q.steps < 1) q.steps = 1;
    return q;
}
template <int SRC, int NW>
__device__ __forceinline__ Request uniform_request(const AttendArgs &a, int r)
{
    Request q;
    q.row0 = clamp64(uniform_load(a.q_offsets + r), 0, a.num_queries);
    q.tokens = (int)(clamp64(uniform_load(a.q_offsets + r + 1), q.row0, a.num_queries) - q.row0);
    q.tiles = (int)(((int64_t)q.tokens * a.group + FEW_ROWS - 1) / FEW_ROWS);
    q.key0 = 0;
    if constexpr (SRC == PLAID_SOURCE_PAGED) {
        q.len = clamp64(uniform_load(a.lengths + r), 0, (int64_t)a.max_blocks << a.block_shift);
    } else {
        q.key0 = clamp64(uniform_load(a.k_offsets + r), 0, a.num_keys);
        q.len = clamp64(uniform_load(a.k_offsets + r + 1), q.key0, a.num_keys) - q.key0;
    }
    q.steps = (int)((q.len + NW * 32 - 1) / (NW * 32));
    if (q.steps < 1) q.steps = 1;
    return q;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
template <typename T>
__device__ __forceinline__ T wave_prefix(T x)  // sum over lower lanes and this one
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// Steps of all requests and of those before r.  The host takes these kernels where the counts of steps fit 32 bits, a request's whatever the
// offsets hold, all requests' if the offsets ascend.  Others may claim a row many times over: the sum is formed in 64 bits, and where it
// does not fit, 0 is returned and nothing is done.
template <int SRC, int NW>
__device__ __forceinline__ int all_work(const AttendArgs &a, int r, int &before)
{
    int64_t all = 0, some = 0;
    for (int i = threadIdx.x & 63; i < a.n; i += 64) {
        const Request q = request<SRC, NW>(a, i);
        const int w = q.tiles * q.steps;
        all += w;
        if (i < r) some += w;
    }
    before = (int)wave_sum(some);
    all = wave_sum(all);
    return all > INT32_MAX ? 0 : (int)all;
}
// The worker's stretch at .. end - 1 of the line, the request that holds its beginning (-1: the stretch is empty) and the
// place where that request begins.
template <int SRC, int NW>
__device__ __forceinline__ int find_work(const AttendArgs &a, int workers, int worker, int &at, int &end, int &first)
{
    const int lane = threadIdx.x & 63, per = (a.n + 63) >> 6;
    int64_t sum = 0;
    for (int i = lane * per; i < min(a.n, (lane + 1) * per); ++i) {
        const Request q = request<SRC, NW>(a, i);
        sum += q.tiles * q.steps;
    }
    const int64_t sums = wave_prefix(sum), all = uniform(__shfl(sums, 63));
    if (all > INT32_MAX) return -1;
    const int mine = (int)sum, upto = (int)sums, total = (int)all, share = (int)(((uint32_t)total + workers - 1) / (uint32_t)workers);
    if ((int64_t)worker * share >= total) return -1;
    at = worker * share;
    end = min(total, at + share);
    const int block = __popcll(__ballot(upto <= at));  // lanes whose requests all end before
    if (per == 1) {
        first = uniform(__shfl(upto - mine, block));
        return block;
    }
    int left = __shfl(upto - mine, block);
    for (int i = block * per; i < a.n; i += 64) {
        int w = 0;
        if (i + lane < a.n) {
            const Request q = request<SRC, NW>(a, i + lane);
            w = q.tiles * q.steps;
        }
        const int to = left + wave_prefix(w), k = __popcll(__ballot(to <= at));
        if (k < 64) {
            first = uniform(__shfl(to - w, k));
            return uniform(i + k);
        }
        left = __shfl(to, 63);
    }
    return -1;
}

template <int DT, int D, int SRC>
struct Piece {  // a wave's 32 keys on their way in
    i32x4 k[2][D / 32], v[D / 16];
    int bias[4];
};
template <int DT, int D>
struct Piece<DT, D, PLAID_SOURCE_PAGED> {
    i32x4 k[2], v[2], vs[2];
    int ks[2];
};

template <int D, int NW, int SRC>
struct FewLds {
    union {
        char v[SRC == PLAID_SOURCE_PAGED ? 16 : NW * 32 * D * 2];  // dense values, a part for each wave
        float o[NW][FEW_ROWS][D + 4];
    };
    float ml[NW][FEW_ROWS][2], shift[NW];
    int any[NW];  // whether a wave has seen a key that is not masked
};

// Keys and values of a piece are loaded apart, each into the registers that its predecessor has just left: the scores of a
// step are formed while its values are still on their way, and the next keys are asked for before the softmax.
template <int DT, int D, int NW, int SRC>
__global__ __launch_bounds__(NW * 64, FEW_PER_SIMD(D, SRC)) void attend_few_kernel(AttendArgs a, int workers)
{
    constexpr int KS = D / 32, OT = D / 16;  // steps of the score product, tiles of the output
    constexpr bool PAGED = SRC == PLAID_SOURCE_PAGED, BIAS = SRC == PLAID_SOURCE_BIAS;
    __shared__ __align__(16) FewLds<D, NW, SRC> lds;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), kg = lane >> 4, m16 = lane & 15;
    const int head_kv = blockIdx.x % a.kv_heads, worker = blockIdx.x / a.kv_heads;
    int at, end, first, r;
    if (workers) {
        r = find_work<SRC, NW>(a, workers, worker, at, end, first);
    } else {  // a workgroup for each tile
        const TilePlace tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, 4, worker);
        r = tp.r;
        if (r >= 0) first = 0, at = tp.tile * uniform_request<SRC, NW>(a, r).steps, end = at + 1;
    }
    if (r < 0) return;
    const float cs = BIAS ? LOG2E : a.scale * LOG2E;

    while (at < end) {
        Request rq = uniform_request<SRC, NW>(a, r);
        while (at >= first + rq.tiles * rq.steps) {  // to the request that owns the place
            first += rq.tiles * rq.steps;
            rq = uniform_request<SRC, NW>(a, ++r);
        }
        const int tile = (int)((uint32_t)(at - first) / (uint32_t)rq.steps), begin = at - first - tile * rq.steps;
        const int stop = workers ? min(rq.steps, begin + (end - at)) : rq.steps;
        const int rows = rq.tokens * a.group, row = tile * FEW_ROWS + m16;
        const bool there = row < rows;
        const int token = row_token(a, there ? row : 0), head = head_kv * a.group + (there ? row : 0) - token * a.group;
        const int len = (int)rq.len;
        int limit = len, least = len;
        if constexpr (PAGED)
            if (a.causal) {
                const int64_t all = uniform_load(a.lengths + r);
                limit = there ? (int)clamp64(all - rq.tokens + token + 1, 0, len) : len;
                // the tile's first token sees the least
                least = (int)clamp64(all - rq.tokens + row_token(a, tile * FEW_ROWS) + 1, 0, len);
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
        Shift shift;
        int bad[KS];  // paged: the first key of those that are hidden from some row whose values of 32 dimensions are not finite
#pragma unroll
        for (int g = 0; g < KS; ++g) bad[g] = INT32_MAX;

        // --- loads of a piece
        Piece<DT, D, SRC> x;
        int ids[2] = {-1, -1}, in[2] = {0, 0};  // paged: the blocks of the cells loaded last, the cells' places in them
        bool ok[2] = {true, true};              // whether the keys' cells have a block
        auto find = [&](int step) {
            if constexpr (PAGED) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int key = step * (NW * 32) + wave * 32 + 16 * c;
                    ids[c] = -1;
                    if (key < len) ids[c] = uniform_load(a.table + r * a.table_stride + (key >> a.block_shift));
                    in[c] = key & ((1 << a.block_shift) - 1);
                }
            }
        };
        auto cell = [&](int c) { return a.cache + ((int64_t)ids[c] * a.kv_heads + head_kv) * ((int64_t)(D * 17 / 16) << a.block_shift); };
        auto load_k = [&](int step) {
            const int key0 = step * (NW * 32) + wave * 32;
            if constexpr (PAGED) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    ok[c] = (uint32_t)ids[c] < (uint64_t)a.num_blocks;
                    x.k[c] = i32x4{0, 0, 0, 0};
                    x.ks[c] = 0;
                    if (ok[c]) {
                        const uint8_t *p = cell(c) + in[c] * (D / 2), *s = cell(c) + (D << a.block_shift) + in[c] * KS;
                        const uint32_t off = m16 * (D / 2) + kg * (D / 8);
                        if constexpr (D == 128) {
                            x.k[c] = *(const i32x4 *)(p + off);
                        } else {
                            const i32x2 y = *(const i32x2 *)(p + off);
                            x.k[c] = i32x4{y[0], y[1], 0, 0};
                        }
                        x.ks[c] = s[(uint32_t)(m16 * KS + (kg * KS) / 4)];
                    }
                }
            } else {
                const char *base = a.k + (rq.key0 + key0) * a.k_token + head_kv * a.k_head;
                const int last = len - 1 - key0;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    // a key past the end is masked whatever it holds: the last one stands for it
                    const uint32_t off = (uint32_t)(16 * c + m16 <= last ? 16 * c + m16 : last) * (uint32_t)a.k_token + kg * (D / 2);
#pragma unroll
                    for (int s = 0; s < KS; ++s) x.k[c][s] = *(const i32x4 *)(base + off + 16 * s);
                }
            }
        };
        auto load_v = [&](int step) {
            const int key0 = step * (NW * 32) + wave * 32;
            if constexpr (PAGED) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    x.v[c] = x.vs[c] = i32x4{0, 0, 0, 0};
                    if ((uint32_t)ids[c] < (uint64_t)a.num_blocks) {
                        const uint8_t *p = cell(c) + ((D / 2) << a.block_shift) + in[c] * (D / 2), *s = cell(c) + ((D + KS) << a.block_shift) + in[c] * KS;
                        const uint32_t off = lane * (D / 8), soff = 4 * kg * KS;
                        if constexpr (D == 128) {
                            x.v[c] = *(const i32x4 *)(p + off), x.vs[c] = *(const i32x4 *)(s + soff);
                        } else {
                            const i32x2 y = *(const i32x2 *)(p + off), z = *(const i32x2 *)(s + soff);
                            x.v[c] = i32x4{y[0], y[1], 0, 0}, x.vs[c] = i32x4{z[0], z[1], 0, 0};
                        }
                    }
                }
            } else {
                const char *base = a.v + (rq.key0 + key0) * a.v_token + head_kv * a.v_head;
                constexpr int AT_ONCE = 512 / D;  // keys that a load of the wave covers
                const int last = len - 1 - key0;
                if (last >= 31) {
                    const uint32_t off = (uint32_t)(lane / (D / 8)) * (uint32_t)a.v_token + lane % (D / 8) * 16;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) x.v[i] = *(const i32x4 *)(base + (uint32_t)(i * AT_ONCE) * (uint32_t)a.v_token + off);
                } else {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        // a value past the end meets a weight of zero; with biases it is left out below
                        const int key = i * AT_ONCE + lane / (D / 8);
                        const char *from = base + (uint32_t)(key < last ? key : last) * (uint32_t)a.v_token + lane % (D / 8) * 16;
                        x.v[i] = *(const i32x4 *)(BIAS || key <= last ? from : (const char *)zero_row);
                    }
                }
                if constexpr (BIAS) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int key = key0 + 16 * c + 4 * kg;
                        const uint16_t *p = (const uint16_t *)a.bias + rq.key0;
                        uint16_t b[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            b[e] = p[min(key + e, len - 1)];
                            if (key + e >= len) b[e] = DT == PLAID_BF16 ? 0xff80 : 0xfc00;
                        }
                        x.bias[2 * c] = b[0] | (b[1] << 16), x.bias[2 * c + 1] = b[2] | (b[3] << 16);
                    }
                }
            }
        };
        // whether the wave has keys in the step; a key past the end stands in for none only where there is one
        auto has = [&](int step) { return step < stop && step * (NW * 32) + wave * 32 < len; };

        if (has(begin)) {
            find(begin);
            load_k(begin);
            load_v(begin);
        }
        for (int step = begin; has(step); ++step) {
            const int key0 = step * (NW * 32) + wave * 32;
            const bool more = has(step + 1);
            const bool held0 = ok[0], held1 = ok[1];
            int bias[4];
            if (more) find(step + 1);
            char *mine = nullptr;
            if constexpr (!PAGED) {
                mine = lds.v + wave * (32 * D * 2);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const int unit = i * 64 + lane;
                    *(i32x4 *)(mine + lds_chunk<D>(unit / (D / 8), unit % (D / 8))) = x.v[i];
                }
                if constexpr (BIAS)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[e] = x.bias[e];
                if (more) load_v(step + 1);
            }
            f32x4 s[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                s[c] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int d = 0; d < KS; ++d) {
                    i32x4 k;
                    if constexpr (PAGED) {
                        const float power = scale_power(x.ks[c], 0);
                        const int w = x.k[c][d];
                        k = i32x4{codes2<DT, 0>(w, power), codes2<DT, 1>(w, power), codes2<DT, 2>(w, power), codes2<DT, 3>(w, power)};
                    } else {
                        k = x.k[c][d];
                    }
                    s[c] = mfma16<DT>(k, q[d], s[c]);
                }
            }
            if (more) load_k(step + 1);
            if constexpr (BIAS) {
                float b[8], largest = -INFINITY;
                bool unusual = false, usual = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    b[e] = unpack<DT>(bias[e >> 1], e & 1);
                    const bool is = unusual_bias(b[e]);
                    unusual = unusual || is;
                    usual = usual || (!is && b[e] != -INFINITY);
                    largest = is ? fmaxf(largest, b[e]) : largest;
                }
                const float c = shift.c;
                shift.add(__ballot(unusual), largest, __any(usual));
                m += c - shift.c;  // m is relative to the shift
                const float scale = beside(shift.c) ? __int_as_float(1) : a.scale;  // what is finite vanishes, an infinity stays one
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e >> 2][e & 3] = b[e] == -INFINITY ? -INFINITY : fmaf(s[e >> 2][e & 3], scale, b[e] - shift.c);
            } else if (key0 + 32 > least || !held0 || !held1) {
                // some key of the piece is hidden from some row
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 16 * c + 4 * kg + e;
                        s[c][e] = key < limit && (c ? held1 : held0) ? s[c][e] : -INFINITY;
                        if constexpr (PAGED) {
                            // a token past the end may hold anything: with the smallest power its products with a weight of 0 are 0
                            if constexpr (D == 128) x.vs[c][e] = key < len ? x.vs[c][e] : 0;
                            else x.vs[c][e >> 1] &= key < len ? -1 : (e & 1 ? 0xffff : (int)0xffff0000);
                            // so may one that only some of the rows see: those get what it holds at the end
                            if (least < len && key >= least) {
#pragma unroll
                                for (int g = 0; g < KS; ++g) {
                                    const int byte = e * KS + g, mask = 255 << 8 * (byte & 3);
                                    if ((x.vs[c][byte >> 2] & mask) == mask) bad[g] = min(bad[g], key), x.vs[c][byte >> 2] &= ~mask;
                                }
                            }
                        }
                    }
            }
            const float top = max_halves(max_rows(larger(larger(larger(s[0][0], s[0][1]), larger(s[0][2], s[0][3])),
                                                         larger(larger(s[1][0], s[1][1]), larger(s[1][2], s[1][3])))));
            if (__any(!((top - m) * cs <= 8.0f))) {  // also where there was no key so far
                const float to = fmaxf(m, top);
                const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - to) * cs);
                m = to;
                l *= alpha;
#pragma unroll
                for (int t = 0; t < OT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][e] *= alpha;
            }
            const float ref_cs = m == -INFINITY ? 0.0f : m * cs;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = fmaf(s[c][e], cs, -ref_cs);
                    s[c][e] = __builtin_amdgcn_exp2f(y);
                    l += s[c][e];
                }
            const i32x4 p{pack2<DT>(s[0][0], s[0][1]), pack2<DT>(s[0][2], s[0][3]), pack2<DT>(s[1][0], s[1][1]), pack2<DT>(s[1][2], s[1][3])};
            if constexpr (PAGED) {
#pragma unroll
                for (int g = 0; g < KS; ++g) {
                    i32x4 lo, hi;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int w = x.v[c][g];
                        int y[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const int byte = t * KS + g;  // scale bytes [token][group]
                            const float power = scale_power(x.vs[c][byte >> 2], byte & 3);
                            y[t] = t == 0   ? codes2<DT, 0>(w, power)
                                   : t == 1 ? codes2<DT, 1>(w, power)
                                   : t == 2 ? codes2<DT, 2>(w, power)
                                            : codes2<DT, 3>(w, power);
                        }
                        lo[2 * c] = (int)__builtin_amdgcn_perm(y[1], y[0], 0x05040100), lo[2 * c + 1] = (int)__builtin_amdgcn_perm(y[3], y[2], 0x05040100);
                        hi[2 * c] = (int)__builtin_amdgcn_perm(y[1], y[0], 0x07060302), hi[2 * c + 1] = (int)__builtin_amdgcn_perm(y[3], y[2], 0x07060302);
                    }
                    o[2 * g] = mfma16<DT>(lo, p, o[2 * g]);
                    o[2 * g + 1] = mfma16<DT>(hi, p, o[2 * g + 1]);
                }
                if (more) load_v(step + 1);
            } else {
                i32x4 keep{-1, -1, -1, -1};  // what masked keys hold must not meet their zero weights
                if constexpr (BIAS) {
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        keep[w] = (unpack<DT>(bias[w], 0) == -INFINITY ? 0 : 0xffff) | (unpack<DT>(bias[w], 1) == -INFINITY ? 0 : (int)0xffff0000);
                }
                const int rr = m16 >> 2, cc = (m16 & 3) >> 1, swz = swizzle<D>(4 * kg + rr);  // rows 16 apart have one number
                typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
                for (int t = 0; t < OT; ++t) {
                    const char *y = mine + (4 * kg + rr) * (D * 2) + (((2 * t + cc) ^ swz) << 4) + (m16 & 1) * 8;
                    const i32x2 u = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)y));
                    const i32x2 w = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(y + 16 * (D * 2))));
                    if constexpr (BIAS) o[t] = mfma16<DT>(i32x4{u[0] & keep[0], u[1] & keep[1], w[0] & keep[2], w[1] & keep[3]}, p, o[t]);
                    else o[t] = mfma16<DT>(i32x4{u[0], u[1], w[0], w[1]}, p, o[t]);
                }
            }
        }

        if (PAGED && least < len) {
#pragma unroll
            for (int g = 0; g < KS; ++g) {
                if (!__any(bad[g] != INT32_MAX)) continue;
                bad[g] = min(bad[g], __shfl_xor(bad[g], 16));
                bad[g] = min(bad[g], __shfl_xor(bad[g], 32));
                if (bad[g] < limit) o[2 * g] = o[2 * g + 1] = f32x4{NAN, NAN, NAN, NAN};
            }
        }

        // --- the waves' sums joined
        l = sum_halves(sum_rows(l));
        const float natural = BIAS ? m : (m == -INFINITY ? m : m * a.scale);
        __syncthreads();  // the values of all waves have been read, and a former tile's sums
#pragma unroll
        for (int t = 0; t < OT; ++t) *(f32x4 *)&lds.o[wave][m16][16 * t + 4 * kg] = o[t];
        if (kg == 0) lds.ml[wave][m16][0] = natural, lds.ml[wave][m16][1] = l;
        if (lane == 0) lds.shift[wave] = shift.c, lds.any[wave] = shift.any();
        __syncthreads();
        const int count = min(FEW_ROWS, rows - tile * FEW_ROWS);  // rows that there are
        for (int u = threadIdx.x; u < count * (D / 4); u += NW * 64) {
            const int y = u / (D / 4), d = u % (D / 4) * 4;  // a row and 4 of its dimensions
            float base = -INFINITY, top = -INFINITY, sum = 0.0f;
            f32x4 acc{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < NW; ++i) base = fmaxf(base, lds.ml[i][y][1] == 0.0f && !(BIAS && lds.any[i]) ? -INFINITY : lds.shift[i]);
            const float c = base == -INFINITY ? 0.0f : base;
#pragma unroll
            for (int i = 0; i < NW; ++i) top = fmaxf(top, lds.shift[i] - c + lds.ml[i][y][0]);
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const float w = __builtin_amdgcn_exp2f((lds.shift[i] - c + lds.ml[i][y][0] - ref) * LOG2E);
                const f32x4 z = *(const f32x4 *)&lds.o[i][y][d];
                sum += w * lds.ml[i][y][1];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += w * z[e];
            }
            const int row_out = tile * FEW_ROWS + y;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const float2 lse = base == -INFINITY ? float2{-INFINITY, 0.0f} : float2{base, top + logf(sum)};
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] *= inv;
            if (begin == 0 && stop == rq.steps) {
                const int tk = row_token(a, row_out);
                const int64_t to = (rq.row0 + tk) * a.heads + head_kv * a.group + row_out - tk * a.group;
                *(i32x2 *)(a.out + (to * D + d) * 2) = i32x2{pack2<DT>(acc[0], acc[1]), pack2<DT>(acc[2], acc[3])};
                if (a.lse && d == 0) *(float2 *)(a.lse + 2 * to) = lse;
            } else {
                const int64_t slot = ((int64_t)worker * 2 + (begin == 0)) * a.kv_heads + head_kv;
                *(f32x4 *)(a.part_o + (slot * FEW_ROWS + y) * D + d) = acc;
                if (d == 0) *(float2 *)(a.part_lse + (slot * FEW_ROWS + y) * 2) = lse;
            }
        }
        __syncthreads();  // before the next tile's values and sums
        at += stop - begin;
    }
}

// Tiles that several workers have parts of, joined in the order of the line.
#define JOIN_THREADS 512
#define JOIN_PARTS 16
template <int DT, int D, int NW, int SRC>
__global__ __launch_bounds__(JOIN_THREADS) void join_workers_kernel(AttendArgs a, int workers)
{
    __shared__ float s_shift[JOIN_THREADS], s_top[JOIN_THREADS], s_sum[JOIN_THREADS];
    __shared__ __align__(16) f32x4 s_acc[JOIN_THREADS];
    const TilePlace tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, 4, blockIdx.x);
    if (tp.r < 0) return;
    const int head_kv = blockIdx.y;
    int before;
    const int total = all_work<SRC, NW>(a, tp.r, before), share = (int)(((uint32_t)total + workers - 1) / (uint32_t)workers);
    if (total == 0) return;
    const Request rq = request<SRC, NW>(a, tp.r);
    const int begin = before + tp.tile * rq.steps, end = begin + rq.steps;
    const int w0 = (int)((uint32_t)begin / (uint32_t)share), w1 = (int)((uint32_t)(end - 1) / (uint32_t)share);
    if (w0 == w1) return;
    // PARTS groups of threads take every PARTS-th worker's sums each, then the groups' sums are joined: the order is fixed
    const int rows = min(FEW_ROWS, rq.tokens * a.group - tp.tile * FEW_ROWS), units = rows * (D / 4);
    const int parts = min(min(w1 - w0 + 1, JOIN_PARTS), JOIN_THREADS / units);
    const int part = threadIdx.x / units, u = threadIdx.x % units, y = u / (D / 4), d = u % (D / 4) * 4;
    auto place = [&](int w) { return (((int64_t)w * 2 + (w == w0)) * a.kv_heads + head_kv) * FEW_ROWS + y; };
    float c = -INFINITY, top = -INFINITY, sum = 0.0f;
    f32x4 acc{0, 0, 0, 0};
    if (part < parts) {
#pragma unroll 4
        for (int w = w0 + part; w <= w1; w += parts) {
            const float2 x = *(const float2 *)(a.part_lse + 2 * place(w));
            // relative to the largest shift so far
            const float to = fmaxf(c, x.x), moved = top + (c == -INFINITY ? 0.0f : c - to), next = x.x - to + x.y;
            if (x.x != -INFINITY) top = fmaxf(moved, next), c = to;
        }
        const float base = c == -INFINITY ? 0.0f : c, ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
        for (int w = w0 + part; w <= w1; w += parts) {
            const int64_t p = place(w);
            const float2 x = *(const float2 *)(a.part_lse + 2 * p);
            const float f = __builtin_amdgcn_exp2f((x.x - base + x.y - ref) * LOG2E);
            sum += f;
            const f32x4 v = *(const f32x4 *)(a.part_o + p * D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += f * v[e];
        }
        s_shift[threadIdx.x] = c, s_top[threadIdx.x] = top, s_sum[threadIdx.x] = sum, s_acc[threadIdx.x] = acc;
    }
    __syncthreads();
    if (part) return;
    for (int i = 0; i < parts; ++i) c = fmaxf(c, s_shift[i * units + u]);
    const float base = c == -INFINITY ? 0.0f : c;
    top = -INFINITY;
    for (int i = 0; i < parts; ++i) top = fmaxf(top, s_shift[i * units + u] - base + s_top[i * units + u]);
    const float ref = top == -INFINITY ? 0.0f : top;
    sum = 0.0f;
    acc = f32x4{0, 0, 0, 0};
    for (int i = 0; i < parts; ++i) {
        const float f = __builtin_amdgcn_exp2f((s_shift[i * units + u] - base + s_top[i * units + u] - ref) * LOG2E);
        const f32x4 v = s_acc[i * units + u];
        sum += f * s_sum[i * units + u];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += f * v[e];
    }
    const int row = tp.tile * FEW_ROWS + y, tk = row_token(a, row);
    const int64_t to = (rq.row0 + tk) * a.heads + head_kv * a.group + row - tk * a.group;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *(i32x2 *)(a.out + (to * D + d) * 2) = i32x2{pack2<DT>(acc[0] * inv, acc[1] * inv), pack2<DT>(acc[2] * inv, acc[3] * inv)};
    if (a.lse && d == 0) *(float2 *)(a.lse + 2 * to) = c == -INFINITY ? float2{-INFINITY, 0.0f} : float2{c, top + logf(sum)};
}

template <int DT, int D, int SRC>
static void launch(hipStream_t st, const AttendArgs &a, int workers, int64_t tiles)
{
    if (!workers) {
        attend_few_kernel<DT, D, 8, SRC><<<dim3((unsigned)(tiles * a.kv_heads)), dim3(512), 0, st>>>(a, 0);
        return;
    }
    attend_few_kernel<DT, D, 4, SRC><<<dim3((unsigned)(workers * a.kv_heads)), dim3(256), 0, st>>>(a, workers);
    if (workers > 1) join_workers_kernel<DT, D, 4, SRC><<<dim3((unsigned)tiles, (unsigned)a.kv_heads), dim3(JOIN_THREADS), 0, st>>>(a, workers);
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
    if (dtype == PLAID_BF16)
        head_dim == 64 ? launch_source<PLAID_BF16, 64>(st, a, source, workers, tiles) : launch_source<PLAID_BF16, 128>(st, a, source, workers, tiles);
    else head_dim == 64 ? launch_source<PLAID_FP16, 64>(st, a, source, workers, tiles) : launch_source<PLAID_FP16, 128>(st, a, source, workers, tiles);
}
