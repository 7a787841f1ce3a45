// Attention where a request has many rows (tokens x heads that share keys): tiles of rows x 64 keys on the matrix units.
#include "reader.h"

// out = softmax(scale q k^T + b) v in one pass over the keys, with the running maximum m and sum l of each row:
//   p = exp(s - m),  l <- l exp(m_old - m) + sum p,  o <- o exp(m_old - m) + p v,  and out = o / l at the end.
// A wave owns 32 rows.  It computes s^T = k q^T, so that a lane holds one row (column l % 32 of the result) and the two halves
// of the wave half of its keys each: the maximum and the sum need one exchange, and the result's registers, rounded, are
// already the operand of o^T = v^T p^T (rows of v^T come from LDS by the transposing read, or lie transposed there).  q stays
// in registers, keys and values of 64 keys at a time go through LDS twice buffered; the next tile's loads are in flight while
// this one is multiplied.  The maximum that p is taken against lags behind the true one by up to 2^8: o is rescaled only
// where it would fall further back.
template <int DT, int D, int NW, int SRC>
struct Stage;  // one tile on its way from memory to LDS

template <int D, int SRC>
struct TileBuffers {
    char k[2][MANY_KEYS * D * 2];
    char v[2][SRC == PLAID_SOURCE_PAGED ? D * (MANY_KEYS + 4) * 2 : MANY_KEYS * D * 2];
    float bias[2][SRC == PLAID_SOURCE_BIAS ? MANY_KEYS : 4];
    int cell[2][4];  // paged: whether the cells of 16 keys have a block
};

struct KeyRange {
    int64_t base;  // dense: the request's first key
    int len;       // keys of the request that there are
    int r, head;   // request, key head
};

template <int DT, int D, int NW, int SRC>
struct Stage {
    static constexpr int THREADS = NW * 64, CHUNKS = D / 8, N = (MANY_KEYS * CHUNKS + THREADS - 1) / THREADS;
    i32x4 k[N], v[N];
    float bias;
    __device__ __forceinline__ void start(const AttendArgs &, const KeyRange &, int) {}
    __device__ __forceinline__ void load(const AttendArgs &a, const KeyRange &kr, int step)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int id = threadIdx.x + i * THREADS, key = id / CHUNKS, c = id % CHUNKS, at = step * MANY_KEYS + key;
            k[i] = v[i] = i32x4{0, 0, 0, 0};
            bool there = id < MANY_KEYS * CHUNKS && at < kr.len;
            // what a masked key holds is never used: infinities there would make products with zero weights not a number
            if constexpr (SRC == PLAID_SOURCE_BIAS) there = there && load16<DT>(a.bias + 2 * (kr.base + at)) != -INFINITY;
            if (there) {
                k[i] = *(const i32x4 *)(a.k + (kr.base + at) * a.k_token + kr.head * a.k_head + c * 16);
                v[i] = *(const i32x4 *)(a.v + (kr.base + at) * a.v_token + kr.head * a.v_head + c * 16);
            }
        }
        if constexpr (SRC == PLAID_SOURCE_BIAS) {
            const int at = step * MANY_KEYS + threadIdx.x;
            if (threadIdx.x < MANY_KEYS) bias = at < kr.len ? load16<DT>(a.bias + 2 * (kr.base + at)) : -INFINITY;
        }
    }
    __device__ __forceinline__ void store(TileBuffers<D, SRC> &b, int buf)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int id = threadIdx.x + i * THREADS, key = id / CHUNKS, c = id % CHUNKS;
            if (id < MANY_KEYS * CHUNKS) {
                *(i32x4 *)(b.k[buf] + lds_chunk<D>(key, c)) = k[i];
                *(i32x4 *)(b.v[buf] + lds_chunk<D>(key, c)) = v[i];
            }
        }
        if constexpr (SRC == PLAID_SOURCE_BIAS)
            if (threadIdx.x < MANY_KEYS) b.bias[buf][threadIdx.x] = bias;
    }
};

// Paged: a unit is 32 dimensions of a key (one scale), or a lane's part of a cell of value codes (4 tokens, D / 16
// dimensions), turned into 16-bit values on the way into LDS.  The block ids are read one tile ahead of the codes.
template <int DT, int D, int NW>
struct Stage<DT, D, NW, PLAID_SOURCE_PAGED> {
    static constexpr int THREADS = NW * 64, G = D / 32, KU = MANY_KEYS * G, VU = MANY_KEYS / 16 * 64, N = (KU + VU + THREADS - 1) / THREADS;
    int id_next[N], ok[N];
    i32x4 code[N], scale[N];
    int len, last[N];

    // first key of a unit in its tile
    static __device__ __forceinline__ int unit_key(int u) { return u < KU ? u / G : ((u - KU) >> 6) * 16 + (((u - KU) >> 4) & 3) * 4; }

    __device__ __forceinline__ void find(const AttendArgs &a, const KeyRange &kr, int step)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, at = step * MANY_KEYS + unit_key(u);
            id_next[i] = u < KU + VU && at < kr.len ? a.table[kr.r * a.table_stride + (at >> a.block_shift)] : -1;
        }
    }
    __device__ __forceinline__ void start(const AttendArgs &a, const KeyRange &kr, int step) { find(a, kr, step); }
    __device__ __forceinline__ void load(const AttendArgs &a, const KeyRange &kr, int step)
    {
        const int64_t bs = 1ll << a.block_shift, region = bs * D * 17 / 16;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, at = step * MANY_KEYS + unit_key(u);
            const int in = at & (int)(bs - 1);
            ok[i] = (uint32_t)id_next[i] < (uint64_t)a.num_blocks;
            last[i] = kr.len - at;  // tokens of the unit that there are
            code[i] = scale[i] = i32x4{0, 0, 0, 0};
            if (ok[i]) {
                const uint8_t *p = a.cache + ((int64_t)id_next[i] * a.kv_heads + kr.head) * region;
                if (u < KU) {
                    code[i] = *(const i32x4 *)(p + in * (D / 2) + (u % G) * 16);
                    scale[i][0] = p[bs * D + in * G + u % G];
                } else {
                    const int l = (u - KU) & 63;
                    const uint8_t *c = p + bs * (D / 2) + (in >> 4) * (8 * D) + l * (D / 8), *s = p + bs * D + bs * G + in * G;
                    if constexpr (D == 128) {
                        code[i] = *(const i32x4 *)c;
                        scale[i] = *(const i32x4 *)s;
                    } else {
                        const i32x2 x = *(const i32x2 *)c, y = *(const i32x2 *)s;
                        code[i][0] = x[0], code[i][1] = x[1], scale[i][0] = y[0], scale[i][1] = y[1];
                    }
                }
            }
        }
        find(a, kr, step + 1);
    }
    __device__ __forceinline__ void store(TileBuffers<D, PLAID_SOURCE_PAGED> &b, int buf)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, key = unit_key(u);
            if (u < KU) {
                const float power = scale_power(scale[i][0], 0);
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    *(i32x4 *)(b.k[buf] + lds_chunk<D>(key, (u % G) * 4 + w)) =
                        i32x4{codes2<DT, 0>(code[i][w], power), codes2<DT, 1>(code[i][w], power), codes2<DT, 2>(code[i][w], power),
                              codes2<DT, 3>(code[i][w], power)};
            } else if (u < KU + VU) {
                const int m = (u - KU) & 15;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    // scale bytes [token][group]; a token past the end gets the smallest power: finite, and its weight is 0
                    float power[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int byte = t * G + g;
                        power[t] = t < last[i] ? scale_power(scale[i][byte >> 2], byte & 3) : 0.0f;
                    }
                    const int w = code[i][g];
                    const int t0 = codes2<DT, 0>(w, power[0]), t1 = codes2<DT, 1>(w, power[1]), t2 = codes2<DT, 2>(w, power[2]),
                              t3 = codes2<DT, 3>(w, power[3]);
                    const i32x2 low{(int)__builtin_amdgcn_perm(t1, t0, 0x05040100), (int)__builtin_amdgcn_perm(t3, t2, 0x05040100)};
                    const i32x2 high{(int)__builtin_amdgcn_perm(t1, t0, 0x07060302), (int)__builtin_amdgcn_perm(t3, t2, 0x07060302)};
                    *(i32x2 *)(b.v[buf] + (32 * g + m) * ((MANY_KEYS + 4) * 2) + key * 2) = low;
                    *(i32x2 *)(b.v[buf] + (32 * g + 16 + m) * ((MANY_KEYS + 4) * 2) + key * 2) = high;
                }
                if (((u - KU) & 63) == 0) b.cell[buf][(u - KU) >> 6] = ok[i];
            }
        }
    }
};

template <int D, int SRC>
__device__ __forceinline__ i32x4 value_operand(const TileBuffers<D, SRC> &b, int buf, int base, int dt)
{
    if constexpr (SRC == PLAID_SOURCE_PAGED) {
        const int lane = threadIdx.x & 63;
        const char *p = b.v[buf] + (32 * dt + (lane & 31)) * ((MANY_KEYS + 4) * 2) + (base + 4 * (lane >> 5)) * 2;
        const i32x2 x = *(const i32x2 *)p, y = *(const i32x2 *)(p + 16);
        return i32x4{x[0], x[1], y[0], y[1]};
    } else {
        return lds_columns<D>(b.v[buf], base, dt);
    }
}

template <int DT, int D, int NW, int SRC>
__global__ __launch_bounds__(NW * 64, 2) void attend_many_kernel(AttendArgs a, int64_t tiles)
{
    constexpr int ROWS = NW * 32, SHIFT = NW == 8 ? 8 : 7, DT_TILES = D / 32;
    __shared__ __align__(16) TileBuffers<D, SRC> lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int64_t place = id % tiles;
    id /= tiles;
    KeyRange kr;
    kr.head = (int)(id % a.kv_heads);
    const int split = (int)(id / a.kv_heads);
    const TilePlace tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, place);
    if (tp.r < 0) return;
    kr.r = tp.r;

    const int tokens = (int)(tp.end - tp.begin), rows = tokens * a.group;
    const int row = tp.tile * ROWS + wave * 32 + (lane & 31);
    const bool there = row < rows;
    const int token = row_token(a, there ? row : 0), head = kr.head * a.group + (there ? row : 0) - token * a.group;

    // keys that the row sees, and that any row of the tile sees
    int limit, reach;
    if constexpr (SRC == PLAID_SOURCE_PAGED) {
        const int64_t held = (int64_t)a.max_blocks << a.block_shift;
        const int64_t all = a.lengths[tp.r];
        kr.base = 0;
        kr.len = (int)clamp64(all, 0, held);
        const int last = tp.tile * ROWS + ROWS - 1;
        const int last_token = row_token(a, last < rows ? last : rows - 1);
        limit = a.causal && there ? (int)clamp64(all - tokens + token + 1, 0, kr.len) : kr.len;
        reach = a.causal ? (int)clamp64(all - tokens + last_token + 1, 0, kr.len) : kr.len;
        kr.len = reach;
    } else {
        kr.base = clamp64(a.k_offsets[tp.r], 0, a.num_keys);
        kr.len = (int)(clamp64(a.k_offsets[tp.r + 1], kr.base, a.num_keys) - kr.base);
        limit = reach = kr.len;
    }
    int least = limit;  // over the wave's rows
    if constexpr (SRC == PLAID_SOURCE_PAGED) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) least = min(least, __shfl_xor(least, o));
    }

    const int steps = (reach + MANY_KEYS - 1) / MANY_KEYS, share = (steps + a.splits - 1) / a.splits;
    const int begin = split * share, end = min(steps, begin + share);

    i32x4 q[D / 16];
    {
        const char *p = a.q + (tp.begin + token) * a.q_token + head * a.q_head + h * 16;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            q[s] = i32x4{0, 0, 0, 0};
            if (there) q[s] = *(const i32x4 *)(p + s * 32);
#pragma unroll
            for (int e = 0; e < 4; ++e) q[s][e] ^= (int)a.negate_q;
        }
    }
    f32x16 o[DT_TILES];
#pragma unroll
    for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = zero16();
    // with a bias the scores are kept as they are, else as q . k: one multiply-add then makes the exponent
    const float cs = SRC == PLAID_SOURCE_BIAS ? LOG2E : a.scale * LOG2E;
    float m = -INFINITY, l = 0.0f;

    Stage<DT, D, NW, SRC> stage;
    if (begin < end) {
        stage.start(a, kr, begin);
        stage.load(a, kr, begin);
        stage.store(lds, 0);
    }
    __syncthreads();
    for (int step = begin; step < end; ++step) {
        const int buf = (step - begin) & 1;
        if (step + 1 < end) stage.load(a, kr, step + 1);

        f32x16 s[2];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            s[mt] = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) s[mt] = mfma32<DT>(lds_rows<D>(lds.k[buf], 32 * mt, d), q[d], s[mt]);
        }
        if constexpr (SRC == PLAID_SOURCE_BIAS) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 b = *(const f32x4 *)&lds.bias[buf][32 * mt + 8 * i + 4 * h];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[mt][4 * i + e] = b[e] == -INFINITY ? -INFINITY : fmaf(s[mt][4 * i + e], a.scale, b[e]);
                }
        } else {
            bool whole = (step + 1) * MANY_KEYS <= least;
            if constexpr (SRC == PLAID_SOURCE_PAGED) whole = whole && (lds.cell[buf][0] & lds.cell[buf][1] & lds.cell[buf][2] & lds.cell[buf][3]);
            if (!whole) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = 32 * mt + 8 * (i >> 2) + 4 * h + (i & 3);
                        bool seen = step * MANY_KEYS + key < limit;
                        if constexpr (SRC == PLAID_SOURCE_PAGED) seen = seen && lds.cell[buf][2 * mt + (i >> 3)];
                        s[mt][i] = seen ? s[mt][i] : -INFINITY;
                    }
            }
        }
        float top = larger(s[0][0], s[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) top = larger(larger(top, s[0][i]), s[1][i]);
        top = max_halves(top);
        if (__any((top - m) * cs > 8.0f)) {
            const float next = fmaxf(m, top);
            const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - next) * cs);
            m = next;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
        }
        const float ref = m == -INFINITY ? 0.0f : m, ref_cs = ref * cs;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                // a bias may be the type's lowest value: the difference is taken before it is scaled
                const float e = SRC == PLAID_SOURCE_BIAS ? (s[mt][i] - ref) * cs : fmaf(s[mt][i], cs, -ref_cs);
                const float p = __builtin_amdgcn_exp2f(e);
                s[mt][i] = p;
                l += p;
            }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const i32x4 p = round8<DT>(s[mt], i);
#pragma unroll
                for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = mfma32<DT>(value_operand<D, SRC>(lds, buf, 32 * mt + 16 * i, dt), p, o[dt]);
            }
        if (step + 1 < end) stage.store(lds, buf ^ 1);
        __syncthreads();
    }

    l = sum_halves(l);
    if (!there) return;
    const int64_t out_row = (tp.begin + token) * a.heads + head;
    const float natural = SRC == PLAID_SOURCE_BIAS ? m : (m == -INFINITY ? m : m * a.scale);
    if (a.splits > 1) {
        const int64_t at = (int64_t)split * a.num_queries * a.heads + out_row;
#pragma unroll
        for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f32x4 *)(a.part_o + at * D + 32 * dt + 8 * i + 4 * h) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        if (h == 0) a.part_ml[2 * at] = natural, a.part_ml[2 * at + 1] = l;
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(i32x2 *)(a.out + (out_row * D + 32 * dt + 8 * i + 4 * h) * 2) =
                i32x2{pack2<DT>(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv), pack2<DT>(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
    if (a.lse && h == 0) a.lse[2 * out_row] = l == 0.0f ? -INFINITY : natural, a.lse[2 * out_row + 1] = l == 0.0f ? 0.0f : logf(l);
}

// The splits of a row joined, in their order: a thread takes 4 dimensions.
template <int DT, int D>
__global__ __launch_bounds__(256) void join_splits_kernel(AttendArgs a)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / (D / 4), rows = a.num_queries * a.heads;
    const int d = threadIdx.x % (D / 4) * 4;
    if (at >= rows) return;
    // a row outside every request has no sums
    const int64_t token = at / a.heads;
    if (token < a.q_offsets[0] || token >= a.q_offsets[a.n]) return;
    float m = -INFINITY;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[2 * (s * rows + at)]);
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    f32x4 o{0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s) {
        const float w = __builtin_amdgcn_exp2f((a.part_ml[2 * (s * rows + at)] - ref) * LOG2E);
        const f32x4 x = *(const f32x4 *)(a.part_o + (s * rows + at) * D + d);
        l += w * a.part_ml[2 * (s * rows + at) + 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += w * x[e];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *(i32x2 *)(a.out + (at * D + d) * 2) = i32x2{pack2<DT>(o[0] * inv, o[1] * inv), pack2<DT>(o[2] * inv, o[3] * inv)};
    if (a.lse && d == 0) a.lse[2 * at] = l == 0.0f ? -INFINITY : m, a.lse[2 * at + 1] = l == 0.0f ? 0.0f : logf(l);
}

template <int DT, int D, int NW>
static void launch_source(hipStream_t st, const AttendArgs &a, int source, int64_t tiles)
{
    const dim3 grid((unsigned)(tiles * a.kv_heads * a.splits)), block(NW * 64);
    if (source == PLAID_SOURCE_DENSE) attend_many_kernel<DT, D, NW, PLAID_SOURCE_DENSE><<<grid, block, 0, st>>>(a, tiles);
    else if (source == PLAID_SOURCE_BIAS) attend_many_kernel<DT, D, NW, PLAID_SOURCE_BIAS><<<grid, block, 0, st>>>(a, tiles);
    else attend_many_kernel<DT, D, NW, PLAID_SOURCE_PAGED><<<grid, block, 0, st>>>(a, tiles);
}

template <int DT, int D>
static void launch_type(hipStream_t st, const AttendArgs &a, int source, int waves, int64_t tiles)
{
    if (waves == 8) launch_source<DT, D, 8>(st, a, source, tiles);
    else launch_source<DT, D, 4>(st, a, source, tiles);
    if (a.splits > 1) {
        const int64_t threads = a.num_queries * a.heads * (D / 4);
        join_splits_kernel<DT, D><<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st>>>(a);
    }
}

void plaid_launch_attend_many(hipStream_t st, const AttendArgs &a, int dtype, int head_dim, int source, int waves, int64_t tiles)
{
    if (dtype == PLAID_BF16) head_dim == 64 ? launch_type<PLAID_BF16, 64>(st, a, source, waves, tiles) : launch_type<PLAID_BF16, 128>(st, a, source, waves, tiles);
    else head_dim == 64 ? launch_type<PLAID_FP16, 64>(st, a, source, waves, tiles) : launch_type<PLAID_FP16, 128>(st, a, source, waves, tiles);
}
