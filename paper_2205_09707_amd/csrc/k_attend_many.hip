// Attention where a request has many rows (tokens x heads that share keys): tiles of rows x 64 keys on the matrix units.
#include <type_traits>

#include "reader.h"

// out = softmax(scale q k^T + b) v in one pass over the keys, with the running maximum m and sum l of each row:
//   p = exp(s - m),  l <- l exp(m_old - m) + sum p,  o <- o exp(m_old - m) + p v,  and out = o / l at the end.
// A wave owns 32 rows.  It computes s^T = k q^T, so that a lane holds one row (column l % 32 of the result) and the two halves
// of the wave half of its keys each: the maximum and the sum need one exchange, and the result's registers, rounded, are
// already the operand of o^T = v^T p^T (rows of v^T come from LDS by the transposing read, or lie transposed there).  q stays
// in registers; keys and values of 64 keys at a time go through LDS, dense ones straight from memory up to three tiles ahead, those of
// the cache as codes in registers that are turned into values on the way.  m lags behind the maximum by up to 2^8: o is rescaled
// only where it would fall further back.  Biases, divided by the scale, are what the matrix instruction adds the products to, so
// that a biased score costs no instruction of its own (565 us in place of 614, below).
// The weights round to the type before they multiply the values (half of the matrix rate is lost with more bits); their sum does not.
//
// What bounds it: one group's vector instructions (exponential 16 cycles, multiply-add, half a maximum, half a rounding and one addition a
// score) against the other's products.  Measured: 16 requests of 456 tokens x 16 heads on 6250 keys of 4 heads, D = 128 (373 GFLOP):
// 378 us without biases, 462 with = 0.99 and 0.81 PFLOP/s, many calls in a row; products first and addresses of loads kept in registers took
// 2 % each off.  6 prompts of 850 tokens x 32 heads behind 4750 in the cache (419 GFLOP): 482 us = 0.87 PFLOP/s; what is left there is the
// codes' way into values, which every 256 rows pay.
//
// Tiles that lie in LDS at a time, and how many tiles ahead of the weights' one keys and values are asked for.  With two groups of
// waves (see below) a tile of keys is read in two phases and one of values in the two after those; a buffer is filled anew from
// the second phase of a step on.
template <int NW, int SRC>
struct Ahead {
    static constexpr bool PAGED = SRC == PLAID_SOURCE_PAGED;
    static constexpr int GROUPS = NW == 8 ? 2 : 1, TILES = PAGED || NW == 4 ? 2 : 4;
    static constexpr int K = PAGED ? 1 : TILES - GROUPS + 1, V = PAGED ? 0 : TILES - GROUPS;
};

template <int D, int NW, int SRC>
struct TileBuffers {
    static constexpr int TILES = Ahead<NW, SRC>::TILES;
    char k[TILES][MANY_KEYS * D * 2];
    char v[TILES][SRC == PLAID_SOURCE_PAGED ? D * (MANY_KEYS + 4) * 2 : MANY_KEYS * D * 2];
    float bias[SRC == PLAID_SOURCE_BIAS ? NW : 1][4][SRC == PLAID_SOURCE_BIAS ? MANY_KEYS : 4];  // each wave's own
    uint32_t raw[SRC == PLAID_SOURCE_BIAS ? NW : 1][4][64];  // biases as they are loaded
    int cell[4][4];  // paged: whether the cells of 16 keys have a block
    int bad[D / 32]; // paged: the first key of those that are hidden from some row whose values of 32 dimensions are not finite
};

struct KeyRange {
    int64_t base;  // dense: the request's first key
    int len;       // keys of the request that there are
    int r, head;   // request, key head
    int least;     // keys that every row of the tile sees
};

// How a workgroup's waves bring tiles into LDS: dense keys and values go there straight from memory, each wave its share.
template <int DT, int D, int NW, int SRC>
struct Stage {
    static constexpr int TILES = Ahead<NW, SRC>::TILES, CHUNKS = D / 8, AT_ONCE = 512 / D, N = MANY_KEYS / AT_ONCE / NW;  // loads of a wave a tile
    static constexpr bool BIAS = SRC == PLAID_SOURCE_BIAS;
    static constexpr uint16_t NONE = DT == PLAID_BF16 ? 0xff80 : 0xfc00;  // -infinity
    uint64_t k_masked, v_masked;  // keys of bias -infinity, and places past the end, in the tiles that are asked for next
    // What a load's address is made of is formed once: a tile's place is a product of 32 bits, a lane's place in a tile is kept.
    const char *keys, *values, *biases;            // the request's first
    uint32_t key_row[N], value_row[N], chunk[N];  // bytes of a lane's row in a tile, and within the row
    uint32_t to_k, to_v, to_raw;                  // in LDS, of the wave

    __device__ __forceinline__ void init(const AttendArgs &a, const KeyRange &kr, const TileBuffers<D, NW, SRC> &b)
    {
        const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
        keys = a.k + kr.base * a.k_token + kr.head * a.k_head, values = a.v + kr.base * a.v_token + kr.head * a.v_head;
        biases = a.bias + 2 * kr.base;
        to_k = lds_address(b.k[0]) + wave * N * 1024, to_v = lds_address(b.v[0]) + wave * N * 1024, to_raw = lds_address(b.raw[BIAS ? wave : 0]);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = (wave * N + i) * AT_ONCE + lane / CHUNKS;
            key_row[i] = (uint32_t)row * (uint32_t)a.k_token, value_row[i] = (uint32_t)row * (uint32_t)a.v_token;
            chunk[i] = ((lane % CHUNKS) ^ swizzle<D>(row)) * 16;
        }
    }
    // Keys past the end repeat the last one (with biases they are zeros, else the last step leaves them out).  The tiles after the last repeat that one, so that a phase's number of loads is fixed.
    __device__ __forceinline__ void load(const KeyRange &kr, const char *first, uint32_t token, const uint32_t (&rows)[N], int tile, uint32_t to,
                                         uint64_t masked)
    {
        const char *base = first + (uint64_t)(uint32_t)(tile * MANY_KEYS) * token;
        const uint32_t last = (uint32_t)min(kr.len - 1 - tile * MANY_KEYS, MANY_KEYS - 1) * token;
        const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
        const uint32_t none = (uint32_t)(masked >> (wave * N * AT_ONCE)) >> (lane / CHUNKS);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t off = min(rows[i], last) + chunk[i];
            if constexpr (BIAS) load_to_lds(none >> (i * AT_ONCE) & 1 ? (const char *)zero_row : base + off, to + i * 1024);
            else load_to_lds(base, off, to + i * 1024);
        }
    }
    __device__ __forceinline__ void load_k(const AttendArgs &a, const KeyRange &kr, int tile, int end)
    {
        load(kr, keys, (uint32_t)a.k_token, key_row, min(tile, end - 1), to_k + (uint32_t)tile % TILES * (MANY_KEYS * D * 2), k_masked);
    }
    __device__ __forceinline__ void load_v(const AttendArgs &a, const KeyRange &kr, int tile, int end)
    {
        load(kr, values, (uint32_t)a.v_token, value_row, min(tile, end - 1), to_v + (uint32_t)tile % TILES * (MANY_KEYS * D * 2), v_masked);
    }
    __device__ __forceinline__ void load_bias(const KeyRange &kr, int tile, int end)
    {
        const int lane = threadIdx.x & 63, t = min(tile, end - 1), last = kr.len - 1 - t * MANY_KEYS;
        load2_to_lds(biases + (uint64_t)(uint32_t)t * (2 * MANY_KEYS), 2 * min(lane, last), to_raw + (tile & 3) * 256);
    }
    // The biases of the tile whose keys are asked for next, in 32 bits, and which of its keys are masked.  They are read some time
    // before they are used.
    uint32_t raw;
    Shift shift;
    int shifts[Ahead<NW, SRC>::K];  // bits of what was subtracted in the tile whose weights are next, and those after it
    __device__ __forceinline__ void read_bias(const TileBuffers<D, NW, SRC> &b, int tile) { raw = b.raw[threadIdx.x >> 6][tile & 3][threadIdx.x & 63]; }
    __device__ __forceinline__ void store_bias(const AttendArgs &a, const KeyRange &kr, int end, TileBuffers<D, NW, SRC> &b, int tile)
    {
        const int lane = threadIdx.x & 63;
        const uint16_t x = min(tile, end - 1) * MANY_KEYS + lane < kr.len ? (uint16_t)raw : NONE;
        const float f = unpack<DT>(x, 0);
        v_masked = k_masked;
        k_masked = __ballot(x == NONE);
        const uint64_t large = __ballot(fabsf(f) > BIAS_USUAL), unusual = large & ~k_masked;
        shift.add(unusual, unusual_bias(f) ? f : -INFINITY, ~(k_masked | large) != 0);
        b.bias[threadIdx.x >> 6][tile & 3][lane] = (f - shift.c) * a.inv_scale;
#pragma unroll
        for (int i = 0; i + 1 < Ahead<NW, SRC>::K; ++i) shifts[i] = shifts[i + 1];
        shifts[Ahead<NW, SRC>::K - 1] = __float_as_int(shift.c);
    }
    // Before the first phase: asks for the first tiles and waits for the first one's keys.
    __device__ __forceinline__ void start(const AttendArgs &a, const KeyRange &kr, int begin, int end, TileBuffers<D, NW, SRC> &b)
    {
        using A = Ahead<NW, SRC>;
        static_assert(A::V == A::K - 1, "values are asked for one tile behind the keys");
        init(a, kr, b);
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i <= A::K; ++i) load_bias(kr, begin + i, end);
            wait_loads<0>();
        }
#pragma unroll
        for (int i = 0; i < A::K; ++i) {
            if constexpr (BIAS) {
                read_bias(b, begin + i);
                store_bias(a, kr, end, b, begin + i);
            }
            load_k(a, kr, begin + i, end);
            if (i > 0) load_v(a, kr, begin + i - 1, end);
        }
        wait_all_loads();  // the queries too
        lds_barrier();
    }
    // In the second phase of a step, before and after its weights.
    __device__ __forceinline__ void before(int step, const TileBuffers<D, NW, SRC> &b)
    {
        if constexpr (BIAS) {
            wait_loads<2 * N>();  // the biases that the step before asked for first
            read_bias(b, step + Ahead<NW, SRC>::K);
        }
    }
    template <bool>
    __device__ __forceinline__ void bring(const AttendArgs &a, const KeyRange &kr, int step, int end, int, TileBuffers<D, NW, SRC> &b)
    {
        using A = Ahead<NW, SRC>;
        if constexpr (BIAS) {
            store_bias(a, kr, end, b, step + A::K);
            load_bias(kr, step + A::K + 1, end);
        }
        load_k(a, kr, step + A::K, end);
        load_v(a, kr, step + A::V, end);
    }
    // At the end of a phase: what the phases after the next barrier need has arrived.  A step asks for 2 N pieces (and its bias);
    // the next step's keys and this one's values must be there after its second phase.
    __device__ __forceinline__ void arrive(bool second, int late)
    {
        constexpr int STEP = 2 * N + BIAS;
        if constexpr (Ahead<NW, SRC>::GROUPS == 2) {
            if (second && !late) wait_loads<STEP *(TILES - 2)>();
            if (!second && late) wait_loads<STEP *(TILES - 3)>();
        } else {
            if (second) wait_loads<STEP *(TILES - 1)>();
        }
    }
};

// Paged: a unit is 32 dimensions of a key (one scale), or a lane's part of a cell of value codes (4 tokens, D / 16 dimensions),
// turned into 16-bit values on the way into LDS.  The units of keys come first, so that a wave has one kind.  Block ids are read
// one tile ahead of the codes.
template <int DT, int D, int NW>
struct Stage<DT, D, NW, PLAID_SOURCE_PAGED> {
    static constexpr int THREADS = NW * 64, G = D / 32, KU = MANY_KEYS * G, VU = MANY_KEYS / 16 * 64, N = (KU + VU + THREADS - 1) / THREADS;
    int id_next[N], ok[N], last[N];
    i32x4 code[N], scale[N];

    // first key of a unit in its tile
    static __device__ __forceinline__ int unit_key(int u) { return u < KU ? u / G : ((u - KU) >> 6) * 16 + (((u - KU) >> 4) & 3) * 4; }

    // As above nothing is loaded under a condition: the last key's block stands for what is past the end, the first block for an id
    // outside the cache (a request of a cache without blocks has no keys).
    template <bool KEYS>
    __device__ __forceinline__ void find(const AttendArgs &a, const KeyRange &kr, int tile)
    {
        const int32_t *row = a.table + kr.r * a.table_stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS;
            if ((u < KU) != KEYS) continue;
            id_next[i] = row[(uint32_t)(min(tile * MANY_KEYS + unit_key(u), kr.len - 1) >> a.block_shift)];
        }
    }
    template <bool KEYS>
    __device__ __forceinline__ void load(const AttendArgs &a, const KeyRange &kr, int tile)
    {
        const uint32_t bs = 1u << a.block_shift, region = bs * (D * 17 / 16);
        const uint8_t *heads = a.cache + (int64_t)kr.head * region;
        const int64_t block = (int64_t)a.kv_heads * region;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, at = tile * MANY_KEYS + unit_key(u);
            if ((u < KU) != KEYS) continue;
            const uint32_t in = at & (bs - 1);
            ok[i] = (uint32_t)id_next[i] < (uint64_t)a.num_blocks;
            last[i] = ok[i] ? kr.len - at : 0;  // tokens of the unit that there are
            const uint8_t *p = heads + (ok[i] ? id_next[i] : 0) * block;
            if constexpr (KEYS) {
                code[i] = *(const i32x4 *)(p + (in * (D / 2) + (u % G) * 16));
                scale[i][0] = p[bs * D + in * G + u % G];
            } else {
                const uint32_t l = (u - KU) & 63;
                const uint8_t *c = p + (bs * (D / 2) + (in >> 4) * (8 * D) + l * (D / 8)), *s = p + (bs * (D + G) + in * G);
                if constexpr (D == 128) {
                    code[i] = *(const i32x4 *)c;
                    scale[i] = *(const i32x4 *)s;
                } else {
                    const i32x2 x = *(const i32x2 *)c, y = *(const i32x2 *)s;
                    code[i][0] = x[0], code[i][1] = x[1], scale[i][0] = y[0], scale[i][1] = y[1];
                }
            }
        }
        find<KEYS>(a, kr, tile + 1);
    }
    __device__ __forceinline__ void load_k(const AttendArgs &a, const KeyRange &kr, int tile) { load<true>(a, kr, tile); }
    __device__ __forceinline__ void load_v(const AttendArgs &a, const KeyRange &kr, int tile) { load<false>(a, kr, tile); }
    __device__ __forceinline__ void store_k(TileBuffers<D, NW, PLAID_SOURCE_PAGED> &b, int tile)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, key = unit_key(u);
            if (u >= KU) continue;
            const float power = scale_power(scale[i][0], 0);
#pragma unroll
            for (int w = 0; w < 4; ++w)
                *(i32x4 *)(b.k[tile & 1] + lds_chunk<D>(key, (u % G) * 4 + w)) =
                    i32x4{codes2<DT, 0>(code[i][w], power), codes2<DT, 1>(code[i][w], power), codes2<DT, 2>(code[i][w], power),
                          codes2<DT, 3>(code[i][w], power)};
            if (u % (16 * G) == 0) b.cell[tile & 3][key >> 4] = ok[i];
        }
    }
    template <bool CAREFUL>
    __device__ __forceinline__ void store_v(const KeyRange &kr, TileBuffers<D, NW, PLAID_SOURCE_PAGED> &b, int tile)
    {
        // A key that only some of the rows see may hold what is not finite, which would meet the zero weights of the others: it goes in
        // as zero, and those that see it get it at the end.
        if (CAREFUL && (tile + 1) * MANY_KEYS > kr.least) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int u = threadIdx.x + i * THREADS, at = tile * MANY_KEYS + unit_key(u);
                if (u < KU || u >= KU + VU) continue;
#pragma unroll
                for (int byte = 0; byte < 4 * G; ++byte) {
                    const int mask = 255 << 8 * (byte & 3), t = byte / G;
                    if (at + t < kr.least || t >= last[i] || (scale[i][byte >> 2] & mask) != mask) continue;
                    atomicMin(&b.bad[byte % G], at + t);
                    scale[i][byte >> 2] &= ~mask;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = threadIdx.x + i * THREADS, key = unit_key(u);
            if (u < KU || u >= KU + VU) continue;
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
                *(i32x2 *)(b.v[tile & 1] + (32 * g + m) * ((MANY_KEYS + 4) * 2) + key * 2) = low;
                *(i32x2 *)(b.v[tile & 1] + (32 * g + 16 + m) * ((MANY_KEYS + 4) * 2) + key * 2) = high;
            }
        }
    }
    __device__ __forceinline__ void start(const AttendArgs &a, const KeyRange &kr, int begin, int end, TileBuffers<D, NW, PLAID_SOURCE_PAGED> &b)
    {
        find<true>(a, kr, begin);
        find<false>(a, kr, begin);
        load_k(a, kr, begin);
        store_k(b, begin);
        if (threadIdx.x < G) b.bad[threadIdx.x] = INT32_MAX;
        if (begin + 1 < end) load_k(a, kr, begin + 1);
        load_v(a, kr, begin);
        lds_barrier();
        if (NW == 8 && threadIdx.x >= 256) bring<true>(a, kr, begin - 1, end, 1, b);
    }
    // In its second phase of step t group g brings keys t + 1 + g and values t + g: nobody reads their buffers in that phase or the
    // one beside it.  Then it asks for the next ones.
    template <bool CAREFUL>
    __device__ __forceinline__ void bring(const AttendArgs &a, const KeyRange &kr, int step, int end, int late, TileBuffers<D, NW, PLAID_SOURCE_PAGED> &b)
    {
        const int tile = step + late;
        if (tile + 1 < end) store_k(b, tile + 1);
        if (tile < end) store_v<CAREFUL>(kr, b, tile);
        if (tile + 2 < end) load_k(a, kr, tile + 2);
        if (tile + 1 < end) load_v(a, kr, tile + 1);
    }
    __device__ __forceinline__ void before(int, const TileBuffers<D, NW, PLAID_SOURCE_PAGED> &) {}
    __device__ __forceinline__ void arrive(bool, int) {}
};

template <int D, int NW, int SRC>
__device__ __forceinline__ i32x4 value_operand(const TileBuffers<D, NW, SRC> &b, int buf, int base, int dt)
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
    __shared__ __align__(16) TileBuffers<D, NW, SRC> lds;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    const WorkPlace w = work_place(a, tiles, a.splits, blockIdx.x);
    KeyRange kr;
    kr.head = w.head;
    const int split = w.split;
    TilePlace tp;
    if (a.n <= SORTED_REQUESTS) {
        const int of = min(lane, a.n - 1);
        const int keys = SRC == PLAID_SOURCE_PAGED ? a.lengths[of] : (int)(a.k_offsets[of + 1] - a.k_offsets[of]);
        tp = find_sorted_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, w.place, keys);
    } else {
        tp = find_tile(a.q_offsets, a.n, a.num_queries, a.group, SHIFT, w.place);
    }
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
        const int64_t all = uniform_load(a.lengths + tp.r);
        kr.base = 0;
        kr.len = a.num_blocks > 0 ? (int)clamp64(all, 0, held) : 0;
        const int last = tp.tile * ROWS + ROWS - 1;
        const int last_token = row_token(a, last < rows ? last : rows - 1);
        limit = a.causal && there ? (int)clamp64(all - tokens + token + 1, 0, kr.len) : kr.len;
        reach = a.causal ? (int)clamp64(all - tokens + last_token + 1, 0, kr.len) : kr.len;
        kr.len = reach;
        kr.least = a.causal ? (int)clamp64(all - tokens + row_token(a, tp.tile * ROWS) + 1, 0, reach) : reach;
    } else {
        kr.base = clamp64(uniform_load(a.k_offsets + tp.r), 0, a.num_keys);
        kr.len = (int)(clamp64(uniform_load(a.k_offsets + tp.r + 1), kr.base, a.num_keys) - kr.base);
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
    // with values that are not finite in q even the zeros that stand for masked keys give scores that are not numbers
    int odd = 0;
    if constexpr (SRC == PLAID_SOURCE_BIAS) {
        constexpr int INF = DT == PLAID_BF16 ? 0x7f80 : 0x7c00;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= (q[s][e] & INF) == INF || ((q[s][e] >> 16) & INF) == INF;
        odd = uniform(__any(odd) ? 1 : 0);
    }
    f32x16 o[DT_TILES];
#pragma unroll
    for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = zero16();
    // scores are kept as q . k + b / scale: one multiply-add then makes the exponent
    const float cs = a.scale * LOG2E;
    float m = -INFINITY, l = 0.0f;
    int shift = 0, alone = 0;  // the shift's bits, and whether it leaves the scores nothing: the same for all lanes

    // Two groups of waves, one of each on every SIMD, half a step apart: while one multiplies, the other forms exponentials.
    // A step of a group is a phase of products (o += v^T p^T of the former tile, s of this one) and one of everything else, with
    // barriers between them.
    using A = Ahead<NW, SRC>;
    const int late = A::GROUPS == 2 ? uniform((int)(threadIdx.x >> 8)) : 0;
    Stage<DT, D, NW, SRC> stage;
    auto phase_end = [&](bool second) {
        __builtin_amdgcn_sched_barrier(0);
        stage.arrive(second, late);
        lds_barrier();
    };
    if (begin < end) {
        stage.start(a, kr, begin, end, lds);
        if (late) lds_barrier();
    }
    f32x16 s[2];
    i32x4 p[4];
    auto before_scores = [&](int step) {
        if constexpr (SRC == PLAID_SOURCE_BIAS) {  // what the products are added to
            typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
            const lds_f32x4 *b = (const lds_f32x4 *)&lds.bias[wave][step & 3][4 * h];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) s[mt] = join16(b[8 * mt], b[8 * mt + 2], b[8 * mt + 4], b[8 * mt + 6]);
        } else {
            s[0] = zero16(), s[1] = zero16();
        }
    };
    constexpr int EARLY = 4, KEY_READS = D / 16 * 2;  // operands of keys that are read before the products with values end
    i32x4 early[EARLY];
    auto key_operand = [&](int step, int i) { return lds_rows<D>(lds.k[step % A::TILES], 32 * (i & 1), i >> 1); };
    auto scores = [&](int step) {
#pragma unroll
        for (int i = 0; i < KEY_READS; ++i) s[i & 1] = mfma32<DT>(i < EARLY ? early[i] : key_operand(step, i), q[i >> 1], s[i & 1]);
    };
    auto add_values = [&](int step, int from, int to) {
#pragma unroll
        for (int i = from; i < to; ++i)
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = mfma32<DT>(value_operand<D, NW, SRC>(lds, step % A::TILES, 16 * i, dt), p[i], o[dt]);
    };
    auto add_weights = [&]() {
        float sums[4] = {l, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[i & 3] += s[0][i] + s[1][i];
        l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    };
    auto weights = [&](int step, auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        if constexpr (SRC == PLAID_SOURCE_DENSE) stage.template bring<CAREFUL>(a, kr, step, end, late, lds);
        else stage.before(step, lds);
        float top;
        if constexpr (SRC == PLAID_SOURCE_BIAS) {
            if (stage.shifts[0] != shift) {  // m is relative to the shift
                // in one operation: the product alone may overflow, and m may be -infinity
                m = fmaf(__int_as_float(shift) - __int_as_float(stage.shifts[0]), a.inv_scale, m);
                shift = stage.shifts[0];
                alone = uniform((int)beside(__int_as_float(shift)));
            }
            if (odd | alone) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 b = *(const f32x4 *)&lds.bias[wave][step & 3][32 * mt + 8 * i + 4 * h];
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[mt][4 * i + e] = b[e] == -INFINITY ? b[e] : alone ? vanish(s[mt][4 * i + e], b[e]) : s[mt][4 * i + e];
                    }
            }
        } else {
            bool whole = (step + 1) * MANY_KEYS <= least;
            if constexpr (SRC == PLAID_SOURCE_PAGED) {
                const int *held = lds.cell[step & 3];
                whole = whole && (held[0] & held[1] & held[2] & held[3]);
            }
            if (!whole) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = 32 * mt + 8 * (i >> 2) + 4 * h + (i & 3);
                        bool seen = step * MANY_KEYS + key < limit;
                        if constexpr (SRC == PLAID_SOURCE_PAGED) seen = seen && lds.cell[step & 3][2 * mt + (i >> 3)];
                        s[mt][i] = seen ? s[mt][i] : -INFINITY;
                    }
            }
        }
        top = larger(s[0][0], s[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) top = larger(larger(top, s[0][i]), s[1][i]);
        top = max_halves(top);
        if (__any(!((top - m) * cs <= 8.0f))) {  // also where there was no key so far
            const float next = fmaxf(m, top);
            const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - next) * cs);
            m = next;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
        }
        const float ref_cs = m == -INFINITY ? 0.0f : m * cs;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[mt][i] = __builtin_amdgcn_exp2f(fmaf(s[mt][i], cs, -ref_cs));
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = round8<DT>(s[i >> 1], i & 1);
        if constexpr (SRC != PLAID_SOURCE_DENSE) stage.template bring<CAREFUL>(a, kr, step, end, late, lds);
    };
    if (begin < end) {
        before_scores(begin);
#pragma unroll
        for (int i = 0; i < EARLY; ++i) early[i] = key_operand(begin, i);
        scores(begin);
        phase_end(false);
        auto both_phases = [&](int step, auto careful) {
            weights(step, careful);
            phase_end(true);
            // products go before the other group's instructions (382 us in place of 391; paged 536 in place of 564)
            __builtin_amdgcn_s_setprio(1);
            // the weights are added up while the first operands are on their way, and their registers then are free
            i32x4 first[DT_TILES];
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt) first[dt] = value_operand<D, NW, SRC>(lds, step % A::TILES, 0, dt);
            __builtin_amdgcn_sched_barrier(0);
            add_weights();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = mfma32<DT>(first[dt], p[0], o[dt]);
            add_values(step, 1, 4);
            before_scores(step + 1);
#pragma unroll
            for (int i = 0; i < EARLY; ++i) early[i] = key_operand(step + 1, i);
            // the order of the phase: operands are asked for some reads ahead of the products that take them
            constexpr int READS = DT_TILES * 6 + (SRC == PLAID_SOURCE_BIAS ? 8 : 0) + EARLY - 6, PAIRS = DT_TILES * 2 - 1;
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (READS + PAIRS - 1) / PAIRS, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            scores(step + 1);
#pragma unroll
            for (int i = 0; i < (KEY_READS - EARLY) / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, EARLY, 0);
            phase_end(false);
            __builtin_amdgcn_s_setprio(0);
        };
        int step = begin;
        if constexpr (SRC == PLAID_SOURCE_PAGED)  // the tiles of values that a step stores: its own and the next one
            for (; step + 1 < end && (step + 2) * MANY_KEYS <= kr.least; ++step) both_phases(step, std::false_type());
        for (; step + 1 < end; ++step) both_phases(step, std::true_type());
        weights(end - 1, std::true_type());
        phase_end(true);
        add_weights();
        if (SRC == PLAID_SOURCE_DENSE && end * MANY_KEYS > kr.len) {
            // what stands in for values past the end may not be finite and must not meet its weights of zero
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                i32x4 keep;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int left = kr.len - ((end - 1) * MANY_KEYS + 16 * i + 8 * (x >> 1) + 4 * h + 2 * (x & 1));
                    keep[x] = left >= 2 ? -1 : left == 1 ? 0xffff : 0;
                }
#pragma unroll
                for (int dt = 0; dt < DT_TILES; ++dt) o[dt] = mfma32<DT>(value_operand<D, NW, SRC>(lds, (end - 1) % A::TILES, 16 * i, dt) & keep, p[i], o[dt]);
            }
        } else {
            add_values(end - 1, 0, 4);
        }
        if (A::GROUPS == 2 && !late) lds_barrier();
        wait_loads<0>();  // nothing may arrive in LDS that is no longer the workgroup's
    }

    if constexpr (SRC == PLAID_SOURCE_PAGED) {
        if (begin < end) {
#pragma unroll
            for (int dt = 0; dt < DT_TILES; ++dt)
                if (lds.bad[dt] < limit) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] = NAN;
                }
        }
    }
    l = sum_halves(l);
    if (!there) return;
    const int64_t out_row = (tp.begin + token) * a.heads + head;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bool any = l != 0.0f;
    if constexpr (SRC == PLAID_SOURCE_BIAS) any = stage.shift.any();
    const float2 lse = any ? float2{__int_as_float(shift), m * a.scale + logf(l)} : float2{-INFINITY, 0.0f};
    if (a.splits > 1) {
        const int64_t at = (int64_t)split * a.num_queries * a.heads + out_row;
#pragma unroll
        for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f32x4 *)(a.part_o + at * D + 32 * dt + 8 * i + 4 * h) =
                    f32x4{o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv, o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv};
        if (h == 0) *(float2 *)(a.part_lse + 2 * at) = lse;
        return;
    }
#pragma unroll
    for (int dt = 0; dt < DT_TILES; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(i32x2 *)(a.out + (out_row * D + 32 * dt + 8 * i + 4 * h) * 2) =
                i32x2{pack2<DT>(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv), pack2<DT>(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
    if (a.lse && h == 0) *(float2 *)(a.lse + 2 * out_row) = lse;
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
    float c = -INFINITY, top = -INFINITY;
    for (int s = 0; s < a.splits; ++s) c = fmaxf(c, a.part_lse[2 * (s * rows + at)]);
    const float base = c == -INFINITY ? 0.0f : c;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_lse[2 * (s * rows + at)] - base + a.part_lse[2 * (s * rows + at) + 1]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    f32x4 o{0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s) {
        const float w = __builtin_amdgcn_exp2f((a.part_lse[2 * (s * rows + at)] - base + a.part_lse[2 * (s * rows + at) + 1] - ref) * LOG2E);
        const f32x4 x = *(const f32x4 *)(a.part_o + (s * rows + at) * D + d);
        l += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += w * x[e];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *(i32x2 *)(a.out + (at * D + d) * 2) = i32x2{pack2<DT>(o[0] * inv, o[1] * inv), pack2<DT>(o[2] * inv, o[3] * inv)};
    if (a.lse && d == 0) *(float2 *)(a.lse + 2 * at) = c == -INFINITY ? float2{-INFINITY, 0.0f} : float2{c, top + logf(l)};
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
    if (dtype == PLAID_BF16)
        head_dim == 64 ? launch_type<PLAID_BF16, 64>(st, a, source, waves, tiles) : launch_type<PLAID_BF16, 128>(st, a, source, waves, tiles);
    else head_dim == 64 ? launch_type<PLAID_FP16, 64>(st, a, source, waves, tiles) : launch_type<PLAID_FP16, 128>(st, a, source, waves, tiles);
}
