// Cross entropy over a vocabulary: the products.
#include <type_traits>

#include "train.h"

// Three products, each of tiles of 256 x 256 over an axis k taken 64 at a time:
//   scores   s[t][v]  = sum over the width of h[t] W[v];      the tile ends as statistics of its rows, or as G, rounded to the type
//   d_hidden dh[t][j] = sum over the vocabulary of G[t][v] W[v][j]
//   d_weight dW[v][j] = sum over rows of G[t][v] h[t][j]
// An operand lies in memory with k along its rows, or across them; the latter goes into LDS as it is and is read transposed.  Eight waves
// have 128 x 64 of a tile each.  The axis that is to lie together in memory is the one of the result's registers (M): four neighbours a lane.
//
// Measured, 7296 rows of 2048, 5107 of them with a target, on 128000 entries in bf16 (2.7 TFLOP a product): statistics of the scores 2160 us = 1.24 PFLOP/s,
// G 2260 = 1.18, both gradients 4370 = 1.23; on other cards 2200 to 2250, 2330 to 2370, 4480; with what G left out 4560.  A step
// of 64 takes 1.6 us (1.34 PFLOP/s), a tile's first loads and its way out 5 (statistics) to 7 (G).
// The matrix units are busy for 63 % of the time at 1.73 GHz, and for 52 % at 1.9 GHz before the reads of operands lay among the products: what is
// left is power and the loads (statistics without loads 1855 in place of 2276, without reads of LDS 2064, without waiting for loads 2243).
// Kept out: lines of later steps touched in advance (2515), a wave's priority raised for its products (no change), four waves with 128 x 128 each, which
// read a third less of LDS (2600), steps that begin at different columns (no change here, but see k_loss.hip).
#define BK LOSS_STEP
#define TILE_BYTES (LOSS_TILE * BK * 2)

// How a wave brings its eighth of an operand's tile into LDS, four loads of 1 KB.  Along: [256 rows][64], a load has 8 rows.  Across: two
// halves [64 k][128], a load has 4 rows of k.  The chunks of 16 bytes of a row change places as lds_chunk says; a load's lanes write
// LDS one after another, so it is the lanes' addresses that do.
template <bool ACROSS>
struct Operand {
    const char *at[4];
    int k[4];  // of the lane's chunk
    // along: rows first .. first + 255 of `rows`, later ones are the last again.  across: columns first .. first + 255 of `columns`; what lies
    // past the end is column 0, and its results are not kept.
    __device__ __forceinline__ void set(const char *base, int64_t stride, int64_t first, int64_t rows, int64_t columns)
    {
        const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int load = wave * 4 + i;
            if constexpr (!ACROSS) {
                const int row = load * 8 + (lane >> 3), chunk = (lane & 7) ^ swizzle<64>(row);
                k[i] = chunk * 8;
                at[i] = base + min(first + row, rows - 1) * stride + chunk * 16;
            } else {
                const int half = load >> 4, row = (load & 15) * 4 + (lane >> 4), chunk = (lane & 15) ^ swizzle<128>(row);
                const int64_t column = first + half * 128 + chunk * 8;
                k[i] = row;
                at[i] = base + row * stride + (column < columns ? column : 0) * 2;
            }
        }
    }
    __device__ __forceinline__ void load(int i, uint32_t tile) const { load_to_lds(at[i], tile + i * 1024); }
    // The last step of an axis that ends inside it: `left` of the 64 are there.  Along: zeros for the others.  Across: the last one again
    // (the other operand has zeros there).
    __device__ __forceinline__ void load_end(int i, uint32_t tile, int left, int64_t stride) const
    {
        const char *p = at[i];
        if constexpr (!ACROSS) p = k[i] < left ? p : (const char *)zero_row;
        else p = k[i] < left ? p : p - (k[i] - (left - 1)) * stride;
        load_to_lds(p, tile + i * 1024);
    }
    __device__ __forceinline__ void step(int64_t bytes)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] += bytes;
    }
};
// Where a lane reads its part of the operand of 32 rows (columns, across) at k = 16 s + 8 (l / 32) .. + 7, for N such blocks.  Along, blocks are
// at a constant distance and s = 0 .. 3 have a place each; across, steps of s are, and blocks have two places each, four rows of k apart.
template <bool ACROSS, int N>
struct Places {
    int at[ACROSS ? 2 * N : 4];
    __device__ __forceinline__ void set(int base)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (!ACROSS) {
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = (base + (lane & 31)) * 128 + (((2 * s + (lane >> 5)) ^ swizzle<64>(lane & 31)) << 4);
        } else {
            const int row = 8 * (lane >> 5) + ((lane >> 2) & 3), x = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                const int r = row + 4 * (i & 1), block = (base >> 5) + i / 2;
                at[i] = (block >> 2) * (TILE_BYTES / 2) + r * 256 + ((((block & 3) * 4 + x) ^ swizzle<128>(r)) << 4) + (lane & 1) * 8;
            }
        }
    }
    __device__ __forceinline__ i32x4 read(const char *tile, int i, int s) const
    {
        if constexpr (!ACROSS) return *(const i32x4 *)(tile + at[s] + i * 4096);
        else {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const i32x2 u = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at[2 * i] + s * 4096)));
            const i32x2 w = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at[2 * i + 1] + s * 4096)));
            return i32x4{u[0], u[1], w[0], w[1]};
        }
    }
};

struct Tile {
    int m, n;
};
// Tile of workgroup `id`: workgroups go to the eight XCDs in turn, and each XCD gets a stretch of panels of four tiles of n, so that what its
// workgroups read together is in its cache.
__device__ __forceinline__ bool find_tile(int id, int ms, int ns, int splits, Tile &t, int &split)
{
    const int tiles = ms * ns, all = tiles * splits, each = (all + 7) / 8;
    int o = (id & 7) * each + (id >> 3);
    if ((id >> 3) >= each || o >= all) return false;
    split = o / tiles, o -= split * tiles;
    const int panels = ns / 4, whole = panels * 4 * ms;
    if (o < whole) t.n = o / (4 * ms) * 4 + o % 4, t.m = o % (4 * ms) / 4;
    else t.n = panels * 4 + (o - whole) % (ns % 4), t.m = (o - whole) / (ns % 4);
    return true;
}

// A tile of results on its way out: 16 bits each, in LDS as rows of n, whose chunks of 16 bytes change places with the row's number, so that
// neither the lanes' columns nor whole rows meet in a bank.  Memory then gets half a kilobyte of a row at a time; straight from the registers it
// would get pieces of 16 bytes (G of 7296 x 128000: 2570 us in place of 2490).
__device__ __forceinline__ int result_place(int n, int m) { return n * (LOSS_TILE * 2) + (((m >> 3) ^ (n & 31)) << 4) + (m & 4) * 2; }

#define KIND_STATISTICS 0
#define KIND_GRADIENT 1
#define KIND_D_HIDDEN 2
#define KIND_D_WEIGHT 3

// Tiles that lie in LDS at a time: three of the operand that comes from memory (the vocabulary for scores, the scores' gradients for the others), for
// which a step is not long enough, two of the other; the results' place afterwards.
struct TileLds {
    char near[2][TILE_BYTES], far[3][TILE_BYTES];
};
template <int DT, int KIND>
__device__ __forceinline__ void product(const LossArgs &a, TileLds &lds, int id)
{
    constexpr bool SCORES = KIND <= KIND_GRADIENT, A_ACROSS = !SCORES, B_ACROSS = KIND == KIND_D_WEIGHT;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), wm = wave >> 2, wn = wave & 3;
    const int live = uniform_load(a.state), row_tiles = (live + LOSS_TILE - 1) / LOSS_TILE;
    const int pieces = (a.piece + LOSS_TILE - 1) / LOSS_TILE, widths = a.columns / LOSS_TILE;
    // a gradient's tiles come once for each part of its axis, those of one part together
    const LossParts parts = SCORES ? LossParts{1, 1} : loss_parts(a, live);
    const int splits = KIND == KIND_D_HIDDEN ? parts.hidden : parts.weight;
    Tile t;
    int split = 0;
    if (!find_tile(id, SCORES ? pieces : widths, KIND == KIND_D_WEIGHT ? pieces : row_tiles, splits, t, split)) return;

    // a piece's gradients lie tile by tile, rows by pieces, 128 KB each; packed states too, of 64 columns, 32 KB each
    constexpr int64_t G_TILE = LOSS_TILE * LOSS_TILE * 2;
    Operand<A_ACROSS> A;
    Operand<B_ACROSS> B;
    int64_t a_step = 2 * BK, b_step = TILE_BYTES;
    int begin = 0, steps, end_left = BK;  // steps of k, what there is of the last
    if constexpr (SCORES) {
        steps = a.pitch / BK, end_left = a.width - (steps - 1) * BK;
        A.set(a.weight, a.weight_stride, a.first + t.m * LOSS_TILE, a.vocabulary, 0);
        B.set(a.packed + (int64_t)t.n * steps * TILE_BYTES, 2 * BK, 0, LOSS_TILE, 0);
    } else if constexpr (KIND == KIND_D_HIDDEN) {
        const int all = (a.piece + BK - 1) / BK, share = (all + splits - 1) / splits;
        begin = min(all, split * share), steps = min(all, begin + share) - begin;
        if (begin + steps == all) end_left = a.piece - (all - 1) * BK;
        a_step = BK * a.weight_stride, b_step = 2 * BK;
        A.set(a.weight + (a.first + (int64_t)begin * BK) * a.weight_stride, a.weight_stride, t.m * LOSS_TILE, 0, a.width);
        B.set(a.gradient + ((int64_t)t.n * pieces + begin / 4) * G_TILE + begin % 4 * (2 * BK), 2 * LOSS_TILE, 0, LOSS_TILE, 0);
    } else {
        const int all = (live + BK - 1) / BK, share = (all + splits - 1) / splits;
        begin = min(all, split * share), steps = min(all, begin + share) - begin;
        a_step = (int64_t)widths * TILE_BYTES;
        A.set(a.scaled + ((int64_t)begin * widths + t.m) * TILE_BYTES, 2 * LOSS_TILE, 0, 0, LOSS_TILE);
        B.set(a.gradient + ((int64_t)(begin / 4) * pieces + t.n) * G_TILE + begin % 4 * TILE_BYTES, 2 * LOSS_TILE, 0, 0, LOSS_TILE);
    }
    Places<A_ACROSS, 4> pa;
    Places<B_ACROSS, 2> pb;
    pa.set(wm * 128), pb.set(wn * 64);

    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = zero16();

    // A wave's loads of a step go to its own 4 KB of both tiles.  The far operand's tile of step s is in place `slot`, s modulo 3.
    const uint32_t near_mine = lds_address(lds.near) + wave * 4096, far_mine = lds_address(lds.far) + wave * 4096;
    int slot = 0;
    const auto bring_a = [&](uint32_t to, int i, bool last) {
        if (KIND != KIND_D_WEIGHT && last && end_left < BK) A.load_end(i, to, end_left, a.weight_stride);
        else A.load(i, to);
    };
    const auto bring_near = [&](int s, int i, bool last) {
        const uint32_t to = near_mine + (s & 1) * TILE_BYTES;
        if constexpr (SCORES) B.load(i, to);
        else bring_a(to, i, last);
    };
    const auto bring_far = [&](int place, int i, bool last) {
        const uint32_t to = far_mine + place * TILE_BYTES;
        if constexpr (SCORES) bring_a(to, i, last);
        else B.load(i, to);
    };
    const auto advance_near = [&]() {
        if constexpr (SCORES) B.step(b_step);
        else A.step(a_step);
    };
    const auto advance_far = [&](int s) {  // from step s to the next; four steps are a tile of gradients
        if constexpr (SCORES) A.step(a_step);
        else if constexpr (KIND == KIND_D_HIDDEN) B.step(((begin + s) & 3) == 3 ? G_TILE - 6 * BK : 2 * BK);
        else B.step(((begin + s) & 3) == 3 ? pieces * G_TILE - 3 * TILE_BYTES : TILE_BYTES);
    };
    // d_weight: which of a wave's next 1024 rows have a target in the tile; a lane's rows are 64 apart, a bit each
    const int end = min(live, (begin + steps) * BK), first_entry = (int)a.first + t.n * LOSS_TILE;
    int looked[16];
    const auto look = [&](int r0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) looked[i] = a.target[min(r0 + wave * 1024 + i * 64 + lane, end - 1)];
    };
    const auto found = [&](int r0) {
        int bits = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) bits |= (int)(r0 + wave * 1024 + i * 64 + lane < end && (unsigned)(looked[i] - first_entry) < LOSS_TILE) << i;
        return bits;
    };
    int bits = 0;
    if (KIND == KIND_D_WEIGHT && end > 0) look(begin * BK);
    i32x4 p[2][4], q[2][2];
    const auto read = [&](int s, int place, int k) {
        const char *x = SCORES ? lds.far[place] : lds.near[s & 1], *y = SCORES ? lds.near[s & 1] : lds.far[place];
#pragma unroll
        for (int j = 0; j < 2; ++j) q[k & 1][j] = pb.read(y, j, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[k & 1][i] = pa.read(x, i, k);
    };
    const auto multiply = [&](int k, int i, int j) { acc[i][j] = mfma32<DT>(p[k & 1][i], q[k & 1][j], acc[i][j]); };
    // A quarter's products, with the next quarter's operands read among them.
    const auto quarter = [&](int s, int k) {
        constexpr int READS = (A_ACROSS ? 8 : 4) + (B_ACROSS ? 4 : 2);
        read(s, slot, k + 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) multiply(k, i >> 1, i & 1);
        // the order: one or two reads before each of the first six products
#define PAIR(I) __builtin_amdgcn_sched_group_barrier(0x100, READS / 6 + (I < READS % 6), 0), __builtin_amdgcn_sched_group_barrier(0x008, 1, 0)
        PAIR(0), PAIR(1), PAIR(2), PAIR(3), PAIR(4), PAIR(5);
#undef PAIR
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // Operands are read a quarter of a step before they are multiplied, those of the next step's first quarter too: its tiles have come when
    // the last quarter's operands are in registers, and the tiles of the steps after may then take this one's places.  The last steps stand
    // apart, so that the others have no branches.
    const auto step = [&](int s, auto stands) {
        constexpr int AFTER = decltype(stands)::value;  // steps that come after this one, 4: more than three
        const int next = slot == 2 ? 0 : slot + 1;
        quarter(s, 0);
        quarter(s, 1);
        quarter(s, 2);
        if constexpr (AFTER > 0) {
            wait_loads<AFTER >= 2 ? 4 : 0>();  // the far operand's of the step after next
            lds_barrier();
            read(s + 1, next, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            multiply(3, i >> 1, i & 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (AFTER >= 2)
                if (i < 4) bring_near(s + 2, i, AFTER == 2);
            if constexpr (AFTER >= 3)
                if (i >= 4) bring_far(slot, i - 4, AFTER == 3);
        }
        if constexpr (AFTER > 2) advance_near();
        if constexpr (AFTER > 3) advance_far(s + 3);
        slot = next;
    };
    if (steps > 0) {
        const auto first = [&](int s, bool with_near) {
            if (s >= steps) return;
            if (with_near) {
#pragma unroll
                for (int i = 0; i < 4; ++i) bring_near(s, i, s == steps - 1);
                advance_near();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) bring_far(s, i, s == steps - 1);
            advance_far(s);
        };
        first(0, true);
        first(1, true);
        first(2, false);
        if (KIND == KIND_D_WEIGHT) bits = found(begin * BK);
        if (steps == 1) wait_loads<0>();
        else if (steps == 2) wait_loads<8>();
        else wait_loads<12>();
        lds_barrier();
        read(0, 0, 0);
        for (int s = 0; s < steps - 4; ++s) step(s, std::integral_constant<int, 4>());
        if (steps > 3) step(steps - 4, std::integral_constant<int, 3>());
        if (steps > 2) step(steps - 3, std::integral_constant<int, 2>());
        if (steps > 1) step(steps - 2, std::integral_constant<int, 1>());
        step(steps - 1, std::integral_constant<int, 0>());
    }

    if constexpr (KIND == KIND_D_WEIGHT) {
        // What the targets' entries left out: the rows whose target is one of the tile's are multiplied again, 64 of them at a time, with a tile that has a
        // single entry in each.  They are looked for among all of the axis, up to 8192 at a time, in order.
        // (Both gradients of 7296 rows of 2048, 5107 with a target, on 128000 entries 4560 us in place of 4480, of 509 rows of 768 on 32128 76 in place
        // of 70; looked for after the other products, and in LossRow: 4710 and 77.  The errors of both, bf16 0.0024 and fp16 0.0003 of the
        // gradients' norm, are 0.0017 and 0.00021, as of one rounding.)
        int *const list = (int *)lds.far[2], *const counts = (int *)lds.far[1];
        for (int r0 = begin * BK; r0 < end; r0 += TILE_BYTES / 4) {
            if (r0 > begin * BK) look(r0), bits = found(r0);
            const int mine0 = r0 + wave * 1024 + lane;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) mine += __popcll(__ballot(bits >> i & 1));
            lds_barrier();  // the tiles have been read
            if (lane == 0) counts[wave] = mine;
            lds_barrier();
            int at = 0, all = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (w < wave) at += counts[w];
                all += counts[w];
            }
            for (int i = 0; i < 16; ++i) {
                const uint64_t votes = __ballot(bits >> i & 1);
                if (bits >> i & 1) list[at + __popcll(votes & ((1ull << lane) - 1))] = mine0 + i * 64;
                at += __popcll(votes);
            }
            for (int b = 0; b < all; b += BK) {
                lds_barrier();  // the list is there; the tiles have been read
                const int here = min(all - b, BK), quarters = (here + 15) / 16;
                const int single = (int)threadIdx.x < here ? list[b + threadIdx.x] : -1;
                const int entry = single < 0 ? 0 : a.target[single] - first_entry;
                const float rest = single < 0 ? 0.0f : a.rest[single];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (((wave * 4 + i) & 15) >= quarters * 4) continue;
                    const int load = wave * 4 + i, k = (load & 15) * 4 + (lane >> 4), column = (load >> 4) * 128 + (((lane & 15) ^ swizzle<128>(k)) * 8);
                    const int row = k < here ? list[b + k] : -1;
                    const char *p = a.scaled + ((int64_t)(row / BK) * widths + t.m) * TILE_BYTES + row % BK * (2 * LOSS_TILE) + column * 2;
                    load_to_lds(row < 0 ? (const char *)zero_row : p, near_mine + i * 1024);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) *(i32x4 *)(lds.far[0] + (i * 512 + threadIdx.x) * 16) = i32x4{0, 0, 0, 0};
                lds_barrier();
                if (single >= 0) {
                    const int k = threadIdx.x;
                    store16<DT>(lds.far[0] + (entry >> 7) * (TILE_BYTES / 2) + k * 256 + ((((entry & 127) >> 3) ^ swizzle<128>(k)) << 4) + (entry & 7) * 2, rest);
                }
                wait_loads<0>();
                lds_barrier();
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if (s >= quarters) break;
                    read(0, 0, s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) multiply(s, i >> 1, i & 1);
                }
            }
        }
    }

    // a lane's results: column n = 64 wn + 32 j + lane % 32, rows m = 128 wm + 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4
    const int m0 = t.m * LOSS_TILE + wm * 128 + 4 * (lane >> 5), n0 = t.n * LOSS_TILE + wn * 64 + (lane & 31);
    char *const results = lds.near[0];
    const auto keep = [&](int i, int j, int c, float x0, float x1, float x2, float x3) {
        *(i32x2 *)(results + result_place((n0 & 255) + 32 * j, (m0 & 255) + 32 * i + 8 * c)) = i32x2{pack2<DT>(x0, x1), pack2<DT>(x2, x3)};
    };
    // The kept tile's rows: 32 lanes a row, in turn.
    const auto send = [&](char *out, int64_t stride, int rows, int columns) {
        __syncthreads();
#pragma unroll 4
        for (int k = 0; k < LOSS_TILE / 16; ++k) {
            const int n = k * 16 + wave * 2 + (lane >> 5), m = (lane & 31) * 8;
            if (n < rows && m < columns) *(i32x4 *)(out + n * stride + m * 2) = *(const i32x4 *)(results + result_place(n, m));
        }
    };
    if (KIND == KIND_GRADIENT || (KIND == KIND_D_WEIGHT && splits == 1)) __syncthreads();  // all waves are done with the operands
    if constexpr (KIND == KIND_STATISTICS) {
        const float f = exponent_factor(a);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = n0 + 32 * j;
            const bool there = row < live;
            const int target = there ? a.row[row].target - (int)a.first - m0 : -1;  // place in the piece, from the lane's first
            if (__any(target >= 0 && target < 128)) {  // the target is kept apart
                float own = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool is = 32 * i + 8 * (r / 4) + r % 4 == target;
                        own = is ? acc[i][j][r] : own;
                        acc[i][j][r] = is ? -INFINITY : acc[i][j][r];
                    }
                if (target >= 0 && target < 128 && !(target & 4) && m0 + target < a.piece) a.own[row] = own;
            }
            if (t.m == pieces - 1)  // entries past the end
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = m0 + 32 * i + 8 * (r / 4) + r % 4 < a.piece ? acc[i][j][r] : -INFINITY;
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
            most = max_halves(most);
            const float base = most == -INFINITY ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * f);
            sum = sum_halves(sum);
            if (lane < 32) a.part[(int64_t)(t.m * 2 + wm) * a.padded_rows + row] = {most, sum};
        }
    } else if constexpr (KIND == KIND_GRADIENT) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = n0 + 32 * j;
            const bool there = row < live;
            const LossRow x = there ? a.row[row] : LossRow{-1, 0, 0.0f, 0.0f, 0.0f};
            const int target = there ? x.target - (int)a.first - m0 : -1;
            const ScoreGradient gradient(x, a, DT);
            if (t.n == row_tiles - 1)  // rows past the end, packed as zeros: whatever the vocabulary holds
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = there ? acc[i][j][r] : 0.0f;
            if (t.m == pieces - 1)  // entries past the end
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = m0 + 32 * i + 8 * (r / 4) + r % 4 < a.piece ? acc[i][j][r] : -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    keep(i, j, c, gradient.other(acc[i][j][4 * c]), gradient.other(acc[i][j][4 * c + 1]), gradient.other(acc[i][j][4 * c + 2]), gradient.other(acc[i][j][4 * c + 3]));
            if (__any(target >= 0 && target < 128)) {
                float own = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) own = 32 * i + 8 * (r / 4) + r % 4 == target ? acc[i][j][r] : own;
                const int n = (n0 & 255) + 32 * j, m = (m0 & 255) + target;
                if (target >= 0 && target < 128 && !(target & 4) && m0 + target < a.piece) {
                    const float g = gradient.target(own);
                    store16<DT>(results + result_place(n, m) + (m & 3) * 2, g);
                    a.rest[row] = left_out<DT>(g);
                }
            }
        }
        send(a.gradient + ((int64_t)t.n * pieces + t.m) * G_TILE, LOSS_TILE * 2, LOSS_TILE, LOSS_TILE);
    } else if (KIND == KIND_D_HIDDEN || splits > 1) {
        // sums over parts stay in the order of the registers: 1 KB of a wave at a time; those of d_hidden go on from piece to piece
        float *out = KIND == KIND_D_HIDDEN ? a.d_part + (((int64_t)split * row_tiles + t.n) * widths + t.m) * (LOSS_TILE * LOSS_TILE)
                                           : a.w_part + (((int64_t)split * pieces + t.n) * widths + t.m) * (LOSS_TILE * LOSS_TILE);
        out += wave * 8192 + lane * 4;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f32x4 *p = (f32x4 *)(out + ((j * 4 + i) * 4 + c) * 256);
                    f32x4 v = {acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]};
                    if (KIND == KIND_D_HIDDEN && a.first > 0) v += *p;
                    *p = v;
                }
    } else {
        const float factor = score_factor(a) * (DT == PLAID_FP16 ? 0x1p-15f : 1.0f);
        const int exponent = uniform_load(a.state + 1);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float g[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) g[r] = ldexpf(acc[i][j][4 * c + r] * factor, exponent);
                    keep(i, j, c, g[0], g[1], g[2], g[3]);
                }
        send(a.d_weight + ((a.first + t.n * LOSS_TILE) * (int64_t)a.width + t.m * LOSS_TILE) * 2, (int64_t)a.width * 2, a.piece - t.n * LOSS_TILE, a.width - t.m * LOSS_TILE);
    }
}

template <int DT, int KIND>
__global__ __launch_bounds__(512, 2) void loss_mm_kernel(LossArgs a)
{
    __shared__ __align__(16) TileLds lds;
    product<DT, KIND>(a, lds, blockIdx.x);
}
// Both gradients: d_hidden's tiles, which take longer, then d_weight's.
template <int DT>
__global__ __launch_bounds__(512, 2) void loss_gradients_kernel(LossArgs a, int hidden)
{
    __shared__ __align__(16) TileLds lds;
    if ((int)blockIdx.x < hidden) product<DT, KIND_D_HIDDEN>(a, lds, blockIdx.x);
    else product<DT, KIND_D_WEIGHT>(a, lds, blockIdx.x - hidden);
}

static int rounded_up(int64_t tiles) { return (int)((tiles + 7) / 8 * 8); }

void plaid_launch_loss_scores(hipStream_t st, const LossArgs &a, int dtype, bool backward)
{
    const int grid = rounded_up((int64_t)((a.piece + LOSS_TILE - 1) / LOSS_TILE) * (a.padded_rows / LOSS_TILE));
#define GO(DT) backward ? loss_mm_kernel<DT, KIND_GRADIENT><<<grid, 512, 0, st>>>(a) : loss_mm_kernel<DT, KIND_STATISTICS><<<grid, 512, 0, st>>>(a)
    if (dtype == PLAID_BF16) GO(PLAID_BF16);
    else GO(PLAID_FP16);
#undef GO
}
void plaid_launch_loss_gradients(hipStream_t st, const LossArgs &a, int dtype)
{
    const int64_t widths = a.columns / LOSS_TILE;
    const int hidden = a.d_hidden ? rounded_up(loss_hidden_parts(a.padded_rows, a.columns, a.hidden_steps)) : 0;
    const int weight = !a.d_weight ? 0 : rounded_up(a.w_part ? loss_weight_parts(a.padded_rows, a.columns, a.hidden_steps) : widths * ((a.piece + LOSS_TILE - 1) / LOSS_TILE));
    if (dtype == PLAID_BF16) loss_gradients_kernel<PLAID_BF16><<<hidden + weight, 512, 0, st>>>(a, hidden);
    else loss_gradients_kernel<PLAID_FP16><<<hidden + weight, 512, 0, st>>>(a, hidden);
}
