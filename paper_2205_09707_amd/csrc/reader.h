// Declarations shared by the kernels of the reader: block tables, the cache in four bits, attention (gfx950 only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plaid.h"

int plaid_fail(int code, const char *fmt, ...);  // sets plaid_last_error's text and returns code

// ---------------------------------------------------------------------------------------------
// Arguments of the attention kernels (by value).  Rows of a request and key head are its tokens and the group's heads, row
// t * group + g, so that heads that share keys share the tiles of them.
// ---------------------------------------------------------------------------------------------
struct AttendArgs {
    const char *q, *k, *v;             // elements of 16 bits
    const char *bias;                  // [num_keys] of the type, or null
    const int64_t *q_offsets, *k_offsets;
    char *out;
    float *lse;                        // pairs whose sum is the logarithm of the sum of exponentials: a shift, and the rest; may be null.
                                       // (-infinity, 0): no key; (the biases' shift, -infinity): keys whose scores are all -infinity
    int64_t num_queries, num_keys;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;  // strides in bytes
    int32_t n, heads, kv_heads, group;
    uint32_t group_magic;              // ceil(2^32 / group): row / group = umulhi(row, magic) for group > 1
    float scale;                       // forward: > 0, negate_q carries the sign
    float inv_scale;                   // 1 / scale, or of the least scale that exponents are formed with
    uint32_t negate_q;                 // 0x80008000 where the caller's scale is negative, else 0
    // paged source
    const uint8_t *cache;
    const int32_t *table, *lengths;
    int64_t table_stride, num_blocks;
    int32_t max_blocks, block_shift, causal;
    // split over keys: partial sums
    int32_t splits;
    float *part_o;                     // outputs of parts of the keys. attend_many: [splits][num_queries][heads][D]; attend_few: [workers][2][kv_heads][16][D]
    float *part_lse;                   // the same without D, pairs as in lse, (-infinity, 0) without a key
};

struct GradArgs {
    AttendArgs a;                      // out and lse are inputs
    float factor;                      // the scale as it was given, of dq and dk
    const char *d_out;
    char *dq, *dk, *dv, *dbias;        // any may be null
    float *delta, *delta_sum;          // [num_queries][heads] -dO . out, corrected in place; corrected, where the keys are cut into parts
    float *row_part;                   // [q_splits][num_queries][heads][2] sums of dS and |dS| over parts of the keys, null with one part
    int32_t *far;                      // [workgroups of dq][4] whether a wave's rows need a second pass, with one part
    float *exponent;                   // [num_queries][heads] -lse / scale without the shift; without a key an infinity that makes weights 0
    float *dbias_part;                 // [splits][kv_heads][num_keys], null without dbias
    float *dk_part, *dv_part;          // [splits][num_keys][kv_heads][D], null with one split
    float *dq_part;                    // [splits][num_queries][heads][D], null with one split
};

#define PLAID_SOURCE_DENSE 0
#define PLAID_SOURCE_BIAS 1
#define PLAID_SOURCE_PAGED 2

// Keys that a step of attend_few's workgroup covers, rows of its tiles.
#define FEW_KEYS 128
#define FEW_ROWS 16
// Waves of attend_few on a SIMD: what its registers allow without spills (dense D = 128 keeps 64 of them for loads under way).
#define FEW_PER_SIMD(D, SRC) ((D) == 64 ? 4 : (SRC) == PLAID_SOURCE_PAGED ? 3 : 2)
// Keys of a tile of attend_many.
#define MANY_KEYS 64

// Launchers.  workers: workgroups of attend_few per key head, 0: one for each tile.
void plaid_launch_attend_few(hipStream_t st, const AttendArgs &a, int dtype, int head_dim, int source, int workers, int64_t tiles);
void plaid_launch_attend_many(hipStream_t st, const AttendArgs &a, int dtype, int head_dim, int source, int waves, int64_t tiles);
void plaid_launch_attend_grad(hipStream_t st, const GradArgs &g, int dtype, int head_dim, int q_splits, int k_waves, int k_splits);
void plaid_launch_cache_write(hipStream_t st, const plaid_paged_cache &c, const char *k, const char *v, int64_t k_token, int64_t k_head,
                              int64_t v_token, int64_t v_head, const int64_t *slots, int64_t n);
void plaid_launch_cache_read(hipStream_t st, const plaid_paged_cache &c, const int64_t *slots, int64_t n, char *k, char *v);
struct TablesArgs {
    const int32_t *lengths, *added, *free_blocks;
    int32_t *table, *totals, *positions;
    int64_t *offsets, *slots, *blocks_wanted;
    int64_t table_stride, capacity;
    int32_t n, max_blocks, n_free, block_shift;
    int64_t *scan;                     // [2][n + 1] prefix sums of tokens and blocks, null where one launch does all
};
void plaid_launch_block_tables(hipStream_t st, const TablesArgs &t);
int64_t plaid_block_tables_scan_bytes(int32_t n, int64_t capacity);

#ifdef __HIP__
// ---------------------------------------------------------------------------------------------
// Device side
// ---------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// C += A . B, 32 x 32 x 16: lane l holds row / column l % 32 of A / B at k = 8 (l / 32) .. + 7; C: column l % 32, register r is
// row 8 (r / 4) + 4 (l / 32) + r % 4.
template <int DT>
__device__ __forceinline__ f32x16 mfma32(i32x4 a, i32x4 b, f32x16 c)
{
    if constexpr (DT == PLAID_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// 16 x 16 x 32: lane l holds row / column l % 16 at k = 8 (l / 16) .. + 7; C: column l % 16, register r is row 4 (l / 16) + r.
template <int DT>
__device__ __forceinline__ f32x4 mfma16(i32x4 a, i32x4 b, f32x4 c)
{
    if constexpr (DT == PLAID_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Two values rounded (to nearest, ties to even) to the type, the first in the low half.
template <int DT>
__device__ __forceinline__ int pack2(float x, float y)
{
    if constexpr (DT == PLAID_BF16) {
        bf16x2 p;
        p[0] = (__bf16)x;
        p[1] = (__bf16)y;
        return __builtin_bit_cast(int, p);
    } else {
        f16x2 p;
        p[0] = (_Float16)x;
        p[1] = (_Float16)y;
        return __builtin_bit_cast(int, p);
    }
}
template <int DT>
__device__ __forceinline__ float unpack(int w, int half)
{
    if constexpr (DT == PLAID_BF16) return __int_as_float(half ? (w & 0xffff0000) : (w << 16));
    else return (float)__builtin_bit_cast(f16x2, w)[half];
}
template <int DT>
__device__ __forceinline__ float load16(const char *p)
{
    return unpack<DT>(*(const uint16_t *)p, 0);
}
template <int DT>
__device__ __forceinline__ void store16(char *p, float x)
{
    *(uint16_t *)p = (uint16_t)pack2<DT>(x, 0.0f);
}
// Two codes of a byte (BYTE of w) times a power of two, exact; the low half's value first.
template <int DT, int BYTE>
__device__ __forceinline__ int codes2(int w, float power)
{
    if constexpr (DT == PLAID_BF16) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((unsigned)w, power, BYTE));
    else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4((unsigned)w, power, BYTE));
}
// The power of byte `byte` of w as codes2 takes it: the conversion reads the exponent's eight bits alone (bits 23 to 30, 255: every
// code is NaN), so what a shift leaves in the others does not matter.
__device__ __forceinline__ float scale_power(int w, int byte) { return __int_as_float(byte == 3 ? (int)((uint32_t)w >> 1) : w << (23 - 8 * byte)); }

// A lane's value and that of the lane 32 (16) further on, exchanged between registers.
__device__ __forceinline__ float2 both_halves(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return {__uint_as_float(y[0]), __uint_as_float(y[1])};
}
__device__ __forceinline__ float2 both_rows(float x)
{
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return {__uint_as_float(y[0]), __uint_as_float(y[1])};
}
__device__ __forceinline__ float max_halves(float x)
{
    const float2 y = both_halves(x);
    return fmaxf(y.x, y.y);
}
__device__ __forceinline__ float sum_halves(float x)
{
    const float2 y = both_halves(x);
    return y.x + y.y;
}
__device__ __forceinline__ float max_rows(float x)
{
    const float2 y = both_rows(x);
    return fmaxf(y.x, y.y);
}
__device__ __forceinline__ float sum_rows(float x)
{
    const float2 y = both_rows(x);
    return y.x + y.y;
}
__device__ __forceinline__ f32x16 join16(f32x4 a, f32x4 b, f32x4 c, f32x4 d)
{
    const auto low = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), high = __builtin_shufflevector(c, d, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15);
}
// The larger of two products' results; fmaxf would first make each of them quiet.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, INFINITY); }

// Loads of what every lane wants alike, through the scalar cache: arguments that no kernel writes while one reads them.
template <typename T>
__device__ __forceinline__ T uniform_load(const T *p)
{
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)p;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)x) | ((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32));
}

// Row / group and row % group.
__device__ __forceinline__ int row_token(const AttendArgs &a, int row) { return a.group == 1 ? row : (int)__umulhi((uint32_t)row, a.group_magic); }

// The request that owns place p of the tiles, with the tiles of request r starting at floor(off[r] * per_token / tile) + r: a
// request of m rows has at least ceil(m / tile) places there, so the grid needs only the totals that the host knows.
// All lanes of a wave call it together and get the same answer; off is not trusted.
struct TilePlace {
    int r;       // request, -1: none
    int tile;    // tile of the request
    int64_t begin, end;  // its rows of the packed tensor
};
__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ TilePlace find_tile(const int64_t *off, int n, int64_t rows, int per_token, int tile_shift, int64_t p)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n - 1;  // the last request whose first place is <= p
    while (lo < hi) {
        const int64_t span = (int64_t)hi - lo;  // candidates lo + 1 .. hi, 64 of them tried at a time
        const int64_t step = (span + 63) >> 6;
        const int64_t at = lo + step * (lane + 1);
        bool below = false;
        if (at <= hi) below = ((clamp64(off[at], 0, rows) * per_token) >> tile_shift) + at <= p;
        const uint64_t votes = __ballot(below);
        const int k = votes ? 64 - __clzll((long long)votes) : 0;  // the highest lane that said yes, plus one
        const int64_t nlo = lo + step * k;
        const int64_t nhi = nlo + step - 1;
        lo = uniform((int)nlo);
        hi = uniform((int)(nhi < hi ? nhi : hi));
    }
    TilePlace t;
    t.begin = clamp64(uniform_load(off + lo), 0, rows);
    t.end = clamp64(uniform_load(off + lo + 1), t.begin, rows);
    const int64_t first = ((t.begin * per_token) >> tile_shift) + lo;
    t.tile = (int)(p - first);
    t.r = p >= first && ((int64_t)t.tile << tile_shift) < (t.end - t.begin) * per_token ? lo : -1;
    return t;
}

// The same with the requests in the order of `work`, what a tile of request r (of lane r) takes, the largest first, and a request's
// last tile, which sees the most of a causal mask, first: what starts last is short, so that all of the chip ends at about the same time.
// 6 prompts behind contexts: 498 us in place of 531; a training step of 16 long answers: 1981 in place of 2050.  Only for n <= 64, a lane for
// each request: with more of them there are many rounds of tiles, whose order matters less.
#define SORTED_REQUESTS 64
__device__ __forceinline__ TilePlace find_sorted_tile(const int64_t *off, int n, int64_t rows, int per_token, int tile_shift, int64_t p, int work)
{
    const int lane = threadIdx.x & 63, of = min(lane, n - 1);
    const int64_t begin = clamp64(off[of], 0, rows), end = clamp64(off[of + 1], begin, rows);
    const int tiles = lane < n ? (int)(((end - begin) * per_token + (1ll << tile_shift) - 1) >> tile_shift) : 0;
    int64_t first = 0;
    for (int j = 0; j < n; ++j) {
        const int other = __builtin_amdgcn_readlane(work, j);
        if (other > work || (other == work && j < lane)) first += __builtin_amdgcn_readlane(tiles, j);
    }
    const uint64_t mine = __ballot(first <= p && p < first + tiles);
    TilePlace t = {-1, 0, 0, 0};
    if (mine) {
        t.r = uniform((int)__ffsll((unsigned long long)mine) - 1);
        t.begin = clamp64(uniform_load(off + t.r), 0, rows);
        t.end = clamp64(uniform_load(off + t.r + 1), t.begin, rows);
        t.tile = __builtin_amdgcn_readlane((int)(first + tiles - 1 - p), t.r);
    }
    return t;
}

// What a workgroup of a grid of tiles x key heads x splits does.  Workgroups go to the eight XCDs in turn.  With an even number of
// key heads the heads come first: the tiles of one head, which share what they read, then meet on as many XCDs as eight has more
// factors of two than the number of heads, and every XCD gets the same mixture of long and short requests.  With an odd number
// the tiles come first, in stretches of four that go round the XCDs.
struct WorkPlace {
    int64_t place;
    int head, split;
};
__device__ __forceinline__ WorkPlace work_place(const AttendArgs &a, int64_t tiles, int splits, int64_t id)
{
    WorkPlace w;
    if (a.kv_heads & 1) {
        if (id < tiles * a.kv_heads * splits / 32 * 32) id = ((id >> 5) * 8 + (id & 7)) * 4 + ((id >> 3) & 3);
        w.place = id % tiles;
        id /= tiles;
        w.head = (int)(id % a.kv_heads), w.split = (int)(id / a.kv_heads);
    } else {
        w.head = (int)(id % a.kv_heads);
        id /= a.kv_heads;
        w.split = (int)(id % splits), w.place = id / splits;
    }
    return w;
}

// ---------------------------------------------------------------------------------------------
// Tiles of 16-bit values in LDS: rows of D values, their 16-byte chunks exchanged by an exclusive-or with a number of the
// row.  At D = 128 a row is as long as the 64 banks: the number's upper bits are row % 4, so that the 64-byte pieces of four
// rows that half a wave's transposing read takes lie in different banks, the lower ones are row / 4 % 4, so that sixteen rows'
// chunks of one column (a read along the rows) do too.  At D = 64 two rows share the banks and row / 2 % 2 does for row % 4.
// ---------------------------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ int swizzle(int row)
{
    return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

template <int D>
__device__ __forceinline__ int lds_chunk(int row, int chunk)
{
    return row * (D * 2) + ((chunk ^ swizzle<D>(row)) << 4);
}
// Operand along the row: rows base + l % 32, values 16 s + 8 (l / 32) .. + 7.  base is a multiple of 32.
template <int D>
__device__ __forceinline__ i32x4 lds_rows(const char *tile, int base, int s)
{
    const int lane = threadIdx.x & 63, f = swizzle<D>(lane & 31);
    return *(const i32x4 *)(tile + base * (D * 2) + (lane & 31) * (D * 2) + (((2 * s + (lane >> 5)) ^ f) << 4));
}
// Transposed operand: columns 32 dt + l % 32, rows base + 4 (l / 32) .. + 3 and base + 8 + 4 (l / 32) .. + 3 (base a multiple
// of 16): the order in which mfma32's result leaves its rows in a lane's registers 8 i .. 8 i + 7.
template <int D>
__device__ __forceinline__ i32x4 lds_columns(const char *tile, int base, int dt)
{
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 5) + ((lane >> 2) & 3), x = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const char *p = tile + base * (D * 2) + row * (D * 2) + (((4 * dt + x) ^ swizzle<D>(row)) << 4) + (lane & 1) * 8;
    const char *r = tile + base * (D * 2) + (row + 8) * (D * 2) + (((4 * dt + x) ^ swizzle<D>(row + 8)) << 4) + (lane & 1) * 8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
    const s16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)r);
    const i32x2 u = __builtin_bit_cast(i32x2, y), w = __builtin_bit_cast(i32x2, z);
    return i32x4{u[0], u[1], w[0], w[1]};
}
// Barrier of the workgroup for what its waves read and write in LDS themselves; loads from memory stay under way.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// Waits until at most N of the wave's loads are under way: loads straight into LDS are not waited for otherwise.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Biases.  Scores s + b are formed as s + (b - c) with a shift c, so that a mask of the type's lowest value, or any other large
// bias that all of a row's keys have, costs the scores nothing.  c depends on the biases of the keys that are not masked alone:
// 0 where the largest of them is within BIAS_USUAL, else the largest.  A part of the keys has its own; parts are joined under the
// largest.  So all rows of a request have one, also a row whose scores are -infinity throughout.  Beside a bias beyond BIAS_ALL a score vanishes, as it does in a sum in 64 bits.
#define BIAS_USUAL 256.0f
#define BIAS_ALL 4503599627370496.0f
struct Shift {
    float c = 0.0f, most = -INFINITY;  // most: the largest unusual bias
    bool usual = false, seen = false;  // whether a usual, an unusual one was seen
    __device__ __forceinline__ bool any() const { return usual || seen; }
    // Takes in a wave's biases: lanes that have an unusual one, their largest (looked at where there are any), whether any lane has
    // a usual one.
    __device__ __forceinline__ void add(uint64_t unusual, float largest, bool any_usual)
    {
        usual |= any_usual;
        seen |= unusual != 0;
        if (seen) {
            if (unusual) {
#pragma unroll
                for (int o = 32; o; o >>= 1) largest = fmaxf(largest, __shfl_xor(largest, o));
                most = fmaxf(most, __int_as_float(uniform(__float_as_int(largest))));
            }
            c = __int_as_float(uniform(__float_as_int(most > BIAS_USUAL ? most : usual ? 0.0f : most)));
        }
    }
};
__device__ __forceinline__ bool unusual_bias(float b) { return fabsf(b) > BIAS_USUAL && b != -INFINITY; }
__device__ __forceinline__ bool beside(float c) { return fabsf(c) > BIAS_ALL; }
// A score that vanishes beside b, unless it is not finite.
__device__ __forceinline__ float vanish(float s, float b) { return fabsf(s) < INFINITY ? b : s; }

// Waits for all of the wave's loads, and lets the compiler know: one that it is unsure of it would wait for in every round of a loop.
__device__ __forceinline__ void wait_all_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Where keys that are masked are loaded from: an infinity in what they hold would make a product with a weight of zero not a number.
static __device__ const i32x4 zero_row[16] = {};

// 16 (4) bytes of every lane, from base + off, into the 1024 (256) bytes of LDS at `to` (the same for all lanes), lane after lane.
// There is no result in registers and the compiler does not count these loads: it would have every transposing read of LDS wait
// for all of them.  (They go by register m0, which is reserved: the compiler keeps nothing there and sets it itself before what
// needs it, so it cannot be named as overwritten.)  What they bring is waited for with
// wait_loads, before the barrier that lets it be read and before the end.
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, char *to) { load_to_lds(base, off, lds_address(to)); }
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *from, char *to) { load_to_lds(from, lds_address(to)); }
__device__ __forceinline__ void load2_to_lds(const char *base, uint32_t off, uint32_t to)  // 2 bytes a lane, 4 in LDS
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load2_to_lds(const char *base, uint32_t off, uint32_t *to) { load2_to_lds(base, off, lds_address(to)); }
__device__ __forceinline__ void load4_to_lds(const float *from, float *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_address(to)), "v"(from) : "memory");
}
// Rows 8 i .. of a result's registers as an operand: registers 8 i .. 8 i + 7 rounded to the type.
template <int DT>
__device__ __forceinline__ i32x4 round8(const f32x16 &x, int i)
{
    return i32x4{pack2<DT>(x[8 * i], x[8 * i + 1]), pack2<DT>(x[8 * i + 2], x[8 * i + 3]), pack2<DT>(x[8 * i + 4], x[8 * i + 5]),
                 pack2<DT>(x[8 * i + 6], x[8 * i + 7])};
}
__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}
#endif
