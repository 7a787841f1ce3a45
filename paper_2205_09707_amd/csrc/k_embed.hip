// Embedding: rows of a table for a list of tokens, and the table's gradient by sorted tokens.
#include "train.h"

// out_t = scale E[id_t].  A team of threads, a power of two of them, has a row, or four where there are many, whose loads are then under way together
// (100000 of 2048 out of 128000: 122 us in place of 151; 2000: 5.4 both).  Bound by memory: 819 MB less what rows asked for twice leave in the caches.
template <int DT, int ROWS>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs e, int team_shift)
{
    const int lane = threadIdx.x & ((1 << team_shift) - 1), teams = 256 >> team_shift;
    const int64_t t0 = (wide_block() * teams + (threadIdx.x >> team_shift)) * ROWS;
    if (t0 >= e.n) return;
    const char *row[ROWS];
    bool there[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t id = t0 + i < e.n ? e.ids[t0 + i] : -1;
        there[i] = id >= 0 && id < e.vocabulary;
        row[i] = e.table + (there[i] ? id : 0) * e.table_stride;
    }
    for (int at = lane * 8; at < e.width; at += 8 << team_shift) {
        i32x4 w[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) w[i] = there[i] ? load_piece(row[i], at, e.width) : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            Eight v = unpack8<DT>(w[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v.x[j] = there[i] ? v.x[j] * e.scale : 0.0f;
            if (t0 + i < e.n) store_piece(e.out + (t0 + i) * e.width * 2, at, e.width, pack8<DT>(v));
        }
    }
}

#define FILL_EACH 4  // pieces of 16 bytes that a thread fills
// --- the tokens in ascending order, equal ones in the order in which they stood -------------------------------------------------
// A radix sort from the lowest digit on; up to SORT_ONE tokens by one workgroup and in one launch (with the gradient of 50000 x 768: 100 tokens 26 us
// in place of 41 with three launches a pass, 4000 34 and 53, 8000 46 and 59).  Each wave has a stretch of places and goes through it 64 at a time:
// lanes with the same digit find each other by votes, so that every place's rank is counted in order and none depends on which atomic came first.
__device__ __forceinline__ int token_key(const EmbedArgs &e, int64_t t)
{
    const int64_t id = e.ids[t];
    return id >= 0 && id < e.vocabulary ? (int)id : (int)e.vocabulary;  // last
}
// Rank of the lane's digit behind what `count` (the wave's own, in LDS) holds of it; counts the 64 of them.  All lanes call it.
__device__ __forceinline__ int rank_digit(int digit, bool there, int bits, volatile int *count)
{
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? ones : ~ones;
    }
    const int lane = threadIdx.x & 63;
    const int before = there ? __popcll(same & ((1ull << lane) - 1)) : 0;
    const int base = there ? count[digit] : 0;
    __builtin_amdgcn_wave_barrier();
    if (there && before == 0) count[digit] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    return base + before;
}

// Up to SORT_ONE tokens: one workgroup, everything in LDS.  The others fill the gradient with zeros meanwhile, rows with a token too: there
// are few of them.
__global__ __launch_bounds__(1024) void sort_one_kernel(EmbedArgs e, int64_t pieces)
{
    constexpr int WAVES = 16, EACH = SORT_ONE / 1024;
    const int64_t block = wide_block();
    if (block > 0) {
        const i32x4 zero = {0, 0, 0, 0};
        const int64_t first = (block - 1) * (1024 * FILL_EACH) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < FILL_EACH; ++i)
            if (first + i * 1024 < pieces) *(i32x4_any *)(e.d_table + (first + i * 1024) * 16) = zero;
        // what is left of a whole number of pieces
        const int64_t rest = pieces * 8 + threadIdx.x;
        if (block == 1 && rest < e.vocabulary * e.width) *(uint16_t *)(e.d_table + 2 * rest) = 0;
        return;
    }
    if (threadIdx.x == 0) *e.shared = 0;
    __shared__ int keys[SORT_ONE], counts[WAVES][256], totals[256];
    __shared__ uint16_t places[SORT_ONE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = (int)e.n;
    const int each = (n + 1023) / 1024, base = wave * (each * 64) + lane;  // a wave's places: each times 64
    int key[EACH], place[EACH], rank[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        place[i] = base + i * 64;
        key[i] = i < each && place[i] < n ? token_key(e, place[i]) : 0;
    }
    for (int shift = 0; shift < e.bits; shift += 8) {
        for (int i = threadIdx.x; i < WAVES * 256; i += 1024) (&counts[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < each) rank[i] = rank_digit((key[i] >> shift) & 255, base + i * 64 < n, 8, counts[wave]);
        __syncthreads();
        int sum = 0;
        if (threadIdx.x < 256)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = counts[w][threadIdx.x];
                counts[w][threadIdx.x] = sum;
                sum += c;
            }
        if (threadIdx.x < 256) {
            int scan = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(scan, o);
                if (lane >= o) scan += y;
            }
            totals[threadIdx.x] = scan;  // inclusive, in the wave's 64 digits
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < each && base + i * 64 < n) {
                const int d = (key[i] >> shift) & 255;
                int to = rank[i] + counts[wave][d] + (d & 63 ? totals[d - 1] : 0);
                for (int w = 0; w < d >> 6; ++w) to += totals[64 * w + 63];
                keys[to] = key[i], places[to] = (uint16_t)place[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = base + i * 64;
            if (i < each && at < n) key[i] = keys[at], place[i] = places[at];
        }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = base + i * 64;
        if (i < each && at < n) e.keys[0][at] = key[i], e.places[0][at] = place[i];
    }
}

// More of them: a pass is three launches.  Counts of the digits of each tile; prefix sums over the tiles, a workgroup for each digit; places.
#define SORT_BINS 512
__device__ __forceinline__ int pass_key(const EmbedArgs &e, int pass, int64_t at) { return pass == 0 ? token_key(e, at) : e.keys[(pass + 1) & 1][at]; }

__global__ __launch_bounds__(256) void sort_count_kernel(EmbedArgs e, int pass, int tiles)
{
    __shared__ int count[SORT_BINS];
    const int bins = 1 << e.digit, shift = pass * e.digit;
    for (int i = threadIdx.x; i < bins; i += 256) count[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * SORT_TILE;
#pragma unroll
    for (int i = 0; i < SORT_TILE / 256; ++i) {
        const int64_t at = first + i * 256 + threadIdx.x;
        if (at < e.n) atomicAdd(&count[(pass_key(e, pass, at) >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += 256) e.counts[(int64_t)i * tiles + blockIdx.x] = count[i];
}

__global__ __launch_bounds__(256) void sort_scan_kernel(EmbedArgs e, int tiles)
{
    __shared__ int wave_sum[4];
    int *c = e.counts + (int64_t)blockIdx.x * tiles;
    if (blockIdx.x == 0 && threadIdx.x == 0) *e.shared = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int first = 0; first < tiles; first += 256) {
        const int at = first + threadIdx.x, mine = at < tiles ? c[at] : 0;
        int scan = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(scan, o);
            if (lane >= o) scan += y;
        }
        if (lane == 63) wave_sum[wave] = scan;
        __syncthreads();
        int base = before;
        for (int w = 0; w < wave; ++w) base += wave_sum[w];
        if (at < tiles) c[at] = base + scan - mine;
        before += wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
        __syncthreads();
    }
    if (threadIdx.x == 0) e.totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(256) void sort_place_kernel(EmbedArgs e, int pass, int tiles)
{
    constexpr int WAVES = 4, EACH = SORT_TILE / 256;
    __shared__ int counts[WAVES][SORT_BINS], wave_sum[WAVES];
    const int bins = 1 << e.digit, shift = pass * e.digit, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * SORT_TILE + wave * (EACH * 64);
    for (int i = threadIdx.x; i < WAVES * SORT_BINS; i += 256) (&counts[0][0])[i] = 0;
    int key[EACH], place[EACH], rank[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int64_t at = first + i * 64 + lane;
        key[i] = at < e.n ? pass_key(e, pass, at) : 0;
        place[i] = pass == 0 || at >= e.n ? (int)at : e.places[(pass + 1) & 1][at];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) rank[i] = rank_digit((key[i] >> shift) & (bins - 1), first + i * 64 + lane < e.n, e.digit, counts[wave]);
    __syncthreads();
    // where each digit starts: two neighbouring digits a thread
    const int d0 = 2 * threadIdx.x, t0 = d0 < bins ? e.totals[d0] : 0, t1 = d0 + 1 < bins ? e.totals[d0 + 1] : 0;
    int scan = t0 + t1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(scan, o);
        if (lane >= o) scan += y;
    }
    if (lane == 63) wave_sum[wave] = scan;
    __syncthreads();
    int base = scan - t0 - t1;
    for (int w = 0; w < wave; ++w) base += wave_sum[w];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (d0 + k < bins) {
            int sum = base + (k ? t0 : 0) + e.counts[(int64_t)(d0 + k) * tiles + blockIdx.x];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = counts[w][d0 + k];
                counts[w][d0 + k] = sum;
                sum += c;
            }
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (first + i * 64 + lane < e.n) {
            const int to = rank[i] + counts[wave][(key[i] >> shift) & (bins - 1)];
            e.keys[pass & 1][to] = key[i], e.places[pass & 1][to] = place[i];
        }
}

// --- sums -----------------------------------------------------------------------------------------------------------------------
// dE[v] = scale times the sum of d_out over the places of token v, in order, held in 32 bits.  The sorted places are cut into chunks, a
// team of threads each, so that a token that stands everywhere is no one's burden.  What a chunk has of a token that it shares with its
// neighbours goes to the workspace: [0] of a token that the chunk before has too, [1] of one that begins here and goes on.  Such beginnings are
// put on a list, in whatever order, and the second launch adds up each one's parts, in theirs.
//
// Measured: 100000 tokens on 128000 x 2048 in bf16, 2 in 100 without a row, as text has them: 35 us for the sort, 189 for sums and zeros (934 MB,
// 4.9 TB/s), 20 for the parts of tokens that several chunks share.  509 tokens on 50021 x 768: 12 for the sort and 77 MB of zeros beside it, 9, 4.
template <int DT>
__device__ __forceinline__ void write_row(const EmbedArgs &e, int key, int at, const Eight &sum)
{
    char *row = e.d_table + (int64_t)key * e.width * 2;
    Eight v;
    if (e.add) v = unpack8<DT>(load_piece(row, at, e.width));
#pragma unroll
    for (int i = 0; i < 8; ++i) v.x[i] = e.add ? v.x[i] + sum.x[i] * e.scale : sum.x[i] * e.scale;
    store_piece(row, at, e.width, pack8<DT>(v));
}
__device__ __forceinline__ void write_part(const EmbedArgs &e, int64_t chunk, int which, int at, const Eight &sum)
{
    float *p = e.part + (chunk * 2 + which) * (int64_t)e.columns() + at;
    *(f32x4 *)p = f32x4{sum.x[0], sum.x[1], sum.x[2], sum.x[3]};
    *(f32x4 *)(p + 4) = f32x4{sum.x[4], sum.x[5], sum.x[6], sum.x[7]};
}

// WIDE: a team is whole waves, whose lanes bring 64 tokens and places at a time; a place is then the same for all lanes.
template <int DT, bool WIDE>
__device__ __forceinline__ void add_chunk(const EmbedArgs &e, int team_shift, int64_t block, int slice)
{
    constexpr int AHEAD = 8;
    const int lane = threadIdx.x & ((1 << team_shift) - 1), teams = 256 >> team_shift;
    const int at = (slice * 256 + lane) * 8, wave_lane = threadIdx.x & 63;
    int64_t chunk = block * teams + (threadIdx.x >> team_shift);
    if (WIDE) chunk = uniform(chunk);
    const int64_t begin = chunk * e.chunk, end = min(begin + e.chunk, e.n);
    if (begin >= e.n || (!WIDE && at >= e.width)) return;
    const bool there = at < e.width;
    const int *keys = e.keys[e.sorted], *places = e.places[e.sorted];
    int key = keys[begin];
    bool shared = begin > 0 && keys[begin - 1] == key;  // with the chunk before
    if (WIDE) key = uniform(key), shared = uniform((int)shared);
    Eight sum = {};
    int many_keys = 0, many_places = 0;
    for (int64_t i = begin; i < end; i += AHEAD) {
        i32x4 w[AHEAD];
        int next[AHEAD];
        if (WIDE && ((i - begin) & 63) == 0) {
            const int64_t p = min(i + wave_lane, end - 1);
            many_keys = keys[p], many_places = places[p];
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            int place;
            if (WIDE) {
                const int from = (int)((i - begin) & 63) + k;
                next[k] = __builtin_amdgcn_readlane(many_keys, from), place = __builtin_amdgcn_readlane(many_places, from);
            } else {
                const int64_t p = min(i + k, end - 1);
                next[k] = keys[p], place = places[p];
            }
            w[k] = next[k] < e.vocabulary ? load_piece(e.d_out + place * e.d_out_stride, at, e.width) : i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i + k < end) {
                if (next[k] != key) {
                    if (there) {
                        if (shared) write_part(e, chunk, 0, at, sum);
                        else write_row<DT>(e, key, at, sum);
                    }
                    key = next[k], shared = false;
                    sum = Eight{};
                }
                const Eight v = unpack8<DT>(w[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum.x[j] += v.x[j];
            }
    }
    if (key >= e.vocabulary || !there) return;  // what has no token is last
    if (shared) write_part(e, chunk, 0, at, sum);
    else if (end < e.n && keys[end] == key) {
        write_part(e, chunk, 1, at, sum);
        if (lane == 0 && slice == 0) e.begins[atomicAdd(e.shared, 1)] = (int32_t)chunk;
    } else write_row<DT>(e, key, at, sum);
}

// Zeros for the rows of tokens that are not there: a wave looks 64 of them up in the sorted list, a lane each.
__device__ __forceinline__ void fill_absent(const EmbedArgs &e, int64_t block)
{
    const int lane = threadIdx.x & 63;
    const int64_t first = (block * 4 + (threadIdx.x >> 6)) * 64, mine = first + lane;
    if (first >= e.vocabulary) return;
    const int *keys = e.keys[e.sorted];
    int64_t lo = 0, hi = e.n;  // the first place whose token is not below mine
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < mine) lo = mid + 1;
        else hi = mid;
    }
    uint64_t absent = __ballot(mine < e.vocabulary && !(lo < e.n && keys[lo] == mine));
    while (absent) {
        const int r = __ffsll((unsigned long long)absent) - 1;
        absent &= absent - 1;
        char *row = e.d_table + (first + r) * e.width * 2;
        for (int at = lane * 8; at < e.width; at += 512) store_piece(row, at, e.width, i32x4{0, 0, 0, 0});
    }
}

// Chunks first, then rows without a token.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedArgs e, int team_shift, unsigned chunk_blocks, unsigned slices)
{
    if (blockIdx.x < chunk_blocks) add_chunk<DT, WIDE>(e, team_shift, blockIdx.x / slices, blockIdx.x % slices);
    else fill_absent(e, blockIdx.x - chunk_blocks);
}

// Up to 256 columns of a token that several chunks share: the threads that have the same four columns have a stretch of its parts each.
template <int DT>
__global__ __launch_bounds__(256) void embed_grad_join_kernel(EmbedArgs e, int lane_shift)
{
    __shared__ f32x4 lds[256];
    const int lane = threadIdx.x & 63, column = threadIdx.x & ((1 << lane_shift) - 1), share = threadIdx.x >> lane_shift, shares = 256 >> lane_shift;
    const int at = (blockIdx.y * 64 + column) * 4, many = *e.shared;
    const int *keys = e.keys[e.sorted];
    const int64_t columns = e.columns();
    for (int i = blockIdx.x; i < many; i += gridDim.x) {
        const int64_t chunk = e.begins[i];
        const int key = keys[chunk * e.chunk + e.chunk - 1];
        int parts = 1;  // this chunk's, and of as many chunks as begin with the token
        for (int more = 64; more == 64; parts += more) {
            const int64_t p = (chunk + parts + lane) * e.chunk;
            const uint64_t same = __ballot(p < e.n && keys[min(p, e.n - 1)] == key);
            more = same == ~0ull ? 64 : __ffsll((unsigned long long)~same) - 1;
        }
        const int each = (parts + shares - 1) / shares, first = share * each, last = min(parts, first + each);
        f32x4 sum = {0, 0, 0, 0};
        if (at < columns) {
            const float *p = e.part + chunk * 2 * columns + at;  // part 0 has place 1 of its chunk, the others place 0
#pragma unroll 8
            for (int k = first; k < last; ++k) sum += *(const f32x4 *)(p + (k == 0 ? 1 : 2 * k) * columns);
        }
        lds[threadIdx.x] = sum;
        __syncthreads();
        if (share == 0 && at < e.width) {
            for (int w = 1; w < min(shares, parts); ++w) sum += lds[(w << lane_shift) + column];
            char *row = e.d_table + ((int64_t)key * e.width + at) * 2;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at + j < e.width) store16<DT>(row + 2 * j, e.add ? load16<DT>(row + 2 * j) + sum[j] * e.scale : sum[j] * e.scale);
        }
        __syncthreads();
    }
}

static int team_shift_of(int width)
{
    int s = 0;
    while (s < 8 && (8 << s) < width) ++s;
    return s;
}

void plaid_launch_embedding(hipStream_t st, const EmbedArgs &e, int dtype)
{
    const int shift = team_shift_of(e.width);
    const int64_t teams = 256 >> shift;
    const bool four = e.n >= 4096 * teams;
    const dim3 grid = wide_grid((e.n + teams * (four ? 4 : 1) - 1) / (teams * (four ? 4 : 1)));
#define GO(DT, R) embed_kernel<DT, R><<<grid, 256, 0, st>>>(e, shift)
    if (dtype == PLAID_BF16) four ? GO(PLAID_BF16, 4) : GO(PLAID_BF16, 1);
    else four ? GO(PLAID_FP16, 4) : GO(PLAID_FP16, 1);
#undef GO
}

template <int DT>
static void launch_backward(hipStream_t st, const EmbedArgs &e)
{
    const bool one = e.n <= SORT_ONE, fill = one && !e.add;
    if (one) {
        const int64_t pieces = fill ? e.vocabulary * e.width / 8 : 0;
        const int64_t blocks = fill ? (pieces + 1024 * FILL_EACH - 1) / (1024 * FILL_EACH) : 0;
        sort_one_kernel<<<wide_grid(1 + (fill && blocks == 0 ? 1 : blocks)), 1024, 0, st>>>(e, pieces);
    } else
        for (int pass = 0; pass < e.passes; ++pass) {
            const int tiles = (int)((e.n + SORT_TILE - 1) / SORT_TILE);
            sort_count_kernel<<<tiles, 256, 0, st>>>(e, pass, tiles);
            sort_scan_kernel<<<1 << e.digit, 256, 0, st>>>(e, tiles);
            sort_place_kernel<<<tiles, 256, 0, st>>>(e, pass, tiles);
        }
    if (e.n == 0) return;
    const int shift = team_shift_of(e.width);
    const int64_t teams = 256 >> shift, chunks = (e.n + e.chunk - 1) / e.chunk, slices = (e.width + 2047) / 2048;
    const unsigned chunk_blocks = (unsigned)((chunks + teams - 1) / teams * slices);
    const unsigned fill_blocks = !one && !e.add ? (unsigned)((e.vocabulary + 255) / 256) : 0;
    if (shift >= 6) embed_grad_kernel<DT, true><<<chunk_blocks + fill_blocks, 256, 0, st>>>(e, shift, chunk_blocks, (unsigned)slices);
    else embed_grad_kernel<DT, false><<<chunk_blocks + fill_blocks, 256, 0, st>>>(e, shift, chunk_blocks, (unsigned)slices);
    if (chunks > 1) {
        const int lane_shift = shift + 1 < 6 ? shift + 1 : 6;  // a team's thread has eight columns, one of these four
        embed_grad_join_kernel<DT><<<dim3((unsigned)(chunks < 1024 ? chunks : 1024), (unsigned)((e.width + 255) / 256)), 256, 0, st>>>(e, lane_shift);
    }
}
void plaid_launch_embedding_backward(hipStream_t st, const EmbedArgs &e, int dtype)
{
    dtype == PLAID_BF16 ? launch_backward<PLAID_BF16>(st, e) : launch_backward<PLAID_FP16>(st, e);
}
