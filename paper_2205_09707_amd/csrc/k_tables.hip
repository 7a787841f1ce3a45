// Block tables and slots of a step's new tokens, from the requests' lengths.
#include "reader.h"

// Two prefix sums over the requests (tokens, blocks) and a pass over the tokens, which is all writing: 12 bytes a token.  Up to
// TABLES_ONE requests each workgroup forms both sums in LDS for itself, so that a step needs one launch and no workspace; the
// sums cost it 8 n bytes from L2, its tokens 12 KB of writes.  More requests take a launch that leaves the sums in the workspace.
// 1000 prompts of 6500 tokens: 22 us, 3.6 TB/s of writes, of which about 5 go before a workgroup's first token; a step of 16 requests 4.6.
#define TABLES_ONE 2048
#define TABLES_THREADS 256
#define TABLES_TOKENS 4  // neighbouring tokens of a thread: 16-byte stores

struct Growth {
    int64_t old, added, have, want;
};
__device__ __forceinline__ Growth growth(const TablesArgs &t, int r)
{
    Growth g;
    g.old = max(t.lengths[r], 0);
    g.added = max(t.added[r], 0);
    const int64_t round = (1ll << t.block_shift) - 1;
    g.have = min((g.old + round) >> t.block_shift, (int64_t)t.max_blocks);
    g.want = min((g.old + g.added + round) >> t.block_shift, (int64_t)t.max_blocks) - g.have;
    return g;
}

// Exclusive prefix sums of all requests by one workgroup; out[n] is the total.  A thread has neighbouring requests, so that there
// is one scan over the threads however many requests there are.
__device__ __forceinline__ void scan_requests(const TablesArgs &t, int64_t *tokens, int64_t *blocks)
{
    __shared__ int64_t wave_sum[2][TABLES_THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int each = (t.n + TABLES_THREADS - 1) / TABLES_THREADS, r0 = min(t.n, (int)threadIdx.x * each), r1 = min(t.n, r0 + each);
    int64_t mine[2] = {0, 0};
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const Growth g = growth(t, r);
        mine[0] += g.added, mine[1] += g.want;
    }
    int64_t at[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int64_t sum = mine[k];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = __shfl_up(sum, o);
            if (lane >= o) sum += y;
        }
        if (lane == 63) wave_sum[k][wave] = sum;
        at[k] = sum - mine[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 0; w < TABLES_THREADS / 64; ++w)
            if (w < wave) at[k] += wave_sum[k][w];
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const Growth g = growth(t, r);
        tokens[r] = at[0], blocks[r] = at[1];
        at[0] += g.added, at[1] += g.want;
    }
    if (threadIdx.x == TABLES_THREADS - 1) tokens[t.n] = at[0], blocks[t.n] = at[1];
}

// The last request whose sum is <= x (sums ascend from 0, x < sums[n]), from request `from` on, where it usually is.
__device__ __forceinline__ int owner(const int64_t *sums, int n, int64_t x, int from = 0)
{
    if (x < sums[from + 1]) return from;
    int lo = from, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The request that a thread is at: kept over its tokens, as most of them have the same.
struct Owner {
    int r;
    int64_t first, end;       // its tokens
    uint32_t old, have, held; // tokens before, blocks before, blocks now
    int64_t fresh;            // block b >= have is the free block fresh + b
    const int32_t *row;
};
__device__ __forceinline__ Owner owner_of(const TablesArgs &t, const int64_t *tokens, const int64_t *blocks, int r)
{
    const Growth g = growth(t, r);
    return {r, tokens[r], tokens[r + 1], (uint32_t)g.old, (uint32_t)g.have, (uint32_t)(g.have + g.want), blocks[r] - g.have, t.table + r * t.table_stride};
}
__device__ __forceinline__ int block_id(const TablesArgs &t, const Owner &o, uint32_t b)
{
    if (b < o.have) return o.row[b];
    return b < o.held && o.fresh + b < t.n_free ? t.free_blocks[o.fresh + b] : -1;
}

__device__ __forceinline__ void fill(const TablesArgs &t, const int64_t *tokens, const int64_t *blocks)
{
    const int64_t first = (int64_t)blockIdx.x * TABLES_THREADS + threadIdx.x, stride = (int64_t)gridDim.x * TABLES_THREADS;
    if (first == 0) t.blocks_wanted[0] = blocks[t.n];
    for (int64_t r = first; r <= t.n; r += stride) {
        t.offsets[r] = tokens[r];
        if (r < t.n) t.totals[r] = max(t.lengths[r], 0) + max(t.added[r], 0);
    }
    for (int64_t j = first; j < blocks[t.n]; j += stride) {
        const int r = owner(blocks, t.n, j);
        t.table[r * t.table_stride + growth(t, r).have + j - blocks[r]] = j < t.n_free ? t.free_blocks[j] : -1;
    }
    const int64_t all = min(tokens[t.n], t.capacity);
    // a workgroup's tokens are neighbours, so that a thread's request mostly stays
    constexpr int64_t SWEEP = TABLES_THREADS * TABLES_TOKENS;
    const int64_t per = (t.capacity + SWEEP * gridDim.x - 1) / (SWEEP * gridDim.x) * SWEEP, from = blockIdx.x * per;
    Owner own = {0, 0, 0, 0, 0, 0, 0, nullptr};
    const uint32_t within = (1u << t.block_shift) - 1;
    for (int64_t i = from + threadIdx.x * TABLES_TOKENS; i < min(t.capacity, from + per); i += SWEEP) {
        int position[TABLES_TOKENS];
        int64_t slot[TABLES_TOKENS];
        if (i < all && i >= own.end) own = owner_of(t, tokens, blocks, owner(tokens, t.n, i, own.r));
        if (i + TABLES_TOKENS <= min(all, own.end)) {  // of one request, in at most two blocks
            const uint32_t at = own.old + (uint32_t)(i - own.first), b = at >> t.block_shift, last = (at + TABLES_TOKENS - 1) >> t.block_shift;
            const int id = block_id(t, own, b), next = last == b ? id : block_id(t, own, last);
#pragma unroll
            for (int k = 0; k < TABLES_TOKENS; ++k) {
                const int of = (at + k) >> t.block_shift == b ? id : next;
                position[k] = (int)(at + k);
                slot[k] = of < 0 ? -1 : ((int64_t)of << t.block_shift) + ((at + k) & within);
            }
        } else {
#pragma unroll
            for (int k = 0; k < TABLES_TOKENS; ++k) {
                position[k] = -1;
                slot[k] = -1;
                if (i + k >= all) continue;
                while (i + k >= own.end) own = owner_of(t, tokens, blocks, own.r + 1);
                const uint32_t at = own.old + (uint32_t)(i + k - own.first);
                const int id = block_id(t, own, at >> t.block_shift);
                position[k] = (int)at;
                slot[k] = id < 0 ? -1 : ((int64_t)id << t.block_shift) + (at & within);
            }
        }
        if (i + TABLES_TOKENS <= t.capacity) {
            *(i32x4 *)(t.positions + i) = i32x4{position[0], position[1], position[2], position[3]};
            typedef __attribute__((ext_vector_type(2))) long long i64x2;
            *(i64x2 *)(t.slots + i) = i64x2{slot[0], slot[1]};
            *(i64x2 *)(t.slots + i + 2) = i64x2{slot[2], slot[3]};
        } else {
#pragma unroll
            for (int k = 0; k < TABLES_TOKENS; ++k)
                if (i + k < t.capacity) t.positions[i + k] = position[k], t.slots[i + k] = slot[k];
        }
    }
}

__global__ __launch_bounds__(TABLES_THREADS) void tables_one_kernel(TablesArgs t)
{
    extern __shared__ int64_t sums[];  // as much as the requests need, so that more workgroups find room
    int64_t *tokens = sums, *blocks = sums + t.n + 1;
    scan_requests(t, tokens, blocks);
    __syncthreads();
    fill(t, tokens, blocks);
}
__global__ __launch_bounds__(TABLES_THREADS) void tables_scan_kernel(TablesArgs t) { scan_requests(t, t.scan, t.scan + t.n + 1); }
__global__ __launch_bounds__(TABLES_THREADS) void tables_fill_kernel(TablesArgs t) { fill(t, t.scan, t.scan + t.n + 1); }

int64_t plaid_block_tables_scan_bytes(int32_t n, int64_t) { return n > TABLES_ONE ? 2 * ((int64_t)n + 1) * 8 : 0; }

void plaid_launch_block_tables(hipStream_t st, const TablesArgs &t)
{
    const int64_t per = TABLES_THREADS * TABLES_TOKENS;
    int64_t groups = (t.capacity + per - 1) / per;
    groups = groups < 1 ? 1 : groups > 2048 ? 2048 : groups;
    if (t.n <= TABLES_ONE) {
        tables_one_kernel<<<dim3((unsigned)groups), dim3(TABLES_THREADS), 2 * (t.n + 1) * sizeof(int64_t), st>>>(t);
    } else {
        tables_scan_kernel<<<dim3(1), dim3(TABLES_THREADS), 0, st>>>(t);
        tables_fill_kernel<<<dim3((unsigned)groups), dim3(TABLES_THREADS), 0, st>>>(t);
    }
}
