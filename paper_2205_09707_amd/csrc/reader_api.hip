// C entry points of the reader (include/plaid.h): argument checks, the choice of kernel and of how the work is cut, workspaces.
#include <cmath>

#include "api_common.h"
#include "reader.h"

namespace {

bool block_size_ok(int32_t b) { return b == 16 || b == 32 || b == 64 || b == 128 || b == 256; }

int check_cache(const plaid_paged_cache *c)
{
    if (!c) FAIL("cache is null");
    if (!block_size_ok(c->block_size)) FAIL("block_size %d is none of 16, 32, 64, 128, 256", c->block_size);
    if (c->head_dim != 64 && c->head_dim != 128) FAIL("head_dim %d is neither 64 nor 128", c->head_dim);
    if (c->dtype != PLAID_BF16 && c->dtype != PLAID_FP16) FAIL("dtype %d is neither PLAID_BF16 nor PLAID_FP16", c->dtype);
    if (c->kv_heads < 1 || c->kv_heads > 65535) FAIL("kv_heads %d out of range", c->kv_heads);
    if (c->num_blocks < 0 || c->num_blocks > INT32_MAX) FAIL("num_blocks out of range");
    if (c->num_blocks > 0 && (!c->data || misaligned(c->data, 16))) FAIL("cache data is null or not 16-byte aligned");
    return PLAID_OK;
}

constexpr int UNITS = 256;             // compute units
constexpr float LEAST_SCALE = 1e-30f;  // that scores are multiplied with

struct Plan {
    bool few;
    int workers, waves, splits, q_splits, k_waves, k_splits;
    int64_t tiles, bytes;
    int64_t o_bytes, row_bytes, part_bytes, bias_bytes, k_bytes, q_bytes;
};

// Parts that an axis of `steps` steps is cut into, at least `least` of them a part, where `groups` workgroups of so many waves leave
// compute units empty: one of eight waves has room on each, two of four.  One part too many would start a second round.
constexpr int64_t split_count(int64_t groups, int waves, int64_t steps, int64_t least)
{
    int64_t s = UNITS * 8 / waves / (groups < 1 ? 1 : groups);
    if (s > steps / least) s = steps / least;
    return s < 1 ? 1 : s > 64 ? 64 : s;
}

// Which forward kernel takes a call whose requests have `rows` rows and `keys` keys on average.  One tile of 16 rows is always the
// few-row kernel's: the other leaves half of its 32 rows empty.  More rows it reads the same keys for once a tile, so it takes
// them while its workgroups all find room at once and have little to read; it then cuts the keys finer.  us, few and many:
//   16 heads on 4, D = 128, 4 requests of 64 tokens x 450 keys: 10.8 and 21.3;  x 2000: 31.6 and 29.5;  16 of 64 x 450: 37.2 and 29.0
//   12 heads on 12, D = 64, 4 requests of 128 tokens x 450 keys: 11.4 and 15.8;  of 64 x 2000: 23.9 and 22.2;  16 of 96 x 450: 26.2 and 23.0
//   paged, 32 heads on 8, 4 requests of 32 tokens x 2000 keys: 17.0 and 31.3;  16 of 8 x 8000: 52.4 and 93.2;  16 of 32 x 2000: 61.5 and 47.4
constexpr bool few_rows(int64_t rows, int64_t n, int64_t kv_heads, int64_t keys, int head_dim, int source)
{
    if (rows <= FEW_ROWS) return true;
    const bool paged = source == PLAID_SOURCE_PAGED;
    const int64_t groups = ceil_div(rows, FEW_ROWS) * n * kv_heads;
    return groups <= (paged || head_dim == 64 ? UNITS * 5 / 2 : UNITS) && groups * keys <= (paged ? 1 << 21 : 1 << 19);
}

// keys: of all requests; longest: that a request can have; usual: to reckon with
constexpr Plan plan_forward(const plaid_attention &a, int source, int64_t keys, int64_t longest, int64_t usual)
{
    Plan p = {};
    const int64_t group = a.heads / a.kv_heads, tokens = ceil_div(a.num_queries, a.n), rows = tokens * group;
    p.tiles = a.num_queries * group / FEW_ROWS + a.n;
    // its counts of steps are 32 bits wide
    p.few = few_rows(rows, a.n, a.kv_heads, usual, a.head_dim, source) && p.tiles * (longest / FEW_KEYS + 1) < INT32_MAX;
    if (p.few) {
        // One workgroup for each tile, no workers, nothing to join: 9.4 us in place of 11.0 at 1024 keys, 14.8 in place of 11.4 at 2048
        // for one request of 8 key heads; 34.6 in place of 39.5 at 2048 for 64 of them.  Packed keys: a request is taken to have at most
        // twice the mean, unless that could make it wait for eight times as many (75 us at 8192).
        const int64_t most = p.tiles * a.kv_heads >= 128 ? 2048 : 1024;
        if (longest <= most || (2 * usual <= most && longest <= 8 * most)) return p;
        const int64_t line = (ceil_div(keys, FEW_KEYS) + a.n) * ceil_div(rows < 1 ? 1 : rows, FEW_ROWS);
        const int64_t w = ceil_div(UNITS * FEW_PER_SIMD(a.head_dim, source), a.kv_heads);
        p.workers = (int)(w < line ? w : line);
        p.o_bytes = p.workers > 1 ? (int64_t)p.workers * 2 * a.kv_heads * FEW_ROWS * a.head_dim * 4 : 0;
        p.bytes = p.o_bytes + p.o_bytes / a.head_dim * 2;
        return p;
    }
    // 8 waves share a tile of keys among 256 rows: 488 us in place of 498 with 4 for 16 x 456 tokens of 16 heads on 6250 keys, 435 in place of
    // 507 where the tile comes out of the cache (6 x 850 tokens of 32 heads behind 4750)
    p.waves = rows > 128 ? 8 : 4;
    p.tiles = a.num_queries * group / (p.waves * 32) + a.n;
    p.splits = (int)split_count(ceil_div(rows, p.waves * 32) * a.n * a.kv_heads, p.waves, ceil_div(usual, MANY_KEYS), 4);
    p.o_bytes = p.splits > 1 ? (int64_t)p.splits * a.num_queries * a.heads * a.head_dim * 4 : 0;
    p.bytes = p.o_bytes + p.o_bytes / a.head_dim * 2;
    return p;
}

constexpr Plan plan_backward(const plaid_attention &a)
{
    Plan p = {};
    const int64_t group = a.heads / a.kv_heads, rows = ceil_div(a.num_queries, a.n) * group, keys = ceil_div(a.num_keys, a.n);
    // Workgroups of dk and dv, us with 8 and with 4 waves.  D = 128, 16 heads on 4: 16 x 456 rows on 6250 keys 1504 and 1552, 16 x 100 on 1000
    // 110 and 106.  D = 64, 12 heads on 12: 16 x 200 on 900 134 and 100, 8 x 500 on 3000 282 and 240: two workgroups of 4 on a unit do more.
    p.k_waves = a.head_dim == 128 && keys > 64 && rows > 128 ? 8 : 4;
    p.q_splits = (int)split_count(ceil_div(rows, 128) * a.n * a.kv_heads, 4, ceil_div(keys, 64), 4);
    p.k_splits = (int)split_count(ceil_div(keys, p.k_waves * 16) * a.n * a.kv_heads, p.k_waves, ceil_div(rows, 64), 4);
    p.row_bytes = round16(a.num_queries * a.heads * 4);  // delta, the rows' exponents
    // what delta was off by: of parts, with the corrected delta, or whether a workgroup's waves need a second pass
    p.part_bytes = p.q_splits > 1 ? round16(a.num_queries * a.heads * 8 * p.q_splits) + p.row_bytes : (a.num_queries * group / 128 + a.n) * a.kv_heads * 16;
    p.bias_bytes = round16((int64_t)p.k_splits * a.kv_heads * a.num_keys * 4);
    p.k_bytes = p.k_splits > 1 ? (int64_t)p.k_splits * a.num_keys * a.kv_heads * a.head_dim * 4 : 0;
    p.q_bytes = p.q_splits > 1 ? (int64_t)p.q_splits * a.num_queries * a.heads * a.head_dim * 4 : 0;
    p.bytes = 2 * p.row_bytes + p.part_bytes + p.bias_bytes + 2 * p.k_bytes + p.q_bytes;
    return p;
}

int check_shape(const plaid_attention *a)
{
    if (!a) FAIL("args is null");
    if (a->dtype != PLAID_BF16 && a->dtype != PLAID_FP16) FAIL("dtype %d is neither PLAID_BF16 nor PLAID_FP16", a->dtype);
    if (a->head_dim != 64 && a->head_dim != 128) FAIL("head_dim %d is neither 64 nor 128", a->head_dim);
    if (a->n < 1) FAIL("n %d: a call needs at least one request", a->n);
    if (a->kv_heads < 1 || a->kv_heads > 65535 || a->heads < 1 || a->heads % a->kv_heads) FAIL("heads %d is no multiple of kv_heads %d", a->heads, a->kv_heads);
    if (a->num_queries < 0 || a->num_keys < 0 || a->num_keys > (1 << 30)) FAIL("num_queries or num_keys out of range");
    const int64_t group = a->heads / a->kv_heads;
    if (a->num_queries > (1ll << 30) || group > 4096 || a->num_queries * group > (1ll << 30) || a->num_queries * group * group >= (1ll << 32))
        FAIL("too many query rows: %lld tokens of %d heads for a key head", (long long)a->num_queries, (int)group);
    return PLAID_OK;
}
int check_rows(const char *what, const void *p, int64_t token, int64_t head)
{
    if (!p || misaligned(p, 16)) FAIL("%s is null or not 16-byte aligned", what);
    if (token % 8 || head % 8) FAIL("the strides of %s are no multiples of 8 elements", what);
    if (token < 0 || token >= 1 << 24 || head < 0 || head >= 1 << 24) FAIL("a stride of %s is out of range", what);  // 64 rows lie within 32 bits
    return PLAID_OK;
}
// Pointers that any attention call reads; out is an input of the backward pass.
int check_queries(const plaid_attention *a)
{
    if (!a->q_offsets || misaligned(a->q_offsets, 8)) FAIL("q_offsets is null or misaligned");
    if (a->num_queries > 0) {
        if (const int rc = check_rows("q", a->q, a->q_token_stride, a->q_head_stride)) return rc;
        if (!a->out || misaligned(a->out, 16)) FAIL("out is null or not 16-byte aligned");
    }
    if (misaligned(a->lse, 8)) FAIL("lse is misaligned");
    return PLAID_OK;
}
int check_keys(const plaid_attention *a)
{
    if (!a->k_offsets || misaligned(a->k_offsets, 8)) FAIL("k_offsets is null or misaligned");
    if (a->num_keys > 0) {
        if (const int rc = check_rows("k", a->k, a->k_token_stride, a->k_head_stride)) return rc;
        if (const int rc = check_rows("v", a->v, a->v_token_stride, a->v_head_stride)) return rc;
    }
    if (misaligned(a->key_bias, 2)) FAIL("key_bias is misaligned");
    return PLAID_OK;
}
AttendArgs attend_args(const plaid_attention &a)
{
    AttendArgs x = {};
    x.q = (const char *)a.q, x.k = (const char *)a.k, x.v = (const char *)a.v, x.bias = (const char *)a.key_bias;
    x.q_offsets = a.q_offsets, x.k_offsets = a.k_offsets;
    x.out = (char *)a.out, x.lse = a.lse;
    x.num_queries = a.num_queries, x.num_keys = a.num_keys;
    x.q_token = 2 * a.q_token_stride, x.q_head = 2 * a.q_head_stride;
    x.k_token = 2 * a.k_token_stride, x.k_head = 2 * a.k_head_stride;
    x.v_token = 2 * a.v_token_stride, x.v_head = 2 * a.v_head_stride;
    x.n = a.n, x.heads = a.heads, x.kv_heads = a.kv_heads, x.group = a.heads / a.kv_heads;
    x.group_magic = x.group > 1 ? (uint32_t)(((1ull << 32) + x.group - 1) / x.group) : 0;
    x.scale = a.scale;
    x.splits = 1;
    return x;
}

int run_forward(const plaid_attention &a, AttendArgs &x, const Plan &p, int source, void *workspace, int64_t workspace_bytes, int device, void *stream)
{
    if (const int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
    const int64_t groups = p.few ? (p.workers ? p.workers : p.tiles) * a.kv_heads : p.tiles * a.kv_heads * p.splits;
    if (groups > INT32_MAX || p.tiles > INT32_MAX) FAIL("too much work for one call");
    if (a.num_queries == 0) return PLAID_OK;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    // the running maximum is that of q . k, so the factor is made positive and q carries its sign
    if (!(a.scale >= 0.0f)) x.negate_q = 0x80008000u, x.scale = -a.scale;
    // a factor of 0 would meet the infinities of keys that are hidden; beside this one every score that is not huge is nothing as well
    if (x.scale < LEAST_SCALE) x.scale = LEAST_SCALE;
    x.inv_scale = 1.0f / x.scale;
    x.part_o = (float *)workspace;
    x.part_lse = (float *)((char *)workspace + p.o_bytes);
    if (p.few) {
        plaid_launch_attend_few((hipStream_t)stream, x, a.dtype, a.head_dim, source, p.workers, p.tiles);
    } else {
        x.splits = p.splits;
        plaid_launch_attend_many((hipStream_t)stream, x, a.dtype, a.head_dim, source, p.waves, p.tiles);
    }
    return launched();
}

}  // namespace

extern "C" int plaid_block_tables_workspace(int32_t n, int64_t capacity, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (n < 1 || capacity < 0) FAIL("n or capacity out of range");
    *bytes = plaid_block_tables_scan_bytes(n, capacity);
    return PLAID_OK;
}

extern "C" int plaid_block_tables(const int32_t *lengths, const int32_t *added, int32_t n, int32_t *table, int64_t table_stride,
                                  int32_t max_blocks, const int32_t *free_blocks, int32_t n_free, int32_t block_size, int64_t *offsets,
                                  int32_t *totals, int32_t *positions, int64_t *slots, int64_t capacity, int64_t *blocks_wanted,
                                  void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (n < 1) FAIL("n %d: a call needs at least one request", n);
    if (!lengths || !added || !table || !offsets || !totals || !blocks_wanted) FAIL("null argument");
    if (!block_size_ok(block_size)) FAIL("block_size %d is none of 16, 32, 64, 128, 256", block_size);
    if (max_blocks < 1 || (int64_t)max_blocks * block_size > INT32_MAX) FAIL("max_blocks %d out of range", max_blocks);
    if (n > 1 && table_stride < max_blocks) FAIL("table_stride %lld is below max_blocks", (long long)table_stride);
    if (n_free < 0 || (n_free > 0 && !free_blocks)) FAIL("free_blocks is null");
    if (capacity < 0 || (capacity > 0 && (!positions || !slots))) FAIL("positions or slots is null");
    if (misaligned(positions, 16) || misaligned(slots, 16) || misaligned(offsets, 8) || misaligned(blocks_wanted, 8)) FAIL("misaligned output");
    const int64_t need = plaid_block_tables_scan_bytes(n, capacity);
    if (const int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    TablesArgs t = {};
    t.lengths = lengths, t.added = added, t.free_blocks = free_blocks;
    t.table = table, t.totals = totals, t.positions = positions, t.offsets = offsets, t.slots = slots, t.blocks_wanted = blocks_wanted;
    t.table_stride = table_stride, t.capacity = capacity;
    t.n = n, t.max_blocks = max_blocks, t.n_free = n_free, t.block_shift = __builtin_ctz((unsigned)block_size);
    t.scan = (int64_t *)workspace;
    plaid_launch_block_tables((hipStream_t)hip_stream, t);
    return launched();
}

extern "C" int plaid_cache_write(const plaid_paged_cache *cache, const void *k, const void *v, int64_t k_token_stride, int64_t k_head_stride,
                                 int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots, int64_t n, int device, void *hip_stream)
{
    if (const int rc = check_cache(cache)) return rc;
    if (n < 0 || n > (1ll << 31)) FAIL("n out of range");
    if (n == 0) return PLAID_OK;
    if (const int rc = check_rows("k", k, k_token_stride, k_head_stride)) return rc;
    if (const int rc = check_rows("v", v, v_token_stride, v_head_stride)) return rc;
    if (!slots || misaligned(slots, 8)) FAIL("slots is null or misaligned");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    plaid_launch_cache_write((hipStream_t)hip_stream, *cache, (const char *)k, (const char *)v, 2 * k_token_stride, 2 * k_head_stride, 2 * v_token_stride,
                             2 * v_head_stride, slots, n);
    return launched();
}

extern "C" int plaid_cache_read(const plaid_paged_cache *cache, const int64_t *slots, int64_t n, void *k, void *v, int device, void *hip_stream)
{
    if (const int rc = check_cache(cache)) return rc;
    if (n < 0 || n > (1ll << 31)) FAIL("n out of range");
    if (n == 0 || (!k && !v)) return PLAID_OK;
    if (misaligned(k, 16) || misaligned(v, 16)) FAIL("k or v is not 16-byte aligned");
    if (!slots || misaligned(slots, 8)) FAIL("slots is null or misaligned");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    plaid_launch_cache_read((hipStream_t)hip_stream, *cache, slots, n, (char *)k, (char *)v);
    return launched();
}

static int check_cached(const plaid_attention *args, int32_t max_blocks, int32_t block_size)
{
    if (const int rc = check_shape(args)) return rc;
    if (!block_size_ok(block_size)) FAIL("block_size %d is none of 16, 32, 64, 128, 256", block_size);
    if (max_blocks < 1 || (int64_t)max_blocks * block_size > (1 << 30)) FAIL("max_blocks %d out of range", max_blocks);
    return PLAID_OK;
}
static constexpr Plan plan_cached(const plaid_attention &a, int32_t max_blocks, int32_t block_size)
{
    const int64_t longest = (int64_t)max_blocks * block_size;
    return plan_forward(a, PLAID_SOURCE_PAGED, longest * a.n, longest, longest);
}

extern "C" int plaid_cached_attention_workspace(const plaid_attention *args, int32_t max_blocks, int32_t block_size, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (const int rc = check_cached(args, max_blocks, block_size)) return rc;
    *bytes = plan_cached(*args, max_blocks, block_size).bytes;
    return PLAID_OK;
}

extern "C" int plaid_cached_attention(const plaid_attention *args, const plaid_paged_cache *cache, const int32_t *table, int64_t table_stride,
                                      int32_t max_blocks, const int32_t *lengths, int32_t causal, void *workspace, int64_t workspace_bytes,
                                      int device, void *hip_stream)
{
    if (const int rc = check_cache(cache)) return rc;
    if (const int rc = check_cached(args, max_blocks, cache->block_size)) return rc;
    if (const int rc = check_queries(args)) return rc;
    if (args->kv_heads != cache->kv_heads || args->head_dim != cache->head_dim || args->dtype != cache->dtype)
        FAIL("kv_heads, head_dim or dtype of the queries is not the cache's");
    if (!table || !lengths || misaligned(table, 4) || misaligned(lengths, 4)) FAIL("table or lengths is null or misaligned");
    if (args->n > 1 && table_stride < max_blocks) FAIL("table_stride %lld is below max_blocks", (long long)table_stride);
    AttendArgs x = attend_args(*args);
    x.bias = nullptr;
    x.cache = cache->data, x.table = table, x.lengths = lengths, x.table_stride = table_stride, x.num_blocks = cache->num_blocks;
    x.max_blocks = max_blocks, x.block_shift = __builtin_ctz((unsigned)cache->block_size), x.causal = causal != 0;
    return run_forward(*args, x, plan_cached(*args, max_blocks, cache->block_size), PLAID_SOURCE_PAGED, workspace, workspace_bytes, device, hip_stream);
}

static constexpr Plan plan_cross(const plaid_attention &a)
{
    return plan_forward(a, a.key_bias ? PLAID_SOURCE_BIAS : PLAID_SOURCE_DENSE, a.num_keys, a.num_keys, ceil_div(a.num_keys, a.n));
}

extern "C" int plaid_cross_attention_workspace(const plaid_attention *args, int32_t backward, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (const int rc = check_shape(args)) return rc;
    *bytes = backward ? plan_backward(*args).bytes : plan_cross(*args).bytes;
    return PLAID_OK;
}

extern "C" int plaid_cross_attention(const plaid_attention *args, void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_shape(args)) return rc;
    if (const int rc = check_queries(args)) return rc;
    if (const int rc = check_keys(args)) return rc;
    AttendArgs x = attend_args(*args);
    return run_forward(*args, x, plan_cross(*args), x.bias ? PLAID_SOURCE_BIAS : PLAID_SOURCE_DENSE,
                       workspace, workspace_bytes, device, hip_stream);
}

extern "C" int plaid_cross_attention_backward(const plaid_attention *args, const void *d_out, void *dq, void *dk, void *dv, void *dbias,
                                              void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_shape(args)) return rc;
    if (const int rc = check_queries(args)) return rc;
    if (const int rc = check_keys(args)) return rc;
    if (args->num_queries > 0 && (!args->lse || !d_out || misaligned(d_out, 16))) FAIL("lse or d_out is null, or d_out is not 16-byte aligned");
    if (misaligned(dq, 16) || misaligned(dk, 16) || misaligned(dv, 16) || misaligned(dbias, 2)) FAIL("misaligned output");
    if (dbias && !args->key_bias) FAIL("dbias without key_bias");
    const Plan p = plan_backward(*args);
    if (const int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
    const int64_t group = args->heads / args->kv_heads;
    if ((args->num_queries * group / 128 + args->n) * args->kv_heads * p.q_splits > INT32_MAX ||
        (args->num_keys / (p.k_waves * 16) + args->n) * args->kv_heads * p.k_splits > INT32_MAX)
        FAIL("too much work for one call");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    GradArgs g = {};
    g.a = attend_args(*args);
    g.factor = args->scale;
    if (std::fabs(g.a.scale) < LEAST_SCALE) g.a.scale = std::copysign(LEAST_SCALE, g.a.scale);
    g.a.inv_scale = 1.0f / g.a.scale;
    g.d_out = (const char *)d_out;
    g.dq = (char *)dq, g.dk = (char *)dk, g.dv = (char *)dv, g.dbias = (char *)dbias;
    char *w = (char *)workspace;
    g.delta = (float *)w, g.exponent = (float *)(w + p.row_bytes), w += 2 * p.row_bytes;
    if (p.q_splits > 1) g.delta_sum = (float *)w, g.row_part = (float *)(w + p.row_bytes);
    else g.far = (int32_t *)w;
    w += p.part_bytes;
    g.dbias_part = dbias ? (float *)w : nullptr, w += p.bias_bytes;
    g.dk_part = p.k_bytes ? (float *)w : nullptr, w += p.k_bytes;
    g.dv_part = p.k_bytes ? (float *)w : nullptr, w += p.k_bytes;
    g.dq_part = p.q_bytes ? (float *)w : nullptr;
    plaid_launch_attend_grad((hipStream_t)hip_stream, g, args->dtype, args->head_dim, p.q_splits, p.k_waves, p.k_splits);
    return launched();
}
