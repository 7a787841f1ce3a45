// C entry points of a reader's training step around its attention (include/plaid.h): argument checks, how the work is cut, workspaces.
#include <cmath>

#include "api_common.h"
#include "train.h"

namespace {

int check_dtype(int32_t dtype)
{
    if (dtype != PLAID_BF16 && dtype != PLAID_FP16) FAIL("dtype %d is neither PLAID_BF16 nor PLAID_FP16", dtype);
    return PLAID_OK;
}
constexpr int UNITS = 256;  // compute units
constexpr int64_t MOST_ROWS = 1ll << 30, MOST_STRIDE = 1ll << 32, MOST_VALUES = 1ll << 40;

int check_table(int64_t n, int64_t vocabulary, int32_t width, const int64_t *ids, int32_t dtype)
{
    if (const int rc = check_dtype(dtype)) return rc;
    if (n < 0 || n > MOST_ROWS) FAIL("n %lld out of range", (long long)n);
    if (vocabulary < 1 || vocabulary > MOST_ROWS) FAIL("vocabulary %lld out of range", (long long)vocabulary);
    if (width < 1 || width > (1 << 20)) FAIL("width %d out of range", width);
    if (vocabulary * width > MOST_VALUES || n * width > MOST_VALUES) FAIL("a table or result of more than 2^40 values");
    if (n > 0 && (!ids || misaligned(ids, 8))) FAIL("ids is null or misaligned");
    return PLAID_OK;
}

struct EmbedPlan {
    int32_t bits, passes, digit, chunk;
    int64_t tiles, key_bytes, count_bytes, begin_bytes, part_bytes, bytes;
};
EmbedPlan plan_embedding(int64_t n, int64_t vocabulary, int32_t width)
{
    EmbedPlan p = {};
    if (n == 0) {  // the gradient is filled with zeros
        p.bytes = p.begin_bytes = 16;
        return p;
    }
    p.bits = 64 - __builtin_clzll((unsigned long long)vocabulary);  // keys are 0 .. vocabulary
    p.passes = (int32_t)ceil_div(p.bits, 9);
    p.digit = (int32_t)ceil_div(p.bits, p.passes);
    p.tiles = ceil_div(n, SORT_TILE);
    // Chunks: as many teams of threads as fill the chip, up to 16384 for narrow rows, at least 2048; their sums are added up one after another where
    // one token has them all.  (200000 tokens of 64 columns: 75 us with 2048 chunks, 23 with 16384.)
    int64_t lanes = 1;
    while (lanes < 256 && lanes * 8 < width) lanes *= 2;
    const int64_t most = (1 << 17) / lanes;
    p.chunk = (int32_t)ceil_div(n, most < 2048 ? 2048 : most > 16384 ? 16384 : most);
    if (p.chunk < 8) p.chunk = 8;
    p.key_bytes = round16(n * 4);
    p.count_bytes = n > SORT_ONE ? round16(((p.tiles + 1) << p.digit) * 4) : 0;
    const int64_t chunks = ceil_div(n, p.chunk);
    p.begin_bytes = 16 + round16(chunks * 4);
    p.part_bytes = chunks > 1 ? chunks * 2 * ((width + 7) / 8 * 8) * 4 : 0;
    p.bytes = (n > SORT_ONE ? 4 : 2) * p.key_bytes + p.count_bytes + p.begin_bytes + p.part_bytes;
    return p;
}

int check_norm(int64_t rows, int32_t width, int32_t dtype)
{
    if (const int rc = check_dtype(dtype)) return rc;
    if (rows < 0 || rows > MOST_ROWS) FAIL("rows %lld out of range", (long long)rows);
    if (width < 1 || width > NORM_WIDEST) FAIL("width %d is not in 1 .. %d", width, NORM_WIDEST);
    return PLAID_OK;
}
int check_stride(const char *what, int64_t stride)
{
    if (stride < 0 || stride >= MOST_STRIDE) FAIL("the stride of %s is out of range", what);
    return PLAID_OK;
}
// Workgroups that go over the rows: teams of as many threads as a row has pieces of eight elements (as the launch has them), and at least two
// rows a team.
int norm_workers(int64_t rows, int32_t width)
{
    const int pieces = (width + 7) / 8, lanes = pieces == 1 ? 1 : pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : pieces <= 192 ? 64 : 256;
    const int64_t teams = 256 / lanes, most = width <= 2048 ? 1024 : width <= 8192 ? 512 : 256, want = ceil_div(rows, teams * 2);
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

struct LossPlan {
    bool few;
    int entries;
    int64_t padded_rows, pitch, columns, piece;
    int64_t list_bytes, row_bytes, packed_bytes, scaled_bytes, part_bytes, running_bytes, own_bytes, gradient_bytes, rest_bytes, reach_bytes, d_part_bytes, w_part_bytes, bytes;
};
LossPlan plan_loss(const plaid_token_loss &a, bool backward)
{
    LossPlan p = {};
    // Tiles of few rows: up to 128 rows, and where all of them then find room on the chip at once, in place of 256 entries and 256 rows.  Of 64 entries
    // where that is so, else of more, so that fewer workgroups read the rows.  us of a forward call by entries of a tile (64, 128 or 256, large):
    //   16 rows on 40000 entries, width 1024: 16.3, 17.1;  48 on 40000: 18.2, 19.3;  48 on 50021: 23.9, 20.9;  90 on 50000: 49, 23, 31
    //   1000 on 2600, width 512: 19, 22, 30;  500 on 11000: 29, 25, 32;  400 on 16000: 32, 27, 31;  250 on 40000: 42, 38, 33
    //   2000 on 2000, width 1024: 27, 32, 46;  200 on 30000: 46, 36, 44;  200 on 50000: 73, 57, 46
    const int64_t row_tiles = ceil_div(a.rows, LOSS_FEW), tiles = ceil_div(a.vocabulary, 64) * row_tiles;
    const int64_t stage = 3 * (64 + 16 * ceil_div(a.rows < LOSS_FEW ? a.rows : LOSS_FEW, 16)) * 128, resident = UNITS * (160 * 1024 / (stage + 2048));
    p.few = row_tiles <= 1 || tiles <= resident || ceil_div(a.vocabulary, 256) * row_tiles <= UNITS;
    p.entries = tiles <= resident ? 64 : a.rows <= 64 ? 128 : 256;
    if (p.few && !backward) {
        p.padded_rows = a.rows;
        p.part_bytes = round16(ceil_div(a.vocabulary, p.entries) * p.padded_rows * 8);
        p.own_bytes = round16(p.padded_rows * 4);
        p.bytes = p.part_bytes + p.own_bytes;
        return p;
    }
    p.padded_rows = ceil_div(a.rows < 1 ? 1 : a.rows, LOSS_TILE) * LOSS_TILE;
    p.pitch = ceil_div(a.width, LOSS_STEP) * LOSS_STEP;
    p.columns = ceil_div(a.width, LOSS_TILE) * LOSS_TILE;
    p.list_bytes = 16 + round16(a.rows * 4);
    p.row_bytes = round16(p.padded_rows * (int64_t)sizeof(LossRow));
    p.packed_bytes = p.padded_rows * p.pitch * 2;
    // pieces of the vocabulary whose statistics (forward) or gradients of the scores (backward) take so much of the workspace, all of a size
    const int64_t room = backward ? (512ll << 20) / (p.padded_rows * 2) : (64ll << 20) / (p.padded_rows * 8) * LOSS_PART;
    int64_t piece = room / LOSS_TILE * LOSS_TILE;
    if (piece < LOSS_TILE) piece = LOSS_TILE;
    const int64_t pieces = ceil_div(a.vocabulary, piece);
    p.piece = ceil_div(ceil_div(a.vocabulary, pieces), LOSS_TILE) * LOSS_TILE;
    if (backward) {
        p.gradient_bytes = p.padded_rows * p.piece * 2;
        p.scaled_bytes = p.padded_rows * p.columns * 2;
        p.rest_bytes = p.padded_rows * 8;
        p.reach_bytes = a.dtype == PLAID_FP16 ? p.padded_rows * 4 : 0;
        p.d_part_bytes = loss_hidden_parts(p.padded_rows, p.columns, ceil_div(p.piece, LOSS_STEP)) * (LOSS_TILE * LOSS_TILE * 4);
        p.w_part_bytes = loss_weight_parts(p.padded_rows, p.columns, ceil_div(p.piece, LOSS_STEP)) * (LOSS_TILE * LOSS_TILE * 4);
        p.bytes = p.list_bytes + p.row_bytes + p.packed_bytes + p.scaled_bytes + p.gradient_bytes + p.rest_bytes + p.reach_bytes + p.d_part_bytes + p.w_part_bytes;
    } else {
        p.part_bytes = p.piece / LOSS_PART * p.padded_rows * 8;
        p.running_bytes = p.padded_rows * 8;
        p.own_bytes = p.padded_rows * 4;
        p.bytes = p.list_bytes + p.row_bytes + p.packed_bytes + p.part_bytes + p.running_bytes + p.own_bytes;
    }
    return p;
}

int check_loss_shape(const plaid_token_loss *a)
{
    if (!a) FAIL("args is null");
    if (const int rc = check_dtype(a->dtype)) return rc;
    if (a->rows < 0 || a->rows > (1 << 24)) FAIL("rows %lld out of range", (long long)a->rows);
    if (a->vocabulary < 1 || a->vocabulary > (1 << 27)) FAIL("vocabulary %lld out of range", (long long)a->vocabulary);
    if (a->width < 8 || a->width > 16384 || a->width % 8) FAIL("width %d is no multiple of 8 in 8 .. 16384", a->width);
    return PLAID_OK;
}
int check_loss_rows(const char *what, const void *p, int64_t stride)
{
    if (!p || misaligned(p, 16)) FAIL("%s is null or not 16-byte aligned", what);
    if (stride < 0 || stride % 8 || stride >= 1 << 24) FAIL("the stride of %s is no multiple of 8 in [0, 2^24)", what);
    return PLAID_OK;
}
int check_loss(const plaid_token_loss *a)
{
    if (const int rc = check_loss_shape(a)) return rc;
    if (const int rc = check_loss_rows("weight", a->weight, a->weight_stride)) return rc;
    if (a->rows > 0) {
        if (const int rc = check_loss_rows("hidden", a->hidden, a->hidden_stride)) return rc;
        if (!a->targets || misaligned(a->targets, 8)) FAIL("targets is null or misaligned");
    }
    if (misaligned(a->loss, 4) || misaligned(a->lse, 8)) FAIL("loss or lse is misaligned");
    return PLAID_OK;
}
// Arguments with the workspace laid out.
LossArgs loss_args(const plaid_token_loss &a, const LossPlan &p, void *workspace, bool backward)
{
    LossArgs x = {};
    x.hidden = (const char *)a.hidden, x.weight = (const char *)a.weight, x.targets = a.targets;
    x.loss = a.loss, x.lse = a.lse;
    x.rows = a.rows, x.vocabulary = a.vocabulary, x.hidden_stride = 2 * a.hidden_stride, x.weight_stride = 2 * a.weight_stride;
    x.width = a.width, x.scale = a.scale;
    x.padded_rows = (int32_t)p.padded_rows, x.pitch = (int32_t)p.pitch, x.columns = (int32_t)p.columns, x.hidden_steps = (int32_t)ceil_div(p.piece, LOSS_STEP);
    char *w = (char *)workspace;
    if (backward || !p.few) {
        x.state = (int32_t *)w, x.list = (int32_t *)(w + 16), w += p.list_bytes;
        x.row = (LossRow *)w, w += p.row_bytes;
        x.packed = w, w += p.packed_bytes;
        if (backward) {
            x.scaled = w, w += p.scaled_bytes;
            x.gradient = w, w += p.gradient_bytes;
            x.target = (int32_t *)w, x.rest = (float *)w + p.padded_rows, w += p.rest_bytes;
            x.reach = p.reach_bytes ? (int32_t *)w : nullptr, w += p.reach_bytes;
            x.d_part = (float *)w, w += p.d_part_bytes;
            x.w_part = p.w_part_bytes ? (float *)w : nullptr;
        }
    }
    if (!backward) {
        x.part = (float2 *)w, w += p.part_bytes;
        x.running = (float2 *)w, w += p.running_bytes;
        x.own = (float *)w;
    }
    return x;
}

}  // namespace

extern "C" int plaid_embedding(const void *table, int64_t table_stride, int64_t vocabulary, int32_t width, const int64_t *ids, int64_t n, float scale,
                               void *out, int32_t dtype, int device, void *hip_stream)
{
    if (const int rc = check_table(n, vocabulary, width, ids, dtype)) return rc;
    if (n == 0) return PLAID_OK;
    if (const int rc = check_stride("table", table_stride)) return rc;
    if (!table || misaligned(table, 2) || !out || misaligned(out, 16)) FAIL("table or out is null or misaligned");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    EmbedArgs e = {};
    e.table = (const char *)table, e.out = (char *)out, e.ids = ids;
    e.n = n, e.vocabulary = vocabulary, e.table_stride = 2 * table_stride, e.width = width, e.scale = scale;
    plaid_launch_embedding((hipStream_t)hip_stream, e, dtype);
    return launched();
}

extern "C" int plaid_embedding_backward_workspace(int64_t n, int64_t vocabulary, int32_t width, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (n < 0 || n > MOST_ROWS || vocabulary < 1 || vocabulary > MOST_ROWS || width < 1 || width > (1 << 20) || vocabulary * width > MOST_VALUES || n * width > MOST_VALUES)
        FAIL("n, vocabulary or width out of range");
    *bytes = plan_embedding(n, vocabulary, width).bytes;
    return PLAID_OK;
}

extern "C" int plaid_embedding_backward(const void *d_out, int64_t d_out_stride, int64_t vocabulary, int32_t width, const int64_t *ids, int64_t n, float scale,
                                        int32_t add, void *d_table, int32_t dtype, void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_table(n, vocabulary, width, ids, dtype)) return rc;
    if (n > 0 && (!d_out || misaligned(d_out, 2))) FAIL("d_out is null or misaligned");
    if (const int rc = check_stride("d_out", d_out_stride)) return rc;
    if (!d_table || misaligned(d_table, 2)) FAIL("d_table is null or misaligned");
    const EmbedPlan p = plan_embedding(n, vocabulary, width);
    if (const int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    EmbedArgs e = {};
    e.d_out = (const char *)d_out, e.d_table = (char *)d_table, e.ids = ids;
    e.n = n, e.vocabulary = vocabulary, e.d_out_stride = 2 * d_out_stride, e.width = width, e.add = add != 0, e.scale = scale;
    e.bits = p.bits, e.passes = p.passes, e.digit = p.digit, e.chunk = p.chunk;
    char *w = (char *)workspace;
    e.keys[0] = (int32_t *)w, w += p.key_bytes, e.places[0] = (int32_t *)w, w += p.key_bytes;
    if (n > SORT_ONE) {
        e.keys[1] = (int32_t *)w, w += p.key_bytes, e.places[1] = (int32_t *)w, w += p.key_bytes;
        e.sorted = (p.passes - 1) & 1;
        e.counts = (int32_t *)w, e.totals = e.counts + (p.tiles << p.digit), w += p.count_bytes;
    }
    e.shared = (int32_t *)w, e.begins = (int32_t *)(w + 16), w += p.begin_bytes;
    e.part = (float *)w;
    plaid_launch_embedding_backward((hipStream_t)hip_stream, e, dtype);
    return launched();
}

extern "C" int plaid_dropout(const void *x, const void *residual, int64_t n, float p, const int64_t *rng, void *out, int32_t dtype, int device,
                             void *hip_stream)
{
    if (const int rc = check_dtype(dtype)) return rc;
    if (n < 0 || n > (1ll << 40)) FAIL("n %lld out of range", (long long)n);
    if (!(p >= 0.0f && p <= 1.0f)) FAIL("p %g is not in [0, 1]", (double)p);
    if (n == 0) return PLAID_OK;
    if (!x || misaligned(x, 2) || !out || misaligned(out, 2) || misaligned(residual, 2)) FAIL("x or out is null, or an array is misaligned");
    if (!rng || misaligned(rng, 8)) FAIL("rng is null or misaligned");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    plaid_launch_dropout((hipStream_t)hip_stream, (const char *)x, (const char *)residual, n, (uint32_t)std::floor(65536.0 * (double)p + 0.5), rng, (char *)out, dtype);
    return launched();
}

extern "C" int plaid_layer_norm(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t rows, int32_t width, float eps, void *out,
                                float *statistics, int32_t dtype, int device, void *hip_stream)
{
    if (const int rc = check_norm(rows, width, dtype)) return rc;
    if (!(eps >= 0.0f)) FAIL("eps %g is negative", (double)eps);
    if (rows == 0) return PLAID_OK;
    if (const int rc = check_stride("x", x_stride)) return rc;
    if (!x || misaligned(x, 2) || !out || misaligned(out, 2) || misaligned(weight, 2) || misaligned(bias, 2) || misaligned(statistics, 8))
        FAIL("x or out is null, or an array is misaligned");
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    NormArgs a = {};
    a.x = (const char *)x, a.weight = (const char *)weight, a.bias = (const char *)bias, a.out = (char *)out, a.statistics = statistics;
    a.rows = rows, a.x_stride = 2 * x_stride, a.width = width, a.eps = eps;
    plaid_launch_layer_norm((hipStream_t)hip_stream, a, dtype);
    return launched();
}

extern "C" int plaid_layer_norm_backward_workspace(int64_t rows, int32_t width, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (const int rc = check_norm(rows, width, PLAID_BF16)) return rc;
    *bytes = (int64_t)norm_workers(rows, width) * 2 * width * 4;
    return PLAID_OK;
}

extern "C" int plaid_layer_norm_backward(const void *d_out, int64_t d_out_stride, const void *x, int64_t x_stride, const void *weight,
                                         const float *statistics, int64_t rows, int32_t width, void *dx, void *dweight, void *dbias, int32_t dtype,
                                         void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_norm(rows, width, dtype)) return rc;
    if (const int rc = check_stride("d_out", d_out_stride)) return rc;
    if (const int rc = check_stride("x", x_stride)) return rc;
    if (rows > 0 && (!d_out || misaligned(d_out, 2) || !x || misaligned(x, 2))) FAIL("d_out or x is null or misaligned");
    if (rows > 0 && (!statistics || misaligned(statistics, 8))) FAIL("statistics is null or misaligned");
    if (misaligned(weight, 2) || misaligned(dx, 2) || misaligned(dweight, 2) || misaligned(dbias, 2)) FAIL("an array is misaligned");
    if (dweight && !weight) FAIL("dweight without weight");
    const int workers = norm_workers(rows, width);
    const bool sums = dweight || dbias;
    if (sums)
        if (const int rc = check_workspace(workspace, workspace_bytes, (int64_t)workers * 2 * width * 4)) return rc;
    if (!sums && (!dx || rows == 0)) return PLAID_OK;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    NormArgs a = {};
    a.x = (const char *)x, a.weight = (const char *)weight, a.d_out = (const char *)d_out, a.statistics = (float *)statistics;
    a.dx = (char *)dx, a.dweight = (char *)dweight, a.dbias = (char *)dbias;
    a.rows = rows, a.x_stride = 2 * x_stride, a.d_out_stride = 2 * d_out_stride, a.width = width, a.workers = workers;
    a.part = sums ? (float *)workspace : nullptr;
    plaid_launch_layer_norm_backward((hipStream_t)hip_stream, a, dtype);
    return launched();
}

extern "C" int plaid_cross_entropy_workspace(const plaid_token_loss *args, int32_t backward, int64_t *bytes)
{
    if (!bytes) FAIL("bytes is null");
    if (const int rc = check_loss_shape(args)) return rc;
    *bytes = args->rows == 0 && !backward ? 0 : plan_loss(*args, backward != 0).bytes;
    return PLAID_OK;
}

extern "C" int plaid_cross_entropy(const plaid_token_loss *args, void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_loss(args)) return rc;
    if (args->rows == 0) return PLAID_OK;
    if (!args->loss) FAIL("loss is null");
    const LossPlan p = plan_loss(*args, false);
    if (const int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    const hipStream_t st = (hipStream_t)hip_stream;
    LossArgs x = loss_args(*args, p, workspace, false);
    if (p.few) {
        x.last = 1;
        plaid_launch_loss_few(st, x, args->dtype, p.entries, false);
        plaid_launch_loss_join(st, x, (int)ceil_div(x.vocabulary, p.entries), false);
        return launched();
    }
    plaid_launch_loss_pack(st, x, args->dtype, false);
    for (x.first = 0; x.first < x.vocabulary; x.first += p.piece) {
        x.piece = (int32_t)(x.vocabulary - x.first < p.piece ? x.vocabulary - x.first : p.piece);
        x.last = x.first + p.piece >= x.vocabulary;
        plaid_launch_loss_scores(st, x, args->dtype, false);
        plaid_launch_loss_join(st, x, (int)ceil_div(x.piece, LOSS_TILE) * (LOSS_TILE / LOSS_PART), true);
    }
    return launched();
}

extern "C" int plaid_cross_entropy_backward(const plaid_token_loss *args, const float *d_loss, int64_t d_loss_stride, void *d_hidden, void *d_weight,
                                            void *workspace, int64_t workspace_bytes, int device, void *hip_stream)
{
    if (const int rc = check_loss(args)) return rc;
    if (args->rows > 0 && (!args->lse || !d_loss || misaligned(d_loss, 4))) FAIL("lse or d_loss is null, or d_loss is misaligned");
    if (d_loss_stride != 0 && d_loss_stride != 1) FAIL("the stride of d_loss is neither 0 nor 1");
    if (misaligned(d_hidden, 16) || misaligned(d_weight, 16)) FAIL("misaligned output");
    const LossPlan p = plan_loss(*args, true);
    if (const int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
    if (!d_weight && (!d_hidden || args->rows == 0)) return PLAID_OK;
    const OnDevice guard(device);
    if (!guard.ok) return plaid_fail(PLAID_EHIP, "device %d cannot be used", device);
    const hipStream_t st = (hipStream_t)hip_stream;
    LossArgs x = loss_args(*args, p, workspace, true);
    x.d_loss = d_loss, x.d_loss_stride = 4 * d_loss_stride;
    x.d_hidden = args->rows > 0 ? (char *)d_hidden : nullptr, x.d_weight = (char *)d_weight;
    if (!d_weight) x.reach = nullptr;
    plaid_launch_loss_pack(st, x, args->dtype, true);
    for (x.first = 0; x.first < x.vocabulary; x.first += p.piece) {
        x.piece = (int32_t)(x.vocabulary - x.first < p.piece ? x.vocabulary - x.first : p.piece);
        x.last = x.first + p.piece >= x.vocabulary;
        if (p.few) plaid_launch_loss_few(st, x, args->dtype, p.entries, true);
        else plaid_launch_loss_scores(st, x, args->dtype, true);
        plaid_launch_loss_gradients(st, x, args->dtype);
        plaid_launch_loss_gradients_join(st, x, args->dtype);
    }
    return launched();
}
