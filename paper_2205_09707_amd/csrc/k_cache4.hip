// The cache in four bits: writing keys and values to their slots, and reading them back.
#include "reader.h"

// 8 values of a lane are 16 bytes; four lanes share a scale.  The codes of 16-bit values leave at a quarter of what came in, so
// both directions are bound by the 16-bit side.  Value codes interleave four tokens: a thread that finds four tokens in a row
// of slots stores their bytes as one piece (16 bytes at D = 128), others byte by byte.  65003 tokens of 8 heads of 128, keys and values
// (266 MB of 16 bits, 71 of codes and scales): written in 75 us (4.5 TB/s), 87 between other calls, read back in 78; a decode step's 64 tokens 3.6 each.
template <int DT>
struct Limits {
    static constexpr int TOP = DT == PLAID_BF16 ? 126 : 14, LOWEST = DT == PLAID_BF16 ? -126 : -23, INF = DT == PLAID_BF16 ? 0x7f80 : 0x7c00;
};

struct CacheArgs {
    uint8_t *data;
    const char *k, *v;
    char *k_out, *v_out;
    int64_t k_token, k_head, v_token, v_head;  // bytes
    const int64_t *slots;
    int64_t n, num_blocks;
    int32_t kv_heads, block_shift;
};

// Codes of a lane's 8 values (4 bits each, in order) and the scale byte that its four lanes agree on.
template <int DT>
__device__ __forceinline__ uint32_t encode8(i32x4 x, int &scale)
{
    int top = 0;  // the largest magnitude's bits: a value that is not finite compares above all others
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7fff, (x[e] >> 16) & 0x7fff));
    top = max(top, __shfl_xor(top, 1));
    top = max(top, __shfl_xor(top, 2));
    // largest = f 2^n with f in [1/2, 1): within 6 2^e = 0.75 2^(e + 3) from e = n - 3 on where f <= 0.75
    const int bits = __float_as_int(unpack<DT>(top, 0));
    int e = (bits >> 23) - 129 + ((bits & 0x7fffff) > 0x400000);
    e = min(max(e, Limits<DT>::LOWEST), Limits<DT>::TOP);
    scale = top >= Limits<DT>::INF ? 255 : e + 127;
    const float power = __int_as_float((e + 127) << 23), most = e == Limits<DT>::TOP ? 3.0f * power : INFINITY;  // 4 2^TOP is not finite in the type
    uint32_t codes = 0;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(unpack<DT>(x[i >> 1], i & 1), -most), most);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], power, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], power, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], power, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], power, 3);
    return codes;
}

template <int DT, int D>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs c)
{
    constexpr int LANES = D / 8, TOKENS = 256 / LANES, G = D / 32;
    __shared__ uint32_t s_v[TOKENS][16];  // per token and dim % 16: a byte for each 32 dimensions
    __shared__ int64_t s_slot[TOKENS + 4];
    const int tok = threadIdx.x / LANES, l = threadIdx.x % LANES, head = blockIdx.y;
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS, t = t0 + tok, bs = 1ll << c.block_shift, region = bs * D * 17 / 16;
    int64_t slot = -1;
    i32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
    if (t < c.n) {
        slot = c.slots[t];
        if ((uint64_t)slot >= (uint64_t)(c.num_blocks << c.block_shift)) slot = -1;
        k = *(const i32x4 *)(c.k + t * c.k_token + head * c.k_head + l * 16);
        v = *(const i32x4 *)(c.v + t * c.v_token + head * c.v_head + l * 16);
    }
    if (l == 0) s_slot[tok] = slot;
    if (threadIdx.x < 4) s_slot[TOKENS + threadIdx.x] = -1;
    int ks, vs;
    const uint32_t kc = encode8<DT>(k, ks), vc = encode8<DT>(v, vs);
    const int in = (int)(slot & (bs - 1));
    uint8_t *p = c.data + ((slot >> c.block_shift) * c.kv_heads + head) * region;
    if (slot >= 0) {
        *(uint32_t *)(p + in * (D / 2) + l * 4) = kc;
        if ((l & 3) == 0) {
            p[bs * D + in * G + l / 4] = (uint8_t)ks;
            p[bs * D + bs * G + in * G + l / 4] = (uint8_t)vs;
        }
    }
    // dims 32 i + m and 32 i + 16 + m share a byte: lanes l and l ^ 2 have its halves; the lower lane of the two makes m .. m + 3
    const uint32_t other = __shfl_xor(vc, 2);
    {
        const int upper = (l >> 1) & 1;  // of the 16 dims' halves
        const uint32_t lo = upper ? other >> 16 : vc, hi = upper ? vc >> 16 : other;
        const int m = (l & 1) * 8 + upper * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) ((uint8_t *)&s_v[tok][m + j])[l >> 2] = (uint8_t)(((lo >> (4 * j)) & 15) | (((hi >> (4 * j)) & 15) << 4));
    }
    __syncthreads();
    for (int u = threadIdx.x; u < TOKENS * 16; u += 256) {
        const int y = u >> 4, m = u & 15;
        const int64_t s = s_slot[y];
        if (s < 0) continue;
        const int quad = (int)(s & 3), at = (int)(s & (bs - 1));
        // whole: the slots of the quad are those of four neighbouring tokens here
        const int lead = y - quad;
        const bool whole = lead >= 0 && s_slot[lead] == s - quad && s_slot[lead + 1] == s - quad + 1 && s_slot[lead + 2] == s - quad + 2 &&
                           s_slot[lead + 3] == s - quad + 3;
        uint8_t *to = c.data + ((s >> c.block_shift) * c.kv_heads + head) * region + bs * (D / 2) + (at >> 4) * (8 * D) + (((at >> 2) & 3) * 16 + m) * (D / 8);
        if (whole) {
            if (quad) continue;
            const uint32_t w0 = s_v[y][m], w1 = s_v[y + 1][m], w2 = s_v[y + 2][m], w3 = s_v[y + 3][m];
            // 4 x 4 bytes [token][i] -> [i][token]
            const uint32_t a = __builtin_amdgcn_perm(w1, w0, 0x05010400), b = __builtin_amdgcn_perm(w3, w2, 0x05010400);
            const uint32_t e = __builtin_amdgcn_perm(w1, w0, 0x07030602), f = __builtin_amdgcn_perm(w3, w2, 0x07030602);
            const int r0 = (int)__builtin_amdgcn_perm(b, a, 0x05040100), r1 = (int)__builtin_amdgcn_perm(b, a, 0x07060302);
            const int r2 = (int)__builtin_amdgcn_perm(f, e, 0x05040100), r3 = (int)__builtin_amdgcn_perm(f, e, 0x07060302);
            if constexpr (D == 128) *(i32x4 *)to = i32x4{r0, r1, r2, r3};
            else *(i32x2 *)to = i32x2{r0, r1};
        } else {
            const uint32_t w = s_v[y][m];
#pragma unroll
            for (int i = 0; i < G; ++i) to[i * 4 + quad] = (uint8_t)(w >> (8 * i));
        }
    }
}

// Value codes are read four tokens at a time where neighbours in the list are neighbours in a quad of the cache (the list's
// alignment is taken from the first token's slot): a lane gets 4 tokens x 8 dimensions and their 16 other halves from 8 words.
// Byte by byte, the same takes eight times the loads (100 us in place of 76 for 65003 tokens of 8 heads).
template <int DT, int D, int TOKENS>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs c)
{
    constexpr int LANES = D / 8, G = D / 32;
    __shared__ int64_t s_slot[TOKENS + 8];
    __shared__ uint8_t s_done[TOKENS];
    const int head = blockIdx.y;
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS, bs = 1ll << c.block_shift, region = bs * D * 17 / 16;
    const int count = (int)min((int64_t)TOKENS, c.n - t0);
    for (int i = threadIdx.x; i < TOKENS + 8; i += 256) {
        int64_t slot = i < count ? c.slots[t0 + i] : -1;
        if ((uint64_t)slot >= (uint64_t)(c.num_blocks << c.block_shift)) slot = -1;
        s_slot[i] = slot;
        if (i < TOKENS) s_done[i] = 0;
    }
    __syncthreads();
    auto cell_of = [&](int64_t slot) { return c.data + ((slot >> c.block_shift) * c.kv_heads + head) * region; };
    auto out_of = [&](char *out, int tok) { return out + ((t0 + tok) * c.kv_heads + head) * (D * 2); };
    if (c.v_out) {
        const int lead = (int)(-s_slot[0] & 3);
        for (int u = threadIdx.x; u < TOKENS / 4 * G * 2; u += 256) {
            const int quad = u / (G * 2), l = u % (G * 2), i = l >> 1, m = (l & 1) * 8, tok = lead + 4 * quad;
            const int64_t s = s_slot[tok];
            if (s < 0 || (s & 3) || s_slot[tok + 1] != s + 1 || s_slot[tok + 2] != s + 2 || s_slot[tok + 3] != s + 3) continue;
            if (l == 0) s_done[tok] = s_done[tok + 1] = s_done[tok + 2] = s_done[tok + 3] = 1;
            const int in = (int)(s & (bs - 1));
            const uint8_t *p = cell_of(s) + bs * (D / 2) + (in >> 4) * (8 * D) + (((in >> 2) & 3) * 16 + m) * (D / 8) + i * 4;
            const uint8_t *scales = cell_of(s) + bs * D + bs * G + in * G + i;
            int w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = *(const int *)(p + j * (D / 8));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float power = scale_power(scales[t * G], 0);
                i32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int x = t == 0   ? codes2<DT, 0>(w[2 * j], power)
                                  : t == 1 ? codes2<DT, 1>(w[2 * j], power)
                                  : t == 2 ? codes2<DT, 2>(w[2 * j], power)
                                           : codes2<DT, 3>(w[2 * j], power);
                    const int y = t == 0   ? codes2<DT, 0>(w[2 * j + 1], power)
                                  : t == 1 ? codes2<DT, 1>(w[2 * j + 1], power)
                                  : t == 2 ? codes2<DT, 2>(w[2 * j + 1], power)
                                           : codes2<DT, 3>(w[2 * j + 1], power);
                    lo[j] = (int)__builtin_amdgcn_perm(y, x, 0x05040100), hi[j] = (int)__builtin_amdgcn_perm(y, x, 0x07060302);
                }
                char *to = out_of(c.v_out, tok + t) + (32 * i + m) * 2;
                *(i32x4 *)to = lo;
                *(i32x4 *)(to + 32) = hi;
            }
        }
        __syncthreads();
    }
    for (int u = threadIdx.x; u < count * LANES; u += 256) {
        const int tok = u / LANES, l = u % LANES;
        const int64_t slot = s_slot[tok];
        const int in = (int)(slot & (bs - 1));
        const uint8_t *p = cell_of(slot);
        if (c.k_out) {
            i32x4 k{0, 0, 0, 0};
            if (slot >= 0) {
                const int w = *(const int *)(p + in * (D / 2) + l * 4);
                const float power = scale_power(p[bs * D + in * G + l / 4], 0);
                k = i32x4{codes2<DT, 0>(w, power), codes2<DT, 1>(w, power), codes2<DT, 2>(w, power), codes2<DT, 3>(w, power)};
            }
            *(i32x4 *)(out_of(c.k_out, tok) + l * 16) = k;
        }
        if (c.v_out && !s_done[tok]) {
            i32x4 v{0, 0, 0, 0};
            if (slot >= 0) {
                // dims 32 i + 8 (l % 4) .. + 7: m = 8 (l % 2) .. and the half that l / 2 % 2 names
                const uint8_t *q = p + bs * (D / 2) + (in >> 4) * (8 * D) + (((in >> 2) & 3) * 16 + 8 * (l & 1)) * (D / 8) + (l >> 2) * 4 + (in & 3);
                const float power = scale_power(p[bs * D + bs * G + in * G + l / 4], 0);
                const int half = ((l >> 1) & 1) * 4;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int w = ((q[2 * j * (D / 8)] >> half) & 15) | (((q[(2 * j + 1) * (D / 8)] >> half) & 15) << 4);
                    v[j] = codes2<DT, 0>(w, power);
                }
            }
            *(i32x4 *)(out_of(c.v_out, tok) + l * 16) = v;
        }
    }
}

static CacheArgs cache_args(const plaid_paged_cache &c, const int64_t *slots, int64_t n)
{
    CacheArgs a = {};
    a.data = c.data;
    a.slots = slots;
    a.n = n;
    a.num_blocks = c.num_blocks;
    a.kv_heads = c.kv_heads;
    a.block_shift = __builtin_ctz((unsigned)c.block_size);
    return a;
}
void plaid_launch_cache_write(hipStream_t st, const plaid_paged_cache &c, const char *k, const char *v, int64_t k_token, int64_t k_head,
                              int64_t v_token, int64_t v_head, const int64_t *slots, int64_t n)
{
    CacheArgs a = cache_args(c, slots, n);
    a.k = k, a.v = v, a.k_token = k_token, a.k_head = k_head, a.v_token = v_token, a.v_head = v_head;
    const int tokens = c.head_dim == 128 ? 16 : 32;
    const dim3 grid((unsigned)((n + tokens - 1) / tokens), (unsigned)c.kv_heads), block(256);
    if (c.dtype == PLAID_BF16) {
        if (c.head_dim == 128) cache_write_kernel<PLAID_BF16, 128><<<grid, block, 0, st>>>(a);
        else cache_write_kernel<PLAID_BF16, 64><<<grid, block, 0, st>>>(a);
    } else {
        if (c.head_dim == 128) cache_write_kernel<PLAID_FP16, 128><<<grid, block, 0, st>>>(a);
        else cache_write_kernel<PLAID_FP16, 64><<<grid, block, 0, st>>>(a);
    }
}
template <int DT, int D>
static void launch_read(hipStream_t st, const CacheArgs &a)
{
    // 64 tokens fill a workgroup's lanes with quads; where that leaves most of the chip idle, 16 (256 tokens of 8 heads: 3.4 us in place of 6.4)
    if (a.n * a.kv_heads >= 64 * 1024) cache_read_kernel<DT, D, 64><<<dim3((unsigned)((a.n + 63) / 64), (unsigned)a.kv_heads), dim3(256), 0, st>>>(a);
    else cache_read_kernel<DT, D, 16><<<dim3((unsigned)((a.n + 15) / 16), (unsigned)a.kv_heads), dim3(256), 0, st>>>(a);
}
void plaid_launch_cache_read(hipStream_t st, const plaid_paged_cache &c, const int64_t *slots, int64_t n, char *k, char *v)
{
    CacheArgs a = cache_args(c, slots, n);
    a.k_out = k, a.v_out = v;
    if (c.dtype == PLAID_BF16) {
        if (c.head_dim == 128) launch_read<PLAID_BF16, 128>(st, a);
        else launch_read<PLAID_BF16, 64>(st, a);
    } else {
        if (c.head_dim == 128) launch_read<PLAID_FP16, 128>(st, a);
        else launch_read<PLAID_FP16, 64>(st, a);
    }
}
