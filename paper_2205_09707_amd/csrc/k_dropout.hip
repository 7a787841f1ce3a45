// Dropout whose mask is never stored.
#include "train.h"

// out_e = residual_e + kept_e x_e / (1 - T / 65536), with kept_e where the sixteen bits of element e are at least T.  The bits of eight
// elements are one value of Philox4x32-10 (Salmon, Moraes, Dror, Shaw, 2011): ten rounds of two products of 32 bits, which make the value
// a function of the counter (group of elements, call) and of the key (seed) alone, so that the backward pass forms the same mask again
// from the same two numbers.  They are read from memory: a captured graph gets new masks where the caller's program counts on.
// What was dropped does not reach the sum, so that an infinity there leaves no trace.
//
// Memory bounds it: 100000 x 2048 in bf16 take 211 us with a residual (1.23 GB, 5.8 TB/s), 128 without (819 MB, 6.4 TB/s).  With sixteen bits an element
// a value serves eight of them, 16 bytes of a thread, and its twenty products of 32 bits hide behind the loads; with 32 bits there would be twice as many.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0, c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1, c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
}

template <int DT, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(const char *x, const char *residual, int64_t n, uint32_t threshold, float factor, const int64_t *rng, char *out)
{
    const uint64_t seed = (uint64_t)uniform_load(rng), call = (uint64_t)uniform_load(rng + 1);
    const int64_t group = wide_block() * 256 + threadIdx.x, at = group * 8;
    if (at >= n) return;
    const int here = (int)min(n - at, (int64_t)8);
    const i32x4 raw = load_piece(x + 2 * at, 0, here);
    i32x4 other = {0, 0, 0, 0};
    if (RESIDUAL) other = load_piece(residual + 2 * at, 0, here);
    uint32_t c[4] = {(uint32_t)group, (uint32_t)((uint64_t)group >> 32), (uint32_t)call, (uint32_t)(call >> 32)};
    philox(c, (uint32_t)seed, (uint32_t)(seed >> 32));
    Eight v = unpack8<DT>(raw);
    const Eight r = unpack8<DT>(other);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? c[i / 2] >> 16 : c[i / 2] & 0xffff;
        const float kept = bits >= threshold ? v.x[i] * factor : 0.0f;
        v.x[i] = RESIDUAL ? r.x[i] + kept : kept;
    }
    store_piece(out + 2 * at, 0, here, pack8<DT>(v));
}

void plaid_launch_dropout(hipStream_t st, const char *x, const char *residual, int64_t n, uint32_t threshold, const int64_t *rng, char *out, int dtype)
{
    const float factor = threshold < 65536 ? 65536.0f / (float)(65536 - threshold) : 0.0f;
    const dim3 grid = wide_grid((n + 2047) / 2048);
#define GO(DT, R) dropout_kernel<DT, R><<<grid, 256, 0, st>>>(x, residual, n, threshold, factor, rng, out)
    if (dtype == PLAID_BF16) residual ? GO(PLAID_BF16, true) : GO(PLAID_BF16, false);
    else residual ? GO(PLAID_FP16, true) : GO(PLAID_FP16, false);
#undef GO
}
