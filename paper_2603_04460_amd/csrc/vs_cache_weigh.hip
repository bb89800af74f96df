// The weight that every token of the 4-bit paged cache gets from the last tokens' queries, added to what it had:
//   w_j = decay old_j + sum over the query heads of a KV head and over the rows r that see j of exp(scale q_r . K_j - lse_r)
// K of a block of 64 tokens is turned into bf16 once and stays in a wavefront's registers (scales in the conversion, exact), query rows pass by in tiles
// of 32: S = K Q^T, keys x rows, 32 x 32 x 16 matrix instructions.  A lane keeps the sums of its 32 keys over its rows, which meet across the
// lanes once at the end: no key belongs to two wavefronts, no atomics, the same call gives the same bits.
// The exponent is scale s - lse near zero for every weight that counts, of terms that are not: what the products' factor c = scale log2(e) loses by its
// rounding is put into lse's factor (c / scale), and what is left of lse's product goes to the row as a factor, which costs nothing since the sum is a
// multiply-add.
#include <float.h>

#include "vs_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;

struct WeighParams {
    CacheParams cache;
    const uint16_t* q;
    const float* lse;
    const float* old;              // or null: zeros
    float* weights;
    int64_t stride;
    int n_q, rows;                 // query rows of a KV head: group * n_q
    int fresh;                     // last tokens that have no weight yet
    float c, ratio, ratio_low;     // scale log2(e); c / scale in two terms
    float decay;
};

// sum over the 32 lanes of a half
__device__ __forceinline__ float half_sum(float x) {
    auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x = dpp(x, std::integral_constant<int, 0xB1>{});
    x = dpp(x, std::integral_constant<int, 0x4E>{});
    x = dpp(x, std::integral_constant<int, 0x141>{});
    x = dpp(x, std::integral_constant<int, 0x140>{});
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned r0 = r[0], r1 = r[1];
    return __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
}

__device__ __forceinline__ bf16x8 operand(uint4 x) { return __builtin_bit_cast(bf16x8, x); }

__global__ __launch_bounds__(64 * kWaves) void weigh_kernel(WeighParams p) {
    const int unit = blockIdx.y, b = unit / p.cache.kv_heads, h = unit - b * p.cache.kv_heads;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int block = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = cache_length_scalar(p.cache, b), first = block * kBlock;
    if (first >= len) return;
    const uint8_t* const from = cache_block(p.cache, b, h, block);
    float sum[2][16];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[t][e] = 0.0f;
    if (from) {
        bf16x8 k[2][8];                                    // channels 64 half + 8 j .. of token 32 t + col
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int token = 32 * t + col;
            const uint4* const codes = reinterpret_cast<const uint4*>(from + 64 * token + 32 * half);
            const uint4 x = codes[0], y = codes[1];
            const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const uint32_t e = from[kKScales + 4 * (16 * (2 * half + g) + (token & 15)) + (token >> 4)];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[t][4 * g + j] = operand(dequantise8(w[4 * g + j], __uint_as_float(e << 23)));
            }
        }
        const bool edge = first + kBlock - 1 > len - p.n_q;
        for (int at = 0; at < p.rows; at += 32) {
            const int row = min(at + col, p.rows - 1);
            const int64_t r = static_cast<int64_t>(unit) * p.rows + row;
            const uint16_t* const q = p.q + r * 128 + 64 * half;
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bf16x8 y = operand(*reinterpret_cast<const uint4*>(q + 8 * j));
#pragma unroll
                for (int t = 0; t < 2; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[t][j], y, s[t], 0, 0, 0);
            }
            // 2^(c s - high) factor; a row without a key has no weights
            const float lse = p.lse[r];
            float high = lse * p.ratio, factor = 1.0f;
            if (fabsf(high) < INFINITY) factor = __builtin_amdgcn_exp2f(-fmaf(lse, p.ratio_low, fmaf(lse, p.ratio, -high)));
            if (lse == -INFINITY) high = INFINITY;
            const int limit = at + col < p.rows ? len - p.n_q + row % p.n_q : -1;   // last key that the row sees
            const bool masked = edge || at + 32 > p.rows;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float x = fmaf(s[t][e], p.c, -high);
                    if (masked && first + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3) > limit) x = -INFINITY;
                    sum[t][e] = fmaf(__builtin_amdgcn_exp2f(x), factor, sum[t][e]);
                }
        }
    }
    // key 32 t + 8 (e / 4) + 4 half + e % 4 to the lane with col = 16 t + e
    float mine = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = half_sum(sum[t][e]);
            if (col == 16 * t + e) mine = x;
        }
    const int e = col & 15, j = first + 32 * (col >> 4) + 8 * (e >> 2) + 4 * half + (e & 3);
    if (j >= len) return;
    const int64_t at = unit * p.stride + j;
    if (p.old && p.decay != 0.0f && j < len - p.fresh) mine = fmaf(p.old[at], p.decay, mine);
    p.weights[at] = mine;
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_MAX_SEQ && q_heads % kv_heads == 0 && q_heads <= 4096 &&
           max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535 && q_heads / kv_heads * n_q <= INT32_MAX / 2;
}

}  // namespace

extern "C" size_t vs_cache_weigh_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    return 0;
}

extern "C" int vs_cache_weigh(const void* q, const float* lse, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens,
                              int64_t max_n, float scale, const float* old, float decay, int64_t fresh, float* weights, int64_t stride, void* ws,
                              size_t ws_bytes, void* stream) {
    if (!q || !lse || !weights || !vs::aligned16(q) || !vs::aligned16(lse) || !vs::aligned4(old) || !vs::aligned4(weights) || !vs::aligned16(ws))
        return VS_ERR_INVALID_ARG;
    WeighParams p;
    p.c = scale * 1.44269504088896340736f;
    if (q_heads <= 0 || n_q <= 0 || fresh < 0 || !(scale > 0.0f) || !(p.c < INFINITY) || !(p.c >= FLT_MIN) || !(decay >= 0.0f && decay <= 1.0f)) return VS_ERR_INVALID_ARG;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_UNSUPPORTED;
    const size_t units = static_cast<size_t>(batch) * cache->kv_heads;
    size_t bytes;
    if (stride < max_n || __builtin_mul_overflow(units * 4, static_cast<size_t>(stride), &bytes)) return VS_ERR_INVALID_ARG;
    if (ws_bytes < vs_cache_weigh_workspace(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.lse = lse;
    p.old = old;
    p.weights = weights;
    p.stride = stride;
    p.n_q = static_cast<int>(n_q);
    p.rows = static_cast<int>(q_heads / cache->kv_heads * n_q);
    p.fresh = static_cast<int>(fresh < max_n ? fresh : max_n);
    const double ratio = static_cast<double>(p.c) / scale;
    p.ratio = static_cast<float>(ratio);
    p.ratio_low = static_cast<float>(ratio - p.ratio);
    p.decay = decay;
    const unsigned blocks = static_cast<unsigned>((max_n + kBlock * kWaves - 1) / (kBlock * kWaves));
    hipLaunchKernelGGL(weigh_kernel, dim3(blocks, static_cast<unsigned>(units)), dim3(64 * kWaves), 0, static_cast<hipStream_t>(stream), p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}
