// Attention of a chunk of new tokens over the 4-bit paged cache, more rows than vs_cache_attend takes.
//   o = softmax(scale q K^T) V over the keys up to the query's own position
// A workgroup has 256 query rows of a KV head, eight row blocks of 32 (hc query heads times 8 / hc stretches of 32 tokens), two to a wavefront:
//   S^T = K Q^T (keys x rows, bf16),  O^T = V^T P^T (channels x rows, fp16), 32 x 32 x 16 matrix instructions
// A block of 64 keys is turned into 16-bit numbers in LDS by all four wavefronts: K in bf16 with its scales (exact); V in fp16.  A wavefront has the
// 32 channels of V that share scales and holds their unit 2^(R - 127), R at least the largest scale byte so far: an element is code 2^(E - R + 13), exact
// for E from R - 27 to R.  What lies below, and groups that are not finite, stays out of the tile and is added to the rows that see it
// in fp32; when R grows, everybody's sums are scaled.  Weights are held as 128 p (up to 2^15: the running maximum may be exceeded by 2^8) in fp16,
// 11 significant bits, which is why V is fp16: weights of 8 bits would double the rounding error of the output.
// The rows of a K tile stand in LDS in the order (bits 3 and 4 of a key's number exchanged) in which a lane of S^T holds the weights that
// the second product wants beside one word of V's codes, eight tokens of a channel: a word becomes one 16-byte operand.
#include <float.h>

#include "vs_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kUnitRows = 256;
constexpr int kTileBytes = kBlock * 256;                   // K or V of a block in 16 bits
constexpr float kGrown = 8.0f;                             // log2 units by which a score may exceed the running maximum
constexpr float kLift = 7.0f;                              // weights are held times 2^7
constexpr int kTop = 13;                                   // fp16 exponent of a code with E = R: 6 * 2^13 < 65504
constexpr int kSpan = 27;                                  // E from R - 27 (2^-14 in fp16) to R

struct PrefillParams {
    CacheParams cache;
    const uint16_t* q;
    uint16_t* o;
    float* lse;
    int q_heads, n_q, group, hc, tok;      // tok: tokens of a unit, 256 / hc
    int tiles;                             // units of a head chunk
    float c;                               // scale * log2(e)
};

__device__ __forceinline__ float half_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const unsigned a = r[0], b = r[1];
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}

// wavefront maximum of whole numbers >= 0
__device__ __forceinline__ int wave_max_int(int x) { return static_cast<int>(wave_max(static_cast<float>(x))); }

struct Raw {
    uint4 k, v, ve;
    uint32_t ke;
};

struct Tiles {
    uint8_t k[2][kTileBytes];
    uint8_t v[2][kTileBytes];
    int unit_of[2][4];                     // R of the buffer's block
    int event[2];                          // block whose R or V needs more than the products
};

__device__ __forceinline__ int row_of_key(int key) { return (key & 0x27) | ((key >> 1) & 8) | ((key << 1) & 16); }

__global__ __launch_bounds__(kThreads, 1) void prefill_kernel(PrefillParams p) {
    extern __shared__ __align__(16) unsigned char smem[];
    Tiles& lds = *reinterpret_cast<Tiles*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int chunks = p.group / p.hc;
    const int tile = blockIdx.x % p.tiles, hchunk = blockIdx.x / p.tiles;
    const int b = blockIdx.y / p.cache.kv_heads, g = blockIdx.y - b * p.cache.kv_heads;
    const int len = cache_length_scalar(p.cache, b), base = len - p.n_q;   // position of row 0
    (void)chunks;

    int head[2], row0[2], limit[2];
    bf16x8 q[2][8];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
        const int w = 2 * wave + rb;
        head[rb] = b * p.q_heads + g * p.group + hchunk * p.hc + w % p.hc;
        row0[rb] = tile * p.tok + 32 * (w / p.hc);
        const int row = min(row0[rb] + col, p.n_q - 1);
        limit[rb] = max(base + row, 0);
        const uint16_t* const from = p.q + (static_cast<int64_t>(head[rb]) * p.n_q + row) * 128 + 8 * half;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[rb][j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(from + 16 * j));
    }
    const int last = base + min((tile + 1) * p.tok, p.n_q) - 1;            // position of the unit's last row
    const int blocks = max(last, 0) / kBlock + 1;

    f32x16 o[2][4];
    float top[2], sum[2];
    int unit_now[4] = {0, 0, 0, 0};                                        // R that the sums of each group are in
    int unit_mine = 0;                                                     // R of this wavefront's channels
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
        top[rb] = -INFINITY;
        sum[rb] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[rb][j][e] = 0.0f;
    }

    const int key = tid >> 2, quarter = tid & 3, key_row = row_of_key(key);
    const uint32_t k_scale = kKScales + 4 * (16 * quarter + (key & 15)) + (key >> 4);
    const int c = lane >> 4, m = lane & 15;
    const uint32_t v_code = kVCodes + 1024 * wave + 16 * lane, v_scale = kVScales + 16 * (4 * c + wave);

    auto block_at = [&](int block) __attribute__((always_inline)) { return len > 0 ? cache_block(p.cache, b, g, block) : nullptr; };
    auto load = [&](Raw& x, const uint8_t* from) __attribute__((always_inline)) {
        x.k = *reinterpret_cast<const uint4*>(from + 16 * tid);
        x.v = *reinterpret_cast<const uint4*>(from + v_code);
        x.ve = *reinterpret_cast<const uint4*>(from + v_scale);
        x.ke = from[k_scale];
    };
    auto put_k = [&](const Raw& x, int buffer) __attribute__((always_inline)) {
        const float scale = __uint_as_float(x.ke << 23);
        const uint32_t w[4] = {x.k.x, x.k.y, x.k.z, x.k.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(lds.k[buffer] + 256 * key_row + 16 * ((4 * quarter + i) ^ (key_row & 15))) = dequantise8(w[i], scale);
    };
    // block: its number, live: tokens of it that the sequence has
    auto put_v = [&](const Raw& x, int buffer, int block, int live) __attribute__((always_inline)) {
        const uint32_t e[4] = {x.ve.x, x.ve.y, x.ve.z, x.ve.w};
        ushort2_t scale[8], most = {0, 0};
        const uint16_t lowest = static_cast<uint16_t>(unit_mine - kSpan), bias = static_cast<uint16_t>((unit_mine - kSpan - 1) << 10);
#pragma unroll
        for (int i = 0; i < 8; ++i) {                      // tokens 16 (i / 2) + 4 c + 2 (i % 2) and the next
            const ushort2_t pair = __builtin_bit_cast(ushort2_t, __builtin_amdgcn_perm(0u, e[i >> 1], i & 1 ? 0x0c030c02u : 0x0c010c00u));
            most = __builtin_elementwise_max(most, pair - lowest);
            scale[i] = pair * static_cast<uint16_t>(1024) - bias;
        }
        if (__any(most[0] > kSpan || most[1] > kSpan)) {   // not all of E in [R - 27, R]
            int largest = 0;
            auto there = [&](int i, int j) { return 16 * (i >> 1) + 4 * c + 2 * (i & 1) + j < live; };
            auto byte = [&](int i, int j) { return static_cast<int>((e[i >> 1] >> (8 * (2 * (i & 1) + j))) & 255); };
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (there(i, j) && byte(i, j) < 255) largest = max(largest, byte(i, j));
            largest = __builtin_amdgcn_readfirstlane(wave_max_int(largest));
            bool event = largest > unit_mine;
            if (largest > unit_mine) unit_mine = min(largest + 2, 254);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int x = byte(i, j) - unit_mine + kSpan + 1;
                    const bool fits = there(i, j) && byte(i, j) < 255 && x > 0;
                    scale[i][j] = fits ? static_cast<uint16_t>(x << 10) : 0;
                    event |= there(i, j) && byte(i, j) > 0 && !fits;
                }
            if (__any(event)) lds.event[buffer] = block;
        }
        lds.unit_of[buffer][wave] = unit_mine;
        const uint32_t w[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {                      // word 2 b + u
            const int u = i & 1, channel = 32 * wave + 16 * (i >> 1) + m;
            half2_t y[4];
            y[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], 1.0f, 0) * __builtin_bit_cast(half2_t, scale[4 * u]);
            y[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], 1.0f, 1) * __builtin_bit_cast(half2_t, scale[4 * u + 1]);
            y[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], 1.0f, 2) * __builtin_bit_cast(half2_t, scale[4 * u + 2]);
            y[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], 1.0f, 3) * __builtin_bit_cast(half2_t, scale[4 * u + 3]);
            *reinterpret_cast<uint4*>(lds.v[buffer] + 128 * channel + 16 * ((4 * u + c) ^ ((channel >> 1) & 7))) =
                make_uint4(__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]), __builtin_bit_cast(uint32_t, y[2]),
                           __builtin_bit_cast(uint32_t, y[3]));
        }
    };

    if (tid < 2) lds.event[tid] = -1;
    __syncthreads();
    for (int block = 0; block < blocks; ++block) {
        const uint8_t* const from = block_at(block);
        Raw raw;
        load(raw, from ? from : p.cache.data);
        put_k(raw, 0);
        put_v(raw, 0, block, from ? min(len - block * kBlock, kBlock) : 0);
        __syncthreads();
        const bool event = lds.event[0] == block;
        if (event) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int unit = __builtin_amdgcn_readfirstlane(lds.unit_of[0][j]);
                if (unit == unit_now[j]) continue;
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[rb][j][e] = __builtin_ldexpf(o[rb][j][e], unit_now[j] - unit);
                unit_now[j] = unit;
            }
        }
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(lds.k[0] + 256 * (32 * t + col) + 16 * ((2 * j + half) ^ (col & 15))));
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[rb][j], s[t], 0, 0, 0);
                }
            // key of element e of tile t: 32 t + 16 (e / 4 % 2) + 8 (e / 8) + 4 half + e % 4
            float most = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = block * kBlock + 32 * t + 16 * ((e >> 2) & 1) + 8 * (e >> 3) + 4 * half + (e & 3);
                    if (j > limit[rb] || !from) s[t][e] = -INFINITY;
                    most = fmaxf(most, s[t][e]);
                }
            const float m_new = fmaxf(top[rb], half_max(most));
            if (__any((m_new - top[rb]) * p.c > kGrown)) {
                const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((top[rb] - m_new) * p.c);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[rb][j] *= alpha;
                sum[rb] *= alpha;
                top[rb] = m_new;
            }
            const float at = top[rb] == -INFINITY ? 0.0f : top[rb];
            half8_t weight[2][2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[t][e] - at, p.c, kLift)), y = __builtin_amdgcn_exp2f(fmaf(s[t][e + 1] - at, p.c, kLift));
                    sum[rb] += x + y;
                    const f32x2 two = {x, y};
                    const half2_t z = __builtin_convertvector(two, half2_t);
                    weight[t][e >> 3][e & 7] = z[0];
                    weight[t][e >> 3][(e & 7) + 1] = z[1];
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const half8_t a = __builtin_bit_cast(half8_t, *reinterpret_cast<const uint4*>(lds.v[0] + 128 * (32 * j + col) + 16 * ((2 * k + half) ^ ((col >> 1) & 7))));
                    o[rb][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, weight[k >> 1][k & 1], o[rb][j], 0, 0, 0);
                }
            if (event && from) {                           // what the tile of V has not
                const int live = min(len - block * kBlock, kBlock);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    for (int token = 0; token < live; ++token) {
                        const int E = __builtin_amdgcn_readfirstlane(from[kVScales + 16 * (4 * ((token >> 2) & 3) + j) + 4 * (token >> 4) + (token & 3)]);
                        if (E == 0 || (E < 255 && E >= unit_now[j] - kSpan)) continue;
                        const int at_row = row_of_key(token), element = 4 * ((at_row >> 3) & 3) + (at_row & 3);
                        float w = 0.0f;
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (32 * t + e == (token & 32) + element) w = static_cast<float>(weight[t][e >> 3][e & 7]);
                        w = __shfl(w, col + 32 * ((at_row >> 2) & 1));
                        const bool seen = block * kBlock + token <= limit[rb];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int channel = 32 * j + 8 * (e >> 2) + 4 * half + (e & 3);
                            const uint32_t word = *reinterpret_cast<const uint32_t*>(from + v_word(channel, (token >> 2) & 3, token >> 5));
                            const uint32_t code = word >> (4 * ((token & 3) + ((token >> 4) & 1) * 4)) & 15u;
                            const uint32_t size = code & 7u;           // 0 .5 1 1.5 2 3 4 6
                            float v = size < 2 ? 0.5f * static_cast<float>(size) : __builtin_ldexpf(size & 1 ? 1.5f : 1.0f, static_cast<int>(size >> 1) - 1);
                            if (code & 8u) v = -v;
                            if (E == 255) v = __uint_as_float(0x7fc00000u);
                            else v = __builtin_ldexpf(v, E - unit_now[j] + kTop);
                            if (seen) o[rb][j][e] = fmaf(w, v, o[rb][j][e]);
                        }
                    }
            }
        }
        __syncthreads();
    }

#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
        const float l = half_swap_sum(sum[rb]);
        const int row = row0[rb] + col;
        if (row >= p.n_q) continue;
        const bool none = base + row < 0 || l == 0.0f;
        const float inv = none ? 0.0f : 1.0f / l;
        const int64_t r = static_cast<int64_t>(head[rb]) * p.n_q + row;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = none ? 0.0f : __builtin_ldexpf(o[rb][j][4 * a + i] * inv, unit_now[j] - 127 - kTop);
                *reinterpret_cast<uint2*>(p.o + r * 128 + 32 * j + 8 * a + 4 * half) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            }
        if (p.lse && half == 0) p.lse[r] = none ? -INFINITY : (top[rb] * p.c + log2f(l) - kLift) * 0.69314718055994530942f;
    }
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_MAX_SEQ && q_heads % kv_heads == 0 && q_heads <= 4096 &&
           max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535;
}

}  // namespace

extern "C" size_t vs_cache_prefill_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    if (n_q <= VS_CACHE_MAX_NEW) return vs_cache_attend_workspace(batch, q_heads, kv_heads, static_cast<int>(n_q), max_n);
    return 0;
}

extern "C" int vs_cache_prefill(const void* q, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens, int64_t max_n,
                                float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (n_q > 0 && n_q <= VS_CACHE_MAX_NEW)
        return vs_cache_attend(q, cache, batch, q_heads, static_cast<int>(n_q), lens, max_n, scale, o, lse, ws, ws_bytes, stream);
    if (!q || !o || !vs::aligned16(q) || !vs::aligned16(o) || !vs::aligned16(lse) || !vs::aligned16(ws)) return VS_ERR_INVALID_ARG;
    PrefillParams p;
    p.c = scale * 1.44269504088896340736f;
    if (q_heads <= 0 || n_q <= 0 || !(scale > 0.0f) || !(p.c < INFINITY)) return VS_ERR_INVALID_ARG;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_UNSUPPORTED;
    if (ws_bytes < vs_cache_prefill_workspace(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.q_heads = q_heads;
    p.n_q = static_cast<int>(n_q);
    p.group = q_heads / cache->kv_heads;
    p.hc = p.group % 4 == 0 ? 4 : p.group % 2 == 0 ? 2 : 1;
    p.tok = kUnitRows / p.hc;
    p.tiles = (p.n_q + p.tok - 1) / p.tok;
    static vs::PerDeviceOnce once;
    const int set = once.run(nullptr, [](int) -> int {
        VS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&prefill_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(Tiles))));
        return VS_OK;
    });
    if (set != VS_OK) return set;
    hipLaunchKernelGGL(prefill_kernel, dim3(static_cast<unsigned>(p.tiles * (p.group / p.hc)), static_cast<unsigned>(batch * cache->kv_heads)), dim3(kThreads),
                       sizeof(Tiles), static_cast<hipStream_t>(stream), p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}
