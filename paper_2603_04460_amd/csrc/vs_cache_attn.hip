// Attention of the last tokens of each sequence over the 4-bit paged cache.
//   o = softmax(scale q K^T) V over the keys up to the query's own position
// A wavefront takes blocks of 64 keys: codes come straight from memory into the registers of the matrix operands (the block is laid
// out for that), are turned into bf16 by the conversion instructions (exact), and meet
//   S^T = K Q^T   (keys x query rows, 16 x 16 x 32 matrix instructions, K's scales inside the conversion)
//   O^T = V^T P^T (channels x query rows): the lane that holds scores 4 c .. 4 c + 3 of a column holds the weights that the second
//                 product wants from it, nothing moves between lanes.
// A word of V codes is eight keys of one channel and each key has its own scale, so V's scales go to the weights instead: P times
// the scale (a power of two: no rounding besides P's own to bf16), one set per 32 channels.
//   up to four query rows of a KV head (FOLD): the 16 columns are four rows x four channel groups; every column has its group's
//     weights, and of each output tile the columns of its group count
//   more: 16 rows a tile, four sets of weights
// Running maximum and sum of the softmax per wavefront, merged in LDS at the end; where there are few (sequence, KV head) pairs, several
// workgroups share the keys and a second kernel adds their parts up.
// Bound by the memory for few rows: 136 bytes a key and KV head.
#include <float.h>

#include "vs_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct AttendParams {
    CacheParams cache;
    const uint16_t* q;
    uint16_t* o;
    float* lse;
    float* part;                   // [splits][total rows][128] sums, then [splits][total rows] (maximum, sum of weights)
    int n_q, rows;                 // new tokens; query rows of a KV head (group * n_q)
    int total_rows;                // of all sequences and heads
    int splits, units;             // units: sequences x KV heads
    float c;                       // scale * log2(e)
};

// over the four lanes that hold the same column
template <typename F>
__device__ __forceinline__ float column_reduce(float x, F op) {
    auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned r0 = r[0], r1 = r[1];
    x = op(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
    auto q = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned q0 = q[0], q1 = q[1];
    return op(__builtin_bit_cast(float, q0), __builtin_bit_cast(float, q1));
}

// Scale byte i of a word as a number.  The lowest bit of the fraction makes the byte 255 a NaN instead of an infinity and is
// far below the weights' rounding.
__device__ __forceinline__ float scale_of(uint32_t w, int i) {
    const uint32_t field = i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1;
    return __uint_as_float((field & 0x7f800000u) | 1u);
}

__device__ __forceinline__ bf16x8 operand(uint4 x) { return __builtin_bit_cast(bf16x8, x); }

template <bool FOLD>
struct Block {
    uint4 k[4], v[4];
    uint32_t ks;
    uint4 vs[FOLD ? 1 : 4];
};

template <bool FOLD>
__device__ __forceinline__ void load_block(Block<FOLD>& x, const uint8_t* at, int lane) {
    const int c = lane >> 4, m = lane & 15;
#pragma unroll
    for (int t = 0; t < 4; ++t) x.k[t] = *reinterpret_cast<const uint4*>(at + 1024 * t + 64 * m + 16 * c);
#pragma unroll
    for (int p = 0; p < 4; ++p) x.v[p] = *reinterpret_cast<const uint4*>(at + kVCodes + 1024 * p + 16 * lane);
    x.ks = *reinterpret_cast<const uint32_t*>(at + kKScales + 4 * lane);
#pragma unroll
    for (int g = 0; g < (FOLD ? 1 : 4); ++g) x.vs[g] = *reinterpret_cast<const uint4*>(at + kVScales + 64 * c + 16 * (FOLD ? m & 3 : g));
}

// TILES tiles of query rows: FOLD four rows, else 16 rows each
template <int TILES, bool FOLD>
__global__ __launch_bounds__(kThreads) void cache_attend_kernel(AttendParams p) {
    constexpr int kTileRows = FOLD ? 4 : 16;
    constexpr int kKept = FOLD ? 2 : 8;                    // output tiles of 16 channels that a lane has values of
    __shared__ float4 sums[kWaves][kKept][64];
    __shared__ float2 stat[kWaves][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, c = lane >> 4;
    const int unit = blockIdx.x / p.splits, split = blockIdx.x - unit * p.splits;
    const int b = unit / p.cache.kv_heads, h = unit - b * p.cache.kv_heads;
    const int len = cache_length(p.cache, b);
    const int blocks = (len + kBlock - 1) / kBlock;
    const int per = (blocks + p.splits - 1) / p.splits;
    const int first = split * per, last = min(first + per, blocks);
    if (p.splits > 1 && first >= last) return;

    bf16x8 q[TILES][4];
    int row[TILES], limit[TILES];                          // last key that the column's row sees
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        row[i] = (blockIdx.y * TILES + i) * kTileRows + (FOLD ? n >> 2 : n);
        const int r = min(row[i], p.rows - 1);
        limit[i] = len - p.n_q + r % p.n_q;
        const uint16_t* from = p.q + (static_cast<int64_t>(unit) * p.rows + r) * 128 + 32 * c;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[i][j] = operand(*reinterpret_cast<const uint4*>(from + 8 * j));
    }

    f32x4 o[TILES][8];
    float top[TILES], sum[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        top[i] = -FLT_MAX;
        sum[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    for (int block = first + wave; block < last; block += kWaves) {
        const uint8_t* at = cache_block(p.cache, b, h, block);
        if (!at) continue;
        Block<FOLD> x;
        load_block<FOLD>(x, at, lane);
        const bool edge = block * kBlock + kBlock - 1 > len - p.n_q;      // some row does not see all of the block

        f32x4 s[TILES][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float scale = __uint_as_float(((x.ks >> (8 * t)) & 0xffu) << 23);
            const uint32_t w[4] = {x.k[t].x, x.k[t].y, x.k[t].z, x.k[t].w};
#pragma unroll
            for (int i = 0; i < TILES; ++i) s[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 a = operand(dequantise8(w[j], scale));
#pragma unroll
                for (int i = 0; i < TILES; ++i) s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[i][j], s[i][t], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            if (edge) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (block * kBlock + 16 * t + 4 * c + e > limit[i]) s[i][t][e] = -INFINITY;
            }
            float m = -FLT_MAX;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, s[i][t][e]);
            m = column_reduce(m, [](float u, float v) { return fmaxf(u, v); });
            m = fmaxf(top[i], m * p.c);
            if (__any(m > top[i])) {
                const float f = __builtin_amdgcn_exp2f(top[i] - m);
                sum[i] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[i][j] *= f;
                top[i] = m;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][t][e] = __builtin_amdgcn_exp2f(fmaf(s[i][t][e], p.c, -top[i]));
                    sum[i] += s[i][t][e];
                }
        }

        bf16x8 w[TILES][2];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (!FOLD || g == 0) {
                const uint32_t e[4] = {x.vs[FOLD ? 0 : g].x, x.vs[FOLD ? 0 : g].y, x.vs[FOLD ? 0 : g].z, x.vs[FOLD ? 0 : g].w};
#pragma unroll
                for (int i = 0; i < TILES; ++i)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float y[8];
#pragma unroll
                        for (int a = 0; a < 8; ++a) {
                            const int t = 2 * u + (a >> 2);
                            y[a] = s[i][t][a & 3] * scale_of(e[t], a & 3);
                            // a key that the row does not see has whatever scale the memory holds
                            if (edge && block * kBlock + 16 * t + 4 * c + (a & 3) > limit[i]) y[a] = 0.0f;
                        }
                        w[i][u] = operand(make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])));
                    }
            }
            const uint32_t v[4] = {x.v[g].x, x.v[g].y, x.v[g].z, x.v[g].w};
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bf16x8 a = operand(dequantise8(v[2 * half + u], 1.0f));
#pragma unroll
                    for (int i = 0; i < TILES; ++i)
                        o[i][2 * g + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[i][u], o[i][2 * g + half], 0, 0, 0);
                }
        }
    }

    // the wavefronts' parts
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        if (i) __syncthreads();
        const float all = column_reduce(sum[i], [](float u, float v) { return u + v; });
        if (c == 0) stat[wave][n] = make_float2(top[i], all);
#pragma unroll
        for (int j = 0; j < kKept; ++j) {
            f32x4 y = o[i][j];
            if (FOLD) {                                    // the tiles of the column's group: 2 g + j
                const int g = n & 3;
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = g == 0 ? o[i][j][k] : g == 1 ? o[i][2 + j][k] : g == 2 ? o[i][4 + j][k] : o[i][6 + j][k];
            }
            sums[wave][j][lane] = make_float4(y[0], y[1], y[2], y[3]);
        }
        __syncthreads();
        float m = -FLT_MAX, l = 0.0f, f[kWaves];
#pragma unroll
        for (int k = 0; k < kWaves; ++k) m = fmaxf(m, stat[k][n].x);
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            f[k] = __builtin_amdgcn_exp2f(stat[k][n].x - m);
            l += f[k] * stat[k][n].y;
        }
        const bool there = row[i] < p.rows;
        const int64_t r = static_cast<int64_t>(unit) * p.rows + row[i];
        for (int j = wave; j < kKept && there; j += kWaves) {
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float4 z = sums[k][j][lane];
                y.x = fmaf(z.x, f[k], y.x);
                y.y = fmaf(z.y, f[k], y.y);
                y.z = fmaf(z.z, f[k], y.z);
                y.w = fmaf(z.w, f[k], y.w);
            }
            const int channel = (FOLD ? 32 * (n & 3) + 16 * j : 16 * j) + 4 * c;
            if (p.splits == 1) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                *reinterpret_cast<uint2*>(p.o + r * 128 + channel) = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
            } else {
                *reinterpret_cast<float4*>(p.part + (static_cast<int64_t>(split) * p.total_rows + r) * 128 + channel) = y;
            }
        }
        if (there && wave == 0 && c == 0 && (!FOLD || (n & 3) == 0)) {
            if (p.splits == 1) {
                if (p.lse) p.lse[r] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
            } else {
                reinterpret_cast<float2*>(p.part + static_cast<int64_t>(p.splits) * p.total_rows * 128)[static_cast<int64_t>(split) * p.total_rows + r] = make_float2(m, l);
            }
        }
    }
}

// One row per workgroup: 32 lanes hold its channels, the eight groups of them take the parts in turn.
__global__ __launch_bounds__(256) void cache_join_kernel(AttendParams p) {
    __shared__ float4 sums[8][32];
    const int r = blockIdx.x, lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int b = r / (p.rows * p.cache.kv_heads);
    const int blocks = (cache_length(p.cache, b) + kBlock - 1) / kBlock;
    const int per = (blocks + p.splits - 1) / p.splits;
    const int parts = per ? (blocks + per - 1) / per : 0;
    const float2* stat = reinterpret_cast<const float2*>(p.part + static_cast<int64_t>(p.splits) * p.total_rows * 128) + r;
    float m = -FLT_MAX, l = 0.0f;
    for (int s = 0; s < parts; ++s) m = fmaxf(m, stat[static_cast<int64_t>(s) * p.total_rows].x);
    for (int s = 0; s < parts; ++s) {
        const float2 x = stat[static_cast<int64_t>(s) * p.total_rows];
        l += x.y * __builtin_amdgcn_exp2f(x.x - m);
    }
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = group; s < parts; s += 8) {
        const float f = __builtin_amdgcn_exp2f(stat[static_cast<int64_t>(s) * p.total_rows].x - m);
        const float4 z = *reinterpret_cast<const float4*>(p.part + (static_cast<int64_t>(s) * p.total_rows + r) * 128 + 4 * lane);
        y.x = fmaf(z.x, f, y.x);
        y.y = fmaf(z.y, f, y.y);
        y.z = fmaf(z.z, f, y.z);
        y.w = fmaf(z.w, f, y.w);
    }
    sums[group][lane] = y;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) {
        const float4 z = sums[k][lane];
        y.x += z.x;
        y.y += z.y;
        y.z += z.z;
        y.w += z.w;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint2*>(p.o + static_cast<int64_t>(r) * 128 + 4 * lane) = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
    if (p.lse && lane == 0) p.lse[r] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}

struct Plan {
    int tiles, fold, groups, splits;       // tiles per wavefront, kernel, workgroups over the rows of a unit, workgroups over the keys
};

Plan plan(int64_t units, int rows, int64_t max_n) {
    Plan x;
    x.fold = rows <= 4;
    x.tiles = !x.fold && rows > 16 ? 2 : 1;
    const int per = (x.fold ? 4 : 16) * x.tiles;
    x.groups = (rows + per - 1) / per;
    const int64_t blocks = (max_n + kBlock - 1) / kBlock;
    int64_t splits = 1024 / (units * x.groups);
    if (splits > blocks / (2 * kWaves)) splits = blocks / (2 * kWaves);
    x.splits = static_cast<int>(splits < 1 ? 1 : splits);
    return x;
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_CACHE_MAX_NEW && q_heads % kv_heads == 0 &&
           q_heads <= 4096 && max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535;
}

}  // namespace

extern "C" size_t vs_cache_attend_workspace(int batch, int q_heads, int kv_heads, int n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    const Plan x = plan(static_cast<int64_t>(batch) * kv_heads, q_heads / kv_heads * n_q, max_n);
    return x.splits == 1 ? 0 : static_cast<size_t>(x.splits) * batch * q_heads * n_q * (VS_HEAD_DIM + 2) * sizeof(float);
}

extern "C" int vs_cache_attend(const void* q, const vs_cache_t* cache, int batch, int q_heads, int n_q, const int32_t* lens, int64_t max_n,
                               float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (!q || !o || !vs::aligned16(q) || !vs::aligned16(o) || !vs::aligned16(lse) || !vs::aligned16(ws)) return VS_ERR_INVALID_ARG;
    if (q_heads <= 0 || n_q <= 0 || !(scale > 0.0f) || !(scale < INFINITY)) return VS_ERR_INVALID_ARG;
    AttendParams p;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_UNSUPPORTED;
    const int64_t units = static_cast<int64_t>(batch) * cache->kv_heads;
    p.rows = q_heads / cache->kv_heads * n_q;
    if (units * p.rows > (1 << 26)) return VS_ERR_UNSUPPORTED;
    const Plan x = plan(units, p.rows, max_n);
    if (x.splits > 1 && (!ws || ws_bytes < vs_cache_attend_workspace(batch, q_heads, cache->kv_heads, n_q, max_n))) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.part = static_cast<float*>(ws);
    p.n_q = n_q;
    p.units = static_cast<int>(units);
    p.total_rows = static_cast<int>(units * p.rows);
    p.splits = x.splits;
    p.c = scale * 1.44269504088896340736f;
    const dim3 grid(static_cast<unsigned>(units * x.splits), x.groups);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    auto* const kernel = x.fold ? cache_attend_kernel<1, true> : x.tiles == 1 ? cache_attend_kernel<1, false> : cache_attend_kernel<2, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, p);
    VS_LAUNCH_CHECK();
    if (x.splits > 1) {
        hipLaunchKernelGGL(cache_join_kernel, dim3(p.total_rows), dim3(256), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    return VS_OK;
}
