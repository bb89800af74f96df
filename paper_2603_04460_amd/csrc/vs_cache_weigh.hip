// The weight that every token of the 4-bit paged cache gets from the last tokens' queries, added to what it had:
//   w_j = decay old_j + sum over the query heads of a KV head and over the rows r that see j of exp(scale q_r . K_j - lse_r)
// K of a block of 64 tokens comes straight from memory into the registers of the matrix operands, is turned into bf16 by the conversions (scales among
// it, exact) and stays there while the rows pass by: S = K Q^T, keys x rows.  A lane keeps the sums of its keys over its rows, which meet across the lanes
// once at the end: no key belongs to two wavefronts, no atomics, the same call gives the same bits.
// The exponent scale s - lse is near zero for every weight that counts, its terms are not: it is a multiply-add, in one rounding, times log2(e).  The kernel for many
// rows saves the product: what its factor c = scale log2(e) loses by its rounding is put into lse's factor (c / scale), and what is left of lse's product goes to the row
// as a factor of its weights, which costs nothing since the sum is a multiply-add.  Past kFar that factor would come to leave the range of fp32, and make NaN of weights that
// are zero: tiles with such an lse have the product, as masked ones do, whose scores are gone over once more in any case.
//   weigh_few_kernel   up to 16 rows of a KV head: 16 x 16 x 32 products, the rows in registers; bound by the memory (68 + 8 bytes a token)
//   weigh_many_kernel  more: 32 x 32 x 16 products, four wavefronts of 64 keys share the rows, which come to LDS in tiles of 32
//   weigh_add_kernel   few keys and many rows: workgroups share the rows, their sums meet here, in the order of the rows
#include <float.h>

#include "vs_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
constexpr int kFewRows = 16;
constexpr int kRing = 8;                                   // tiles of rows in LDS
constexpr int kAhead = 4;                                  // tiles that are asked for in advance (6: the same)
constexpr int kTileBytes = 32 * 256;

struct WeighParams {
    CacheParams cache;
    const uint16_t* q;
    const float* lse;
    const float* old;              // or null: zeros
    float* weights;
    int64_t stride;
    float* part;                   // [parts][units][padded] sums, or null: one workgroup has all rows of its keys
    int64_t padded;
    int parts;
    int n_q, rows;                 // query rows of a KV head: group * n_q
    int runs, run_rows, tiles;     // rows are taken in `runs` runs (all of them, or a head each) of run_rows rows, `tiles` tiles each
    int blocks;                    // of a wavefront
    int fresh;                     // last tokens that have no weight yet
    float scale;
    float c, ratio, ratio_low;     // scale log2(e); c / scale in two terms
    float decay;
};

__device__ __forceinline__ bf16x8 operand(uint4 x) { return __builtin_bit_cast(bf16x8, x); }

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kFar = 4194304.0f;                         // 2^22: up to here what is left of lse's product is below 1

// A row without a key (lse = -inf) has no weights.
__device__ __forceinline__ float lse_for(float lse) { return lse == -INFINITY ? INFINITY : lse; }

// A row's weights are 2^(c s - high) factor, where its lse is not far.
struct RowConst {
    float high, factor;
};

__device__ __forceinline__ RowConst row_const(const WeighParams& p, float lse) {
    RowConst x;
    x.high = lse * p.ratio;
    x.factor = __builtin_amdgcn_exp2f(-fmaf(lse, p.ratio_low, fmaf(lse, p.ratio, -x.high)));
    return x;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// Sixteen values of each lane, summed over a row of 16 lanes: lane m gets the sum of value m.  Lanes that differ in a bit of their number exchange the
// halves that the other one keeps.
__device__ __forceinline__ float sum_to_lane(float (&v)[16], int lane) {
    static_for<8>([&](auto i) __attribute__((always_inline)) {
        const bool b = lane & 8;
        const float keep = b ? v[i + 8] : v[i], send = b ? v[i] : v[i + 8];
        v[i] = keep + dpp<0x140>(send);                    // lane 15 - m
    });
    static_for<4>([&](auto i) __attribute__((always_inline)) {
        const bool b = lane & 4;
        const float keep = b ? v[i + 4] : v[i], send = b ? v[i] : v[i + 4];
        v[i] = keep + dpp<0x141>(send);                    // 7 - m
    });
    static_for<2>([&](auto i) __attribute__((always_inline)) {
        const bool b = lane & 2;
        const float keep = b ? v[i + 2] : v[i], send = b ? v[i] : v[i + 2];
        v[i] = keep + dpp<0x1B>(send);                     // 3 - m
    });
    const bool b = lane & 1;
    const float keep = b ? v[1] : v[0], send = b ? v[0] : v[1];
    return keep + dpp<0xB1>(send);                         // m ^ 1
}

__global__ __launch_bounds__(64 * kWaves) void weigh_few_kernel(WeighParams p) {
    const int unit = blockIdx.y, b = unit / p.cache.kv_heads, h = unit - b * p.cache.kv_heads;
    const int lane = threadIdx.x & 63, col = lane & 15, c = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = cache_length_scalar(p.cache, b), end = (len + kBlock - 1) / kBlock;
    int block = blockIdx.x * kWaves * p.blocks + wave;
    const int last = min(block + kWaves * (p.blocks - 1), end - 1);
    if (block > last) return;
    struct Held {
        uint4 k[4];
        uint32_t scale;
        float old;
        bool paged;
    };
    // after the turning round a lane has one key
    const int key = 16 * (col >> 2) + 4 * c + (col & 3);
    auto load = [&](Held& x, int block) __attribute__((always_inline)) {
        const uint8_t* from = cache_block(p.cache, b, h, block);
        x.paged = from != nullptr;
        if (!from) from = p.cache.data;
#pragma unroll
        for (int t = 0; t < 4; ++t) x.k[t] = *reinterpret_cast<const uint4*>(from + 1024 * t + 64 * col + 16 * c);
        x.scale = *reinterpret_cast<const uint32_t*>(from + kKScales + 4 * lane);
        const int j = block * kBlock + key;
        x.old = p.old && p.decay != 0.0f && j < len - p.fresh ? p.old[unit * p.stride + j] : 0.0f;
    };
    Held x;
    load(x, block);
    const int row = min(col, p.rows - 1);
    const int64_t r = static_cast<int64_t>(unit) * p.rows + row;
    bf16x8 q[4];                                           // channels 32 c + 8 j ..
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = operand(*reinterpret_cast<const uint4*>(p.q + r * 128 + 32 * c + 8 * j));
    const float lse = lse_for(p.lse[r]);
    const int limit = col < p.rows ? len - p.n_q + row % p.n_q : -1;       // last key that the row sees
    for (;; block += kWaves) {
        Held next;
        const bool more = block + kWaves <= last;
        load(next, more ? block + kWaves : block);
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t w = j == 0 ? x.k[t].x : j == 1 ? x.k[t].y : j == 2 ? x.k[t].z : x.k[t].w;
                const float scale = __uint_as_float(t == 0 ? x.scale << 23 : t == 1 ? x.scale << 15 : t == 2 ? x.scale << 7 : x.scale >> 1);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(dequantise8(w, scale)), q[j], s[t], 0, 0, 0);
            }
        float v[16];
        const int before = limit - block * kBlock - 4 * c;                 // key 16 t + i of the lane's is seen up to here
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y = fmaf(s[t][i], p.scale, -lse) * kLog2e;
                if (16 * t + i > before) y = -INFINITY;
                v[4 * t + i] = __builtin_amdgcn_exp2f(y);
            }
        float mine = sum_to_lane(v, lane);
        if (!x.paged) mine = 0.0f;
        const int j = block * kBlock + key;
        if (j < len) p.weights[unit * p.stride + j] = fmaf(x.old, p.decay, mine);
        if (!more) return;
        x = next;
    }
}

// Workgroup (x, unit, part): wavefronts take blocks 4 i + wave of the workgroup's p.blocks groups of four; part: a stretch of the tiles of rows.
// A tile of rows is in LDS as it is in memory, but for its 16-byte chunks: chunk c of row r stands at c ^ (r % 16), so that 16 lanes that read a
// chunk of 16 rows use all banks.  Where all of a part's tiles fit in LDS they are read once; otherwise two at a time are asked for, kAhead tiles ahead.
// The two halves of a group's keys run half a step apart: between the products of one stand the exponentials of the other.  Operands of the next
// tile are read behind the last products of this one's.
// What bounds it is power: the clock falls under this load, and a loop of these instructions alone, with operands from LDS and numbers like these, takes 220 ns
// for 32 x 32 scores and weights on a SIMD with one wavefront or two (1.2 PFLOP/s; without exponentials and LDS 1.77).  2048 tokens of 131072, 32 / 8 heads: 2100 us,
// 256 ns;  1024 of 32749 285 to 300 us;  64 of 131072 69 us, where eight tiles have to pay for a block's conversion and sums.
template <bool RESIDENT>
__global__ __launch_bounds__(64 * kWaves, 2) void weigh_many_kernel(WeighParams p) {
    __shared__ __align__(16) uint8_t tile_of[kRing][kTileBytes];
    __shared__ __align__(16) float lse_of[kRing][kWaves][64];
    const int unit = blockIdx.y, b = unit / p.cache.kv_heads, h = unit - b * p.cache.kv_heads, part = blockIdx.z;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = cache_length_scalar(p.cache, b), end = (len + kBlock - 1) / kBlock;
    const int group0 = blockIdx.x * p.blocks, groups = min(p.blocks, (end + kWaves - 1) / kWaves - group0);
    if (groups <= 0) return;
    const int base = len - p.n_q;                          // position of row 0
    const int all = p.runs * p.tiles, i0 = static_cast<int>(static_cast<int64_t>(all) * part / p.parts), i1 = static_cast<int>(static_cast<int64_t>(all) * (part + 1) / p.parts);
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)tile_of));
    const uint32_t lds1 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)lse_of));

    // A tile of 32 rows: the run's rows from `at` on.
    struct Tile {
        int64_t row;                                       // of the call
        int at;
    };
    auto tile_number = [&](int i) { return Tile{static_cast<int64_t>(unit) * p.rows + i / p.tiles * p.run_rows + i % p.tiles * 32, i % p.tiles * 32}; };
    // the next one; of a run those from row `skip` on
    auto forward = [&](Tile& t, int skip) __attribute__((always_inline)) {
        t.at += 32;
        t.row += 32;
        if (t.at >= p.run_rows) {
            t.row += p.run_rows - t.at + skip;
            t.at = skip;
        }
    };
    const uint32_t chunk0 = 16 * ((lane & 15) ^ ((8 * wave + (lane >> 4)) & 15)), chunk1 = chunk0 ^ 64;    // (row + 4: bit 2 of the row, which is clear in the first)
    const int row_mine = 8 * wave + (lane >> 4);
    auto request = [&](const Tile& t, int slot) __attribute__((always_inline)) {
        const int most = p.run_rows - 1 - t.at;            // (the last tile's rows behind the last one: that one again, masked)
        const uint16_t* const from = p.q + t.row * 128;
        lds_load16(256 * min(row_mine, most) + chunk0, from, lds0 + slot * kTileBytes + 2048 * wave);
        lds_load16(256 * min(row_mine + 4, most) + chunk1, from, lds0 + slot * kTileBytes + 2048 * wave + 1024);
        lds_load4(static_cast<uint32_t>(4 * min(col, most)), p.lse + t.row, lds1 + 256 * (kWaves * slot + wave));
    };

    struct Held {
        uint4 k[2][2];
        uint32_t scale[2];                                 // of groups 2 half, 2 half + 1: words of tokens 16 t + col % 16
        bool paged;
    };
    auto load = [&](Held& x, int block) __attribute__((always_inline)) {
        const uint8_t* from = block < end ? cache_block(p.cache, b, h, block) : nullptr;
        x.paged = from != nullptr;
        if (!from) from = p.cache.data;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint4* const codes = reinterpret_cast<const uint4*>(from + 64 * (32 * t + col) + 32 * half);
            x.k[t][0] = codes[0];
            x.k[t][1] = codes[1];
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) x.scale[g] = *reinterpret_cast<const uint32_t*>(from + kKScales + 4 * (16 * (2 * half + g) + (col & 15)));
    };
    const uint32_t chunk_at = 256 * col + 16 * ((8 * half) ^ (col & 15));                 // of channels 64 half of row `col`; 8 j further on: ^ 16 j

    bf16x8 y[8];                                           // channels 64 half + 8 j .. of row `col` of a tile
    Held next;
    if constexpr (RESIDENT) {
        load(next, group0 * kWaves + wave);
        Tile t = tile_number(i0);
        for (int i = i0; i < i1; ++i) {
            request(t, i - i0);
            forward(t, 0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    for (int group = group0; group < group0 + groups; ++group) {
        const int block = group * kWaves + wave, first = block * kBlock;
        if constexpr (!RESIDENT) load(next, block);
        const bool paged = next.paged;
        bf16x8 k[2][8];                                    // channels 64 half + 8 j .. of token 32 t + col
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4& x = next.k[t][j >> 2];
                k[t][j] = operand(dequantise8((j & 3) == 0 ? x.x : (j & 3) == 1 ? x.y : (j & 3) == 2 ? x.z : x.w, __uint_as_float((next.scale[j >> 2] >> (8 * (2 * t + (col >> 4)))) << 23)));
            }
        if constexpr (RESIDENT) load(next, group + 1 < group0 + groups ? block + kWaves : block);
        float sum[2][16];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[t][e] = 0.0f;
        const bool edge = first + kBlock - 1 > base;

        f32x16 s[2];                                       // scores of the group's first and second 32 keys
        float used = 0.0f, factor = 0.0f, by = 0.0f;       // of the tile that is weighed: weights 2^(by s - used) factor
        float lse = 0.0f;                                  // of the tile whose operands are there
        auto read = [&](int slot, int j) __attribute__((always_inline)) {
            y[j] = operand(*reinterpret_cast<const uint4*>(tile_of[slot] + (chunk_at ^ (16 * j))));
            if (j == 0) lse = lse_of[slot][wave][lane];    // (there when `step` looks at it)
        };
        auto weigh = [&](int u, int j) __attribute__((always_inline)) {    // elements 2 j and 2 j + 1
#pragma unroll
            for (int e = 2 * j; e < 2 * j + 2; ++e) {
                sum[u][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[u][e], by, -used)), factor, sum[u][e]);
                asm volatile("" : "+v"(sum[u][e]));        // (at this place)
            }
        };
        // Products of the tile whose operands are there with keys 32 u ..; OTHER: weights of the other 32 keys (of this tile for u = 1, of the one in front for u = 0)
        auto products = [&](auto half_of, auto other, int next_slot) __attribute__((always_inline)) {
            constexpr int U = decltype(half_of)::value;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j == 0) {
                    f32x16 zero;
#pragma unroll
                    for (int e = 0; e < 16; ++e) zero[e] = 0.0f;
                    s[U] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[U][0], y[0], zero, 0, 0, 0);
                } else {
                    s[U] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[U][j], y[j], s[U], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (U == 1) read(next_slot, j);
                if constexpr (decltype(other)::value) weigh(1 - U, j);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // exponents as they are, where the row sees the key, for rows of any lse
        auto mask = [&](int u, const Tile& t, float lse) __attribute__((always_inline)) {
            const int in_run = t.at + col, row = p.runs == 1 ? in_run % p.n_q : in_run;
            const int before = (in_run < p.run_rows ? base + row : -1) - first - 4 * half - 32 * u;
            lse = lse_for(lse);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = fmaf(s[u][e], p.scale, -lse) * kLog2e;
                if (8 * (e >> 2) + (e & 3) > before) s[u][e] = -INFINITY;
            }
        };
        using Z = std::integral_constant<int, 0>;
        using O = std::integral_constant<int, 1>;
        auto step = [&](auto old, const Tile& t, int next_slot) __attribute__((always_inline)) {
            const float lse_now = lse;
            const bool masked = edge || t.at + 32 > p.run_rows || __ballot(fabsf(lse_now) > kFar) != 0;
            products(Z{}, old, 0);
            const RowConst row = row_const(p, lse_now);
            by = p.c;
            used = row.high;
            factor = row.factor;
            if (__builtin_expect(masked, 0)) {
                mask(0, t, lse_now);
                by = 1.0f;
                used = 0.0f;
                factor = 1.0f;
            }
            products(O{}, std::true_type{}, next_slot);
            if (masked) mask(1, t, lse_now);
        };
        if constexpr (RESIDENT) {
            Tile t = tile_number(i0);
#pragma unroll
            for (int j = 0; j < 8; ++j) read(0, j);
            step(std::false_type{}, t, i0 + 1 < i1 ? 1 : 0);
            for (int i = 1; i < i1 - i0; ++i) {
                forward(t, 0);
                step(std::true_type{}, t, i0 + i + 1 < i1 ? i + 1 : 0);
            }
        } else {
            // (the first tile has none in front: weights of 2^-inf)
            by = 0.0f;
            used = INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[1][e] = 0.0f;
            // rows in front of the group's first key see nothing of it: of a run the tiles from `skip` on
            const int skip = p.runs == 1 ? 0 : min(max(group * kWaves * kBlock - base, 0) >> 5, p.tiles - 1);
            const int at0 = max(i0 % p.tiles, skip), last_run = (i1 - 1) / p.tiles - i0 / p.tiles, last = (i1 - 1) % p.tiles;
            const int count = last_run == 0 ? last + 1 - at0 : p.tiles - at0 + (last_run - 1) * (p.tiles - skip) + max(last + 1 - skip, 0);
            if (count > 0) {
                Tile now = tile_number(i0 / p.tiles * p.tiles + at0), ahead = now;
                int asked = 0;
                auto ask = [&]() __attribute__((always_inline)) {          // for the next two tiles (behind the last one: that one again)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        request(ahead, asked & (kRing - 1));
                        if (++asked < count) forward(ahead, 32 * skip);
                    }
                };
                __syncthreads();                           // the group before this one is out of the ring
                for (int i = 0; i < kAhead; i += 2) ask();
                asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(3 * (kAhead - 1)) : "memory");
#pragma unroll
                for (int j = 0; j < 8; ++j) read(0, j);
                for (int i = 0; i < count; i += 2) {
                    // tiles i, i + 1 and i + 2 are there, tile i - 1 has been read
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(3 * (kAhead - 3)) : "memory");
                    ask();
                    step(std::true_type{}, now, (i + 1) & (kRing - 1));
                    forward(now, 32 * skip);
                    if (i + 1 >= count) break;
                    step(std::true_type{}, now, (i + 2) & (kRing - 1));
                    forward(now, 32 * skip);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) weigh(1, j);
        // key 32 u + 8 (e / 4) + 4 half + e % 4 to a lane: first over 16 lanes, then over the two rows of 16
        float total[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float x = sum_to_lane(sum[u], lane);
            const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
            const unsigned r0 = r[0], r1 = r[1];
            total[u] = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
        }
        const int e = lane & 15, j = first + 32 * (col >> 4) + 8 * (e >> 2) + 4 * half + (e & 3);
        const float mine = !paged ? 0.0f : col < 16 ? total[0] : total[1];
        if (j < len) {
            if (p.part) {
                p.part[(static_cast<int64_t>(part) * gridDim.y + unit) * p.padded + j] = mine;
            } else {
                const int64_t at = unit * p.stride + j;
                p.weights[at] = p.old && p.decay != 0.0f && j < len - p.fresh ? fmaf(p.old[at], p.decay, mine) : mine;
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (what was asked for beyond the last tile)
}

__global__ __launch_bounds__(256) void weigh_add_kernel(WeighParams p) {
    const int unit = blockIdx.y, len = cache_length_scalar(p.cache, unit / p.cache.kv_heads), j = blockIdx.x * 256 + threadIdx.x;
    if (j >= len) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int part = 0; part < p.parts; ++part) sum += p.part[(static_cast<int64_t>(part) * gridDim.y + unit) * p.padded + j];
    const int64_t at = unit * p.stride + j;
    p.weights[at] = p.old && p.decay != 0.0f && j < len - p.fresh ? fmaf(p.old[at], p.decay, sum) : sum;
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_MAX_SEQ && q_heads % kv_heads == 0 && q_heads <= 4096 &&
           max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535 && q_heads / kv_heads * n_q <= INT32_MAX / 2;
}

// The form, and how workgroups share the work.
void plan(WeighParams& p, int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    const int64_t units = static_cast<int64_t>(batch) * kv_heads, blocks = (max_n + kBlock - 1) / kBlock;
    p.n_q = static_cast<int>(n_q);
    p.rows = static_cast<int>(q_heads / kv_heads * n_q);
    p.parts = 1;
    p.padded = blocks * kBlock;
    if (p.rows <= kFewRows) {
        const int64_t each = units * blocks / 8192;        // a wavefront's, with eight on a SIMD
        p.blocks = static_cast<int>(each < 1 ? 1 : each < 16 ? each : 16);
        return;
    }
    // A run for each head leaves out what its first rows do not see, at the price of a last tile that is not full.  All heads in one / one for each, us: 400 tokens of
    // 32768 126 / 129, 200 of 32768 70 / 76, 256 of 2000 12.6 / 12.3, 160 of 32768 57.4 / 56.8.
    const int64_t groups = (blocks + kWaves - 1) / kWaves;
    p.runs = n_q * n_q >= 2 * ((32 - n_q % 32) % 32) * groups * kWaves * kBlock ? static_cast<int>(q_heads / kv_heads) : 1;
    p.run_rows = p.runs == 1 ? p.rows : p.n_q;
    p.tiles = (p.run_rows + 31) / 32;
    const int64_t all = static_cast<int64_t>(p.runs) * p.tiles;
    // Two workgroups run on a compute unit, the older one faster: with fewer than 16 for each the last ones run alone.  512 / 2048 / 4096 / 8192 workgroups, us:
    // 1024 tokens of 32749 335 / 303 / 293 / 298, 128 of 32768 48.2 / 46.4 / 46.2 / -, 4096 of 4096 177 / 171 / 178 / 178.
    int64_t parts = (4096 + units * groups - 1) / (units * groups);
    if (parts > (all + 7) / 8) parts = (all + 7) / 8;      // of eight tiles at least
    // .. of four, up to two workgroups a compute unit.  Eight / four / two tiles at least, us: 300 tokens of 300 12.1 / 10.2 / 10.2, 128 of 2000 12.3 / 10.2 / 10.5,
    // 400 of 2000 16.8 / 15.9 / 16.1, 32 of 2000 7.1 / 7.4 / 10.4;  four for all: 1000 of 1000 18.2 / 19.8.
    const int64_t few = 512 / (units * groups), most = (all + 3) / 4;
    if (parts < few) parts = few < most ? few : most;
    if (parts > 64) parts = 64;
    p.parts = static_cast<int>(parts);
    // Rows that stay in LDS are worth several groups for a workgroup: all that there are at once on the card (512) where that fills 85 % of them and the one sequence is as
    // long as it may be, else small ones that even out.  Groups for 1024 / for 512, us: 64 tokens of 131072 (all of 512) 70.2 / 68.9, 32 of 32768 (all) 14.2 / 12.4, 64 of 70000 (86 %)
    // 46.1 / 42.3, of 36000 (73 %) 25.4 / 26.9, of 20000 (62 %) 17.3 / 19.5, 33 of seven sequences of up to 10000 17.1 / 31.2.
    const int64_t once = (units * groups + 511) / 512;
    const int64_t each = all > kRing ? 1 : batch == 1 && units * groups * 100 >= 85 * 512 * once ? once : units * groups / 1024 < 16 ? units * groups / 1024 : 16;
    p.blocks = static_cast<int>(each < 1 ? 1 : each);
}

size_t part_bytes(const WeighParams& p, int64_t units) { return p.parts > 1 ? static_cast<size_t>(p.parts * units * p.padded) * sizeof(float) : 0; }

}  // namespace

extern "C" size_t vs_cache_weigh_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    // (fewer groups of blocks are shared by more workgroups: the most that any length up to max_n takes)
    size_t most = 0;
    const int64_t units = static_cast<int64_t>(batch) * kv_heads;
    for (int64_t n = kBlock * kWaves;; n += kBlock * kWaves) {
        WeighParams p;
        plan(p, batch, q_heads, kv_heads, n_q, n < max_n ? n : max_n);
        const size_t x = part_bytes(p, units);
        if (x > most) most = x;
        if (n >= max_n || p.parts == 1) break;
    }
    return most;
}

extern "C" int vs_cache_weigh(const void* q, const float* lse, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens,
                              int64_t max_n, float scale, const float* old, float decay, int64_t fresh, float* weights, int64_t stride, void* ws,
                              size_t ws_bytes, void* stream) {
    if (!q || !lse || !weights || !vs::aligned16(q) || !vs::aligned16(lse) || !vs::aligned4(old) || !vs::aligned4(weights) || !vs::aligned16(ws))
        return VS_ERR_INVALID_ARG;
    WeighParams p;
    p.scale = scale;
    p.c = scale * kLog2e;
    if (q_heads <= 0 || n_q <= 0 || fresh < 0 || !(scale > 0.0f) || !(p.c < INFINITY) || !(p.c >= FLT_MIN) || !(decay >= 0.0f && decay <= 1.0f)) return VS_ERR_INVALID_ARG;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_UNSUPPORTED;
    const int64_t units = static_cast<int64_t>(batch) * cache->kv_heads;
    int64_t bytes;
    if (stride < max_n || __builtin_mul_overflow(units * 4, stride, &bytes)) return VS_ERR_INVALID_ARG;
    plan(p, batch, q_heads, cache->kv_heads, n_q, max_n);
    const size_t need = part_bytes(p, units);
    if (need && (!ws || ws_bytes < need)) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.lse = lse;
    p.old = old;
    p.weights = weights;
    p.stride = stride;
    p.part = p.parts > 1 ? static_cast<float*>(ws) : nullptr;
    p.fresh = static_cast<int>(fresh < max_n ? fresh : max_n);
    const double ratio = static_cast<double>(p.c) / scale;
    p.ratio = static_cast<float>(ratio);
    p.ratio_low = static_cast<float>(ratio - p.ratio);
    p.decay = decay;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned y = static_cast<unsigned>(units), x = static_cast<unsigned>((max_n + kBlock * kWaves * p.blocks - 1) / (kBlock * kWaves * p.blocks));
    if (p.rows <= kFewRows) {
        hipLaunchKernelGGL(weigh_few_kernel, dim3(x, y), dim3(64 * kWaves), 0, s, p);
        VS_LAUNCH_CHECK();
        return VS_OK;
    }
    hipLaunchKernelGGL(p.runs * p.tiles <= kRing * p.parts ? weigh_many_kernel<true> : weigh_many_kernel<false>, dim3(x, y, p.parts), dim3(64 * kWaves), 0, s, p);
    VS_LAUNCH_CHECK();
    if (p.part) {
        hipLaunchKernelGGL(weigh_add_kernel, dim3(static_cast<unsigned>((max_n + 255) / 256), y), dim3(256), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    return VS_OK;
}
