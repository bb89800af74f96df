// Attention of many query rows of a KV head over the 4-bit paged cache (a short chunk, proposed tokens of many heads).
// A workgroup turns a block of 64 keys into bf16 once, K and V with their scales (exact: three significant bits times a power of two), in
// LDS, and its eight wavefronts, 32 query rows each, read their operands from there:
//   S^T = K Q^T (keys x rows), O^T = V^T P^T (channels x rows), 32 x 32 x 16 matrix instructions
// A lane of S^T holds one row's scores of the keys 8 a + 4 (lane / 32) + 0 .. 3; V lies in LDS by channel, keys in the order in which the lanes
// hold their weights, so that nothing moves between lanes.  16-byte chunks are exchanged inside a row of LDS (by the key, by half the channel)
// so that 16 lanes reading a chunk of 16 rows use all banks.
// The codes of the block after next are on their way into registers while one block is worked on and the next one's are written to the other
// buffer: one barrier a block.
// P goes into the second product as two bf16 terms, which read the same operand of V (see vs_cache_attn.hip): 84 us with one term, 97 with two.
// 32 / 8 heads, 32768 tokens, 100 new ones (400 rows) 97 us (54 Gflop, 81 with the second terms: 830 TFLOP/s), 64 62 (with 16 rows a wavefront and every
// wavefront turning its blocks into bf16 for itself 135 and 87).  A block takes about 6400 clocks: 5500 with one term (the two products 1100 each, the
// softmax 800 to 1000, the turning into bf16 1700 to 2200), 900 more for the second terms; the matrix unit is busy for 40 % of the kernel.  With one term: the two wavefronts of a SIMD in opposite orders (one turns
// while the other multiplies) 94 against 91, 64 rows a wavefront, four wavefronts 114; with two: the second terms of four channels' tiles behind their first 98, each 16 keys' weights
// evaluated in front of their products 100, the reads of V's operands left to the compiler 102: not taken.
#include "vs_cache_attend.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTileBytes = kBlock * 256;                   // K or V of a block in bf16

struct Raw {                                               // a thread's codes: 16 channels of a key, 8 + 8 tokens of a channel
    uint2 k, v;
    uint32_t ke;
    uint4 ve;
};

__device__ __forceinline__ float half_reduce_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const unsigned a = r[0], b = r[1];
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}

__global__ __launch_bounds__(64 * vs::kTileWaves, 2) void attend_tile_kernel(AttendParams p) {
    __shared__ __align__(16) uint8_t tile[2][2][kTileBytes];               // buffer, K / V
    __shared__ int tainted[2];                             // step whose V has a group that is not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int share = blockIdx.x;
    Place at;
    int left;
    {
        const Lengths lens = look(p, lane);
        const int begin = share * lens.chunk;
        left = min(lens.total * p.cache.kv_heads - begin, lens.chunk);
        if (left <= 0) return;
        at = find(p, lens, lane, begin, -1, 0);
    }
    if (threadIdx.x < 2) tainted[threadIdx.x] = -1;
    const int row = (blockIdx.y * vs::kTileWaves + wave) * 32 + col;
    const bool idle = row - col >= p.rows;

    // a thread's piece of a block: 16 channels of a key, and 16 tokens of a channel of V with their scales
    const int key = threadIdx.x >> 3, chunk = 2 * (threadIdx.x & 7);
    // (so that 32 lanes, writing 8 bytes each, use all banks: 16 channels and both c of a 16-byte chunk)
    const int group = threadIdx.x >> 7, c = ((threadIdx.x >> 6) & 1) + 2 * ((threadIdx.x >> 4) & 1);
    const int channel = 32 * group + 16 * ((threadIdx.x >> 5) & 1) + (threadIdx.x & 15);
    const uint32_t k_scale = kKScales + 4 * (16 * (chunk >> 2) + (key & 15)) + (key >> 4), v_scale = kVScales + 16 * (4 * c + group);
    const uint32_t v_code = v_word(channel, c, 0);
    auto load = [&](Raw& x, const uint8_t* from) __attribute__((always_inline)) {
        x.k = *reinterpret_cast<const uint2*>(from + 8 * threadIdx.x);
        x.v = *reinterpret_cast<const uint2*>(from + v_code);
        x.ke = from[k_scale];
        x.ve = *reinterpret_cast<const uint4*>(from + v_scale);
    };
    // Into buffer `to`.  Of V, what must not reach rows that do not see it (their weight is zero, but zero times it is not): tokens from `live`
    // on, which may hold anything, and groups that are not finite, which are put into the rows that see them afterwards.
    auto spread = [&](const Raw& x, int to, int live, int step) __attribute__((always_inline)) {
        {
            const float scale = __uint_as_float(x.ke << 23);
            uint8_t* const out = tile[to][0] + 256 * key;
            *reinterpret_cast<uint4*>(out + 16 * (chunk ^ (key & 15))) = dequantise8(x.k.x, scale);
            *reinterpret_cast<uint4*>(out + 16 * ((chunk + 1) ^ (key & 15))) = dequantise8(x.k.y, scale);
        }
        uint8_t* const out = tile[to][1] + 128 * channel;
        const uint32_t e[4] = {x.ve.x, x.ve.y, x.ve.z, x.ve.w};
        uint32_t y[8];                                     // tokens 16 t + 4 c + 2 i, + 1 at 2 t + i: a word converted with the scale of either
        static_for<8>([&](auto k) __attribute__((always_inline)) {
            constexpr int t = k / 2, i = k % 2, two = 2 * (t & 1) + i;
            const uint32_t w = t < 2 ? x.v.x : x.v.y;
            const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_field(e[t], 2 * i), two));
            const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_field(e[t], 2 * i + 1), two));
            y[k] = __builtin_amdgcn_perm(d, a, 0x07060100u);
        });
        uint32_t nan = 0;                                  // some byte of the four words is 255
#pragma unroll
        for (int t = 0; t < 4; ++t) nan |= (0xfefefefeu - e[t]) & e[t];
        if (live < kBlock || __any((nan & 0x80808080u) != 0)) {
            bool bad = false;
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t half = j ? 0xffff0000u : 0xffffu;
                    const bool there = 16 * (k >> 1) + 4 * c + 2 * (k & 1) + j < live, finite = ((y[k] & half) >> 16 * j & 0x7f80u) != 0x7f80u;
                    bad |= there && !finite;
                    if (!there || !finite) y[k] &= ~half;
                }
            if (bad) tainted[to] = step;
            asm volatile("" ::: "memory");                 // (a branch, not selects for every block)
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
            *reinterpret_cast<uint2*>(out + 16 * ((2 * t + (c & 1)) ^ ((channel >> 1) & 7)) + 8 * (c >> 1)) = make_uint2(y[2 * t], y[2 * t + 1]);
    };

    // the block behind the one at x; the last one of the share stays
    int remain = left;
    auto next = [&](Place& x) __attribute__((always_inline)) {
        if (remain <= 1) return;
        --remain;
        if (++x.in_page == p.cache.page_blocks) {
            x.in_page = 0;
            ++x.page;
        }
        if (++x.block < blocks_of(x.len)) return;
        x.block = x.page = x.in_page = 0;
        if (++x.h < p.cache.kv_heads) return;
        x.h = 0;
        do x.len = cache_length_scalar(p.cache, ++x.b);
        while (x.len == 0 && x.b < p.batch - 1);
    };
    struct Tag {
        int unit, block, len, key;
        const uint8_t* from;
    };
    int page = cache_page(p.cache, at.b, at.page);         // looked up a block ahead
    auto fetch = [&](Raw& x) __attribute__((always_inline)) {
        const bool paged = cache_paged(p.cache, page);
        Tag y;
        y.from = p.cache.data + (paged ? cache_offset(p.cache, page, at.h, at.in_page) : 0);
        y.unit = at.b * p.cache.kv_heads + at.h;
        y.block = at.block;
        y.len = at.len;
        y.key = paged ? at.block * kBlock : kNowhere;
        load(x, y.from);
        next(at);
        page = cache_page(p.cache, at.b, at.page);
        return y;
    };
    auto live_of = [&](const Tag& y) __attribute__((always_inline)) { return y.key == kNowhere ? 0 : min(y.len - y.key, kBlock); };

    bf16x8 q[8];
    f32x16 o[4];
    float top = -FLT_MAX, less = -FLT_MAX, sum = 0.0f;     // less: top, or 0 where it is taken off before
    bool large = false;                                    // some row's running maximum is past kLarge
    int limit = -1, unit = -1, from_block = 0;             // last key that the row sees; head at work, its first block here
    auto begin = [&](const Tag& y) __attribute__((always_inline)) {
        unit = y.unit;
        from_block = y.block;
        const int r = min(row, p.rows - 1);
        limit = y.len - p.n_q + r % p.n_q;
        const uint16_t* from = p.q + (static_cast<int64_t>(unit) * p.rows + r) * 128 + 8 * half;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = operand(*reinterpret_cast<const uint4*>(from + 16 * j));
        top = less = -FLT_MAX;
        large = false;
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;
    };
    auto finish = [&](int len, int upto) __attribute__((always_inline)) {
        const bool whole = from_block == 0 && upto == blocks_of(len);
        const float l = half_swap_sum(sum);
        if (row >= p.rows) return;
        const int64_t r = static_cast<int64_t>(unit) * p.rows + row, slot = static_cast<int64_t>(share + unit) * p.rows + row;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int first = 32 * (j >> 2) + 8 * (j & 3) + 4 * half;
            const f32x16& t = o[j >> 2];
            const float4 y = make_float4(t[4 * (j & 3)], t[4 * (j & 3) + 1], t[4 * (j & 3) + 2], t[4 * (j & 3) + 3]);
            if (whole) put_row(p, r, first, y, l);
            else *reinterpret_cast<float4*>(p.part + slot * 128 + first) = y;
        }
        if (half == 0) {
            if (whole) put_lse(p, r, top, l);
            else part_stat(p)[slot] = make_float2(top, l);
        }
    };

    // The operands' LDS reads run six ahead of the products that take them, `each` products an operand.
    auto ahead_of_products = [&](auto id, auto each) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_group_barrier(0x100, 6, id);                // LDS reads
        static_for<10>([&](auto) __attribute__((always_inline)) {
            __builtin_amdgcn_sched_group_barrier(0x008, each, id);         // matrix instructions
            __builtin_amdgcn_sched_group_barrier(0x100, 1, id);
        });
        __builtin_amdgcn_sched_group_barrier(0x008, 6 * each, id);
    };
    auto take = [&](int buffer, const Tag& y, int step) __attribute__((always_inline)) {
        const bool edge = y.key + kBlock - 1 > y.len - p.n_q;
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8 a = operand(*reinterpret_cast<const uint4*>(tile[buffer][0] + 256 * (32 * t + col) + 16 * ((2 * j + half) ^ (col & 15))));
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[j], s[t], 0, 0, 0);
            }
        ahead_of_products(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
        if (edge) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (y.key + 32 * t + 8 * (i >> 2) + 4 * half + (i & 3) > limit) s[t][i] = -INFINITY;
            asm volatile("" ::: "memory");
        }
        float most[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            most[k] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) most[k] = fmaxf(most[k], s[k >> 1][8 * (k & 1) + i]);
        }
        float m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * p.c;
        if (large || __any(m > top + kStale)) {                     // the maximum may be exceeded by 2^8, as in the kernels for few rows
            m = fmaxf(top, half_reduce_max(m));
            const float f = __builtin_amdgcn_exp2f(top - m);
            sum *= f;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] *= f;
            top = m;
            large = __any(fabsf(m) > kLarge && m > -FLT_MAX);
            less = top;
            if (large) {                                   // (the row's largest weight is to be 1)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[t][i] = (s[t][i] * p.c - top) * p.inverse_c;
                less = 0.0f;
            }
        }
        float part[4] = {sum, 0.0f, 0.0f, 0.0f};
        bf16x8 high[4], low[4];                            // the weights in two terms
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            TwoTerms y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][8 * (k & 1) + 2 * i], p.c, -less));
                const float b = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][8 * (k & 1) + 2 * i + 1], p.c, -less));
                part[k] += a + b;
                y[i] = two_terms(a, b);
            }
            high[k] = operand(make_uint4(y[0].high, y[1].high, y[2].high, y[3].high));
            low[k] = operand(make_uint4(y[0].low, y[1].low, y[2].low, y[3].low));
        }
        sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 a = operand(*reinterpret_cast<const uint4*>(tile[buffer][1] + 128 * (32 * j + col) + 16 * ((2 * k + half) ^ ((col >> 1) & 7))));
                o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, high[k], o[j], 0, 0, 0);
                o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, low[k], o[j], 0, 0, 0);
            }
        ahead_of_products(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
        if (tainted[buffer] == step) {
            const int live = live_of(y);
            for (int g = 0; g < 4; ++g)
                for (int token = 0; token < live; ++token) {
                    if (y.from[kVScales + 16 * (4 * ((token >> 2) & 3) + g) + 4 * (token >> 4) + (token & 3)] != 255) continue;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j == g && y.key + token <= limit)
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[j][i] = __uint_as_float(0x7fc00000u);
                }
        }
    };

    Raw raw;
    __syncthreads();                                       // tainted
    Tag now = fetch(raw), ahead;
    spread(raw, 0, live_of(now), 0);
    ahead = fetch(raw);
    int len_at = 0, upto = 0;
    for (int step = 0;; ++step) {
        __syncthreads();                                   // this step's buffer is written, the other one read
        if (now.unit != unit) {
            if (unit >= 0 && !idle) finish(len_at, upto);
            begin(now);
            len_at = now.len;
        }
        upto = now.block + 1;
        if (left > 1) spread(raw, (step + 1) & 1, live_of(ahead), step + 1);
        const Tag after = fetch(raw);
        if (!idle) take(step & 1, now, step);
        if (--left == 0) break;
        now = ahead;
        ahead = after;
    }
    if (!idle) finish(len_at, upto);
}

}  // namespace

namespace vs {

int launch_attend_tile(const AttendParams& p, int groups, hipStream_t stream) {
    hipLaunchKernelGGL(attend_tile_kernel, dim3(p.shares, groups), dim3(64 * kTileWaves), 0, stream, p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}

}  // namespace vs
