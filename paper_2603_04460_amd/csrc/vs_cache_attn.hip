// Attention of the last tokens of each sequence over the 4-bit paged cache.
//   o = softmax(scale q K^T) V over the keys up to the query's own position
// A wavefront takes blocks of 64 keys: codes come straight from memory into the registers of the matrix operands (the block is laid
// out for that), are turned into bf16 by the conversion instructions (exact), and meet
//   S^T = K Q^T   (keys x query rows, 16 x 16 x 32 matrix instructions, K's scales inside the conversion)
//   O^T = V^T P^T (channels x query rows): the lane that holds scores 4 c .. 4 c + 3 of a column holds the weights that the second
//                 product wants from it, nothing moves between lanes.
// P goes into the second product as two bf16 terms: rounded to one it would be as far off as the output's own rounding (error against 64 bits 0.0023
// relative, in two terms 0.0016, the same as the output's rounding alone; one token of 131072 33.4 us with one term, 34.1 with two, five tokens of four
// sequences of 20011 20.0 and 21.9).
// A word of V codes is eight keys of one channel and each key has its own scale, so V's scales go to the weights instead: P's terms times
// the scale (a power of two: no rounding), one set per 32 channels.  As exponents of bf16 numbers that is a subtraction for two
// weights, of words that the wavefront makes in LDS once a block (with weights of one term, five tokens of four sequences of 20011 22.9 -> 20.3 us against
// words made by every lane for itself, 16 rows of 131072 39 -> 36, 64 rows of 32768 30 -> 26).
//   up to four query rows of a KV head (FOLD): the 16 columns are four rows x four channel groups; every column has its group's
//     weights, and of each output tile the columns of its group count
//   more: 16 rows a tile, four sets of weights
// A wavefront has the running maximum and sum of its keys' softmax and everything it needs in registers, two blocks of codes among it, so
// that the next one's loads are in flight while one is worked on.
//   attend_head_kernel  short sequences: eight wavefronts share a head's keys and add up in LDS
//   attend_row_kernel   all blocks of all heads and sequences in a row, divided evenly among the wavefronts of the GPU whatever the sequences'
//                       lengths (which only the GPU knows); attend_join_kernel adds the parts up
// Bound by the memory for few rows: 136 bytes a key and KV head.  32 / 8 heads, one token of 131072 34 us (142 MB; a plain read of as much
// 24): 28 to 29.7 of them the first kernel, with a start of 2, then the second kernel and the gap in front of it.
#include "vs_cache_attend.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kHeadWaves = 8;                              // that share the keys of a head
constexpr int kDepth = 2;                                  // blocks in a wavefront's registers
template <bool FOLD>
constexpr int kRows = FOLD ? 4 : 16;                       // query rows of a tile

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

struct Block {
    uint4 k[4], v[4];
    uint32_t ks, vs;                                       // four scales each, all of the block's over the wavefront
};

// lane's offsets into a block: beside a block's address, the same for the wavefront, they are all that a load needs
struct Offsets {
    uint32_t k, v, ks, vs;
    __device__ __forceinline__ explicit Offsets(int lane) {
        const uint32_t c = lane >> 4, m = lane & 15;
        k = 64 * m + 16 * c;
        v = kVCodes + 16 * lane;
        ks = kKScales + 4 * lane;
        vs = kVScales + 4 * lane;
    }
};

__device__ __forceinline__ void load_block(Block& x, const uint8_t* at, const Offsets& off) {
#pragma unroll
    for (int t = 0; t < 4; ++t) x.k[t] = *reinterpret_cast<const uint4*>(at + off.k + 1024 * t);
#pragma unroll
    for (int p = 0; p < 4; ++p) x.v[p] = *reinterpret_cast<const uint4*>(at + off.v + 1024 * p);
    x.ks = *reinterpret_cast<const uint32_t*>(at + off.ks);
    x.vs = *reinterpret_cast<const uint32_t*>(at + off.vs);
}

// V's scales meet the weights as what they take off a bf16 number's exponent: 2^(e - 127) = 2^kRaise 2^-(127 + kRaise - e), where the
// first factor goes to V.  So a pair of weights takes one subtraction, and the words that are subtracted are the same for all rows: the
// wavefront makes them once a block, in LDS (word 2 x + i: scales 2 i and 2 i + 1 of the x-th word of V's scales).
// What falls below the smallest number becomes less than 2^-126: a key loses less than 2^-126 2^kRaise 6 of the sum.  Scales past 2^kRaise
// and small ones, where that would count, take the way of weights multiplied in fp32.
constexpr int kRaise = 16;
constexpr uint32_t kScaleMost = 127 + kRaise, kScaleLeast = 56;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t less_pair(uint32_t a, uint32_t b) {      // a - b in both halves
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2, a) - __builtin_bit_cast(u16x2, b));
}

__device__ __forceinline__ uint2 scale_words(uint32_t e) {
    constexpr uint32_t most = (kScaleMost << 7) * 0x10001u;
    return make_uint2(less_pair(most, __builtin_amdgcn_perm(e, e, 0x010c000cu) >> 1), less_pair(most, __builtin_amdgcn_perm(e, e, 0x030c020cu) >> 1));
}

__device__ __forceinline__ uint32_t scaled_pair(uint32_t weights, uint32_t word) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, weights), __builtin_bit_cast(u16x2, word)));
}

// the same for any scales: the byte 255 is a NaN, by the lowest bit of the fraction
__device__ __forceinline__ TwoTerms scaled_pair_any(float a, float b, uint32_t word) {
    const uint32_t e = less_pair((kScaleMost << 7) * 0x10001u, word);
    return two_terms(a * __uint_as_float(e << 16 | 1u), b * __uint_as_float((e & 0xffff0000u) | 1u));
}

// Lane's word of V's scales with those of keys that no row sees (they have no weight, whatever the memory holds) replaced by an ordinary one;
// `live`: keys of the block that hold a token.
__device__ __forceinline__ uint32_t live_scales(uint32_t e, int lane, int live) {
    const int n = live - 16 * (lane & 3) - 4 * (lane >> 4);
    const uint32_t mine = n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1;
    return (e & mine) | (0x7f7f7f7fu & ~mine);
}

// a byte of the word is above kScaleMost, or below kScaleLeast and not 0 (a group of zeros takes any weights)
__device__ __forceinline__ bool odd_scales(uint32_t e) {
    const uint32_t low = (e - kScaleLeast * 0x01010101u) & ~e & (((e & 0x7f7f7f7fu) + 0x7f7f7f7fu) | e);
    return ((((kScaleMost * 0x01010101u - e) & e) | low) & 0x80808080u) != 0;
}

// all lanes' words of scales to the wavefront's 512 bytes of LDS
__device__ __forceinline__ void put_scales(uint2* words, uint32_t e, int lane) {
    words[lane] = scale_words(e);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What a wavefront knows of its query rows (FOLD: four, else 16) and keeps of the keys so far.
template <bool FOLD>
struct Rows {
    static constexpr int kKept = FOLD ? 2 : 8;             // output tiles of 16 channels that a lane has values of
    bf16x8 q[4];
    int row, limit;                                        // of the lane's column; last key that the row sees
    f32x4 o[8];
    float top, sum;
    float less;                                            // top, or 0 where it is taken off the scores before their weights are evaluated
    bool large;                                            // some column's running maximum is past kLarge

    __device__ __forceinline__ void begin(const AttendParams& p, int lane, int unit, int len) {
        const int n = lane & 15, c = lane >> 4;
        row = blockIdx.y * kRows<FOLD> + (FOLD ? n >> 2 : n);
        const int r = min(row, p.rows - 1);
        limit = len - p.n_q + r % p.n_q;
        const uint16_t* from = p.q + (static_cast<int64_t>(unit) * p.rows + r) * 128 + 32 * c;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = operand(*reinterpret_cast<const uint4*>(from + 8 * j));
        top = less = -FLT_MAX;
        sum = 0.0f;
        large = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // 64 keys from position `key` on; edge: some row does not see all of them
    __device__ __forceinline__ void take(const AttendParams& p, const Block& x, int lane, int key, bool edge, int len, uint2* words) {
        const int c = lane >> 4;
        put_scales(words, x.vs, lane);
        f32x4 s[4];
        float scale[4];
        uint32_t word[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            scale[t] = scale_field(x.ks, t);
            word[t][0] = x.k[t].x;
            word[t][1] = x.k[t].y;
            word[t][2] = x.k[t].z;
            word[t][3] = x.k[t].w;
            s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)                        // four independent products at a time
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(dequantise8(word[t][j], scale[t])), q[j], s[t], 0, 0, 0);
        if (edge) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (key + 16 * t + 4 * c + e > limit) s[t][e] = -INFINITY;
            asm volatile("" ::: "memory");                 // (a branch, not selects for every block)
        }
        float most[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) most[t] = fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3]));
        float m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * p.c;
        // The maximum may be exceeded by 2^8: weights relative to a stale one are as exact, and the search across lanes and the rescaling are
        // left out for most blocks.
        if (large || __any(m > top + kStale)) {
            m = fmaxf(top, column_reduce(m, [](float u, float v) { return fmaxf(u, v); }));
            const float f = __builtin_amdgcn_exp2f(top - m);
            sum *= f;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] *= f;
            top = m;
            large = __any(fabsf(m) > kLarge && m > -FLT_MAX);
            less = top;
            if (large) {                                   // (the row's largest weight is to be 1)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][e] = (s[t][e] * p.c - top) * p.inverse_c;
                less = 0.0f;
            }
        }
        float part[4] = {sum, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], p.c, -less));
                part[t] += s[t][e];
            }
        sum = (part[0] + part[1]) + (part[2] + part[3]);

        TwoTerms pair[8];                                  // weights of keys 2 i and 2 i + 1 of the lane's 16
        uint32_t scales = x.vs;
        if (edge) {
            scales = live_scales(scales, lane, len - key);
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) pair[i] = two_terms(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1]);
        const bool plain = !__any(odd_scales(scales));
        // ordinary: no scale is out of the ordinary
        auto products = [&](auto ordinary) __attribute__((always_inline)) {
            bf16x8 high[2], low[2];
            const uint4* const of = reinterpret_cast<const uint4*>(words) + 8 * c + (FOLD ? 2 * (lane & 3) : 0);
            uint4 ahead[2] = {of[0], of[1]};               // words of V's scales, requested a step ahead
            int base = key;
            asm volatile("" : "+s"(base));                 // (positions of keys are not evaluated before)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if (!FOLD || g == 0) {
                    const uint32_t e[8] = {ahead[0].x, ahead[0].y, ahead[0].z, ahead[0].w, ahead[1].x, ahead[1].y, ahead[1].z, ahead[1].w};
                    if (!FOLD) {
                        if (g < 3) {
                            ahead[0] = of[2 * g + 2];
                            ahead[1] = of[2 * g + 3];
                        }
                        __builtin_amdgcn_sched_barrier(0xf);       // (reads stay in front)
                    }
                    TwoTerms y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (ordinary) {
                            y[i] = {scaled_pair(pair[i].high, e[i]), scaled_pair(pair[i].low, e[i])};
                        } else {                           // a key that the row does not see has whatever scale the memory holds
                            y[i] = scaled_pair_any(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1], e[i]);
                            const int at = base + 16 * (i >> 1) + 4 * c + 2 * (i & 1);
                            const uint32_t seen = at > limit ? 0u : at + 1 > limit ? 0xffffu : ~0u;
                            y[i] = {y[i].high & seen, y[i].low & seen};
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        high[u] = operand(make_uint4(y[4 * u].high, y[4 * u + 1].high, y[4 * u + 2].high, y[4 * u + 3].high));
                        low[u] = operand(make_uint4(y[4 * u].low, y[4 * u + 1].low, y[4 * u + 2].low, y[4 * u + 3].low));
                    }
                }
                const uint32_t v[4] = {x.v[g].x, x.v[g].y, x.v[g].z, x.v[g].w};
#pragma unroll
                for (int u = 0; u < 2; ++u)
                {
                    bf16x8 values[2];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        values[half] = operand(dequantise8(v[2 * half + u], ordinary ? static_cast<float>(1 << kRaise) : 1.0f));
                        o[2 * g + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values[half], high[u], o[2 * g + half], 0, 0, 0);
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        o[2 * g + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values[half], low[u], o[2 * g + half], 0, 0, 0);
                }
            }
        };
        if (plain) products(std::integral_constant<bool, true>{});
        else products(std::integral_constant<bool, false>{});
    }

    // output tile j of those that count in this lane
    __device__ __forceinline__ float4 kept(int j, int lane) const {
        f32x4 y = o[j];
        if (FOLD) {                                        // the tiles of the column's group: 2 g + j
            const int g = lane & 3;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = g == 0 ? o[j][k] : g == 1 ? o[2 + j][k] : g == 2 ? o[4 + j][k] : o[6 + j][k];
        }
        return make_float4(y[0], y[1], y[2], y[3]);
    }
    // its first channel
    static __device__ __forceinline__ int channel(int j, int lane) { return (FOLD ? 32 * (lane & 3) : 0) + 16 * j + 4 * (lane >> 4); }
    // one lane of those that hold a row's statistics
    static __device__ __forceinline__ bool speaks(int lane) { return lane < 16 && (!FOLD || (lane & 3) == 0); }
    __device__ __forceinline__ float total() const {
        return column_reduce(sum, [](float u, float v) { return u + v; });
    }
};

// A workgroup for each (sequence, KV head): kHeadWaves wavefronts take its blocks in turn and add up in LDS.
template <bool FOLD>
__global__ __launch_bounds__(64 * kHeadWaves) void attend_head_kernel(AttendParams p) {
    using R = Rows<FOLD>;
    __shared__ float4 sums[kHeadWaves][R::kKept][64];
    __shared__ float2 stat[kHeadWaves][16];
    __shared__ __align__(16) uint2 words[kHeadWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x, b = unit / p.cache.kv_heads, h = unit - b * p.cache.kv_heads;
    const int len = cache_length_scalar(p.cache, b), last = blocks_of(len);
    R rows;
    rows.begin(p, lane, unit, len);

    // Two blocks in registers: the next one's loads are in flight while one is worked on, and its address is known before.  Loads and
    // work are unconditional (a branch around them would make the wait for the older loads a wait for all): past the end
    // the last block is fetched again, without a page the begin of the cache, and no row sees it.
    const Offsets off(lane);
    auto address = [&](int i, bool* there) __attribute__((always_inline)) {
        const uint8_t* x = cache_block(p.cache, b, h, min(i, last - 1));
        *there = i < last && x;
        return x ? x : p.cache.data;
    };
    auto take = [&](const Block& x, int i, bool there) __attribute__((always_inline)) {
        const int key = there ? i * kBlock : kNowhere;
        rows.take(p, x, lane, key, key + kBlock - 1 > len - p.n_q, len, words[wave]);
    };
    if (wave < last) {
        bool there0, there1, there2;
        const uint8_t *at0 = address(wave, &there0), *at1 = address(wave + kHeadWaves, &there1);
        Block x0, x1;
        load_block(x0, at0, off);
        for (int block = wave;;) {
            at0 = address(block + 2 * kHeadWaves, &there2);
            load_block(x1, at1, off);
            take(x0, block, there0);
            there0 = there2;
            if ((block += kHeadWaves) >= last) break;
            at1 = address(block + 2 * kHeadWaves, &there2);
            load_block(x0, at0, off);
            take(x1, block, there1);
            there1 = there2;
            if ((block += kHeadWaves) >= last) break;
        }
    }

    const float all = rows.total();
    if (lane < 16) stat[wave][lane] = make_float2(rows.top, all);
#pragma unroll
    for (int j = 0; j < R::kKept; ++j) sums[wave][j][lane] = rows.kept(j, lane);
    __syncthreads();
    if (rows.row >= p.rows) return;
    const int n = lane & 15;
    float m = -FLT_MAX, l = 0.0f, f[kHeadWaves];
#pragma unroll
    for (int k = 0; k < kHeadWaves; ++k) m = fmaxf(m, stat[k][n].x);
#pragma unroll
    for (int k = 0; k < kHeadWaves; ++k) {
        f[k] = __builtin_amdgcn_exp2f(stat[k][n].x - m);
        l += f[k] * stat[k][n].y;
    }
    const int64_t r = static_cast<int64_t>(unit) * p.rows + rows.row;
    for (int j = wave; j < R::kKept; j += kHeadWaves) {
        float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kHeadWaves; ++k) {
            const float4 z = sums[k][j][lane];
            y.x = fmaf(z.x, f[k], y.x);
            y.y = fmaf(z.y, f[k], y.y);
            y.z = fmaf(z.z, f[k], y.z);
            y.w = fmaf(z.w, f[k], y.w);
        }
        put_row(p, r, R::channel(j, lane), y, l);
    }
    if (wave == 0 && R::speaks(lane)) put_lse(p, r, m, l);
}

// Every wavefront by itself takes `chunk` consecutive blocks of the row of all blocks, from one head and sequence to the next.
template <bool FOLD>
__global__ __launch_bounds__(256, 2) void attend_row_kernel(AttendParams p) {
    using R = Rows<FOLD>;
    const int lane = threadIdx.x & 63;
    __shared__ __align__(16) uint2 words[4][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = blockIdx.x * 4 + wave;
    Place at;
    int left;
    {
        const Lengths lens = look(p, lane);
        const int begin = share * lens.chunk;              // below 2^31: the last share begins less than `shares` chunks from the end
        left = min(lens.total * p.cache.kv_heads - begin, lens.chunk);
        if (left <= 0) return;
        at = find(p, lens, lane, begin, -1, 0);
    }
    // the block behind the one at x; the last one of the share stays
    auto next = [&](Place& x, int* remain) __attribute__((always_inline)) {
        if (*remain <= 1) return;
        --*remain;
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
    // A block's codes are requested kDepth - 1 blocks ahead, its page one more.  Loads and work are unconditional (a branch around them
    // would make the wait for the older loads a wait for all): without a page the begin of the cache is fetched and no row sees it.
    const Offsets off(lane);
    struct Held {
        Block x;
        int unit, block, len, key;
    };
    int remain = left, page;
    auto look_up = [&]() __attribute__((always_inline)) { page = cache_page(p.cache, at.b, at.page); };
    auto fetch = [&](Held& y) __attribute__((always_inline)) {
        const bool paged = cache_paged(p.cache, page);
        load_block(y.x, p.cache.data + (paged ? cache_offset(p.cache, page, at.h, at.in_page) : 0), off);
        y.unit = at.b * p.cache.kv_heads + at.h;
        y.block = at.block;
        y.len = at.len;
        y.key = paged ? at.block * kBlock : kNowhere;
        next(at, &remain);
        look_up();
    };

    R rows;
    int unit = -1, from = 0;                               // head at work, its first block here
    auto finish = [&](int len, int upto) __attribute__((always_inline)) {
        const bool whole = from == 0 && upto == blocks_of(len);
        const float l = rows.total();
        if (rows.row >= p.rows) return;
        const int64_t r = static_cast<int64_t>(unit) * p.rows + rows.row, slot = static_cast<int64_t>(share + unit) * p.rows + rows.row;
        if (whole) {
#pragma unroll
            for (int j = 0; j < R::kKept; ++j) put_row(p, r, R::channel(j, lane), rows.kept(j, lane), l);
            if (R::speaks(lane)) put_lse(p, r, rows.top, l);
        } else {
            float4* const to = reinterpret_cast<float4*>(p.part + slot * 128 + R::channel(0, lane));
#pragma unroll
            for (int j = 0; j < R::kKept; ++j) to[(R::channel(j, 0) - R::channel(0, 0)) / 4] = rows.kept(j, lane);
            if (R::speaks(lane)) part_stat(p)[slot] = make_float2(rows.top, l);
        }
    };
    int len_at = 0, upto = 0;
    // in front of the request for a later block, so that waiting for the rows is no wait for that block
    auto enter = [&](const Held& y) __attribute__((always_inline)) {
        if (y.unit == unit) return;
        if (unit >= 0) finish(len_at, upto);
        unit = y.unit;
        from = y.block;
        len_at = y.len;
        rows.begin(p, lane, unit, y.len);
    };
    auto take = [&](const Held& y) __attribute__((always_inline)) {
        rows.take(p, y.x, lane, y.key, y.key + kBlock - 1 > y.len - p.n_q, y.len, words[wave]);
        upto = y.block + 1;
    };

    Held ring[kDepth];
    look_up();
    static_for<kDepth - 1>([&](auto k) __attribute__((always_inline)) { fetch(ring[k]); });
    for (; left >= kDepth; left -= kDepth)
        static_for<kDepth>([&](auto k) __attribute__((always_inline)) {
            enter(ring[k]);
            fetch(ring[(k + kDepth - 1) % kDepth]);
            take(ring[k]);
        });
    static_for<kDepth - 1>([&](auto k) __attribute__((always_inline)) {
        if (k < left) {
            enter(ring[k]);
            take(ring[k]);
        }
    });
    finish(len_at, upto);
}

// The parts of a row added up.  A workgroup has SLICE channels of a row: SLICE / 4 lanes hold them, the other lanes are that many groups,
// which take the parts in turn, four at a time, each with a running maximum of its own; they meet inside the wavefronts, then once in LDS.
// 8 heads of 131072 tokens (128 parts of each) 4 us, the second kernel of a call; one head of 131072 (1024 parts) 13.5 with the first.
template <int SLICE>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendParams p) {
    constexpr int kLanes = SLICE / 4, kGroups = 256 / kLanes, kAhead = 4;
    static_assert(kLanes == 8 || kLanes == 32);
    __shared__ float4 sums[4][kLanes];
    __shared__ float2 stat[4];
    const int unit = blockIdx.x / p.rows, row = blockIdx.x - unit * p.rows;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, wave = threadIdx.x >> 6, b = unit / p.cache.kv_heads;
    const int channel = blockIdx.y * SLICE + 4 * lane;
    const Lengths lens = look(p, threadIdx.x & 63);
    const Place at = find(p, lens, threadIdx.x & 63, 0, b, unit - b * p.cache.kv_heads);
    const int blocks = blocks_of(at.len);
    const int from_share = at.start / lens.chunk;
    const int parts = blocks ? (at.start + blocks - 1) / lens.chunk - from_share + 1 : 0;
    if (parts == 1) return;                                // written by the wavefront that has all of the keys
    const int64_t slot = static_cast<int64_t>(from_share + unit) * p.rows + row;
    const float4* from = reinterpret_cast<const float4*>(p.part + slot * 128 + channel);
    const float2* from_stat = part_stat(p) + slot;
    float m = -FLT_MAX, l = 0.0f;
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = group; s < parts; s += kAhead * kGroups) {
        float4 z[kAhead];
        float2 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = min(s + kGroups * k, parts - 1);
            z[k] = from[i * p.rows * 32];
            x[k] = from_stat[i * p.rows];
        }
        float most = m;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (s + kGroups * k >= parts) {                // the last part again: no weight
                x[k] = make_float2(-FLT_MAX, 0.0f);
                z[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            most = fmaxf(most, x[k].x);
        }
        const float f = __builtin_amdgcn_exp2f(m - most);
        m = most;
        l *= f;
        y = make_float4(y.x * f, y.y * f, y.z * f, y.w * f);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float g = __builtin_amdgcn_exp2f(x[k].x - m);
            l = fmaf(x[k].y, g, l);
            y.x = fmaf(z[k].x, g, y.x);
            y.y = fmaf(z[k].y, g, y.y);
            y.z = fmaf(z[k].z, g, y.z);
            y.w = fmaf(z[k].w, g, y.w);
        }
    }
    // over the wavefront's groups: lanes that differ in bit 5, and bits 3 and 4
    auto across = [&](float v, auto op) __attribute__((always_inline)) {
        if (kLanes == 8) {
            v = op(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true)));   // row_ror 8
            return column_reduce(v, op);
        }
        const auto w = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        const unsigned w0 = w[0], w1 = w[1];
        return op(__builtin_bit_cast(float, w0), __builtin_bit_cast(float, w1));
    };
    const auto plus = [](float u, float v) { return u + v; };
    const float most = across(m, [](float u, float v) { return fmaxf(u, v); }), f = __builtin_amdgcn_exp2f(m - most);
    l = across(l * f, plus);
    y = make_float4(across(y.x * f, plus), across(y.y * f, plus), across(y.z * f, plus), across(y.w * f, plus));
    if ((threadIdx.x & 63) < kLanes) sums[wave][lane] = y;
    if ((threadIdx.x & 63) == 0) stat[wave] = make_float2(most, l);
    __syncthreads();
    if (group) return;
    m = fmaxf(fmaxf(stat[0].x, stat[1].x), fmaxf(stat[2].x, stat[3].x));
    l = 0.0f;
    y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float g = __builtin_amdgcn_exp2f(stat[k].x - m);
        const float4 z = sums[k][lane];
        l = fmaf(stat[k].y, g, l);
        y.x = fmaf(z.x, g, y.x);
        y.y = fmaf(z.y, g, y.y);
        y.z = fmaf(z.z, g, y.z);
        y.w = fmaf(z.w, g, y.w);
    }
    put_row(p, r, channel, y, l);
    if (channel == 0) put_lse(p, r, m, l);
}

constexpr int kSliced = 512;                               // fewer rows than this: the joining kernel has four workgroups a row

struct Plan {
    bool fold;
    bool many;                     // rows: the kernel of vs_cache_tile.hip
    int groups;                    // workgroups over the rows of a sequence and KV head
    int shares;                    // see AttendParams
    int64_t items;
};

// The form with the least time by these estimates (us), each a line in the number of blocks that the bound of the lengths allows: a start, the blocks of one worker,
// and `join`, the second kernel, the parts and the scans over the lengths.  Sequences of a batch differ in length and are counted as 2/5 of the bound (the
// batches below: spread evenly in their logarithm from a sixteenth of it to all of it).
//   head   a workgroup for each head and tile of rows, eight wavefronts to its blocks, one workgroup on a compute unit at a time, no second kernel
//   row    all blocks in a row, divided among the wavefronts of the GPU
//   tile   all blocks in a row, turned into bf16 once for 256 rows
// The estimates' starts grow in this order, so that with more blocks the form goes from head to row to tile and never back, and so does the workspace.
// Measured, head / row, 32 / 8 heads (sequences x new tokens x longest): 1 x 1 x 1000 7.5 / 7.6, 1500 9.2 / 7.8, 4 x 1 x 1000 7.4 / 7.9, 1500 9.2 / 8.2, 8 x 1 x 1500 9.2 / 9.2,
// 2000 10.8 / 9.3, 12 x 1 x 1500 9.2 / 10.2, 2000 11.0 / 10.4, 16 x 1 x 1500 9.6 / 10.8, 2000 11.4 / 11.2, 4000 18.5 / 14.8, 32 x 1 x 2000 12.9 / 14.8, 3000 16.4 / 16.0, 4000 19.8 / 17.2,
// 64 x 1 x 2000 20.1 / 19.6, 3000 23.2 / 22.1, 4 heads on one, 64 x 1 x 1500 9.1 / 9.1, 200 10.3 / 15.3, 300 14.7 / 18.0; 1 x 5 x 1000 7.9 / 8.8, 1500 9.7 / 9.2, 2000 11.5 / 9.7, 4 x 5 x 1500 9.7 / 9.7, 2000 11.6 / 10.8, 16 x 5 x 4000 20.1 / 20.9, 6000 27.1 / 23.3,
// 64 x 5 x 2000 33 / 38, 4000 59 / 61, 8000 99 / 82; 1 x 25 x 2000 11.8 / 12.2, 3000 15.5 / 13.4, 1 x 50 x 3000 15.7 / 17.7, 4000 19.4 / 19.6, 6000 26.7 / 24.1, 1 x 75 x 8000 34 / 36,
// 1 x 100 x 4000 20 / 29, 8000 34 / 42, 12000 48 / 59; 4 x 25 x 4000 19.5 / 20.5, 6000 27 / 21, 16 x 16 x 4000 36 / 36, 8000 53 / 44, 4 x 50 x 2000 22 / 24, 4000 37 / 31.
// Batches whose sequences are all as long as the bound (only the GPU knows): 8 x 1 x 2000 11.6 / 12.2, 16 x 1 x 2000 12.2 / 14.0, 4000 19.1 / 19.7, 6000 29 / 26, 32 x 1 x 4000 31 / 36, 64 x 1 x 4000 58 / 63,
// 16 x 5 x 4000 22 / 31, 5000 26 / 36, 6000 32 / 42, 64 x 5 x 4000 106 / 95, 4 x 25 x 4000 20 / 30, 6000 27 / 38, 4 x 50 x 4000 38 / 50: up to 45 % for the estimate's 2/5; counted full, the
// batches above would lose as much (32 x 1 x 8000 33 / 21, 16 x 5 x 12000 48 / 34).
// Row / tile: 1 x 24 (96 rows of a KV head) x 32768 41 / 42, 131072 130 / 128, 1 x 32 (128) x 24000 39 / 39, 32768 48 / 44, 131072 164 / 132, 1 x 40 (160) x 16000 35 / 39,
// 24000 48 / 48, 32768 60 / 55, 131072 211 / 172, 1 x 48 x 16000 41 / 41, 24000 55 / 51, 1 x 64 x 10000 35 / 40, 16000 49 / 46, 32768 88 / 63, 1 x 100 x 16000 73 / 64, 32768 136 / 98;
// 4 x 50 x 8000 50 / 48; 8 / 8 heads, 1 x 100 x 30000 42 / 44, 1 x 128 x 60000 80 / 72; 16 / 2 heads, 1 x 32 x 131072 86 / 62.
Plan plan(int64_t batch, int kv_heads, int rows, int64_t max_n) {
    Plan x;
    x.fold = rows <= 4;
    const int per = x.fold ? kRows<true> : kRows<false>;
    x.groups = (rows + per - 1) / per;
    const int64_t units = batch * kv_heads, blocks = (max_n + kBlock - 1) / kBlock;
    const double all = static_cast<double>(units * blocks) * (batch > 1 ? 0.4 : 1.0);
    const int64_t total = units * rows;
    const double join = 0.0016 * static_cast<double>(total < kSliced ? 4 * total : total) + 1.3 * static_cast<double>((batch - 1) / 64);

    const int64_t rounds = (units * x.groups + 255) / 256;
    const double head = 4.2 + (x.fold ? 1.68 : 1.86) * static_cast<double>(rounds * blocks) / kHeadWaves;
    // A wavefront for every SIMD: with two blocks in registers each that is enough to keep the memory busy, and more of them only make more
    // parts.  512 / 1024 / 1536 / 2048 wavefronts (weights of one term), us: 32 / 8 heads, one sequence of 32768 tokens 16.4 / 14.0 / 16.6 / 16.5, 131072 41 / 34 /
    // 37 / 36, 64 of 8000 59 / 45 / 47 / 44, four new tokens of 131072 54 / 38 / 43 / 41.
    x.shares = 1024 / x.groups < 4 ? 4 : 1024 / x.groups / 4 * 4;
    const double row = (x.fold ? 7.8 + 0.006 * static_cast<double>(units) : 9.1) + (x.fold ? 1.0 : 1.15) * all / x.shares + join;
    // One workgroup on every compute unit; with fewer than six blocks for each, its start and its parts are more than the estimate.  Up to 64 rows it has no gain,
    // and from 65 on no fewer shares than above: shorter sequences need no larger workspace.
    const int tile_groups = (rows + vs::kTileRows - 1) / vs::kTileRows, tile_shares = 256 / tile_groups < 4 ? 4 : 256 / tile_groups;
    const int waves = (rows < vs::kTileRows ? rows + 31 : vs::kTileRows) / 32;
    const double tile = 16.0 + (waves <= 4 ? 1.8 : 1.65 + 0.15 * waves) * all / tile_shares + join;
    x.many = rows > 64 && all >= 6.0 * tile_shares && tile < row;
    // Head up to 24 blocks for each of its wavefronts: beyond, a hundred tokens would still gain (1 x 100 x 14000 55 / 59 with tile, 1 x 128 56 / 63, x 16000 63 / 67), which
    // is left.
    if (blocks <= 24 * kHeadWaves && head < (x.many ? tile : row)) {
        x.many = false;
        x.shares = 0;
    } else if (x.many) {
        x.groups = tile_groups;
        x.shares = tile_shares;
    }
    x.items = x.shares ? units + x.shares : units;
    return x;
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_CACHE_MAX_NEW && q_heads % kv_heads == 0 &&
           q_heads <= 4096 && max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535;
}

}  // namespace

extern "C" size_t vs_cache_attend_workspace(int batch, int q_heads, int kv_heads, int n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    const Plan x = plan(batch, kv_heads, q_heads / kv_heads * n_q, max_n);
    return x.shares ? static_cast<size_t>(x.items) * (q_heads / kv_heads * n_q) * (VS_HEAD_DIM + 2) * sizeof(float) : 0;
}

extern "C" int vs_cache_attend(const void* q, const vs_cache_t* cache, int batch, int q_heads, int n_q, const int32_t* lens, int64_t max_n,
                               float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (!q || !o || !vs::aligned16(q) || !vs::aligned16(o) || !vs::aligned16(lse) || !vs::aligned16(ws)) return VS_ERR_INVALID_ARG;
    AttendParams p;
    p.c = scale * 1.44269504088896340736f;
    p.inverse_c = 1.0f / p.c;
    if (q_heads <= 0 || n_q <= 0 || !(scale > 0.0f) || !(p.c < INFINITY)) return VS_ERR_INVALID_ARG;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n)) return VS_ERR_UNSUPPORTED;
    const int64_t units = static_cast<int64_t>(batch) * cache->kv_heads;
    p.rows = q_heads / cache->kv_heads * n_q;
    if (units * p.rows >= 1 << 24) return VS_ERR_UNSUPPORTED;     // threads of the joining kernel: 256 a row, 32 bits
    const Plan x = plan(batch, cache->kv_heads, p.rows, max_n);
    if (x.shares && (!ws || ws_bytes < vs_cache_attend_workspace(batch, q_heads, cache->kv_heads, n_q, max_n))) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.part = static_cast<float*>(ws);
    p.batch = batch;
    p.n_q = n_q;
    p.shares = x.shares;
    p.items = static_cast<int>(x.items);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!x.shares) {
        hipLaunchKernelGGL(x.fold ? attend_head_kernel<true> : attend_head_kernel<false>, dim3(static_cast<unsigned>(units), x.groups),
                           dim3(64 * kHeadWaves), 0, s, p);
        VS_LAUNCH_CHECK();
        return VS_OK;
    }
    if (x.many) {
        const int tile_rc = vs::launch_attend_tile(p, x.groups, s);
        if (tile_rc != VS_OK) return tile_rc;
    } else {
        hipLaunchKernelGGL(x.fold ? attend_row_kernel<true> : attend_row_kernel<false>, dim3(x.shares / 4, x.groups), dim3(256), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    const unsigned total = static_cast<unsigned>(units * p.rows);
    if (total < kSliced) hipLaunchKernelGGL(attend_join_kernel<32>, dim3(total, 4), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(attend_join_kernel<128>, dim3(total), dim3(256), 0, s, p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}
