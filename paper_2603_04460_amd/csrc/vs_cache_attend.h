// Attention over the 4-bit paged cache, what its kernels share: parameters, the division of all blocks among workgroups or wavefronts whatever the
// sequences' lengths are, and the form of a result and of a part.
#pragma once
#include <float.h>

#include "vs_cache.h"

namespace vs {

struct AttendParams {
    CacheParams cache;
    const uint16_t* q;
    uint16_t* o;
    float* lse;
    float* part;                   // [items][rows][128] sums, then [items][rows] (maximum, sum of weights)
    int batch, n_q, rows;          // sequences; new tokens; query rows of a KV head (group * n_q)
    int shares;                    // workers (workgroups or wavefronts) that divide the blocks among them; 0: one for each head
    int items;                     // room in part: shares + sequences x KV heads
    float c, inverse_c;            // scale * log2(e), 1 / c
};

// many query rows of a KV head (vs_cache_tile.hip): a workgroup has eight wavefronts of 32 rows, `groups` workgroups all rows
constexpr int kTileWaves = 8, kTileRows = 32 * kTileWaves;
int launch_attend_tile(const AttendParams& p, int groups, hipStream_t stream);

}  // namespace vs

namespace {

using vs::AttendParams;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kStale = 8.0f;                             // log2 units by which a score may exceed the running maximum
constexpr float kLarge = 16777216.0f;                      // 2^24: from here on a score's rounding, times log2(e) and scale, is a unit and more

// Scale byte i of a word for the conversions, which look at the exponent only: what is in the other bits does not matter.
__device__ __forceinline__ float scale_field(uint32_t w, int i) {
    return __uint_as_float(i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1);
}

__device__ __forceinline__ bf16x8 operand(uint4 x) { return __builtin_bit_cast(bf16x8, x); }

// Two weights as two bf16 terms each, 15 significant bits: the first cut off (so that the second is not negative), the second rounded.
struct TwoTerms {
    uint32_t high, low;
};

__device__ __forceinline__ TwoTerms two_terms(float a, float b) {
    const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
    return {__builtin_amdgcn_perm(v, u, 0x07060302u), pack_bf16(a - __uint_as_float(u & 0xffff0000u), b - __uint_as_float(v & 0xffff0000u))};
}

// position of the first key of a block without a page: no row sees it
constexpr int kNowhere = 1 << 30;

// inclusive sum over the lanes up to this one
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);    // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // last of a row of 16 to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);    // last of the lower half to the upper
    return x;
}

// The blocks of all sequences and KV heads in a row (sequence, head, block) are divided evenly among the workers, whatever the
// lengths are; a worker may end one head and go on with the next.  A (worker, head) pair has the slot `worker + head's
// number` for its part: from one pair of the row to the next at least one of the two grows.
// Every wavefront finds its place by a scan over lens, 64 sequences at a time.
struct Lengths {
    int first;                     // of sequence `lane`: the usual batch is read once
    int total;                     // blocks of one head over all sequences
    int chunk;                     // blocks of a worker
};

__device__ __forceinline__ int length_at(const AttendParams& p, int b) { return b < p.batch ? cache_length(p.cache, b) : 0; }

__device__ __forceinline__ int blocks_of(int len) { return (len + kBlock - 1) / kBlock; }

__device__ __forceinline__ Lengths look(const AttendParams& p, int lane) {
    Lengths x;
    x.first = length_at(p, lane);
    x.total = __builtin_amdgcn_readlane(wave_scan(blocks_of(x.first)), 63);
    for (int at = 64; at < p.batch; at += 64) x.total += __builtin_amdgcn_readlane(wave_scan(blocks_of(length_at(p, at + lane))), 63);
    const int all = x.total * p.cache.kv_heads;            // below 2^31: at most 65535 pairs of at most 16384 blocks
    x.chunk = max((all + p.shares - 1) / p.shares, 1);
    return x;
}

struct Place {
    int b, h, len;
    int block;                     // of the sequence
    int start;                     // of (b, h) in the row of all blocks
    int page, in_page;             // entry of the page table and block of the page that `block` is
};

// place `x` of the row (below its end), or the begin of head h of sequence b (b >= 0)
__device__ __forceinline__ Place find(const AttendParams& p, const Lengths& lens, int lane, int x, int b, int h) {
    Place y;
    int before = 0;
    for (int at = 0;; at += 64) {
        const int len = at == 0 ? lens.first : length_at(p, at + lane);
        const int blocks = blocks_of(len);
        const int upto = before + wave_scan(blocks);
        const int l = b >= 0 ? b - at : __popcll(__ballot(upto * p.cache.kv_heads <= x));
        if (l < 64) {
            const int of = __builtin_amdgcn_readlane(blocks, l), base = (__builtin_amdgcn_readlane(upto, l) - of) * p.cache.kv_heads;
            y.b = at + l;
            y.len = __builtin_amdgcn_readlane(len, l);
            y.h = b >= 0 ? h : (x - base) / of;
            y.start = base + y.h * of;
            y.block = b >= 0 ? 0 : x - y.start;
            y.page = y.block / p.cache.page_blocks;
            y.in_page = y.block - y.page * p.cache.page_blocks;
            return y;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
}

__device__ __forceinline__ float2* part_stat(const AttendParams& p) {
    return reinterpret_cast<float2*>(p.part + static_cast<int64_t>(p.items) * p.rows * 128);
}

__device__ __forceinline__ void put_row(const AttendParams& p, int64_t r, int channel, float4 y, float l) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint2*>(p.o + r * 128 + channel) = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
}

__device__ __forceinline__ void put_lse(const AttendParams& p, int64_t r, float m, float l) {
    if (p.lse) p.lse[r] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}

}  // namespace
