// The paged 4-bit cache: its layout and checks, shared by the calls that write, read and attend over it.
//
// A block is 64 tokens of one KV head in VS_CACHE_BLOCK_BYTES contiguous bytes, laid out for the operands of the 16 x 16 x 32
// matrix instructions of the attention, whose lane 16 c + m holds row (or column) m and the c-th quarter of the contraction:
//   K codes     token 16 t + m, channels 32 c + 8 j + 0 .. 7 (word j) at 64 (16 t + m) + 16 c + 4 j: the token's 64 bytes in order
//   V codes     channel 32 p + 16 b + m, tokens 32 u + 4 c + 0 .. 3 and 32 u + 16 + 4 c + 0 .. 3 (the nibbles of a word, from the
//               lowest) at 4096 + 1024 p + 16 (16 c + m) + 8 b + 4 u
//   K scales    token 16 t + m, channels 32 g .. 32 g + 31 at 8192 + 4 (16 g + m) + t
//   V scales    token 16 t + 4 c + i, channels 32 g .. at 8448 + 16 (4 c + g) + 4 t + i
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vs_common.h"
#include "vs_wave.h"

namespace vs {

struct CacheParams {
    uint8_t* data;
    const int32_t* table;          // null: sequence b has the pages b * max_pages ..
    const int32_t* lens;           // null: every sequence holds max_n tokens
    int64_t pages;
    int max_pages;                 // of a sequence
    int kv_heads;
    int page_blocks;               // blocks of a page
    int max_n;
};

// Host checks that the calls on a cache share; fills p.
int cache_params(const vs_cache_t* cache, int batch, const int32_t* lens, int64_t max_n, CacheParams* p);

}  // namespace vs

namespace {

using vs::CacheParams;

constexpr int kBlock = VS_CACHE_BLOCK;
constexpr int kBlockBytes = VS_CACHE_BLOCK_BYTES;
constexpr int kVCodes = 4096, kKScales = 8192, kVScales = 8448;

__device__ __forceinline__ int cache_length(const CacheParams& p, int b) {
    return p.lens ? min(max(p.lens[b], 0), p.max_n) : p.max_n;
}

// block `block` of sequence b, head h; null where the page table names no page
__device__ __forceinline__ uint8_t* cache_block(const CacheParams& p, int b, int h, int block) {
    const int at = block / p.page_blocks;
    const int64_t entry = static_cast<int64_t>(b) * p.max_pages + at;
    const int64_t page = p.table ? static_cast<int64_t>(p.table[entry]) : entry;
    if (page < 0 || page >= p.pages) return nullptr;
    return p.data + ((page * p.kv_heads + h) * p.page_blocks + (block - at * p.page_blocks)) * kBlockBytes;
}

__device__ __forceinline__ uint32_t v_word(int channel, int c, int u) {
    return kVCodes + (channel >> 5) * 1024 + (c * 16 + (channel & 15)) * 16 + ((channel >> 4) & 1) * 8 + u * 4;
}

typedef __bf16 bf16x2c __attribute__((ext_vector_type(2)));

// eight codes -> eight bf16 numbers, times 2^(e - 127) given as the fp32 number (exact: three significant bits; e = 255: NaN)
__device__ __forceinline__ uint4 dequantise8(uint32_t w, float scale) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}

}  // namespace
