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
    int64_t head_bytes;            // of a head in a page
    int pages;
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

// Element i of an array that no kernel writes while this one runs, i the same for the wavefront: through the scalar cache, so that no wait
// for it is a wait for the vector loads in flight.
__device__ __forceinline__ int32_t scalar_load(const int32_t* x, int64_t i) {
    const auto* at = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(x));
    return at[i];
}

__device__ __forceinline__ int cache_length(const CacheParams& p, int b) {
    return p.lens ? min(max(p.lens[b], 0), p.max_n) : p.max_n;
}

// the same, b the same for the wavefront
__device__ __forceinline__ int cache_length_scalar(const CacheParams& p, int b) {
    return p.lens ? min(max(scalar_load(p.lens, b), 0), p.max_n) : p.max_n;
}

// entry i of sequence b in the page table; outside [0, pages): no page
__device__ __forceinline__ int cache_page(const CacheParams& p, int b, int i) {
    const int64_t entry = static_cast<int64_t>(b) * p.max_pages + i;
    return p.table ? scalar_load(p.table, entry) : static_cast<int>(entry);
}

__device__ __forceinline__ bool cache_paged(const CacheParams& p, int page) { return static_cast<uint32_t>(page) < static_cast<uint32_t>(p.pages); }

__device__ __forceinline__ int64_t cache_offset(const CacheParams& p, int page, int h, int in_page) {
    return (static_cast<int64_t>(page) * p.kv_heads + h) * p.head_bytes + static_cast<int64_t>(in_page) * kBlockBytes;
}

// block `block` of sequence b, head h; null where the page table names no page
__device__ __forceinline__ uint8_t* cache_block(const CacheParams& p, int b, int h, int block) {
    const int i = block / p.page_blocks, page = cache_page(p, b, i);
    return cache_paged(p, page) ? p.data + cache_offset(p, page, h, block - i * p.page_blocks) : nullptr;
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
