// The 4-bit paged cache of keys and values: quantising tokens as they are written, and reading them back.
//   s = 2^(E - 127), the smallest power of two (E in 2 .. 252) with max |x| <= 7 s over 32 channels of a token,
//   code = the E2M1 number (0 .5 1 1.5 2 3 4 6 and a sign) nearest to x / s, the even one of two as near, 6 beyond
// (7 is where 6 and the next power's 8 would meet: no element is further off than half of its step).  Three significant bits and
// a power of two: the values are bf16 numbers, reading them back is exact.
// Both kernels move a block of 64 tokens of one head per workgroup: rows of 256 bytes on the one side, the block's 8704 bytes on
// the other; codes of V change from rows of a token to words of eight tokens of a channel on the way, in LDS.  Bound by the memory: 131072 tokens of 8
// heads are written in 133 us (5.1 TB/s) and read back in 135 (5.0), one token of each of 64 sequences in 3.5 and 3.
#include "vs_cache.h"

namespace {

constexpr int kThreads = 256;

// scale byte of a group from its largest magnitude (bf16 bits without the sign; NaN and infinity are the largest of all)
__device__ __forceinline__ int scale_byte(uint32_t top) {
    const int e = static_cast<int>(top >> 7);
    if (e == 255) return 255;
    if (top == 0) return 0;
    return min(max(e - 2 + ((top & 0x7f) > 0x60 ? 1 : 0), 2), 252);
}

// A piece of eight channels per lane, four lanes to a group: code word and scale byte.
__device__ __forceinline__ uint32_t quantise8(uint4 x, int* e_out) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0xB1, 0xf, 0xf, true)));
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0x4E, 0xf, 0xf, true)));
    const int e = scale_byte(top);
    *e_out = e;
    if (e == 0 || e == 255) return 0;
    const float scale = __uint_as_float(static_cast<uint32_t>(e) << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2c, w[0]), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2c, w[1]), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2c, w[2]), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2c, w[3]), scale, 3);
    return r;
}

// Eight codes of V for each of 64 tokens in `codes` -> the four words of piece (p, c, m) of the block: channels 32 p + m and 16 more, u = 0, 1;
// `mine`: nibbles of tokens in [lo, hi).
__device__ __forceinline__ uint4 v_piece(const uint32_t (*codes)[17], int piece, int lo, int hi, uint4* mine) {
    const int p = piece >> 6, c = (piece >> 4) & 3, m = piece & 15;
    uint32_t value[4] = {0, 0, 0, 0}, mask[4] = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int token = 32 * u + (e < 4 ? 0 : 16) + 4 * c + (e & 3);
#pragma unroll
            for (int b = 0; b < 2; ++b)
                value[2 * b + u] |= ((codes[token][4 * p + 2 * b + (m >> 3)] >> (4 * (m & 7))) & 15u) << (4 * e);
            if (token >= lo && token < hi) {
                mask[u] |= 15u << (4 * e);
                mask[2 + u] |= 15u << (4 * e);
            }
        }
    *mine = make_uint4(mask[0], mask[1], mask[2], mask[3]);
    return make_uint4(value[0], value[1], value[2], value[3]);
}

// Workgroup (x, y): the x-th block that the new tokens of sequence b touch, of head h (y = b kv_heads + h).  A block of new tokens
// only is put together in LDS and written in pieces of 16 bytes; of others every thread writes what belongs to new tokens, and a word of
// V codes, which belongs to one thread, keeps the other tokens' nibbles.
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheParams p, const uint16_t* k, const uint16_t* v, int rows) {
    __shared__ __align__(16) uint32_t k_codes[kBlock][16];
    __shared__ uint32_t codes[kBlock][17];               // V: token, piece of eight channels
    __shared__ __align__(16) uint8_t scales[512];
    const int b = blockIdx.y / p.kv_heads, h = blockIdx.y - b * p.kv_heads;
    const int len = cache_length_scalar(p, b);
    const int first = len - rows;                        // position of row 0
    const int block = max(first, 0) / kBlock + blockIdx.x;
    const int lo = max(first, 0) - block * kBlock, hi = len - block * kBlock;   // new tokens of the block: lo <= token < hi
    if (hi <= 0) return;
    uint8_t* const to = cache_block(p, b, h, block);
    if (!to) return;
    const int l = threadIdx.x & 15, g = l >> 2, token0 = threadIdx.x >> 4;
    const int64_t head = static_cast<int64_t>(blockIdx.y) * rows;
    const uint16_t* const from_k = k + (head + block * kBlock - first) * 128 + 8 * l;
    const uint16_t* const from_v = v + (head + block * kBlock - first) * 128 + 8 * l;
    if (lo <= 0 && hi >= kBlock) {
        uint4 x[kBlock / 16][2];
#pragma unroll
        for (int i = 0; i < kBlock / 16; ++i) {
            x[i][0] = *reinterpret_cast<const uint4*>(from_k + (token0 + 16 * i) * 128);
            x[i][1] = *reinterpret_cast<const uint4*>(from_v + (token0 + 16 * i) * 128);
        }
#pragma unroll
        for (int i = 0; i < kBlock / 16; ++i) {
            const int token = token0 + 16 * i;
            int ek, ev;
            k_codes[token][l] = quantise8(x[i][0], &ek);
            codes[token][l] = quantise8(x[i][1], &ev);
            if ((l & 3) == 0) {
                scales[4 * (16 * g + (token & 15)) + (token >> 4)] = static_cast<uint8_t>(ek);
                scales[256 + 16 * (4 * ((token >> 2) & 3) + g) + 4 * (token >> 4) + (token & 3)] = static_cast<uint8_t>(ev);
            }
        }
        __syncthreads();
        uint4 mine;
        reinterpret_cast<uint4*>(to)[threadIdx.x] = reinterpret_cast<const uint4*>(k_codes)[threadIdx.x];
        reinterpret_cast<uint4*>(to + kVCodes)[threadIdx.x] = v_piece(codes, threadIdx.x, 0, kBlock, &mine);
        if (threadIdx.x < 32) reinterpret_cast<uint4*>(to + kKScales)[threadIdx.x] = reinterpret_cast<const uint4*>(scales)[threadIdx.x];
        return;
    }
    const int begin = max(lo, 0), end = min(hi, kBlock);
    for (int token = begin + token0; token < end; token += 16) {
        int ek, ev;
        const uint4 xk = *reinterpret_cast<const uint4*>(from_k + token * 128), xv = *reinterpret_cast<const uint4*>(from_v + token * 128);
        *reinterpret_cast<uint32_t*>(to + token * 64 + 4 * l) = quantise8(xk, &ek);
        codes[token][l] = quantise8(xv, &ev);
        if ((l & 3) == 0) {
            to[kKScales + 4 * (16 * g + (token & 15)) + (token >> 4)] = static_cast<uint8_t>(ek);
            to[kVScales + 16 * (4 * ((token >> 2) & 3) + g) + 4 * (token >> 4) + (token & 3)] = static_cast<uint8_t>(ev);
        }
    }
    __syncthreads();
    uint4 mine;
    const uint4 value = v_piece(codes, threadIdx.x, lo, hi, &mine);
    const uint32_t w[4] = {value.x, value.y, value.z, value.w}, mask[4] = {mine.x, mine.y, mine.z, mine.w};
    uint32_t* const at = reinterpret_cast<uint32_t*>(to + kVCodes) + 4 * threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (mask[i]) at[i] = mask[i] == 0xffffffffu ? w[i] : (at[i] & ~mask[i]) | (w[i] & mask[i]);
}

__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheParams p, uint16_t* k, uint16_t* v, int rows) {
    __shared__ __align__(16) uint8_t held[kBlockBytes - kVCodes];           // V codes, K scales, V scales
    const int b = blockIdx.y / p.kv_heads, h = blockIdx.y - b * p.kv_heads;
    const int len = cache_length_scalar(p, b);
    const int first = len - rows;
    const int block = max(first, 0) / kBlock + blockIdx.x;
    const int lo = max(first, 0) - block * kBlock, hi = len - block * kBlock;
    if (hi <= 0) return;
    const uint8_t* const from = cache_block(p, b, h, block);
    if (!from) return;
    for (int i = threadIdx.x; i < (kBlockBytes - kVCodes) / 16; i += kThreads)
        reinterpret_cast<uint4*>(held)[i] = reinterpret_cast<const uint4*>(from + kVCodes)[i];
    __syncthreads();
    const int l = threadIdx.x & 15, g = l >> 2;
    const int64_t head = static_cast<int64_t>(blockIdx.y) * rows;
#pragma unroll
    for (int i = 0; i < kBlock / 16; ++i) {
        const int token = (threadIdx.x >> 4) + 16 * i;
        if (token < lo || token >= hi) continue;
        const int64_t at = (head + (block * kBlock + token - first)) * 128 + 8 * l;
        if (k) {
            const uint32_t e = held[kKScales - kVCodes + 4 * (16 * g + (token & 15)) + (token >> 4)];
            *reinterpret_cast<uint4*>(k + at) = dequantise8(*reinterpret_cast<const uint32_t*>(from + token * 64 + 4 * l), __uint_as_float(e << 23));
        }
        if (v) {
            const int c = (token >> 2) & 3, u = token >> 5, shift = 4 * ((token & 3) + ((token >> 4) & 1) * 4);
            const uint32_t e = held[kVScales - kVCodes + 16 * (4 * c + g) + 4 * (token >> 4) + (token & 3)];
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w |= ((*reinterpret_cast<const uint32_t*>(held + v_word(8 * l + j, c, u) - kVCodes) >> shift) & 15u) << (4 * j);
            *reinterpret_cast<uint4*>(v + at) = dequantise8(w, __uint_as_float(e << 23));
        }
    }
}

// workgroups along the tokens: blocks that `rows` tokens can touch wherever they begin
unsigned blocks_of(int64_t rows) { return static_cast<unsigned>((rows + kBlock - 2) / kBlock + 1); }

// at most 2^12 heads of 2^14 blocks: below 2^40
int64_t page_bytes(int kv_heads, int page_size) { return static_cast<int64_t>(kv_heads) * (page_size / kBlock) * kBlockBytes; }

}  // namespace

namespace vs {

int cache_params(const vs_cache_t* cache, int batch, const int32_t* lens, int64_t max_n, CacheParams* p) {
    if (!cache || !cache->data || !aligned16(cache->data) || !aligned4(cache->table) || !aligned4(lens)) return VS_ERR_INVALID_ARG;
    if (batch <= 0 || max_n <= 0 || cache->pages <= 0 || cache->kv_heads <= 0 || cache->page_size <= 0 || cache->max_pages <= 0) return VS_ERR_INVALID_ARG;
    if (cache->page_size % kBlock || cache->page_size > VS_MAX_SEQ || max_n > VS_MAX_SEQ || cache->kv_heads > 4096 || batch > 65535 ||
        static_cast<int64_t>(batch) * cache->kv_heads > 65535 || cache->pages > INT32_MAX) return VS_ERR_UNSUPPORTED;
    int64_t bytes;                                         // offsets into the cache have to fit in 64 bits
    if (__builtin_mul_overflow(cache->pages, page_bytes(cache->kv_heads, cache->page_size), &bytes)) return VS_ERR_UNSUPPORTED;
    if (max_n > static_cast<int64_t>(cache->max_pages) * cache->page_size) return VS_ERR_INVALID_ARG;
    if (!cache->table && static_cast<int64_t>(batch) * cache->max_pages > cache->pages) return VS_ERR_INVALID_ARG;
    p->data = static_cast<uint8_t*>(cache->data);
    p->table = cache->table;
    p->lens = lens;
    p->pages = static_cast<int>(cache->pages);
    p->head_bytes = static_cast<int64_t>(cache->page_size / kBlock) * kBlockBytes;
    p->max_pages = cache->max_pages;
    p->kv_heads = cache->kv_heads;
    p->page_blocks = cache->page_size / kBlock;
    p->max_n = static_cast<int>(max_n);
    return VS_OK;
}

}  // namespace vs

extern "C" size_t vs_cache_bytes(int64_t pages, int kv_heads, int page_size) {
    if (pages <= 0 || kv_heads <= 0 || page_size <= 0 || page_size % kBlock || pages > INT32_MAX || kv_heads > 4096 || page_size > VS_MAX_SEQ) return 0;
    size_t bytes;
    const size_t page = static_cast<size_t>(page_bytes(kv_heads, page_size));
    return __builtin_mul_overflow(static_cast<size_t>(pages), page, &bytes) ? 0 - page : bytes;
}

extern "C" int vs_cache_write(const vs_cache_t* cache, const void* k, const void* v, int batch, int64_t rows, const int32_t* lens,
                              int64_t max_n, void* stream) {
    if (!k || !v || !vs::aligned16(k) || !vs::aligned16(v) || rows <= 0) return VS_ERR_INVALID_ARG;
    if (rows > VS_MAX_SEQ) return VS_ERR_UNSUPPORTED;
    CacheParams p;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p);
    if (rc != VS_OK) return rc;
    hipLaunchKernelGGL(cache_write_kernel, dim3(blocks_of(rows), batch * p.kv_heads), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p,
                       static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), static_cast<int>(rows));
    VS_LAUNCH_CHECK();
    return VS_OK;
}

extern "C" int vs_cache_read(const vs_cache_t* cache, int batch, int64_t rows, const int32_t* lens, int64_t max_n, void* k, void* v, void* stream) {
    if ((!k && !v) || !vs::aligned16(k) || !vs::aligned16(v) || rows <= 0) return VS_ERR_INVALID_ARG;
    if (rows > VS_MAX_SEQ) return VS_ERR_UNSUPPORTED;
    CacheParams p;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p);
    if (rc != VS_OK) return rc;
    hipLaunchKernelGGL(cache_read_kernel, dim3(blocks_of(rows), batch * p.kv_heads), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p,
                       static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), static_cast<int>(rows));
    VS_LAUNCH_CHECK();
    return VS_OK;
}
