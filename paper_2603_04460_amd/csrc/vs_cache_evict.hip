// Eviction from the 4-bit paged cache: of every sequence and KV head the first tokens, the last ones and those with the largest weights stay, in
// their order, at the front of the same cache or of another one.
//   select_kernel  a workgroup for each head: the smallest key that stays by four passes over the weights, 8 bits each (weights as unsigned numbers in
//                  their order; first and last tokens above all, NaN below all), then the numbers of the tokens that stay, ascending
//   gather_kernel  a workgroup for each block of 64 tokens that stay: codes and scales of 64 tokens from wherever they are
//   put_kernel     a cache that is made smaller in place: blocks go through the workspace, so that all are read before one is written
// Moving a token moves codes, nothing is rounded again.
#include "vs_cache.h"

namespace {

constexpr int kThreads = 256;
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr uint32_t kAlways = 0xffffffffu, kNever = 0;      // keys of tokens that stay in any case, and that are not there

struct EvictParams {
    CacheParams from, to;
    const float* weights;          // [units][stride]
    float* weights_out;            // [units][stride_out] or null
    int64_t stride, stride_out;
    int32_t* kept;                 // [units][keep] or null
    int32_t* lens_out;
    int32_t* count;                // [batch]
    int32_t* index;                // [units][keep]
    float* weight_stage;           // [units][keep] or null: weights_out is written at once
    uint8_t* block_stage;          // [units][blocks][kBlockBytes] or null: `to` is written at once
    int keep, n_sink, n_recent, blocks;
    bool same;                     // `to` is `from`
};

// The token's place in the order of staying.
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return kNever + 1;
    const uint32_t x = __float_as_uint(w + 0.0f);          // (one zero)
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

__device__ __forceinline__ uint32_t key_at(const EvictParams& p, const float* weights, int j, int n, bool paged) {
    if (j >= n || !paged) return kNever;
    return j < p.n_sink || j >= n - p.n_recent ? kAlways : key_of(weights[j]);
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictParams p) {
    __shared__ int hist[kSelectWaves][256];
    __shared__ int above[kSelectWaves], equal[kSelectWaves];
    __shared__ int shared_need, shared_digit;
    const int unit = blockIdx.x, b = unit / p.from.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = cache_length_scalar(p.from, b);
    const float* const weights = p.weights + unit * p.stride;
    // a wavefront's share: blocks [first, last)
    const int blocks = (n + kBlock - 1) / kBlock, each = (blocks + kSelectWaves - 1) / kSelectWaves;
    const int first = min(wave * each, blocks), last = min(first + each, blocks);
    auto for_keys = [&](auto f) __attribute__((always_inline)) {
        for (int block = first; block < last; ++block) {
            const bool paged = cache_paged(p.from, cache_page(p.from, b, block / p.from.page_blocks));
            f(block * kBlock + lane, key_at(p, weights, block * kBlock + lane, n, paged));
        }
    };
    // tokens that are there
    int there = 0;
    for_keys([&](int, uint32_t key) { there += __popcll(__ballot(key != kNever)); });
    if (lane == 0) above[wave] = there;
    __syncthreads();
    int present = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) present += above[w];
    const int count = min(p.keep, present);
    uint32_t prefix = 0;                                   // of the smallest key that stays
    int need = count;                                      // tokens that stay among those with that prefix
    for (int shift = 24; shift >= 0 && count > 0; shift -= 8) {
        for (int i = lane; i < 256; i += 64) hist[wave][i] = 0;
        __syncthreads();
        for_keys([&](int, uint32_t key) {
            if (key != kNever && (shift == 24 || key >> (shift + 8) == prefix)) atomicAdd(&hist[wave][(key >> shift) & 255], 1);
        });
        __syncthreads();
        if (wave == 0) {                                   // four digits a lane, from the largest down
            int sum[4], total = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] = 0;
                for (int w = 0; w < kSelectWaves; ++w) sum[i] += hist[w][255 - 4 * lane - i];
                total += sum[i];
            }
            int upto = total;
            for (int d = 1; d < 64; d *= 2) {
                const int x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            int before = upto - total;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < need && need <= before + sum[i]) {
                    shared_digit = 255 - 4 * lane - i;
                    shared_need = need - before;
                }
                before += sum[i];
            }
        }
        __syncthreads();
        prefix = prefix << 8 | static_cast<uint32_t>(shared_digit);
        need = shared_need;
    }
    int more = 0, same = 0;
    for_keys([&](int, uint32_t key) {
        more += __popcll(__ballot(key > prefix));
        same += __popcll(__ballot(key == prefix));
    });
    __syncthreads();
    if (lane == 0) {
        above[wave] = more;
        equal[wave] = same;
    }
    __syncthreads();
    int at = 0, ties = 0;                                  // larger ones, and equal ones, in front of this share
    for (int w = 0; w < wave; ++w) {
        at += above[w];
        ties += equal[w];
    }
    at += min(ties, need);
    int32_t* const index = p.index + static_cast<int64_t>(unit) * p.keep;
    int32_t* const kept = p.kept ? p.kept + static_cast<int64_t>(unit) * p.keep : nullptr;
    if (count > 0)
        for_keys([&](int j, uint32_t key) {
            const uint64_t below = (1ull << lane) - 1, tied = __ballot(key == prefix);
            const bool stays = key > prefix || (key == prefix && ties + __popcll(tied & below) < need);
            const uint64_t staying = __ballot(stays);
            if (stays) {
                const int i = at + __popcll(staying & below);
                index[i] = j;
                if (kept) kept[i] = j;
            }
            at += __popcll(staying);
            ties += __popcll(tied);
        });
    if (kept)
        for (int i = count + threadIdx.x; i < p.keep; i += kSelectThreads) kept[i] = -1;
    if (threadIdx.x == 0 && unit == b * p.from.kv_heads) p.count[b] = count;
}

// block `block` of sequence b, head h; null where the page table names no page.  (cache_block for a block that differs from lane to lane)
__device__ __forceinline__ uint8_t* block_of_lane(const CacheParams& p, int b, int h, int block) {
    const int i = block / p.page_blocks;
    const int64_t entry = static_cast<int64_t>(b) * p.max_pages + i;
    const int page = p.table ? p.table[entry] : static_cast<int>(entry);
    return cache_paged(p, page) ? p.data + cache_offset(p, page, h, block - i * p.page_blocks) : nullptr;
}

// A block all of whose tokens are where they were.
__device__ __forceinline__ bool unmoved(const EvictParams& p, int unit, int block, int count) {
    const int last = min(block * kBlock + kBlock, count) - 1;
    return p.same && p.index[static_cast<int64_t>(unit) * p.keep + last] == last;
}

__global__ __launch_bounds__(kThreads) void gather_kernel(EvictParams p) {
    __shared__ const uint8_t* from[kBlock];
    __shared__ int place[kBlock];
    const int unit = blockIdx.y, b = unit / p.from.kv_heads, h = unit - b * p.from.kv_heads, block = blockIdx.x;
    const int count = p.count[b];
    if (!p.block_stage && !p.weight_stage && block == 0 && h == 0 && threadIdx.x == 0) p.lens_out[b] = count;
    if (block * kBlock >= count) return;
    const int64_t head = static_cast<int64_t>(unit) * p.keep;
    uint8_t* const there = cache_block(p.to, b, h, block);
    uint8_t* const to = p.block_stage ? p.block_stage + (static_cast<int64_t>(unit) * p.blocks + block) * kBlockBytes : there;
    if (threadIdx.x < kBlock) {
        const int i = block * kBlock + threadIdx.x;
        if (i < count) {
            const int j = p.index[head + i];
            from[threadIdx.x] = block_of_lane(p.from, b, h, j / kBlock);
            place[threadIdx.x] = j % kBlock;
            if (p.weights_out) {
                const float w = p.weights[unit * p.stride + j];
                if (p.weight_stage) p.weight_stage[head + i] = w;
                else p.weights_out[unit * p.stride_out + i] = w;
            }
        } else {                                           // what the cache holds behind the last token stays
            from[threadIdx.x] = there;
            place[threadIdx.x] = threadIdx.x;
        }
    }
    __syncthreads();
    if (!there || unmoved(p, unit, block, count)) return;
    {
        const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
        const uint4 x = *reinterpret_cast<const uint4*>(from[token] + 64 * place[token] + 16 * quarter);
        // words (channel, u) of tokens 32 u + 4 c + 0 .. 3 and 16 more: two channels, u = 0, 1
        const int c = (threadIdx.x >> 4) & 3, channel = 32 * (threadIdx.x >> 6) + (threadIdx.x & 15);
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = 32 * u + (e < 4 ? 0 : 16) + 4 * c + (e & 3), j = place[i];
                const uint8_t* const at = from[i];
                const int shift = 4 * ((j & 3) + ((j >> 4) & 1) * 4);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    w[2 * half + u] |= ((*reinterpret_cast<const uint32_t*>(at + v_word(channel + 16 * half, (j >> 2) & 3, j >> 5)) >> shift) & 15u) << (4 * e);
            }
        uint32_t scales = 0;
        if (threadIdx.x < 128) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // K: group g, tokens 16 k + m;  V: tokens 16 t + 4 c + k of group g
                const int x = threadIdx.x & 63;
                const bool is_k = threadIdx.x < 64;
                const int i = is_k ? 16 * k + (x & 15) : 16 * (x & 3) + 4 * (x >> 4) + k, g = is_k ? x >> 4 : (x >> 2) & 3, j = place[i];
                const int at = is_k ? kKScales + 4 * (16 * g + (j & 15)) + (j >> 4) : kVScales + 16 * (4 * ((j >> 2) & 3) + g) + 4 * (j >> 4) + (j & 3);
                scales |= static_cast<uint32_t>(from[i][at]) << (8 * k);
            }
        }
        __syncthreads();                                   // (`to` may be where some of it was read)
        reinterpret_cast<uint4*>(to)[threadIdx.x] = x;
        reinterpret_cast<uint4*>(to + kVCodes)[threadIdx.x] = make_uint4(w[0], w[1], w[2], w[3]);
        if (threadIdx.x < 128) reinterpret_cast<uint32_t*>(to + kKScales)[threadIdx.x] = scales;
    }
}

__global__ __launch_bounds__(kThreads) void put_kernel(EvictParams p) {
    const int unit = blockIdx.y, b = unit / p.from.kv_heads, h = unit - b * p.from.kv_heads, block = blockIdx.x;
    const int count = p.count[b];
    if (block == 0 && h == 0 && threadIdx.x == 0) p.lens_out[b] = count;
    if (block * kBlock >= count) return;
    const int i = block * kBlock + threadIdx.x;
    if (p.weight_stage && threadIdx.x < kBlock && i < count) p.weights_out[unit * p.stride_out + i] = p.weight_stage[static_cast<int64_t>(unit) * p.keep + i];
    uint8_t* const to = cache_block(p.to, b, h, block);
    if (!p.block_stage || !to || unmoved(p, unit, block, count)) return;
    const uint4* const from = reinterpret_cast<const uint4*>(p.block_stage + (static_cast<int64_t>(unit) * p.blocks + block) * kBlockBytes);
    for (int k = threadIdx.x; k < kBlockBytes / 16; k += kThreads) reinterpret_cast<uint4*>(to)[k] = from[k];
}

bool sizes_ok(int batch, int kv_heads, int64_t max_n, int64_t keep) {
    return batch > 0 && kv_heads > 0 && max_n > 0 && keep > 0 && max_n <= VS_MAX_SEQ && keep <= VS_MAX_SEQ && batch <= 65535 && kv_heads <= 4096 &&
           static_cast<int64_t>(batch) * kv_heads <= 65535;
}

struct Parts {                                             // of the workspace: bytes in front of each
    size_t index, weights, blocks, all;
};

Parts parts(int batch, int kv_heads, int64_t keep) {
    const size_t units = static_cast<size_t>(batch) * kv_heads, k = static_cast<size_t>(keep);
    Parts x;
    x.index = vs::round_up(static_cast<size_t>(batch) * 4, 256);
    x.weights = x.index + vs::round_up(units * k * 4, 256);
    x.blocks = x.weights + vs::round_up(units * k * 4, 256);
    x.all = x.blocks + units * ((k + kBlock - 1) / kBlock) * kBlockBytes;
    return x;
}

// do the bytes [a, a + n) and [b, b + m) meet
bool meet(const void* a, size_t n, const void* b, size_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y ? y - x < n : x - y < m;
}

}  // namespace

extern "C" size_t vs_cache_evict_workspace(int batch, int kv_heads, int64_t max_n, int64_t keep) {
    return sizes_ok(batch, kv_heads, max_n, keep) ? parts(batch, kv_heads, keep).all : 0;
}

extern "C" int vs_cache_evict(const vs_cache_t* cache, const float* weights, int64_t stride, int batch, const int32_t* lens, int64_t max_n,
                              int64_t keep, int64_t n_sink, int64_t n_recent, const vs_cache_t* to, float* weights_out, int64_t stride_out,
                              int32_t* kept, int32_t* lens_out, void* ws, size_t ws_bytes, void* stream) {
    if (!weights || !lens_out || !vs::aligned4(weights) || !vs::aligned4(weights_out) || !vs::aligned4(kept) || !vs::aligned4(lens_out) ||
        !vs::aligned16(ws)) return VS_ERR_INVALID_ARG;
    if (keep <= 0 || n_sink < 0 || n_recent < 0 || n_sink > keep || n_recent > keep - n_sink) return VS_ERR_INVALID_ARG;
    if (keep > VS_MAX_SEQ) return VS_ERR_UNSUPPORTED;
    EvictParams p;
    int rc = vs::cache_params(cache, batch, lens, max_n, &p.from);
    if (rc == VS_OK) rc = vs::cache_params(to ? to : cache, batch, nullptr, keep, &p.to);
    if (rc != VS_OK) return rc;
    if (p.to.kv_heads != p.from.kv_heads || stride < max_n || (weights_out && stride_out < keep)) return VS_ERR_INVALID_ARG;
    const size_t units = static_cast<size_t>(batch) * p.from.kv_heads;
    size_t in, out;                                        // bytes of the weights: in 64 bits, or they are no array
    if (__builtin_mul_overflow(units * 4, static_cast<size_t>(stride), &in) ||
        (weights_out && __builtin_mul_overflow(units * 4, static_cast<size_t>(stride_out), &out))) return VS_ERR_INVALID_ARG;
    const Parts x = parts(batch, p.from.kv_heads, keep);
    if (!ws || ws_bytes < x.all) return VS_ERR_WORKSPACE;
    uint8_t* const base = static_cast<uint8_t*>(ws);
    p.weights = weights;
    p.weights_out = weights_out;
    p.stride = stride;
    p.stride_out = stride_out;
    p.kept = kept;
    p.lens_out = lens_out;
    p.count = reinterpret_cast<int32_t*>(base);
    p.index = reinterpret_cast<int32_t*>(base + x.index);
    p.keep = static_cast<int>(keep);
    p.n_sink = static_cast<int>(n_sink);
    p.n_recent = static_cast<int>(n_recent);
    p.blocks = static_cast<int>((keep + kBlock - 1) / kBlock);
    p.same = p.from.data == p.to.data && p.from.table == p.to.table && p.from.page_blocks == p.to.page_blocks && p.from.max_pages == p.to.max_pages;
    const bool one_memory = meet(p.from.data, static_cast<size_t>(p.from.pages) * p.from.kv_heads * p.from.head_bytes, p.to.data,
                                 static_cast<size_t>(p.to.pages) * p.to.kv_heads * p.to.head_bytes);
    p.block_stage = one_memory ? base + x.blocks : nullptr;
    p.weight_stage = weights_out && meet(weights, in, weights_out, out) ? reinterpret_cast<float*>(base + x.weights) : nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(select_kernel, dim3(static_cast<unsigned>(units)), dim3(kSelectThreads), 0, s, p);
    VS_LAUNCH_CHECK();
    hipLaunchKernelGGL(gather_kernel, dim3(p.blocks, static_cast<unsigned>(units)), dim3(kThreads), 0, s, p);
    VS_LAUNCH_CHECK();
    if (p.block_stage || p.weight_stage) {
        hipLaunchKernelGGL(put_kernel, dim3(p.blocks, static_cast<unsigned>(units)), dim3(kThreads), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    return VS_OK;
}
