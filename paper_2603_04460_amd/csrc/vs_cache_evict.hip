// Eviction from the 4-bit paged cache: of every sequence and KV head the first tokens, the last ones and those with the largest weights stay, in
// their order, at the front of the same cache or of another one.
// Weights become unsigned numbers in their order (first and last tokens above all, NaN below all); the smallest one that stays is found by three counts
// of 11, 11 and 10 bits, and of those that equal it the first ones stay.
//   select_kernel  up to 32768 tokens: a workgroup has a head, its keys in registers, the counts in LDS (8 us for 1088 tokens, 12 for 16384)
//   count_kernel, emit_kernel  more: workgroups share a head.  Each writes the counts of its tokens, the next kernel adds up those of the head; three
//                  counts, then the numbers are written (131072 tokens of 8 heads: 5.4, 8.2, 8.3 and 9.7 us, of each 5 to start and to read what the last left)
//   gather_kernel  a workgroup for each block of 64 tokens that stay: codes and scales of 64 tokens from wherever they are
//   put_kernel     a cache that is made smaller in place: blocks go through the workspace, so that all are read before one is written
// Moving a token moves codes, nothing is rounded again.
#include "vs_cache.h"

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kAlways = 0xffffffffu, kNever = 0;      // keys of tokens that stay in any case, and that are not there
constexpr int kBins = 2048, kRounds = 3;
// Tokens up to which one workgroup has a head.  Alone / shared, us with the tokens that stay read back: 8 heads, to 2048 tokens from 10000 22.6 / 40.5, 20000 32.5 / 41.4,
// 32768 35.3 / 41.9 (64 keys a lane would be the next), four sequences of 32768 41.9 / 48.4, 16 of 32768 86 / 113.  The more heads the more sharing costs, and past the line there
// is no other form: eight heads to 4000 tokens, not read back, 64 sequences of 32768 386, of 40000 578 (130 of them bytes).
constexpr int kAlone = 32768;
constexpr int kAtOnce = 8;                                 // blocks of a wavefront that are asked for at once
constexpr int kCountThreads = 1024, kCountBlocks = 128, kMaxChunks = 32;   // workgroups that share a head: blocks of each at least, and their number

__device__ __forceinline__ constexpr int shift_of(int round) { return round == 0 ? 21 : round == 1 ? 10 : 0; }
__device__ __forceinline__ constexpr uint32_t digit_of(uint32_t key, int round) { return (key >> shift_of(round)) & (round == 2 ? 1023u : 2047u); }

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
    int32_t* hist;                 // [kRounds][units][chunks][kBins] counts of the workgroups that share a head
    int32_t* above;                // [2][units][chunks]: tokens of a workgroup that the first and second count already let stay
    int2* state;                   // [2][units]: digits found so far, tokens still to be found
    int keep, n_sink, n_recent, blocks;
    int chunks, chunk_blocks;      // workgroups that share a head, blocks of each
    bool same;                     // `to` is `from`
};

// The token's place in the order of staying.
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return kNever + 1;
    const uint32_t x = __float_as_uint(w + 0.0f);          // (one zero)
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// Keys of R blocks from `block` on (those from `end` on have none), a token of each for every lane: all that they need is asked for at once, and waited for
// where the keys are made.
template <int R>
struct Keys {
    float w[R];
    int block, page;                                      // page of block `lane`
    bool mine;
    __device__ __forceinline__ void ask(const EvictParams& p, int b, const float* weights, int n, int from, int end, int lane) {
        block = from;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = (block + i) * kBlock + lane;
            w[i] = j < n ? weights[j] : 0.0f;
        }
        mine = lane < R && block + lane < end;
        page = 0;
        if (mine) {
            const int64_t entry = static_cast<int64_t>(b) * p.from.max_pages + (block + lane) / p.from.page_blocks;
            page = p.from.table ? p.from.table[entry] : static_cast<int>(entry);
        }
    }
    __device__ __forceinline__ void make(const EvictParams& p, int n, int lane, uint32_t (&key)[R]) const {
        const uint64_t there = __ballot(mine && cache_paged(p.from, page));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = (block + i) * kBlock + lane;
            key[i] = (there >> i & 1) == 0 || j >= n ? kNever : j < p.n_sink || j >= n - p.n_recent ? kAlways : key_of(w[i]);
        }
    }
};

// Counts in LDS: bin d at d + d / 32.  Neighbouring bins, which weights of one size go to, are in different banks, and so are the bins that the lanes read at once,
// 32 apart.
constexpr int kHist = kBins + kBins / 32;
__device__ __forceinline__ int bin_at(uint32_t d) { return static_cast<int>(d + (d >> 5)); }

struct Found {
    int digit, need, total;        // digit that the `need`-th largest key has, how many with that digit stay, how many stay in all
};

// By one wavefront: lane l has the bins 2047 - 32 l down to 2016 - 32 l.  No more than there are can be needed.
__device__ __forceinline__ Found find_digit(const int* hist, int need, int lane) {
    int sum = 0;
    const int mine = 63 - lane;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += hist[33 * mine + i];
    const int upto = wave_scan(sum);
    Found x;
    need = min(need, __builtin_amdgcn_readlane(upto, 63));
    if (need <= 0) return {0, 0, 0};
    x.total = need;
    const int l = __popcll(__ballot(upto < need));         // the lane that has it (need between 1 and the total)
    const int before = __builtin_amdgcn_readlane(upto - sum, l & 63);
    const int count = lane < 32 ? hist[33 * (63 - l) + 31 - lane] : 0;     // its bins, the largest first
    const int within = wave_scan(count);
    const int k = __popcll(__ballot(before + within < need));
    x.digit = 2047 - 32 * l - k;
    x.need = need - before - __builtin_amdgcn_readlane(within - count, k & 63);
    return x;
}

// Numbers of a wavefront's tokens that stay, ascending.  at: place of the first of them; ties: tokens in front whose key is the smallest that stays.
struct Emit {
    int32_t *index, *kept;
    uint32_t least;
    int need, at, ties;
    __device__ __forceinline__ void take(int j, uint32_t key, int lane) {
        const uint64_t below = (1ull << lane) - 1, tied = __ballot(key == least);
        const bool stays = key > least || (key == least && ties + __popcll(tied & below) < need);
        const uint64_t staying = __ballot(stays);
        if (stays) {
            const int i = at + __popcll(staying & below);
            index[i] = j;
            if (kept) kept[i] = j;
        }
        at += __popcll(staying);
        ties += __popcll(tied);
    }
};

// A wavefront has the tokens from 64 R * its number on, R of each lane.  Bound by latency: the keys, then three times counts, a barrier, a search by one wavefront
// and a barrier.  256 threads with 8 keys / 512 with 4 / 1024 with 2, us with the tokens that stay moved and read back: 600 tokens of one sequence 15.9 / 15.3 / 15.3, 64 of up to
// 1088 106.0 / 104.8 / 105.2.
template <int T, int R>
__global__ __launch_bounds__(T) void select_kernel(EvictParams p) {
    __shared__ __align__(16) int hist[kRounds][kHist];
    __shared__ int more_of[T / 64], same_of[T / 64];
    __shared__ Found found[kRounds];
    const int unit = blockIdx.x, b = unit / p.from.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = cache_length_scalar(p.from, b);
    const float* const weights = p.weights + unit * p.stride;
    uint32_t key[R];
    Keys<R> of;
    of.ask(p, b, weights, n, wave * R, (n + kBlock - 1) / kBlock, lane);
    static_assert(kRounds * kHist % 4 == 0, "");
    for (int i = threadIdx.x; i < kRounds * kHist / 4; i += T) reinterpret_cast<int4*>(hist[0])[i] = make_int4(0, 0, 0, 0);
    of.make(p, n, lane, key);
    __syncthreads();
    uint32_t prefix = 0;
    int need = p.keep, count = 0;
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (key[i] != kNever && (round == 0 || key[i] >> shift_of(round - 1) == prefix)) atomicAdd(&hist[round][bin_at(digit_of(key[i], round))], 1);
        __syncthreads();
        if (wave == 0) {
            const Found x = find_digit(hist[round], need, lane);
            if (lane == 0) found[round] = x;
        }
        __syncthreads();
        const Found x = found[round];
        if (round == 0) count = x.total;
        prefix = prefix << (round == 2 ? 10 : 11) | static_cast<uint32_t>(round == 2 ? x.digit & 1023 : x.digit);
        need = x.need;
    }
    int more = 0, same = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        more += __popcll(__ballot(key[i] > prefix));
        same += __popcll(__ballot(key[i] == prefix));
    }
    if (lane == 0) {
        more_of[wave] = more;
        same_of[wave] = same;
    }
    __syncthreads();
    Emit out;
    out.index = p.index + static_cast<int64_t>(unit) * p.keep;
    out.kept = p.kept ? p.kept + static_cast<int64_t>(unit) * p.keep : nullptr;
    out.least = prefix;
    out.need = need;
    out.at = out.ties = 0;
    for (int w = 0; w < wave; ++w) {
        out.at += more_of[w];
        out.ties += same_of[w];
    }
    out.at += min(out.ties, need);
    if (count > 0)
#pragma unroll
        for (int i = 0; i < R; ++i) out.take((wave * R + i) * kBlock + lane, key[i], lane);
    if (out.kept)
        for (int i = count + threadIdx.x; i < p.keep; i += T) out.kept[i] = -1;
    if (threadIdx.x == 0 && unit == b * p.from.kv_heads) p.count[b] = count;
}

// ---- workgroups that share a head ----
__device__ __forceinline__ int32_t* chunk_hist(const EvictParams& p, int round, int unit, int chunk) {
    return p.hist + ((static_cast<int64_t>(round) * gridDim.y + unit) * p.chunks + chunk) * kBins;
}

// The counts of a round of all of the head's workgroups into `hist`, this one's or (FRONT) those in front of it into `other`.
template <bool FRONT>
__device__ __forceinline__ void add_up(const EvictParams& p, int round, int unit, int live, int* hist, int* other) {
    static_assert(kBins == 2 * kCountThreads, "a thread has two bins");
    const int d = 2 * threadIdx.x;
    int2 sum = make_int2(0, 0), some = sum;
    for (int c = 0; c < live; c += kMaxChunks / 2) {
        int2 x[kMaxChunks / 2];
#pragma unroll
        for (int k = 0; k < kMaxChunks / 2; ++k) x[k] = *reinterpret_cast<const int2*>(chunk_hist(p, round, unit, min(c + k, live - 1)) + d);
#pragma unroll
        for (int k = 0; k < kMaxChunks / 2; ++k) {
            const bool in = FRONT ? c + k < static_cast<int>(blockIdx.x) : c + k == static_cast<int>(blockIdx.x);
            some.x += in ? x[k].x : 0;
            some.y += in ? x[k].y : 0;
            sum.x += c + k < live ? x[k].x : 0;
            sum.y += c + k < live ? x[k].y : 0;
        }
    }
    hist[bin_at(d)] = sum.x;
    hist[bin_at(d) + 1] = sum.y;                           // (an even bin and the next one stand together)
    other[bin_at(d)] = some.x;
    other[bin_at(d) + 1] = some.y;
}

// What round `round` is about: keys that begin with prefix, need of them stay.  By all threads of the workgroup; the first count's total is count.
template <bool FRONT>
__device__ __forceinline__ void find_round(const EvictParams& p, int round, int unit, int live, int* hist, int* other, Found* found, uint32_t* prefix, int* need,
                                           int* count) {
    const int lane = threadIdx.x & 63;
    int2 last = make_int2(0, p.keep);
    if (round > 0) last = p.state[(round - 1) * gridDim.y + unit];
    add_up<FRONT>(p, round, unit, live, hist, other);
    __syncthreads();
    if (threadIdx.x < 64) {
        const Found x = find_digit(hist, last.y, lane);
        if (lane == 0) *found = x;
    }
    __syncthreads();
    *prefix = static_cast<uint32_t>(last.x) << (round == 2 ? 10 : 11) | static_cast<uint32_t>(round == 2 ? found->digit & 1023 : found->digit);
    *need = found->need;
    if (round == 0) *count = found->total;
}

// sum over the workgroup of the bins of `hist` above digit
__device__ __forceinline__ int bins_above(const int* hist, int digit, int* scratch) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = 0;
    for (int d = threadIdx.x; d < kBins; d += kCountThreads)
        if (d > digit) sum += hist[bin_at(d)];
    sum = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    __syncthreads();
    if (lane == 0) scratch[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kCountThreads / 64; ++w) sum += scratch[w];
    return sum;
}

// Workgroup (chunk, unit): counts of its tokens in round ROUND; what the rounds before found is added up first.
template <int ROUND>
__global__ __launch_bounds__(kCountThreads) void count_kernel(EvictParams p) {
    __shared__ int hist[kHist], own[kHist], scratch[kCountThreads / 64];
    __shared__ Found found;
    const int unit = blockIdx.y, b = unit / p.from.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = cache_length_scalar(p.from, b), blocks = (n + kBlock - 1) / kBlock, live = (blocks + p.chunk_blocks - 1) / p.chunk_blocks;
    const int first = blockIdx.x * p.chunk_blocks, last = min(first + p.chunk_blocks, blocks);
    if (first >= last) {
        if (ROUND == 0 && blocks == 0 && blockIdx.x == 0 && threadIdx.x == 0 && unit == b * p.from.kv_heads) p.count[b] = 0;
        return;
    }
    const float* const weights = p.weights + unit * p.stride;
    Keys<kAtOnce> of;
    of.ask(p, b, weights, n, first + kAtOnce * wave, last, lane);
    uint32_t prefix = 0;
    int need = p.keep, count = 0;
    if constexpr (ROUND > 0) {
        find_round<false>(p, ROUND - 1, unit, live, hist, own, &found, &prefix, &need, &count);
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            p.state[(ROUND - 1) * gridDim.y + unit] = make_int2(static_cast<int>(prefix), need);
            if (ROUND == 1 && unit == b * p.from.kv_heads) p.count[b] = count;
        }
        const int above = bins_above(own, found.digit, scratch);
        if (threadIdx.x == 0) p.above[((ROUND - 1) * gridDim.y + unit) * p.chunks + blockIdx.x] = above;
    }
    for (int d = threadIdx.x; d < kHist; d += kCountThreads) hist[d] = 0;
    __syncthreads();
    for (int block = first + kAtOnce * wave; block < last; block += kAtOnce * (kCountThreads / 64)) {
        uint32_t key[kAtOnce];
        of.make(p, n, lane, key);
        of.ask(p, b, weights, n, block + kAtOnce * (kCountThreads / 64), last, lane);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (key[i] != kNever && (ROUND == 0 || key[i] >> shift_of(ROUND - 1) == prefix)) atomicAdd(&hist[bin_at(digit_of(key[i], ROUND))], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kBins; d += kCountThreads) chunk_hist(p, ROUND, unit, blockIdx.x)[d] = hist[bin_at(d)];
}

__global__ __launch_bounds__(kCountThreads) void emit_kernel(EvictParams p) {
    __shared__ int hist[kHist], before[kHist], scratch[kCountThreads / 64], more_of[kCountThreads / 64], same_of[kCountThreads / 64];
    __shared__ Found found;
    const int unit = blockIdx.y, b = unit / p.from.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = cache_length_scalar(p.from, b), blocks = (n + kBlock - 1) / kBlock, live = (blocks + p.chunk_blocks - 1) / p.chunk_blocks;
    const int first = blockIdx.x * p.chunk_blocks, last = min(first + p.chunk_blocks, blocks);
    // a wavefront's share of the workgroup's blocks
    const float* const weights = p.weights + unit * p.stride;
    const int each = (last - first + kCountThreads / 64 - 1) / (kCountThreads / 64), from = min(first + wave * each, last), to = min(from + each, last);
    Keys<kAtOnce> of;
    if (first < last) of.ask(p, b, weights, n, from, to, lane);
    const int count = p.count[b];
    int32_t* const kept = p.kept ? p.kept + static_cast<int64_t>(unit) * p.keep : nullptr;
    if (kept && blockIdx.x == 0)
        for (int i = count + threadIdx.x; i < p.keep; i += kCountThreads) kept[i] = -1;
    if (first >= last || count == 0) return;
    Emit out;
    {                                                      // (a lane for each workgroup in front: there are kMaxChunks at most)
        const bool front = lane < static_cast<int>(blockIdx.x);
        const int x = front ? p.above[unit * p.chunks + lane] : 0, y = front ? p.above[(gridDim.y + unit) * p.chunks + lane] : 0;
        out.at = __builtin_amdgcn_readlane(wave_scan(x + y), 63);
    }
    uint32_t prefix;
    int need, unused;
    find_round<true>(p, 2, unit, live, hist, before, &found, &prefix, &need, &unused);
    out.index = p.index + static_cast<int64_t>(unit) * p.keep;
    out.kept = kept;
    out.least = prefix;
    out.need = need;
    out.at += bins_above(before, found.digit, scratch);
    out.ties = before[bin_at(found.digit)];
    // the keys are in registers, where the wavefront has no more blocks than it asks for at once
    uint32_t key[kAtOnce];
    int more = 0, same = 0;
    for (int block = from; block < to; block += kAtOnce) {
        if (block > from) of.ask(p, b, weights, n, block, to, lane);
        of.make(p, n, lane, key);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            more += __popcll(__ballot(key[i] > prefix));
            same += __popcll(__ballot(key[i] == prefix));
        }
    }
    if (lane == 0) {
        more_of[wave] = more;
        same_of[wave] = same;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        out.at += more_of[w];
        out.ties += same_of[w];
    }
    out.at += min(out.ties, need);
    for (int block = from; block < to; block += kAtOnce) {
        if (each > kAtOnce) {
            of.ask(p, b, weights, n, block, to, lane);
            of.make(p, n, lane, key);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) out.take((block + i) * kBlock + lane, key[i], lane);
    }
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

// Blocks of which the codes of V and all scales go through LDS.  0 / 2 / 4 / 8 of them, us: 64 sequences of up to 1088 tokens to 1024, read back 114 / 107 / 106 / 123, 16 of
// 4160 to 4096 112 / 103 / 103 / 118, 12 of up to 12001 to 2000 44.3 / 44.7 / 44.8 / 49.2, one of 131072 to 16384 63 / 63 / 63 / 67 (8 take the room of other workgroups).
constexpr int kSpan = 2;
constexpr int kHeldBytes = kBlockBytes - kVCodes;

// Bound by latency and memory: the numbers, then the page table, then the codes.  1024 of up to 1088 tokens of 64 sequences 47 us, 3.1 TB/s; where few tokens of a
// block stay, the block's V is read for them (a token's codes lie in every 16 bytes of a half of it): 16384 of 131072 18 us for 90 MB.  Workgroups of a head are
// gridDim.x apart: on one XCD where the number of heads is a multiple of eight, so that a block that two of them read comes from memory once (47 against 49 us).
// K's rows come from where they are.  Of V a word is eight tokens of a channel: a thread puts its four words (two channels, 16 tokens) together from 16 pieces
// of 16 bytes, each with both channels of one token.  Where the tokens stand in no more than kSpan blocks, which is so while most of them stay, those
// blocks' codes of V and scales are read once, into LDS.
__global__ __launch_bounds__(kThreads) void gather_kernel(EvictParams p) {
    __shared__ __align__(16) uint8_t held[kSpan][kHeldBytes];
    __shared__ const uint8_t* from[kBlock];
    __shared__ int place[kBlock];
    __shared__ const uint8_t* source[kSpan];
    const int unit = blockIdx.x, b = unit / p.from.kv_heads, h = unit - b * p.from.kv_heads, block = blockIdx.y;
    const int64_t head = static_cast<int64_t>(unit) * p.keep;
    // numbers of its tokens, asked for together with how many there are (behind `count` they are whatever the workspace held, and not used)
    const int slot = block * kBlock + (threadIdx.x & (kBlock - 1));
    const int number = slot < p.keep ? p.index[head + slot] : 0;
    const int count = p.count[b];
    if (!p.block_stage && !p.weight_stage && block == 0 && h == 0 && threadIdx.x == 0) p.lens_out[b] = count;
    if (block * kBlock >= count) return;
    uint8_t* const there = cache_block(p.to, b, h, block);
    uint8_t* const to = p.block_stage ? p.block_stage + (static_cast<int64_t>(unit) * p.blocks + block) * kBlockBytes : there;
    const int tokens = min(count - block * kBlock, kBlock);
    const int j0 = __builtin_amdgcn_readfirstlane(number) / kBlock, j1 = __builtin_amdgcn_readlane(number, tokens - 1) / kBlock;     // blocks of the first and the last
    const bool still = __builtin_amdgcn_readlane(number, tokens - 1) == block * kBlock + tokens - 1;       // all tokens are where they were
    const bool near = tokens == kBlock && j1 - j0 < kSpan;
    if (threadIdx.x < kBlock) {
        const int i = slot;
        if (threadIdx.x < tokens) {
            const int j = number;
            from[threadIdx.x] = block_of_lane(p.from, b, h, j / kBlock);
            place[threadIdx.x] = (j / kBlock - j0) * kBlock + j % kBlock;
            if (p.weights_out) {
                const float w = p.weights[unit * p.stride + j];
                if (p.weight_stage) p.weight_stage[head + i] = w;
                else p.weights_out[unit * p.stride_out + i] = w;
            }
        } else {                                           // what the cache holds behind the last token stays
            from[threadIdx.x] = there;
            place[threadIdx.x] = threadIdx.x;
        }
    } else if (threadIdx.x < kBlock + kSpan) {
        const int k = threadIdx.x - kBlock;
        source[k] = near && j0 + k <= j1 ? block_of_lane(p.from, b, h, j0 + k) : nullptr;
    }
    __syncthreads();
    if (!there || (p.same && still)) return;
    const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
    const uint4 x = *reinterpret_cast<const uint4*>(from[token] + 64 * (place[token] & 63) + 16 * quarter);
    // words (channel, u) of tokens 32 u + 4 c + 0 .. 3 and 16 more: channels 32 p + m and 16 more, u = 0, 1
    const int c = (threadIdx.x >> 4) & 3, piece = 1024 * (threadIdx.x >> 6) + 16 * (threadIdx.x & 15);
    const int scale_lane = threadIdx.x & 63;
    const bool is_k = threadIdx.x < 64;                    // scales: threads 0 .. 63 of K (group g, tokens 16 k + m), 64 .. 127 of V (tokens 16 t + 4 c + k of group g)
    uint32_t w[4] = {0, 0, 0, 0}, scales = 0;
    auto put_together = [&](auto v_piece, auto byte) __attribute__((always_inline)) {
        static_for<2>([&](auto u) __attribute__((always_inline)) {         // eight tokens at once
            uint4 y[8];
            static_for<8>([&](auto e) __attribute__((always_inline)) {
                const int i = 32 * u + 16 * (e >> 2) + 4 * c + (e & 3);
                y[e] = v_piece(i, piece + 256 * ((place[i] >> 2) & 3));
            });
            static_for<8>([&](auto e) __attribute__((always_inline)) {
                const int j = place[32 * u + 16 * (e >> 2) + 4 * c + (e & 3)];
                const int shift = 4 * ((j & 3) + ((j >> 4) & 1) * 4);
                const uint32_t low = j & 32 ? y[e].y : y[e].x, high = j & 32 ? y[e].w : y[e].z;
                w[u] |= ((low >> shift) & 15u) << (4 * e);
                w[2 + u] |= ((high >> shift) & 15u) << (4 * e);
            });
        });
        if (threadIdx.x < 128) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = is_k ? 16 * k + (scale_lane & 15) : 16 * (scale_lane & 3) + 4 * (scale_lane >> 4) + k, g = is_k ? scale_lane >> 4 : (scale_lane >> 2) & 3, j = place[i] & 63;
                const int at = is_k ? kKScales + 4 * (16 * g + (j & 15)) + (j >> 4) : kVScales + 16 * (4 * ((j >> 2) & 3) + g) + 4 * (j >> 4) + (j & 3);
                scales |= static_cast<uint32_t>(byte(i, at)) << (8 * k);
            }
        }
    };
    if (near) {
        for (int i = threadIdx.x; i < (j1 - j0 + 1) * (kHeldBytes / 16); i += kThreads) {
            const int k = i / (kHeldBytes / 16), at = 16 * (i - k * (kHeldBytes / 16));
            if (source[k]) *reinterpret_cast<uint4*>(held[k] + at) = *reinterpret_cast<const uint4*>(source[k] + kVCodes + at);
        }
        __syncthreads();
        put_together([&](int i, int at) { return *reinterpret_cast<const uint4*>(held[place[i] >> 6] + at); },
                     [&](int i, int at) { return held[place[i] >> 6][at - kVCodes]; });
    } else {
        put_together([&](int i, int at) { return *reinterpret_cast<const uint4*>(from[i] + kVCodes + at); }, [&](int i, int at) { return from[i][at]; });
    }
    __syncthreads();                                       // (`to` may be where some of it was read)
    reinterpret_cast<uint4*>(to)[threadIdx.x] = x;
    reinterpret_cast<uint4*>(to + kVCodes)[threadIdx.x] = make_uint4(w[0], w[1], w[2], w[3]);
    if (threadIdx.x < 128) reinterpret_cast<uint32_t*>(to + kKScales)[threadIdx.x] = scales;
}

__global__ __launch_bounds__(kThreads) void put_kernel(EvictParams p) {
    const int unit = blockIdx.x, b = unit / p.from.kv_heads, h = unit - b * p.from.kv_heads, block = blockIdx.y;
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
    size_t index, weights, blocks, above, state, hist, all;
    int chunks, chunk_blocks;
};

Parts parts(int batch, int kv_heads, int64_t max_n, int64_t keep) {
    const size_t units = static_cast<size_t>(batch) * kv_heads, k = static_cast<size_t>(keep);
    Parts x;
    const int64_t all = (max_n + kBlock - 1) / kBlock;
    x.chunk_blocks = static_cast<int>(all > kMaxChunks * kCountBlocks ? (all + kMaxChunks - 1) / kMaxChunks : kCountBlocks);
    x.chunks = max_n <= kAlone ? 0 : static_cast<int>((all + x.chunk_blocks - 1) / x.chunk_blocks);
    x.index = vs::round_up(static_cast<size_t>(batch) * 4, 256);
    x.weights = x.index + vs::round_up(units * k * 4, 256);
    x.blocks = x.weights + vs::round_up(units * k * 4, 256);
    x.above = x.blocks + units * ((k + kBlock - 1) / kBlock) * kBlockBytes;
    x.state = x.above + vs::round_up(2 * units * kMaxChunks * 4, 256);
    x.hist = x.state + vs::round_up(2 * units * 8, 256);
    // (as many chunks as any length up to max_n has)
    x.all = x.hist + (x.chunks ? kRounds * units * static_cast<size_t>(all < kMaxChunks * kCountBlocks ? x.chunks : kMaxChunks) * kBins * 4 : 0);
    return x;
}

// do the bytes [a, a + n) and [b, b + m) meet
bool meet(const void* a, size_t n, const void* b, size_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y ? y - x < n : x - y < m;
}

}  // namespace

extern "C" size_t vs_cache_evict_workspace(int batch, int kv_heads, int64_t max_n, int64_t keep) {
    return sizes_ok(batch, kv_heads, max_n, keep) ? parts(batch, kv_heads, max_n, keep).all : 0;
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
    const Parts x = parts(batch, p.from.kv_heads, max_n, keep);
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
    p.above = reinterpret_cast<int32_t*>(base + x.above);
    p.state = reinterpret_cast<int2*>(base + x.state);
    p.hist = reinterpret_cast<int32_t*>(base + x.hist);
    p.chunks = x.chunks;
    p.chunk_blocks = x.chunk_blocks;
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
    const unsigned y = static_cast<unsigned>(units);
    if (x.chunks) {
        const dim3 grid(x.chunks, y);
        hipLaunchKernelGGL(count_kernel<0>, grid, dim3(kCountThreads), 0, s, p);
        VS_LAUNCH_CHECK();
        hipLaunchKernelGGL(count_kernel<1>, grid, dim3(kCountThreads), 0, s, p);
        VS_LAUNCH_CHECK();
        hipLaunchKernelGGL(count_kernel<2>, grid, dim3(kCountThreads), 0, s, p);
        VS_LAUNCH_CHECK();
        hipLaunchKernelGGL(emit_kernel, grid, dim3(kCountThreads), 0, s, p);
    } else if (max_n <= 2048) {
        hipLaunchKernelGGL((select_kernel<512, 4>), dim3(y), dim3(512), 0, s, p);
    } else if (max_n <= 4096) {
        hipLaunchKernelGGL((select_kernel<512, 8>), dim3(y), dim3(512), 0, s, p);
    } else if (max_n <= 8192) {
        hipLaunchKernelGGL((select_kernel<1024, 8>), dim3(y), dim3(1024), 0, s, p);
    } else if (max_n <= 16384) {
        hipLaunchKernelGGL((select_kernel<1024, 16>), dim3(y), dim3(1024), 0, s, p);
    } else {
        hipLaunchKernelGGL((select_kernel<1024, 32>), dim3(y), dim3(1024), 0, s, p);
    }
    VS_LAUNCH_CHECK();
    hipLaunchKernelGGL(gather_kernel, dim3(y, p.blocks), dim3(kThreads), 0, s, p);
    VS_LAUNCH_CHECK();
    if (p.block_stage || p.weight_stage) {
        hipLaunchKernelGGL(put_kernel, dim3(y, p.blocks), dim3(kThreads), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    return VS_OK;
}
