// Attention of a chunk of new tokens over the 4-bit paged cache, for more rows than vs_cache_attend takes or serves well.
//   o = softmax(scale q K^T) V over the keys up to the query's own position
// A workgroup has 256 query rows of a KV head, eight row blocks of 32 (hc query heads times 8 / hc stretches of 32 tokens), two to a wavefront:
//   S^T = K Q^T (keys x rows, bf16),  O^T = V^T P^T (channels x rows, fp16), 32 x 32 x 16 matrix instructions
// A block of 64 keys is turned into 16-bit numbers in LDS by all four wavefronts: K in bf16 with its scales (exact); V in fp16.  A wavefront has the
// 32 channels of V that share scales and holds their unit 2^(R - 127), R at least the largest scale byte so far: an element is code 2^(E - R + 13), exact
// for E from R - 27 to R.  Where a value of a block lies below, or a group is not finite, all of the block stays out of the tile in these 32 channels: a bit for the block and
// the channels says so, and the unit goes over such blocks once more at its end (bf16, weights in two terms; NaN to the rows that see it).  So which of the two has a value is
// settled once, whatever R becomes behind it.  When R grows, everybody's sums are scaled.  Weights are held as 128 p (up to 2^15: the running
// maximum may be exceeded by 2^8) in fp16, 11 significant bits down to 2^-21 of the maximum, which is why V is fp16: weights of 8 bits would double the rounding error of the output.
// The rows of a K tile stand in LDS in the order (bits 3 and 4 of a key's number exchanged) in which a lane of S^T holds the weights that
// the second product wants beside one word of V's codes, eight tokens of a channel: a word becomes one 16-byte operand.
#include <float.h>

#include "vs_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kUnitRows = 256;
constexpr float kGrown = 8.0f;                             // log2 units by which a score may exceed the running maximum
constexpr float kLift = 7.0f;                              // weights are held times 2^7
constexpr float kGrownSum = 32768.0f;                      // 2^(8 + 7): no weight of a lane is larger if their sum is not
constexpr float kSafe = 1024.0f;                           // scores (log2 units) up to which a product and a difference in one rounding are good enough
constexpr int kPartFloats = kUnitRows * 128 + 1088;          // (4352 bytes more: parts a power of two apart would all begin in the same memory channels)
constexpr int kShares = 256;                               // a workgroup for every compute unit
// What a unit's start and end (about 12 us) count for in the division, in steps (1.8 us); kEmpty: all of a unit whose rows have no position (zeros).  kStart of 3 / 5 / 6 /
// 7 / 8 / 10, us: 32 / 8 heads, 1000 rows of six prompts of up to 9001 tokens - / 392 / 384 / 380 / 383 / 387, 512 of twelve of up to 3000 133 / 125 / 118 / 117 / 118 / 122,
// 2000 of four of up to 2000 102 / 89 / 82 / 83 / 81 / 83, 512 of one of 32768 250.8 / 250.1 / 249.3 / 248.6 / 251.6 / 250.9.  kEmpty of 1 / 2 / 3 / 6 (with 6): the first
// 447 / 385 / 390 / 396, 4000 rows of eight prompts of up to 4000 482 / 393 / 404 / 458.
constexpr int kStart = 7, kEmpty = 2;
constexpr int kAhead = 4;                                  // parts that are asked for at once
// Small calls: shorter shares against more parts to join.  Us with 2 / 3 / 6 / 8: 8 / 2 heads, 300 rows of 1201 26.0 / 26.5 / 30.3 / 35.0, 32 / 8 heads, 130 of 1000
// 29.6 / 28.5 / 31.9 / 35.7 (with 4 26.5 and 29.3).
constexpr int kSteps = 2;                                  // of a workgroup, if there are so few
constexpr int kTop = 13;                                   // fp16 exponent of a code with E = R: 6 * 2^13 < 65504
constexpr int kSpan = 27;                                  // E from R - 27 (2^-14 in fp16) to R

struct PrefillParams {
    CacheParams cache;
    const uint16_t* q;
    uint16_t* o;
    float* lse;
    float* part;                           // [2 shares][kPartFloats] sums, rows of 128, then [2 shares][256] (maximum, sum of weights), then [shares] Joined
    int batch, q_heads, n_q, group, hc;
    int tok, tok_blocks;                   // tokens of a unit, 256 / hc, and that in blocks
    int tiles;                             // units of a sequence's head chunk
    int heads;                             // head chunks of a sequence: kv_heads * group / hc
    int shares;
    float c;                               // scale * log2(e)
};

// ---- the work of a call in a row: steps by sequence, head chunk, unit, block, which the workgroups divide evenly ----
// A unit of sequence b has start() steps in front (its start and end cost as much) and one for each block up to its last row's position.
__device__ __forceinline__ int start(int blocks) { return blocks > 0 ? kStart : kEmpty; }

struct Sequence {
    int len, base, first;                  // base: position of row 0;  first: blocks up to row 0, may be negative
    __device__ __forceinline__ Sequence(const PrefillParams& p, int length) {
        len = length;
        base = len - p.n_q;
        first = (base + kBlock - 1) >> 6;
    }
    __device__ __forceinline__ int blocks(const PrefillParams& p, int tile) const {
        return max(tile + 1 < p.tiles ? first + (tile + 1) * p.tok_blocks : (len + kBlock - 1) >> 6, 0);
    }
    // steps of the units in front of `tile` (tile < tiles: none of them is the last one)
    __device__ __forceinline__ int64_t before(const PrefillParams& p, int tile) const {
        const int64_t z = min(max(-first, 0) / p.tok_blocks, tile), t = tile;      // units that end in front of position 0
        return kEmpty * z + kStart * (t - z) + (t - z) * first + p.tok_blocks * ((t * (t + 1) - z * (z + 1)) >> 1);
    }
    __device__ __forceinline__ int64_t steps(const PrefillParams& p) const {
        const int last = blocks(p, p.tiles - 1);
        return before(p, p.tiles - 1) + start(last) + last;
    }
};

// inclusive sum over the lanes up to this one
__device__ __forceinline__ int64_t scan64(int64_t x) {
    auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        x += static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});        // row_shr 1, 2, 4, 8
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});        // last of a row of 16 to the next row
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});        // last of the lower half to the upper
    return x;
}

__device__ __forceinline__ int64_t lane64(int64_t x, int l) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), l), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), l);
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

struct Place {
    int b = 0, head = 0, tile = 0, step = 0, blocks = 0;       // head: of the sequence's head chunks;  step: of the unit, which has start(blocks) + blocks
    int len = 0, base = 0;
    __device__ __forceinline__ void next(const PrefillParams& p) {                 // the unit behind this one
        step = 0;
        if (++tile == p.tiles) {
            tile = 0;
            if (++head == p.heads) {
                head = 0;
                if (++b < p.batch) len = cache_length_scalar(p.cache, b);
            }
        }
        enter(p);
    }
    __device__ __forceinline__ void enter(const PrefillParams& p) {
        const Sequence s(p, len);
        base = s.base;
        blocks = s.blocks(p, tile);
    }
};

// Steps of a share, and where share `share` begins (false: behind the end).
__device__ __forceinline__ bool find(const PrefillParams& p, int share, int lane, int64_t* per, int64_t* total, Place* at) {
    auto length = [&](int b) { return b < p.batch ? cache_length(p.cache, b) : 0; };
    auto steps = [&](int b, int len) { return b < p.batch ? Sequence(p, len).steps(p) : 0; };
    int len = length(lane);
    int64_t mine = steps(lane, len), upto = scan64(mine), all = lane64(upto, 63);
    for (int b = 64; b < p.batch; b += 64) all += lane64(scan64(steps(b + lane, length(b + lane))), 63);
    all *= p.heads;
    *total = all;
    *per = (all + p.shares - 1) / p.shares;
    int64_t x = *per * share;
    if (x >= all) return false;
    for (int b = 0;; b += 64) {
        if (b > 0) {
            len = length(b + lane);
            mine = steps(b + lane, len);
            upto = scan64(mine);
        }
        const int l = __popcll(__ballot(upto * p.heads <= x));
        if (l < 64) {
            at->b = b + l;
            at->len = __builtin_amdgcn_readlane(len, l);
            x -= lane64(upto - mine, l) * p.heads;
            break;
        }
        x -= lane64(upto, 63) * p.heads;
    }
    const Sequence s(p, at->len);
    const int64_t each = s.steps(p);
    at->head = all >> 31 ? static_cast<int>(x / each) : static_cast<int>(static_cast<uint32_t>(x) / static_cast<uint32_t>(each));
    x -= at->head * each;
    int low = 0, high = p.tiles - 1;
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (s.before(p, mid) <= x) low = mid;
        else high = mid - 1;
    }
    at->tile = low;
    at->step = static_cast<int>(x - s.before(p, low));
    at->enter(p);
    return true;
}

__device__ __forceinline__ float2* part_stat(const PrefillParams& p) { return reinterpret_cast<float2*>(p.part + static_cast<int64_t>(2 * p.shares) * kPartFloats); }

// The unit that a share ends and that others began, for the second kernel; parts: shares that have some of its blocks, 0: there is none.
struct Joined {
    int parts, b, head, tile, base, pad[3];
};

__device__ __forceinline__ Joined* joined(const PrefillParams& p) { return reinterpret_cast<Joined*>(part_stat(p) + static_cast<int64_t>(2 * p.shares) * kUnitRows); }

__device__ __forceinline__ float half_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const unsigned a = r[0], b = r[1];
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}

// wavefront maximum of whole numbers >= 0
__device__ __forceinline__ int wave_max_int(int x) { return __builtin_amdgcn_readfirstlane(static_cast<int>(wave_max(static_cast<float>(x)))); }

// K in LDS: chunk (eight channels) after chunk, 64 rows of 16 bytes each; a chunk's pad spreads the four chunks that four lanes write over the banks.
// V: word (eight tokens) after word, 128 channels of 16 bytes each.  Every read is 512 bytes in a row for a half of the wavefront.
constexpr int kChunkBytes = 64 * 16 + 16, kKBytes = 16 * kChunkBytes, kWordBytes = 128 * 16, kVBytes = 8 * kWordBytes;

// A block as it comes from memory.  Codes are read by the wavefront that asked for them, scales by all (wavefronts 2 and 3 ask for what 0 and 1 do).
constexpr int kRawBytes = 16384, kRing = 4;                // (a power of two: a stage's place is a shift and a mask)

struct Lds {
    uint8_t k[2][kKBytes];
    uint8_t v[2][kVBytes];
    uint8_t raw[kRing][kRawBytes];
    uint16_t scale[kThreads / 64][64];     // V's scales of a wavefront's channels in fp16, by token in the order of the words
    int unit_of[2][4];                     // R of the buffer's block
    int event[2];                          // last step (its number in the workgroup's life) that had a new R
    int any_far;                           // last step with values out of the products' range
    uint32_t far[4][VS_MAX_SEQ / kBlock / 32];             // for a wavefront's channels: a bit for every stage that has some
};

__device__ __forceinline__ int row_of_key(int key) { return (key & 0x27) | ((key >> 1) & 8) | ((key << 1) & 16); }

// Rows in front of their sequence.
__device__ __forceinline__ void no_keys(const PrefillParams& p, const Place& at, int tid) {
    const int g = at.head / (p.group / p.hc), hchunk = at.head - g * (p.group / p.hc), shift = 31 - __builtin_clz(p.hc);        // (hc is a power of two)
    const int64_t head0 = at.b * p.q_heads + g * p.group + hchunk * p.hc;
#pragma unroll
    for (int k = 0; k < kUnitRows * 16 / kThreads; ++k) {
        const int i = k * kThreads + tid, w = i >> 9, row = at.tile * p.tok + 32 * (w >> shift) + ((i >> 4) & 31);
        if (row >= p.n_q) continue;
        const int64_t r = (head0 + (w & (p.hc - 1))) * p.n_q + row;
        reinterpret_cast<uint4*>(p.o + r * 128)[i & 15] = make_uint4(0, 0, 0, 0);
        if (p.lse && (i & 15) == 0) p.lse[r] = -INFINITY;
    }
}

// A step of 64 keys x 256 rows is 64 matrix instructions of 32 cycles a wavefront, 2048 of about 3400 cycles, and the clock is at 1.9 GHz.  What stands beside them is as many
// vector instructions, 15 % of them the turning of codes into 16 bits: vs_dense_kernel, which has no codes to turn, goes over the same numbers read back at 1.36 PFLOP/s
// (2048 rows of 131072, 32 / 8 heads: 3220 us, and 136 for reading them back) where this one takes 3590 to 3790 us, 1.15 to 1.21;  512 rows 974 and 977;  512 of 32768 250.
// Small calls are bound by their start (codes on their way, the search of a share's place) and the join: 300 rows of 1201, 8 / 2 heads, 23 us for 5 us of products.
// Eight row blocks for a workgroup: the turning of a block is shared by 256 rows; 160 KB of LDS hold one workgroup, whose wavefronts have 512 registers each.
//
// Softmax, products and the turning into 16 bits in one instruction stream, written out in issue order (one wavefront a SIMD hides nothing): the two row
// blocks run half a stage apart, as in vs_dense_kernel.
//   slot X(i): matrix: scores of block 0 for stage i, P V of block 0 for stage i - 1;  vector: softmax of block 1, stage i - 1, and V of stage i to LDS
//   slot Y(i): matrix: scores of block 1 for stage i, P V of block 1 for stage i - 1;  vector: softmax of block 0, stage i, and K of stage i + 2 to LDS
// One barrier a stage, at the start of Y(i): it publishes V of stage i and K of stage i + 1, whose buffers' last readers are in front of it.
__global__ __launch_bounds__(kThreads, 1) void prefill_kernel(const PrefillParams p) {
    extern __shared__ __align__(16) unsigned char smem[];
    Lds& lds = *reinterpret_cast<Lds*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int share = blockIdx.x;
    int64_t per, total;
    Place at;
    const bool some = find(p, share, lane, &per, &total, &at);
    const int64_t mine = some ? min(per, total - per * share) : 0;
    if (tid == 0) {
        // (the first of them has the unit's first block)
        const int front = start(at.blocks);
        const bool ends = some && at.step > front && front + at.blocks - at.step <= mine;
        *(joined(p) + share) = {ends ? share + 1 - static_cast<int>((per * share - at.step + front) / per) : 0, at.b, at.head, at.tile, at.base, {0, 0, 0}};
    }
    if (tid < 2) lds.event[tid] = -1;
    if (tid == 0) lds.any_far = -1;
    for (int w = tid; w < 4 * (VS_MAX_SEQ / kBlock / 32); w += kThreads) (&lds.far[0][0])[w] = 0;

    // a thread's piece of a block: 32 channels of a key, and of V the words of eight tokens 4 c .. of two channels of the wavefront's 32
    const int key = tid >> 2, quarter = tid & 3, c = lane >> 4, m = lane & 15;
    const uint32_t k_code = 16 * tid, k_scale = kKScales + 4 * (16 * quarter + (key & 15));       // (a word: byte key / 16, the wavefront's number)
    const uint32_t scales = kKScales + 4 * (tid & 127);                    // what it asks for of the scales
    const uint32_t v_code = kVCodes + 1024 * wave + 16 * lane, v_scale = kVScales + 16 * (4 * c + wave);
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)smem));
    // buffer 0; the other one is kKBytes and kVBytes behind
    const uint32_t k_to0 = lds0 + 4 * quarter * kChunkBytes + 16 * row_of_key(key), v_to0 = lds0 + 2 * kKBytes + c * kWordBytes + 16 * (32 * wave + m);
    const uint32_t k_from0 = lds0 + half * kChunkBytes + 16 * col, v_from0 = lds0 + 2 * kKBytes + half * kWordBytes + 16 * col;
    uint32_t k_to, v_to, k_from, v_from;                                   // of the stage that is next to be written and read
    const uint32_t raw0 = lds0 + offsetof(Lds, raw);
    // the scale byte of token `lane` for the wavefront's channels, and where it goes: word (c, u), token of the word
    const uint32_t e_from = raw0 + kVScales + 16 * (4 * ((lane >> 2) & 3) + wave) + 4 * (lane >> 4) + (lane & 3);
    const uint32_t e_to = lds0 + offsetof(Lds, scale) + 128 * wave + 2 * (16 * ((lane >> 2) & 3) + 8 * (lane >> 5) + 4 * ((lane >> 4) & 1) + (lane & 3));
    const uint32_t scale_from = lds0 + offsetof(Lds, scale) + 128 * wave + 32 * c;
    typedef __attribute__((address_space(3))) u32x4* lds_u4;
    typedef __attribute__((address_space(3))) uint32_t* lds_u1;
    typedef __attribute__((address_space(3))) uint16_t* lds_h1;
    typedef __attribute__((address_space(3))) uint8_t* lds_b1;

    bf16x8 qf[2][8], kf[2][8];
    half8_t vf[4][4], pb[2][2][2];
    f32x16 sc[2][2], oacc[2][4];
    float m_run[2], l_run[2];
    u32x4 raw_k, raw_v, scale[2];          // codes of K, codes of V and their scales (tokens 0 .. 3, 16 .. 19 from 4 c on, and 32 further on)
    uint32_t raw_s;                        // K's scale
    int steps_done = 0;                    // numbers the steps for lds.event
    int64_t left = mine;

    for (; left > 0; at.next(p)) {
        const int front = start(at.blocks), end = at.step + static_cast<int>(min(left, static_cast<int64_t>(front + at.blocks - at.step)));
        left -= end - at.step;
        const int b = at.b, g = at.head / (p.group / p.hc), hchunk = at.head - g * (p.group / p.hc), len = at.len;
        const int first_block = max(at.step - front, 0), nst = max(end - front, 0) - first_block;
        if (nst == 0) {                                                    // the start alone, or (rows without a position) no more than that
            if (at.blocks == 0) no_keys(p, at, tid);
            continue;
        }
        // ---- the unit's rows ----
        int head[2], row0[2], limit[2], sure = INT32_MAX;                  // limit: last key that the lane's row sees;  sure: that every row of the wavefront sees
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            const int w = 2 * wave + rb;
            head[rb] = b * p.q_heads + g * p.group + hchunk * p.hc + w % p.hc;
            row0[rb] = at.tile * p.tok + 32 * (w / p.hc);
            const int row = min(row0[rb] + col, p.n_q - 1);                // (rows behind the last one are not stored)
            limit[rb] = max(at.base + row, 0);                             // (nor are rows in front of their sequence)
            sure = min(sure, max(at.base + min(row0[rb], p.n_q - 1), 0));
            m_run[rb] = -INFINITY;
            l_run[rb] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[rb][j][e] = 0.0f;
        }
        int unit_now[4] = {0, 0, 0, 0};                                    // R that the sums of each group are in
        int unit_mine = 0;                                                 // R of this wavefront's channels
        bool ready = false;                                                // stages without a mask need no search for a maximum

        // ---- blocks: addresses a stage and more ahead ----
        int page = first_block / p.cache.page_blocks, in_page = first_block - page * p.cache.page_blocks, ahead = 0;
        uint32_t there = 0;                                                // bit i: stage `now` + i has a page
        const uint8_t* next_at = nullptr;                                  // the block that is asked for next
        bool next_paged = false;
        auto enter_page = [&]() __attribute__((always_inline)) {
            const int entry = cache_page(p.cache, b, page);
            next_paged = len > 0 && cache_paged(p.cache, entry);
            next_at = p.cache.data + (next_paged ? cache_offset(p.cache, entry, g, in_page) : 0);
        };
        enter_page();
        auto next_block = [&]() __attribute__((always_inline)) -> const uint8_t* {
            const uint8_t* const from = next_at;
            there = there >> 1 | (next_paged ? 16u : 0u);
            if (++ahead < nst) {                                           // (behind the last stage: that one again)
                if (++in_page == p.cache.page_blocks) {
                    in_page = 0;
                    ++page;
                    enter_page();
                } else if (next_paged) {
                    next_at += kBlockBytes;
                }
            }
            return from;
        };
        auto request = [&](int st, int piece, const uint8_t* from) __attribute__((always_inline)) {       // piece 0 .. 2 of the block at `from`, for stage st
            const uint32_t to = raw0 + (st & (kRing - 1)) * kRawBytes;
            if (piece == 0) lds_load16(k_code, from, to + 1024 * wave);
            if (piece == 1) lds_load16(v_code, from, to + kVCodes + 1024 * wave);
            if (piece == 2) lds_load4(scales, from, to + kKScales + 256 * (wave & 1));
        };
        auto take_k = [&](int st) __attribute__((always_inline)) {
            const uint32_t at = raw0 + (st & (kRing - 1)) * kRawBytes;
            raw_k = *(lds_u4)(at + k_code);
            raw_s = *(lds_u1)(at + k_scale);
        };
        auto take_v = [&](int st) __attribute__((always_inline)) {
            raw_v = *(lds_u4)(raw0 + (st & (kRing - 1)) * kRawBytes + v_code);
            scale[0] = *(lds_u4)scale_from;
            scale[1] = *(lds_u4)(scale_from + 16);
        };
        auto live_of = [&](int st) __attribute__((always_inline)) { return min(len - (first_block + st) * kBlock, kBlock); };
        const uint8_t* ahead_at = nullptr;                                 // block of stage sq + 4

        // chunk i of this thread's four of K
        auto put_k = [&](int i) __attribute__((always_inline)) {
            if (i == 0) raw_s = (raw_s >> (8 * wave)) << 23;
            *(lds_u4)(k_to + i * kChunkBytes) = __builtin_bit_cast(u32x4, dequantise8(raw_k[i], __uint_as_float(raw_s)));
        };
        // Scales of stage st's V: a lane turns one token's E into fp16, 2^(E - R + 13).
        int e_of = 0;
        auto ask_scale = [&](int st) __attribute__((always_inline)) { e_of = *(lds_b1)(e_from + (st & (kRing - 1)) * kRawBytes); };
        auto put_scale = [&](int st, bool paged) __attribute__((always_inline)) {
            int x = e_of - unit_mine + kSpan + 1;                          // 1 .. 28, or V is out of the range of fp16
            bool fits = e_of != 0;
            if (__builtin_expect(__ballot(fits && static_cast<uint32_t>(x - 1) > kSpan) != 0, 0)) {
                const bool in = st < nst && lane < (paged ? live_of(st) : 0);
                const int largest = wave_max_int(in && e_of < 255 ? e_of : 0);
                if (largest > unit_mine) {
                    unit_mine = min(largest + 2, 254);
                    lds.event[st & 1] = steps_done + st;
                    x = e_of - unit_mine + kSpan + 1;
                }
                fits = in && e_of < 255 && x > 0;
                if (__ballot(in && e_of > 0 && !fits)) {                   // zeros for all of the stage: R may grow before the unit ends
                    fits = false;
                    lds.any_far = steps_done;
                    if (lane == 0) lds.far[wave][st >> 5] |= 1u << (st & 31);
                }
            }
            lds.unit_of[st & 1][wave] = unit_mine;
            *(lds_h1)e_to = static_cast<uint16_t>(fits ? x << 10 : 0);
        };
        uint32_t word[4];
        auto put_v = [&](int piece) __attribute__((always_inline)) {   // word 2 b + u (piece / 4), tokens 2 k, 2 k + 1 of its eight
            const int i = piece >> 2, k = piece & 3, u = i & 1;
            const uint32_t w = raw_v[i];
            const uint32_t of_tokens = scale[u][k];
            const half2_t s = __builtin_bit_cast(half2_t, of_tokens);
            half2_t y;
            if (k == 0) y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0);
            if (k == 1) y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
            if (k == 2) y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2);
            if (k == 3) y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
            word[k] = __builtin_bit_cast(uint32_t, y * s);
            if (k == 3) *(lds_u4)(v_to + 4 * u * kWordBytes + 256 * (i >> 1)) = u32x4{word[0], word[1], word[2], word[3]};
        };

        auto read_k = [&](int i) __attribute__((always_inline)) {  // fragment i % 8 of tile i / 8
            const u32x4 x = *(lds_u4)(k_from + 512 * (i >> 3) + 2 * kChunkBytes * (i & 7));
            kf[i >> 3][i & 7] = __builtin_bit_cast(bf16x8, x);
        };
        auto read_v = [&](int i) __attribute__((always_inline)) {  // tokens 16 (i / 4) .., channels 32 (i % 4) ..
            const u32x4 x = *(lds_u4)(v_from + 2 * kWordBytes * (i >> 2) + 512 * (i & 3));
            vf[i >> 2][i & 3] = __builtin_bit_cast(half8_t, x);
        };

        // What the products of stage st's V do not have: a new unit for the sums (in front of them), values out of their range (behind them).
        auto new_units = [&](int st) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int unit = __builtin_amdgcn_readfirstlane(lds.unit_of[st & 1][j]);
                if (unit == unit_now[j]) continue;
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[rb][j][e] = __builtin_ldexpf(oacc[rb][j][e], unit_now[j] - unit);
                unit_now[j] = unit;
            }
        };
        int event = -1;                                                    // lds.event of the stage whose P V is next
#define VS_FENCE() __builtin_amdgcn_sched_barrier(0)
        // MR: the row block whose matrix products are issued; VR = 1 - MR: the one whose softmax runs.  sq: stage whose scores are computed (HAS_Q);
        // sq - 1: stage whose P V is accumulated (HAS_P); sv: stage whose scores go through the softmax (HAS_S).
        auto slot = [&](auto mr_tag, auto has_q, auto has_p, auto has_s, bool search, int sq, int sv) __attribute__((always_inline)) {
            constexpr int MR = decltype(mr_tag)::value, VR = 1 - MR;
            constexpr bool HAS_Q = decltype(has_q)::value, HAS_P = decltype(has_p)::value, HAS_S = decltype(has_s)::value;
            auto qmfma = [&](int kk, int u) __attribute__((always_inline)) {
                if (kk == 0) {
                    f32x16 zero;
#pragma unroll
                    for (int e = 0; e < 16; ++e) zero[e] = 0.0f;
                    sc[MR][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][0], qf[MR][0], zero, 0, 0, 0);
                } else {
                    sc[MR][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][kk], qf[MR][kk], sc[MR][u], 0, 0, 0);
                }
            };
            auto pmfma = [&](int i) __attribute__((always_inline)) {       // tokens 16 (i / 4) .., channels 32 (i % 4) ..
                oacc[MR][i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i >> 2][i & 3], pb[MR][i >> 3][(i >> 2) & 1], oacc[MR][i & 3], 0, 0, 0);
            };
            if constexpr (MR == 1) {
                if constexpr (HAS_Q) ahead_at = next_block();
                asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // (stage sq + 3 is on its way)
                VS_FENCE();
            }
            if constexpr (MR == 0 && HAS_P) {
                if (__builtin_expect(__builtin_amdgcn_readfirstlane(event) == steps_done + sq - 1, 0)) new_units(sq - 1);
                VS_FENCE();
            }
            // Softmax elements as a three-deep pipeline: step k scales element k, takes the exponential of element k - 1 and adds element k - 2 to the row
            // sum (packing a finished pair): no instruction uses the result of its predecessor.
            float mc = 0.0f, lsum = 0.0f;
            float tq[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            int estep = 0;
            auto pack_pair = [&](int u, int e, float x0, float x1) __attribute__((always_inline)) {       // weights of elements e - 1 and e
                const f32x2 two = {x0, x1};
                uint32_t packed = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, half2_t));
                asm volatile("" : "+v"(packed));
                const half2_t r = __builtin_bit_cast(half2_t, packed);
                pb[VR][u][e >> 3][(e & 7) - 1] = r[0];
                pb[VR][u][e >> 3][e & 7] = r[1];
            };
            auto expstep = [&]() __attribute__((always_inline)) {
                if constexpr (HAS_S) {
                    const int k = estep;
                    if (k < 32) {
                        float t = fmaf(sc[VR][k >> 4][k & 15], p.c, -mc);
                        asm volatile("" : "+v"(t));
                        tq[k & 3] = t;
                    }
                    if (k >= 1 && k <= 32) {
                        float x = tq[(k - 1) & 3];
                        x = __builtin_amdgcn_exp2f(x);
                        asm volatile("" : "+v"(x));
                        tq[(k - 1) & 3] = x;
                    }
                    if (k >= 2 && k <= 33) {
                        const int idx = k - 2, u = idx >> 4, e = idx & 15;
                        lsum += tq[idx & 3];
                        asm volatile("" : "+v"(lsum));
                        if (e & 1) pack_pair(u, e, tq[(idx - 1) & 3], tq[idx & 3]);
                    }
                    ++estep;
                }
            };
            auto expsteps_upto = [&](int target) __attribute__((always_inline)) {
                while (estep < target) expstep();
            };
            auto exp_share = [&](int j) __attribute__((always_inline)) {   // behind matrix instruction j
                expsteps_upto(min(34, ((j + 1) * 34 + 30) / 31));
            };
            // what goes to LDS, behind matrix instruction j
            auto turn = [&](auto index) __attribute__((always_inline)) {
                constexpr int j = decltype(index)::value;
                if constexpr (HAS_Q && MR == 0) {
                    if constexpr (j == 0) take_v(sq);
                    if constexpr (j >= 14 && j < 30) put_v(j - 14);
                    if constexpr (j == 30) v_to = 2 * v_to0 + kVBytes - v_to;
                }
                if constexpr (HAS_Q && MR == 1) {
                    if constexpr (j == 0) take_k(sq + 2);
                    if constexpr (j >= 4 && j < 12 && j % 2 == 0) put_k((j - 4) / 2);
                    if constexpr (j == 14) k_to = 2 * k_to0 + kKBytes - k_to;
                    if constexpr (j == 15) ask_scale(sq + 1);
                    if constexpr (j == 6 || j == 9 || j == 12) request(sq + 4, (j - 6) / 3, ahead_at);
                    if constexpr (j == 22) put_scale(sq + 1, there & 2);
                    if constexpr (j == 30) event = lds.event[sq & 1];
                }
            };
            auto rescale = [&](float mx) __attribute__((always_inline)) -> bool {
                const float m_new = fmaxf(m_run[VR], half_max(mx));
                if (!__ballot((m_new - m_run[VR]) * p.c > kGrown)) return false;
                const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m_run[VR] - m_new) * p.c);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[VR][j][e] *= alpha;
                l_run[VR] *= alpha;
                m_run[VR] = m_new;
                return true;
            };
            auto look_again = [&]() __attribute__((always_inline)) {
                if (__builtin_expect(__ballot(lsum > kGrownSum) != 0ull, 0)) {
                    float mx[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        mx[u] = sc[VR][u][0];
#pragma unroll
                        for (int e = 1; e < 16; ++e) mx[u] = fmaxf(mx[u], sc[VR][u][e]);
                    }
                    if (rescale(fmaxf(mx[0], mx[1]))) {
                        lsum = 0.0f;
#pragma unroll
                        for (int idx = 0; idx < 32; idx += 2) {
                            const int u = idx >> 4, e = idx & 15;
                            const float x0 = __builtin_amdgcn_exp2f(fmaf(sc[VR][u][e] - m_run[VR], p.c, kLift));
                            const float x1 = __builtin_amdgcn_exp2f(fmaf(sc[VR][u][e + 1] - m_run[VR], p.c, kLift));
                            lsum += x0;
                            lsum += x1;
                            pack_pair(u, e + 1, x0, x1);
                        }
                        if (__ballot(fabsf(m_run[VR]) * p.c > kSafe)) ready = false;
                    }
                }
            };
            if constexpr (HAS_S) {
                if (search) {
                    // key of element e of tile u: 32 u + 16 (e / 4 % 2) + 8 (e / 8) + 4 half + e % 4
                    const int last = there & 1u ? limit[VR] - (first_block + sv) * kBlock - 4 * half : -1;
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (32 * u + 16 * ((e >> 2) & 1) + 8 * (e >> 3) + (e & 3) > last) sc[VR][u][e] = -INFINITY;
                            mx[e & 3] = fmaxf(mx[e & 3], sc[VR][u][e]);
                        }
                    rescale(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
                    const float at_least = m_run[VR] == -INFINITY ? 0.0f : m_run[VR];
                    mc = fmaf(at_least, p.c, -kLift);
                    if (__ballot(fabsf(at_least) * p.c > kSafe)) {         // (the row's largest weight is to be 1)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int e = 0; e < 16; ++e) sc[VR][u][e] -= at_least;
                        mc = -kLift;
                    }
                } else {
                    mc = fmaf(m_run[VR], p.c, -kLift);
                }
                VS_FENCE();
            }
            static_for<16>([&](auto index) __attribute__((always_inline)) {
                constexpr int j = decltype(index)::value;
                if constexpr (HAS_Q) qmfma(j >> 1, j & 1);
                VS_FENCE();
                if constexpr (MR == 0 && HAS_P) read_v(j);
                turn(index);
                if constexpr (HAS_S) exp_share(j);
                VS_FENCE();
            });
            static_for<16>([&](auto index) __attribute__((always_inline)) {
                constexpr int j = decltype(index)::value;
                if constexpr (HAS_S && j == 15)
                    if (!search) look_again();
                if constexpr (HAS_P) pmfma(j);
                VS_FENCE();
                if constexpr (MR == 1 && HAS_Q) read_k(j);
                turn(std::integral_constant<int, 16 + j>{});
                if constexpr (HAS_S) exp_share(16 + j);
                VS_FENCE();
            });
            if constexpr (HAS_S) {
                expsteps_upto(34);
                l_run[VR] += lsum;
            }
            if constexpr (MR == 1 && HAS_Q) k_from = 2 * k_from0 + kKBytes - k_from;
            if constexpr (MR == 0 && HAS_P) v_from = 2 * v_from0 + kVBytes - v_from;
            VS_FENCE();
        };
#undef VS_FENCE

        using T = std::true_type;
        using F = std::false_type;
        using R0 = std::integral_constant<int, 0>;
        using R1 = std::integral_constant<int, 1>;

        // ---- the first blocks ----
        k_to = k_to0;
        v_to = v_to0;
        k_from = k_from0;
        v_from = v_from0;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the unit before this one is out of every buffer
#pragma unroll
        for (int st = 0; st < kRing; ++st) {
            const uint8_t* const from = next_block();
#pragma unroll
            for (int piece = 0; piece < 3; ++piece) request(st, piece, from);
        }
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            const int row = min(row0[rb] + col, p.n_q - 1);
            const uint16_t* const from = p.q + (static_cast<int64_t>(head[rb]) * p.n_q + row) * 128 + 8 * half;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                u32x4 x = *reinterpret_cast<const u32x4*>(from + 16 * j);
                asm volatile("" : "+a"(x));                                // (else it is copied from there in front of every product)
                qf[rb][j] = __builtin_bit_cast(bf16x8, x);
            }
        }
        asm volatile("s_waitcnt vmcnt(6)\n\ts_barrier" ::: "memory");           // (scales are read by all)
        ask_scale(0);
        put_scale(0, there & 2);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            take_k(st);
#pragma unroll
            for (int i = 0; i < 4; ++i) put_k(i);
            k_to = 2 * k_to0 + kKBytes - k_to;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int i = 0; i < 16; ++i) read_k(i);
        k_from = 2 * k_from0 + kKBytes - k_from;
        slot(R0{}, T{}, F{}, F{}, true, 0, 0);                              // X(0): scores of block 0
        slot(R1{}, T{}, F{}, T{}, true, 0, 0);                              // Y(0): scores of block 1; softmax of block 0
        // Y(i) and X(i + 1) have the softmax of stage i: without a mask and a search for the maximum where every row of the wavefront sees all of it and has
        // a maximum that serves already
        bool search = true;
        slot(R0{}, T{}, T{}, T{}, true, 1, 0);                             // X(1): softmax of block 1 for stage 0
        for (int i = 1; i < nst; ++i) {
            if (search) {
                const float least = fminf(m_run[0], m_run[1]), largest = fmaxf(m_run[0], m_run[1]);
                ready = __all(least * p.c >= -kSafe && largest * p.c <= kSafe);
            }
            search = !(ready && (there & 2) && (first_block + i) * kBlock + kBlock - 1 <= sure);
            slot(R1{}, T{}, T{}, T{}, search, i, i);
            slot(R0{}, T{}, T{}, T{}, search, i + 1, i);
        }
        slot(R1{}, F{}, T{}, F{}, true, nst, nst);                          // Y(nst): P V of block 1

        // ---- what the products of V do not have (and nothing that was asked for beyond the last stage is on its way any more) ----
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(lds.any_far) == steps_done, 0)) {
            for (int w = 0; 32 * w < nst; ++w) {
                const uint32_t bits_mine = __builtin_amdgcn_readfirstlane(lds.far[wave][w]);
                for (uint32_t bits = __builtin_amdgcn_readfirstlane(lds.far[0][w] | lds.far[1][w] | lds.far[2][w] | lds.far[3][w]); bits; bits &= bits - 1) {
                    const int bit = __builtin_ctz(bits), st = 32 * w + bit, live = live_of(st);
                    const bool mine = bits_mine >> bit & 1;                // (else the tile had this wavefront's channels)
                    const uint8_t* const from = cache_block(p.cache, b, g, first_block + st);     // (a block without a page has no bit)
                    raw_k = *reinterpret_cast<const u32x4*>(from + k_code);
                    raw_s = *reinterpret_cast<const uint32_t*>(from + k_scale);
                    raw_v = *reinterpret_cast<const u32x4*>(from + v_code);
                    const u32x4 raw_e = *reinterpret_cast<const u32x4*>(from + v_scale);
                    k_to = k_to0;
                    k_from = k_from0;
                    v_from = v_from0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) put_k(i);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int u = i & 1;
                        uint32_t y[4];
                        static_for<4>([&](auto k) __attribute__((always_inline)) {
                            uint32_t x[2];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const int which = 4 * u + k, E = static_cast<int>((raw_e[which >> 1] >> (8 * (2 * (which & 1) + j))) & 255);
                                const int up = E - unit_mine + kTop + 127;                        // exponent of the scale in fp32
                                const bool far = 16 * (which >> 1) + 4 * c + 2 * (which & 1) + j < live && mine && E > 0 && E < 255 && up > 0;
                                x[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw_v[i], __uint_as_float(static_cast<uint32_t>(far ? up : 127) << 23), decltype(k)::value));
                                if (!far) x[j] = 0;
                            }
                            y[k] = __builtin_amdgcn_perm(x[1], x[0], 0x07060100u);
                        });
                        *(lds_u4)(v_to0 + 4 * u * kWordBytes + 256 * (i >> 1)) = u32x4{y[0], y[1], y[2], y[3]};
                    }
                    __syncthreads();
                    static_for<2>([&](auto rb_tag) __attribute__((always_inline)) {
                        constexpr int rb = decltype(rb_tag)::value;
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) sc[rb][u][e] = 0.0f;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                read_k(8 * u + k);
                                sc[rb][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][k], qf[rb][k], sc[rb][u], 0, 0, 0);
                            }
                        }
                        const float at_least = m_run[rb] == -INFINITY ? 0.0f : m_run[rb];
                        const int last = limit[rb] - (first_block + st) * kBlock - 4 * half;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {                      // 16 tokens
                            uint32_t high[4], low[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                float x[2];
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const int e = 8 * (i & 1) + 2 * k + j;
                                    const bool seen = 32 * (i >> 1) + 16 * ((e >> 2) & 1) + 8 * (e >> 3) + (e & 3) <= last;
                                    x[j] = seen ? __builtin_amdgcn_exp2f(fmaf(sc[rb][i >> 1][e] - at_least, p.c, kLift)) : 0.0f;
                                }
                                high[k] = pack_bf16(x[0], x[1]);
                                low[k] = pack_bf16(x[0] - __uint_as_float(high[k] << 16), x[1] - __uint_as_float(high[k] & 0xffff0000u));
                            }
                            const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{high[0], high[1], high[2], high[3]});
                            const bf16x8 z = __builtin_bit_cast(bf16x8, u32x4{low[0], low[1], low[2], low[3]});
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                read_v(4 * i + j);
                                const bf16x8 y = __builtin_bit_cast(bf16x8, vf[i][j]);
                                oacc[rb][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, a, oacc[rb][j], 0, 0, 0);
                                oacc[rb][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, z, oacc[rb][j], 0, 0, 0);
                            }
                        }
                        // groups that are not finite, to the rows that see them
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int E = from[kVScales + 16 * (4 * ((lane >> 2) & 3) + j) + 4 * (lane >> 4) + (lane & 3)];      // of token `lane`
                            const uint64_t bad = __ballot(lane < live && E == 255);
                            if (bad && (first_block + st) * kBlock + __builtin_ctzll(bad) <= limit[rb])
#pragma unroll
                                for (int e = 0; e < 16; ++e) oacc[rb][j][e] = __uint_as_float(0x7fc00000u);
                        }
                    });
                    __syncthreads();
                }
            }
            __syncthreads();                                               // (every wavefront has seen the bits)
            for (int w = lane; 32 * w < nst; w += 64) lds.far[wave][w] = 0;
        }

        // ---- results ----
        const bool whole = first_block == 0 && nst == at.blocks;
        const int slot_of = 2 * share + (first_block == 0 ? 1 : 0);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            const float l = half_swap_sum(l_run[rb]);
            const int row = row0[rb] + col;
            if (row >= p.n_q) continue;
            if (whole) {
                const bool none = at.base + row < 0 || l == 0.0f;
                const float inv = none ? 0.0f : 1.0f / l;
                const int64_t r = static_cast<int64_t>(head[rb]) * p.n_q + row;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        float y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = none ? 0.0f : __builtin_ldexpf(oacc[rb][j][4 * a + i] * inv, unit_now[j] - 127 - kTop);
                        *reinterpret_cast<uint2*>(p.o + r * 128 + 32 * j + 8 * a + 4 * half) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
                    }
                if (p.lse && half == 0) p.lse[r] = none ? -INFINITY : (m_run[rb] * p.c + (log2f(l) - kLift)) * 0.69314718055994530942f;
            } else {
                // (in the order of the registers: lanes write memory in a row)
                float4* const to = reinterpret_cast<float4*>(p.part + static_cast<int64_t>(slot_of) * kPartFloats) + 16 * 64 * (2 * wave + rb) + lane;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        float y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = __builtin_ldexpf(oacc[rb][j][4 * a + i], unit_now[j] - 127 - kTop);
                        to[64 * (4 * j + a)] = make_float4(y[0], y[1], y[2], y[3]);
                    }
                if (half == 0) part_stat(p)[static_cast<int64_t>(slot_of) * kUnitRows + 32 * (2 * wave + rb) + col] = make_float2(m_run[rb] * p.c, l);
            }
        }
        steps_done += nst + 2;
    }
}

// The parts of a unit that several workgroups shared.  Workgroup (x, s): the unit that share s ends, if others began it; channels of one of its row blocks.  The
// first part stands in its share's second slot, the others in their shares' first.  WAYS 4: each wavefront takes every fourth part, their sums meet in LDS; 1: a
// wavefront takes all parts of its channels.  us with 1 / 4: 4 / 1 heads, 300 rows of 8000 (19 parts) 38.1 / 34.7, 200 of 2000 (8) 23.0 / 21.7, one head, 267 rows of 61864
// (128) 60.5 / 42.8;  32 / 8 heads, six prompts of up to 9001 (two or three; four times the workgroups find nothing to do) 398.6 / 405.5.
template <int WAYS>
__global__ __launch_bounds__(kThreads) void prefill_join_kernel(const PrefillParams p) {
    const int share = blockIdx.y;
    const Joined at = joined(p)[share];
    const int parts = at.parts, first = share + 1 - parts;
    if (parts <= 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int x0 = blockIdx.x * 4 / WAYS + (WAYS == 1 ? wave : 0), w = x0 >> 3, piece = 2 * (x0 & 7);       // and the next: channels 8 piece + 4 half ..
    const int row = at.tile * p.tok + 32 * (w / p.hc) + col;
    float m = -INFINITY, l = 0.0f;
    float4 y[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
    // adds sums z (of weights that are large by x.x, their own sum x.y)
    auto add = [&](float2 x, const float4 (&z)[2]) __attribute__((always_inline)) {
        if (x.y == 0.0f) return;                                           // (a sum that is not a number has to stay one)
        const float h = __builtin_amdgcn_exp2f(x.x - m);
        l = fmaf(x.y, h, l);
#pragma unroll
        for (int j = 0; j < 2; ++j) y[j] = make_float4(fmaf(z[j].x, h, y[j].x), fmaf(z[j].y, h, y[j].y), fmaf(z[j].z, h, y[j].z), fmaf(z[j].w, h, y[j].w));
    };
    for (int i = WAYS == 1 ? 0 : wave; i < parts; i += WAYS * kAhead) {
        float4 z[kAhead][2];
        float2 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int part = min(i + WAYS * k, parts - 1);
            const int64_t slot = part == 0 ? 2 * first + 1 : 2 * (first + part);
            x[k] = part_stat(p)[slot * kUnitRows + 32 * w + col];
            const float4* const from = reinterpret_cast<const float4*>(p.part + slot * kPartFloats) + 64 * (16 * w + piece) + lane;
            z[k][0] = from[0];
            z[k][1] = from[64];
        }
        float most = m;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + WAYS * k >= parts) x[k] = make_float2(-INFINITY, 0.0f);   // the last one again: no weight
            most = fmaxf(most, x[k].x);
        }
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - most);
        m = most;
        l *= f;
#pragma unroll
        for (int j = 0; j < 2; ++j) y[j] = make_float4(y[j].x * f, y[j].y * f, y[j].z * f, y[j].w * f);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) add(x[k], z[k]);
    }
    if constexpr (WAYS > 1) {
        __shared__ float sums[WAYS][10][64];
        const float mine[10] = {m, l, y[0].x, y[0].y, y[0].z, y[0].w, y[1].x, y[1].y, y[1].z, y[1].w};
#pragma unroll
        for (int i = 0; i < 10; ++i) sums[wave][i][lane] = mine[i];
        __syncthreads();
        if (wave != 0) return;
        l = 0.0f;
        y[0] = y[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 1; k < WAYS; ++k) m = fmaxf(m, sums[k][0][lane]);
#pragma unroll
        for (int k = 0; k < WAYS; ++k) {
            auto of = [&](int i) { return sums[k][i][lane]; };
            const float4 z[2] = {make_float4(of(2), of(3), of(4), of(5)), make_float4(of(6), of(7), of(8), of(9))};
            add(make_float2(of(0), of(1)), z);
        }
    }
    if (row >= p.n_q) return;
    const int g = at.head / (p.group / p.hc), hchunk = at.head - g * (p.group / p.hc);
    const int64_t r = static_cast<int64_t>(at.b * p.q_heads + g * p.group + hchunk * p.hc + w % p.hc) * p.n_q + row;
    const bool none = at.base + row < 0 || l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (none) y[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        *reinterpret_cast<uint2*>(p.o + r * 128 + 8 * (piece + j) + 4 * half) =
            make_uint2(pack_bf16(y[j].x * inv, y[j].y * inv), pack_bf16(y[j].z * inv, y[j].w * inv));
    }
    if (p.lse && piece == 0 && half == 0) p.lse[r] = none ? -INFINITY : (m + (log2f(l) - kLift)) * 0.69314718055994530942f;
}

bool sizes_ok(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    return batch > 0 && q_heads > 0 && kv_heads > 0 && n_q > 0 && max_n > 0 && n_q <= VS_MAX_SEQ && q_heads % kv_heads == 0 && q_heads <= 4096 &&
           max_n <= VS_MAX_SEQ && batch <= 65535 && static_cast<int64_t>(batch) * kv_heads <= 65535;
}

// p.n_q, p.group, .. and the workgroups from the sizes; steps of the longest sequences: fewer workgroups where there are few.
void plan(PrefillParams& p, int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    p.batch = batch;
    p.q_heads = q_heads;
    p.n_q = static_cast<int>(n_q);
    p.group = q_heads / kv_heads;
    p.hc = p.group % 4 == 0 ? 4 : p.group % 2 == 0 ? 2 : 1;
    p.tok = kUnitRows / p.hc;
    p.tok_blocks = p.tok / kBlock;
    p.tiles = (p.n_q + p.tok - 1) / p.tok;
    p.heads = kv_heads * (p.group / p.hc);
    const int64_t units = static_cast<int64_t>(batch) * p.heads * p.tiles;
    const int64_t steps = units * (kStart + (max_n + kBlock - 1) / kBlock);  // no fewer than there are
    const int64_t shares = (steps + kSteps - 1) / kSteps;
    p.shares = static_cast<int>(shares < kShares ? shares : kShares);
}

// Up to VS_CACHE_MAX_NEW rows vs_cache_attend's kernels start faster; this one has the cheaper step.  It takes those rows where they fill more than half of its
// units and there is work for 12 blocks of 256 rows a workgroup.  Us there / here, 32 / 8 heads: 128 rows of 8000 tokens (7.8 blocks) 34 / 48, 40 of 32768 (10) 54 / 55,
// 48 of 32768 (12) 56 / 56, 100 of 16000 (12.2) 63 / 59, 128 of 16000 (15.6) 67 / 58, 128 of 131072 363 / 263, 64 of 131072 191 / 146, 128 of four sequences of 4000
// (15.6) 66 / 44, of sixteen 193 / 100;  16 / 8 heads (units of 128 tokens), 65 rows of eight sequences of 32768 129 / 100;  8 / 8 heads (256 tokens), the same
// 82 / 101, 128 rows 115 / 107.  32 rows or fewer would win by 1.5 at best, in large batches, and lose by 3.
bool many_rows(const PrefillParams& p, int64_t max_n) {
    if (p.n_q > VS_CACHE_MAX_NEW) return true;
    const int64_t blocks = (max_n + kBlock - 1) / kBlock;
    return 2 * p.n_q > p.tok && static_cast<int64_t>(p.batch) * p.q_heads * p.n_q * blocks >= static_cast<int64_t>(12) * kUnitRows * kShares;
}

size_t part_bytes(const PrefillParams& p) { return static_cast<size_t>(p.shares) * (2 * kPartFloats * sizeof(float) + 2 * kUnitRows * sizeof(float2) + sizeof(Joined)); }

}  // namespace

extern "C" size_t vs_cache_prefill_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n) {
    if (!sizes_ok(batch, q_heads, kv_heads, n_q, max_n)) return 0;
    PrefillParams p;
    plan(p, batch, q_heads, kv_heads, n_q, max_n);
    const size_t here = many_rows(p, max_n) ? part_bytes(p) : 0;
    const size_t there = n_q <= VS_CACHE_MAX_NEW ? vs_cache_attend_workspace(batch, q_heads, kv_heads, static_cast<int>(n_q), max_n) : 0;
    return here > there ? here : there;                                      // (a smaller max_n may go there)
}

extern "C" int vs_cache_prefill(const void* q, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens, int64_t max_n,
                                float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    PrefillParams p;
    const bool sizes = cache && sizes_ok(batch, q_heads, cache->kv_heads, n_q, max_n);
    if (sizes) plan(p, batch, q_heads, cache->kv_heads, n_q, max_n);
    if (n_q > 0 && n_q <= VS_CACHE_MAX_NEW && !(sizes && many_rows(p, max_n)))
        return vs_cache_attend(q, cache, batch, q_heads, static_cast<int>(n_q), lens, max_n, scale, o, lse, ws, ws_bytes, stream);
    if (!q || !o || !vs::aligned16(q) || !vs::aligned16(o) || !vs::aligned16(lse) || !vs::aligned16(ws)) return VS_ERR_INVALID_ARG;
    p.c = scale * 1.44269504088896340736f;
    if (q_heads <= 0 || n_q <= 0 || !(scale > 0.0f) || !(p.c < INFINITY)) return VS_ERR_INVALID_ARG;
    const int rc = vs::cache_params(cache, batch, lens, max_n, &p.cache);
    if (rc != VS_OK) return rc;
    if (!sizes) return VS_ERR_UNSUPPORTED;
    if (!ws || ws_bytes < part_bytes(p)) return VS_ERR_WORKSPACE;
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.part = static_cast<float*>(ws);
    static vs::PerDeviceOnce once;
    const int set = once.run(nullptr, [](int) -> int {
        VS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&prefill_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(Lds))));
        return VS_OK;
    });
    if (set != VS_OK) return set;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(prefill_kernel, dim3(p.shares), dim3(kThreads), sizeof(Lds), s, p);
    VS_LAUNCH_CHECK();
    if (p.shares > 1) {
        const bool few = p.shares > 4 * static_cast<int64_t>(batch) * p.heads * p.tiles;       // units: more than four parts each
        if (few) hipLaunchKernelGGL(prefill_join_kernel<4>, dim3(kUnitRows / 32 * 8, p.shares), dim3(kThreads), 0, s, p);
        else hipLaunchKernelGGL(prefill_join_kernel<1>, dim3(kUnitRows / 32 * 2, p.shares), dim3(kThreads), 0, s, p);
        VS_LAUNCH_CHECK();
    }
    return VS_OK;
}
