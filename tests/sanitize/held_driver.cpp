// The host side of the calls on held tokens (attention of a chunk over the 4-bit cache, weights of its tokens, eviction), compiled under AddressSanitizer
// and UndefinedBehaviorSanitizer: sizes at both ends of their ranges, and calls that are refused before anything is launched.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "vsprefill.h"

#define EXPECT(call, want) do { const long long got_ = static_cast<long long>(call); if (got_ != static_cast<long long>(want)) { \
    std::fprintf(stderr, "line %d: %s returned %lld, expected %lld\n", __LINE__, #call, got_, static_cast<long long>(want)); return 1; } } while (0)

int main() {
    alignas(16) static unsigned char buf[4096];
    void* p = buf;                      // never dereferenced by a refused call
    void* odd = buf + 4;
    const int32_t* ip = reinterpret_cast<const int32_t*>(buf);
    int32_t* op = reinterpret_cast<int32_t*>(buf);
    float* fp = reinterpret_cast<float*>(buf);

    // workspaces: none for sizes that are refused, never less for a longer bound of the lengths
    const int batches[] = {1, 2, 63, 64, 65, 512, 8191, 65535}, heads[] = {1, 4, 8, 12, 32, 33, 4096};
    const int64_t rows[] = {1, 2, 16, 17, 33, 65, 128, 129, 255, 2048, 1 << 20}, lengths[] = {1, 63, 64, 1000, 2049, 40000, 131072, 1 << 20};
    for (int b : batches)
        for (int hk : {1, 8, 11})
            for (int hq : heads)
                for (int64_t n_q : rows) {
                    size_t last[2] = {0, 0};
                    for (int64_t n : lengths) {
                        const size_t x[2] = {vs_cache_prefill_workspace(b, hq, hk, n_q, n), vs_cache_weigh_workspace(b, hq, hk, n_q, n)};
                        for (int i = 0; i < 2; ++i) {
                            if (x[i] < last[i] || x[i] % 4) return 3;
                            if (hq % hk && x[i]) return 4;
                            last[i] = x[i];
                        }
                    }
                }
    for (int b : batches)
        for (int hk : {1, 8, 11})
            for (int64_t n : lengths)
                for (int64_t keep : lengths) {
                    const size_t x = vs_cache_evict_workspace(b, hk, n, keep);
                    if (x % 4 || !x != (static_cast<int64_t>(b) * hk > 65535)) return 5;
                }
    for (int64_t bad : {int64_t{0}, int64_t{-1}, int64_t{(1 << 20) + 1}, INT64_MAX, INT64_MIN}) {
        EXPECT(vs_cache_prefill_workspace(1, 8, 8, bad, 1000), 0);
        EXPECT(vs_cache_prefill_workspace(1, 8, 8, 200, bad), 0);
        EXPECT(vs_cache_weigh_workspace(1, 8, 8, bad, 1000), 0);
        EXPECT(vs_cache_weigh_workspace(1, 8, 8, 200, bad), 0);
        EXPECT(vs_cache_evict_workspace(1, 8, bad, 10), 0);
        EXPECT(vs_cache_evict_workspace(1, 8, 1000, bad), 0);
    }
    EXPECT(vs_cache_prefill_workspace(INT32_MAX, 4096, 4096, 1 << 20, 1 << 20), 0);
    EXPECT(vs_cache_weigh_workspace(INT32_MAX, 4096, 4096, 1 << 20, 1 << 20), 0);
    EXPECT(vs_cache_evict_workspace(INT32_MAX, INT32_MAX, 1 << 20, 1), 0);

    const vs_cache_t c = {p, 8, 2, 64, ip, 4}, null = {nullptr, 8, 2, 64, ip, 4};
    vs_cache_t big = {p, INT32_MAX, 1, 1 << 20, ip, INT32_MAX};

    // attention of a chunk
    auto prefill = [&](const vs_cache_t* cache, int64_t n_q, int64_t n, float scale, size_t ws) {
        return vs_cache_prefill(p, cache, 1, 4, n_q, ip, n, scale, p, fp, p, ws, nullptr);
    };
    for (int64_t n_q : {1, 128, 129, 5000}) {
        EXPECT(prefill(nullptr, n_q, 10, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&null, n_q, 10, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&c, n_q, 257, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&c, n_q, 10, -0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&c, n_q, 10, NAN, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&c, n_q, INT64_MIN, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(prefill(&c, n_q, INT64_MAX, 0.1f, 0), VS_ERR_UNSUPPORTED);
        EXPECT(prefill(&big, n_q, 1 << 20, 0.1f, 16), VS_ERR_WORKSPACE);
    }
    EXPECT(prefill(&c, INT64_MAX, 10, 0.1f, 0), VS_ERR_UNSUPPORTED);
    EXPECT(prefill(&c, INT64_MIN, 10, 0.1f, 0), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_prefill(odd, &c, 1, 4, 200, ip, 10, 0.1f, p, fp, p, 0, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_prefill(p, &c, INT32_MAX, 4, 200, ip, 10, 0.1f, p, fp, p, 0, nullptr), VS_ERR_UNSUPPORTED);

    // weights of held tokens
    auto weigh = [&](const vs_cache_t* cache, int64_t n_q, int64_t n, float decay, float scale, size_t ws) {
        return vs_cache_weigh(p, fp, cache, 1, 4, n_q, ip, n, scale, nullptr, decay, 0, fp, 1 << 20, p, ws, nullptr);
    };
    for (int64_t n_q : {1, 17, 1000}) {
        EXPECT(weigh(nullptr, n_q, 10, 1.0f, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(weigh(&null, n_q, 10, 1.0f, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(weigh(&c, n_q, 257, 1.0f, 0.1f, 0), VS_ERR_INVALID_ARG);
        EXPECT(weigh(&c, n_q, 10, 1.0f, NAN, 0), VS_ERR_INVALID_ARG);
        EXPECT(weigh(&c, n_q, INT64_MAX, 1.0f, 0.1f, 0), VS_ERR_UNSUPPORTED);
    }
    EXPECT(weigh(&c, INT64_MAX, 10, 1.0f, 0.1f, 0), VS_ERR_UNSUPPORTED);
    EXPECT(weigh(&c, INT64_MIN, 10, 1.0f, 0.1f, 0), VS_ERR_INVALID_ARG);
    if (vs_cache_weigh_workspace(1, 4, 1, 4096, 2000) <= 16) return 6;
    EXPECT(weigh(&big, 4096, 2000, 1.0f, 0.1f, 16), VS_ERR_WORKSPACE);

    // eviction
    auto evict = [&](const vs_cache_t* from, const vs_cache_t* to, int64_t n, int64_t keep, int64_t sink, int64_t recent, size_t ws) {
        return vs_cache_evict(from, fp, 1 << 20, 1, ip, n, keep, sink, recent, to, nullptr, 0, nullptr, op, p, ws, nullptr);
    };
    EXPECT(evict(nullptr, nullptr, 100, 10, 0, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&null, nullptr, 100, 10, 0, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, &null, 100, 10, 0, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 257, 10, 0, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 100, 0, 0, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 100, 10, -1, 0, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 100, 10, 0, INT64_MIN, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 100, 10, 6, 5, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, 100, 10, INT64_MAX, INT64_MAX, 0), VS_ERR_INVALID_ARG);
    EXPECT(evict(&c, nullptr, INT64_MAX, 10, 0, 0, 0), VS_ERR_UNSUPPORTED);
    EXPECT(evict(&big, nullptr, 1 << 20, 1000, 0, 0, 16), VS_ERR_WORKSPACE);
    std::printf("run ok\n");
    return 0;
}
