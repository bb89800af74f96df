// The host side of the calls around the prefill (norm and rotation, the 4-bit cache, the attention over it), compiled under AddressSanitizer and
// UndefinedBehaviorSanitizer: sizes at both ends of their ranges, and calls that are refused before anything is launched.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "vsprefill.h"

#define EXPECT(call, want) do { const long long got_ = static_cast<long long>(call); if (got_ != static_cast<long long>(want)) { \
    std::fprintf(stderr, "line %d: %s returned %lld, expected %lld\n", __LINE__, #call, got_, static_cast<long long>(want)); return 1; } } while (0)

int main() {
    alignas(16) static unsigned char buf[4096];
    void* p = buf;                      // never dereferenced by a refused call
    void* odd = buf + 4;
    const int32_t* ip = reinterpret_cast<const int32_t*>(buf);
    const float* fp = reinterpret_cast<const float*>(buf);

    // frequencies, into arrays that end where they have to
    for (int rot = 8; rot <= 128; rot += 8)
        for (int scaling = 0; scaling < 3; ++scaling) {
            std::vector<double> f(rot / 2);
            EXPECT(vs_rope_frequencies(1e6, rot, scaling, 8.0, 1.0, 4.0, 8192.0, f.data()), VS_OK);
            for (double x : f)
                if (!(x > 0.0 && x <= 1.0)) return 2;
        }
    double one = 0.0;
    EXPECT(vs_rope_frequencies(NAN, 8, 0, 1, 1, 4, 1, &one), VS_ERR_INVALID_ARG);
    EXPECT(vs_rope_frequencies(1e6, 132, 0, 1, 1, 4, 1, &one), VS_ERR_UNSUPPORTED);
    EXPECT(vs_rope_frequencies(1e6, 8, 2, 8, 4, 1, 8192, &one), VS_ERR_INVALID_ARG);

    // sizes
    EXPECT(vs_cache_bytes(0x7fffffffll, 4096, 1 << 20), 0x7fffffffull * 4096ull * 16384ull * VS_CACHE_BLOCK_BYTES);
    EXPECT(vs_cache_bytes(1ll << 31, 1, 64), 0);
    EXPECT(vs_cache_bytes(1, 1, 96), 0);
    const int batches[] = {1, 2, 63, 64, 65, 512, 65535}, heads[] = {1, 4, 8, 32, 33, 4096}, news[] = {1, 2, 5, 17, 100, 128};
    const int64_t lengths[] = {1, 63, 64, 1000, 2049, 40000, 131072, 1 << 20};
    for (int b : batches)
        for (int hk : {1, 8, 11})
            for (int hq : heads)
                for (int n_q : news) {
                    size_t last = 0;
                    for (int64_t n : lengths) {
                        const size_t x = vs_cache_attend_workspace(b, hq, hk, n_q, n);
                        if (x < last || x % 4) return 3;
                        if (hq % hk && x) return 4;
                        last = x;
                    }
                }
    EXPECT(vs_cache_attend_workspace(1, 8, 8, 129, 1000), 0);
    EXPECT(vs_cache_attend_workspace(65535, 16, 8, 1, 1 << 20), 0);
    EXPECT(vs_cache_attend_workspace(1, 8, 8, 1, (1 << 20) + 1), 0);

    // norm and rotation
    const vs_rows_t x = {p, 128, 128}, narrow = {p, 64, 128}, null = {nullptr, 128, 128};
    vs_rotation_t t = {reinterpret_cast<const double*>(buf), 128, 0, 1.0f};
    auto norm = [&](const vs_rows_t* q, int batch, int64_t rows, float eps, int64_t pos0) {
        return vs_qk_norm_rope(q, &x, nullptr, batch, rows, 4, 1, fp, fp, eps, &t, nullptr, pos0, p, p, nullptr, nullptr);
    };
    EXPECT(norm(nullptr, 1, 1, 1e-6f, 0), VS_ERR_INVALID_ARG);
    EXPECT(norm(&null, 1, 1, 1e-6f, 0), VS_ERR_INVALID_ARG);
    EXPECT(norm(&narrow, 1, 1, 1e-6f, 0), VS_ERR_INVALID_ARG);
    EXPECT(norm(&x, 1, 1, NAN, 0), VS_ERR_INVALID_ARG);
    EXPECT(norm(&x, 1, 1, 1e-6f, INT64_MIN), VS_ERR_INVALID_ARG);
    EXPECT(norm(&x, 1, 1, 1e-6f, INT64_MAX), VS_ERR_UNSUPPORTED);
    EXPECT(norm(&x, 1, INT64_MAX, 1e-6f, 0), VS_ERR_UNSUPPORTED);
    EXPECT(norm(&x, INT32_MAX, 1 << 20, 1e-6f, 0), VS_ERR_UNSUPPORTED);

    // the cache
    vs_cache_t c = {p, 8, 2, 64, ip, 4};
    EXPECT(vs_cache_write(nullptr, p, p, 1, 1, ip, 10, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_write(&c, odd, p, 1, 1, ip, 10, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_write(&c, p, p, 1, INT64_MAX, ip, 10, nullptr), VS_ERR_UNSUPPORTED);
    EXPECT(vs_cache_write(&c, p, p, 1, 1, ip, INT64_MAX, nullptr), VS_ERR_UNSUPPORTED);
    EXPECT(vs_cache_write(&c, p, p, INT32_MAX, 1, ip, 10, nullptr), VS_ERR_UNSUPPORTED);
    EXPECT(vs_cache_read(&c, 1, 1, ip, 10, nullptr, nullptr, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_read(&c, 1, 1, ip, 257, p, p, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_attend(p, &c, 1, 4, 1, ip, 10, -1.0f, p, nullptr, p, 0, nullptr), VS_ERR_INVALID_ARG);
    EXPECT(vs_cache_attend(p, &c, 1, 4, 129, ip, 10, 0.1f, p, nullptr, p, 0, nullptr), VS_ERR_UNSUPPORTED);
    vs_cache_t big = {p, INT32_MAX, 1, 1 << 20, ip, INT32_MAX};
    EXPECT(vs_cache_attend(p, &big, 1, 4, 1, ip, 1 << 20, 0.1f, p, nullptr, p, 16, nullptr), VS_ERR_WORKSPACE);
    big.table = nullptr;
    EXPECT(vs_cache_attend(p, &big, 2, 4, 1, ip, 1 << 20, 0.1f, p, nullptr, p, 16, nullptr), VS_ERR_INVALID_ARG);
    big.page_size = INT32_MAX;
    EXPECT(vs_cache_read(&big, 1, 1, ip, 10, p, p, nullptr), VS_ERR_UNSUPPORTED);
    std::printf("run ok\n");
    return 0;
}
