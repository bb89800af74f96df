// Norm of queries and keys per head and rotary embedding in one pass, from a layer's projection (token-major, strided) to the
// library's layout [batch, heads, rows, 128]:
//   y = x w / sqrt(mean(x^2) + eps) over the 128 elements of a head (w optional), then on the first rot_dim elements
//   (a, b) -> magnitude (a cos t - b sin t, a sin t + b cos t),  t = position * freq[plane],
// rounded once to bf16; the values are copied to the same layout where they are asked for.
//
// 16 lanes hold a row, eight elements each, as two 8-byte pieces: lanes below rot_dim / 8 have whole planes 4 l .. 4 l + 3 (with half
// pairing the pieces are rot_dim / 2 apart), the others plain elements, so that a rotation needs no lane's neighbour.  The angle
// is reduced to a fraction of a turn in fp64, its sine and cosine are fp32.  Before its rounding an element is within 2^-19 of |a| + |b|, the rotated pair, for
// |position * freq| up to 2^31: 3 * 2^-53 of the angle from the reduction (2^-20.4 there, nothing at 2^20), 2 pi 2^-26 where the fraction
// becomes fp32, 2^-23 of sine and cosine, fewer than 13 roundings of 2^-24 in norm, weights, magnitude and products; 2^11 times finer than
// the rounding to bf16.  The angles serve all heads of a position that a thread walks over.
// A head's row costs a norm and four products a plane: the weights are folded into the angles' sines and cosines.
// Bound by the memory: every element is read and written once.  131072 positions of 32 / 8 heads 675 us (4.8 TB/s; a large copy reaches 5.1),
// with one row's loads in flight, weights apart and all parts in one loop 860.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "vs_common.h"
#include "vs_wave.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPositions = kThreads / 16;      // of a workgroup
constexpr int kBatch = 4;                      // heads of a position whose loads are in flight together

struct Part {                                  // q, k or v
    const uint16_t* x;
    uint16_t* out;
    const float* w;                            // null: no norm
    int64_t token, head;                       // strides of x in elements
    int heads;
    int groups, per;                           // workgroups that share the heads, heads of each
    int plain;                                 // copied as it is
};

struct NormRopeParams {
    Part part[3];
    uint32_t tokens, rows;                     // batch * rows, rows per sequence
    const int32_t* lens;
    int64_t pos0;
    const double* freq;
    int rot_dim, pairing;
    float eps, magnitude;
};

__device__ __forceinline__ float row16_sum(float x) {
    auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x += dpp(x, std::integral_constant<int, 0xB1>{});
    x += dpp(x, std::integral_constant<int, 0x4E>{});
    x += dpp(x, std::integral_constant<int, 0x141>{});
    x += dpp(x, std::integral_constant<int, 0x140>{});
    return x;
}

// one row: norm, then the planes (x, y) -> (x ca - y sb, x sa + y cb) where ca .. sb are cosine and sine times the weights of x and y
struct Turn {
    float ca[4], cb[4], sa[4], sb[4];
};

template <bool PAIRED_HALVES>
__device__ __forceinline__ void norm_turn(uint2& u0, uint2& u1, const Turn& t, bool norm, float eps, bool turned) {
    float e[8];
    const uint32_t word[4] = {u0.x, u0.y, u1.x, u1.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[2 * i] = __uint_as_float(word[i] << 16);
        e[2 * i + 1] = __uint_as_float(word[i] & 0xffff0000u);
    }
    float inv = 1.0f;
    if (norm) {
        float sum = 0.0f, other = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            sum = fmaf(e[i], e[i], sum);
            other = fmaf(e[i + 1], e[i + 1], other);
        }
        sum = row16_sum(sum + other);
        inv = rsqrtf(fmaf(sum, 1.0f / 128.0f, eps));
        if (!(sum < INFINITY)) {                  // squares past fp32: again with the row scaled down (eps is nothing beside it)
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] *= 8.470329472543003e-22f;                              // 2^-70
                sum = fmaf(e[i], e[i], sum);
            }
            inv = rsqrtf(row16_sum(sum) * (1.0f / 128.0f));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float& a = PAIRED_HALVES ? e[i] : e[2 * i];
        float& b = PAIRED_HALVES ? e[4 + i] : e[2 * i + 1];
        const float x = a * inv, y = b * inv;
        a = x * t.ca[i];
        b = y * t.cb[i];
        if (turned) {
            a = fmaf(-y, t.sb[i], a);
            b = fmaf(x, t.sa[i], b);
        }
    }
    u0 = make_uint2(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]));
    u1 = make_uint2(pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7]));
}

// Workgroup (x, y): 16 positions, the y-th group of heads of q, k or v.
template <bool PAIRED_HALVES>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRopeParams p) {
    const int l = threadIdx.x & 15;
    const uint32_t t = blockIdx.x * kPositions + (threadIdx.x >> 4);
    if (t >= p.tokens) return;
    int group = blockIdx.y, which = 0;
    while (group >= p.part[which].groups) group -= p.part[which++].groups;
    const Part part = p.part[which];
    const uint32_t b = t / p.rows, r = t - b * p.rows;
    const bool turned = 8 * l < p.rot_dim;
    // the two pieces of four elements
    const int at0 = turned && PAIRED_HALVES ? 4 * l : 8 * l;
    const int at1 = turned && PAIRED_HALVES ? p.rot_dim / 2 + 4 * l : 8 * l + 4;
    const int h0 = group * part.per, h1 = min(h0 + part.per, part.heads);
    const uint16_t* x = part.x + t * part.token;
    uint16_t* out = part.out + (static_cast<int64_t>(b) * part.heads * p.rows + r) * 128;
    const int64_t out_head = static_cast<int64_t>(p.rows) * 128;

    uint2 u[kBatch][2];
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint16_t* from = x + min(h + j, part.heads - 1) * part.head;
            u[j][0] = *reinterpret_cast<const uint2*>(from + at0);
            u[j][1] = *reinterpret_cast<const uint2*>(from + at1);
        }
    };
    auto store = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (h + j < h1) {
                uint16_t* to = out + (h + j) * out_head;
                *reinterpret_cast<uint2*>(to + at0) = u[j][0];
                *reinterpret_cast<uint2*>(to + at1) = u[j][1];
            }
    };
    load(h0);                                      // requested before the angles are evaluated
    Turn turn;
    if (!part.plain) {
        float w0[4] = {1.0f, 1.0f, 1.0f, 1.0f}, w1[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        if (part.w) {
            const float4 a = *reinterpret_cast<const float4*>(part.w + at0), c = *reinterpret_cast<const float4*>(part.w + at1);
            w0[0] = a.x, w0[1] = a.y, w0[2] = a.z, w0[3] = a.w;
            w1[0] = c.x, w1[1] = c.y, w1[2] = c.z, w1[3] = c.w;
        }
        double pos = 0.0;
        if (turned) pos = static_cast<double>(p.lens ? static_cast<int64_t>(p.lens[b]) - p.rows + r : p.pos0 + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s = 0.0f, c = 1.0f;
            if (turned) {
                const double turns = pos * p.freq[4 * l + i] * 0.15915494309189533577;   // 1 / (2 pi)
                sincospif(2.0f * static_cast<float>(turns - rint(turns)), &s, &c);
                c *= p.magnitude;
                s *= p.magnitude;
            }
            const float wa = PAIRED_HALVES ? w0[i] : i < 2 ? w0[2 * i] : w1[2 * i - 4];
            const float wb = PAIRED_HALVES ? w1[i] : i < 2 ? w0[2 * i + 1] : w1[2 * i - 3];
            turn.ca[i] = c * wa;
            turn.sa[i] = s * wa;
            turn.cb[i] = c * wb;
            turn.sb[i] = s * wb;
        }
    }
    for (int h = h0;;) {
        if (!part.plain) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) norm_turn<PAIRED_HALVES>(u[j][0], u[j][1], turn, part.w, p.eps, turned);
        }
        store(h);
        h += kBatch;
        if (h >= h1) break;
        load(h);
    }
}

}  // namespace

extern "C" int vs_rope_frequencies(double theta_base, int rot_dim, int scaling, double factor, double low, double high, double original,
                                   double* freq_host) {
    if (!freq_host || !(theta_base > 1.0) || !isfinite(theta_base)) return VS_ERR_INVALID_ARG;
    if (rot_dim < 8 || rot_dim > VS_HEAD_DIM || rot_dim % 8) return VS_ERR_UNSUPPORTED;
    if (scaling < 0 || scaling > 2) return VS_ERR_INVALID_ARG;
    if (scaling && (!(factor >= 1.0) || !isfinite(factor))) return VS_ERR_INVALID_ARG;
    if (scaling == 2 && (!(low > 0.0) || !(high > low) || !isfinite(high) || !(original > 0.0) || !isfinite(original))) return VS_ERR_INVALID_ARG;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(theta_base, -2.0 * i / rot_dim);
        if (scaling == 1) {
            f /= factor;
        } else if (scaling == 2) {
            double keep = (original * f / 6.283185307179586477 - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f *= (1.0 - keep) / factor + keep;
        }
        freq_host[i] = f;
    }
    return VS_OK;
}

extern "C" int vs_qk_norm_rope(const vs_rows_t* q, const vs_rows_t* k, const vs_rows_t* v, int batch, int64_t rows, int q_heads, int kv_heads,
                               const float* w_q, const float* w_k, float eps, const vs_rotation_t* rotation, const int32_t* lens,
                               int64_t pos0, void* q_out, void* k_out, void* v_out, void* stream) {
    if (!q || !k || !rotation || !q_out || !k_out || (v == nullptr) != (v_out == nullptr)) return VS_ERR_INVALID_ARG;
    if (batch <= 0 || rows <= 0 || q_heads <= 0 || kv_heads <= 0 || pos0 < 0) return VS_ERR_INVALID_ARG;
    if (!vs::aligned16(q_out) || !vs::aligned16(k_out) || !vs::aligned16(v_out) || !vs::aligned16(w_q) || !vs::aligned16(w_k) ||
        !vs::aligned4(lens)) return VS_ERR_INVALID_ARG;
    if ((w_q || w_k) && !(eps >= FLT_MIN && eps <= 1.0f)) return VS_ERR_INVALID_ARG;
    if (!rotation->freq || !vs::aligned16(rotation->freq) || !isfinite(rotation->magnitude)) return VS_ERR_INVALID_ARG;
    if (rotation->pairing != 0 && rotation->pairing != 1) return VS_ERR_INVALID_ARG;
    const vs_rows_t* in[3] = {q, k, v};
    for (const vs_rows_t* x : in) {
        if (!x) continue;
        if (!x->data || !vs::aligned16(x->data) || x->token_stride < VS_HEAD_DIM || x->head_stride < VS_HEAD_DIM) return VS_ERR_INVALID_ARG;
        if (x->token_stride % 8 || x->head_stride % 8) return VS_ERR_INVALID_ARG;
    }
    if (rotation->rot_dim < 8 || rotation->rot_dim > VS_HEAD_DIM || rotation->rot_dim % 8) return VS_ERR_UNSUPPORTED;
    if (pos0 > (1ll << 31) - rows) return VS_ERR_UNSUPPORTED;      // (with freq <= 1 the angle's reduction keeps 2^-20)
    if (rows > VS_MAX_SEQ || batch > 65535 || static_cast<int64_t>(batch) * rows > (1 << 26) || q_heads > 4096 || kv_heads > 4096) return VS_ERR_UNSUPPORTED;

    NormRopeParams p;
    const float* w[3] = {w_q, w_k, nullptr};
    void* out[3] = {q_out, k_out, v_out};
    for (int i = 0; i < 3; ++i) {
        p.part[i].x = in[i] ? static_cast<const uint16_t*>(in[i]->data) : nullptr;
        p.part[i].token = in[i] ? in[i]->token_stride : 0;
        p.part[i].head = in[i] ? in[i]->head_stride : 0;
        p.part[i].out = static_cast<uint16_t*>(out[i]);
        p.part[i].w = w[i];
        p.part[i].plain = i == 2;
        p.part[i].heads = i == 0 ? q_heads : in[i] ? kv_heads : 0;
    }
    p.tokens = static_cast<uint32_t>(batch * rows);
    p.rows = static_cast<uint32_t>(rows);
    p.lens = lens;
    p.pos0 = pos0;
    p.freq = rotation->freq;
    p.rot_dim = rotation->rot_dim;
    p.pairing = rotation->pairing;
    p.magnitude = rotation->magnitude;
    p.eps = eps;
    const unsigned blocks = (p.tokens + kPositions - 1) / kPositions;
    // Short calls: the heads are shared out over about two workgroups per compute unit, whole batches of heads together; every
    // workgroup evaluates the angles of its positions.  One workgroup over all heads / shared out: 16 x 1 position, 32 / 8 heads 33.6 / 4.2 us,
    // 4099 positions 92 / 22.7 (2048 workgroups 23.7, 8192 26.0), 131072 positions the same; shares of whole batches / of ceil(heads / workgroups) heads:
    // 1000 positions 8.3 / 9.0, 2000 11.6 / 12.4, 33 / 11 heads x 1000 8.8 / 9.4, 16 sequences x 1 4.0 / 4.2, 700, 1500, 4099 and 32768 positions the same.
    unsigned groups = 0;
    for (Part& x : p.part) {
        const int batches = (x.heads + kBatch - 1) / kBatch;
        int64_t share = (512ll * x.heads / (q_heads + 2 * kv_heads) + blocks - 1) / blocks;
        share = share < 1 ? 1 : share > batches ? batches : share;
        x.per = batches ? static_cast<int>((batches + share - 1) / share) * kBatch : kBatch;
        x.groups = (x.heads + x.per - 1) / x.per;
        groups += x.groups;
    }
    const dim3 grid(blocks, groups);
    auto* const kernel = rotation->pairing ? norm_rope_kernel<true> : norm_rope_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}
