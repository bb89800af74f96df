// Norm of queries and keys per head and rotary embedding in one pass, from a layer's projection (token-major, strided) to the
// library's layout [batch, heads, rows, 128]:
//   y = x w / sqrt(mean(x^2) + eps) over the 128 elements of a head (w optional), then on the first rot_dim elements
//   (a, b) -> magnitude (a cos t - b sin t, a sin t + b cos t),  t = position * freq[plane],
// rounded once to bf16; the values are copied to the same layout where they are asked for.
//
// 16 lanes hold a row, eight elements each, as two 8-byte pieces: lanes below rot_dim / 8 have whole planes 4 l .. 4 l + 3 (with half
// pairing the pieces are rot_dim / 2 apart), the others plain elements, so that a rotation needs no lane's neighbour.  The angle
// is reduced to a fraction of a turn in fp64 (positions reach 2^20), its sine and cosine are fp32: within 2^-23 of the
// rotated pair's size, 2^14 times finer than a bf16 step.  They serve all heads of a position that a thread walks over.
// Bound by the memory: every element is read and written once.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "vs_common.h"
#include "vs_wave.h"

namespace {

constexpr int kThreads = 256;
constexpr int kSlots = kThreads / 16;          // rows of 128 that a workgroup holds at a time

struct Part {                                  // q, k or v
    const uint16_t* x;
    uint16_t* out;
    const float* w;                            // null: no norm
    int64_t token, head;                       // strides of x in elements
    int heads;
};

struct NormRopeParams {
    Part part[3];
    int heads;                                 // of all parts together
    int heads_per_group;                       // heads that a workgroup walks over
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

// POSITIONS positions per workgroup, 16 / POSITIONS heads of each at a time
template <int POSITIONS>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRopeParams p) {
    constexpr int kHeads = kSlots / POSITIONS;
    const int l = threadIdx.x & 15, slot = threadIdx.x >> 4;
    const uint32_t t = blockIdx.x * POSITIONS + slot % POSITIONS;
    if (t >= p.tokens) return;
    const uint32_t b = t / p.rows, r = t - b * p.rows;
    const bool turned = 8 * l < p.rot_dim;
    // the two pieces of four elements
    const int at0 = turned && p.pairing ? 4 * l : 8 * l;
    const int at1 = turned && p.pairing ? p.rot_dim / 2 + 4 * l : 8 * l + 4;

    float c[4], s[4];
    if (turned) {
        const double pos = static_cast<double>(p.lens ? static_cast<int64_t>(p.lens[b]) - p.rows + r : p.pos0 + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double turns = pos * p.freq[4 * l + i] * 0.15915494309189533577;   // 1 / (2 pi)
            const float f = static_cast<float>(turns - rint(turns));
            sincospif(2.0f * f, &s[i], &c[i]);
            c[i] *= p.magnitude;
            s[i] *= p.magnitude;
        }
    }

    const int h0 = blockIdx.y * p.heads_per_group, h1 = min(h0 + p.heads_per_group, p.heads);
    for (int hh = h0 + slot / POSITIONS; hh < h1; hh += kHeads) {
        const int which = hh < p.part[0].heads ? 0 : hh < p.part[0].heads + p.part[1].heads ? 1 : 2;
        const int h = hh - (which > 0 ? p.part[0].heads : 0) - (which > 1 ? p.part[1].heads : 0);
        const Part& part = p.part[which];
        const uint16_t* x = part.x + t * part.token + h * part.head;
        uint2 u0 = *reinterpret_cast<const uint2*>(x + at0), u1 = *reinterpret_cast<const uint2*>(x + at1);
        if (which < 2) {
            const uint32_t word[4] = {u0.x, u0.y, u1.x, u1.y};
            float e[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[2 * i] = __uint_as_float(word[i] << 16);
                e[2 * i + 1] = __uint_as_float(word[i] & 0xffff0000u);
            }
            if (part.w) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(e[i], e[i], sum);
                sum = row16_sum(sum);
                float inv = rsqrtf(fmaf(sum, 1.0f / 128.0f, p.eps));
                if (!(sum < INFINITY)) {          // squares past fp32: again with the row scaled down (eps is nothing beside it)
                    sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        e[i] *= 8.470329472543003e-22f;                              // 2^-70
                        sum = fmaf(e[i], e[i], sum);
                    }
                    inv = rsqrtf(row16_sum(sum) * (1.0f / 128.0f));
                }
                const float4 w0 = *reinterpret_cast<const float4*>(part.w + at0), w1 = *reinterpret_cast<const float4*>(part.w + at1);
                const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = e[i] * inv * w[i];
            }
            if (turned) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float& a = p.pairing ? e[i] : e[2 * i];
                    float& d = p.pairing ? e[4 + i] : e[2 * i + 1];
                    const float a0 = a, d0 = d;
                    a = fmaf(a0, c[i], -(d0 * s[i]));
                    d = fmaf(a0, s[i], d0 * c[i]);
                }
            }
            u0 = make_uint2(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]));
            u1 = make_uint2(pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7]));
        }
        uint16_t* out = part.out + ((static_cast<int64_t>(b) * part.heads + h) * p.rows + r) * 128;
        *reinterpret_cast<uint2*>(out + at0) = u0;
        *reinterpret_cast<uint2*>(out + at1) = u1;
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
    if ((w_q || w_k) && (!(eps > 0.0f) || !isfinite(eps))) return VS_ERR_INVALID_ARG;
    if (!rotation->freq || !vs::aligned16(rotation->freq) || !isfinite(rotation->magnitude)) return VS_ERR_INVALID_ARG;
    if (rotation->pairing != 0 && rotation->pairing != 1) return VS_ERR_INVALID_ARG;
    const vs_rows_t* in[3] = {q, k, v};
    for (const vs_rows_t* x : in) {
        if (!x) continue;
        if (!x->data || !vs::aligned16(x->data) || x->token_stride < VS_HEAD_DIM || x->head_stride < VS_HEAD_DIM) return VS_ERR_INVALID_ARG;
        if (x->token_stride % 8 || x->head_stride % 8) return VS_ERR_INVALID_ARG;
    }
    if (rotation->rot_dim < 8 || rotation->rot_dim > VS_HEAD_DIM || rotation->rot_dim % 8) return VS_ERR_UNSUPPORTED;
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
        p.part[i].heads = i == 0 ? q_heads : in[i] ? kv_heads : 0;
    }
    p.heads = p.part[0].heads + p.part[1].heads + p.part[2].heads;
    p.tokens = static_cast<uint32_t>(batch * rows);
    p.rows = static_cast<uint32_t>(rows);
    p.lens = lens;
    p.pos0 = pos0;
    p.freq = rotation->freq;
    p.rot_dim = rotation->rot_dim;
    p.pairing = rotation->pairing;
    p.magnitude = rotation->magnitude;
    p.eps = eps;
    constexpr int kPositions = 16;
    const unsigned blocks = (p.tokens + kPositions - 1) / kPositions;
    p.heads_per_group = p.heads;
    const dim3 grid(blocks, 1);
    hipLaunchKernelGGL(norm_rope_kernel<kPositions>, grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
    VS_LAUNCH_CHECK();
    return VS_OK;
}
