// kv_append.hip -- a step's new keys and values into the pool, rotated on the
// way, and the upload of a batch's tables.
//
// Each token's heads are independent rows of D values: queries and keys are
// rotated, keys and values rounded to the pool's type and written to their slot.
// Bound by memory: a row is read once and written once.  A lane makes 8 values
// (16 bytes in, so that a wave reads whole lines), and for pairs (j, j + R/2) reads
// the 8 partners as well, which the row's other half of lanes has just fetched into
// the cache.  The lanes of a row are in one wave, whose loads all end before its
// stores begin, so q may be rotated in place.  A workgroup takes one token's rows,
// all or, where there are few tokens, some of them: a lane's cosines and sines are
// loaded once for all the heads that it turns.
#include <algorithm>

#include "kv_device.h"

namespace aqua {
namespace {

using namespace kv;

// Tokens from which a workgroup takes all of a token's heads.  Measured with 80 rows of
// 128 a token, whole against a workgroup for every 16 rows: 256 tokens 5.7 against
// 4.2 us, 512 7.3 against 7.7, 1024 9.9 against 11.1, 4096 37 against 44.
constexpr uint32_t kWholeTokens = 512;

template <int CTRL>
__device__ inline float quad(float x) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// a / b from b's correctly rounded reciprocal: one correction of the product gives the
// correctly rounded quotient (Markstein, "Computation of elementary functions on the
// IBM RISC System/6000 processor", 1990), so that a value halfway between two codes
// is found there.  Three instructions instead of a division's ten: thirteen prompts of 17
// to 3001 tokens into a 4-bit pool took 39 instead of 42 us.  a * inverse is finite.
__device__ inline float quotient(float a, float b, float inverse) {
    const float q = a * inverse;
    return __builtin_fmaf(__builtin_fmaf(-q, b, a), inverse, q);
}

// 8 values of a row as a 4-bit pool holds them: the lane's word of codes and, in
// every lane of the group's four, the pair.  fp32 throughout; a value halfway between two
// codes goes to the even one.
__device__ inline uint32_t to_int4(const float (&in)[8], uint32_t* pair) {
    float x[8], lo = __builtin_inff(), hi = -__builtin_inff();
    float nan = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        nan = in[i] != in[i] ? 1.0f : nan;
        x[i] = fminf(fmaxf(in[i], -16384.0f), 16384.0f);
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
    }
    lo = fminf(lo, quad<0xb1>(lo));
    lo = fminf(lo, quad<0x4e>(lo));
    hi = fmaxf(hi, quad<0xb1>(hi));
    hi = fmaxf(hi, quad<0x4e>(hi));
    nan = fmaxf(nan, quad<0xb1>(nan));
    nan = fmaxf(nan, quad<0x4e>(nan));
    const f16 s16 = (f16)((hi - lo) / 15.0f);
    const float scale = (float)s16;
    const f16 b16 = (f16)(lo - scale * 16.0f);
    const float base = (float)b16, step = scale > 0.0f ? scale : 1.0f;
    const float inverse = 1.0f / step;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = __builtin_rintf(quotient(x[i] - base, step, inverse)) - 16.0f;
        w |= (uint32_t)fminf(fmaxf(c, 0.0f), 15.0f) << ((i & 1) * 16 + (i >> 1) * 4);
    }
    const f16x2 p = {nan > 0.0f ? (f16)__builtin_nanf("") : s16, b16};
    *pair = __builtin_bit_cast(uint32_t, p);
    return w;
}

__device__ inline float to_range8(float x) {
    return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f);
}

template <typename Q>
__device__ inline void load8(const uint8_t* p, float (&x)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = lo_float<Q>(w[i]);
        x[2 * i + 1] = hi_float<Q>(w[i]);
    }
}

// Rotation without fused multiply-adds: products and their sum each rounded.
template <typename Q>
__device__ inline void rotate(float (&x)[8], const uint8_t* row, uint32_t at, uint32_t half,
                              bool interleaved, const float (&co)[8], const float (&si)[8]) {
#pragma clang fp contract(off)
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * co[i] - b * si[i];
            x[2 * i + 1] = b * co[i] + a * si[i];
        }
        return;
    }
    float y[8];
    const bool first = at < half;
    load8<Q>(row + 2 * (first ? at + half : at - half), y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float p = x[i] * co[i], r = y[i] * si[i];
        x[i] = first ? p - r : p + r;
    }
}

template <int POOL, typename Q>
__global__ __launch_bounds__(256) void append_kernel(const KvAppend a, const uint32_t parts) {
    const uint32_t tok = blockIdx.x / parts, part = blockIdx.x % parts;
    if (tok >= a.t.head->append_tokens) return;
    const KvToken where = a.t.tokens[tok];
    if (a.rope && where.position >= a.rope_rows) return;
    const uint32_t D = a.layer.D, H = a.layer.H;
    const uint32_t lanes = D / 8, per = 256 / lanes;
    const uint32_t at = threadIdx.x % lanes * 8;    // first of the lane's values in a row
    const uint32_t half = a.rope_dim / 2;
    const bool turns = a.rope && at < a.rope_dim;
    float co[8], si[8];
    if (turns) {
        const float* r = a.rope + (uint64_t)where.position * a.rope_dim;
        const uint32_t j = a.interleaved ? at / 2 : at % half;
        const int n = a.interleaved ? 4 : 8;
#pragma unroll
        for (int i = 0; i < 8; i += 4)
            if (i < n) {
                const f32x4 c = *reinterpret_cast<const f32x4*>(r + j + i);
                const f32x4 s = *reinterpret_cast<const f32x4*>(r + half + j + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    co[i + e] = c[e];
                    si[i + e] = s[e];
                }
            }
    }
    uint8_t* const chunk = a.layer.base + (uint64_t)where.block * a.layer.chunk_bytes;
    const uint32_t slot = where.position & (a.layer.T - 1);
    const uint32_t heads = a.q_heads + 2 * H;
    for (uint32_t h = part * per + threadIdx.x / lanes; h < heads; h += parts * per) {
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + H;
        const uint32_t own = is_q ? h : is_v ? h - a.q_heads - H : h - a.q_heads;
        const uint64_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
        const uint8_t* row = (is_q ? a.q : is_v ? a.v : a.k) + 2 * (tok * stride + own * D);
        float x[8];
        load8<Q>(row + 2 * at, x);
        if (turns && !is_v) rotate<Q>(x, row, at, half, a.interleaved, co, si);
        if (is_q || POOL == kF16 || POOL == kBF16) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2<Q>(x[2 * i], x[2 * i + 1]);
            uint8_t* to = is_q ? a.q_out + 2 * (tok * a.q_out_stride + own * D + at)
                               : chunk + 2 * (((is_v ? H : 0) + own) * a.layer.T + slot) * D + 2 * at;
            *reinterpret_cast<u32x4*>(to) = w;
            continue;
        }
        const uint32_t r = ((is_v ? H : 0) + own) * a.layer.T + slot;   // row of the chunk
        if constexpr (POOL == kFP8) {
            const float scale = is_v ? a.v_scale : a.k_scale;
            if (scale >= 0x1p-100f && scale <= 0x1p100f) {
                const float inverse = 1.0f / scale;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float q = x[i] * inverse;   // infinite or NaN: what it is
                    x[i] = __builtin_isfinite(q) ? quotient(x[i], scale, inverse) : q;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] / scale;
            }
            u32x2 w;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int v = __builtin_amdgcn_cvt_pk_fp8_f32(to_range8(x[4 * i]), to_range8(x[4 * i + 1]),
                                                        0, false);
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
                    to_range8(x[4 * i + 2]), to_range8(x[4 * i + 3]), v, true);
            }
            *reinterpret_cast<u32x2*>(chunk + (uint64_t)r * D + at) = w;
        }
        if constexpr (POOL == kInt4) {
            uint32_t pair;
            const uint32_t w = to_int4(x, &pair);
            *reinterpret_cast<uint32_t*>(chunk + (uint64_t)r * (D / 2) + at / 2) = w;
            uint8_t* const pairs = chunk + (uint64_t)2 * H * a.layer.T * (D / 2);
            if (at % 32 == 0)
                *reinterpret_cast<uint32_t*>(pairs + 4 * ((uint64_t)r * (D / 32) + at / 32)) = pair;
        }
    }
}

__global__ __launch_bounds__(256) void upload_kernel(const KvUpload u) {
    for (uint32_t p = 0; p < KvUpload::kPieces; ++p)
        for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < u.piece[p].n; i += gridDim.x * 256u)
            u.piece[p].dst[i] = u.piece[p].src[i];
}

template <int POOL, typename Q>
hipError_t append(const KvAppend& a, uint32_t tokens, hipStream_t stream) {
    const uint32_t per = 256 / (a.layer.D / 8), heads = a.q_heads + 2 * a.layer.H;
    // (Fewer than 2^32 threads in all.)
    const uint32_t parts =
        tokens >= kWholeTokens ? 1 : std::min<uint32_t>((heads + per - 1) / per, 8192);
    (void)hipGetLastError();
    hipLaunchKernelGGL((append_kernel<POOL, Q>), dim3(tokens * parts), dim3(256), 0, stream, a,
                       parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const KvAppend& a, const KvCounts& n, hipStream_t stream) {
    if (!n.tokens) return hipSuccess;
    const bool half = a.dtype == AQUA_F16;
    switch (a.layer.dtype) {
        case AQUA_F16: return append<kF16, f16>(a, n.tokens, stream);
        case AQUA_BF16: return append<kBF16, bf16>(a, n.tokens, stream);
        case AQUA_FP8_E4M3:
            return half ? append<kFP8, f16>(a, n.tokens, stream)
                        : append<kFP8, bf16>(a, n.tokens, stream);
        default:
            return half ? append<kInt4, f16>(a, n.tokens, stream)
                        : append<kInt4, bf16>(a, n.tokens, stream);
    }
}

hipError_t launch_upload(const KvUpload& u, hipStream_t stream) {
    uint32_t most = 0;
    for (const auto& p : u.piece) most = p.n > most ? p.n : most;
    if (!most) return hipSuccess;
    const uint32_t grid = (most + 255) / 256;
    (void)hipGetLastError();
    hipLaunchKernelGGL(upload_kernel, dim3(grid < 256 ? grid : 256), dim3(256), 0, stream, u);
    return hipGetLastError();
}

}  // namespace aqua
