// kv_device.h -- what the operators' kernels share: element types, conversions,
// cross-lane sums.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "kv_ops.h"

namespace aqua {
namespace kv {

using f16 = _Float16;
using bf16 = __bf16;
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Pool element types as template arguments.
enum : int { kF16 = AQUA_F16, kBF16 = AQUA_BF16, kFP8 = AQUA_FP8_E4M3, kInt4 = AQUA_INT4 };

// A 16-bit type that the matrix instructions take.
template <typename T>
struct Mat;
template <>
struct Mat<f16> {
    using v2 = f16x2;
    using v8 = f16x8;
    static constexpr uint32_t kExp = 0x7c00u;  // exponent bits: all set in inf and NaN
    __device__ static f32x4 mfma16(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    __device__ static f32x16 mfma32(v8 a, v8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    // Two e4m3 bytes (low or high half of a word): exact in 16 bits.
    template <bool HI>
    __device__ static uint32_t from_fp8(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
    }
};
template <>
struct Mat<bf16> {
    using v2 = bf16x2;
    using v8 = bf16x8;
    static constexpr uint32_t kExp = 0x7f80u;
    __device__ static f32x4 mfma16(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    __device__ static f32x16 mfma32(v8 a, v8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    template <bool HI>
    __device__ static uint32_t from_fp8(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    }
};

// Two floats rounded to nearest even, low half first.
template <typename T>
__device__ inline uint32_t pack2(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, typename Mat<T>::v2));
}

template <typename T>
__device__ inline float lo_float(uint32_t w) {
    return (float)__builtin_bit_cast(typename Mat<T>::v2, w)[0];
}
template <typename T>
__device__ inline float hi_float(uint32_t w) {
    return (float)__builtin_bit_cast(typename Mat<T>::v2, w)[1];
}

// Halves of two words paired: (low of a, low of b) and (high of a, high of b).
__device__ inline uint32_t pair_lo(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ inline uint32_t pair_hi(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// Codes 4i..4i+3 of each 16-bit half of w, as the fp16 numbers 16 + code: the code
// goes to the top of the mantissa of 2^4.
template <int I>
__device__ inline f16x2 codes4(uint32_t w) {
    const uint32_t s = I == 0 ? w << 6 : I == 1 ? w << 2 : I == 2 ? w >> 2 : w >> 6;
    // (Constants in registers, one of them a vector register: an instruction takes one
    // scalar.  Then it is one and-or, and not an and and an or.)
    uint32_t mask = 0x03c003c0u, sixteen = 0x4c004c00u;
    asm("" : "+s"(mask));
    asm("" : "+v"(sixteen));
    return __builtin_bit_cast(f16x2, (s & mask) | sixteen);
}
// The two values that they stand for: one rounding, as the format has it.
__device__ inline uint32_t value4(f16x2 c, f16x2 scale, f16x2 base) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, scale, base));
}

// A load; ONCE: of data that nothing else reads.
template <bool ONCE, typename T>
__device__ inline T load(const void* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
    return *reinterpret_cast<const T*>(p);
}

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The other half's (lanes xor 32) and the other row's (lanes xor 16) values
// combined with one's own, in every lane.
template <typename F>
__device__ inline float over_halves(float x, F f) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x),
                                                    __builtin_bit_cast(uint32_t, x), false, false);
    return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
template <typename F>
__device__ inline float over_rows(float x, F f) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x),
                                                    __builtin_bit_cast(uint32_t, x), false, false);
    return over_halves(
        f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])), f);
}
struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// Values at positions that some columns see and others do not.  A weight of 0 keeps
// neither infinity nor NaN out of a product, so these enter it as 0 (`odd` tells that
// there were any), and the columns that do see them are given them afterwards, one by
// one (odd_value).
template <typename T>
__device__ inline uint32_t finite_or_zero(uint32_t w, bool* odd) {
    constexpr uint32_t e = Mat<T>::kExp;
    if ((w & e) == e) {
        w &= 0xffff0000u;
        *odd = true;
    }
    if (((w >> 16) & e) == e) {
        w &= 0xffffu;
        *odd = true;
    }
    return w;
}
// Value d of a row if it is not finite, else 0.
template <int POOL, typename M>
__device__ inline float odd_value(const uint8_t* row, const uint8_t* pairs, uint32_t d) {
    float x = 0.0f;
    if constexpr (POOL == kInt4) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(row + d / 8 * 4);
        const f16x2 p = *reinterpret_cast<const f16x2*>(pairs + d / 32 * 4);
        const uint32_t c = w >> (d % 2 * 16 + d % 8 / 2 * 4) & 15u;
        x = (float)(f16)__builtin_fmaf(16.0f + (float)c, (float)p[0], (float)p[1]);
    } else if constexpr (POOL == kFP8) {
        x = (row[d] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
    } else {
        x = (float)*reinterpret_cast<const M*>(row + 2 * d);
    }
    return __builtin_isfinite(x) ? 0.0f : x;
}

// Queries of type Q as operands of products of type M.  Where Q has more range (bf16
// queries, fp16 products), the column is scaled by a power of two that makes its
// largest value 2^8 to 2^9: values 2^-22 of it and more keep all their bits, and the
// scores' scale takes the power back.  `share` combines the lanes of a column.
template <typename M, typename Q, int N, typename F>
__device__ inline void fit_queries(typename Mat<M>::v8 (&qf)[N], float* scale2, F share) {
    if constexpr (!std::is_same_v<M, Q>) {
        float top = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const u32x4 w = __builtin_bit_cast(u32x4, qf[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                top = fmaxf(top, fmaxf(fabsf(lo_float<Q>(w[i])), fabsf(hi_float<Q>(w[i]))));
        }
        top = share(top);
        const int e = top > 0.0f && top < __builtin_inff() ? 9 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            u32x4 w = __builtin_bit_cast(u32x4, qf[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = pack2<M>(__builtin_amdgcn_ldexpf(lo_float<Q>(w[i]), e),
                                __builtin_amdgcn_ldexpf(hi_float<Q>(w[i]), e));
            qf[n] = __builtin_bit_cast(typename Mat<M>::v8, w);
        }
        *scale2 = __builtin_amdgcn_ldexpf(*scale2, -e);
    }
}

// Makes the scores' scale positive: queries change their sign with it, so that the
// largest product is the largest score.  A scale of 0 becomes the least there is, 2^-149,
// with which all scores are next to 0 (2^-21 at most) and masked ones, -inf, stay what
// they are.
template <typename V8, int N>
__device__ inline void fit_scale(V8 (&qf)[N], float* scale2) {
    if (*scale2 < 0.0f)
#pragma unroll
        for (int n = 0; n < N; ++n)
            qf[n] = __builtin_bit_cast(V8, __builtin_bit_cast(u32x4, qf[n]) ^ 0x80008000u);
    *scale2 = fmaxf(fabsf(*scale2), 0x1p-149f);
}

// The softmax is computed in powers of two.  The running maximum is raised only when
// a score exceeds it by kSlack, so that sums are rarely scaled; weights carry
// 2^kLift, so that small ones keep their bits in fp16 (2^14 at most).
constexpr float kSlack = 8.0f, kLift = 6.0f;
constexpr float kLn2 = 0.69314718f;

// Bytes of a token's row of one head, without a 4-bit pool's pairs.
template <int POOL>
__host__ __device__ constexpr uint32_t row_bytes(uint32_t D) {
    return POOL == kInt4 ? D / 2 : POOL == kFP8 ? D : 2 * D;
}

}  // namespace kv
}  // namespace aqua
