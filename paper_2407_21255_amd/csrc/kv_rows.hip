// kv_rows.hip -- attention for few columns (decode steps): 16 columns a
// workgroup, the tokens split over its waves and over workgroups, and the join
// of the split sums.
//
// One pass over the tokens with a running maximum and sum.  Bound by reading the
// cache, each key and value byte once:
//   S^T = K Q^T   16x16x32: A = keys (a lane holds one token's 8 values), B =
//                 queries, so a lane's scores are of one column (lane % 16) and
//                 of four tokens of each 16;
//   O^T += V^T P^T  A = values, B = weights.  The order of the tokens inside a product
//                 is free, so the lane's eight scores of 32 tokens are its B operand
//                 as they stand, and the values are taken in that order.  A lane takes
//                 D/16 consecutive values of its 8 tokens, and pairing their halves
//                 gives the operands of D/16 products.
// Pools of 16 bits are loaded straight into the registers that the products take
// (Direct).  In 8 and 4 bits a lane's share of a value row would be 8 or 4 bytes, and
// there a wave loads whole pieces of 16 bytes a lane and exchanges them through LDS
// that is its own (Staged).  Either way the next step is on its way while one is
// computed.  All statistics and sums are fp32.
#include <algorithm>

#include "kv_device.h"

namespace aqua {
namespace {

using namespace kv;

constexpr int kWaves = 4;

// Keys of a 16-token tile as a lane holds them, and the values of 32 tokens.
// first_of(ks, kg): first of the 8 values of a head that lane group kg puts into
// product ks.
template <int POOL, int D>
struct Load;

template <int D, int POOL16>
struct Load16 {
    static constexpr int kK = D / 32, E = D / 16, kV = E / 2;  // 16-byte pieces; words
    struct Key { u32x4 w[kK]; };
    struct Val { uint32_t w[8][kV]; };
    __device__ static constexpr int first_of(int ks, int kg) { return ks * 32 + kg * 8; }
    template <bool ONCE>
    __device__ static void key(Key& k, const uint8_t* row, const uint8_t*, int kg) {
#pragma unroll
        for (int i = 0; i < kK; ++i)
            k.w[i] = load<ONCE, u32x4>(row + i * 64 + kg * 16);
    }
    template <typename M>
    __device__ static u32x4 key_of(const Key& k, int ks) { return k.w[ks]; }
    template <bool ONCE>
    __device__ static void val(Val& v, int i, const uint8_t* row, const uint8_t*, int m) {
        if constexpr (kV == 2) {
            const u32x2 w = load<ONCE, u32x2>(row + m * 8);
            v.w[i][0] = w[0];
            v.w[i][1] = w[1];
        } else {
#pragma unroll
            for (int j = 0; j < kV; j += 4) {
                const u32x4 w = load<ONCE, u32x4>(row + m * (4 * kV) + 4 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) v.w[i][j + e] = w[e];
            }
        }
    }
    __device__ static void clear(Val& v, int i) {
#pragma unroll
        for (int j = 0; j < kV; ++j) v.w[i][j] = 0;
    }
    template <typename M>
    __device__ static void tame(Val& v, int i, bool* odd) {
#pragma unroll
        for (int j = 0; j < kV; ++j) v.w[i][j] = finite_or_zero<M>(v.w[i][j], odd);
    }
    template <typename M>
    __device__ static void vals_of(const Val& v, u32x4 (&out)[E]) {
#pragma unroll
        for (int j = 0; j < kV; ++j)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                out[2 * j][p] = pair_lo(v.w[2 * p][j], v.w[2 * p + 1][j]);
                out[2 * j + 1][p] = pair_hi(v.w[2 * p][j], v.w[2 * p + 1][j]);
            }
    }
};
template <int D>
struct Load<kF16, D> : Load16<D, kF16> {};
template <int D>
struct Load<kBF16, D> : Load16<D, kBF16> {};

template <int D>
struct Load<kFP8, D> {
    static constexpr int kK = D / 64, E = D / 16, kV = E / 4;
    struct Key { u32x4 w[kK]; };
    struct Val { uint32_t w[8][kV]; };
    __device__ static constexpr int first_of(int ks, int kg) {
        return ks / 2 * 64 + kg * 16 + ks % 2 * 8;
    }
    __device__ static void key(Key& k, const uint8_t* row, const uint8_t*, int kg) {
#pragma unroll
        for (int i = 0; i < kK; ++i)
            k.w[i] = *reinterpret_cast<const u32x4*>(row + i * 64 + kg * 16);
    }
    template <typename M>
    __device__ static u32x4 key_of(const Key& k, int ks) {
        const uint32_t a = k.w[ks / 2][ks % 2 * 2], b = k.w[ks / 2][ks % 2 * 2 + 1];
        return {Mat<M>::template from_fp8<false>(a), Mat<M>::template from_fp8<true>(a),
                Mat<M>::template from_fp8<false>(b), Mat<M>::template from_fp8<true>(b)};
    }
    __device__ static void val(Val& v, int i, const uint8_t* row, const uint8_t*, int m) {
        if constexpr (kV == 1) {
            v.w[i][0] = *reinterpret_cast<const uint32_t*>(row + m * 4);
        } else if constexpr (kV == 2) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(row + m * 8);
            v.w[i][0] = w[0];
            v.w[i][1] = w[1];
        } else {
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + m * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) v.w[i][e] = w[e];
        }
    }
    __device__ static void clear(Val& v, int i) {
#pragma unroll
        for (int j = 0; j < kV; ++j) v.w[i][j] = 0;
    }
    template <typename M>
    __device__ static void tame(Val& v, int i, bool* odd) {
#pragma unroll
        for (int j = 0; j < kV; ++j)
#pragma unroll
            for (int b = 0; b < 32; b += 8)
                if ((v.w[i][j] >> b & 0x7fu) == 0x7fu) {   // NaN, e4m3's only such value
                    v.w[i][j] &= ~(0xffu << b);
                    *odd = true;
                }
    }
    // Bytes of two tokens are paired before they are widened: one permutation and
    // two conversions for four values.
    template <typename M>
    __device__ static void vals_of(const Val& v, u32x4 (&out)[E]) {
#pragma unroll
        for (int j = 0; j < kV; ++j)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t a = v.w[2 * p][j], b = v.w[2 * p + 1][j];
                const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
                const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07030602u);  // a2 b2 a3 b3
                out[4 * j][p] = Mat<M>::template from_fp8<false>(x);
                out[4 * j + 1][p] = Mat<M>::template from_fp8<true>(x);
                out[4 * j + 2][p] = Mat<M>::template from_fp8<false>(y);
                out[4 * j + 3][p] = Mat<M>::template from_fp8<true>(y);
            }
    }
};

template <int D>
struct Load<kInt4, D> {
    // A lane's share of a key: D/4 codes (D/32 words), in groups kg (D = 128), half a
    // group (64) or groups kg and 4 + kg (256).
    static constexpr int kW = D / 32, kG = D == 256 ? 2 : 1, E = D / 16, kV = D == 256 ? 2 : 1;
    struct Key { uint32_t w[kW]; uint32_t pair[kG]; };
    struct Val { uint32_t w[8][kV]; uint32_t pair[8]; };
    __device__ static constexpr int first_of(int ks, int kg) {
        return D == 64 ? kg * 16 + ks * 8 : (ks / 4 * 4 + kg) * 32 + ks % 4 * 8;
    }
    __device__ static void key(Key& k, const uint8_t* row, const uint8_t* pairs, int kg) {
        if constexpr (D == 64) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(row + kg * 8);
            k.w[0] = w[0];
            k.w[1] = w[1];
            k.pair[0] = *reinterpret_cast<const uint32_t*>(pairs + kg / 2 * 4);
        } else {
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(row + i * 64 + kg * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) k.w[4 * i + e] = w[e];
                k.pair[i] = *reinterpret_cast<const uint32_t*>(pairs + (i * 4 + kg) * 4);
            }
        }
    }
    template <typename M>
    __device__ static u32x4 key_of(const Key& k, int ks) {
        const uint32_t w = k.w[ks], p = k.pair[D == 64 ? 0 : ks / 4];
        const f16x2 s = __builtin_bit_cast(f16x2, pair_lo(p, p));
        const f16x2 b = __builtin_bit_cast(f16x2, pair_hi(p, p));
        return {value4(codes4<0>(w), s, b), value4(codes4<1>(w), s, b),
                value4(codes4<2>(w), s, b), value4(codes4<3>(w), s, b)};
    }
    __device__ static void val(Val& v, int i, const uint8_t* row, const uint8_t* pairs, int m) {
        if constexpr (D == 64) {
            v.w[i][0] = *reinterpret_cast<const uint32_t*>(row + m / 2 * 4);
        } else if constexpr (D == 128) {
            v.w[i][0] = *reinterpret_cast<const uint32_t*>(row + m * 4);
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2*>(row + m * 8);
            v.w[i][0] = w[0];
            v.w[i][1] = w[1];
        }
        v.pair[i] = *reinterpret_cast<const uint32_t*>(pairs + m * E / 32 * 4);
        if constexpr (D == 64) v.w[i][0] >>= (m & 1) * 8;
    }
    __device__ static void clear(Val& v, int i) {
        v.pair[i] = 0;
    }
    // (A pair that is not finite leaves no finite value in its group.)
    template <typename M>
    __device__ static void tame(Val& v, int i, bool* odd) {
        if ((v.pair[i] & 0x7c00u) == 0x7c00u || (v.pair[i] >> 16 & 0x7c00u) == 0x7c00u) {
            v.pair[i] = 0;
            *odd = true;
        }
    }
    // Words of two tokens are paired by halves; a shift and a mask then leave the same
    // value of both in the two halves of a register, and one packed fma with their
    // scales and bases makes the operand.
    template <typename M>
    __device__ static void vals_of(const Val& v, u32x4 (&out)[E]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t pa = v.pair[2 * p], pb = v.pair[2 * p + 1];
            const f16x2 s = __builtin_bit_cast(f16x2, pair_lo(pa, pb));
            const f16x2 b = __builtin_bit_cast(f16x2, pair_hi(pa, pb));
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                const uint32_t x = pair_lo(v.w[2 * p][j], v.w[2 * p + 1][j]);
                const uint32_t y = pair_hi(v.w[2 * p][j], v.w[2 * p + 1][j]);
                out[8 * j][p] = value4(codes4<0>(x), s, b);
                out[8 * j + 1][p] = value4(codes4<0>(y), s, b);
                out[8 * j + 2][p] = value4(codes4<1>(x), s, b);
                out[8 * j + 3][p] = value4(codes4<1>(y), s, b);
                if constexpr (D != 64) {
                    out[8 * j + 4][p] = value4(codes4<2>(x), s, b);
                    out[8 * j + 5][p] = value4(codes4<2>(y), s, b);
                    out[8 * j + 6][p] = value4(codes4<3>(x), s, b);
                    out[8 * j + 7][p] = value4(codes4<3>(y), s, b);
                }
            }
        }
    }
};

// Where a head's keys and values are, and a sequence's blocks.
struct Cache {
    const uint8_t *keys, *vals, *kpairs, *vpairs;  // of block 0
    uint64_t chunk;
    const int32_t* table;
    uint32_t last, shift, mask;  // table entries are read up to `last`; slots
    // (A step may reach behind the context: the last block is read there instead.)
    __device__ uint32_t block(uint32_t token) const { return table[min(token >> shift, last)]; }
};

// Keys and values that are loaded as the products take them: a lane's token of keys is
// lane % 16 of each 16, and lane group kg takes the values of tokens 4 kg + 0..3.
template <int POOL, int D>
struct Direct {
    using L = Load<POOL, D>;
    static constexpr int kStep = 32;
    static constexpr bool kStaged = false;
    static constexpr uint32_t kRow = row_bytes<POOL>(D), kBytes = 0;
    typename L::Key keys[2];
    typename L::Val vals;
    uint32_t kb[2], vb[2];
    __device__ static int token(int kg, int r) { return 4 * kg + r; }
    __device__ void blocks(const Cache& c, uint32_t t, int lane) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            kb[i] = c.block(t + 16 * i + lane % 16);
            vb[i] = c.block(t + 16 * i + 4 * (lane / 16));
        }
    }
    template <bool ONCE>
    __device__ void fetch_keys(const Cache& c, uint32_t t, int lane) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            L::template key<ONCE>(
                keys[i], c.keys + kb[i] * c.chunk + ((t + 16 * i + lane % 16) & c.mask) * kRow,
                nullptr, lane / 16);
    }
    template <bool ONCE>
    __device__ void fetch_vals(const Cache& c, uint32_t t, int lane) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* r =
                c.vals + vb[i] * c.chunk + ((t + 16 * i + 4 * (lane / 16)) & c.mask) * kRow;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                L::template val<ONCE>(vals, 4 * i + j, r + j * kRow, nullptr, lane % 16);
        }
    }
    __device__ void settle(uint8_t*, int) {}
    __device__ typename L::Key key(const uint8_t*, int i, int) const { return keys[i]; }
    __device__ typename L::Val val(const uint8_t*, int, int) const { return vals; }
};

// Keys and values that pass through LDS: pieces of 16 bytes in the rows' order.
// Product row m of 16 is token 4 (m % 4) + m / 4, so that lane group kg takes the
// values of tokens 4 r + kg: the four groups' reads are of four rows that follow each
// other, and fall on different banks.
template <int POOL, int D, int STEP>
struct Staged {
    using L = Load<POOL, D>;
    static constexpr int kStep = STEP;
    static constexpr bool kStaged = true;
    static constexpr uint32_t kRow = row_bytes<POOL>(D), kPairs = POOL == kInt4 ? D / 32 * 4 : 0;
    static constexpr int kPieces = STEP * kRow / 1024;             // a lane's, of keys
    static constexpr uint32_t kPair = STEP * kPairs < 1024 ? 8 : 16;  // bytes of a piece of pairs
    static constexpr int kPairPieces = STEP * kPairs / (64 * kPair);
    static_assert(kPieces * 1024 == STEP * kRow && kPairPieces * 64 * kPair == STEP * kPairs,
                  "whole pieces");
    static constexpr uint32_t kRowPairs = kPairs ? kPairs / kPair : 1;  // pieces of a row
    static constexpr uint32_t kKeyAt = 0, kValAt = STEP * kRow, kKeyPairAt = 2 * STEP * kRow,
                              kValPairAt = kKeyPairAt + STEP * kPairs,
                              kBytes = kValPairAt + STEP * kPairs;
    u32x4 k[kPieces], v[kPieces], kp[kPairPieces + 1], vp[kPairPieces + 1];
    uint32_t b[kPieces], pb[kPairPieces + 1];
    __device__ static int token(int kg, int r) { return 4 * r + kg; }
    __device__ static uint32_t row_of(int j, int lane) { return (j * 64 + lane) / (kRow / 16); }
    __device__ static uint32_t pair_row_of(int j, int lane) {
        return (j * 64 + lane) / kRowPairs;
    }
    __device__ void blocks(const Cache& c, uint32_t t, int lane) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) b[j] = c.block(t + row_of(j, lane));
#pragma unroll
        for (int j = 0; j < kPairPieces; ++j) pb[j] = c.block(t + pair_row_of(j, lane));
    }
    template <bool ONCE>
    __device__ void fetch_keys(const Cache& c, uint32_t t, int lane) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const uint64_t at = b[j] * c.chunk + ((t + row_of(j, lane)) & c.mask) * kRow +
                                (j * 64 + lane) % (kRow / 16) * 16;
            k[j] = load<ONCE, u32x4>(c.keys + at);
            v[j] = load<ONCE, u32x4>(c.vals + at);
        }
#pragma unroll
        for (int j = 0; j < kPairPieces; ++j) {
            const uint64_t at = pb[j] * c.chunk + ((t + pair_row_of(j, lane)) & c.mask) * kPairs +
                                (j * 64 + lane) % kRowPairs * kPair;
            if constexpr (kPair == 16) {
                kp[j] = load<ONCE, u32x4>(c.kpairs + at);
                vp[j] = load<ONCE, u32x4>(c.vpairs + at);
            } else {
                const u32x2 x = load<ONCE, u32x2>(c.kpairs + at), y = load<ONCE, u32x2>(c.vpairs + at);
                kp[j] = u32x4{x[0], x[1], 0, 0};
                vp[j] = u32x4{y[0], y[1], 0, 0};
            }
        }
    }
    template <bool ONCE>
    __device__ void fetch_vals(const Cache&, uint32_t, int) {}
    __device__ void settle(uint8_t* lds, int lane) {
        // A wave's LDS instructions are done in their order; the fences keep the compiler
        // from changing it.
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            *reinterpret_cast<u32x4*>(lds + kKeyAt + (j * 64 + lane) * 16) = k[j];
            *reinterpret_cast<u32x4*>(lds + kValAt + (j * 64 + lane) * 16) = v[j];
        }
#pragma unroll
        for (int j = 0; j < kPairPieces; ++j) {
            uint8_t* const x = lds + kKeyPairAt + (j * 64 + lane) * kPair;
            uint8_t* const y = lds + kValPairAt + (j * 64 + lane) * kPair;
            if constexpr (kPair == 16) {
                *reinterpret_cast<u32x4*>(x) = kp[j];
                *reinterpret_cast<u32x4*>(y) = vp[j];
            } else {
                *reinterpret_cast<u32x2*>(x) = u32x2{kp[j][0], kp[j][1]};
                *reinterpret_cast<u32x2*>(y) = u32x2{vp[j][0], vp[j][1]};
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
    __device__ typename L::Key key(const uint8_t* lds, int i, int lane) const {
        const uint32_t row = 16 * i + lane % 4 * 4 + lane % 16 / 4;
        typename L::Key x;
        L::key(x, lds + kKeyAt + row * kRow, lds + kKeyPairAt + row * kPairs, lane / 16);
        return x;
    }
    __device__ typename L::Val val(const uint8_t* lds, int half, int lane) const {
        typename L::Val x;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t row = 32 * half + i / 4 * 16 + token(lane / 16, i % 4);
            L::val(x, i, lds + kValAt + row * kRow, lds + kValPairAt + row * kPairs, lane % 16);
        }
        return x;
    }
};

template <int POOL, int D>
struct Source : Direct<POOL, D> {};
template <int D>
struct Source<kFP8, D> : Staged<kFP8, D, 32> {};
template <int D>
struct Source<kInt4, D> : Staged<kInt4, D, D == 64 ? 64 : 32> {};   // whole pieces a wave

// Q: type of the queries and the result.  M: type of the products: fp16 for a 4-bit
// pool, whose values are fp16 numbers.
// Three waves a SIMD, where their registers allow it (heads up to 128): one was left
// to two of them by three registers, and took 50 instead of 45 us for 64 chats in 4
// bits.
template <int POOL, typename Q, int D>
__global__ __launch_bounds__(256, D > 128 ? 1 : 3) void rows_kernel(const KvAttend a) {
    using M = std::conditional_t<POOL == kInt4, f16, Q>;
    using L = Load<POOL, D>;
    using S = Source<POOL, D>;
    using V8 = typename Mat<M>::v8;
    constexpr int E = L::E, kStep = S::kStep, kRuns = kStep / 16;
    constexpr bool kTwo = std::is_same_v<M, Q>;
    static_assert(kRows.step % (kWaves * kStep) == 0, "parts are whole steps of a workgroup");
    const uint32_t H = a.layer.H;
    const uint32_t item = blockIdx.x / H, head = blockIdx.x % H;
    const KvPart part = a.t.rows[item];   // (an old one, where there is none)
    if (item >= a.t.head->rows) return;
    const KvSeq seq = part.seq;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col = lane % 16, kg = lane / 16;
    const uint32_t G = a.group, T = a.layer.T;
    const uint32_t columns = G * seq.fresh;
    const uint32_t c = min(part.tile * kRowColumns + col, columns - 1);
    const uint32_t token = c / G;
    // The column sees tokens below its limit.
    const uint32_t limit = seq.context - seq.fresh + token + 1;
    const uint32_t least = seq.context - seq.fresh + part.tile * kRowColumns / G + 1;

    // Queries, in the order in which the lanes load the keys.
    const uint8_t* q = a.q + 2 * ((uint64_t)(seq.row + token) * a.q_stride +
                                  (uint64_t)(head * G + c % G) * D);
    V8 qf[D / 32];
    float scale2 = a.scale2;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
        qf[ks] = __builtin_bit_cast(
            V8, *reinterpret_cast<const u32x4*>(q + 2 * L::first_of(ks, kg)));
    fit_queries<M, Q>(qf, &scale2, [](float x) { return over_rows(x, Max()); });
    fit_scale(qf, &scale2);

    constexpr uint32_t kRow = row_bytes<POOL>(D), kPairs = D / 32 * 4;
    Cache cache;
    cache.keys = a.layer.base + (uint64_t)head * T * kRow;
    cache.vals = cache.keys + (uint64_t)H * T * kRow;
    cache.kpairs = a.layer.base + (uint64_t)2 * H * T * kRow + (uint64_t)head * T * kPairs;
    cache.vpairs = cache.kpairs + (uint64_t)H * T * kPairs;
    cache.chunk = a.layer.chunk_bytes;
    cache.table = a.t.blocks + seq.first;
    cache.last = (seq.context - 1) >> a.layer.shift;
    cache.shift = a.layer.shift;
    cache.mask = T - 1;

    // Steps of the waves, then the waves' sums.
    constexpr uint32_t kSumRow = D + 4;
    __shared__ __attribute__((aligned(16)))
    uint8_t shared[std::max<uint32_t>(kWaves * S::kBytes, kWaves * 16 * kSumRow * 4)];
    uint8_t* const lds = shared + wave * S::kBytes;

    f32x4 acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = f32x4{0, 0, 0, 0};
    float top = -__builtin_inff(), sum = 0.0f;
    bool odd = false;
    S src;

    const auto steps = [&](auto once) __attribute__((always_inline)) {
        constexpr bool kOnce = decltype(once)::value;
        uint32_t t = part.begin + wave * kStep;
        if (t < part.end) {
            src.blocks(cache, t, lane);
            src.template fetch_keys<kOnce>(cache, t, lane);
            src.template fetch_vals<kOnce>(cache, t, lane);
            src.blocks(cache, t + kWaves * kStep, lane);
        }
        for (; t < part.end; t += kWaves * kStep) {
            const uint32_t next = t + kWaves * kStep;
            const bool more = next < part.end;
            src.settle(lds, lane);
            if (S::kStaged && more) {
                src.template fetch_keys<kOnce>(cache, next, lane);
                src.blocks(cache, next + kWaves * kStep, lane);
            }
            f32x4 s[kRuns];
#pragma unroll
            for (int i = 0; i < kRuns; ++i) {
                s[i] = f32x4{0, 0, 0, 0};
                const typename L::Key key = src.key(lds, i, lane);
#pragma unroll
                for (int ks = 0; ks < D / 32; ++ks)
                    s[i] = Mat<M>::mfma16(
                        __builtin_bit_cast(V8, L::template key_of<M>(key, ks)), qf[ks], s[i]);
            }
            if (!S::kStaged && more) src.template fetch_keys<kOnce>(cache, next, lane);

            // Tokens behind a column's limit, or another part's, get no weight.
            const uint32_t stop = min(limit, part.end);
            const bool masked = t + kStep > min(least, part.end);
            if (masked)
#pragma unroll
                for (int i = 0; i < kRuns; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (t + 16 * i + S::token(kg, r) >= stop) s[i][r] = -__builtin_inff();
            float high = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < kRuns; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) high = fmaxf(high, s[i][r]);
            high = over_rows(high, Max()) * scale2;
            if (__any(high > top + kSlack)) {
                // (A column that has seen nothing keeps its -inf, and sums of 0.)
                const float raised = fmaxf(top, high);
                const float f = raised > -__builtin_inff() ? exp2_(top - raised) : 1.0f;
                top = raised;
                sum *= f;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= f;
            }
            const float off = top > -__builtin_inff() ? top - kLift : 0.0f;
#pragma unroll
            for (int half = 0; half < kRuns / 2; ++half) {
                // Where the products' type is no finer than the result's, weights are in two
                // terms, the second what the first's rounding left: the products have time to
                // spare, and the result is as exact as its own rounding.  (Weights in fp16 for
                // a bf16 result, of a 4-bit pool: off by 0.00167 of its size against 64 bits,
                // with weights in fp32 by 0.00166.)
                u32x4 pw, pr = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = exp2_(__builtin_fmaf(s[2 * half + i / 2][i % 2 * 2], scale2, -off));
                    const float y =
                        exp2_(__builtin_fmaf(s[2 * half + i / 2][i % 2 * 2 + 1], scale2, -off));
                    sum += x + y;
                    const uint32_t w = pack2<M>(x, y);
                    pw[i] = w;
                    if (kTwo) pr[i] = pack2<M>(x - lo_float<M>(w), y - hi_float<M>(w));
                }
                const V8 pf = __builtin_bit_cast(V8, pw), pg = __builtin_bit_cast(V8, pr);

                typename L::Val val = src.val(lds, half, lane);
                if (masked) {
                    // What stands behind the context may be anything: no weight is no help
                    // against NaN.
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (t + 32 * half + i / 4 * 16 + S::token(kg, i % 4) >= seq.context)
                            L::clear(val, i);
                        else if (seq.fresh > 1)
                            L::template tame<M>(val, i, &odd);
                }
                u32x4 vf[E];
                L::template vals_of<M>(val, vf);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    acc[e] = Mat<M>::mfma16(__builtin_bit_cast(V8, vf[e]), pf, acc[e]);
                if (kTwo)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        acc[e] = Mat<M>::mfma16(__builtin_bit_cast(V8, vf[e]), pg, acc[e]);
            }
            if (!S::kStaged && more) {
                src.template fetch_vals<kOnce>(cache, next, lane);
                src.blocks(cache, next + kWaves * kStep, lane);
            }
        }
    };
    // Loads that tell that no other workgroup reads the data leave the caches to others:
    // 64 chats in bf16 took 91 instead of 102 us.  Where several tiles of columns share
    // a context they would read it from memory each: 32 columns took 98 instead of
    // 74 us.
    if (columns <= kRowColumns)
        steps(std::true_type());
    else
        steps(std::false_type());

    if (__any(odd))
        for (uint32_t t = part.begin + wave * kStep; t < part.end; t += kWaves * kStep) {
            if (t + kStep <= min(least, part.end)) continue;
            for (uint32_t k = t; k < min(t + kStep, part.end); ++k) {
                const uint64_t at = cache.block(k) * cache.chunk;
                const uint32_t slot = k & cache.mask;
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = odd_value<POOL, M>(cache.vals + at + slot * kRow,
                                                           cache.vpairs + at + slot * kPairs,
                                                           (kg * 4 + r) * E + e);
                        acc[e][r] += k < min(limit, part.end) ? x : 0.0f;
                    }
            }
        }

    // The waves' sums, on a common maximum.
    __shared__ float tops[kWaves][16], sums[kWaves][16];
    float (*part_sum)[16][kSumRow] = reinterpret_cast<float (*)[16][kSumRow]>(shared);
    sum = over_rows(sum, Sum());
    if (kg == 0) tops[wave][col] = top;
    __syncthreads();   // and the waves are done with their steps
    float all = tops[0][col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w][col]);
    const float f = top > -__builtin_inff() ? exp2_(top - all) : 0.0f;
    if (kg == 0) sums[wave][col] = sum * f;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<f32x4*>(&part_sum[wave][col][(kg * 4 + r) * E + e]) =
                f32x4{acc[e][r], acc[e + 1][r], acc[e + 2][r], acc[e + 3][r]} * f;
    __syncthreads();

    // 16 lanes a column, D/16 values a lane.
    const int oc = threadIdx.x / 16, od = threadIdx.x % 16 * E;
    const uint32_t oc_all = part.tile * kRowColumns + oc;
    if (oc_all >= columns) return;
    float total = 0.0f, high = tops[0][oc];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        total += sums[w][oc];
        high = fmaxf(high, tops[w][oc]);
    }
    float o[E];
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        f32x4 x = *reinterpret_cast<const f32x4*>(&part_sum[0][oc][od + e]);
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            x += *reinterpret_cast<const f32x4*>(&part_sum[w][oc][od + e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[e + i] = x[i];
    }
    if (part.slot != kNoSlot) {
        float* slot = a.t.slots + ((uint64_t)part.slot * H + head) * slot_floats(D);
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<f32x4*>(slot + oc * D + od + e) =
                f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
        if (od == 0) {
            slot[16 * D + oc] = high;
            slot[16 * D + 16 + oc] = total;
        }
        return;
    }
    const uint64_t row = seq.row + oc_all / G, h = head * G + oc_all % G;
    // (The values' scale by itself: over the sum it may be too small for fp32.  Only fp8
    // pools have one.)
    const float norm = 1.0f / total;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= norm;
    if (POOL == kFP8)
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= a.v_scale;
    uint8_t* out = a.out + 2 * (row * a.out_stride + h * D + od);
    if constexpr (E == 4) {
        *reinterpret_cast<u32x2*>(out) = u32x2{pack2<Q>(o[0], o[1]), pack2<Q>(o[2], o[3])};
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 8)
            *reinterpret_cast<u32x4*>(out + 2 * e) =
                u32x4{pack2<Q>(o[e], o[e + 1]), pack2<Q>(o[e + 2], o[e + 3]),
                      pack2<Q>(o[e + 4], o[e + 5]), pack2<Q>(o[e + 6], o[e + 7])};
    }
    if (a.lse && od == 0)
        a.lse[row * a.q_heads + h] = (high - kLift + __builtin_log2f(total)) * kLn2;
}

// A running maximum, sum of weights and weighted values.
struct Sums {
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    // Brings the sums to a maximum that is at least their own.
    __device__ void raise(float to) {
        // (Where nothing has been seen, -inf, the sums are 0.)
        const float f = exp2_(top - (to > -__builtin_inff() ? to : 0.0f));
        total *= f;
        o *= f;
        top = to;
    }
    __device__ void add(float high, float sum, f32x4 x) {
        const float w = exp2_(high - (top > -__builtin_inff() ? top : 0.0f));
        total += w * sum;
        o += w * x;
    }
};

// Parts p, p + turns, ... of a column: AHEAD of them in flight.
template <int AHEAD>
__device__ inline void join_parts(Sums& s, const float* first, uint64_t step, uint32_t at,
                                  uint32_t stat, uint32_t p, uint32_t turns, uint32_t parts) {
    for (; p < parts; p += AHEAD * turns) {
        float high[AHEAD], sum[AHEAD], raised = s.top;
        f32x4 x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            // (The last turn reads the last part again, and drops it.)
            const float* slot = first + min(p + i * turns, parts - 1) * step;
            high[i] = slot[stat];
            sum[i] = slot[stat + kRowColumns];
            x[i] = *reinterpret_cast<const f32x4*>(slot + at);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) raised = fmaxf(raised, high[i]);
        s.raise(raised);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (p + i * turns < parts) s.add(high[i], sum[i], x[i]);
    }
}

// Joins the parts of some columns of a tile of 16.  A lane takes four values of a
// column; the groups of lanes that the columns leave over share out the parts.  Bound by
// latency, so each lane has up to kJoinAhead parts in flight, and there is one
// pass with a running maximum.  Every sum has a fixed order.
template <typename Q, int D>
__global__ __launch_bounds__(256) void join_kernel(const KvAttend a) {
    constexpr uint32_t kLanes = D / 4, kGroups = join_groups(D);
    static_assert(kLanes * kGroups == 256, "a workgroup's lanes");
    __shared__ f32x4 os[kGroups][kLanes];
    __shared__ float tops[kGroups][kLanes], totals[kGroups][kLanes];
    const uint32_t H = a.layer.H, group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t items = a.t.head->joins * H;
    // (A captured launch may have fewer workgroups than joins.)
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const KvJoin join = a.t.joins[n / H];
        const uint32_t head = n % H, turns = kGroups / join.count;
        const uint32_t mine = group / turns, turn = group % turns;
        const bool live = mine < join.count;
        const uint32_t c = join.column + min(mine, join.count - 1), col = c % kRowColumns;
        const uint64_t step = (uint64_t)join.stride * H * slot_floats(D);
        const float* first = a.t.slots + ((uint64_t)join.slot * H + head) * slot_floats(D);
        const uint32_t at = col * D + lane * 4, stat = 16 * D + col;
        Sums s;
        if (join.parts <= 2 * turns)
            join_parts<2>(s, first, step, at, stat, turn, turns, join.parts);
        else
            join_parts<kJoinAhead>(s, first, step, at, stat, turn, turns, join.parts);
        if (turns > 1) {
            os[group][lane] = s.o;
            tops[group][lane] = s.top;
            totals[group][lane] = s.total;
            __syncthreads();
            if (turn == 0 && live) {
                float top = s.top;
                for (uint32_t t = 1; t < turns; ++t) top = fmaxf(top, tops[group + t][lane]);
                s.raise(top);
                for (uint32_t t = 1; t < turns; ++t)
                    s.add(tops[group + t][lane], totals[group + t][lane], os[group + t][lane]);
            }
            __syncthreads();
        }
        if (!live || turn) continue;
        const uint64_t row = join.row + c / a.group, h = head * a.group + c % a.group;
        s.o *= 1.0f / s.total;
        *reinterpret_cast<u32x2*>(a.out + 2 * (row * a.out_stride + h * D + lane * 4)) =
            u32x2{pack2<Q>(s.o[0] * a.v_scale, s.o[1] * a.v_scale),
                  pack2<Q>(s.o[2] * a.v_scale, s.o[3] * a.v_scale)};
        if (a.lse && lane == 0)
            a.lse[row * a.q_heads + h] = (s.top - kLift + __builtin_log2f(s.total)) * kLn2;
    }
}

template <typename K>
hipError_t launch(K kernel, uint32_t grid, uint32_t block, hipStream_t stream, const KvAttend& a) {
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(block), 0, stream, a);
    return hipGetLastError();
}

template <int POOL, typename Q>
hipError_t rows(const KvAttend& a, uint32_t grid, hipStream_t stream) {
    switch (a.layer.D) {
        case 64: return launch(rows_kernel<POOL, Q, 64>, grid, 256, stream, a);
        case 128: return launch(rows_kernel<POOL, Q, 128>, grid, 256, stream, a);
        default: return launch(rows_kernel<POOL, Q, 256>, grid, 256, stream, a);
    }
}

template <typename Q>
hipError_t join(const KvAttend& a, uint32_t grid, hipStream_t stream) {
    switch (a.layer.D) {
        case 64: return launch(join_kernel<Q, 64>, grid, 256, stream, a);
        case 128: return launch(join_kernel<Q, 128>, grid, 256, stream, a);
        default: return launch(join_kernel<Q, 256>, grid, 256, stream, a);
    }
}

// Workgroups of a join's launch at most.
constexpr uint32_t kJoinGrid = 4096;

}  // namespace

hipError_t launch_rows(const KvAttend& a, uint32_t items, hipStream_t stream) {
    if (!items) return hipSuccess;
    const uint32_t grid = items * a.layer.H;
    const bool half = a.dtype == AQUA_F16;
    switch (a.layer.dtype) {
        case AQUA_F16: return rows<kF16, f16>(a, grid, stream);
        case AQUA_BF16: return rows<kBF16, bf16>(a, grid, stream);
        case AQUA_FP8_E4M3: return half ? rows<kFP8, f16>(a, grid, stream)
                                        : rows<kFP8, bf16>(a, grid, stream);
        default: return half ? rows<kInt4, f16>(a, grid, stream)
                             : rows<kInt4, bf16>(a, grid, stream);
    }
}

hipError_t launch_join(const KvAttend& a, uint32_t joins, hipStream_t stream) {
    if (!joins) return hipSuccess;
    const uint32_t all = joins * a.layer.H, grid = all < kJoinGrid ? all : kJoinGrid;
    return a.dtype == AQUA_F16 ? join<f16>(a, grid, stream) : join<bf16>(a, grid, stream);
}

hipError_t launch_attend(const KvAttend& a, const KvCounts& n, hipStream_t stream) {
    hipError_t e = launch_tiles(a, n.tiles, stream);
    if (e == hipSuccess) e = launch_rows(a, n.rows, stream);
    if (e == hipSuccess) e = launch_join(a, n.joins, stream);
    return e;
}

}  // namespace aqua
