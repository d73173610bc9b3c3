// kv_rows.hip -- attention for few columns (decode steps): 16 columns a
// workgroup, the tokens split over its waves and over workgroups, and the join
// of the split sums.
//
// One pass over the tokens with a running maximum and sum.  Bound by reading the
// cache: each key and value byte is read once, straight from the pool's blocks into
// the registers that the matrix instructions take, with no LDS in between:
//   S^T = K Q^T   16x16x32: A = keys (a lane holds one token's 8 values), B =
//                 queries, so a lane's scores are of one column (lane % 16) and
//                 of tokens 4 (lane / 16) + 0..3 of each 16;
//   O^T += V^T P^T  A = values, B = weights.  The order of the tokens inside a product
//                 is free, so the lane's eight scores of 32 tokens are its B operand
//                 as they stand, and the values are loaded in that order: lane
//                 group kg takes tokens 4 kg + 0..3 and 16 + 4 kg + 0..3.  A lane
//                 loads D/16 consecutive values of its 8 tokens, and pairing their
//                 halves gives the operands of D/16 products.
// All statistics and sums are fp32.
#include "kv_device.h"

namespace aqua {
namespace {

using namespace kv;

constexpr int kWaves = 4, kStep = 32;  // tokens of a wave's step
static_assert(kRowsStep == kWaves * kStep, "parts are whole steps of a workgroup");

// Keys of a 16-token tile as a lane loads them, and the values of a 32-token step.
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
    __device__ static void key(Key& k, const uint8_t* row, const uint8_t*, int kg) {
#pragma unroll
        for (int i = 0; i < kK; ++i)
            k.w[i] = *reinterpret_cast<const u32x4*>(row + i * 64 + kg * 16);
    }
    template <typename M>
    __device__ static u32x4 key_of(const Key& k, int ks) { return k.w[ks]; }
    __device__ static void val(Val& v, int i, const uint8_t* row, const uint8_t*, int m) {
        if constexpr (kV == 2) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(row + m * 8);
            v.w[i][0] = w[0];
            v.w[i][1] = w[1];
        } else {
#pragma unroll
            for (int j = 0; j < kV; j += 4) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(row + m * (4 * kV) + 4 * j);
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

// Q: type of the queries and the result.  M: type of the products: fp16 for a 4-bit
// pool, whose values are fp16 numbers.
template <int POOL, typename Q, int D>
__global__ __launch_bounds__(256) void rows_kernel(const KvAttend a) {
    using M = std::conditional_t<POOL == kInt4, f16, Q>;
    using L = Load<POOL, D>;
    using V8 = typename Mat<M>::v8;
    constexpr int E = L::E;
    const uint32_t H = a.layer.H;
    const uint32_t item = blockIdx.x / H, head = blockIdx.x % H;
    if (item >= a.t.head->rows) return;
    const KvPart part = a.t.rows[item];
    const KvSeq seq = a.t.seqs[part.seq];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int col = lane % 16, kg = lane / 16;
    const uint32_t G = a.group, T = a.layer.T, shift = a.layer.shift;
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

    constexpr uint32_t kRow = row_bytes<POOL>(D), kPairs = D / 32 * 4;
    const uint64_t C = a.layer.chunk_bytes;
    const uint8_t* const kbase = a.layer.base + (uint64_t)head * T * kRow;
    const uint8_t* const vbase = kbase + (uint64_t)H * T * kRow;
    const uint8_t* const kpair = a.layer.base + (uint64_t)2 * H * T * kRow + (uint64_t)head * T * kPairs;
    const uint8_t* const vpair = kpair + (uint64_t)H * T * kPairs;
    const int32_t* const table = a.t.blocks + seq.first;
    const uint32_t last = (seq.context - 1) >> shift;   // table entries are read up to here

    f32x4 acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = f32x4{0, 0, 0, 0};
    float top = -__builtin_inff(), sum = 0.0f;
    bool odd = false;

    typename L::Key key[2];
    typename L::Val val;
    uint32_t kb[2], vb[2];
    // Blocks of the lane's tokens in the step at t: two keys, two runs of 4 values.
    // A step may reach behind the context: the last block is read there instead.
    const auto blocks = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            kb[i] = table[min((t + 16 * i + col) >> shift, last)];
            vb[i] = table[min((t + 16 * i + 4 * kg) >> shift, last)];
        }
    };
    const auto load_keys = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t slot = (t + 16 * i + col) & (T - 1);
            L::key(key[i], kbase + kb[i] * C + slot * kRow, kpair + kb[i] * C + slot * kPairs, kg);
        }
    };
    const auto load_vals = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t slot = (t + 16 * i + 4 * kg) & (T - 1);
            const uint8_t* r = vbase + vb[i] * C + slot * kRow;
            const uint8_t* p = vpair + vb[i] * C + slot * kPairs;
#pragma unroll
            for (int j = 0; j < 4; ++j) L::val(val, 4 * i + j, r + j * kRow, p + j * kPairs, col);
        }
    };

    uint32_t t = part.begin + wave * kStep;
    if (t < part.end) {
        blocks(t);
        load_keys(t);
        load_vals(t);
        blocks(t + kWaves * kStep);
    }
    for (; t < part.end; t += kWaves * kStep) {
        f32x4 s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
                s[i] = Mat<M>::mfma16(
                    __builtin_bit_cast(V8, L::template key_of<M>(key[i], ks)), qf[ks], s[i]);
        }
        const uint32_t next = t + kWaves * kStep;
        const bool more = next < part.end;
        if (more) load_keys(next);

        // Tokens behind a column's limit, or another part's, get no weight.
        const uint32_t stop = min(limit, part.end);
        const bool masked = t + kStep > min(least, part.end);
        float high = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[i][r] *= scale2;
                if (masked && t + 16 * i + 4 * kg + r >= stop) s[i][r] = -__builtin_inff();
                high = fmaxf(high, s[i][r]);
            }
        high = over_rows(high, Max());
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
        u32x4 pw;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[r] = exp2_(s[i][r] - off);
                sum += p[r];
            }
            pw[2 * i] = pack2<M>(p[0], p[1]);
            pw[2 * i + 1] = pack2<M>(p[2], p[3]);
        }
        const V8 pf = __builtin_bit_cast(V8, pw);

        u32x4 vf[E];
        if (masked) {
            // What stands behind the context may be anything: no weight is no help
            // against NaN.
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t + 16 * i + 4 * kg + j >= seq.context) L::clear(val, 4 * i + j);
        }
        L::template vals_of<M>(val, vf);
        if (masked && seq.fresh > 1)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int p = 0; p < 4; ++p) vf[e][p] = finite_or_zero<M>(vf[e][p], &odd);
#pragma unroll
        for (int e = 0; e < E; ++e)
            acc[e] = Mat<M>::mfma16(__builtin_bit_cast(V8, vf[e]), pf, acc[e]);
        if (more) {
            load_vals(next);
            blocks(next + kWaves * kStep);
        }
    }

    if (__any(odd))
        for (t = part.begin + wave * kStep; t < part.end; t += kWaves * kStep) {
            if (t + kStep <= min(least, part.end)) continue;
            for (uint32_t k = t; k < min(t + kStep, part.end); ++k) {
                const uint64_t at = table[k >> shift] * C;
                const uint32_t slot = k & (T - 1);
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = odd_value<POOL, M>(vbase + at + slot * kRow,
                                                           vpair + at + slot * kPairs,
                                                           (kg * 4 + r) * E + e);
                        acc[e][r] += k < min(limit, part.end) ? x : 0.0f;
                    }
            }
        }

    // The waves' sums, on a common maximum.
    __shared__ float tops[kWaves][16], sums[kWaves][16];
    __shared__ __attribute__((aligned(16))) float part_sum[kWaves][16][D + 4];
    sum = over_rows(sum, Sum());
    if (kg == 0) tops[wave][col] = top;
    __syncthreads();
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
    const float norm = a.v_scale / total;
    uint8_t* out = a.out + 2 * (row * a.out_stride + h * D + od);
    if constexpr (E == 4) {
        *reinterpret_cast<u32x2*>(out) =
            u32x2{pack2<Q>(o[0] * norm, o[1] * norm), pack2<Q>(o[2] * norm, o[3] * norm)};
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 8)
            *reinterpret_cast<u32x4*>(out + 2 * e) =
                u32x4{pack2<Q>(o[e] * norm, o[e + 1] * norm),
                      pack2<Q>(o[e + 2] * norm, o[e + 3] * norm),
                      pack2<Q>(o[e + 4] * norm, o[e + 5] * norm),
                      pack2<Q>(o[e + 6] * norm, o[e + 7] * norm)};
    }
    if (a.lse && od == 0)
        a.lse[row * a.q_heads + h] = (high - kLift + __builtin_log2f(total)) * kLn2;
}

// Joins the parts of 16 columns: a wave a column, four columns a workgroup.
// Lanes take four values each and, where a column has fewer than 256, the parts in
// turn.  Every sum has a fixed order.
template <typename Q, int D>
__global__ __launch_bounds__(256) void join_kernel(const KvAttend a) {
    const uint32_t H = a.layer.H;
    const uint32_t quarter = blockIdx.x % 4, head = blockIdx.x / 4 % H, item = blockIdx.x / 4 / H;
    if (item >= a.t.head->joins) return;
    const KvJoin join = a.t.joins[item];
    const KvSeq seq = a.t.seqs[join.seq];
    const uint32_t col = quarter * 4 + threadIdx.x / 64, c = join.tile * kRowColumns + col;
    if (c >= a.group * seq.fresh) return;
    const int lane = threadIdx.x % 64;
    constexpr int kLanes = D / 4, kTurns = 64 / kLanes;
    const uint64_t step = (uint64_t)join.stride * H * slot_floats(D);
    const float* first = a.t.slots + ((uint64_t)join.slot * H + head) * slot_floats(D);

    float top = -__builtin_inff();
    for (uint32_t p = lane; p < join.parts; p += 64)
        top = fmaxf(top, first[p * step + 16 * D + col]);
#pragma unroll
    for (int m = 32; m; m /= 2) top = fmaxf(top, __shfl_xor(top, m));
    const int turn = lane / kLanes, d = lane % kLanes * 4;
    f32x4 o = {0, 0, 0, 0};
    float total = 0.0f;
#pragma unroll 4
    for (uint32_t p = turn; p < join.parts; p += kTurns) {
        const float* slot = first + p * step;
        const float w = exp2_(slot[16 * D + col] - top);
        total += w * slot[16 * D + 16 + col];
        o += w * *reinterpret_cast<const f32x4*>(slot + col * D + d);
    }
#pragma unroll
    for (int m = kLanes; m < 64; m *= 2) {
        total += __shfl_xor(total, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m);
    }
    if (turn) return;
    const uint64_t row = seq.row + c / a.group, h = head * a.group + c % a.group;
    const float norm = a.v_scale / total;
    *reinterpret_cast<u32x2*>(a.out + 2 * (row * a.out_stride + h * D + d)) =
        u32x2{pack2<Q>(o[0] * norm, o[1] * norm), pack2<Q>(o[2] * norm, o[3] * norm)};
    if (a.lse && d == 0)
        a.lse[row * a.q_heads + h] = (top - kLift + __builtin_log2f(total)) * kLn2;
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
    const uint32_t grid = joins * a.layer.H * 4;
    return a.dtype == AQUA_F16 ? join<f16>(a, grid, stream) : join<bf16>(a, grid, stream);
}

hipError_t launch_attend(const KvAttend& a, const KvCounts& n, hipStream_t stream) {
    hipError_t e = launch_tiles(a, n.tiles, stream);
    if (e == hipSuccess) e = launch_rows(a, n.rows, stream);
    if (e == hipSuccess) e = launch_join(a, n.joins, stream);
    return e;
}

}  // namespace aqua
