// kv_tiles.hip -- attention for many columns (prompts and chunks of them): 256
// columns a workgroup (128 for heads of 256), a wave 32, over tiles of 64 tokens (32)
// that the waves share through LDS.
//
// One pass over the tokens with a running maximum and sum.  Bound by the matrix
// products and, next to them, by the exponentials of the weights.  Per tile and wave:
//   S^T = K Q^T     32x32x16: A = keys from LDS, B = queries, which stay in
//                   registers; a lane's scores are of one column (lane % 32);
//   O^T += V^T P^T  A = values from LDS, B = the lane's weights as they stand: a
//                   16-token product takes, from lane half h, tokens 4h + 0..3 and
//                   8 + 4h + 0..3 of its 16, and V^T lies in LDS in that order.
// While a tile is computed the next one is on its way from the pool's blocks to
// registers; it is then widened to 16 bits and put into the other of two LDS
// buffers, so that one barrier a tile is enough.  LDS rows are whole multiples of the
// banks; 16-byte pieces are exchanged by the row's number (key_at, val_at), so that
// the lanes of a read fall on different banks.
#include "kv_device.h"

namespace aqua {
namespace {

using namespace kv;

// Tokens of a tile: heads of 256 leave no registers for more.
constexpr int tile_tokens(int D) { return D > 128 ? 32 : 64; }

// What a thread brings of a tile: units of 16 keys' values (of one token) and of 4
// tokens times 4 values.
template <int POOL, int D>
struct Raw;

template <int D>
struct Raw16 {
    u32x4 k[2];
    u32x2 v[4];
    __device__ void key(const uint8_t* row, const uint8_t*, int u) {
        k[0] = *reinterpret_cast<const u32x4*>(row + u * 32);
        k[1] = *reinterpret_cast<const u32x4*>(row + u * 32 + 16);
    }
    __device__ void val(int i, const uint8_t* row, const uint8_t*, int u) {
        v[i] = *reinterpret_cast<const u32x2*>(row + u * 8);
    }
    __device__ void clear(int i) { v[i] = u32x2{0, 0}; }
    template <typename M>
    __device__ void keys_of(u32x4 (&out)[2]) const {
        out[0] = k[0];
        out[1] = k[1];
    }
    template <typename M>
    __device__ void vals_of(u32x2 (&out)[4], int) const {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                out[2 * j][p] = pair_lo(v[2 * p][j], v[2 * p + 1][j]);
                out[2 * j + 1][p] = pair_hi(v[2 * p][j], v[2 * p + 1][j]);
            }
    }
};
template <int D>
struct Raw<kF16, D> : Raw16<D> {};
template <int D>
struct Raw<kBF16, D> : Raw16<D> {};

template <int D>
struct Raw<kFP8, D> {
    u32x4 k;
    uint32_t v[4];
    __device__ void key(const uint8_t* row, const uint8_t*, int u) {
        k = *reinterpret_cast<const u32x4*>(row + u * 16);
    }
    __device__ void val(int i, const uint8_t* row, const uint8_t*, int u) {
        v[i] = *reinterpret_cast<const uint32_t*>(row + u * 4);
    }
    __device__ void clear(int i) { v[i] = 0; }
    template <typename M>
    __device__ void keys_of(u32x4 (&out)[2]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            out[i / 2][i % 2 * 2] = Mat<M>::template from_fp8<false>(k[i]);
            out[i / 2][i % 2 * 2 + 1] = Mat<M>::template from_fp8<true>(k[i]);
        }
    }
    template <typename M>
    __device__ void vals_of(u32x2 (&out)[4], int) const {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint32_t a = v[2 * p], b = v[2 * p + 1];
            const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
            const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07030602u);  // a2 b2 a3 b3
            out[0][p] = Mat<M>::template from_fp8<false>(x);
            out[1][p] = Mat<M>::template from_fp8<true>(x);
            out[2][p] = Mat<M>::template from_fp8<false>(y);
            out[3][p] = Mat<M>::template from_fp8<true>(y);
        }
    }
};

template <int D>
struct Raw<kInt4, D> {
    u32x2 k;
    uint32_t kp, v[4], vp[4];
    __device__ void key(const uint8_t* row, const uint8_t* pairs, int u) {
        k = *reinterpret_cast<const u32x2*>(row + u * 8);
        kp = *reinterpret_cast<const uint32_t*>(pairs + u / 2 * 4);
    }
    // Four values are two codes of each half of a word.
    __device__ void val(int i, const uint8_t* row, const uint8_t* pairs, int u) {
        v[i] = *reinterpret_cast<const uint32_t*>(row + u / 2 * 4);
        vp[i] = *reinterpret_cast<const uint32_t*>(pairs + u / 8 * 4);
    }
    __device__ void clear(int i) { vp[i] = 0; }
    template <typename M>
    __device__ void keys_of(u32x4 (&out)[2]) const {
        const f16x2 s = __builtin_bit_cast(f16x2, pair_lo(kp, kp));
        const f16x2 b = __builtin_bit_cast(f16x2, pair_hi(kp, kp));
#pragma unroll
        for (int i = 0; i < 2; ++i)
            out[i] = {value4(codes4<0>(k[i]), s, b), value4(codes4<1>(k[i]), s, b),
                      value4(codes4<2>(k[i]), s, b), value4(codes4<3>(k[i]), s, b)};
    }
    template <typename M>
    __device__ void vals_of(u32x2 (&out)[4], int u) const {
        const int shift = (u & 1) * 8;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const f16x2 s = __builtin_bit_cast(f16x2, pair_lo(vp[2 * p], vp[2 * p + 1]));
            const f16x2 b = __builtin_bit_cast(f16x2, pair_hi(vp[2 * p], vp[2 * p + 1]));
            const uint32_t x = pair_lo(v[2 * p], v[2 * p + 1]) >> shift;
            const uint32_t y = pair_hi(v[2 * p], v[2 * p + 1]) >> shift;
            out[0][p] = value4(codes4<0>(x), s, b);
            out[1][p] = value4(codes4<0>(y), s, b);
            out[2][p] = value4(codes4<1>(x), s, b);
            out[3][p] = value4(codes4<1>(y), s, b);
        }
    }
};

// Byte offset of 16-byte piece `piece` of key row `row`, and of value row `d` (the
// tile's tokens of one value), in a buffer.
template <int D>
__device__ inline uint32_t key_at(uint32_t row, uint32_t piece) {
    const uint32_t x = D == 64 ? (row >> 1) & 7 : row & 15;
    return row * (2 * D) + (piece ^ x) * 16;
}
template <int TILE>
__device__ inline uint32_t val_at(uint32_t d, uint32_t piece) {
    const uint32_t x = TILE == 64 ? ((d >> 1) ^ (d >> 4)) & 7 : ((d >> 2) ^ (d >> 4)) & 3;
    return d * (2 * TILE) + (piece ^ x) * 16;
}

template <int POOL, typename Q, int D>
__global__ __launch_bounds__(2 * (int)tile_columns(D)) void tiles_kernel(const KvAttend a) {
    using M = std::conditional_t<POOL == kInt4, f16, Q>;
    using V8 = typename Mat<M>::v8;
    constexpr int kColumns = tile_columns(D), kThreads = 2 * kColumns;
    constexpr int kTile = tile_tokens(D), kRuns = kTile / 16, kWide = kTile / 32;
    static_assert(kTiles.step % kTile == 0, "parts are whole tiles");
    constexpr int kUnits = kTile * D / 16, kPer = (kUnits + kThreads - 1) / kThreads;
    constexpr int kSteps = D / 16, kOut = D / 32;
    const uint32_t H = a.layer.H;
    const uint32_t item = blockIdx.x / H, head = blockIdx.x % H;
    const KvPart part = a.t.tiles[item];   // (an old one, where there is none)
    if (item >= a.t.head->tiles) return;
    const KvSeq seq = part.seq;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col = lane % 32, half = lane / 32;
    const uint32_t G = a.group, T = a.layer.T, shift = a.layer.shift;
    const uint32_t columns = G * seq.fresh;
    const uint32_t c_all = part.tile * kColumns + wave * 32 + col;
    const uint32_t c = min(c_all, columns - 1);
    const uint32_t token = c / G;
    const uint32_t before = seq.context - seq.fresh;
    // The column sees tokens below its limit; the wave's columns see `least` tokens
    // all, and `most` at most.
    const uint32_t stop = min(before + token + 1, part.end);
    const uint32_t first = part.tile * kColumns + wave * 32;
    const uint32_t least = min(before + min(first, columns - 1) / G + 1, part.end);
    const uint32_t most = min(before + min(first + 31, columns - 1) / G + 1, part.end);

    const uint8_t* q = a.q + 2 * ((uint64_t)(seq.row + token) * a.q_stride +
                                  (uint64_t)(head * G + c % G) * D);
    V8 qf[kSteps];
    float scale2 = a.scale2;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
        qf[ks] = __builtin_bit_cast(
            V8, *reinterpret_cast<const u32x4*>(q + 2 * (ks * 16 + half * 8)));
    fit_queries<M, Q>(qf, &scale2, [](float x) { return over_halves(x, Max()); });
    fit_scale(qf, &scale2);

    constexpr uint32_t kRow = row_bytes<POOL>(D), kPairs = D / 32 * 4;
    const uint64_t C = a.layer.chunk_bytes;
    const uint8_t* const kbase = a.layer.base + (uint64_t)head * T * kRow;
    const uint8_t* const vbase = kbase + (uint64_t)H * T * kRow;
    const uint8_t* const kpair =
        a.layer.base + (uint64_t)2 * H * T * kRow + (uint64_t)head * T * kPairs;
    const uint8_t* const vpair = kpair + (uint64_t)H * T * kPairs;
    const int32_t* const table = a.t.blocks + seq.first;
    const uint32_t last = (seq.context - 1) >> shift;   // table entries are read up to here

    // Tokens that all of the workgroup's columns see, and whether values behind them
    // are not finite.
    const uint32_t shared_by_all = min(before + part.tile * kColumns / G + 1, part.end);
    __shared__ int odd;
    if (threadIdx.x == 0) odd = 0;
    __syncthreads();

    __shared__ __attribute__((aligned(16))) uint8_t keys[2][kTile * D * 2];
    __shared__ __attribute__((aligned(16))) uint8_t vals[2][kTile * D * 2];

    Raw<POOL, D> raw[kPer];
    uint32_t kb[kPer], vb[kPer];
    // Unit n of keys: token n / (D/16), its values from 16 (n % (D/16)) on.  Unit n of
    // values: tokens 4 (n / (D/4)) + 0..3, values 4 (n % (D/4)) + 0..3.
    const auto blocks = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t n = threadIdx.x + i * kThreads;
            kb[i] = table[min((t + n / (D / 16)) >> shift, last)];
            vb[i] = table[min((t + n / (D / 4) * 4) >> shift, last)];
        }
    };
    const auto fetch = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t n = threadIdx.x + i * kThreads;
            if (kUnits % kThreads && n >= kUnits) break;
            const uint32_t ks = (t + n / (D / 16)) & (T - 1);
            raw[i].key(kbase + kb[i] * C + ks * kRow, kpair + kb[i] * C + ks * kPairs, n % (D / 16));
            const uint32_t vs = (t + n / (D / 4) * 4) & (T - 1);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                raw[i].val(j, vbase + vb[i] * C + (vs + j) * kRow,
                           vpair + vb[i] * C + (vs + j) * kPairs, n % (D / 4));
        }
    };
    const auto put = [&](uint32_t t, int buf) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t n = threadIdx.x + i * kThreads;
            if (kUnits % kThreads && n >= kUnits) break;
            u32x4 kw[2];
            raw[i].template keys_of<M>(kw);
            const uint32_t row = n / (D / 16), piece = n % (D / 16) * 2;
            *reinterpret_cast<u32x4*>(&keys[buf][key_at<D>(row, piece)]) = kw[0];
            *reinterpret_cast<u32x4*>(&keys[buf][key_at<D>(row, piece + 1)]) = kw[1];
            const uint32_t quad = n / (D / 4), d4 = n % (D / 4);
            // What stands behind the context may be anything: no weight is no help
            // against NaN.
            if (t + kTile > seq.context)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t + quad * 4 + j >= seq.context) raw[i].clear(j);
            u32x2 vw[4];
            raw[i].template vals_of<M>(vw, d4);
            if (t + kTile > shared_by_all) {
                bool found = false;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int w = 0; w < 2; ++w) vw[j][w] = finite_or_zero<M>(vw[j][w], &found);
                if (found) odd = 1;
            }
            const uint32_t p = quad / 4 * 2 + quad % 2, at = quad / 2 % 2 * 8;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<u32x2*>(&vals[buf][val_at<kTile>(d4 * 4 + j, p) + at]) = vw[j];
        }
    };
    // Value row 32 dt + col's piece of run kt: the exchange makes it the piece that
    // row col has for run kt xor dt.
    uint32_t val_pos[kRuns];
#pragma unroll
    for (int k = 0; k < kRuns; ++k) val_pos[k] = val_at<kTile>(col, k * 2 + half);
    const auto val_of = [&](int buf, int dt, int kt) {
        return *reinterpret_cast<const u32x4*>(
            &vals[buf][val_pos[kt ^ (dt & (kRuns - 1))] + dt * 64 * kTile]);
    };

    f32x16 acc[kOut];
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
    float top = -__builtin_inff(), sum = 0.0f;

    blocks(part.begin);
    fetch(part.begin);
    blocks(part.begin + kTile);
    put(part.begin, 0);
    if (part.begin + kTile < part.end) {
        fetch(part.begin + kTile);
        blocks(part.begin + 2 * kTile);
    }
    __syncthreads();
    // The tile at t, in buffer `buf`; the next goes into the other.
    const auto tile = [&](auto buffer, uint32_t t) {
        constexpr int buf = decltype(buffer)::value;
        if (t < most) {
            f32x16 s[kWide];
#pragma unroll
            for (int i = 0; i < kWide; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                for (int i = 0; i < kWide; ++i) {
                    const u32x4 k = *reinterpret_cast<const u32x4*>(
                        &keys[buf][key_at<D>(i * 32 + col, ks * 2 + half)]);
                    s[i] = Mat<M>::mfma32(__builtin_bit_cast(V8, k), qf[ks], s[i]);
                }
            if (t + kTile > least) {
#pragma unroll
                for (int i = 0; i < kWide; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (t + 32 * i + 8 * (r / 4) + 4 * half + r % 4 >= stop)
                            s[i][r] = -__builtin_inff();
            }
            float high = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < kWide; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) high = fmaxf(high, s[i][r]);
            high = over_halves(high, Max()) * scale2;
            if (__any(high > top + kSlack)) {
                // (A column that has seen nothing keeps its -inf, and sums of 0.)
                const float raised = fmaxf(top, high);
                const float f = raised > -__builtin_inff() ? exp2_(top - raised) : 1.0f;
                top = raised;
                sum *= f;
#pragma unroll
                for (int d = 0; d < kOut; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[d][r] *= f;
            }
            const float off = top > -__builtin_inff() ? top - kLift : 0.0f;
            // Weights are rounded once, to the products' type: a second term with what that
            // leaves, as the rows kernel has it, would be half as many products again
            // where these are what takes the time.  An 8192-token bf16 prompt is off by
            // 0.0020 of its size against 64 bits, with weights in fp32 by 0.0015 (the
            // result's own rounding to bf16).
            V8 pf[kRuns];
#pragma unroll
            for (int kt = 0; kt < kRuns; ++kt) {
                u32x4 w;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int r = kt % 2 * 8 + 2 * p;
                    const float x = exp2_(__builtin_fmaf(s[kt / 2][r], scale2, -off));
                    const float y = exp2_(__builtin_fmaf(s[kt / 2][r + 1], scale2, -off));
                    sum += x + y;
                    w[p] = pack2<M>(x, y);
                }
                pf[kt] = __builtin_bit_cast(V8, w);
            }
#pragma unroll
            for (int kt = 0; kt < kRuns; ++kt)
#pragma unroll
                for (int d = 0; d < kOut; ++d)
                    acc[d] = Mat<M>::mfma32(__builtin_bit_cast(V8, val_of(buf, d, kt)), pf[kt],
                                            acc[d]);
        }
        if (t + kTile < part.end) {
            put(t + kTile, buf ^ 1);
            if (t + 2 * kTile < part.end) {
                fetch(t + 2 * kTile);
                blocks(t + 3 * kTile);
            }
        }
        __syncthreads();
    };
    for (uint32_t t = part.begin; t < part.end; t += 2 * kTile) {
        tile(std::integral_constant<int, 0>(), t);
        if (t + kTile < part.end) tile(std::integral_constant<int, 1>(), t + kTile);
    }

    if (odd) {
        uint32_t k = part.begin;
        if (shared_by_all > k) k += (shared_by_all - k) / kTile * kTile;
        for (; k < most; ++k) {
            const uint64_t at = table[k >> shift] * C;
            const uint32_t slot = k & (T - 1);
#pragma unroll
            for (int d = 0; d < kOut; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float x = odd_value<POOL, M>(vbase + at + slot * kRow,
                                                       vpair + at + slot * kPairs,
                                                       d * 32 + r / 4 * 8 + half * 4 + r % 4);
                    acc[d][r] += k < stop ? x : 0.0f;
                }
        }
    }
    sum = over_halves(sum, Sum());
    if (c_all >= columns) return;
    if (part.slot != kNoSlot) {
        const uint32_t w = wave * 32 + col, oc = w % kRowColumns;
        float* slot =
            a.t.slots + ((uint64_t)(part.slot + w / kRowColumns) * H + head) * slot_floats(D);
#pragma unroll
        for (int d = 0; d < kOut; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4*>(slot + oc * D + d * 32 + r * 2 + half * 4) =
                    f32x4{acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]};
        if (!half) {
            slot[16 * D + oc] = top;
            slot[16 * D + 16 + oc] = sum;
        }
        return;
    }
    const uint64_t row = seq.row + token, h = head * G + c % G;
    // (The values' scale by itself: over the sum it may be too small for fp32.  Only fp8
    // pools have one.)
    const float norm = 1.0f / sum;
#pragma unroll
    for (int d = 0; d < kOut; ++d) acc[d] *= norm;
    if (POOL == kFP8)
#pragma unroll
        for (int d = 0; d < kOut; ++d) acc[d] *= a.v_scale;
    uint8_t* out = a.out + 2 * (row * a.out_stride + h * D);
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<u32x2*>(out + 2 * (d * 32 + r * 2 + half * 4)) =
                u32x2{pack2<Q>(acc[d][r], acc[d][r + 1]), pack2<Q>(acc[d][r + 2], acc[d][r + 3])};
    if (a.lse && !half)
        a.lse[row * a.q_heads + h] = (top - kLift + __builtin_log2f(sum)) * kLn2;
}

template <int POOL, typename Q, int D>
hipError_t launch(const KvAttend& a, uint32_t grid, hipStream_t stream) {
    (void)hipGetLastError();
    hipLaunchKernelGGL((tiles_kernel<POOL, Q, D>), dim3(grid), dim3(2 * tile_columns(D)), 0,
                       stream, a);
    return hipGetLastError();
}

template <int POOL, typename Q>
hipError_t tiles(const KvAttend& a, uint32_t grid, hipStream_t stream) {
    switch (a.layer.D) {
        case 64: return launch<POOL, Q, 64>(a, grid, stream);
        case 128: return launch<POOL, Q, 128>(a, grid, stream);
        default: return launch<POOL, Q, 256>(a, grid, stream);
    }
}

}  // namespace

hipError_t launch_tiles(const KvAttend& a, uint32_t items, hipStream_t stream) {
    if (!items) return hipSuccess;
    const uint32_t grid = items * a.layer.H;
    const bool half = a.dtype == AQUA_F16;
    switch (a.layer.dtype) {
        case AQUA_F16: return tiles<kF16, f16>(a, grid, stream);
        case AQUA_BF16: return tiles<kBF16, bf16>(a, grid, stream);
        case AQUA_FP8_E4M3: return half ? tiles<kFP8, f16>(a, grid, stream)
                                        : tiles<kFP8, bf16>(a, grid, stream);
        default: return half ? tiles<kInt4, f16>(a, grid, stream)
                             : tiles<kInt4, bf16>(a, grid, stream);
    }
}

}  // namespace aqua
