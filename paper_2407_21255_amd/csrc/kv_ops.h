// kv_ops.h -- launch interface of the operators on the pool: append, the two
// attention kernels and the join of split sums.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "kv_plan.h"

namespace aqua {

// A batch's tables in device memory, as aqua_kv_batch_set left them.
struct KvTables {
    const KvHeader* head;
    const KvPart* rows;
    const KvPart* tiles;
    const KvJoin* joins;
    const KvToken* tokens;
    const int32_t* blocks;
    float* slots;  // per slot: [16][D] sums, [16] maxima, [16] totals
};

// Work items to launch for: the step's own, or a captured launch's limits.
struct KvCounts {
    uint32_t rows, tiles, joins, tokens;
};

// One layer of a pool.
struct KvLayer {
    uint8_t* base;         // of the layer's first block
    uint64_t chunk_bytes;  // C
    uint32_t H, T, D;
    uint32_t shift;        // T = 1 << shift
    int32_t dtype;
};

struct KvAppend {
    KvTables t;
    KvLayer layer;
    const uint8_t *k, *v, *q;
    uint8_t* q_out;
    uint64_t k_stride, v_stride, q_stride, q_out_stride;  // elements
    uint32_t q_heads;  // 0: no queries
    int32_t dtype;
    const float* rope;
    uint32_t rope_rows, rope_dim, interleaved;
    float k_scale, v_scale;
};

struct KvAttend {
    KvTables t;
    KvLayer layer;
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    uint64_t q_stride, out_stride;
    uint32_t q_heads, group;
    int32_t dtype;
    float scale2;   // of the scores, times log2(e): the softmax is in powers of two
    float v_scale;
};

hipError_t launch_append(const KvAppend& a, const KvCounts& n, hipStream_t stream);
hipError_t launch_attend(const KvAttend& a, const KvCounts& n, hipStream_t stream);

// The two attention kernels by themselves (launch_attend and the files that
// hold them).
hipError_t launch_rows(const KvAttend& a, uint32_t items, hipStream_t stream);
hipError_t launch_tiles(const KvAttend& a, uint32_t items, hipStream_t stream);
hipError_t launch_join(const KvAttend& a, uint32_t joins, hipStream_t stream);

// Floats of a workspace slot.
constexpr uint64_t slot_floats(uint32_t head_dim) { return kRowColumns * (head_dim + 2ull); }

// Copies pieces of pinned memory to device memory with one launch.
struct KvUpload {
    static constexpr uint32_t kPieces = 6;
    struct {
        const uint4* src;
        uint4* dst;
        uint32_t n;  // 16-byte vectors
    } piece[kPieces];
};
hipError_t launch_upload(const KvUpload& u, hipStream_t stream);

}  // namespace aqua
