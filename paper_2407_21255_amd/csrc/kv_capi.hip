// kv_capi.hip -- C entry points of the operators on the pool: a batch's tables
// and staging memory, the checks of a call's tensors, the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <utility>

#include <rocprofiler-sdk-roctx/roctx.h>

#include "aqua.h"
#include "kv_ops.h"
#include "kv_plan.h"
#include "pool_view.h"

namespace {

constexpr int kStages = 4;  // sets that may be in flight
constexpr uint64_t kAlign = 256;

struct Range {
    explicit Range(const char* name) { roctxRangePushA(name); }
    ~Range() { roctxRangePop(); }
    Range(const Range&) = delete;
    Range& operator=(const Range&) = delete;
};

// Makes the batch's device current for the duration of a call.
struct OnDevice {
    int before = -1;
    bool ok;
    explicit OnDevice(int device) {
        ok = hipGetDevice(&before) == hipSuccess &&
             (before == device || hipSetDevice(device) == hipSuccess);
        if (before == device) before = -1;
    }
    ~OnDevice() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

// Where the tables lie in the device memory and in each staging slot.
struct Layout {
    uint64_t rows, tiles, joins, tokens, blocks, bytes;
};

Layout layout_of(const aqua::KvLimits& m) {
    Layout l;
    uint64_t at = kAlign;  // the header's
    const auto take = [&at](uint64_t n) {
        const uint64_t here = at;
        at += (n + kAlign - 1) / kAlign * kAlign;
        return here;
    };
    l.rows = take(m.rows * sizeof(aqua::KvPart));
    l.tiles = take(m.tiles * sizeof(aqua::KvPart));
    l.joins = take(m.joins * sizeof(aqua::KvJoin));
    l.tokens = take(m.tokens * sizeof(aqua::KvToken));
    l.blocks = take(m.blocks * sizeof(int32_t));
    l.bytes = at;
    return l;
}

// [ptr, ptr + n) in one allocation of device memory of `device`.
bool device_range(int device, const void* ptr, uint64_t n) {
    if (!ptr) return false;
    hipPointerAttribute_t attr;
    std::memset(&attr, 0, sizeof(attr));
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipPointerGetAttributes(&attr, ptr) != hipSuccess ||
        hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)ptr) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    const uintptr_t b = (uintptr_t)base, x = (uintptr_t)ptr;
    return attr.type == hipMemoryTypeDevice && attr.device == device && x >= b &&
           x - b <= size && n <= size - (x - b);
}

// A tensor [rows][heads][D] of 16-bit elements, `stride` elements from row to row.
bool tensor_ok(int device, const void* ptr, uint64_t rows, uint64_t heads, uint64_t D,
               uint64_t stride) {
    if ((uintptr_t)ptr % 16 || stride % 8 || stride < heads * D || stride > (1ull << 40)) return false;
    return !rows || device_range(device, ptr, 2 * ((rows - 1) * stride + heads * D));
}

// Whether rows of aw elements at a and of bw at b, with strides as and bs, share bytes:
// exact where the strides are equal, else by the tensors' extents.
bool rows_meet(const void* a, uint64_t as, uint64_t aw, const void* b, uint64_t bs, uint64_t bw,
               uint64_t rows) {
    if (!rows) return false;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    if (x + 2 * ((rows - 1) * as + aw) <= y || y + 2 * ((rows - 1) * bs + bw) <= x)
        return false;
    if (as != bs) return true;
    // Bytes from the start of a's row to the start of b's next.
    const uint64_t apart = x <= y ? (y - x) % (2 * as) : 2 * as - 1 - (x - y - 1) % (2 * as);
    return apart < 2 * aw || 2 * as - apart < 2 * bw;
}

// Bytes of a tensor from its first element to its last.
uint64_t extent(uint64_t rows, uint64_t stride, uint64_t width) {
    return rows ? 2 * ((rows - 1) * stride + width) : 0;
}

// Whether [a, a + an) and [b, b + bn) share bytes.
bool bytes_meet(const void* a, uint64_t an, const void* b, uint64_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return an && bn && x < y + bn && y < x + an;
}

bool positive(float x) { return std::isfinite(x) && x > 0.0f; }

bool capturing(hipStream_t stream) {
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    if (!stream) return false;  // the null stream cannot be captured
    if (hipStreamIsCapturing(stream, &st) != hipSuccess) (void)hipGetLastError();
    return st != hipStreamCaptureStatusNone;
}

}  // namespace

struct aqua_kv_batch {
    aqua::PoolView pool;
    aqua::KvLimits limits;
    aqua::KvPlan plan;              // of the last set
    aqua::KvPlan scratch;           // of the one being made
    Layout layout{};
    uint8_t* device = nullptr;      // the tables
    float* slots = nullptr;         // split sums
    uint8_t* stage[kStages] = {};   // pinned, as the host writes them
    uint8_t* stage_dev[kStages] = {};
    hipEvent_t staged[kStages] = {};
    bool used[kStages] = {};
    int next = 0;

    aqua::KvTables tables() const {
        return {reinterpret_cast<const aqua::KvHeader*>(device),
                reinterpret_cast<const aqua::KvPart*>(device + layout.rows),
                reinterpret_cast<const aqua::KvPart*>(device + layout.tiles),
                reinterpret_cast<const aqua::KvJoin*>(device + layout.joins),
                reinterpret_cast<const aqua::KvToken*>(device + layout.tokens),
                reinterpret_cast<const int32_t*>(device + layout.blocks), slots};
    }
    aqua::KvLayer layer(uint32_t l) const {
        const aqua::Shape& s = pool.shape;
        return {pool.base + (uint64_t)l * s.N * s.C, s.C, s.H, s.T, s.D,
                (uint32_t)__builtin_ctz(s.T), s.dtype};
    }
    aqua::KvCounts counts(bool captured) const {
        if (captured) return {limits.rows, limits.tiles, limits.joins, limits.tokens};
        return {plan.head.rows, plan.head.tiles, plan.head.joins, plan.new_tokens};
    }
    bool takes(int32_t dtype) const {
        if (dtype != AQUA_F16 && dtype != AQUA_BF16) return false;
        const int32_t d = pool.shape.dtype;
        return d == AQUA_FP8_E4M3 || d == AQUA_INT4 || d == dtype;
    }
    bool scales_ok(float k, float v) const {
        return pool.shape.dtype == AQUA_FP8_E4M3 ? positive(k) && positive(v)
                                                 : k == 1.0f && v == 1.0f;
    }
};

namespace {

void free_batch(aqua_kv_batch* b) {
    (void)hipFree(b->device);
    (void)hipFree(b->slots);
    for (int k = 0; k < kStages; ++k) {
        if (b->stage[k]) (void)hipHostFree(b->stage[k]);
        if (b->staged[k]) (void)hipEventDestroy(b->staged[k]);
    }
    (void)hipGetLastError();
    delete b;
}

// Launches each source file's kernels once with nothing to do, so that the runtime
// loads their code at the first batch of a device and not in its first step.
hipError_t warm(const aqua_kv_batch* b) {
    static std::mutex mu;
    static uint64_t done = 0;  // a bit a device; devices from 64 on load lazily
    std::lock_guard<std::mutex> lk(mu);
    const uint64_t bit = b->pool.device < 64 ? 1ull << b->pool.device : 0;
    if (!bit || (done & bit)) return hipSuccess;
    aqua::KvAttend a{};
    a.t = b->tables();  // whose header is 0: every workgroup ends at once
    a.layer = b->layer(0);
    a.group = 1;
    a.dtype = b->takes(AQUA_F16) ? AQUA_F16 : AQUA_BF16;
    aqua::KvAppend p{};
    p.t = a.t;
    p.layer = a.layer;
    p.dtype = a.dtype;
    hipError_t e = aqua::launch_append(p, {0, 0, 0, 1}, nullptr);
    if (e == hipSuccess) e = aqua::launch_attend(a, {1, 1, 1, 0}, nullptr);
    const hipError_t es = hipDeviceSynchronize();
    if (e == hipSuccess) e = es;
    if (e == hipSuccess) done |= bit;
    (void)hipGetLastError();
    return e;
}

}  // namespace

extern "C" {

aqua_status aqua_kv_batch_create(aqua_kv_pool_t pool, const aqua_kv_batch_desc* desc,
                                 aqua_kv_batch_t* out) {
    Range trace("aqua_kv_batch_create");
    if (!pool || !out) return AQUA_ERR_INVALID;
    const aqua::PoolView view = aqua::view_of(pool);
    aqua::KvLimits limits;
    const aqua_status st = aqua::kv_limits(view.shape, desc, &limits);
    if (st != AQUA_OK) return st;
    OnDevice on(view.device);
    if (!on.ok) return AQUA_ERR_HIP;
    aqua_kv_batch* b = new (std::nothrow) aqua_kv_batch();
    if (!b) return AQUA_ERR_HIP;
    b->pool = view;
    b->limits = limits;
    b->layout = layout_of(limits);
    const uint64_t slots =
        (uint64_t)limits.slots * view.shape.H * aqua::slot_floats(view.shape.D) * sizeof(float);
    bool ok = hipMalloc(reinterpret_cast<void**>(&b->device), b->layout.bytes) == hipSuccess &&
              hipMalloc(reinterpret_cast<void**>(&b->slots), slots) == hipSuccess &&
              hipMemset(b->device, 0, kAlign) == hipSuccess &&
              hipStreamSynchronize(nullptr) == hipSuccess;  // a set's stream may not wait for it
    for (int k = 0; ok && k < kStages; ++k)
        ok = hipHostMalloc(reinterpret_cast<void**>(&b->stage[k]), b->layout.bytes,
                           hipHostMallocMapped | hipHostMallocCoherent) == hipSuccess &&
             hipHostGetDevicePointer(reinterpret_cast<void**>(&b->stage_dev[k]), b->stage[k], 0) ==
                 hipSuccess &&
             hipEventCreateWithFlags(&b->staged[k], hipEventDisableTiming) == hipSuccess;
    if (!ok || warm(b) != hipSuccess) {
        free_batch(b);
        return AQUA_ERR_HIP;
    }
    *out = b;
    return AQUA_OK;
}

aqua_status aqua_kv_batch_destroy(aqua_kv_batch_t b) {
    Range trace("aqua_kv_batch_destroy");
    if (!b) return AQUA_ERR_INVALID;
    OnDevice on(b->pool.device);
    const bool ok = on.ok && hipDeviceSynchronize() == hipSuccess;
    free_batch(b);
    return ok ? AQUA_OK : AQUA_ERR_HIP;
}

aqua_status aqua_kv_batch_set(aqua_kv_batch_t b, uint32_t num_seqs, const int32_t* block_ids,
                              const uint64_t* seq_offsets, const uint32_t* context_tokens,
                              const uint32_t* new_tokens, void* stream) {
    Range trace("aqua_kv_batch_set");
    if (!b) return AQUA_ERR_INVALID;
    const hipStream_t s = (hipStream_t)stream;
    OnDevice on(b->pool.device);
    if (!on.ok) return AQUA_ERR_HIP;
    if (capturing(s)) return AQUA_ERR_INVALID;
    aqua_status st;
    try {
        st = aqua::kv_plan(b->limits, num_seqs, block_ids, seq_offsets, context_tokens,
                           new_tokens, &b->scratch);
    } catch (const std::bad_alloc&) {
        st = AQUA_ERR_HIP;  // no memory, as where a handle cannot be allocated
    }
    if (st != AQUA_OK) return st;
    const int k = b->next;
    b->next = (k + 1) % kStages;
    if (b->used[k] && hipEventSynchronize(b->staged[k]) != hipSuccess) return AQUA_ERR_HIP;
    b->used[k] = false;

    const aqua::KvPlan& p = b->scratch;
    uint8_t* const host = b->stage[k];
    aqua::KvUpload up{};
    uint32_t pieces = 0;
    const auto piece = [&](uint64_t at, const void* from, uint64_t bytes) {
        if (bytes) std::memcpy(host + at, from, bytes);
        up.piece[pieces++] = {reinterpret_cast<const uint4*>(b->stage_dev[k] + at),
                              reinterpret_cast<uint4*>(b->device + at),
                              (uint32_t)((bytes + 15) / 16)};
    };
    piece(0, &p.head, sizeof(p.head));
    piece(b->layout.rows, p.rows.data(), p.rows.size() * sizeof(aqua::KvPart));
    piece(b->layout.tiles, p.tiles.data(), p.tiles.size() * sizeof(aqua::KvPart));
    piece(b->layout.joins, p.joins.data(), p.joins.size() * sizeof(aqua::KvJoin));
    piece(b->layout.tokens, p.tokens.data(), p.tokens.size() * sizeof(aqua::KvToken));
    piece(b->layout.blocks, block_ids, (uint64_t)p.entries * sizeof(int32_t));
    hipError_t e = aqua::launch_upload(up, s);
    if (e == hipSuccess) e = hipEventRecord(b->staged[k], s);
    if (e != hipSuccess) {
        (void)hipStreamSynchronize(s);
        (void)hipGetLastError();
        return AQUA_ERR_HIP;
    }
    b->used[k] = true;
    std::swap(b->plan, b->scratch);
    return AQUA_OK;
}

aqua_status aqua_kv_append(aqua_kv_batch_t b, uint32_t layer, const aqua_kv_append_args* x,
                           void* stream) {
    Range trace("aqua_kv_append");
    if (!b || !x || layer >= b->pool.shape.L) return AQUA_ERR_INVALID;
    const aqua::Shape& s = b->pool.shape;
    if (!b->takes(x->dtype) || !b->scales_ok(x->k_scale, x->v_scale)) return AQUA_ERR_INVALID;
    if (x->interleaved != 0 && x->interleaved != 1) return AQUA_ERR_INVALID;
    const hipStream_t st = (hipStream_t)stream;
    OnDevice on(b->pool.device);
    if (!on.ok) return AQUA_ERR_HIP;
    const bool captured = capturing(st);
    const uint32_t rows = captured ? b->limits.tokens : b->plan.new_tokens;
    const uint32_t q_heads = x->q ? b->limits.q_heads : 0;
    const int dev = b->pool.device;
    if (!tensor_ok(dev, x->k, rows, s.H, s.D, x->k_stride) ||
        !tensor_ok(dev, x->v, rows, s.H, s.D, x->v_stride))
        return AQUA_ERR_INVALID;
    if (x->q) {
        if (!tensor_ok(dev, x->q, rows, q_heads, s.D, x->q_stride) ||
            !tensor_ok(dev, x->q_out, rows, q_heads, s.D, x->q_out_stride))
            return AQUA_ERR_INVALID;
        const uint64_t width = (uint64_t)q_heads * s.D, own = (uint64_t)s.H * s.D;
        const bool in_place = x->q == x->q_out && x->q_stride == x->q_out_stride;
        const auto meets = [&](const void* p, uint64_t stride, uint64_t w) {
            return rows_meet(x->q_out, x->q_out_stride, width, p, stride, w, rows);
        };
        if ((!in_place && meets(x->q, x->q_stride, width)) || meets(x->k, x->k_stride, own) ||
            meets(x->v, x->v_stride, own) ||
            bytes_meet(x->q_out, extent(rows, x->q_out_stride, width), b->pool.base, s.pool_bytes))
            return AQUA_ERR_INVALID;
    }
    if (x->rope) {
        if (!x->rope_dim || x->rope_dim % 16 || x->rope_dim > s.D || (uintptr_t)x->rope % 16 ||
            x->rope_rows < b->plan.longest ||
            !device_range(dev, x->rope, 4ull * x->rope_rows * x->rope_dim) ||
            (x->q && bytes_meet(x->q_out, extent(rows, x->q_out_stride, (uint64_t)q_heads * s.D),
                                x->rope, 4ull * x->rope_rows * x->rope_dim)))
            return AQUA_ERR_INVALID;
    }
    if (!b->plan.append_ok) return AQUA_ERR_DUPLICATE;
    aqua::KvAppend a;
    a.t = b->tables();
    a.layer = b->layer(layer);
    a.k = (const uint8_t*)x->k;
    a.v = (const uint8_t*)x->v;
    a.q = (const uint8_t*)x->q;
    a.q_out = (uint8_t*)x->q_out;
    a.k_stride = x->k_stride;
    a.v_stride = x->v_stride;
    a.q_stride = x->q_stride;
    a.q_out_stride = x->q_out_stride;
    a.q_heads = q_heads;
    a.dtype = x->dtype;
    a.rope = x->rope;
    a.rope_rows = x->rope_rows;
    a.rope_dim = x->rope ? x->rope_dim : 0;
    a.interleaved = (uint32_t)x->interleaved;
    a.k_scale = x->k_scale;
    a.v_scale = x->v_scale;
    return aqua::launch_append(a, b->counts(captured), st) == hipSuccess ? AQUA_OK : AQUA_ERR_HIP;
}

aqua_status aqua_kv_attend(aqua_kv_batch_t b, uint32_t layer, const aqua_kv_attend_args* x,
                           void* stream) {
    Range trace("aqua_kv_attend");
    if (!b || !x || layer >= b->pool.shape.L) return AQUA_ERR_INVALID;
    const aqua::Shape& s = b->pool.shape;
    const float scale2 = (float)((double)x->scale * x->k_scale * 1.4426950408889634);
    if (!b->takes(x->dtype) || !b->scales_ok(x->k_scale, x->v_scale) || !std::isfinite(scale2))
        return AQUA_ERR_INVALID;
    const hipStream_t st = (hipStream_t)stream;
    OnDevice on(b->pool.device);
    if (!on.ok) return AQUA_ERR_HIP;
    const bool captured = capturing(st);
    const uint32_t rows = captured ? b->limits.tokens : b->plan.new_tokens;
    const uint32_t heads = b->limits.q_heads;
    const int dev = b->pool.device;
    const uint64_t width = (uint64_t)heads * s.D;
    if (!tensor_ok(dev, x->q, rows, heads, s.D, x->q_stride) ||
        !tensor_ok(dev, x->out, rows, heads, s.D, x->out_stride) ||
        rows_meet(x->q, x->q_stride, width, x->out, x->out_stride, width, rows))
        return AQUA_ERR_INVALID;
    const uint64_t out_bytes = extent(rows, x->out_stride, width), lse_bytes = 4ull * rows * heads;
    if (bytes_meet(x->out, out_bytes, b->pool.base, s.pool_bytes)) return AQUA_ERR_INVALID;
    if (x->lse && ((uintptr_t)x->lse % 4 || (rows && !device_range(dev, x->lse, lse_bytes)) ||
                   bytes_meet(x->lse, lse_bytes, x->out, out_bytes) ||
                   bytes_meet(x->lse, lse_bytes, x->q, extent(rows, x->q_stride, width)) ||
                   bytes_meet(x->lse, lse_bytes, b->pool.base, s.pool_bytes)))
        return AQUA_ERR_INVALID;
    aqua::KvAttend a;
    a.t = b->tables();
    a.layer = b->layer(layer);
    a.q = (const uint8_t*)x->q;
    a.out = (uint8_t*)x->out;
    a.lse = x->lse;
    a.q_stride = x->q_stride;
    a.out_stride = x->out_stride;
    a.q_heads = heads;
    a.group = b->limits.group;
    a.dtype = x->dtype;
    a.scale2 = scale2;
    a.v_scale = x->v_scale;
    return aqua::launch_attend(a, b->counts(captured), st) == hipSuccess ? AQUA_OK : AQUA_ERR_HIP;
}

}  // extern "C"
