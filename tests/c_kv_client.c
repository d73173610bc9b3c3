/*
 * c_kv_client.c -- a plain C program that uses the operators on the pool through
 * include/aqua.h alone, with memory and streams from the HIP runtime: no Python
 * and no torch in the process.
 *
 * Two sequences of a small fp16 pool (2 layers, 32 blocks of 16 tokens, 2 KV heads of
 * 64, 4 query heads): one of 70 tokens of which 5 are new, and a whole prompt of 33.
 * Their new keys and values are appended to layer 1, rotated, and attended over;
 * then both are swapped out, swapped in to other blocks, and a captured attention of
 * each sequence's last token over the new tables is replayed twice.  Calls that the
 * header says are refused are made on the way.  Into a directory go, for the
 * test that compares them with the definitions:
 *
 *   pool_before.bin, k.bin, v.bin, q.bin, rope.bin        what the calls were given
 *   q_out.bin, pool_after.bin, out.bin, lse.bin           what the step gave
 *   out_moved.bin, lse_moved.bin                          what the replays gave
 *
 * The tables are fixed below.  Exit status 0 and a last line "c_kv_client: ok" mean
 * every call returned what the header says.
 */
#define _POSIX_C_SOURCE 200112L
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "aqua.h"

#define L 2u
#define N 32u
#define H 2u
#define T 16u
#define D 64u
#define HQ 4u
#define LAYER 1u
#define POOL_BYTES (2ull * L * N * 2 * H * T * D)
#define NEW 38u
#define NBLK 8u
#define ROPE_ROWS 70u
#define IMG_BYTES (POOL_BYTES / N * NBLK)

static const int32_t IDS[NBLK] = {30, 2, 17, 4, 9, 0, 31, 11};
static const int32_t MOVED[NBLK] = {1, 3, 5, 7, 8, 10, 12, 14};
static const int32_t WRONG[NBLK] = {30, 2, 17, 4, 9, 0, 32, 11};
static const int32_t SHARED[NBLK] = {30, 2, 17, 4, 9, 0, 9, 11};
static const uint64_t OFFS[3] = {0, 5, 8};
static const uint32_t CONTEXT[2] = {70, 33};
static const uint32_t FRESH[2] = {5, 33};
static const uint32_t LAST[2] = {1, 1};

static uint64_t seed = 1;

static uint64_t next(void) {
    seed ^= seed << 13;
    seed ^= seed >> 7;
    seed ^= seed << 17;
    return seed >> 16;
}

/* fp16 numbers of 2^-3 to 2 in size. */
static void fill16(uint16_t* p, uint64_t n) {
    for (uint64_t i = 0; i < n; ++i) {
        const uint64_t x = next();
        p[i] = (uint16_t)((x & 0x83ffu) | ((12u + (x >> 20) % 4u) << 10));
    }
}

static int hip(hipError_t e, const char* what) {
    if (e != hipSuccess) fprintf(stderr, "c_kv_client: %s: %s\n", what, hipGetErrorString(e));
    return e != hipSuccess;
}

static int returns(aqua_status want, aqua_status got, const char* what) {
    if (got != want)
        fprintf(stderr, "c_kv_client: %s: %s, not %s\n", what, aqua_status_str(got),
                aqua_status_str(want));
    return got != want;
}

static int dump(const char* dir, const char* name, const void* device, uint64_t n) {
    char path[4096];
    void* p = malloc(n);
    snprintf(path, sizeof path, "%s/%s", dir, name);
    FILE* f = fopen(path, "wb");
    int bad = !p || !f || hip(hipMemcpy(p, device, n, hipMemcpyDeviceToHost), "read") ||
              fwrite(p, 1, n, f) != n;
    if (bad) fprintf(stderr, "c_kv_client: cannot write %s\n", path);
    if (f) bad |= fclose(f) != 0;
    free(p);
    return bad;
}

static void* upload(const void* host, uint64_t n) {
    void* p = NULL;
    if (hip(hipMalloc(&p, n), "hipMalloc")) exit(1);
    if (host ? hip(hipMemcpy(p, host, n, hipMemcpyHostToDevice), "upload")
             : hip(hipMemset(p, 0, n), "clear"))
        exit(1);
    return p;
}

int main(int argc, char** argv) {
    if (argc != 2) {
        fprintf(stderr, "usage: %s OUT_DIR\n", argv[0]);
        return 2;
    }
    const char* dir = argv[1];
    static uint16_t host[POOL_BYTES / 2], k_h[NEW * H * D], v_h[NEW * H * D], q_h[NEW * HQ * D];
    static float rope_h[ROPE_ROWS * D];
    fill16(host, POOL_BYTES / 2);
    fill16(k_h, NEW * H * D);
    fill16(v_h, NEW * H * D);
    fill16(q_h, NEW * HQ * D);
    for (uint32_t i = 0; i < ROPE_ROWS * D; ++i) rope_h[i] = (float)(next() % 2001u) / 1000.0f - 1.0f;
    if (hip(hipSetDevice(0), "hipSetDevice")) return 1;
    void *pool = upload(host, POOL_BYTES), *image = upload(NULL, IMG_BYTES);
    void *k = upload(k_h, sizeof k_h), *v = upload(v_h, sizeof v_h), *q = upload(q_h, sizeof q_h);
    void *rope = upload(rope_h, sizeof rope_h), *q_out = upload(NULL, sizeof q_h);
    void *out = upload(NULL, sizeof q_h), *lse = upload(NULL, NEW * HQ * 4);
    hipStream_t s = NULL;
    if (hip(hipStreamCreate(&s), "hipStreamCreate") ||
        dump(dir, "pool_before.bin", pool, POOL_BYTES) || dump(dir, "k.bin", k, sizeof k_h) ||
        dump(dir, "v.bin", v, sizeof v_h) || dump(dir, "q.bin", q, sizeof q_h) ||
        dump(dir, "rope.bin", rope, sizeof rope_h))
        return 1;

    const aqua_kv_desc shape = {L, N, H, T, D, AQUA_F16};
    const aqua_kv_batch_desc most = {HQ, 2, NEW, NBLK}, odd_heads = {HQ + 1, 2, NEW, NBLK};
    aqua_kv_pool_t kv = NULL;
    aqua_kv_batch_t batch = NULL;
    if (returns(AQUA_OK, aqua_kv_pool_create(&shape, pool, POOL_BYTES, &kv), "pool") ||
        returns(AQUA_ERR_INVALID, aqua_kv_batch_create(kv, &odd_heads, &batch), "odd heads") ||
        returns(AQUA_ERR_INVALID, aqua_kv_batch_create(kv, NULL, &batch), "no limits") ||
        returns(AQUA_OK, aqua_kv_batch_create(kv, &most, &batch), "batch"))
        return 1;

    /* A step that cannot be, and one that an append may not write. */
    aqua_kv_append_args a = {k, v, q, q_out, H * D, H * D, HQ * D, HQ * D, AQUA_F16, 0,
                             rope, ROPE_ROWS, D, 1.0f, 1.0f};
    if (returns(AQUA_ERR_RANGE, aqua_kv_batch_set(batch, 2, WRONG, OFFS, CONTEXT, FRESH, s),
                "a block outside the pool") ||
        returns(AQUA_ERR_CAPACITY, aqua_kv_batch_set(batch, 2, IDS, OFFS, CONTEXT, CONTEXT, s),
                "more tokens than the batch holds") ||
        returns(AQUA_OK, aqua_kv_batch_set(batch, 2, SHARED, OFFS, CONTEXT, FRESH, s), "shared") ||
        returns(AQUA_ERR_DUPLICATE, aqua_kv_append(batch, LAYER, &a, s), "a shared block"))
        return 1;

    /* The step. */
    aqua_kv_attend_args t = {q_out, out, lse, HQ * D, HQ * D, AQUA_F16, 0.125f, 1.0f, 1.0f};
    if (returns(AQUA_OK, aqua_kv_batch_set(batch, 2, IDS, OFFS, CONTEXT, FRESH, s), "set") ||
        returns(AQUA_ERR_INVALID, aqua_kv_append(batch, L, &a, s), "a layer too many") ||
        returns(AQUA_ERR_INVALID, aqua_kv_append(batch, LAYER, NULL, s), "no arguments"))
        return 1;
    a.rope_rows = ROPE_ROWS - 1;
    if (returns(AQUA_ERR_INVALID, aqua_kv_append(batch, LAYER, &a, s), "a short table")) return 1;
    a.rope_rows = ROPE_ROWS;
    if (returns(AQUA_OK, aqua_kv_append(batch, LAYER, &a, s), "append") ||
        returns(AQUA_OK, aqua_kv_attend(batch, LAYER, &t, s), "attend"))
        return 1;
    t.out = q_out;
    if (returns(AQUA_ERR_INVALID, aqua_kv_attend(batch, LAYER, &t, s), "onto the queries")) return 1;
    t.out = out;
    if (hip(hipStreamSynchronize(s), "step") || dump(dir, "q_out.bin", q_out, sizeof q_h) ||
        dump(dir, "pool_after.bin", pool, POOL_BYTES) || dump(dir, "out.bin", out, sizeof q_h) ||
        dump(dir, "lse.bin", lse, NEW * HQ * 4))
        return 1;

    /* Preempted, and on from other blocks. */
    uint64_t ticket = 0;
    if (returns(AQUA_OK, aqua_swap_out(kv, 2, IDS, OFFS, image, IMG_BYTES, NULL,
                                       AQUA_TARGET_DEVICE, s, &ticket), "swap out") ||
        returns(AQUA_OK, aqua_sync(kv, ticket), "sync") ||
        hip(hipMemset(pool, 0xff, POOL_BYTES), "overwrite") ||
        hip(hipDeviceSynchronize(), "overwrite") ||
        returns(AQUA_OK, aqua_swap_in(kv, 2, MOVED, OFFS, image, IMG_BYTES, NULL,
                                      AQUA_TARGET_DEVICE, s, &ticket), "swap in") ||
        returns(AQUA_OK, aqua_stream_wait(kv, ticket, s), "wait"))
        return 1;
    /* Rows 0 and 1 are the last tokens' queries; a captured call's tensors have
     * max_tokens rows. */
    const uint64_t row = HQ * D * 2;
    hipGraph_t graph = NULL;
    hipGraphExec_t exec = NULL;
    if (hip(hipMemcpyAsync(q, (char*)q_out + 4 * row, row, hipMemcpyDeviceToDevice, s), "query") ||
        hip(hipMemcpyAsync((char*)q + row, (char*)q_out + (NEW - 1) * row, row,
                           hipMemcpyDeviceToDevice, s), "query") ||
        hip(hipStreamSynchronize(s), "queries"))
        return 1;
    t.q = q;
    if (hip(hipStreamBeginCapture(s, hipStreamCaptureModeThreadLocal), "capture") ||
        returns(AQUA_ERR_INVALID, aqua_kv_batch_set(batch, 2, MOVED, OFFS, CONTEXT, LAST, s),
                "a set in a capture") ||
        returns(AQUA_OK, aqua_kv_attend(batch, LAYER, &t, s), "captured") ||
        hip(hipStreamEndCapture(s, &graph), "end of capture") ||
        hip(hipGraphInstantiate(&exec, graph, NULL, NULL, 0), "instantiate"))
        return 1;
    for (int i = 0; i < 2; ++i)
        if (returns(AQUA_OK, aqua_kv_batch_set(batch, 2, MOVED, OFFS, CONTEXT, LAST, s), "set") ||
            hip(hipMemset(out, 0, 2 * row), "clear") || hip(hipDeviceSynchronize(), "clear") ||
            hip(hipGraphLaunch(exec, s), "replay") || hip(hipStreamSynchronize(s), "replay"))
            return 1;
    if (dump(dir, "out_moved.bin", out, 2 * row) || dump(dir, "lse_moved.bin", lse, 2 * HQ * 4))
        return 1;

    (void)hipGraphExecDestroy(exec);
    (void)hipGraphDestroy(graph);
    if (returns(AQUA_OK, aqua_kv_batch_destroy(batch), "destroy the batch") ||
        returns(AQUA_ERR_INVALID, aqua_kv_batch_destroy(NULL), "destroy nothing") ||
        returns(AQUA_OK, aqua_kv_pool_destroy(kv), "destroy the pool"))
        return 1;
    (void)hipStreamDestroy(s);
    void* all[] = {pool, image, k, v, q, rope, q_out, out, lse};
    for (unsigned i = 0; i < sizeof all / sizeof *all; ++i) (void)hipFree(all[i]);
    printf("c_kv_client: ok\n");
    return 0;
}
