// kv_testapi.cpp -- C entry points into the operators' host planning for CPU
// tests (libaqua_core.so only).
#include <algorithm>
#include <cstring>

#include "kv_plan.h"

extern "C" {

// out: group, rows, tiles, joins, slots.
aqua_status aqua_core_kv_limits(const aqua_kv_desc* pool, const aqua_kv_batch_desc* d,
                                uint32_t* out) {
    aqua::Shape s;
    aqua_status st = aqua::make_shape(pool, &s);
    if (st != AQUA_OK) return st;
    aqua::KvLimits m;
    st = aqua::kv_limits(s, d, &m);
    if (st != AQUA_OK) return st;
    const uint32_t v[5] = {m.group, m.rows, m.tiles, m.joins, m.slots};
    std::memcpy(out, v, sizeof(v));
    return AQUA_OK;
}

// Plans a step; counts: rows, tiles, joins, tokens, append_ok, longest, slots.
// rows, tiles: 8 words an item (first, context, fresh, row, tile, begin, end, slot);
// joins: 6 words (row, column, count, slot, parts, stride); tokens: 2 words (block,
// position); at most `most` of each are written.
aqua_status aqua_core_kv_plan(const aqua_kv_desc* pool, const aqua_kv_batch_desc* d,
                              uint32_t num_seqs, const int32_t* ids, const uint64_t* offs,
                              const uint32_t* context, const uint32_t* fresh, uint32_t most,
                              uint32_t* counts, uint32_t* rows, uint32_t* tiles, uint32_t* joins,
                              uint32_t* tokens) {
    aqua::Shape s;
    aqua_status st = aqua::make_shape(pool, &s);
    if (st != AQUA_OK) return st;
    aqua::KvLimits m;
    st = aqua::kv_limits(s, d, &m);
    if (st != AQUA_OK) return st;
    aqua::KvPlan p;
    st = aqua::kv_plan(m, num_seqs, ids, offs, context, fresh, &p);
    if (st != AQUA_OK) return st;
    const uint32_t c[7] = {p.head.rows, p.head.tiles,  p.head.joins, p.new_tokens,
                           p.append_ok, p.longest, p.slots};
    std::memcpy(counts, c, sizeof(c));
    for (uint32_t i = 0; i < std::min<uint32_t>(most, p.head.rows); ++i)
        std::memcpy(rows + 8 * i, &p.rows[i], 32);
    for (uint32_t i = 0; i < std::min<uint32_t>(most, p.head.tiles); ++i)
        std::memcpy(tiles + 8 * i, &p.tiles[i], 32);
    for (uint32_t i = 0; i < std::min<uint32_t>(most, p.head.joins); ++i)
        std::memcpy(joins + 6 * i, &p.joins[i], 24);
    for (uint32_t i = 0; i < std::min<uint32_t>(most, p.new_tokens); ++i)
        std::memcpy(tokens + 2 * i, &p.tokens[i], 8);
    return AQUA_OK;
}

}  // extern "C"
