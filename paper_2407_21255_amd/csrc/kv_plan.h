// kv_plan.h -- host planning of the operators on the pool (aqua_kv_batch_set):
// validation of a step and its split into work items.  Pure C++17, no HIP
// types, so that it builds and is tested on a machine without a GPU.
#pragma once

#include <cstdint>
#include <vector>

#include "aqua_core.h"

namespace aqua {

// A column is one (new token, query head) pair of a KV head: column c of
// sequence s is token c / G, head c % G of the G query heads that share the KV
// head.  Two kernels share the attention by the columns that a (sequence, KV
// head) has:
//   rows   16 columns a workgroup, whose four waves split the tokens: bound by
//          reading the cache;
//   tiles  many columns a workgroup, whose waves split the columns and share
//          the tokens through LDS: bound by the matrix products.
// Both take parts of a context where a whole one would leave compute units
// without work; the parts' sums are joined by a third kernel.
constexpr uint32_t kRowColumns = 16;

// Columns of a tiles workgroup, by head size: 8 waves of 32, or 4 where a
// wave's sums take twice the registers.
constexpr uint32_t tile_columns(uint32_t head_dim) { return head_dim > 128 ? 128 : 256; }

// Up to this many columns go to the rows kernel.  Measured with 32 contexts of 128 to
// 8192 tokens and 8 KV heads, us: rows with 16, 32 and 64 columns 56, 74 and 110; tiles
// with 72 and 128 columns 109 and 123.
constexpr uint32_t kRowsMostColumns = 64;

// How a kernel's items are split into parts of at most `most` tokens (part_tokens):
//   wide     workgroups that a round is counted as, for all head sizes: two a compute
//            unit (rows) and one (tiles).  By the kernels' registers and LDS, a compute unit
//            has room for three rows workgroups with heads of 128, three or four with
//            64 and one with 256, and for one of tiles; what follows was measured with
//            heads of 128;
//   step     tokens that a workgroup takes in a step: parts are whole ones;
//   fewest   tokens of a part that is worth a join;
//   rounds   parts of split items are at most `wide` times this many workgroups, and so are
//            all together, but where whole items take as many by themselves and a part
//            would be longer than all the work spread evenly: then splitting adds fewer
//            than this many rounds (600 contexts of 100 tokens and one of 131072, 8 KV
//            heads of 128: 148 us, and with the long one whole 1893);
//   start    what starting a part costs, and
//   join     what a launch that joins costs, in tokens (of 16 bits, where reading the
//            tokens is what takes the time: scaled by a pool's own).
// Measured on MI355X, us.  Rows, parts of 256 / 512 / 1024 tokens at least: one chat of
// 512 tokens 14.6 / 11.6 / 11.5 (a join is a launch more), three documents of 30001 to
// 131072 on one KV head 23.6 / 23.5 / 25.5, 64 chats the same.  `start` 64 / 320: 64
// chats in bf16 91 / 94, in 4 bits 47 / 42 (there 64 and 205 are one); 256 chats of up to
// 600 tokens, joined because nothing said what a join costs, 38, and left whole 35.
// Tiles, 512 tokens and a start of 128 / 128 and 256: a chunk of 100 tokens behind 4000
// 34.4 / 31.3, 1000 tokens of 64 heads 42.7 / 39.9, six prompts of 300 to 700
// 41.0 / 42.9.
struct KvSplit {
    uint32_t wide, step, fewest, rounds, start, join;
};
constexpr KvSplit kRows{512, 256, 512, 8, 64, 150};
constexpr KvSplit kTiles{256, 64, 256, 4, 256, 0};

constexpr uint32_t kMostContext = 1u << 30;
constexpr uint32_t kNoSlot = 0xffffffffu;

// Device structures, shared with the kernels.
struct KvHeader {
    uint32_t rows, tiles, joins;
    uint32_t append_tokens;  // tokens that an append writes: none where it must not
};
struct KvSeq {
    uint32_t first;  // of its table entries
    uint32_t context;
    uint32_t fresh;  // new tokens
    uint32_t row;    // of the first of them
};
struct alignas(8) KvToken {
    uint32_t block, position;
};
// One workgroup's work, for each KV head: the columns of tile `tile` (of 16, or
// of tile_columns) of a sequence over the tokens [begin, end).  slot: where the part's
// sums go in the workspace, in groups of H slots; kNoSlot: the part is the whole.
// It holds all that its workgroup has to know, so that one load brings it.
struct alignas(16) KvPart {
    KvSeq seq;
    uint32_t tile, begin, end, slot;
};
// One workgroup's join, for each KV head: `count` columns from `column` on (of the
// sequence's), all of one tile of 16, whose sums are in `parts` slots from `slot` on,
// one every `stride` groups.
struct alignas(16) KvJoin {
    uint32_t row, column, count, slot, parts, stride, reserved[2];
};
// A joining workgroup has this many groups of lanes, each with four values of a column
// a lane, and takes so many columns that a group has about kJoinAhead parts.
constexpr uint32_t join_groups(uint32_t head_dim) { return 1024 / head_dim; }
constexpr uint32_t kJoinAhead = 8;
static_assert(sizeof(KvHeader) == 16 && sizeof(KvToken) == 8 && sizeof(KvPart) == 32 &&
                  sizeof(KvJoin) == 32,
              "shared with the kernels");

// What a batch can hold at most.
struct KvLimits {
    Shape shape;
    uint32_t q_heads = 0, seqs = 0, tokens = 0, blocks = 0;
    uint32_t group = 0;                         // G
    uint32_t rows = 0, tiles = 0, joins = 0;    // work items
    uint32_t row_parts = 0, tile_parts = 0;     // of them, parts of items that are split
    uint32_t slots = 0;                         // groups of H slots of 16 columns
};

// Fills *out; AQUA_ERR_INVALID for a pool or limits that the operators do not take.
aqua_status kv_limits(const Shape& s, const aqua_kv_batch_desc* d, KvLimits* out);

// A step as planned.  Keeps its memory from one to the next.
struct KvPlan {
    KvHeader head{};
    std::vector<KvSeq> seqs;
    std::vector<KvPart> rows, tiles;
    std::vector<KvJoin> joins;
    std::vector<KvToken> tokens;
    uint32_t entries = 0;        // table entries
    uint32_t new_tokens = 0;
    uint32_t longest = 0;        // context with new tokens
    uint32_t slots = 0;          // groups used
    bool append_ok = true;       // no written block is in another table
    std::vector<uint32_t> ends;  // scratch: tokens of a kernel's items
    std::vector<uint64_t> mark;  // scratch: per block, (epoch, table entry)
    uint32_t epoch = 0;
};

// Validates the step and plans it; *plan is untouched unless it returns AQUA_OK.
// Precedence: invalid -> capacity -> range.
aqua_status kv_plan(const KvLimits& lim, uint32_t num_seqs, const int32_t* ids,
                    const uint64_t* offs, const uint32_t* context, const uint32_t* fresh,
                    KvPlan* plan);

}  // namespace aqua
