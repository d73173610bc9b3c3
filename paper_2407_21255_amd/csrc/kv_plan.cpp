// kv_plan.cpp -- validation and work split of the operators on the pool (host
// only).
#include "kv_plan.h"

#include <algorithm>

namespace aqua {

namespace {

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Tokens of a part at most, for items of `ends` tokens (whose order is not kept).
// Workgroups start longest first, so a launch of r rounds of `wide` ends after r parts of
// the longest size, or the work of all spread evenly and one part more, whichever is less;
// every round starts its parts anew.  For each number of rounds, from what whole items
// take on, the smallest parts that fit them are found by bisection, and the rounds that
// end first are taken.  More than sp.rounds are looked at only where a part is still
// longer than all the work spread evenly, which the other workgroups cannot hide: one
// long context among so many short ones that these fill the rounds by themselves.
// `bits`: of a value; at most `most_items` items come of it, and `most_parts` parts of
// items that are split.
uint64_t part_tokens(std::vector<uint32_t>& ends, uint32_t H, const KvSplit& sp, uint32_t bits,
                     uint64_t most_items, uint64_t most_parts) {
    uint64_t work = 0, longest = 0;
    for (uint32_t e : ends) {
        work += (uint64_t)H * e;
        longest = std::max<uint64_t>(longest, e);
    }
    if (longest <= sp.fewest) return sp.fewest;
    // Those that may be split, first: often few.
    const auto split = std::partition(ends.begin(), ends.end(),
                                      [&](uint32_t e) { return e > sp.fewest; });
    const auto fits = [&](uint32_t most, uint64_t added) {
        uint64_t parts = 0;
        for (auto e = ends.begin(); e != split; ++e) {
            if (*e <= most) continue;
            const uint32_t n = (*e + most - 1) / most;
            parts += n;
            if (parts > most_parts || n - 1 > added) return false;
            added -= n - 1;
        }
        return true;
    };
    const uint64_t n = ends.size(), first = ceil_div(n * H, sp.wide);
    const uint64_t whole = ceil_div(longest, sp.step) * sp.step, even = ceil_div(work, sp.wide);
    const auto cost = [&](uint64_t rounds, uint64_t most) {
        return std::min(rounds * most, even + most) + rounds * sp.start * 16 / bits;
    };
    const uint64_t join = sp.join * 16 / bits;
    uint64_t best = whole, least = cost(first, longest);
    uint64_t hi = whole / sp.step;  // fits
    for (uint64_t r = first; r < first + sp.rounds; ++r) {
        if (r > sp.rounds && best <= even) break;
        if (cost(r, sp.fewest) + join >= least) break;  // nor do more rounds end before
        const uint64_t items = std::min(most_items, r * sp.wide / H);
        if (items < n) continue;
        uint64_t lo = sp.fewest / sp.step;
        while (lo < hi) {
            const uint64_t mid = (lo + hi) / 2;
            if (fits((uint32_t)(mid * sp.step), items - n))
                hi = mid;
            else
                lo = mid + 1;
        }
        const uint64_t c = cost(r, hi * sp.step) + join;
        if (c < least) {
            least = c;
            best = hi * sp.step;
        }
        if (hi == sp.fewest / sp.step) break;
    }
    return best;
}

// Tokens that the columns of a tile see at most.
uint32_t tile_end(const KvSeq& q, uint32_t G, uint32_t columns, uint32_t tile) {
    const uint64_t last = std::min<uint64_t>((uint64_t)(tile + 1) * columns,
                                             (uint64_t)G * q.fresh) - 1;
    return q.context - q.fresh + (uint32_t)(last / G) + 1;
}

}  // namespace

aqua_status kv_limits(const Shape& s, const aqua_kv_batch_desc* d, KvLimits* out) {
    if (!d || !out) return AQUA_ERR_INVALID;
    if (s.T < 4 || s.T > 1024 || (s.T & (s.T - 1))) return AQUA_ERR_INVALID;
    if (s.D != 64 && s.D != 128 && s.D != 256) return AQUA_ERR_INVALID;
    if (!d->num_q_heads || d->num_q_heads > 65536 || d->num_q_heads % s.H)
        return AQUA_ERR_INVALID;
    if (!d->max_seqs || !d->max_tokens || !d->max_blocks) return AQUA_ERR_INVALID;
    if (d->max_seqs > (1u << 20) || d->max_tokens > (1u << 22) || d->max_blocks > (1u << 28))
        return AQUA_ERR_INVALID;
    KvLimits m;
    m.shape = s;
    m.q_heads = d->num_q_heads;
    m.seqs = d->max_seqs;
    m.tokens = d->max_tokens;
    m.blocks = d->max_blocks;
    m.group = m.q_heads / s.H;
    const uint64_t G = m.group, H = s.H;
    // Items of whole contexts: a sequence's columns round up to a tile.
    const uint64_t busy = std::min(m.seqs, m.tokens);
    const uint64_t wide = std::min<uint64_t>(busy, G * m.tokens / (kRowsMostColumns + 1));
    const uint32_t tc = tile_columns(s.D);
    const uint64_t rows = busy + std::min<uint64_t>(G * m.tokens / kRowColumns,
                                                    busy * kRowsMostColumns / kRowColumns);
    // (A single token's heads may be more columns than kRowsMostColumns; they go to
    // the tiles kernel, whose items are fewer.)
    const uint64_t tiles = wide ? wide + G * m.tokens / tc : 0;
    // The parts of items that are split are at most wide * rounds workgroups, and no more
    // than the tables' tokens make.  A context of e > fewest tokens has at most e / fewest + 1
    // parts for each of its items; rows items are one for each 16 of its columns, which
    // are at most kRowsMostColumns.
    const uint64_t held = (uint64_t)m.blocks * s.T;
    const uint64_t row_items =
        ceil_div(std::min<uint64_t>(G * m.tokens, kRowsMostColumns), kRowColumns);
    const uint64_t row_parts =
        held > kRows.fewest
            ? std::min(row_items * (held / kRows.fewest + std::min(busy, held / (kRows.fewest + 1))),
                       (uint64_t)kRows.wide * kRows.rounds / H)
            : 0;
    const uint64_t tile_parts =
        held > kTiles.fewest ? std::min(tiles * ceil_div(held, kTiles.fewest),
                                        (uint64_t)kTiles.wide * kTiles.rounds / H)
                             : 0;
    const uint64_t tile_slots = tile_parts * (tc / kRowColumns);
    // A tile of 16 with p >= 2 parts makes at most 1 + 16 turns / groups joins, with
    // turns <= p / kJoinAhead + 1 (and groups / turns rounded down: twice that).
    const uint64_t slots = row_parts + tile_slots, groups = join_groups(s.D);
    const uint64_t joins = slots ? slots * (kRowColumns + groups) / groups + 16 : 0;
    // A launch has fewer than 2^32 threads, 256 or 512 a workgroup; columns are counted in
    // 32 bits.
    const uint64_t row_room = ((1ull << 24) - 1) / H, tile_room = ((1ull << 23) - 1) / H;
    if (rows > row_room || tiles > tile_room ||
        joins * H >= (1ull << 31) || G * m.tokens >= (1ull << 31))
        return AQUA_ERR_INVALID;
    m.rows = (uint32_t)std::min(rows + row_parts, row_room);
    m.tiles = (uint32_t)std::min(tiles + tile_parts, tile_room);
    m.row_parts = (uint32_t)row_parts;
    m.tile_parts = (uint32_t)tile_parts;
    m.joins = (uint32_t)joins;
    m.slots = (uint32_t)slots;
    *out = m;
    return AQUA_OK;
}

aqua_status kv_plan(const KvLimits& lim, uint32_t num_seqs, const int32_t* ids,
                    const uint64_t* offs, const uint32_t* context, const uint32_t* fresh,
                    KvPlan* plan) {
    if (!plan) return AQUA_ERR_INVALID;
    const uint32_t T = lim.shape.T, N = lim.shape.N, H = lim.shape.H, G = lim.group;
    if (num_seqs && (!offs || !context || !fresh)) return AQUA_ERR_INVALID;
    if (num_seqs && offs[0] != 0) return AQUA_ERR_INVALID;
    for (uint32_t s = 0; s < num_seqs; ++s)
        if (offs[s + 1] < offs[s] || fresh[s] > context[s] || context[s] > kMostContext)
            return AQUA_ERR_INVALID;
    const uint64_t entries = num_seqs ? offs[num_seqs] : 0;
    if (entries && !ids) return AQUA_ERR_INVALID;
    if (num_seqs > lim.seqs || entries > lim.blocks) return AQUA_ERR_CAPACITY;
    uint64_t tokens = 0;
    for (uint32_t s = 0; s < num_seqs; ++s) {
        if (ceil_div(context[s], T) > offs[s + 1] - offs[s]) return AQUA_ERR_CAPACITY;
        tokens += fresh[s];
    }
    if (tokens > lim.tokens) return AQUA_ERR_CAPACITY;
    uint32_t bad = 0;
    for (uint64_t i = 0; i < entries; ++i) bad |= (uint32_t)ids[i] >= N;
    if (bad) return AQUA_ERR_RANGE;

    plan->seqs.clear();
    plan->rows.clear();
    plan->tiles.clear();
    plan->joins.clear();
    plan->tokens.clear();
    plan->entries = (uint32_t)entries;
    plan->longest = 0;

    // Tokens, and whether an append may write them: a block that is written
    // stands in one place of one table only.
    if (plan->mark.size() != N || plan->epoch == 0xffffffffu) {
        plan->mark.assign(N, 0);
        plan->epoch = 0;
    }
    const uint64_t epoch = (uint64_t)++plan->epoch << 32;
    plan->append_ok = true;
    uint32_t row = 0;
    for (uint32_t s = 0; s < num_seqs; ++s) {
        plan->seqs.push_back({(uint32_t)offs[s], context[s], fresh[s], row});
        row += fresh[s];
        if (!fresh[s]) continue;
        plan->longest = std::max(plan->longest, context[s]);
        for (uint32_t p = context[s] - fresh[s]; p < context[s]; ++p)
            plan->tokens.push_back({(uint32_t)ids[offs[s] + p / T], p});
        for (uint32_t b = (context[s] - fresh[s]) / T; b <= (context[s] - 1) / T; ++b) {
            uint64_t& m = plan->mark[ids[offs[s] + b]];
            if ((m & ~0xffffffffull) == epoch) plan->append_ok = false;
            m = epoch | (offs[s] + b);
        }
    }
    for (uint32_t s = 0; s < num_seqs && plan->append_ok; ++s)
        for (uint64_t i = offs[s]; i < offs[s] + ceil_div(context[s], T); ++i) {
            const uint64_t m = plan->mark[ids[i]];
            if ((m & ~0xffffffffull) == epoch && m != (epoch | i)) plan->append_ok = false;
        }

    // Work items.  A tile of columns sees [0, end) of the context.
    const uint32_t tc = tile_columns(lim.shape.D), per = tc / kRowColumns;
    const auto wide = [&](const KvSeq& q) {
        return (uint64_t)G * q.fresh > kRowsMostColumns && lim.tiles;
    };
    const uint32_t bits = (uint32_t)(lim.shape.C * 8 / (2ull * H * T * lim.shape.D));
    plan->slots = 0;
    for (int w = 0; w < 2; ++w) {
        const KvSplit& sp = w ? kTiles : kRows;
        const uint32_t columns = w ? tc : kRowColumns, sub = w ? per : 1;
        std::vector<KvPart>& items = w ? plan->tiles : plan->rows;
        plan->ends.clear();
        for (const KvSeq& q : plan->seqs)
            if (q.fresh && wide(q) == (w == 1))
                for (uint64_t t = 0; t * columns < (uint64_t)G * q.fresh; ++t)
                    plan->ends.push_back(tile_end(q, G, columns, (uint32_t)t));
        if (plan->ends.empty()) continue;
        const uint64_t most =
            w ? part_tokens(plan->ends, H, sp, 16, lim.tiles, lim.tile_parts)
              : part_tokens(plan->ends, H, sp, bits, lim.rows, lim.row_parts);
        for (const KvSeq& q : plan->seqs) {
            if (!q.fresh || wide(q) != (w == 1)) continue;
            const uint64_t all = (uint64_t)G * q.fresh;
            for (uint32_t t = 0; (uint64_t)t * columns < all; ++t) {
                const uint32_t end = tile_end(q, G, columns, t);
                const uint32_t n = (uint32_t)ceil_div(end, most);
                if (n == 1) {
                    items.push_back({q, t, 0, end, kNoSlot});
                    continue;
                }
                // Parts of one size, in whole steps: n of them or fewer.
                const uint32_t size = (uint32_t)(ceil_div(ceil_div(end, n), sp.step) * sp.step);
                const uint32_t parts = (uint32_t)ceil_div(end, size);
                for (uint32_t k = 0; k < parts; ++k)
                    items.push_back({q, t, k * size, std::min(end, (k + 1) * size),
                                     plan->slots + k * sub});
                const uint32_t groups = join_groups(lim.shape.D);
                const uint32_t turns =
                    std::min<uint32_t>(groups, (uint32_t)ceil_div(parts, kJoinAhead));
                const uint32_t take = std::min(groups / turns, kRowColumns);
                const uint32_t last =
                    (uint32_t)std::min<uint64_t>((uint64_t)(t + 1) * columns, all);
                for (uint32_t c = t * columns; c < last;) {
                    const uint32_t room = kRowColumns - c % kRowColumns;
                    const uint32_t n16 = std::min({take, room, last - c});
                    plan->joins.push_back({q.row, c, n16,
                                           plan->slots + (c - t * columns) / kRowColumns, parts,
                                           sub, {}});
                    c += n16;
                }
                plan->slots += parts * sub;
            }
        }
        // Longest first, so that the last to start are the shortest.
        std::stable_sort(items.begin(), items.end(), [](const KvPart& a, const KvPart& b) {
            return a.end - a.begin > b.end - b.begin;
        });
    }
    plan->head = {};
    plan->head.rows = (uint32_t)plan->rows.size();
    plan->head.tiles = (uint32_t)plan->tiles.size();
    plan->head.joins = (uint32_t)plan->joins.size();
    plan->new_tokens = (uint32_t)plan->tokens.size();
    plan->head.append_tokens = plan->append_ok ? plan->new_tokens : 0;
    return AQUA_OK;
}

}  // namespace aqua
