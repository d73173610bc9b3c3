"""CPU tests of the operators' host planning: what a batch refuses, and that its
work items cover every (column, token) once and stay within the batch's limits."""
import ctypes

import numpy as np
import pytest

from tests import core_lib

OK, INVALID, RANGE, CAPACITY = 0, -1, -2, -4
F16, BF16, FP8, INT4 = 1, 2, 3, 4


class BatchDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in ("num_q_heads", "max_seqs", "max_tokens",
                                               "max_blocks")]


def _lib():
    L = core_lib.lib()
    P, u32 = ctypes.c_void_p, ctypes.c_uint32
    L.aqua_core_kv_limits.argtypes = [P, P, P]
    L.aqua_core_kv_plan.argtypes = [P, P, u32, P, P, P, P, u32, P, P, P, P, P]
    L.aqua_core_kv_limits.restype = L.aqua_core_kv_plan.restype = ctypes.c_int32
    return L


def limits(pool, batch):
    out = np.zeros(5, dtype=np.uint32)
    st = _lib().aqua_core_kv_limits(ctypes.byref(core_lib.Desc(*pool)),
                                    ctypes.byref(BatchDesc(*batch)), out.ctypes.data)
    return st, dict(zip(("group", "rows", "tiles", "joins", "slots"), out.tolist()))


def plan(pool, batch, tables, ctx, new, offs=None, most=1 << 16):
    ids = np.ascontiguousarray(np.concatenate([np.asarray(t, dtype=np.int32) for t in tables])
                               if tables else np.zeros(0, np.int32))
    if offs is None:
        offs = np.concatenate([[0], np.cumsum([len(t) for t in tables])])
    offs = np.ascontiguousarray(offs, dtype=np.uint64)
    ctx, new = (np.ascontiguousarray(x, dtype=np.uint32) for x in (ctx, new))
    counts = np.zeros(7, dtype=np.uint32)
    rows, tiles, joins = (np.zeros((most, n), dtype=np.uint32) for n in (8, 8, 6))
    tokens = np.zeros((most, 2), dtype=np.uint32)
    st = _lib().aqua_core_kv_plan(
        ctypes.byref(core_lib.Desc(*pool)), ctypes.byref(BatchDesc(*batch)), len(tables),
        ids.ctypes.data, offs.ctypes.data, ctx.ctypes.data, new.ctypes.data, most,
        *(a.ctypes.data for a in (counts, rows, tiles, joins, tokens)))
    if st:
        return st, None
    c = dict(zip(("rows", "tiles", "joins", "tokens", "append_ok", "longest", "slots"),
                 counts.tolist()))
    return st, {"counts": c, "rows": rows[:c["rows"]], "tiles": tiles[:c["tiles"]],
                "joins": joins[:c["joins"]], "tokens": tokens[:c["tokens"]]}


def _tables(ctx, T, N, rng, spare=0):
    free = rng.permutation(N)
    out, at = [], 0
    for c in ctx:
        n = -(-c // T) + spare
        out.append(free[at:at + n])
        at += n
    return out


def _check_cover(pool, batch, starts, ctx, new, p, lim):
    """Every column's tokens once, in parts whose slots are apart and joined."""
    L, N, H, T, D, dtype = pool
    G = batch[0] // H
    c = p["counts"]
    assert c["rows"] <= lim["rows"] and c["tiles"] <= lim["tiles"]
    assert c["joins"] <= lim["joins"] and c["slots"] <= lim["slots"]
    wide = 128 if D > 128 else 256
    firsts = np.concatenate([[0], np.cumsum(new)]).tolist()
    by_row = {firsts[s]: s for s in range(len(ctx)) if new[s]}
    used = {}                       # slot group -> (seq, 16-column tile)
    parts = {}                      # (seq, columns, tile) -> [(begin, end, slot)]
    for items, columns in ((p["rows"], 16), (p["tiles"], wide)):
        for at, context, fresh, row, tile, begin, end, slot in items.tolist():
            s = by_row[row]
            assert (at, context, fresh) == (starts[s], ctx[s], new[s])
            assert begin < end and begin % (256 if columns == 16 else 64) == 0
            parts.setdefault((s, columns, tile), []).append((begin, end, slot))
            if slot != 0xFFFFFFFF:
                for k in range(columns // 16):
                    assert slot + k < lim["slots"]
                    assert slot + k not in used, "two parts in one slot"
                    used[slot + k] = (s, tile * (columns // 16) + k, begin)
    joins = {}
    for row, column, count, slot, n, stride in p["joins"].tolist():
        assert count and column // 16 == (column + count - 1) // 16
        for k in range(column, column + count):
            assert (by_row[row], k) not in joins, "a column is joined twice"
            joins[by_row[row], k] = (slot, n, stride)
    seen = set()
    for (s, columns, tile), items in parts.items():
        R = G * new[s]
        first, last = tile * columns, min((tile + 1) * columns, R) - 1
        assert first <= last
        seen |= {(s, k) for k in range(first, last + 1)}
        items.sort()
        end = ctx[s] - new[s] + last // G + 1
        assert items[0][0] == 0 and items[-1][1] == end
        assert all(a[1] == b[0] for a, b in zip(items, items[1:]))
        if len(items) == 1:
            assert items[0][2] == 0xFFFFFFFF
            continue
        for k in range(columns // 16):
            tile16 = tile * (columns // 16) + k
            for column in range(tile16 * 16, min((tile16 + 1) * 16, R)):
                slot, n, stride = joins.pop((s, column))
                assert n == len(items)
                assert sorted(slot + i * stride for i in range(n)) == \
                    sorted(it[2] + k for it in items)
    assert not joins
    assert seen == {(s, k) for s in range(len(ctx)) for k in range(G * new[s])}


@pytest.mark.parametrize("heads", [(8, 32), (1, 71), (5, 5), (40, 40), (2, 64)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_items_cover_every_column_once(heads, D):
    H, Hq = heads
    rng = np.random.default_rng(H * 1000 + D)
    for trial in range(25):
        T = int(rng.choice([4, 8, 16, 64]))
        n = int(rng.integers(1, 40))
        ctx = [int(x) for x in np.exp(rng.uniform(0, np.log(40000 if trial % 3 else 300), n))]
        kind = trial % 4
        new = [1 if kind == 0 else int(rng.integers(0, min(c, 7) + 1)) if kind == 1
               else c if kind == 2 and c < 3000 else int(rng.integers(0, min(c, 700) + 1))
               for c in ctx]
        tables = _tables(ctx, T, sum(-(-c // T) for c in ctx) + n, rng, spare=trial % 2)
        pool = (2, sum(len(t) for t in tables) + n, H, T, D, BF16)
        batch = (Hq, n, max(1, sum(new)), sum(len(t) for t in tables))
        st, lim = limits(pool, batch)
        assert st == OK
        st, p = plan(pool, batch, tables, ctx, new)
        assert st == OK and p["counts"]["append_ok"] == 1
        assert p["counts"]["longest"] == max([c for c, m in zip(ctx, new) if m], default=0)
        _check_cover(pool, batch, np.cumsum([0] + [len(t) for t in tables])[:-1].tolist(), ctx, new,
                     p, lim)
        want = [(int(t[q // T]), q) for t, c, m in zip(tables, ctx, new) for q in range(c - m, c)]
        assert [tuple(x) for x in p["tokens"].tolist()] == want


def test_long_contexts_are_split_and_short_ones_are_not():
    pool, batch = (1, 9000, 8, 16, 128, BF16), (32, 64, 64, 9000)
    rng = np.random.default_rng(2)
    st, p = plan(pool, batch, _tables([131072], 16, 9000, rng), [131072], [1])
    assert st == OK and 64 <= p["counts"]["rows"] <= 260
    st, p = plan(pool, batch, _tables([200] * 64, 16, 9000, rng), [200] * 64, [1] * 64)
    assert st == OK and p["counts"]["rows"] == 64 and p["counts"]["joins"] == 0
    st, p = plan(pool, batch, [], [], [])
    assert st == OK and p["counts"]["rows"] == p["counts"]["tokens"] == 0


def test_blocks_that_two_tables_hold():
    pool, batch = (1, 100, 2, 16, 128, BF16), (4, 4, 200, 100)
    a, b = list(range(0, 8)), list(range(10, 18))
    ok = lambda t, c, n: plan(pool, batch, t, c, n)[1]["counts"]["append_ok"]
    assert ok([a, b], [100, 100], [1, 1]) == 1
    assert ok([a, a[:6] + b[6:]], [100, 100], [1, 1]) == 1      # shared full blocks
    assert ok([a, a], [100, 100], [1, 1]) == 0                  # both write block 6
    assert ok([a, a], [100, 97], [1, 0]) == 0                   # one writes, one reads it
    assert ok([a, a], [97, 96], [1, 0]) == 1                    # 96 tokens end before it
    assert ok([a, a], [100, 100], [0, 0]) == 1                  # both read
    assert ok([a, a], [100, 100], [20, 0]) == 0                 # writes reach block 5
    assert ok([a[:6] + [0], b], [100, 100], [1, 1]) == 0        # a block twice in a table
    assert ok([a + [6], b], [100, 100], [1, 1]) == 1            # entries past the context
    assert ok([a, b[:3] + [5, 6]], [100, 48], [1, 1]) == 1      # ... of another table


def test_what_a_batch_refuses():
    ok = (1, 64, 2, 16, 128, BF16)
    assert limits(ok, (4, 1, 1, 1))[0] == OK
    for pool in [(1, 64, 2, 2, 128, BF16), (1, 64, 2, 2048, 128, BF16), (1, 64, 2, 12, 128, BF16),
                 (1, 64, 2, 16, 96, BF16), (1, 64, 2, 16, 32, BF16), (1, 64, 2, 16, 512, BF16)]:
        assert limits(pool, (4, 1, 1, 1))[0] == INVALID, pool
    for batch in [(3, 1, 1, 1), (0, 1, 1, 1), (4, 0, 1, 1), (4, 1, 0, 1), (4, 1, 1, 0),
                  (65538, 1, 1, 1), (4, (1 << 20) + 1, 1, 1), (4, 1, (1 << 22) + 1, 1),
                  (4, 1, 1, (1 << 28) + 1), (65536, 1 << 20, 1 << 22, 1)]:
        assert limits(ok, batch)[0] == INVALID, batch
    # As large as the header promises.
    for H, Hq, tokens in [(1, 64, 1 << 17), (64, 64, 1 << 17), (1, 2, 1 << 22), (8, 8, 1 << 20)]:
        assert limits((1, 64, H, 16, 128, BF16), (Hq, min(tokens, 1 << 20), tokens, 1))[0] == OK


def test_what_a_step_refuses():
    pool, batch = (1, 64, 2, 16, 128, BF16), (4, 2, 40, 10)
    t = [[1, 2, 3, 4], [5, 6]]
    cases = [
        (CAPACITY, [[1], [2], [3]], [1, 1, 1], [1, 1, 1], None),    # sequences
        (CAPACITY, t, [64, 32], [20, 21], None),                    # tokens
        (CAPACITY, [list(range(11))], [1], [1], None),              # table entries
        (CAPACITY, t, [65, 32], [1, 1], None),                      # context past its table
        (CAPACITY, [[], [1]], [1, 1], [1, 1], None),                # an empty table
        (INVALID, t, [64, 32], [1, 33], None),                      # more new than context
        (INVALID, t, [(1 << 30) + 1, 32], [1, 1], None),
        (INVALID, t, [64, 32], [1, 1], [0, 4, 3]),                  # offsets
        (INVALID, t, [64, 32], [1, 1], [1, 4, 6]),
        (RANGE, [[1, 2, 3, 64], [5, 6]], [64, 32], [1, 1], None),
        (RANGE, [[1, 2, 3, -1], [5, 6]], [64, 32], [1, 1], None),
        (RANGE, [[1, 2, 3, 64], [5, 6]], [10, 32], [1, 1], None),   # unused, and still wrong
    ]
    for want, tables, ctx, new, offs in cases:
        assert plan(pool, batch, tables, ctx, new, offs)[0] == want, (tables, ctx, new)
    assert plan(pool, batch, t, [64, 32], [20, 20])[0] == OK
    assert plan(pool, batch, [[], [1]], [0, 1], [0, 1])[0] == OK


def test_four_bit_chunks():
    """A 4-bit chunk is 5 bits a value; its head size is made of groups of 32."""
    v = lambda desc, nbytes: core_lib.lib().aqua_core_validate(
        ctypes.byref(core_lib.Desc(*desc)), 1, np.zeros(1, np.int32).ctypes.data,
        np.array([0, 1], np.uint64).ctypes.data, 4096, nbytes, None, 0)
    assert v((1, 4, 8, 16, 128, INT4), 20480) == OK            # 2*8*16*128 * 5/8
    assert v((1, 4, 8, 16, 128, INT4), 20479) == CAPACITY
    assert v((2, 4, 2, 4, 64, INT4), 2 * 640) == OK
    for desc in [(1, 4, 8, 16, 80, INT4), (1, 4, 8, 16, 16, INT4), (1, 4, 1, 1, 32, INT4)]:
        assert v(desc, 1 << 20) == INVALID, desc


def _mixed(H, Hq, short, long, new, D=128):
    """`short` contexts of 100 tokens and one long one, with `new` tokens each."""
    T, rng = 16, np.random.default_rng(short)
    ctx = [100] * short + [long]
    ctx = [int(x) for x in rng.permutation(ctx)]
    fresh = [min(c, new) for c in ctx]
    blocks = sum(-(-c // T) for c in ctx)
    pool = (1, blocks, H, T, D, BF16)
    batch = (Hq, len(ctx), sum(fresh), blocks)
    tables = _tables(ctx, T, blocks, rng)
    st, lim = limits(pool, batch)
    assert st == OK
    st, p = plan(pool, batch, tables, ctx, fresh)
    assert st == OK
    _check_cover(pool, batch, np.cumsum([0] + [len(t) for t in tables])[:-1].tolist(), ctx,
                 fresh, p, lim)
    return p


@pytest.mark.parametrize("H,short", [(8, 63), (8, 500), (8, 511), (8, 600), (8, 4000), (32, 128),
                                     (32, 600), (1, 5000)])
def test_a_long_context_among_many_short_ones_is_split(H, short):
    """Whatever whole items there are beside it: no part is longer than what a
    workgroup has to do when the work is spread evenly."""
    p = _mixed(H, 32, short, 131072, 1)
    longest = int((p["rows"][:, 6].astype(int) - p["rows"][:, 5]).max())
    even = -(-(short * 100 + 131072) * H // 512)
    assert longest <= max(512, -(-even // 256) * 256)


@pytest.mark.parametrize("short", [20, 101, 128, 400])
@pytest.mark.parametrize("D,columns", [(128, 256), (256, 128)])
def test_a_chunk_behind_a_long_context_beside_many_prompts_is_split(D, columns, short):
    p = _mixed(8, 32, short, 131072, 100, D)
    n = p["tiles"][:, 6].astype(int) - p["tiles"][:, 5]
    even = -(-int(n.sum()) * 8 // 256)
    assert int(n.max()) <= max(256, -(-even // 64) * 64)


def _workspace(pool, lim):
    """Bytes of split sums: 16 columns of D values, maxima and totals a slot and KV head."""
    return lim["slots"] * pool[2] * 16 * (pool[4] + 2) * 4


def test_the_workspace_is_what_a_split_of_the_batchs_blocks_can_need():
    pool = (1, 1 << 20, 8, 16, 128, BF16)
    # Contexts that are never split: 32 blocks hold 512 tokens, 16 hold 256.
    for batch in [(32, 1, 1, 1), (32, 1, 1, 32), (32, 64, 16, 32), (32, 1, 64, 4), (32, 1, 512, 16)]:
        st, lim = limits(pool, batch)
        assert st == OK and lim["slots"] == lim["joins"] == 0, batch
    # One more block, and there are two parts; more grow with it.
    st, lim = limits(pool, (32, 1, 1, 33))
    assert st == OK and 2 <= lim["slots"] <= 4
    st, more = limits(pool, (32, 1, 1, 330))
    assert lim["slots"] < more["slots"] <= 40
    # Decode batches take no room for prompts' tiles; at most what the header says.
    for D, rows, tiles in ((64, 17.4e6, 69.3e6), (128, 34.1e6, 136.4e6), (256, 67.7e6, 135.3e6)):
        big = (1, 1 << 20, 8, 16, D, BF16)
        assert 0.99 * rows < _workspace(big, limits(big, (32, 16, 16, 1 << 20))[1]) <= rows
        assert 0.99 * (rows + tiles) < _workspace(big, limits(big, (32, 64, 64, 1 << 20))[1]) <= \
            rows + tiles


@pytest.mark.parametrize("heads", [(8, 32), (1, 71), (5, 5), (2, 64)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_room_for_the_batchs_blocks_takes_no_part_from_a_step(heads, D):
    """A step is planned alike in a batch that just holds its tables and in a larger one."""
    H, Hq = heads
    rng = np.random.default_rng(H * 7 + D)
    for trial in range(40):
        T = int(rng.choice([4, 16, 256]))
        n = int(rng.integers(1, 12))
        ctx = [int(x) for x in np.exp(rng.uniform(0, np.log(120000 if trial % 2 else 3000), n))]
        if trial % 5 == 0:
            ctx = [int(x) for x in rng.choice([256, 257, 512, 513, 768, 1024, 1025], n)]
        new = [1 if trial % 3 == 0 else int(rng.integers(0, min(c, 5) + 1)) if trial % 3 == 1
               else int(rng.integers(0, min(c, 300) + 1)) for c in ctx]
        if not sum(new):
            continue
        tables = _tables(ctx, T, sum(-(-c // T) for c in ctx) + n, rng)
        blocks = sum(len(t) for t in tables)
        pool = (2, blocks + n, H, T, D, BF16)
        exact, wide = (Hq, n, sum(new), blocks), (Hq, n, sum(new), blocks + (1 << 20))
        st, lim = limits(pool, exact)
        (sa, a), (sb, b) = plan(pool, exact, tables, ctx, new), plan(pool, wide, tables, ctx, new)
        assert st == sa == sb == OK
        for name in ("rows", "tiles", "joins", "tokens"):
            assert np.array_equal(a[name], b[name]), (trial, name)
            assert len(a[name]) <= lim.get(name, 1 << 32)
        assert a["counts"]["slots"] <= lim["slots"]


def test_the_longest_context():
    """2^30 tokens in blocks of 1024: parts and their ends stay within 32 bits."""
    most = 1 << 30
    for H, Hq in ((1, 1), (8, 64)):
        table = np.arange(most // 1024, dtype=np.int32)
        pool, batch = (1, most // 1024, H, 1024, 64, INT4), (Hq, 1, 20, most // 1024)
        st, lim = limits(pool, batch)
        assert st == OK
        for new in (1, 20):
            st, p = plan(pool, batch, [table], [most], [new])
            assert st == OK and p["counts"]["longest"] == most
            _check_cover(pool, batch, [0], [most], [new], p, lim)
            assert p["tokens"].tolist()[-1] == [most // 1024 - 1, most - 1]
            n = np.concatenate([x[:, 6].astype(int) - x[:, 5] for x in (p["rows"], p["tiles"])])
            assert int(n.max()) <= most * H // 256 + 512
