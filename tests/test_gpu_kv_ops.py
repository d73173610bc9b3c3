"""GPU tests of the operators on the pool (aqua_kv_append, aqua_kv_attend) against
plain 64-bit forms, with tolerances from the roundings that the header names
(tests/kv_ref.py)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2407_21255_amd import aqua
from tests import kv_ref as ref
from tests.gpu_util import say
from tests.kv_ref import BF16, F16, F64, FP8, INT4

pytestmark = pytest.mark.gpu

KINDS = [(F16, torch.float16), (BF16, torch.bfloat16), (FP8, torch.float16),
         (FP8, torch.bfloat16), (INT4, torch.float16), (INT4, torch.bfloat16)]
KIND_IDS = [f"{ref.NAMES[p]}-{str(t)[6:]}" for p, t in KINDS]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    aqua.load()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class Step:
    """A pool with a batch set to a step, and its tensors."""

    def __init__(self, shape, Hq, ctx, new, q_dtype, seed=1, spare=0, limits=None, padding=0,
                 poison=True, blocks_past=5, spread=1.0):
        L, N, H, T, D, dtype = shape
        self.shape, self.Hq, self.ctx, self.new, self.dtype = shape, Hq, ctx, new, q_dtype
        self.tables = ref.tables_for(ctx, T, N, seed, spare)
        self.pool = ref.random_pool(shape, seed, spread=spread)
        if poison:
            ref.poison_unused(self.pool, shape, self.tables, ctx)
        self.tokens = int(sum(new))
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        rows = self.tokens + padding
        self.qkv = torch.randn(max(rows, 1), Hq + 2 * H, D, device="cuda",
                               generator=gen).to(q_dtype)[:rows]
        self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + H], self.qkv[:, Hq + H:]
        self.kv = aqua.KVPool(shape, self.pool)
        blocks = sum(len(t) for t in self.tables)
        m = limits or (max(1, len(ctx)), max(1, rows), max(1, blocks))
        self.batch = aqua.KVBatch(self.kv, Hq, *m)
        self.batch.set(self.tables, ctx, new)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.kv.close()

    def reference(self, layer, q, **kw):
        return ref.attend(ref.values(self.pool, self.shape), layer, self.tables, self.ctx,
                          self.new, q, **kw)

    def check_attend(self, layer, q, what, got=None, k_scale=1.0, v_scale=1.0, scale=None):
        n = self.tokens
        out, lse = got if got is not None else self.batch.attend(
            layer, q, lse=True, k_scale=k_scale, v_scale=v_scale, scale=scale)
        torch.cuda.synchronize()
        o, l, mass, reach = self.reference(layer, q[:n], k_scale=k_scale, v_scale=v_scale,
                                           scale=scale)
        vals = ref.values(self.pool, self.shape)
        vmax = float(vals[vals.isfinite()].abs().amax()) * v_scale
        bo, bl = ref.attend_bounds(o, l, mass, reach, self.shape[4], max(self.ctx), self.dtype,
                                   self.shape[5], vmax)
        ref.assert_within(lse[:n], l, bl, what + ": lse")
        ref.assert_within(out[:n], o, bo, what + ": out")
        return out, lse


# -- attention -----------------------------------------------------------------

# Contexts and new tokens that meet the edges: one token, a full and a barely begun
# block, the ends of a wave's 32 tokens and a workgroup's 128, parts that split;
# single tokens, a few, whole prompts.
CTX = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 300, 511, 1000]
NEW1 = [1] * len(CTX)
FEW = [1, 2, 3, 16, 5, 1, 8, 4, 2, 64, 3, 7, 1, 0, 4, 2, 5]
MANY = [1, 1, 15, 16, 17, 31, 20, 33, 63, 40, 65, 100, 129, 255, 200, 0, 333]


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("heads", [(2, 8), (3, 3), (1, 20)], ids=["g4", "g1", "g20"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attend_one_token_each(D, heads, kind):
    H, Hq = heads
    shape = (2, 300, H, 16, D, kind[0])
    ks, vs = (0.5, 1.5) if kind[0] == FP8 else (1.0, 1.0)
    with Step(shape, Hq, CTX, NEW1, kind[1], seed=D + H) as s:
        s.check_attend(1, s.q, "decode", k_scale=ks, v_scale=vs)


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("D,T", [(64, 4), (128, 8), (128, 64), (256, 32)])
@pytest.mark.parametrize("new", [FEW, MANY], ids=["few", "many"])
def test_attend_several_tokens(new, D, T, kind):
    shape = (1, 6000 // T, 2, T, D, kind[0])
    with Step(shape, 10, CTX, new, kind[1], seed=T) as s:
        s.check_attend(0, s.q, "chunks")


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
def test_attend_splits_long_contexts(kind):
    """Contexts of many parts, for one token and for a chunk, beside short ones."""
    ctx, new = [20001, 7, 9000, 4097], [1, 1, 300, 2]
    shape = (1, 2200, 2, 16, 128, kind[0])
    with Step(shape, 8, ctx, new, kind[1], seed=3) as s:
        s.check_attend(0, s.q, "splits")


@pytest.mark.parametrize("kind", [KINDS[1], KINDS[4]], ids=[KIND_IDS[1], KIND_IDS[4]])
def test_attend_scores_of_any_size_and_sign(kind):
    """Large scores (weights of one token only), negative and zero scales."""
    ctx, new = [700, 300], [3, 100]
    shape = (1, 100, 2, 16, 128, kind[0])
    for scale in (3.0, -0.4, 0.0):
        with Step(shape, 4, ctx, new, kind[1], seed=7) as s:
            s.check_attend(0, s.q, f"scale {scale}", scale=scale)


def test_queries_beyond_the_range_of_fp16_on_a_4_bit_pool():
    """bf16 queries of 2^100 and of 2^-100 keep their meaning."""
    ctx, new = [200, 90], [2, 80]
    shape = (1, 40, 2, 16, 128, INT4)
    with Step(shape, 4, ctx, new, torch.bfloat16, seed=9) as s:
        for p in (100, -100):
            q = s.q * 2.0 ** p
            s.check_attend(0, q, f"2^{p}", scale=2.0 ** -p / 11)


def test_rows_behind_the_last_sequence_are_left():
    shape = (1, 40, 2, 16, 128, BF16)
    for new in ([1, 1], [3, 90], [0, 0], [0, 1]):
        with Step(shape, 4, [200, 90], new, torch.bfloat16, padding=7) as s:
            out = torch.full_like(s.q, 7.0)
            lse = torch.full(s.q.shape[:2], 7.0, device="cuda")
            s.batch.attend(0, s.q, out=out, lse=lse)
            torch.cuda.synchronize()
            assert bool((out[s.tokens:] == 7).all()) and bool((lse[s.tokens:] == 7).all())
            if s.tokens:
                s.check_attend(0, s.q, "padded", got=(out, lse))
    with Step(shape, 4, [], [], torch.bfloat16, limits=(4, 8, 16), padding=3) as s:
        out = torch.full_like(s.q, 7.0)
        s.batch.attend(0, s.q, out=out)
        s.batch.append(0, s.k, s.v)
        torch.cuda.synchronize()
        assert bool((out == 7).all())


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[1], KINDS[3], KINDS[4]],
                         ids=[KIND_IDS[i] for i in (0, 1, 3, 4)])
@pytest.mark.parametrize("m", [3, 150], ids=["rows", "tiles"])
def test_what_a_query_does_not_see_has_no_influence(m, kind):
    """Values (and keys) of later positions that are infinite or NaN: queries before
    them are as without them, those at and behind them are not finite in those
    values."""
    pool_dtype, dt = kind
    ctx, new = [400], [m]
    shape = (1, 30, 1, 16, 128, pool_dtype)
    bad_at, d = ctx[0] - m // 2 - 1, 37
    with Step(shape, 4, ctx, new, dt, seed=5) as s:
        clean, clean_lse = s.batch.attend(0, s.q, lse=True)
        block, slot = int(s.tables[0][bad_at // 16]), bad_at % 16
        if pool_dtype == INT4:
            pairs = ref.codes_and_pairs(s.pool, shape)[1]
            pairs[0, block, 1, 0, slot, d // 32, 0] = float("nan")
            hit = torch.arange(128, device="cuda") // 32 == d // 32
        else:
            row = s.pool[:s.pool.numel()].view(ref.TORCH[pool_dtype]).view(1, 30, 2, 1, 16, 128)
            row[0, block, 1, 0, slot, d] = float("inf") if pool_dtype != FP8 else float("nan")
            hit = torch.arange(128, device="cuda") == d
        out, lse = s.batch.attend(0, s.q, lse=True)
        torch.cuda.synchronize()
        sees = torch.arange(ctx[0] - m, ctx[0], device="cuda") >= bad_at
        assert torch.equal(lse, clean_lse)
        assert torch.equal(out[~sees], clean[~sees])
        assert torch.equal(out[sees][..., ~hit], clean[sees][..., ~hit])
        assert not bool(out[sees][..., hit].isfinite().any())
        if pool_dtype in (F16, BF16):
            assert bool((out[sees][..., hit] == float("inf")).all())
            # A key that is not finite.
            row[0, block, 1, 0, slot, d] = 1.0
            row[0, block, 0, 0, slot, d] = float("nan")
            out, lse = s.batch.attend(0, s.q, lse=True)
            torch.cuda.synchronize()
            assert bool(out[~sees].isfinite().all()) and bool(out[sees].isnan().all())
            assert bool(lse[~sees].isfinite().all()) and bool(lse[sees].isnan().all())


def test_offsets_past_32_bits():
    """Blocks and a layer beyond 4 GiB, for both operators."""
    shape = (3, 36000, 4, 16, 128, BF16)               # 3 x 1.1 GiB ... blocks of 32 KiB
    ctx, new = [1000, 77], [2, 77]
    L, N, H, T, D, dtype = shape
    pool = torch.zeros(L * N * ref.chunk_bytes(H, T, D, dtype) + (5 << 30), dtype=torch.uint8,
                       device="cuda")
    big = (L, pool.numel() // L // ref.chunk_bytes(H, T, D, dtype), H, T, D, dtype)
    N = big[1]
    tables = [np.arange(N - 63, N, dtype=np.int32), np.arange(N - 80, N - 75, dtype=np.int32)]
    tail = pool[2 * N * 32768 + (N - 100) * 32768:3 * N * 32768]
    assert 2 * N * 32768 > 1 << 32
    tail.copy_(torch.randn(tail.numel() // 2, device="cuda").bfloat16().view(torch.uint8))
    small = [t - (N - 100) for t in tables]
    with aqua.KVPool(big, pool) as kv:
        b = aqua.KVBatch(kv, 8, 2, 79, 68)
        b.set(tables, ctx, new)
        q, k = torch.randn(79, 8, 128, device="cuda").bfloat16(), \
            torch.randn(79, 4, 128, device="cuda").bfloat16()
        b.append(2, k, k)
        out, lse = b.attend(2, q, lse=True)
        torch.cuda.synchronize()
        vals = tail.view(torch.bfloat16).to(F64).view(1, 100, 2, H, T, D)
        blk, slot = ref.slots(small, ctx, new, T)
        assert torch.equal(vals[0, blk, 0, :, slot], k.to(F64))
        assert torch.equal(vals[0, blk, 1, :, slot], k.to(F64))
        o, l, mass, reach = ref.attend(vals, 0, small, ctx, new, q)
        bo, bl = ref.attend_bounds(o, l, mass, reach, 128, 1000, torch.bfloat16, BF16, 5.0)
        ref.assert_within(lse, l, bl, "lse")
        ref.assert_within(out, o, bo, "out")
        assert int(pool[:2 * N * 32768 + (N - 100) * 32768].count_nonzero()) == 0


def test_so_many_heads_that_nothing_is_split():
    """More KV heads than parts that a launch is split into: no room for split sums."""
    H, T, D = 8192, 64, 128
    shape = (1, 1, H, T, D, BF16)
    pool = torch.zeros(ref.chunk_bytes(*shape[2:]), dtype=torch.uint8, device="cuda")
    with aqua.KVPool(shape, pool) as kv, aqua.KVBatch(kv, H, 1, 1, 1) as batch:
        q, k, v = (torch.randn(1, H, D, device="cuda").bfloat16() for _ in range(3))
        batch.set([np.array([0])], [T], [1])
        batch.append(0, k, v)
        out, lse = batch.attend(0, q, lse=True, scale=1.0 / 16)
        torch.cuda.synchronize()
        rows = pool.view(torch.bfloat16).view(2, H, T, D)
        assert torch.equal(rows[0, :, -1], k[0]) and torch.equal(rows[1, :, -1], v[0])
        assert not bool(rows[:, :, :-1].any())
        # T - 1 keys of zeros, whose scores are 0, and values of zeros.
        s = (q[0].to(F64) * k[0].to(F64)).sum(-1) / 16
        w = s.exp() / (s.exp() + T - 1)
        want = w[:, None] * v[0].to(F64)
        # A score's fp32 sum of D products, and T weights' fp32 sum; then the weight's
        # two 16-bit terms and the result's rounding.
        score = D * 2.0 ** -24 * (q[0].to(F64) * k[0].to(F64)).abs().sum(-1) / 16
        off = score + T * 2.0 ** -24
        assert bool(((lse[0].to(F64) - (s.exp() + T - 1).log()).abs() <= off).all())
        off = (2 * off + 2.0 ** -16 + 2.0 ** -8)[:, None]
        assert bool(((out[0].to(F64) - want).abs() <= off * want.abs()).all())


def test_attend_twice_gives_the_same_bits():
    ctx, new = [20001, 9000, 33], [1, 300, 1]
    shape = (1, 1900, 2, 16, 128, INT4)
    with Step(shape, 8, ctx, new, torch.float16, seed=3) as s:
        a = s.batch.attend(0, s.q, lse=True)
        for _ in range(5):
            b = s.batch.attend(0, s.q, lse=True)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# -- append --------------------------------------------------------------------

def check_append(s, layer, rope, interleaved, before, q_out, k_scale=1.0, v_scale=1.0,
                 k=None, v=None, q=None):
    """The pool and the queries after an append, against the definition; every other
    byte of the pool as it was."""
    L, N, H, T, D, dtype = s.shape
    n = s.tokens
    k, v = (s.k if k is None else k)[:n], (s.v if v is None else v)[:n]
    q = (s.q if q is None else q)[:n]
    pos = torch.from_numpy(ref.positions(s.ctx, s.new)).cuda()
    blk, slot = ref.slots(s.tables, s.ctx, s.new, T)
    turn = (lambda x: ref.rotate(x, pos, rope, interleaved)) if rope is not None else \
        (lambda x: (x.to(F64), x.to(F64).abs()))
    u = ref.half_step(s.dtype)
    if q_out is not None:
        y, size = turn(q)
        f32 = size * 3 * 2.0 ** -24
        tiny = 2.0 ** -25 if s.dtype == torch.float16 else 0.0
        ref.assert_within(q_out[:n], y, y.abs() * u + f32 * (1 + u) + tiny, "queries")
    after = ref.values(s.pool, s.shape)
    for which, x, scale in ((0, k, k_scale), (1, v, v_scale)):
        y, size = turn(x) if which == 0 else (x.to(F64), x.to(F64).abs() * (0 if which else 1))
        got = after[layer, blk, which, :, slot]
        f32 = size * 3 * 2.0 ** -24 if which == 0 and rope is not None else torch.zeros_like(y)
        name = "values" if which else "keys"
        if dtype in (F16, BF16):
            tiny = 2.0 ** -25 if dtype == F16 else 0.0
            ref.assert_within(got, y, y.abs() * u + f32 * (1 + u) + tiny, name)
        elif dtype == FP8:
            # One more fp32 rounding, of the division; half of the least step, 2^-9.
            y, f32 = y / scale, f32 / scale + y.abs() / scale * 2.0 ** -24
            y = y.clamp(-448, 448)
            ref.assert_within(got, y, y.abs() * 2.0 ** -4 + f32 * 1.1 + 2.0 ** -10, name)
        else:
            check_int4(s, layer, blk, which, slot, y, f32, got, name)
    # Everything else is untouched.
    e = {F16: 2, BF16: 2, FP8: 1, INT4: 0}[dtype]
    if dtype == INT4:
        for a, b in zip(ref.codes_and_pairs(s.pool, s.shape),
                        ref.codes_and_pairs(before, s.shape)):
            if a.dtype == torch.float16:
                a, b = a.view(torch.int16), b.view(torch.int16)
            b = b.clone()
            b[layer, blk, :, :, slot] = a[layer, blk, :, :, slot]
            assert torch.equal(a, b)
    else:
        a, b = (p[:L * N * 2 * H * T * D * e].view(L, N, 2, H, T, D * e) for p in (s.pool, before))
        b = b.clone()
        b[layer, blk, :, :, slot] = a[layer, blk, :, :, slot]
        assert torch.equal(a, b)


def check_int4(s, layer, blk, which, slot, y, f32, got, name):
    words, pairs = ref.codes_and_pairs(s.pool, s.shape)
    p = pairs[layer, blk, which, :, slot].to(F64)
    scale, base = p[..., 0], p[..., 1]
    g = y.clamp(-16384, 16384).unflatten(-1, (-1, 32))
    lo, hi = g.amin(-1), g.amax(-1)
    e = f32.unflatten(-1, (-1, 32)).amax(-1)
    # scale: the fp32 roundings of a value, the difference and the quotient, then fp16's.
    want = (hi - lo) / 15
    ref.assert_within(scale, want, want * (2.0 ** -11 + 2.0 ** -22) + 2 * e / 15 + 2.0 ** -25,
                      name + ": scales")
    want = lo - 16 * scale                             # the product is exact
    ref.assert_within(base, want, want.abs() * (2.0 ** -11 + 2.0 ** -23) + e + 2.0 ** -25,
                      name + ": bases")
    # Each value: half a step, what the rounded base and scale cut off at the ends
    # (base's rounding below; 15 scale's above), fp32's and the value's own rounding.
    cut = want.abs() * 2.0 ** -11 + 31 * scale * 2.0 ** -11 + 2.0 ** -24
    bound = (scale / 2 + cut + 2 * e)[..., None] * (1 + 2.0 ** -10) + \
        g.abs() * 2.0 ** -11 + 2.0 ** -24
    ref.assert_within(got.unflatten(-1, (-1, 32)), g, bound, name)


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("D,R,interleaved", [(128, 128, False), (128, 128, True), (64, 32, False),
                                             (64, 16, True), (256, 256, False), (256, 48, True),
                                             (128, 0, False)])
def test_append(D, R, interleaved, kind):
    ctx, new = [1, 16, 17, 33, 300, 64, 700], [1, 16, 1, 33, 2, 0, 250]
    shape = (3, 100, 3, 16, D, kind[0])
    ks, vs = (0.37, 2.0) if kind[0] == FP8 else (1.0, 1.0)
    with Step(shape, 6, ctx, new, kind[1], seed=R + D, poison=False, padding=5) as s:
        rope = ref.rope_table(max(ctx), R) if R else None
        before = s.pool.clone()
        q = s.batch.append(1, s.k, s.v, q=s.q, rope=rope, interleaved=interleaved,
                           k_scale=ks, v_scale=vs)
        torch.cuda.synchronize()
        check_append(s, 1, rope, interleaved, before, q, ks, vs)


@pytest.mark.parametrize("tokens", [1, 3, 511, 512, 2500])
@pytest.mark.parametrize("T", [4, 32])
def test_append_lengths_and_in_place(tokens, T):
    """From one token to the counts at which a workgroup takes a token's heads
    whole; the queries in place; padding rows left."""
    shape = (1, 2600 // T + 8, 8, T, 64, BF16)
    with Step(shape, 64, [tokens + 40], [tokens], torch.bfloat16, poison=False, padding=9) as s:
        rope = ref.rope_table(tokens + 40, 64)
        before, q0 = s.pool.clone(), s.qkv.clone()
        got = s.batch.append(0, s.k, s.v, q=s.q, q_out=s.q, rope=rope)
        torch.cuda.synchronize()
        assert got is s.q
        check_append(s, 0, rope, False, before, s.q, q=q0[:, :64])
        assert torch.equal(s.qkv[tokens:], q0[tokens:])
        assert torch.equal(s.qkv[:, 64:], q0[:, 64:])


def test_append_strange_values():
    """Infinities, NaN, subnormals, zeros of both signs and groups of equal values."""
    for dtype, dt in KINDS:
        shape = (1, 4, 1, 16, 128, dtype)
        with Step(shape, 1, [20], [20], dt, poison=False) as s:
            x = torch.zeros(20, 1, 128, device="cuda")
            x[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0])
            x[1] = 3.25
            x[2] = 1e-7
            x[3, 0, 5] = 60000.0
            x[4, 0, 33] = -1e30
            x[5, 0, 64:] = torch.linspace(-6e-8, 6e-8, 64)
            v = x.to(dt)
            s.batch.append(0, v, v)
            torch.cuda.synchronize()
            got = ref.values(s.pool, shape)[0, torch.from_numpy(s.tables[0]).long().cuda()]
            got = got.permute(1, 2, 0, 3, 4).flatten(2, 3)[0, 0, :20]
            want = v[:, 0].to(F64)
            if dtype in (F16, BF16):
                assert torch.equal(got.isnan(), want.isnan())
                assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
            elif dtype == FP8:
                assert torch.equal(got.isnan(), want.isnan())
                w = want.clamp(-448, 448).float().to(torch.float8_e4m3fn).to(F64)
                assert torch.equal(got.nan_to_num(7.0), w.nan_to_num(7.0))
            else:
                assert bool(got[0, :32].isnan().all()) and not bool(got[0, 32:].isnan().any())
                assert not bool(got[1:].isnan().any())
                assert bool((got[1] == 3.25).all())
                assert got[3, 5] == 16384 or abs(got[3, 5] - 16384) <= 16
                # A scale under 2^-25 (half of fp16's least) is 0: then the values are
                # at most 15 * 2^-25 apart, and the base is off by 2^-25 at most.
                assert float((got[2] - want[2]).abs().max()) <= 16 * 2.0 ** -25
                assert float((got[5] - want[5]).abs().max()) <= 16 * 2.0 ** -25


@pytest.mark.parametrize("scale", [2.0 ** -120, 1e-3, 0.3, 7.0, 2.0 ** 120])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_append_fp8_scales(dt, scale):
    """The fp32 quotient, rounded to nearest even: every 16-bit pattern, infinities and
    NaN among them, and halfway cases of the type."""
    shape = (1, 80, 2, 16, 256, FP8)
    n = 256
    with Step(shape, 2, [n], [n], dt, poison=False) as s:
        x = torch.arange(1 << 16, device="cuda").to(torch.int16).view(dt).view(128, 2, 256)
        half = (torch.randint(1, 64, (128, 2, 256), device="cuda") * 0.125 * scale).to(dt)
        v = torch.cat([x, half])
        s.batch.append(0, v, v.flip(0), k_scale=scale, v_scale=scale)
        torch.cuda.synchronize()
        ids = torch.from_numpy(s.tables[0]).long().cuda()
        got = s.pool.view(torch.float8_e4m3fn).view(80, 2, 2, 16, 256)[ids]
        got = got.to(F64).permute(1, 2, 0, 3, 4).flatten(2, 3)          # [2, H, n, D]
        q = v.float() / torch.full_like(v, scale, dtype=torch.float32)   # IEEE division
        want = q.clamp(-448, 448).to(torch.float8_e4m3fn).to(F64).permute(1, 0, 2)
        for which, w in ((0, want), (1, want.flip(1))):
            assert torch.equal(got[which].isnan(), w.isnan())
            assert torch.equal(got[which].nan_to_num(9.0), w.nan_to_num(9.0))


# -- together, as a program uses them --------------------------------------------

@pytest.mark.parametrize("kind", [KINDS[1], KINDS[3], KINDS[4]],
                         ids=[KIND_IDS[i] for i in (1, 3, 4)])
def test_a_preempted_prompt_goes_on_where_it_was(kind):
    """Prompts are computed, decoded, swapped out, swapped in to other blocks and
    decoded on: every step's result equals a run that was never preempted, bit for
    bit, and the 64-bit form."""
    dtype, dt = kind
    shape = (2, 200, 2, 16, 128, dtype)
    L, N, H, T, D, _ = shape
    Hq = 8
    gen = torch.Generator(device="cuda").manual_seed(11)
    lens = [150, 33, 470]
    perm = np.random.default_rng(4).permutation(N).astype(np.int32)
    here = [perm[:12], perm[12:20], perm[20:52]]
    there = [perm[60:72], perm[72:80], perm[80:112]]
    pools = [torch.zeros(L * N * ref.chunk_bytes(H, T, D, dtype), dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    kvs = [aqua.KVPool(shape, p) for p in pools]
    batches = [aqua.KVBatch(kv, Hq, 3, sum(lens), 52) for kv in kvs]
    rope = ref.rope_table(600, D)
    image = torch.zeros(L * 52 * ref.chunk_bytes(H, T, D, dtype), dtype=torch.uint8, device="cuda")
    ctx = np.array(lens)

    def step(i, tables, ctx, new, qkv):
        b = batches[i]
        b.set(tables, ctx, new)
        res = []
        for layer in range(L):
            x = qkv[layer]
            q = b.append(layer, x[:, Hq:Hq + H], x[:, Hq + H:], q=x[:, :Hq], rope=rope)
            res.append((q, *b.attend(layer, q, lse=True)))
        return res

    try:
        tables = here
        for k in range(6):
            new = ctx if k == 0 else np.ones(3, dtype=int)
            if k:
                ctx = ctx + 1
            qkv = torch.randn(L, int(sum(new)), Hq + 2 * H, D, device="cuda", generator=gen).to(dt)
            want, got = step(0, here, ctx, new, qkv), step(1, tables, ctx, new, qkv)
            torch.cuda.synchronize()
            for layer in range(L):
                for a, b in zip(want[layer], got[layer]):
                    assert torch.equal(a, b), (k, layer)
            vals = ref.values(pools[1], shape)
            o, l, mass, reach = ref.attend(vals, 1, tables, ctx, new, got[1][0])
            bo, bl = ref.attend_bounds(o, l, mass, reach, D, int(max(ctx)), dt, dtype,
                                       float(vals[vals.isfinite()].abs().amax()))
            ref.assert_within(got[1][1], o, bo, f"step {k}: out")
            if k in (1, 3):
                t = kvs[1].swap_out(tables, image)
                kvs[1].sync(t)
                pools[1].fill_(0xFF)
                tables = there if tables is here else here
                kvs[1].swap_in(tables, image)
                kvs[1].sync()
    finally:
        for kv in kvs:
            kv.close()


def test_a_captured_step_follows_its_batch():
    """One graph of two layers serves steps of other sequences, lengths and tables,
    with eager work between the replays; a decode step, a mixed one and none."""
    dtype, dt = BF16, torch.bfloat16
    shape = (2, 400, 2, 16, 128, dtype)
    L, N, H, T, D, _ = shape
    Hq, most = 8, 130
    steps = [([300, 20, 1500], [1, 1, 1]), ([40, 500], [40, 90]), ([2000], [1]),
             ([17, 18, 19, 900], [1, 3, 0, 100]), ([64], [64])]
    pool = ref.random_pool(shape, 8)
    rope = ref.rope_table(2001, D)
    side = torch.cuda.Stream()
    with aqua.KVPool(shape, pool) as kv:
        b = aqua.KVBatch(kv, Hq, 4, most, 200)
        q = torch.zeros(most, Hq, D, dtype=dt, device="cuda")
        k, v = (torch.zeros(most, H, D, dtype=dt, device="cuda") for _ in range(2))
        out = torch.zeros(L, most, Hq, D, dtype=dt, device="cuda")
        lse = torch.zeros(L, most, Hq, device="cuda")
        turned = torch.zeros(L, most, Hq, D, dtype=dt, device="cuda")

        def layers():
            for i in range(L):
                b.append(i, k, v, q=q, q_out=turned[i], rope=rope)
                b.attend(i, turned[i], out=out[i], lse=lse[i])

        tables = ref.tables_for([300, 20, 1500], T, N, 1)
        b.set(tables, *steps[0])
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            layers()
            for call in (lambda: b.set(tables, *steps[0]),
                         lambda: b.attend(0, q[:3], out=out[0][:3]),     # max_tokens rows
                         lambda: b.append(0, k[:3], v[:3])):
                with pytest.raises(aqua.AquaError) as err:
                    call()
                assert err.value.status == aqua.AQUA_ERR_INVALID
        for turn in range(3):
            for n, (ctx, new) in enumerate(steps):
                say("replay", turn, n)
                gen = torch.Generator(device="cuda").manual_seed(100 * turn + n)
                for x in (q, k, v):
                    x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
                tables = ref.tables_for(ctx, T, N, 10 * turn + n)
                before = pool.clone()
                b.set(tables, ctx, new)
                layers()                               # eager, for comparison
                torch.cuda.synchronize()
                want = [x.clone() for x in (pool, out, lse, turned)]
                pool.copy_(before)
                for x in (out, lse, turned):
                    x.fill_(3.0)
                graph.replay()
                torch.cuda.synchronize()
                m = sum(new)
                assert torch.equal(pool, want[0])
                for x, y in zip((out, lse, turned), want[1:]):
                    assert torch.equal(x[:, :m], y[:, :m])
                    assert bool((x[:, m:] == 3.0).all())
        del graph


def test_sets_without_a_wait_between_them():
    """More steps in a row than the batch has staging slots, with no host wait."""
    shape = (1, 300, 2, 16, 64, F16)
    ctxs = [[100 + 7 * i, 30 + i] for i in range(12)]
    with Step(shape, 4, ctxs[0], [1, 1], torch.float16, limits=(2, 2, 40), poison=False) as s:
        tables = [ref.tables_for(c, 16, 300, i) for i, c in enumerate(ctxs)]
        outs = []
        for c, t in zip(ctxs, tables):
            s.batch.set(t, c, [1, 1])
            outs.append(s.batch.attend(0, s.q, lse=True))
        torch.cuda.synchronize()
        for c, t, got in zip(ctxs, tables, outs):
            s.ctx, s.tables = c, t
            s.check_attend(0, s.q, "step", got=got)


def test_another_stream_and_two_batches():
    """Calls on a stream that is not the current one, and two batches at once."""
    shape = (1, 600, 2, 16, 128, BF16)
    with Step(shape, 8, [5000, 40], [1, 1], torch.bfloat16) as s:
        other = aqua.KVBatch(s.kv, 8, 2, 2, 400)
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        s.batch.set(s.tables, s.ctx, s.new, stream=a)
        other.set(s.tables, s.ctx, s.new, stream=b)
        got = [(x.attend(0, s.q, lse=True, stream=st))
               for _ in range(4) for x, st in ((s.batch, a), (other, b))]
        torch.cuda.synchronize()
        for g in got:
            assert torch.equal(g[0], got[0][0]) and torch.equal(g[1], got[0][1])
        s.check_attend(0, s.q, "streams", got=got[0])


def test_results_on_another_stream_are_its_own_memory():
    """What the current stream has let go may still be read there: a result on another
    stream does not lie in it."""
    with Step((1, 20, 2, 16, 128, BF16), 4, [100, 50], [2, 50], torch.bfloat16) as s:
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        gone = []
        for shape, dt in [((s.tokens, 4, 128), torch.bfloat16), ((s.tokens, 4), torch.float32)]:
            t = torch.empty(shape, dtype=dt, device="cuda")
            gone.append(t.data_ptr())
            del t
        q_out = s.batch.append(0, s.k, s.v, q=s.q, stream=side)
        out, lse = s.batch.attend(0, q_out, lse=True, stream=side)
        raw = s.batch.attend(0, q_out, stream=side.cuda_stream)
        side.synchronize()
        for t in (q_out, out, lse, raw):
            assert t.data_ptr() not in gone
        assert torch.equal(q_out, s.q) and torch.equal(raw, out)
        s.check_attend(0, s.q, "side stream", got=(out, lse))


def test_shared_prefix_is_read_by_both():
    """Two sequences whose tables share full blocks; appending to a shared block is
    refused."""
    shape = (1, 60, 2, 16, 128, BF16)
    with Step(shape, 4, [100, 120], [1, 1], torch.bfloat16, poison=False) as s:
        shared = s.tables[0].copy()
        other = np.concatenate([shared[:5], s.tables[1][5:]])
        s.tables = [shared, other]
        s.batch.set(s.tables, [100, 120], [1, 1])
        s.check_attend(0, s.q, "shared")
        s.batch.append(0, s.k, s.v)                    # the last blocks are their own
        same = [shared, shared]
        s.batch.set(same, [100, 100], [1, 1])
        s.tables, s.ctx = same, [100, 100]
        s.check_attend(0, s.q, "the same table twice")
        before = s.pool.clone()
        with pytest.raises(aqua.AquaError) as e:
            s.batch.append(0, s.k, s.v)
        assert e.value.status == aqua.AQUA_ERR_DUPLICATE
        torch.cuda.synchronize()
        assert torch.equal(s.pool, before)


# -- refusals ---------------------------------------------------------------------

def test_refusals():
    shape = (2, 60, 2, 16, 128, BF16)
    INV = aqua.AQUA_ERR_INVALID
    with Step(shape, 4, [100, 50], [2, 50], torch.bfloat16) as s:
        b, n = s.batch, s.tokens
        before = s.pool.clone()
        out = torch.full((n, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        rope = ref.rope_table(100, 128)
        wide = torch.zeros(n, 4, 256, dtype=torch.bfloat16, device="cuda")

        def refused(what, fn, status=INV):
            with pytest.raises(aqua.AquaError) as e:
                fn()
            say(what, e.value)
            assert e.value.status == status, what

        at = lambda **kw: b.attend(kw.pop("layer", 0), kw.pop("q", s.q), out=kw.pop("out", out),
                                   **kw)
        refused("layer", lambda: at(layer=2))
        refused("type", lambda: at(q=s.q.half(), out=out.half()))
        refused("float queries", lambda: at(q=s.q.float()))
        refused("host queries", lambda: at(q=s.q.cpu()))
        refused("few rows", lambda: at(q=s.q[:n - 1]))
        refused("few rows of the result", lambda: at(out=out[:n - 1]))
        refused("heads", lambda: at(q=s.q[:, :2]))
        refused("head size", lambda: at(q=wide))
        refused("strided head", lambda: at(q=wide[:, :, ::2]))
        refused("heads apart", lambda: at(q=wide[:, :, :128]))
        refused("misaligned", lambda: at(q=torch.zeros(n * 512 + 1, dtype=torch.bfloat16,
                                                       device="cuda")[1:].view(n, 4, 128)))
        refused("the result is the queries", lambda: at(out=s.q))
        refused("infinite scale", lambda: at(scale=float("inf")))
        refused("scale past fp32 in powers of two", lambda: at(scale=3e38))
        refused("no number", lambda: at(scale=float("nan")))
        refused("scale of another pool", lambda: at(k_scale=2.0))
        refused("lse type", lambda: at(lse=torch.zeros(n, 4, device="cuda", dtype=F64)))
        refused("lse rows", lambda: at(lse=torch.zeros(n - 1, 4, device="cuda")))

        ap = lambda **kw: b.append(kw.pop("layer", 0), kw.pop("k", s.k), kw.pop("v", s.v), **kw)
        refused("layer", lambda: ap(layer=2))
        refused("types", lambda: ap(v=s.v.half()))
        refused("rows", lambda: ap(k=s.k[:n - 1]))
        refused("short table", lambda: ap(rope=rope[:99].contiguous()))
        refused("odd rotation", lambda: ap(rope=torch.zeros(100, 24, device="cuda")))
        refused("wide rotation", lambda: ap(rope=torch.zeros(100, 144, device="cuda")))
        refused("half table", lambda: ap(rope=rope.half()))
        refused("no queries", lambda: ap(q_out=out))
        refused("queries shifted", lambda: ap(q=s.q, q_out=s.qkv[:, 1:5]))
        refused("v scale", lambda: ap(v_scale=0.5))
        refused("queries onto keys", lambda: ap(q=s.q.clone(), q_out=s.qkv[:, 1:5]))
        refused("queries onto values", lambda: ap(q=s.q.clone(), q_out=s.qkv[:, 4:8]))
        x = torch.zeros(n + 1, 8, 128, dtype=torch.bfloat16, device="cuda")
        shifted = torch.as_strided(x, (n, 4, 128), x.stride(), 6 * 128)   # 2 heads of the next row
        refused("queries onto the next row's keys", lambda: ap(k=x[:n, :2], q=s.q, q_out=shifted))

        CAP, RANGE = aqua.AQUA_ERR_CAPACITY, aqua.AQUA_ERR_RANGE
        t = s.tables
        refused("three sequences", lambda: b.set([t[0], t[1], []], [1, 1, 0], [1, 1, 0]), CAP)
        refused("tokens", lambda: b.set(t, [100, 50], [3, 50]), CAP)
        refused("blocks", lambda: b.set([np.arange(30), t[1]], [100, 50], [1, 1]), CAP)
        refused("context", lambda: b.set(t, [113, 50], [1, 1]), CAP)
        refused("new > context", lambda: b.set(t, [1, 50], [2, 1]))
        refused("negative", lambda: b.set(t, [100, 50], [-1, 1]))
        refused("lengths", lambda: b.set(t, [100], [1]))
        refused("block id", lambda: b.set([np.where(t[0] == t[0][3], 60, t[0]), t[1]],
                                          [100, 50], [1, 1]), RANGE)
        refused("negative id", lambda: b.set([np.where(t[0] == t[0][3], -1, t[0]), t[1]],
                                             [100, 50], [1, 1]), RANGE)
        torch.cuda.synchronize()
        assert torch.equal(s.pool, before) and bool((out == 5).all())
        s.check_attend(0, s.q, "the batch is as it was set")    # after refused sets

        D = aqua.aqua_kv_batch_desc
        for what, args in {"heads": (3, 1, 1, 1), "no heads": (0, 1, 1, 1), "seqs": (4, 0, 1, 1),
                           "tokens": (4, 1, 0, 1), "blocks": (4, 1, 1, 0),
                           "many heads": (65538, 1, 1, 1)}.items():
            st, _ = aqua.aqua_kv_batch_create(s.kv.handle, D(*args))
            assert st == INV, what
        assert aqua.aqua_kv_batch_create(None, D(4, 1, 1, 1))[0] == INV
        L = aqua.load()
        assert L.aqua_kv_append(b.handle, 0, None, None) == INV
        assert L.aqua_kv_attend(b.handle, 0, None, None) == INV
        assert L.aqua_kv_attend(None, 0, ctypes.byref(aqua.aqua_kv_attend_args()), None) == INV
        # Addresses that torch would not make.
        a = aqua.aqua_kv_attend_args(q=s.q.data_ptr(), out=out.data_ptr(), q_stride=s.q.stride(0),
                                     out_stride=1 << 30, dtype=BF16, scale=1.0, k_scale=1.0,
                                     v_scale=1.0)
        assert aqua.aqua_kv_attend(b.handle, 0, a, None) == INV      # past its allocation
        a.out_stride, a.q_stride = 512, 500
        assert aqua.aqua_kv_attend(b.handle, 0, a, None) == INV
    for shape in [(1, 8, 2, 2, 128, BF16), (1, 8, 2, 12, 128, BF16), (1, 8, 2, 16, 96, BF16)]:
        pool = torch.zeros(8 * ref.chunk_bytes(*shape[2:]), dtype=torch.uint8, device="cuda")
        with aqua.KVPool(shape, pool) as kv:
            with pytest.raises(aqua.AquaError):
                aqua.KVBatch(kv, 4, 1, 1, 1)


# -- a step's shape ----------------------------------------------------------------

@pytest.mark.parametrize("kind", [KINDS[1], KINDS[4]], ids=[KIND_IDS[1], KIND_IDS[4]])
def test_a_long_context_among_many_short_ones(kind):
    """So many short contexts that they fill a launch's rounds by themselves, and one that
    is split all the same; called and captured."""
    ctx = [1 + (37 * i) % 61 for i in range(530)]
    ctx[200] = 20011
    shape = (1, sum(-(-c // 16) for c in ctx) + 3, 8, 16, 64, kind[0])
    with Step(shape, 24, ctx, [1] * len(ctx), kind[1], seed=5) as s:
        out, lse = s.check_attend(0, s.q, "many")
        graph, again = torch.cuda.CUDAGraph(), torch.empty_like(out)
        with torch.cuda.graph(graph):
            s.batch.attend(0, s.q, out=again)
        for _ in range(3):
            again.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(again, out)
        del graph


def test_tensors_of_a_model_under_no_grad():
    """A model's parameters require gradients; what it makes under no_grad does not, and a
    leaf is read there as any other tensor."""
    with Step((1, 40, 2, 16, 128, BF16), 4, [200, 90], [2, 80], torch.bfloat16) as s:
        leaf = s.q.clone().requires_grad_()
        with pytest.raises(aqua.AquaError, match="gradient"):
            s.batch.attend(0, leaf)
        with torch.no_grad():
            got = s.batch.attend(0, leaf, lse=True)
            assert s.batch.append(0, s.k, s.v, q=leaf).equal(leaf)
        with torch.inference_mode():
            again = s.batch.attend(0, leaf, lse=True)
        torch.cuda.synchronize()
        assert not got[0].requires_grad
        want = s.batch.attend(0, leaf.detach(), lse=True)
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


def test_results_that_share_memory_are_refused():
    """Outputs lie apart from each other, from what a call reads, and from the pool."""
    shape = (1, 60, 2, 16, 128, BF16)
    with Step(shape, 4, [100, 50], [2, 50], torch.bfloat16, poison=False) as s:
        b, n = s.batch, s.tokens
        q = s.q.contiguous()
        out, rope = torch.empty_like(q), ref.rope_table(100, 128)
        before = s.pool.clone()
        bf16 = lambda t: t.view(torch.bfloat16)[:q.numel()].view(q.shape)
        f32 = lambda t: t.view(-1)[:2 * 4 * n].view(torch.float32).view(n, 4)
        last = lambda t: t.view(-1)[-2 * 4 * n:].view(torch.float32).view(n, 4)
        wide = torch.zeros(n, 12, 128, dtype=torch.bfloat16, device="cuda")
        calls = {
            "lse on the result": lambda: b.attend(0, q, out=out, lse=f32(out)),
            "lse on the result's end": lambda: b.attend(0, q, out=out, lse=last(out)),
            "lse on the queries": lambda: b.attend(0, q, out=out, lse=f32(q)),
            "lse on the last queries": lambda: b.attend(0, q, out=out, lse=last(q)),
            "lse on the pool": lambda: b.attend(0, q, out=out, lse=f32(bf16(s.pool))),
            "result on the pool": lambda: b.attend(0, q, out=bf16(s.pool)),
            "result on the pool's end": lambda: b.attend(0, q, out=bf16(s.pool[-2 * q.numel():])),
            "queries on the pool": lambda: b.append(0, s.k, s.v, q=q, q_out=bf16(s.pool)),
            "queries on the table": lambda: b.append(
                0, s.k, s.v, q=q, q_out=bf16(big), rope=big[:100 * 128].view(100, 128)),
            "queries on the table's end": lambda: b.append(
                0, s.k, s.v, q=q, q_out=bf16(big[99 * 128:]), rope=big[:100 * 128].view(100, 128)),
        }
        big = torch.zeros(100 * 128 + q.numel(), device="cuda")
        for what, call in calls.items():
            with pytest.raises(aqua.AquaError) as e:
                call()
            say(what, e.value)
            assert e.value.status == aqua.AQUA_ERR_INVALID, what
        torch.cuda.synchronize()
        assert torch.equal(s.pool, before) and not bool(big.any())
        # Side by side is apart: results and queries in one tensor's heads, the sums and the
        # result in one allocation, the queries rotated next to their table.
        wide[:, :4] = q
        one = torch.zeros(2 * q.numel() + 4 * 4 * n, dtype=torch.uint8, device="cuda")
        side, sums = one[:2 * q.numel()].view(torch.bfloat16).view(q.shape), \
            one[2 * q.numel():].view(torch.float32).view(n, 4)
        want = b.attend(0, q, lse=True)
        for o, l in ((wide[:, 4:8], None), (side, sums), (wide[:, 8:], sums)):
            got = b.attend(0, wide[:, :4], out=o, lse=True if l is None else l)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        big[:100 * 128] = rope.flatten()
        turned = b.append(0, s.k, s.v, q=q, q_out=bf16(big[100 * 128:]),
                          rope=big[:100 * 128].view(100, 128))
        torch.cuda.synchronize()
        pos = torch.from_numpy(ref.positions(s.ctx, s.new)).cuda()
        y, size = ref.rotate(q, pos, rope, False)
        f = size * 3 * 2.0 ** -24
        ref.assert_within(turned, y, y.abs() * 2.0 ** -8 + f * (1 + 2.0 ** -8), "queries")


@pytest.mark.parametrize("vs", [2.0 ** -124, 2.0 ** 115])
def test_value_scales_at_the_ends_of_fp32(vs):
    """The scale of the values does not underflow on its way to the result, over long
    contexts too, whose sums of weights are large."""
    ctx, new = [30000, 7, 900, 1300], [1, 1, 300, 3]
    shape = (1, 2100, 2, 16, 128, FP8)
    with Step(shape, 8, ctx, new, torch.bfloat16, seed=3) as s:
        # Values of 64 to 120, so that results are normal numbers of bf16.
        vals = s.pool.view(1, 2100, 2, 2, 16, 128)[:, :, 1]
        vals.copy_(torch.where(vals == 0xFF, vals, vals % 8 + 0x68))
        for scale in (None, 0.0):                      # 0: sums of weights as large as can be
            out, lse = s.batch.attend(0, s.q, lse=True, v_scale=vs, scale=scale)
            torch.cuda.synchronize()
            s.check_attend(0, s.q, f"scaled, {scale}", got=(out.to(F64) / vs, lse), scale=scale)


@pytest.mark.parametrize("m", [3, 150], ids=["rows", "tiles"])
def test_a_scale_of_zero_with_products_as_large_as_they_come(m):
    """All scores are 0 then, and below fp32's normal scales what the product makes of
    them."""
    ctx = [400]
    with Step((1, 30, 2, 16, 128, BF16), 4, ctx, [m], torch.bfloat16, seed=5) as s:
        used = s.pool.view(torch.bfloat16).view(30, 2, 2, 16, 128)
        keys = used[:, 0]
        keys.copy_(torch.where(keys.isfinite(), keys * 2.0 ** 58, keys))
        q = s.q * 2.0 ** 58                            # products of 2^116 to 2^123
        vals = ref.values(s.pool, s.shape)
        for scale in (0.0, 2.0 ** -130, -(2.0 ** -130)):
            out, lse = s.batch.attend(0, q, lse=True, scale=scale)
            torch.cuda.synchronize()
            # scale * log2(e) has a subnormal's bits: 2^-149 of 2^-130 at most.
            o, l, mass, reach = ref.attend(vals, 0, s.tables, ctx, [m], q, scale=scale)
            bo, bl = ref.attend_bounds(o, l, mass, reach, 128, 400, torch.bfloat16, BF16, 6.0)
            extra = reach * 2.0 ** -19 + 2.0 ** 123 * 2.0 ** -148
            ref.assert_within(lse, l, bl + extra, f"{scale}: lse")
            ref.assert_within(out, o, bo + 2.1 * extra[..., None] * mass, f"{scale}: out")


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("m", [2, 150], ids=["rows", "tiles"])
def test_scores_as_large_as_the_header_has_them(m, kind):
    """Scores up to 2^24 in size: each query's weight is all on the key that stands out
    for it, and the log sum is that score."""
    D, ctx = 64, [700]
    shape = (1, 50, 1, 16, D, kind[0])
    with Step(shape, 2, ctx, [m], kind[1], seed=5) as s:
        q = torch.zeros_like(s.q)
        q[:, 0, 0], q[:, 1, 0] = 4.0, -4.0
        # Keys of one value: 1, and 3 at position 300; -2 at position 301.
        k = torch.zeros(700, 1, D, dtype=kind[1], device="cuda")
        k[:, 0, 0] = 1
        k[300, 0, 0], k[301, 0, 0] = 3, -2
        v = torch.randn(700, 1, D, device="cuda").to(kind[1])
        one = aqua.KVBatch(s.kv, 2, 1, 700, 44)
        one.set(s.tables, ctx, ctx)
        one.append(0, k, v)
        held = ref.cached(ref.values(s.pool, shape), 0, s.tables[0], 700)[1][0]
        scale = 2.0 ** 20
        out, lse = s.batch.attend(0, q, lse=True, scale=scale)
        torch.cuda.synchronize()
        # Scores of 12 * 2^20 (products of 3 and 4) and 8 * 2^20; a key's 4-bit rounding (a
        # group of 0 and 3: half a step of 1/5, times 4) and log2(e)'s in fp32.
        off = 0.4 if kind[0] == INT4 else 0.0
        for h, at, want in ((0, 300, 12.0), (1, 301, 8.0)):
            assert float((lse[:, h].to(F64) - want * scale).abs().max()) <= \
                (want * 2.0 ** -21 + off) * scale
            assert bool(((out[:, h].to(F64) - held[at]).abs() <=
                         held[at].abs() * 2.0 ** -7 + 2.0 ** -24).all())


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[1], KINDS[3], KINDS[4]],
                         ids=[KIND_IDS[i] for i in (0, 1, 3, 4)])
@pytest.mark.parametrize("m", [1, 3, 150], ids=["one", "rows", "tiles"])
def test_values_that_are_not_finite_and_seen(m, kind):
    """An element of a value that every query sees and that is not finite leaves that
    element of the results not finite, and the others as they are."""
    pool_dtype, dt = kind
    shape, ctx, d = (1, 60, 1, 16, 128, pool_dtype), [900], 37
    with Step(shape, 4, ctx, [m], dt, seed=5) as s:
        clean, clean_lse = s.batch.attend(0, s.q, lse=True)
        block, slot = int(s.tables[0][20]), 3
        if pool_dtype == INT4:
            ref.codes_and_pairs(s.pool, shape)[1][0, block, 1, 0, slot, d // 32, 1] = float("inf")
            hit = torch.arange(128, device="cuda") // 32 == d // 32
        else:
            row = s.pool.view(ref.TORCH[pool_dtype]).view(60, 2, 1, 16, 128)
            row[block, 1, 0, slot, d] = float("nan") if pool_dtype == FP8 else -float("inf")
            hit = torch.arange(128, device="cuda") == d
        out, lse = s.batch.attend(0, s.q, lse=True)
        torch.cuda.synchronize()
        assert torch.equal(lse, clean_lse)
        assert torch.equal(out[..., ~hit], clean[..., ~hit])
        assert not bool(out[..., hit].isfinite().any())


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("D", [64, 256])
def test_heads_of_64_and_256_split_long_contexts(D, kind):
    """Contexts of so many parts that groups of a join's lanes share them, with a tile of 16
    columns that is partly filled."""
    ctx, new = [20001, 7, 9000, 4097], [1, 1, 100, 3]
    shape = (1, 2200, 2, 16, D, kind[0])
    with Step(shape, 10, ctx, new, kind[1], seed=3) as s:
        s.check_attend(0, s.q, "splits")


@pytest.mark.parametrize("kind", [KINDS[1], KINDS[3], KINDS[4]],
                         ids=[KIND_IDS[i] for i in (1, 3, 4)])
@pytest.mark.parametrize("T", [128, 1024])
def test_large_blocks(T, kind):
    ctx, new = [3000, 1, T, T + 1, 900], [1, 1, 2, 1, 200]
    shape = (2, 40, 2, T, 128, kind[0])
    with Step(shape, 8, ctx, new, kind[1], seed=T) as s:
        s.check_attend(1, s.q, "large blocks")
        before, rope = s.pool.clone(), ref.rope_table(3000, 128)
        q = s.batch.append(1, s.k, s.v, q=s.q, rope=rope)
        torch.cuda.synchronize()
        # (What no context holds is NaN here, and compared bit for bit.)
        check_append(s, 1, rope, False, before, q)


@pytest.mark.parametrize("kind", [KINDS[1], KINDS[4]], ids=[KIND_IDS[1], KIND_IDS[4]])
def test_very_many_query_heads(kind):
    """More columns of one token than a workgroup takes."""
    shape = (1, 40, 1, 16, 64, kind[0])
    with Step(shape, 4099, [300, 20], [2, 1], kind[1], seed=4, poison=False) as s:
        s.check_attend(0, s.q, "heads")
        before, rope = s.pool.clone(), ref.rope_table(300, 64)
        q = s.batch.append(0, s.k, s.v, q=s.q, rope=rope)
        torch.cuda.synchronize()
        check_append(s, 0, rope, False, before, q)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_append_int4_code_by_code(dt):
    """Scales, bases and codes are the fp32 formulas' to the last bit, at values halfway
    between two codes too."""
    shape, n = (1, 40, 2, 16, 256, INT4), 512
    with Step(shape, 2, [n], [n], dt, poison=False) as s:
        gen = torch.Generator(device="cuda").manual_seed(3)
        x = torch.randn(n, 2, 256, device="cuda", generator=gen)
        x = x * 2.0 ** torch.randint(-12, 14, (n, 2, 1), device="cuda", generator=gen)
        # Groups of steps p = 2^-3 ... 2^4 from -8 p to 7 p, at and between the codes: exact.
        p = 2.0 ** torch.randint(-3, 5, (n // 2, 2, 8, 1), device="cuda", generator=gen)
        half = torch.randint(-15, 14, (n // 2, 2, 8, 32), device="cuda", generator=gen) * 0.5 * p
        half[..., 3:4], half[..., 17:18] = -8 * p, 7 * p
        x[::2] = half.flatten(2)
        x = x.to(dt)
        v = x.flip(0).contiguous()
        s.batch.append(0, x, v)
        torch.cuda.synchronize()
        words, pairs = ref.codes_and_pairs(s.pool, shape)
        ids = torch.from_numpy(s.tables[0]).long().cuda()[:n // 16]
        rows = lambda t: t[0, ids].permute(1, 0, 3, 2, *range(4, t.dim() - 1)).flatten(1, 2)
        code, pair = rows(ref.codes(words)).cpu(), rows(pairs).cpu()     # [2, n, H, ...]
        for which, t in ((0, x), (1, v)):
            g = t.cpu().float().clamp(-16384, 16384).unflatten(-1, (8, 32))
            lo, hi = g.amin(-1), g.amax(-1)
            scale = ((hi - lo) / torch.full_like(lo, 15.0)).half()       # IEEE divisions
            base = (lo - 16 * scale.float()).half()
            assert torch.equal(pair[which][..., 0], scale)
            assert torch.equal(pair[which][..., 1], base)
            step = torch.where(scale > 0, scale.float(), torch.ones_like(lo))[..., None]
            want = (((g - base.float()[..., None]) / step).round() - 16).clamp(0, 15)
            assert torch.equal(code[which].unflatten(-1, (8, 32)).float(), want)
            if which == 0:                                               # the exact groups
                e = ((g.double() - base.double()[..., None]) / step.double())[::2]
                assert int(((e - e.floor()) == 0.5).sum()) > 10000
                assert torch.equal((e.round() - 16).clamp(0, 15).float(), want[::2])


def test_a_replayed_append_writes_what_the_call_itself_would():
    """Nothing where two tables hold a block that is written; and of a context that reaches
    behind the rotation table, the tokens before its end."""
    shape = (1, 60, 2, 16, 128, BF16)
    n, R = 40, 64
    # A table of 100 rows within a larger tensor, whose other rows would show.
    rope = torch.cat([ref.rope_table(100, R), torch.full((60, R), 3.0, device="cuda")])
    with Step(shape, 4, [90, 50], [20, 20], torch.bfloat16, poison=False,
              limits=(2, n, 60)) as s:
        out = torch.full_like(s.q, 7.0)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            s.batch.append(0, s.k, s.v, q=s.q, q_out=out, rope=rope[:100])
        free = np.random.default_rng(1).permutation(60).astype(np.int32)
        a, b = free[:12], free[12:24]
        for turn in range(3):
            say("turn", turn)
            # Both sequences write block 5 of a's.
            s.batch.set([a, a], [90, 90], [20, 20])
            before = s.pool.clone()
            out.fill_(7.0)
            with pytest.raises(aqua.AquaError) as e:
                s.batch.append(0, s.k, s.v, q=s.q, q_out=out, rope=rope[:100])
            assert e.value.status == aqua.AQUA_ERR_DUPLICATE
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(s.pool, before) and bool((out == 7).all())
            # Positions 75 .. 114 and, one step later, one sequence that ends before the table does.
            for tables, ctx, new in (([a, b], [115, 33], [30, 10]), ([b], [100], [40])):
                s.batch.set(tables, ctx, new)
                if ctx[0] > 100:
                    with pytest.raises(aqua.AquaError) as e:
                        s.batch.append(0, s.k, s.v, q=s.q, q_out=out, rope=rope[:100])
                    assert e.value.status == aqua.AQUA_ERR_INVALID
                s.pool.fill_(0)
                out.fill_(7.0)
                graph.replay()
                torch.cuda.synchronize()
                pos = torch.from_numpy(ref.positions(ctx, new)).cuda()
                blk, slot = ref.slots(tables, ctx, new, 16)
                m, held = len(pos), s.pool.view(torch.bfloat16).view(60, 2, 2, 16, 128)
                there = pos < 100
                assert int(there.sum()) == min(m, m - (ctx[0] - 100))
                for x, got in ((s.q, out[:m]), (s.k, held[blk, 0, :, slot])):
                    y, size = ref.rotate(x[:m], pos.clamp(max=99), rope[:100], False)
                    f = size * 3 * 2.0 ** -24
                    bound = y.abs() * 2.0 ** -8 + f * (1 + 2.0 ** -8)
                    ref.assert_within(got[there], y[there], bound[there], "rotated")
                assert torch.equal(held[blk, 1, :, slot][there], s.v[:m][there])
                assert bool((out[:m][~there] == 7).all()) and bool((out[m:] == 7).all())
                # Nothing else: as many values as tokens have, all of them not 0 in the main.
                held[blk[there], :, :, slot[there]] = 0
                assert not bool(s.pool.any())
        del graph
