"""CPU tests of what aqua.KVBatch checks before the library sees a call: the library is
given addresses and 32-bit numbers, so what does not fit them has to be refused here."""
import types

import numpy as np
import pytest
import torch

from paper_2407_21255_amd import aqua

INVALID, RANGE = aqua.AQUA_ERR_INVALID, aqua.AQUA_ERR_RANGE


@pytest.fixture
def calls(monkeypatch):
    """The arguments of each aqua_kv_batch_set that gets through."""
    seen = []

    def take(batch, n, ids, offs, ctx, new, stream):
        read = lambda at, count, t: np.ctypeslib.as_array(
            (np.ctypeslib.as_ctypes_type(t) * count).from_address(at)).tolist() if count else []
        o = read(offs, n + 1, np.uint64)
        seen.append((read(ids, o[-1], np.int32), o, read(ctx, n, np.uint32),
                     read(new, n, np.uint32)))
        return aqua.AQUA_OK

    monkeypatch.setattr(aqua, "aqua_kv_batch_set", take)
    monkeypatch.setattr(aqua, "_raw_stream", lambda device: 0)
    return seen


def batch(layers=2):
    b = aqua.KVBatch.__new__(aqua.KVBatch)
    b.handle, b.num_q_heads, b.head_dim, b.max_tokens, b.tokens = None, 4, 128, 100, 0
    b.device, b.num_layers, b.num_kv_heads = 0, layers, 2
    b.pool = types.SimpleNamespace(
        handle=None, _spaces=[b], desc=aqua.aqua_kv_desc(layers, 100, 2, 16, 128, aqua.AQUA_BF16))
    return b


def refused(status, *args):
    with pytest.raises(aqua.AquaError) as e:
        batch().set(*args)
    assert e.value.status == status, args


@pytest.mark.parametrize("dtype", [np.int32, np.int64, np.uint64, np.int16, np.float64])
def test_tables_of_any_type_that_holds_their_ids(calls, dtype):
    a, b = np.array([3, 9, 1], dtype=dtype), np.array([70], dtype=dtype)
    batch().set([a, b], [40, 16], [1, 2])
    batch().set([np.array([3, 9, 1]), b], np.array([40, 16]), np.array([1, 2], dtype=np.uint8))
    batch().set((np.concatenate([a, b]), np.array([0, 3, 4])), [40, 16], [1, 2])
    batch().set([[3, 9, 1], (70,)], [40, 16], [1, 2])
    batch().set([np.array([3, 0, 9, 0, 1, 0], dtype=dtype)[::2], b], [40, 16], [1, 2])
    assert calls == [([3, 9, 1, 70], [0, 3, 4], [40, 16], [1, 2])] * 5


def test_nothing_to_do(calls):
    for tables, n in (([], 0), ([np.array([])], 1), ([[]], 1), ([np.zeros(0, np.int32)], 1),
                      ((np.zeros(0, np.int32), np.zeros(1, np.uint64)), 0)):
        batch().set(tables, [0] * n, [0] * n)
    batch().set([np.array([]), np.array([5, 6])], [0, 20], [0, 1])
    assert calls == [([], [0] * (n + 1), [0] * n, [0] * n) for n in (0, 1, 1, 1, 0)] + \
        [([5, 6], [0, 0, 2], [0, 20], [0, 1])]


@pytest.mark.parametrize("bad", [np.array([1 << 32, 5]), np.array([5, (1 << 40) + 2]),
                                 np.array([5, -(1 << 32)]), np.array([1 << 31, 0], dtype=np.uint32),
                                 np.array([1 << 63, 0], dtype=np.uint64), np.array([1.5, 2.0]),
                                 np.array([np.nan, 2.0])])
def test_an_id_is_not_wrapped_into_another_blocks(calls, bad):
    refused(RANGE, [bad], [20], [1])
    refused(RANGE, [np.array([7], dtype=np.int32), bad], [1, 20], [1, 1])
    refused(RANGE, (bad, np.array([0, 2])), [20], [1])
    assert not calls


def test_tables_of_another_shape_are_refused(calls):
    two = np.array([[1, 2], [3, 4]])
    for tables, n in (([two], 1), ([two, two], 2), ([two, np.array([5])], 2), ([np.array(5)], 1),
                      ([[[1, 2], [3, 4]]], 1), ((two, np.array([0, 2])), 1),
                      ((np.array([1, 2]), np.array([[0, 1], [1, 2]])), 1),
                      ((np.array([1, 2]), np.array([0, 3])), 1),          # past the ids
                      ((np.array([1, 2]), np.zeros(0)), 0)):
        refused(INVALID, tables, [16] * n, [1] * n)
    assert not calls


def test_counts_are_whole_numbers_in_a_row(calls):
    t = [np.array([1, 2]), np.array([3, 4])]
    for ctx, new in (([20.5, 20], [1, 1]), ([20, 20], [1, 0.5]), ([[20, 20]], [[1, 1]]),
                     ([[20], [20]], [1, 1]), ([20, 20], [[1], [1]]), ([20, 1 << 32], [1, 1]),
                     ([20, 20], [1, -1]), ([20, np.nan], [1, 1]), (20, 1), ([20], [1]),
                     (np.array([20, (1 << 64) - 1], dtype=np.uint64), [1, 1])):
        refused(INVALID, t, ctx, new)
    assert not calls
    batch().set(t, [20.0, 20.0], np.array([1.0, 2.0]))
    assert calls == [([1, 2, 3, 4], [0, 2, 4], [20, 20], [1, 2])]


def test_numbers_that_32_bits_do_not_hold(monkeypatch):
    """ctypes takes the low 32 bits of a number without a word."""
    monkeypatch.setattr(aqua, "aqua_kv_batch_create", lambda pool, desc: (aqua.AQUA_OK, 1))
    x = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    for layer in (-1, 2, 1 << 32, (1 << 32) + 1):
        for call in (lambda: batch().append(layer, x, x), lambda: batch().attend(layer, x)):
            with pytest.raises(aqua.AquaError) as e:
                call()
            assert e.value.status == INVALID
    pool = batch().pool
    pool.pool = torch.zeros(1)
    for args in ((4 + (1 << 32), 1, 1, 1), (4, 1 + (1 << 32), 1, 1), (4, 1, 1 + (1 << 32), 1),
                 (4, 1, 1, 1 + (1 << 32)), (4, -1, 1, 1)):
        with pytest.raises(aqua.AquaError) as e:
            aqua.KVBatch(pool, *args)
        assert e.value.status == INVALID


def test_tensors_that_require_a_gradient_are_refused():
    """A result without a gradient would cut the caller's graph without a word."""
    x = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    q = torch.zeros(1, 4, 128, dtype=torch.bfloat16)
    rope = torch.zeros(8, 128)
    g = lambda t: t.clone().requires_grad_()
    for call in (lambda b: b.append(0, g(x), x), lambda b: b.append(0, x, g(x) * 2),
                 lambda b: b.append(0, x, x, q=g(q)), lambda b: b.append(0, x, x, q=q, q_out=g(q)),
                 lambda b: b.append(0, x, x, rope=g(rope)), lambda b: b.attend(0, g(q)),
                 lambda b: b.attend(0, q, out=g(q)), lambda b: b.attend(0, q, lse=g(rope[:, :4]))):
        with pytest.raises(aqua.AquaError, match="gradient") as e:
            call(batch())
        assert e.value.status == INVALID


def test_the_stream_is_the_pools_devices_current_one(calls, monkeypatch):
    """... whichever device is the current one, as for torch's own operators."""
    monkeypatch.undo()
    streams, entered = [], []
    monkeypatch.setattr(aqua, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(aqua, "_cur_device", lambda: 0)
    monkeypatch.setattr(aqua, "aqua_kv_batch_set", lambda *a: streams.append(a[-1]) or aqua.AQUA_OK)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    b = batch()
    b.device = 1
    b.set([np.array([1])], [1], [1])
    b.set([np.array([1])], [1], [1], stream=7)
    b.device = 0
    b.set([np.array([1])], [1], [1])
    assert streams == [1001, 7, 1000]

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            entered.append(self.device)

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(aqua, "_capturing", lambda: len(entered) > 0)
    assert b._needed(None) == 1 and entered == []      # the current device: not asked for
    b.device = 1
    assert b._needed(None) == b.max_tokens and entered == [1]
