"""The operators on the pool from a plain C program (tests/c_kv_client.c, built by
build()): what it was given and what it got, against the 64-bit forms."""
import os
import subprocess

import numpy as np
import pytest
import torch

from tests import kv_ref as ref
from tests.gpu_util import say
from tests.kv_ref import F16

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLIENT = os.path.join(ROOT, "tests", "c_kv_client")

# The program's fixed shape, tables and step.
SHAPE = (2, 32, 2, 16, 64, F16)
HQ, LAYER = 4, 1
TABLES = [np.array([30, 2, 17, 4, 9]), np.array([0, 31, 11])]
CTX, NEW = [70, 33], [5, 33]


@pytest.mark.gpu
def test_c_program_appends_and_attends_through_the_abi(tmp_path):
    assert os.path.exists(CLIENT), "build() compiles tests/c_kv_client"
    say("c_kv_client", tmp_path)
    r = subprocess.run([CLIENT, str(tmp_path)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip().endswith("c_kv_client: ok")

    L, N, H, T, D, _ = SHAPE
    load = lambda name, dtype, *shape: torch.from_numpy(
        np.fromfile(tmp_path / name, dtype=np.uint8)).cuda().view(dtype).view(*shape)
    half = lambda name, heads: load(name, torch.float16, -1, heads, D)
    k, v, q, turned = half("k.bin", H), half("v.bin", H), half("q.bin", HQ), half("q_out.bin", HQ)
    rope = load("rope.bin", torch.float32, -1, D)
    before, after = (load(n, torch.uint8, -1) for n in ("pool_before.bin", "pool_after.bin"))

    # The append: rotated rows in their slots, all else as it was.
    pos = torch.from_numpy(ref.positions(CTX, NEW)).cuda()
    blk, slot = ref.slots(TABLES, CTX, NEW, T)
    rows = lambda p: p.view(torch.float16).view(L, N, 2, H, T, D)
    held, want = rows(after), rows(before).clone()
    u = ref.half_step(torch.float16)
    for x, got, what in ((q, turned, "queries"), (k, held[LAYER, blk, 0, :, slot], "keys")):
        y, size = ref.rotate(x, pos, rope, False)
        f32 = size * 3 * 2.0 ** -24
        ref.assert_within(got, y, y.abs() * u + f32 * (1 + u) + 2.0 ** -25, what)
    assert torch.equal(held[LAYER, blk, 1, :, slot], v)
    want[LAYER, blk, :, :, slot] = held[LAYER, blk, :, :, slot]
    assert torch.equal(after.view(torch.int16), want.view(torch.int16).flatten())

    # The step's attention, and that of the last tokens after the swap to other blocks.
    vals = ref.values(after, SHAPE)
    last = turned[[4, 37]]
    for new, x, out, lse in ((NEW, turned, "out.bin", "lse.bin"),
                             ([1, 1], last, "out_moved.bin", "lse_moved.bin")):
        o, l, mass, reach = ref.attend(vals, LAYER, TABLES, CTX, new, x, scale=0.125)
        bo, bl = ref.attend_bounds(o, l, mass, reach, D, 70, torch.float16, F16, 2.0)
        ref.assert_within(half(out, HQ), o, bo, out)
        ref.assert_within(load(lse, torch.float32, -1, HQ), l, bl, lse)
