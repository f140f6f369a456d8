"""Cache attention of queries that bf16 does not hold: the largest fp32 numbers, which round to infinity there, and infinities."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
from gpu_util import DEV
from test_gpu_cache import DTYPES, hold, i32

pytestmark = pytest.mark.gpu
PAGE, HELD = 64, 300


def call(q, k, v, dtype, scale, rows, wide):
    """out and lse of the last `rows` tokens, the pool and the table; wide: a table of 2^21 tokens, for tiles of 32 or 128."""
    hq, d = q.shape[1:]
    heads = P.Heads(hq, 1, d, dtype, None, scale)
    pages = -(-HELD // PAGE)
    pool = O.put(np.zeros((pages, 1, PAGE // 16, 17 * d), np.uint8), np.arange(HELD), k, v)
    table = np.zeros((1, (1 << 21) // PAGE if wide else pages), np.int64)
    table[0, :pages] = np.arange(pages)
    out, lse = torch.full_like(q, 5.0), torch.full((rows, hq), 5.0, device=DEV)
    P.pevlm_cache_attn_kv4(q, out, P.KvCache(torch.from_numpy(pool).to(DEV), i32(table), PAGE), heads, i32([0]), i32([rows]), i32([HELD]), lse=lse)
    return out, lse, pool, table[:, :pages]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,wide", [(1, False), (7, True)])
def test_the_largest_numbers(rows, wide, d):
    rng = np.random.default_rng(d + rows)
    top = np.float32(np.finfo(np.float32).max)
    q = (rng.uniform(0.25, 1, (rows, 4, d)) * rng.choice([-1, 1], (rows, 4, d)) * 2.0 ** 127).astype(np.float32)
    q[:, :, ::5] = top * rng.choice([-1, 1], q[:, :, ::5].shape).astype(np.float32)
    q[:, 1, 3] = np.float32(3.3954e38)  # halfway between bf16's largest number and 2^128
    k, v = rng.standard_normal((HELD, 1, d)) * 2.0 ** -95, rng.standard_normal((HELD, 1, d))
    qd, scale = torch.from_numpy(q).to(DEV), 2.0 ** -34
    out, lse, pool, table = call(qd, k, v, "f32", scale, rows, wide)
    want = O.attention(q.astype(np.float64), pool, table, [0] * 4, [0], [rows], [HELD], scale=scale)
    assert np.isfinite(want["out"]).all() and 0.5 < np.abs(want["spread"]).max() < 1e3
    hold(out, lse, want, "f32", d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,rows,wide", [("bf16", 2, False), ("f32", 2, False), ("bf16", 9, True), ("f32", 9, True), ("bf16", 30, True)])
def test_infinities(dtype, rows, wide, d):
    """A score of -inf has no weight: a row that has no other gets what one that sees nothing gets; one of +inf leaves no number."""
    rng = np.random.default_rng(d + rows)
    k, v = rng.standard_normal((HELD, 1, d)), rng.standard_normal((HELD, 1, d))
    k[:, :, 0] = 4.0  # the largest of its block or near it: never the code of 0
    q = rng.standard_normal((rows, 4, d))
    q[0, 0, 0], q[0, 1, 0], q[rows - 1, 2, 0] = -np.inf, np.inf, -np.inf
    out, lse, pool, table = call(torch.from_numpy(q).to(DTYPES[dtype]).to(DEV), k, v, dtype, 0.0, rows, wide)
    for row, head, want in ((0, 0, 0.0), (rows - 1, 2, 0.0), (0, 1, np.nan)):
        w = torch.full((d,), want, dtype=out.dtype, device=DEV)
        assert torch.equal(out[row, head].isnan(), w.isnan()) and (want != 0 or (out[row, head] == 0).all()), (row, head)
        assert lse[row, head].isnan() if np.isnan(want) else lse[row, head] == -np.inf
    # the other rows and heads of the tile have their numbers
    fine = np.isfinite(q).all(-1)
    qf = torch.from_numpy(np.where(fine[..., None], q, 0.0)).to(DTYPES[dtype]).double().numpy()
    ref = O.attention(qf, pool, table, [0] * 4, [0], [rows], [HELD])
    assert out[torch.from_numpy(fine).to(DEV)].isfinite().all()
    some = np.argwhere(fine)[::7]
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20
    for r, h in some:
        bound = step * np.abs(ref["out"][r, h]) + 2 * (step + 2.0 ** -13) * ref["mass"][r, h]
        assert (np.abs(out[r, h].double().cpu().numpy() - ref["out"][r, h]) <= bound).all()
