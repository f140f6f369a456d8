"""The cache attention's workspace holds the parts of units that are cut, and of no others: cut requests between whole ones, in every kind of tile, and
calls of many rows with no more than the size query asks for."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
from gpu_util import DEV
from test_gpu_cache import DTYPES, U, attn_case, i32
from test_gpu_cache_long import exact, far

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [9, 70])
@pytest.mark.parametrize("dtype,hq,hkv,d,wide", [("bf16", 8, 2, 128, None), ("f32", 14, 2, 64, None), ("bf16", 14, 2, 64, "32"), ("f32", 8, 2, 128, "32"),
                                                 ("bf16", 8, 2, 128, "128"), ("bf16", 14, 2, 64, "128")])
def test_cut_requests_between_whole_ones(n, dtype, hq, hkv, d, wide):
    rng = np.random.default_rng(n + d)
    held = rng.integers(20, 90, n)
    held[[0, 3, n - 3]] = 1500, 2100, 700
    short, mean = (16, 17) if d == 64 else (28, 30)  # rows of a tile of 128: 119 and 120 pairs a request on average
    rows = {None: np.ones(n, int), "32": np.full(n, 5), "128": np.minimum(held, short)}[wide]
    if wide == "128":
        rows[held > 100] += (mean * n - rows.sum()) // 3 + 1
    assert (rows > 0).all() and (rows <= held).all()
    attn_case(hq, hkv, d, dtype, 64 if wide == "32" else 16, held.tolist(), rows.tolist(), wide=wide)


@pytest.mark.parametrize("dtype,hq,hkv,d,rows,held", [("bf16", 16, 4, 128, 4500, 5000), ("bf16", 14, 2, 64, 9001, 9100), ("f32", 8, 4, 64, 3000, 3500),
                                                      ("bf16", 28, 4, 128, 700, 9000)])
def test_many_rows_of_one_request(dtype, hq, hkv, d, rows, held):
    page = 64
    rng = np.random.default_rng(rows)
    columns = -(-held // page)
    pool = rng.integers(0, 256, (columns, hkv, page // 16, 17 * d)).astype(np.uint8)
    pool[..., 16 * d:] = rng.integers(123, 126, pool[..., 16 * d:].shape)
    order = rng.permutation(columns)
    heads = P.Heads(hq, hkv, d, dtype)
    need = P.pevlm_cache_attn_workspace_bytes(heads, 1, rows)
    assert need < 100 << 20
    block = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device=DEV)
    q = (torch.randn((rows, hq, d), generator=torch.Generator().manual_seed(rows)) * 0.4).to(DTYPES[dtype]).to(DEV)
    out, lse = torch.empty_like(q), torch.empty((rows, hq), device=DEV)
    P.pevlm_cache_attn_kv4(q, out, P.KvCache(torch.from_numpy(pool).to(DEV), i32(order[None]), page), heads, i32([0]), i32([rows]), i32([held]), lse=lse,
                           workspace=block[:need])
    k, v = (torch.from_numpy(x).to(DEV) for x in O.get(pool, order[np.arange(held) // page] * page + np.arange(held) % page))
    want = exact(q.double(), k, v, torch.arange(held - rows, held, device=DEV), 1 / np.sqrt(d), [h * hkv // hq for h in range(hq)])
    assert max(far(out, lse, want, dtype, d, held + 600, U if dtype == "f32" else 2.0 ** -8)) <= 1
    assert (block[need:] == 77).all()
