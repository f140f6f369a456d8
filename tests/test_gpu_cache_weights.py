"""What the weights of the cache attention are rounded to, tile by tile: two bf16 parts (2^-16) in tiles of 16 and 32 pairs of bf16 tensors, one
(2^-8) in tiles of 128, 2^-24 for fp32 tensors; and values of single tokens that count for much, where records and pages end."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
import test_gpu_cache as T
from test_gpu_cache import U, attn_case, i32

pytestmark = pytest.mark.gpu


def holds_to(weight_step):
    """The bound of test_gpu_cache.hold with the weights' own rounding beside the result's: out within half a step of its type of numbers whose weights
    are off by what their scores' sums, the exponential and weight_step make of them."""
    def hold(out, lse, want, dtype, d):
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        rows = want["rows"]
        assert (got[~rows] == 5).all() and (got_lse[~rows] == 5).all()
        step, n = 2.0 ** -8 if dtype == "bf16" else U, np.maximum(want["keys"][rows], 1)[:, None]
        weight = (3 * d + 8) * U * want["spread"][rows] + 2.0 ** -22
        ref, ref_lse = want["out"][rows], want["lse"][rows]
        fine = np.isfinite(ref_lse)
        assert np.array_equal(got_lse[rows][~fine], ref_lse[~fine])
        assert (np.abs(got_lse[rows] - ref_lse)[fine] <= (weight + 2 * n * U + 4 * U * np.abs(ref_lse) + 4 * U)[fine]).all()
        bound = step * np.abs(ref) + 2 * (weight + weight_step + 2 * n * U)[..., None] * want["mass"][rows] + 1e-30
        assert (np.abs(got[rows] - ref) <= bound).all(), (np.abs(got[rows] - ref) / bound).max()
    return hold


TILES = [("bf16", None, 2.0 ** -16), ("bf16", "32", 2.0 ** -16), ("bf16", "128", 2.0 ** -8), ("f32", None, U), ("f32", "32", U)]


@pytest.mark.parametrize("dtype,wide,weight_step", TILES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (14, 2, 64)])
def test_values_that_count_for_much(monkeypatch, hq, hkv, d, dtype, wide, weight_step):
    """V of the first and last token of a page, of a record's last and of the request's last, 128 times the others'."""
    page = 64
    held = [1, 17, 63, 64, 65, 200, 463]
    rows = {None: [1, 1, 2, 1, 1, 1, 1], "32": [1, 4, 9, 5, 3, 6, 5], "128": [1, 17, 40, 50, 30, 32, 60]}[wide]

    def edit(a):
        for s, n in enumerate(held):
            for t in {0, 15, 16, page - 1, page, 5 * page - 1, n // 16 * 16 - 1, n // 16 * 16, n - 2, n - 1}:
                if 0 <= t < n:
                    slot = a["table"][s, t // page] * page + t % page
                    scales = a["pool"][slot // page, :, slot % page // 16, 16 * d:].reshape(hkv, d // 32, 16, 2)
                    scales[:, :, slot % 16, 1] += 7
                    a["pool"][slot // page, :, slot % page // 16, 16 * d:] = scales.reshape(hkv, d)
    monkeypatch.setattr(T, "hold", holds_to(weight_step))
    attn_case(hq, hkv, d, dtype, page, held, rows, edit=edit, wide=wide)
    attn_case(hq, hkv, d, dtype, page, held, rows, sink=[0, 3, 0, 16, 17, 64, 20], window=[1, 2, 20, 16, 33, 80, 70], edit=edit, wide=wide)


@pytest.mark.parametrize("dtype,wide,weight_step", [x for x in TILES if x[1] != "128"])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_between_two_bf16_numbers(dtype, wide, weight_step, d):
    """Every other key has the weight 1/2 + 2^-9, halfway between two bf16 numbers, and -2 as value where the others have 1: out is what the
    rounding of the weight makes of it."""
    n, rows, page, hq = 256, {None: 2, "32": 9}[wide], 64, 4
    scale, w = -float(np.log(np.float64(0.5 + 2.0 ** -9))), 0.5 + 2.0 ** -9
    k, v = np.zeros((n, 1, d)), np.where(np.arange(n) % 2 == 0, 1.0, -2.0)[:, None, None] * np.ones((n, 1, d))
    k[::2, 0, 0] = 1
    heads = P.Heads(hq, 1, d, dtype, None, scale)
    width = (1 << 21) // page if wide else n // page
    pool, table = np.zeros((n // page, 1, page // 16, 17 * d), np.uint8), np.zeros((1, width), np.int64)
    table[0, :n // page] = np.arange(n // page)
    O.put(pool, np.arange(n), k, v)
    q = torch.zeros((rows, hq, d), dtype=T.DTYPES[dtype], device=T.DEV)
    q[:, :, 0] = 1
    tiles16 = -(-rows * hq // 16)  # tiles of 32 from 64 steps of a workgroup on, in a table of 2^21 tokens
    steps = tiles16 * (width * page // 32) / ((4 if d == 64 else 3) * torch.cuda.get_device_properties(0).multi_processor_count)
    assert (tiles16 > 1 and steps >= 64) == (wide == "32") and tiles16 <= 4
    out, lse = torch.full_like(q, 5.0), torch.full((rows, hq), 5.0, device=T.DEV)
    P.pevlm_cache_attn_kv4(q, out, P.KvCache(torch.from_numpy(pool).to(T.DEV), i32(table), page), heads, i32([0]), i32([rows]), i32([n]), lse=lse)
    want = O.attention(q.double().cpu().numpy(), pool, table[:, :n // page], [0] * hq, [0], [rows], [n], scale=scale)
    holds_to(weight_step)(out, lse, want, dtype, d)
    # one bf16 part of the weight would be 1/2 or 1/2 + 2^-8
    even = np.arange(n - rows, n) // 2 + 1
    odd = (np.arange(n - rows, n) + 1) // 2
    for part in (0.5, 0.5 + 2.0 ** -8):
        one = torch.from_numpy((even - 2 * part * odd) / (even + w * odd)).to(T.DTYPES[dtype]).to(T.DEV)
        with pytest.raises(AssertionError):
            holds_to(weight_step)(one[:, None, None].expand(rows, hq, d), lse, want, dtype, d)
