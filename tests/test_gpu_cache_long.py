"""Cache attention where a wavefront's list of records is read again (every 64 of its steps): long requests in items that no other workgroup shares.
Every page is another one, and those that weigh most lie behind the first such reading."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
from gpu_util import DEV
from test_gpu_cache import DTYPES, U, i32

pytestmark = pytest.mark.gpu


def exact(q, k, v, pos, scale, kv_of_q):
    """(out, lse, spread, mass) in 64 bits: the row at position pos[r] sees the keys up to there."""
    rows, hq, d = q.shape
    out, mass = torch.zeros(rows, hq, d, dtype=torch.float64, device=DEV), torch.zeros(rows, hq, d, dtype=torch.float64, device=DEV)
    lse, spread = torch.zeros(rows, hq, dtype=torch.float64, device=DEV), torch.zeros(rows, hq, dtype=torch.float64, device=DEV)
    seen = torch.arange(len(k), device=DEV) <= pos[:, None]
    for h in range(hq):
        kk, vv = k[:, kv_of_q[h]], v[:, kv_of_q[h]]
        s = (q[:, h] @ kk.T.contiguous() * scale).masked_fill(~seen, -np.inf)
        lse[:, h] = torch.logsumexp(s, -1)
        w = torch.exp(s - lse[:, h, None])
        out[:, h], mass[:, h] = w @ vv, w @ vv.abs()
        spread[:, h] = (q[:, h].abs() @ kk.abs().T.contiguous()).masked_fill(~seen, 0).amax(-1) * scale
    return out, lse, spread, mass


def far(got, got_lse, want, dtype, d, depth, weight_step):
    """By how much out and lse are further from the definition than their roundings allow: scores within (3 d + 8) U of the products that they add up,
    weights within 2^-22 of them and rounded to weight_step, sums of `depth` terms one after another, one rounding of the result."""
    out, lse, spread, mass = want
    weight = (3 * d + 8) * U * spread + 2.0 ** -22
    step = 2.0 ** -8 if dtype == "bf16" else U
    bound = step * out.abs() + 2 * (weight[..., None] + weight_step + 2 * depth * U) * mass + 1e-30
    bound_lse = weight + 2 * depth * U + 4 * U * lse.abs() + 4 * U
    return ((got.double() - out).abs() / bound).amax().item(), ((got_lse.double() - lse).abs() / bound_lse).amax().item()


# tile: pairs of a tile; the steps of a wavefront after which its list is read again, in tokens of the request, follow from it
CASES = [(16, 64, "bf16", 64, 16, 16, 1), (16, 64, "f32", 64, 16, 16, 1), (16, 128, "bf16", 64, 12, 12, 1), (16, 128, "f32", 64, 24, 12, 1),
         (16, 64, "bf16", 130, 8, 8, 1), (32, 64, "bf16", 64, 24, 12, 9), (32, 128, "bf16", 64, 24, 8, 7), (32, 128, "f32", 64, 8, 8, 20),
         (32, 64, "f32", 70, 24, 12, 9), (128, 64, "bf16", 16, 32, 32, 119), (128, 128, "bf16", 16, 32, 32, 125), (128, 64, "bf16", 65, 16, 8, 60),
         (128, 128, "bf16", 70, 16, 8, 40)]


@pytest.mark.parametrize("tile,d,dtype,n,hq,hkv,rows", CASES)
def test_records_behind_the_first_list(tile, d, dtype, n, hq, hkv, rows):
    page, again = 64, 4096 if tile == 128 else 8192
    longest = again + 700
    group, units = hq // hkv, torch.cuda.get_device_properties(0).multi_processor_count
    # the cut that the call takes, and items that are whole units: as many as the chip holds, or more
    pairs = rows * group
    tiles16, tiles128 = -(-pairs // 16), -(-pairs // 128)
    many = dtype == "bf16" and tiles16 > (4 if d == 128 else 7) * tiles128
    assert many == (tile == 128) and (tiles16 == 1) == (tile == 16) and pairs <= tile
    resident = 2 if tile == 128 else (4 if d == 64 else 3) - (tile == 32)
    # an item has work / target steps, work / (target - units) or half of that where they leave no room: more than the longest request
    assert n * hkv >= resident * units * (1 if n <= 64 else 0.55)

    rng = np.random.default_rng(tile + d + n)
    columns = -(-longest // page)
    pool = rng.integers(0, 256, (columns + 3, hkv, page // 16, 17 * d)).astype(np.uint8)
    pool[..., 16 * d:] = rng.integers(123, 126, pool[..., 16 * d:].shape)
    order = rng.permutation(columns + 3)[:columns]
    heavy = again // page + 2  # a page whose keys weigh most, behind the first list
    pool[order[heavy], :, :, 16 * d::2] += 3
    held = longest - 11 * (np.arange(n) % 40)
    heads = P.Heads(hq, hkv, d, dtype)
    cache = P.KvCache(torch.from_numpy(pool).to(DEV), i32(np.broadcast_to(order, (n, columns)).copy()), page)
    q = (torch.randn((n * rows, hq, d), generator=torch.Generator().manual_seed(n + d)) * 0.4).to(DTYPES[dtype]).to(DEV)
    out, lse = torch.empty_like(q), torch.empty((n * rows, hq), device=DEV)
    P.pevlm_cache_attn_kv4(q, out, cache, heads, i32(np.arange(n) * rows), i32([rows] * n), i32(held), lse=lse)

    kv = [h // group for h in range(hq)]
    pos = torch.from_numpy((held - rows)[:, None] + np.arange(rows)).flatten().to(DEV)
    depth = longest if tile == 128 else longest // 4 + 96  # the wavefronts share the pairs, or take the steps in turn
    weight_step = U if dtype == "f32" else (2.0 ** -8 if tile == 128 else 2.0 ** -16)

    def want(columns_read):
        slots = columns_read[np.arange(longest) // page].astype(np.int64) * page + np.arange(longest) % page
        k, v = (torch.from_numpy(x).to(DEV) for x in O.get(pool, slots))
        return exact(q.double(), k, v, pos, 1 / np.sqrt(d), kv)
    assert max(far(out, lse, want(order), dtype, d, depth, weight_step)) <= 1
    # the definition with a list that was not read again is further away than that
    stale = order.copy()
    stale[again // page:] = order[:columns - again // page]
    assert min(far(out, lse, want(stale), dtype, d, depth, weight_step)) > 3
