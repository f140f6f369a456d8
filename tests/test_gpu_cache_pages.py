"""Pages that a request gives back when it ends, as the header says, go to the requests after it."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
from gpu_util import DEV
from test_gpu_cache import hold, i32

pytestmark = pytest.mark.gpu


def test_pages_come_back_and_go_to_another_request():
    """Three requests share a pool that holds two of them at their longest; the second ends, and a new one takes its place and its pages."""
    page, hq, hkv, d, n = 16, 8, 2, 64, 3
    heads, rng = P.Heads(hq, hkv, d, "bf16"), np.random.default_rng(12)
    cache = P.KvCache(P.KvCache.new_pool(heads, 9, page, DEV), i32(np.full((n, 8), -1)), page)
    free, num_free = i32(rng.permutation(9)), i32([9])
    seq_len, row_start, row_len = i32([0] * n), i32([0] * n), i32([0] * n)
    kept = {s: (np.zeros((0, hkv, d)), np.zeros((0, hkv, d))) for s in range(n)}  # what every request put in

    def step(new, served):
        rows = sum(new)
        slot_map = i32([0] * rows)
        P.pevlm_cache_slots(cache, seq_len, i32(new), free, num_free, seq_len, num_free, row_start, row_len, slot_map)
        assert row_len.tolist() == served
        k, v = (torch.from_numpy(rng.standard_normal((rows, hkv, d))).to(torch.bfloat16).to(DEV) for _ in range(2))
        q = torch.from_numpy(rng.standard_normal((rows, hq, d))).to(torch.bfloat16).to(DEV)
        P.pevlm_cache_store_kv4(k, v, slot_map, cache, heads)
        out, lse = torch.full_like(q, 5.0), torch.full((rows, hq), 5.0, device=DEV)
        P.pevlm_cache_attn_kv4(q, out, cache, heads, row_start, row_len, seq_len, lse=lse)
        at = 0
        for s in range(n):
            if served[s]:
                kept[s] = tuple(np.concatenate([a, x[at:at + new[s]].double().cpu().numpy()]) for a, x in zip(kept[s], (k, v)))
            at += new[s]
        # the definition over a pool of its own, where the requests' tokens lie one after another
        lens = [len(kept[s][0]) for s in range(n)]
        assert seq_len.tolist() == lens
        table, pool = np.arange(n * 8).reshape(n, 8), np.zeros((n * 8, hkv, 1, 17 * d), np.uint8)
        for s in range(n):
            O.put(pool, s * 8 * page + np.arange(lens[s]), *kept[s])
        hold(out, lse, O.attention(q.double().cpu().numpy(), pool, table, [h // (hq // hkv) for h in range(hq)], row_start.cpu().numpy(), row_len.cpu().numpy(),
                                   seq_len.cpu().numpy()), "bf16", d)

    def end(s):  # on the GPU, without a look at the lengths from the host
        count = (seq_len[s] + page - 1) // page
        column = torch.arange(8, device=DEV)
        to = torch.where(column < count, num_free.long() + column, torch.full_like(column, 9))
        grown = torch.cat([free, free.new_zeros(1)])
        grown[to] = cache.block_table[s]
        free.copy_(grown[:9])
        num_free.add_(count)
        seq_len[s] = 0
        kept[s] = (np.zeros((0, hkv, d)), np.zeros((0, hkv, d)))

    step([40, 50, 20], [40, 50, 20])        # 3 + 4 + 2 pages: all of them
    assert num_free.item() == 0
    step([8, 14, 13], [8, 14, 0])           # the third would need one more
    end(1)
    assert num_free.item() == 4 and sorted(free.tolist()[:4]) == sorted(cache.block_table[1, :4].tolist())
    step([1, 0, 13], [1, 0, 13])            # two of the pages that came back
    step([15, 30, 1], [15, 30, 1])          # a new request in the second one's place, on the other two
    assert num_free.item() == 0
    used = [p for s, m in zip(range(n), seq_len.tolist()) for p in cache.block_table[s, :-(-m // page)].tolist()]
    assert sorted(used) == list(range(9))
