"""Size of the cache attention's workspace (no GPU): it goes by the items that a call is cut into, not by its rows."""
import pytest

import paper_2506_19651_amd as P


@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (14, 2, 64, "bf16"), (32, 8, 128, "f32"), (8, 8, 64, "f32")])
def test_many_rows_need_no_more_than_a_round_of_items(heads):
    h = P.Heads(*heads)
    # two rounds of 1024 workgroups at most, 128 pairs each of head_dim values and two numbers
    most = 1.1 * 2048 * 128 * (heads[2] + 2) * 4 * (0.5 if heads[3] == "bf16" else 0.25)
    for seqs in (1, 64, 1000):
        for rows in (1, 100, 4096, 32768, 200000):
            assert 0 < P.pevlm_cache_attn_workspace_bytes(h, seqs, rows) < most, (seqs, rows)
    assert P.pevlm_cache_attn_workspace_bytes(h, 1, 32768) == P.pevlm_cache_attn_workspace_bytes(h, 1, 262144)
