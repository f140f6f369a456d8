"""The 4-bit cache's oracle against what the format fixes, worked out by hand, and the package's refusals (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P


def test_codes_of_the_format():
    # sign, two exponent bits with bias 1, one mantissa bit
    for code in range(16):
        s, e, m = code >> 3, code >> 1 & 3, code & 1
        value = (m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)) * (-1) ** s
        assert O.VALUES[code] == value


def test_ties_go_to_the_even_code_and_the_scale_is_the_smallest_that_fits():
    x = np.zeros(32)
    x[:10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5]
    codes, s = O.encode_block(x)
    assert s == 127 and codes[:10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14]
    for amax, e in ((6, 0), (np.nextafter(6, 7), 1), (12, 1), (3, -1), (1, -2), (0.75, -3), (0, 0), (2.0 ** -140, -100), (3.4e38, 125)):
        assert O.exponent(amax) == e, amax
    assert O.encode_block([np.inf] + [1] * 31)[1] == 255 and O.encode_block([np.nan] + [1] * 31)[1] == 255
    codes, s = O.encode_block([2.0 ** 127 * 1.99] + [2.0 ** 126] * 31)  # beyond 6 * 2^125: saturates
    assert s == 252 and codes[0] == 7 and O.VALUES[codes[1]] == 2


def test_the_array_form_is_the_block_form():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 2, 64)) * 2.0 ** rng.integers(-130, 128, (5, 2, 1))
    x[0, 0, 3], x[1, 1, 40], x[2] = np.inf, np.nan, 0
    codes, scales = O.encode(x)
    for n in range(5):
        for h in range(2):
            for b in range(2):
                c, s = O.encode_block(x[n, h, b * 32:b * 32 + 32])
                assert s == scales[n, h, b] and (s == 255 or np.array_equal(c, codes[n, h, b * 32:b * 32 + 32]))


def test_a_value_is_kept_to_half_a_step():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((200, 1, 64))
    y = O.values(*O.encode(x))
    top = np.abs(x.reshape(200, 1, 2, 32)).max(-1).repeat(32, -1)
    # the step at the top is 2 * 2^e, and 6 * 2^e < 2 * top
    assert (np.abs(x - y) <= np.maximum(top / 3, 0)).all() and np.abs(x - y).mean() < 0.1


def test_bytes_of_a_record_by_hand():
    pool = np.zeros((2, 1, 2, 17 * 64), np.uint8)
    k, v = np.zeros((1, 1, 64)), np.zeros((1, 1, 64))
    k[0, 0, 33], k[0, 0, 32], v[0, 0, 0] = 6, -3, 1.5
    O.put(pool, [32 + 16 + 5], k, v)  # page 1, record 1, token 5
    rec = pool[1, 0, 1]
    assert rec[(16 + 5) * 16] == 13 + 16 * 7  # K, block 1, byte 0: element 32 low, 33 high
    assert rec[512 + 5 * 16] == 7             # V, block 0, element 0: 1.5 = 6 * 2^-2
    assert rec[1024 + (16 + 5) * 2] == 127 and rec[1024 + 5 * 2 + 1] == 125 and rec[1024 + 5 * 2] == 127
    assert np.count_nonzero(pool) == 6
    kk, vv = O.get(pool, [53])
    assert np.array_equal(kk, k) and np.array_equal(vv, v)


def test_attention_of_the_oracle_against_the_formula_spelt_out():
    rng = np.random.default_rng(5)
    pool, table = np.zeros((4, 2, 1, 17 * 64), np.uint8), np.array([[2, 0, 3]])
    k, v = rng.standard_normal((37, 2, 64)), rng.standard_normal((37, 2, 64))
    O.put(pool, [table[0, t // 16] * 16 + t % 16 for t in range(37)], k, v)
    k, v = O.values(*O.encode(k)), O.values(*O.encode(v))
    q = rng.standard_normal((3, 2, 64))
    r = O.attention(q, pool, table, [1, 0], [1], [2], [37], [2], [5])
    assert r["rows"].tolist() == [False, True, True]
    for i, p in ((1, 35), (2, 36)):
        for h, g in ((0, 1), (1, 0)):
            keys = [0, 1] + list(range(p - 4, p + 1))
            w = [math.exp(float(k[j, g] @ q[i, h]) / 8) for j in keys]
            want = sum(a * v[j, g] for a, j in zip(w, keys)) / sum(w)
            assert np.abs(r["out"][i, h] - want).max() < 1e-12 and abs(r["lse"][i, h] - math.log(sum(w))) < 1e-12
    empty = O.attention(q, pool, table, [1, 0], [0], [1], [37], [0], [0])
    assert (empty["out"][0] == 0).all() and (empty["lse"][0] == -np.inf).all()
    # planted mistakes show: a window off by one, a sink that is lost, the other KV head, keys behind the row
    for wrong in (([1, 0], [2], [6]), ([1, 0], [1], [5]), ([0, 1], [2], [5])):
        o = O.attention(q, pool, table, wrong[0], [1], [2], [37], wrong[1], wrong[2])
        assert np.abs(o["out"][1:] - r["out"][1:]).max() > 1e-3


def test_slots_of_the_oracle_by_hand():
    r = O.slots([[9, -1, -1], [-1, -1, -1], [4, -1, -1]], [5, 7, 8], 3, [15, 0, 16], [2, 17, 1], 20, 16, 10, [0, 100, 0])
    # request 0 takes page 8, request 1 wants two and gets 7 and 5, request 2 finds the list empty
    assert r["table"].tolist() == [[9, 8, -1], [7, 5, -1], [4, -1, -1]]
    assert r["row_len"].tolist() == [2, 17, 0] and r["row_start"].tolist() == [0, 2, 19] and r["seq_len_out"].tolist() == [17, 17, 16]
    assert r["slot_map"].tolist() == [9 * 16 + 15, 8 * 16] + [7 * 16 + i for i in range(16)] + [5 * 16, -1]
    assert r["pos_ids"][2].tolist() == [15, 16] + [100 + i for i in range(17)] + [0] and r["num_free_out"].tolist() == [0]


# ------------------------------------------------------------------------------------------ refusals
INVALID, UNSUPPORTED, SMALL = P.binding.PEVLM_ERR_INVALID_ARG, P.binding.PEVLM_ERR_UNSUPPORTED, P.binding.PEVLM_ERR_WORKSPACE_TOO_SMALL
FAKE = 0x1000  # aligned, never dereferenced on these paths


def _cache(**changes):
    c = P.binding._CCache(FAKE, 10, 16, 2, 4, FAKE)
    for name, value in changes.items():
        setattr(c, name, value)
    return ctypes.byref(c)


BAD_POOLS = [dict(page_size=8), dict(page_size=24), dict(page_size=8192), dict(num_pages=0), dict(num_pages=1 << 27)]
BAD_TABLES = [dict(num_seqs=0), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(max_pages=1 << 27), dict(block_table=None), dict(block_table=FAKE + 2)]


@pytest.mark.parametrize("changes", BAD_POOLS + [dict(pool=None), dict(pool=FAKE + 8)])
def test_store_load_and_attention_refuse_a_bad_pool(changes):
    lib, heads = P.load_library(), P.Heads(4, 2, 64, "bf16")
    for fn in (lib.pevlm_cache_store_kv4, lib.pevlm_cache_load_kv4):
        assert fn(FAKE, FAKE, 0, 0, FAKE, 3, _cache(**changes), heads.ref(), None) == INVALID
    assert lib.pevlm_cache_attn_kv4(FAKE, FAKE, None, _cache(**changes), heads.ref(), 3, FAKE, FAKE, FAKE, None, None, FAKE, 1 << 40, None) == INVALID
    assert P.pevlm_last_error()


@pytest.mark.parametrize("changes", BAD_POOLS + BAD_TABLES)
def test_slots_refuse_a_bad_cache(changes):
    lib = P.load_library()
    assert lib.pevlm_cache_slots(_cache(**changes), FAKE, None, FAKE, 3, FAKE, 4, None, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 20, None) == INVALID


def test_slots_refuse_bad_arguments():
    lib = P.load_library()
    good = [_cache(), FAKE, None, FAKE, 3, FAKE, 4, None, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 20, None]
    for at, value in ((0, None), (1, None), (3, None), (4, -1), (5, None), (6, -1), (8, None), (9, None), (10, None), (11, None), (12, None), (1, FAKE + 2),
                      (2, FAKE + 1), (7, FAKE + 3), (12, FAKE + 2), (13, FAKE + 2)):
        args = list(good)
        args[at] = value
        assert lib.pevlm_cache_slots(*args) == INVALID, at
    for at, value in ((14, None), (14, FAKE + 16), (15, 4)):
        args = list(good)
        args[at] = value
        assert lib.pevlm_cache_slots(*args) == SMALL, at
    assert P.pevlm_cache_slots_workspace_bytes(0) == 0 and P.pevlm_cache_slots_workspace_bytes(100) >= 400


def test_store_and_load_refuse_bad_arguments():
    lib, heads = P.load_library(), P.Heads(4, 2, 64, "bf16")
    for fn in (lib.pevlm_cache_store_kv4, lib.pevlm_cache_load_kv4):
        good = [FAKE, FAKE, 0, 0, FAKE, 3, _cache(), heads.ref(), None]
        for at, value, status in ((0, None, INVALID), (1, None, INVALID), (0, FAKE + 8, INVALID), (2, 64, INVALID), (3, 132, INVALID), (3, -128, INVALID),
                                  (4, None, INVALID), (4, FAKE + 2, INVALID), (5, -1, INVALID), (6, None, INVALID), (7, None, INVALID),
                                  (7, P.Heads(4, 2, 96, "bf16").ref(), UNSUPPORTED), (7, P.Heads(4, 2, 64, 7).ref(), UNSUPPORTED), (7, P.Heads(4, 3, 64, "bf16").ref(), INVALID)):
            args = list(good)
            args[at] = value
            assert fn(*args) == status, (at, value)
        assert fn(None, None, 0, 0, None, 0, _cache(pool=None), heads.ref(), None) == P.binding.PEVLM_OK  # no rows: nothing to do


def test_attention_refuses_bad_arguments():
    lib, heads = P.load_library(), P.Heads(4, 2, 64, "bf16")
    good = [FAKE, FAKE, None, _cache(), heads.ref(), 3, FAKE, FAKE, FAKE, None, None, FAKE, 1 << 40, None]
    for at, value, status in ((0, None, INVALID), (0, FAKE + 8, INVALID), (1, None, INVALID), (2, FAKE + 2, INVALID), (3, None, INVALID), (4, None, INVALID),
                              (4, P.Heads(4, 2, 96, "bf16").ref(), UNSUPPORTED), (4, P.Heads(4, 2, 64, 5).ref(), UNSUPPORTED),
                              (4, P.Heads(4, 2, 64, "bf16", kv_head_of_q=[0, 1, 2, 0]).ref(), INVALID), (5, -1, INVALID), (6, None, INVALID), (7, None, INVALID),
                              (8, None, INVALID), (9, FAKE + 2, INVALID), (10, FAKE + 1, INVALID), (11, None, SMALL), (11, FAKE + 16, SMALL)):
        args = list(good)
        args[at] = value
        assert lib.pevlm_cache_attn_kv4(*args) == status, (at, value)
    for changes in BAD_TABLES:
        args = list(good)
        args[3] = _cache(**changes)
        assert lib.pevlm_cache_attn_kv4(*args) == INVALID, changes
    assert lib.pevlm_cache_attn_kv4(None, None, None, _cache(), heads.ref(), 0, None, None, None, None, None, None, 0, None) == P.binding.PEVLM_OK
    assert P.pevlm_cache_attn_workspace_bytes(heads, 0, 1) == 0 and P.pevlm_cache_attn_workspace_bytes(heads, 1, -1) == 0


def test_more_rows_than_a_launch_has_lanes_are_refused():
    lib = P.load_library()
    for d, hkv, rows in ((128, 8, 1 << 27), (64, 8, 1 << 28), (64, 1, (1 << 30) + 1), (64, 1, 2 ** 31 - 1)):
        for fn in (lib.pevlm_cache_store_kv4, lib.pevlm_cache_load_kv4):
            assert fn(FAKE, FAKE, 0, 0, FAKE, rows, _cache(), P.Heads(8, hkv, d, "bf16").ref(), None) == UNSUPPORTED, (d, hkv, rows)
    for rows in ((1 << 30) + 1, 2 ** 31 - 1):
        assert lib.pevlm_cache_slots(_cache(), FAKE, None, FAKE, 3, FAKE, rows, None, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 20, None) == UNSUPPORTED
    for hq, hkv, d, dtype, width in ((32, 8, 128, "bf16", 16), (32, 1, 64, "bf16", 1 << 12), (8, 8, 128, "f32", 1 << 12)):
        cache = _cache(max_pages=width // 16 * 16)
        for rows in (1 << 25, 2 ** 31 - 1):
            assert lib.pevlm_cache_attn_kv4(FAKE, FAKE, None, cache, P.Heads(hq, hkv, d, dtype).ref(), rows, FAKE, FAKE, FAKE, None, None, FAKE, 1 << 62,
                                            None) == UNSUPPORTED, (hq, hkv, d, dtype, rows)


def test_pool_bytes():
    assert P.pevlm_cache_pool_bytes(P.Heads(28, 4, 128, "bf16"), 10, 64) == 10 * 64 * 4 * 136
    assert P.pevlm_cache_pool_bytes(P.Heads(14, 2, 64, "f32"), 3, 16) == 3 * 16 * 2 * 68
    assert P.pevlm_cache_pool_bytes(P.Heads(14, 2, 64, "f32"), 3, 20) == 0 and P.pevlm_cache_pool_bytes(P.Heads(14, 2, 64, "f32"), 0, 16) == 0
    assert P.pevlm_cache_pool_bytes(P.Heads(32, 8, 128, "bf16"), 1 << 20, 256) == (1 << 28) * 8 * 136  # beyond 32 bits


def test_the_binding_refuses_what_the_tensors_say():
    heads = P.Heads(4, 2, 64, "bf16")
    pool, table = P.KvCache.new_pool(heads, 3, 32, "cpu"), torch.zeros((2, 4), dtype=torch.int32)
    cache = P.KvCache(pool, table, 32)
    assert (cache.num_pages, cache.n_kv_heads, cache.head_dim, cache.num_seqs, cache.max_pages) == (3, 2, 64, 2, 4)
    for bad in (lambda: P.KvCache(pool, table, 16), lambda: P.KvCache(pool.float(), table, 32), lambda: P.KvCache(pool[:, :, ::2], table, 16),
                lambda: P.KvCache(pool, table.long(), 32), lambda: P.KvCache(pool, table[:, ::2], 32), lambda: P.KvCache.new_pool(heads, 3, 20, "cpu")):
        with pytest.raises(P.PevlmError):
            bad()
    k, i32 = torch.zeros((5, 2, 64), dtype=torch.bfloat16), lambda n: torch.zeros(n, dtype=torch.int32)
    wide = torch.zeros((5, 3, 64), dtype=torch.bfloat16)
    for args in ((k.float(), k, i32(5)), (k, k[:4], i32(5)), (k, k, i32(4)), (k, k, i32(5).long()), (k, k.transpose(1, 2), i32(5)),
                 (k, torch.zeros((5, 64, 2), dtype=torch.bfloat16).transpose(1, 2), i32(5)), (wide[:, ::2], k, i32(5)),
                 (k, k, i32(5))):  # the last is in order but not in device memory
        with pytest.raises(P.PevlmError):
            P.pevlm_cache_store_kv4(*args, cache, heads)
        with pytest.raises(P.PevlmError):
            P.pevlm_cache_load_kv4(*args, cache, heads)
    with pytest.raises(P.PevlmError, match="KV heads"):
        P.pevlm_cache_store_kv4(k, k, i32(5), cache, P.Heads(4, 1, 64, "bf16"))
    q = torch.zeros((5, 4, 64), dtype=torch.bfloat16)
    ok = dict(row_start=i32(2), row_len=i32(2), seq_len=i32(2), workspace=torch.zeros(256, dtype=torch.uint8))
    for qq, out, more in ((q.float(), q, {}), (q, q[:4], {}), (q[:, :2], q[:, :2], {}), (q.transpose(0, 1), q, {}), (q, q, dict(row_len=i32(3))),
                          (q, q, dict(seq_len=None)), (q, q, dict(window=i32(2).long())), (q, q, dict(sink_len=i32(1))),
                          (q, q, dict(lse=torch.zeros((5, 4), dtype=torch.bfloat16))), (q, q, dict(lse=torch.zeros(5, 2))), (q, q, {})):
        with pytest.raises(P.PevlmError):
            P.pevlm_cache_attn_kv4(qq, out, cache, heads, **dict(ok, **more))
    for at in range(8):
        args = [i32(2), i32(2), i32(7), i32(1), i32(2), i32(1), i32(2), i32(2)]
        args[at] = args[at].float() if at != 2 else args[at].long()
        with pytest.raises(P.PevlmError):
            P.pevlm_cache_slots(cache, *args, i32(9), workspace=ok["workspace"])


def test_the_binding_refuses_rows_that_share_memory():
    """A row stride of 0 means contiguous rows to the library: one row that stands for five must not get there."""
    heads = P.Heads(4, 2, 64, "bf16")
    cache = P.KvCache(P.KvCache.new_pool(heads, 3, 32, "cpu"), torch.zeros((2, 4), dtype=torch.int32), 32)
    k, slots = torch.zeros((5, 2, 64), dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    one = torch.zeros((1, 2, 64), dtype=torch.bfloat16).expand(5, 2, 64)
    near = torch.zeros(5 * 128, dtype=torch.bfloat16).as_strided((5, 2, 64), (64, 64, 1))
    for bad in (one, near):
        for args in ((bad, k), (k, bad)):
            for call in (P.pevlm_cache_store_kv4, P.pevlm_cache_load_kv4):
                with pytest.raises(P.PevlmError, match="apart"):
                    call(*args, slots, cache, heads)


def test_the_binding_refuses_a_dtype_that_no_tensor_has():
    heads = P.Heads(4, 2, 64, 7)
    cache = P.KvCache(P.KvCache.new_pool(P.Heads(4, 2, 64, "bf16"), 3, 32, "cpu"), torch.zeros((2, 4), dtype=torch.int32), 32)
    rows, ints = torch.zeros((5, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((5, 4, 64), dtype=torch.bfloat16)
    for call in (P.pevlm_cache_store_kv4, P.pevlm_cache_load_kv4):
        with pytest.raises(P.PevlmError):
            call(rows, rows, torch.zeros(5, dtype=torch.int32), cache, heads)
    with pytest.raises(P.PevlmError):
        P.pevlm_cache_attn_kv4(q, q, cache, heads, ints, ints, ints, workspace=torch.zeros(256, dtype=torch.uint8))
