"""The paged 4-bit KV cache on the GPU against its definition in 64 bits: rows in and out, slots, attention, and the calls together."""
import numpy as np
import pytest
import torch

import kv4_oracle as O
import paper_2506_19651_amd as P
import workloads as W
from gpu_util import DEV

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def rounded(x, dtype):
    """x as the device tensor that a caller has, and its values in 64 bits."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(DTYPES[dtype])
    return t.to(DEV), t.double().numpy()


def pages_for(lengths, page, rng, spare=2, width=None):
    """A block table over shuffled pages (entries behind a request's pages: far outside the pool) and the number of pages."""
    counts = [-(-n // page) for n in lengths]
    order = rng.permutation(sum(counts) + spare)
    table = np.full((len(lengths), width or max(max(counts), 1)), 0x7fffffff, np.int64)
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    return table, sum(counts) + spare


# ------------------------------------------------------------------------------------------ rows in and out
def special_rows(hkv, d, rng):
    """Rows of every magnitude, halves of steps, powers of two, zeros, and blocks that hold an infinity or a NaN."""
    x = rng.standard_normal((41, hkv, d))
    x[1] *= 2.0 ** -60
    x[2] = 0
    x[3] = -0.0
    x[4] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -2.5, 6, -6], (hkv, d)) * 2.0 ** rng.integers(-20, 20, (hkv, 1))
    x[5] = 2.0 ** rng.integers(-126, 127, (hkv, d))
    x[6] = 2.0 ** -140
    x[7] = 3.0e38 * rng.choice([1, -1], (hkv, d))
    x[8, :, 7] = np.inf
    x[9, 0, d - 1] = np.nan
    x[10, :, 33] = -np.inf
    x[11, :, ::32] = 6 * 2.0 ** 5
    x[12] = 1.9921875 * 2.0 ** 126  # above 6 * 2^124
    x[13] *= 2.0 ** 100
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,d,page", [(1, 64, 16), (3, 128, 32), (4, 128, 256), (8, 64, 64)])
def test_rows_go_in_and_come_out_as_defined(dtype, hkv, d, page):
    rng = np.random.default_rng(d + hkv)
    heads = P.Heads(2 * hkv, hkv, d, dtype)
    pages = 3 + 80 // page
    slots = rng.permutation(pages * page)[:41]
    slots[[17, 30, 35]] = [-1, pages * page, -(2 ** 31)]  # nowhere
    before = rng.integers(0, 256, (pages, hkv, page // 16, 17 * d)).astype(np.uint8)
    pool = torch.from_numpy(before).to(DEV)
    cache = P.KvCache(pool, i32([[0]]), page)
    (k, k64), (v, v64) = rounded(special_rows(hkv, d, rng), dtype), rounded(special_rows(hkv, d, rng)[::-1].copy(), dtype)
    P.pevlm_cache_store_kv4(k, v, i32(slots), cache, heads)
    want = O.put(before.copy(), slots, k64, v64)
    assert np.array_equal(pool.cpu().numpy(), want)  # every byte of it, the other slots' among them
    back = torch.full((41, hkv, d), 7.0, dtype=DTYPES[dtype], device=DEV), torch.full((41, hkv, d), 7.0, dtype=DTYPES[dtype], device=DEV)
    P.pevlm_cache_load_kv4(*back, i32(slots), cache, heads)
    inside = (slots >= 0) & (slots < pages * page)
    for got, ref in zip(back, O.get(want, slots[inside])):
        got = got.double().cpu().numpy()
        assert (got[~inside] == 7).all() and np.array_equal(got[inside], ref, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_may_lie_inside_wider_ones(dtype):
    rng = np.random.default_rng(8)
    heads, n = P.Heads(4, 2, 128, dtype), 77
    wide, w64 = rounded(rng.standard_normal((n, 8, 128)), dtype)  # a projection's output: 4 query heads, 2 of K, 2 of V
    cache = P.KvCache(P.KvCache.new_pool(heads, 6, 16, DEV), i32([[0]]), 16)
    slots = rng.permutation(96)[:n]
    P.pevlm_cache_store_kv4(wide[:, 4:6], wide[:, 6:8], i32(slots), cache, heads)
    want = O.put(np.zeros(cache.pool.shape, np.uint8), slots, w64[:, 4:6], w64[:, 6:8])
    assert np.array_equal(cache.pool.cpu().numpy(), want)
    back = torch.full_like(wide, 3.0)
    P.pevlm_cache_load_kv4(back[:, 2:4], back[:, :2], i32(slots), cache, heads)
    k, v = O.get(want, slots)
    got = back.double().cpu().numpy()
    assert np.array_equal(got[:, 2:4], k) and np.array_equal(got[:, :2], v) and (got[:, 4:] == 3).all()
    one = torch.ones((1, 2, 128), dtype=DTYPES[dtype], device=DEV)  # one row, and none
    P.pevlm_cache_store_kv4(one, one, i32([5]), cache, heads)
    P.pevlm_cache_load_kv4(back[:1, :2], back[:1, 2:4], i32([5]), cache, heads)
    assert (back[0, :4] == 1).all()
    P.pevlm_cache_store_kv4(one[:0], one[:0], i32([]), cache, heads)


def test_every_number_of_sixteen_bits_is_rounded_as_defined():
    x = np.arange(65536, dtype=np.uint32)
    x = x[(x & 0x7f80) != 0x7f80]  # finite
    rng = np.random.default_rng(2)
    x = np.concatenate([x, x[: (-len(x)) % 64]])
    values = (rng.permutation(x) << 16).astype(np.uint32).view(np.float32)  # mixed magnitudes share a block
    near = np.sort(values)  # neighbours do
    for a in (values, near):
        k, k64 = rounded(a.reshape(-1, 1, 64), "bf16")
        n = len(k)
        heads = P.Heads(1, 1, 64, "bf16")
        cache = P.KvCache(P.KvCache.new_pool(heads, -(-n // 1024), 1024, DEV), i32([[0]]), 1024)
        P.pevlm_cache_store_kv4(k, k, torch.arange(n, dtype=torch.int32, device=DEV), cache, heads)
        got = torch.empty_like(k), torch.empty_like(k)
        P.pevlm_cache_load_kv4(*got, torch.arange(n, dtype=torch.int32, device=DEV), cache, heads)
        want = O.values(*O.encode(k64))
        assert np.array_equal(got[0].double().cpu().numpy(), want) and torch.equal(got[0], got[1])


# ------------------------------------------------------------------------------------------ slots
def run_slots(table, free, num_free, seq_len, new_len, rows, page, num_pages, pos_offset=None, in_place=False, want_pos=True):
    n = len(seq_len)
    pool = torch.zeros((num_pages, 1, page // 16, 17 * 64), dtype=torch.uint8, device=DEV)
    cache = P.KvCache(pool, i32(table), page)
    seq, count = i32(seq_len), i32([num_free])
    out = dict(seq_len_out=seq if in_place else i32([-9] * n), num_free_out=count if in_place else i32([-9]), row_start=i32([-9] * n),
               row_len=i32([-9] * n), slot_map=i32([-9] * rows), pos_ids=torch.full((3, rows), -9, dtype=torch.int32, device=DEV))
    ws = torch.full((P.pevlm_cache_slots_workspace_bytes(n),), 255, dtype=torch.uint8, device=DEV)
    P.pevlm_cache_slots(cache, seq, None if new_len is None else i32(new_len), i32(free), count, out["seq_len_out"], out["num_free_out"], out["row_start"],
                        out["row_len"], out["slot_map"], pos_ids=out["pos_ids"] if want_pos else None,
                        pos_offset=None if pos_offset is None else i32(pos_offset), workspace=ws)
    want = O.slots(table, free, num_free, seq_len, [1] * n if new_len is None else new_len, rows, page, num_pages, pos_offset)
    for name, w in want.items():
        got = (cache.block_table if name == "table" else out[name]).cpu().numpy()
        if name == "pos_ids" and not want_pos:
            w = np.full_like(w, -9)
        assert np.array_equal(got, w), (name, got, w)


SLOT_CASES = {
    "one request, empty": ([0], [1], 1),
    "none gets any": ([3, 16, 0], [0, 0, 0], 0),
    "page ends": ([15, 16, 17, 31, 32, 0], [1, 1, 1, 2, 17, 16], 38),
    "rows to spare": ([7, 40], [3, 5], 13),
    "rows end inside a request": ([7, 40, 3], [3, 5, 0], 6),
    "negative lengths": ([-4, 10, -1], [3, -7, 2], 5),
    "long and short": ([0, 0, 5, 100], [700, 1, 0, 333], 1034),
}


@pytest.mark.parametrize("name", SLOT_CASES)
@pytest.mark.parametrize("in_place", [False, True])
def test_slots(name, in_place):
    held, new, rows = SLOT_CASES[name]
    rng = np.random.default_rng(len(name))
    table, used = pages_for([max(h, 0) for h in held], 16, rng, 0, 50)
    free = rng.permutation(200)[:90]
    run_slots(table, free, 90, held, new, rows, 16, 200, in_place=in_place)
    run_slots(table, free, 90, held, new, rows, 16, 200, pos_offset=rng.integers(-1000, 1000, len(held)), in_place=in_place)
    run_slots(table, free, 90, held, None, len(held) + 2, 16, 200, in_place=in_place, want_pos=False)


def test_slots_when_pages_or_columns_run_out():
    rng = np.random.default_rng(1)
    table, _ = pages_for([20, 64, 100, 5, 32], 32, rng, 0, 4)
    free = rng.permutation(300)[:40]
    for num_free in (0, 1, 2, 3, 5, 8, 40, 1000, -3):  # 1000: more than the list has entries
        run_slots(table, free, num_free, [20, 64, 100, 5, 32], [13, 40, 20, 1, 70], 150, 32, 300)
        run_slots(table, free, num_free, [20, 64, 100, 5, 32], [12, 64, 29, 90, 0], 300, 32, 300)  # 100 + 29: one more than the table holds
    run_slots(table, free, 40, [2 ** 31 - 1, 64, 129, 5, 32], [2 ** 31 - 1, 1, 0, 1, 2 ** 31 - 1], 7, 32, 300)  # sums beyond 32 bits
    run_slots(table, [], 0, [20, 64, 100, 5, 32], [1, 1, 1, 1, 0], 5, 32, 300)
    run_slots(table, free - 150, 40, [20, 64, 100, 5, 32], [13, 40, 20, 1, 30], 150, 32, 100)  # pages of the list outside the pool


@pytest.mark.parametrize("n", [63, 64, 65, 1023, 1024, 1025, 2500])
def test_slots_of_many_requests(n):
    rng = np.random.default_rng(n)
    held, new = rng.integers(0, 100, n), rng.integers(0, 40, n) * (rng.random(n) < 0.7)
    table, used = pages_for(held, 16, rng, 0, 9)
    free = used + rng.permutation(4 * n)
    run_slots(table, free, 3 * n, held, new, int(new.sum()) + 1, 16, used + 4 * n)
    run_slots(table, free, n // 2, held, None, n, 16, used + 4 * n, in_place=True)


# ------------------------------------------------------------------------------------------ attention
def attn_case(hq, hkv, d, dtype, page, lengths, rows, sink=None, window=None, kv_of_q=None, scale=0.0, seed=0, order=None, edit=None, q_scale=1.0,
              wide=None):
    """Makes a cache and queries, calls, and holds out and lse to the oracle.  order: row_start of every request (default: packed).  wide: how the call
    is to be cut, "128" for tiles of 128 (row, head) pairs, with a table of 4096 tokens a request and more, "32" for tiles of 32, with one of 2^20."""
    rng = np.random.default_rng(seed + hq + d)
    heads = P.Heads(hq, hkv, d, dtype, kv_of_q, scale)
    table, pages = pages_for([max(n, 0) for n in lengths], page, rng, width=max(-(-max(lengths) // page), {"128": 4096, "32": 1 << 20}[wide] // page) if wide else None)
    pool = np.zeros((pages, hkv, page // 16, 17 * d), np.uint8)
    for s, n in enumerate(lengths):
        j = np.arange(max(n, 0))
        O.put(pool, table[s, j // page] * page + j % page, rng.standard_normal((len(j), hkv, d)) + 0.3, rng.standard_normal((len(j), hkv, d)) + 0.1)
    # what no row sees must not matter: unwritten slots hold every byte, NaN scales among them
    used = {int(table[s, t // page]) * page + t % page for s, n in enumerate(lengths) for t in range(n)}
    for slot in sorted(set(range(pages * page)) - used):
        for b in range(d // 32):
            t = slot % 16
            for which in range(2):
                pool[slot // page, :, slot % page // 16, which * 8 * d + (b * 16 + t) * 16:][:, :16] = 0x77
            pool[slot // page, :, slot % page // 16, 16 * d + (b * 16 + t) * 2:][:, :2] = 255
    num_rows = max([a + b for a, b in zip(order, rows)] if order else [sum(rows)])
    row_start = np.array(order) if order else np.concatenate([[0], np.cumsum(rows)[:-1]])
    q, q64 = rounded(rng.standard_normal((num_rows, hq, d)) * q_scale, dtype)
    a = dict(pool=pool, table=table, row_start=row_start, row_len=np.array(rows), seq_len=np.array(lengths), num_rows=num_rows)
    if edit:
        edit(a)
        q, q64 = q[:a["num_rows"]].contiguous(), q64[:a["num_rows"]]
    if wide:
        group, asking = max(np.bincount(kv_of_q)) if kv_of_q is not None else hq // hkv, min(len(rows), len(q))
        tiles16, tiles128 = (-(-len(q) * group // asking // n) for n in (16, 128))
        many = dtype == "bf16" and tiles16 > (4 if d == 128 else 7) * tiles128
        steps = asking * tiles16 * hkv * (1 << 15) / ((4 if d == 64 else 3) * torch.cuda.get_device_properties(0).multi_processor_count)
        assert many if wide == "128" else not many and tiles16 > 1 and steps >= 64
    cache = P.KvCache(torch.from_numpy(a["pool"]).to(DEV), i32(a["table"]), page)
    out = torch.full_like(q, 5.0)
    lse = torch.full(q.shape[:2], 5.0, device=DEV)
    ws = torch.full((P.pevlm_cache_attn_workspace_bytes(heads, len(lengths), len(q)),), 255, dtype=torch.uint8, device=DEV)
    P.pevlm_cache_attn_kv4(q, out, cache, heads, i32(a["row_start"]), i32(a["row_len"]), i32(a["seq_len"]), None if sink is None else i32(sink),
                           None if window is None else i32(window), lse=lse, workspace=ws)
    kv = kv_of_q if kv_of_q is not None else [h // (hq // hkv) for h in range(hq)]
    want = O.attention(q64, a["pool"], a["table"], kv, a["row_start"], a["row_len"], a["seq_len"], sink, window, scale if scale > 0 else None)
    hold(out, lse, want, dtype, d)
    again = torch.full_like(q, 5.0)
    P.pevlm_cache_attn_kv4(q, again, cache, heads, i32(a["row_start"]), i32(a["row_len"]), i32(a["seq_len"]), None if sink is None else i32(sink),
                           None if window is None else i32(window))
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))  # without lse, in other scratch memory: the same bits
    return want


def hold(out, lse, want, dtype, d):
    """A score is a sum of d products (of three parts each in fp32), each rounding within U of what it adds to; a weight's relative error is that
    plus the exponential's 2^-22; it is rounded to bf16 (2^-8) for bf16 tensors and to 2^-24 for fp32 ones; n weights are added up.  Numerator and
    denominator both have these errors, and the result is rounded once to its type (2^-8, 2^-24)."""
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    rows = want["rows"]
    assert (got[~rows] == 5).all() and (got_lse[~rows] == 5).all()
    for r in np.flatnonzero(rows):
        n = max(int(want["keys"][r]), 1)
        weight = (3 * d + 8) * U * want["spread"][r] + 2.0 ** -22  # [heads]
        step = 2.0 ** -8 if dtype == "bf16" else U
        fine = np.isfinite(want["lse"][r])
        assert np.array_equal(np.isnan(got_lse[r]), np.isnan(want["lse"][r])) and np.array_equal(got_lse[r][~fine & ~np.isnan(want["lse"][r])],
                                                                                              want["lse"][r][~fine & ~np.isnan(want["lse"][r])])
        far = np.abs(got_lse[r][fine] - want["lse"][r][fine]) - (weight[fine] + 2 * n * U + 4 * U * np.abs(want["lse"][r][fine]) + 4 * U)
        assert (far <= 0).all(), (r, n, far)
        known = np.isfinite(want["out"][r])
        assert np.array_equal(np.isnan(got[r]), ~known)
        bound = step * np.abs(want["out"][r]) + 2 * (weight[:, None] + step + 2 * n * U) * want["mass"][r] + 1e-30
        far = np.abs(got[r][known] - want["out"][r][known]) - bound[known]
        assert (far <= 0).all(), (r, n, far.max())


HEADS = [(2, 1, 64), (14, 2, 64), (28, 4, 128), (8, 8, 128), (32, 1, 128), (33, 3, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_one_token_of_every_request(hq, hkv, d, dtype):
    attn_case(hq, hkv, d, dtype, 16, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 500], [1] * 13)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 512])
def test_pages_of_every_size(page, dtype):
    attn_case(14, 2, 64, dtype, page, [1, 600, 511, 513, 300], [1, 1, 1, 1, 1], seed=page)
    attn_case(4, 1, 128, dtype, page, [1100, 40], [3, 5], [20, 0], [100, 17], seed=page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (14, 2, 64), (3, 3, 64)])
def test_questions_of_several_tokens(hq, hkv, d, dtype):
    attn_case(hq, hkv, d, dtype, 32, [70, 1, 300, 129, 33], [7, 1, 40, 129, 2])
    attn_case(hq, hkv, d, dtype, 64, [700, 300], [130, 64], [3, 0], [65, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_sinks_and_rows_that_see_nothing(dtype):
    n = 9
    want = attn_case(8, 2, 128, dtype, 16, [200] * n, [1, 2, 3, 1, 2, 3, 1, 20, 40], sink=[0, 1, 16, 17, 300, 5, -3, 0, 90],
                     window=[0, 0, 1, 16, 33, 1000, 0, 7, 2 ** 31 - 1])
    assert (want["keys"][[0, 12]] == 0).all()
    # a window without sinks, sinks without a window
    attn_case(8, 2, 128, dtype, 16, [200, 90], [2, 5], window=[10, 3])
    attn_case(8, 2, 128, dtype, 16, [200, 90], [2, 5], sink=[10, 3])
    # a request with more rows than tokens: the first ones see nothing
    want = attn_case(14, 2, 64, dtype, 16, [3, 0, 20], [5, 2, 30])
    assert (want["keys"][[0, 1, 5, 6, 7]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_requests_beside_short_ones(dtype):
    attn_case(7, 1, 128, dtype, 16, [5000, 3, 1700, 64, 1], [1] * 5)
    attn_case(7, 1, 128, dtype, 64, [4100, 900], [1, 1], [100, 0], [2000, 64])
    attn_case(5, 1, 64, dtype, 128, [3500], [9])


def test_many_requests():
    rng = np.random.default_rng(6)
    attn_case(4, 2, 64, "bf16", 16, rng.integers(1, 60, 300).tolist(), [1] * 300)
    attn_case(2, 1, 64, "f32", 16, rng.integers(0, 40, 1100).tolist(), rng.integers(0, 3, 1100).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_maps(dtype):
    attn_case(6, 3, 64, dtype, 16, [50, 200], [1, 4], kv_of_q=[2, 0, 2, 2, 0, 2])  # uneven, one KV head without queries
    attn_case(8, 2, 128, dtype, 32, [300, 31], [1, 1], kv_of_q=[1, 0, 0, 1, 1, 0, 1, 0])
    attn_case(40, 2, 64, dtype, 32, [100, 31], [1, 2], kv_of_q=[1] * 39 + [0], scale=0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    """Weights of one or two keys, maxima that come late."""
    attn_case(8, 2, 128, dtype, 16, [400, 77], [1, 6], q_scale=12.0)
    attn_case(2, 1, 64, dtype, 16, [1500], [1], scale=6.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_padded_batch(dtype):
    """Rows [request][3] of which some are not used, in another order than the requests: they stay as they were."""
    attn_case(4, 2, 64, dtype, 16, [40, 0, 17, 90], [2, 0, 3, 1], order=[9, 6, 0, 3])

    def short(a):  # rows that end behind the tensors
        a["num_rows"] = 11
        a["row_len"][2] = 8
        a["row_start"][:] = [9, 6, 5, -1]
    attn_case(4, 2, 64, dtype, 16, [40, 0, 17, 90], [2, 0, 3, 1], order=[9, 6, 0, 3], edit=short)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1, 1, 1], [1, 40, 3]])
def test_bad_pages_and_lengths(rows, dtype):
    def edit(a):
        a["table"][0, 2] = -1
        a["table"][1, [0, 3]] = [len(a["pool"]), 2 ** 31 - 1]
        a["table"][2, :] = -(2 ** 31)
        a["seq_len"][0] = 2 ** 31 - 1  # as long as the table is wide
    attn_case(8, 2, 64, dtype, 16, [96, 90, 33], rows, edit=edit)

    def negative(a):
        a["seq_len"][:] = [-5, 0, 12]
        a["row_len"][1] = -(2 ** 31)
    attn_case(8, 2, 64, dtype, 16, [96, 90, 33], rows, edit=negative)


@pytest.mark.parametrize("dtype,rows,wide", [("bf16", [1, 1], None), ("f32", [1, 1], None), ("bf16", [3, 40], None), ("f32", [3, 40], None),
                                             ("bf16", [3, 40], "128"), ("bf16", [19, 47], "128"), ("bf16", [6, 7], "32"), ("f32", [19, 47], "32")])
def test_blocks_without_a_value(dtype, rows, wide):
    """NaN blocks reach the rows that see them: a key's all of the row, a value's its 32 elements; masked ones nobody."""
    def nan_at(a, s, token, which, block):
        slot = a["table"][s, token // 16] * 16 + token % 16
        a["pool"][slot // 16, 0, 0, 16 * 128 + (block * 16 + token % 16) * 2 + which] = 255

    def value(a):
        nan_at(a, 0, 60, 1, 2)
        nan_at(a, 1, 5, 1, 0)

    def key(a):
        nan_at(a, 0, 100, 0, 1)

    def hidden(a):
        nan_at(a, 0, 30, 1, 3)
        nan_at(a, 0, 31, 0, 3)
    lengths = [120, 50]
    first = [120 - rows[0], 50 - rows[1]]
    want = attn_case(4, 1, 128, dtype, 16, lengths, rows, edit=value, wide=wide)
    assert np.isnan(want["out"][0][:, 64:96]).all() and np.isfinite(want["out"][0][:, :64]).all()
    want = attn_case(4, 1, 128, dtype, 16, lengths, rows, edit=key, wide=wide)
    assert np.isnan(want["out"][0]).all() and np.isfinite(want["out"][rows[0]:]).all()
    want = attn_case(4, 1, 128, dtype, 16, lengths, rows, sink=[29, 0], window=[first[0] - 31, -1], edit=hidden, wide=wide)
    assert np.isfinite(want["out"]).all()
    # a value that some rows of a question see and earlier ones do not
    want = attn_case(4, 1, 128, dtype, 16, lengths, rows, edit=lambda a: nan_at(a, 1, 49, 1, 1), wide=wide)
    assert np.isnan(want["out"][-1][:, 32:64]).all() and np.isfinite(want["out"][:-1]).all()


@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (14, 2, 64), (3, 3, 64), (8, 8, 128), (33, 3, 64)])
@pytest.mark.parametrize("page", [16, 64, 512])
def test_many_rows(page, hq, hkv, d):
    attn_case(hq, hkv, d, "bf16", page, [1500], [128], wide="128")
    attn_case(hq, hkv, d, "bf16", page, [200, 119, 300, 135], [100, 119, 161, 129], wide="128")


def test_many_rows_with_masks():
    n = [200, 333, 64, 500, 90]
    attn_case(8, 2, 128, "bf16", 16, n, [40, 64, 70, 33, 80], sink=[0, 16, 300, 5, -3], window=[0, 1, 16, 100, 2 ** 31 - 1], wide="128")
    attn_case(8, 2, 128, "bf16", 16, n, [40, 64, 60, 33, 80], window=[-1, 50, 64, 65, 63], wide="128")
    attn_case(14, 2, 64, "bf16", 32, [2500, 700], [77, 130], sink=[100, 17], window=[600, 1], wide="128")
    want = attn_case(14, 2, 64, "bf16", 16, [30, 0, 320], [150, 2, 250], wide="128")  # more rows than tokens
    assert (want["keys"][:120] == 0).all() and (want["keys"][150:152] == 0).all() and want["keys"][120] == 1


def test_many_rows_of_mapped_heads():
    attn_case(6, 3, 64, "bf16", 16, [150, 600], [100, 200], kv_of_q=[2, 0, 2, 2, 0, 2], wide="128")
    attn_case(8, 2, 128, "bf16", 32, [300, 131], [60, 40], kv_of_q=[1, 0, 0, 1, 1, 0, 1, 0], wide="128")
    attn_case(40, 2, 64, "bf16", 32, [100, 31], [20, 12], kv_of_q=[1] * 39 + [0], scale=0.2, wide="128")


def test_many_rows_with_scores_far_apart():
    attn_case(8, 2, 128, "bf16", 16, [400, 77], [60, 70], q_scale=12.0, wide="128")
    attn_case(2, 1, 64, "bf16", 16, [1500], [127], scale=6.0, wide="128")


def test_many_rows_of_a_padded_batch():
    attn_case(4, 2, 64, "bf16", 16, [140, 0, 117, 190], [120, 0, 101, 77], order=[380, 360, 0, 200], wide="128")

    def short(a):  # rows that end behind the tensors
        a["num_rows"] = 499
        a["row_start"][:] = [380, 360, 90, -1]
    attn_case(4, 2, 64, "bf16", 16, [140, 0, 117, 190], [120, 0, 101, 77], order=[380, 360, 0, 200], edit=short, wide="128")


def test_many_rows_with_bad_pages_and_lengths():
    def edit(a):
        a["table"][0, 2] = -1
        a["table"][1, [0, 3]] = [len(a["pool"]), 2 ** 31 - 1]
        a["table"][2, :] = -(2 ** 31)
        a["seq_len"][0] = 2 ** 31 - 1  # as long as the table is wide
    attn_case(8, 2, 128, "bf16", 16, [96, 90, 33], [40, 90, 60], edit=edit, wide="128")

    def negative(a):
        a["seq_len"][:] = [-5, 0, 212]
        a["row_len"][1] = -(2 ** 31)
    attn_case(8, 2, 128, "bf16", 16, [96, 90, 212], [40, 90, 60], edit=negative, wide="128")


def test_many_requests_with_many_rows():
    rng = np.random.default_rng(6)
    attn_case(4, 1, 128, "bf16", 16, rng.integers(1, 100, 150).tolist(), rng.integers(20, 40, 150).tolist(), wide="128")

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (14, 2, 64), (32, 1, 128), (24, 3, 64)])
def test_tiles_of_32(hq, hkv, d, dtype):
    attn_case(hq, hkv, d, dtype, 64, [700, 31, 300, 33], [2, 2, 1, 3] if hkv == 1 else [3, 5, 1, 8], wide="32")
    attn_case(hq, hkv, d, dtype, 512, [1500], [31 * hkv // hq + 2], wide="32")
    if dtype == "f32":
        attn_case(hq, hkv, d, dtype, 64, [300, 119], [60, 119], wide="32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_32_with_masks(dtype):
    n = [200, 333, 64, 500, 90]
    attn_case(8, 2, 128, dtype, 64, n, [4, 9, 12, 10, 17], sink=[0, 16, 300, 5, -3], window=[0, 1, 16, 100, 2 ** 31 - 1], wide="32")
    attn_case(14, 2, 64, dtype, 64, [900, 700], [9, 5], sink=[100, 17], window=[600, 1], wide="32")
    want = attn_case(14, 2, 64, dtype, 64, [3, 0, 320], [15, 2, 5], wide="32")  # more rows than tokens
    assert (want["keys"][:12] == 0).all() and want["keys"][12] == 1
    attn_case(6, 3, 64, dtype, 64, [50, 200], [13, 9], kv_of_q=[2, 0, 2, 2, 0, 2], wide="32")
    attn_case(8, 2, 128, dtype, 64, [400, 77], [6, 7], q_scale=12.0, wide="32")

    def short(a):  # rows that end behind the tensors
        a["num_rows"] = 40
        a["row_start"][:] = [30, 20, 10, -1]
    attn_case(8, 2, 64, dtype, 64, [40, 0, 17, 90], [11, 0, 6, 7], order=[30, 20, 0, 10], edit=short, wide="32")

    def bad(a):
        a["table"][0, 2] = -1
        a["table"][1, [0, 3]] = [len(a["pool"]), 2 ** 31 - 1]
        a["seq_len"][2] = -5
    attn_case(8, 2, 64, dtype, 16, [96, 90, 33], [6, 8, 7], edit=bad, wide="32")



@pytest.mark.parametrize("width,rows", [(64, 3), (8192, 3), (8192, 70), (1 << 20, 9)])
def test_requests_that_name_the_same_rows_write_nothing_else(width, rows):
    """Not allowed, and their rows hold no result; but nothing outside the tensors and the workspace is written."""
    heads, n, page = P.Heads(8, 2, 128, "bf16"), 700, 64
    pool = torch.zeros((4, 2, 4, 17 * 128), dtype=torch.uint8, device=DEV)
    cache = P.KvCache(pool, torch.zeros((n, width // page), dtype=torch.int32, device=DEV), page)
    need = P.pevlm_cache_attn_workspace_bytes(heads, n, rows)
    block = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device=DEV)
    around = torch.full((rows + 64, 8, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((rows + 64, 8), 5.0, device=DEV)
    q = torch.randn((rows, 8, 128), device=DEV).bfloat16()
    for per in (rows, 1):
        P.pevlm_cache_attn_kv4(q, around[32:32 + rows], cache, heads, i32([0] * n), i32([per] * n), i32([2 ** 31 - 1] * n), lse=lse[32:32 + rows],
                               workspace=block[:need])
    torch.cuda.synchronize()
    assert (block[need:] == 77).all() and (around[:32] == 5).all() and (around[32 + rows:] == 5).all()
    assert (lse[:32] == 5).all() and (lse[32 + rows:] == 5).all()


def test_lengths_of_many_millions():
    """Every page of the table is the same one: the rows before the last see n copies of its tokens, so out is that of one page and lse more by log(n)."""
    page, width = 4096, 1 << 13  # 2^25 tokens
    rng = np.random.default_rng(3)
    for rows, d in ((1, 128), (1, 64), (130, 128), (130, 64)):
        pool = np.zeros((1, 1, page // 16, 17 * d), np.uint8)
        O.put(pool, np.arange(page), rng.standard_normal((page, 1, d)), rng.standard_normal((page, 1, d)))
        q, q64 = rounded(rng.standard_normal((rows, 1, d)), "bf16")
        heads = P.Heads(1, 1, d, "bf16")
        cache = P.KvCache(torch.from_numpy(pool).to(DEV), torch.zeros((1, width), dtype=torch.int32, device=DEV), page)
        out, lse = torch.empty_like(q), torch.empty((rows, 1), device=DEV)
        P.pevlm_cache_attn_kv4(q, out, cache, heads, i32([0]), i32([rows]), i32([page * width]), lse=lse)
        last = O.attention(q64[-1:], pool, np.array([[0]]), [0], [0], [1], [page])
        got, got_lse = out[-1:].double().cpu().numpy(), lse[-1:].double().cpu().numpy()
        n = page * width / 512 * U  # an item's tokens, of at least 512 items: its sums in fp32 are within n of them, relative to what they add up
        assert (np.abs(got_lse - last["lse"] - np.log(width)) <= 2 * n + 1e-5).all()
        assert (np.abs(got - last["out"]) <= 2.0 ** -8 * np.abs(last["out"]) + (2.0 ** -8 + 8 * n) * last["mass"]).all()


def test_a_pool_beyond_32_bits():
    """Pages at the end of a pool of 5 GiB."""
    heads, page = P.Heads(28, 4, 128, "bf16"), 256
    pages = (5 << 30) // (page * 4 * 136)
    pool = torch.empty((pages, 4, 16, 17 * 128), dtype=torch.uint8, device=DEV)
    assert pool.numel() > 1 << 32
    rng = np.random.default_rng(9)
    k, k64 = rounded(rng.standard_normal((600, 4, 128)), "bf16")
    v, v64 = rounded(rng.standard_normal((600, 4, 128)), "bf16")
    table = np.array([[pages - 1, 3, pages // 2 + 7]])
    slots = table[0, np.arange(600) // page] * page + np.arange(600) % page
    cache = P.KvCache(pool, i32(np.pad(table, ((0, 0), (0, 13)))), page)
    P.pevlm_cache_store_kv4(k, v, i32(slots), cache, heads)
    back = torch.empty_like(k), torch.empty_like(v)
    P.pevlm_cache_load_kv4(*back, i32(slots), cache, heads)
    assert np.array_equal(back[0].double().cpu().numpy(), O.values(*O.encode(k64))) and np.array_equal(back[1].double().cpu().numpy(), O.values(*O.encode(v64)))
    small = np.zeros((3, 4, 16, 17 * 128), np.uint8)
    O.put(small, np.arange(600), k64, v64)
    for rows in (1, 40):
        q, q64 = rounded(rng.standard_normal((rows, 28, 128)), "bf16")
        out, lse = torch.full_like(q, 5.0), torch.full((rows, 28), 5.0, device=DEV)
        P.pevlm_cache_attn_kv4(q, out, cache, heads, i32([0]), i32([rows]), i32([600]), lse=lse)
        hold(out, lse, O.attention(q64, small, np.array([[0, 1, 2]]), [h // 7 for h in range(28)], [0], [rows], [600]), "bf16", 128)


# ------------------------------------------------------------------------------------------ the calls together
class Server:
    """A program's own state: a prompt goes through the prefill calls, then tokens are generated against the cache."""

    def __init__(self, seqs, dtype="bf16", hq=8, hkv=2, d=128, page=32, pages=64, width=40, steps=8):
        self.w = W.Workload("served", 77, dtype, hq, hkv, d, 1.0e6, seqs, 0.5)
        self.lay, self.heads = P.Layout.from_seqs(seqs), P.Heads(hq, hkv, d, dtype)
        n = self.n = len(seqs)
        self.cache = P.KvCache(P.KvCache.new_pool(self.heads, pages, page, DEV), i32(np.full((n, width), -1)), page)
        self.free, self.num_free = torch.randperm(pages, device=DEV).int(), i32([pages])
        self.seq_len, self.row_start, self.row_len = i32([0] * n), i32([0] * n), i32([0] * n)
        self.ws = torch.empty(P.pevlm_cache_attn_workspace_bytes(self.heads, n, n), dtype=torch.uint8, device=DEV)
        self.ws_slots = torch.empty(P.pevlm_cache_slots_workspace_bytes(n), dtype=torch.uint8, device=DEV)

    def slots(self, new_len, rows):
        slot_map, pos = i32([0] * rows), torch.zeros((3, rows), dtype=torch.int32, device=DEV)
        self.slots_into(new_len, slot_map, pos)
        return slot_map, pos

    def slots_into(self, new_len, slot_map, pos):
        P.pevlm_cache_slots(self.cache, self.seq_len, new_len, self.free, self.num_free, self.seq_len, self.num_free, self.row_start, self.row_len,
                            slot_map, pos_ids=pos, workspace=self.ws_slots)

    def prefill(self):
        data = W.generate(self.w)
        to = lambda a: (torch.from_numpy(a.view(np.int16)).to(DEV).view(torch.bfloat16) if a.dtype == np.uint16 else torch.from_numpy(a).to(DEV))  # noqa: E731
        q, k, v = (to(data[x]) for x in "qkv")
        out = torch.empty_like(q)
        P.pevlm_rope_seq(q, k, self.lay, self.heads, self.w.rope_base)
        P.pevlm_block_prefill_attn(q, k, v, out, self.lay, self.heads)
        P.pevlm_query_attn(q, k, v, out, self.lay, self.heads)
        slot_map, pos = self.slots(i32(np.diff(self.lay.cu)), self.lay.total_tokens)
        P.pevlm_cache_store_kv4(k, v, slot_map, self.cache, self.heads)
        return q, k, v, out, slot_map, pos

    def step(self, q, k, v, out, lse, slot_map, pos):
        """One layer of one step: q, k, v of a token of every request, in place."""
        self.slots_into(None, slot_map, pos)
        P.pevlm_rope_mrope(q, k, self.n, self.heads, self.w.rope_base, pos, [self.heads.head_dim // 2, 0, 0])
        P.pevlm_cache_store_kv4(k, v, slot_map, self.cache, self.heads)
        P.pevlm_cache_attn_kv4(q, out, self.cache, self.heads, self.row_start, self.row_len, self.seq_len, lse=lse, workspace=self.ws)

    def want(self, q):
        args = [x.cpu().numpy() for x in (self.row_start, self.row_len, self.seq_len)]
        g = self.heads.n_q_heads // self.heads.n_kv_heads
        return O.attention(q.double().cpu().numpy(), self.cache.pool.cpu().numpy(), self.cache.block_table.cpu().numpy().astype(np.int64),
                           [h // g for h in range(self.heads.n_q_heads)], *args)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_and_its_answer(dtype):
    """Prefill, the prompt's K and V into the cache, then three tokens of every request."""
    seqs = [(40, 64, 300, 9), (3, 16, 77, 1), (0, 8, 31, 0)]
    srv = Server(seqs, dtype)
    q, k, v, out, slot_map, pos = srv.prefill()
    lens = np.diff(srv.lay.cu)
    assert srv.seq_len.tolist() == lens.tolist() and srv.num_free.item() == 64 - sum(-(-n // 32) for n in lens)
    assert pos[1].cpu().tolist() == [t for n in lens for t in range(n)]
    back = torch.empty_like(k), torch.empty_like(v)
    P.pevlm_cache_load_kv4(*back, slot_map, srv.cache, srv.heads)
    for x, y in zip(back, (k, v)):
        assert np.array_equal(x.double().cpu().numpy(), O.values(*O.encode(y.double().cpu().numpy())))
    gen = torch.Generator(device=DEV).manual_seed(5)
    rows = lambda h: torch.randn((3, h, 128), generator=gen, device=DEV).to(DTYPES[dtype])  # noqa: E731
    slot_map, pos = i32([0] * 3), torch.zeros((3, 3), dtype=torch.int32, device=DEV)
    for t in range(3):
        q, k, v = rows(8), rows(2), rows(2)
        plain_k, out, lse = k.clone(), torch.empty_like(q), torch.empty((3, 8), device=DEV)
        srv.step(q, k, v, out, lse, slot_map, pos)
        assert srv.seq_len.tolist() == (lens + t + 1).tolist()
        # the keys were turned at their tokens' places
        lay = P.Layout.from_seqs([(1, 1, 0, 0)] * 3)
        P.pevlm_rope_seq(None, plain_k, lay, srv.heads, 1.0e6, pos_offset=(lens + t).tolist())
        assert torch.equal(plain_k, k)
        hold(out, lse, srv.want(q), dtype, 128)


def test_a_step_that_is_captured_and_replayed():
    """The lengths grow on the GPU from replay to replay; pages are taken; eager work of the program in between."""
    servers = [Server([(16, 16, 40, 3), (0, 16, 9, 2)], page=16, pages=80) for _ in range(2)]
    servers[1].free.copy_(servers[0].free)
    for s in servers:
        s.prefill()
    gen = torch.Generator(device=DEV).manual_seed(6)
    shapes = (8, 2, 2)
    bufs = [torch.zeros((2, h, 128), dtype=torch.bfloat16, device=DEV) for h in shapes]
    out, lse = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 8), device=DEV)
    slot_map, pos = i32([0] * 2), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        servers[0].step(*bufs, out, lse, slot_map, pos)
    for t in range(20):
        new = [torch.randn((2, h, 128), generator=gen, device=DEV).bfloat16() for h in shapes]
        for b, x in zip(bufs, new):
            b.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
        e_slots, e_pos = torch.zeros_like(slot_map), torch.zeros_like(pos)
        servers[1].step(*new, e_out, e_lse, e_slots, e_pos)
        torch.cuda.synchronize()
        assert torch.equal(out, e_out) and torch.equal(lse, e_lse) and torch.equal(slot_map, e_slots) and torch.equal(pos, e_pos), t
        assert torch.equal(servers[0].seq_len, servers[1].seq_len) and torch.equal(servers[0].cache.pool, servers[1].cache.pool)
        if t in (0, 7, 19):
            hold(out, lse, servers[0].want(bufs[0]), "bf16", 128)


def test_two_streams_at_once():
    rng = np.random.default_rng(4)
    heads = P.Heads(28, 4, 128, "bf16")
    table, pages = pages_for([3000, 700], 32, rng)
    pool = torch.from_numpy(np.concatenate([rng.integers(0, 256, (pages, 4, 2, 2048)), rng.integers(120, 130, (pages, 4, 2, 128))], -1).astype(np.uint8)).to(DEV)
    cache = P.KvCache(pool, i32(table), 32)
    args = i32([0, 1]), i32([1, 1]), i32([3000, 700])
    qs = [torch.randn((2, 28, 128), device=DEV).bfloat16() for _ in range(2)]
    want = [torch.empty_like(q) for q in qs]
    for q, o in zip(qs, want):
        P.pevlm_cache_attn_kv4(q, o, cache, heads, *args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    outs = [[torch.empty_like(q) for _ in range(20)] for q in qs]
    spaces = [torch.empty(P.pevlm_cache_attn_workspace_bytes(heads, 2, 2), dtype=torch.uint8, device=DEV) for _ in qs]
    torch.cuda.synchronize()
    for t in range(20):
        for q, o, ws, s in zip(qs, outs, spaces, streams):
            P.pevlm_cache_attn_kv4(q, o[t], cache, heads, *args, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x, w) for x in o)
