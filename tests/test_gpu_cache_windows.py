"""Cache attention where a request has more rows than tokens and its window ends near 2^31: the edge of a row before the first token
does not fit 32 bits, and the rows behind it see what they see."""
import pytest

from test_gpu_cache import attn_case

pytestmark = pytest.mark.gpu
TOP = 2 ** 31 - 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sink", [None, [0, 2, 400, 1, -7, 16]])
def test_tiles_of_16(dtype, sink):
    held, rows = [3, 3, 5, 40, 0, 17], [6, 5, 30, 60, 4, 20]
    want = attn_case(8, 2, 64, dtype, 16, held, rows, sink, [TOP] * 6)
    assert want["keys"][:6].tolist() == [0, 0, 0, 1, 2, 3]
    # rows - tokens is 3, 2, 25, 20, 4, 3: the edge wraps, or is the last number that does not
    attn_case(8, 2, 128, dtype, 16, held, rows, sink, [TOP - 1, TOP - 1, TOP - 24, TOP - 18, TOP - 3, TOP - 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_32(dtype):
    attn_case(14, 2, 64, dtype, 64, [3, 20, 320], [9, 25, 5], [1, 0, 5], [TOP] * 3, wide="32")
    attn_case(8, 2, 64, dtype, 64, [3, 20, 1], [6, 23, 9], None, [TOP, TOP - 1, TOP - 3], wide="32")


def test_tiles_of_128():
    for hq, hkv, d, rows in ((8, 2, 128, [31, 40, 33]), (14, 2, 64, [150, 29, 20])):
        attn_case(hq, hkv, d, "bf16", 16, [30 if rows[0] < 100 else 120, 25, 3], rows, [7, 0, 1], [TOP] * 3, wide="128")
        attn_case(hq, hkv, d, "bf16", 16, [rows[0] - 3, 20, 1], rows, None, [TOP, TOP - 5, TOP - 1], wide="128")
