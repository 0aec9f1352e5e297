"""GPU: appending to 8-bit caches with a scale per block: what is not finite, and scales that are none, code by code."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


INF, NAN = float("inf"), float("nan")


def bytes_of(k):
    import torch
    return k.view(torch.uint8)


def append(marlin, k_cache, k_scale, length, rows):
    """kv_append of rows [n, 16] (keys and values alike, one head) behind length - n tokens of one sequence on page 0; codes and scale of keys."""
    import torch
    n = len(rows)
    qkv = torch.tensor(rows, dtype=torch.float16, device="cuda").repeat(1, 3).contiguous()
    v_cache, v_scale = k_cache.clone(), k_scale.clone()
    ws = torch.zeros(marlin.attention_workspace_bytes(16), dtype=torch.uint8, device="cuda")
    pages, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    marlin.kv_append(qkv, k_cache, v_cache, pages, lengths, ws, starts=starts, k_scale=k_scale, v_scale=v_scale)
    assert marlin.read_status(ws) == 0
    assert torch.equal(k_cache.view(torch.uint8), v_cache.view(torch.uint8)) and torch.equal(k_scale.view(torch.int32), v_scale.view(torch.int32))
    return k_cache.view(torch.uint8)[0, 0].cpu().numpy(), k_scale[0, 0].cpu().numpy()


def cache_of(kind, code=0x31, scale=7.0):
    import torch
    k = torch.full((1, 1, 16, 16), code, dtype=torch.uint8, device="cuda").view(torch.int8 if kind == "int8" else torch.float8_e4m3fn)
    return k, torch.full((1, 1, 2), scale, device="cuda")


LARGEST = {"int8": (0x7f, 0x81), "e4m3": (0x7e, 0xfe)}  # plus and minus 127, 448


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_an_infinity_becomes_the_largest_code(marlin, kind):
    rows = np.zeros((2, 16))
    rows[0, :4], rows[1, 5:7] = [INF, -INF, NAN, 1.0], [INF, 0.5]
    codes, scale = append(marlin, *cache_of(kind), 2, rows)
    assert scale[0] == np.float32(1.0) * (np.float32(1) / np.float32(127 if kind == "int8" else 448)) and scale[1] == 7
    most, least = LARGEST[kind]
    assert list(codes[0, :2]) == [most, least] and codes[0, 3] == most and codes[1, 5] == most
    assert codes[0, 2] & 0x7f == (0 if kind == "int8" else 0x7f)  # a NaN stays one in e4m3 and is 0 in two's complement
    # under a scale that is there, also where nothing else is new
    rows = np.zeros((1, 16))
    rows[0, :3] = [INF, -INF, NAN]
    codes, after = append(marlin, *cache_of(kind), 3, rows)
    assert list(codes[2, :2]) == [most, least] and codes[2, 2] & 0x7f == (0 if kind == "int8" else 0x7f) and not codes[2, 3:].any()
    assert after[0] == 7 and (codes[:2] == 0x31).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [1, 3, 8])
def test_codes_are_0_where_the_largest_finite_magnitude_is_0(marlin, kind, n):
    # "where a is 0 and the block has no scale yet, s is 0 and all codes are 0, also those of infinities; a NaN stays one in e4m3"
    rows = np.zeros((n, 16))
    rows[:, 3], rows[0, 4], rows[-1, 5], rows[-1, 6] = INF, -INF, -0.0, INF
    codes, scale = append(marlin, *cache_of(kind), n, rows)
    assert scale[0] == 0 and not codes[:n].any()
    rows[:] = INF
    codes, scale = append(marlin, *cache_of(kind), n, rows)
    assert scale[0] == 0 and not codes[:n].any()
    rows[0, 9] = NAN
    codes, scale = append(marlin, *cache_of(kind), n, rows)
    assert scale[0] == 0 and codes[0, 9] & 0x7f == (0 if kind == "int8" else 0x7f)
    codes[0, 9] = 0
    assert not codes[:n].any()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("scale", [0.0, -1.0, NAN, INF, -INF])
@pytest.mark.parametrize("new", [0.0, 2.0, INF])
def test_a_scale_that_is_not_finite_and_above_0_stands_for_codes_of_0(marlin, kind, scale, new):
    # "the codes of its earlier tokens become 0, those of NaN too"
    k, s = cache_of(kind, 0x7f, scale)
    bytes_of(k)[0, 0, 1] = 0xc5
    rows = np.full((2, 16), new)
    codes, after = append(marlin, k, s, 5, rows)
    assert not codes[:3].any() and (codes[5:] == 0x7f).all()
    assert after[0] == (np.float32(2) * (np.float32(1) / np.float32(127 if kind == "int8" else 448)) if new == 2 else 0)
    assert (codes[3:5] == (LARGEST[kind][0] if new == 2 else 0)).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_scale_that_doubles_more_often_than_fp32_has_powers(marlin, kind):
    # 2^-149 doubled until 60000 / L fits: codes that are there vanish, but a NaN stays one
    k, s = cache_of(kind, 0x7e, 2.0 ** -149)
    bytes_of(k)[0, 0, 0, 0] = 0x7f
    codes, after = append(marlin, k, s, 2, np.full((1, 16), 60000.0))
    assert np.isfinite(after[0]) and after[0] >= np.float32(60000) * (np.float32(1) / np.float32(127 if kind == "int8" else 448))
    assert codes[0, 0] == (0 if kind == "int8" else 0x7f) and not (codes[0, 1:] & 0x7f).any()
