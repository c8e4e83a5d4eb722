"""What the cache calls refuse, before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1711_06505_amd import ams

OK, NULL, SIZE, DTYPE, DIMS, WS = range(6)
FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
R = ctypes.byref
BAD = [((0, 16, 16, 4, 10), DIMS), ((2, 0, 16, 4, 10), DIMS), ((2, 129, 16, 4, 10), DIMS), ((2, 16, 8, 4, 10), DIMS),
       ((2, 16, 48, 4, 10), DIMS), ((2, 16, 256, 4, 10), DIMS), ((2, 16, 0, 4, 10), DIMS), ((2, 16, 16, 0, 10), SIZE),
       ((2, 16, 16, 4, 0), SIZE), ((2, 16, 128, 2 ** 24, 10), SIZE), ((2, 16, 16, 4, 2 ** 31), SIZE)]


def test_write_host_errors():
    lib = ams.load()
    good = ams.make_cache(2, 16, 16, 4, 10)
    w = [R(good), 0, 3, FAKE, 5, FAKE, FAKE, FAKE, 32, FAKE, 32, FAKE, FAKE, FAKE, FAKE, None, None]
    for at, value, code in [(0, None, NULL), (1, 2, DTYPE), (2, -1, SIZE), (4, -1, SIZE), (4, 2 ** 31, SIZE),
                            (8, 31, SIZE), (10, 31, SIZE), *[(i, None, NULL) for i in (3, 5, 6, 7, 9, 11, 12, 13, 14)]]:
        a = list(w)
        a[at] = value
        assert lib.ams_cache_write(*a) == code, (at, value)
    for bad, code in BAD:
        assert lib.ams_cache_write(R(ams.make_cache(*bad)), *w[1:]) == code, bad
    for at in (2, 4):
        a = list(w)
        a[at] = 0
        assert lib.ams_cache_write(*a) == OK


def test_attn_host_errors():
    lib = ams.load()
    attn, cache = ams.make_attn(4, 2, 16, "f32"), ams.make_cache(2, 16, 16, 4, 10)
    f = [R(attn), R(cache), 3, FAKE, 5, FAKE, FAKE, FAKE, 64, FAKE, FAKE, FAKE, FAKE, FAKE, 64, None, FAKE, 16, None]
    assert lib.ams_cache_attn(*f) == WS
    for at, value, code in [(0, None, NULL), (1, None, NULL), (2, -1, SIZE), (4, -1, SIZE), (4, 2 ** 30, SIZE),
                            (8, 63, SIZE), (14, 63, SIZE),
                            *[(i, None, NULL) for i in (3, 5, 6, 7, 9, 10, 11, 12, 13, 16)]]:
        a = list(f)
        a[at] = value
        assert lib.ams_cache_attn(*a) == code, (at, value)
    for bad, code in BAD:
        assert lib.ams_cache_attn(R(attn), R(ams.make_cache(*bad)), *f[2:]) == code, bad
        assert ams.ams_cache_workspace(attn, ams.make_cache(*bad), 3, 5) == 0
    for bad, code in [(ams.ams_attn(2, 4, 2, 16, 1.0), DTYPE), (ams.make_attn(4, 1, 16), DIMS),
                      (ams.make_attn(4, 2, 12), DIMS), (ams.make_attn(5, 2, 16), DIMS)]:
        assert lib.ams_cache_attn(R(bad), *f[1:]) == code
    a = list(f)
    a[4] = 0
    assert lib.ams_cache_attn(*a) == OK


def test_binding_refusals():
    cache = ams.make_cache(2, 16, 16, 2, 4)
    off, start = torch.tensor([0, 1], dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    table = torch.zeros((1, 2), dtype=torch.int32)
    k = torch.zeros((1, 2, 16))
    codes, scale = torch.zeros((4, 2, 16, 16), dtype=torch.uint8), torch.ones((4, 2))
    pool = (codes, scale, codes.clone(), scale.clone())
    with pytest.raises(ValueError, match="not on a GPU"):
        ams.ams_cache_write(cache, off, start, table, k, k, *pool)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ams.ams_cache_write(cache, off, start, table, k.half(), k, *pool)
    with pytest.raises(ValueError, match="k and v have"):
        ams.ams_cache_write(cache, off, start, table, k, torch.zeros((2, 2, 16)), *pool)
    with pytest.raises(ams.AmsError, match="DIMS"):
        ams.ams_cache_attn(ams.make_attn(4, 2, 12, "f32"), cache, off, start, table, torch.zeros((1, 4, 12)), *pool,
                           torch.zeros((1, 4, 12)), torch.zeros(1, dtype=torch.uint8))
    c = ams._Call("x", k)
    c.device = -1                       # the tensors'
    with pytest.raises(ValueError, match="elements"):
        ams._cache_arrays(c, cache, 1, table, codes[:3], scale, codes, scale)
    with pytest.raises(ValueError, match="page_table has"):
        ams._cache_arrays(c, cache, 2, table, *pool)
    with pytest.raises(ValueError, match="contiguous"):
        ams._cache_arrays(c, cache, 1, table, codes.transpose(2, 3), scale, codes, scale)
