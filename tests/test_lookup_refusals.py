"""What the lookup calls refuse, before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1711_06505_amd import ams

OK, NULL, SIZE, DTYPE, DIMS, WS = range(6)
FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first


def test_lookup_host_errors():
    lib = ams.load()
    f = [0, 12, 1.0, -1, FAKE, 100, FAKE, 50, 12, FAKE, 12, None]
    for at, value, code in [(0, 2, DTYPE), (0, -1, DTYPE), (1, 0, DIMS), (1, 65537, DIMS), (4, None, NULL),
                            (5, -1, SIZE), (5, 2 ** 30, SIZE), (6, None, NULL), (7, -1, SIZE), (8, 11, SIZE),
                            (9, None, NULL), (10, 11, SIZE)]:
        a = list(f)
        a[at] = value
        assert lib.ams_lookup_fwd(*a) == code, (at, value)
    a = list(f)
    a[5] = 0
    assert lib.ams_lookup_fwd(*a) == OK
    b = [0, 12, 1.0, -1, 100, FAKE, FAKE, FAKE, FAKE, FAKE, 100, FAKE, 12, FAKE, FAKE, 16, None]
    assert lib.ams_lookup_bwd(*b) == WS
    for at, value, code in [(0, 2, DTYPE), (1, 0, DIMS), (4, -1, SIZE), (10, -1, SIZE), (12, 11, SIZE),
                            *[(i, None, NULL) for i in (5, 6, 7, 8, 9, 11, 13, 14)]]:
        a = list(b)
        a[at] = value
        assert lib.ams_lookup_bwd(*a) == code, (at, value)
    a = list(b)
    a[4] = 0
    assert lib.ams_lookup_bwd(*a) == OK


def test_lookup_workspace_serves_smaller_calls():
    for D in (1, 12, 2048):
        ws = [ams.ams_lookup_workspace(n, D) for n in [*range(0, 2000, 37), 131_000, 131_071, 131_072, 131_073,
                                                       140_000, 600_000, 2 ** 30 - 1]]
        assert all(b >= a for a, b in zip(ws, ws[1:])), D
    assert ams.ams_lookup_workspace(-1, 4) == ams.ams_lookup_workspace(2 ** 30, 4) == 0
    assert ams.ams_lookup_workspace(10, 0) == ams.ams_lookup_workspace(10, 65537) == 0


def test_lookup_binding_refusals():
    ids = torch.zeros(4, dtype=torch.int32)
    T, out = torch.zeros((5, 8)), torch.zeros((4, 8))
    with pytest.raises(ValueError, match="not on a GPU"):
        ams.ams_lookup_fwd(ids, T, out)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ams.ams_lookup_fwd(ids, T.half(), out)
    with pytest.raises(ValueError, match="ids must be"):
        ams.ams_lookup_fwd(ids.long(), T, out)
    d = [torch.zeros(4, dtype=torch.int32) for _ in range(3)]
    off, nu = torch.zeros(5, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="a row of dout must be contiguous"):
        ams.ams_lookup_bwd(*d, off, nu, 4, torch.zeros((8, 4)).t(), torch.zeros((4, 8)), torch.zeros(1))
    with pytest.raises(ValueError, match="rows of dout overlap"):
        ams.ams_lookup_bwd(*d, off, nu, 4, torch.zeros((1, 8)).expand(4, 8), torch.zeros((4, 8)), torch.zeros(1))
