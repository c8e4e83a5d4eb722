"""What the cross attention calls refuse, before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1711_06505_amd import ams

OK, NULL, SIZE, DTYPE, DIMS, WS = range(6)
FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first


def test_host_errors():
    lib = ams.load()
    good = ams.make_attn(4, 2, 16, "f32")
    R = ctypes.byref
    f = [R(good), 3, FAKE, 10, FAKE, 50, FAKE, 64, FAKE, 32, FAKE, 32, None, FAKE, 64, None, FAKE, 16, None]
    assert lib.ams_xattn_fwd(*f) == WS
    b = [*f[:13], FAKE, 64, FAKE, FAKE, 64, FAKE, 64, FAKE, 32, FAKE, 32, FAKE, 16, None]
    assert lib.ams_xattn_bwd(*b) == WS
    for call, args in ((lib.ams_xattn_fwd, f), (lib.ams_xattn_bwd, b)):
        for at, value, code in [(0, None, NULL), (1, -1, SIZE), (2, None, NULL), (3, -1, SIZE), (4, None, NULL),
                                (5, -1, SIZE), (5, 2 ** 31, SIZE), (6, None, NULL), (7, 63, SIZE), (8, None, NULL),
                                (9, 31, SIZE), (10, None, NULL), (11, 31, SIZE), (13, None, NULL), (14, 63, SIZE),
                                (3, 2 ** 31 // 2, SIZE)]:
            a = list(args)
            a[at] = value
            assert call(*a) == code, (at, value)
        for bad, code in [((4, 2, 16, "f32", 9), DTYPE), ((4, 3, 16), DIMS), ((0, 1, 16), DIMS), ((4, 0, 16), DIMS),
                          ((4, 2, 0), DIMS), ((4, 2, 129), DIMS), ((4097, 4097, 1), DIMS), ((-4, -2, 16), DIMS)]:
            s = ams.ams_attn(bad[4] if len(bad) > 4 else 0, bad[0], bad[1], bad[2], 1.0)
            assert call(*[R(s), *args[1:]]) == code, bad
            assert ams.ams_xattn_workspace(s, 3, 10, 50) == 0
        a = list(args)
        a[1] = 0
        assert call(*a) == OK
    for at in (15, 16, 18, 20, 22, 24):
        a = list(b)
        a[at] = None
        assert lib.ams_xattn_bwd(*a) == NULL, at
    for at, value in ((17, 63), (19, 63), (21, 31), (23, 31)):
        a = list(b)
        a[at] = value
        assert lib.ams_xattn_bwd(*a) == SIZE, at


def test_binding_refusals():
    attn = ams.make_attn(4, 2, 16, "f32")
    off = torch.tensor([0, 2], dtype=torch.int32)
    q, k = torch.zeros((2, 4, 16)), torch.zeros((2, 2, 16))
    ws = torch.zeros(8, dtype=torch.uint8)
    ok = dict(q_off=off, k_off=off, q=q, k=k, v=k, out=q.clone(), lse=None, ws=ws)
    for change, text in [({}, "not on a GPU"), ({"q": q.bfloat16()}, "must be"), ({"q_off": off.long()}, "q_off must be"),
                         ({"k": torch.zeros((2, 4, 16))}, "needed"), ({"v": torch.zeros((3, 2, 16))}, "rows"),
                         ({"out": torch.zeros((1, 4, 16))}, "needed"),
                         ({"k": torch.zeros((2, 16, 2)).transpose(1, 2)}, "must be contiguous"),
                         ({"q": torch.zeros((1, 4, 16)).expand(2, 4, 16)}, "overlap"),
                         ({"key_mask": torch.zeros(2)}, "key_mask must be")]:
        with pytest.raises(ValueError, match=text):
            if change:     # these are seen before the device is asked for
                args = {**ok, **change}
                c = ams._Call("ams_xattn_fwd", q)
                c.device = -1                   # the tensors'
                ams._xattn_inputs(c, attn, args["q_off"], args["k_off"], args["q"], args["k"], args["v"],
                                  args.get("key_mask"))
                c.rows("out", args["out"], q.dtype, 2, (4, 16))
            else:
                ams.ams_xattn_fwd(attn, **ok)
    with pytest.raises(ams.AmsError):
        ams.ams_xattn_fwd(ams.ams_attn(7, 4, 2, 16, 1.0), **ok)
