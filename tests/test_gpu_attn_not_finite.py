"""Infinities and NaN in rows that do take part: the results of their own sample
and key head are unspecified, every other one is what it is without them."""
import numpy as np
import pytest
import torch

from paper_1711_06505_amd import ams
from test_gpu_cache import Cache
from test_gpu_xattn import Problem

pytestmark = pytest.mark.gpu


def results(p):
    out, lse = p.forward()
    return (out, lse, *p.backward(out, lse))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_len,k_len,D", [
    ([3, 2, 4], [40, 33, 70], 12), ([17, 1, 2], [300, 65, 9], 64),              # samples of few rows and others
    ([90, 70, 40], [130, 65, 100], 64), ([90, 70, 40], [130, 65, 100], 40), ([140, 33, 20], [90, 200, 70], 128)])
def test_other_samples_and_heads_are_untouched(q_len, k_len, D, dtype, bad):
    H, Hk, G = 4, 2, 2
    p = Problem(q_len, k_len, H, Hk, D, dtype, seed=D)
    want = results(p)
    q0, q1, k0, k1 = q_len[0], q_len[0] + q_len[1], k_len[0], k_len[0] + k_len[1]
    p.k[k0 + 3, 1, 0] = bad                                # sample 1, key head 1
    p.v[k0 + 4, 1, D - 1] = bad
    p.q[q0, G, 0] = p.do[q0, G + 1, D // 2] = bad
    got = results(p)
    for x, y, a, b, h in zip(want, got, (q0, q0, q0, k0, k0), (q1, q1, q1, k1, k1), (G, G, G, 1, 1)):
        assert torch.equal(x[:a], y[:a]) and torch.equal(x[b:], y[b:])
        assert torch.equal(x[a:b, :h], y[a:b, :h])         # the other key head's


@pytest.mark.parametrize("q", [2, 110])
def test_over_pages(q):
    c = Cache(3, 2, 64, 16, 6, seed=q)
    c.write([70, 90, 33])
    off = torch.arange(4, dtype=torch.int32, device="cuda") * q
    x = torch.from_numpy(np.random.default_rng(q).standard_normal((3 * q, 4, 64))).bfloat16().cuda()
    attn = ams.make_attn(4, 2, 64, "bf16")
    outs = []
    for nan in (False, True):
        if nan:
            for codes in c.dev[:2]:
                codes[int(c.table[1, 2]), 1, 5, 7] = 127   # sample 1, token 37, key head 1
        out = torch.zeros_like(x)
        ws = torch.empty(ams.ams_cache_workspace(attn, c.cache, 3, 3 * q), dtype=torch.uint8, device="cuda")
        ams.ams_cache_attn(attn, c.cache, off, torch.from_numpy(c.len).cuda(), torch.from_numpy(c.table).cuda(), x,
                           *c.arrays(), out, ws)
        outs.append(out)
    a, b = outs
    assert torch.equal(a[:q], b[:q]) and torch.equal(a[2 * q:], b[2 * q:]) and torch.equal(a[q:2 * q, :2], b[q:2 * q, :2])
    assert torch.isnan(b[q:2 * q, 2:]).all()
