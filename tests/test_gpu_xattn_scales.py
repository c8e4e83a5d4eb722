"""Scales of the scores at the ends of their range, for few and many rows: zero
over products up to 2^126 (equal weights all the same), and NaN."""
import pytest
import torch

from test_gpu_xattn import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q", [2, 150])
def test_zero_over_large_products(q, dtype):
    p = Problem([q, 3], [130, 70], 2, 1, 64, dtype, seed=q, drop=0.1)
    for x in (p.q, p.k):
        x.copy_(torch.sign(x.float()) * 2.0 ** 60)
    p.attn.scale = 0.0
    out, lse = p.forward()
    live = p.mask[:200].double()
    for rows, keys in ((slice(0, q), slice(0, 130)), (slice(q, q + 3), slice(130, 200))):
        n, v = float(live[keys].sum()), p.v[keys, 0].double()
        want = (live[keys, None] * v).sum(0) / n
        # a sum of n + 1 float32 terms, each weight and the result rounded to the storage type (2^-8, 2^-24)
        tol = ((live[keys, None] * v.abs()).sum(0) / n) * 1.1 * (2 * (2.0 ** -8 if dtype == "bf16" else 0) + (n + 20) * 2.0 ** -24)
        assert ((out[rows].double() - want).abs() <= tol).all()
        assert ((lse[rows].double() - torch.log(torch.tensor(n).double())).abs() <= (n + 20) * 2.0 ** -24 * 6).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q", [2, 150])
def test_not_a_number(q, dtype):
    """NaN goes through to every row that attends to something, and to no other one."""
    p = Problem([q, 3], [130, 0], 2, 1, 64, dtype, seed=q)
    p.attn.scale = float("nan")
    out, lse = p.forward()
    assert torch.isnan(out[:q]).all() and torch.isnan(lse[:q]).all()
    assert (out[q:q + 3] == 0).all() and (out[q + 3:] == -3.0).all()
