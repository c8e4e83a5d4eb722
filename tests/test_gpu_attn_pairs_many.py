"""The gradient of the queries of heads up to 32 wide: its weights' gradients
enter the product as a pair of bf16 values for samples of many rows too.  Inputs
and bounds are those of test_gpu_attn_pairs; the backward is given the
definition's output (rounded once) and log-sum-exp."""
import pytest
import torch

from test_gpu_attn_pairs import attention, inputs, once
from test_gpu_xattn import Problem

SHAPES = [(40, 80, 32), (140, 200, 8), (48, 70, 12), (36, 300, 16)]


@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_the_bounds_tell_one_rounding_from_two(rows, keys, D):
    x = [t.double() for t in inputs(rows, keys, D, 1)]
    (_, right, _, _), (_, tol, _, _) = attention(*x, D ** -0.5)
    assert ((attention(*x, D ** -0.5, once)[0][1] - right).abs() > tol).any()


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_queries_gradient(rows, keys, D, extra):
    heads, samples = 2, 2
    p = Problem([rows] * samples, [keys] * samples, heads, heads, D, "bf16", extra=extra, behind=0)
    out, lse = p.fresh(p.q), torch.zeros((rows * samples, heads), device="cuda")
    want = {}
    for i in range(samples):
        for h in range(heads):
            x = inputs(rows, keys, D, 10 * i + h)
            r, c = slice(i * rows, (i + 1) * rows), slice(i * keys, (i + 1) * keys)
            for t, at, n in zip(x, (p.q, p.k, p.v, p.do), (r, c, c, r)):
                at[n, h] = t.cuda()
            q, k, v, do = (t.double() for t in x)
            want[i, h] = r, attention(q, k, v, do, p.attn.scale)
            s = p.attn.scale * q @ k.T
            out[r, h], lse[r, h] = (torch.softmax(s, 1) @ v).bfloat16().cuda(), torch.logsumexp(s, 1).float().cuda()
    dq = p.backward(out, lse)[0].double().cpu()
    for (i, h), (r, (vals, tols)) in want.items():
        err = (dq[r, h] - vals[1]).abs()
        assert (err <= tols[1]).all(), (i, h, float((err / tols[1]).max()))
