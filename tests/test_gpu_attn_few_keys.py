"""Gradients in bf16 over lists of up to 16 keys, whose delta = sum_j p_j <dO, V_j>
is formed from the keys, not from the stored output, which is rounded to bf16.
The values of a list are nearly alike, so that dP - delta, and with it dQ and dK,
is small beside the terms it comes from, and what delta is off by shows.

Bounds, with attn_ref's symbols and p = 2^-17 for a dS on its way into a product:
dp is off by e = (D + 4) u sum_d |do v|, a weight by the factor f, so delta by
sum_j w (f |dp| + e) + (n + 2) u sum_j w |dp|; dS then by m + |scale| (m |dp - delta| +
w (f |dp - delta| + e + e_delta + 2 u (|dp| + |delta|)))."""
import numpy as np
import pytest
import torch

import attn_ref
from test_gpu_xattn import Problem

U, M, H, PAIR = attn_ref.U, attn_ref.M, 2.0 ** -8, 2.0 ** -17


def gradients(q, k, v, do, scale, live, stored=False):
    """dq, dk and their bounds for one head, float64; stored: delta from the output rounded to bf16."""
    keep = live.nonzero()[:, 0]
    K, V = k[keep], v[keep]
    D, n, rows = q.shape[1], K.shape[0], q.shape[0]
    w = torch.softmax(scale * q @ K.T, 1)
    dp = do @ V.T
    out = w @ V
    delta = (do * out.float().bfloat16().double()).sum(1, keepdim=True) if stored else (w * dp).sum(1, keepdim=True)
    ds = scale * w * (dp - delta)
    f = 2 * (D + 8) * U * abs(scale) * (q.abs() @ K.abs().T).amax(1, keepdim=True) + (n + 16) * U
    e = (D + 4) * U * (do.abs() @ V.abs().T)
    e_delta = (w * (f * dp.abs() + e) + (n + 2) * U * w * dp.abs()).sum(1, keepdim=True)
    e_ds = M + abs(scale) * (M * (dp - delta).abs() + w * (f * (dp - delta).abs() + e + e_delta
                                                          + 2 * U * (dp.abs() + delta.abs())))
    dq, dk, bk = ds @ K, torch.zeros_like(k), torch.zeros_like(k)
    dk[keep] = ds.T @ q
    bq = (e_ds + (PAIR + n * U) * ds.abs()) @ K.abs() + (H + U) * dq.abs()
    bk[keep] = (e_ds + (PAIR + rows * U) * ds.abs()).T @ q.abs() + (H + U) * dk[keep].abs()
    return (dq, dk), (1.1 * bq + 1e-37, 1.1 * bk + 1e-37)


def sample(rows, keys, D, seed):
    """q, k, v, do of one head, the values within about 2 % of each other."""
    g = torch.Generator().manual_seed(seed)
    q, k, do = (torch.randn((n, D), generator=g).bfloat16() for n in (rows, keys, rows))
    v = (torch.randn(D, generator=g) * (1 + 0.02 * torch.randn((keys, D), generator=g))).bfloat16()
    return q, k, v, do


# rows a sample, keys of each sample, width: one pass for all gradients, and two kernels
SHAPES = [(1, [2, 16, 1, 5], 64), (9, [3, 16, 7], 16), (16, [2, 12], 128), (20, [4, 9], 32), (40, [3, 16, 1, 2], 64),
          (70, [5, 15], 12), (33, [16, 2], 100)]


@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_the_bounds_tell_the_stored_output_from_the_sum(rows, keys, D):
    missed = [False, False]
    for i, n in enumerate(keys):
        x = [t.double() for t in sample(rows, n, D, i)]
        on = torch.ones(n, dtype=torch.bool)
        right, tols = gradients(*x, D ** -0.5, on)
        wrong, _ = gradients(*x, D ** -0.5, on, stored=True)
        missed = [m or bool(((a - b).abs() > tol).any()) for m, a, b, tol in zip(missed, right, wrong, tols)]
    assert all(missed)


@pytest.mark.gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_few_keys(rows, keys, D, extra, masked):
    heads, B = 2, len(keys)
    p = Problem([rows] * B, keys, heads, heads, D, "bf16", extra=extra, behind=1, drop=0.4 * masked, seed=3)
    k_at = np.concatenate([[0], np.cumsum(keys)])
    for i, n in enumerate(keys):
        for h in range(heads):
            q, k, v, do = sample(rows, n, D, 10 * i + h)
            p.q[i * rows:(i + 1) * rows, h], p.do[i * rows:(i + 1) * rows, h] = q.cuda(), do.cuda()
            p.k[k_at[i]:k_at[i + 1], h], p.v[k_at[i]:k_at[i + 1], h] = k.cuda(), v.cuda()
    live = torch.ones(sum(keys), dtype=torch.bool) if not masked else p.mask[:sum(keys)].cpu() != 0
    if masked:
        p.k[p.mask == 0], p.v[p.mask == 0] = float("nan"), float("inf")
    out, lse = p.forward()
    dq, dk, _ = (x.double().cpu() for x in p.backward(out, lse))
    for i, n in enumerate(keys):
        r, c = slice(i * rows, (i + 1) * rows), slice(k_at[i], k_at[i + 1])
        for h in range(heads):
            q, k, v, do = (t.double() for t in sample(rows, n, D, 10 * i + h))
            if not live[c].any():
                assert (dq[r, h] == 0).all() and (dk[c, h] == 0).all()
                continue
            vals, tols = gradients(q, k, v, do, p.attn.scale, live[c])
            for name, x, want, tol in zip(("dq", "dk"), (dq[r, h], dk[c, h]), vals, tols):
                err = (x - want).abs()
                assert (err <= tol).all(), (name, i, h, float((err / tol).max()))
