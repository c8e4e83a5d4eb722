"""The weights of the softmax and their gradients in bf16, which enter the second
product as a pair of bf16 values within 2^-17 of the float32 one.  The inputs come
in pairs of rows that cancel: keys 2j and 2j + 1 nearly alike with opposite
values, queries likewise with opposite upstream rows.  So results are small
beside the sums of their terms' magnitudes, their own rounding (2^-8 of the
result) too, and an error of the weights shows: rounded to bf16 once they would
miss these bounds, which is asserted for the definition in float64.

The bounds are attn_ref's, with p = 2^-17 for a weight or dS on its way into a
product and h = 2^-8 for the rounding of a stored result."""
import pytest
import torch

import attn_ref
from paper_1711_06505_amd import ams
from test_gpu_cache import Cache
from test_gpu_xattn import Problem

U, M, H, PAIR = attn_ref.U, attn_ref.M, 2.0 ** -8, 2.0 ** -17


def once(x):
    """Rounded to bf16 once."""
    return x.float().bfloat16().double()


def attention(q, k, v, do, scale, weights=lambda w: w):
    """(out, dq, dk, dv) and their bounds for one head, float64; `weights` is applied to what enters a second product."""
    D, n, rows = q.shape[1], k.shape[0], q.shape[0]
    s = scale * q @ k.T
    e = torch.exp(s - s.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    w, out = e / total, weights(e) @ v / total
    es = (D + 8) * U * abs(scale) * (q.abs() @ k.abs().T)
    f = 2 * es.amax(1, keepdim=True) + (n + 16) * U
    b_out = w @ v.abs() * (f + PAIR + n * U) + M * v.abs().sum(0) + (H + U) * out.abs()
    dp = do @ v.T
    stored = w @ v
    delta = (do * stored).sum(1, keepdim=True)
    ds = scale * w * (dp - delta)
    e_dp = (D + 4) * U * (do.abs() @ v.abs().T) + (do.abs() * b_out).sum(1, keepdim=True) \
        + (D + 4) * U * (do.abs() * out.abs()).sum(1, keepdim=True)
    e_ds = M + abs(scale) * (M * (dp - delta).abs() + w * (f * (dp - delta).abs() + e_dp))
    dq, dk, dv = weights(ds) @ k, weights(ds).T @ q, weights(w).T @ do
    b_dq = (e_ds + (PAIR + n * U) * ds.abs()) @ k.abs() + (H + U) * dq.abs()
    b_dk = (e_ds + (PAIR + rows * U) * ds.abs()).T @ q.abs() + (H + U) * dk.abs()
    b_dv = (M + w * (f + PAIR + rows * U)).T @ do.abs() + (H + U) * dv.abs()
    return (out, dq, dk, dv), [1.1 * b + 1e-37 for b in (b_out, b_dq, b_dk, b_dv)]


def alike(x):
    """Rows 2j + 1 within about 2 % of rows 2j."""
    g = torch.Generator().manual_seed(x.shape[0])
    x[1::2] = x[::2] * (1 + 0.02 * torch.randn(x[::2].shape, generator=g))
    return x.bfloat16()


def opposite(x):
    x = x.bfloat16()
    x[1::2] = -x[::2]
    return x


def inputs(rows, keys, D, seed):
    """Of one head: q, k, v, do."""
    g = torch.Generator().manual_seed(seed)
    return [f(0.5 * torch.randn((n, D), generator=g)) for n, f in
            ((rows, alike), (keys, alike), (keys, opposite), (rows, opposite))]


# rows of a sample, its keys, width: gradients in one pass; in two kernels (more rows, fewer than 64 keys)
SHAPES = [(16, 32, 64), (8, 200, 16), (32, 48, 32), (8, 60, 128), (40, 48, 64), (24, 60, 128)]


@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_the_bounds_tell_one_rounding_from_two(rows, keys, D):
    x = [t.double() for t in inputs(rows, keys, D, 1)]
    right, tols = attention(*x, D ** -0.5)
    wrong, _ = attention(*x, D ** -0.5, once)
    for a, b, tol in zip(right, wrong, tols):
        assert ((a - b).abs() > tol).any()


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("rows,keys,D", SHAPES)
def test_pairs(rows, keys, D, extra):
    heads, samples = 2, 3
    p = Problem([rows] * samples, [keys] * samples, heads, heads, D, "bf16", extra=extra, behind=0)
    for i in range(samples):
        for h in range(heads):
            q, k, v, do = inputs(rows, keys, D, 10 * i + h)
            p.q[i * rows:(i + 1) * rows, h], p.do[i * rows:(i + 1) * rows, h] = q.cuda(), do.cuda()
            p.k[i * keys:(i + 1) * keys, h], p.v[i * keys:(i + 1) * keys, h] = k.cuda(), v.cuda()
    out, lse = p.forward()
    got = [x.double().cpu() for x in (out, *p.backward(out, lse))]
    for i in range(samples):
        for h in range(heads):
            vals, tols = attention(*(t.double() for t in inputs(rows, keys, D, 10 * i + h)), p.attn.scale)
            for name, x, want, tol, n in zip(("out", "dq", "dk", "dv"), got, vals, tols, (rows, rows, keys, keys)):
                err = (x[i * n:(i + 1) * n, h] - want).abs()
                assert (err <= tol).all(), (name, i, h, float((err / tol).max()))


SCALE = 0.004                     # of the scores over pages: weights nearly alike, whose opposite values cancel


@pytest.mark.gpu
@pytest.mark.parametrize("q,G,D,page,n", [(1, 1, 64, 16, 64), (3, 4, 128, 32, 60), (20, 1, 64, 16, 48), (40, 2, 32, 16, 32)])
def test_pairs_over_pages(q, G, D, page, n):
    """Up to 96 rows a sample; the definition with weights rounded once misses the bound here too."""
    c = Cache(1, 1, D, page, -(-n // page), seed=D + q)
    keys = iter((True, False))                              # then the values

    def rows(rng, shape):
        x = rng.standard_normal(shape)
        if not next(keys):
            x[1::2] = -x[::2]
        return x
    c.write([n], make=rows)
    (k, v), _ = c.entries(0)
    x = torch.from_numpy(c.rng.standard_normal((q, G, D))).bfloat16().cuda()
    out = torch.zeros_like(x)
    attn = ams.make_attn(G, 1, D, "bf16", SCALE)
    off = torch.tensor([0, q], dtype=torch.int32, device="cuda")
    ws = torch.empty(ams.ams_cache_workspace(attn, c.cache, 1, q), dtype=torch.uint8, device="cuda")
    print(f"pairs over pages q={q} G={G} D={D} n={n}", flush=True)
    ams.ams_cache_attn(attn, c.cache, off, torch.from_numpy(c.len).cuda(), torch.from_numpy(c.table).cuda(), x,
                       *c.arrays(), out, ws)
    missed = False
    for h in range(G):
        a = x[:, h].double().cpu()
        args = (a, k[:, 0], v[:, 0], torch.zeros_like(a), attn.scale)
        vals, tols = attention(*args)
        missed |= bool(((attention(*args, once)[0][0] - vals[0]).abs() > tols[0]).any())
        assert ((out[:, h].double().cpu() - vals[0]).abs() <= tols[0]).all(), h
    assert missed
