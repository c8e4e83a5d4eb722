"""Cross attention and its gradients against float64 (bounds derived in attn_ref)."""
import numpy as np
import pytest
import torch

import attn_ref
from paper_1711_06505_amd import ams

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device="cuda")


def rows_in(x, extra, offset):
    """x [n, heads, dim] as rows of a wider buffer that starts `offset` elements late."""
    n, w = x.shape[0], x.shape[1] * x.shape[2]
    flat = torch.full((n * (w + extra) + offset + 8,), 7.0, dtype=x.dtype, device="cuda")
    v = flat[offset:offset + n * (w + extra)].view(n, w + extra)[:, :w].view(n, *x.shape[1:]) if n else x.cuda()
    v.copy_(x)
    return v


class Problem:
    """Inputs of one call; `behind` rows that no sample owns follow the last sequence."""

    def __init__(self, q_len, k_len, H, Hk, D, dtype, drop=0.0, extra=0, offset=0, behind=3, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed + 7 * sum(q_len) + D)
        self.q_len, self.k_len, self.H, self.Hk, self.D, self.dtype = q_len, k_len, H, Hk, D, dtype
        nq, nk = sum(q_len) + behind, sum(k_len) + behind
        normal = lambda *s: (torch.randn(s, generator=g) * spread).to(DT[dtype])       # noqa: E731
        self.q, self.k = rows_in(normal(nq, H, D), extra, offset), rows_in(normal(nk, Hk, D), extra, offset)
        self.v, self.do = rows_in(normal(nk, Hk, D), extra, offset), rows_in(normal(nq, H, D), extra, offset)
        self.mask = (torch.rand(nk, generator=g) >= drop).to(torch.uint8).cuda() if drop else None
        self.extra, self.offset = extra, offset
        self.attn = ams.make_attn(H, Hk, D, dtype)
        self.q_off, self.k_off = offsets(q_len), offsets(k_len)

    def fresh(self, like):
        x = rows_in(torch.zeros_like(like), self.extra, self.offset)
        x.fill_(-3.0)
        return x

    def workspace(self):
        need = ams.ams_xattn_workspace(self.attn, len(self.q_len), self.q.shape[0], self.k.shape[0])
        assert need > 0
        return torch.full((need,), 255, dtype=torch.uint8, device="cuda")      # NaN in every float

    def forward(self, ws=None, out=None, lse=None, stream=None):
        out = self.fresh(self.q) if out is None else out
        lse = torch.full((self.q.shape[0], self.H), -3.0, device="cuda") if lse is None else lse
        print(f"xattn fwd q={self.q_len[:4]} k={self.k_len[:4]} B={len(self.q_len)} H={self.H}/{self.Hk} D={self.D} "
              f"{self.dtype} +{self.extra}@{self.offset}", flush=True)
        ams.ams_xattn_fwd(self.attn, self.q_off, self.k_off, self.q, self.k, self.v, out, lse,
                          self.workspace() if ws is None else ws, key_mask=self.mask, stream=stream)
        return out, lse

    def backward(self, out, lse, ws=None, grads=None, stream=None):
        dq, dk, dv = [self.fresh(x) for x in (self.q, self.k, self.v)] if grads is None else grads
        print("xattn bwd", flush=True)
        ams.ams_xattn_bwd(self.attn, self.q_off, self.k_off, self.q, self.k, self.v, out, lse, self.do, dq, dk, dv,
                          self.workspace() if ws is None else ws, key_mask=self.mask, stream=stream)
        return dq, dk, dv

    def check(self):
        out, lse = self.forward()
        grads = self.backward(out, lse)
        torch.cuda.synchronize()
        nq, nk = sum(self.q_len), sum(self.k_len)
        live = None if self.mask is None else self.mask[:nk]
        vals, tols = attn_ref.batch(self.q[:nq], self.k[:nk], self.v[:nk], self.do[:nq], self.q_len, self.k_len,
                                    self.attn.scale, live, self.dtype == "bf16")
        for name, x, want, tol, n in zip(("out", "dq", "dk", "dv"), (out, *grads), vals, tols, (nq, nq, nk, nk)):
            got = x.double().cpu()
            assert (got[n:] == -3.0).all(), name                  # rows behind the last sequence
            err = (got[:n] - want).abs()
            assert (err <= tol).all(), (name, float((err / tol).max()))
        self.check_lse(lse.double().cpu(), nq, live)

    def check_lse(self, lse, nq, live):
        assert (lse[nq:] == -3.0).all()
        q0 = k0 = 0
        for a, b in zip(self.q_len, self.k_len):
            q, k = self.q[q0:q0 + a].double().cpu(), self.k[k0:k0 + b].double().cpu()
            on = slice(None) if live is None else live[k0:k0 + b].cpu() != 0
            k = k.repeat_interleave(self.H // self.Hk, 1)[on]
            s = torch.einsum("qhd,khd->qhk", q, k) * self.attn.scale
            want = torch.logsumexp(s, 2) if k.shape[0] else torch.full((a, self.H), -np.inf, dtype=torch.float64)
            big = torch.einsum("qhd,khd->qhk", q.abs(), k.abs()).amax(2) * abs(self.attn.scale) if k.shape[0] else 0
            if k.shape[0]:
                tol = (self.D + 12) * attn_ref.U * big + (b + 20) * attn_ref.U * (1 + want.abs())
                assert ((lse[q0:q0 + a] - want).abs() <= tol).all()
            else:
                assert torch.equal(lse[q0:q0 + a], want)
            q0, k0 = q0 + a, k0 + b


SHAPES = [
    # q_len, k_len, heads, key heads, dim
    ([1], [1], 1, 1, 1),
    ([1], [1], 2, 1, 12),
    ([1, 0, 1, 2], [3, 5, 0, 33], 4, 2, 16),
    ([2, 1], [31, 32], 3, 1, 20),
    ([17], [129], 4, 4, 12),
    ([5, 16, 33], [64, 63, 65], 8, 2, 64),
    ([3], [200], 6, 2, 40),
    ([130, 1], [1, 300], 2, 2, 128),
    ([40, 7], [70, 260], 5, 1, 100),
    ([1, 1, 1], [1000, 3, 517], 8, 8, 128),
    ([1], [9000], 4, 1, 128),
    ([600], [3], 4, 2, 32),
    ([300, 5], [200, 900], 4, 2, 128),
    ([64], [64], 16, 2, 65),
    ([0, 0], [10, 2], 2, 1, 8),
    ([3, 2], [0, 0], 2, 1, 8),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"q{sum(s[0])}k{sum(s[1])}h{s[2]}_{s[3]}d{s[4]}")
def test_against_float64(shape, dtype):
    Problem(*shape, dtype).check()


MANY = [                                     # samples of many rows: several tiles of rows and of keys
    ([128], [64], 1, 1, 64), ([129, 70], [65, 127], 4, 2, 128), ([33, 260, 0], [300, 1, 9], 8, 2, 64),
    ([257], [513], 2, 1, 32), ([100], [1000], 4, 1, 128), ([90, 90], [5, 0], 2, 2, 96), ([150], [190], 3, 1, 40),
    ([700], [300], 2, 2, 72), ([70], [2500], 2, 1, 64), ([1500], [130], 2, 2, 16), ([64, 64], [64, 128], 5, 1, 8)]


@pytest.mark.parametrize("drop", [0.0, 0.4])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: f"q{sum(s[0])}k{sum(s[1])}h{s[2]}_{s[3]}d{s[4]}")
def test_many_rows(shape, drop):
    p = Problem(*shape, "bf16", drop=drop, seed=13, extra=8)
    if drop:
        p.k[p.mask == 0] = float("nan")
        p.v[p.mask == 0] = float("nan")
    p.check()
    if shape[4] == 64:
        Problem(*shape, "f32", drop=drop, seed=14).check()


@pytest.mark.parametrize("D,extra,offset", [(89, 0, 0), (33, 3, 1), (12, 4, 4), (100, 0, 2), (127, 1, 0), (64, 1, 3)])
def test_many_rows_of_any_alignment(D, extra, offset):
    p = Problem([150, 40], [130, 260], 4, 2, D, "bf16", drop=0.2, extra=extra, offset=offset, seed=16)
    p.k[p.mask == 0] = float("nan")
    p.v[p.mask == 0] = float("nan")
    p.check()


def test_many_rows_without_a_key():
    """Every key of one sample masked: zero rows, whatever the upstream gradient holds there."""
    p = Problem([100, 80], [90, 70], 2, 1, 64, "bf16", seed=15, drop=0.1)
    p.mask[:90] = 0
    p.k[:90] = float("nan")
    p.do[:100] = float("nan")
    out, lse = p.forward()
    dq, dk, dv = p.backward(out, lse)
    assert (out[:100] == 0).all() and (dq[:100] == 0).all() and (dk[:90] == 0).all() and (dv[:90] == 0).all()
    assert all(torch.isfinite(x.float()).all() for x in (out, dq[100:180], dk[90:160], dv[90:160]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drop", [0.3, 0.97, 1.0])
def test_key_mask(drop, dtype):
    """Masked keys take no part, also where they leave a query nothing; their
    rows hold NaN and infinities."""
    p = Problem([3, 1, 20, 2], [40, 5, 700, 64], 4, 2, 24, dtype, drop=drop, seed=1)
    dead = p.mask == 0
    p.k[dead] = float("nan")
    p.v[dead] = float("inf")
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("extra,offset", [(8, 0), (4, 4), (1, 0), (3, 1), (0, 2)])
@pytest.mark.parametrize("D", [12, 64])
def test_strides_and_alignment(D, extra, offset, dtype):
    Problem([5, 1, 18], [70, 300, 2], 4, 2, D, dtype, extra=extra, offset=offset, seed=2).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales(dtype):
    """A negative scale, and one of zero (equal weights), for few and many rows."""
    for scale in (-0.3, 0.0):
        for shape in (([3, 2], [40, 70], 2, 2, 16), ([200], [150], 2, 1, 64)):
            p = Problem(*shape, dtype, seed=8)
            p.attn.scale = scale
            p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_short_samples(dtype):
    rng = np.random.default_rng(3)
    Problem(rng.integers(0, 3, 700).tolist(), rng.integers(0, 60, 700).tolist(), 4, 2, 16, dtype, seed=3).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [12, 64, 128])
def test_one_large_sample_among_small_ones(D, dtype):
    """Gradients of samples of few rows and of the others come from different
    kernels of one call; with few samples also in several shares of the keys."""
    Problem([1] * 30 + [90, 0, 2], [25] * 15 + [0] * 5 + [7] * 10 + [150, 9, 60], 4, 2, D, dtype, seed=17).check()
    Problem([1, 25], [3000, 500], 2, 2, D, dtype, drop=0.1, seed=18).check()
    Problem([35, 1], [40, 2500], 2, 1, D, dtype, seed=19).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of several hundred: the maximum is what keeps the softmax finite."""
    Problem([9], [150], 2, 1, 64, dtype, seed=4, spread=8.0).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_upstream_of_a_row_without_keys_is_not_used(dtype):
    p = Problem([2, 2], [5, 0], 2, 1, 16, dtype, seed=5)
    p.do[2:4] = float("nan")
    out, lse = p.forward()
    dq, dk, dv = p.backward(out, lse)
    assert (out[2:4] == 0).all() and (dq[2:4] == 0).all()
    assert all(torch.isfinite(x[:5]).all() for x in (dk, dv))


def test_gradient_against_differences():
    """d<dO, out>/dx by central differences of the float32 forward along random
    directions: truncation h^2 and rounding 2^-22 / h, at h = 2^-7, on values of order 1."""
    p = Problem([3, 2], [9, 20], 4, 2, 8, "f32", behind=0, seed=6)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    g = torch.Generator().manual_seed(9)
    h = 2.0 ** -7
    for name, x, dx in zip("qkv", (p.q, p.k, p.v), grads):
        d = torch.randn(x.shape, generator=g).cuda()
        d /= d.norm()
        keep = x.clone()
        f = []
        for s in (h, -h):
            x.copy_(keep + s * d)
            f.append(float((p.forward()[0].double() * p.do.double()).sum()))
        x.copy_(keep)
        slope, want = (f[0] - f[1]) / (2 * h), float((dx.double() * d.double()).sum())
        mag = float((out.abs() * p.do.abs()).sum())
        assert abs(slope - want) <= 8 * h * h * mag + 2.0 ** -22 / h * mag, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_graph(dtype):
    """Forward and backward captured and replayed on new inputs beside eager
    calls with another workspace: bit-equal."""
    p = Problem([1, 4, 0], [700, 90, 30], 4, 2, 32, dtype, seed=7)
    e = Problem([1, 4, 0], [700, 90, 30], 4, 2, 32, dtype, seed=7)
    ws, ws_e = p.workspace(), e.workspace()
    buf = [p.fresh(p.q), torch.zeros((p.q.shape[0], 4), device="cuda"), p.fresh(p.q), p.fresh(p.k), p.fresh(p.v)]

    def step():
        p.forward(ws, buf[0], buf[1])
        p.backward(buf[0], buf[1], ws, buf[2:])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        g = torch.Generator().manual_seed(k)
        for x, y in ((p.q, e.q), (p.k, e.k), (p.v, e.v), (p.do, e.do)):
            x.copy_(torch.randn(x.shape, generator=g).to(x.dtype))
            y.copy_(x)
        out, lse = e.forward(ws_e)
        grads = e.backward(out, lse, ws_e)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(buf, (out, lse, *grads)):
            assert torch.equal(a[:5], b[:5]), k


@pytest.mark.parametrize("q_len,k_len", [([3, 1, 2], [40, 70, 9]), ([90, 70], [130, 100])])
def test_rows_before_the_first_sample(q_len, k_len):
    """Offsets that begin behind 0: the rows in front are nobody's, and the
    samples' results are what they are without them."""
    a = Problem(q_len, k_len, 4, 2, 32, "bf16", seed=20)
    b = Problem([5] + q_len, [7] + k_len, 4, 2, 32, "bf16", seed=20)
    nq, nk = sum(q_len), sum(k_len)
    for x, y, lead, n in ((a.q, b.q, 5, nq), (a.do, b.do, 5, nq), (a.k, b.k, 7, nk), (a.v, b.v, 7, nk)):
        y[lead:lead + n] = x[:n]
        y[:lead] = float("nan")
    b.q_off, b.k_off = b.q_off[1:].contiguous(), b.k_off[1:].contiguous()
    b.q_len, b.k_len = q_len, k_len
    res = []
    for p in (a, b):
        out, lse = p.forward()
        res.append((out, *p.backward(out, lse)))
    for x, y, lead, n in zip(*res, (5, 5, 7, 7), (nq, nq, nk, nk)):
        assert torch.equal(x[:n], y[lead:lead + n])
        assert (y[:lead] == -3.0).all() and (y[lead + n:] == -3.0).all()


def test_two_streams_at_once():
    ps = [Problem([1, 9], [5000, 300], 4, 2, 64, "bf16", seed=s) for s in (10, 11)]
    alone = [[x.clone() for x in (o, *p.backward(o, l))] for p in ps for o, l in [p.forward()]]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    held, got = [], []
    for p, s in zip(ps, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            ws = p.workspace()
            o, l = p.forward(ws)
            got.append((o, *p.backward(o, l, ws)))
            held.append((ws, l))
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_keys_and_values_in_one_array():
    """k is v: the gradient is dk + dv (as for a query over plain embeddings)."""
    p = Problem([4, 2], [30, 7], 2, 2, 12, "f32", seed=12)
    p.v = p.k
    p.check()
