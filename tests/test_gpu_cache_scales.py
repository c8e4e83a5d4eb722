"""Attention over 8-bit pages with any scale of the scores: zero (equal weights),
one so small that its product with a page's scale has no float32 value, and
negative ones, where pages of zeros (whose scale is 2^-100) lie beside others."""
import numpy as np
import pytest
import torch

import attn_ref
from paper_1711_06505_amd import ams
from test_gpu_cache import DT, Cache

pytestmark = pytest.mark.gpu


def attend(c, q_len, H, dtype, scale, q=None):
    """Calls with `scale` and compares every row and log-sum-exp with float64 (bounds of attn_ref)."""
    off = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    n = int(off[-1])
    q = (torch.from_numpy(c.rng.standard_normal((n, H, c.D))) if q is None else q).to(DT[dtype]).cuda()
    out, lse = torch.full_like(q, -3.0), torch.full((n, H), -3.0, device="cuda")
    attn = ams.make_attn(H, c.Hk, c.D, dtype, scale)
    ws = torch.full((ams.ams_cache_workspace(attn, c.cache, c.B, n),), 255, dtype=torch.uint8, device="cuda")
    print(f"cache attn scale={scale} q={q_len[:4]} len={c.len[:4]} H={H}/{c.Hk} D={c.D} P={c.P} {dtype}", flush=True)
    ams.ams_cache_attn(attn, c.cache, torch.from_numpy(off).cuda(), torch.from_numpy(c.len).cuda(),
                       torch.from_numpy(c.table).cuda(), q, *c.arrays(), out, ws, lse=lse)
    torch.cuda.synchronize()
    q, out, lse = q.double().cpu(), out.double().cpu(), lse.double().cpu()
    for i in range(c.B):
        (k, v), ok = c.entries(i)
        rows = slice(off[i], off[i + 1])
        for head in range(H):
            x, kh = q[rows, head], head // (H // c.Hk)
            vals, tols = attn_ref.attention(x, k[:, kh], v[:, kh], torch.zeros_like(x), attn.scale, ok,
                                            2.0 ** -8 if dtype == "bf16" else 0.0)
            assert ((out[rows, head] - vals[0]).abs() <= 1.1 * tols[0] + 1e-37).all(), (i, head)
            s = x @ k[ok][:, kh].T * attn.scale
            want = torch.logsumexp(s, 1)
            big = (x.abs() @ k[ok][:, kh].abs().T).amax(1) * abs(attn.scale)
            tol = (c.D + 12) * attn_ref.U * big + (s.shape[1] + 20) * attn_ref.U * (1 + want.abs())
            assert ((lse[rows, head] - want).abs() <= tol).all(), (i, head)


def zeros_in(spans):
    """Normal rows with zeros in head 0 of the tokens of `spans` (both keys and values)."""
    def rows(rng, shape):
        x = rng.standard_normal(shape)
        for lo, hi in spans:
            x[lo:hi, 0] = 0.0
        return x
    return rows


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 1e-20, -1e-20, 1e-39, -0.3])
@pytest.mark.parametrize("q,G,D,page", [(2, 2, 64, 16), (200, 1, 64, 16), (60, 4, 128, 16), (130, 1, 32, 64)])
def test_pages_of_zeros(q, G, D, page, scale, dtype):
    """Few and many rows; the last page's keys are zero in one head, and its last tokens fill no tile."""
    lens = [64 + 6, 3, 4 * page + 1]
    ends = np.cumsum(lens)
    first = [(n - 1) // page * page for n in lens]              # of the last page
    spans = [(e - n + f, e) for e, n, f in zip(ends, lens, first)]
    c = Cache(3, 2, D, page, -(-max(lens) // page), seed=D + q)
    c.write(lens, make=zeros_in(spans))
    assert all((c.scale[0][c.table[i, f // page], 0] == 2.0 ** -100) for i, f in enumerate(first))
    attend(c, [q, q + 3, q], 2 * G, dtype, scale)


@pytest.mark.parametrize("q", [2, 150])
def test_zero_scale_over_large_entries(q):
    """A scale of zero gives equal weights whatever the products are (up to 2^166 here, 2^74 in the codes' units)."""
    c = Cache(1, 1, 64, 16, 5, seed=q)
    c.write([70], make=lambda r, s: np.sign(r.standard_normal(s)) * 2.0 ** 100)
    rows = torch.from_numpy(np.sign(c.rng.standard_normal((q, 1, 64))) * 2.0 ** 60)
    attend(c, [q], 1, "bf16", 0.0, rows)


@pytest.mark.parametrize("q", [2, 150])
def test_a_scale_that_is_not_a_number(q):
    """NaN goes through to every row that attends to something."""
    c = Cache(1, 1, 64, 16, 5, seed=q)
    c.write([70])
    off = torch.tensor([0, q], dtype=torch.int32, device="cuda")
    x = torch.ones((q, 1, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(x)
    attn = ams.make_attn(1, 1, 64, "bf16", float("nan"))
    ws = torch.empty(ams.ams_cache_workspace(attn, c.cache, 1, q), dtype=torch.uint8, device="cuda")
    ams.ams_cache_attn(attn, c.cache, off, torch.from_numpy(c.len).cuda(), torch.from_numpy(c.table).cuda(), x,
                       *c.arrays(), out, ws)
    assert torch.isnan(out).all()
