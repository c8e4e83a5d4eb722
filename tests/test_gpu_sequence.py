"""The sequence operators together, as a program uses them: a training step of
an ID table through lookup, attention and back, and the same histories served
from 8-bit pages.  Tolerances are those of attn_ref carried through the sums."""
import numpy as np
import pytest
import torch

import attn_ref
from paper_1711_06505_amd import ams

pytestmark = pytest.mark.gpu
U = attn_ref.U


class Batch:
    """Padded histories: B users, L places each, some of them padding (ID 0), and nq ads each."""

    def __init__(self, B, L, nq, rows, H, D, seed):
        rng = np.random.default_rng(seed)
        self.B, self.L, self.nq, self.rows, self.H, self.D = B, L, nq, rows, H, D
        lens = rng.integers(0, L + 1, B)
        lens[0], lens[1] = 0, L                       # a user without a history, one without padding
        hist = rng.integers(1, rows, (B, L)) * (np.arange(L) < lens[:, None])
        self.lens = lens
        self.ids = torch.from_numpy(np.concatenate([hist.ravel(), rng.integers(1, rows, B * nq)]).astype(np.int32)).cuda()
        self.k_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * L
        self.q_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * nq
        self.table = torch.from_numpy(rng.standard_normal((rows, H * D)).astype(np.float32)).cuda()
        self.do = torch.from_numpy(rng.standard_normal((B * nq, H, D)).astype(np.float32)).cuda()
        self.scale = float(np.float32(1.5))


def training_step(b, table, accum, lr):
    """One step; returns what a test looks at (the table and accum are updated)."""
    n, nk, H, D = b.ids.numel(), b.B * b.L, b.H, b.D
    dev = dict(device="cuda")
    emb, demb = torch.empty((n, H * D), **dev), torch.empty((n, H * D), **dev)
    ams.ams_lookup_fwd(b.ids, table, emb, b.scale, pad_id=0)
    keys, ads = emb[:nk].view(nk, H, D), emb[nk:].view(-1, H, D)
    mask = (b.ids[:nk] != 0).to(torch.uint8)
    attn = ams.make_attn(H, H, D, "f32")
    ws = torch.empty(ams.ams_xattn_workspace(attn, b.B, n - nk, nk), dtype=torch.uint8, **dev)
    out, lse = torch.empty_like(ads), torch.empty((n - nk, H), **dev)
    ams.ams_xattn_fwd(attn, b.q_off, b.k_off, ads, keys, keys, out, lse, ws, key_mask=mask)
    dk, dv = torch.empty_like(keys), torch.empty_like(keys)
    ams.ams_xattn_bwd(attn, b.q_off, b.k_off, ads, keys, keys, out, lse, b.do, demb[nk:].view(-1, H, D), dk, dv, ws,
                      key_mask=mask)
    demb[:nk] = (dk + dv).view(nk, H * D)
    i32 = lambda m: torch.empty(m, dtype=torch.int32, **dev)      # noqa: E731
    uniq, inv, perm, off, nu, status = i32(n), i32(n), i32(n), i32(n + 1), i32(1), i32(1)
    dws = torch.empty(max(ams.ams_dedup_workspace(n, b.rows), ams.ams_lookup_workspace(n, H * D)), dtype=torch.uint8,
                      **dev)
    grad = torch.empty((n, H * D), **dev)
    ams.ams_dedup(b.ids, b.rows, uniq, inv, perm, off, nu, status, dws)
    ams.ams_lookup_bwd(uniq, inv, perm, off, nu, n, demb, grad, dws, b.scale, pad_id=0)
    ams.ams_adagrad_rows(uniq, nu, n, grad, table, accum, lr, 1e-8)
    torch.cuda.synchronize()
    k = int(nu.item())
    assert int(status.item()) == 0
    return emb, out, uniq[:k].cpu().numpy(), grad[:k].double().cpu(), attn


@pytest.mark.parametrize("B,L,nq,H,D", [(6, 40, 1, 2, 12), (5, 70, 3, 4, 16), (3, 90, 40, 2, 32)])
def test_training_step(B, L, nq, H, D):
    b = Batch(B, L, nq, 50, H, D, seed=L)
    print(f"sequence training B={B} L={L} q={nq} H={H} D={D}", flush=True)
    table, accum = b.table.clone(), torch.zeros_like(b.table)
    emb, out, uniq, grad, attn = training_step(b, table, accum, 0.1)
    nk, ids = B * L, b.ids.cpu().numpy()
    want_emb = np.where((ids != 0)[:, None], b.table.cpu().numpy()[ids] * np.float32(b.scale), np.float32(0))
    np.testing.assert_array_equal(emb.cpu().numpy(), want_emb)
    keys, ads = emb[:nk].view(nk, H, D), emb[nk:].view(-1, H, D)
    vals, tols = attn_ref.batch(ads, keys, keys, b.do, [nq] * B, [L] * B, attn.scale, b.ids[:nk] != 0, False)
    assert ((out.double().cpu() - vals[0]).abs() <= tols[0]).all()
    assert (out[:nq] == 0).all()                                   # the user without a history
    # each token's gradient and how far it may be off, then the rows' sums of them
    dkv, tkv = vals[2] + vals[3], tols[2] + tols[3]
    tkv = tkv + U * (dkv.abs() + tkv)
    tok = torch.cat([dkv, vals[1]]).view(len(ids), -1)
    tol = torch.cat([tkv, tols[1]]).view(len(ids), -1)
    np.testing.assert_array_equal(uniq, np.unique(ids))
    for r, u in enumerate(uniq):
        at = torch.from_numpy(np.flatnonzero(ids == u))
        want, m = tok[at].sum(0) * b.scale * (u != 0), len(at)
        allow = b.scale * (tol[at].sum(0) + m * U * 1.01 * (tok[at].abs() + tol[at]).sum(0)) * (u != 0)
        assert ((grad[r] - want).abs() <= allow + 1e-37).all(), u
    # Adagrad from zero accumulators moves each entry by lr g / (|g| + eps)
    moved = (b.table.double().cpu() - table.double().cpu())[torch.from_numpy(uniq).long()]
    step = 0.1 * grad / (grad.abs() + 1e-8)
    assert ((moved - step).abs() <= 8 * U * (b.table.double().cpu()[torch.from_numpy(uniq).long()].abs() + 0.2)).all()
    gone = np.setdiff1d(np.arange(50), uniq)
    assert torch.equal(table[torch.from_numpy(gone).cuda()], b.table[torch.from_numpy(gone).cuda()])


def test_served_from_pages():
    """Histories embedded, written in two parts and attended to: within what the
    codes' rounding allows of the attention over the embeddings themselves.  An
    entry is off by at most e = 2^-4 of it (half a step of 4 bits) + 2^-10 of its
    scale (half a subnormal step), a score by scale |q| (e_k), so a weight by the factor
    f = exp(2 max e_s) - 1, and the result by sum w (f |v| + (1 + f) e_v)."""
    B, L, nq, H, D = 4, 60, 5, 2, 32
    b = Batch(B, L, nq, 80, H, D, seed=3)
    emb = torch.empty((b.ids.numel(), H * D), device="cuda")
    ams.ams_lookup_fwd(b.ids, b.table, emb, 0.3, pad_id=0)
    nk = B * L
    hist, ads = emb[:nk].view(B, L, H, D), emb[nk:].view(-1, H, D)
    cache = ams.make_cache(H, D, 16, 4, B * 4)
    table = torch.randperm(B * 4, device="cuda").int().view(B, 4)
    kc, vc = (torch.zeros((B * 4, H, 16, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((B * 4, H), device="cuda") for _ in range(2))
    first = b.lens // 2
    for lo, hi in ((np.zeros_like(first), first), (first, b.lens)):
        rows = torch.cat([hist[i, lo[i]:hi[i]] for i in range(B)])
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(hi - lo)]).astype(np.int32)).cuda()
        ams.ams_cache_write(cache, off, torch.from_numpy(lo.astype(np.int32)).cuda(), table, rows, rows, kc, ks, vc, vs)
    attn = ams.make_attn(H, H, D, "f32")
    ws = torch.empty(ams.ams_cache_workspace(attn, cache, B, B * nq), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(ads)
    print("sequence served from pages", flush=True)
    ams.ams_cache_attn(attn, cache, b.q_off, torch.from_numpy(b.lens.astype(np.int32)).cuda(), table, ads, kc, ks, vc,
                       vs, out, ws)
    top = float(ks.max())
    for i in range(B):
        x = hist[i, :b.lens[i]].double().cpu()
        for h in range(H):
            q, k = ads[i * nq:(i + 1) * nq, h].double().cpu(), x[:, h]
            got = out[i * nq:(i + 1) * nq, h].double().cpu()
            if not len(k):
                assert (got == 0).all()
                continue
            # a page's second write may round its first tokens again: twice the error
            e = 2 * (k.abs() * 2.0 ** -4 + top * 2.0 ** -10)
            w = torch.softmax(q @ k.T * attn.scale, 1)
            f = torch.expm1(2 * attn.scale * (q.abs() @ e.T).amax(1, keepdim=True))
            assert ((got - w @ k).abs() <= f * (w @ k.abs()) + (1 + f) * (w @ e) + 1e-5).all()
