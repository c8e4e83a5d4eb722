"""The 8-bit cache: codes and scales against their definition (equal, bit by
bit), attention over them against float64 on the entries that the codes stand
for (bounds of attn_ref, whose k and v are exact here)."""
import numpy as np
import pytest
import torch

import attn_ref
from paper_1711_06505_amd import ams

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def scale_for(most):
    """Least 2^e >= 2^-100 with 448 2^e >= most."""
    m, e = np.frexp(np.asarray(most, np.float64))           # most = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    return np.exp2(np.maximum(e - 9 + (m > 0.875), -100) * (most > 0) + -100.0 * (most == 0))


def encode(x):
    """float64 to e4m3 bytes: nearest of the 127 magnitudes, ties to the even code."""
    mags = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=-1e9)), 448.0)
    hi = np.minimum(np.searchsorted(mags, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = mags[hi] - a, a - mags[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def decode(codes):
    return torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()


class Cache:
    """A pool on the GPU and its model: what write() should leave in every byte."""

    def __init__(self, B, Hk, D, page, max_pages, seed=0, spare=2):
        self.B, self.Hk, self.D, self.P, self.max_pages = B, Hk, D, page, max_pages
        self.rng = np.random.default_rng(seed)
        self.n_pages = B * max_pages + spare
        self.cache = ams.make_cache(Hk, D, page, max_pages, self.n_pages)
        self.table = self.rng.permutation(self.n_pages)[:B * max_pages].astype(np.int32).reshape(B, max_pages)
        self.codes = [self.rng.integers(0, 256, (self.n_pages, Hk, page, D)).astype(np.uint8) for _ in range(2)]
        self.scale = [np.exp2(self.rng.integers(-3, 3, (self.n_pages, Hk))).astype(np.float32) for _ in range(2)]
        self.dev = [torch.from_numpy(x).cuda() for x in (*self.codes, *self.scale)]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.len = np.zeros(B, np.int32)

    def arrays(self):
        kc, vc, ks, vs = self.dev
        return kc, ks, vc, vs

    def write(self, n_new, dtype="f32", make=None, extra=0):
        n_new = np.asarray(n_new, np.int32)
        off = np.concatenate([[0], np.cumsum(n_new)]).astype(np.int32)
        n, w = int(off[-1]), self.Hk * self.D
        rows = []
        for _ in range(2):
            x = make(self.rng, (n, self.Hk, self.D)) if make else self.rng.standard_normal((n, self.Hk, self.D))
            buf = torch.zeros((n, w + extra), dtype=DT[dtype], device="cuda")
            v = buf[:, :w].view(n, self.Hk, self.D) if n else buf.view(0, self.Hk, self.D)
            v.copy_(torch.from_numpy(np.asarray(x, np.float64)).to(DT[dtype]))
            rows.append(v)
        print(f"cache write {n_new[:4]} at {self.len[:4]} Hk={self.Hk} D={self.D} P={self.P} {dtype}", flush=True)
        ams.ams_cache_write(self.cache, torch.from_numpy(off).cuda(), torch.from_numpy(self.len).cuda(),
                            torch.from_numpy(self.table).cuda(), *rows, *self.arrays(), self.status)
        torch.cuda.synchronize()
        for x, codes, scale in zip(rows, self.codes, self.scale):
            x = x.double().cpu().numpy()
            for i in range(self.B):
                s, e = int(self.len[i]), int(self.len[i]) + int(n_new[i])
                for p in range(max(s, 0) // self.P, -(-e // self.P)):
                    lo, hi = max(s, p * self.P), min(e, (p + 1) * self.P)
                    page = self.table[i, p] if s >= 0 and p < self.max_pages else -1
                    if lo >= hi or not 0 <= page < self.n_pages:
                        continue
                    new = x[off[i] + lo - s:off[i] + hi - s].transpose(1, 0, 2)
                    t0, t1 = lo - p * self.P, hi - p * self.P
                    for h in range(self.Hk):
                        mag = np.abs(new[h])
                        sc = scale_for(np.max(mag[np.isfinite(mag)], initial=0.0))
                        if t0 and scale[page, h] >= sc:
                            sc = np.float64(scale[page, h])
                        elif t0:
                            codes[page, h, :t0] = encode(decode(codes[page, h, :t0]) * (scale[page, h] / sc))
                        codes[page, h, t0:t1] = encode(new[h] / sc)
                        scale[page, h] = sc
        self.len = self.len + n_new

    def check(self):
        for got, want in zip(self.dev[:2], self.codes):
            g, nan = got.cpu().numpy(), (want & 127) == 127
            np.testing.assert_array_equal(g[~nan], want[~nan])
            assert ((g[nan] & 127) == 127).all()                    # NaN of either sign
        for got, want in zip(self.dev[2:], self.scale):
            np.testing.assert_array_equal(got.cpu().numpy(), want)

    def entries(self, i):
        """float64 k and v rows [tokens, Hk, D] of sample i; None for tokens whose page is nowhere."""
        out = []
        for codes, scale in zip(self.codes, self.scale):
            x = np.zeros((self.len[i], self.Hk, self.D))
            for t in range(self.len[i]):
                page = self.table[i, t // self.P]
                if 0 <= page < self.n_pages:
                    x[t] = decode(codes[page, :, t % self.P]) * scale[page][:, None]
            out.append(torch.from_numpy(x))
        ok = [0 <= self.table[i, t // self.P] < self.n_pages for t in range(self.len[i])]
        return out, torch.tensor(ok, dtype=torch.bool)

    def attend(self, q_len, H, dtype, extra=0, with_lse=True):
        off = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
        n, w = int(off[-1]) + 2, H * self.D                         # two rows that nobody owns
        q, out = (torch.zeros((n, w + extra), dtype=DT[dtype], device="cuda")[:, :w].view(n, H, self.D)
                  for _ in range(2))
        q.copy_(torch.from_numpy(self.rng.standard_normal((n, H, self.D))).to(DT[dtype]))
        out.fill_(-3.0)
        attn = ams.make_attn(H, self.Hk, self.D, dtype)
        ws = torch.full((ams.ams_cache_workspace(attn, self.cache, self.B, n),), 255, dtype=torch.uint8, device="cuda")
        lse = torch.full((n, H), -3.0, device="cuda") if with_lse else None
        print(f"cache attn q={q_len[:4]} len={self.len[:4]} H={H}/{self.Hk} D={self.D} P={self.P} {dtype}", flush=True)
        ams.ams_cache_attn(attn, self.cache, torch.from_numpy(off).cuda(), torch.from_numpy(self.len).cuda(),
                           torch.from_numpy(self.table).cuda(), q, *self.arrays(), out, ws, lse=lse)
        torch.cuda.synchronize()
        assert (out[off[-1]:] == -3.0).all()
        h = 2.0 ** -8 if dtype == "bf16" else 0.0
        for i in range(self.B):
            (k, v), ok = self.entries(i)
            for head in range(H):
                x = q[off[i]:off[i + 1], head].double().cpu()
                if not x.shape[0]:
                    continue
                kh = head // (H // self.Hk)
                vals, tols = attn_ref.attention(x, k[:, kh], v[:, kh], torch.zeros_like(x), attn.scale, ok, h)
                got = out[off[i]:off[i + 1], head].double().cpu()
                assert ((got - vals[0]).abs() <= 1.1 * tols[0] + 1e-37).all(), (i, head)
                if with_lse:
                    s = x @ k[ok][:, kh].T * attn.scale
                    want = torch.logsumexp(s, 1) if s.shape[1] else torch.full((x.shape[0],), -np.inf).double()
                    got = lse[off[i]:off[i + 1], head].double().cpu()
                    tol = (self.D + 12) * attn_ref.U * (x.abs() @ k[ok][:, kh].abs().T).amax(1) * attn.scale \
                        + (s.shape[1] + 20) * attn_ref.U * (1 + want.abs()) if s.shape[1] else 0
                    assert (got == want).all() if not s.shape[1] else ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hk,D,page", [(1, 1, 16), (2, 12, 16), (3, 64, 32), (1, 128, 128), (2, 20, 64), (4, 33, 16)])
def test_prompts_then_single_tokens(Hk, D, page, dtype):
    """Prompts of ragged lengths, then tokens one at a time over page borders, some of them larger than before."""
    c = Cache(4, Hk, D, page, 5, seed=D)
    c.write([page + 3, 0, 1, 2 * page], dtype, extra=8)
    c.check()
    for k in range(5):
        c.write([1, 1, k % 2, 1], dtype, make=lambda r, s: r.standard_normal(s) * 4.0 ** r.integers(-3, 4, (s[0], 1, 1)))
        c.check()
    c.write([page - 2, 2 * page + 1, 5, 0], dtype)
    c.check()
    assert c.status.item() == 0
    c.attend([1, 3, 0, 2], 2 * Hk, dtype)


def test_every_value_and_tie():
    """All bf16 magnitudes of a page's range, so every tie between codes, with the scale that 448 gives."""
    b = torch.arange(0, 2 ** 15, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double().numpy()
    b = b[np.isfinite(b) & (b <= 448) & (b >= 2.0 ** -12)]
    b = np.concatenate([b, -b, [448.0]])
    n = -(-b.size // 64)
    vals = np.zeros(n * 64)
    vals[:b.size] = b
    c = Cache(1, 1, 64, 128, -(-n // 128))

    def rows(r, s):
        x = vals.reshape(s).copy()
        x[::128, :, -1] = 448.0                                    # every page's scale is 1
        return x
    c.write([n], "bf16", make=rows)
    c.check()
    assert (c.scale[0][c.table[0]] == 1.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_ordinary(dtype):
    """Zeros, infinities, NaN, subnormal and huge values."""
    def rows(r, s):
        x = r.standard_normal(s)
        x[0] = 0.0
        x[1] = 1e-39
        x[2, :, 0], x[2, :, 1], x[2, :, 2] = np.inf, -np.inf, np.nan
        x[3] *= 1e38
        x[20:] = 0.0
        return x
    c = Cache(2, 2, 8, 16, 4, seed=3)
    c.write([40, 0], dtype, make=rows)
    c.check()
    c.write([1, 17], dtype, make=lambda r, s: np.full(s, -0.0))
    c.check()


def test_tokens_with_nowhere_to_go():
    c = Cache(3, 2, 16, 16, 2, seed=4)
    c.table[1, 1] = c.n_pages                       # a bad page
    c.write([32, 30, 40])                           # sample 2 has room for 32
    c.check()
    assert c.status.item() == 7                     # AMS_ERR_ID_RANGE
    c.len[2] = 32
    c.attend([2, 2, 2], 4, "f32")                   # sample 1's second page takes no part
    c.table[1, 0] = -1
    c.attend([1, 1, 1], 4, "bf16")                  # now it has no page: a zero row
    c.status.zero_()
    c.len[:] = [-3, 0, 0]
    c.table[1] = c.rng.permutation(2)
    c.table[0], c.table[2] = [2, 3], [4, 5]
    c.write([5, 1, 1])
    c.len[0] = 0
    c.check()
    assert c.status.item() == 7


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hk,G,D,page,lens,q_len", [
    (1, 1, 12, 16, [1, 0, 17], [1, 2, 1]),
    (2, 4, 64, 32, [500, 3, 64, 33], [1, 1, 1, 1]),
    (2, 2, 32, 128, [129, 127], [20, 37]),
    (1, 8, 128, 64, [4000], [1]),
    (3, 1, 100, 16, [40, 700], [3, 0]),
    (8, 4, 128, 16, [90, 5], [1, 1]),
    # many rows a sample: one tile and several, of keys too, widths that fill none
    (2, 4, 64, 32, [700, 0, 64], [40, 30, 33]), (1, 2, 128, 16, [65, 1, 300], [129, 20, 64]),
    (1, 1, 32, 64, [1500], [200]), (2, 1, 80, 128, [200, 129], [70, 300]), (1, 4, 16, 16, [63, 900], [50, 3])])
def test_attention(Hk, G, D, page, lens, q_len, dtype):
    c = Cache(len(lens), Hk, D, page, -(-max(lens) // page) + 1, seed=D + page)
    c.write(lens)
    c.attend(q_len, Hk * G, dtype)
    c.attend(q_len, Hk * G, dtype, extra=3, with_lse=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,D,q", [(1, 64, 2), (4, 64, 2), (8, 32, 50), (16, 128, 50), (2, 12, 1)])
def test_pools_at_any_address(offset, D, q, dtype):
    c = Cache(2, 2, D, 16, 8, seed=offset)
    for i in range(2):
        x = c.dev[i]
        c.dev[i] = torch.zeros(x.numel() + offset, dtype=torch.uint8, device="cuda")[offset:].view(x.shape)
        c.dev[i].copy_(x)
    c.write([100, 37], dtype)
    c.write([1, 20], dtype)
    c.check()
    c.attend([q, q + 1], 4, dtype)


def test_lengths_beyond_the_table_and_unwritten_slots():
    """A length is taken as max_pages pages at most; what unwritten slots hold
    (NaN codes) does not count."""
    c = Cache(2, 1, 16, 16, 2, seed=5)
    for x in c.codes:
        x[:] = 127
    c.dev = [torch.from_numpy(x).cuda() for x in (*c.codes, *c.scale)]
    c.write([20, 32])
    c.attend([2, 1], 2, "bf16")
    off, q = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.ones((2, 2, 16), device="cuda")
    attn = ams.make_attn(2, 1, 16, "f32")
    ws = torch.empty(ams.ams_cache_workspace(attn, c.cache, 2, 2), dtype=torch.uint8, device="cuda")
    outs = []
    for n in (32, 2_000_000_000):
        out = torch.zeros((2, 2, 16), device="cuda")
        ams.ams_cache_attn(attn, c.cache, off, torch.tensor([20, n], dtype=torch.int32, device="cuda"),
                           torch.from_numpy(c.table).cuda(), q, *c.arrays(), out, ws)
        outs.append(out)
    assert torch.equal(*outs) and torch.isfinite(outs[0]).all()


def test_shared_pages():
    """Two samples that read one history's pages get what each alone gets."""
    c = Cache(2, 2, 32, 16, 4, seed=6)
    c.write([60, 0])
    c.table[1], c.len[1] = c.table[0], 60
    c.attend([3, 2], 4, "bf16")


def test_codes_beyond_32_bit_offsets():
    """A pool of 2.4 GB of codes: the pages at its end."""
    Hk, D, P, n = 8, 128, 128, 18_500
    cache = ams.make_cache(Hk, D, P, 1, n)
    kc, vc = (torch.zeros((n, Hk, P, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((n, Hk), device="cuda") for _ in range(2))
    table = torch.tensor([[n - 1]], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    k = torch.ones((2, Hk, D), device="cuda")
    v = torch.stack([torch.full((Hk, D), 1.0), torch.full((Hk, D), 3.0)]).cuda()
    print("cache beyond 32 bits", flush=True)
    ams.ams_cache_write(cache, off, torch.zeros(1, dtype=torch.int32, device="cuda"), table, k, v, kc, ks, vc, vs)
    attn = ams.make_attn(Hk, Hk, D, "f32")
    ws = torch.empty(ams.ams_cache_workspace(attn, cache, 1, 2), dtype=torch.uint8, device="cuda")
    out = torch.zeros((2, Hk, D), device="cuda")
    ams.ams_cache_attn(attn, cache, off, off[1:], table, k, kc, ks, vc, vs, out, ws)
    assert (out == 2.0).all()
    assert int(kc[:-1].max()) == 0 and int(vc[:-1].max()) == 0


def test_captured_serving_step():
    """Append and attend captured once, replayed for token after token with the
    lengths advanced between replays: bit-equal to eager calls on a second pool."""
    a, b = Cache(3, 2, 64, 16, 6, seed=7), Cache(3, 2, 64, 16, 6, seed=7)
    for c in (a, b):
        c.write([15, 40, 7], "bf16")
    attn = ams.make_attn(8, 2, 64, "bf16")
    off = torch.arange(4, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(a.table).cuda()
    start = torch.from_numpy(a.len).cuda()
    total = start + 1
    x = [torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]
    ws = [torch.empty(ams.ams_cache_workspace(attn, a.cache, 3, 3), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(c, out, w):
        ams.ams_cache_write(c.cache, off, start, table, *x, *c.arrays(), c.status)
        ams.ams_cache_attn(attn, c.cache, off, total, table, q, *c.arrays(), out, w)

    kept = [t.clone() for t in a.dev]
    step(a, outs[0], ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, outs[0], ws[0])
    for t, s in zip(a.dev, kept):
        t.copy_(s)
    for k in range(20):
        g = torch.Generator().manual_seed(k)
        for t in (*x, q):
            t.copy_((torch.randn(t.shape, generator=g) * 2.0 ** (k % 5)).to(t.dtype))
        step(b, outs[1], ws[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(*outs), k
        assert all(torch.equal(s, t) for s, t in zip(a.dev, b.dev)), k
        start.add_(1)
        total.add_(1)
