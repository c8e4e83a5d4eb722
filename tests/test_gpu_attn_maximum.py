"""The running maximum over a long list: keys whose scores grow (or fall) from
tile to tile of 64, for some rows and not for others, so that the sums of the
tiles before have to be scaled anew, by much, by little, or not at all.
Against float64, with the bounds of attn_ref."""
import numpy as np
import pytest
import torch

from paper_1711_06505_amd import ams
from test_gpu_cache import Cache
from test_gpu_cache_scales import attend
from test_gpu_xattn import Problem

pytestmark = pytest.mark.gpu

# a row's factor: its scores rise by factor * 0.18 * rise (base 2) a tile of 64 keys
FACTORS = np.array([0.0, 4.0, 1.0, -4.0, 0.0, 2.0, -0.5, 0.25])


def levels(n, rise):
    """Of the keys' first element: `rise` more for every tile of 64."""
    return np.arange(n) // 64 * float(rise)


def scale_of(D):
    return 0.125                              # log2(e) / 8 = 0.18 per unit of the first elements' product


@pytest.mark.parametrize("scale", [0.125, -0.125])
@pytest.mark.parametrize("rise", [32, 8, 40])
@pytest.mark.parametrize("q_len,k_len,H,Hk,D,dtype,extra", [
    ([140, 70], [461, 130], 4, 2, 64, "bf16", 0),
    ([140], [700], 2, 1, 128, "bf16", 0),
    ([130, 40], [333, 90], 2, 2, 32, "bf16", 0),
    ([150, 40], [461, 130], 2, 1, 64, "bf16", 1),          # rows that are not aligned
    ([60], [2600], 2, 1, 64, "bf16", 0),                   # the keys in shares
    ([40, 3], [461, 130], 2, 2, 64, "f32", 0),
    ([3, 1], [461, 130], 4, 2, 64, "bf16", 0),
    ([2], [2600], 2, 1, 32, "f32", 0)])
def test_keys_that_grow(q_len, k_len, H, Hk, D, dtype, extra, rise, scale):
    p = Problem(q_len, k_len, H, Hk, D, dtype, extra=extra, seed=rise + D, spread=0.5)
    p.attn.scale = scale
    n = p.q.shape[0]
    p.q[:, :, 0] = torch.from_numpy(np.resize(FACTORS, (n, H))).to(p.q.dtype).cuda()
    tops = np.concatenate([levels(b, rise) for b in k_len] + [np.zeros(p.k.shape[0] - sum(k_len))])
    p.k[:, :, 0] = torch.from_numpy(tops)[:, None].to(p.k.dtype).cuda()
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.125, -0.125])
@pytest.mark.parametrize("rise", [32, 8, 40])
@pytest.mark.parametrize("q,G,D,page,lens", [
    (130, 1, 64, 16, [461, 130]), (60, 4, 128, 32, [300, 461]), (140, 1, 32, 128, [333, 64]),
    (110, 1, 64, 64, [2600]), (2, 2, 64, 16, [461, 130])])
def test_pages_that_grow(q, G, D, page, lens, rise, scale, dtype):
    c = Cache(len(lens), 1, D, page, -(-max(lens) // page), seed=rise + D)
    tops = np.concatenate([levels(b, rise) for b in lens])

    def rows(rng, shape):
        x = rng.standard_normal(shape) * 0.5
        if rows.keys:
            x[:, :, 0] = tops[:, None]
        rows.keys = False                                  # the values come second
        return x
    rows.keys = True
    c.write(lens, dtype, make=rows)
    n = q * len(lens)
    x = torch.from_numpy(c.rng.standard_normal((n, G, D)) * 0.5)
    x[:, :, 0] = torch.from_numpy(np.resize(FACTORS, (n, G)))
    attend(c, [q] * len(lens), G, dtype, scale, x)
