"""Batches large enough for the kernels that small ones never reach: one wave
per tile of rows (many samples with short lists), and grids that walk several
tiles a block (a few larger samples behind hundreds of small ones).  Against
float64, with the bounds of attn_ref."""
import numpy as np
import pytest

from test_gpu_cache import Cache
from test_gpu_xattn import Problem

pytestmark = pytest.mark.gpu


def lens(seed, n, lo, hi):
    return np.random.default_rng(seed).integers(lo, hi + 1, n).tolist()


@pytest.mark.parametrize("q,H,Hk,D,dtype,extra", [
    ((18, 32), 4, 4, 16, "f32", 0), ((18, 32), 4, 4, 64, "bf16", 0),       # two row tiles a wave
    ((5, 8), 16, 4, 64, "bf16", 0), ((5, 8), 16, 4, 32, "f32", 0),         # of grouped heads
    ((1, 16), 4, 4, 12, "f32", 0), ((1, 16), 4, 4, 12, "bf16", 0), ((1, 10), 4, 4, 128, "bf16", 0),
    ((18, 32), 4, 4, 20, "bf16", 1)])
def test_short_lists(q, H, Hk, D, dtype, extra):
    """300 samples of 0..60 keys; some of them masked in every second case."""
    Problem(lens(1, 300, *q), lens(2, 300, 0, 60), H, Hk, D, dtype, extra=extra, drop=0.1 * (D != 64), seed=D).check()


@pytest.mark.parametrize("D,dtype,extra", [(16, "f32", 0), (64, "f32", 0), (100, "f32", 0), (64, "f32", 1),
                                           (64, "bf16", 0), (128, "bf16", 0), (33, "bf16", 0)])
def test_short_lists_of_more_rows(D, dtype, extra):
    """Gradients where samples have more rows than one pass takes, and lists too short for shared tiles."""
    Problem(lens(3, 300, 33, 45), lens(4, 300, 0, 60), 4, 4, D, dtype, extra=extra, drop=0.1, seed=D).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q,D,page", [((1, 1), 64, 16), ((1, 2), 20, 32), ((17, 22), 64, 16), ((17, 20), 128, 16),
                                      ((17, 20), 33, 64)])
def test_short_histories_in_pages(q, D, page, dtype):
    """130 samples of 8 key heads, each wave a tile of its own."""
    n = lens(5, 130, 0, 40)
    c = Cache(130, 8, D, page, -(-40 // page), seed=D)
    c.write(n, dtype)
    c.attend(lens(6, 130, *q), 8, dtype)


@pytest.mark.parametrize("D,dtype", [(16, "f32"), (64, "bf16"), (12, "bf16"), (128, "f32")])
def test_larger_samples_behind_many_small_ones(D, dtype):
    """1600 blocks of work in a grid of 1024: the larger samples' tiles come in a block's second round."""
    Problem(lens(7, 400, 0, 2) + [90, 0, 70, 40], lens(8, 400, 0, 30) + [80, 5, 0, 200], 4, 4, D, dtype, drop=0.1,
            seed=D).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_larger_samples_behind_long_lists(dtype):
    """The same with the keys in two shares."""
    Problem([1] * 197 + [50, 1, 120], lens(9, 200, 500, 620), 4, 4, 16, dtype, seed=5).check()
