"""The lookup gradient around 262144 tokens, from where on a wave takes four
rounds of 64 of them: runs over one, several and many chunks, against float64
sums (tolerances of test_gpu_lookup)."""
import numpy as np
import pytest
import torch

from paper_1711_06505_amd import ams
from test_gpu_lookup import DT, check_backward, make_ids, strided


def test_workspace_serves_smaller_calls():
    for D in (1, 12, 2048):
        ws = [ams.ams_lookup_workspace(n, D) for n in [*range(262_000, 262_300), 400_000, 1_048_575, 1_048_576, 1_100_000]]
        assert all(b >= a for a, b in zip(ws, ws[1:])), D


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,n,rows,D,extra,offset", [
    ("runs", 262_143, 262_143, 5, 0, 0), ("runs", 262_144, 262_144, 7, 0, 0), ("runs", 300_001, 20_000, 12, 0, 0),
    ("same", 262_145, 3, 16, 0, 0), ("zipf", 280_000, 20_000, 32, 0, 0), ("zipf", 262_200, 1000, 132, 0, 0),
    ("runs", 263_000, 263_000, 136, 0, 8), ("zipf", 290_001, 300_000, 24, 1, 1), ("same", 270_000, 9, 260, 0, 0)])
def test_backward(kind, n, rows, D, extra, offset, dtype):
    rng = np.random.default_rng(n + D)
    ids = make_ids(kind, n, rows, rng)
    x = strided(torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).to(DT[dtype]).cuda(), extra, offset)
    check_backward(ids, rows, x, D ** 0.5, 1)
