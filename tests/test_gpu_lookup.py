"""Token lookups and their gradient against float64 sums.

Tolerances, derived: the float32 forward is one rounded product (equal to
numpy's); the bf16 forward rounds that product once more, 2^-24 + 2^-8 of the
value.  A gradient row of m tokens is m - 1 rounded additions in some order and
one product: m 2^-24 (1 + 2^-20) of the sum of the terms' magnitudes."""
import numpy as np
import pytest
import torch

from paper_1711_06505_amd import ams

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_ids(kind, n, rows, rng):
    if kind == "same":
        return np.full(n, rows // 2, np.int32)
    if kind == "distinct":
        return rng.permutation(rows)[:n].astype(np.int32)
    if kind == "runs":          # runs that end at, before and behind multiples of 64 and 256
        ids = np.repeat(np.arange(n), rng.choice([1, 2, 63, 64, 65, 255, 256, 257], n))[:n]
        return rng.permutation(ids.astype(np.int32) % rows)
    p = 1.0 / np.arange(1, rows + 1) ** 1.1
    return rng.permutation(rows)[rng.choice(rows, n, p=p / p.sum())].astype(np.int32)


def strided(x, extra, offset):
    """The rows of x inside a wider buffer that starts `offset` elements late."""
    n, D = x.shape
    flat = torch.full((n * (D + extra) + offset + 8,), 7.0, dtype=x.dtype, device="cuda")
    v = flat[offset:offset + n * (D + extra)].view(n, D + extra)[:, :D]
    v.copy_(x)
    return v


def dedup(ids, rows):
    n = ids.numel()
    i32 = lambda m: torch.full((m,), -9, dtype=torch.int32, device="cuda")      # noqa: E731
    d = dict(uniq=i32(max(n, 1)), inv=i32(max(n, 1)), perm=i32(max(n, 1)), off=i32(n + 1), nu=i32(1), status=i32(1))
    ws = torch.empty(max(ams.ams_dedup_workspace(n, rows), 256), dtype=torch.uint8, device="cuda")
    ams.ams_dedup(ids, rows, d["uniq"], d["inv"], d["perm"], d["off"], d["nu"], d["status"], ws)
    return d


def backward(ids, rows, dout, scale, pad_id, D):
    d, n = dedup(ids, rows), ids.numel()
    nu = int(d["nu"].item())
    grad = torch.full((nu + 2, D), -5.0, device="cuda")
    ws = torch.empty(ams.ams_lookup_workspace(n, D), dtype=torch.uint8, device="cuda")
    ams.ams_lookup_bwd(d["uniq"], d["inv"], d["perm"], d["off"], d["nu"], nu, dout, grad, ws, scale, pad_id)
    torch.cuda.synchronize()
    assert (grad[nu:] == -5.0).all()
    return d["uniq"][:nu].cpu().numpy(), grad[:nu].double().cpu().numpy()


def check_backward(ids, rows, dout, scale, pad_id):
    n, D = dout.shape
    print(f"lookup bwd n={n} D={D} {dout.dtype} ld={dout.stride(0)}", flush=True)
    uniq, grad = backward(torch.from_numpy(ids).cuda(), rows, dout, scale, pad_id, D)
    x = dout.double().cpu().numpy()
    want_u, inv, count = np.unique(ids, return_inverse=True, return_counts=True)
    np.testing.assert_array_equal(uniq, want_u)
    order = np.argsort(inv, kind="stable")
    start = np.concatenate([[0], np.cumsum(count)[:-1]])
    want = np.add.reduceat(x[order], start, axis=0) * np.float32(scale)
    mag = np.add.reduceat(np.abs(x[order]), start, axis=0) * abs(np.float32(scale))
    live = (want_u != pad_id)[:, None]
    tol = count[:, None] * U32 * mag * (1 + 2.0 ** -20)
    assert (np.abs(grad - want * live) <= tol * live).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,extra,offset", [
    (1, 1, 0, 0), (1, 12, 0, 0), (63, 3, 0, 0), (64, 12, 4, 0), (65, 32, 0, 1), (1000, 5, 3, 2), (777, 100, 0, 0),
    (300, 257, 7, 3), (129, 2048, 8, 0), (65, 4100, 0, 0), (20011, 64, 0, 0), (70001, 2, 0, 0)])
def test_forward(n, D, extra, offset, dtype):
    rng = np.random.default_rng(n * 31 + D)
    rows, scale, pad = max(50, n // 3), np.float32(D ** 0.5), 3
    ids = rng.integers(-2, rows + 2, n).astype(np.int32)      # some outside the table
    T = strided(torch.from_numpy(rng.standard_normal((rows, D)).astype(np.float32)).to(DT[dtype]).cuda(), extra, offset)
    out = strided(torch.zeros((n + 1, D), dtype=DT[dtype], device="cuda"), extra, offset)
    out.fill_(-3.0)
    print(f"lookup fwd n={n} D={D} {dtype}", flush=True)
    ams.ams_lookup_fwd(torch.from_numpy(ids).cuda(), T, out, float(scale), pad)
    torch.cuda.synchronize()
    live = ((ids >= 0) & (ids < rows) & (ids != pad))[:, None]
    t = T.float().cpu().numpy()[np.clip(ids, 0, rows - 1)]
    got = out.double().cpu().numpy()
    assert (got[n] == -3.0).all()                              # the row behind the last token
    if dtype == "f32":
        np.testing.assert_array_equal(got[:n].astype(np.float32), np.where(live, t * scale, np.float32(0)))
    else:
        want = t.astype(np.float64) * np.float64(scale) * live
        assert (np.abs(got[:n] - want) <= np.abs(want) * (U16 + U32)).all()


def test_forward_rows_beyond_32_bit_offsets():
    T = torch.zeros((2_300_000, 1024), dtype=torch.bfloat16, device="cuda")       # 2.4e9 elements
    T[-1] = 2.0
    T[2_097_152] = 3.0                                                             # element 2^31
    ids = torch.tensor([2_299_999, 0, 2_097_152], dtype=torch.int32, device="cuda")
    out = torch.empty((3, 1024), dtype=torch.bfloat16, device="cuda")
    print("lookup fwd beyond 32 bits", flush=True)
    ams.ams_lookup_fwd(ids, T, out, 0.5)
    assert (out.float().cpu() == torch.tensor([1.0, 0.0, 1.5])[:, None]).all()


def test_nothing_to_look_up():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    out = torch.full((2, 4), 5.0, device="cuda")
    ams.ams_lookup_fwd(e, torch.ones((3, 4), device="cuda"), out)
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert (out == 5.0).all()
    ams.ams_lookup_fwd(ids, torch.empty((0, 4), device="cuda"), out)               # a table without rows
    assert (out == 0.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,n,rows,D,extra,offset", [
    ("zipf", 1, 5, 12, 0, 0), ("zipf", 2, 5, 1, 0, 0), ("same", 64, 9, 3, 0, 0), ("same", 65, 9, 4, 0, 0),
    ("distinct", 500, 600, 2, 1, 0), ("zipf", 1000, 300, 1, 0, 0), ("runs", 5000, 4000, 12, 0, 0),
    ("runs", 7001, 8000, 5, 2, 1), ("runs", 3000, 3000, 64, 0, 0), ("zipf", 4097, 1000, 100, 4, 0),
    ("same", 20000, 3, 257, 0, 0), ("zipf", 3001, 900, 2048, 0, 0), ("runs", 140_001, 140_001, 7, 0, 0),
    ("same", 200_000, 3, 16, 0, 0), ("zipf", 150_000, 20_000, 32, 0, 0), ("runs", 131_072, 9000, 128, 0, 8)])
def test_backward(kind, n, rows, D, extra, offset, dtype):
    rng = np.random.default_rng(n + D)
    ids = make_ids(kind, n, rows, rng)
    x = strided(torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).to(DT[dtype]).cuda(), extra, offset)
    check_backward(ids, rows, x, D ** 0.5, -1)


def test_backward_skips_padding():
    """Padded tokens give no gradient, whatever their upstream rows hold."""
    rng = np.random.default_rng(5)
    ids = make_ids("zipf", 5000, 200, rng)
    ids[::3] = 0
    x = rng.standard_normal((5000, 24)).astype(np.float32)
    x[::3] = np.nan
    x = np.where((ids == 0)[:, None], np.nan, x).astype(np.float32)
    uniq, grad = backward(torch.from_numpy(ids).cuda(), 200, torch.from_numpy(x).cuda(), 2.0, 0, 24)
    assert uniq[0] == 0 and (grad[0] == 0).all() and np.isfinite(grad).all()


def test_backward_below_the_unique_count_stays_in_its_buffer():
    """Rows past n_uniq_cap are dropped; the rows below it are complete."""
    rng = np.random.default_rng(6)
    ids = make_ids("zipf", 4000, 900, rng)
    d = dedup(torch.from_numpy(ids).cuda(), 900)
    x = torch.from_numpy(rng.integers(-8, 9, (4000, 20)).astype(np.float32)).cuda()      # integers: sums are exact
    cap = 100
    grad = torch.full((cap + 1, 20), -5.0, device="cuda")
    ws = torch.empty(ams.ams_lookup_workspace(4000, 20), dtype=torch.uint8, device="cuda")
    print("lookup bwd below the unique count", flush=True)
    ams.ams_lookup_bwd(d["uniq"], d["inv"], d["perm"], d["off"], d["nu"], cap, x, grad, ws)
    uniq = np.unique(ids)[:cap]
    want = np.stack([x.cpu().numpy()[ids == u].sum(0) for u in uniq])
    np.testing.assert_array_equal(grad[:cap].cpu().numpy(), want)
    assert (grad[cap] == -5.0).all()


def test_training_step_of_a_table_in_a_graph():
    """Lookup, sorted tokens, gradient and the Adagrad rows, captured once and
    replayed on new tokens: bit-equal to the eager calls each time."""
    rng = np.random.default_rng(7)
    n, rows, D = 3000, 500, 24
    table0 = torch.from_numpy(rng.standard_normal((rows, D)).astype(np.float32)).cuda()
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    dout = torch.zeros((n, D), device="cuda")
    i32 = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")      # noqa: E731
    d = dict(uniq=i32(n), inv=i32(n), perm=i32(n), off=i32(n + 1), nu=i32(1), status=i32(1))
    dws = torch.empty(ams.ams_dedup_workspace(n, rows), dtype=torch.uint8, device="cuda")
    ws = torch.empty(ams.ams_lookup_workspace(n, D), dtype=torch.uint8, device="cuda")

    def step(table, accum, out, grad):
        ams.ams_lookup_fwd(ids, table, out, 2.0)
        ams.ams_dedup(ids, rows, d["uniq"], d["inv"], d["perm"], d["off"], d["nu"], d["status"], dws)
        ams.ams_lookup_bwd(d["uniq"], d["inv"], d["perm"], d["off"], d["nu"], n, dout, grad, ws, 2.0)
        ams.ams_adagrad_rows(d["uniq"], d["nu"], n, grad, table, accum, 0.05, 1e-8)

    def buffers():
        return table0.clone(), torch.zeros_like(table0), torch.zeros((n, D), device="cuda"), \
            torch.zeros((n, D), device="cuda")

    eager, captured = buffers(), buffers()
    step(*buffers())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for x, y in zip(captured, buffers()):
        x.copy_(y)
    for k in range(4):
        ids.copy_(torch.from_numpy(make_ids("zipf", n, rows, rng)))
        dout.copy_(torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)))
        step(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        nu = int(d["nu"].item())
        for x, y, rows_of in zip(eager, captured, (rows, rows, n, nu)):
            assert torch.equal(x[:rows_of], y[:rows_of]), k


def test_gradient_twice_is_the_same():
    """Fixed orders: the same bits again, hot rows over many chunks included."""
    rng = np.random.default_rng(9)
    ids = torch.from_numpy(make_ids("zipf", 150_000, 700, rng)).cuda()
    x = torch.from_numpy(rng.standard_normal((150_000, 24)).astype(np.float32)).cuda()
    first, again = (backward(ids, 700, x, 1.5, -1, 24)[1] for _ in range(2))
    np.testing.assert_array_equal(first, again)


def test_on_another_stream():
    rng = np.random.default_rng(8)
    T = torch.from_numpy(rng.standard_normal((100, 16)).astype(np.float32)).cuda()
    ids = torch.from_numpy(make_ids("zipf", 900, 100, rng)).cuda()
    a, b = torch.zeros((900, 16), device="cuda"), torch.zeros((900, 16), device="cuda")
    ams.ams_lookup_fwd(ids, T, a, 3.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ams.ams_lookup_fwd(ids, T, b, 3.0, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
