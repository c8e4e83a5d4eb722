"""The sequence operators of the library, timed as a training or serving program
calls them: behavior tokens looked up in an embedding table, queries (candidate
ads) that attend to a user's behavior states, and the same attention over
states kept in 8 bits.

Three kinds of calls, twelve listed cases, and draw() for more of the same
kinds and ranges:

  lookup  rows of an embedding table times a scale, one per token; in training
          also the tokens' sorted order and the merged gradient of every
          touched row
  attend  multi-head attention of each sample's queries to that sample's keys,
          lists of different lengths; in training also the gradients of the
          queries, keys and values
  cache   keys and values written into 8-bit pages, with one scale for each
          page and head, and/or queries attending to what the pages hold

`own` False computes them from elementary torch operations, True calls the
library.  Sizes are those of the library's own workloads (1024 samples with
10..100 behaviors, 4096 samples with lists of mean 200 capped at 500, ID
tables of 10,000 to 10,000,000 rows, requests of 37 candidates) and generic
ones for wider heads and longer histories.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------ cases

def _lookup(n, D, rows, zipf, dtype, train, pad):
    """pad: the share of the tokens that are padding (their ID is row 0)."""
    return {"kind": "lookup", "n": n, "D": D, "rows": rows, "zipf": zipf, "dtype": dtype, "train": train, "pad": pad}


def _attend(B, q_lo, q_hi, k_law, k_lo, k_hi, heads, kv_heads, dim, dtype, train, drop):
    """Queries per sample uniform in [q_lo, q_hi]; keys "uniform" in [k_lo, k_hi]
    or "geometric" with mean k_lo capped at k_hi; drop: share of masked keys."""
    return {"kind": "attend", "B": B, "q_lo": q_lo, "q_hi": q_hi, "k_law": k_law, "k_lo": k_lo, "k_hi": k_hi,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "train": train, "drop": drop}


def _cache(B, page, k_lo, k_hi, new, q_lo, q_hi, heads, kv_heads, dim, dtype):
    """B samples that hold uniform [k_lo, k_hi] tokens after the call; of these
    `new` (-1: all) are written by it.  Then q_lo..q_hi queries attend (q_hi 0: none)."""
    return {"kind": "cache", "B": B, "page": page, "k_lo": k_lo, "k_hi": k_hi, "new": new, "q_lo": q_lo,
            "q_hi": q_hi, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype}


def listed():
    return [
        # The ad IDs of a serving batch: the smallest call, launch latency counts.
        {"name": "lookup_1024_f32", **_lookup(1024, 12, 10_000, 1.05, "f32", False, 0.0)},
        # A training step's behavior IDs over a large ID table, forward and merged row gradients.
        {"name": "lookup_train_823k_f32", **_lookup(823_191, 32, 1_000_000, 1.05, "f32", True, 0.0)},
        # Wide bf16 token embeddings in padded batches, forward and gradient.
        {"name": "lookup_train_64k_bf16", **_lookup(65_536, 2048, 50_000, 1.05, "bf16", True, 0.15)},
        # One request: 37 candidates against one user's hundred behaviors, latency counts.
        {"name": "attend_37_f32", **_attend(1, 37, 37, "uniform", 100, 100, 4, 4, 16, "f32", False, 0.0)},
        # The float32 training step: one ad per sample, 10..100 behaviors, heads of image-embedding width.
        {"name": "attend_train_1024_f32", **_attend(1024, 1, 1, "uniform", 10, 100, 4, 4, 12, "f32", True, 0.0)},
        # Long behavior lists with some behaviors masked, up to 8 ads a sample, grouped heads.
        {"name": "attend_train_4096_bf16", **_attend(4096, 1, 8, "geometric", 200, 500, 8, 2, 64, "bf16", True, 0.1)},
        # One query a sample over very long histories: work has to be split along the keys.
        {"name": "attend_long_bf16", **_attend(3, 1, 1, "uniform", 60_000, 100_000, 8, 8, 128, "bf16", False, 0.0)},
        # Long query and key sequences, wide grouped heads: the largest call, bound by matrix products.
        {"name": "attend_train_8x2048_bf16",
         **_attend(8, 1024, 2048, "uniform", 2048, 4096, 16, 4, 128, "bf16", True, 0.0)},
        # Histories of a batch of users written into empty pages.
        {"name": "cache_write_64_bf16", **_cache(64, 32, 100, 2000, -1, 0, 0, 8, 4, 64, "bf16")},
        # A few users' serving step: one token appended, one query each; latency counts.
        {"name": "cache_step_3_f32", **_cache(3, 16, 40, 130, 1, 1, 1, 4, 2, 32, "f32")},
        # A serving step of a batch: one token appended, one query each over long grouped-head pages.
        {"name": "cache_step_32_bf16", **_cache(32, 64, 512, 4096, 1, 1, 1, 32, 8, 128, "bf16")},
        # Candidates of several users ranked against their cached histories.
        {"name": "cache_rank_24_bf16", **_cache(24, 32, 200, 4000, 0, 20, 60, 8, 2, 64, "bf16")},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8])
    return kv * rng.choice([1, 1, 2, 4]), kv


def draw(rng):
    kind = rng.choice(["lookup", "attend", "attend", "cache"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "lookup":
        D = rng.choice([12, rng.randint(1, 64), _log(rng, 64, 4096)])
        n = _log(rng, 1, min(1_000_000, 134_000_000 // D))
        rows = _log(rng, 100, min(10_000_000, 2_000_000_000 // D))
        return _lookup(n, D, rows, rng.choice([0.0, 1.05, 1.1]), dtype, rng.random() < 0.6, rng.choice([0.0, 0.15]))
    heads, kv = _draw_heads(rng)
    dim = rng.choice([12, 16, 32, 64, 128, rng.randint(4, 128)])
    if kind == "cache":
        page = rng.choice([16, 32, 64, 128])
        B = _log(rng, 1, 64)
        hi = _log(rng, 8, max(16, min(16_000, 90_000_000 // (B * kv * dim))))
        lo = rng.randint(1, hi)
        new = rng.choice([-1, 0, 1, rng.randint(1, lo)])
        q = rng.choice([1, 1, _log(rng, 1, 60)])
        return _cache(B, page, lo, hi, new, 1 if new != -1 else 0, q if new != -1 else 0, heads, kv, dim, dtype)
    train = rng.random() < 0.6
    B = _log(rng, 1, 4096)
    k_hi = _log(rng, 4, max(8, min(60_000, 60_000_000 // (B * kv * dim))))
    q_hi = min(_log(rng, 1, 2000), max(1, 200_000_000 // (B * k_hi * heads)), max(1, 30_000_000 // (B * heads * dim)))
    drop = rng.choice([0.0, 0.0, 0.1])
    if k_hi >= 40 and rng.random() < 0.4:
        return _attend(B, 1, q_hi, "geometric", max(8, k_hi // 3), k_hi, heads, kv, dim, dtype, train, drop)
    least = 0 if B >= 8 else 1
    return _attend(B, rng.randint(least, q_hi), q_hi, "uniform", rng.randint(least, k_hi), k_hi, heads, kv, dim, dtype,
                   train, drop)


# ------------------------------------------------------- sizes and work

@functools.lru_cache(maxsize=64)
def _n_unique(rows, zipf, n):
    """Expected number of distinct IDs among n draws."""
    p = np.arange(1, rows + 1, dtype=np.float64) ** (-zipf)
    p /= p.sum()
    return float(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _mean_keys(case):
    if case.get("k_law") != "geometric":
        return (case["k_lo"] + case["k_hi"]) / 2
    p = 1.0 / case["k_lo"]
    return (1 - (1 - p) ** case["k_hi"]) / p


def work(case):
    e = _size(case)
    if case["kind"] == "lookup":
        n, D = case["n"], case["D"]
        u = _n_unique(case["rows"], case["zipf"], n)
        byts, flops = 4 * n + e * D * u + e * n * D, n * D
        if case["train"]:       # the IDs' sorted order; upstream rows in, one float32 row per touched row out
            byts, flops = byts + 4 * n + 4 * u + e * n * D + 4 * u * D, flops + n * D
        return {"bytes": float(byts), "flops": float(flops)}
    B, H, Hk, D = case["B"], case["heads"], case["kv_heads"], case["dim"]
    nk, nq = B * _mean_keys(case), B * (case["q_lo"] + case["q_hi"]) / 2
    pairs = nq * _mean_keys(case) * H
    if case["kind"] == "attend":
        byts, flops = e * D * (2 * nq * H + 2 * nk * Hk), 4 * pairs * D
        if case["train"]:
            byts, flops = byts + e * D * (4 * nq * H + 4 * nk * Hk), flops + 10 * pairs * D
        return {"bytes": float(byts), "flops": float(flops)}
    new = nk if case["new"] < 0 else B * case["new"]
    byts, flops = new * Hk * D * 2 * (e + 1), 4 * new * Hk * D
    if case["q_hi"]:
        byts, flops = byts + nk * Hk * D * 2 + 2 * e * nq * H * D, flops + 4 * pairs * D
    return {"bytes": float(byts), "flops": float(flops)}


# ----------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(g, dtype, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g).to(dtype)


def _ids(g, n, rows, zipf, pad):
    """n int32 IDs in [1, rows), Zipf by rank; a share of them row 0 (padding).
    The ranks are the same for every seed, so the number of distinct IDs is
    too; the seed scatters them over the table and over the batch."""
    fixed, m = _gen(n), max(1, rows - 1)
    cdf = torch.arange(1, m + 1, device="cuda", dtype=torch.float64).pow_(-zipf).cumsum_(0)
    u = torch.rand(n, generator=fixed, device="cuda", dtype=torch.float64) * cdf[-1]
    rank = torch.searchsorted(cdf, u).clamp_max_(m - 1)
    padded = torch.rand(n, generator=fixed, device="cuda") < pad
    ids = torch.randperm(m, generator=g, device="cuda", dtype=torch.int32)[rank] + 1
    ids = torch.where(padded, torch.zeros_like(ids), ids).clamp_max_(rows - 1)
    return ids[torch.randperm(n, generator=g, device="cuda")]


def _lengths(g, B, law, lo, hi):
    """The same lengths for every seed, in another order."""
    fixed = _gen(B)
    if law == "geometric":
        u = torch.rand(B, generator=fixed, device="cuda", dtype=torch.float64)
        n = (torch.log1p(-u) / math.log1p(-1.0 / lo)).floor_().long().add_(1).clamp_(1, hi)
    else:
        n = torch.randint(lo, hi + 1, (B,), generator=fixed, device="cuda")
    return n[torch.randperm(B, generator=g, device="cuda")]


def _offsets(n):
    off = torch.zeros(n.numel() + 1, dtype=torch.int64, device="cuda")
    torch.cumsum(n, 0, out=off[1:])
    return off.int()


def prepare(case, seed):
    g = _gen(seed)
    dt = _dtype(case)
    st = {"case": case}
    if case["kind"] == "lookup":
        n, D = case["n"], case["D"]
        st["ids"] = _ids(g, n, case["rows"], case["zipf"], case["pad"])
        st["pad_id"] = 0 if case["pad"] else -1
        st["scale"] = math.sqrt(D)
        st["table"] = torch.empty((case["rows"], D), dtype=dt, device="cuda").normal_(std=D ** -0.5, generator=g)
        if case["train"]:
            st["dout"] = _normal(g, dt, n, D)
            st["n_u"] = int(torch.unique(st["ids"]).numel())    # the rows of the answer that hold something
    else:
        B, H, Hk, D = case["B"], case["heads"], case["kv_heads"], case["dim"]
        q_len = _lengths(g, B, "uniform", case["q_lo"], case["q_hi"])
        k_len = _lengths(g, B, case.get("k_law", "uniform"), case["k_lo"], case["k_hi"])
        st["q_off"], st["max_q"], st["max_k"] = _offsets(q_len), int(q_len.max()), int(k_len.max())
        n_q, n_k = int(q_len.sum()), int(k_len.sum())
        st["q"] = _normal(g, dt, n_q, H, D)
        st["scale"] = D ** -0.5
        if case["kind"] == "attend":
            st["k_off"] = _offsets(k_len)
            st["k"], st["v"] = _normal(g, dt, n_k, Hk, D), _normal(g, dt, n_k, Hk, D)
            st["mask"] = (torch.rand(n_k, generator=g, device="cuda") >= case["drop"]).to(torch.uint8) \
                if case["drop"] else None
            if case["train"]:
                st["dout"] = _normal(g, dt, n_q, H, D)
        else:
            _prepare_cache(case, st, g, k_len)
    _prepare_plan(case, st)
    return st


def _prepare_cache(case, st, g, k_len):
    """Pages of every sample scattered over the pool (a few pages belong to
    nobody); what is there before the call has the scale that its page's
    largest value asks for, slots not yet written hold code 0."""
    B, Hk, D, P = case["B"], case["kv_heads"], case["dim"], case["page"]
    max_pages = -(-case["k_hi"] // P)
    n_pages = B * max_pages + 3
    perm = torch.randperm(n_pages, generator=g, device="cuda", dtype=torch.int32)
    st["page_table"] = perm[:B * max_pages].view(B, max_pages).contiguous()
    st["len"] = k_len.int()
    new = k_len if case["new"] < 0 else torch.full_like(k_len, case["new"])
    st["start"] = (k_len - new).int()
    st["new_off"], st["max_new"] = _offsets(new), int(new.max())
    n_new = int(new.sum())
    st["k"], st["v"] = _normal(g, _dtype(case), n_new, Hk, D), _normal(g, _dtype(case), n_new, Hk, D)
    pos = torch.arange(max_pages * P, device="cuda")
    held = torch.zeros((n_pages, P), dtype=torch.bool, device="cuda")
    held[st["page_table"].long()] = (pos[None] < st["start"][:, None]).view(B, max_pages, P)
    for name in ("k", "v"):
        x = _normal(g, torch.float32, n_pages, Hk, P, D).mul_(held[:, None, :, None])
        s = _scale_of(x.abs().amax((2, 3)))
        st[name + "_codes"] = (x / s[..., None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        st[name + "_scale"] = s


def _prepare_plan(case, st):
    """What a program allocates once for calls of these sizes: outputs and a workspace."""
    dev = "cuda"
    if case["kind"] == "lookup":
        n, D = case["n"], case["D"]
        st["out"] = torch.empty((n, D), dtype=_dtype(case), device=dev)
        if case["train"]:
            i32 = functools.partial(torch.empty, dtype=torch.int32, device=dev)
            st.update(uniq=i32(n), inv=i32(n), perm=i32(n), off=i32(n + 1), n_uniq=i32(1), status=i32(1),
                      grad=torch.empty((n, D), dtype=torch.float32, device=dev))
    else:
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=dev)
        st["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
        if case.get("train"):
            st.update(dq=torch.empty_like(st["q"]), dk=torch.empty_like(st["k"]), dv=torch.empty_like(st["v"]))
    if own:
        st.update(_plan_own(case, st))


def _plan_own(case, st):
    """The library's shapes and workspace for these sizes."""
    from paper_1711_06505_amd import ams
    if case["kind"] == "lookup":
        need = max(ams.ams_dedup_workspace(case["n"], case["rows"]),
                   ams.ams_lookup_workspace(case["n"], case["D"])) if case["train"] else 0
        plan = {}
    else:
        plan = {"attn": ams.make_attn(case["heads"], case["kv_heads"], case["dim"], case["dtype"])}
        if case["kind"] == "attend":
            need = ams.ams_xattn_workspace(plan["attn"], case["B"], st["q"].shape[0], st["k"].shape[0])
        else:
            plan["cache"] = ams.make_cache(case["kv_heads"], case["dim"], case["page"], st["page_table"].shape[1],
                                           st["k_codes"].shape[0])
            need = ams.ams_cache_workspace(plan["attn"], plan["cache"], case["B"], st["q"].shape[0])
    plan["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return plan


# -------------------------------------------------------------------- run

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"lookup": _own_lookup, "attend": _own_attend, "cache": _own_cache}[kind](state)
    return {"lookup": _plain_lookup, "attend": _plain_attend, "cache": _plain_cache}[kind](state)


def _own_lookup(st):
    from paper_1711_06505_amd import ams
    c = st["case"]
    ams.ams_lookup_fwd(st["ids"], st["table"], st["out"], st["scale"], st["pad_id"])
    if not c["train"]:
        return st["out"]
    ams.ams_dedup(st["ids"], c["rows"], st["uniq"], st["inv"], st["perm"], st["off"], st["n_uniq"], st["status"],
                  st["ws"])
    ams.ams_lookup_bwd(st["uniq"], st["inv"], st["perm"], st["off"], st["n_uniq"], c["n"], st["dout"], st["grad"], st["ws"],
                       st["scale"], st["pad_id"])
    return st["out"], st["uniq"][:st["n_u"]], st["grad"][:st["n_u"]]


def _own_attend(st):
    from paper_1711_06505_amd import ams
    ams.ams_xattn_fwd(st["attn"], st["q_off"], st["k_off"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["ws"],
                      key_mask=st["mask"])
    if not st["case"]["train"]:
        return st["out"]
    ams.ams_xattn_bwd(st["attn"], st["q_off"], st["k_off"], st["q"], st["k"], st["v"], st["out"], st["lse"],
                      st["dout"], st["dq"], st["dk"], st["dv"], st["ws"], key_mask=st["mask"])
    return st["out"], st["dq"], st["dk"], st["dv"]


def _own_cache(st):
    from paper_1711_06505_amd import ams
    c, outs = st["case"], []
    if c["new"]:
        ams.ams_cache_write(st["cache"], st["new_off"], st["start"], st["page_table"], st["k"], st["v"],
                            st["k_codes"], st["k_scale"], st["v_codes"], st["v_scale"], st["status"])
        outs = [_values(st["k_codes"]), st["k_scale"], _values(st["v_codes"]), st["v_scale"]]
    if c["q_hi"]:
        ams.ams_cache_attn(st["attn"], st["cache"], st["q_off"], st["len"], st["page_table"], st["q"],
                           st["k_codes"], st["k_scale"], st["v_codes"], st["v_scale"], st["out"], st["ws"])
        outs.append(st["out"])
    return outs


def _values(codes):
    """Codes as the 8-bit values they stand for (times their page's scale: the entry)."""
    return codes.view(torch.float8_e4m3fn)


# ------------------------------------------------------------ plain forms

def _plain_lookup(st):
    c, ids = st["case"], st["ids"].long()
    live = (ids != st["pad_id"])[:, None]
    out = torch.where(live, st["table"][ids].float() * st["scale"], 0.0).to(st["table"].dtype)
    if not c["train"]:
        return out
    # tokens sorted by ID; a row's sum is a difference of prefix sums, which 32 bits would not hold
    tokens, order = torch.sort(ids, stable=True)
    last = torch.nonzero(torch.cat([tokens[1:] != tokens[:-1], torch.ones_like(tokens[:1], dtype=torch.bool)]))[:, 0]
    sums = torch.where(live, st["dout"].double() * st["scale"], 0.0)[order].t().contiguous().cumsum_(1)[:, last]
    sums[:, 1:] -= sums[:, :-1].clone()
    return out, tokens[last].int(), sums.t().float().contiguous()


def _padded(x, off, most):
    """[B, most, ...] float32 rows of each list, and which of them are real."""
    pos = off[:-1, None].long() + torch.arange(most, device="cuda")
    real = pos < off[1:, None]
    return x[pos.clamp_max(max(x.shape[0] - 1, 0))].float(), real


def _unpadded(x, real):
    return x[real]


def _plain_attend(st):
    c = st["case"]
    B, H, Hk, D, dt = c["B"], c["heads"], c["kv_heads"], c["dim"], _dtype(c)
    if not st["q"].shape[0] or not st["k"].shape[0]:
        z = [torch.zeros_like(st[x]) for x in "qkv"]
        return (z[0].clone(), *z) if c["train"] else z[0]
    q, q_real = _padded(st["q"], st["q_off"], st["max_q"])
    k, live = _padded(st["k"], st["k_off"], st["max_k"])
    v, k_real = _padded(st["v"], st["k_off"], st["max_k"])
    if st["mask"] is not None:
        live = live & (_padded(st["mask"], st["k_off"], st["max_k"])[0] > 0)
    k, v = (torch.where(live[:, :, None, None], x, 0.0).transpose(1, 2) for x in (k, v))
    rows = lambda x: torch.where(q_real[:, :, None, None], x, 0.0).view(B, st["max_q"], Hk, H // Hk, D) \
        .permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)                                # noqa: E731
    back = lambda x: _unpadded(x.view(B, Hk, st["max_q"], H // Hk, D).permute(0, 2, 1, 3, 4)
                               .reshape(B, st["max_q"], H, D), q_real).to(dt)        # noqa: E731
    q = rows(q)
    p = _softmax((q @ k.transpose(2, 3)) * st["scale"], live)
    out = back(p @ v)
    if not c["train"]:
        return out
    do = rows(_padded(st["dout"], st["q_off"], st["max_q"])[0])
    dv = p.transpose(2, 3) @ do
    dp = do @ v.transpose(2, 3)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * st["scale"]
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    return out, back(dq), _unpadded(dk.transpose(1, 2), k_real).to(dt), _unpadded(dv.transpose(1, 2), k_real).to(dt)


def _softmax(s, live):
    """Over the last axis, among the keys that are there; a row without any is 0."""
    s = torch.where(live[:, None, None], s, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    return e / e.sum(-1, keepdim=True).clamp_min(1e-37)


def _scale_of(most):
    """The least power of two (2^-100 at least) whose product with 448, the
    largest 8-bit value, reaches `most`."""
    m, e = torch.frexp(most.float())                     # most = m 2^e with m in [0.5, 1); 448 = 0.875 2^9
    return _power_of_two((e - 9 + (m > 0.875).int()).clamp_min(-100).masked_fill(most == 0, -100))


def _power_of_two(e):
    """2^e in 32 bits, by its exponent field (torch.ldexp and exp2 may be off by a rounding)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _plain_cache(st):
    c, outs = st["case"], []
    codes = [st["k_codes"], st["v_codes"]]
    scales = [st["k_scale"], st["v_scale"]]
    if c["new"]:
        pairs = [_plain_write(st, a, b, x) for a, b, x in zip(codes, scales, (st["k"], st["v"]))]
        codes, scales = zip(*pairs)
        outs = [_values(codes[0]), scales[0], _values(codes[1]), scales[1]]
    if c["q_hi"]:
        outs.append(_plain_cache_attend(st, codes, scales))
    return outs


def _plain_write(st, codes, scale, x):
    """Each touched page gets the scale that its new tokens ask for, if that is
    larger; what it held is rounded to the new scale."""
    P, n = st["case"]["page"], x.shape[0]
    pos = torch.arange(n, device="cuda")
    i = torch.searchsorted(st["new_off"][1:].long(), pos, right=True)
    at = st["start"][i].long() + pos - st["new_off"][i].long()
    page = st["page_table"][i, at // P].long()
    n_pages, Hk = scale.shape
    most = torch.zeros((n_pages, Hk), device="cuda").index_reduce_(0, page, x.float().abs().amax(2), "amax")
    pos_in = torch.arange(P, device="cuda")
    first = torch.full((n_pages,), P, device="cuda").index_reduce_(0, page, at % P, "amin")
    touched = (first < P)[:, None]
    fresh = torch.where((first == 0)[:, None], _scale_of(most), torch.maximum(scale, _scale_of(most)))
    new_scale = torch.where(touched, fresh, scale)
    grown = (pos_in < first[:, None])[:, None, :, None] & touched[:, :, None, None]
    old = _values(codes).float()
    ratio = (scale / new_scale)[:, :, None, None]
    old = torch.where(grown, old * ratio, old)
    old[page, :, at % P] = x.float() / new_scale[page][..., None]
    return old.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), new_scale


def _plain_cache_attend(st, codes, scales):
    c = st["case"]
    B, H, Hk, D, P = c["B"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    table = st["page_table"].long()
    live = torch.arange(table.shape[1] * P, device="cuda") < st["len"][:, None]
    k, v = ((_values(x)[table].float() * s[table][..., None, None]).transpose(1, 2).reshape(B, Hk, -1, D)
            for x, s in zip(codes, scales))
    q, real = _padded(st["q"], st["q_off"], st["max_q"])
    q = q.view(B, st["max_q"], Hk, H // Hk, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)
    k, v = (torch.where(live[:, None, :, None], x, 0.0) for x in (k, v))
    out = _softmax((q @ k.transpose(2, 3)) * st["scale"], live) @ v
    out = out.view(B, Hk, st["max_q"], H // Hk, D).permute(0, 2, 1, 3, 4).reshape(B, st["max_q"], H, D)
    return _unpadded(out, real).to(_dtype(c))


# ------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"lookup": _exact_lookup, "attend": _exact_attend, "cache": _exact_cache}[case["kind"]](st)


def _exact_lookup(st):
    """One-hot rows summed by autograd: the lookup is out = scale (1 - padded) table[ids]."""
    ids = st["ids"].long()
    uniq, inv = torch.unique(ids, return_inverse=True)
    rows = st["table"][uniq].double().requires_grad_(True)
    factor = st["scale"] * (ids != st["pad_id"]).double()
    out = rows.index_select(0, inv) * factor[:, None]
    if not st["case"]["train"]:
        return out.detach()
    (grad,) = torch.autograd.grad(out, rows, st["dout"].double())
    return out.detach(), uniq.int(), grad


def _exact_one(q, k, v, scale):
    """softmax(scale q k^T) v of one sample by query head ([queries, H, D], [keys, Hk, D])."""
    G = q.shape[1] // k.shape[1]
    s = torch.einsum("qhd,khd->hqk", q, k.repeat_interleave(G, 1)) * scale
    return torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v.repeat_interleave(G, 1))


def _exact_attend(st):
    c = st["case"]
    q_off, k_off = st["q_off"].tolist(), st["k_off"].tolist()
    q, k, v = (st[x].double() for x in "qkv")
    do = st["dout"].double() if c["train"] else None
    out, dq, dk, dv = (torch.zeros_like(x) for x in (q, q, k, v))
    for i in range(c["B"]):
        rows = slice(q_off[i], q_off[i + 1])
        keys = torch.arange(k_off[i], k_off[i + 1], device="cuda")
        if st["mask"] is not None:
            keys = keys[st["mask"][keys] > 0]
        if not keys.numel() or rows.start == rows.stop:
            continue
        leaves = [x.requires_grad_(c["train"]) for x in (q[rows].clone(), k[keys], v[keys])]
        o = _exact_one(*leaves, st["scale"])
        out[rows] = o.detach()
        if c["train"]:
            dq[rows], dk[keys], dv[keys] = torch.autograd.grad(o, leaves, do[rows])
    return (out, dq, dk, dv) if c["train"] else out


def _round_e4m3(x):
    """To 4 significant bits (multiples of 2^-9 below 2^-6), ties to even, at most 448."""
    _, e = torch.frexp(x)
    step = (((e - 4).clamp_min(-9).long() + 1023) << 52).view(torch.float64)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_scale(most):
    """The first of the powers of two from 2^-100 on that is enough."""
    powers = torch.tensor([2.0 ** e for e in range(-100, 121)], dtype=torch.float64, device=most.device)
    return powers[torch.searchsorted(powers * 448, most.double().contiguous())]


def _exact_cache(st):
    c, P = st["case"], st["case"]["page"]
    table, start, length = st["page_table"].tolist(), st["start"].tolist(), st["len"].tolist()
    new_off, q_off = st["new_off"].tolist(), st["q_off"].tolist()
    held = [[_values(st[n + "_codes"]).double(), st[n + "_scale"].double()] for n in "kv"]
    if c["new"]:
        for (codes, scale), x in zip(held, (st["k"].double(), st["v"].double())):
            for i in range(c["B"]):
                for p in range(start[i] // P, -(-length[i] // P)):
                    lo, hi = max(start[i], p * P), min(length[i], (p + 1) * P)
                    if lo >= hi:
                        continue
                    page, t0, t1 = table[i][p], lo - p * P, hi - p * P
                    rows = x[new_off[i] + lo - start[i]:new_off[i] + hi - start[i]].transpose(0, 1)
                    s = _exact_scale(rows.abs().amax((1, 2)))
                    if t0:
                        s = torch.maximum(s, scale[page])
                        codes[page, :, :t0] = _round_e4m3(codes[page, :, :t0] * (scale[page] / s)[:, None, None])
                    codes[page, :, t0:t1] = _round_e4m3(rows / s[:, None, None])
                    scale[page] = s
    outs = [held[0][0], held[0][1], held[1][0], held[1][1]] if c["new"] else []
    if c["q_hi"]:
        q = st["q"].double()
        out = torch.zeros_like(q)
        for i in range(c["B"]):
            rows, n = slice(q_off[i], q_off[i + 1]), length[i]
            if not n or rows.start == rows.stop:
                continue
            pages = torch.tensor(table[i][:-(-n // P)], device="cuda")
            k, v = ((codes[pages] * scale[pages][..., None, None]).permute(0, 2, 1, 3).reshape(-1, *codes.shape[1::2])[:n]
                    for codes, scale in held)
            out[rows] = _exact_one(q[rows], k, v, st["scale"])
        outs.append(out)
    return outs
