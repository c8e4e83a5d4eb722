"""Attention of one sample in float64, its gradients, and bounds on what the
kernels may be off by.

u = 2^-24 (float32), h = half a step of the storage type (2^-8 for bf16; 0 for
float32, whose results are float32 already and counted with u).  With
a_ij = scale sum_d |q_id k_jd|, a score is off by at most e_s = (D + 8) u a
(D products and sums, the scale, the change to base 2, the subtraction of the
maximum or of the log-sum-exp), so a weight is off by the factor 2 e_s (its own
score and the sum's) + (n + 16) u (the sum's additions, exp2 and division),
with the row's largest e_s; call that f.  Then, every sum of n terms adding
n u of its magnitudes and h standing for each rounding to the storage type:
  out:  sum_j w |v| (f + h + n u) + (h + u) |out|
  dS:   ds = scale w (dp - delta), dp and delta off by (D + 4) u sum_d |do v| and
        by (h + (D + 4) u) sum_d |do o|, with the weight's f for the product
  dV:   sum_i w |do| (f + h + n u) + (h + u) |dV|
  dK:   sum_i (e_ds + (h + n u) |ds|) |q| + (h + u) |dK|; dQ likewise over keys.
Second-order terms: all bounds times 1.1.
A weight, or a dS, below the smallest normal number 2^-126 may be flushed to
zero (the hardware's exp2 gives no subnormal results): m = 2^-126 is added to
each weight's and each dS's own error, so it enters the results times what the
weight is multiplied by: |v|, |do|, |dp - delta| |q| ...
"""
import torch

U = 2.0 ** -24
M = 2.0 ** -126


def attention(q, k, v, do, scale, live, h):
    """[rows, D], [keys, D], [keys, D], [rows, D] float64 and live [keys]:
    (out, dq, dk, dv) and their bounds, for one query head; a row without live
    keys gives zeros."""
    keep = live.nonzero()[:, 0]
    K, V = k[keep], v[keep]
    D, n, rows = q.shape[1], K.shape[0], q.shape[0]
    dk, dv, bk, bv = (torch.zeros_like(k) for _ in range(4))
    if n == 0:
        z = torch.zeros_like(q)
        return (z, z, dk, dv), (z, z, bk, bv)
    w = torch.softmax(scale * q @ K.T, 1)
    out = w @ V
    es = (D + 8) * U * abs(scale) * (q.abs() @ K.abs().T)
    f = 2 * es.amax(1, keepdim=True) + (n + 16) * U
    b_out = w @ V.abs() * (f + h + n * U) + M * V.abs().sum(0) + (h + U) * out.abs()
    dp = do @ V.T
    delta = (do * out).sum(1, keepdim=True)
    ds = scale * w * (dp - delta)
    e_dp = (D + 4) * U * (do.abs() @ V.abs().T) + (do.abs() * b_out).sum(1, keepdim=True) \
        + (D + 4) * U * (do.abs() * out.abs()).sum(1, keepdim=True)
    e_ds = M + abs(scale) * (M * (dp - delta).abs() + w * (f * (dp - delta).abs() + e_dp))
    dq = ds @ K
    b_dq = (e_ds + (h + n * U) * ds.abs()) @ K.abs() + (h + U) * dq.abs()
    dk[keep], dv[keep] = ds.T @ q, w.T @ do
    bk[keep] = (e_ds + (h + rows * U) * ds.abs()).T @ q.abs()
    bv[keep] = (M + w * (f + h + rows * U)).T @ do.abs()
    return (out, dq, dk, dv), (b_out, b_dq, bk, bv)


def batch(q, k, v, do, q_len, k_len, scale, live, bf16):
    """All samples and heads: [n_q, H, D] and [n_k, Hk, D] arrays; a key head's
    gradients (and their bounds) are summed over its query heads."""
    h = 2.0 ** -8 if bf16 else 0.0
    q, k, v, do = (x.double().cpu() for x in (q, k, v, do))
    live = torch.ones(k.shape[0], dtype=torch.bool) if live is None else live.cpu() != 0
    G = q.shape[1] // k.shape[1]
    vals = [torch.zeros_like(x) for x in (q, q, k, v)]
    tols = [torch.zeros_like(x) for x in (q, q, k, v)]
    q0 = k0 = 0
    for nq, nk in zip(q_len, k_len):
        qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
        for head in range(q.shape[1]):
            kh = head // G
            if nq:
                # what a masked key holds does not enter
                kk, vv = (torch.where(live[ks, None], x[ks, kh], 0.0) for x in (k, v))
                x, t = attention(q[qs, head], kk, vv, do[qs, head], scale, live[ks], h)
                for i, (s, at) in enumerate(((qs, head), (qs, head), (ks, kh), (ks, kh))):
                    vals[i][s, at] += x[i]
                    tols[i][s, at] += t[i]
        q0, k0 = q0 + nq, k0 + nk
    for i in (2, 3):                          # the one rounding of the summed gradients
        tols[i] += (h + U) * vals[i].abs()
    # a float32 result below its smallest normal number may be flushed
    return vals, [1.1 * t + 1e-37 for t in tols]
