"""Softmax attention over ordered tokens in 64 bits, with its gradients and how far a kernel may be from them.

Bounds, with u = 2^-24 (a rounding to fp32) and r = half a step of the storage type (bf16: 2^-8; fp32: 0, its own roundings are in the sums
of u below), to first order and times 2 for what is left out:
  scores   a sum of d products, scaled, capped (slope at most 1), a bias added, turned into units of log 2 and back:
           e_ij = (d + 8) u (scale sum |q||k| + |bias| + |s| + cap)
  P        one exponential of s - lse; lse's error is a mean of the e over the row and (n + 4) u:  f_i = 2 max_j e_ij + (n + 8) u (1 + |lse|), relative
  out      sum P (f + r) |v| + n u sum P |v| + r |out|        (the products take P rounded to storage)
  dS       f |dS| + P (d u sum |dout||v| + d u sum |dout||out| + r sum |dout||out|)      (out is given in storage)
  dX       the slope 1 - t^2 of the cap, t = c / cap off by e / cap + 4 u:  |dS| 2 |t| (e / cap + 4 u) + error of dS, then rounded: r |dX|
  dQ, dK   scale sum (error of dX) |k| + n u sum |dX||k| + r |dQ|, the same for dK; dV like out; dtable sum of dS errors + N u sum |dS|."""
import math

import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


def bucket(first, delta, two_sided):
    n = np.abs(delta) if two_sided else np.maximum(-delta, 0)
    b = np.searchsorted(np.asarray(first), n, side="right") - 1
    return b + (delta > 0) * len(first) if two_sided else b


def visible(B, nq, nk, mask="full", k_len=None, q_start=None, prefix=None, q_doc=None, k_doc=None):
    """bool [B, nq, nk] and relative positions [B, nq, nk]."""
    start = np.full(B, nk - nq, np.int64) if q_start is None else np.asarray(q_start, np.int64)
    p = start[:, None] + np.arange(nq)
    j = np.arange(nk)
    delta = j[None, None, :] - p[:, :, None]
    see = np.ones((B, nq, nk), bool) if mask == "full" else delta <= 0
    if mask == "prefix":
        see = see | (j[None, :] < np.asarray(prefix)[:, None])[:, None, :]
    if k_len is not None:
        see = see & (j[None, :] < np.asarray(k_len)[:, None])[:, None, :]
    if q_doc is not None:
        q_doc, k_doc = np.asarray(q_doc), np.asarray(k_doc)
        see = see & (q_doc[:, :, None] == k_doc[:, None, :]) & (q_doc[:, :, None] >= 0)
    return see, delta


def _host(x):
    return None if x is None else x.detach().cpu().double().numpy()


def reference(q, k, v, dout=None, scale=None, cap=0.0, mask="full", k_len=None, q_start=None, prefix=None, q_doc=None, k_doc=None,
              slopes=None, table=None, first=None, two_sided=False):
    """dict of 64-bit numpy results: out, lse and, with dout, dq, dk, dv, dtable; the same with _tol: the bounds above."""
    r = HALF_STEP[q.dtype]
    cpu = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    B, H, nq, d = q.shape
    KV, nk = k.shape[1], k.shape[2]
    g = H // KV
    scale = d ** -0.5 if scale is None else scale
    see, delta = visible(B, nq, nk, mask, cpu(k_len), cpu(q_start), cpu(prefix), cpu(q_doc), cpu(k_doc))
    Q, K, V = _host(q), np.repeat(_host(k), g, 1), np.repeat(_host(v), g, 1)
    see4 = np.broadcast_to(see[:, None], (B, H, nq, nk))
    # what nobody sees does not matter, whatever it holds
    used_k, used_q = see.any(1)[:, None, :, None], see.any(2)[:, None, :, None]
    Q, K, V = np.where(used_q, Q, 0.0), np.where(used_k, K, 0.0), np.where(used_k, V, 0.0)
    z = scale * (Q @ K.transpose(0, 1, 3, 2))
    z_abs = abs(scale) * (np.abs(Q) @ np.abs(K).transpose(0, 1, 3, 2))
    t = np.tanh(z / cap) if cap else np.zeros_like(z)
    c = cap * t if cap else z
    bias = np.zeros((1, 1, 1, 1))
    if table is not None:
        T = _host(table)
        bias = T[:, bucket(first, delta, two_sided)].transpose(1, 0, 2, 3)
    elif slopes is not None:
        bias = -_host(slopes)[None, :, None, None] * np.abs(delta)[:, None]
    s = np.where(see4, c + bias, -np.inf)
    top = s.max(-1, keepdims=True)
    top = np.where(np.isneginf(top), 0.0, top)
    e = np.exp(s - top)
    total = e.sum(-1, keepdims=True)
    P = e / np.where(total == 0, 1.0, total)
    with np.errstate(divide="ignore"):
        lse = np.where(total[..., 0] > 0, top[..., 0] + np.log(total[..., 0]), -np.inf)
    out = P @ V
    err = (d + 8) * U * (z_abs + np.where(np.isfinite(bias), np.abs(bias), 0.0) + np.where(see4 & np.isfinite(s), np.abs(s), 0.0) + cap)
    f = 2 * np.where(see4, err, 0.0).max(-1, keepdims=True) + (nk + 8) * U * (1 + np.abs(np.where(np.isfinite(lse), lse, 0.0)))[..., None]
    ans = {"out": out, "lse": lse, "P": P, "see": see,
           "out_tol": 2 * ((f + nk * U) * (P @ np.abs(V))) + r * (P @ np.abs(V)) + r * np.abs(out) + 1e-30,
           "lse_tol": 2 * (f[..., 0])}
    if dout is None:
        return ans
    G = np.where(used_q, _host(dout), 0.0)
    dP = G @ V.transpose(0, 1, 3, 2)
    D = (G * out).sum(-1, keepdims=True)
    dS = P * (dP - D)
    G_out = (np.abs(G) * np.abs(out)).sum(-1, keepdims=True)
    dS_err = f * np.abs(dS) + P * (d * U * (np.abs(G) @ np.abs(V).transpose(0, 1, 3, 2) + G_out) + r * G_out)
    dX = dS * (1 - t * t) if cap else dS
    dX_err = dS_err + (np.abs(dS) * 2 * np.abs(t) * (err / cap + 4 * U) if cap else 0.0)
    share = lambda x: x.reshape(B, KV, g, *x.shape[2:]).sum(2)  # noqa: E731
    ans["dq"] = scale * (dX @ K)
    ans["dk"] = share(scale * (dX.transpose(0, 1, 3, 2) @ Q))
    ans["dv"] = share(P.transpose(0, 1, 3, 2) @ G)
    a = abs(scale)
    ans["dq_tol"] = a * ((2 * dX_err + (r + 2 * nk * U) * np.abs(dX)) @ np.abs(K)) + r * np.abs(ans["dq"]) + 1e-30
    ans["dk_tol"] = share(a * ((2 * dX_err + (r + 2 * g * nq * U) * np.abs(dX)).transpose(0, 1, 3, 2) @ np.abs(Q))) + r * np.abs(ans["dk"]) + 1e-30
    ans["dv_tol"] = share(((2 * f + r + 2 * g * nq * U) * P).transpose(0, 1, 3, 2) @ np.abs(G)) + r * np.abs(ans["dv"]) + 1e-30
    if table is not None:
        cols = T.shape[1]
        b = np.broadcast_to(bucket(first, delta, two_sided)[:, None], dS.shape)
        by = lambda x: np.stack([np.bincount(b[:, h].ravel(), x[:, h].ravel(), cols) for h in range(H)])  # noqa: E731
        ans["dtable"] = by(dS)
        ans["dtable_tol"] = by(2 * dS_err) + 2 * math.log2(B * nq * nk + 2) * 64 * U * by(np.abs(dS)) + r * np.abs(ans["dtable"]) + 1e-30
    ans["dS"] = dS
    return ans


def assert_close(got, want, tol, what):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, f"{what}: {got.shape} instead of {want.shape}"
    same = (got == want) | (np.isneginf(got) & np.isneginf(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} beyond the bound, first at {np.argwhere(bad)[0].tolist()}: "
                           f"{got[tuple(np.argwhere(bad)[0])]} for {want[tuple(np.argwhere(bad)[0])]}, bound {np.broadcast_to(tol, want.shape)[tuple(np.argwhere(bad)[0])]:.3g}")
