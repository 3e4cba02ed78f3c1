"""Softmax attention on the GPU: values that are not finite, unusual documents, steep slopes, and what a training call keeps of its outputs."""
import numpy as np
import pytest
import torch

from tests import softmax_reference as R
from tests.test_gpu_softmax import DT, check, lib, make, route  # noqa: F401

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
MODIFIERS = [(cap, bias, mask) for cap in (0.0, 20.0) for bias in ("none", "slopes", "table") for mask in ("full", "causal", "prefix")]


def outputs_only(lib, x, how, what=""):
    """The call that keeps nothing for a backward pass: kernels of its own in bf16."""
    api, _, ctx = lib
    want = R.reference(x["q"], x["k"], x["v"], **how)
    R.assert_close(api.softmax_attn(ctx, x["q"], x["k"], x["v"], **how), want["out"], want["out_tol"], what + "out")
    return want


def unseen_by_all(x, how):
    """(keys that no query sees [B, nk], queries that see no key [B, nq])"""
    B, _, nq, _ = x["q"].shape
    host = {n: how[n].cpu() for n in ("k_len", "q_start", "prefix", "q_doc", "k_doc") if n in how}
    see, _ = R.visible(B, nq, x["k"].shape[2], how["mask"], **host)
    return torch.from_numpy(~see.any(1)).cuda(), torch.from_numpy(~see.any(2)).cuda()


def spoil_unseen(lib, x, how, dout, what):
    """Outputs and gradients with NaN and infinities in all that nobody sees, against 64 bits."""
    keys, queries = unseen_by_all(x, how)
    assert keys.any()
    for bad in (NAN, INF):
        for t in (x["k"], x["v"]):
            t.masked_fill_(keys[:, None, :, None], bad)
        for t in (x["q"], dout):
            t.masked_fill_(queries[:, None, :, None], bad)
        check(lib, x, how, dout, f"{what}, {bad}: ")
        outputs_only(lib, x, how, f"{what}, {bad}, nothing kept: ")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias,mask", MODIFIERS)
def test_unseen_values_in_every_kernel(lib, route, cap, bias, mask, d):  # noqa: F811
    """What a token holds that nobody sees does not matter, with and without caps, biases and orders."""
    for nq in (150, 6):
        spoil_unseen(lib, *make(53, 2, 4, 2, nq, 300, d, "bf16", mask=mask, bias=bias, cap=cap, ragged=True), f"{nq} queries")


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("nq,start", [(150, False), (300, False), (200, True)])
@pytest.mark.parametrize("docs", ["few", "many", "unsorted"])
@pytest.mark.parametrize("cap,bias,mask", [(0.0, "none", "full"), (20.0, "slopes", "causal"), (0.0, "table", "prefix")])
def test_unseen_values_of_documents(lib, route, cap, bias, mask, docs, nq, start, dtype, d):  # noqa: F811
    """Among them keys of documents that no query is of, and those behind the last query of theirs."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    x, how, dout = make(103, 2, 4, 2, nq, 300, d, dtype, mask=mask, bias=bias, cap=cap, docs=docs, start=start)
    if start:
        how["q_doc"] = how["q_doc"].roll(37, 1).contiguous()
    spoil_unseen(lib, x, how, dout, "")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("docs", ["few", "many", "unsorted"])
@pytest.mark.parametrize("cap,bias,mask", [(0.0, "table", "full"), (20.0, "none", "causal"), (0.0, "slopes", "prefix")])
def test_negative_documents(lib, route, dtype, docs, cap, bias, mask):  # noqa: F811
    """Any negative document is none: tokens of equal negative numbers, the lowest one among them, do not see one another."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    for nq in (300, 8):
        x, how, dout = make(59, 2, 2, 1, nq, 300, 64, dtype, mask=mask, bias=bias, cap=cap, docs=docs)
        g = torch.Generator().manual_seed(2)
        for name in ("q_doc", "k_doc"):
            ids = how[name].cpu()
            none = torch.tensor([-1, -7, -2**31, -2**31], dtype=torch.int32)[torch.randint(0, 4, ids.shape, generator=g)]
            how[name] = torch.where((ids < 0) | (torch.rand(ids.shape, generator=g) < 0.1), none, ids).cuda()
        check(lib, x, how, dout, f"{nq} queries: ")
        for t, ids in ((x["k"], "k_doc"), (x["v"], "k_doc"), (dout, "q_doc")):
            t.masked_fill_((how[ids] < 0)[:, None, :, None], NAN)
        check(lib, x, how, dout, f"{nq} queries, NaN in padding: ")


@pytest.mark.parametrize("nq,nk", [(40, 40), (150, 170)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias,mask", [(0.0, "none", "full"), (0.0, "none", "causal"), (5.0, "none", "causal"), (0.0, "table", "full"), (0.0, "slopes", "prefix")])
def test_rest_holds_what_rounding_took(lib, cap, bias, mask, nq, nk, d):  # noqa: F811
    """out + rest comes from probabilities of 2^-16: within a bound that probabilities rounded to bf16 do not meet."""
    api, _, ctx = lib
    x, how, _ = make(61, 2, 2, 1, nq, nk, d, "bf16", mask=mask, bias=bias, cap=cap)
    want = R.reference(x["q"], x["k"], x["v"], **how)
    V = np.repeat(x["v"].double().cpu().numpy(), 2, 1)
    r, size = R.HALF_STEP[torch.bfloat16], want["P"] @ np.abs(V)
    # the bound of out without the roundings of P and of out, for which each leaves a rounding of its own remainder: r r
    bound = want["out_tol"] - r * size - r * np.abs(want["out"]) + r * r * (size + np.abs(want["out"]))
    rounded = torch.from_numpy(want["P"] / want["P"].max(-1, keepdims=True)).bfloat16().double().numpy() * want["P"].max(-1, keepdims=True)
    assert (np.abs(rounded @ V - want["out"]) > bound).sum() > 20
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    R.assert_close(out.double() + saved.rest.double(), want["out"], bound, "out + rest")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("mask", ["causal", "prefix"])
def test_rest_of_rows_that_are_summed_again(lib, mask, cap, d):  # noqa: F811
    """An infinity in a value that a row does not see, in a tile that it does: the row's out + rest is as good as without."""
    api, _, ctx = lib
    nq = nk = 120
    x, how, _ = make(67, 1, 2, 1, nq, nk, d, "bf16", mask=mask, cap=cap)
    if mask == "prefix":
        how["prefix"].fill_(30)
    want = R.reference(x["q"], x["k"], x["v"], **how)
    V = np.repeat(x["v"].double().cpu().numpy(), 2, 1)
    r, size = R.HALF_STEP[torch.bfloat16], want["P"] @ np.abs(V)
    bound = want["out_tol"] - r * size - r * np.abs(want["out"]) + r * r * (size + np.abs(want["out"]))
    v = x["v"].clone()
    v[0, 0, nk - 1, ::3] = INF                          # seen by the last query alone
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], v, want_lse=True, **how)
    assert not out[0, :, -1, ::3].isfinite().any()
    both = (out.double() + saved.rest.double())[:, :, :-1]
    R.assert_close(both, want["out"][:, :, :-1], bound[:, :, :-1], "out + rest")


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_lse_of_a_call_without_rest(lib, scale):  # noqa: F811
    """lse as fp32 sums of fp32 exponentials, where all of a row's weight lies on one or two keys, whichever they are."""
    api, B, ctx = lib
    nq = nk = 128
    d = 128
    q, k = torch.zeros(1, 1, nq, d), torch.zeros(1, 1, nk, d)
    q[0, 0, :, 0] = 1 + torch.arange(nq) / 128.0        # products of eight bits by eight: exact in fp32
    pair = torch.arange(nk) // 2
    v = torch.randn(1, 1, nk, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    for first in range(64):
        k[0, 0, :, 0] = torch.where(pair == first, 1.5 + (torch.arange(nk) & 1) * 0.75, torch.tensor(-30.0))
        qc, kc = q.bfloat16().cuda(), k.bfloat16().cuda()
        want = R.reference(qc, kc, v, scale=scale)
        s = api._softmax_desc(ctx, qc, kc, v, scale, 0.0, "full", None, None, None, None, None, None, None, None, False)
        out, lse = torch.empty_like(v), torch.empty(1, 1, nq, device="cuda")
        B.grf_softmax_attn(ctx.handle, s, qc, kc, v, out, lse, None, None, 0)
        R.assert_close(out, want["out"], want["out_tol"], "out")
        # scores below 16 in units of log 2, three roundings; an exponential of 2^-22; a logarithm and two roundings of lse below 8
        R.assert_close(lse, want["lse"], 3 * 8 * R.U + 2.0**-22 + 3 * 8 * R.U, f"lse, keys {2 * first} and the next")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [5, 300])
@pytest.mark.parametrize("mask", ["causal", "full"])
@pytest.mark.parametrize("slope", [1.0e4, 1.0e6, 1.0e37, 3.0e38])
def test_steep_slopes(lib, route, dtype, mask, nq, slope):  # noqa: F811
    """Slopes so steep that a query is left with its own position: that score is not rounded to the steps of the others' biases."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    api, _, ctx = lib
    d = 64
    x, _, dout = make(71, 1, 2, 1, nq, 300, d, dtype)
    how = {"mask": mask, "slopes": torch.full((2,), slope, device="cuda")}
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    Q, K, V, G = (t.double().cpu().numpy() for t in (x["q"], x["k"], x["v"], dout))
    own = slice(300 - nq, 300)
    s = (Q * K[:, :, own]).sum(-1) * d ** -0.5
    e = (d + 8) * R.U * ((np.abs(Q) * np.abs(K[:, :, own])).sum(-1) * d ** -0.5 + np.abs(s) + 1)
    R.assert_close(saved.lse, s, 2 * e, "lse")
    r = R.HALF_STEP[DT[dtype]]
    R.assert_close(out, np.broadcast_to(V[:, :, own], out.shape), 4 * e[..., None] * np.abs(V[:, :, own]) + 1e-30, "out")
    dq, dk, dv, _ = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], out, saved, dout, **how)
    # P = 1 within the error of s - lse, then rounded; dv of a key: the two heads' dout of its query
    want = np.zeros(V.shape)
    want[:, 0, own] = G.sum(1)
    bound = np.zeros(V.shape)
    bound[:, 0, own] = ((4 * e[..., None] + r) * np.abs(G)).sum(1) + (r + 8 * R.U) * np.abs(G.sum(1))
    R.assert_close(dv, want, bound, "dv")
    # dS = P (dP - D) of two sums of the same products
    ds = (4 * d * R.U) * (np.abs(G) * np.abs(V[:, :, own])).sum(-1) + 1e-30
    assert (np.abs(dq.double().cpu().numpy()) <= (1 + 2 * r) * ds[..., None] * d ** -0.5 * np.abs(K[:, :, own]) + 1e-30).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("d", [40, 128])
def test_rows_whose_scores_are_all_lowest(lib, route, dtype, cap, d):  # noqa: F811
    """Queries that only see keys with a bias of -infinity, in tiles that they see whole: nothing of theirs reaches a gradient, NaN neither."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    api, _, ctx = lib
    nq, nk = 256, 64
    x, how, dout = make(73, 1, 2, 1, nq, nk, d, dtype, cap=cap)
    how.update(first=[0, 200], table=torch.tensor([[0.5, -INF], [1.0, -INF]], dtype=DT[dtype], device="cuda"), two_sided=False,
               q_start=torch.tensor([100], dtype=torch.int32, device="cuda"))
    o, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    want = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], o, saved, dout, **how)
    gone = torch.arange(nq) >= 163
    assert torch.equal(saved.lse[0, 0].cpu() == -INF, gone) and (o[:, :, 163:] == 0).all()
    dout[:, :, 163:] = NAN
    dout[:, :, 170:] = INF
    for y, z in zip(api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], o, saved, dout, **how), want):
        assert torch.equal(y, z)
    if cap:                                             # (a cap makes an infinite product finite, and -infinity of it still)
        k, clean = x["k"].abs(), dout.clone()
        clean[:, :, 163:] = 0
        ref = R.reference(x["q"], k, x["v"], clean, **how)
        o, saved = api.softmax_attn(ctx, x["q"], k, x["v"], want_lse=True, **how)
        q = x["q"].clone()
        q[:, :, 180:] = INF
        for name, y in zip(("dq", "dk", "dv", "dtable"), api.softmax_attn_backward(ctx, q, k, x["v"], o, saved, dout, **how)):
            # (out and lse are the kernel's: each bound counts once more)
            R.assert_close(y, ref[name], 2 * ref[name + "_tol"], name)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("who", ["q", "k"])
def test_gradients_of_infinite_capped_scores(lib, route, dtype, bad, who):  # noqa: F811
    """A value that is not finite in what is seen leaves no finite gradient beside it: 0 times infinity is NaN."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    api, _, ctx = lib
    x, how, dout = make(79, 2, 2, 1, 100, 100, 64, dtype, mask="causal", cap=10.0)
    x[who][0, 0, 50, 7] = bad
    o = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    dq, dk, dv, _ = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *o, dout, **how)
    if who == "k":
        assert not dq[0, :, 50:, 7].isfinite().any()
    else:
        assert not dk[0, 0, :51, 7].isfinite().any()
    assert dq[1].isfinite().all() and dk[1].isfinite().all() and dv[1].isfinite().all()


INFERENCE = [(19, 8, 4, 150, 170, 128), (1, 2, 1, 300, 300, 96), (2, 4, 2, 129, 500, 128), (1, 3, 1, 257, 255, 64), (2, 2, 2, 70, 70, 24)]


@pytest.mark.parametrize("shape", INFERENCE, ids=str)
@pytest.mark.parametrize("cap,bias,mask", MODIFIERS)
def test_outputs_only(lib, shape, cap, bias, mask):  # noqa: F811
    """Calls that keep nothing for a backward pass, which bf16 has kernels of its own for."""
    for more in (dict(), dict(ragged="empty", start=True), dict(docs="few")):
        x, how, _ = make(83, *shape, "bf16", mask=mask, bias=bias, cap=cap, **more)
        outputs_only(lib, x, how, f"{more}: ")
    for scale in (-0.1, 0.0):
        x, how, _ = make(89, *shape, "bf16", mask=mask, bias=bias, cap=cap)
        outputs_only(lib, x, dict(how, scale=scale), f"scale {scale}: ")


@pytest.mark.parametrize("mask", ["full", "causal"])
def test_outputs_only_of_long_rows(lib, mask):  # noqa: F811
    """The plain call at d = 128, some of whose exponentials are sums of products: over sharp rows and flat ones."""
    for sharp in (0.1, 1.5, 12.0):
        x, how, _ = make(97, 1, 2, 1, 300, 2000, 128, "bf16", mask=mask)
        x["q"] = (x["q"].float() * sharp).bfloat16()
        outputs_only(lib, x, how, f"times {sharp}: ")


def test_refusals_of_the_backward_calls(lib):  # noqa: F811
    """What the library refuses is its error in every call, whoever brings the workspace."""
    api, B, ctx = lib
    x, how, dout = make(101, 1, 2, 1, 20, 20, 136, "bf16")
    with pytest.raises(B.GrfError) as e:
        api.softmax_attn(ctx, x["q"], x["k"], x["v"])
    assert e.value.code == B.GRF_ERR_INVALID
    saved = api.SoftmaxSaved(torch.zeros(1, 2, 20, device="cuda"), None)
    with pytest.raises(B.GrfError) as e:
        api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], x["q"], saved, dout)
    assert e.value.code == B.GRF_ERR_INVALID
    with pytest.raises(B.GrfError) as e:
        api.relative_bias_backward(ctx, torch.zeros(2, 20, 20, device="cuda"), list(range(65)))
    assert e.value.code == B.GRF_ERR_INVALID
    x, how, dout = make(101, 1, 2, 1, 20, 20, 64, "bf16")
    with pytest.raises(ValueError):
        api.softmax_attn(ctx, x["q"], x["k"], x["v"], mask="casual")


def test_waits_beside_rows_that_are_summed_again(lib):  # noqa: F811
    """Every multiprocessor sums all rows of its first block again, over 2^18 keys, while its other warps wait with the second."""
    api, B, ctx = lib
    H, nq, nk, d = 148, 512, 1 << 18, 128
    g = torch.Generator(device="cuda").manual_seed(6)
    q = torch.randn(1, H, nq, d, device="cuda", generator=g).bfloat16()
    k, v = (torch.randn(1, 1, nk, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    for x in range(4):                                  # the last key of a tile, seen by that tile's last query and later ones; a column in either half
        v[0, 0, nk - 1 - 128 * x, [x, 64 + x]] = INF
    torch.cuda.synchronize()
    at = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    at[0].record()
    out = api.softmax_attn(ctx, q, k, v, mask="causal")
    at[1].record()
    torch.cuda.synchronize()
    B.grf_ctx_check(ctx.handle)
    print(f"{at[0].elapsed_time(at[1]):.1f} ms")
    for h, i in ((0, 0), (1, 100), (70, 254), (71, 383), (147, 510), (147, 511)):
        s = (k[0, 0].double() @ q[0, h, i].double()) * d ** -0.5
        s[nk - nq + i + 1:] = -INF
        p = torch.softmax(s, 0)
        w = v[0, 0].double()
        sees = (w[:nk - nq + i + 1] == INF).any(0)
        clean = torch.where(w.isfinite(), w, 0.0)
        want, size = p @ clean, p @ clean.abs()
        assert torch.equal(out[0, h, i] == INF, sees) and int(sees.sum()) == 2 * ((i + 1) // 128)
        # P and out to bf16; scores, of a size of 8 or less, and sums in 32 bits
        bound = size * (2 * 2.0**-8 + 2.0**-16) + 1e-9
        assert ((out[0, h, i].double() - want).abs() <= bound)[~sees].all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("mask", ["causal", "prefix"])
def test_unseen_values_behind_the_last_query(lib, route, mask, cap, d):  # noqa: F811
    """Keys behind the last query, in blocks of keys that earlier ones are seen in, where the last block of queries is not full."""
    for seed, nq, nk in ((1, 95, 225), (2, 8, 100), (3, 234, 444), (4, 128, 300)):
        x, how, dout = make(seed, 3, 2, 1, nq, nk, d, "bf16", mask=mask, cap=cap)
        how["q_start"] = torch.tensor([0, nk // 3, nk - nq - 5], dtype=torch.int32, device="cuda")
        if mask == "prefix":
            how["prefix"].clamp_(max=nk // 4)
        spoil_unseen(lib, x, how, dout, f"{nq} queries, {nk} keys")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [3, 140])
def test_numbers_at_the_ends_of_their_range(lib, route, dtype, nq):  # noqa: F811
    """Starts, lengths, prefixes and documents of any 32 bits."""
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    low, high = -2**31, 2**31 - 1
    ends = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for mask in ("full", "causal", "prefix"):
        for bias, buckets in (("none", (32, 128)), ("table", (32, 128)), ("table", (64, 1 << 24))):
            x, how, dout = make(107, 6, 2, 1, nq, 150, 64, dtype, mask=mask, bias=bias, buckets=buckets)
            if mask == "prefix":
                how["prefix"] = ends(low, high, 0, 40, high, low)
            how["q_start"] = ends(low, high, -nq // 2, 100, low, high)
            how["k_len"] = ends(high, high, 150, high, 70, low)
            check(lib, x, how, dout, f"{mask} {bias}: ")
            g = torch.Generator().manual_seed(1)
            ids = ends(low, -1, 0, 1, high - 1, high)
            pick = lambda n: ids[torch.randint(0, 6, (6, n), generator=g).cuda()]  # noqa: E731
            x, how, dout = make(109, 6, 2, 1, nq, 150, 64, dtype, mask=mask, bias=bias, buckets=buckets)
            check(lib, x, dict(how, q_doc=pick(nq), k_doc=pick(150)), dout, f"{mask} {bias} documents: ")
