"""Softmax attention over ordered tokens on the GPU: outputs and gradients against 64 bits, at sizes and masks where they can go wrong."""
import numpy as np
import pytest
import torch

from tests import softmax_reference as R

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def lib():
    from paper_2410_03462_b200 import api, binding
    ctx = api.Context(0)
    yield api, binding, ctx
    ctx.close()


@pytest.fixture(params=["default", "alu"])
def route(request, lib):
    """bf16 once by the default kernels and once without the tensor cores."""
    api, B, ctx = lib
    B.grf_ctx_use_tensor_cores(ctx.handle, request.param == "default")
    yield request.param
    B.grf_ctx_check(ctx.handle)
    B.grf_ctx_use_tensor_cores(ctx.handle, True)


def make(seed, B, H, KV, nq, nk, d, dtype, mask="full", bias="none", cap=0.0, ragged=False, docs=None, start=False, buckets=(32, 128),
         two_sided=None, grad=True):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = {"q": (n(B, H, nq, d) * (3.0 if cap else 1.5)).to(dt).cuda(), "k": n(B, KV, nk, d).to(dt).cuda(), "v": n(B, KV, nk, d).to(dt).cuda()}
    how = {"mask": mask, "cap": cap}
    if bias == "table":
        from paper_2410_03462_b200 import api
        how["first"] = api.relative_buckets(*buckets)
        how["two_sided"] = mask == "full" if two_sided is None else two_sided
        how["table"] = n(H, buckets[0] * (2 if how["two_sided"] else 1)).to(dt).cuda()
    elif bias == "slopes":
        how["slopes"] = torch.tensor([0.5 ** (h + 1) for h in range(H)]).cuda()
    if mask == "prefix":
        how["prefix"] = torch.randint(0, nk + 1, (B,), generator=g, dtype=torch.int32).cuda()
    if ragged:
        lens = torch.randint(0, nk + 1, (B,), generator=g, dtype=torch.int32)
        lens[0] = 0 if ragged == "empty" else max(1, nk - 1)
        how["k_len"] = lens.cuda()
    if start:
        how["q_start"] = torch.randint(-3, nk + 1, (B,), generator=g, dtype=torch.int32).cuda()
    if docs:
        many = {"few": 3, "many": max(nk // 5, 1), "unsorted": 4}[docs]
        kd = torch.randint(0, many, (B, nk), generator=g, dtype=torch.int32)
        if docs != "unsorted":
            kd = kd.sort(1).values
        kd[:, nk - nk // 7:] = -1
        qd = kd if nq == nk else torch.nn.functional.pad(kd, (max(nq - nk, 0), 0), value=-1)[:, -nq:].contiguous()
        how["q_doc"], how["k_doc"] = qd.cuda(), kd.cuda()
    dout = n(B, H, nq, d).to(dt).cuda() if grad else None
    return x, how, dout


def check(lib, x, how, dout, what=""):
    api, _, ctx = lib
    want = R.reference(x["q"], x["k"], x["v"], dout, **how)
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    lse = saved.lse
    R.assert_close(out, want["out"], want["out_tol"], what + "out")
    if saved.rest is not None:      # out and its rest: the fp32 result, but for a rounding of the rest
        both = out.double() + saved.rest.double()
        R.assert_close(both, want["out"], want["out_tol"] - R.HALF_STEP[x["q"].dtype] * np.abs(want["out"]) * (1 - 2 ** -7), what + "rest")
    R.assert_close(lse, want["lse"], want["lse_tol"], what + "lse")
    empty = ~want["see"].any(2)[:, None] & np.ones(lse.shape, bool)
    assert (out.float().cpu().numpy()[empty] == 0).all() and np.isneginf(lse.cpu().numpy()[empty]).all()
    if dout is None:
        return
    got = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], torch.from_numpy(want["out"]).to(x["q"].dtype).cuda(),
                                    api.SoftmaxSaved(torch.from_numpy(want["lse"]).float().cuda(), None), dout, **how)
    for name, y in zip(("dq", "dk", "dv", "dtable"), got):
        if y is None:
            assert name == "dtable" and "table" not in how
            continue
        R.assert_close(y, want[name], want[name + "_tol"], what + name)
    assert (got[0].float().cpu().numpy()[empty] == 0).all()
    unseen = ~want["see"].any(1)
    for y in got[1:3]:
        assert (y.float().cpu().numpy().transpose(0, 2, 1, 3)[unseen] == 0).all()


SHAPES = [
    # B, H, KV, nq, nk, d
    (1, 1, 1, 17, 17, 8), (2, 3, 3, 64, 64, 32), (1, 2, 1, 65, 65, 40), (1, 4, 2, 127, 129, 64), (2, 2, 2, 128, 128, 128),
    (1, 6, 2, 200, 333, 72), (1, 1, 1, 257, 100, 96), (3, 2, 1, 31, 300, 128), (1, 7, 7, 196, 196, 64), (1, 2, 2, 385, 385, 16),
    (1, 2, 1, 130, 1, 64), (1, 3, 1, 500, 640, 128),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("how", [dict(), dict(mask="causal", cap=20.0), dict(mask="causal", bias="slopes", ragged=True),
                                 dict(mask="prefix", bias="table"), dict(bias="table", cap=5.0), dict(mask="causal", bias="table", docs="few")],
                         ids=lambda h: "-".join(map(str, h.values())) or "plain")
def test_outputs_and_gradients(lib, route, shape, dtype, how):
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    check(lib, *make(7, *shape, dtype, **how))


@pytest.mark.parametrize("shape", [(40, 8, 4, 150, 170, 64), (21, 16, 2, 300, 129, 128), (100, 4, 4, 33, 257, 40)], ids=str)
@pytest.mark.parametrize("how", [dict(), dict(mask="causal", ragged="empty", bias="table"), dict(mask="prefix", cap=10.0, start=True, bias="slopes"),
                                 dict(mask="causal", docs="few", bias="table"), dict(start=True, ragged="empty", bias="table")],
                         ids=lambda h: "-".join(map(str, h.values())) or "plain")
def test_more_blocks_than_multiprocessors(lib, shape, how):
    """CTAs that go from block to block, some of which see nothing."""
    check(lib, *make(21, *shape, "bf16", **how))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("docs", ["few", "many", "unsorted"])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_documents(lib, route, dtype, docs, mask):
    check(lib, *make(11, 2, 2, 1, 333, 333, 64, dtype, mask=mask, docs=docs))
    check(lib, *make(12, 1, 2, 2, 150, 420, 32, dtype, mask=mask, docs=docs, bias="slopes"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [40, 200])
def test_starts_and_lengths(lib, route, dtype, nq):
    """Queries anywhere: before the first key (rows that see nothing), behind the last one, sequences without a key."""
    for mask in ("full", "causal", "prefix"):
        check(lib, *make(13, 4, 2, 1, nq, 190, 64, dtype, mask=mask, start=True, ragged="empty", bias="table", two_sided=True))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [3, 150])
@pytest.mark.parametrize("scale", [0.0, -0.2, 0.5])
def test_scales(lib, route, dtype, nq, scale):
    """Scores that are all alike, or turned round; caps that many scores reach."""
    for cap in (0.0, 0.5, 8.0):
        x, how, dout = make(15, 2, 2, 1, nq, 150, 64, dtype, mask="causal", cap=cap)
        check(lib, x, dict(how, scale=scale), dout)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("buckets", [(2, 2), (3, 1000), (64, 100000), (5, 7)])
@pytest.mark.parametrize("two_sided", [False, True])
def test_bucket_tables(lib, route, dtype, buckets, two_sided):
    check(lib, *make(17, 2, 2, 1, 150, 150, 32, dtype, mask="full", bias="table", buckets=buckets, two_sided=two_sided))


FEW = [(1, 1, 1, 1, 1, 64), (1, 8, 8, 1, 1000, 64), (3, 8, 2, 1, 257, 128), (2, 4, 1, 5, 130, 40), (1, 7, 1, 16, 300, 96), (5, 6, 3, 2, 64, 8),
       (2, 2, 2, 16, 15, 32), (1, 1, 1, 1, 20000, 128), (1, 32, 1, 3, 9000, 16)]


@pytest.mark.parametrize("shape", FEW, ids=str)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("how", [dict(), dict(mask="causal", cap=20.0, ragged="empty"), dict(mask="causal", bias="slopes", start=True),
                                 dict(mask="prefix", bias="table", docs="few")], ids=lambda h: "-".join(map(str, h.values())) or "plain")
def test_few_queries(lib, route, shape, dtype, how):
    if dtype == "fp32" and route == "alu":
        pytest.skip("fp32 has one route")
    check(lib, *make(19, *shape, dtype, grad=shape[4] < 1000, **how))


def test_one_pass_of_all_of_them(lib):
    """Rows of the bias, attention with that bias, its gradients, and the table's gradient from the rows' one."""
    api, _, ctx = lib
    x, how, dout = make(23, 2, 4, 2, 100, 100, 32, "fp32", bias="table", cap=30.0)
    rows = api.relative_bias(ctx, how["table"], how["first"], 100, 100, two_sided=True)
    delta = np.arange(100)[None, :] - np.arange(100)[:, None]
    assert np.array_equal(rows.cpu().numpy(), how["table"].cpu().numpy()[:, R.bucket(how["first"], delta, True)])
    want = R.reference(x["q"], x["k"], x["v"], dout, **how)
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    dq, dk, dv, dtable = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], out, saved, dout, **how)
    for name, y in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv), ("dtable", dtable)):
        # (out comes from the kernel: its error enters D as an rounding would)
        extra = 0.0 if name in ("out", "dv") else 2 * np.abs(want["out_tol"]).max() * float(dout.abs().sum(-1).max()) * 32
        R.assert_close(y, want[name], want[name + "_tol"] + extra, name)
    again = api.relative_bias_backward(ctx, torch.from_numpy(want["dS"]).float().cuda(), how["first"], two_sided=True)
    R.assert_close(again, want["dtable"], 64 * R.U * np.abs(want["dS"]).sum((0, 2, 3))[:, None], "dtable from rows")


def test_gradients_against_differences(lib):
    """The kernel's gradients along random directions against central differences of the loss in 64 bits."""
    api, _, ctx = lib
    x, how, dout = make(29, 1, 2, 1, 70, 70, 32, "fp32", mask="causal", bias="table", cap=10.0)
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    got = dict(zip(("q", "k", "v", "table"), api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], out, saved, dout, **how)))
    g = torch.Generator().manual_seed(1)

    def loss(name, step):
        y = {n: t.double().cpu() for n, t in x.items()}
        h = dict(how, table=how["table"].double().cpu())
        if name == "table":
            h["table"] = h["table"] + step
        else:
            y[name] = y[name] + step
        return float((_loss64(y["q"], y["k"], y["v"], h) * dout.double().cpu()).sum())

    def _loss64(q, k, v, h):
        see, delta = R.visible(1, 70, 70, "causal")
        z = 10.0 * torch.tanh((q @ k.repeat_interleave(2, 1).transpose(2, 3)) * 32 ** -0.5 / 10.0)
        z = z + h["table"][:, torch.from_numpy(R.bucket(h["first"], delta[0], False))]
        z = z.masked_fill(~torch.from_numpy(see)[:, None], float("-inf"))
        return torch.softmax(z, -1) @ v.repeat_interleave(2, 1)

    eps = 1e-4
    for name, grad in got.items():
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        slope = (loss(name, eps * u) - loss(name, -eps * u)) / (2 * eps)
        mine = float((grad.double().cpu() * u).sum())
        scale = float((grad.double().cpu().abs() * u.abs()).sum())
        # third derivatives times eps^2 are about 1e-6 of the terms; fp32 gradients are off by some 1e-6 of them
        assert abs(mine - slope) <= 2e-5 * scale, f"{name}: {mine} for {slope}"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [4, 140])
def test_strides_and_broadcasts(lib, route, dtype, nq):
    """Tokens before heads, a slice of a packed projection, keys broadcast over heads and batch, and outputs of other strides."""
    api, _, ctx = lib
    dt = DT[dtype]
    g = torch.Generator().manual_seed(3)
    packed = torch.randn(2, nq, 3, 4, 48, generator=g).to(dt).cuda()
    q = packed[:, :, 1].transpose(1, 2)[..., 8:40]
    shared = torch.randn(1, 1, 150, 32, generator=g).to(dt).cuda()
    k, v = shared.expand(2, 2, 150, 32), torch.randn(150, 2, 2, 32, generator=g).to(dt).cuda().permute(1, 2, 0, 3)
    dout = torch.randn(1, 4, nq, 32, generator=g).to(dt).cuda().expand(2, 4, nq, 32)
    want = R.reference(q, k, v, dout, mask="causal")
    room = torch.full((2, nq, 4, 40), 7.0, dtype=dt, device="cuda")
    out = room.transpose(1, 2)[..., :32]
    got, saved = api.softmax_attn(ctx, q, k, v, mask="causal", want_lse=True, out=out)
    assert got is out
    R.assert_close(out, want["out"], want["out_tol"], "out")
    assert (room[..., 32:] == 7.0).all()
    grads = api.softmax_attn_backward(ctx, q, k, v, out, saved, dout, mask="causal")
    for name, y in zip(("dq", "dk", "dv"), grads):
        # (out and lse are the kernel's: out's own error stands in D as its rounding does, so each bound counts once more)
        R.assert_close(y, want[name], want[name + "_tol"] * 2, name)


@pytest.mark.parametrize("nq", [2, 130])
def test_offsets_past_32_bits(lib, route, nq):
    """Sequences, heads and tokens more than 2^32 bytes apart."""
    api, _, ctx = lib
    far = (1 << 31) + (1 << 16)
    room = torch.zeros(far + (1 << 22), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(8)
    for axis in range(3):
        shape = [(2, 1, 140, 64), (1, 2, 140, 64), (1, 1, 140, 64)][axis]
        strides = [(far, 64, 64, 1), (64, far, 64, 1), (64, 64, far // 139 // 8 * 8, 1)][axis]
        k, v = room.as_strided(shape, strides, 0), room.as_strided(shape, strides, 1 << 20)
        k.copy_(torch.randn(shape, generator=g))
        v.copy_(torch.randn(shape, generator=g))
        q = torch.randn(shape[0], shape[1], nq, 64, generator=g).to(torch.bfloat16).cuda()
        dout = torch.randn(q.shape, generator=g).to(torch.bfloat16).cuda()
        check(lib, {"q": q, "k": k, "v": v}, {"mask": "causal"}, dout)
        room.zero_()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("nq", [3, 150])
def test_what_nobody_sees_does_not_matter(lib, route, dtype, bad, nq):
    """Infinities and NaN behind the lengths, in padding, and in later tokens (forward: whoever does not see them)."""
    api, _, ctx = lib
    x, how, dout = make(31, 2, 4, 2, nq, 200, 64, dtype, mask="causal", docs="few" if nq > 16 else None, ragged=True, bias="table")
    clean = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    want = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *clean, dout, **how)
    see, _ = R.visible(2, nq, 200, "causal", how["k_len"].cpu(), None, None,
                       *(how[n].cpu() if n in how else None for n in ("q_doc", "k_doc")))
    unseen, empty = torch.from_numpy(~see.any(1)).cuda(), torch.from_numpy(~see.any(2)).cuda()
    assert unseen.any()
    q, k, v, do = (t.clone() for t in (x["q"], x["k"], x["v"], dout))
    for t in (k, v):
        t.masked_fill_(unseen[:, None, :, None], bad)
    for t in (q, do):
        t.masked_fill_(empty[:, None, :, None], bad)
    out, saved = api.softmax_attn(ctx, q, k, v, want_lse=True, **how)
    assert torch.equal(out, clean[0]) and torch.equal(saved.lse, clean[1].lse)
    for a, b in zip(api.softmax_attn_backward(ctx, q, k, v, out, saved, do, **how), want):
        assert torch.equal(a, b)
    # one value that some queries see and some do not: it reaches the former in its column, and nobody else
    j = int(np.flatnonzero(see[0].any(0) & ~see[0].all(0))[0])
    v = x["v"].clone()
    v[0, 1, j, 5] = bad
    out = api.softmax_attn(ctx, x["q"], x["k"], v, **how).float().cpu().numpy()
    hit = np.zeros(out.shape, bool)
    hit[0, 2:, :, 5] = see[0][:, j]
    assert not np.isfinite(out[hit]).any()
    same = api.softmax_attn(ctx, x["q"], x["k"], x["v"], **how).float().cpu().numpy()
    # (a spoilt column of a row that does not see the value may be summed again, in another order: one rounding to storage)
    again = np.zeros(out.shape, bool)
    again[0, 2:, :, 5] = True
    assert np.array_equal(out[~again], same[~again])
    again &= ~hit
    assert (np.abs(out[again] - same[again]) <= (2 * R.HALF_STEP[DT[dtype]] + 2 * 200 * R.U) * np.abs(same[again]) + 1e-4).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nq", [2, 100])
def test_lowest_and_infinite_biases(lib, route, dtype, nq):
    """A table of the type's lowest values beside ordinary ones masks; a row of lowest values only is a mean; -inf everywhere is an empty row."""
    api, _, ctx = lib
    x, how, dout = make(37, 1, 2, 2, nq, 100, 32, dtype, mask="causal", bias="table", buckets=(4, 8))
    low = torch.finfo(DT[dtype]).min
    how["table"][0, 2:] = low
    how["table"][1, :] = -float("inf")
    out, saved = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    lse = saved.lse
    near = dict(how, table=how["table"].clone())
    near["table"][0, 2:] = -float("inf")
    near["table"][1, :] = 0
    want = R.reference(x["q"], x["k"], x["v"], **near)
    R.assert_close(out[:, :1], want["out"][:, :1], want["out_tol"][:, :1], "masked by the lowest value")
    assert (out[:, 1] == 0).all() and (lse[:, 1] == -float("inf")).all()
    dq, dk, dv, dtable = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], out, saved, dout, **how)
    assert (dq[:, 1] == 0).all() and (dk[:, 1] == 0).all() and (dv[:, 1] == 0).all() and (dtable[1] == 0).all()
    assert all(torch.isfinite(y.float()).all() for y in (dq, dk, dv, dtable))
    how["table"][0, :] = low
    out = api.softmax_attn(ctx, x["q"], x["k"], x["v"], **how)
    V = x["v"][0, 0].double().cpu().numpy()
    see, _ = R.visible(1, nq, 100, "causal")
    P = see[0] / see[0].sum(1, keepdims=True)
    R.assert_close(out[0, 0], P @ V, (2 * R.HALF_STEP[DT[dtype]] + 300 * R.U) * (P @ np.abs(V)), "a mean")


def test_equal_calls_give_equal_bits(lib, route):
    api, _, ctx = lib
    for shape in ((2, 8, 2, 300, 300, 64), (3, 8, 2, 1, 3000, 128)):
        x, how, dout = make(41, *shape, "bf16", mask="causal", bias="table", cap=30.0)
        a = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
        ga = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *a, dout, **how)
        for _ in range(3):
            b = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
            gb = api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *b, dout, **how)
            assert all(torch.equal(s, t) for s, t in zip((a[0], *a[1], *ga), (b[0], *b[1], *gb)))


def test_streams_and_captured_calls(lib):
    """Two contexts at once on streams of their own, and a captured pass replayed on new inputs beside eager calls."""
    api, B, ctx = lib
    sides = []
    for seed in (1, 2):
        stream = torch.cuda.Stream()
        x, how, dout = make(seed, 1, 4, 2, 260, 260, 64, "bf16", mask="causal", bias="table", docs="few")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            sides.append((stream, api.Context(0), x, how, dout))
    want = []
    for _, _, x, how, dout in sides:
        o = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
        want.append((o[0], *o[1], *api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *o, dout, **how)))
    torch.cuda.synchronize()
    got = []
    for stream, c, x, how, dout in sides:
        with torch.cuda.stream(stream):
            o = api.softmax_attn(c, x["q"], x["k"], x["v"], want_lse=True, **how)
            got.append((o[0], *o[1], *api.softmax_attn_backward(c, x["q"], x["k"], x["v"], *o, dout, **how)))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    stream, c, x, how, dout = sides[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        o = api.softmax_attn(c, x["q"], x["k"], x["v"], want_lse=True, **how)
        held = (o[0], *o[1], *api.softmax_attn_backward(c, x["q"], x["k"], x["v"], *o, dout, **how))
        few = api.softmax_attn(c, x["q"][:, :, :4], x["k"], x["v"], mask="causal")
    other = make(5, 1, 4, 2, 260, 260, 64, "bf16", mask="causal", bias="table", docs="few")
    for name in x:
        x[name].copy_(other[0][name])
    dout.copy_(other[2])
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    o = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
    fresh = (o[0], *o[1], *api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *o, dout, **how))
    assert all(torch.equal(s, t) for s, t in zip(held, fresh))
    assert torch.equal(few, api.softmax_attn(ctx, x["q"][:, :, :4], x["k"], x["v"], mask="causal"))
    del graph
    for _, c, *_ in sides:
        c.close()


def test_spoilt_values_at_the_end_of_a_long_cache(lib):
    """Infinities that some queries of a tile see and others do not, and one that all see, with keys so many that summing rows again takes long."""
    api, B, ctx = lib
    nq, nk, d = 256, 1 << 20, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(1, 1, nq, d, device="cuda", generator=g).bfloat16()
    k, v = (torch.randn(1, 1, nk, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    inf = float("inf")
    v[0, 0, nk - 60, 7] = inf               # query nq - 60 and those behind it
    v[0, 0, nk - 200, 9] = -inf
    v[0, 0, 5, 11] = inf                    # everyone
    torch.cuda.synchronize()
    at = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    at[0].record()
    out = api.softmax_attn(ctx, q, k, v, mask="causal")[0, 0]
    at[1].record()
    torch.cuda.synchronize()
    B.grf_ctx_check(ctx.handle)
    print(f"{at[0].elapsed_time(at[1]):.1f} ms")
    rows = torch.arange(nq, device="cuda")
    assert (out[:, 11] == inf).all()
    assert torch.equal(out[:, 7] == inf, rows >= nq - 60) and torch.equal(out[:, 9] == -inf, rows >= nq - 200)
    other = torch.ones_like(out, dtype=torch.bool)
    other[:, 11] = False
    other[nq - 60:, 7] = False
    other[nq - 200:, 9] = False
    assert out[other].isfinite().all()
    ones = [0, 20, 56, 57, 100, 195, 196, 255]
    s = (q[0, 0, ones].double() @ k[0, 0].double().T) * d ** -0.5
    s[torch.arange(nk, device="cuda")[None] > (nk - nq + rows[ones])[:, None]] = -inf
    p = torch.softmax(s, 1)
    w = v[0, 0].double()
    clean = torch.where(w.isfinite(), w, 0.0)
    want, size = p @ clean, p @ clean.abs()
    # P and out to bf16; scores, of a size of 6 or less, and sums in 32 bits
    bound = size * (2 * 2.0**-8 + 2.0**-16) + 1e-9
    diff = (out[ones].double() - want).abs()
    assert (diff <= bound)[other[ones]].all()


def test_workspace_of_a_call_on_a_stream_that_is_not_current(lib, monkeypatch):
    """Memory of a call's workspace is not handed out on the current stream while the call may still run on the context's."""
    api, B, ctx = lib
    x, how, dout = make(8, 2, 2, 2, 300, 300, 64, "bf16", docs="few", bias="table")
    drows = torch.randn(2, 2, 300, 300, device="cuda")
    places = []
    for name, at in (("grf_softmax_attn", -2), ("grf_softmax_attn_backward", -2), ("grf_relative_bias_backward", -2)):
        call = getattr(B, name)
        monkeypatch.setattr(B, name, lambda *a, call=call, at=at: (places.append((a[at].data_ptr(), a[at].numel())), call(*a)))
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        o = api.softmax_attn(ctx, x["q"], x["k"], x["v"], want_lse=True, **how)
        taken = [torch.empty(places[-1][1], dtype=torch.uint8, device="cuda")]
        api.softmax_attn_backward(ctx, x["q"], x["k"], x["v"], *o, dout, **how)
        taken.append(torch.empty(places[-1][1], dtype=torch.uint8, device="cuda"))
        api.relative_bias_backward(ctx, drows, how["first"])
        taken.append(torch.empty(places[-1][1], dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert len(places) == 3 and all(n > 0 for _, n in places)
    assert not {p for p, _ in places} & {t.data_ptr() for t in taken}


def test_threads_with_contexts_of_their_own(lib):
    """Calls of the same kernels with and without what takes more shared memory, from two threads at once."""
    import threading
    api, B, ctx = lib
    sides = []
    for seed, docs, last in ((1, "few", 64), (2, None, 5000)):
        x, how, dout = make(seed, 1, 2, 2, 130, 130, 64, "bf16", mask="causal", bias="table", docs=docs)
        first = api.relative_buckets(32, last)
        drows = torch.randn(1, 2, 130, 130, device="cuda")

        def run(c, x=x, how=how, dout=dout, first=first, drows=drows):
            o = api.softmax_attn(c, x["q"], x["k"], x["v"], want_lse=True, **how)
            return (o[0], *o[1], *api.softmax_attn_backward(c, x["q"], x["k"], x["v"], *o, dout, **how), api.relative_bias_backward(c, drows, first))
        sides.append((run, run(ctx)))
    torch.cuda.synchronize()
    failures = []

    def work(run, want):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                c = api.Context(0)
                for _ in range(300):
                    got = run(c)
                stream.synchronize()
                assert all(torch.equal(s, t) for s, t in zip(got, want))
                stream.synchronize()
                c.close()
        except Exception as e:  # noqa: BLE001
            failures.append(e)
    threads = [threading.Thread(target=work, args=side) for side in sides]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (1, 3, 7, 9), (2, 5, 77, 130), (3, 2, 200, 1), (1, 4, 513, 515), (2, 1, 33, 3000)], ids=str)
@pytest.mark.parametrize("two_sided,buckets", [(False, (32, 128)), (True, (32, 128)), (True, (64, 5000)), (False, (2, 2))])
def test_bias_rows_and_table_gradient(lib, dtype, shape, two_sided, buckets):
    api, _, ctx = lib
    B, H, nq, nk = shape
    g = torch.Generator().manual_seed(9)
    first = api.relative_buckets(*buckets)
    cols = len(first) * (2 if two_sided else 1)
    table = torch.randn(H, cols, generator=g).to(DT[dtype]).cuda()
    drows = torch.randn(B, H, nq, nk, generator=g).to(DT[dtype]).cuda()
    for start in (None, 0, -100, 5000, 2**31 - 1, -2**31):
        delta = np.arange(nk)[None, :] - (np.arange(nq)[:, None] + (nk - nq if start is None else start))
        b = R.bucket(first, delta, two_sided)
        rows = api.relative_bias(ctx, table, first, nq, nk, two_sided=two_sided, q_start=start)
        assert torch.equal(rows.cpu(), table.cpu()[:, torch.from_numpy(b)])
        got = api.relative_bias_backward(ctx, drows, first, two_sided=two_sided, q_start=start)
        x = drows.double().cpu().numpy()
        sums = lambda y: np.stack([np.bincount(b.ravel(), y[:, h].sum(0).ravel(), cols) for h in range(H)])  # noqa: E731
        want, size = sums(x), sums(np.abs(x))
        # a lane's bin takes at most n / 256 additions, the joins 20 more
        R.assert_close(got, want, (B * nq * nk / 256 + 32) * R.U * size + R.HALF_STEP[DT[dtype]] * np.abs(want) + 1e-30, "dtable")


@pytest.mark.parametrize("two_sided", [False, True])
@pytest.mark.parametrize("last", [300, 5000, 1 << 29])
def test_table_gradient_with_buckets_far_beyond_the_tokens(lib, last, two_sided):
    """Right, and in a time that goes with the matrix, not with the distances of buckets that it does not reach."""
    api, _, ctx = lib
    H, nq, nk, first = 2, 300, 900, [0, 3, 200, last]
    cols = len(first) * (2 if two_sided else 1)
    drows = torch.randn(1, H, nq, nk, generator=torch.Generator().manual_seed(3)).cuda()
    x = drows.double().cpu().numpy()
    for start in (None, 0, last):
        b = R.bucket(np.array(first), np.arange(nk)[None, :] - (np.arange(nq)[:, None] + (nk - nq if start is None else start)), two_sided)
        for _ in range(3):
            at = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            at[0].record()
            got = api.relative_bias_backward(ctx, drows, first, two_sided=two_sided, q_start=start)
            at[1].record()
            torch.cuda.synchronize()
        assert at[0].elapsed_time(at[1]) < 10.0
        sums = lambda y: np.stack([np.bincount(b.ravel(), y[:, h].sum(0).ravel(), cols) for h in range(H)])  # noqa: E731
        want, size = sums(x), sums(np.abs(x))
        R.assert_close(got, want, (nq * nk / 256 + 32) * R.U * size + R.HALF_STEP[torch.float32] * np.abs(want) + 1e-30, "dtable")


def test_refusals_leave_outputs_alone(lib):
    api, B, ctx = lib
    x, how, dout = make(43, 1, 2, 1, 20, 20, 32, "bf16")
    s = api._softmax_desc(ctx, x["q"], x["k"], x["v"], None, 0.0, "full", None, None, None, None, None, None, None, None, False)
    out = torch.full_like(x["q"], 3.0)
    lse = torch.empty(1, 2, 20, device="cuda")
    for field, value, code in (("dim", 12, -1), ("dim", 136, -1), ("kv_heads", 3, -1), ("cap", -1.0, -1), ("cap", float("nan"), -1), ("order", 3, -1),
                               ("order", 2, -1), ("bias", 1, -1), ("n_q", 0, -1), ("n_k", (1 << 22) + 1, -2), ("batch", 70000, -2), ("dtype", 2, -1)):
        old = getattr(s, field)
        setattr(s, field, value)
        with pytest.raises(B.GrfError) as e:
            B.grf_softmax_attn(ctx.handle, s, x["q"], x["k"], x["v"], out, lse, None, None, 0)
        assert e.value.code == code, field
        setattr(s, field, old)
    torch.cuda.synchronize()
    assert (out == 3.0).all()
    with pytest.raises(ValueError):
        api.softmax_attn(ctx, x["q"], x["k"].float(), x["v"])
    with pytest.raises(ValueError):
        api.softmax_attn(ctx, x["q"].transpose(2, 3), x["k"], x["v"])
    with pytest.raises(ValueError):
        api.softmax_attn(ctx, x["q"], x["k"], x["v"], k_len=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        api.softmax_attn(ctx, x["q"], x["k"], x["v"], table=torch.zeros(2, 4, dtype=torch.bfloat16, device="cuda"))
