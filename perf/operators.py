"""Performance cases of softmax attention with score modifiers and of the learned relative position bias.

A case has a kind:

  "prefill"  one forward pass over whole sequences
  "train"    forward and backward pass: outputs and the gradients of Q, K, V and of the bias table
  "decode"   a few new tokens (mostly one) of every sequence against its cache of keys and values
  "bias"     the relative position bias as rows of a matrix, and the gradient of its table

Scores are x = scale q.k, capped as cap tanh(x / cap) where the case has a cap, plus a bias that depends on the distance of key
and query: a slope per head times the distance ("slopes"), or a learned value per head and bucket of distances ("table").  Masks:
"full", "causal", "prefix" (causal, and a stretch at the start that every query sees); documents packed into one sequence;
lengths per sequence.  Positions of the queries are the last ones of the keys unless they are given per sequence."""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BUCKETS, FAR = 32, 128          # values of a table per head and side; distances from FAR on share the last one


def _case(name, kind, B, H, kv, nq, nk, d, dtype, mask="full", bias="none", cap=0.0, docs=False, ragged=False):
    c = {"kind": kind, "B": B, "H": H, "kv": kv, "nq": nq, "nk": nk, "d": d, "dtype": dtype, "mask": mask, "bias": bias,
         "cap": cap, "docs": docs, "ragged": ragged}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: the next token of one sequence, eight heads; latency is all of it
        _case("decode_one", "decode", 1, 8, 8, 1, 1000, 64, "bf16", "causal", "table"),
        # a serving batch with shared key heads and caches of uneven length: the bandwidth of the memory
        _case("decode_batch", "decode", 64, 32, 8, 1, 8192, 128, "bf16", "causal", "none", 30.0, ragged=True),
        # five drafted tokens of seven sequences in full precision, odd lengths
        _case("decode_drafts_fp32", "decode", 7, 6, 2, 5, 5003, 64, "fp32", "causal", "slopes", ragged=True),
        # one layer of an image transformer: 64 images of 14 x 14 patches, 12 heads, learned bias to both sides
        _case("patches_196", "prefill", 64, 12, 12, 196, 196, 64, "bf16", "full", "table"),
        # a language model's prompt: causal, capped scores, shared key heads
        _case("prompt_4096_capped", "prefill", 2, 16, 4, 4096, 4096, 128, "bf16", "causal", "none", 50.0),
        # documents packed into one long sequence, distance slopes, an odd length
        _case("packed_8191", "prefill", 1, 8, 8, 8191, 8191, 64, "bf16", "causal", "slopes", docs=True),
        # full precision, everything odd, a prefix that all queries see
        _case("prefix_1003_fp32", "prefill", 3, 5, 5, 1003, 1003, 32, "fp32", "prefix", "table"),
        # training step of the image transformer's layer
        _case("train_patches_196", "train", 64, 12, 12, 196, 196, 64, "bf16", "full", "table"),
        # training step of a language model's layer, capped scores, shared key heads
        _case("train_4096_capped", "train", 1, 16, 4, 4096, 4096, 128, "bf16", "causal", "none", 50.0),
        # training step in full precision over packed documents with padding behind them
        _case("train_packed_1531_fp32", "train", 2, 4, 2, 1531, 1531, 40, "fp32", "causal", "table", docs=True),
        # the bias by itself, and the gradient of its table from a batch of eight
        _case("bias_1024", "bias", 8, 12, 12, 1024, 1024, 64, "bf16", "full", "table"),
        # the same in full precision, more keys than queries
        _case("bias_777_fp32", "bias", 3, 5, 5, 777, 1003, 64, "fp32", "causal", "table"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "train", "train", "decode", "decode", "bias"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    d = rng.choice([32, 40, 64, 64, 80, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 5, 8])
    H = kv * rng.choice([1, 1, 2, 4, 7])
    mask = rng.choice(["full", "causal", "causal", "prefix"])
    bias = rng.choice(["none", "slopes", "table", "table"])
    cap = rng.choice([0.0, 0.0, 30.0, 50.0])
    if kind == "decode":
        B, nk = _log(rng, 1, 64), _log(rng, 64, 8192)
        while B * kv * nk * d > 64 * 8 * 8192 * 128 // (4 if dtype == "fp32" else 1):
            B = max(1, B // 2)
        return _case(None, kind, B, H, kv, rng.choice([1, 1, 1, 2, 5, 8]), nk, d, dtype, "causal", bias, cap, ragged=rng.random() < 0.7)
    if kind == "bias":
        nq, nk = _log(rng, 16, 2048), _log(rng, 16, 2048)
        B = max(1, min(_log(rng, 1, 16), 8 * 12 * 1024 * 1024 // (H * nq * nk)))
        return _case(None, kind, B, H, H, nq, nk, d, dtype, rng.choice(["full", "causal"]), "table")
    n = _log(rng, 16, 8192 if dtype == "bf16" else 2048)
    while H * n * n * d > 16 * 4096 * 4096 * 128 // (8 if dtype == "fp32" else 1):
        n = n * 2 // 3
    B = max(1, min(_log(rng, 1, 64), 16 * 4096 * 4096 * 128 // (8 if dtype == "fp32" else 1) // (H * n * n * d)))
    docs = n >= 64 and rng.random() < 0.3
    return _case(None, kind, B, H, kv, n, n, d, dtype, mask, bias, cap, docs=docs, ragged=not docs and mask != "prefix" and rng.random() < 0.3)


def _first():
    """Smallest distance of each bucket: the first half one distance each, the rest by even steps of the logarithm up to FAR."""
    half = BUCKETS // 2
    steps = BUCKETS - half
    first = list(range(half))
    for k in range(steps):
        n = half                                    # smallest n with (n / half)^steps >= (FAR / half)^k, in integers
        while n ** steps * half ** k < FAR ** k * half ** steps:
            n += 1
        first.append(max(n, first[-1] + 1))
    return first


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 11)
    dev, dt = "cuda", DTYPES[case["dtype"]]
    B, H, kv, nq, nk, d = (case[k] for k in ("B", "H", "kv", "nq", "nk", "d"))
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    state = {"case": case, "first": _first(), "two_sided": case["mask"] == "full", "start": None, "k_len": None, "prefix": None,
             "docs": None, "slopes": None, "table": None}
    columns = BUCKETS * (2 if state["two_sided"] else 1)
    if case["bias"] == "table":
        state["table"] = (0.5 * normal(H, columns)).to(dt)
    elif case["bias"] == "slopes":
        state["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=dev)
    if case["kind"] == "bias":
        state["dbias"] = normal(B, H, nq, nk).to(dt)
        return state
    # scores of a few units; wider where they are capped, so that the cap is felt
    state["q"] = (normal(B, H, nq, d) * (4.0 if case["cap"] else 1.5)).to(dt)
    state["k"] = normal(B, kv, nk, d).to(dt)
    state["v"] = normal(B, kv, nk, d).to(dt)
    state["scale"] = d ** -0.5
    if case["kind"] == "train":
        state["dout"] = normal(B, H, nq, d).to(dt)
    if case["mask"] == "prefix":
        state["prefix"] = torch.randint(0, max(1, nk // 2) + 1, (B,), generator=g, device=dev, dtype=torch.int32)
    if case["ragged"]:
        low = max(nq, nk // 4)
        state["k_len"] = torch.randint(min(low, nk), nk + 1, (B,), generator=g, device=dev, dtype=torch.int32)
        if case["kind"] == "decode":
            state["start"] = state["k_len"] - nq
    if case["docs"]:
        ends = torch.rand(B, nk, generator=g, device=dev) < 8.0 / nk            # about eight documents a sequence
        ids = torch.cumsum(ends.to(torch.int32), 1, dtype=torch.int32)
        ids[:, nk - nk // 32:] = -1                                              # padding behind the last one
        state["docs"] = ids.contiguous()
    return state


# ------------------------------------------------------------------------------------------------ plain forms

def _distance_bucket(state, delta):
    """Bucket of each relative position (key minus query) of an integer tensor."""
    first = torch.tensor(state["first"], device=delta.device)
    n = delta.abs() if state["two_sided"] else (-delta).clamp(min=0)
    b = torch.bucketize(n, first, right=True) - 1
    return b + (delta > 0) * len(state["first"]) if state["two_sided"] else b


def _positions(state, nq, nk, device):
    """Relative positions [B or 1, nq, nk]."""
    start = state["start"].long() if state["start"] is not None else torch.full((1,), nk - nq, device=device)
    p = start[:, None] + torch.arange(nq, device=device)
    return torch.arange(nk, device=device) - p[:, :, None]


def _sum_by_bucket(state, ds, delta):
    """ds [H, nq, nk] summed by bucket: first along diagonals, then over the diagonals of a bucket."""
    H, nq, nk = ds.shape
    w = nq + nk
    skew = torch.nn.functional.pad(ds.flip(1), (0, nq)).reshape(H, nq * w)[:, : nq * (w - 1)]
    diag = skew.reshape(H, nq, w - 1).sum(1, dtype=torch.float64)               # column x: j - i = x - (nq - 1)
    rel = torch.arange(w - 1, device=ds.device) - (nq - 1) + delta[0, 0, 0]
    columns = len(state["first"]) * (2 if state["two_sided"] else 1)
    out = torch.zeros(H, columns, dtype=torch.float64, device=ds.device)
    return out.index_add_(1, _distance_bucket(state, rel), diag)


def _scores(state):
    """(scores, capped without bias, visible), all [B, kv, H / kv, nq, nk]."""
    c = state["case"]
    B, H, kv, nq, nk, d = (c[k] for k in ("B", "H", "kv", "nq", "nk", "d"))
    dev = state["q"].device
    q = state["q"].float().reshape(B, kv, H // kv * nq, d)
    x = (q @ state["k"].float().transpose(2, 3)).mul_(state["scale"]).reshape(B, kv, H // kv, nq, nk)
    if c["cap"]:
        x = torch.tanh(x / c["cap"]).mul_(c["cap"])
    delta = _positions(state, nq, nk, dev)
    s = x
    if state["table"] is not None:
        rows = state["table"].float()[:, _distance_bucket(state, delta)]         # [H, B or 1, nq, nk]
        s = x + rows.reshape(kv, H // kv, *delta.shape).permute(2, 0, 1, 3, 4)
    elif state["slopes"] is not None:
        s = x - state["slopes"].reshape(1, kv, H // kv, 1, 1) * delta.abs()[:, None, None].float()
    see = torch.ones(1, 1, 1, nq, nk, dtype=torch.bool, device=dev)
    if c["mask"] != "full":
        see = (delta <= 0)[:, None, None]
    if state["prefix"] is not None:
        see = see | (torch.arange(nk, device=dev) < state["prefix"][:, None]).reshape(B, 1, 1, 1, nk)
    if state["k_len"] is not None:
        see = see & (torch.arange(nk, device=dev) < state["k_len"][:, None]).reshape(B, 1, 1, 1, nk)
    if state["docs"] is not None:
        ids = state["docs"]
        see = see & ((ids[:, :, None] == ids[:, None, :]) & (ids >= 0)[:, :, None]).reshape(B, 1, 1, nq, nk)
    return s, x, see


def _weights(state):
    s, x, see = _scores(state)
    top = s.masked_fill(~see, -math.inf).amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = (s - top).exp_().masked_fill_(~see, 0.0)
    total = p.sum(-1, keepdim=True)
    return p.div_(total.masked_fill(total == 0, 1.0)), x


def _plain_attention(state):
    c = state["case"]
    B, H, kv, nq, nk, d = (c[k] for k in ("B", "H", "kv", "nq", "nk", "d"))
    dt = DTYPES[c["dtype"]]
    p, x = _weights(state)
    pf = p.reshape(B, kv, H // kv * nq, nk)
    v = state["v"].float()
    out = (pf @ v).reshape(B, H, nq, d)
    if c["kind"] != "train":
        return out.to(dt)
    do = state["dout"].float()
    dog = do.reshape(B, kv, H // kv * nq, d)
    dv = pf.transpose(2, 3) @ dog
    ds = (dog @ v.transpose(2, 3)).reshape(p.shape)
    ds = ds.sub_((do * out).sum(-1).reshape(B, kv, H // kv, nq, 1)).mul_(p)
    answer = [out.to(dt)]
    dtable = None
    if state["table"] is not None:
        dtable = _sum_by_bucket(state, ds.reshape(B, H, nq, nk).sum(0), _positions(state, nq, nk, ds.device)).to(dt)
    if c["cap"]:
        ds = ds.mul_(1.0 - (x / c["cap"]).square())
    ds = ds.mul_(state["scale"]).reshape(pf.shape)
    dq = (ds @ state["k"].float()).reshape(B, H, nq, d)
    dk = ds.transpose(2, 3) @ state["q"].float().reshape(B, kv, H // kv * nq, d)
    answer += [dq.to(dt), dk.to(dt), dv.to(dt)]
    return answer + [dtable] if dtable is not None else answer


def _plain_bias(state):
    c = state["case"]
    delta = _positions(state, c["nq"], c["nk"], state["table"].device)
    rows = state["table"][:, _distance_bucket(state, delta)[0]]
    return rows, _sum_by_bucket(state, state["dbias"].float().sum(0), delta).to(DTYPES[c["dtype"]])


# ------------------------------------------------------------------------------------------------ the framework's calls

_contexts = {}


def _context():
    """A program's library context, one per device."""
    from paper_2410_03462_b200 import api
    dev = torch.cuda.current_device()
    if dev not in _contexts:
        _contexts[dev] = api.Context(dev)
    return api, _contexts[dev]


def _own(state):
    api, ctx = _context()
    c = state["case"]
    if c["kind"] == "bias":
        rows = api.relative_bias(ctx, state["table"], state["first"], c["nq"], c["nk"], two_sided=state["two_sided"])
        return rows, api.relative_bias_backward(ctx, state["dbias"], state["first"], two_sided=state["two_sided"])
    how = {"scale": state["scale"], "cap": c["cap"], "mask": c["mask"], "k_len": state["k_len"], "q_start": state["start"],
           "prefix": state["prefix"], "q_doc": state["docs"], "k_doc": state["docs"], "slopes": state["slopes"],
           "table": state["table"], "first": state["first"], "two_sided": state["two_sided"]}
    if c["kind"] != "train":
        return api.softmax_attn(ctx, state["q"], state["k"], state["v"], **how)
    out, lse = api.softmax_attn(ctx, state["q"], state["k"], state["v"], want_lse=True, **how)
    dq, dk, dv, dtable = api.softmax_attn_backward(ctx, state["q"], state["k"], state["v"], out, lse, state["dout"], **how)
    return [out, dq, dk, dv] + ([dtable] if dtable is not None else [])


def run(state):
    if own:
        return _own(state)
    return _plain_bias(state) if state["case"]["kind"] == "bias" else _plain_attention(state)


# ------------------------------------------------------------------------------------------------ sizes, and 64 bits

def work(case):
    B, H, kv, nq, nk, d = (case[k] for k in ("B", "H", "kv", "nq", "nk", "d"))
    e = 4 if case["dtype"] == "fp32" else 2
    columns = BUCKETS * (2 if case["mask"] == "full" else 1)
    if case["kind"] == "bias":
        return {"bytes": (H * nq * nk + B * H * nq * nk + 2 * H * columns) * e, "flops": B * H * nq * nk}
    keys = nk * (0.625 if case["ragged"] else 1.0)                  # mean length
    causal = nq * (keys - nq) + nq * (nq + 1) / 2 if case["kind"] == "decode" else nq * (nq + 1) / 2
    pairs = nq * keys if case["mask"] == "full" else causal
    if case["kind"] != "decode" and case["ragged"] and case["mask"] != "full":
        pairs = nq * nq * 0.41                                       # keys behind the length are seen by none
    if case["mask"] == "prefix":
        pairs = causal + (nk / 4) ** 2 * 2 / 3                       # mean over prefixes up to half
    if case["docs"]:
        pairs = pairs * 0.2                                          # about eight documents of uneven length
    read = (B * H * nq + 2 * B * kv * keys) * d * e
    wrote = B * H * nq * d * e
    if case["kind"] == "train":
        read += 2 * B * H * nq * d * e
        wrote += (B * H * nq + 2 * B * kv * nk) * d * e
    return {"bytes": read + wrote, "flops": (14 if case["kind"] == "train" else 4) * d * B * H * pairs}


def exact(case, seed):
    """From the definition, in 64 bits, one sequence and head at a time."""
    state = prepare(case, seed)
    B, H, kv, nq, nk, d = (case[k] for k in ("B", "H", "kv", "nq", "nk", "d"))
    if B * H * nq * nk > 6e8 or B * H > 4096:
        return None
    dev = "cuda"
    first, sides = state["first"], state["two_sided"]
    columns = len(first) * (2 if sides else 1)
    lut_n = torch.arange(nq + nk + 1, device=dev)
    lut = sum((lut_n >= f).long() for f in first) - 1               # bucket of a distance
    if case["kind"] == "bias":
        rel = torch.arange(nk, device=dev)[None, :] - (torch.arange(nq, device=dev)[:, None] + nk - nq)
        b = lut[rel.abs()] + (rel > 0).long() * len(first) if sides else lut[(-rel).clamp(min=0)]
        rows = torch.stack([state["table"][h].double()[b] for h in range(H)])
        grad = torch.stack([torch.stack([state["dbias"][:, h].double().sum(0)[b == y].sum() for y in range(columns)]) for h in range(H)])
        return rows, grad
    scale, cap = float(state["scale"]), float(case["cap"])
    train = case["kind"] == "train"
    out = torch.zeros(B, H, nq, d, dtype=torch.float64, device=dev)
    dq, dk, dv = torch.zeros_like(out), *(torch.zeros(B, kv, nk, d, dtype=torch.float64, device=dev) for _ in range(2))
    dtable = torch.zeros(H, columns, dtype=torch.float64, device=dev)
    j = torch.arange(nk, device=dev)
    for y in range(B):
        start = int(state["start"][y]) if state["start"] is not None else nk - nq
        i = torch.arange(nq, device=dev) + start
        see = torch.ones(nq, nk, dtype=torch.bool, device=dev) if case["mask"] == "full" else j[None, :] <= i[:, None]
        if state["prefix"] is not None:
            see = see | (j < int(state["prefix"][y]))[None, :]
        if state["k_len"] is not None:
            see = see & (j < int(state["k_len"][y]))[None, :]
        if state["docs"] is not None:
            w = state["docs"][y]
            see = see & (w[:, None] == w[None, :]) & (w[:, None] >= 0)
        rel = j[None, :] - i[:, None]
        b = lut[rel.abs().clamp(max=nq + nk)] + (rel > 0).long() * len(first) if sides else lut[(-rel).clamp(min=0, max=nq + nk)]
        some = see.any(1)
        for h in range(H):
            Q, K, V = state["q"][y, h].double(), state["k"][y, h // (H // kv)].double(), state["v"][y, h // (H // kv)].double()
            z = (Q @ K.T) * scale
            t = torch.tanh(z / cap) if cap else None
            a = cap * t if cap else z
            if state["table"] is not None:
                a = a + state["table"][h].double()[b]
            if state["slopes"] is not None:
                a = a - state["slopes"][h].double() * rel.abs()
            a = torch.where(see, a, torch.full_like(a, -math.inf))
            P = torch.zeros_like(a)
            P[some] = torch.softmax(a[some], dim=1)
            out[y, h] = P @ V
            if not train:
                continue
            G = state["dout"][y, h].double()
            dP = G @ V.T
            dA = P * (dP - (P * dP).sum(1, keepdim=True))
            dv[y, h // (H // kv)] += P.T @ G
            if state["table"] is not None:
                flat = torch.zeros(columns, dtype=torch.float64, device=dev)
                dtable[h] += flat.index_add_(0, b.reshape(-1), dA.reshape(-1))
            dZ = dA * (1 - t * t) * scale if cap else dA * scale
            dq[y, h] = dZ @ K
            dk[y, h // (H // kv)] += dZ.T @ Q
    if not train:
        return out
    return [out, dq, dk, dv] + ([dtable] if state["table"] is not None else [])
