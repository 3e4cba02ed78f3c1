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
