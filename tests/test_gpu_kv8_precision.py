"""Attention over the 8-bit KV cache where most of the weight is on values of
zero, against 64 bits: every output element within fp32's error of its own sum
of |weight * value|, not of the largest value."""

import numpy as np
import pytest
import torch

import paper_2608_00528_amd as s4r
from tests import kv8_reference as R
from tests.test_gpu_kv8 import cfg, dev, ints

pytestmark = pytest.mark.gpu


def attention_by_element(ref, q, lengths, waves):
    """(out, tol) of R.attention, the bound per element.  R.attention's count of roundings holds for each weight and
    each sum in relative terms: a weight is off by 25 * 2^-24 S and exp2's error, a sum by the roundings of its chain
    relative to the absolute sum of what it adds.  So an element is off by that times sum p |v_d| / sum p, for which
    R.attention takes max |v|.  Weights below 2^-126 of the largest may be flushed."""
    out, tol = R.attention(ref, q, lengths, waves)
    B, n, hq, dh = q.shape
    G = hq // ref.H
    by_element = np.zeros_like(out)
    for b in range(B):
        N = int(lengths[b])
        k, v = (ref.values(s, b, N) for s in "kv")
        for i in range(n):
            m = N - (n - 1 - i)
            for h in range(hq if m > 0 else 0):
                kk, vv = k[h // G, :m], np.abs(v[h // G, :m])
                z = kk @ q[b, i, h] / np.sqrt(dh)
                p = np.exp(z - z.max())
                unit = tol[b, i, h] / vv.max() if vv.max() > 0 else 0.0
                by_element[b, i, h] = unit * (p @ vv / p.sum()) + m * 2.0 ** -126 * vv.max()
    return out, by_element


@pytest.mark.parametrize("margin", [10, 15, 23, 40, 60])
@pytest.mark.parametrize("fmt,dtype,hq,hkv,dh,nq,n,cap,copies", [
    ("int8", "bf16", 4, 1, 128, 1, 1000, 1008, 1),        # a workgroup per pair
    ("e4m3", "bf16", 8, 2, 64, 5, 700, 2304, 1),          # cut into runs, two chunks of query rows
    ("int8", "fp32", 4, 2, 128, 1, 2300, 2304, 1),        # cut into runs
    ("e4m3", "fp32", 16, 1, 128, 2, 130, 144, 640)])      # a wave per pair
def test_first_token_holds_the_weight_and_no_value(fmt, dtype, hq, hkv, dh, nq, n, cap, copies, margin):
    """An attention sink: the first token's logit is `margin` above every other, and its value is zero."""
    rng = np.random.default_rng(margin + dh)
    q = 1 + 0.05 * rng.standard_normal((1, nq, hq, dh))
    q = R.round_to(q, dtype)
    x = {s: 0.02 * rng.standard_normal((1, n, hkv, dh)) for s in "kv"}
    x["v"] *= 50
    x["k"][:, 0] = margin / np.sqrt(dh)                   # q . k / sqrt(dh) is about `margin`
    x["v"][:, 0] = 0
    ref = R.RefCache(fmt, 1, hkv, dh, cap)
    ref.write({s: R.round_to(x[s].reshape(1, n, -1), dtype) for s in "kv"}, [0], [n])
    want, tol = attention_by_element(ref, q, [n], 1 if copies > 1 else 4)
    c = cfg(copies, hq, hkv, dh, cap, dtype)
    t = {}
    for s in "kv":
        t[s + "_codes"] = torch.from_numpy(ref.codes[s]).cuda().repeat(copies, 1, 1, 1)
        t[s + "_scales"] = torch.from_numpy(ref.scales[s]).cuda().repeat(copies, 1, 1)
    got = s4r.kv8_decode(c, s4r.KV8Cache(fmt, **t), cap, dev(np.tile(q, (copies, 1, 1, 1)), c),
                         s4r.alloc_kv8_workspace(c, nq), lengths=ints([n] * copies)).double().cpu().numpy()
    err = np.abs(got - want)
    assert np.all(err <= tol), f"worst {(err / np.maximum(tol, 1e-300)).max():.3g} of the bound"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("copies,cap", [(1, 64), (1, 4096), (640, 64)])
def test_fp32_queries_keep_their_last_bits(fmt, dh, copies, cap):
    """Four query heads that differ in their last two bits alone: c (1 + 2^-11 + i 2^-23).  The one key element that
    they meet is a power of two after its scale, so a logit is the query's element times a power of two, exactly:
    Z (1 + 2^-11 + i 2^-23), Z = 64 or 45 nats above the second token's, whose value alone is not zero.  The output
    is exp(-logit): head i is off head 0 by i Z 2^-23 in the exponent.  Roundings, in each head: the logit's last
    factor (2^-24 Z), exp2 (its own 2^-22), the sum and the division (below 2^-22 together)."""
    hq, n = 4, 2
    q = np.zeros((1, 1, hq, dh))
    q[0, 0, :, 0] = 8 * (1 + 2.0 ** -11 + np.arange(hq) * 2.0 ** -23)
    q = R.round_to(q, "fp32")
    assert np.array_equal(q[0, 0, :, 0] / q[0, 0, 0, 0] > 1, np.arange(hq) > 0)
    x = {s: np.zeros((1, n, 1, dh)) for s in "kv"}
    x["k"][0, 0, 0, 0], x["k"][0, 0, 0, 1] = 64, 127
    x["v"][0, 1] = 1
    ref = R.RefCache(fmt, 1, 1, dh, cap)
    ref.write({s: x[s].reshape(1, n, dh) for s in "kv"}, [0], [n])
    logit = 64 * q[0, 0, :, 0] / np.sqrt(dh)
    assert logit[0] > 40
    c = cfg(copies, hq, 1, dh, cap, "fp32")
    t = {}
    for s in "kv":
        t[s + "_codes"] = torch.from_numpy(ref.codes[s]).cuda().repeat(copies, 1, 1, 1)
        t[s + "_scales"] = torch.from_numpy(ref.scales[s]).cuda().repeat(copies, 1, 1)
    got = s4r.kv8_decode(c, s4r.KV8Cache(fmt, **t), cap, dev(np.tile(q, (copies, 1, 1, 1)), c),
                         s4r.alloc_kv8_workspace(c), lengths=ints([n] * copies)).double().cpu().numpy()
    assert np.all(got > 0)
    apart = np.log(got / got[:, :, :1])
    want = -(logit - logit[0])[:, None]
    assert np.all(np.abs(apart - want) <= logit[0] * 2.0 ** -23 + 2 * 2.0 ** -21)
