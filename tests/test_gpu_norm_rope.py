"""Norms of query and key heads with the rotation (`qk_norm_rope`) against the
64-bit reference, and the whole cache path of a decoding program."""

import numpy as np
import pytest
import torch

import paper_2608_00528_amd as s4r
from tests import kv8_reference as R

pytestmark = pytest.mark.gpu


def cfg(hq, hkv, dh, theta, dtype="bf16", **kw):
    kw = dict(dict(batch=1, capacity=64, rank=32), **kw)
    return s4r.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, rope_theta=theta, dtype=dtype, **kw)


def dev(x, c):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", s4r.storage_dtype(c))


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bound(x, weight, y, dtype):
    """|error| of an output: the pair's size times the angle's and the products' errors, and the last rounding.
    Angle: 2^-25 of a revolution from the fraction's fp32 rounding, and the hardware's sine and cosine, whose
    error is taken as 2^-20 of one (a bound for 24-bit fractions); two products and a sum: 3 * 2^-24; the norm's
    factor and the weight: 4 * 2^-24.  Half a step of the storage type."""
    half = y.shape[-1] // 2
    pair = np.hypot(y[..., :half], y[..., half:])
    pair = np.concatenate([pair, pair], -1)
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return pair * (2 * np.pi * 2.0 ** -25 + 2.0 ** -20 + 7 * 2.0 ** -24) * 1.5 + np.abs(y) * step * 1.01


def check(got, x, weight, eps, pos, theta, dtype):
    want = R.norm_rope(x, weight, eps, pos, theta)
    err = np.abs(got.double().cpu().numpy() - want)
    tol = bound(x, weight, want, dtype)
    assert np.all(err <= tol), f"worst {(err / np.maximum(tol, 1e-300)).max():.3g} of the bound"


@pytest.mark.parametrize("hq,hkv,dh,theta", [(32, 8, 128, 1e6), (8, 2, 64, 1e4), (28, 4, 128, 5e5), (4, 4, 128, 1e4),
                                             (5, 1, 64, 1e4), (16, 1, 128, 0.0), (3, 3, 64, 0.0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens", [1, 7, 301, 900])
def test_heads_in_rows_of_a_fused_projection(hq, hkv, dh, theta, dtype, tokens):
    rng = np.random.default_rng(tokens + hq)
    c = cfg(hq, hkv, dh, theta, dtype)
    x = R.round_to(rng.standard_normal((tokens, hq + 2 * hkv, dh)) * rng.uniform(0.01, 30, (tokens, 1, 1)), dtype)
    wq, wk = (R.round_to(1 + 0.3 * rng.standard_normal(dh), dtype) for _ in range(2))
    pos = rng.integers(0, 131072, tokens)
    f = dev(x, c)
    before = f.clone()
    q, k = s4r.qk_norm_rope(c, f[:, :hq], f[:, hq:hq + hkv], ints(pos) if theta else None, dev(wq, c), dev(wk, c))
    assert torch.equal(f, before) and q.is_contiguous() and k.is_contiguous()
    check(q, x[:, :hq], wq, 1e-6, pos, theta, dtype)
    check(k, x[:, hq:hq + hkv], wk, 1e-6, pos, theta, dtype)
    # the same in place: the value heads stay, the results are the same bits
    s4r.qk_norm_rope(c, f[:, :hq], f[:, hq:hq + hkv], ints(pos) if theta else None, dev(wq, c), dev(wk, c),
                     q_out=f[:, :hq], k_out=f[:, hq:hq + hkv])
    assert torch.equal(f[:, :hq], q) and torch.equal(f[:, hq:hq + hkv], k)
    assert torch.equal(f[:, hq + hkv:], before[:, hq + hkv:])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_side_without_weights(dtype):
    rng = np.random.default_rng(4)
    c = cfg(8, 2, 64, 1e4, dtype)
    x = R.round_to(rng.standard_normal((2, 9, 10, 64)), dtype)     # two sequences of nine tokens
    pos = rng.integers(0, 5000, 18)
    w = R.round_to(1 + 0.3 * rng.standard_normal(64), dtype)
    q, k = s4r.qk_norm_rope(c, dev(x[:, :, :8], c), dev(x[:, :, 8:], c), ints(pos), None, dev(w, c), eps=1e-5)
    assert q.shape == (2, 9, 8, 64)
    check(q.flatten(0, 1), x[:, :, :8].reshape(18, 8, 64), None, 1e-5, pos, 1e4, dtype)
    check(k.flatten(0, 1), x[:, :, 8:].reshape(18, 2, 64), w, 1e-5, pos, 1e4, dtype)
    q2, none = s4r.qk_norm_rope(c, dev(x[:, :, :8], c), None, ints(pos))
    assert none is None and torch.equal(q2, q)
    none, k2 = s4r.qk_norm_rope(c, None, dev(x[:, :, 8:], c), ints(pos), k_weight=dev(w, c), eps=1e-5)
    assert none is None and torch.equal(k2, k)


def test_more_tokens_than_a_grid_holds():
    """Rows past 2^32 elements and more tokens than one wave each: the first, the last and some between."""
    hq, hkv, dh, n, width = 2, 2, 64, (1 << 22) + 77, 1024
    c = cfg(hq, hkv, dh, 1e4)
    assert n * width > 2 ** 32
    f = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(5)
    at = np.array([0, 1, 12345, 1 << 21, (1 << 22) - 1, 1 << 22, n - 2, n - 1])
    x = R.round_to(rng.standard_normal((len(at), hq + hkv, dh)), "bf16")
    f[torch.from_numpy(at).cuda(), :(hq + hkv) * dh] = dev(x, c).flatten(1)
    heads = f[:, :(hq + hkv) * dh].view(n, hq + hkv, dh)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    w = torch.ones(dh, dtype=torch.bfloat16, device="cuda")
    q, k = s4r.qk_norm_rope(c, heads[:, :hq], heads[:, hq:], pos, w, w, k_out=heads[:, hq:])
    index = torch.from_numpy(at).cuda()
    # the angle's error grows with the position: 2^-53 of the frequency times 2^22
    check(q[index], x[:, :hq], np.ones(dh), 1e-6, at, 1e4, "bf16")
    check(k[index], x[:, hq:], np.ones(dh), 1e-6, at, 1e4, "bf16")
    q[index] = 0
    heads[index] = 0
    assert not q.any() and not f.any()


def test_far_and_negative_positions():
    c = cfg(4, 4, 128, 5e5, "fp32")
    pos = np.array([0, 1, -1, -131072, 2 ** 20 + 1, 2 ** 24 + 3, 5, 131071])
    rng = np.random.default_rng(6)
    x = R.round_to(rng.standard_normal((8, 4, 128)), "fp32")
    q, _ = s4r.qk_norm_rope(c, dev(x, c), None, ints(pos))
    check(q, x, None, 0, pos, 5e5, "fp32")
    # the largest positions: 2^-53 of the frequency times 2^31 is 2^-22 of a revolution more
    far = np.array([2 ** 31 - 1, -2 ** 31])
    q, _ = s4r.qk_norm_rope(c, dev(x[:2], c), None, ints(far))
    want = R.norm_rope(x[:2], None, 0, far, 5e5)
    assert np.abs(q.double().cpu().numpy() - want).max() <= np.abs(x).max() * 1.5 * (2 * np.pi * 2.0 ** -20 + 2.0 ** -19)


def test_values_at_the_ends_of_the_range():
    c = cfg(6, 6, 64, 0.0, "fp32")
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 6, 64))
    x[0, 0] = 0                                   # no length: zeros
    x[0, 1] *= 1e38 / np.abs(x[0, 1]).max()       # squares beyond fp32
    x[0, 2] *= 1e-25                              # squares below fp32, under eps
    x[0, 3, 1:] = 0                               # one large number alone
    x[0, 3, 0] = 3e38
    x = R.round_to(x, "fp32")
    one = torch.ones(64, device="cuda")
    q, k = s4r.qk_norm_rope(c, dev(x, c), dev(x, c), None, one, None)
    check(q, x, np.ones(64), 1e-6, [0], 0, "fp32")
    assert torch.equal(k, dev(x, c))
    q, _ = s4r.qk_norm_rope(c, dev(x[:, 1:], c).repeat(1, 2, 1)[:, :6].contiguous(), None, None, one, eps=0.0)
    check(q, np.tile(x[:, 1:], (1, 2, 1))[:, :6], np.ones(64), 0.0, [0], 0, "fp32")
    x[0, 4, 3], x[0, 5, 7] = np.nan, np.inf
    q, _ = s4r.qk_norm_rope(c, dev(x, c), None, None, one)
    q = q[0].cpu().numpy()
    assert np.isfinite(q[:4]).all() and np.isnan(q[4]).all() and np.isnan(q[5, 7]) and not np.delete(q[5], 7).any()


def test_refusals():
    c = cfg(8, 2, 64, 1e4)
    f = torch.zeros(5, 12, 64, dtype=torch.bfloat16, device="cuda")
    q, k, pos = f[:, :8], f[:, 8:10], ints(np.arange(5))
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for call, text in [
            (lambda: s4r.qk_norm_rope(c, q, k, None), "positions"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos[:4]), "entries"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos.long()), "dtype"),
            (lambda: s4r.qk_norm_rope(c, q, k[:4], pos), "tokens"),
            (lambda: s4r.qk_norm_rope(c, q.float(), k, pos), "dtype"),
            (lambda: s4r.qk_norm_rope(c, f[:, :7], k, pos), "shape|packed|expected"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos, w[:32]), "entries"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos, eps=-1.0), "eps"),
            (lambda: s4r.qk_norm_rope(c, q[:0], k[:0], pos[:0]), "no rows"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos, q_out=f[:, 2:10]), "overlap"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos, q_out=f[:, 4:12], k_out=k), "overlap"),
            (lambda: s4r.qk_norm_rope(c, q, k, pos, k_out=f[:, 7:9]), "overlap")]:
        with pytest.raises((ValueError, s4r.S4RError), match=text):
            call()
    assert not f.any()


THETA = 1e6


def layer(rng, B, n, hq, hkv, dh):
    """Rows of a fused projection for n tokens of B sequences."""
    return R.round_to(rng.standard_normal((B, n, hq + 2 * hkv, dh)) * 2, "bf16")


@pytest.mark.parametrize("fmt,cap", [("int8", 272), ("e4m3", 272), ("int8", 4096), ("e4m3", 4096)])
def test_prompt_then_decoding_eager_and_replayed(fmt, cap):
    """A decoding program: prompts of unequal lengths go in, then every step norms and rotates its heads, appends its
    token and attends.  Two steps' graphs share a workspace and are replayed in turn while lengths live on the
    device; eager steps run between the replays.  Every step is compared with the 64-bit attention over the
    reference's cache, whose keys are the kernel's own rotated rows (compared with the reference apart)."""
    B, hq, hkv, dh = 3, 8, 2, 128
    rng = np.random.default_rng(11)
    c = cfg(hq, hkv, dh, THETA, batch=B, capacity=cap)
    wq, wk = (R.round_to(1 + 0.2 * rng.standard_normal(dh), "bf16") for _ in range(2))
    gq, gk = dev(wq, c), dev(wk, c)
    prompt = [130, 1, 61]
    n = max(prompt)
    x = layer(rng, B, n, hq, hkv, dh)
    f = dev(x, c)
    at = np.tile(np.arange(n), (B, 1))
    _, k = s4r.qk_norm_rope(c, None, f[:, :, hq:hq + hkv], ints(at), k_weight=gk)
    check(k.flatten(0, 1), x[:, :, hq:hq + hkv].reshape(B * n, hkv, dh), wk, 1e-6, at.ravel(), THETA, "bf16")
    cache, ws = s4r.kv8_alloc(c, fmt), s4r.alloc_kv8_workspace(c)
    lengths = ints(prompt)
    s4r.kv8_write(c, cache, k, f[:, :, hq + hkv:], counts=lengths)
    ref = R.RefCache(fmt, B, hkv, dh, cap)
    ref.write({"k": k.double().cpu().numpy().reshape(B, n, -1), "v": x[:, :, hq + hkv:].reshape(B, n, -1)}, [0] * B, prompt)

    token = torch.zeros(B, hq + 2 * hkv, dh, dtype=torch.bfloat16, device="cuda")
    outs = [{}, {}]

    def step(o):
        q, k = s4r.qk_norm_rope(c, token[:, :hq], token[:, hq:hq + hkv], lengths, gq, gk)
        s4r.kv8_write(c, cache, k, token[:, hq + hkv:], starts=lengths)
        lengths.add_(1)
        o.update(q=q, k=k, out=s4r.kv8_decode(c, cache, cap, q, ws, lengths=lengths))

    state = [t.clone() for t in (lengths, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(o)
        graphs.append(g)
    for t, was in zip((lengths, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), state):
        t.copy_(was)
    for i in range(72):
        x = layer(rng, B, 1, hq, hkv, dh)[:, 0]
        token.copy_(dev(x, c))
        o = {}
        if i % 3 == 2:
            step(o)
        else:
            graphs[i % 3].replay()
            o = outs[i % 3]
        torch.cuda.synchronize()
        held = [p + i for p in prompt]
        check(o["q"], x[:, :hq], wq, 1e-6, held, THETA, "bf16")
        check(o["k"], x[:, hq:hq + hkv], wk, 1e-6, held, THETA, "bf16")
        ref.write({"k": o["k"].double().cpu().numpy().reshape(B, 1, -1), "v": x[:, hq + hkv:].reshape(B, 1, -1)}, held, [1] * B)
        want, tol = R.attention(ref, o["q"].double().cpu().numpy()[:, None], [p + 1 for p in held])
        assert np.all(np.abs(o["out"].double().cpu().numpy() - want[:, 0]).max(-1) <= tol[:, 0]), f"step {i}"
    for s in "kv":
        assert np.array_equal(getattr(cache, s + "_codes").cpu().numpy(), ref.codes[s])
        assert np.array_equal(getattr(cache, s + "_scales").cpu().numpy(), ref.scales[s])


def test_pre_rope_rows_reach_the_compressed_path():
    """Without the rotation the rows are what the compressed path takes: a prompt kept in 8 bits is read back,
    compressed, and decoded with the library's own step."""
    hq, hkv, dh, n, s = 8, 2, 128, 500, 4
    rng = np.random.default_rng(21)
    c = cfg(hq, hkv, dh, 0.0, capacity=512, rank=64, window=16, topk=64)
    x = layer(rng, 1, n, hq, hkv, dh)
    f = dev(x, c)
    w = torch.ones(dh, dtype=torch.bfloat16, device="cuda")
    q, k = s4r.qk_norm_rope(c, f[:, :, :hq], f[:, :, hq:hq + hkv], None, w, w)
    cache = s4r.kv8_alloc(c, "e4m3")
    s4r.kv8_write(c, cache, k, f[:, :, hq + hkv:])
    back_k, back_v = s4r.kv8_read(c, cache, n)
    # e4m3 keeps half a step of 2^-4 of a number, or of the smallest normal one (2^-6 of the scale)
    for got, had, scales in ((back_k, k, cache.k_scales), (back_v, f[:, :, hq + hkv:], cache.v_scales)):
        a, b = got.float().view(1, n, hkv, dh), had.float()
        unit = scales.repeat_interleave(64, 2)[:, :, :n].transpose(1, 2)[..., None]
        assert torch.all((a - b).abs() <= torch.maximum(b.abs(), unit * 2.0 ** -6) * (2.0 ** -4 + 2.0 ** -8))
    c2 = cfg(hq, hkv, dh, THETA, capacity=512, rank=64, window=16, topk=64)
    g = s4r.prefill(c2, back_k, back_v, eta=0.9)
    out = s4r.decode_step(c2, n - s, q[:, -1].contiguous(), g["sink_k"], g["sink_v"], g["bases_k"], g["bases_v"],
                          g["coef_k"], g["coef_v"], s4r.alloc_workspace(c2))
    assert torch.isfinite(out).all() and out.any()
