"""Axes of the tensors around the 8-bit KV cache: rows that come in another order than the library takes them
are refused, whatever the number of elements; the same order in other axes is taken."""

import pytest
import torch

import paper_2608_00528_amd as s4r
from tests.test_gpu_kv8 import cfg, ints

pytestmark = pytest.mark.gpu

B, N, HQ, HKV, DH, CAP = 2, 3, 6, 3, 64, 128


def rand(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda").to(dtype)


def refused(call, text):
    with pytest.raises((ValueError, s4r.S4RError), match=text):
        call()


def test_rows_written_sequence_by_sequence():
    c = cfg(B, HQ, HKV, DH, CAP)
    k, v = rand(B, N, HKV, DH), rand(B, N, HKV, DH)
    cache = s4r.kv8_alloc(c)
    s4r.kv8_write(c, cache, k, v)
    held = s4r.kv8_read(c, cache, N)
    for x in (k.transpose(0, 1).contiguous(), k.transpose(0, 1), k.transpose(0, 1).flatten(2)):
        refused(lambda: s4r.kv8_write(c, cache, x, v), "sequences|evenly")
        refused(lambda: s4r.kv8_write(c, cache, k, x), "sequences|evenly")
    # the elements of a head in the axis before the heads
    refused(lambda: s4r.kv8_write(c, cache, k.transpose(2, 3).contiguous(), v), "expected")
    assert all(torch.equal(a, b) for a, b in zip(held, s4r.kv8_read(c, cache, N)))
    # the same rows in other axes
    for shape in ((B * N, HKV, DH), (B * N, HKV * DH), (B, 1, N, HKV * DH), (B, N, HKV, 1, DH)):
        other = s4r.kv8_alloc(c)
        s4r.kv8_write(c, other, k.view(shape), v.view(shape))
        assert all(torch.equal(a, b) for a, b in zip(held, s4r.kv8_read(c, other, N)))
    # one sequence, and one row of each
    one = cfg(1, HQ, HKV, DH, CAP)
    s4r.kv8_write(one, s4r.kv8_alloc(one), k.flatten(0, 1), v)
    four = cfg(4, HQ, HKV, DH, CAP)
    s4r.kv8_write(four, s4r.kv8_alloc(four), rand(2, 2, HKV, DH), rand(4, HKV * DH), row0=9)


def test_query_tokens_sequence_by_sequence():
    c = cfg(B, HQ, HKV, DH, CAP)
    cache, ws = s4r.kv8_alloc(c), s4r.alloc_kv8_workspace(c, N)
    s4r.kv8_write(c, cache, rand(B, 100, HKV, DH), rand(B, 100, HKV, DH))
    q = rand(B, N, HQ, DH)
    want = s4r.kv8_decode(c, cache, 100, q, ws)
    turned = q.transpose(0, 1).contiguous()
    refused(lambda: s4r.kv8_decode(c, cache, 100, turned, ws), "axes")
    refused(lambda: s4r.kv8_decode(c, cache, 100, q.transpose(2, 3).contiguous(), ws), "axes")
    out = torch.full((N, B, HQ, DH), 7.0, device="cuda")
    refused(lambda: s4r.kv8_decode(c, cache, 100, q, ws, out=out), "axes")
    refused(lambda: s4r.kv8_decode(c, cache, 100, q, ws, out=out.view(B, N, DH, HQ)), "axes")
    assert bool((out == 7).all())
    # the same rows in other axes
    for shape in ((B * N, HQ, DH), (B, N * HQ, DH), (B, N, HQ * DH), (B, N, HKV, HQ // HKV, DH), (B * N * HQ * DH,)):
        got = s4r.kv8_decode(c, cache, 100, q.view(shape), ws)
        assert got.shape == shape and torch.equal(got.view_as(want), want)
        got = s4r.kv8_decode(c, cache, 100, q, ws, out=torch.empty(shape, device="cuda"))
        assert got.shape == shape and torch.equal(got.view_as(want), want)
    one = s4r.kv8_decode(c, cache, 98, q[:, 0].contiguous(), ws)
    assert one.shape == (B, HQ, DH) and torch.equal(one, want[:, 0])


def test_rows_read_into_two_tensors_sequence_by_sequence():
    c = cfg(B, HQ, HKV, DH, CAP)
    cache = s4r.kv8_alloc(c)
    s4r.kv8_write(c, cache, rand(B, N, HKV, DH), rand(B, N, HKV, DH))
    k, v = s4r.kv8_read(c, cache, N)
    a = torch.zeros(2, B, N, HKV * DH, dtype=torch.bfloat16, device="cuda")
    refused(lambda: s4r.kv8_read(c, cache, N, k=a[0], v=a[0]), "overlap")
    flat = a.flatten()
    n = k.numel()
    refused(lambda: s4r.kv8_read(c, cache, N, k=flat[:n], v=flat[n - 8:2 * n - 8]), "overlap")
    refused(lambda: s4r.kv8_read(c, cache, N, k=flat[n - 8:2 * n - 8], v=flat[:n]), "overlap")
    refused(lambda: s4r.kv8_read(c, cache, N, k=a[0].view(N, B, HKV * DH)), "axes")
    refused(lambda: s4r.kv8_read(c, cache, N, v=a[0].view(B, N, DH, HKV)), "axes")
    assert not a.any()
    # side by side, and the same rows in other axes
    s4r.kv8_read(c, cache, N, k=a[1], v=a[0])
    assert torch.equal(a[1], k) and torch.equal(a[0], v)
    a.zero_()
    s4r.kv8_read(c, cache, N, k=flat[:n], v=a[1].view(B * N, HKV, DH))
    assert torch.equal(a[0], k) and torch.equal(a[1], v)


def test_heads_of_the_same_tokens():
    c = s4r.make_config(batch=1, n_q_heads=HQ, n_kv_heads=HKV, head_dim=DH, rank=32, capacity=64, rope_theta=1e4)
    q, k = rand(B, N, HQ, DH), rand(B, N, HKV, DH)
    pos = ints(range(B * N)).view(B, N)
    want = s4r.qk_norm_rope(c, q, k, pos)
    refused(lambda: s4r.qk_norm_rope(c, q, k.transpose(0, 1).contiguous(), pos), "axes")
    refused(lambda: s4r.qk_norm_rope(c, q, k, pos.t().contiguous()), "axes")
    refused(lambda: s4r.qk_norm_rope(c, q, None, pos.t().contiguous()), "axes")
    refused(lambda: s4r.qk_norm_rope(c, q.transpose(2, 3).contiguous(), k, pos), "expected")
    out = torch.zeros(N, B, HQ, DH, dtype=torch.bfloat16, device="cuda")
    refused(lambda: s4r.qk_norm_rope(c, q, k, pos, q_out=out), "axes")
    refused(lambda: s4r.qk_norm_rope(c, q, k, pos, q_out=out.view(B, N, DH, HQ)), "expected")
    assert not out.any()
    # the same tokens in other axes
    for a, b, p in ((q.flatten(0, 1), k, pos), (q, k.flatten(0, 1), pos.flatten()), (q.flatten(2), k.flatten(2), pos),
                    (q.view(B, N, HKV, HQ // HKV, DH), k.view(B, 1, N, HKV, DH), pos.view(1, B, N)),
                    (q.flatten(0, 1).flatten(1), k.flatten(0, 1), pos)):
        got = s4r.qk_norm_rope(c, a, b, p)
        assert got[0].shape == a.shape and got[1].shape == b.shape
        assert all(torch.equal(x.flatten(), y.flatten()) for x, y in zip(got, want))
        got = s4r.qk_norm_rope(c, a, b, p, q_out=out.view(B * N, HQ, DH), k_out=torch.empty_like(k))
        assert all(torch.equal(x.flatten(), y.flatten()) for x, y in zip(got, want))


def test_cache_of_another_config():
    """As many elements, other sequences and heads."""
    c, other = cfg(B, HQ, HKV, DH, CAP), cfg(HKV, HQ, B, DH, CAP)
    cache, ws = s4r.kv8_alloc(other), s4r.alloc_kv8_workspace(c)
    x = rand(B, N, HKV, DH)
    refused(lambda: s4r.kv8_write(c, cache, x, x), "axes")
    refused(lambda: s4r.kv8_read(c, cache, N), "axes")
    refused(lambda: s4r.kv8_decode(c, cache, 100, rand(B, HQ, DH), ws), "axes")
    mine = s4r.kv8_alloc(c)
    mine.v_scales = cache.v_scales
    refused(lambda: s4r.kv8_write(c, mine, x, x), "axes")
    assert not cache.k_codes.any() and not mine.k_codes.any() and not cache.v_scales.any()
    # flat memory of the program's own
    mine = s4r.kv8_alloc(c)
    flat = s4r.KV8Cache("int8", *[t.view(-1) for t in (mine.k_codes, mine.k_scales, mine.v_codes, mine.v_scales)])
    s4r.kv8_write(c, flat, x, x)
    assert all(torch.equal(a, b) for a, b in zip(s4r.kv8_read(c, flat, N), s4r.kv8_read(c, mine, N)))
    assert mine.k_scales.any()


@pytest.mark.parametrize("n", [2, 5])
def test_heads_before_tokens_are_refused(n):
    """[B, heads, n, d_h], the order in which other attention calls take them."""
    c = cfg(B, HQ, HKV, DH, CAP)
    plain = s4r.make_config(batch=1, n_q_heads=HQ, n_kv_heads=HKV, head_dim=DH, rank=32, capacity=64)
    cache, ws = s4r.kv8_alloc(c), s4r.alloc_kv8_workspace(c, n)
    q, k = rand(B, HQ, n, DH), rand(B, HKV, n, DH)
    refused(lambda: s4r.kv8_write(c, cache, k, k), "expected")
    refused(lambda: s4r.kv8_decode(c, cache, 100, q, ws), "axes")
    out = torch.zeros(B, HQ, n, DH, device="cuda")
    refused(lambda: s4r.kv8_decode(c, cache, 100, q.transpose(1, 2).contiguous(), ws, out=out), "axes")
    refused(lambda: s4r.kv8_read(c, cache, n, k=k.zero_()), "axes")
    refused(lambda: s4r.qk_norm_rope(plain, q, None, None), "expected|spaced")
    assert not cache.k_codes.any() and not out.any() and not k.any()
    s4r.kv8_write(c, cache, k.transpose(1, 2).contiguous(), k.transpose(1, 2).contiguous())
