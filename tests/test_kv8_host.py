"""The 8-bit cache's and the head norms' checks on the host (no GPU): refusals of
the C ABI, sizes, refusals of the binding, and the reference's own layout."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_00528_amd as s4r
from paper_2608_00528_amd import _lib as L
from tests import kv8_reference as R

host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers never reach a machine with a GPU")

P = 0x10000                 # aligned, never dereferenced
MIS = 0x10004               # 4-byte aligned only
ODD = 0x10002


def cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, rank=32, capacity=1008, rope_theta=10000.0)
    base.update(kw)
    return s4r.make_config(**base)


def kv8(**kw):
    f = dict(format=0, k_codes=P, k_scales=P, v_codes=P, v_scales=P)
    f.update(kw)
    return L.KV8(*[f[n] for n, _ in L.KV8._fields_])


def refused(status, text):
    assert L.STATUS_NAMES[status[0]] == status[1], L.load().s4r_last_error()
    assert text in L.load().s4r_last_error().decode()


def test_sizes():
    # 1008 tokens: 15.75 blocks
    assert s4r.kv8_size(cfg()) == (2 * 2 * 16 * 64 * 64, 2 * 2 * 16)
    assert s4r.kv8_size(cfg(head_dim=128, batch=1, capacity=64)) == (2 * 64 * 128, 2)
    one, two = s4r.kv8_workspace_size(cfg()), s4r.kv8_workspace_size(cfg(), 32)
    assert 0 < one < two and one % 256 == 0 and two % 256 == 0
    # a workspace serves every smaller number of query tokens
    for c in (cfg(), cfg(capacity=131072), cfg(n_q_heads=16, n_kv_heads=1, head_dim=128), cfg(n_q_heads=4, n_kv_heads=4, capacity=16)):
        g = c.n_q_heads // c.n_kv_heads
        sizes = [s4r.kv8_workspace_size(c, n) for n in range(1, 128 // g + 1)]
        assert sizes == sorted(sizes)
    for n in (0, 33):                                   # n * G = 132 > 128
        with pytest.raises(s4r.S4RError):
            s4r.kv8_workspace_size(cfg(), n)
    with pytest.raises(s4r.S4RError, match="NULL_ARG"):
        L.check(L.load().s4r_kv8_size(ctypes.byref(cfg()), None, None))
    with pytest.raises(s4r.S4RError, match="BAD_SHAPE"):
        s4r.kv8_size(cfg(capacity=1000))


@host_only
def test_write_and_read_refusals():
    lib = L.load()

    def write(c=None, k=None, n=4, row0=0, starts=None, counts=None, kr=P, ks=128, vr=P, vs=128):
        return lib.s4r_kv8_write(ctypes.byref(c or cfg()), ctypes.byref(k or kv8()), n, row0, starts, counts, kr, ks,
                                 vr, vs, None)

    for kw, text in [(dict(k=kv8(format=2)), "format"), (dict(n=0), "n_rows"), (dict(n=1009), "n_rows"),
                     (dict(row0=-1), "rows"), (dict(row0=1005), "rows"), (dict(row0=1009, counts=P), "rows"),
                     (dict(ks=127), "stride"), (dict(vs=64), "stride")]:
        refused((write(**kw), "BAD_SHAPE"), text)
    for kw, text in [(dict(k=kv8(k_codes=None)), "k_codes"), (dict(k=kv8(v_scales=None)), "v_scales"),
                     (dict(kr=None), "k_rows"), (dict(vr=None), "v_rows")]:
        refused((write(**kw), "NULL_ARG"), text)
    for kw, text in [(dict(k=kv8(v_codes=MIS)), "v_codes"), (dict(kr=MIS), "k_rows"), (dict(starts=ODD), "starts"),
                     (dict(counts=ODD), "counts"), (dict(ks=132), "k_rows"),
                     (dict(c=cfg(dtype="fp32"), vs=130), "v_rows")]:
        refused((write(**kw), "MISALIGNED"), text)
    refused((write(ks=1 << 32), "UNSUPPORTED"), "stride")
    refused((lib.s4r_kv8_write(ctypes.byref(cfg()), None, 4, 0, None, None, P, 128, P, 128, None), "NULL_ARG"), "cache")
    refused((write(c=cfg(batch=40000)), "UNSUPPORTED"), "batch")
    refused((write(c=cfg(batch=20000, n_q_heads=32, n_kv_heads=32, capacity=1 << 17)), "UNSUPPORTED"), "blocks")

    def read(k=None, n=4, row0=0, starts=None, counts=None, ko=P, vo=P):
        return lib.s4r_kv8_read(ctypes.byref(cfg()), ctypes.byref(k or kv8()), n, row0, starts, counts, ko, vo, None)

    refused((read(n=0), "BAD_SHAPE"), "n_rows")
    refused((read(row0=1005), "BAD_SHAPE"), "rows")
    refused((read(ko=None), "NULL_ARG"), "k_out")
    refused((read(vo=MIS), "MISALIGNED"), "v_out")
    refused((read(starts=ODD), "MISALIGNED"), "starts")


@host_only
def test_decode_refusals():
    lib = L.load()
    W = 0x100000

    def decode(c=None, k=None, N=100, lengths=None, nq=1, q=P, out=P, ws=W, nbytes=None):
        c = c or cfg()
        nbytes = s4r.kv8_workspace_size(c, nq) if nbytes is None else nbytes
        return lib.s4r_kv8_decode(ctypes.byref(c), ctypes.byref(k or kv8()), N, lengths, nq, q, out, ws, nbytes, None)

    refused((decode(N=0), "BAD_SHAPE"), "N = 0")
    refused((decode(N=1009), "BAD_SHAPE"), "N = 1009")
    refused((decode(nq=0, nbytes=1), "BAD_SHAPE"), "n_q")
    refused((decode(nq=33, nbytes=1), "UNSUPPORTED"), "n_q")
    refused((decode(q=None), "NULL_ARG"), "q")
    refused((decode(out=None), "NULL_ARG"), "out")
    refused((decode(ws=None), "NULL_ARG"), "ws")
    refused((decode(q=MIS), "MISALIGNED"), "q")
    refused((decode(lengths=ODD), "MISALIGNED"), "lengths")
    refused((decode(ws=W + 16), "MISALIGNED"), "ws")
    refused((decode(nbytes=s4r.kv8_workspace_size(cfg()) - 1), "WORKSPACE"), "workspace")
    refused((decode(k=kv8(format=-1)), "BAD_SHAPE"), "format")
    refused((decode(c=cfg(head_dim=96), nbytes=1), "UNSUPPORTED"), "head_dim")
    refused((decode(c=cfg(n_q_heads=34), nbytes=1), "UNSUPPORTED"), "G")


@host_only
def test_norm_refusals():
    lib = L.load()

    def norm(c=None, n=3, q=P, qs=512, k=P, ks=128, eps=1e-6, pos=P, qo=P, qos=512, ko=P, kos=128, qw=P, kw=P):
        return lib.s4r_qk_norm_rope(ctypes.byref(c or cfg()), n, q, qs, k, ks, qw, kw, eps, pos, qo, qos, ko, kos, None)

    for kw, text in [(dict(n=0), "n_tokens"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                     (dict(eps=float("inf")), "eps"), (dict(qs=511), "q stride"), (dict(kos=64), "k_out stride")]:
        refused((norm(**kw), "BAD_SHAPE"), text)
    for kw, text in [(dict(q=None), "q and q_out"), (dict(ko=None), "k and k_out"), (dict(pos=None), "positions"),
                     (dict(q=None, qo=None, k=None, ko=None), "both")]:
        refused((norm(**kw), "NULL_ARG"), text)
    for kw, text in [(dict(q=MIS), "q"), (dict(qos=516), "q_out"), (dict(ks=132), "k"), (dict(kw=MIS), "k_weight"),
                     (dict(pos=ODD), "positions")]:
        refused((norm(**kw), "MISALIGNED"), text)


def test_binding_refuses_cpu_tensors_and_wrong_sizes():
    c = cfg()
    x = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        s4r.qk_norm_rope(c, x, None, None)
    with pytest.raises(ValueError, match="q or k"):
        s4r.qk_norm_rope(c, None, None, None)
    with pytest.raises(ValueError, match="q_out without q"):
        s4r.qk_norm_rope(c, None, None, None, q_out=x)
    with pytest.raises(ValueError, match="format"):
        s4r.kv8_alloc(c, "int4")
    with pytest.raises(ValueError, match="format"):
        s4r.KV8Cache("fp8", x, x, x, x)
    with pytest.raises(ValueError, match="GPU"):
        s4r.kv8_alloc(c, device="cpu")
    with pytest.raises(ValueError, match="KV8Cache"):
        s4r.kv8_write(c, None, x, x)


@pytest.mark.parametrize("dh", [64, 128])
def test_reference_layout_is_a_permutation(dh):
    for side in "kv":
        assert np.array_equal(np.sort(R.offsets(side, dh).ravel()), np.arange(64 * dh))
    # the two orders as reshapes
    x = np.arange(64 * dh).reshape(64, dh)
    k = x.reshape(4, 16, dh // 64, 4, 16).transpose(0, 2, 3, 1, 4).ravel()
    v = x.reshape(4, 4, 4, dh // 16, 16).transpose(3, 1, 4, 2, 0).ravel()
    for side, want in (("k", k), ("v", v)):
        got = np.empty(64 * dh, int)
        got[R.offsets(side, dh)] = x
        assert np.array_equal(got, want)


def test_reference_rounding():
    y = np.array([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 0.49999999])
    assert np.array_equal(R.nearest(y, "int8"), [0, 2, 2, 0, -2, 126, 0])
    # every e4m3 number is its own nearest; halfway values go to the even code
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    x = R.from_bytes(codes, "e4m3")
    assert np.array_equal(R.nearest(x, "e4m3"), x)
    pos = x[:127]
    mid = (pos[:-1] + pos[1:]) / 2
    even = np.where(np.arange(126) % 2 == 0, pos[:-1], pos[1:])
    assert np.array_equal(R.nearest(mid, "e4m3"), even)
    assert np.array_equal(R.nearest(mid * (1 + 2.0 ** -30), "e4m3"), pos[1:])
    t = torch.linspace(-448, 448, 100001, dtype=torch.float32)
    assert np.array_equal(R.nearest(t.double().numpy(), "e4m3"), t.to(torch.float8_e4m3fn).double().numpy())
    assert R.scale_of(np.array([448.0]), "e4m3") == 1 and R.scale_of(np.array([448.1]), "e4m3") == 2
    assert R.scale_of(np.array([127.0]), "int8") == 1


def test_reference_growth_by_hand():
    c = R.RefCache("int8", 1, 1, 64, 64)
    row = np.zeros((1, 1, 64))
    row[0, 0, :3] = [127, 63, -1]
    c.write({"k": row, "v": row}, [0], [1])
    assert c.scales["k"][0, 0, 0] == 1 and list(c.block("k", 0, 0, 0)[0, :3]) == [127, 63, -1]
    row = row * 2
    c.write({"k": row, "v": row}, [1], [1])
    # the first token anew on the doubled scale: 63.5 -> 64 (even), 31.5 -> 32, -0.5 -> 0
    assert c.scales["k"][0, 0, 0] == 2
    assert list(c.block("k", 0, 0, 0)[0, :3]) == [64, 32, 0] and list(c.block("v", 0, 0, 0)[1, :3]) == [127, 63, -1]
