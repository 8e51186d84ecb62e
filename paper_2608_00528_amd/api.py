"""Python binding of the S^4R C ABI (include/s4r.h).

Thin marshalling only: every function checks tensor placement / dtype /
contiguity, allocates outputs with torch when the caller passes none, and
calls the library on torch's current HIP stream.  All arithmetic happens in
the gfx950 kernels of libs4r.so; there is no CPU path.
"""

import ctypes
import math

import torch

from . import _lib as L

_DTYPES = {"bf16": (L.S4R_BF16, torch.bfloat16), "fp32": (L.S4R_FP32, torch.float32)}
_POOL = {"max": L.S4R_POOL_MAX, "avg": L.S4R_POOL_AVG}
_AGG = {"mean": L.S4R_AGG_MEAN, "max": L.S4R_AGG_MAX}
_KV_FORMATS = {"int8": L.S4R_KV_INT8, "e4m3": L.S4R_KV_E4M3}


def make_config(*, batch, n_q_heads, n_kv_heads, head_dim, rank, capacity, basis_groups=1, n_sink=4,
                window=64, q_window=1, topk=1024, pool_kernel=7, pool_mode="max", group_agg="mean",
                bases_shared=False, rope_theta=0.0, dtype="bf16", rank_v=0):
    c = L.Config()
    c.batch, c.n_q_heads, c.n_kv_heads, c.head_dim = batch, n_q_heads, n_kv_heads, head_dim
    c.basis_groups, c.rank, c.n_sink, c.window = basis_groups, rank, n_sink, window
    c.q_window, c.topk, c.pool_kernel = q_window, topk, pool_kernel
    c.pool_mode, c.group_agg = _POOL[pool_mode], _AGG[group_agg]
    c.bases_shared = int(bool(bases_shared))
    c.capacity = capacity
    c.rope_theta = float(rope_theta)
    c.dtype = _DTYPES[dtype][0]
    c.rank_v = rank_v
    return c


def value_config(cfg):
    """The configuration whose `rank` is the value rank: the layout helpers
    (pack_coef / unpack_coef) take a cache's width from `rank`, so a value
    cache of an asymmetric configuration is converted with this one."""
    c = L.Config()
    ctypes.pointer(c)[0] = cfg
    if cfg.rank_v:
        c.rank, c.rank_v = cfg.rank_v, 0
    return c


def storage_dtype(cfg):
    return torch.bfloat16 if cfg.dtype == L.S4R_BF16 else torch.float32


def _ptr(t, name, dtype=None, required=True):
    """The device address of a tensor argument, as an int (0.3 us a call: a step
    marshals up to 18 of them beside its launches)."""
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    return t.data_ptr()


# torch's getter of a device's current stream handle, where this torch has it: it
# is no public name
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    """The current stream's handle, without the torch.cuda.Stream object around
    it where torch offers that (0.3 against 3 us)."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _cfgp(cfg):
    return ctypes.byref(cfg)


def version():
    return L.load().s4r_version().decode()


def workspace_size(cfg):
    n = ctypes.c_size_t()
    L.check(L.load().s4r_workspace_size(_cfgp(cfg), ctypes.byref(n)))
    return n.value


def alloc_workspace(cfg, device="cuda"):
    return torch.empty(workspace_size(cfg), dtype=torch.uint8, device=device)


def num_selected(cfg, length):
    m = L.load().s4r_num_selected(_cfgp(cfg), length)
    if m < 0:
        raise L.S4RError(L.S4R_ERR_BAD_SHAPE, L.load().s4r_last_error().decode())
    return m


def _G(cfg):
    return cfg.n_q_heads // cfg.n_kv_heads


def rank_stride(rank):
    """Storage width of a rank: the rank rounded up to a multiple of 32 (the
    coefficient layout works in 32-column blocks; the extra columns hold zeros)."""
    return (rank + 31) // 32 * 32


def _R(cfg):
    return rank_stride(cfg.rank) * cfg.basis_groups


def pad_latent(x, rank, basis_groups=1):
    """Lay latent data out in the library's storage width: the last axis of
    `x` holds basis_groups blocks of `rank` columns (bases: one block); each
    block moves to its own rank_stride(rank) columns, the padding columns zero.
    Works on torch tensors and numpy arrays; returns `x` itself when the rank
    is already a multiple of 32."""
    rs = rank_stride(rank)
    if rs == rank:
        return x
    if x.shape[-1] != rank * basis_groups:
        raise ValueError(f"last axis {x.shape[-1]} is not {basis_groups} x rank {rank}")
    shape = tuple(x.shape[:-1]) + (basis_groups * rs,)
    if isinstance(x, torch.Tensor):
        out = torch.zeros(shape, dtype=x.dtype, device=x.device)
    else:
        import numpy as np
        out = np.zeros(shape, dtype=x.dtype)
    for g in range(basis_groups):
        out[..., g * rs:g * rs + rank] = x[..., g * rank:(g + 1) * rank]
    return out


def score_latent(cfg, length, q, bases_k, coef_k, ws, qwin_prev=None, scores=None, qcoef=None):
    dt = storage_dtype(cfg)
    dev = q.device
    if scores is None:
        scores = torch.empty((cfg.batch, length), dtype=torch.float32, device=dev)
    L.check(L.load().s4r_score_latent(
        _cfgp(cfg), length, _ptr(q, "q", dt), _ptr(qwin_prev, "qwin_prev", torch.float32, False),
        _ptr(bases_k, "bases_k", dt), _ptr(coef_k, "coef_k", dt), _ptr(scores, "scores", torch.float32),
        _ptr(qcoef, "qcoef", torch.float32, False), _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))
    return scores


def select_topk(cfg, length, scores, ws, idx=None):
    if idx is None:
        idx = torch.empty((cfg.batch, num_selected(cfg, length)), dtype=torch.int32, device=scores.device)
    L.check(L.load().s4r_select_topk(_cfgp(cfg), length, _ptr(scores, "scores", torch.float32),
                                     _ptr(idx, "idx", torch.int32), _ptr(ws, "ws", torch.uint8), ws.numel(),
                                     _stream()))
    return idx


def reconstruct(cfg, length, idx, bases_k, bases_v, coef_k, coef_v, k_hat=None, v_hat=None):
    dt = storage_dtype(cfg)
    m = idx.shape[1]
    Dp = cfg.n_kv_heads * cfg.head_dim
    if k_hat is None:
        k_hat = torch.empty((cfg.batch, m, Dp), dtype=torch.float32, device=idx.device)
    if v_hat is None:
        v_hat = torch.empty((cfg.batch, m, Dp), dtype=torch.float32, device=idx.device)
    L.check(L.load().s4r_reconstruct(_cfgp(cfg), length, m, _ptr(idx, "idx", torch.int32),
                                     _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt),
                                     _ptr(coef_k, "coef_k", dt), _ptr(coef_v, "coef_v", dt),
                                     _ptr(k_hat, "k_hat", torch.float32), _ptr(v_hat, "v_hat", torch.float32),
                                     _stream()))
    return k_hat, v_hat


def sparse_attn(cfg, length, q, sink_k, sink_v, idx, k_sel, v_sel, ws, out=None):
    dt = storage_dtype(cfg)
    m = idx.shape[1] if idx is not None else 0
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_sparse_attn(_cfgp(cfg), length, m, _ptr(q, "q", dt),
                                     _ptr(sink_k, "sink_k", dt, need_sink), _ptr(sink_v, "sink_v", dt, need_sink),
                                     _ptr(idx, "idx", torch.int32, m > 0), _ptr(k_sel, "k_sel", torch.float32, m > 0),
                                     _ptr(v_sel, "v_sel", torch.float32, m > 0), _ptr(out, "out", torch.float32),
                                     _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))
    return out


def decode_step(cfg, length, q, sink_k, sink_v, bases_k, bases_v, coef_k, coef_v, ws, qwin_prev=None,
                win_k=None, win_v=None, k_new=None, v_new=None, out=None, idx_out=None, scores_out=None):
    dt = storage_dtype(cfg)
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_decode_step(
        _cfgp(cfg), length, _ptr(q, "q", dt), _ptr(qwin_prev, "qwin_prev", torch.float32, False),
        _ptr(sink_k, "sink_k", dt, need_sink), _ptr(sink_v, "sink_v", dt, need_sink),
        _ptr(win_k, "win_k", dt, False), _ptr(win_v, "win_v", dt, False),
        _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt), _ptr(coef_k, "coef_k", dt),
        _ptr(coef_v, "coef_v", dt), _ptr(k_new, "k_new", dt, False), _ptr(v_new, "v_new", dt, False),
        _ptr(out, "out", torch.float32), _ptr(idx_out, "idx_out", torch.int32, False),
        _ptr(scores_out, "scores_out", torch.float32, False), _ptr(ws, "ws", torch.uint8), ws.numel(),
        _stream()))
    return out


def window_state_size(cfg):
    """Bytes of the window state: [B, q_window, G, capacity] fp32 softmax rows,
    and for longer windows the older rows' running sum [2, B, G, capacity]
    fp64 after them."""
    n = ctypes.c_size_t()
    L.check(L.load().s4r_window_state_size(_cfgp(cfg), ctypes.byref(n)))
    return n.value


def alloc_window_state(cfg, device="cuda"):
    """A zeroed window state of window_state_size(cfg) bytes (fp32 elements)."""
    return torch.zeros((window_state_size(cfg) // 4,), dtype=torch.float32, device=device)


def window_state_init(cfg, length, qwin_prev, coef_k, state, ws):
    """Softmax rows of the window's q_window - 1 older queries (their
    coefficient rows qwin_prev [B, G, q_window - 1, R]) for a windowed step at
    `length`."""
    dt = storage_dtype(cfg)
    L.check(L.load().s4r_window_state_init(
        _cfgp(cfg), length, _ptr(qwin_prev, "qwin_prev", torch.float32), _ptr(coef_k, "coef_k", dt),
        _ptr(state, "state", torch.float32), _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))
    return state


def decode_step_windowed(cfg, length, q, state, sink_k, sink_v, bases_k, bases_v, coef_k, coef_v, ws,
                         win_k=None, win_v=None, k_new=None, v_new=None, out=None, idx_out=None, scores_out=None):
    """The fused step with the window state in place of qwin_prev (steps at
    consecutive lengths); the newest query row's softmax is stored in it."""
    dt = storage_dtype(cfg)
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_decode_step_windowed(
        _cfgp(cfg), length, _ptr(q, "q", dt), _ptr(state, "state", torch.float32),
        _ptr(sink_k, "sink_k", dt, need_sink), _ptr(sink_v, "sink_v", dt, need_sink),
        _ptr(win_k, "win_k", dt, False), _ptr(win_v, "win_v", dt, False),
        _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt), _ptr(coef_k, "coef_k", dt),
        _ptr(coef_v, "coef_v", dt), _ptr(k_new, "k_new", dt, False), _ptr(v_new, "v_new", dt, False),
        _ptr(out, "out", torch.float32), _ptr(idx_out, "idx_out", torch.int32, False),
        _ptr(scores_out, "scores_out", torch.float32, False), _ptr(ws, "ws", torch.uint8), ws.numel(),
        _stream()))
    return out


def decode_step_noalloc(cfg, length, q, sink_k, sink_v, bases_k, bases_v, coef_k, coef_v, qwin_prev=None,
                        win_k=None, win_v=None, k_new=None, v_new=None, out=None, idx_out=None, scores_out=None):
    """The fused step on the library's own per-device scratch (no workspace
    argument); configurations needing more than 64 MiB of it are refused."""
    dt = storage_dtype(cfg)
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_decode_step_noalloc(
        _cfgp(cfg), length, _ptr(q, "q", dt), _ptr(qwin_prev, "qwin_prev", torch.float32, False),
        _ptr(sink_k, "sink_k", dt, need_sink), _ptr(sink_v, "sink_v", dt, need_sink),
        _ptr(win_k, "win_k", dt, False), _ptr(win_v, "win_v", dt, False),
        _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt), _ptr(coef_k, "coef_k", dt),
        _ptr(coef_v, "coef_v", dt), _ptr(k_new, "k_new", dt, False), _ptr(v_new, "v_new", dt, False),
        _ptr(out, "out", torch.float32), _ptr(idx_out, "idx_out", torch.int32, False),
        _ptr(scores_out, "scores_out", torch.float32, False), _stream()))
    return out


def decode_step_ragged(cfg, lengths, q, sink_k, sink_v, bases_k, bases_v, coef_k, coef_v, ws, qwin_prev=None,
                       win_k=None, win_v=None, k_new=None, v_new=None, out=None, idx_out=None, scores_out=None):
    """The fused step over a ragged batch: lengths is a sequence of B ints
    (each sequence's L, the appended token included)."""
    dt = storage_dtype(cfg)
    if len(lengths) != cfg.batch:
        raise ValueError(f"lengths has {len(lengths)} entries for a batch of {cfg.batch}")
    lens = (ctypes.c_int64 * cfg.batch)(*[int(x) for x in lengths])
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_decode_step_ragged(
        _cfgp(cfg), lens, _ptr(q, "q", dt), _ptr(qwin_prev, "qwin_prev", torch.float32, False),
        _ptr(sink_k, "sink_k", dt, need_sink), _ptr(sink_v, "sink_v", dt, need_sink),
        _ptr(win_k, "win_k", dt, False), _ptr(win_v, "win_v", dt, False),
        _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt), _ptr(coef_k, "coef_k", dt),
        _ptr(coef_v, "coef_v", dt), _ptr(k_new, "k_new", dt, False), _ptr(v_new, "v_new", dt, False),
        _ptr(out, "out", torch.float32), _ptr(idx_out, "idx_out", torch.int32, False),
        _ptr(scores_out, "scores_out", torch.float32, False), _ptr(ws, "ws", torch.uint8), ws.numel(),
        _stream()))
    return out


def project_queries(cfg, q_rows, bases_k, ws, out=None):
    """C^Q rows [B, G, n, R] fp32 of the queries q_rows [B, n, h_q, d_h] (the
    initial query window of the prefill: qwin_prev for n = W_q - 1)."""
    dt = storage_dtype(cfg)
    n = q_rows.shape[1]
    G = cfg.n_q_heads // cfg.n_kv_heads
    if out is None:
        out = torch.empty((cfg.batch, G, n, _R(cfg)), dtype=torch.float32, device=q_rows.device)
    L.check(L.load().s4r_project_queries(_cfgp(cfg), n, _ptr(q_rows, "q_rows", dt), _ptr(bases_k, "bases_k", dt),
                                         _ptr(out, "out", torch.float32), _ptr(ws, "ws", torch.uint8), ws.numel(),
                                         _stream()))
    return out


def prefill_bases(cfg, n_rows, s_k, s_v, eta=0.2, center=False, bases_k=None, bases_v=None, sample_idx=None,
                  ws=None):
    """Bases of a prompt's non-sink raw K/V rows [B, n_rows, Dp] (hybrid
    sample, token-wise normalisation, truncated SVD; Section 3.1.2).  Returns
    (bases_k, bases_v); sample_idx (int32, num_samples entries) receives the
    sampled positions when given."""
    dt = storage_dtype(cfg)
    lib = L.load()
    dg = cfg.n_kv_heads * cfg.head_dim // cfg.basis_groups
    shape = lambda r: (cfg.batch, cfg.basis_groups, dg, rank_stride(r))  # noqa: E731
    if bases_k is None:
        bases_k = torch.empty(shape(cfg.rank), dtype=dt, device=s_k.device)
    if bases_v is None:
        bases_v = torch.empty(shape(cfg.rank_v or cfg.rank), dtype=dt, device=s_k.device)
    if ws is None:
        ws = torch.empty(prefill_bases_workspace_size(cfg, n_rows, eta), dtype=torch.uint8, device=s_k.device)
    L.check(lib.s4r_prefill_bases(_cfgp(cfg), n_rows, _ptr(s_k, "s_k", dt), _ptr(s_v, "s_v", dt), float(eta),
                                  int(bool(center)), _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt),
                                  _ptr(sample_idx, "sample_idx", torch.int32, False), _ptr(ws, "ws", torch.uint8),
                                  ws.numel(), _stream()))
    return bases_k, bases_v


def prefill_bases_workspace_size(cfg, n_rows, eta=0.2):
    sz = ctypes.c_size_t()
    L.check(L.load().s4r_prefill_bases_workspace_size(_cfgp(cfg), n_rows, float(eta), ctypes.byref(sz)))
    return sz.value


def num_samples(n_rows, eta=0.2):
    return L.load().s4r_prefill_num_samples(n_rows, float(eta))


def prefill_project(cfg, n_rows, s_k, s_v, bases_k, bases_v, coef_k, coef_v, ws):
    """Bulk projection of a prompt's non-sink raw K/V rows [B, n_rows, Dp]
    into rows [0, n_rows) of the tiled coefficient caches (ws: the decode
    workspace)."""
    dt = storage_dtype(cfg)
    L.check(L.load().s4r_prefill_project(_cfgp(cfg), n_rows, _ptr(s_k, "s_k", dt), _ptr(s_v, "s_v", dt),
                                         _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt),
                                         _ptr(coef_k, "coef_k", dt), _ptr(coef_v, "coef_v", dt),
                                         _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))


def prefill(cfg, S_k, S_v, eta=0.2, center=False, ws=None):
    """The prefill stage of Section 3.1 on the GPU for a prompt's raw pre-RoPE
    keys / values S_k, S_v [B, N, Dp] (sinks first): the first n_sink rows
    kept as the sinks, the bases of the non-sink rows (s4r_prefill_bases:
    hybrid sample with ratio eta, token-wise normalisation, optional
    centring, truncated SVD) and their bulk projection into tiled coefficient
    caches of cfg.capacity rows (s4r_prefill_project).  Returns a dict of
    device tensors sink_k, sink_v, bases_k, bases_v, coef_k, coef_v."""
    s = cfg.n_sink
    n = S_k.shape[1] - s
    sink_k, sink_v = S_k[:, :s].contiguous(), S_v[:, :s].contiguous()
    X_k, X_v = S_k[:, s:].contiguous(), S_v[:, s:].contiguous()
    bases_k, bases_v = prefill_bases(cfg, n, X_k, X_v, eta=eta, center=center)
    dt = storage_dtype(cfg)
    coef_k = torch.zeros((cfg.batch, cfg.capacity, _R(cfg)), dtype=dt, device=S_k.device)
    coef_v = torch.zeros((cfg.batch, cfg.capacity, _R(value_config(cfg))), dtype=dt, device=S_k.device)
    if ws is None:
        ws = alloc_workspace(cfg, S_k.device)
    prefill_project(cfg, n, X_k, X_v, bases_k, bases_v, coef_k, coef_v, ws)
    return {"sink_k": sink_k, "sink_v": sink_v, "bases_k": bases_k, "bases_v": bases_v, "coef_k": coef_k,
            "coef_v": coef_v}


def full_recon_decode(cfg, length, q, sink_k, sink_v, bases_k, bases_v, coef_k, coef_v, ws, out=None):
    """Comparator (Appendix B.1): attention over the sinks and every one of
    the `length` tokens reconstructed from the coefficient caches."""
    dt = storage_dtype(cfg)
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    need_sink = cfg.n_sink > 0
    L.check(L.load().s4r_full_recon_decode(
        _cfgp(cfg), length, _ptr(q, "q", dt), _ptr(sink_k, "sink_k", dt, need_sink),
        _ptr(sink_v, "sink_v", dt, need_sink), _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt),
        _ptr(coef_k, "coef_k", dt), _ptr(coef_v, "coef_v", dt), _ptr(out, "out", torch.float32),
        _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))
    return out


def dense_decode(cfg, n_tokens, q, k_cache, v_cache, ws, out=None):
    """Comparator: dense GQA decode over an uncompressed bf16 KV cache
    [B, capacity, Dp] (keys stored after RoPE) for tokens 0..n_tokens-1."""
    if out is None:
        out = torch.empty((cfg.batch, cfg.n_q_heads, cfg.head_dim), dtype=torch.float32, device=q.device)
    dt = storage_dtype(cfg)
    L.check(L.load().s4r_dense_decode(_cfgp(cfg), n_tokens, _ptr(q, "q", dt), _ptr(k_cache, "k_cache", dt),
                                      _ptr(v_cache, "v_cache", dt), _ptr(out, "out", torch.float32),
                                      _ptr(ws, "ws", torch.uint8), ws.numel(), _stream()))
    return out


def _device():
    """The current device's index; None without a GPU, where no tensor argument passes its checks."""
    try:
        return torch.cuda.current_device()
    except (RuntimeError, AssertionError):
        return None


def _here(t, name, dev):
    """The tensor's device has to be the current one: the launch goes to its stream."""
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on the current device {dev}")


def _same_order(a, b, names):
    """Axes a and b of as many elements count them in the same order: they are equal, or one's are the other's with
    some of them as one."""
    if a == b:
        return
    ends = []
    for shape in (a, b):
        n, e = 1, {1}
        for x in shape:
            n *= x
            e.add(n)
        ends.append(e)
    if not (ends[0] <= ends[1] or ends[1] <= ends[0]):
        raise ValueError(f"{names} have axes {tuple(a)} and {tuple(b)}")


def _batch_first(shape, name, batch, width):
    """The rows of `width` elements in `shape` come sequence by sequence: leading axes that make up the batch, or
    rows in one axis (sequence b's before b + 1's)."""
    if shape[0] == batch:
        return
    rows = math.prod(shape) // width
    if rows == batch or batch == 1:
        return
    n = 1
    for a in shape:
        if a == 1:
            continue
        if n == 1 and a % rows == 0:
            return
        n *= a
        if n >= batch:
            break
    if n != batch:
        raise ValueError(f"{name} has shape {tuple(shape)}: the {batch} sequences of the batch were expected first")


def _heads_last(shape, name, heads, dh):
    """The last axis holds whole heads: rows of heads * dh elements, or heads of dh."""
    if not shape or shape[-1] % dh:
        raise ValueError(f"{name} has shape {tuple(shape)}: rows of {heads} heads of {dh} elements were expected")


def _rows(t, name, dtype, heads, dh, dev):
    """(address, rows, elements between rows) of a GPU tensor [..., heads, dh] or [..., heads * dh] whose last
    axes are packed to rows and whose leading axes step evenly from row to row."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    _here(t, name, dev)
    shape, width = t.shape, heads * dh
    d = len(shape)
    # the usual cases first: a packed tensor, one leading axis
    if d > 1:
        lead = d - 1 if shape[-1] == width else d - 2
        if lead == d - 1 or (shape[-1] == dh and shape[-2] == heads):
            n = t.numel()
            if n and t.is_contiguous():
                return t.data_ptr(), n // width, width
    _heads_last(shape, name, heads, dh)
    strides, n = t.stride(), 1
    while d and n < width:
        d -= 1
        if strides[d] != n and shape[d] != 1:
            raise ValueError(f"{name}: the elements of a row must be packed")
        n *= shape[d]
    if n != width:
        raise ValueError(f"{name} has shape {tuple(shape)}: rows of {width} elements were expected")
    rows, stride = 1, None
    for i in range(d - 1, -1, -1):
        if shape[i] != 1:
            if stride is None:
                stride = strides[i]
            elif strides[i] != rows * stride:
                raise ValueError(f"{name}: the rows must be evenly spaced")
            rows *= shape[i]
    if rows == 0:
        raise ValueError(f"{name} has no rows")
    return t.data_ptr(), rows, width if stride is None else stride


def _ints(t, name, n, dev):
    if t is None:
        return None
    p = _ptr(t, name, torch.int32)
    _here(t, name, dev)
    if t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} entries, expected {n}")
    return p


def _tokens(t, heads, dh):
    """The axes of a tensor's rows where they are several."""
    shape = t.shape
    d, n = len(shape), 1
    if d < 3 or (d == 3 and shape[-1] == dh):
        return None
    while d and n < heads * dh:
        d -= 1
        n *= shape[d]
    return shape[:d]


def qk_norm_rope(cfg, q, k, positions, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
    """Query heads q [..., h_q, d_h] and key heads k [..., h_kv, d_h] of the same tokens in the same order, each head
    normalised (x / sqrt(mean(x^2) + eps) * weight [d_h]; not where its weight is None) and rotated by its token's position
    (int32, one per token; rope_theta = 0: not rotated, positions may be None).  q or k may be None.  The tokens may
    be slices of a fused projection's rows; outputs (new packed tensors by default) may be the inputs themselves.
    Returns (q_out, k_out)."""
    dt, dh, dev, n = storage_dtype(cfg), cfg.head_dim, _device(), None
    args, outs, axes = [], [], None
    for name, x, o, heads in (("q", q, q_out, cfg.n_q_heads), ("k", k, k_out, cfg.n_kv_heads)):
        if x is None:
            if o is not None:
                raise ValueError(f"{name}_out without {name}")
            args += (None, 0, None, 0)
            outs.append(None)
            continue
        p, rows, stride = _rows(x, name, dt, heads, dh, dev)
        if n is not None and rows != n:
            raise ValueError(f"q has {n} tokens and k {rows}")
        n, own = rows, _tokens(x, heads, dh) if x.dim() > 3 or x.shape[-1] != dh else None
        if own is not None:
            if axes is not None:
                _same_order(axes, own, "the tokens of q and k")
            axes = own
        if o is None:
            o = x.new_empty(x.shape)
            args += (p, stride, o.data_ptr(), heads * dh)
        else:
            po, ro, so = _rows(o, name + "_out", dt, heads, dh, dev)
            if ro != n:
                raise ValueError(f"{name}_out has {ro} tokens, expected {n}")
            to = _tokens(o, heads, dh)
            if own is not None and to is not None:
                _same_order(own, to, f"the tokens of {name} and {name}_out")
            args += (p, stride, po, so)
        outs.append(o)
    if n is None:
        raise ValueError("q or k is required")
    if q_out is not None or k_out is not None:
        _apart(args, n, cfg, dt)
    pos = _ints(positions, "positions", n, dev)
    if pos is not None and axes is not None:
        _same_order(axes, positions.shape, "the tokens and positions")
    weights = []
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        weights.append(_ptr(w, name, dt, False))
        if w is not None:
            _here(w, name, dev)
            if w.numel() != dh:
                raise ValueError(f"{name} has {w.numel()} entries, expected {dh}")
    L.check(L.load().s4r_qk_norm_rope(
        _cfgp(cfg), n, args[0], args[1], args[4], args[5], weights[0], weights[1], eps,
        pos, args[2], args[3], args[6], args[7], _stream()))
    return tuple(outs)


def _apart(args, n, cfg, dt):
    """An output's rows may be its own input's, and otherwise no other rows of the call.  Rows of one fused
    buffer (equal strides) interleave without overlapping."""
    es = 2 if dt == torch.bfloat16 else 4
    dh = cfg.head_dim
    wq, wk = cfg.n_q_heads * dh * es, cfg.n_kv_heads * dh * es
    q, k = (args[0], args[1] * es, wq), (args[4], args[5] * es, wk)
    qo, ko = (args[2], args[3] * es, wq), (args[6], args[7] * es, wk)

    def overlap(a, b):
        if a[0] is None or b[0] is None:
            return False
        if a[0] + (n - 1) * a[1] + a[2] <= b[0] or b[0] + (n - 1) * b[1] + b[2] <= a[0]:
            return False
        if a[1] != b[1] or n == 1:
            return True
        off = (b[0] - a[0]) % a[1]
        return off < a[2] or off + b[2] > a[1]

    for name, o, own, others in (("q_out", qo, q, (k,)), ("k_out", ko, k, (q,))):
        if o[0] is None:
            continue
        if any(overlap(o, x) for x in others) or (o[:2] != own[:2] and overlap(o, own)):
            raise ValueError(f"{name} overlaps an input of the call that is not its own")
    if overlap(qo, ko):
        raise ValueError("q_out and k_out overlap")


class KV8Cache:
    """The tensors of an 8-bit KV cache (kv8_alloc): codes [B, h_kv, T, 64 d_h] uint8 and scales [B, h_kv, T]
    fp32 of both sides, T = ceil(capacity / 64); format "int8" or "e4m3"."""

    __slots__ = ("format", "k_codes", "k_scales", "v_codes", "v_scales")

    def __init__(self, format, k_codes, k_scales, v_codes, v_scales):
        if format not in _KV_FORMATS:
            raise ValueError(f"format {format!r}: one of {sorted(_KV_FORMATS)} was expected")
        self.format = format
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales


def kv8_size(cfg):
    """(bytes of codes, scales) of one side of the 8-bit cache."""
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    L.check(L.load().s4r_kv8_size(_cfgp(cfg), ctypes.byref(n), ctypes.byref(m)))
    return n.value, m.value


def kv8_alloc(cfg, format="int8", device="cuda"):
    """An empty 8-bit cache of cfg.capacity tokens per sequence."""
    if format not in _KV_FORMATS:
        raise ValueError(f"format {format!r}: one of {sorted(_KV_FORMATS)} was expected")
    kv8_size(cfg)                                    # the library's own checks of cfg
    if torch.device(device).type != "cuda":
        raise ValueError(f"device {device}: a GPU was expected")
    shape = (cfg.batch, cfg.n_kv_heads, (cfg.capacity + L.KV8_BLOCK - 1) // L.KV8_BLOCK)
    sides = []
    for _ in range(2):
        sides += [torch.zeros(shape + (L.KV8_BLOCK * cfg.head_dim,), dtype=torch.uint8, device=device),
                  torch.zeros(shape, dtype=torch.float32, device=device)]
    return KV8Cache(format, *sides)


def _kv8(cfg, cache, dev):
    """The C view of a cache, its tensors checked against cfg."""
    if not isinstance(cache, KV8Cache):
        raise ValueError("cache must be a KV8Cache")
    batch, heads, tiles = cfg.batch, cfg.n_kv_heads, (cfg.capacity + L.KV8_BLOCK - 1) // L.KV8_BLOCK
    scales, codes = (batch, heads, tiles), (batch, heads, tiles, L.KV8_BLOCK * cfg.head_dim)
    kc, ks, vc, vs = cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales
    view = L.KV8(_KV_FORMATS[cache.format], _ptr(kc, "k_codes", torch.uint8), _ptr(ks, "k_scales", torch.float32),
                 _ptr(vc, "v_codes", torch.uint8), _ptr(vs, "v_scales", torch.float32))
    for name, t, shape in (("k_codes", kc, codes), ("k_scales", ks, scales), ("v_codes", vc, codes),
                           ("v_scales", vs, scales)):
        if t.shape != shape:
            if t.numel() != math.prod(shape):
                raise ValueError(f"{name} has {t.numel()} elements, expected {shape}")
            _same_order(t.shape, shape, f"{name} and cfg's cache")
        if t.get_device() != dev:
            _here(t, name, dev)
    return ctypes.byref(view)


def kv8_write(cfg, cache, k, v, row0=0, starts=None, counts=None):
    """Quantise rows k, v [B, n, h_kv d_h] (or [B, n, h_kv, d_h]; evenly spaced rows; B and n may be one axis) into
    the cache as tokens starts[b] + i (int32 GPU tensor; row0 + i without it) for i < counts[b] (all without it).  A
    sequence whose range does not fit is left as it is, without an error: the program keeps its lengths below
    cfg.capacity."""
    dt, batch, heads, dh = storage_dtype(cfg), cfg.batch, cfg.n_kv_heads, cfg.head_dim
    dev = _device()
    c = _kv8(cfg, cache, dev)
    pk, rows, sk = _rows(k, "k", dt, heads, dh, dev)
    pv, rv, sv = _rows(v, "v", dt, heads, dh, dev)
    if rows != rv or rows % batch:
        raise ValueError(f"k has {rows} rows and v {rv}: a multiple of the batch {batch}, the same for both, was expected")
    if k.shape[0] != batch or v.shape[0] != batch:
        _batch_first(k.shape, "k", batch, heads * dh)
        _batch_first(v.shape, "v", batch, heads * dh)
    L.check(L.load().s4r_kv8_write(_cfgp(cfg), c, rows // batch, row0, _ints(starts, "starts", batch, dev),
                                   _ints(counts, "counts", batch, dev), pk, sk, pv, sv, _stream()))


def kv8_read(cfg, cache, n_rows, row0=0, starts=None, counts=None, k=None, v=None):
    """The tokens starts[b] + i (row0 + i), i < n_rows, of every sequence in the storage dtype: (k, v)
    [B, n_rows, h_kv d_h].  Rows from counts[b] on are zeros."""
    dt = storage_dtype(cfg)
    dev = _device()
    c = _kv8(cfg, cache, dev)
    shape = (cfg.batch, max(n_rows, 0), cfg.n_kv_heads * cfg.head_dim)
    out = []
    for name, t in (("k", k), ("v", v)):
        if t is None:
            t = cache.k_codes.new_empty(shape, dtype=dt)
        elif t.numel() != shape[0] * shape[1] * shape[2]:
            raise ValueError(f"{name} has {t.numel()} elements, expected {shape}")
        elif t.shape != shape:
            _same_order(t.shape, shape[:2] + (cfg.n_kv_heads, cfg.head_dim), f"{name} and the rows")
        out.append(t)
    ptrs = [_ptr(t, name, dt) for t, name in zip(out, "kv")]
    for t, name in zip(out, "kv"):
        _here(t, name, dev)
    L.check(L.load().s4r_kv8_read(_cfgp(cfg), c, n_rows, row0, _ints(starts, "starts", cfg.batch, dev),
                                  _ints(counts, "counts", cfg.batch, dev), ptrs[0], ptrs[1], _stream()))
    return tuple(out)


def kv8_workspace_size(cfg, n_queries=1):
    n = ctypes.c_size_t()
    L.check(L.load().s4r_kv8_workspace_size(_cfgp(cfg), n_queries, ctypes.byref(n)))
    return n.value


def alloc_kv8_workspace(cfg, n_queries=1, device="cuda"):
    return torch.empty(kv8_workspace_size(cfg, n_queries), dtype=torch.uint8, device=device)


def kv8_decode(cfg, cache, n_tokens, q, ws, lengths=None, out=None):
    """Attention of the newest query tokens q [B, h_q, d_h] or [B, n, h_q, d_h] (rotated as the cached keys are)
    over the 8-bit cache: tokens 0 .. n_tokens - 1 of every sequence, or of lengths[b] (int32 GPU tensor, at most
    n_tokens are used).  Query token i of n sees all but the newest n - 1 - i tokens.  ws: alloc_kv8_workspace.
    Returns fp32 of q's shape."""
    dt = storage_dtype(cfg)
    dev = _device()
    c = _kv8(cfg, cache, dev)
    batch, hq, dh = cfg.batch, cfg.n_q_heads, cfg.head_dim
    p = _ptr(q, "q", dt)
    _here(q, "q", dev)
    shape, n = q.shape, q.numel()
    n_q, left = divmod(n, batch * hq * dh)
    if left or not n_q:
        raise ValueError(f"q has shape {tuple(shape)}: [batch, n, n_q_heads, head_dim] was expected")
    order = (batch, n_q, hq, dh)
    if shape != order and (n_q > 1 or shape != (batch, hq, dh)):
        _same_order(shape, order, "q and the query tokens")
    if out is None:
        out = q.new_empty(shape, dtype=torch.float32)
    elif out.shape != shape:
        if out.numel() != n:
            raise ValueError(f"out has {out.numel()} elements, expected {n}")
        _same_order(out.shape, order, "out and the query tokens")
    po, pw = _ptr(out, "out", torch.float32), _ptr(ws, "ws", torch.uint8)
    _here(out, "out", dev)
    _here(ws, "ws", dev)
    L.check(L.load().s4r_kv8_decode(_cfgp(cfg), c, n_tokens, _ints(lengths, "lengths", batch, dev), n_q, p, po, pw,
                                    ws.numel(), _stream()))
    return out


def project_append(cfg, row, k_new, v_new, bases_k, bases_v, coef_k, coef_v):
    dt = storage_dtype(cfg)
    L.check(L.load().s4r_project_append(_cfgp(cfg), row, _ptr(k_new, "k_new", dt), _ptr(v_new, "v_new", dt),
                                        _ptr(bases_k, "bases_k", dt), _ptr(bases_v, "bases_v", dt),
                                        _ptr(coef_k, "coef_k", dt), _ptr(coef_v, "coef_v", dt), _stream()))


def pack_coef(cfg, n_rows, src, dst=None):
    dt = storage_dtype(cfg)
    if dst is None:
        dst = torch.zeros((cfg.batch, cfg.capacity, _R(cfg)), dtype=dt, device=src.device)
    L.check(L.load().s4r_pack_coef(_cfgp(cfg), n_rows, _ptr(src, "src", dt), _ptr(dst, "dst", dt), _stream()))
    return dst


def unpack_coef(cfg, n_rows, src, dst=None):
    dt = storage_dtype(cfg)
    if dst is None:
        dst = torch.empty((cfg.batch, n_rows, _R(cfg)), dtype=dt, device=src.device)
    L.check(L.load().s4r_unpack_coef(_cfgp(cfg), n_rows, _ptr(src, "src", dt), _ptr(dst, "dst", dt), _stream()))
    return dst


TIMED_KERNELS = ("prepare", "score_stream", "relevance", "select", "attn_split", "attn_combine")


def timing_enable(max_steps):
    L.check(L.load().s4r_timing_enable(max_steps))


def timing_read():
    """-> ({kernel name: summed ms}, timed steps)"""
    ms = (ctypes.c_double * len(TIMED_KERNELS))()
    n = ctypes.c_int64()
    L.check(L.load().s4r_timing_read(ms, ctypes.byref(n)))
    return dict(zip(TIMED_KERNELS, list(ms))), n.value


def read_bandwidth(buf, sink=None):
    """One read pass over the bytes of GPU tensor `buf` (roofline reference).
    Returns the per-thread XOR sink (uint32 viewed as int32)."""
    lib = L.load()
    if sink is None:
        sink = torch.empty(lib.s4r_read_bandwidth_sink_len(), dtype=torch.int32, device=buf.device)
    L.check(lib.s4r_read_bandwidth(_ptr(buf, "buf"), buf.numel() * buf.element_size(), _ptr(sink, "sink", torch.int32),
                                   _stream()))
    return sink
