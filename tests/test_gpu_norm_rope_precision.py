"""The rotation of fp32 heads against 64 bits: sine and cosine to fp32's rounding of their own size."""

import numpy as np
import pytest
import torch

import paper_2608_00528_amd as s4r
from tests import kv8_reference as R
from tests.test_gpu_norm_rope import cfg, dev, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("theta", [1.0, 1e4, 5e5])
def test_sine_and_cosine_of_fp32_heads(theta, dh):
    """A head of ones and zeros leaves the cosine and the sine themselves.  Positions next to multiples of a quarter
    turn (355 radians are 113 half turns less 3e-5), of both signs, and any.  Relative error: the fraction's two
    roundings 2u (u = 2^-24), the series 2u, a cosine's half of them again where it is 0.71: below 5u; and the
    frequency's own error, 2^-52 of a revolution per position, in absolute terms."""
    c = cfg(2, 2, dh, theta, "fp32")
    rng = np.random.default_rng(dh)
    pos = np.concatenate([[0, 1, -1, 3, 11, 22, 33, 44, 333, 355, -355, 710, 52174, 103993, -104348, 131071],
                          rng.integers(-131072, 131072, 200)])
    x = np.zeros((len(pos), 2, dh))
    x[:, 0, :dh // 2] = 1                          # (cos, sin)
    x[:, 1, dh // 2:] = 1                          # (-sin, cos)
    want = R.norm_rope(x, None, 0, pos, float(np.float32(theta)))
    for got in s4r.qk_norm_rope(c, dev(x, c), dev(x, c), ints(pos)):
        err = np.abs(got.double().cpu().numpy() - want)
        tol = 5 * 2.0 ** -24 * np.abs(want) + 2 * np.pi * 2.0 ** -52 * np.abs(pos)[:, None, None]
        assert np.all(err <= tol), f"worst {(err / np.maximum(tol, 1e-300)).max():.3g} of the bound"


def test_fp32_pairs_far_out():
    """Positions up to 2^26, where the frequency's error reaches a rounding of the pair's size."""
    dh = 128
    c = cfg(4, 4, dh, 5e5, "fp32")
    rng = np.random.default_rng(1)
    pos = rng.integers(-2 ** 26, 2 ** 26, 300)
    x = R.round_to(rng.standard_normal((len(pos), 4, dh)), "fp32")
    got, _ = s4r.qk_norm_rope(c, dev(x, c), None, ints(pos))
    want = R.norm_rope(x, None, 0, pos, 5e5)
    pair = np.tile(np.hypot(x[..., :dh // 2], x[..., dh // 2:]), 2)
    # cosine and sine 5u each, of which a pair's element takes at most sqrt(2); two products and a sum 3u
    tol = pair * ((5 * 2 ** 0.5 + 3) * 2.0 ** -24 + 2 * np.pi * 2.0 ** -52 * np.abs(pos)[:, None, None])
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= tol), f"worst {(err / tol).max():.3g} of the bound"
