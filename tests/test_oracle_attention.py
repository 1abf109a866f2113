"""The oracle of the cache and its attention against independent computations: torch's softmax in fp64, the quantiser's bounds, the mask by cases."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao


@pytest.mark.parametrize("L,window,causal", [(1, 0, True), (17, 0, True), (17, 5, True), (17, 0, False)])
def test_row_is_the_masked_softmax(L, window, causal):
    rng = np.random.default_rng(L + window)
    q, k, v = rng.normal(size=24), rng.normal(size=(L, 24)), rng.normal(size=(L, 24))
    for i in range(L):
        seen = ao.visible(L, i, causal, window)
        want = [t for t in range(L) if not causal or (t <= i and (not window or i - t < window))]
        assert list(np.flatnonzero(seen)) == want
        o, lse, a = ao.attention_row(q, k, v, seen, 0.2)
        s = torch.from_numpy(0.2 * (k @ q)).masked_fill(torch.from_numpy(~seen), -torch.inf)
        p = torch.softmax(s, 0).numpy()
        assert np.allclose(o, p @ v, rtol=1e-12, atol=1e-14) and np.isclose(lse, torch.logsumexp(s, 0).item(), rtol=1e-12)
        assert np.allclose(a, p @ np.abs(v), rtol=1e-12)


def test_a_row_that_sees_nothing():
    o, lse, _ = ao.attention_row(np.ones(4), np.ones((3, 4)), np.ones((3, 4)), ao.visible(3, -1), 1.0)
    assert not o.any() and lse == -np.inf


def test_quantiser():
    x = np.random.default_rng(0).normal(size=(64, 33)).astype(np.float32)
    x[3] = 0
    x[4] = 1e-7
    x[5, 2] = np.inf
    x[6, 1] = np.nan
    codes, step = ao.quantise(x)
    assert not codes[3].any() and (codes[4] == 1).all() and not codes[5:7].any()        # (1e-7 is 1.28 steps of 1e-5 / 128)
    assert np.isnan(step[5:7]).all() and (step[3:5] == np.float32(1e-5) / 128).all()
    good = [i for i in range(64) if i not in (5, 6)]
    y = ao.stored(x, True)
    top = np.abs(x[good]).max(1)
    # half a step of rounding; the largest positive value is held back by the top code 127, one step.  fl32(code * step) adds at most
    # 2^-24 * 128 steps, and the two roundings of x * (128 / top) move where a code begins by twice that.
    ulp = 128 * 2.0 ** -24
    assert (np.abs(y[good] - x[good]) <= np.maximum(top, 1e-5)[:, None] / 128 * (1 + ulp)).all()
    inner = np.abs(x[good]) < 127 / 128 * top[:, None]
    assert (np.abs(y[good] - x[good])[inner] <= (np.maximum(top, 1e-5)[:, None] / 128 * (0.5 + 3 * ulp) * np.ones_like(x[good]))[inner]).all()
    assert np.isnan(y[5:7]).all()


def test_bf16_is_torchs():
    x = np.concatenate([np.random.default_rng(1).normal(size=1000), [0, np.inf, -np.inf, np.nan, 3.4e38, 1e-40, 1.00390625, 1.01171875]]).astype(np.float32)
    want = torch.from_numpy(x).bfloat16().float().numpy()
    assert np.array_equal(ao.bf16(x), want, equal_nan=True)
