"""Attention over a paged cache in 4 bits where one channel, the same in every key, has
far larger products than the channels that tell the keys apart.

Tolerance of an element: that of test_gpu_paged.py and what such a channel adds.  Only
eight products of a score are not zero.  They are exact, and their sum, kept in 32
bits, is off by at most eight times 2^-23 of the largest, T; the reference that the
exponential subtracts is rounded too, at most 2^-23 of 1.5 T.  So a score is off by less
than 10 * 2^-23 T (the scale is 1), a weight by e to that, and the weighted mean of the
values by twice that of the largest value: with T <= 2^11 2 * 10 * 2^-12 < 2^-7."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests import serve_ref as S
from tests.test_gpu_cache4 import put
from tests.test_gpu_paged4 import Case4
from tests.test_gpu_serve_range import KERNELS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", [32.0, 512.0])
@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_a_large_channel_beside_small_ones(n, ctx, hq, hkv, b, large):
    rng = np.random.default_rng(n + int(large))
    c = Case4(b, n, ctx, hq, hkv, 16, seed=40)
    c.q = S.bf16(rng.normal(size=c.q.shape))
    c.q[..., 8:] = 0.0
    c.q[..., 0] = large
    k = R.GRID[rng.integers(0, 8, size=c.k.shape)] * rng.choice([-1.0, 1.0], size=c.k.shape)
    k[..., 0], k[..., 1] = 4.0, 6.0 * np.sign(k[..., 1] + 0.25)     # blocks of powers 2^0: held as they are
    v = S.bf16(c.v)
    D.cache_write(c.p, c.c, put(k), put(v), ctx)
    c.k, c.v = R.held(k), R.held(v)
    assert np.array_equal(c.k[..., :32], k[..., :32])
    c.kt = S.bf16(rng.normal(size=c.kt.shape) * 3.0)
    c.kt[..., 0] = 4.0
    c.dq, c.dk = put(c.q), put(c.kt)
    c.a.scale = 1.0
    got = c.run().double().cpu().numpy()
    assert np.isfinite(got).all()
    for r in sorted({0, b - 1}):
        for h in sorted({0, hq - 1}):
            g = h // (hq // hkv)
            see = np.concatenate([np.ones((n, ctx), bool), c.see[r]], axis=1)
            keys, values = np.concatenate([c.k[r, :, g], c.kt[r, :, g]]), np.concatenate([c.v[r, :, g], c.vt[r, :, g]])
            want = S.attention(c.q[r, :, h].astype(np.float64), keys, values, see, 1.0)
            tol = (2.0 ** -8 + 2.0 ** -9 + 2.0 ** -7) * np.abs(values).max(axis=0) + 2.0 ** -8 * np.abs(want)
            assert (np.abs(got[r, :, h] - want) <= tol).all(), (r, h, np.abs(got[r, :, h] - want).max())
