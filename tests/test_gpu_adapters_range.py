"""Adapted 1 x 1 convolutions on the tensor cores over the range of what they are given: filters that are zero or tiny beside their adapters,
filters and adapters' rows of very different size, long reductions, sums that lose nothing.  Formula as in test_gpu_adapters; the tolerances are the
math modes' own (gpu_util.TOL) where nothing else is said, taken for each output channel by itself where channels differ in size."""
import numpy as np
import pytest

import test_gpu_adapters as A
from gpu_util import B, TOL, ctx, dev, from_blk, new_blk, rel_err, to_blk

pytestmark = pytest.mark.gpu


def on_tensor_cores(layer, N, H, W):
    assert B.small_adapted_conv2d_workspace_bytes(N, layer.C, layer.K, H, W, layer.R) > 0


def by_channel(got, ref):
    """The largest of the channels' errors: each output channel (N, pixels) measured against its own size."""
    return max(rel_err(got[:, k], ref[:, k]) for k in range(ref.shape[1]))


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("exponent", [None, -115, -100])
def test_adapters_beside_filters_of_next_to_nothing(exponent, mode):
    """A projection that starts at zero, or far below its adapters: their part, some hundreds here, is the result."""
    rng = np.random.default_rng(71)
    layer, x = A.Layer(rng, 96, 160, 16, 3), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    layer.w *= np.float32(0 if exponent is None else 2.0 ** exponent)
    layer.up *= 100
    on_tensor_cores(layer, 80, 9, 10)
    ids = (np.arange(80) % 4 - 1).astype(np.int32)
    got, ref = layer.run(x, ids, mode), layer.ref(x, ids)
    assert np.isfinite(got).all() and rel_err(got, ref) <= TOL[mode]
    none = np.full(80, -1, np.int32)
    layer.b[:] = 0
    assert rel_err(layer.run(x, none, mode) * 2.0 ** 100, layer.ref(x, none) * 2.0 ** 100) <= TOL[mode]


@pytest.mark.parametrize("fill", [1e20, float("inf"), float("nan")])
def test_pad_lanes_that_hold_anything_have_no_part(fill):
    rng = np.random.default_rng(76)
    layer, x = A.Layer(rng, 72, 160, 16, 3), rng.standard_normal((80, 72, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    ids = (np.arange(80) % 4 - 1).astype(np.int32)
    layer.pack("3xtf32")
    blk, out = to_blk(x), new_blk(80, 160, 9, 10)
    blk.view(80, 3, 90, 32)[:, 2, :, 8:] = fill
    layer.call(blk, dev(ids), out, layer.workspace(80, 9, 10), 80, 9, 10, B.MATH_3XTF32)
    assert rel_err(from_blk(out, 80, 160, 9, 10), layer.ref(x, ids)) <= TOL["3xtf32"]
    assert B.small_device_status(ctx()) == B.OK


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("C", [512, 2048, 8192])
def test_sums_that_lose_nothing_are_exact(C, mode):
    """Ones times ones, and small integers picked out one by one: every product and every sum is a number of few bits."""
    rng = np.random.default_rng(72)
    layer = A.Layer(rng, C, 64, 16, 1, bias=False, scale=False)
    layer.w[:], ids = 1, np.full(80, -1, np.int32)
    on_tensor_cores(layer, 80, 8, 8)
    assert np.array_equal(layer.run(np.ones((80, C, 8, 8), np.float32), ids, mode), np.full((80, 64, 8, 8), C, np.float32))
    layer.w[:] = 0
    pick = rng.permutation(C)[:64]
    layer.w[np.arange(64), pick] = 1
    x = rng.integers(-500, 501, (80, C, 8, 8)).astype(np.float32)
    assert np.array_equal(layer.run(x, ids, mode), x[:, pick])
    # the adapter alone: x -> sums over the channels, one for each rank -> the filters that pick a rank
    layer.w[:], layer.down[:], layer.up[:] = 0, 1, 0
    layer.up[0, np.arange(64), np.arange(64) % 16] = 1
    assert np.array_equal(layer.run(np.ones((80, C, 8, 8), np.float32), np.zeros(80, np.int32), mode), np.full((80, 64, 8, 8), C, np.float32))


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("C,K,R", [(1000, 96, 20), (2048, 64, 16), (8192, 40, 9), (8192, 33, 128)])
def test_long_reductions(C, K, R, mode):
    rng = np.random.default_rng(C + K)
    layer, x = A.Layer(rng, C, K, R, 3), rng.standard_normal((80, C, 8, 8)).astype(np.float32)
    ids = (np.arange(80) % 4 - 1).astype(np.int32)
    on_tensor_cores(layer, 80, 8, 8)
    # inputs and filters with a mean of their own, so that the sums grow with the number of terms, as the running sums then do
    for x_, w in ((x, layer.w), (np.abs(x), np.abs(layer.w))):
        layer.w, layer.down = w, np.abs(layer.down) if w is not layer.w else layer.down
        got, ref = layer.run(x_, ids, mode), layer.ref(x_, ids)
        assert rel_err(got, ref) <= TOL[mode]
    layer.w, layer.b[:] = np.zeros_like(layer.w), 0                 # the adapters' products by themselves
    some = ids >= 0
    assert rel_err(layer.run(x, ids, mode)[some], layer.ref(x, ids)[some]) <= TOL[mode]
