"""Adapted 1 x 1 convolutions on the tensor cores over the range of what they are given: filters that are zero or tiny beside their adapters,
filters and adapters' rows of very different size, long reductions, sums that lose nothing.  Formula as in test_gpu_adapters; the tolerances are the
math modes' own (gpu_util.TOL) where nothing else is said, taken for each output channel by itself where channels differ in size."""
import numpy as np
import pytest
import torch

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


SIZES = np.array([0, -24, -28, -32, -40, -60, 20, -90], np.float64)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("R", [12, 40])
def test_filters_and_rows_of_up_of_very_different_size(R, mode):
    """Every output channel has a size of its own, and in half of them the adapter's row another one than the filter: each keeps its own accuracy."""
    rng = np.random.default_rng(73 + R)
    layer, x = A.Layer(rng, 96, 160, R, 3, bias=False), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    k = np.arange(160)
    layer.w = (layer.w * 2.0 ** SIZES[k % 8][:, None]).astype(np.float32)
    layer.up = (layer.up * 2.0 ** SIZES[np.where(k % 3 < 2, k, k // 8) % 8][:, None]).astype(np.float32)
    for ids in (np.full(80, -1, np.int32), (np.arange(80) % 3).astype(np.int32)):
        assert by_channel(layer.run(x, ids, mode), layer.ref(x, ids)) <= TOL[mode]


@pytest.mark.parametrize("mode", A.MODES)
def test_ranks_of_very_different_size(mode):
    """Rows of Down far below and above one another, and columns of Up that make up for it: every rank has the same part in the result."""
    rng = np.random.default_rng(74)
    layer, x = A.Layer(rng, 96, 160, 16, 3, bias=False), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    size = 2.0 ** SIZES[np.arange(16) % 8]
    layer.down, layer.up = (layer.down * size[:, None]).astype(np.float32), (layer.up / size).astype(np.float32)
    layer.w *= 0.1
    ids = (np.arange(80) % 3).astype(np.int32)
    assert rel_err(layer.run(x, ids, mode), layer.ref(x, ids)) <= TOL[mode]


@pytest.mark.parametrize("mode", ["fp32", "3xtf32"])
def test_scales_of_adapters_far_from_one(mode):
    rng = np.random.default_rng(75)
    layer, x = A.Layer(rng, 96, 160, 16, 5, bias=False), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    layer.scale = np.array([0.0, -1e-30, 1e30, -3.0, 1e-38], np.float32)
    layer.up[1] *= 1e30
    layer.up[2] *= 1e-30
    ids = (np.arange(80) % 6 - 1).astype(np.int32)
    assert rel_err(layer.run(x, ids, mode), layer.ref(x, ids)) <= TOL[mode]


@pytest.mark.parametrize("mode", ["3xtf32", "tf32"])
def test_repeatable_on_streams_and_in_a_graph(mode):
    """The tensor-core form: two calls at once with workspaces of their own, then a captured one whose adapters and inputs change between replays."""
    rng = np.random.default_rng(77)
    N, H, W = 80, 12, 11
    layer, x = A.Layer(rng, 200, 300, 20, 5), rng.standard_normal((N, 200, H, W)).astype(np.float32)
    on_tensor_cores(layer, N, H, W)
    ids = rng.integers(-1, 5, N).astype(np.int32)
    first = layer.run(x, ids, mode)
    assert np.array_equal(layer.run(x, ids, mode), first)
    blk, idt = to_blk(x), dev(ids)
    outs, wss = [new_blk(N, 300, H, W) for _ in range(2)], [layer.workspace(N, H, W) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o, ws in zip(streams, outs, wss):
            with torch.cuda.stream(s):
                layer.call(blk, idt, o, ws, N, H, W, B.MATH[mode])
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(from_blk(o, N, 300, H, W), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.call(blk, idt, outs[0], wss[0], N, H, W, B.MATH[mode])
    for i in range(3):
        y, other = (x * (i + 1)).astype(np.float32), rng.integers(-1, 5, N).astype(np.int32)
        blk.copy_(to_blk(y))
        idt.copy_(dev(other))
        graph.replay()
        assert rel_err(from_blk(outs[0], N, 300, H, W), layer.ref(y, other)) <= TOL[mode]
    assert B.small_device_status(ctx()) == B.OK


@pytest.mark.parametrize("mode", ["3xtf32", "tf32"])
@pytest.mark.parametrize("N,C,K,H,W,R", [(80, 33, 290, 8, 8, 9), (9, 70, 1111, 21, 19, 128), (80, 130, 257, 8, 9, 33), (300, 64, 32, 8, 8, 100), (3, 500, 800, 56, 55, 17)])
def test_every_edge_of_a_tile(N, C, K, H, W, R, mode):
    """Pixels that end inside a warp's 32, filters that end inside a block and inside a tile, the previous output added, with and without ReLU."""
    rng = np.random.default_rng(78)
    layer, x = A.Layer(rng, C, K, R, 3), rng.standard_normal((N, C, H, W)).astype(np.float32)
    on_tensor_cores(layer, N, H, W)
    ids = (np.arange(N) % 4 - 1).astype(np.int32)
    before = rng.standard_normal((N, K, H, W)).astype(np.float32)
    plain = layer.ref(x, ids)
    assert by_channel(layer.run(x, ids, mode), plain) <= TOL[mode]
    assert rel_err(layer.run(x, ids, mode, before=before), plain + before) <= TOL[mode]
    assert rel_err(layer.run(x, ids, mode, relu=True, before=before), np.maximum(plain + before, 0)) <= TOL[mode]


@pytest.mark.parametrize("mode", ["3xtf32", "tf32"])
def test_values_that_are_not_finite_stay_with_their_pixel(mode):
    rng = np.random.default_rng(79)
    layer, x = A.Layer(rng, 96, 160, 16, 4), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    ids = (np.arange(80) % 5 - 1).astype(np.int32)
    ref = layer.ref(x, ids)
    x[7, 50, 3, 4], x[11, 0, 8, 9], x[20, 95, 0, 0] = np.nan, np.inf, -np.inf
    layer.up[3, 10, 5] = np.nan                                 # filter 10 of the images that use adapter 3
    got = layer.run(x, ids, mode)
    for n, p in ((7, (3, 4)), (11, (8, 9)), (20, (0, 0))):
        assert not np.isfinite(got[(n, slice(None)) + p]).any()
        got[(n, slice(None)) + p] = ref[(n, slice(None)) + p]
    assert np.isnan(got[ids == 3, 10]).all()
    got[ids == 3, 10] = ref[ids == 3, 10]
    assert rel_err(got, ref) <= TOL[mode]


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("w_size", [1.0, 2.0 ** 70, 2.0 ** -70])
def test_pixels_at_the_ends_of_the_range(w_size, mode):
    """Pixels from 1e-33 to 1e35, beside filters that bring the results back in, or not so far out: each pixel keeps its own accuracy."""
    rng = np.random.default_rng(80)
    layer, x = A.Layer(rng, 96, 160, 12, 3, bias=False), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    on_tensor_cores(layer, 80, 9, 10)
    sizes = np.array([1e-33, 1e-20, 1.0, 1e12] + [1e16 if w_size > 1 else 1e35])
    size = sizes[np.arange(90) % 5].reshape(9, 10)
    x = (x * size).astype(np.float32)
    layer.w, layer.up = (layer.w * w_size).astype(np.float32), (layer.up * w_size).astype(np.float32)
    ids = (np.arange(80) % 4 - 1).astype(np.int32)
    seen = size * w_size > 1e-30                                # below it, TF32 pairs and FP32's own products lose bits to the smallest numbers
    got, ref = layer.run(x, ids, mode)[:, :, seen] / (size * w_size)[seen], layer.ref(x, ids)[:, :, seen] / (size * w_size)[seen]
    assert rel_err(got, ref) <= TOL[mode]
