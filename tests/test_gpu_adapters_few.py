"""Adapted 1 x 1 convolutions of few pixels, which are one launch in FP32 whatever the mode: pixels that fill no whole block of eight, images that
share one, ragged channels and filters, ranks up to three groups of eight.  Formula and tolerances are those of test_gpu_adapters."""
import numpy as np
import pytest
import torch

import test_gpu_adapters as A
from gpu_util import B, TOL, ctx, dev, from_blk, new_blk, rel_err, to_blk

pytestmark = pytest.mark.gpu

SHAPES = [  # N, C, K, H, W, rank, adapters
    (7, 64, 64, 1, 1, 17, 3), (1, 512, 96, 2, 3, 8, 2), (9, 33, 31, 1, 1, 24, 4), (3, 20, 70, 3, 5, 1, 2), (64, 256, 256, 1, 1, 8, 9), (1, 96, 40, 1, 2, 9, 2),
    (2, 512, 128, 7, 7, 4, 3), (20, 32, 32, 1, 1, 20, 4), (37, 5, 3, 2, 2, 2, 5), (1, 32, 1000, 1, 1, 8, 1), (3, 500, 30, 5, 5, 7, 2), (2, 64, 64, 28, 28, 16, 2)]


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_the_formula(shape, mode):
    A.test_matches_the_formula(shape, mode)


@pytest.mark.parametrize("mode", A.MODES)
def test_results_are_those_of_fp32_and_the_same_each_time(mode):
    """No mode rounds operands here; the order of the sums is fixed."""
    rng = np.random.default_rng(41)
    layer, x = A.Layer(rng, 96, 130, 8, 4), rng.standard_normal((11, 96, 2, 2)).astype(np.float32)
    ids = rng.integers(-1, 4, 11).astype(np.int32)
    got = layer.run(x, ids, mode)
    assert rel_err(got, layer.ref(x, ids)) <= TOL["fp32"]
    assert np.array_equal(got, layer.run(x, ids, mode)) and np.array_equal(got, layer.run(x, ids, "fp32"))


def test_pad_lanes_that_hold_anything_have_no_part():
    rng = np.random.default_rng(42)
    layer, x = A.Layer(rng, 40, 50, 8, 2), rng.standard_normal((5, 40, 3, 1)).astype(np.float32)
    ids = np.array([0, -1, 1, 7, 0], np.int32)
    layer.pack("3xtf32")
    blk, out = to_blk(x), new_blk(5, 50, 3, 1)
    blk.view(5, 2, 3, 32)[:, 1, :, 8:] = float("nan")
    layer.call(blk, dev(ids), out, None, 5, 3, 1, B.MATH_3XTF32)
    assert rel_err(from_blk(out, 5, 50, 3, 1), layer.ref(x, ids)) <= TOL["fp32"]


def test_on_streams_and_in_a_graph():
    rng = np.random.default_rng(43)
    layer, x = A.Layer(rng, 64, 96, 8, 3), rng.standard_normal((6, 64, 2, 3)).astype(np.float32)
    ids = rng.integers(-1, 3, 6).astype(np.int32)
    first = layer.run(x, ids, "3xtf32")
    blk, idt, outs = to_blk(x), dev(ids), [new_blk(6, 96, 2, 3) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                layer.call(blk, idt, o, None, 6, 2, 3, B.MATH_3XTF32)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer.call(blk, idt, outs[2], None, 6, 2, 3, B.MATH_3XTF32)
    idt.fill_(-1)                                               # read when the work runs
    graph.replay()
    for o in outs[:2]:
        assert np.array_equal(from_blk(o, 6, 96, 2, 3), first)
    assert rel_err(from_blk(outs[2], 6, 96, 2, 3), layer.ref(x, np.full(6, -1, np.int32))) <= TOL["fp32"]
    assert B.small_device_status(ctx()) == B.OK
