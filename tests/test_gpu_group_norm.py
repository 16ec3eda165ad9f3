"""Group normalisation with an activation against its formula in 64 bits.

Tolerance: FP32's (gpu_util.TOL).  A mean of n values is off by a few roundings of 2^-24 (sums are trees of short runs), and that
is an error of |mean| / spread such roundings in the result: far below 1e-5 for the activations here, added where a test's mean is large."""
import numpy as np
import pytest
import torch

import attention_ref as R
from gpu_util import B, TOL, ctx, dev, from_blk, new_blk, pad_lanes_are_zero, rel_err, to_blk

pytestmark = pytest.mark.gpu
FLAGS = {"none": 0, "relu": B.RELU, "silu": B.SILU}


def run(x, gamma, beta, groups, eps=1e-5, act="none", in_place=False, blk=None):
    N, C, H, W = x.shape
    blk = to_blk(x) if blk is None else blk
    out = blk if in_place else new_blk(N, C, H, W)
    need = B.small_group_norm_workspace_bytes(N, C, H, W, groups)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    g, b = (None if t is None else dev(t) for t in (gamma, beta))
    B.small_group_norm(ctx(), blk, g, b, out, ws, N, C, H, W, groups, eps, FLAGS[act])
    assert pad_lanes_are_zero(out, N, C, H, W)
    return from_blk(out, N, C, H, W)


def make(rng, N, C, H, W, mean=0.7, spread=1.0):
    x = rng.standard_normal((N, C, H, W)) * (0.3 + spread * rng.random((1, C, 1, 1))) + mean * rng.standard_normal((1, C, 1, 1))
    return x.astype(np.float32), (1 + 0.2 * rng.standard_normal(C)).astype(np.float32), (0.2 * rng.standard_normal(C)).astype(np.float32)


@pytest.mark.parametrize("shape", [
    (1, 1, 1, 1, 1), (1, 64, 25, 5, 8), (3, 32, 1, 1, 4), (2, 40, 1, 3, 5), (2, 33, 7, 7, 33), (2, 33, 7, 7, 1), (1, 31, 5, 9, 31),
    (2, 72, 13, 29, 6), (2, 96, 9, 11, 32), (2, 320, 6, 5, 32), (1, 256, 56, 56, 32), (2, 64, 56, 56, 1), (1, 62, 17, 3, 2),
    (1, 1024, 3, 2, 1), (300, 16, 4, 4, 2), (1, 32, 96, 96, 4), (1, 8, 97, 115, 8), (1, 48, 130, 129, 3), (2, 32, 150, 120, 32), (1, 256, 64, 64, 1)])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_matches_the_formula(shape, act):
    N, C, H, W, groups = shape
    rng = np.random.default_rng(C * 1000 + H * 10 + N)
    x, gamma, beta = make(rng, N, C, H, W)
    # a group of one value has no spread: what is left is beta, exactly 0 / sqrt(eps)
    assert rel_err(run(x, gamma, beta, groups, act=act), R.group_norm(x, gamma, beta, groups, 1e-5, act)) <= TOL["fp32"]


def test_both_forms_are_reached():
    assert B.small_group_norm_workspace_bytes(1, 256, 56, 56, 32) == 0 and B.small_group_norm_workspace_bytes(1, 32, 96, 96, 4) == 0
    assert B.small_group_norm_workspace_bytes(1, 48, 130, 129, 3) > 0 and B.small_group_norm_workspace_bytes(1, 256, 64, 64, 1) > 0


@pytest.mark.parametrize("H", [9, 150])
def test_without_affine_and_in_place(H):
    rng = np.random.default_rng(3)
    x, gamma, beta = make(rng, 2, 40, H, 140)
    ref = R.group_norm(x, None, None, 4, 1e-3, "silu")
    assert rel_err(run(x, None, None, 4, eps=1e-3, act="silu", in_place=True), ref) <= TOL["fp32"]
    assert rel_err(run(x, gamma, None, 4), R.group_norm(x, gamma, None, 4, 1e-5, "none")) <= TOL["fp32"]
    assert rel_err(run(x, None, beta, 4), R.group_norm(x, None, beta, 4, 1e-5, "none")) <= TOL["fp32"]


@pytest.mark.parametrize("H", [12, 150])
def test_a_mean_far_from_zero(H):
    rng = np.random.default_rng(4)
    x = (1000.0 + rng.standard_normal((2, 32, H, 130))).astype(np.float32)
    # the mean of a group is off by at most 16 roundings (runs of 16 to 64 values joined by trees, their errors of either sign): 1000 * 16 * 2^-24
    assert rel_err(run(x, None, None, 2), R.group_norm(x, None, None, 2, 1e-5, "none")) <= TOL["fp32"] + 1000 * 16 * 2.0 ** -24 / 8


def test_constant_groups_and_eps_zero():
    x = np.full((2, 16, 5, 5), 3.0, np.float32)
    x[1] = np.random.default_rng(5).standard_normal((16, 5, 5))
    beta = np.arange(16, dtype=np.float32)
    got = run(x, None, beta, 4, eps=1e-5)
    assert np.array_equal(got[0], np.broadcast_to(beta[:, None, None], (16, 5, 5)))
    assert rel_err(run(x, None, beta, 4, eps=0.0)[1], R.group_norm(x, None, beta, 4, 0.0, "none")[1]) <= TOL["fp32"]


@pytest.mark.parametrize("H", [10, 150])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_stays_in_its_group(H, bad):
    rng = np.random.default_rng(6)
    x, gamma, beta = make(rng, 2, 48, H, 120)
    y = x.copy()
    y[1, 20, H // 2, 7] = bad                                   # group 1 of image 1: channels 16 to 31
    got, ref = run(y, gamma, beta, 3), R.group_norm(x, gamma, beta, 3, 1e-5, "none")
    assert np.isnan(got[1, 16:32]).all()
    got[1, 16:32] = ref[1, 16:32]
    assert rel_err(got, ref) <= TOL["fp32"]


def test_silu_far_out():
    x = np.linspace(-1, 1, 64, dtype=np.float32).reshape(1, 1, 8, 8)
    for size in (30.0, 300.0):
        gamma = np.array([size], np.float32)
        ref = R.group_norm(x, gamma, None, 1, 1e-5, "silu")
        assert rel_err(run(x, gamma, None, 1, act="silu"), ref) <= TOL["fp32"]


def test_whatever_lies_in_pad_lanes_has_no_part():
    rng = np.random.default_rng(7)
    x, gamma, beta = make(rng, 2, 40, 6, 6)
    blk = to_blk(x)
    blk.view(2, 2, 36, 32)[:, 1, :, 8:] = float("nan")
    assert rel_err(run(x, gamma, beta, 4, blk=blk), R.group_norm(x, gamma, beta, 4, 1e-5, "none")) <= TOL["fp32"]


@pytest.mark.parametrize("shape", [(4, 64, 14, 14, 8), (1, 64, 140, 130, 8)])
def test_repeatable_on_streams_and_in_a_graph(shape):
    N, C, H, W, groups = shape
    rng = np.random.default_rng(8)
    x, gamma, beta = make(rng, N, C, H, W)
    first = run(x, gamma, beta, groups)
    blk, out, g, b = to_blk(x), new_blk(N, C, H, W), dev(gamma), dev(beta)
    ws = torch.empty(max(16, B.small_group_norm_workspace_bytes(N, C, H, W, groups)), dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.small_group_norm(ctx(), blk, g, b, out, ws, N, C, H, W, groups)
    torch.cuda.synchronize()
    assert np.array_equal(from_blk(out, N, C, H, W), first)
    with torch.cuda.graph(graph):
        B.small_group_norm(ctx(), blk, g, b, out, ws, N, C, H, W, groups)
    out.fill_(0)
    for _ in range(3):
        graph.replay()
    assert np.array_equal(from_blk(out, N, C, H, W), first)


@pytest.mark.parametrize("shape", [(1, 4096, 16, 16, 1), (1, 8192, 12, 12, 1), (2, 4128, 16, 17, 32), (1, 6144, 9, 9, 1)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_units_of_thousands_of_channels(shape, act):
    """The second form's second kernel: means, scales and shifts of a unit's channels take more than the 48 KB a kernel has unasked."""
    N, C, H, W, groups = shape
    rng = np.random.default_rng(C + H)
    x, gamma, beta = make(rng, N, C, H, W)
    assert B.small_group_norm_workspace_bytes(*shape) > 0
    assert rel_err(run(x, gamma, beta, groups, act=act), R.group_norm(x, gamma, beta, groups, 1e-5, act)) <= TOL["fp32"]


@pytest.mark.parametrize("shape", [(1, 9984, 10, 11, 1), (1, 11520, 7, 9, 1), (2, 10240, 3, 3, 1)])
def test_the_largest_units(shape):
    """Two or more pixels of these are too many for a block, one is not."""
    N, C, H, W, groups = shape
    rng = np.random.default_rng(C + H)
    x, gamma, beta = make(rng, N, C, H, W)
    assert rel_err(run(x, gamma, beta, groups), R.group_norm(x, gamma, beta, groups, 1e-5, "none")) <= TOL["fp32"]


@pytest.mark.parametrize("H", [10, 150])
def test_a_group_without_spread_far_from_zero(H):
    """2^70 everywhere in one group: its sums are exact, their squares are beyond FP32's range and have no part."""
    rng = np.random.default_rng(11)
    x, gamma, beta = make(rng, 2, 48, H, 120)
    x[1, 16:32] = np.float32(2.0 ** 70)
    got = run(x, gamma, beta, 3)
    assert np.array_equal(got[1, 16:32], np.broadcast_to(beta[16:32, None, None], (16, H, 120)))


@pytest.mark.parametrize("H", [10, 150])
def test_a_variance_beyond_the_range(H):
    """Values whose squares are more than FP32 holds: an infinite variance, and what the formula makes of one."""
    rng = np.random.default_rng(9)
    x, gamma, beta = make(rng, 2, 48, H, 120)
    y = x.copy()
    y[1, 16:32] *= 1e25                                         # group 1 of image 1
    got, ref = run(y, gamma, beta, 3), R.group_norm(x, gamma, beta, 3, 1e-5, "none")
    assert np.array_equal(got[1, 16:32], np.broadcast_to(beta[16:32, None, None], (16, H, 120)))
    got[1, 16:32] = ref[1, 16:32]
    assert rel_err(got, ref) <= TOL["fp32"]


@pytest.mark.parametrize("H", [10, 150])
def test_a_value_that_is_not_finite_before_an_activation(H):
    rng = np.random.default_rng(10)
    x, gamma, beta = make(rng, 1, 48, H, 120)
    ref = {act: R.group_norm(x, gamma, beta, 3, 1e-5, act) for act in ("relu", "silu")}
    x[0, 20, H // 2, 7] = np.nan                                # group 1
    for act, left in (("relu", 0.0), ("silu", np.nan)):         # max(NaN, 0) is 0 in every layer of the library
        got = run(x, gamma, beta, 3, act=act)
        assert np.array_equal(got[0, 16:32], np.full((16, H, 120), left, np.float32), equal_nan=True)
        got[0, 16:32] = ref[act][0, 16:32]
        assert rel_err(got, ref[act]) <= TOL["fp32"]
