"""Attention over the pixels of a plane against its formula in 64 bits, in every math mode.

Tolerances: the modes' own (gpu_util.TOL).  FP32 and 3xTF32: a score of size s is off by some 1e-7 s (a sum of at most 128 products), its
exponential by that much relatively, and the weighted sum averages over the keys: below 2e-6 for the scores here (|s| < 10).  TF32: operands
are off by at most 2^-12 each, so a score of unit size by 3e-4 and the result by 5e-4 at the most seen by a single key."""
import numpy as np
import pytest
import torch

import attention_ref as R
from gpu_util import B, TOL, ctx, dev, from_blk, new_blk, pad_lanes_are_zero, rel_err, to_blk

pytestmark = pytest.mark.gpu
MODES = ["fp32", "3xtf32", "tf32"]


def workspace(N, heads, kv, D, qp, kp, mode):
    return torch.empty(max(16, B.small_attention_workspace_bytes(N, heads, kv, D, qp, kp, B.MATH[mode])), dtype=torch.uint8, device="cuda")


def run(q, k, v, heads, kv, mode, scale=None, cap=0.0, bias=None, qe=None, ke=None):
    N, C, QH, QW = q.shape
    KH, KW = k.shape[2:]
    D = C // heads
    out = new_blk(N, C, QH, QW)
    ws = workspace(N, heads, kv, D, (QH, QW), (KH, KW), mode)
    up = lambda t: None if t is None else dev(t)          # noqa: E731
    B.small_attention(ctx(), to_blk(q), to_blk(k), to_blk(v), out, ws, ws.numel(), N, heads, kv, D, (QH, QW), (KH, KW), scale, cap, up(bias), up(qe), up(ke),
                      flags=B.MATH[mode])
    assert pad_lanes_are_zero(out, N, C, QH, QW)
    got = from_blk(out, N, C, QH, QW)
    assert B.small_device_status(ctx()) == B.OK
    return got


def make(rng, N, heads, kv, D, qp, kp, size=1.0):
    f = lambda c, p: (size * rng.standard_normal((N, c, *p))).astype(np.float32)       # noqa: E731
    return f(heads * D, qp), f(kv * D, kp), (f(kv * D, kp) + 0.5).astype(np.float32)


def table(rng, heads, qp, kp):
    return (0.7 * rng.standard_normal((heads, qp[0] + kp[0] - 1, qp[1] + kp[1] - 1))).astype(np.float32)


def close(got, ref, mode):
    assert np.isfinite(got).all()
    assert rel_err(got, ref) <= TOL[mode]


SHAPES = [  # N, heads, kv heads, D, query plane, key plane
    (1, 1, 1, 1, (1, 1), (1, 1)), (2, 2, 1, 8, (1, 1), (1, 1)), (2, 3, 3, 32, (5, 3), (5, 3)), (2, 4, 2, 64, (7, 7), (7, 7)), (1, 2, 2, 32, (14, 14), (14, 14)),
    (1, 4, 2, 40, (25, 13), (25, 13)), (1, 2, 2, 64, (28, 28), (28, 28)), (2, 2, 1, 128, (12, 11), (12, 11)), (1, 3, 1, 96, (9, 16), (9, 16)), (1, 1, 1, 5, (11, 12), (11, 12)),
    (1, 2, 2, 33, (13, 13), (13, 13)), (1, 1, 1, 64, (16, 16), (8, 16)), (1, 1, 1, 64, (1, 128), (1, 129)), (1, 1, 1, 32, (127, 1), (128, 1)), (1, 2, 1, 64, (16, 17), (3, 1)),
    (2, 8, 8, 64, (1, 1), (7, 7)), (3, 8, 2, 64, (1, 1), (31, 33)), (1, 6, 2, 48, (1, 3), (20, 21)), (1, 16, 1, 32, (1, 1), (40, 41)), (1, 1, 1, 128, (2, 1), (96, 96)),
    (1, 1, 1, 64, (3, 1), (1, 1)), (1, 5, 5, 20, (1, 1), (9, 9)), (1, 1, 1, 7, (1, 1), (33, 3)), (1, 2, 2, 64, (50, 41), (50, 41)), (1, 1, 1, 128, (1, 300), (2, 150)),
    (25, 8, 4, 48, (7, 7), (7, 7)), (2, 2, 2, 64, (1, 16), (12, 12)), (2, 2, 2, 64, (1, 17), (12, 12)), (1, 4, 1, 128, (4, 4), (8, 8)), (1, 40, 8, 32, (2, 3), (10, 10))]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_the_formula(shape, mode):
    N, heads, kv, D, qp, kp = shape
    rng = np.random.default_rng(D * 100 + qp[0] + kp[1])
    q, k, v = make(rng, N, heads, kv, D, qp, kp)
    close(run(q, k, v, heads, kv, mode), R.attention(q, k, v, heads, kv, D ** -0.5), mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_bias_cap_and_padded_images(shape, cap, mode):
    N, heads, kv, D, qp, kp = shape
    N += 2
    rng = np.random.default_rng(D * 100 + qp[1] + kp[0] + 1)
    q, k, v = make(rng, N, heads, kv, D, qp, kp)
    bias = table(rng, heads, qp, kp)
    ke = np.stack([rng.integers(0, kp[0] + 1, N), rng.integers(0, kp[1] + 1, N)], 1).astype(np.int32)
    qe = np.stack([rng.integers(0, qp[0] + 1, N), rng.integers(0, qp[1] + 1, N)], 1).astype(np.int32)
    ke[0], qe[0] = kp, (qp[0] + 3, 1 << 30)                     # whole planes; more than the plane counts as the plane
    qe[1] = (-5, qp[1])                                         # and less than none as none
    args = dict(scale=1.3 * D ** -0.5, cap=cap, bias=bias)
    close(run(q, k, v, heads, kv, mode, qe=qe, ke=ke, **args), R.attention(q, k, v, heads, kv, q_extents=qe, k_extents=ke, **args), mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("qp", [(1, 1), (12, 13)])
def test_what_lies_outside_the_extents_has_no_part(qp, mode):
    rng = np.random.default_rng(11)
    kp = (12, 13)
    q, k, v = make(rng, 4, 2, 1, 64, qp, kp)
    ke = np.array([[12, 13], [5, 13], [12, 3], [0, 13]], np.int32)
    qe = ke if qp == kp else None
    ref = R.attention(q, k, v, 2, 1, 0.125, k_extents=ke, q_extents=qe)
    for fill in (np.nan, np.inf, -np.inf, 3e38):
        a, b, c = q.copy(), k.copy(), v.copy()
        for n in range(4):
            for t in (b, c) + ((a,) if qp == kp else ()):
                t[n, :, ke[n, 0]:], t[n, :, :, ke[n, 1]:] = fill, fill
        got = run(a, b, c, 2, 1, mode, ke=ke, qe=qe)
        close(got, ref, mode)
        assert (got[3] == 0).all()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("plane", [(4, 5), (17, 16)])
def test_infinite_and_lowest_values_in_the_table(plane, mode):
    rng = np.random.default_rng(12)
    q, k, v = make(rng, 2, 2, 2, 32, plane, plane)
    low = float(np.finfo(np.float32).min)
    bias = table(rng, 2, plane, plane)
    bias[:, plane[0]:] = -np.inf                                # keys above the query are out of reach (a mask as a table of displacements)
    close(run(q, k, v, 2, 2, mode, bias=bias), R.attention(q, k, v, 2, 2, 32 ** -0.5, bias=bias), mode)
    bias[:, plane[0]:] = low
    close(run(q, k, v, 2, 2, mode, bias=bias), R.attention(q, k, v, 2, 2, 32 ** -0.5, bias=bias), mode)
    # nothing left: 0.  The lowest value everywhere: a number like any other, all keys weigh the same
    bias[:] = -np.inf
    assert (run(q, k, v, 2, 2, mode, bias=bias) == 0).all()
    bias[:] = low
    mean = np.broadcast_to(v.astype(np.float64).mean((2, 3), keepdims=True), v.shape)
    close(run(q, k, v, 2, 2, mode, bias=bias), mean, mode)
    # one head only; the other one as before
    bias[0] = -np.inf
    bias[1] = table(rng, 1, plane, plane)[0]
    got = run(q, k, v, 2, 2, mode, bias=bias)
    assert (got[:, :32] == 0).all()
    close(got, R.attention(q, k, v, 2, 2, 32 ** -0.5, bias=bias), mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("qp", [(1, 1), (15, 15)])
def test_values_that_are_not_finite_are_not_hidden(qp, mode):
    rng = np.random.default_rng(13)
    q, k, v = make(rng, 3, 1, 1, 32, qp, (15, 15))
    ref = R.attention(q, k, v, 1, 1, 32 ** -0.5)
    v[1, 4, 3, 3] = np.nan                                      # one channel of one image
    k[2, 0, 5, 5] = np.nan                                      # one key: every weight of the image
    got = run(q, k, v, 1, 1, mode)
    assert np.isnan(got[1, 4]).all() and np.isnan(got[2]).all()
    got[1, 4], got[2] = ref[1, 4], ref[2]
    close(got, ref, mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("qp", [(1, 1), (13, 12)])
@pytest.mark.parametrize("qs,ks,vs", [(1e4, 1e-4, 1.0), (1e-15, 1e15, 1e20), (1.0, 1.0, 1e-20), (1e-20, 1e19, 1e-30)])
def test_scales_of_the_operands(qp, qs, ks, vs, mode):
    """Magnitudes far outside half precision, values of very different size within a tile."""
    rng = np.random.default_rng(14)
    q, k, v = make(rng, 2, 2, 2, 32, qp, (13, 12))
    v[:, :, ::2] *= 1e-3
    q, k, v = (q * qs).astype(np.float32), (k * ks).astype(np.float32), (v * vs).astype(np.float32)
    scale = 1.0 / (32 ** 0.5 * qs * ks)
    close(run(q, k, v, 2, 2, mode, scale=scale) / vs, R.attention(q, k, v, 2, 2, scale) / vs, mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("qp", [(1, 1), (13, 12)])
@pytest.mark.parametrize("scale", [0.0, -0.15])
def test_scales_that_are_not_positive(qp, scale, mode):
    rng = np.random.default_rng(19)
    q, k, v = make(rng, 2, 2, 1, 40, qp, (13, 12))
    for args in (dict(), dict(bias=table(rng, 2, qp, (13, 12))), dict(cap=2.0)):
        close(run(q, k, v, 2, 1, mode, scale=scale, **args), R.attention(q, k, v, 2, 1, scale, **args), mode)


@pytest.mark.parametrize("mode", ["fp32", "3xtf32"])
def test_large_scores(mode):
    """Scores of some hundreds: nearly all weight on one key; the largest score may come last or first."""
    rng = np.random.default_rng(15)
    q, k, v = make(rng, 1, 1, 1, 64, (16, 16), (20, 20))
    for order in (1, -1):
        kk = np.ascontiguousarray((k.reshape(1, 64, -1) * np.linspace(0.1, 12, 400, dtype=np.float32)[::order]).reshape(k.shape))
        got, ref = run(q, kk, v, 1, 1, mode, scale=1.0), R.attention(q, kk, v, 1, 1, 1.0)
        # scores up to 400 are off by some 1e-7 of |q| |k| (at most 130 here... 1600 at the largest key): 2e-4 relatively in a weight
        assert rel_err(got, ref) <= 4e-4


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("qp", [(14, 14), (1, 1)])
def test_slices_of_a_stacked_tensor(qp, mode):
    """q, k and v as runs of channel blocks of one tensor, as one projection writes them."""
    rng = np.random.default_rng(16)
    N, heads, D, kp = 3, 2, 32, (14, 14)
    x = rng.standard_normal((N, 3 * heads * D, *kp)).astype(np.float32)
    q, k, v = (np.ascontiguousarray(x[:, i * 64:(i + 1) * 64]) for i in range(3))
    if qp == (1, 1):
        q = rng.standard_normal((N, 64, 1, 1)).astype(np.float32)
    blk, out, ws = to_blk(x), new_blk(N, 64, *qp), workspace(N, heads, heads, D, qp, kp, mode)
    image, part = 6 * 196 * 32, 4 * 2 * 196 * 32
    first = blk.data_ptr() if qp == kp else to_blk(q)
    B.small_attention(ctx(), first, blk.data_ptr() + part, blk.data_ptr() + 2 * part, out, ws, ws.numel(), N, heads, heads, D, qp, kp,
                      strides=(image if qp == kp else 0, image, image), flags=B.MATH[mode])
    close(from_blk(out, N, 64, *qp), R.attention(q, k, v, heads, heads, D ** -0.5), mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", [(2, 4, 2, 64, (16, 17), (16, 17)), (2, 4, 2, 64, (1, 1), (30, 30))])
def test_repeatable_on_streams_and_in_a_graph(shape, mode):
    N, heads, kv, D, qp, kp = shape
    rng = np.random.default_rng(17)
    q, k, v = make(rng, N, heads, kv, D, qp, kp)
    bias = table(rng, heads, qp, kp)
    first = run(q, k, v, heads, kv, mode, bias=bias)
    qb, kb, vb, tb, out = to_blk(q), to_blk(k), to_blk(v), dev(bias), new_blk(N, heads * D, *qp)
    outs = [new_blk(N, heads * D, *qp) for _ in range(2)]
    wss = [workspace(N, heads, kv, D, qp, kp, mode) for _ in range(3)]
    call = lambda o, ws: B.small_attention(ctx(), qb, kb, vb, o, ws, ws.numel(), N, heads, kv, D, qp, kp, bias=tb, flags=B.MATH[mode])       # noqa: E731
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):                                          # two calls at once, each with a workspace of its own
        for s, o, ws in zip(streams, outs, wss):
            with torch.cuda.stream(s):
                call(o, ws)
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(from_blk(o, N, heads * D, *qp), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, wss[2])
    out.fill_(0)
    for _ in range(3):
        graph.replay()
    assert np.array_equal(from_blk(out, N, heads * D, *qp), first)


def test_between_kernels_that_hold_tensor_memory():
    """Attention whose blocks take turns on an SM's tensor memory, with convolutions right behind it that want some too, over and over."""
    rng = np.random.default_rng(20)
    N, heads, D, plane = 24, 8, 32, (11, 11)
    q, k, v = make(rng, N, heads, heads, D, plane, plane)
    qb, kb, vb, out = to_blk(q), to_blk(k), to_blk(v), new_blk(N, heads * D, *plane)
    ws = workspace(N, heads, heads, D, plane, plane, "3xtf32")
    w = dev((rng.standard_normal((256, 256, 3, 3)) / 48).astype(np.float32))
    wb, y = torch.empty(B.small_conv_weight_elems(256, 256, 3, 3, B.MATH_3XTF32), device="cuda"), new_blk(N, 256, *plane)
    B.small_pack_conv_weights(ctx(), w, wb, 256, 256, 3, 3, B.MATH_3XTF32)
    for _ in range(40):
        B.small_attention(ctx(), qb, kb, vb, out, ws, ws.numel(), N, heads, heads, D, plane, plane, flags=B.MATH_3XTF32)
        B.small_conv2d(ctx(), out, wb, None, y, N, 256, 256, *plane, 3, 3, 1, (1, 1, 1, 1), B.MATH_3XTF32)
    close(from_blk(out, N, heads * D, *plane), R.attention(q, k, v, heads, heads, D ** -0.5), "3xtf32")
    assert np.isfinite(from_blk(y, N, 256, *plane)).all() and B.small_device_status(ctx()) == B.OK


@pytest.mark.parametrize("mode", MODES)
def test_random_shapes(mode):
    rng = np.random.default_rng(18)
    for _ in range(24):
        kv, share, D = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 129))
        kp = (int(rng.integers(1, 24)), int(rng.integers(1, 24)))
        qp = (1, 1) if rng.random() < 0.3 else kp if rng.random() < 0.6 else (int(rng.integers(1, 20)), int(rng.integers(1, 20)))
        N, heads = int(rng.integers(1, 4)), kv * share
        q, k, v = make(rng, N, heads, kv, D, qp, kp)
        bias = table(rng, heads, qp, kp) if rng.random() < 0.5 else None
        ke = np.stack([rng.integers(0, kp[0] + 1, N), rng.integers(0, kp[1] + 1, N)], 1).astype(np.int32) if rng.random() < 0.4 else None
        cap = float(rng.choice([0.0, 2.0]))
        close(run(q, k, v, heads, kv, mode, cap=cap, bias=bias, ke=ke), R.attention(q, k, v, heads, kv, D ** -0.5, cap=cap, bias=bias, k_extents=ke), mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", [(2, 2, 1, 32, (1, 1), (20, 21)), (2, 2, 2, 40, (5, 6), (5, 6)), (2, 4, 2, 64, (19, 19), (19, 19))])
def test_caps_at_both_ends_of_the_range(shape, mode):
    """Far above every score a cap has no part; next to nothing it leaves all keys alike, a score of exactly 0 (a query of zeros) among them."""
    N, heads, kv, D, qp, kp = shape
    rng = np.random.default_rng(21)
    q, k, v = make(rng, N, heads, kv, D, qp, kp)
    bias = table(rng, heads, qp, kp)
    q[:, :, 0, 0] = 0
    for b in (None, bias):
        free = R.attention(q, k, v, heads, kv, D ** -0.5, bias=b)
        for cap in (3.4e38, 2.4e38, 1e33):
            close(run(q, k, v, heads, kv, mode, cap=cap, bias=b), free, mode)
        alike = R.attention(q * 0, k, v, heads, kv, D ** -0.5, bias=b)
        for cap in (1e-39, 1e-38, 1e-30):
            close(run(q, k, v, heads, kv, mode, cap=cap, bias=b), alike, mode)
