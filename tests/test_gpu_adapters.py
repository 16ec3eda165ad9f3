"""1 x 1 convolutions with an adapter for each image against the formula in 64 bits, and the layers of an attention block run together.
Tolerances: the math modes' own (gpu_util.TOL); the sums have at most C + R terms."""
import numpy as np
import pytest
import torch

import attention_ref as R
from gpu_util import B, TOL, ctx, dev, from_blk, new_blk, pad_lanes_are_zero, rel_err, to_blk

pytestmark = pytest.mark.gpu
MODES = ["fp32", "3xtf32", "tf32"]


class Layer:
    def __init__(self, rng, C, K, rank, A, bias=True, scale=True):
        f = lambda *s: rng.standard_normal(s).astype(np.float32)          # noqa: E731
        self.C, self.K, self.R, self.A = C, K, rank, A
        self.w, self.b = f(K, C) * np.float32(C ** -0.5), f(K) if bias else None
        self.down, self.up = f(A, rank, C) * np.float32(C ** -0.5), f(A, K, rank) * np.float32(rank ** -0.5)
        self.scale = (0.5 + rng.random(A)).astype(np.float32) if scale else None

    def pack(self, mode):
        self.w_blk = torch.empty(B.small_conv_weight_elems(self.C, self.K, 1, 1, B.MATH[mode]), device="cuda")
        B.small_pack_conv_weights(ctx(), dev(self.w), self.w_blk, self.C, self.K, 1, 1, B.MATH[mode])
        self.packed = torch.full((B.small_adapter_elems(self.A, self.C, self.K, self.R),), float("nan"), device="cuda")
        B.small_pack_adapters(ctx(), dev(self.down), dev(self.up), self.packed, self.A, self.C, self.K, self.R)
        self.bt, self.st = (None if t is None else dev(t) for t in (self.b, self.scale))

    def call(self, blk, ids, out, ws, N, H, W, flags):
        B.small_adapted_conv2d(ctx(), blk, self.w_blk, self.bt, self.packed, ids, self.st, out, ws, N, self.C, self.K, H, W, self.R, self.A, flags)

    def workspace(self, N, H, W):
        need = B.small_adapted_conv2d_workspace_bytes(N, self.C, self.K, H, W, self.R)
        return torch.full((max(4, need // 4),), float("nan"), device="cuda")

    def run(self, x, ids, mode, relu=False, before=None):
        N, _, H, W = x.shape
        self.pack(mode)
        out = new_blk(N, self.K, H, W) if before is None else to_blk(before)
        self.call(to_blk(x), dev(ids), out, self.workspace(N, H, W), N, H, W, B.MATH[mode] | (B.RELU if relu else 0) | (0 if before is None else B.ACCUMULATE))
        assert pad_lanes_are_zero(out, N, self.K, H, W)
        got = from_blk(out, N, self.K, H, W)
        assert B.small_device_status(ctx()) == B.OK
        return got

    def ref(self, x, ids, relu=False, before=None):
        return R.adapted(x, self.w, self.b, self.down, self.up, ids, self.scale, relu, before)


SHAPES = [  # N, C, K, H, W, rank, adapters
    (1, 1, 1, 1, 1, 1, 1), (8, 512, 512, 1, 1, 8, 16), (3, 64, 64, 1, 1, 128, 2), (33, 96, 40, 1, 1, 4, 5), (130, 64, 128, 1, 1, 16, 7), (4, 96, 130, 13, 14, 5, 7),
    (2, 128, 128, 28, 28, 16, 3), (5, 40, 200, 7, 7, 33, 4), (2, 31, 33, 5, 9, 3, 2), (1, 256, 768, 14, 14, 64, 2), (3, 64, 96, 31, 29, 20, 9), (6, 320, 64, 3, 3, 8, 3),
    (1, 100, 300, 56, 56, 16, 1), (2, 32, 32, 1, 300, 100, 2), (9, 200, 1000, 1, 1, 16, 4),
    (40, 70, 300, 12, 11, 17, 6), (90, 33, 45, 8, 9, 128, 3), (75, 160, 64, 16, 16, 48, 80), (150, 64, 200, 10, 13, 5, 9)]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_the_formula(shape, mode):
    N, C, K, H, W, rank, A = shape
    rng = np.random.default_rng(C + K + rank)
    layer, x = Layer(rng, C, K, rank, A), rng.standard_normal((N, C, H, W)).astype(np.float32)
    ids = rng.integers(-1, A, N).astype(np.int32)
    ids[0] = A - 1
    before = rng.standard_normal((N, K, H, W)).astype(np.float32)
    assert rel_err(layer.run(x, ids, mode), layer.ref(x, ids)) <= TOL[mode]
    assert rel_err(layer.run(x, ids, mode, relu=True), layer.ref(x, ids, relu=True)) <= TOL[mode]
    assert rel_err(layer.run(x, ids, mode, relu=True, before=before), layer.ref(x, ids, relu=True, before=before)) <= TOL[mode]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("plane", [(1, 1), (9, 8)])
def test_indexes_outside_the_table_and_the_same_one_twice(plane, mode):
    rng = np.random.default_rng(21)
    layer, x = Layer(rng, 64, 64, 8, 3, bias=False, scale=False), rng.standard_normal((8, 64, *plane)).astype(np.float32)
    ids = np.array([-1, 3, -(1 << 31), (1 << 31) - 1, 2, 2, 0, 2], np.int32)
    got = layer.run(x, ids, mode)
    assert rel_err(got, layer.ref(x, ids)) <= TOL[mode]
    none = layer.run(x, np.full(8, -1, np.int32), mode)
    assert np.array_equal(none[:4], got[:4])                    # images without one: the shared projection's values, whatever the others use
    assert rel_err(none, layer.ref(x, np.full(8, -1))) <= TOL[mode]


@pytest.mark.parametrize("mode", MODES)
def test_images_do_not_reach_one_another(mode):
    """A value that is not finite in one image, or in an adapter that others use, stays where it belongs."""
    rng = np.random.default_rng(22)
    for plane in ((1, 1), (5, 5)):
        layer, x = Layer(rng, 64, 96, 8, 4), rng.standard_normal((6, 64, *plane)).astype(np.float32)
        ids = np.array([0, 1, 2, -1, 1, 0], np.int32)
        ref = layer.ref(x, ids)
        layer.down[2, 3, 7] = np.nan
        x[4, 10, 0, 0] = np.nan
        got = layer.run(x, ids, mode)
        assert np.isnan(got[2]).all() and np.isnan(got[4, :, 0, 0]).all()
        got[2], got[4, :, 0, 0] = ref[2], ref[4, :, 0, 0]
        assert rel_err(got, ref) <= TOL[mode]


@pytest.mark.parametrize("mode", ["fp32", "3xtf32"])
@pytest.mark.parametrize("R_", [4, 40])
def test_pixels_and_adapters_of_very_different_size(R_, mode):
    """One pixel far larger than its neighbours, and adapters far larger and smaller than the filters: each pixel keeps its own accuracy."""
    rng = np.random.default_rng(25)
    layer, x = Layer(rng, 96, 160, R_, 3), rng.standard_normal((80, 96, 9, 10)).astype(np.float32)
    x[:, :, 4, 5] *= 1e12
    x[:, :, 7, 1] *= 1e-12
    layer.b[:] = 0
    layer.up[1] *= 1e6
    layer.down[2] *= 1e-6
    ids = (np.arange(80) % 4 - 1).astype(np.int32)
    got, ref = layer.run(x, ids, mode), layer.ref(x, ids)
    size = np.sqrt((ref ** 2).mean(1, keepdims=True))
    assert rel_err(got / size, ref / size) <= TOL[mode]


@pytest.mark.parametrize("plane", [(1, 1), (14, 13)])
def test_repeatable_on_streams_and_in_a_graph(plane):
    rng = np.random.default_rng(23)
    N, (H, W) = 5, plane
    layer, x, ids = Layer(rng, 96, 128, 12, 3), rng.standard_normal((5, 96, *plane)).astype(np.float32), np.array([0, 2, -1, 1, 0], np.int32)
    first = layer.run(x, ids, "3xtf32")
    blk, idt = to_blk(x), dev(ids)
    outs, wss = [new_blk(N, 128, H, W) for _ in range(2)], [layer.workspace(N, H, W) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o, ws in zip(streams, outs, wss):
            with torch.cuda.stream(s):
                layer.call(blk, idt, o, ws, N, H, W, B.MATH_3XTF32)
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(from_blk(o, N, 128, H, W), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.call(blk, idt, outs[0], wss[0], N, H, W, B.MATH_3XTF32)
    outs[0].fill_(0)
    idt.copy_(torch.tensor([1, 1, 1, -1, 2], dtype=torch.int32))          # indexes are read when the kernel runs
    for _ in range(2):
        graph.replay()
    assert rel_err(from_blk(outs[0], N, 128, H, W), layer.ref(x, idt.cpu().numpy())) <= TOL["3xtf32"]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("N,C,heads,plane", [(3, 64, 2, (14, 14)), (2, 80, 2, (9, 13)), (1, 128, 2, (28, 20))])
def test_an_attention_block(N, C, heads, plane, mode):
    """x + Wo attention(Wqkv norm(x)): all layers behind one another in one stream, q, k and v as slices of one tensor."""
    rng = np.random.default_rng(24)
    H, W = plane
    D, blocks = C // heads, (C + 31) // 32
    CP = blocks * 32                                                       # each of q, k and v begins with a channel block
    x = rng.standard_normal((N, C, H, W)).astype(np.float32)
    gamma, beta = (1 + 0.1 * rng.standard_normal(C)).astype(np.float32), (0.1 * rng.standard_normal(C)).astype(np.float32)
    qkv, proj = Layer(rng, C, 3 * CP, 8, 4), Layer(rng, C, C, 8, 4)
    pad = (np.arange(3 * CP) % CP) >= C                                    # their pad lanes stay zero
    qkv.w[pad], qkv.b[pad], qkv.up[:, pad] = 0, 0, 0
    ids = rng.integers(-1, 4, N).astype(np.int32)
    bias = (0.5 * rng.standard_normal((heads, 2 * H - 1, 2 * W - 1))).astype(np.float32)
    for layer in (qkv, proj):
        layer.pack(mode)
    blk, y, stacked, mixed, out, idt = to_blk(x), new_blk(N, C, H, W), new_blk(N, 3 * CP, H, W), new_blk(N, C, H, W), to_blk(x), dev(ids)
    wss = [qkv.workspace(N, H, W), proj.workspace(N, H, W)]
    aws = torch.empty(max(16, B.small_attention_workspace_bytes(N, heads, heads, D, plane, plane, B.MATH[mode])), dtype=torch.uint8, device="cuda")
    nws = torch.empty(max(16, B.small_group_norm_workspace_bytes(N, C, H, W, 8)), dtype=torch.uint8, device="cuda")
    g, b, t = dev(gamma), dev(beta), dev(bias)
    image, part = 3 * CP * H * W, 4 * CP * H * W
    B.small_group_norm(ctx(), blk, g, b, y, nws, N, C, H, W, 8)
    qkv.call(y, idt, stacked, wss[0], N, H, W, B.MATH[mode])
    p = stacked.data_ptr()
    B.small_attention(ctx(), p, p + part, p + 2 * part, mixed, aws, aws.numel(), N, heads, heads, D, plane, plane, bias=t, strides=(image,) * 3, flags=B.MATH[mode])
    proj.call(mixed, idt, out, wss[1], N, H, W, B.MATH[mode] | B.ACCUMULATE)
    a = qkv.ref(R.group_norm(x, gamma, beta, 8, 1e-5, "none"), ids)
    z = R.attention(a[:, :C], a[:, CP:CP + C], a[:, 2 * CP:2 * CP + C], heads, heads, D ** -0.5, bias=bias)
    # four layers behind one another: each one's error, and the first projection's once more through the scores
    assert rel_err(from_blk(out, N, C, H, W), proj.ref(z, ids, before=x)) <= 2 * TOL[mode]
    assert B.small_device_status(ctx()) == B.OK


@pytest.mark.parametrize("mode", MODES)
def test_more_filters_than_stay_in_registers(mode):
    """300 and 486 blocks of 32 x 32 weights; a converting team keeps six."""
    rng = np.random.default_rng(61)
    for N, C, K in ((80, 320, 960), (76, 840, 570)):
        layer, x = Layer(rng, C, K, 9, 3), rng.standard_normal((N, C, 8, 8)).astype(np.float32)
        ids = rng.integers(-1, 3, N).astype(np.int32)
        assert B.small_adapted_conv2d_workspace_bytes(N, C, K, 8, 8, 9) > 0
        assert rel_err(layer.run(x, ids, mode), layer.ref(x, ids)) <= TOL[mode]
