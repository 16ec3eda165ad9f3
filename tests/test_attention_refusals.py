"""Calls of the attention block's layers that are refused: found on the host before anything is launched, so they are tested
without a device, on a context that is only looked at (zeroed) and addresses that nothing reads."""
import ctypes

import pytest

B = pytest.importorskip("paper_2303_04769_b200.binding")

CTX = ctypes.c_void_p()
_room = (ctypes.c_char * 8192)()
INVALID, SHAPE, ALIGN, OVERLAP, WORKSPACE, NOT_INIT = 1, 2, 3, 4, 5, 9
STREAM = 0


@pytest.fixture(scope="module", autouse=True)
def context():
    from paper_2303_04769_b200 import build
    build.build()
    CTX.value = ctypes.addressof(_room)
    yield
    CTX.value = None


def at(i):
    return (i + 1) << 36


def status(f, *args, **kw):
    with pytest.raises(B.SmallError) as e:
        f(*args, **kw)
    return e.value.status


def norm(ctx=CTX, x=at(0), gamma=at(1), beta=at(2), out=at(3), ws=at(4), N=2, C=64, H=8, W=8, groups=8, eps=1e-5, flags=0):
    return status(B.small_group_norm, ctx, x, gamma, beta, out, ws, N, C, H, W, groups, eps, flags, STREAM)


def test_group_norm():
    assert norm(ctx=0) == NOT_INIT
    assert norm(x=None) == INVALID and norm(out=None) == INVALID
    assert norm(flags=B.RELU | B.SILU) == INVALID and norm(flags=B.ACCUMULATE) == INVALID and norm(flags=B.MATH_TF32) == INVALID
    assert norm(eps=-1e-5) == INVALID and norm(eps=float("nan")) == INVALID and norm(eps=float("inf")) == INVALID
    assert norm(x=at(0) + 4) == ALIGN and norm(gamma=at(1) + 8) == ALIGN and norm(ws=at(4) + 4) == ALIGN
    for bad in (dict(N=0), dict(C=0), dict(H=0), dict(W=-1), dict(groups=0), dict(groups=7), dict(groups=128), dict(H=1 << 13, W=1 << 12)):
        assert norm(**bad) == SHAPE
        full = dict(N=2, C=64, H=8, W=8, groups=8) | bad
        assert B.small_group_norm_workspace_bytes(full["N"], full["C"], full["H"], full["W"], full["groups"]) == 0
    assert norm(N=1, C=65536, H=2, W=2, groups=1) == 6                   # a group that no block's shared memory holds the sums of
    assert norm(out=at(0) + 1024) == OVERLAP and norm(gamma=at(3) + 16) == OVERLAP and norm(beta=at(3)) == OVERLAP
    big = dict(H=512, W=512)
    assert B.small_group_norm_workspace_bytes(2, 64, 512, 512, 8) > 0 and B.small_group_norm_workspace_bytes(2, 64, 8, 8, 8) == 0
    assert norm(ws=None, **big) == WORKSPACE and norm(ws=at(0), **big) == OVERLAP and norm(ws=at(3), **big) == OVERLAP and norm(ws=at(1), **big) == OVERLAP


def attend(ctx=CTX, q=at(0), k=at(1), v=at(2), out=at(3), ws=at(4), ws_bytes=1 << 40, N=2, heads=4, kv=2, D=32, qp=(8, 8), kp=(8, 8), bias=at(5), qe=at(6),
           ke=at(7), strides=(0, 0, 0), scale=0.1, cap=0.0, flags=B.MATH_3XTF32 if B else 0):
    return status(B.small_attention, ctx, q, k, v, out, ws, ws_bytes, N, heads, kv, D, qp, kp, scale, cap, bias, qe, ke, strides, flags, STREAM)


def test_attention():
    assert attend(ctx=0) == NOT_INIT
    for name in ("q", "k", "v", "out"):
        assert attend(**{name: None}) == INVALID and attend(**{name: at(9) + 4}) == ALIGN
    for name in ("bias", "qe", "ke", "ws"):
        assert attend(**{name: at(9) + 8}) == ALIGN
    assert attend(flags=B.RELU) == INVALID and attend(flags=3 << 4) == INVALID and attend(flags=B.SILU | B.MATH_TF32) == INVALID
    for bad in (dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf"))):
        assert attend(**bad) == INVALID
    for bad in (dict(N=0), dict(heads=0), dict(kv=0), dict(heads=3), dict(D=0), dict(D=129), dict(qp=(0, 8)), dict(qp=(8, -1)), dict(kp=(8, 0)),
                dict(kp=(1 << 13, 1 << 12)), dict(N=1 << 17), dict(heads=1 << 17, kv=1)):
        assert attend(**bad) == SHAPE
        f = dict(N=2, heads=4, kv=2, D=32, qp=(8, 8), kp=(8, 8)) | bad
        assert B.small_attention_workspace_bytes(f["N"], f["heads"], f["kv"], f["D"], f["qp"], f["kp"], B.MATH_3XTF32) == 0
    assert B.small_attention_workspace_bytes(2, 4, 2, 32, (8, 8), (8, 8), 3 << 4) == 0
    # strides: an image's run has to fit, whole vectors, and stay inside 64 bits
    run, krun = 4 * 64 * 32, 2 * 64 * 32
    assert attend(strides=(run - 4, 0, 0)) == SHAPE and attend(strides=(0, krun - 32, 0)) == SHAPE and attend(strides=(0, 0, -4)) == SHAPE
    assert attend(strides=(run + 2, 0, 0)) == ALIGN and attend(strides=(0, krun + 1, 0)) == ALIGN
    assert attend(strides=(0, 1 << 60, 0)) == SHAPE
    for name in ("q", "k", "v", "bias", "qe", "ke"):
        assert attend(**{name: at(3)}) == OVERLAP
    assert attend(k=at(3) - 4 * (3 * krun + krun) + 16, strides=(0, 3 * krun, 0)) == OVERLAP            # the last image reaches the output
    need = B.small_attention_workspace_bytes(1, 8, 8, 64, (56, 56), (56, 56), B.MATH_3XTF32)
    if need:
        large = dict(N=1, heads=8, kv=8, D=64, qp=(56, 56), kp=(56, 56))
        assert attend(ws_bytes=need - 1, **large) == WORKSPACE and attend(ws=None, **large) == WORKSPACE
        for name in ("q", "k", "v", "bias", "qe", "ke", "out"):
            assert attend(**{name: at(4)}, **large) == OVERLAP


def adapt(ctx=CTX, x=at(0), w=at(1), b=at(2), packed=at(3), ids=at(4), scale=at(5), out=at(6), ws=at(7), N=80, C=64, K=96, H=8, W=8, R=9, A=4,
          flags=B.MATH_3XTF32 if B else 0):
    return status(B.small_adapted_conv2d, ctx, x, w, b, packed, ids, scale, out, ws, N, C, K, H, W, R, A, flags, STREAM)


def test_adapters():
    assert adapt(ctx=0) == NOT_INIT
    for name in ("x", "w", "packed", "ids", "out"):
        assert adapt(**{name: None}) == INVALID and adapt(**{name: at(9) + 4}) == ALIGN
    for name in ("b", "scale", "ws"):
        assert adapt(**{name: at(9) + 4}) == ALIGN
    assert adapt(ws=None) == WORKSPACE and B.small_adapted_conv2d_workspace_bytes(80, 64, 96, 8, 8, 9) > 0
    assert B.small_adapted_conv2d_workspace_bytes(2, 64, 96, 8, 8, 9) == 0 and adapt(ws=None, N=2) not in (WORKSPACE, INVALID)        # not needed: gets as far as the device
    assert adapt(flags=B.SILU) == INVALID and adapt(flags=B.RELU_MID) == INVALID and adapt(flags=3 << 4) == INVALID
    for bad in (dict(N=0), dict(C=0), dict(K=0), dict(H=0), dict(W=0), dict(R=0), dict(R=129), dict(A=0), dict(H=1 << 13, W=1 << 12)):
        assert adapt(**bad) == SHAPE
    for name in ("x", "w", "b", "packed", "ids", "scale", "ws"):
        assert adapt(**{name: at(6)}) == OVERLAP
    for name in ("x", "w", "b", "packed", "ids", "scale"):
        assert adapt(**{name: at(7)}) == OVERLAP
    assert B.small_adapter_elems(0, 64, 64, 8) == 0 and B.small_adapter_elems(2, 64, 64, 129) == 0
    assert B.small_adapted_conv2d_workspace_bytes(2, 64, 64, 0, 8, 8) == 0
    pack = lambda ctx=CTX, down=at(0), up=at(1), packed=at(2), A=4, C=64, K=96, R=8: status(B.small_pack_adapters, ctx, down, up, packed, A, C, K, R, STREAM)  # noqa: E731
    assert pack(ctx=0) == NOT_INIT and pack(down=None) == INVALID and pack(up=at(1) + 4) == ALIGN and pack(R=0) == SHAPE and pack(A=0) == SHAPE
    assert pack(down=at(2)) == OVERLAP and pack(up=at(2) + 64) == OVERLAP


def test_attention_without_channels_and_a_scale():
    for D in (0, -1):
        assert attend(D=D, scale=None) == SHAPE


CUDA = 7


def test_a_context_without_a_device_goes_no_further():
    """Calls with nothing else wrong: a zeroed context has no SMs to plan for, with a GPU in the machine or without one."""
    for refused in (norm(), attend(), attend(qp=(1, 1)), attend(flags=B.MATH_FP32), adapt(), adapt(N=2, ws=None), adapt(N=2, H=1, W=1), adapt(flags=B.MATH_FP32),
                    status(B.small_pack_adapters, CTX, at(0), at(1), at(2), 4, 64, 96, 8, STREAM)):
        assert refused == CUDA


def test_fp32_needs_no_workspace():
    """The products of halves are the other modes': FP32 gets as far as the device without their room, and does not look at what is given."""
    assert B.small_adapted_conv2d_workspace_bytes(80, 64, 96, 8, 8, 9) > 0
    for ws in (None, at(6), at(0)):
        assert adapt(ws=ws, flags=B.MATH_FP32) == CUDA
    for flags in (B.MATH_TF32, B.MATH_3XTF32):
        assert adapt(ws=None, flags=flags) == WORKSPACE and adapt(ws=at(6), flags=flags) == OVERLAP
