"""The layers of an attention block in a convolutional network, as cases to time.

Such a block normalises a feature map (`small_group_norm`), projects it with a 1 x 1 convolution that the images of a batch
share while each request may bring a low-rank adapter of its own (`small_adapted_conv2d`), and lets every pixel attend to
every other one (`small_attention`).  Three kinds of case:

  norm      group normalisation with its affine and an activation
  attend    attention over the pixels of a plane: heads of their own or shared between queries, a learned bias for each
            displacement, scores capped by a tanh, images padded to a common plane.  A query plane of one pixel is the
            attention pooling in front of a classifier, the form for a single query.
  adapt     a 1 x 1 convolution (a full reduction where the plane is one pixel) whose images use adapters picked by index,
            or none

All tensors are float, in the blocked layout [N][ceil(C / 32)][H][W][32] with zero pad lanes; arithmetic is asked for at FP32
accuracy (`MATH_3XTF32`).  Planes, channels and batches are those of the layer sweep and the networks of synth/configs.py, and ragged
ones like them.
"""
import math

import torch

own = False

_ctx = {}


def listed():
    return [
        # behind the last pair of the keyword-spotting network, one recording: a few microseconds, where the launch counts
        dict(name="norm_c64_25x5_n1", op="norm", N=1, C=64, H=25, W=5, groups=8, act="silu"),
        # a residual stage's normalisation at a serving batch
        dict(name="norm_c128_hw28_n64", op="norm", N=64, C=128, H=28, W=28, groups=32, act="relu"),
        # channels that fill no whole block, groups that no block holds a whole number of, an odd plane, no activation
        dict(name="norm_c72_13x29_n16", op="norm", N=16, C=72, H=13, W=29, groups=6, act="none"),
        # the sweep's largest plane at its batch and 256 channels
        dict(name="norm_c256_hw56_n128", op="norm", N=128, C=256, H=56, W=56, groups=32, act="silu"),
        # attention pooling: one query an image over a 7 x 7 plane
        _attend("attend_pool_hw7_n8", 8, 8, 8, 64, 1, 1, 7, 7),
        # one query an image over a long axis: the plane of the depthwise-separable network's input, shared heads
        _attend("attend_pool_hw96_n4", 4, 8, 4, 64, 1, 1, 96, 96),
        # self-attention on a 14 x 14 plane with a bias for each displacement
        _attend("attend_hw14_n32", 32, 4, 4, 32, 14, 14, 14, 14, bias=True),
        # an odd plane, shared heads of 40 channels, capped scores, padded images
        _attend("attend_25x13_n8", 8, 6, 2, 40, 25, 13, 25, 13, bias=True, cap=20.0, ragged=True),
        # self-attention on the sweep's largest plane: 3136 pixels
        _attend("attend_hw56_n4", 4, 8, 8, 64, 56, 56, 56, 56, bias=True),
        # eight requests of one vector each, eight adapters in use: a classifier's full reduction
        dict(name="adapt_c512_n8", op="adapt", N=8, C=512, K=512, H=1, W=1, R=8, adapters=16, relu=False),
        # ragged channels, filters and plane, an odd rank
        dict(name="adapt_c96_k130_n24", op="adapt", N=24, C=96, K=130, H=13, W=14, R=5, adapters=7, relu=True),
        # the projection to queries, keys and values of a batch
        dict(name="adapt_c256_k768_n64", op="adapt", N=64, C=256, K=768, H=28, W=28, R=16, adapters=32, relu=False),
    ]


def _attend(name, N, heads, kv, D, QH, QW, KH, KW, bias=False, cap=0.0, ragged=False):
    return dict(name=name, op="attend", N=N, heads=heads, kv=kv, D=D, QH=QH, QW=QW, KH=KH, KW=KW, bias=bias, cap=cap, ragged=ragged)


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["norm", "attend", "adapt"])
    if kind == "norm":
        while True:
            g = rng.choice([1, 2, 3, 4, 6, 8, 16, 32])
            C, H, W = g * _log(rng, 1, 512 // g), _log(rng, 2, 130), _log(rng, 2, 130)
            N = _log(rng, 1, 128)
            if N * C * H * W <= 128 * 256 * 56 * 56:
                return dict(op="norm", N=N, C=C, H=H, W=W, groups=g, act=rng.choice(["none", "relu", "silu"]))
    if kind == "attend":
        while True:
            kv, share, D = _log(rng, 1, 8), rng.choice([1, 1, 2, 3, 4]), rng.choice([8, 16, 20, 32, 40, 48, 64, 96, 128])
            KH, KW, N = _log(rng, 1, 96), _log(rng, 1, 96), _log(rng, 1, 64)
            pool = rng.random() < 0.35
            QH, QW = (1, 1) if pool else (KH, KW)
            work = N * kv * share * QH * QW * KH * KW * D
            if kv * share * D <= 1024 and work <= 4 * 8 * 3136 * 3136 * 64 and N * kv * D * KH * KW <= 1 << 26:
                return dict(op="attend", N=N, heads=kv * share, kv=kv, D=D, QH=QH, QW=QW, KH=KH, KW=KW, bias=rng.random() < 0.5,
                            cap=rng.choice([0.0, 0.0, 15.0]), ragged=rng.random() < 0.4)
    while True:
        C, K, N = _log(rng, 8, 512), _log(rng, 8, 1024), _log(rng, 1, 128)
        H, W = (1, 1) if rng.random() < 0.3 else (_log(rng, 2, 56), _log(rng, 2, 56))
        if N * H * W * C * K <= 64 * 784 * 256 * 768 and N * H * W * (C + K) <= 64 * 784 * 1024:
            return dict(op="adapt", N=N, C=C, K=K, H=H, W=W, R=_log(rng, 1, 64), adapters=_log(rng, 1, 32), relu=rng.random() < 0.4)


def _blocks(C):
    return -(-C // 32)


def _random(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _blocked(x):
    """[N][C][pixels] -> [N][ceil(C / 32)][pixels][32], pad lanes zero."""
    N, C, P = x.shape
    CB = _blocks(C)
    if C % 32:
        x = torch.cat([x, x.new_zeros(N, CB * 32 - C, P)], 1)
    return x.view(N, CB, 32, P).transpose(2, 3).contiguous()


def _plain(x, C):
    """[N][ceil(C / 32)][pixels][32] -> [N][C][pixels]."""
    N, CB, P, _ = x.shape
    return x.transpose(2, 3).reshape(N, CB * 32, P)[:, :C]


def _empty(N, C, P):
    return torch.empty(N, _blocks(C), P, 32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = dict(case)
    N = c["N"]
    if c["op"] == "norm":
        C, P = c["C"], c["H"] * c["W"]
        # activations behind a convolution: every channel with a mean and a spread of its own
        x = _random(gen, N, C, P) * (0.3 + _random(gen, 1, C, 1).abs()) + 0.7 * _random(gen, 1, C, 1)
        s = dict(c, x=_blocked(x), gamma=1.0 + 0.2 * _random(gen, C), beta=0.2 * _random(gen, C), out=_empty(N, C, P))
        if own:
            B, ctx = _library()
            s["ws"] = torch.empty(max(16, B.small_group_norm_workspace_bytes(N, C, c["H"], c["W"], c["groups"])), dtype=torch.uint8, device="cuda")
    elif c["op"] == "attend":
        heads, kv, D, QP, KP = c["heads"], c["kv"], c["D"], c["QH"] * c["QW"], c["KH"] * c["KW"]
        s = dict(c, q=_blocked(1.2 * _random(gen, N, heads * D, QP)), k=_blocked(1.2 * _random(gen, N, kv * D, KP)),
                 v=_blocked(_random(gen, N, kv * D, KP) + 0.5 * _random(gen, 1, kv * D, 1)), out=_empty(N, heads * D, QP), table=None, qe=None, ke=None)
        if c["bias"]:
            # a learned table: near pixels are favoured, each head with a slope of its own
            dy = torch.arange(c["QH"] + c["KH"] - 1, device="cuda") - (c["KH"] - 1)
            dx = torch.arange(c["QW"] + c["KW"] - 1, device="cuda") - (c["KW"] - 1)
            far = (dy[:, None].abs() + dx[None, :].abs()).float()
            slope = 0.5 ** (1.0 + 6.0 * torch.arange(heads, device="cuda") / heads)
            s["table"] = (0.5 * _random(gen, heads, far.shape[0], far.shape[1]) - slope[:, None, None] * far).contiguous()
        if c["ragged"]:
            # images padded to a common plane; the first one fills it
            def extent(n):
                e = (torch.rand(N, generator=gen, device="cuda") * (n + 1)).long().clamp(max=n)       # 0: a slot without an image
                e[0] = n
                return e
            s["ke"] = torch.stack([extent(c["KH"]), extent(c["KW"])], 1).int().contiguous()
            s["qe"] = s["ke"] if QP == KP else None
        if own:
            B, ctx = _library()
            s["ws"] = torch.empty(max(16, B.small_attention_workspace_bytes(N, heads, kv, D, (c["QH"], c["QW"]), (c["KH"], c["KW"]), B.MATH_3XTF32)),
                                  dtype=torch.uint8, device="cuda")
    else:
        C, K, R, P, A = c["C"], c["K"], c["R"], c["H"] * c["W"], c["adapters"]
        ids = (torch.rand(N, generator=gen, device="cuda") * (A + 1)).long().clamp(max=A) - 1        # -1: no adapter
        s = dict(c, x=_blocked(_random(gen, N, C, P)), w=_random(gen, K, C) * math.sqrt(2.0 / C), b=0.1 * _random(gen, K),
                 down=_random(gen, A, R, C) / math.sqrt(C), up=_random(gen, A, K, R) / math.sqrt(R),
                 scale=0.25 + 0.5 * torch.rand(A, generator=gen, device="cuda"), ids=ids.int(), out=_empty(N, K, P))
        if own:
            B, ctx = _library()
            s["w_blk"] = torch.empty(B.small_conv_weight_elems(C, K, 1, 1, B.MATH_3XTF32), device="cuda")
            B.small_pack_conv_weights(ctx, s["w"], s["w_blk"], C, K, 1, 1, B.MATH_3XTF32)
            s["ad_blk"] = torch.empty(B.small_adapter_elems(A, C, K, R), device="cuda")
            B.small_pack_adapters(ctx, s["down"], s["up"], s["ad_blk"], A, C, K, R)
            s["ws"] = torch.empty(max(16, B.small_adapted_conv2d_workspace_bytes(N, C, K, c["H"], c["W"], R)), dtype=torch.uint8, device="cuda")
    return s


def _library():
    from paper_2303_04769_b200 import binding as B
    device = torch.cuda.current_device()
    if device not in _ctx:
        _ctx[device] = B.small_init(device)
    return B, _ctx[device]


def run(state):
    return {"norm": _norm, "attend": _attention, "adapt": _adapted}[state["op"]](state)


def _norm(s):
    N, C, H, W, G = s["N"], s["C"], s["H"], s["W"], s["groups"]
    if own:
        B, ctx = _library()
        flags = {"none": 0, "relu": B.RELU, "silu": B.SILU}[s["act"]]
        B.small_group_norm(ctx, s["x"], s["gamma"], s["beta"], s["out"], s["ws"], N, C, H, W, G, 1e-5, flags)
        return s["out"]
    x = _plain(s["x"], C).reshape(N, G, -1)
    x = x - x.mean(2, keepdim=True)
    x = x / torch.sqrt((x * x).mean(2, keepdim=True) + 1e-5)
    y = x.view(N, C, H * W) * s["gamma"][:, None] + s["beta"][:, None]
    if s["act"] == "relu":
        y = y.clamp(min=0.0)
    elif s["act"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    return _blocked(y)


def _displacements(s):
    """[queries][keys]: where in the bias table a query and a key meet."""
    def at(h, w):
        i = torch.arange(h * w, device="cuda")
        return i // w, i % w
    qy, qx = at(s["QH"], s["QW"])
    ky, kx = at(s["KH"], s["KW"])
    return (qy[:, None] - ky[None, :] + s["KH"] - 1) * (s["QW"] + s["KW"] - 1) + qx[:, None] - kx[None, :] + s["KW"] - 1


def _inside(extents, h, w):
    """[N][pixels]: the pixels inside each image's extent."""
    i = torch.arange(h * w, device="cuda")
    return (i // w < extents[:, :1]) & (i % w < extents[:, 1:])


def _attention(s):
    N, heads, kv, D = s["N"], s["heads"], s["kv"], s["D"]
    scale = 1.0 / math.sqrt(D)
    if own:
        B, ctx = _library()
        B.small_attention(ctx, s["q"], s["k"], s["v"], s["out"], s["ws"], s["ws"].numel(), N, heads, kv, D, (s["QH"], s["QW"]), (s["KH"], s["KW"]),
                          scale=scale, cap=s["cap"], bias=s["table"], q_extents=s["qe"], k_extents=s["ke"], flags=B.MATH_3XTF32)
        return s["out"]
    q = _plain(s["q"], heads * D).reshape(N, kv, heads // kv, D, -1)
    k = _plain(s["k"], kv * D).reshape(N, kv, 1, D, -1)
    v = _plain(s["v"], kv * D).reshape(N, kv, 1, D, -1)
    x = torch.matmul(q.transpose(3, 4), k) * scale                    # [N][kv][share][queries][keys]
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    if s["table"] is not None:
        x = x + s["table"].reshape(kv, heads // kv, -1)[:, :, _displacements(s)]
    if s["ke"] is not None:
        x = x.masked_fill(~_inside(s["ke"], s["KH"], s["KW"])[:, None, None, None, :], -math.inf)
    top = x.amax(4, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(4, keepdim=True)
    y = torch.matmul(p / torch.where(total == 0, torch.ones_like(total), total), v.transpose(3, 4))
    if s["qe"] is not None:
        y = y * _inside(s["qe"], s["QH"], s["QW"])[:, None, None, :, None]
    return _blocked(y.transpose(3, 4).reshape(N, heads * D, -1))


def _adapted(s):
    N, C, K, H, W = s["N"], s["C"], s["K"], s["H"], s["W"]
    if own:
        B, ctx = _library()
        B.small_adapted_conv2d(ctx, s["x"], s["w_blk"], s["b"], s["ad_blk"], s["ids"], s["scale"], s["out"], s["ws"], N, C, K, H, W, s["R"], s["adapters"],
                               B.MATH_3XTF32 | (B.RELU if s["relu"] else 0))
        return s["out"]
    x = _plain(s["x"], C)
    ids = s["ids"].long()
    pick = ids.clamp(min=0)
    factor = torch.where(ids >= 0, s["scale"][pick], torch.zeros_like(s["scale"][pick]))
    y = torch.matmul(s["w"], x) + s["b"][:, None]
    y = y + factor[:, None, None] * torch.matmul(s["up"][pick], torch.matmul(s["down"][pick], x))
    return _blocked(y.clamp(min=0.0) if s["relu"] else y)


def work(case):
    """Each tensor once (channels without pad lanes, the adapters that can be in use), a multiplication and an addition as two."""
    c, N = case, case["N"]
    if c["op"] == "norm":
        n = N * c["C"] * c["H"] * c["W"]
        return {"bytes": 4.0 * (2 * n + 2 * c["C"]), "flops": 9.0 * n}
    if c["op"] == "attend":
        QP, KP = c["QH"] * c["QW"], c["KH"] * c["KW"]
        table = c["heads"] * (c["QH"] + c["KH"] - 1) * (c["QW"] + c["KW"] - 1) if c["bias"] else 0
        # padded images: the first one whole, of the others a quarter of the keys on the average, and a ninth of the pairs
        keys = (1 + (N - 1) / 4) if c["ragged"] else N
        pairs = keys if QP != KP else (1 + (N - 1) / 9) if c["ragged"] else N
        return {"bytes": 4.0 * (c["heads"] * c["D"] * QP * ((keys if QP == KP else N) + N) + 2 * keys * c["kv"] * c["D"] * KP + table),
                "flops": 4.0 * pairs * c["heads"] * QP * KP * c["D"]}
    P, used = c["H"] * c["W"], min(N, c["adapters"])
    return {"bytes": 4.0 * (N * P * (c["C"] + c["K"]) + c["C"] * c["K"] + c["K"] + used * c["R"] * (c["C"] + c["K"]) + N),
            "flops": 2.0 * N * P * (c["C"] * c["K"] + c["R"] * (c["C"] + c["K"]))}


def exact(case, seed):
    s = prepare(case, seed)
    N = s["N"]

    def channels(x, C):                          # blocked -> [N][pixels][C] in 64 bits
        return x.double().permute(0, 2, 1, 3).flatten(2)[..., :C]

    def back(y):                                 # [N][pixels][C] -> blocked
        C = y.shape[2]
        full = y.new_zeros(y.shape[0], y.shape[1], _blocks(C) * 32)
        full[..., :C] = y
        return full.unflatten(2, (-1, 32)).permute(0, 2, 1, 3).contiguous()

    if s["op"] == "norm":
        parts = []
        for x in s["x"].split(16):
            g = channels(x, s["C"]).unflatten(2, (s["groups"], -1))
            mean = g.mean((1, 3), keepdim=True)
            var = ((g - mean) ** 2).mean((1, 3), keepdim=True)
            y = ((g - mean) * torch.rsqrt(var + 1e-5)).flatten(2) * s["gamma"].double() + s["beta"].double()
            y = y.clamp(min=0) if s["act"] == "relu" else y * torch.sigmoid(y) if s["act"] == "silu" else y
            parts.append(back(y))
        return torch.cat(parts)
    if s["op"] == "attend":
        heads, kv, D = s["heads"], s["kv"], s["D"]
        q, k, v = channels(s["q"], heads * D), channels(s["k"], kv * D), channels(s["v"], kv * D)
        out = torch.zeros_like(q)
        where = _displacements(s) if s["table"] is not None else None
        for n in range(N):
            keys = torch.ones(s["KH"] * s["KW"], dtype=torch.bool, device="cuda")
            rows = torch.ones(s["QH"] * s["QW"], dtype=torch.bool, device="cuda")
            if s["ke"] is not None:
                keys = _inside(s["ke"][n:n + 1], s["KH"], s["KW"])[0]
            if s["qe"] is not None:
                rows = _inside(s["qe"][n:n + 1], s["QH"], s["QW"])[0]
            for h in range(heads):
                j = h // (heads // kv)
                x = q[n][rows][:, h * D:(h + 1) * D] @ k[n][keys][:, j * D:(j + 1) * D].T * (D ** -0.5)
                if s["cap"]:
                    x = torch.tanh(x / s["cap"]) * s["cap"]
                if where is not None:
                    x = x + s["table"][h].double().flatten()[where[rows][:, keys]]
                out[n, rows, h * D:(h + 1) * D] = torch.softmax(x, 1) @ v[n][keys][:, j * D:(j + 1) * D]
        return back(out)
    x = channels(s["x"], s["C"])
    y = x @ s["w"].double().T + s["b"].double()
    for n, i in enumerate(s["ids"].tolist()):
        if i >= 0:
            y[n] += s["scale"][i].double() * (x[n] @ s["down"][i].double().T) @ s["up"][i].double().T
    return back(y.clamp(min=0) if s["relu"] else y)
