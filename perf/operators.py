"""The operators of the gated feed-forward block, the linear layer's gradient and the rotary embedding with several
axes, as cases with real sizes: what a program has in hand, one call of the operator, and the same value in plain
torch operations (`own` false) and from the definition in 64 bits (`exact`).

Widths are those of the encoder configurations of this repository (0.6B-class 1152 / 4304, 0.7B-class 1280 / 5120,
6B-class 3200 / 12800, the small float one 256 / 1024); token counts are those of its workloads, one token, and
odd numbers in between.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
GATES = ("silu", "gelu_tanh", "gelu_erf")
LAYOUTS = ("blocks", "sections", "interleaved")


def listed():
    return [
        # one token through the 0.6B-class block: the step of a token-by-token loop, weights streamed once
        dict(name="mlp_one_token", op="mlp", dtype=BF16, M=1, K=1152, N=4304, gate="silu", bias=True),
        # a handful of tokens through the 6B-class block: still bound by the weights
        dict(name="mlp_16_tokens_6b", op="mlp", dtype=BF16, M=16, K=3200, N=12800, gate="gelu_erf", bias=True),
        # 16 images of 448 x 448 through the 6B-class block
        dict(name="mlp_16_images_6b", op="mlp", dtype=BF16, M=16384, K=3200, N=12800, gate="silu", bias=True),
        # a training step of the block: 8 images of 448 x 448, 0.6B class
        dict(name="mlp_train_8_images", op="mlp_train", dtype=BF16, M=6272, K=1152, N=4304, gate="silu", bias=True),
        # a training step on one image whose token count is no multiple of any tile, 0.7B class, no biases
        dict(name="mlp_train_ragged", op="mlp_train", dtype=BF16, M=1197, K=1280, N=5120, gate="gelu_tanh", bias=False),
        # the float configuration's block, trained on two small images
        dict(name="mlp_train_float", op="mlp_train", dtype=F32, M=512, K=256, N=1024, gate="gelu_tanh", bias=True),
        # gradient of the 0.6B-class QKV projection
        dict(name="linear_grad_qkv", op="linear_grad", dtype=BF16, M=6272, K=1152, N=3456, bias=True),
        # gradient of a projector layer (four merged tokens of the 0.7B class in, hand-off width out) for one small image
        dict(name="linear_grad_projector", op="linear_grad", dtype=BF16, M=391, K=5120, N=3584, bias=True),
        # one token of a decoder with shared key / value heads, far into a long sequence
        dict(name="rope_one_token", op="rope", dtype=BF16, T=1, heads=40, skip=8, dh=128, s0=16, s1=24, s2=24,
             layout="sections", start=100000, inverse=False),
        # queries and keys of a prompt with one large image, read out of the packed projection
        dict(name="rope_prompt", op="rope", dtype=F32, T=16206, heads=20, skip=4, dh=128, s0=24, s1=20, s2=20,
             layout="interleaved", start=1000, inverse=False),
        # 32 images of mixed sizes, 0.6B class: rotary embedding and head split in front of the attention
        dict(name="rope_split_images", op="rope_split", dtype=BF16, T=81628, heads=16, dh=72, s0=12, s1=12, s2=12,
             layout="blocks", start=0),
        # a training step's rotary part on a clip, 6B-class heads: forward and gradient
        dict(name="rope_split_train_clip", op="rope_split_train", dtype=BF16, T=12543, heads=25, dh=128, s0=16, s1=24,
             s2=24, layout="sections", start=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _widths(rng, dtype):
    """A configuration's widths, or a generic pair; bf16 widths are multiples of 8 as in every bf16 configuration."""
    if rng.random() < 0.5:
        return rng.choice([(256, 1024), (1152, 4304), (1280, 5120), (3200, 12800)])
    step = 8 if dtype == BF16 else 1
    K = max(step, _log(rng, 64, 2500) // step * step)
    N = max(step, _log(rng, 128, 8000) // step * step)
    return K, N


def draw(rng):
    op = rng.choice(["mlp", "mlp", "mlp_train", "mlp_train", "linear_grad", "rope", "rope_split", "rope_split_train"])
    dtype = F32 if rng.random() < 0.2 else BF16
    if op in ("mlp", "mlp_train", "linear_grad"):
        K, N = _widths(rng, dtype)
        M = _log(rng, 1, 16384) if op == "mlp" else _log(rng, 30, 7000)
        # work below the largest listed case's; float cases are small, as the float configuration is
        most = 4e9 if dtype == F32 else 5e11 if op == "mlp" else 1e11
        M = max(1, min(M, int(most / (K * N))))
        if op == "linear_grad":
            return dict(op=op, dtype=dtype, M=M, K=K, N=N, bias=rng.random() < 0.7)
        return dict(op=op, dtype=dtype, M=M, K=K, N=N, gate=rng.choice(GATES), bias=rng.random() < 0.7)
    heads = rng.randint(1, 32)
    dh = rng.choice([64, 72, 80, 96, 128])
    T = max(1, min(_log(rng, 1, 82000), int(9e7 / (heads * dh))))
    pairs = dh // 2
    s0 = rng.randint(1, pairs // 2)
    s1 = rng.randint(1, pairs - s0 - 1)
    case = dict(op=op, dtype=dtype, T=T, heads=heads, dh=dh, s0=s0, s1=s1, s2=pairs - s0 - s1,
                layout=rng.choice(LAYOUTS), start=rng.choice([0, 0, 1000, 100000]))
    if op == "rope":
        case.update(skip=rng.randint(0, 8), inverse=rng.random() < 0.5)
    return case


# --------------------------------------------------------------------------------------- inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == F32 else torch.bfloat16


def _positions(case, gen):
    """(time, row, column) of every token: clips of 8 frames of 28 x 28 patches one after the other, the whole shifted
    to where the sequence stands."""
    T = case["T"]
    shift = int(torch.randint(0, 64, (1,), generator=gen, device="cuda"))
    j = torch.arange(T, device="cuda") + 784 * shift
    local = j % (8 * 784)
    first = case["start"] + (j // (8 * 784)) * 40
    pos = torch.stack([first + local // 784, first + local % 784 // 28, first + local % 28])
    return pos.to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _dtype(case)

    def normal(std, *shape):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).to(dt)

    s = {"case": case}
    op = case["op"]
    if op in ("mlp", "mlp_train"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = normal(1.0, M, K)                           # behind a norm
        s["w_in"] = normal(0.7 / math.sqrt(K), 2 * N, K)     # gate rows, then up rows
        s["w_out"] = normal(0.7 / math.sqrt(N), K, N)
        s["b_in"] = normal(0.1, 2 * N) if case["bias"] else None
        s["b_out"] = normal(0.1, K) if case["bias"] else None
        if op == "mlp_train":
            s["dout"] = normal(0.05, M, K)
    elif op == "linear_grad":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = normal(1.0, M, K)
        s["w"] = normal(0.7 / math.sqrt(K), N, K)
        s["dout"] = normal(0.05, M, N)
    else:
        T, H, dh = case["T"], case["heads"], case["dh"]
        s["pos"] = _positions(case, gen)
        s["sections"] = (case["s0"], case["s1"], case["s2"])
        s["theta"] = 10000.0
        axis, freq, first, second = _plan(case)
        s["axis"] = torch.tensor(axis, device="cuda")
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["first"] = torch.tensor(first, device="cuda")
        s["second"] = torch.tensor(second, device="cuda")
        if op == "rope":
            # the heads to rotate lead a packed row; the others (values) are not touched
            s["x"] = normal(1.0, T, H + case["skip"], dh)[:, :H]
        else:
            s["qkv"] = normal(1.0, T, 3 * H * dh)
            s["q_scale"] = 1.4426950408889634 / math.sqrt(dh)
            if op == "rope_split_train":
                pad = (dh + 15) // 16 * 16
                s["grads"] = [normal(0.05, H, T, pad) for _ in range(3)]
    return s


def _plan(case):
    """Per rotation pair: axis, frequency, and the two head dimensions it turns."""
    sections = (case["s0"], case["s1"], case["s2"])
    pairs = sum(sections)
    axis, freq, first, second = [], [], [], []
    if case["layout"] == "blocks":
        base = 0
        for a, n in enumerate(sections):
            for f in range(n):
                axis.append(a)
                freq.append(10000.0 ** (-f / n))
                first.append(base + f)
                second.append(base + n + f)
            base += 2 * n
        return axis, freq, first, second
    if case["layout"] == "sections":
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    else:
        left = list(sections)
        while len(axis) < pairs:
            for a in range(3):
                if left[a] > 0:
                    left[a] -= 1
                    axis.append(a)
    return axis, [10000.0 ** (-i / pairs) for i in range(pairs)], list(range(pairs)), list(range(pairs, 2 * pairs))


# --------------------------------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2601_11590_b200 as epd

    c = s["case"]
    dt = epd.DTYPE_F32 if c["dtype"] == F32 else epd.DTYPE_BF16
    op = c["op"]
    if op == "mlp":
        return epd.op_gated_mlp(dt, s["x"], s["w_in"], s["b_in"], s["w_out"], s["b_out"], _gate(epd, c))
    if op == "mlp_train":
        out, hidden, pre = epd.op_gated_mlp(dt, s["x"], s["w_in"], s["b_in"], s["w_out"], s["b_out"], _gate(epd, c),
                                            save=True)
        g = epd.op_gated_mlp_backward(dt, s["dout"], s["x"], s["w_in"], s["w_out"], hidden, pre, _gate(epd, c),
                                      bias=c["bias"])
        return {"out": out, **g}
    if op == "linear_grad":
        return epd.op_linear_backward(dt, s["dout"], s["x"], s["w"], bias=c["bias"])
    layout = {"blocks": epd.ROPE_BLOCKS, "sections": epd.ROPE_SECTIONS, "interleaved": epd.ROPE_INTERLEAVED}[c["layout"]]
    if op == "rope":
        return epd.op_rope_axes(dt, s["x"], s["pos"], s["sections"], layout, s["theta"], inverse=c["inverse"])
    q, k, v = epd.op_rope_axes_split(dt, s["qkv"], s["pos"], c["heads"], c["dh"], s["sections"], layout, s["theta"],
                                     s["q_scale"])
    if op == "rope_split":
        return [q, k, v]
    d = epd.op_rope_axes_split_backward(dt, *s["grads"], s["pos"], c["dh"], s["sections"], layout, s["theta"],
                                        s["q_scale"])
    return [q, k, v, d]


def _gate(epd, c):
    return {"silu": epd.GATE_SILU, "gelu_tanh": epd.GATE_GELU_TANH, "gelu_erf": epd.GATE_GELU_ERF}[c["gate"]]


def _act(kind, g):
    """Activation and its derivative."""
    if kind == "silu":
        sg = torch.sigmoid(g)
        return g * sg, sg * (1 + g * (1 - sg))
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    phi = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def _plain(s):
    c, dt = s["case"], _dtype(s["case"])
    op = c["op"]
    if op in ("mlp", "mlp_train"):
        N = c["N"]
        x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
        pre = x @ w_in.t()
        if s["b_in"] is not None:
            pre += s["b_in"].float()
        g, u = pre[:, :N], pre[:, N:]
        act, slope = _act(c["gate"], g)
        hidden = act * u
        out = hidden @ w_out.t()
        if s["b_out"] is not None:
            out += s["b_out"].float()
        if op == "mlp":
            return out.to(dt)
        dout = s["dout"].float()
        da = dout @ w_out
        dpre = torch.cat([da * u * slope, da * act], 1)
        grads = {"out": out.to(dt), "dx": (dpre @ w_in).to(dt), "dw_in": (dpre.t() @ x).to(dt),
                 "dw_out": (dout.t() @ hidden).to(dt)}
        if c["bias"]:
            grads["db_in"], grads["db_out"] = dpre.sum(0).to(dt), dout.sum(0).to(dt)
        return grads
    if op == "linear_grad":
        x, w, dout = s["x"].float(), s["w"].float(), s["dout"].float()
        grads = {"dx": (dout @ w).to(dt), "dw": (dout.t() @ x).to(dt)}
        if c["bias"]:
            grads["db"] = dout.sum(0).to(dt)
        return grads
    # angles in 64 bits: a far position times a frequency loses its fraction of a turn in 32
    ang = s["pos"][s["axis"]].double().t() * s["freq"]
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    if op == "rope":
        return _turn(s, s["x"].float(), cos, -sin if c["inverse"] else sin).to(dt)
    T, H, dh = c["T"], c["heads"], c["dh"]
    q, k, v = s["qkv"].float().view(T, 3, H, dh).unbind(1)
    q, k = _turn(s, q, cos, sin) * s["q_scale"], _turn(s, k, cos, sin)
    pad = (dh + 15) // 16 * 16
    outs = []
    for n, t in enumerate((q, k, v)):
        o = torch.zeros(H, T, pad, dtype=dt, device="cuda")
        o[:, :, :dh] = t.transpose(0, 1)
        if n == 2 and pad > dh:
            o[:, :, dh] = 1
        outs.append(o)
    if op == "rope_split":
        return outs
    dq, dk, dv = (t[:, :, :dh].transpose(0, 1).float() for t in s["grads"])
    d = torch.stack([_turn(s, dq, cos, -sin) * s["q_scale"], _turn(s, dk, cos, -sin), dv], 1)
    return outs + [d.reshape(T, 3 * H * dh).to(dt)]


def _turn(s, x, cos, sin):
    a, b = x[..., s["first"]], x[..., s["second"]]
    y = x.clone()
    y[..., s["first"]] = a * cos - b * sin
    y[..., s["second"]] = b * cos + a * sin
    return y


# --------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    es = 4 if case["dtype"] == F32 else 2
    op = case["op"]
    if op in ("mlp", "mlp_train"):
        M, K, N = case["M"], case["K"], case["N"]
        weights = 3 * N * K + (2 * N + K if case["bias"] else 0)
        if op == "mlp":
            return {"bytes": es * (2 * M * K + weights), "flops": 6.0 * M * N * K}
        return {"bytes": es * (4 * M * K + 2 * weights), "flops": 18.0 * M * N * K}
    if op == "linear_grad":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": es * (2 * M * K + M * N + 2 * N * K + (N if case["bias"] else 0)), "flops": 4.0 * M * N * K}
    T, H, dh = case["T"], case["heads"], case["dh"]
    pad = (dh + 15) // 16 * 16
    if op == "rope":
        return {"bytes": 2 * es * T * H * dh + 12 * T, "flops": 3.0 * T * H * dh}
    split = {"bytes": es * 3 * T * H * (dh + pad) + 12 * T, "flops": 6.0 * T * H * dh}
    if op == "rope_split":
        return split
    return {"bytes": split["bytes"] + es * 6 * T * H * dh, "flops": 2 * split["flops"]}


# --------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    op = case["op"]
    if op in ("mlp", "mlp_train"):
        N = case["N"]
        x, wg, wu, wo = s["x"].to(D), s["w_in"][:N].to(D), s["w_in"][N:].to(D), s["w_out"].to(D)
        g, u = torch.mm(x, wg.T), torch.mm(x, wu.T)
        if case["bias"]:
            g, u = g + s["b_in"][:N].to(D), u + s["b_in"][N:].to(D)
        one = torch.ones((), dtype=D, device="cuda")
        if case["gate"] == "silu":
            e = torch.exp(-g)
            act = g / (one + e)
            slope = (one + e + g * e) / (one + e) ** 2
        elif case["gate"] == "gelu_tanh":
            z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
            act = g * (one + torch.tanh(z)) / 2
            slope = (one + torch.tanh(z)) / 2 + g / (2 * torch.cosh(z) ** 2) * math.sqrt(2 / math.pi) * (one + 0.134145 * g ** 2)
        else:
            cdf = torch.erfc(-g / math.sqrt(2)) / 2
            act = g * cdf
            slope = cdf + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
        a = act * u
        y = torch.mm(a, wo.T)
        if case["bias"]:
            y = y + s["b_out"].to(D)
        if op == "mlp":
            return y
        dy = s["dout"].to(D)
        da = torch.mm(dy, wo)
        dg, du = da * u * slope, da * act
        r = {"out": y, "dx": torch.mm(dg, wg) + torch.mm(du, wu), "dw_out": torch.mm(dy.T, a),
             "dw_in": torch.cat([torch.mm(dg.T, x), torch.mm(du.T, x)])}
        if case["bias"]:
            r["db_in"] = torch.cat([dg.sum(0), du.sum(0)])
            r["db_out"] = dy.sum(0)
        return r
    if op == "linear_grad":
        x, w, dy = s["x"].to(D), s["w"].to(D), s["dout"].to(D)
        r = {"dx": torch.mm(dy, w), "dw": torch.mm(dy.T, x)}
        if case["bias"]:
            r["db"] = dy.sum(0)
        return r
    # a pair as one complex number, turned by exp(i t)
    axis, freq, first, second = _plan(case)
    angle = torch.stack([s["pos"][a].to(D) * f for a, f in zip(axis, freq)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotate(x, t):
        z = torch.complex(x[..., first], x[..., second]) * t
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if op == "rope":
        return rotate(s["x"].to(D), turn.conj() if case["inverse"] else turn)
    T, H, dh = case["T"], case["heads"], case["dh"]
    pad = (dh + 15) // 16 * 16
    x = s["qkv"].to(D).reshape(T, 3, H, dh)
    outs = []
    for n in range(3):
        y = x[:, n] if n == 2 else rotate(x[:, n], turn) * (s["q_scale"] if n == 0 else 1.0)
        tail = torch.zeros(T, H, pad - dh, dtype=D, device="cuda")
        if n == 2 and pad > dh:
            tail[..., 0] = 1
        outs.append(torch.cat([y, tail], 2).permute(1, 0, 2))
    if op == "rope_split":
        return outs
    back = []
    for n, t in enumerate(s["grads"]):
        y = t.to(D)[..., :dh].permute(1, 0, 2)
        back.append(y if n == 2 else rotate(y, turn.conj()) * (s["q_scale"] if n == 0 else 1.0))
    return outs + [torch.stack(back, 1).reshape(T, -1)]
