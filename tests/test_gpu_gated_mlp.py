"""Gated feed-forward block, its gradient and the gradient of a linear layer against the definition in float64.

Tolerances (relative Frobenius error, worst row within the factor of tests/metrics.py).  Rounding to bf16 is off by at
most 2^-8 = 3.9e-3 of a value.
  one rounding (hidden, pre, dw_out from given bf16 inputs, ...)     4e-3
  two roundings in a row (out behind the rounded hidden; dx, dw_in, db_in behind the rounded gradient of pre):
  independent errors of at most 2^-8 each, sqrt(2) * 2^-8 = 5.6e-3    6e-3
  float: sums of up to K terms in float, error about sqrt(K) * 2^-24 of the result, K <= 6000: 4.6e-6;   1e-5
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2601_11590_b200 as epd
from tests.metrics import assert_parity

pytestmark = pytest.mark.gpu

F32, BF16 = epd.DTYPE_F32, epd.DTYPE_BF16
GATES = [epd.GATE_SILU, epd.GATE_GELU_TANH, epd.GATE_GELU_ERF]
ONE = {BF16: 4e-3, F32: 1e-5}
TWO = {BF16: 6e-3, F32: 1e-5}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2601_11590_b200 import build
    build.build_library()
    epd.load_library()


def act_and_slope(gate, g):
    if gate == epd.GATE_SILU:
        s = 1 / (1 + torch.exp(-g))
        return g * s, s + g * s * (1 - s)
    if gate == epd.GATE_GELU_TANH:
        c = np.sqrt(2 / np.pi)
        t = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    phi = 0.5 * torch.erfc(-g / np.sqrt(2))
    return g * phi, phi + g * torch.exp(-g * g / 2) / np.sqrt(2 * np.pi)


def f64(t):
    return None if t is None else t.detach().double()


def reference_forward(x, w_in, b_in, gate):
    N = w_in.shape[0] // 2
    pre = f64(x) @ f64(w_in).T
    if b_in is not None:
        pre = pre + f64(b_in)
    return pre, act_and_slope(gate, pre[:, :N])[0] * pre[:, N:]


def reference_backward(dout, x, w_in, w_out, hidden, pre, gate):
    """Gradients from the saved values as they stand (the operator's contract)."""
    N = w_in.shape[0] // 2
    dout, x, w_in, w_out, hidden, pre = map(f64, (dout, x, w_in, w_out, hidden, pre))
    act, slope = act_and_slope(gate, pre[:, :N])
    da = dout @ w_out
    dpre = torch.cat([da * pre[:, N:] * slope, da * act], 1)
    return {"dx": dpre @ w_in, "dw_in": dpre.T @ x, "db_in": dpre.sum(0), "dw_out": dout.T @ hidden, "db_out": dout.sum(0)}


class Draw:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt = torch.float32 if dtype == F32 else torch.bfloat16

    def __call__(self, std, *shape):
        return (torch.randn(*shape, generator=self.g, device="cuda") * std).to(self.dt)


def block(seed, dtype, M, N, K, D=None, bias=True):
    D = K if D is None else D
    n = Draw(seed, dtype)
    return dict(x=n(1.0, M, K), w_in=n(K ** -0.5, 2 * N, K), b_in=n(0.3, 2 * N) if bias else None,
                w_out=n(N ** -0.5, D, N), b_out=n(0.3, D) if bias else None, dout=n(0.1, M, D))


def parity(got, ref, tol, what):
    assert_parity(got.double().cpu().numpy(), ref.double().cpu().numpy(), tol, what)


def check_block(dtype, b, gate):
    out, hidden, pre = epd.op_gated_mlp(dtype, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], gate, save=True)
    pre_ref, hid_ref = reference_forward(b["x"], b["w_in"], b["b_in"], gate)
    out_ref = hid_ref @ f64(b["w_out"]).T
    if b["b_out"] is not None:
        out_ref = out_ref + f64(b["b_out"])
    parity(pre, pre_ref, ONE[dtype], "pre")
    parity(hidden, hid_ref, ONE[dtype], "hidden")
    parity(out, out_ref, TWO[dtype], "out")
    # without saving the projections, and as a single step: the same bits
    assert torch.equal(epd.op_gated_mlp(dtype, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], gate), out)
    assert torch.equal(epd.op_gated_linear(dtype, b["x"], b["w_in"], b["b_in"], gate), hidden)
    g = epd.op_gated_mlp_backward(dtype, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, gate,
                                  bias=b["b_in"] is not None)
    ref = reference_backward(b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, gate)
    for name in g:
        parity(g[name], ref[name], ONE[dtype] if name in ("dw_out", "db_out") else TWO[dtype], name)
    return out, hidden, pre, g


# token counts on both sides of every kernel's limit, and of its tiles
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 32, 33, 64, 65, 127, 129, 255, 257, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_over_token_counts(dtype, M):
    check_block(dtype, block(100 + M, dtype, M, 320, 192, bias=M % 2 == 1), GATES[M % 3])


@pytest.mark.parametrize("N,K,D", [
    (8, 8, 8),            # smaller than one tile in every direction
    (136, 72, 40),        # ragged in every direction, D != K
    (1080, 1152, 1152),   # several tiles
    (1152, 264, 4304),    # ragged last output tile
    (24, 5120, 16),       # long contraction, few columns
    (4304, 64, 64),       # short contraction
])
@pytest.mark.parametrize("M", [1, 5, 40, 300])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_over_widths(dtype, M, N, K, D):
    check_block(dtype, block(7, dtype, M, N, K, D), epd.GATE_SILU)


@pytest.mark.parametrize("N,K,D", [(7, 5, 3), (33, 100, 11), (1, 1, 1)])
@pytest.mark.parametrize("M", [1, 3, 130])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_odd_widths(dtype, M, N, K, D):
    """Widths that are no multiples of 8: the plain-FMA kernels in bf16."""
    b = block(8, dtype, M, N, K, D)
    out, hidden, pre = epd.op_gated_mlp(dtype, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_GELU_ERF,
                                        save=True)
    pre_ref, hid_ref = reference_forward(b["x"], b["w_in"], b["b_in"], epd.GATE_GELU_ERF)
    # element by element (a result may be a single number): 2^-8 of the value per rounding in bf16, and the terms' sum
    # of moduli times the number of additions times 2^-24 for the float sums
    def near(got, ref, moduli, terms, roundings):
        step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
        bound = roundings * step * ref.abs() + (terms + 8) * 2.0 ** -23 * moduli + 1e-30
        assert bool(((got.double() - ref).abs() <= bound).all())
    near(pre, pre_ref, f64(b["x"]).abs() @ f64(b["w_in"]).abs().T + 2, K, 1)
    out_from_saved = f64(hidden) @ f64(b["w_out"]).T + f64(b["b_out"])
    near(out, out_from_saved, f64(hidden).abs() @ f64(b["w_out"]).abs().T + 2, N, 1)
    parity(hidden, hid_ref, TWO[dtype], "hidden")
    g = epd.op_gated_mlp_backward(dtype, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_GELU_ERF)
    ref = reference_backward(b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_GELU_ERF)
    near(g["dw_out"], ref["dw_out"], f64(b["dout"]).abs().T @ f64(hidden).abs(), M, 1)
    near(g["db_out"], ref["db_out"], f64(b["dout"]).abs().sum(0), M, 1)
    # behind the rounded gradient of pre every term carries its own 2^-8
    act, slope = act_and_slope(epd.GATE_GELU_ERF, f64(pre)[:, :N])
    da = f64(b["dout"]) @ f64(b["w_out"])
    da_mod = f64(b["dout"]).abs() @ f64(b["w_out"]).abs()
    mod = torch.cat([da_mod * (f64(pre)[:, N:] * slope).abs(), da_mod * act.abs()], 1)
    dmod = torch.cat([(da * f64(pre)[:, N:] * slope).abs(), (da * act).abs()], 1)
    step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    for name, lead, last in (("dx", lambda t: t, f64(b["w_in"])), ("dw_in", lambda t: t.T, f64(b["x"]))):
        r = ref[name]
        term = lead(dmod) @ last.abs()
        total = lead(mod) @ last.abs()
        bound = step * (r.abs() + 1.01 * term) + (D + 2 * N + M + 16) * 2.0 ** -22 * total + 1e-30
        assert bool(((g[name].double() - r).abs() <= bound).all()), name


@pytest.mark.parametrize("M,N,K,D", [
    (2000, 520, 264, 264),     # several tiles, whole contraction per tile
    (671, 1031, 391, 397),     # odd in every direction
    (64, 4304, 1024, 512),     # few rows: contraction shared among pairs
    (193, 1301, 1103, 77),     # just over three blocks of rows, few output columns
    (4099, 200, 352, 360),     # many rows, narrow
    (257, 1152, 1152, 1152),
])
@pytest.mark.parametrize("gate", GATES)
def test_large_float_block_on_the_tensor_cores(M, N, K, D, gate):
    """A float as three bf16 parts, six products of parts: what is left out is 2^-26 of a product, the float sums are those of
    the plain path, so the same 1e-5 holds."""
    assert epd.load_library().epd_gated_mlp_workspace_bytes(F32, M, N, K, D) > 0
    b = block(M, F32, M, N, K, D, bias=gate != epd.GATE_SILU)
    out, hidden, pre, g = check_block(F32, b, gate)
    # the plain-FMA path of the same call: no workspace.  Two results within 1e-5 of the definition each.
    lib = epd.load_library()
    out2, hid2 = torch.empty_like(out), torch.empty_like(hidden)
    p = lambda t: None if t is None else t.data_ptr()   # noqa: E731
    assert lib.epd_op_gated_mlp(F32, p(b["x"]), K, p(b["w_in"]), K, p(b["b_in"]), p(b["w_out"]), N, p(b["b_out"]), p(hid2), N, None,
                                0, p(out2), D, None, 0, M, N, K, D, gate, 0, torch.cuda.current_stream().cuda_stream) == 0
    parity(out2, out.double(), 2e-5, "the two paths")
    n = Draw(M, F32)
    lin = epd.op_linear_backward(F32, n(1.0, M, N), b["x"], b["w_in"][:N])
    parity(lin["dw"], f64(Draw(M, F32)(1.0, M, N)).T @ f64(b["x"]), ONE[F32], "dw")
    parity(lin["dx"], f64(Draw(M, F32)(1.0, M, N)) @ f64(b["w_in"][:N]), ONE[F32], "dx")


def test_float_parts_over_the_whole_range():
    """Values over the whole range of float, the largest ones among them: every operand value is the exact sum of its parts (24
    bits, above 2^-110), products and sums stay finite.  A diagonal weight leaves one product per result: relative error
    2^-24 of the final rounding and 2^-25 of the parts left out, element by element."""
    M = K = 1024
    x = torch.zeros(M, K, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    e = torch.randint(-100, 127, (M, K), generator=g, device="cuda").double()
    x = ((1 + torch.rand(M, K, generator=g, device="cuda", dtype=torch.float64)) * 2.0 ** e).float()
    x[0, :8] = torch.tensor([3.4028235e38, -3.4028235e38, 3.39e38, 3.3961775e38, 0.0, -0.0, 1.0, 1e-30], device="cuda")
    eye = torch.eye(K, device="cuda") * 0.75
    dw = epd.op_linear_backward(F32, x, torch.eye(M, device="cuda"), eye, bias=False)
    assert torch.allclose(dw["dx"].double(), x.double() * 0.75, rtol=2.0 ** -22, atol=0)
    assert torch.allclose(dw["dw"].double(), x.double().T, rtol=2.0 ** -22, atol=0)


def test_block_at_the_encoder_widths():
    for M, N, K, gate in ((777, 4304, 1152, epd.GATE_GELU_TANH), (30, 12800, 3200, epd.GATE_GELU_ERF),
                          (1, 12800, 3200, epd.GATE_SILU)):
        check_block(BF16, block(M, BF16, M, N, K), gate)


@pytest.mark.parametrize("M,offset", [(1, 0), (1, 8), (20, 0), (20, 8), (300, 8), (20, 1), (300, 3)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_operands_and_untouched_neighbours(dtype, M, offset):
    """Every matrix a window of a larger one filled with NaN: nothing outside is read into a result or written.  Offsets
    that are no multiples of 8 leave the tensor-core kernels."""
    N, K, D = 88, 72, 56
    dt = torch.float32 if dtype == F32 else torch.bfloat16
    b = block(3, dtype, M, N, K, D)

    def window(t, rows, cols):
        big = torch.full((rows + 3, cols + 40), float("nan"), dtype=dt, device="cuda")
        w = big[1:1 + rows, offset:offset + cols]
        if t is not None:
            w.copy_(t)
        return big, w
    ins = {n: window(b[n], *b[n].shape)[1] for n in ("x", "w_in", "w_out", "dout")}
    outs = {n: window(None, *s) for n, s in (("out", (M, D)), ("hidden", (M, N)), ("pre", (M, 2 * N)))}
    epd.op_gated_mlp(dtype, ins["x"], ins["w_in"], b["b_in"], ins["w_out"], b["b_out"], epd.GATE_SILU,
                     out=outs["out"][1], hidden=outs["hidden"][1], pre=outs["pre"][1])
    pre_ref, hid_ref = reference_forward(b["x"], b["w_in"], b["b_in"], epd.GATE_SILU)
    parity(outs["pre"][1], pre_ref, ONE[dtype], "pre")
    parity(outs["hidden"][1], hid_ref, ONE[dtype], "hidden")
    parity(outs["out"][1], hid_ref @ f64(b["w_out"]).T + f64(b["b_out"]), TWO[dtype], "out")
    g = epd.op_gated_mlp_backward(dtype, ins["dout"], ins["x"], ins["w_in"], ins["w_out"], outs["hidden"][1],
                                  outs["pre"][1], epd.GATE_SILU)
    ref = reference_backward(b["dout"], b["x"], b["w_in"], b["w_out"], outs["hidden"][1], outs["pre"][1], epd.GATE_SILU)
    for name in g:
        parity(g[name], ref[name], TWO[dtype], name)
    for n, (big, w) in outs.items():
        w.fill_(float("nan"))
        assert bool(torch.isnan(big).all()), n


@pytest.mark.parametrize("M", [1, 3, 8, 11, 16, 17])
def test_residual_update_of_a_float_block(M):
    """Widths that end inside a lane's stretch of the contraction and inside a warp's rows; gaps behind the rows."""
    N, K, D = 1001, 204, 333
    b = block(5, F32, M, N + 3, K, D)
    w_in = torch.cat([b["w_in"][:N], b["w_in"][-N:]])
    big = torch.full((D, N + 15), float("nan"), device="cuda")
    big[:, :N] = b["w_out"][:, :N]
    w_out, b_in = big[:, :N], b["b_in"][:2 * N].contiguous()
    pre_ref, hid_ref = reference_forward(b["x"], w_in, b_in, epd.GATE_GELU_ERF)
    hid = torch.full((M, N + 7), float("nan"), device="cuda")[:, :N]
    out = torch.randn(M, D, device="cuda")
    ref = out.double() + hid_ref @ f64(w_out).T + f64(b["b_out"])
    pre = torch.empty(M, 2 * N, device="cuda")
    epd.op_gated_mlp(F32, b["x"], w_in, b_in, w_out, b["b_out"], epd.GATE_GELU_ERF, out=out, hidden=hid, pre=pre,
                     flags=epd.LINEAR_ACCUMULATE)
    parity(pre, pre_ref, ONE[F32], "pre")
    parity(hid, hid_ref, ONE[F32], "hidden")
    parity(out, ref, TWO[F32], "residual")


@pytest.mark.parametrize("D", [2371, 2500, 3200, 3600, 4800])      # groups of 24, 32 and 16 columns; a last group cut short
@pytest.mark.parametrize("M", [9, 16, 25])
def test_few_tokens_wide_output(M, D):
    b = block(6, BF16, M, 264, 72, D)
    _, hid_ref = reference_forward(b["x"], b["w_in"], b["b_in"], epd.GATE_SILU)
    ref = hid_ref @ f64(b["w_out"]).T + f64(b["b_out"])
    args = (BF16, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_SILU)
    big = torch.full((M + 1, D + 5), float("nan"), dtype=torch.bfloat16, device="cuda")
    parity(epd.op_gated_mlp(*args, out=big[:M, :D]), ref, TWO[BF16], "out")
    big[:M, :D] = float("nan")
    assert bool(torch.isnan(big).all())
    x = torch.randn(M, D, device="cuda")
    want = ref + x.double()
    epd.op_gated_mlp(*args, out=x, flags=epd.LINEAR_ACCUMULATE)
    parity(x, want, ONE[BF16], "residual")


@pytest.mark.parametrize("dtype,M,N,K", [(BF16, 3000, 1152, 1152), (BF16, 500, 136, 72), (F32, 900, 100, 60),
                                         (F32, 700, 640, 640), (BF16, 300, 33, 15)])
def test_gradients_follow_what_is_in_front_of_them(dtype, M, N, K):
    """The bias sums run beside the products and must still see what the stream did in front of the call, whoever wrote it: a copy,
    or another step of this library, whose successors may start early."""
    n = Draw(77, dtype)
    x, w = n(1.0, M, K), n(K ** -0.5, N, K)
    sources = [n(1.0, M, N) for _ in range(6)]
    want = [epd.op_linear_backward(dtype, s, x, w) for s in sources]
    torch.cuda.synchronize()
    ws = torch.empty(epd.load_library().epd_linear_backward_workspace_bytes(dtype, M, N, K), dtype=torch.uint8, device="cuda")
    pos = torch.zeros(1, M * N, dtype=torch.int32, device="cuda")
    dout = torch.empty_like(sources[0])
    got = []
    for rep in range(3):
        for i, s in enumerate(sources):
            if (i + rep) % 2:
                dout.copy_(s)
            else:      # position 0 turns nothing: a copy by one of this library's kernels
                epd.op_rope_axes(dtype, s.view(M * N, 1, 1), pos, (0,), epd.ROPE_BLOCKS, 10000.0, out=dout.view(M * N, 1, 1))
            got.append(epd.op_linear_backward(dtype, dout, x, w, workspace=ws))
    for i, g in enumerate(got):
        for name in g:
            assert torch.equal(g[name], want[i % len(sources)][name]), (i, name)


@pytest.mark.parametrize("M", [1, 12, 200])
def test_residual_update_and_float_output(M):
    b = block(4, BF16, M, 320, 192)
    _, hid_ref = reference_forward(b["x"], b["w_in"], b["b_in"], epd.GATE_GELU_TANH)
    ref = hid_ref @ f64(b["w_out"]).T + f64(b["b_out"])
    r0 = torch.randn(M, 192, device="cuda")
    args = (BF16, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_GELU_TANH)
    # one rounding (hidden) behind float sums
    parity(epd.op_gated_mlp(*args, flags=epd.LINEAR_OUT_F32), ref, ONE[BF16], "float out")
    x = r0.clone()
    epd.op_gated_mlp(*args, out=x, flags=epd.LINEAR_ACCUMULATE)
    parity(x, ref + r0.double(), ONE[BF16], "residual")
    with pytest.raises(ValueError):
        epd.op_gated_mlp(*args, flags=epd.LINEAR_ACCUMULATE)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M", [3, 150])
def test_large_and_infinite_gates(dtype, M):
    """Gates far out on both sides: the activation and its slope reach their limits, nothing overflows to NaN."""
    N, K = 64, 64
    x = torch.zeros(M, K, device="cuda")
    x[:, 0] = 1
    w = torch.zeros(2 * N, K, device="cuda")
    w[:N, 0] = torch.tensor([-1e37, -1e20, -1e5, -200.0, -30.0, -1.0, -0.0, 0.0, 1.0, 30.0, 200.0, 1e5, 1e20, 1e37, 8.0, -8.0],
                            device="cuda").repeat(N // 16)
    w[N:, 0] = 0.5
    n = Draw(5, dtype)
    dt = n.dt
    x, w = x.to(dt), w.to(dt)
    w_out, dout = torch.eye(N, device="cuda").to(dt), n(1.0, M, N)
    for gate in GATES:
        _, hidden, pre = epd.op_gated_mlp(dtype, x, w, None, w_out, None, gate, save=True)
        hid_ref = reference_forward(x, w, None, gate)[1]
        assert bool(torch.isfinite(hidden.float()).all())
        assert torch.allclose(hidden.double(), hid_ref, rtol=2.0 ** -7, atol=1e-6)
        g = epd.op_gated_mlp_backward(dtype, dout, x, w, w_out, hidden, pre, gate, bias=False, need_dw=False)
        # dx[:, 0] = sum of dg * w_gate + du * w_up: check the gradient of pre itself through an identity in place of w_in
        eye = torch.eye(2 * N, device="cuda").to(dt)
        xe = torch.zeros(M, 2 * N, device="cuda", dtype=dt)
        d = epd.op_gated_mlp_backward(dtype, dout, xe, eye, w_out, hidden, pre, gate, bias=False, need_dw=False)["dx"]
        p = pre.double()
        act, slope = act_and_slope(gate, p[:, :N].clamp(-1e3, 1e3))
        act = torch.where(p[:, :N] > 1e3, p[:, :N], act)
        ref = torch.cat([dout.double() * p[:, N:] * slope, dout.double() * act], 1)
        assert torch.allclose(d.double(), ref, rtol=2.0 ** -6, atol=1e-6)
        assert "dw_in" not in g and "db_in" not in g


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M", [6, 140])
def test_rows_do_not_mix(dtype, M):
    """A row of NaN or infinities changes its own row of hidden, out and dx, and no other."""
    b = block(11, dtype, M, 96, 64)
    args = (b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_SILU)
    out, hidden, pre = epd.op_gated_mlp(dtype, b["x"], *args, save=True)
    dx = epd.op_gated_mlp_backward(dtype, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_SILU)["dx"]
    x2, d2 = b["x"].clone(), b["dout"].clone()
    x2[M // 2] = float("nan")
    d2[M // 3] = float("inf")
    out2, hidden2, pre2 = epd.op_gated_mlp(dtype, x2, *args, save=True)
    dx2 = epd.op_gated_mlp_backward(dtype, d2, x2, b["w_in"], b["w_out"], hidden2, pre2, epd.GATE_SILU)["dx"]
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[M // 2] = False
    assert torch.equal(out[keep], out2[keep]) and torch.equal(hidden[keep], hidden2[keep])
    assert bool(torch.isnan(out2[M // 2].float()).all())
    keep[M // 3] = False
    assert torch.equal(dx[keep], dx2[keep])


def test_gradient_against_differences():
    """Directional derivatives of the 64-bit definition by central differences against the float kernel's gradient: the
    kernel is off by at most 1e-5 of the gradient's norm, times the direction's norm (Cauchy-Schwarz); the quotient's own
    error is step^2 = 1e-10 of the third derivative and 1e-9 of rounding."""
    M, N, K = 37, 48, 40
    for gate in GATES:
        b = block(21, F32, M, N, K)
        _, hidden, pre = epd.op_gated_mlp(F32, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], gate, save=True)
        g = epd.op_gated_mlp_backward(F32, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, gate)
        names = {"x": "dx", "w_in": "dw_in", "b_in": "db_in", "w_out": "dw_out", "b_out": "db_out"}

        def loss(v):
            h = reference_forward(v["x"], v["w_in"], v["b_in"], gate)[1]
            return float(((h @ f64(v["w_out"]).T + f64(v["b_out"])) * f64(b["dout"])).sum())
        for i, (name, grad) in enumerate(names.items()):
            dirn = torch.randn(b[name].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda()
            up, down = dict(b), dict(b)
            up[name], down[name] = f64(b[name]) + 1e-5 * dirn, f64(b[name]) - 1e-5 * dirn
            quotient = (loss(up) - loss(down)) / 2e-5
            along = float((g[grad].double() * dirn).sum())
            scale = float((g[grad].double() ** 2).sum() ** 0.5)
            assert abs(quotient - along) <= 1e-5 * scale * float(dirn.norm()), (gate, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K", [(1, 8, 8), (130, 136, 72), (391, 520, 264), (600, 24, 1032), (65, 3456, 128)])
def test_linear_backward(dtype, M, N, K):
    n = Draw(31, dtype)
    x, w, dout = n(1.0, M, K), n(K ** -0.5, N, K), n(0.1, M, N)
    g = epd.op_linear_backward(dtype, dout, x, w)
    parity(g["dx"], f64(dout) @ f64(w), ONE[dtype], "dx")
    parity(g["dw"], f64(dout).T @ f64(x), ONE[dtype], "dw")
    parity(g["db"], f64(dout).sum(0), ONE[dtype], "db")
    only = epd.op_linear_backward(dtype, dout, x, w, bias=False, need_dw=False)
    assert set(only) == {"dx"} and torch.equal(only["dx"], g["dx"])
    only = epd.op_linear_backward(dtype, dout, x, w, bias=False, need_dx=False)
    assert set(only) == {"dw"} and torch.equal(only["dw"], g["dw"])


def test_many_rows_in_the_gradient():
    """Row counts beyond one block of the column sums, and a contraction over many rows."""
    check_block(BF16, block(41, BF16, 5000, 136, 72), epd.GATE_SILU)
    check_block(F32, block(42, F32, 3001, 40, 24), epd.GATE_GELU_ERF)


def test_no_rows():
    for dtype in (BF16, F32):
        b = block(51, dtype, 0, 16, 24)
        out, hidden, pre = epd.op_gated_mlp(dtype, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], 0, save=True)
        assert out.shape == (0, 24)
        g = epd.op_gated_mlp_backward(dtype, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, 0)
        for name in ("dw_in", "db_in", "dw_out", "db_out"):
            assert not bool(g[name].any()), name
        g = epd.op_linear_backward(dtype, b["dout"], b["x"], torch.ones(24, 24, device="cuda").to(b["x"].dtype))
        assert not bool(g["dw"].any()) and not bool(g["db"].any())


@pytest.mark.parametrize("M", [1, 24, 333])
def test_repeated_calls_streams_and_graphs_give_the_same_bits(M):
    b = block(61, BF16, M, 320, 192)
    args = (BF16, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_SILU)

    def step():
        out, hidden, pre = epd.op_gated_mlp(*args, save=True)
        return [out] + list(epd.op_gated_mlp_backward(BF16, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre,
                                                      epd.GATE_SILU).values())
    want = step()
    assert all(torch.equal(p, q) for p, q in zip(want, step()))
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for s in (s1, s2, s1, s2):
        with torch.cuda.stream(s):
            got.append(step())
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(p, q) for p, q in zip(want, r))
    graph = torch.cuda.CUDAGraph()
    x0 = b["x"].clone()
    with torch.cuda.graph(graph):
        captured = step()
    b["x"].zero_()
    graph.replay()
    b["x"].copy_(x0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, captured))


@pytest.mark.parametrize("dtype,M,N,K", [(BF16, 2500, 1152, 1024), (BF16, 90, 33, 20), (F32, 300, 256, 128), (F32, 700, 640, 640)])
def test_captured_training_steps_back_to_back(dtype, M, N, K):
    """A graph with a copy in front of a training step, replayed over other inputs without a pause: launches that run beside one
    another in the graph see what it copied."""
    sets = [block(80 + i, dtype, M, N, K) for i in range(3)]
    b = {k: v.clone() for k, v in sets[0].items()}

    def step():
        out, hidden, pre = epd.op_gated_mlp(dtype, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_GELU_TANH, save=True)
        g = epd.op_gated_mlp_backward(dtype, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_GELU_TANH)
        return [out] + list(g.values())
    want = []
    for s in sets:
        for k in b:
            b[k].copy_(s[k])
        want.append(step())
    source = {k: v.clone() for k, v in sets[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for k in b:
            b[k].copy_(source[k])
        captured = step()
    got = []
    for i in (1, 2, 0, 2, 1):
        for k in b:
            source[k].copy_(sets[i][k])
        graph.replay()
        got.append((i, [t.clone() for t in captured]))
    torch.cuda.synchronize()
    for i, r in got:
        assert all(torch.equal(p, q) for p, q in zip(want[i], r)), i


def test_limited_sms_change_no_result():
    b = block(71, BF16, 700, 520, 264)
    want = check_block(BF16, b, epd.GATE_SILU)
    epd.set_sm_limit(20)
    try:
        got = check_block(BF16, b, epd.GATE_SILU)
    finally:
        epd.set_sm_limit(0)
    for p, q in zip(want[:3], got[:3]):
        assert torch.equal(p, q)
    assert all(torch.equal(want[3][n], got[3][n]) for n in want[3])


@pytest.mark.parametrize("M,N,K", [(700, 520, 1032), (40, 264, 2056)])   # whole tiles; tiles shared in clusters
def test_expired_waits_end_and_leave_the_device_usable(M, N, K):
    """With a wait limit of 1000 cycles ordinary waits (a first tile on its way from memory) run out: the kernels drain and
    return, their results are undefined.  With the ordinary limit the same calls give the same bits as before."""
    b = block(91, BF16, M, N, K)

    def step():
        out, hidden, pre = epd.op_gated_mlp(BF16, b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"], epd.GATE_SILU, save=True)
        g = epd.op_gated_mlp_backward(BF16, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_SILU)
        torch.cuda.synchronize()
        return [out, hidden, pre] + list(g.values())
    want = step()
    epd.set_wait_limit(1000)
    try:
        step()
    finally:
        epd.set_wait_limit(0)
    assert all(torch.equal(p, q) for p, q in zip(want, step()))


def test_binding_refuses_mismatched_tensors():
    b = block(81, BF16, 4, 16, 24)
    ok = (b["x"], b["w_in"], b["b_in"], b["w_out"], b["b_out"])
    for i, bad in ((0, b["x"].float()), (0, b["x"].cpu()), (1, b["w_in"][:-1]), (2, b["b_in"][:3]), (3, b["w_out"].t()),
                   (0, b["x"].t().contiguous().t())):
        a = list(ok)
        a[i] = bad
        with pytest.raises((ValueError, epd.EpdError)):
            epd.op_gated_mlp(BF16, *a, epd.GATE_SILU)
    with pytest.raises(epd.EpdError) as e:
        epd.op_gated_mlp(BF16, *ok, 3)
    assert e.value.status == epd.EPD_EINVAL
    _, hidden, pre = epd.op_gated_mlp(BF16, *ok, epd.GATE_SILU, save=True)
    with pytest.raises(epd.EpdError) as e:
        epd.op_gated_mlp_backward(BF16, b["dout"], b["x"], b["w_in"], b["w_out"], hidden, pre, epd.GATE_SILU,
                                  workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == epd.EPD_ENOMEM
