"""Rotary embedding with several axes against complex multiplication in float64.

Tolerances: bf16 one rounding, at most 2^-8 of a value: 4e-3 (relative Frobenius error).  Float: the fraction of a turn
is rounded to float (2^-25 of a turn, 1.9e-7 rad), sine and cosine to 2^-23, three roundings of products and sums at
2^-24 each: below 1e-6.
"""
import numpy as np
import pytest
import torch

import paper_2601_11590_b200 as epd
from tests.metrics import assert_parity

pytestmark = pytest.mark.gpu

F32, BF16 = epd.DTYPE_F32, epd.DTYPE_BF16
TOL = {BF16: 4e-3, F32: 1e-6}
THETA = 10000.0


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2601_11590_b200 import build
    build.build_library()
    epd.load_library()


def plan(sections, layout, theta):
    R = sum(sections)
    if layout == epd.ROPE_BLOCKS:
        rows, base = [], 0
        for a, n in enumerate(sections):
            rows += [(a, theta ** (-f / n), base + f, base + n + f) for f in range(n)]
            base += 2 * n
        return rows
    if layout == epd.ROPE_SECTIONS:
        axes = [a for a, n in enumerate(sections) for _ in range(n)]
    else:
        axes, left = [], list(sections)
        while sum(left):
            for a in range(len(left)):
                if left[a]:
                    left[a] -= 1
                    axes.append(a)
    return [(a, theta ** (-i / R), i, i + R) for i, a in enumerate(axes)]


def rotate(x, pos, sections, layout, theta=THETA, sign=1.0):
    """x [T, heads, dh] float64."""
    y = x.clone()
    for a, w, i, j in plan(sections, layout, theta):
        ang = (pos[a].double() * w)[:, None] * sign
        z = torch.complex(x[:, :, i], x[:, :, j]) * torch.polar(torch.ones_like(ang), ang)
        y[:, :, i], y[:, :, j] = z.real, z.imag
    return y


def normal(seed, dtype, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(torch.float32 if dtype == F32 else torch.bfloat16)


def positions(seed, axes, T, lo=0, hi=2000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(lo, hi, (axes, T), generator=g, device="cuda", dtype=torch.int32)


def parity(got, ref, tol, what=""):
    assert_parity(got.double().cpu().numpy(), ref.double().cpu().numpy(), tol, what)


LAYOUTS = [epd.ROPE_BLOCKS, epd.ROPE_SECTIONS, epd.ROPE_INTERLEAVED]
HEADS = [
    # (head_dim, sections): widths that leave 8-, 4-, 2- and 1-element vectors; partial rotation; one to four axes
    (128, (16, 24, 24)), (128, (24, 20, 20)), (72, (12, 12, 12)), (72, (18, 18)), (64, (11, 13, 8)), (80, (40,)),
    (96, (8, 8, 8)), (128, (7, 0, 9, 30)), (40, (0, 0, 3)), (6, (1, 1, 1)), (5, (2,)), (16, (0, 0)),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dh,sections", HEADS)
def test_rotation(dtype, layout, dh, sections):
    for T, heads in ((1, 1), (1, 40), (3, 5), (300, 3), (2501, 2)):
        x, pos = normal(T, dtype, T, heads, dh), positions(T, len(sections), T)
        ref = rotate(x.double(), pos, sections, layout)
        y = epd.op_rope_axes(dtype, x, pos, sections, layout, THETA)
        parity(y, ref, TOL[dtype], "forward")
        y = epd.op_rope_axes(dtype, x, pos, sections, layout, THETA, scale=0.37, inverse=True)
        parity(y, rotate(x.double(), pos, sections, layout, sign=-1.0) * 0.37, TOL[dtype], "inverse")
        # in place
        z = x.clone()
        assert epd.op_rope_axes(dtype, z, pos, sections, layout, THETA, scale=0.37, inverse=True, out=z) is z
        assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_and_negative_positions(dtype):
    """Angles formed in double precision: at 2^31 positions a turn count of 3.4e8 is known to 2^-53 of itself on either
    side, 2.4e-7 rad each, on top of the float path's 1e-6."""
    dh, sections = 64, (10, 11, 11)
    vals = torch.tensor([0, 1, -1, 99999, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32)
    T = vals.numel()
    pos = torch.stack([vals, vals.flip(0), vals.roll(3)]).cuda()
    x = normal(1, dtype, T, 4, dh)
    for layout in LAYOUTS:
        y = epd.op_rope_axes(dtype, x, pos, sections, layout, THETA)
        parity(y, rotate(x.double(), pos, sections, layout), TOL[dtype] + 1e-6)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", [0, 8, 4, 1])
def test_strided_views(dtype, offset):
    """Heads of a packed row (fewer key heads than query heads), head-major input, gaps between tokens; nothing outside
    the view is written."""
    T, heads, skip, dh, sections = 45, 6, 3, 64, (8, 12, 12)
    dt = torch.float32 if dtype == F32 else torch.bfloat16
    pos_all = positions(9, 3, T + 7)
    pos = pos_all[:, 3:3 + T]
    row = torch.full((T, (heads + skip) * dh + 24), float("nan"), dtype=dt, device="cuda")
    view = row[:, offset:offset + heads * dh].unflatten(1, (heads, dh))
    x = normal(2, dtype, T, heads, dh)
    view.copy_(x)
    for layout in LAYOUTS:
        ref = rotate(x.double(), pos, sections, layout)
        parity(epd.op_rope_axes(dtype, view, pos, sections, layout, THETA), ref, TOL[dtype], "packed row")
        major = x.transpose(0, 1).contiguous().transpose(0, 1)
        parity(epd.op_rope_axes(dtype, major, pos, sections, layout, THETA), ref, TOL[dtype], "head-major")
        big = torch.full_like(row, float("nan"))
        into = big[:, offset:offset + heads * dh].unflatten(1, (heads, dh))
        epd.op_rope_axes(dtype, view, pos, sections, layout, THETA, out=into)
        parity(into, ref, TOL[dtype], "into a packed row")
        into.fill_(float("nan"))
        assert bool(torch.isnan(big).all())


@pytest.mark.parametrize("dtype,heads,dh,sections", [(BF16, 20, 128, (16, 24, 24)), (F32, 20, 72, (11, 7, 12)),
                                                     (BF16, 9, 96, (6, 5, 3)), (F32, 124, 128, (20, 20)),
                                                     (BF16, 16, 72, (12, 12, 12)), (F32, 3, 64, (0, 0))])
def test_many_tokens_in_every_arrangement(dtype, heads, dh, sections):
    """Enough tokens for whole blocks of them: rows back to back, gaps behind tokens or heads, head-major rows, on either side;
    a last block with fewer tokens; NaN in dimensions that do not turn stays where it is."""
    T = 1333
    dt = torch.float32 if dtype == F32 else torch.bfloat16
    pos = positions(5, len(sections), T)
    x = normal(6, dtype, T, heads, dh)
    R = sum(sections)
    if 2 * R < dh:
        x[1::3, :, 2 * R] = float("nan")

    def empty(kind):
        if kind == "packed":
            return torch.full((T, heads, dh), float("nan"), dtype=dt, device="cuda"), None
        if kind == "token gap":
            big = torch.full((T, heads * dh + 24), 7.0, dtype=dt, device="cuda")
            return big[:, :heads * dh].unflatten(1, (heads, dh)), big[:, heads * dh:]
        if kind == "head gap":
            big = torch.full((T, heads, dh + 8), 7.0, dtype=dt, device="cuda")
            return big[:, :, :dh], big[:, :, dh:]
        big = torch.full((heads, T, dh), 7.0, dtype=dt, device="cuda")
        return big.transpose(0, 1), None
    for n, layout in enumerate(LAYOUTS):
        ref = rotate(x.double(), pos, sections, layout) * 0.37
        known = torch.isfinite(ref)
        for kind in ("packed", "token gap", "head gap", "head-major"):
            src, _ = empty(kind)
            src.copy_(x)
            for into in ("packed", "token gap", "head gap", "head-major"):
                if n and into != kind:
                    continue
                out, gap = empty(into)
                epd.op_rope_axes(dtype, src, pos, sections, layout, THETA, scale=0.37, out=out)
                parity(torch.where(known, out, torch.zeros_like(out)), torch.where(known, ref, torch.zeros_like(ref)), TOL[dtype],
                       f"{kind} -> {into}")
                assert torch.equal(torch.isnan(out), torch.isnan(ref))
                assert gap is None or bool((gap == 7.0).all())
            epd.op_rope_axes(dtype, src, pos, sections, layout, THETA, scale=0.37, out=src)     # in place
            assert torch.equal(src[known], epd.op_rope_axes(dtype, x, pos, sections, layout, THETA, scale=0.37)[known])


def split_reference(qkv, pos, heads, dh, sections, layout, q_scale):
    T = qkv.shape[0]
    x = qkv.double().view(T, 3, heads, dh)
    dhp = epd.padded_head_dim(dh)
    outs = []
    for n in range(3):
        y = x[:, n] if n == 2 else rotate(x[:, n], pos, sections, layout) * (q_scale if n == 0 else 1.0)
        o = torch.zeros(heads, T, dhp, dtype=torch.float64, device="cuda")
        o[:, :, :dh] = y.transpose(0, 1)
        if n == 2 and dhp > dh:
            o[:, :, dh] = 1
        outs.append(o)
    return outs


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads,dh,sections", [(16, 72, (12, 12, 12)), (2, 128, (16, 24, 24)), (3, 64, (11, 13, 8)),
                                               (1, 80, (10, 10)), (5, 20, (3, 4, 2)), (2, 7, (1, 1))])
def test_split_and_its_gradient(dtype, layout, heads, dh, sections):
    q_scale = 1.4426950408889634 / np.sqrt(dh)
    for T, ldpad in ((1, 0), (9, 0), (300, 16), (1217, 3)):
        pos = positions(T, len(sections), T)
        big = torch.full((T, 3 * heads * dh + ldpad), float("nan"), device="cuda").to(
            torch.float32 if dtype == F32 else torch.bfloat16)
        big[:, :3 * heads * dh] = normal(5, dtype, T, 3 * heads * dh)
        qkv = big[:, :3 * heads * dh]
        got = epd.op_rope_axes_split(dtype, qkv, pos, heads, dh, sections, layout, THETA, q_scale)
        for name, g, r in zip("qkv", got, split_reference(qkv, pos, heads, dh, sections, layout, q_scale)):
            parity(g, r, TOL[dtype], name)
        assert torch.equal(got[2][:, :, :dh].transpose(0, 1).reshape(T, -1), qkv[:, 2 * heads * dh:])
        # gradient: padding columns hold NaN and must not be read
        dhp = epd.padded_head_dim(dh)
        grads = []
        for n in range(3):
            t = torch.full((heads, T, dhp), float("nan"), device="cuda").to(got[0].dtype)
            t[:, :, :dh] = normal(20 + n, dtype, heads, T, dh)
            grads.append(t)
        d = epd.op_rope_axes_split_backward(dtype, *grads, pos, dh, sections, layout, THETA, q_scale)
        g64 = [t[:, :, :dh].transpose(0, 1).double() for t in grads]
        ref = torch.stack([rotate(g64[0], pos, sections, layout, sign=-1.0) * q_scale,
                           rotate(g64[1], pos, sections, layout, sign=-1.0), g64[2]], 1).reshape(T, -1)
        parity(d, ref, TOL[dtype], "gradient")


def test_gradient_against_differences():
    """<g, f(x + h v) - f(x - h v)> / 2h of the 64-bit definition: the map is linear, so the quotient is exact up to
    double rounding and the gradient's own 1e-6."""
    T, heads, dh, sections, q_scale = 50, 3, 64, (8, 12, 12), 0.18
    for layout in LAYOUTS:
        pos = positions(3, 3, T)
        qkv, v = normal(1, F32, T, 3 * heads * dh), normal(2, F32, T, 3 * heads * dh).double()
        grads = [normal(30 + n, F32, heads, T, dh) for n in range(3)]
        d = epd.op_rope_axes_split_backward(F32, *grads, pos, dh, sections, layout, THETA, q_scale)
        f = lambda z: split_reference(z, pos, heads, dh, sections, layout, q_scale)   # noqa: E731
        up, down = f(qkv.double() + 1e-3 * v), f(qkv.double() - 1e-3 * v)
        quotient = sum(float((g.double() * (a - b)).sum()) for g, a, b in zip(grads, up, down)) / 2e-3
        along = float((d.double() * v).sum())
        scale = float(d.double().norm() * v.norm())
        assert abs(quotient - along) <= 1e-6 * scale


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_two_blocks_are_the_two_axis_form(dtype):
    """Two blocks of head_dim / 4 pairs are epd_op_rope_split's rotation by row and column."""
    T, heads, dh = 500, 16, 72
    qkv, pos = normal(3, dtype, T, 3 * heads * dh), positions(4, 2, T, 0, 64)
    q_scale = 1.4426950408889634 / np.sqrt(dh)
    a = epd.op_rope_split(dtype, qkv, pos[0].contiguous(), pos[1].contiguous(), heads, dh, THETA, q_scale)
    b = epd.op_rope_axes_split(dtype, qkv, pos, heads, dh, (dh // 4, dh // 4), epd.ROPE_BLOCKS, THETA, q_scale)
    for p, q in zip(a, b):
        parity(q, p, TOL[dtype])


def test_no_rotation_and_no_tokens():
    x, pos = normal(1, BF16, 10, 2, 64), positions(1, 2, 10)
    assert torch.equal(epd.op_rope_axes(BF16, x, pos, (16, 16), epd.ROPE_SECTIONS, 0.0), x)
    assert epd.op_rope_axes(BF16, x[:0], pos[:, :0], (16, 16), epd.ROPE_SECTIONS, THETA).shape == (0, 2, 64)
    q, k, v = epd.op_rope_axes_split(BF16, normal(1, BF16, 0, 384), pos[:, :0], 2, 64, (16, 16), 0, THETA, 1.0)
    assert q.shape == (2, 0, 64)
    assert epd.op_rope_axes_split_backward(BF16, q, k, v, pos[:, :0], 64, (16, 16), 0, THETA, 1.0).shape == (0, 384)


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^31 elements: its last tokens."""
    T, heads, dh = 17, 1, 128
    step = (1 << 31) // 16 + 8
    store = torch.empty(step * 16 + 128, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((T, heads, dh), (step, dh, 1))
    x.copy_(normal(1, BF16, T, heads, dh))
    pos = positions(2, 3, T)
    y = epd.op_rope_axes(BF16, x, pos, (16, 24, 24), epd.ROPE_SECTIONS, THETA)
    parity(y, rotate(x.double(), pos, (16, 24, 24), epd.ROPE_SECTIONS), TOL[BF16])


def test_streams_and_graphs():
    T, heads, dh, sections = 333, 4, 72, (12, 12, 12)
    qkv, pos = normal(1, BF16, T, 3 * heads * dh), positions(2, 3, T)
    args = (pos, heads, dh, sections, epd.ROPE_BLOCKS, THETA, 0.2)
    want = epd.op_rope_axes_split(BF16, qkv, *args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = epd.op_rope_axes_split(BF16, qkv, *args)
    got2 = epd.op_rope_axes_split(BF16, qkv, *args, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, got2))
    graph = torch.cuda.CUDAGraph()
    keep = qkv.clone()
    with torch.cuda.graph(graph):
        q = epd.op_rope_axes_split(BF16, qkv, *args)
        d = epd.op_rope_axes_split_backward(BF16, *q, pos, dh, sections, epd.ROPE_BLOCKS, THETA, 0.2)
    qkv.zero_()
    graph.replay()
    qkv.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, q))
    assert torch.equal(d, epd.op_rope_axes_split_backward(BF16, *want, pos, dh, sections, epd.ROPE_BLOCKS, THETA, 0.2))


def test_binding_refuses_mismatched_tensors():
    x, pos = normal(1, BF16, 10, 2, 64), positions(1, 2, 10)
    for bad in (pos.long(), pos[:1], pos[:, :9], pos.cpu(), pos.t().contiguous().t(), pos[:1].expand(2, 10)):
        with pytest.raises(ValueError):
            epd.op_rope_axes(BF16, x, bad, (16, 16), 0, THETA)
    for sections, layout, theta in (((16, 17), 0, THETA), ((-1, 4), 0, THETA), ((16, 16), 3, THETA),
                                    ((16, 16), 0, float("nan")), ((16, 16), 0, float("inf"))):
        with pytest.raises(epd.EpdError) as e:
            epd.op_rope_axes(BF16, x, pos, sections, layout, theta)
        assert e.value.status == epd.EPD_EINVAL
    with pytest.raises(epd.EpdError):          # tokens that run into one another
        epd.op_rope_axes(BF16, x[:, :1].expand(10, 2, 64), pos, (16, 16), 0, THETA)
    with pytest.raises(ValueError):
        epd.op_rope_axes(F32, x, pos, (16, 16), 0, THETA)
