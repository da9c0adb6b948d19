"""The new operators as they are used together: one encoder block with (time, row, column) positions and a gated
feed-forward part, forward against the 64-bit definition; and its gradients chained back to the block's input."""
import numpy as np
import pytest
import torch

import paper_2601_11590_b200 as epd
from tests.metrics import assert_parity
from tests.test_gpu_gated_mlp import act_and_slope, reference_forward
from tests.test_gpu_rope_axes import rotate

pytestmark = pytest.mark.gpu

BF16 = epd.DTYPE_BF16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2601_11590_b200 import build
    build.build_library()
    epd.load_library()


def clip_positions(grids):
    rows = [(t, r, c) for (n, h, w) in grids for t in range(n) for r in range(h) for c in range(w)]
    return torch.tensor(rows, dtype=torch.int32, device="cuda").t().contiguous()


@pytest.mark.parametrize("heads,dh,sections,grids", [(4, 72, (12, 12, 12), [(3, 6, 8), (1, 10, 4)]),
                                                     (2, 128, (16, 24, 24), [(1, 2, 2), (4, 14, 14)])])
def test_block_with_three_axes_and_gated_mlp(heads, dh, sections, grids):
    h, m = heads * dh, 536
    pos = clip_positions(grids)
    T = pos.shape[1]
    cu = np.cumsum([0] + [t * a * b for t, a, b in grids]).astype(np.int32)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda std, *s: (torch.randn(*s, generator=g, device="cuda") * std).to(torch.bfloat16)   # noqa: E731
    x0 = torch.randn(T, h, generator=g, device="cuda")
    g1, g2 = 1 + n(0.1, h), 1 + n(0.1, h)
    w_qkv, b_qkv, w_o, b_o = n(h ** -0.5, 3 * h, h), n(0.1, 3 * h), n(h ** -0.5, h, h), n(0.1, h)
    w_in, b_in, w_out, b_out = n(h ** -0.5, 2 * m, h), n(0.1, 2 * m), n(m ** -0.5, h, m), n(0.1, h)
    q_scale = 1.4426950408889634 / np.sqrt(dh)

    x = x0.clone()
    a = torch.empty(T, h, dtype=torch.bfloat16, device="cuda")
    epd.op_rmsnorm(BF16, x, g1, a, 1e-6)
    qkv = torch.empty(T, 3 * h, dtype=torch.bfloat16, device="cuda")
    epd.op_linear(BF16, a, w_qkv, b_qkv, qkv, T, 3 * h, h)
    q, k, v = epd.op_rope_axes_split(BF16, qkv, pos, heads, dh, sections, epd.ROPE_BLOCKS, 1e4, q_scale)
    o = epd.op_attention(BF16, q, k, v, torch.from_numpy(cu).cuda(), cu, dh)
    epd.op_linear(BF16, o, w_o, b_o, x, T, h, h, epd.LINEAR_ACCUMULATE)
    a2 = torch.empty_like(a)
    epd.op_rmsnorm(BF16, x, g2, a2, 1e-6)
    epd.op_gated_mlp(BF16, a2, w_in, b_in, w_out, b_out, epd.GATE_SILU, out=x, flags=epd.LINEAR_ACCUMULATE)

    d = lambda t: t.double()   # noqa: E731
    norm = lambda t, w: t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6) * d(w)   # noqa: E731
    r = d(x0)
    y = norm(r, g1) @ d(w_qkv).T + d(b_qkv)
    qr, kr, vr = y.view(T, 3, heads, dh).unbind(1)
    qr, kr = (rotate(t, pos, sections, epd.ROPE_BLOCKS) for t in (qr, kr))
    att = torch.zeros(T, heads, dh, dtype=torch.float64, device="cuda")
    for lo, hi in zip(cu[:-1], cu[1:]):
        s = torch.einsum("qhd,khd->hqk", qr[lo:hi], kr[lo:hi]) / np.sqrt(dh)
        att[lo:hi] = torch.einsum("hqk,khd->qhd", torch.softmax(s, 2), vr[lo:hi])
    r = r + att.reshape(T, h) @ d(w_o).T + d(b_o)
    r = r + reference_forward(norm(r, g2), w_in, b_in, epd.GATE_SILU)[1] @ d(w_out).T + d(b_out)
    # the bound for one encoder block in bf16
    assert_parity(x.double().cpu().numpy(), r.cpu().numpy(), 1e-2)


def test_gradients_chain_back_through_the_projection_and_the_block():
    """d loss / d input of  a -> QKV projection -> rotation -> head split  (rope_axes_split_backward, then
    linear_backward) and of the gated block behind it, all in float, against automatic differentiation of the 64-bit
    definition.  Two products of float sums in a row: 2e-5."""
    F32 = epd.DTYPE_F32
    T, heads, dh, m, sections = 70, 3, 32, 56, (4, 6, 6)
    h = heads * dh
    g = torch.Generator(device="cuda").manual_seed(5)
    n = lambda std, *s: torch.randn(*s, generator=g, device="cuda") * std   # noqa: E731
    x, w_qkv, grads = n(1, T, h), n(h ** -0.5, 3 * h, h), [n(1, heads, T, dh) for _ in range(3)]
    pos = torch.randint(0, 500, (3, T), generator=g, device="cuda", dtype=torch.int32)
    w_in, w_out = n(h ** -0.5, 2 * m, h), n(m ** -0.5, h, m)
    out, hidden, pre = epd.op_gated_mlp(F32, x, w_in, None, w_out, None, epd.GATE_GELU_ERF, save=True)
    qkv = torch.empty(T, 3 * h, device="cuda")
    epd.op_linear(F32, out, w_qkv, None, qkv, T, 3 * h, h)
    epd.op_rope_axes_split(F32, qkv, pos, heads, dh, sections, epd.ROPE_INTERLEAVED, 1e4, 0.3)
    dqkv = epd.op_rope_axes_split_backward(F32, *grads, pos, dh, sections, epd.ROPE_INTERLEAVED, 1e4, 0.3)
    lin = epd.op_linear_backward(F32, dqkv, out, w_qkv, bias=False)
    got = epd.op_gated_mlp_backward(F32, lin["dx"], x, w_in, w_out, hidden, pre, epd.GATE_GELU_ERF, bias=False)

    leaves = [t.double().requires_grad_() for t in (x, w_in, w_out, w_qkv)]
    xd, wi, wo, wq = leaves
    p = xd @ wi.T
    y = (act_and_slope(epd.GATE_GELU_ERF, p[:, :m])[0] * p[:, m:]) @ wo.T
    q, k, v = (y @ wq.T).view(T, 3, heads, dh).unbind(1)

    def turned(t):
        rows = rotate_differentiable(t, pos, sections)
        return rows
    q, k = turned(q) * 0.3, turned(k)
    loss = sum((t.transpose(0, 1) * gr.double()).sum() for t, gr in zip((q, k, v), grads))
    loss.backward()
    for got_t, leaf, name in ((got["dx"], xd, "dx"), (got["dw_in"], wi, "dw_in"), (got["dw_out"], wo, "dw_out"),
                              (lin["dw"], wq, "dw_qkv")):
        assert_parity(got_t.double().cpu().numpy(), leaf.grad.cpu().numpy(), 2e-5, name)


def rotate_differentiable(x, pos, sections):
    """The interleaved layout as one out-of-place expression."""
    from tests.test_gpu_rope_axes import plan
    rows = plan(sections, epd.ROPE_INTERLEAVED, 1e4)
    ang = torch.stack([pos[a].double() * w for a, w, _, _ in rows], 1)[:, None]
    R = len(rows)
    a, b = x[..., :R], x[..., R:]
    return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)
