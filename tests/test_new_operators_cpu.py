"""Refusals of the gated block, the linear gradient and the rotary embedding with several axes, without a GPU: every
argument is checked on the host before anything is enqueued, so a bad call never reaches a device."""
import ctypes

import pytest

import paper_2601_11590_b200 as epd
from paper_2601_11590_b200 import build

P = 1 << 20          # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return epd.load_library()


def replace(args, **kw):
    return [kw.get(n, v) for n, v in args.items()]


def test_gated_linear_refusals(lib):
    ok = dict(dtype=1, x=P, ldx=64, w=P, ldw=64, bias=None, out=P, ldo=32, pre=None, ldp=0, ws=None, bytes=0,
              M=4, N=32, K=64, gate=0, stream=None)
    for bad in (dict(dtype=2), dict(x=None), dict(w=None), dict(out=None), dict(ldx=63), dict(ldw=63), dict(ldo=31),
                dict(pre=P, ldp=63), dict(M=-1), dict(N=0), dict(K=0), dict(gate=3), dict(gate=-1), dict(x=P + 1),
                dict(M=(1 << 28) + 1), dict(N=1 << 29, ldo=1 << 29), dict(ws=P + 16)):
        assert lib.epd_op_gated_linear(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    assert lib.epd_op_gated_linear(*replace(ok, M=0, x=None, w=None, out=None)) == epd.EPD_OK


def test_gated_mlp_refusals(lib):
    ok = dict(dtype=1, x=P, ldx=64, w_in=P, ldw_in=64, b_in=None, w_out=P, ldw_out=32, b_out=None, hidden=P, ldh=32,
              pre=None, ldp=0, out=P, ldo=48, ws=None, bytes=0, M=4, N=32, K=64, D=48, gate=0, flags=0, stream=None)
    for bad in (dict(dtype=-1), dict(x=None), dict(w_in=None), dict(w_out=None), dict(hidden=None), dict(out=None),
                dict(ldx=60), dict(ldw_in=60), dict(ldw_out=31), dict(ldh=31), dict(ldo=47), dict(pre=P, ldp=60), dict(M=-4),
                dict(N=-1), dict(D=0), dict(gate=9), dict(flags=1), dict(flags=16), dict(hidden=P + 1),
                dict(flags=8, out=P + 2), dict(ws=P + 128)):
        assert lib.epd_op_gated_mlp(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    assert lib.epd_op_gated_mlp(*replace(ok, M=0, hidden=None)) == epd.EPD_OK


def test_gated_mlp_backward_refusals(lib):
    need = lib.epd_gated_mlp_backward_workspace_bytes(1, 4, 32, 64, 48)
    assert need >= 4 * 64 * 2
    ok = dict(dtype=1, dout=P, lddo=48, x=P, ldx=64, w_in=P, ldw_in=64, w_out=P, ldw_out=32, hidden=P, ldh=32, pre=P, ldp=64,
              dx=P, lddx=64, dw_in=P, lddw_in=64, db_in=P, dw_out=P, lddw_out=32, db_out=P, ws=P, bytes=need, M=4, N=32,
              K=64, D=48, gate=0, stream=None)
    for bad in (dict(dtype=5), dict(dout=None), dict(x=None), dict(w_in=None), dict(w_out=None), dict(hidden=None),
                dict(pre=None), dict(lddo=47), dict(ldx=63), dict(ldw_in=63), dict(ldw_out=31), dict(ldh=31), dict(ldp=63),
                dict(lddx=63), dict(lddw_in=63), dict(lddw_out=31), dict(ws=None), dict(ws=P + 8), dict(gate=4), dict(M=-1),
                dict(N=0), dict(K=0), dict(D=0), dict(dx=P + 1)):
        assert lib.epd_op_gated_mlp_backward(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    assert lib.epd_op_gated_mlp_backward(*replace(ok, bytes=need - 1)) == epd.EPD_ENOMEM
    for bad in ((2, 4, 32, 64, 48), (1, -1, 32, 64, 48), (1, 4, 0, 64, 48), (1, 4, 32, 0, 48), (1, 4, 32, 64, 0),
                (1, 1 << 29, 32, 64, 48)):
        assert lib.epd_gated_mlp_backward_workspace_bytes(*bad) == 0


def test_linear_backward_refusals(lib):
    need = lib.epd_linear_backward_workspace_bytes(1, 4, 32, 64)
    ok = dict(dtype=1, dout=P, lddo=32, x=P, ldx=64, w=P, ldw=64, dx=P, lddx=64, dw=P, lddw=64, db=P, ws=P, bytes=need, M=4,
              N=32, K=64, stream=None)
    for bad in (dict(dtype=3), dict(dout=None), dict(x=None), dict(w=None), dict(lddo=31), dict(ldx=1), dict(ldw=1),
                dict(lddx=1), dict(lddw=1), dict(ws=None), dict(ws=P + 128), dict(M=-1), dict(N=0), dict(K=0), dict(dw=P + 1)):
        assert lib.epd_op_linear_backward(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    assert lib.epd_op_linear_backward(*replace(ok, bytes=need - 1)) == epd.EPD_ENOMEM


def sections(*s):
    return (ctypes.c_int32 * len(s))(*s)


def test_rope_axes_refusals(lib):
    ok = dict(dtype=1, x=P, xt=256, xh=64, pos=P, ps=4, out=2 * P, ot=256, oh=64, T=4, heads=4, dh=64, s=sections(8, 12, 12),
              n=3, layout=1, theta=1e4, scale=1.0, inverse=0, stream=None)
    for bad in (dict(dtype=2), dict(x=None), dict(pos=None), dict(out=None), dict(xt=255), dict(xh=63), dict(ot=0), dict(oh=0),
                dict(ps=3), dict(T=-1), dict(heads=0), dict(heads=65536), dict(dh=0), dict(dh=129), dict(s=None),
                dict(s=sections(8, 12, 13)), dict(s=sections(8, -1, 12)), dict(n=0), dict(n=5), dict(layout=-1),
                dict(layout=3), dict(theta=float("nan")), dict(theta=float("inf")), dict(out=P, ot=512), dict(x=P + 1),
                dict(pos=P + 2), dict(s=sections(1 << 30, 1 << 30, 1 << 30)), dict(xt=-256)):
        assert lib.epd_op_rope_axes(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    assert lib.epd_op_rope_axes(*replace(ok, T=0, x=None, out=None, pos=None)) == epd.EPD_OK


def test_rope_axes_split_refusals(lib):
    ok = dict(dtype=1, qkv=P, ld=768, pos=P, ps=4, q=P, k=P, v=P, T=4, heads=4, dh=64, s=sections(8, 12, 12), n=3, layout=0,
              theta=1e4, q_scale=1.0, stream=None)
    bads = (dict(dtype=2), dict(qkv=None), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(ld=767), dict(ps=1),
            dict(T=-1), dict(heads=0), dict(dh=130), dict(s=sections(30, 1, 2)), dict(n=0), dict(layout=7), dict(qkv=P + 1))
    for bad in bads:
        assert lib.epd_op_rope_axes_split(*replace(ok, **bad)) == epd.EPD_EINVAL, bad
    back = dict(dtype=1, q=P, k=P, v=P, pos=P, ps=4, qkv=P, ld=768, T=4, heads=4, dh=64, s=sections(8, 12, 12), n=3, layout=0,
                theta=1e4, q_scale=1.0, stream=None)
    for bad in bads:
        assert lib.epd_op_rope_axes_split_backward(*replace(back, **bad)) == epd.EPD_EINVAL, bad
