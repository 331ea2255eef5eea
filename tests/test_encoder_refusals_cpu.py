"""Arguments that the encoder operators refuse, and the workspaces they ask for: host code that answers before anything is
launched, so it needs no GPU."""
import ctypes

import pytest

from paper_2604_18780_amd import binding as sb

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3
A = 1 << 20  # an address that is never followed: every call here is refused


def call(entry, args, **changes):
    """The entry's status, with named arguments of `args` changed."""
    assert set(changes) <= set(args), changes
    return getattr(sb.load(), entry)(*{**args, **changes}.values())


EMBED = dict(tokens=A, lengths=None, table=A, scale=1.0, B=2, T=8, V=16, D=16, flags=0, out=A, stream=None)
EMBED_BWD = dict(tokens=A, lengths=None, grad_out=A, scale=1.0, B=2, T=8, V=16, D=16, flags=0, workspace=A, bytes=1 << 30,
                 grad_table=A, stream=None)
CONV = dict(u=A, u_row=16, weight=A, bias=None, lengths=None, seen=None, ring=None, B=2, T=8, C=16, W=4, flags=0, out=A,
            out_row=16, ring_out=None, stream=None)
CONV_BWD = dict(u=A, u_row=16, weight=A, bias=None, lengths=None, gy=A, gy_row=16, B=2, T=8, C=16, W=4, flags=0, workspace=A,
                bytes=1 << 30, gu=A, gu_row=16, gw=A, gb=None, stream=None)
SSM = dict(x=A, x_row=128, b=A, b_row=16, c=A, c_row=16, dt=A, dt_row=2, rate=A, skip=None, dt_bias=None, lengths=None,
           state=None, B=2, T=8, H=2, P=64, G=1, N=16, flags=0, workspace=A, bytes=1 << 30, y=A, y_row=128, state_out=None,
           stream=None)
SSM_BWD = dict(x=A, x_row=128, b=A, b_row=16, c=A, c_row=16, dt=A, dt_row=2, rate=A, skip=None, dt_bias=None, lengths=None,
               state=None, gy=A, gy_row=128, glast=None, B=2, T=8, H=2, P=64, G=1, N=16, flags=0, workspace=A, bytes=1 << 30,
               gx=A, gx_row=128, gb=A, gb_row=16, gc=A, gc_row=16, gdt=A, gdt_row=2, grate=A, gskip=None, gbias=None,
               gstate=None, stream=None)
STEP = dict(u=A, u_row=160, weight=A, bias=None, dt=A, dt_row=2, rate=A, skip=None, dt_bias=None, seen=A, ring=A, state=A, B=2,
            H=2, P=64, G=1, N=16, W=4, flags=0, y=A, ring_out=A, state_out=A, stream=None)
BOTH = sb.SEMICRF_EMIS_F16 | sb.SEMICRF_EMIS_BF16

CASES = [
    ("semicrf_embed_fwd", EMBED, EINVAL, [dict(tokens=None), dict(table=None), dict(out=None), dict(B=0), dict(T=0), dict(V=0),
                                          dict(table=A + 8), dict(out=A + 4), dict(flags=BOTH)]),
    ("semicrf_embed_fwd", EMBED, EUNSUPPORTED, [dict(D=12), dict(V=(1 << 24) + 1), dict(B=1 << 15, T=1 << 16)]),
    ("semicrf_embed_bwd", EMBED_BWD, EINVAL, [dict(grad_out=None), dict(grad_table=None), dict(grad_table=A + 4)]),
    ("semicrf_embed_bwd", EMBED_BWD, EWORKSPACE, [dict(workspace=None), dict(workspace=A + 16), dict(bytes=100)]),
    ("semicrf_conv_fwd", CONV, EINVAL, [dict(u=None), dict(weight=None), dict(out=None), dict(u_row=8), dict(out_row=18),
                                        dict(u_row=1 << 20), dict(ring=A), dict(W=0), dict(C=0), dict(flags=BOTH)]),
    ("semicrf_conv_fwd", CONV, EUNSUPPORTED, [dict(W=5), dict(C=12), dict(T=(1 << 30) + 1)]),
    ("semicrf_conv_bwd", CONV_BWD, EINVAL, [dict(gy=None), dict(gu=None), dict(gw=None), dict(gu=A + 8), dict(gy_row=17)]),
    ("semicrf_conv_bwd", CONV_BWD, EWORKSPACE, [dict(workspace=None), dict(workspace=A + 16), dict(bytes=100)]),
    ("semicrf_ssm_fwd", SSM, EINVAL, [dict(x=None), dict(b=None), dict(c=None), dict(dt=None), dict(rate=None), dict(y=None),
                                      dict(x_row=120), dict(b_row=18), dict(dt_row=1), dict(dt_row=1 << 23), dict(H=3, G=2),
                                      dict(state=A + 4), dict(state_out=A + 8), dict(x=A + 2), dict(flags=BOTH), dict(T=0)]),
    ("semicrf_ssm_fwd", SSM, EUNSUPPORTED, [dict(P=60), dict(N=12), dict(P=136), dict(N=136), dict(T=1 << 30, H=2)]),
    ("semicrf_ssm_fwd", {**SSM, "T": 4096}, EWORKSPACE, [dict(workspace=None), dict(workspace=A + 16), dict(bytes=100)]),
    ("semicrf_ssm_bwd", SSM_BWD, EINVAL, [dict(gy=None), dict(gx=None), dict(gb=None), dict(gc=None), dict(gdt=None),
                                          dict(grate=None), dict(gdt_row=1), dict(glast=A + 4), dict(gstate=A + 4)]),
    ("semicrf_ssm_bwd", SSM_BWD, EWORKSPACE, [dict(workspace=None), dict(workspace=A + 16), dict(bytes=100)]),
    ("semicrf_ssm_step", STEP, EINVAL, [dict(u=None), dict(weight=None), dict(dt=None), dict(rate=None), dict(seen=None),
                                        dict(ring=None), dict(state=None), dict(y=None), dict(ring_out=None),
                                        dict(state_out=None), dict(u_row=159), dict(dt_row=1), dict(state=A + 4), dict(W=0),
                                        dict(H=3, G=2), dict(flags=BOTH)]),
    ("semicrf_ssm_step", STEP, EUNSUPPORTED, [dict(W=5), dict(P=60), dict(N=136)]),
]


@pytest.mark.parametrize("entry,args,status,changes", CASES, ids=["%s%d" % (c[0], c[2]) for c in CASES])
def test_refused(entry, args, status, changes):
    for change in changes:
        assert call(entry, args, **change) == status, change


def size(entry, *sizes):
    n = ctypes.c_size_t(1 << 60)
    assert getattr(sb.load(), entry)(*sizes, ctypes.byref(n)) == 0
    return n.value


def test_workspaces():
    # one segment forwards needs none; several need the states at their boundaries
    assert size("semicrf_ssm_workspace_bytes", 64, 251, 8, 64, 1, 64, 0) == 0
    long = size("semicrf_ssm_workspace_bytes", 1, 100_000, 8, 64, 1, 64, 0)
    assert 0 < long < 100_000 * 8 * 64 * 2 * 2  # less than two bytes for each element of x and of y
    # gradients: at most a few times the inputs, and sublinear parts do not depend on the length of a short one
    grad = size("semicrf_ssm_workspace_bytes", 4, 100_000, 8, 64, 1, 64, 1)
    assert grad < 4 * 100_000 * (8 * 64 * 4 + 8 * 64 * 4)
    assert size("semicrf_embed_bwd_workspace_bytes", 1, 1, 4, 8) < 1 << 16
    assert size("semicrf_conv_bwd_workspace_bytes", 4, 100_000, 640, 4) < 64 << 20
    for entry, bad in (("semicrf_ssm_workspace_bytes", (0, 8, 2, 64, 1, 64, 0)), ("semicrf_embed_bwd_workspace_bytes", (1, 0, 4, 8)),
                       ("semicrf_conv_bwd_workspace_bytes", (1, 1, 8, 0))):
        n = ctypes.c_size_t(7)
        assert getattr(sb.load(), entry)(*bad, ctypes.byref(n)) == EINVAL and n.value == 7
        assert getattr(sb.load(), entry)(*bad, None) == EINVAL
