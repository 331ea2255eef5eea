"""GPU tests that nothing beside an output's rows is written: outputs lie inside larger arrays whose other elements keep their
values, with lengths and last blocks of every kind, and rows wider than what is written of them."""
import ctypes

import pytest
import torch

from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_scan import DEV, TYPES, forward, make

pytestmark = pytest.mark.gpu

MARK = 37.0


class Guarded:
    """An array of `rows` rows, `row` elements apart and `width` wide, with room before, behind and between."""

    def __init__(self, rows, width, row, dtype):
        self.rows, self.width, self.row, self.first = rows, width, row, 160 * row
        self.all = torch.full((self.first + (rows + 160) * row,), MARK, dtype=dtype, device=DEV)
        self.ptr = self.all.data_ptr() + self.first * self.all.element_size()

    def check(self, name):
        v = self.all.view(-1, self.row)
        inside = v[160:160 + self.rows, :self.width]
        assert (v[:160] == MARK).all() and (v[160 + self.rows:] == MARK).all(), name
        assert (v[160:160 + self.rows, self.width:] == MARK).all(), name
        assert inside.isfinite().all() and not (inside == MARK).all(), name


def check(status):
    assert status == 0, status


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,P,G,N,lengths", [
    (1, 1, 1, 64, 1, 64, [1]), (2, 5, 2, 16, 1, 24, [5, 3]), (2, 17, 3, 40, 1, 8, [0, 17]), (1, 31, 2, 128, 1, 128, [20]),
    (3, 33, 4, 32, 2, 64, [33, 32, 1]), (1, 65, 2, 64, 1, 40, [49]), (1, 300, 2, 64, 1, 64, [290]), (260, 3, 3, 64, 1, 64, None)])
def test_scan_and_its_gradients(B, T, H, P, G, N, lengths, dtype):
    print("[case] ssm bounds", B, T, H, P, G, N, dtype, flush=True)
    d, _ = make(B, T, H, P, G, N, dtype, lengths, seed=109)
    lib, flags = sb.load(), sb._act(d["x"])
    pad = 16
    y = Guarded(B * T, H * P, H * P + pad, dtype)
    state = Guarded(B * H * P, N, N, torch.float32)
    n = ctypes.c_size_t(0)
    sizes = (B, T, H, P, G, N)
    inputs = sb._ssm_inputs(d["x"], d["b"], d["c"], d["dt"], d["rate"], d["skip"], d["dt_bias"], d["lengths"], d["state"])[1]
    for grad in (0, 1):
        check(lib.semicrf_ssm_workspace_bytes(*sizes, grad, ctypes.byref(n)))
        room = torch.full((n.value + 8192,), 77, dtype=torch.uint8, device=DEV)
        work = room.data_ptr() + 4096
        if not grad:
            check(lib.semicrf_ssm_fwd(*inputs, *sizes, flags, work, n.value, y.ptr, y.row, state.ptr, sb._stream()))
            y.check("y"), state.check("state")
        else:
            gx, gb, gc = Guarded(B * T, H * P, H * P + pad, dtype), Guarded(B * T, G * N, G * N + 8, dtype), Guarded(B * T, G * N, G * N + 16, dtype)
            gdt = Guarded(B * T, H, H + 3, dtype)
            heads = [Guarded(1, H, H, torch.float32) for _ in range(3)]
            gstate = Guarded(B * H * P, N, N, torch.float32)
            check(lib.semicrf_ssm_bwd(*inputs, *sb._rows(d["gy"], dtype, d["gy"].shape), d["glast"].data_ptr(), *sizes, flags, work,
                                      n.value, gx.ptr, gx.row, gb.ptr, gb.row, gc.ptr, gc.row, gdt.ptr, gdt.row,
                                      *[v.ptr for v in heads], gstate.ptr, sb._stream()))
            for name, v in dict(gx=gx, gb=gb, gc=gc, gdt=gdt, grate=heads[0], gskip=heads[1], gbias=heads[2], gstate=gstate).items():
                v.check(name)
        assert (room[:4096] == 77).all() and (room[4096 + n.value:] == 77).all()
    # the same values as in arrays of their own
    own, last = forward(d)
    inside = y.all.view(-1, y.row)[160:160 + B * T, :H * P]
    assert torch.equal(inside, own.reshape(B * T, H * P)) and torch.equal(state.all.view(-1, N)[160:-160].reshape(last.shape), last)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,C,W", [(1, 1, 8, 4), (2, 9, 24, 3), (3, 33, 136, 4), (70, 7, 16, 2)])
def test_convolution_and_its_gradient(B, T, C, W, dtype):
    print("[case] conv bounds", B, T, C, W, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(113)
    u, gy = (torch.randn(B, T, C, generator=g, device=DEV).to(dtype) for _ in range(2))
    weight, bias = torch.randn(C, W, generator=g, device=DEV), torch.randn(C, generator=g, device=DEV)
    lib, flags, n = sb.load(), sb._act(u), ctypes.c_size_t(0)
    out, gu = Guarded(B * T, C, C + 8, dtype), Guarded(B * T, C, C + 16, dtype)
    gw, gb, ring = Guarded(C, W, W, torch.float32), Guarded(1, C, C, torch.float32), Guarded(B * C, W, W, dtype)
    check(lib.semicrf_conv_fwd(u.data_ptr(), C, weight.data_ptr(), bias.data_ptr(), None, None, None, B, T, C, W, flags, out.ptr,
                               out.row, ring.ptr, sb._stream()))
    check(lib.semicrf_conv_bwd_workspace_bytes(B, T, C, W, ctypes.byref(n)))
    room = torch.full((n.value + 8192,), 77, dtype=torch.uint8, device=DEV)
    check(lib.semicrf_conv_bwd(u.data_ptr(), C, weight.data_ptr(), bias.data_ptr(), None, gy.data_ptr(), C, B, T, C, W, flags,
                               room.data_ptr() + 4096, n.value, gu.ptr, gu.row, gw.ptr, gb.ptr, sb._stream()))
    for name, v in dict(out=out, gu=gu, gw=gw, gb=gb, ring=ring).items():
        v.check(name)
    assert (room[:4096] == 77).all() and (room[4096 + n.value:] == 77).all()


@pytest.mark.parametrize("n,V,D", [(1, 1, 8), (17, 5, 24), (1000, 300, 72), (5000, 700, 520)])
def test_embedding_and_its_gradient(n, V, D):
    g = torch.Generator(device=DEV).manual_seed(127)
    tokens = torch.randint(0, V, (1, n), generator=g, device=DEV, dtype=torch.int32)
    table, grad = torch.randn(V, D, generator=g, device=DEV), torch.randn(1, n, D, generator=g, device=DEV)
    lib, size = sb.load(), ctypes.c_size_t(0)
    out, gt = Guarded(n, D, D, torch.float32), Guarded(V, D, D, torch.float32)
    check(lib.semicrf_embed_fwd(tokens.data_ptr(), None, table.data_ptr(), 1.5, 1, n, V, D, 0, out.ptr, sb._stream()))
    check(lib.semicrf_embed_bwd_workspace_bytes(1, n, V, D, ctypes.byref(size)))
    room = torch.full((size.value + 8192,), 77, dtype=torch.uint8, device=DEV)
    check(lib.semicrf_embed_bwd(tokens.data_ptr(), None, grad.data_ptr(), 1.5, 1, n, V, D, 0, room.data_ptr() + 4096, size.value,
                                gt.ptr, sb._stream()))
    out.check("out"), gt.check("table")
    assert (room[:4096] == 77).all() and (room[4096 + size.value:] == 77).all()
