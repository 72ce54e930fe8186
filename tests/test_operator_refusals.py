"""What the layer norm, the balance loss and the orthogonalisation refuse: C entries with arguments that are no arrays (nothing is
launched), and the binding with tensors that do not fit."""
import os

import pytest
import torch

N, S, P, D, W, OK = -1, -2, -3, -4, -5, 0


@pytest.fixture(scope="module")
def lib():
    from paper_2506_15050_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load()


def test_layer_norm(lib):
    def call(x=256, n_rows=4, H=64, ld_x=64, dt=0, weight=256, bias=None, dt_w=0, eps=1e-5, rows=None, M=4, y=256, ld_y=64):
        return lib.tppo_layer_norm(x, n_rows, H, ld_x, dt, weight, bias, dt_w, eps, rows, M, None, y, ld_y, None, None, None, None)
    assert call(dt=2) == D and call(dt_w=-1) == D and call(dt=0, dt_w=1) == D
    assert call(M=-1) == S and call(n_rows=-1) == S and call(H=0) == S and call(H=16385, ld_x=16385, ld_y=16385) == S
    assert call(ld_x=63) == S and call(ld_y=63) == S and call(M=5) == S and call(n_rows=0, rows=256) == S
    assert call(eps=-1e-5) == P and call(eps=float("nan")) == P and call(eps=float("inf")) == P
    assert call(x=None) == N and call(weight=None) == N and call(y=None) == N
    assert call(x=258) == P and call(y=258) == P and call(weight=254) == P and call(bias=257) == P
    assert call(dt=1, dt_w=1, x=257) == P
    assert call(M=0, x=None, y=None) == OK


def test_layer_norm_backward(lib):
    big = lib.tppo_layer_norm_backward_workspace_bytes(4, 64)

    def call(gy=256, ld_gy=64, dt_gy=0, x=256, n_rows=4, H=64, ld_x=64, dt=0, weight=256, dt_w=0, mean=256, rstd=256, rows=None, M=4,
             gx=256, ld_gx=64, dt_gx=0, out_index=None, n_out=4, gw=256, gb=256, ws=256, ws_bytes=big):
        return lib.tppo_layer_norm_backward(gy, ld_gy, dt_gy, x, n_rows, H, ld_x, dt, weight, dt_w, mean, rstd, rows, M, None, gx, ld_gx,
                                            dt_gx, out_index, n_out, gw, gb, 0, ws, ws_bytes, None, None)
    assert big >= 2 * 4 * 64 * 4
    assert call(dt=3) == D and call(dt_gy=1) == D and call(dt_gx=1) == D and call(dt_w=1) == D
    assert call(H=0) == S and call(H=16385) == S and call(ld_gy=60) == S and call(ld_x=60) == S and call(ld_gx=60) == S
    assert call(M=5) == S and call(n_out=3) == S and call(n_out=-1) == S and call(n_rows=0, rows=256) == S
    assert call(gy=None) == N and call(x=None) == N and call(weight=None) == N and call(mean=None) == N and call(rstd=None) == N
    assert call(gy=258) == P and call(gx=258) == P and call(gw=258) == P and call(gb=258) == P
    assert call(ws=None) == W and call(ws=264) == W and call(ws_bytes=big - 1) == W
    assert call(gx=None, gw=None, gb=None, gy=None) == OK


def test_balance_loss(lib):
    big = lib.tppo_balance_loss_workspace_bytes(4, 8)

    def call(z=256, n_rows=4, E=8, ld=8, dt=0, ids=256, k=2, ld_ids=2, rows=None, M=4, coefficient=0.1, ws=256, ws_bytes=big, loss=256):
        return lib.tppo_balance_loss(z, n_rows, E, ld, dt, ids, k, ld_ids, rows, M, None, coefficient, loss, None, None, ws, ws_bytes, None,
                                     None)

    def back(grad=256, ld_grad=8, out_index=None, n_out=4, scale=1.0, denominator=0, E=8):
        return lib.tppo_balance_loss_backward(256, 4, E, 8, 0, 256, 2, 2, None, 4, None, 0.1, scale, None, denominator, grad, ld_grad,
                                              out_index, n_out, None, None, None, 256, 0, None, None)
    assert call(dt=2) == D
    assert call(E=0) == S and call(E=2049, ld=2049) == S and call(E=1 << 33, ld=1 << 33) == S and call(k=0) == S and call(k=1025, ld_ids=1025) == S
    assert call(ld=7) == S and call(ld_ids=1) == S and call(M=5) == S and call(M=-1) == S and call(n_rows=0, rows=256) == S
    assert call(M=1 << 31, rows=256) == S and call(M=1 << 30, rows=256, k=128, ld_ids=128) == S
    assert call(coefficient=float("nan")) == P and call(coefficient=float("inf")) == P
    assert call(z=None) == N and call(ids=None) == N and call(z=258) == P and call(ids=258) == P
    assert call(ws=None) == W and call(ws=264) == W and call(ws_bytes=big - 1) == W
    assert call(loss=None, ws=None) == OK
    assert back(scale=float("nan")) == P and back(denominator=-1) == S and back(ld_grad=7) == S and back(n_out=3) == S
    assert back(grad=None) == N and back(grad=258) == P and back() == W and back(E=0) == S


def test_orthogonalize(lib):
    big = lib.tppo_orthogonalize_workspace_bytes(2, 100, 70)

    def call(g=256, count=2, rows=100, cols=70, ld_g=70, stride_g=7000, dt=0, steps=5, a=3.4, b=-4.8, c=2.0, eps=1e-7, scale=1.0, out=256,
             ld_out=70, stride_out=7000, ws=256, ws_bytes=big):
        return lib.tppo_orthogonalize(g, count, rows, cols, ld_g, stride_g, dt, steps, a, b, c, eps, scale, out, ld_out, stride_out, ws,
                                      ws_bytes, None)
    assert call(dt=2) == D
    assert call(rows=0) == S and call(cols=0) == S and call(rows=65537) == S and call(ld_g=69) == S and call(ld_out=69) == S
    assert call(count=-1) == S and call(count=65536) == S and call(stride_g=-1) == S and call(stride_out=6999) == S
    assert call(steps=-1) == P and call(steps=65) == P and call(eps=-1.0) == P and call(eps=float("nan")) == P
    for name in ("a", "b", "c", "scale", "eps"):
        assert call(**{name: float("inf")}) == P
    assert call(g=None) == N and call(out=None) == N and call(g=258) == P and call(out=257) == P
    assert call(ws=None) == W and call(ws=264) == W and call(ws_bytes=big - 1) == W
    assert call(count=0, g=None) == OK


def test_the_binding_takes_device_tensors_only():
    from paper_2506_15050_amd import binding as tp
    x, w, ids = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: tp.tppo_layer_norm(x, w), lambda: tp.tppo_layer_norm_backward(x, x, w, w, w),
                 lambda: tp.tppo_balance_loss(x, ids), lambda: tp.tppo_balance_loss_backward(x, ids), lambda: tp.tppo_orthogonalize(x)):
        with pytest.raises(ValueError):
            call()
