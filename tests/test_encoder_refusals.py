"""CPU tests: what the encoder's entry points refuse, before anything is launched (device pointers are made up: a call that
touched one would not come back with the status asked for)."""
import pytest
import torch

import paper_2211_00839_amd as rcd

P = 1 << 20      # any aligned address
F32, BF16, MX = 0, 1, 2
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 4, 5


@pytest.fixture(scope="module")
def lib():
    import os

    from paper_2211_00839_amd import binding
    if not os.path.exists(binding.lib_path()):
        from paper_2211_00839_amd import build
        build.build()
    return binding.load_library()


def norm(lib, dt=F32, rows=4, d=64, ld_x=64, r=None, ld_r=64, eps=1e-6, s=None, ld_s=64, y=P, out=F32, ld_y=64, scale=None, ld_scale=2, x=P):
    return lib.rcd_rms_norm(x, dt, rows, d, ld_x, r, ld_r, None, eps, s, ld_s, y, out, ld_y, scale, ld_scale, None, None)


def test_norm(lib):
    assert norm(lib, rows=0) == OK
    assert norm(lib, rows=0, x=None, y=None) == OK
    assert norm(lib, dt=7, out=7) == UNSUPPORTED
    assert norm(lib, dt=MX, out=MX) == UNSUPPORTED
    assert norm(lib, dt=BF16, out=F32) == UNSUPPORTED
    assert norm(lib, rows=-1) == INVALID
    assert norm(lib, d=0) == INVALID
    assert norm(lib, ld_x=63) == INVALID
    assert norm(lib, ld_y=63) == INVALID
    assert norm(lib, r=P, ld_r=63) == INVALID
    assert norm(lib, s=P, ld_s=63) == INVALID
    assert norm(lib, x=None) == INVALID
    assert norm(lib, y=None) == INVALID
    assert norm(lib, s=P, y=P) == INVALID
    assert norm(lib, eps=-1.0) == INVALID
    assert norm(lib, eps=float("nan")) == INVALID
    assert norm(lib, eps=float("inf")) == INVALID
    assert norm(lib, out=MX) == INVALID                       # no scales
    assert norm(lib, out=MX, scale=P, ld_scale=1) == INVALID
    assert norm(lib, d=1 << 31, ld_x=1 << 31, ld_y=1 << 31) == UNSUPPORTED


def test_norm_backward(lib):
    def call(dt=F32, rows=4, d=64, ld=64, rstd=P, dw=P, ws=P, nbytes=1 << 20, h=P):
        return lib.rcd_rms_norm_backward(P, dt, rows, d, ld, h, ld, rstd, None, None, 0, P, ld, dw, ws, nbytes, None)

    assert call(dt=MX) == UNSUPPORTED
    assert call(rows=0, dw=None) == OK
    assert call(rows=-1) == INVALID
    assert call(d=0) == INVALID
    assert call(ld=63) == INVALID
    assert call(rstd=None) == INVALID
    assert call(h=None) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(ws=P + 8) == WORKSPACE
    assert call(nbytes=lib.rcd_rms_norm_backward_workspace_bytes(4, 64) - 1) == WORKSPACE
    assert lib.rcd_rms_norm_backward_workspace_bytes(0, 64) == 0


def test_quantize(lib):
    def call(dt=F32, rows=4, d=64, ld_x=64, q=P, ld_q=64, s=P, ld_s=2):
        return lib.rcd_quantize_mxfp8(P, dt, rows, d, ld_x, q, ld_q, s, ld_s, None)

    assert call(rows=0) == OK
    assert call(dt=MX) == UNSUPPORTED
    assert call(d=0) == INVALID
    assert call(ld_x=1) == INVALID
    assert call(ld_q=1) == INVALID
    assert call(ld_s=1) == INVALID
    assert call(q=None) == INVALID
    assert call(s=None) == INVALID


def linear(lib, dt=F32, out=F32, M=4, N=8, K=64, a=P, sa=None, lda=64, w=P, sw=None, ldw=64, act=0, r=None, ldr=8, z=None, ldz=8,
           y=P, ldy=8, ws=P, nbytes=1 << 40):
    return lib.rcd_linear(a, sa, lda, 2, w, sw, ldw, 2, dt, out, M, N, K, None, act, r, ldr, z, ldz, y, ldy, ws, nbytes, None)


def test_linear(lib):
    assert linear(lib, M=0) == OK
    assert linear(lib, M=0, a=None, y=None, ws=None, nbytes=0) == OK
    assert linear(lib, dt=3) == UNSUPPORTED
    assert linear(lib, dt=F32, out=BF16) == UNSUPPORTED
    assert linear(lib, out=MX) == UNSUPPORTED
    assert linear(lib, act=4) == UNSUPPORTED
    assert linear(lib, act=-1) == UNSUPPORTED
    assert linear(lib, M=-1) == INVALID
    assert linear(lib, N=0) == INVALID
    assert linear(lib, K=0) == INVALID
    assert linear(lib, lda=63) == INVALID
    assert linear(lib, ldw=63) == INVALID
    assert linear(lib, ldy=7) == INVALID
    assert linear(lib, r=P, ldr=7) == INVALID
    assert linear(lib, z=P, ldz=7) == INVALID
    for name in ("a", "w", "y"):
        assert linear(lib, **{name: None}) == INVALID
    assert linear(lib, dt=MX, out=BF16) == INVALID             # no scales
    assert linear(lib, dt=MX, out=BF16, sa=P) == INVALID
    assert linear(lib, dt=MX, out=BF16, sa=P, sw=P, K=65, lda=65, ldw=65) == INVALID      # three scales to a row, two apart
    assert linear(lib, M=1 << 31) == UNSUPPORTED
    long = (1 << 22) + 1
    assert linear(lib, K=long, lda=long, ldw=long) == UNSUPPORTED
    assert linear(lib, N=long, ldy=long) == UNSUPPORTED
    assert lib.rcd_linear_workspace_bytes(64, 64, long, F32) == 0


def test_linear_backward(lib):
    def call(dt=F32, M=4, N=8, K=64, act=0, dy=P, a=P, w=P, z=None, da=P, ldda=64, dw=P, lddw=64, ws=P, nbytes=1 << 40):
        return lib.rcd_linear_backward(dy, N, a, K, w, K, dt, M, N, K, z, N, act, da, ldda, dw, lddw, None, ws, nbytes, None)

    assert call(dt=MX) == UNSUPPORTED
    assert call(M=0, dw=None) == OK
    assert call(M=-1) == INVALID
    assert call(act=2) == INVALID                              # no z
    assert call(act=9) == UNSUPPORTED
    assert call(a=None) == INVALID
    assert call(w=None) == INVALID
    assert call(dy=None) == INVALID
    assert call(ldda=63) == INVALID
    assert call(lddw=63) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(ws=P + 16) == WORKSPACE
    assert call(nbytes=lib.rcd_linear_backward_workspace_bytes(4, 8, 64, F32) - 1) == WORKSPACE


def test_gated(lib):
    def forward(dt=F32, out=F32, M=4, F=8, K=64, a=P, g=P, u=P, h=P, ldh=8, act=2, s=None):
        return lib.rcd_gated_linear(a, s, 64, 2, g, s, 64, 2, u, s, 64, 2, dt, out, M, F, K, act, None, h, ldh, P, 1 << 40, None)

    assert forward(M=0) == OK
    assert forward(dt=5) == UNSUPPORTED
    assert forward(act=7) == UNSUPPORTED
    assert forward(F=0) == INVALID
    assert forward(K=65) == INVALID
    assert forward(ldh=7) == INVALID
    for name in ("a", "g", "u", "h"):
        assert forward(**{name: None}) == INVALID
    assert forward(dt=MX, out=BF16) == INVALID

    def backward(dt=F32, M=4, F=8, K=64, saved=P, da=P, dg=P, du=P, ws=P, nbytes=1 << 40, act=2):
        return lib.rcd_gated_linear_backward(P, F, P, K, P, K, P, K, dt, M, F, K, saved, act, da, K, dg, K, du, K, ws, nbytes, None)

    assert backward(dt=MX) == UNSUPPORTED
    assert backward(M=0, dg=None, du=None) == OK
    assert backward(saved=None) == INVALID
    assert backward(dg=None) == INVALID                        # one without the other
    assert backward(du=None) == INVALID
    assert backward(ws=None) == WORKSPACE
    assert backward(nbytes=lib.rcd_gated_linear_backward_workspace_bytes(4, 8, 64, F32) - 1) == WORKSPACE


def test_workspace_sizes(lib):
    for f in (lib.rcd_linear_workspace_bytes, lib.rcd_linear_backward_workspace_bytes, lib.rcd_gated_linear_workspace_bytes,
              lib.rcd_gated_linear_backward_workspace_bytes):
        for sizes in ((1, 1, 1), (1000, 511, 300), (16384, 2048, 2048)):
            for dt in (F32, BF16):
                assert f(*sizes, dt) % 256 == 0
        assert f(0, 8, 8, F32) == 0 and f(-1, 8, 8, F32) == 0
        # no call with these extents is served: the sizes asked for must not wrap round into small ones
        assert f(8, 1 << 40, 8, F32) == 0 and f(8, 8, 0, F32) == 0


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    t = torch.zeros(4, 8)
    for call in (lambda: rcd.rms_norm(t), lambda: rcd.linear(t, t), lambda: rcd.gated_linear(t, t, t), lambda: rcd.quantize_mxfp8(t),
                 lambda: rcd.linear_backward(t, t, t), lambda: rcd.rms_norm_backward(t, t, None)):
        with pytest.raises(rcd.RcdError):
            call()
