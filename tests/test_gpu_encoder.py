"""GPU tests of the feature encoder's operators against plain 64-bit forms, at the sizes, strides and values where they can go
wrong.  The bounds are derived in encoder_reference.py, before any run."""
import pytest
import torch

import encoder_reference as ref
import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6


def normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def strided(t, pitch, offset=0):
    """The same matrix with rows `pitch` apart, starting `offset` elements into its memory; the rest holds NaN."""
    rows, cols = t.shape
    room = torch.full((rows * pitch + offset + 64,), float("nan"), device="cuda").to(t.dtype)
    view = room[offset: offset + rows * pitch].view(rows, pitch)[:, :cols] if rows else room[:0].view(0, cols)
    view.copy_(t)
    return view


def check(got, want, bound, dtype, what):
    """|got - want| <= bound + the rounding of the stored type; NaN where want has NaN, infinities equal."""
    got = got.double()
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN"
    inf = ~fine & ~torch.isnan(want)
    assert torch.equal(got[inf], want[inf]), what + ": infinities"
    off = (got - want).abs()[fine]
    allowed = (bound + ref.unit(dtype) * (want.abs() + bound) + 1e-37)[fine] if torch.is_tensor(bound) else bound
    worst = (off / allowed).max().item() if off.numel() else 0.0
    print("%s: %.3f of the bound" % (what, worst), flush=True)
    assert worst <= 1.0, what


# ---- norm -----------------------------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 7), (1, 2048), (5, 511), (130, 64), (9, 513), (4, 1024), (7, 1025), (6, 2047), (3, 4096), (5, 5000), (2, 8192),
              (3, 8193), (2, 20001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d", NORM_SIZES)
def test_norm_and_its_gradients(rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows * 10007 + d)
    for layout, with_r, with_w in (("plain", True, True), ("strided", True, False), ("odd", False, True)):
        print("norm", rows, d, dtype, layout, flush=True)
        lay = {"plain": lambda t: t, "strided": lambda t: strided(t, -(-t.shape[1] // 8) * 8 + 16),
               "odd": lambda t: strided(t, t.shape[1] + 3, 1)}[layout]
        x, r = lay(normal(gen, rows, d, dtype=dtype)), lay(normal(gen, rows, d, dtype=dtype)) if with_r else None
        w = (1 + 0.2 * normal(gen, d)).to(dtype) if with_w else None
        dy, ds = lay(normal(gen, rows, d, dtype=dtype)), lay(normal(gen, rows, d, dtype=dtype)) if with_r else None
        got = rcd.rms_norm(x, w, EPS, residual=r, want_sum=True, want_rstd=True)
        h, rstd, y = ref.norm(x, w, EPS, r)
        check(got.sum, h, 0.0 * h, dtype, "sum")
        check(got.rstd[:, None], rstd, (d + 24) * ref.U32 * rstd, F32, "rstd")
        check(got.y, y, ref.norm_error(x, r, y, w, rstd, h, d), dtype, "y")
        # 8 bits with scales: every block's scale the least that holds it, every element within half a step of its value
        q = rcd.rms_norm(x, w, EPS, residual=r, quantize=True)
        err = ref.norm_error(x, r, y, w, rstd, h, d)
        e = q.scale.view(torch.uint8).double() - 127
        blocks = torch.nn.functional.pad(y.abs(), (0, -d % 32)).view(rows, -1, 32).amax(2)
        step = torch.pow(2.0, e)
        assert torch.all(blocks * (1 - 1e-5) <= 448 * step)
        assert torch.all((blocks * (1 + 1e-5) > 224 * step) | (e == -127))
        back = ref.mx_values(q.y, q.scale)
        fine = y.abs() / 16 + step.repeat_interleave(32, 1)[:, :d] * 2.0 ** -10 + 2 * err
        assert torch.all((back - y).abs() <= fine)
        # gradients, at the h and rstd that the forward call stored
        dx, dw = rcd.rms_norm_backward(dy, got.sum, got.rstd, w, dsum=ds)
        hs, rs = got.sum.double(), got.rstd.double()[:, None]
        xh, g = hs * rs, dy.double() * (1 if w is None else w.double())
        mean = (g * xh).mean(1, keepdim=True)
        emean = (d + 16) * ref.U32 * (g * xh).abs().mean(1, keepdim=True)
        dx_ref = rs * (g - xh * mean) + (0 if ds is None else ds.double())
        bound = rs * (xh.abs() * emean + 8 * ref.U32 * (g.abs() + (xh * mean).abs())) + 2 * ref.U32 * dx_ref.abs()
        check(dx, dx_ref, bound, dtype, "dx")
        check(dw[None], (dy.double() * xh).sum(0)[None], (rows + 16) * 2 * ref.U32 * (dy.double() * xh).abs().sum(0)[None], dtype, "dweight")


def test_norm_of_many_rows_and_of_none():
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dy = normal(gen, 40001, 72, dtype=BF16), normal(gen, 40001, 72, dtype=BF16)
    n = rcd.rms_norm(x, None, EPS, want_rstd=True)
    dx, dw = rcd.rms_norm_backward(dy, x, n.rstd)
    xh = x.double() * n.rstd.double()[:, None]
    check(dw[None], (dy.double() * xh).sum(0)[None], 200 * ref.U32 * (dy.double() * xh).abs().sum(0)[None], BF16, "dweight")
    none = torch.empty(0, 72, dtype=BF16, device="cuda")
    n = rcd.rms_norm(none, None, EPS, quantize=True, want_sum=True, want_rstd=True)
    assert n.y.shape == (0, 72) and n.scale.shape == (0, 3) and n.rstd.shape == (0,)
    dx, dw = rcd.rms_norm_backward(none, none, n.rstd)
    assert dx.shape == (0, 72) and torch.all(dw == 0)


def test_norm_of_zeros_infinities_and_nans():
    x = torch.zeros(5, 96, device="cuda")
    x[1, 3] = float("inf")
    x[2, 40] = float("nan")
    x[3] = torch.arange(96, device="cuda") - 48.0
    x[4] = 1e-42      # denormal
    n = rcd.rms_norm(x, None, EPS, quantize=False)
    _, _, y = ref.norm(x, None, EPS)
    assert torch.all(n.y[0] == 0)
    assert torch.isnan(n.y[1, 3]) and torch.all(n.y[1, :3] == 0)
    assert torch.all(torch.isnan(n.y[2]))
    assert torch.allclose(n.y[3].double(), y[3], rtol=1e-6)
    q = rcd.rms_norm(x, None, EPS, quantize=True)
    assert torch.all(q.y[0].float() == 0) and torch.all(q.scale[0].view(torch.uint8) == 0)
    assert torch.isnan(q.y[1, 3].float()) and torch.all(q.y[1, :3].float() == 0)
    assert torch.all(torch.isnan(q.y[2].float()))
    # eps = 0 on a row of zeros: 0 * infinity
    assert torch.all(torch.isnan(rcd.rms_norm(x[:1], None, 0.0).y))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 31), (3, 33), (2, 2048), (5, 100), (2, 9000)])
def test_quantized_rows_are_the_definitions(rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = normal(gen, rows, d)
    x *= torch.pow(2.0, torch.randint(-140, 120, (rows, d), generator=gen, device="cuda").float() / 4)
    x = x.to(dtype)
    if d > 32:
        x[0, :32] = 0
        x[-1, 32:] = 448.0 * 2.0 ** torch.randint(-9, 0, (d - 32,), generator=gen, device="cuda")
    for v in (x, strided(x, d + 5, 1)):
        q, scale = rcd.quantize_mxfp8(v)
        b = torch.nn.functional.pad(v.double(), (0, -d % 32)).view(rows, -1, 32)
        e = torch.ceil(torch.log2(b.abs().amax(2) / 448)).clamp(min=-127)     # (448 = 2^8 1.75: no power of two is met inexactly)
        assert torch.equal(scale.view(torch.uint8), (e + 127).to(torch.uint8))
        want = (b / torch.pow(2.0, e)[..., None]).view(rows, -1)[:, :d].float().to(torch.float8_e4m3fn)
        assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))


def test_norm_in_place_leaves_the_same_bits():
    gen = torch.Generator(device="cuda").manual_seed(3)
    lib = rcd.load_library()
    from paper_2211_00839_amd.binding import _dev_ptr, _stream
    for d in (512, 2048, 9000):
        x, r = normal(gen, 6, d, dtype=BF16), normal(gen, 6, d, dtype=BF16)
        want = rcd.rms_norm(x, None, EPS, residual=r, want_sum=True)
        x2, r2 = x.clone(), r.clone()      # the sum into the residual, y into x
        assert lib.rcd_rms_norm(_dev_ptr(x2), 1, 6, d, d, _dev_ptr(r2), d, None, EPS, _dev_ptr(r2), d, _dev_ptr(x2), 1, d, None, 0,
                                None, _stream()) == 0
        assert torch.equal(r2, want.sum) and torch.equal(x2, want.y)


# ---- products -------------------------------------------------------------------------------------------------------------

# M, N, K: single elements, single tokens, tile edges on either side, lengths that are multiples of nothing
SIZES = [(1, 1, 1), (1, 64, 2048), (2, 100, 64), (7, 33, 500), (16, 256, 512), (17, 65, 96), (33, 130, 257), (64, 200, 1000), (128, 128, 128),
         (129, 127, 65), (200, 384, 72), (255, 257, 320), (300, 512, 1100), (513, 260, 40), (1000, 511, 300)]
ACTS = ["none", "relu", "silu", "gelu"]


def layouts(i):
    return [lambda t: t, lambda t: strided(t, -(-t.shape[1] // 8) * 8 + 8), lambda t: strided(t, t.shape[1] + 1, 3)][i % 3]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_linear_and_its_gradients(i, dtype):
    M, N, K = SIZES[i]
    gen = torch.Generator(device="cuda").manual_seed(i)
    for turn, act in enumerate(ACTS):
        print("linear", M, N, K, dtype, act, flush=True)
        lay = layouts(i + turn)
        a, w = lay(normal(gen, M, K, dtype=dtype)), lay(normal(gen, N, K, dtype=dtype, scale=K ** -0.5))
        b = normal(gen, N, dtype=dtype, scale=0.2) if turn != 1 else None
        r = lay(normal(gen, M, N, dtype=dtype)) if turn != 2 else None
        y, z = rcd.linear(a, w, b, act=act, residual=r, want_preact=True)
        ad, wd, bd, rd = (None if t is None else t.double() for t in (a, w, b, r))
        z_ref, y_ref = ref.linear(ad, wd, bd, act, rd)
        ez, ev = ref.linear_error(ad, wd, bd, act, z_ref)
        check(z, z_ref, ez, F32, "z")
        check(y, y_ref, ev + ref.U32 * y_ref.abs(), dtype, "y")
        assert torch.equal(y, rcd.linear(a, w, b, act=act, residual=r))
        dy = lay(normal(gen, M, N, dtype=dtype))
        da, dw, db = rcd.linear_backward(dy, a, w, z, act=act)
        dyd = dy.double()
        dz, da_ref, dw_ref, db_ref = ref.linear_backward(dyd, ad, wd, z_ref, act)
        edz = dyd.abs() * ref.act_error(z_ref, ez, act)[1] + 2 * ref.U32 * dz.abs()
        rounded = edz + (0 if dtype == F32 or act == "none" else ref.U16 * (dz.abs() + edz))
        check(da, da_ref, rounded @ wd.abs() + ref.sum_error(N, (dz.abs() + edz) @ wd.abs()), dtype, "da")
        check(dw, dw_ref, rounded.t() @ ad.abs() + ref.sum_error(M, (dz.abs() + edz).t() @ ad.abs()), dtype, "dw")
        check(db[None], db_ref[None], (edz.sum(0) + ref.sum_error(M, (dz.abs() + edz).sum(0)))[None], dtype, "db")
        only = rcd.linear_backward(dy, a, w, z, act=act, want_da=False, want_dbias=False)
        assert only[0] is None and only[2] is None and torch.equal(only[1], dw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_gated_and_its_gradients(i, dtype):
    M, F, K = SIZES[i]
    gen = torch.Generator(device="cuda").manual_seed(100 + i)
    for turn, act in enumerate(["silu", ACTS[i % 4]]):
        print("gated", M, F, K, dtype, act, flush=True)
        lay = layouts(i + turn)
        a = lay(normal(gen, M, K, dtype=dtype))
        wg, wu = (lay(normal(gen, F, K, dtype=dtype, scale=K ** -0.5)) for _ in range(2))
        h, saved = rcd.gated_linear(a, wg, wu, act=act, want_saved=True)
        ad, wgd, wud = a.double(), wg.double(), wu.double()
        g, u, h_ref = ref.gated(ad, wgd, wud, act)
        eg, eu = (ref.sum_error(K, ad.abs() @ w.abs().t()) for w in (wgd, wud))
        ev, es = ref.act_error(g, eg, act)
        value, slope = ref.act_both(g, act)
        check(saved[..., 0], g, eg, F32, "g")
        check(saved[..., 1], u, eu, F32, "u")
        check(h, h_ref, ev * (u.abs() + eu) + value.abs() * eu + 2 * ref.U32 * h_ref.abs(), dtype, "h")
        assert torch.equal(h, rcd.gated_linear(a, wg, wu, act=act))
        dh = lay(normal(gen, M, F, dtype=dtype))
        da, dwg, dwu = rcd.gated_linear_backward(dh, a, wg, wu, saved, act=act)
        dhd = dh.double()
        dg, du, da_ref, dwg_ref, dwu_ref = ref.gated_backward(dhd, ad, wgd, wud, g, u, act)
        edg = dhd.abs() * (es * (u.abs() + eu) + slope.abs() * eu) + 4 * ref.U32 * dg.abs()
        edu = dhd.abs() * ev + 2 * ref.U32 * du.abs()
        more = 0 if dtype == F32 else ref.U16
        rg, ru = edg + more * (dg.abs() + edg), edu + more * (du.abs() + edu)
        mg, mu = dg.abs() + edg, du.abs() + edu
        check(da, da_ref, rg @ wgd.abs() + ru @ wud.abs() + ref.sum_error(2 * F, mg @ wgd.abs() + mu @ wud.abs()), dtype, "da")
        check(dwg, dwg_ref, rg.t() @ ad.abs() + ref.sum_error(M, mg.t() @ ad.abs()), dtype, "dw_gate")
        check(dwu, dwu_ref, ru.t() @ ad.abs() + ref.sum_error(M, mu.t() @ ad.abs()), dtype, "dw_up")
        assert torch.equal(rcd.gated_linear_backward(dh, a, wg, wu, saved, act=act, want_dw=False)[0], da)


def mx(gen, rows, K, scale=1.0, lay=lambda t: t):
    v = normal(gen, rows, K, scale=scale) * torch.pow(2.0, torch.randint(-6, 7, (rows, 1), generator=gen, device="cuda").float())
    v[:, ::37] *= 16
    q, s = rcd.quantize_mxfp8(v)
    return lay(q.view(torch.uint8)).view(torch.float8_e4m3fn), s


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_products_of_8_bit_operands(i, out_dtype):
    M, N, K = SIZES[i]
    gen = torch.Generator(device="cuda").manual_seed(200 + i)
    print("8 bits", M, N, K, out_dtype, flush=True)

    def lay(t):
        if i % 3 == 0:
            return t
        pitch, offset = (-(-t.shape[1] // 16) * 16 + 16, 0) if i % 3 == 1 else (t.shape[1] + 3, 1)
        room = torch.full((t.shape[0] * pitch + offset + 64,), 0x7f, dtype=torch.uint8, device="cuda")      # NaN codes around
        view = room[offset: offset + t.shape[0] * pitch].view(t.shape[0], pitch)[:, : t.shape[1]]
        view.copy_(t)
        return view

    (a, sa), (w, sw), (w2, sw2) = mx(gen, M, K, lay=lay), mx(gen, N, K, K ** -0.5, lay), mx(gen, N, K, K ** -0.5, lay)
    ad, wd, w2d = ref.mx_values(a, sa), ref.mx_values(w, sw), ref.mx_values(w2, sw2)
    b, r = normal(gen, N, dtype=out_dtype), normal(gen, M, N, dtype=out_dtype)
    act = ACTS[i % 4]
    y, z = rcd.linear(a, w, b, act=act, residual=r, a_scale=sa, w_scale=sw.view(torch.uint8), out_dtype=out_dtype, want_preact=True)
    z_ref, y_ref = ref.linear(ad, wd, b.double(), act, r.double())
    ez, ev = ref.linear_error(ad, wd, b.double(), act, z_ref)
    check(z, z_ref, ez, F32, "z")
    check(y, y_ref, ev + ref.U32 * y_ref.abs(), out_dtype, "y")
    h = rcd.gated_linear(a, w, w2, act="silu", a_scale=sa, gate_scale=sw, up_scale=sw2, out_dtype=out_dtype)
    g, u, h_ref = ref.gated(ad, wd, w2d, "silu")
    eg, eu = (ref.sum_error(K, ad.abs() @ v.abs().t()) for v in (wd, w2d))
    ev, _ = ref.act_error(g, eg, "silu")
    check(h, h_ref, ev * (u.abs() + eu) + ref.act_both(g, "silu")[0].abs() * eu + 2 * ref.U32 * h_ref.abs(), out_dtype, "h")


def test_bf16_operands_with_an_fp32_result_and_the_residual_in_place():
    gen = torch.Generator(device="cuda").manual_seed(4)
    for M in (1, 300):
        a, w, r = normal(gen, M, 128, dtype=BF16), normal(gen, 96, 128, dtype=BF16), normal(gen, M, 96)
        z, y = ref.linear(a.double(), w.double(), None, "none", r.double())
        want = rcd.linear(a, w, residual=r, out_dtype=F32)
        check(want, y, ref.linear_error(a.double(), w.double(), None, "none", z)[1] + ref.U32 * y.abs(), F32, "y")
        r2 = r.clone()
        assert rcd.linear(a, w, residual=r2, out=r2, out_dtype=F32) is r2 and torch.equal(r2, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows_at_all(dtype):
    a, w = torch.empty(0, 40, dtype=dtype, device="cuda"), torch.randn(24, 40, device="cuda").to(dtype)
    y, z = rcd.linear(a, w, want_preact=True)
    assert y.shape == (0, 24) and z.shape == (0, 24)
    da, dw, db = rcd.linear_backward(y, a, w, z)
    assert da.shape == (0, 40) and torch.all(dw == 0) and torch.all(db == 0)
    h, saved = rcd.gated_linear(a, w, w, want_saved=True)
    da, dwg, dwu = rcd.gated_linear_backward(h, a, w, w, saved)
    assert h.shape == (0, 24) and torch.all(dwg == 0) and torch.all(dwu == 0)


@pytest.mark.parametrize("M", [3, 70, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nans_travel_as_the_formula_says(M, dtype):
    """A lone infinity makes its row's results infinite, opposite ones and NaN make them NaN; no other row sees them."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    K, N = 200, 96
    a, w = normal(gen, M, K, dtype=dtype), normal(gen, N, K, dtype=dtype, scale=K ** -0.5)
    w[5] = 0.5                                        # exactly representable: its lower pieces are zero
    a[0, 17] = float("inf")
    a[1, 3], a[1, 150] = float("inf"), float("-inf")
    a[2, 199] = float("nan")
    w[7, 0] = float("-inf")
    z, y = ref.linear(a.double(), w.double(), None, "none", None)
    got = rcd.linear(a, w)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[:3] = True
    bad[:, 7] = True
    clean_a, clean_w = a.double().nan_to_num(0, 0, 0), w.double().nan_to_num(0, 0, 0)
    bound = ref.linear_error(clean_a, clean_w, None, "none", clean_a @ clean_w.t())[1]
    check(got, y, bound, dtype, "y")
    assert torch.all(torch.isfinite(got[~bad])) and torch.isinf(got[0, 5]) and got[0, 5] > 0
    # large finite values stay finite where the sum does
    big = torch.full((M, 8), 3.0e38, device="cuda").to(dtype)
    eighth = torch.full((4, 8), 0.03125, device="cuda").to(dtype)
    assert torch.all(torch.isfinite(rcd.linear(big, eighth)))
    # a gradient's infinity stays in its own row of dA
    dy = normal(gen, M, N, dtype=dtype)
    dy[0, 2] = float("inf")
    w[7, 0] = 0.0
    da, dw, db = rcd.linear_backward(dy, a.nan_to_num(0, 0, 0), w)
    dz, da_ref, dw_ref, db_ref = ref.linear_backward(dy.double(), a.nan_to_num(0, 0, 0).double(), w.double(), z, "none")
    assert torch.equal(torch.isfinite(da), torch.isfinite(da_ref)) and torch.equal(torch.isnan(da), torch.isnan(da_ref))
    assert torch.equal(torch.isfinite(dw), torch.isfinite(dw_ref)) and torch.isinf(db[2])


def test_offsets_pass_32_bits():
    """Rows over 2^31 elements apart."""
    pitch = (1 << 31) // 2 + 64
    room = torch.zeros(3 * pitch, dtype=BF16, device="cuda")
    a = room.view(3, pitch)[:, :136]
    gen = torch.Generator(device="cuda").manual_seed(1)
    a.copy_(normal(gen, 3, 136, dtype=BF16))
    w = normal(gen, 40, 136, dtype=BF16)
    assert torch.equal(rcd.linear(a, w), rcd.linear(a.contiguous(), w))
    assert torch.equal(rcd.rms_norm(a).y, rcd.rms_norm(a.contiguous()).y)
    many = normal(gen, 600, 136, dtype=BF16)
    assert torch.equal(rcd.linear(many, a), rcd.linear(many, a.contiguous()))
    h, saved = rcd.gated_linear(many, a, a, want_saved=True)
    back = rcd.gated_linear_backward(h, many, a, a, saved)
    for x, y in zip(back, rcd.gated_linear_backward(h, many, a.contiguous(), a.contiguous(), saved)):
        assert torch.equal(x, y)


def test_gradients_against_differences():
    """Central differences of the forward calls (fp32, step 2^-6 along random directions): loss = sum(y * c)."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    M, N, K, step = 20, 24, 30, 2.0 ** -6

    def along(f, t, grad):
        v = normal(gen, *t.shape)
        slope = (f(t + step * v) - f(t - step * v)) / (2 * step)
        want = (grad.double() * v.double()).sum().item()
        # the third derivative of these smooth functions times step^2 / 6 stays below 1e-3 of the directions' size
        size = (grad.double().norm() * v.double().norm()).item()
        assert abs(slope - want) <= 2e-3 * size, (slope, want, size)

    a, w, w2 = normal(gen, M, K), normal(gen, N, K, scale=K ** -0.5), normal(gen, N, K, scale=K ** -0.5)
    b, c, r = normal(gen, N, scale=0.1), normal(gen, M, N), normal(gen, M, K)
    for act in ("none", "silu", "gelu"):
        loss = lambda a_, w_, b_: (rcd.linear(a_, w_, b_, act=act).double() * c.double()).sum().item()  # noqa: E731
        _, z = rcd.linear(a, w, b, act=act, want_preact=True)
        da, dw, db = rcd.linear_backward(c, a, w, z, act=act)
        along(lambda t: loss(t, w, b), a, da)
        along(lambda t: loss(a, t, b), w, dw)
        along(lambda t: loss(a, w, t), b, db)
        loss = lambda a_, g_, u_: (rcd.gated_linear(a_, g_, u_, act=act).double() * c.double()).sum().item()  # noqa: E731
        _, saved = rcd.gated_linear(a, w, w2, act=act, want_saved=True)
        da, dg, du = rcd.gated_linear_backward(c, a, w, w2, saved, act=act)
        along(lambda t: loss(t, w, w2), a, da)
        along(lambda t: loss(a, t, w2), w, dg)
        along(lambda t: loss(a, w, t), w2, du)
    scale, cy, cs = 1 + 0.1 * normal(gen, K), normal(gen, M, K), normal(gen, M, K)

    def loss(x_, w_):
        n = rcd.rms_norm(x_, w_, EPS, residual=r, want_sum=True)
        return (n.y.double() * cy.double() + n.sum.double() * cs.double()).sum().item()

    n = rcd.rms_norm(a, scale, EPS, residual=r, want_sum=True, want_rstd=True)
    dx, dw = rcd.rms_norm_backward(cy, n.sum, n.rstd, scale, dsum=cs)
    along(lambda t: loss(t, scale), a, dx)
    along(lambda t: loss(a, t), scale, dw)


def layer(x, r, p):
    """One encoder layer, forward and backward, as a training step runs it."""
    n = rcd.rms_norm(x, p["scale"], EPS, residual=r, want_sum=True, want_rstd=True)
    h, saved = rcd.gated_linear(n.y, p["wg"], p["wu"], want_saved=True)
    y = rcd.linear(h, p["wd"], residual=n.sum)
    dh, dwd, _ = rcd.linear_backward(y, h, p["wd"], want_dbias=False)
    da, dwg, dwu = rcd.gated_linear_backward(dh, n.y, p["wg"], p["wu"], saved)
    dx, dscale = rcd.rms_norm_backward(da, n.sum, n.rstd, p["scale"], dsum=y)
    return [y, dx, dscale, dwg, dwu, dwd]


def layer_inputs(seed, M, K, F, dtype):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    p = {"scale": (1 + 0.1 * normal(gen, K)).to(dtype), "wg": normal(gen, F, K, dtype=dtype, scale=K ** -0.5),
         "wu": normal(gen, F, K, dtype=dtype, scale=K ** -0.5), "wd": normal(gen, K, F, dtype=dtype, scale=F ** -0.5)}
    return normal(gen, M, K, dtype=dtype), normal(gen, M, K, dtype=dtype), p


@pytest.mark.parametrize("M,K,F,dtype", [(300, 256, 640, BF16), (5, 256, 640, BF16), (130, 120, 200, F32)])
def test_same_inputs_give_the_same_bits_on_any_stream_and_in_a_graph(M, K, F, dtype):
    x, r, p = layer_inputs(M, M, K, F, dtype)
    want = layer(x, r, p)
    for a, b in zip(want, layer(x, r, p)):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer(x, r, p)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer(x, r, p)
    for turn in range(4):
        x2, r2, _ = layer_inputs(50 + turn, M, K, F, dtype)
        x.copy_(x2)
        r.copy_(r2)
        eager = [t.clone() for t in layer(x2, r2, p)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            assert torch.equal(a, b), turn


def test_rows_beside_the_output_are_left_alone():
    gen = torch.Generator(device="cuda").manual_seed(9)
    for M in (2, 150):
        a, w = normal(gen, M, 64, dtype=BF16), normal(gen, 50, 64, dtype=BF16)
        room = torch.full((M + 2, 61), 7.0, dtype=BF16, device="cuda")
        rcd.linear(a, w, out=room[1:-1, 5:55])
        assert torch.equal(room[1:-1, 5:55], rcd.linear(a, w))
        assert torch.all(room[0] == 7) and torch.all(room[-1] == 7) and torch.all(room[:, :5] == 7) and torch.all(room[:, 55:] == 7)


def test_a_given_workspace_is_enough_and_a_smaller_one_is_refused():
    gen = torch.Generator(device="cuda").manual_seed(8)
    lib = rcd.load_library()
    M, N, K = 200, 100, 70
    a, w, dy = normal(gen, M, K), normal(gen, N, K), normal(gen, M, N)
    need = lib.rcd_linear_backward_workspace_bytes(M, N, K, 0)
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")      # NaN wherever it is read before it is written
    for x, y in zip(rcd.linear_backward(dy, a, w, workspace=ws[:need]), rcd.linear_backward(dy, a, w)):
        assert torch.equal(x, y) and torch.all(torch.isfinite(x))
    assert torch.all(ws[need:] == 0xff)
    with pytest.raises(rcd.RcdError) as e:
        rcd.linear_backward(dy, a, w, workspace=ws[: need - 256])
    assert e.value.status == 5
