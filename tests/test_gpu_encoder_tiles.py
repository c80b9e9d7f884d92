"""GPU tests of the encoder's products at sizes that reach every cut of the tile kernels (encoder_shapes.py), against plain
64-bit forms with the bounds derived in encoder_reference.py."""
import pytest
import torch

import encoder_reference as ref
import paper_2211_00839_amd as rcd
from encoder_shapes import TILES, TILES_8_BITS
from test_gpu_encoder import BF16, F32, check, layer, layer_inputs, mx, normal, strided

pytestmark = pytest.mark.gpu


def laid_out(i):
    """In place, with padded rows, and with rows that start and end anywhere."""
    return [lambda t: t, lambda t: strided(t, -(-t.shape[1] // 8) * 8 + 8), lambda t: strided(t, t.shape[1] + 1, 3)][i % 3]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(TILES)))
def test_linear_and_its_gradients(i, dtype):
    M, N, K = TILES[i]
    gen = torch.Generator(device="cuda").manual_seed(1000 + i)
    lay = laid_out(i)
    act = ["gelu", "silu", "relu", "none"][i % 4]
    print("linear", M, N, K, dtype, act, flush=True)
    a, w, b = lay(normal(gen, M, K, dtype=dtype)), lay(normal(gen, N, K, dtype=dtype, scale=K ** -0.5)), normal(gen, N, dtype=dtype, scale=0.2)
    r, dy = lay(normal(gen, M, N, dtype=dtype)), lay(normal(gen, M, N, dtype=dtype))
    y, z = rcd.linear(a, w, b, act=act, residual=r, want_preact=True)
    ad, wd, dyd = a.double(), w.double(), dy.double()
    z_ref, y_ref = ref.linear(ad, wd, b.double(), act, r.double())
    ez, ev = ref.linear_error(ad, wd, b.double(), act, z_ref)
    check(z, z_ref, ez, F32, "z")
    check(y, y_ref, ev + ref.U32 * y_ref.abs(), dtype, "y")
    assert torch.equal(y, rcd.linear(a, w, b, act=act, residual=r))
    da, dw, db = rcd.linear_backward(dy, a, w, z, act=act)
    dz, da_ref, dw_ref, db_ref = ref.linear_backward(dyd, ad, wd, z_ref, act)
    edz = dyd.abs() * ref.act_error(z_ref, ez, act)[1] + 2 * ref.U32 * dz.abs()
    rounded = edz + (0 if dtype == F32 or act == "none" else ref.U16 * (dz.abs() + edz))
    check(da, da_ref, rounded @ wd.abs() + ref.sum_error(N, (dz.abs() + edz) @ wd.abs()), dtype, "da")
    check(dw, dw_ref, rounded.t() @ ad.abs() + ref.sum_error(M, (dz.abs() + edz).t() @ ad.abs()), dtype, "dw")
    check(db[None], db_ref[None], (edz.sum(0) + ref.sum_error(M, (dz.abs() + edz).sum(0)))[None], dtype, "db")
    assert torch.equal(rcd.linear_backward(dy, a, w, z, act=act, want_dw=False)[0], da)
    assert torch.equal(rcd.linear_backward(dy, a, w, z, act=act, want_da=False, want_dbias=False)[1], dw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(TILES)))
def test_gated_and_its_gradients(i, dtype):
    M, F, K = TILES[i]
    gen = torch.Generator(device="cuda").manual_seed(1100 + i)
    lay, other = laid_out(i), laid_out(i + (i % 2))       # (every other time the two weights are laid out differently)
    act = ["silu", "gelu"][i % 2]
    print("gated", M, F, K, dtype, act, flush=True)
    a, wg, wu = lay(normal(gen, M, K, dtype=dtype)), lay(normal(gen, F, K, dtype=dtype, scale=K ** -0.5)), other(normal(gen, F, K, dtype=dtype, scale=K ** -0.5))
    dh = lay(normal(gen, M, F, dtype=dtype))
    h, saved = rcd.gated_linear(a, wg, wu, act=act, want_saved=True)
    ad, wgd, wud, dhd = a.double(), wg.double(), wu.double(), dh.double()
    g, u, h_ref = ref.gated(ad, wgd, wud, act)
    eg, eu = (ref.sum_error(K, ad.abs() @ w.abs().t()) for w in (wgd, wud))
    ev, es = ref.act_error(g, eg, act)
    value, slope = ref.act_both(g, act)
    check(saved[..., 0], g, eg, F32, "g")
    check(saved[..., 1], u, eu, F32, "u")
    check(h, h_ref, ev * (u.abs() + eu) + value.abs() * eu + 2 * ref.U32 * h_ref.abs(), dtype, "h")
    assert torch.equal(h, rcd.gated_linear(a, wg, wu, act=act))
    da, dwg, dwu = rcd.gated_linear_backward(dh, a, wg, wu, saved, act=act)
    dg, du, da_ref, dwg_ref, dwu_ref = ref.gated_backward(dhd, ad, wgd, wud, g, u, act)
    edg = dhd.abs() * (es * (u.abs() + eu) + slope.abs() * eu) + 4 * ref.U32 * dg.abs()
    edu = dhd.abs() * ev + 2 * ref.U32 * du.abs()
    more = 0 if dtype == F32 else ref.U16
    rg, ru = edg + more * (dg.abs() + edg), edu + more * (du.abs() + edu)
    mg, mu = dg.abs() + edg, du.abs() + edu
    check(da, da_ref, rg @ wgd.abs() + ru @ wud.abs() + ref.sum_error(2 * F, mg @ wgd.abs() + mu @ wud.abs()), dtype, "da")
    check(dwg, dwg_ref, rg.t() @ ad.abs() + ref.sum_error(M, mg.t() @ ad.abs()), dtype, "dw_gate")
    check(dwu, dwu_ref, ru.t() @ ad.abs() + ref.sum_error(M, mu.t() @ ad.abs()), dtype, "dw_up")
    only = rcd.gated_linear_backward(dh, a, wg, wu, saved, act=act, want_da=False)
    assert torch.equal(only[1], dwg) and torch.equal(only[2], dwu)


@pytest.mark.parametrize("i", range(len(TILES_8_BITS)))
def test_products_of_8_bit_operands(i):
    M, N, K = TILES_8_BITS[i]
    gen = torch.Generator(device="cuda").manual_seed(1200 + i)
    print("8 bits", M, N, K, flush=True)

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
    b, r = normal(gen, N, dtype=BF16), normal(gen, M, N, dtype=BF16)
    y = rcd.linear(a, w, b, residual=r, a_scale=sa, w_scale=sw)
    z_ref, y_ref = ref.linear(ad, wd, b.double(), "none", r.double())
    ez, ev = ref.linear_error(ad, wd, b.double(), "none", z_ref)
    check(y, y_ref, ev + ref.U32 * y_ref.abs(), BF16, "y")
    h = rcd.gated_linear(a, w, w2, a_scale=sa, gate_scale=sw, up_scale=sw2)
    g, u, h_ref = ref.gated(ad, wd, w2d, "silu")
    eg, eu = (ref.sum_error(K, ad.abs() @ v.abs().t()) for v in (wd, w2d))
    ev, _ = ref.act_error(g, eg, "silu")
    check(h, h_ref, ev * (u.abs() + eu) + ref.act_both(g, "silu")[0].abs() * eu + 2 * ref.U32 * h_ref.abs(), BF16, "h")


@pytest.mark.parametrize("M,N,K", [(4104, 2056, 200), (600, 700, 2000), (2600, 1400, 520)])
def test_infinities_and_nans_in_products_of_pieces(M, N, K):
    """fp32 operands in pieces: a lone infinity makes its row's results infinite (a piece that is zero must not make them
    NaN), opposite ones and NaN make them NaN, values near the largest stay finite; no other row sees any of it."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    a, w = normal(gen, M, K), normal(gen, N, K, scale=K ** -0.5)
    w[5] = 0.5
    a[0, 17] = float("inf")
    a[1, 3], a[1, 150] = float("inf"), float("-inf")
    a[2, 199] = float("nan")
    a[M - 1, 0] = float("-inf")
    w[7, 0] = float("-inf")
    a[9] = 0.0
    a[9, 11] = 3.0e38
    z, y = ref.linear(a.double(), w.double(), None, "none", None)
    got = rcd.linear(a, w)
    clean_a, clean_w = a.double().nan_to_num(0, 0, 0), w.double().nan_to_num(0, 0, 0)
    bound = ref.linear_error(clean_a, clean_w, None, "none", clean_a @ clean_w.t())[1]
    check(got, y, bound, F32, "y")
    assert torch.isinf(got[0, 5]) and got[0, 5] > 0 and torch.isfinite(got[9, 5])
    h, saved = rcd.gated_linear(a, w, w, act="none", want_saved=True)
    check(saved[..., 0], y, bound, F32, "g")
    check(saved[..., 1], y, bound, F32, "u")
    ok = a.nan_to_num(0, 0, 0).clamp(-10, 10)
    w[7, 0] = 0.0
    dy = normal(gen, M, N)
    dy[0, 2] = float("inf")
    dy[3, 5] = float("nan")
    da, dw, db = rcd.linear_backward(dy, ok, w)
    _, da_ref, dw_ref, db_ref = ref.linear_backward(dy.double(), ok.double(), w.double(), z, "none")
    for x, want in ((da, da_ref), (dw, dw_ref), (db, db_ref)):
        assert torch.equal(torch.isnan(x), torch.isnan(want)) and torch.equal(torch.isinf(x), torch.isinf(want))
        assert torch.equal(x[torch.isinf(x)].double(), want[torch.isinf(want)])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tiles_give_the_same_bits_on_any_stream_and_in_a_graph(dtype):
    M, K, F = 2100, 520, 1400
    x, r, p = layer_inputs(7, M, K, F, dtype)
    want = layer(x, r, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer(x, r, p)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer(x, r, p)
    for turn in range(3):
        x2, r2, _ = layer_inputs(60 + turn, M, K, F, dtype)
        x.copy_(x2)
        r.copy_(r2)
        eager = [t.clone() for t in layer(x2, r2, p)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            assert torch.equal(a, b), turn


def test_rows_beside_a_large_result_are_left_alone():
    gen = torch.Generator(device="cuda").manual_seed(9)
    for M, N, K in ((4104, 2056, 72), (600, 700, 2000)):
        a, w = normal(gen, M, K, dtype=BF16), normal(gen, N, K, dtype=BF16)
        room = torch.full((M + 2, N + 11), 7.0, dtype=BF16, device="cuda")
        rcd.linear(a, w, out=room[1:-1, 5:N + 5])
        assert torch.equal(room[1:-1, 5:N + 5], rcd.linear(a, w))
        assert torch.all(room[0] == 7) and torch.all(room[-1] == 7) and torch.all(room[:, :5] == 7) and torch.all(room[:, N + 5:] == 7)


def test_workspaces_full_of_nan_do_not_show():
    """What is read of a workspace has been written before, in every route."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    lib = rcd.load_library()
    for M, N, K in ((4104, 2056, 200), (700, 300, 4000), (300, 520, 1100)):
        for dtype, code in ((F32, 0), (BF16, 1)):
            a, w, dy = strided(normal(gen, M, K, dtype=dtype), K + 1), normal(gen, N, K, dtype=dtype, scale=K ** -0.5), normal(gen, M, N, dtype=dtype)

            def dirty(need):
                return torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")

            ws = dirty(lib.rcd_linear_workspace_bytes(M, N, K, code))
            assert torch.equal(rcd.linear(a, w, workspace=ws[:-256]), rcd.linear(a, w)) and torch.all(ws[-256:] == 0xff)
            ws = dirty(lib.rcd_linear_backward_workspace_bytes(M, N, K, code))
            for x, y in zip(rcd.linear_backward(dy, a, w, workspace=ws[:-256]), rcd.linear_backward(dy, a, w)):
                assert torch.equal(x, y) and torch.all(torch.isfinite(x))
            assert torch.all(ws[-256:] == 0xff)
            ws = dirty(lib.rcd_gated_linear_workspace_bytes(M, N, K, code))
            h, saved = rcd.gated_linear(a, w, w, want_saved=True)
            assert torch.equal(rcd.gated_linear(a, w, w, workspace=ws[:-256]), h) and torch.all(ws[-256:] == 0xff)
            ws = dirty(lib.rcd_gated_linear_backward_workspace_bytes(M, N, K, code))
            for x, y in zip(rcd.gated_linear_backward(dy, a, w, w, saved, workspace=ws[:-256]), rcd.gated_linear_backward(dy, a, w, w, saved)):
                assert torch.equal(x, y) and torch.all(torch.isfinite(x))
            assert torch.all(ws[-256:] == 0xff)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("over", [1, 31, 32, 33, 68, 129, 224, 255])
def test_rows_of_a_tile_that_is_not_full_are_the_full_ones(dtype, over):
    """A row's results do not depend on how many rows come after it in its tile: the same bits with `over` of a tile's rows as
    with all of them, whether the bands of 32 rows that hold them are full or not, infinities among them."""
    M, N, K, full = 4096 + over, 2056, 200, 4352
    gen = torch.Generator(device="cuda").manual_seed(over)
    a, w, w2 = normal(gen, full, K, dtype=dtype), normal(gen, N, K, dtype=dtype, scale=K ** -0.5), normal(gen, N, K, dtype=dtype, scale=K ** -0.5)
    b, r = normal(gen, N, dtype=dtype), normal(gen, full, N, dtype=dtype)
    a[4100, 7] = a[4350, 3] = float("inf")
    for x, y in zip(rcd.linear(a[:M], w, b, act="gelu", residual=r[:M], want_preact=True),
                    rcd.linear(a, w, b, act="gelu", residual=r, want_preact=True)):
        assert torch.equal(torch.nan_to_num(x, 1e9, 2e9, -2e9), torch.nan_to_num(y[:M], 1e9, 2e9, -2e9))
        assert torch.equal(torch.isfinite(x).all(1), torch.isfinite(a[:M].float()).all(1))
    for x, y in zip(rcd.gated_linear(a[:M], w, w2, act="silu", want_saved=True), rcd.gated_linear(a, w, w2, act="silu", want_saved=True)):
        assert torch.equal(torch.nan_to_num(x, 1e9, 2e9, -2e9), torch.nan_to_num(y[:M], 1e9, 2e9, -2e9))
