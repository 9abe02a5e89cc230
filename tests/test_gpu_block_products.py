"""The projection with bias, activation and residual and the gated pair, forward and backward, against the plain 64-bit form: every element within the bound
that the roundings give (block_reference.py)."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu


def _dev(t, dtype):
    return None if t is None else t.to(R.TD[dtype]).cuda()


def _case(B, K, M, H, W, dtype, act, bias, residual, gated, seed=0, step=True):
    import paper_2512_07884_amd as G
    print(f"product B{B} K{K} M{M} {H}x{W} {dtype} {act} bias={bias} residual={residual} gated={gated}", flush=True)
    gen = torch.Generator().manual_seed(1000 + seed)
    rows = 2 * M if gated else M
    rnd = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64).to(R.TD[dtype]).double()
    x, P = rnd(B, K, H, W), (rnd(rows, K) * K ** -0.5).to(R.TD[dtype]).double()
    b = rnd(rows) if bias else None
    res = rnd(B, M, H, W) if residual else None
    g = rnd(B, M, H, W) if step else None
    val, err = R.product(x, P, b, res, g, act, dtype, gated)
    code = {"none": G.GSPN_ACT_NONE, "silu": G.GSPN_ACT_SILU, "gelu": G.GSPN_ACT_GELU, "sigmoid": G.GSPN_ACT_SIGMOID}[act]
    dx, dP, db, dr, dg = (_dev(t, dtype) for t in (x, P, b, res, g))
    nan = lambda *s: torch.full(s, float("nan"), dtype=R.TD[dtype], device="cuda")
    got = {"out": nan(B, M, H, W)}
    if gated:
        G.gspn_gated_project(dx, dP, got["out"], bias=db, act=code)
    else:
        G.gspn_proxy_project_fused(dx, dP, got["out"], bias=db, residual=dr, act=code)
    torch.cuda.synchronize()
    if step:
        got.update(gin=nan(B, K, H, W), gP=nan(rows, K), gbias=nan(rows))
        bwd = G.gspn_gated_project_bwd if gated else G.gspn_proxy_project_fused_bwd
        bwd(dg, dx, dP, got["gin"], got["gP"], got["gbias"], bias=db, act=code)
        torch.cuda.synchronize()
    R.check(got, val, err, (B, K, M, H, W, dtype, act, gated))


# one pixel; fewer pixels and channels than a request, a stage, a tile; odd ones around each; several tiles of every kind
SHAPES = [(1, 1, 1, 1, 1), (1, 3, 2, 1, 5), (2, 8, 8, 1, 7), (3, 17, 33, 3, 3), (1, 64, 64, 8, 8), (2, 65, 40, 7, 7), (1, 96, 31, 5, 13), (2, 100, 130, 9, 11),
          (1, 40, 257, 4, 33), (3, 72, 24, 14, 14), (1, 200, 129, 16, 17), (1, 129, 96, 1, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("gated", [False, True], ids=["project", "gated"])
def test_small_and_odd_sizes(shape, dtype, gated):
    i = SHAPES.index(shape)
    _case(*shape, dtype, ("silu", "gelu", "sigmoid", "none")[i % 4], i % 3 != 0, not gated and i % 2 == 0, gated, i)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("gated", [False, True], ids=["project", "gated"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_activation(act, gated, dtype):
    _case(2, 48, 40, 6, 11, dtype, act, True, not gated, gated, 50)
    _case(1, 24, 16, 5, 5, dtype, act, False, False, gated, 51)


# as many tiles as run on each of the tiles: 128x128, 64x64 and 32x128 at the sizes that choose them
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(8, 72, 256, 64, 33), (6, 136, 140, 31, 33), (9, 40, 20, 63, 63)], ids=lambda s: "x".join(map(str, s)))
def test_tiles_of_many(shape, dtype):
    _case(*shape, dtype, "silu", True, True, False, 60)
    if shape[2] < 200:
        _case(*shape, dtype, "gelu", True, False, True, 61)


# every tile with several stages, in 16-byte requests straight to LDS and (odd rows) through registers; 256x256 for the result, the map's gradient and the
# matrix's; 128x128, 64x64 and 64x32; stretches of the pixels over several images
TILES = [(3, 1024, 1024, 64, 64), (1, 3584, 3584, 16, 16), (4, 1152, 1152, 28, 28), (8, 512, 1024, 31, 33), (8, 512, 1024, 32, 32), (20, 96, 96, 56, 56), (20, 96, 96, 55, 57),
         (8, 384, 384, 14, 14), (8, 384, 384, 13, 15), (64, 200, 136, 7, 7), (2, 300, 200, 7, 9)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", TILES, ids=lambda s: "x".join(map(str, s)))
def test_every_tile(shape, dtype):
    _case(*shape, dtype, "silu", True, True, False, 70)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3, 512, 512, 64, 64), (8, 512, 512, 31, 33), (20, 96, 48, 56, 56), (8, 384, 192, 13, 15), (32, 200, 100, 7, 7)], ids=lambda s: "x".join(map(str, s)))
def test_every_tile_of_the_gated_pair(shape, dtype):
    _case(*shape, dtype, "gelu", True, False, True, 71)


def test_large_values_of_the_activations():
    """Far from zero the activations are 0, z or 1, without infinities or NaN."""
    import paper_2512_07884_amd as G
    z = torch.tensor([-1e4, -200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 200.0, 1e4])
    x = z.reshape(1, 1, 1, -1).cuda()
    P = torch.ones(1, 1, device="cuda")
    g = torch.ones_like(x)
    for code, out, slope in ((G.GSPN_ACT_SILU, z.clamp(min=0), (z > 0).float()), (G.GSPN_ACT_GELU, z.clamp(min=0), (z > 0).float()), (G.GSPN_ACT_SIGMOID, (z > 0).float(), z * 0)):
        y, gx, gP, gb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(P), torch.empty(1, device="cuda")
        G.gspn_proxy_project_fused(x, P, y, act=code)
        G.gspn_proxy_project_fused_bwd(g, x, P, gx, gP, gb, act=code)
        torch.cuda.synchronize()
        away = z != 0
        # at |z| = 20: silu is off its limits by 20 exp(-20) = 4.2e-8, sigmoid by 2.1e-9
        assert torch.allclose(y.cpu().flatten()[away], out[away], rtol=2.0 ** -20, atol=5e-8), code
        assert torch.allclose(gx.cpu().flatten()[away], slope[away], rtol=2.0 ** -20, atol=5e-8), code
        assert torch.isfinite(gP).all() and torch.isfinite(gb).all()


@pytest.mark.parametrize("gated", [False, True], ids=["project", "gated"])
def test_gradients_asked_for_one_by_one(gated):
    """Each of gin, gP, gbias alone is what the call for all of them gives, bit for bit; twice the same bits."""
    import paper_2512_07884_amd as G
    gen = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    B, K, M, H, W = 3, 72, 48, 13, 15
    rows = 2 * M if gated else M
    x, P, b, g = rnd(B, K, H, W), rnd(rows, K), rnd(rows), rnd(B, M, H, W)
    bwd = G.gspn_gated_project_bwd if gated else G.gspn_proxy_project_fused_bwd
    for act in (G.GSPN_ACT_SILU, G.GSPN_ACT_NONE):
        new = lambda: [torch.full_like(t, float("nan")) for t in (x, P, b)]
        whole, again = new(), new()
        bwd(g, x, P, *whole, bias=b, act=act)
        bwd(g, x, P, *again, bias=b, act=act)
        for i in range(3):
            one = new()
            bwd(g, x, P, *[t if j == i else None for j, t in enumerate(one)], bias=b, act=act)
            torch.cuda.synchronize()
            assert torch.equal(one[i], whole[i]) and torch.equal(again[i], whole[i]), (act, i)


def test_rows_behind_the_outputs_stay_as_they_are():
    """Outputs within a larger allocation: nothing before or after them is written."""
    import paper_2512_07884_amd as G
    for dtype in (torch.bfloat16, torch.float32):
        for (B, K, M, H, W) in ((1, 24, 17, 3, 7), (2, 40, 33, 11, 13), (1, 130, 129, 12, 11)):
            gen = torch.Generator(device="cuda").manual_seed(3)
            rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
            x, P, b, g = rnd(B, K, H, W), rnd(2 * M, K), rnd(2 * M), rnd(B, M, H, W)
            shapes = [(B, M, H, W), (B, K, H, W), (2 * M, K), (2 * M,)]
            pad = 64
            store = [torch.full((2 * pad + torch.Size(s).numel(),), 7.0, dtype=dtype, device="cuda") for s in shapes]
            y, gx, gP, gb = (t[pad:pad + torch.Size(s).numel()].view(s) for t, s in zip(store, shapes))
            G.gspn_gated_project(x, P, y, bias=b)
            G.gspn_gated_project_bwd(g, x, P, gx, gP, gb, bias=b)
            torch.cuda.synchronize()
            for t, s in zip(store, shapes):
                n = torch.Size(s).numel()
                assert (t[:pad] == 7).all() and (t[pad + n:] == 7).all() and torch.isfinite(t.float()).all(), (dtype, s)


def test_what_lies_beyond_the_operands_is_never_used():
    """NaN right behind every operand, which an unmasked tail of a row, a matrix or an image would multiply by zero."""
    import paper_2512_07884_amd as G
    for dtype in (torch.bfloat16, torch.float32):
        B, K, M, H, W = 2, 37, 21, 5, 9
        gen = torch.Generator(device="cuda").manual_seed(4)

        def fenced(*s):
            n = torch.Size(s).numel()
            t = torch.full((n + 128,), float("nan"), dtype=dtype, device="cuda")
            t[64:64 + n] = torch.randn(n, generator=gen, device="cuda").to(dtype)
            return t[64:64 + n].view(s)

        x, P, b, g, r = fenced(B, K, H, W), fenced(M, K), fenced(M), fenced(B, M, H, W), fenced(B, M, H, W)
        y, gx, gP, gb = torch.empty_like(g), torch.empty_like(x), torch.empty_like(P), torch.empty_like(b)
        G.gspn_proxy_project_fused(x, P, y, bias=b, residual=r, act=G.GSPN_ACT_GELU)
        G.gspn_proxy_project_fused_bwd(g, x, P, gx, gP, gb, bias=b, act=G.GSPN_ACT_GELU)
        torch.cuda.synchronize()
        assert all(torch.isfinite(t.float()).all() for t in (y, gx, gP, gb)), dtype
