"""Cross attention of a map's positions to tokens, forward and backward, against the plain 64-bit form: every element within the bound that the roundings give
(block_reference.py)."""
import math

import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu


def _inputs(B, heads, kv, D, H, W, L, dtype, seed, spread=1.0):
    gen = torch.Generator().manual_seed(2000 + seed)
    rnd = lambda *s: (torch.randn(s, generator=gen, dtype=torch.float64) * spread).to(R.TD[dtype]).double()
    return rnd(B, heads * D, H, W), rnd(B, L, kv * D), rnd(B, L, kv * D), rnd(B, heads * D, H, W), gen


def _run(q, k, v, mask, g, heads, kv, scale, dtype, workspace=True):
    import paper_2512_07884_amd as G
    td = R.TD[dtype]
    dq, dk, dv, dg = (None if t is None else t.to(td).cuda() for t in (q, k, v, g))
    dm = None if mask is None else mask.cuda()
    B, _, H, W = q.shape
    nan = lambda t: torch.full_like(t, float("nan"))
    got = {"out": nan(dq), "lse": torch.full((B, heads, H, W), float("nan"), device="cuda")}
    kw = {"heads": heads, "kv_heads": kv, "mask": dm, "scale": scale}
    if not workspace:
        kw["workspace"] = None
    G.gspn_cross_attention(dq, dk, dv, got["out"], got["lse"], **kw)
    torch.cuda.synchronize()
    if g is not None:
        got.update(gq=nan(dq), gk=nan(dk), gv=nan(dv))
        G.gspn_cross_attention_bwd(dg, dq, dk, dv, got["out"], got["lse"], got["gq"], got["gk"], got["gv"], **kw)
        torch.cuda.synchronize()
    return got


def _case(B, heads, kv, D, H, W, L, dtype, mask=None, seed=0, scale=None, spread=1.0, step=True):
    print(f"attend B{B} heads{heads}/{kv} D{D} {H}x{W} L{L} {dtype} mask={mask}", flush=True)
    q, k, v, g, gen = _inputs(B, heads, kv, D, H, W, L, dtype, seed, spread)
    m = None
    if mask == "padded":
        n = torch.randint(1, L + 1, (B, 1), generator=gen)
        m = torch.arange(L) < n
    elif mask == "holes":
        m = torch.rand((B, L), generator=gen) > 0.5
        m[0] = False                                     # an image without a token
        if B > 1:
            m[1, L - 1] = True
    elif mask == "last":
        m = torch.arange(L).expand(B, L) == L - 1
    scale = D ** -0.5 if scale is None else scale
    if not step:
        g = None
    val, err = R.attend(q, k, v, m, g, heads, kv, scale, dtype)
    R.check(_run(q, k, v, None if m is None else m.contiguous(), g, heads, kv, scale, dtype), val, err, (B, heads, kv, D, H, W, L, dtype, mask))


LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 77, 127, 128, 129, 200, 300]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("L", LENGTHS)
def test_lengths(L, dtype):
    i = LENGTHS.index(L)
    _case(2, 2, (1, 2)[i % 2], (64, 40, 32)[i % 3], 5, 7, L, dtype, (None, "padded", "holes")[i % 3], i)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", list(range(8, 129, 8)))
def test_head_sizes(D, dtype):
    _case(1, 2, 1, D, 3, 13, 40 + D, dtype, "padded", D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 31), (1, 32), (3, 11), (8, 8), (5, 13), (1, 129), (16, 17)], ids=str)
def test_map_sizes(shape, dtype):
    _case(2, 4, 2, 24, *shape, 50, dtype, "padded", shape[1])


# the forms of the forward kernel: 64 and 32 positions per wave (many positions), the waves on the tokens, stretches of the tokens; of the backward call 1,
# 2 and 4 waves along the tokens, several stretches of the positions
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [16, 64, 96, 128])
@pytest.mark.parametrize("shape", [(4, 16, 16, 47, 47, 3), (4, 16, 8, 31, 17, 70), (1, 4, 2, 3, 3, 1500)], ids=["many", "some", "few"])
def test_forms(shape, D, dtype):
    B, heads, kv, H, W, L = shape
    if H > 40:
        B, heads, kv = (2, 8, 8) if D > 16 else (B, heads, kv)
        H, W = (91, 91) if D > 16 else (H, W)
    _case(B, heads, kv, D, H, W, L, dtype, "padded", D, step=D in (16, 64) or H < 40)


# many positions: a head's tokens in LDS for four and eight waves with several turns, and more tokens than LDS holds (16 bits: D 128, 300 of them), in both calls;
# odd positions, positions short of a wave's 32
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(2, 16, 16, 128, 32, 32, 300), (2, 16, 4, 128, 31, 33, 301), (2, 16, 8, 64, 47, 47, 200), (1, 32, 32, 104, 27, 31, 700),
                                   (4, 16, 16, 32, 31, 31, 90), (1, 8, 4, 104, 3, 5, 700)], ids=str)
def test_tokens_in_lds_and_streamed(shape, dtype):
    _case(*shape, dtype, "padded", shape[6], step=True)


@pytest.mark.parametrize("per", [1, 2, 4, 7])
@pytest.mark.parametrize("positions", [1, 5, 33])
def test_few_positions_over_many_tokens(per, positions):
    for mask in (None, "holes", "last"):
        _case(2, 2 * per, 2, 64, 1, positions, 2100, "bf16", mask, per, step=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("mask", ["holes", "last"])
def test_masks(mask, dtype):
    for L in (1, 5, 64, 100, 161):
        _case(3, 2, 1, 32, 6, 7, L, dtype, mask, L)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_and_flat_scores(dtype):
    _case(1, 2, 2, 32, 6, 6, 90, dtype, None, 1, scale=1e-3)
    _case(1, 2, 2, 32, 6, 6, 90, dtype, "padded", 2, scale=0.7, spread=1.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_what_masked_tokens_hold_is_never_used(dtype):
    """NaN and infinities at tokens that take no part change no bit of any output, and get gradients of 0."""
    import paper_2512_07884_amd as G
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    for L, shape in ((50, (4, 5)), (100, (1, 3)), (1400, (2, 2)), (300, (20, 30))):
        B, heads, D = 2, 2, 40
        q, g = rnd(B, heads * D, *shape), rnd(B, heads * D, *shape)
        k, v = rnd(B, L, heads * D), rnd(B, L, heads * D)
        mask = torch.rand((B, L), generator=gen, device="cuda") > 0.4
        mask[:, 3] = True
        res = []
        for bad in (0.0, float("nan"), float("inf"), -float("inf")):
            kk, vv = (torch.where(mask[:, :, None], t, torch.full((), bad, dtype=dtype, device="cuda")) for t in (k, v))
            out, lse = torch.empty_like(q), torch.empty(B, heads, *shape, device="cuda")
            gq, gk, gv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
            G.gspn_cross_attention(q, kk, vv, out, lse, heads=heads, mask=mask)
            G.gspn_cross_attention_bwd(g, q, kk, vv, out, lse, gq, gk, gv, heads=heads, mask=mask)
            torch.cuda.synchronize()
            assert (gk[~mask] == 0).all() and (gv[~mask] == 0).all(), (dtype, L, bad)
            res.append([t.clone() for t in (out, lse, gq, gk, gv)])
        for other in res[1:]:
            assert all(torch.equal(a, b) for a, b in zip(res[0], other)), (dtype, L)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("L, D, shape", [(80, 8, (9, 11)), (77, 64, (8, 8)), (200, 72, (5, 13)), (900, 128, (6, 9))], ids=str)
def test_gradient_of_q_where_few_tokens_take_part(L, D, shape, dtype):
    """A batch padded to L of which an image has 1, 2, 3, 10 or 64 tokens: gq has its own rounding alone, not that of out as well (with one token it is zero but for fp32).

    Bounds: the kernel's weights are off by at most 2^-16 (scores of up to 16 in powers of two, a hundred roundings of 2^-24 at the most), its products by less, and ds
    is multiplied to 2^-15 of itself in 16 bits (two roundings of 2^-8 at the worst): 2^-13 of the magnitudes that gq adds, and a rounding of gq."""
    heads, counts = 2, (1, 2, 3, 10, 64)
    B = len(counts)
    q, k, v, g, _ = _inputs(B, heads, heads, D, *shape, L, dtype, 40)
    mask = torch.arange(L)[None] < torch.tensor(counts)[:, None]
    scale = D ** -0.5
    val, _ = R.attend(q, k, v, mask, g, heads, heads, scale, dtype)
    got = _run(q, k, v, mask, g, heads, heads, scale, dtype)["gq"].double().cpu()
    N = shape[0] * shape[1]
    Q, Gm = q.reshape(B, heads, D, N), g.reshape(B, heads, D, N)
    K, V = (t.reshape(B, L, heads, D).permute(0, 2, 1, 3) for t in (k, v))
    p = torch.softmax(torch.where(mask[:, None, :, None], scale * (K @ Q), -math.inf), 2)
    mag = V.abs() @ Gm.abs()
    mag = p * (mag + (p * mag).sum(2, keepdim=True))
    bound = 2.0 ** -13 * scale * (K.abs().transpose(2, 3) @ mag).reshape(q.shape) + R.half(dtype) * val["gq"].abs() + R.TINY[dtype]
    worst = ((got - val["gq"]).abs() - bound).amax((1, 2, 3))
    assert (worst <= 0).all(), (L, D, dtype, worst.tolist())


def test_stretches_give_what_one_pass_gives():
    """The same call with and without the workspace it asks for."""
    import paper_2512_07884_amd as G
    from paper_2512_07884_amd import binding
    gen = torch.Generator(device="cuda").manual_seed(6)
    B, heads, kv, D, L = 1, 8, 2, 64, 3000
    q, k, v = (torch.randn(s, generator=gen, device="cuda") for s in ((B, heads * D, 1, 3), (B, L, kv * D), (B, L, kv * D)))
    assert G.gspn_cross_attention_bytes(B, heads, kv, D, 1, 3, L, 0) > 0
    outs = []
    for nothing in (False, True):
        out, lse = torch.empty_like(q), torch.empty(B, heads, 1, 3, device="cuda")
        if nothing:
            lib = binding.load_library()
            assert lib.gspn_cross_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), None, out.data_ptr(), lse.data_ptr(), None, 0, B, heads, kv, D, 1, 3, L,
                                            D ** -0.5, 0, torch.cuda.current_stream().cuda_stream) == 0
        else:
            G.gspn_cross_attention(q, k, v, out, lse, heads=heads, kv_heads=kv)
        torch.cuda.synchronize()
        outs.append((out, lse))
    # sums of 3000 terms in another order, fp32
    assert torch.allclose(outs[0][0], outs[1][0], rtol=0, atol=3000 * 2.0 ** -24) and torch.allclose(outs[0][1], outs[1][1], rtol=2.0 ** -20)


def test_gradients_asked_for_one_by_one_and_twice():
    import paper_2512_07884_amd as G
    gen = torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    for L in (20, 50, 150):
        q, g, k, v = rnd(2, 64, 9, 11), rnd(2, 64, 9, 11), rnd(2, L, 32), rnd(2, L, 32)
        out, lse = torch.empty_like(q), torch.empty(2, 2, 9, 11, device="cuda")
        G.gspn_cross_attention(q, k, v, out, lse, heads=2, kv_heads=1)
        new = lambda: [torch.full_like(t, float("nan")) for t in (q, k, v)]
        whole, again = new(), new()
        for t in (whole, again):
            G.gspn_cross_attention_bwd(g, q, k, v, out, lse, *t, heads=2, kv_heads=1)
        for i in range(3):
            one = new()
            G.gspn_cross_attention_bwd(g, q, k, v, out, lse, *[t if j == i else None for j, t in enumerate(one)], heads=2, kv_heads=1)
            torch.cuda.synchronize()
            assert torch.equal(one[i], whole[i]) and torch.equal(again[i], whole[i]), (L, i)


def test_gradients_against_differences():
    """Directional derivatives of sum(out * gout) by central differences in 64 bits of the plain form's forward pass."""
    B, heads, kv, D, H, W, L = 2, 4, 2, 16, 3, 5, 21
    q, k, v, g, gen = _inputs(B, heads, kv, D, H, W, L, "f32", 30)
    mask = torch.rand((B, L), generator=gen) > 0.3
    mask[:, 0] = True
    got = _run(q, k, v, mask, g, heads, kv, 0.25, "f32")
    f = lambda a, b, c: float((R.attend(a, b, c, mask, None, heads, kv, 0.25, "f32")[0]["out"] * g).sum())
    for i, name in enumerate(("gq", "gk", "gv")):
        t = [q, k, v]
        step = torch.randn(t[i].shape, generator=gen, dtype=torch.float64)
        lo, hi = list(t), list(t)
        lo[i], hi[i] = t[i] - 1e-5 * step, t[i] + 1e-5 * step
        want = (f(*hi) - f(*lo)) / 2e-5
        have = float((got[name].double().cpu() * step).sum())
        # fp32 gradients of some 1e2 values, each within 1e-5 of its size; the difference itself within 1e-9
        assert abs(want - have) <= 1e-5 * float((got[name].double().cpu().abs() * step.abs()).sum()), name
