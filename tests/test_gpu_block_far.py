"""The operators around the scan on maps whose offsets pass 32 bits: the last rows of the last planes against the 64-bit form of those rows alone."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu


def _room(nbytes):
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip("not enough device memory")


@pytest.mark.parametrize("W", [8192, 8191])
def test_projection_of_a_map_of_many_gigabytes(W):
    """64 channels of 16384 x W in bf16: an image of 2^33 values (16 GB).  gout is zero but for the last rows, so that these alone make the matrix's gradient."""
    import paper_2512_07884_amd as G
    _room(90 << 30)
    K, M, H, last = 64, 16, 16384, 2
    print(f"far product K{K} M{M} {H}x{W}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1, K, H, W, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    P = (torch.randn(M, K, generator=gen, device="cuda") / 8).bfloat16()
    b = torch.randn(M, generator=gen, device="cuda").bfloat16()
    out = torch.empty(1, M, H, W, device="cuda", dtype=torch.bfloat16)
    G.gspn_proxy_project_fused(x, P, out, bias=b, act=G.GSPN_ACT_SILU)
    torch.cuda.synchronize()
    tail = lambda t: t[:, :, -last:].double().cpu()
    g = torch.zeros_like(out)
    g[:, :, -last:] = torch.randn(1, M, last, W, generator=gen, device="cuda").bfloat16()
    val, err = R.product(tail(x), P.double().cpu(), b.double().cpu(), None, tail(g), "silu", "bf16", False)
    R.check({"out": tail(out)}, val, err, ("far", W))
    gin, gP, gb = torch.empty_like(x), torch.empty_like(P), torch.empty_like(b)
    G.gspn_proxy_project_fused_bwd(g, x, P, gin, gP, gb, bias=b, act=G.GSPN_ACT_SILU)
    torch.cuda.synchronize()
    assert (gin[0, K - 1, :-last] == 0).all()
    R.check({"gin": tail(gin), "gP": gP, "gbias": gb}, val, err, ("far", W))


def test_attention_of_a_map_of_many_gigabytes():
    """One head of 72 channels on 8192 x 8191 positions (2^32 values and more), seven tokens."""
    import paper_2512_07884_amd as G
    _room(60 << 30)
    D, H, W, L, last = 72, 8191, 8191, 7, 2
    print(f"far attention D{D} {H}x{W} L{L}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.empty(1, D, H, W, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    k, v = (torch.randn(1, L, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty(1, 1, H, W, device="cuda")
    G.gspn_cross_attention(q, k, v, out, lse, heads=1)
    torch.cuda.synchronize()
    tail = lambda t: t[:, :, -last:].double().cpu()
    g = torch.zeros_like(q)
    g[:, :, -last:] = torch.randn(1, D, last, W, generator=gen, device="cuda").bfloat16()
    val, err = R.attend(tail(q), k.double().cpu(), v.double().cpu(), None, tail(g), 1, 1, D ** -0.5, "bf16")
    R.check({"out": tail(out), "lse": tail(lse)}, val, err, "far")
    gq, gk, gv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    G.gspn_cross_attention_bwd(g, q, k, v, out, lse, gq, gk, gv, heads=1)
    torch.cuda.synchronize()
    assert (gq[0, D - 1, :-last] == 0).all()
    R.check({"gq": tail(gq), "gk": gk, "gv": gv}, val, err, "far")
