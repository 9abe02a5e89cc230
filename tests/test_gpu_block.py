"""The operators around the scan together, as a block uses them: proxy projections and scan, cross attention, feed-forward pair, each added to the map, forward and
backward, eager, captured and on streams of their own."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu

B, C, CP, H, W, GR, HEADS, KV, L, F = 2, 64, 16, 13, 14, 4, 4, 2, 37, 96


class Block:
    """y = x + up(scan(down(x)));  z = y + o(cross attention(q(y)));  out = z + d(gated(z)), parameters and buffers of one dtype."""

    def __init__(self, dtype, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.td = R.TD[dtype]
        rnd = lambda *s, scale=1.0: (torch.randn(s, generator=gen) * scale).to(self.td).cuda()
        self.p = {"down": rnd(CP, C, scale=C ** -0.5), "up": rnd(C, CP, scale=CP ** -0.5), "upb": rnd(C, scale=0.1), "q": rnd(C, C, scale=C ** -0.5),
                  "o": rnd(C, C, scale=C ** -0.5), "ob": rnd(C, scale=0.1), "g": rnd(2 * F, C, scale=C ** -0.5), "gb": rnd(2 * F, scale=0.1),
                  "d": rnd(C, F, scale=F ** -0.5), "db": rnd(C, scale=0.1), "lp": rnd(4 * CP, C, scale=C ** -0.5), "lb": rnd(4 * CP, scale=0.1)}
        self.x, self.k, self.v, self.gout = rnd(B, C, H, W), rnd(B, L, C // HEADS * KV), rnd(B, L, C // HEADS * KV), rnd(B, C, H, W)
        self.mask = (torch.rand((B, L), generator=gen) > 0.3).cuda()
        self.mask[:, 0] = True
        self.z = (torch.randn((4, B, GR, 3, H, W), generator=gen)).to(self.td).cuda()
        self.u = torch.rand((4, B, CP, H, W), generator=gen).to(self.td).cuda()
        new = lambda c: torch.empty(B, c, H, W, dtype=self.td, device="cuda")
        self.b = {n: new(c) for n, c in (("px", CP), ("lam", 4 * CP), ("s", CP), ("y", C), ("qm", C), ("a", C), ("z", C), ("h", F), ("out", C),
                                         ("gz", C), ("gh", F), ("ga", C), ("gqm", C), ("gy", C), ("gs", CP), ("t", C), ("t2", C))}
        self.lam = torch.empty(4, B, CP, H, W, dtype=self.td, device="cuda")
        self.lse = torch.empty(B, HEADS, H, W, device="cuda")
        self.grads = {n: torch.empty_like(t) for n, t in self.p.items() if n not in ("down", "lp", "lb")}
        self.gk, self.gv = torch.empty_like(self.k), torch.empty_like(self.v)

    def forward(self, **kw):
        import paper_2512_07884_amd as G
        p, b = self.p, self.b
        G.gspn_proxy_project_fused(self.x, p["down"], b["px"], **kw)
        G.gspn_proxy_project_fused(self.x, p["lp"], b["lam"], bias=p["lb"], act=G.GSPN_ACT_SIGMOID, **kw)
        self.lam.copy_(b["lam"].view(B, 4, CP, H, W).transpose(0, 1))
        G.gspn_scan_fwd_logits(b["px"], self.z, self.lam, self.u, b["s"], None, G=GR, **kw)
        G.gspn_proxy_project_fused(b["s"], p["up"], b["y"], bias=p["upb"], residual=self.x, **kw)
        G.gspn_proxy_project_fused(b["y"], p["q"], b["qm"], **kw)
        G.gspn_cross_attention(b["qm"], self.k, self.v, b["a"], self.lse, heads=HEADS, kv_heads=KV, mask=self.mask, **kw)
        G.gspn_proxy_project_fused(b["a"], p["o"], b["z"], bias=p["ob"], residual=b["y"], **kw)
        G.gspn_gated_project(b["z"], p["g"], b["h"], bias=p["gb"], act=G.GSPN_ACT_GELU, **kw)
        G.gspn_proxy_project_fused(b["h"], p["d"], b["out"], bias=p["db"], residual=b["z"], **kw)

    def backward(self, **kw):
        """Gradients down to the scan's output."""
        import paper_2512_07884_amd as G
        p, b, g = self.p, self.b, self.grads
        G.gspn_proxy_project_fused_bwd(self.gout, b["h"], p["d"], b["gh"], g["d"], g["db"], bias=p["db"], **kw)
        G.gspn_gated_project_bwd(b["gh"], b["z"], p["g"], b["t"], g["g"], g["gb"], bias=p["gb"], act=G.GSPN_ACT_GELU, **kw)
        torch.add(self.gout, b["t"], out=b["gz"])
        G.gspn_proxy_project_fused_bwd(b["gz"], b["a"], p["o"], b["ga"], g["o"], g["ob"], bias=p["ob"], **kw)
        G.gspn_cross_attention_bwd(b["ga"], b["qm"], self.k, self.v, b["a"], self.lse, b["gqm"], self.gk, self.gv, heads=HEADS, kv_heads=KV, mask=self.mask, **kw)
        G.gspn_proxy_project_fused_bwd(b["gqm"], b["y"], p["q"], b["t2"], g["q"], None, **kw)
        torch.add(b["gz"], b["t2"], out=b["gy"])
        G.gspn_proxy_project_fused_bwd(b["gy"], b["s"], p["up"], b["gs"], g["up"], g["upb"], bias=p["upb"], **kw)

    def results(self):
        return {"out": self.b["out"], "gs": self.b["gs"], "gk": self.gk, "gv": self.gv, **{"g_" + n: t for n, t in self.grads.items()}}

    def reference(self):
        """The same from the scan's output on, differentiated in 64 bits."""
        d = lambda t: t.detach().double().cpu()
        p = {n: d(t).requires_grad_(True) for n, t in self.p.items()}
        s, k, v = d(self.b["s"]).requires_grad_(True), d(self.k).requires_grad_(True), d(self.v).requires_grad_(True)
        proj = lambda P, x, bias: torch.einsum("mk,bkhw->bmhw", P, x) + bias[:, None, None]
        y = proj(p["up"], s, p["upb"]) + d(self.x)
        q = torch.einsum("mk,bkhw->bmhw", p["q"], y).reshape(B, HEADS, C // HEADS, H * W)
        rep = lambda t: t.reshape(B, L, KV, C // HEADS).repeat_interleave(HEADS // KV, 2)
        score = torch.einsum("bhdn,blhd->bhnl", q, rep(k)) * (C // HEADS) ** -0.5
        score = score.masked_fill(~self.mask.cpu()[:, None, None, :], -float("inf"))
        a = torch.einsum("bhnl,blhd->bhdn", torch.softmax(score, 3), rep(v)).reshape(B, C, H, W)
        z = proj(p["o"], a, p["ob"]) + y
        pre = proj(p["g"], z, p["gb"])
        h = torch.nn.functional.gelu(pre[:, :F]) * pre[:, F:]
        out = proj(p["d"], h, p["db"]) + z
        names = list(self.grads)
        grads = torch.autograd.grad(out, [s, k, v] + [p[n] for n in names], d(self.gout))
        return {"out": out.detach(), "gs": grads[0], "gk": grads[1], "gv": grads[2], **{"g_" + n: t for n, t in zip(names, grads[3:])}}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_block_forward_and_backward(dtype):
    """From the scan's output to the block's and back, through seven of the calls: each tensor that passes between two calls is rounded once to the storage type,
    a relative error of at most h = eps / 2 in the 2-norm that the calls after it (of gain about 1, as the matrices are scaled) hand on: at most 16 tensors lie
    between any input and a result, so 16 h; fp32 sums add (F + C + L) 2^-24 each."""
    block = Block(dtype)
    block.forward()
    block.backward()
    torch.cuda.synchronize()
    ref, tol = block.reference(), 16 * (R.half(dtype) + (F + C + L) * 2.0 ** -24)
    for n, t in block.results().items():
        a, r = t.double().cpu(), ref[n]
        assert torch.isfinite(a).all(), n
        assert float((a - r).norm() / r.norm()) <= tol, (n, float((a - r).norm() / r.norm()), tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_block_replays_like_eager(dtype):
    """Forward and backward captured together (workspaces from the graph's pool), replayed with changed inputs between eager work; every replay has the bits of
    the eager step.  A second graph of other tensors is captured and replayed in between."""
    block, other = Block(dtype, 1), Block(dtype, 2)
    for b in (block, other):
        b.forward()
        b.backward()
    torch.cuda.synchronize()
    graphs = []
    for b in (block, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.forward()
            b.backward()
        graphs.append(graph)
    gen = torch.Generator(device="cuda").manual_seed(9)
    bits = torch.int32 if dtype == "f32" else torch.int16
    for rep in range(3):
        for b in (block, other):
            for t in (b.x, b.k, b.gout):
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda").to(t.dtype))
        want = []
        for b in (block, other):
            b.forward()
            b.backward()
            torch.cuda.synchronize()
            want.append({n: t.clone() for n, t in b.results().items()})
            for t in b.results().values():
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for b, w in zip((block, other), want):
            for n, t in b.results().items():
                assert torch.equal(t.view(bits), w[n].view(bits)), (rep, n)


def test_blocks_on_streams_of_their_own():
    """Two blocks at once, each on a stream that its calls are given, with the bits of the default stream's."""
    blocks = [Block("bf16", 3), Block("bf16", 4)]
    want = []
    for b in blocks:
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in b.results().items()})
        for t in b.results().values():
            t.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(3):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):                   # (torch's own steps of the block too)
                b.forward(stream=s)
                b.backward(stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for n, t in b.results().items():
            assert torch.equal(t.view(torch.int16), w[n].view(torch.int16)), n


def test_workspaces_of_the_callers():
    """The backward calls with memory of the caller's of exactly the bytes asked for, nothing behind it written; fewer bytes are refused."""
    import paper_2512_07884_amd as G
    from paper_2512_07884_amd import binding as b
    gen = torch.Generator(device="cuda").manual_seed(12)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    x, P, g = rnd(2, 40, 9, 10), rnd(96, 40), rnd(2, 48, 9, 10)
    q, k, go = rnd(2, 32, 9, 10), rnd(2, 45, 32), rnd(2, 32, 9, 10)
    out, lse = torch.empty_like(q), torch.empty(2, 4, 9, 10, device="cuda")
    G.gspn_cross_attention(q, k, k, out, lse, heads=4)
    calls = [(G.gspn_gated_project_bwd_bytes(2, 40, 48, 9, 10, G.GSPN_ACT_SILU, b.GSPN_BF16), (x, P), lambda ws, gr: G.gspn_gated_project_bwd(g, x, P, *gr, None, workspace=ws)),
             (G.gspn_proxy_project_fused_bwd_bytes(2, 40, 48, 9, 10, G.GSPN_ACT_GELU, b.GSPN_BF16), (x, P[:48]),
              lambda ws, gr: G.gspn_proxy_project_fused_bwd(g, x, P[:48], *gr, None, act=G.GSPN_ACT_GELU, workspace=ws)),
             (G.gspn_cross_attention_bwd_bytes(2, 4, 4, 8, 9, 10, 45, b.GSPN_BF16), (q, k, k),
              lambda ws, gr: G.gspn_cross_attention_bwd(go, q, k, k, out, lse, *gr, heads=4, workspace=ws))]
    for need, like, call in calls:
        want, got = [torch.full_like(t, float("nan")) for t in like], [torch.full_like(t, float("nan")) for t in like]
        call(None, want)
        ws = torch.full((need + 1024,), 0x5a, dtype=torch.uint8, device="cuda")
        call(ws, got)
        torch.cuda.synchronize()
        assert (ws[need:] == 0x5a).all()
        assert all(torch.equal(a, c) for a, c in zip(want, got))
        with pytest.raises(G.GspnError):
            call(ws[:need - 256], got)
