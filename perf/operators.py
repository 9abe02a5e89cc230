"""The operators of a block around the scan, as a model that uses this library calls them, and their plain forms.

A GSPN block has more on its feature maps than the scan: projections with a bias, an activation or the residual (the scan's parameters,
the way back up), cross attention to the states of an encoder (a text prompt), a gated feed-forward block.

``listed()`` holds the fixed cases, ``draw`` one more case from the same ranges, ``prepare`` what a program has in hand before the call,
``run`` one pass, ``work`` the bytes and operations of a pass, ``exact`` its results in 64 bits.  With ``own`` the passes are calls of this
package, else elementary torch operations in 32 bits.

A case is a dict of plain values:
    op       "project": out = act(P x + bias) + residual.  "gated": out = act(P1 x + b1) * (P2 x + b2).  "attend": pixels attend to tokens.
    step     False: forward alone.  True: forward and backward (a training step of the operator).
    B, H, W  batch and map;  dtype: storage type of every tensor, "f32", "bf16" or "f16"
    K, M     project: channels in and out;  gated: channels in, hidden channels out
    act      "none", "silu", "gelu" or "sigmoid";  bias, residual: whether there is one
    heads, kv_heads, D, L   attend: heads of the map, heads of the tokens, channels of a head, tokens;  mask: whether tokens are masked,
             empty: whether the first image's mask leaves no token at all
"""
import math

import torch

own = False

TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _project(name, step, B, H, W, dtype, K, M, act, bias=True, residual=False, op="project"):
    c = {"op": op, "step": step, "B": B, "H": H, "W": W, "dtype": dtype, "K": K, "M": M, "act": act, "bias": bias, "residual": residual}
    return {"name": name, **c} if name else c


def _gated(name, step, B, H, W, dtype, K, M, act, bias=True):
    return _project(name, step, B, H, W, dtype, K, M, act, bias, False, "gated")


def _attend(name, step, B, H, W, dtype, heads, kv_heads, D, L, mask=True, empty=False):
    c = {"op": "attend", "step": step, "B": B, "H": H, "W": W, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "D": D, "L": L,
         "mask": mask, "empty": empty}
    return {"name": name, **c} if name else c


def listed():
    return [
        # serving one image: lambda of four directions of 24 proxy channels, third stage of the classifier; latency is the cost
        _project("project_14x14_one_image", False, 1, 14, 14, "bf16", 384, 96, "sigmoid"),
        # batched classification, first stage: the weight logits of four directions, eight groups, three taps
        _project("project_56x56_logits", False, 64, 56, 56, "bf16", 96, 96, "none"),
        # dense prediction, an odd width: back up from the proxy channels, with the residual
        _project("project_100x167_up_f16", False, 2, 100, 167, "f16", 64, 256, "none", residual=True),
        # a training step of a projection on two latents, all channels
        _project("project_64x64_step", True, 2, 64, 64, "bf16", 1152, 1152, "gelu", residual=True),
        # serving one image: the feed-forward block of the third stage
        _gated("gated_14x14_one_image", False, 1, 14, 14, "bf16", 384, 1024, "silu"),
        # full precision on a small odd map, training
        _gated("gated_25x42_step_f32", True, 4, 25, 42, "f32", 192, 512, "silu"),
        # the feed-forward block of a latent layer, training (the largest listed case)
        _gated("gated_64x64_step", True, 2, 64, 64, "bf16", 1152, 4608, "gelu"),
        # serving one image with one prompt: 77 tokens, some of them padding
        _attend("attend_14x14_one_image", False, 1, 14, 14, "bf16", 6, 6, 64, 77),
        # one denoising step of a 1024-px latent, the guided and the free half, 77 tokens
        _attend("attend_128x128_latent", False, 2, 128, 128, "bf16", 16, 16, 64, 77),
        # a training step on two latents, long prompts, heads of 72 channels
        _attend("attend_64x64_step_f16", True, 2, 64, 64, "f16", 16, 16, 72, 300),
        # a single query position per image over a long encoder, shared token heads
        _attend("attend_one_pixel_long", False, 4, 1, 1, "bf16", 16, 4, 64, 8192),
        # full precision on an odd map, shared token heads, training
        _attend("attend_50x83_step_f32", True, 2, 50, 83, "f32", 6, 3, 32, 129),
    ]


def _spread(rng, lo, hi):
    """An integer between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Channels: mostly a multiple of 8, now and then any number."""
    n = _spread(rng, lo, hi)
    return n if rng.random() < 0.2 else max(8, n - n % 8)


def draw(rng):
    op = rng.choice(["project", "gated", "attend"])
    step = rng.random() < 0.5
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    H, W = _spread(rng, 1, 170), _spread(rng, 1, 170)
    if rng.random() < 0.6:                    # square maps of the usual sides
        H = W = rng.choice([7, 14, 28, 32, 56, 64, 96, 128])
    B = _spread(rng, 1, 64)
    if op == "project":
        act = rng.choice(["none", "none", "silu", "gelu", "sigmoid"])
        case = _project("", step, B, H, W, dtype, _channels(rng, 8, 1152), _channels(rng, 8, 1152), act, rng.random() < 0.8, rng.random() < 0.4)
    elif op == "gated":
        K = _channels(rng, 32, 1152)
        case = _gated("", step, B, H, W, dtype, K, _channels(rng, K, 4 * K), rng.choice(["silu", "gelu", "gelu", "sigmoid"]), rng.random() < 0.8)
    else:
        kv = rng.choice([1, 2, 3, 4, 6, 8, 16])
        heads = kv * rng.choice([1, 1, 1, 2, 4])
        if not step and rng.random() < 0.3:   # few positions over a long encoder
            H, W, L = 1, _spread(rng, 1, 40), _spread(rng, 500, 16384)
        else:
            L = _spread(rng, 2 if step else 1, 1024)        # (over a single token the scores have no gradient)
        mask = rng.random() < 0.7
        case = _attend("", step, B, H, W, dtype, heads, kv, 8 * rng.randint(1, 16), L, mask, mask and B > 1 and rng.random() < 0.3)
    most = {"bytes": 0.0, "flops": 0.0}
    for c in listed():
        w = work(c)
        most = {k: max(most[k], w[k]) for k in most}
    if dtype == "f32":                        # (the rate of full precision is a sixteenth)
        most["flops"] /= 8
    while True:
        w = work(case)
        heavy = w["bytes"] > most["bytes"] or w["flops"] > most["flops"]
        heavy = heavy or (op == "attend" and case["B"] * case["heads"] * case["H"] * case["W"] * case["L"] > 1.6e8)
        if not heavy:
            return case
        if case["B"] > 1:
            case["B"] = (case["B"] + 1) // 2
            case["empty"] = case.get("empty", False) and case["B"] > 1
            if op != "attend":
                case.pop("empty")
        elif case["H"] * case["W"] > 1024:
            case["H"], case["W"] = (case["H"] + 1) // 2, (case["W"] + 1) // 2
        elif op == "attend" and case["L"] > 1:
            case["L"] = (case["L"] + 1) // 2
        else:
            case["K"], case["M"] = (case["K"] + 1) // 2, (case["M"] + 1) // 2


def _inputs(case, seed):
    """The tensors of a case by name, on the GPU, in the storage type."""
    td = TORCH_TYPE[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(td)

    B, H, W = case["B"], case["H"], case["W"]
    t = {}
    if case["op"] == "attend":
        C, E = case["heads"] * case["D"], case["kv_heads"] * case["D"]
        t["q"], t["k"], t["v"] = normal(B, C, H, W, scale=1.5), normal(B, case["L"], E), normal(B, case["L"], E)
        t["mask"] = None
        if case["mask"]:                      # prompts of other lengths, padded; now and then a token left out
            n = torch.randint(min(max(2, case["L"] // 4), case["L"]), case["L"] + 1, (B, 1), generator=gen, device="cuda")
            if case["empty"]:
                n[0] = 0
            at = torch.arange(case["L"], device="cuda")
            t["mask"] = (at < n) & ((at < 2) | (torch.rand((B, case["L"]), generator=gen, device="cuda") > 0.03))
        if case["step"]:
            t["gout"] = normal(B, C, H, W)
        return t
    K, M = case["K"], case["M"]
    rows = 2 * M if case["op"] == "gated" else M
    t["x"], t["P"] = normal(B, K, H, W), normal(rows, K, scale=K ** -0.5)
    t["bias"] = normal(rows, scale=0.3) if case["bias"] else None
    t["residual"] = normal(B, M, H, W) if case["residual"] else None
    if case["step"]:
        t["gout"] = normal(B, M, H, W)
    return t


def prepare(case, seed):
    """Inputs of the operator on the GPU and the buffers its outputs go to, as a program keeps them."""
    s = {"case": case, **_inputs(case, seed)}
    if case["op"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        if case["step"]:
            s["lse"] = torch.empty((case["B"], case["heads"], case["H"], case["W"]), dtype=torch.float32, device="cuda")
            s["gq"], s["gk"], s["gv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    else:
        s["out"] = torch.empty((case["B"], case["M"], case["H"], case["W"]), dtype=s["x"].dtype, device="cuda")
        if case["step"]:
            s["gx"], s["gP"] = torch.empty_like(s["x"]), torch.empty_like(s["P"])
            s["gbias"] = torch.empty_like(s["bias"]) if case["bias"] else None
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2512_07884_amd as G
    c = s["case"]
    if c["op"] == "attend":
        kw = {"heads": c["heads"], "kv_heads": c["kv_heads"], "mask": s["mask"]}
        G.gspn_cross_attention(s["q"], s["k"], s["v"], s["out"], s["lse"] if c["step"] else None, **kw)
        if not c["step"]:
            return {"out": s["out"]}
        G.gspn_cross_attention_bwd(s["gout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["gq"], s["gk"], s["gv"], **kw)
        return {k: s[k] for k in ("out", "gq", "gk", "gv")}
    act = {"none": G.GSPN_ACT_NONE, "silu": G.GSPN_ACT_SILU, "gelu": G.GSPN_ACT_GELU, "sigmoid": G.GSPN_ACT_SIGMOID}[c["act"]]
    if c["op"] == "gated":
        G.gspn_gated_project(s["x"], s["P"], s["out"], bias=s["bias"], act=act)
    else:
        G.gspn_proxy_project_fused(s["x"], s["P"], s["out"], bias=s["bias"], residual=s["residual"], act=act)
    if not c["step"]:
        return {"out": s["out"]}
    bwd = G.gspn_gated_project_bwd if c["op"] == "gated" else G.gspn_proxy_project_fused_bwd
    bwd(s["gout"], s["x"], s["P"], s["gx"], s["gP"], s["gbias"], bias=s["bias"], act=act)
    return {k: s[k] for k in ("out", "gx", "gP", "gbias") if s[k] is not None}


def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, None
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(z * (1.0 / math.sqrt(2.0))))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-z))
    if act == "sigmoid":
        return g, g * (1.0 - g)
    return z * g, g + z * g * (1.0 - g)


def _run_plain(s):
    c = s["case"]
    td = TORCH_TYPE[c["dtype"]]
    if c["op"] == "attend":
        return _attend_plain(s, c, td)
    B, H, W, K, M = c["B"], c["H"], c["W"], c["K"], c["M"]
    x, P = s["x"].float().view(B, K, H * W), s["P"].float()
    pre = torch.matmul(P, x)
    if s["bias"] is not None:
        pre = pre + s["bias"].float()[:, None]
    if c["op"] == "gated":
        a, da = _act(pre[:, :M], c["act"])
        out = a * pre[:, M:]
    else:
        a, da = _act(pre, c["act"])
        out = a if s["residual"] is None else a + s["residual"].float().view(B, M, H * W)
    res = {"out": out.to(td).view(B, M, H, W)}
    if not c["step"]:
        return res
    g = s["gout"].float().view(B, M, H * W)
    if c["op"] == "gated":
        g = torch.cat((g * pre[:, M:] * da, g * a), dim=1)
    elif da is not None:
        g = g * da
    res["gx"] = torch.matmul(P.t().contiguous(), g).to(td).view(B, K, H, W)
    res["gP"] = torch.matmul(g.transpose(0, 1).reshape(P.shape[0], B * H * W), x.permute(0, 2, 1).reshape(B * H * W, K)).to(td)
    if s["bias"] is not None:
        res["gbias"] = g.sum(dim=(0, 2)).to(td)
    return res


def _attend_plain(s, c, td):
    B, N, L, h, kv, D = c["B"], c["H"] * c["W"], c["L"], c["heads"], c["kv_heads"], c["D"]
    per = h // kv
    scale = 1.0 / math.sqrt(D)
    q = s["q"].float().view(B, kv, per, D, N).permute(0, 1, 2, 4, 3).reshape(B, kv, per * N, D)      # rows: positions of the heads that share tokens
    k = s["k"].float().view(B, L, kv, D).permute(0, 2, 1, 3).contiguous()
    v = s["v"].float().view(B, L, kv, D).permute(0, 2, 1, 3).contiguous()
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    if s["mask"] is not None:
        keep = s["mask"][:, None, None, :]
        p = torch.where(keep, p, torch.full((), float("-inf"), device=p.device))
        top = p.amax(dim=3, keepdim=True)
        p = torch.exp(p - torch.where(torch.isfinite(top), top, torch.zeros((), device=p.device)))
    else:
        p = torch.exp(p - p.amax(dim=3, keepdim=True))
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones((), device=p.device))
    out = torch.matmul(p, v)

    def image(t):
        return t.to(td).view(B, kv, per, N, D).permute(0, 1, 2, 4, 3).reshape(B, h * D, c["H"], c["W"])

    def tokens(t):
        return t.to(td).permute(0, 2, 1, 3).reshape(B, L, kv * D)

    res = {"out": image(out)}
    if not c["step"]:
        return res
    g = s["gout"].float().view(B, kv, per, D, N).permute(0, 1, 2, 4, 3).reshape(B, kv, per * N, D)
    ds = p * (torch.matmul(g, v.transpose(2, 3).contiguous()) - (g * out).sum(dim=3, keepdim=True)) * scale
    res["gq"] = image(torch.matmul(ds, k))
    res["gk"] = tokens(torch.matmul(ds.transpose(2, 3).contiguous(), q))
    res["gv"] = tokens(torch.matmul(p.transpose(2, 3).contiguous(), g))
    return res


def work(case):
    """Every input once, every output once; the forward and the backward call lie either side of the loss, so the backward call has to read again
    what the forward call read.  Operations: a multiply-add is two; of a backward call the products of its gradients, and for attention the
    scores again (no program keeps those); the mask's share of the tokens is not taken off."""
    e = 4 if case["dtype"] == "f32" else 2
    B, N = case["B"], case["H"] * case["W"]
    if case["op"] == "attend":
        L, D = case["L"], case["D"]
        n, t = B * case["heads"] * D * N, B * case["kv_heads"] * D * L
        elems = 2 * n + 2 * t
        flops = 4.0 * B * case["heads"] * N * L * D
        if case["step"]:
            elems += 4 * n + 4 * t                                  # q, gout, out, gq; k, v, gk, gv
            flops *= 3.5
        return {"bytes": float(e * elems + (B * L if case["mask"] else 0)), "flops": flops}
    K, M = case["K"], case["M"]
    rows = 2 * M if case["op"] == "gated" else M
    elems = B * N * (K + M * (2 if case["residual"] else 1)) + rows * K + (rows if case["bias"] else 0)
    flops = 2.0 * B * N * K * rows
    if case["step"]:
        elems += B * N * (2 * K + M) + 2 * rows * K + (2 * rows if case["bias"] else 0)
        flops *= 3
    return {"bytes": float(e * elems), "flops": flops}


def exact(case, seed):
    """The results in 64 bits: the operators' definitions, with the gradients by differentiating them."""
    if work(case)["flops"] > 2e12:
        return None
    t = {k: v if v is None or v.dtype == torch.bool else v.double() for k, v in _inputs(case, seed).items()}
    B, H, W = case["B"], case["H"], case["W"]
    if case["op"] == "attend":
        leaves = [t["q"], t["k"], t["v"]]
        names = ["gq", "gk", "gv"]
    else:
        leaves = [t["x"], t["P"]] + ([t["bias"]] if case["bias"] else [])
        names = ["gx", "gP", "gbias"]
    if case["step"]:
        for leaf in leaves:
            leaf.requires_grad_(True)
    with torch.set_grad_enabled(case["step"]):
        if case["op"] == "attend":
            h, kv, D, L = case["heads"], case["kv_heads"], case["D"], case["L"]
            # the heads that share tokens each get their own copy of them
            k = t["k"].view(B, L, kv, D).repeat_interleave(h // kv, dim=2).permute(0, 2, 1, 3)
            v = t["v"].view(B, L, kv, D).repeat_interleave(h // kv, dim=2).permute(0, 2, 3, 1)
            score = torch.matmul(k, t["q"].view(B, h, D, H * W)) / math.sqrt(D)         # [B, h, L, N]
            if case["mask"]:
                score = score.masked_fill(~t["mask"][:, None, :, None], -1e300)
            weight = torch.exp(score - score.detach().max(dim=2, keepdim=True).values)
            if case["mask"]:
                weight = weight * t["mask"][:, None, :, None]
            out = torch.matmul(v, weight) / weight.sum(dim=2, keepdim=True).clamp_min(1e-300)
            out = out.view(B, h * D, H, W)
        else:
            pre = torch.matmul(t["P"], t["x"].view(B, case["K"], H * W))
            if case["bias"]:
                pre = pre + t["bias"].view(1, -1, 1)
            z = pre[:, :case["M"]]
            out = {"none": lambda: z, "silu": lambda: z * torch.sigmoid(z), "sigmoid": lambda: torch.sigmoid(z),
                   "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2.0))}[case["act"]]()
            if case["op"] == "gated":
                out = out * pre[:, case["M"]:]
            out = out.view(B, case["M"], H, W)
            if case["residual"]:
                out = out + t["residual"]
        res = {"out": out.detach()}
        if case["step"]:
            res.update(zip(names, torch.autograd.grad(out, leaves, t["gout"])))
    return res
