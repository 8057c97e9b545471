"""The operators around the attention core of a DiT block, case by case: the fused gate + residual + norm + modulation
(``adaln``) and attention over selected key blocks (``sparse``), each forward, with tangents (JVP) and in training.

``run`` computes a case in plain torch operations (32-bit arithmetic, 64-bit block scores) where ``own`` is false and
through the framework's entry points where it is true; ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

BLOCK = 128            # queries and keys of a block of the selection
NEG = -math.inf


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _adaln(name, direction, B, L, C, x="bf16", norm="layer", post="none", weights=False):
    return dict(name=name, op="adaln", direction=direction, B=B, L=L, C=C, x=x, norm=norm, post=post, weights=weights)


def _sparse(name, direction, B, H, Lq, Lk, D, topk=0, density=0.0, kv_tangents=True):
    return dict(name=name, op="sparse", direction=direction, B=B, H=H, Lq=Lq, Lk=Lk, D=D, topk=topk, density=density,
                kv_tangents=kv_tangents)


def listed():
    return [
        # one conditioning token of a 14B-shaped block with an fp32 residual stream: launch latency
        _adaln("adaln_token", "forward", 1, 1, 5120, x="fp32"),
        # every block of a 14B-shaped video DiT at 832x480x81 (32760 tokens), sampling
        _adaln("adaln_video_14b", "forward", 1, 32760, 5120),
        # image DiT in JVP mode, residual stream kept in fp32
        _adaln("adaln_jvp_image_2b", "jvp", 2, 4096, 2048, x="fp32"),
        # blocks with a norm on both sides, odd length, JVP mode
        _adaln("adaln_jvp_sandwich", "jvp", 3, 10007, 1536, norm="rms", post="rms", weights=True),
        # student step of the 14B-shaped block: forward and gradients
        _adaln("adaln_train_video_14b", "train", 1, 32760, 5120),
        # short ragged batch, fp32 residual, learnt norm weights
        _adaln("adaln_train_short", "train", 2, 257, 1536, x="fp32", norm="rms", post="layer", weights=True),
        # a short sequence against a short context: launch latency
        _sparse("sparse_short", "forward", 1, 2, 200, 333, 64, topk=2),
        # 1.3B-shaped video DiT, one key block in eight kept
        _sparse("sparse_video_1p3b", "forward", 1, 12, 32760, 32760, 128, topk=32),
        # image DiT in JVP mode, one key block in four kept
        _sparse("sparse_jvp_image_2b", "jvp", 2, 16, 4096, 4096, 128, topk=8),
        # a given mask with empty rows over a constant context (no K/V tangents), odd lengths
        _sparse("sparse_jvp_mask_d64", "jvp", 1, 24, 4100, 8000, 64, density=0.3, kv_tangents=False),
        # student step of the 1.3B-shaped video DiT: selection, forward, gradients
        _sparse("sparse_train_video_1p3b", "train", 1, 12, 32760, 32760, 128, topk=32),
        # training under a given mask that leaves query and key blocks out, odd lengths
        _sparse("sparse_train_mask_d64", "train", 2, 6, 4001, 3977, 64, density=0.25),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    if rng.random() < 0.5:
        # channel counts H * D of the configurations, or any multiple of 8
        C = rng.choice([1536, 2048, 5120, 8 * _log_int(rng, 8, 640)])
        B = rng.randint(1, 4)
        L = _log_int(rng, 1, 32760 // B)
        post = rng.choice(["none", "none", "rms", "layer"])
        return dict(op="adaln", direction=rng.choice(["forward", "jvp", "train"]), B=B, L=L, C=C,
                    x=rng.choice(["bf16", "fp32"]), norm=rng.choice(["layer", "rms"]), post=post,
                    weights=rng.random() < 0.5)
    D = rng.choice([64, 128])
    B, H = rng.randint(1, 2), rng.randint(1, 6)
    Lq = _log_int(rng, 1, 32760)
    # two keys at least: with a single one every gradient and tangent that is left is exactly 0, and only rounding is compared
    Lk = max(2, Lq if rng.random() < 0.5 else _log_int(rng, 2, 32760))
    n_k = -(-Lk // BLOCK)
    direction = rng.choice(["forward", "jvp", "train"])
    case = dict(op="sparse", direction=direction, B=B, H=H, Lq=Lq, Lk=Lk, D=D, topk=0, density=0.0,
                kv_tangents=rng.random() < 0.7)
    if Lq * Lk <= 8192 * 8192 and rng.random() < 0.4:
        case["density"] = rng.uniform(0.05, 0.9)
    else:
        case["topk"] = _log_int(rng, 1, max(1, min(n_k, 32)))
    return case


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, sigma=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)

    s = dict(case=case)
    if case["op"] == "adaln":
        B, L, C = case["B"], case["L"], case["C"]
        xt = torch.bfloat16 if case["x"] == "bf16" else torch.float32
        # a residual stream with a few large channels, as trained blocks have
        loud = torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        s["x"] = (randn(B, L, C) * loud + randn(1, 1, C, sigma=0.3)).to(xt)
        s["h"] = randn(B, L, C, dtype=torch.bfloat16)
        s["mod"] = randn(B, 3, C, sigma=0.4)        # gate, scale, shift: one row of the block's modulation each
        s["w"] = 1 + randn(C, sigma=0.1) if case["weights"] else None
        s["wp"] = 1 + randn(C, sigma=0.1) if case["weights"] and case["post"] != "none" else None
        if case["direction"] == "jvp":
            s["tx"], s["th"] = randn(B, L, C, sigma=0.5, dtype=xt), randn(B, L, C, sigma=0.5, dtype=torch.bfloat16)
            s["tmod"] = randn(B, 3, C, sigma=0.2)
        if case["direction"] == "train":
            s["dxn"], s["dy"] = randn(B, L, C, dtype=xt), randn(B, L, C, dtype=torch.bfloat16)
        return s

    B, H, Lq, Lk, D = (case[k] for k in ("B", "H", "Lq", "Lk", "D"))
    n_q, n_k = -(-Lq // BLOCK), -(-Lk // BLOCK)

    def tokens(L, n):
        # unit-variance rows around a direction of their block, as neighbouring patches have
        x = randn(B, L, H, D)
        x += randn(B, n, H, D, sigma=0.5).repeat_interleave(BLOCK, 1)[:, :L]
        return x.to(torch.bfloat16)

    s["q"], s["k"] = tokens(Lq, n_q), tokens(Lk, n_k)
    s["v"] = randn(B, Lk, H, D, dtype=torch.bfloat16)
    if case["direction"] == "jvp":
        s["tq"] = randn(B, Lq, H, D, sigma=0.5, dtype=torch.bfloat16)
        if case["kv_tangents"]:
            s["tk"] = randn(B, Lk, H, D, sigma=0.5, dtype=torch.bfloat16)
            s["tv"] = randn(B, Lk, H, D, sigma=0.5, dtype=torch.bfloat16)
    if case["direction"] == "train":
        s["do"] = randn(B, Lq, H, D, dtype=torch.bfloat16)
    if not case["topk"]:
        # a mask drawn block by block, a tenth of the query blocks left without any key
        mask = torch.rand(B, H, n_q, n_k, generator=g, device="cuda") < case["density"]
        s["mask"] = mask & (torch.rand(B, H, n_q, 1, generator=g, device="cuda") >= 0.1)
    return s


# ---------------------------------------------------------------------------------------------------------------
# adaln, plain
# ---------------------------------------------------------------------------------------------------------------
EPS = 1e-6


def _normed(x, kind):
    """Normalised rows and their 1 / deviation."""
    if kind == "none":
        return x, None
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    r = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * r, r


def _normed_tangent(n, r, t, kind):
    if kind == "none":
        return t
    c = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    return r * (c - n * (n * c).mean(-1, keepdim=True))


def _adaln_plain(s):
    case = s["case"]
    norm, post, xt = case["norm"], case["post"], s["x"].dtype
    gate, scale, shift = (m.unsqueeze(1) for m in s["mod"].unbind(1))
    w = 1.0 if s["w"] is None else s["w"]
    wp = 1.0 if s["wp"] is None else s["wp"]
    hn, rp = _normed(s["h"].float(), post)
    xn = s["x"].float() + gate * (wp * hn)
    n, r = _normed(xn, norm)
    out = dict(x=xn.to(xt), y=(n * (w * (1 + scale)) + shift).to(torch.bfloat16))
    if case["direction"] == "jvp":
        tgate, tscale, tshift = (m.unsqueeze(1) for m in s["tmod"].unbind(1))
        thn = _normed_tangent(hn, rp, s["th"].float(), post)
        txn = s["tx"].float() + tgate * (wp * hn) + gate * (wp * thn)
        tn = _normed_tangent(n, r, txn, norm)
        out["tx"] = txn.to(xt)
        out["ty"] = (tn * (w * (1 + scale)) + n * (w * tscale) + tshift).to(torch.bfloat16)
    if case["direction"] == "train":
        dy = s["dy"].float()
        # the derivative of a normalisation is symmetric: the tangent's formula is the gradient's
        dx = s["dxn"].float() + _normed_tangent(n, r, dy * (w * (1 + scale)), norm)
        a, b = (dy * n).sum(1), (dx * hn).sum(1)
        out["dx"] = dx.to(xt)
        out["dh"] = _normed_tangent(hn, rp, dx * (gate * wp), post).to(torch.bfloat16)
        out["dgate"], out["dscale"], out["dshift"] = wp * b, w * a, dy.sum(1)
        if s["w"] is not None:
            out["dw"] = ((1 + scale[:, 0]) * a).sum(0)
        if s["wp"] is not None:
            out["dwp"] = (gate[:, 0] * b).sum(0)
    return out


def _adaln_own(s):
    import paper_2510_08431_b200 as aj
    case = s["case"]
    gate, scale, shift = s["mod"].unbind(1)
    args = dict(x=s["x"], h=s["h"], gate=gate, scale=scale, shift=shift, weight=s["w"], post_weight=s["wp"],
                norm=case["norm"], post_norm=None if case["post"] == "none" else case["post"], eps=EPS)
    if case["direction"] == "jvp":
        tgate, tscale, tshift = s["tmod"].unbind(1)
        x, y, tx, ty = aj.adaln_jvp(**args, tx=s["tx"], th=s["th"], tgate=tgate, tscale=tscale, tshift=tshift)
        return dict(x=x, y=y, tx=tx, ty=ty)
    x, y, _, _ = aj.adaln_jvp(**args)
    out = dict(x=x, y=y)
    if case["direction"] == "train":
        d = aj.adaln_backward(s["dxn"], s["dy"], **args)
        out.update(dx=d.x, dh=d.h, dgate=d.gate, dscale=d.scale, dshift=d.shift)
        if s["w"] is not None:
            out["dw"] = d.weight
        if s["wp"] is not None:
            out["dwp"] = d.post_weight
    return out


# ---------------------------------------------------------------------------------------------------------------
# Attention over selected key blocks, plain
# ---------------------------------------------------------------------------------------------------------------
def _blocks(x, n, dtype=torch.float32):
    """[B][L][H][D] -> [B][H][n][BLOCK][D], rows past L zero."""
    B, L, H, D = x.shape
    x = torch.nn.functional.pad(x.to(dtype), (0, 0, 0, 0, 0, n * BLOCK - L))
    return x.view(B, n, BLOCK, H, D).permute(0, 3, 1, 2, 4)


def _unblocks(x, L):
    B, H, n, _, D = x.shape
    return x.permute(0, 2, 3, 1, 4).reshape(B, n * BLOCK, H, D)[:, :L].to(torch.bfloat16)


def _block_means(x, n):
    L = x.shape[1]
    rows = (L - BLOCK * torch.arange(n, device=x.device)).clamp(max=BLOCK)
    return _blocks(x, n, torch.float64).sum(3) / rows[:, None]


def _sparse_plain(s):
    case = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    B, Lq, H, D = q.shape
    Lk = k.shape[1]
    n_q, n_k = -(-Lq // BLOCK), -(-Lk // BLOCK)
    scale = 1 / math.sqrt(D)
    if case["topk"]:
        # mean-pooled scores, in 64 bits: which of two blocks a hair apart is larger decides whole outputs
        score = _block_means(q, n_q) @ _block_means(k, n_k).transpose(-1, -2)
        index = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :case["topk"]]
        mask = torch.zeros(B, H, n_q, n_k, dtype=torch.bool, device=q.device).scatter_(-1, index, True)
        kept = torch.ones_like(index, dtype=torch.bool)
    else:
        mask = s["mask"]
        kept, index = torch.sort(mask.to(torch.uint8), dim=-1, descending=True, stable=True)
        kept = kept.bool()
    flat = (torch.arange(B * H, device=q.device).view(B, H, 1, 1) * n_k + index)    # which block of all (b, h)
    span = index.shape[-1] * BLOCK

    def gathered(x):
        return _blocks(x, n_k).reshape(B * H * n_k, BLOCK, D)[flat].view(B, H, n_q, span, D)

    inside = index.unsqueeze(-1) * BLOCK + torch.arange(BLOCK, device=q.device) < Lk
    inside = (inside & kept.unsqueeze(-1)).view(B, H, n_q, 1, span)
    qb, kg, vg = _blocks(q, n_q), gathered(k), gathered(v)
    S = (qb @ kg.transpose(-1, -2)).mul_(scale).masked_fill_(~inside, NEG)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == NEG, 0.0, m)
    P = S.sub_(m).exp_()
    l = P.sum(-1, keepdim=True)
    lse = (m + l.log())[..., 0].reshape(B, H, n_q * BLOCK)[..., :Lq]
    P.div_(torch.where(l == 0, 1.0, l))
    o = P @ vg
    out = dict(o=_unblocks(o, Lq), lse=lse.contiguous(), mask=mask)
    if case["direction"] == "jvp":
        tS = _blocks(s["tq"], n_q) @ kg.transpose(-1, -2)
        if case["kv_tangents"]:
            tS += qb @ gathered(s["tk"]).transpose(-1, -2)
        H_ = tS.mul_(scale).mul_(P)
        to = H_ @ vg - H_.sum(-1, keepdim=True) * o
        if case["kv_tangents"]:
            to += P @ gathered(s["tv"])
        out["to"] = _unblocks(to, Lq)
    if case["direction"] == "train":
        do = _blocks(s["do"], n_q)

        def scattered(x):
            sums = torch.zeros(B * H * n_k, BLOCK, D, device=q.device)
            sums.index_add_(0, flat.reshape(-1), x.reshape(-1, BLOCK, D))
            return _unblocks(sums.view(B, H, n_k, BLOCK, D), Lk)

        out["dv"] = scattered(P.transpose(-1, -2) @ do)
        dS = (do @ vg.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(P).mul_(scale)
        out["dq"] = _unblocks(dS @ kg, Lq)
        out["dk"] = scattered(dS.transpose(-1, -2) @ qb)
    return out


def _sparse_own(s):
    import paper_2510_08431_b200 as aj
    case = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    if case["topk"]:
        sel = aj.block_select(q, k, case["topk"])
    else:
        sel = aj.block_selection(s["mask"], q.shape[1], k.shape[1])
    if case["direction"] == "jvp":
        o, to, lse = aj.sparse_attention_jvp(q, k, v, sel, s["tq"], s.get("tk"), s.get("tv"))
        return dict(o=o, lse=lse, mask=sel.mask, to=to)
    o, _, lse = aj.sparse_attention_jvp(q, k, v, sel, fwd_only=True)
    out = dict(o=o, lse=lse, mask=sel.mask)
    if case["direction"] == "train":
        out["dq"], out["dk"], out["dv"] = aj.sparse_attention_backward(s["do"], q, k, v, o, lse, sel)
    return out


def run(state):
    if state["case"]["op"] == "adaln":
        return _adaln_own(state) if own else _adaln_plain(state)
    return _sparse_own(state) if own else _sparse_plain(state)


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "adaln":
        B, L, C = case["B"], case["L"], case["C"]
        cells, xb = B * L * C, 2 if case["x"] == "bf16" else 4
        rows = 3 * B * C * 4 + (8 * C if case["weights"] else 0)       # modulation rows, norm weights
        fwd = cells * (2 * xb + 2 * 2)
        if case["direction"] == "forward":
            return dict(bytes=fwd + rows, flops=12 * cells)
        if case["direction"] == "jvp":
            return dict(bytes=2 * (fwd + rows), flops=30 * cells)
        return dict(bytes=fwd + cells * (2 * xb + 2 * 2) + 2 * rows, flops=40 * cells)
    B, H, Lq, Lk, D = (case[k] for k in ("B", "H", "Lq", "Lk", "D"))
    q_bytes, k_bytes = 2 * B * H * Lq * D, 2 * B * H * Lk * D
    keys = min(Lk, case["topk"] * BLOCK) if case["topk"] else 0.9 * case["density"] * Lk
    pairs = int(B * H * Lq * keys)
    mask = B * H * -(-Lq // BLOCK) * -(-Lk // BLOCK)
    lse = 4 * B * H * Lq
    fwd = 2 * q_bytes + 2 * k_bytes + lse + mask
    if case["direction"] == "forward":
        return dict(bytes=fwd, flops=4 * D * pairs)
    if case["direction"] == "jvp":
        t = 2 * q_bytes + (2 * k_bytes if case["kv_tangents"] else 0)
        return dict(bytes=fwd + t, flops=(12 if case["kv_tangents"] else 8) * D * pairs)
    return dict(bytes=fwd + 2 * q_bytes + 2 * k_bytes, flops=14 * D * pairs)


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_adaln(s):
    case = s["case"]
    f = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor)}
    one = torch.ones(case["C"], dtype=torch.float64, device=f["x"].device)
    w, wp = f.get("w", one), f.get("wp", one)

    def norm(kind, x):
        if kind == "none":
            return x
        if kind == "layer":
            return (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)

    def block(x, h, mod, w, wp):
        gate, scale, shift = mod[:, None, 0], mod[:, None, 1], mod[:, None, 2]
        xn = x + gate * wp * norm(case["post"], h)
        return xn, (1 + scale) * w * norm(case["norm"], xn) + shift

    if case["direction"] == "jvp":
        zero = torch.zeros_like(one)
        (xn, y), (txn, ty) = torch.func.jvp(block, (f["x"], f["h"], f["mod"], w, wp),
                                            (f["tx"], f["th"], f["tmod"], zero, zero))
        return dict(x=xn, y=y, tx=txn, ty=ty)
    if case["direction"] == "forward":
        xn, y = block(f["x"], f["h"], f["mod"], w, wp)
        return dict(x=xn, y=y)
    args = [t.clone().requires_grad_() for t in (f["x"], f["h"], f["mod"], w, wp)]
    with torch.enable_grad():
        xn, y = block(*args)
        dx, dh, dmod, dw, dwp = torch.autograd.grad((xn, y), args, (f["dxn"], f["dy"]), allow_unused=True)
    out = dict(x=xn.detach(), y=y.detach(), dx=dx, dh=dh, dgate=dmod[:, 0], dscale=dmod[:, 1], dshift=dmod[:, 2])
    if s["w"] is not None:
        out["dw"] = dw
    if s["wp"] is not None:
        out["dwp"] = dwp
    return out


def _exact_sparse(s):
    """Query block by query block of every head, over all keys under the mask."""
    case = s["case"]
    q, k, v = (s[n].double() for n in "qkv")
    B, Lq, H, D = q.shape
    Lk = k.shape[1]
    n_q, n_k = -(-Lq // BLOCK), -(-Lk // BLOCK)
    scale = D ** -0.5
    direction = case["direction"]
    if case["topk"]:
        qm = torch.stack([b.mean(1) for b in q.split(BLOCK, 1)], 1)
        km = torch.stack([b.mean(1) for b in k.split(BLOCK, 1)], 1)
        score = torch.einsum("bihd,bjhd->bhij", qm, km)
        rank = torch.sort(torch.sort(score, dim=-1, descending=True, stable=True).indices, dim=-1).indices
        mask = rank < case["topk"]
    else:
        mask = s["mask"]
    o, lse = torch.zeros_like(q), torch.full((B, H, Lq), NEG, dtype=torch.float64, device=q.device)
    names = {"jvp": ["to"], "train": ["dq", "dk", "dv"], "forward": []}[direction]
    more = {n: torch.zeros_like(k if n in ("dk", "dv") else q) for n in names}
    key_mask = mask.repeat_interleave(BLOCK, -1)[..., :Lk].repeat_interleave(BLOCK, 2)[:, :, :Lq]
    step = max(BLOCK, (1 << 26) // Lk)
    for b in range(B):
        for h in range(H):
            K, V = k[b, :, h], v[b, :, h]
            for i in range(0, Lq, step):
                rows = slice(i, i + step)
                keep = key_mask[b, h, rows]
                some = keep.any(-1, keepdim=True)
                S = torch.where(keep, q[b, rows, h] @ K.T * scale, NEG)
                L = torch.logsumexp(S, -1)
                P = torch.where(some, torch.softmax(S, -1), 0.0)
                O = P @ V
                o[b, rows, h], lse[b, h, rows] = O, L
                if direction == "jvp":
                    tS = s["tq"][b, rows, h].double() @ K.T * scale
                    if case["kv_tangents"]:
                        tS += q[b, rows, h] @ s["tk"][b, :, h].double().T * scale
                    G = P * (tS - (P * tS).sum(-1, keepdim=True))
                    t = G @ V
                    if case["kv_tangents"]:
                        t += P @ s["tv"][b, :, h].double()
                    more["to"][b, rows, h] = t
                if direction == "train":
                    do = s["do"][b, rows, h].double()
                    dP = do @ V.T
                    dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * scale
                    more["dq"][b, rows, h] = dS @ K
                    more["dk"][b, :, h] += dS.T @ q[b, rows, h]
                    more["dv"][b, :, h] += P.T @ do
    return dict(o=o, lse=lse, mask=None, **more)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adaln(s) if case["op"] == "adaln" else _exact_sparse(s)
