"""The operators in front of and behind the attention core in training, case by case: rotary tables (``table``), the per-head
norm and rotation of queries and keys (``rotary``: forward, with tangents, in training) and dense attention with shared
heads, padded contexts and a causal mask (``attention``: forward and in training).

``run`` computes a case in plain torch operations (32-bit arithmetic, 64-bit angles) where ``own`` is false and through the
framework's entry points where it is true; ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
NEG = -math.inf


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _table(name, L, dims, scaling="none", factor=1.0, fractional=False):
    return dict(name=name, op="table", L=L, dims=dims, scaling=scaling, factor=factor, fractional=fractional)


def _rotary(name, direction, B, L, H, Hk, D, R, layout="interleaved", norm="rms", affine=True, fused=False, index=False):
    return dict(name=name, op="rotary", direction=direction, B=B, L=L, H=H, Hk=Hk, D=D, R=R, layout=layout, norm=norm,
                affine=affine, fused=fused, index=index)


def _attention(name, direction, B, H, Hk, Lq, Lk, D, causal=False, lengths="", fused=False):
    return dict(name=name, op="attention", direction=direction, B=B, H=H, Hk=Hk, Lq=Lq, Lk=Lk, D=D, causal=causal,
                lengths=lengths, fused=fused)


def listed():
    return [
        # positions (frame, row, column) of the 32760 latent tokens of an 832x480x81 video, frames at their times
        _table("table_video", 32760, "44,42,42", fractional=True),
        # one long sequence, stretched eight times beyond the length of training
        _table("table_long", 262144, "128", scaling="yarn", factor=8.0),
        # one new token for each of eight requests at places of their own, shared key heads: launch latency
        _rotary("rotary_token", "forward", 8, 1, 40, 8, 128, 128, layout="half", index=True),
        # queries and keys of a 14B-shaped video DiT, slices of one projection, sampling
        _rotary("rotary_video_14b", "forward", 1, 32760, 40, 40, 128, 128, fused=True),
        # image DiT in JVP mode
        _rotary("rotary_jvp_image_2b", "jvp", 2, 4096, 16, 16, 128, 128),
        # student step of the 1.3B-shaped video DiT, with the gradients of the norms' weights
        _rotary("rotary_train_video_1p3b", "train", 1, 32760, 12, 12, 128, 128),
        # half of each head rotated, layer norm, shared key heads, odd length, D = 64
        _rotary("rotary_train_part_d64", "train", 3, 4001, 24, 6, 64, 32, layout="half", norm="layer", fused=True),
        # a short sequence against a short context: launch latency
        _attention("attention_train_short", "train", 1, 2, 2, 200, 333, 64),
        # image DiT, student step
        _attention("attention_train_image_2b", "train", 2, 16, 16, 4096, 4096, 128),
        # 1.3B-shaped video DiT, student step
        _attention("attention_train_video_1p3b", "train", 1, 12, 12, 32760, 32760, 128),
        # image tokens against padded text contexts, one of them dropped (guidance)
        _attention("attention_train_context", "train", 3, 16, 16, 8190, 512, 128, lengths="77,0,512"),
        # causal student step with shared key heads, slices of one projection, odd length, D = 64
        _attention("attention_train_causal_d64", "train", 2, 24, 6, 4001, 4001, 64, causal=True, lengths="4001,3277", fused=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["table", "rotary", "rotary", "attention", "attention"])
    if op == "table":
        dims = rng.choice(["128", "64", "32", "44,42,42", "16,24,24", "64,64"])
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return dict(op=op, L=_log_int(rng, 1, 262144), dims=dims, scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0), fractional=rng.random() < 0.3)
    B, D = rng.randint(1, 4), rng.choice([64, 128])
    Hk = rng.randint(1, 8)
    H = Hk * rng.choice([1, 1, 2, 4])
    if op == "rotary":
        norm = rng.choice(["none", "rms", "rms", "layer"])
        return dict(op=op, direction=rng.choice(["forward", "jvp", "train"]), B=B, L=_log_int(rng, 1, 32760 // B), H=H,
                    Hk=rng.choice([0, Hk, Hk, Hk]), D=D, R=16 * rng.randint(1, D // 16), layout=rng.choice(["interleaved", "half"]),
                    norm=norm, affine=norm != "none" and rng.random() < 0.7, fused=rng.random() < 0.5, index=rng.random() < 0.3)
    B = rng.randint(1, 3)
    Lq = _log_int(rng, 1, 16000)
    same = rng.random() < 0.5
    # two keys at least: with a single one every gradient that is left is exactly 0, and only rounding is compared
    Lk = max(2, Lq if same else _log_int(rng, 2, 16000))
    Lq = Lk if same else Lq
    H, Hk = min(H, 16), min(Hk, min(H, 16))
    H -= H % Hk
    lengths = ""
    if rng.random() < 0.5:
        lengths = ",".join(str(rng.choice([Lk, Lk, _log_int(rng, 2, Lk), rng.choice([0, _log_int(rng, 2, Lk)])])) for _ in range(B))
        if all(n == "0" for n in lengths.split(",")):
            lengths = ""
    return dict(op=op, direction=rng.choice(["forward", "train", "train"]), B=B, H=H, Hk=Hk, Lq=Lq, Lk=Lk, D=D,
                causal=same and rng.random() < 0.5, lengths=lengths, fused=same and rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
ORIGINAL_LENGTH = 4096         # of training, before a table is stretched
TABLE_ROWS = 40000             # rows of a table that is read by index


def _dims(case):
    return [int(d) for d in case["dims"].split(",")]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, sigma=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)

    def randint(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda")

    s = dict(case=case)
    if case["op"] == "table":
        L, A = case["L"], len(_dims(case))
        t = torch.arange(L, device="cuda")
        if A == 1:
            pos = t + randint(0, 1 << 20, 1)
        else:
            rows, cols = 30, 52                                 # a latent frame of 480 x 832
            grid = [t // (rows * cols), t // cols % rows, t % cols] if A == 3 else [t // cols, t % cols]
            pos = torch.stack(grid, -1) + randint(0, 64, 1, A)
        # times of frames that are not a whole number of steps apart, else token places
        s["positions"] = (pos * 0.9375).float() if case["fractional"] else pos.int()
        return s

    if case["op"] == "rotary":
        B, L, H, Hk, D, R = (case[k] for k in ("B", "L", "H", "Hk", "D", "R"))
        # head channels of unlike size, as trained projections have
        loud = torch.exp(randn(H + 2 * Hk, D, sigma=0.5, dtype=torch.float32))

        def heads():
            x = (torch.randn(B, L, H + 2 * Hk, D, generator=g, device="cuda") * loud).to(torch.bfloat16)
            q, k = x[:, :, :H], x[:, :, H:H + Hk] if Hk else None
            return (q, k) if case["fused"] else (q.contiguous(), None if k is None else k.contiguous())

        s["q"], s["k"] = heads()
        rows = TABLE_ROWS if case["index"] else L
        theta = 10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) / (R // 2))
        angle = (torch.arange(rows, device="cuda") + randint(0, 1000, 1)).double()[:, None] * theta
        s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["index"] = None
        if case["index"]:
            # every request somewhere else in its sequence
            start = randint(0, TABLE_ROWS - L + 1, B, 1)
            s["index"] = (start + torch.arange(L, device="cuda")).int()
        for n in ("qw", "kw", "qb", "kb"):
            wanted = case["affine"] and (n[0] == "q" or Hk) and (n[1] == "w" or case["norm"] == "layer")
            s[n] = randn(D, sigma=0.2, dtype=torch.float32) + (1 if n[1] == "w" else 0) if wanted else None
        if case["direction"] == "jvp":
            s["tq"], s["tk"] = heads()
        if case["direction"] == "train":
            s["dq"] = randn(B, L, H, D)
            s["dk"] = randn(B, L, Hk, D) if Hk else None
        return s

    B, H, Hk, Lq, Lk, D = (case[k] for k in ("B", "H", "Hk", "Lq", "Lk", "D"))
    if case["fused"]:
        x = randn(B, Lq, H + 2 * Hk, D)
        s["q"], s["k"], s["v"] = x[:, :, :H], x[:, :, H:H + Hk], x[:, :, H + Hk:]
    else:
        s["q"], s["k"], s["v"] = randn(B, Lq, H, D), randn(B, Lk, Hk, D), randn(B, Lk, Hk, D)
    s["lengths"] = None
    if case["lengths"]:
        s["lengths"] = torch.tensor([int(n) for n in case["lengths"].split(",")], dtype=torch.int32, device="cuda")
    if case["direction"] == "train":
        s["do"] = randn(B, Lq, H, D)
    return s


# ---------------------------------------------------------------------------------------------------------------
# table, plain
# ---------------------------------------------------------------------------------------------------------------
def _table_plain(s):
    case, pos = s["case"], s["positions"].double()
    pos = pos.view(case["L"], -1)
    scaling, f = case["scaling"], case["factor"]
    angles, size = [], 1.0
    for a, d in enumerate(_dims(case)):
        step = torch.arange(d // 2, device=pos.device, dtype=torch.float64) * (2.0 / d)
        base = 10000.0 * f ** (d / (d - 2)) if scaling == "ntk" else 10000.0
        theta = torch.exp(-math.log(base) * step)
        if scaling == "linear":
            theta = theta / f
        if scaling == "yarn":
            # turns within the original length: frequencies below 1 are stretched, above 32 kept, a ramp between
            keep = ((ORIGINAL_LENGTH * theta / (2 * math.pi) - 1) / 31).clamp(0, 1)
            theta = theta / f * (1 - keep) + theta * keep
            size = 0.1 * math.log(f) + 1
        angles.append(pos[:, a, None] * theta)
    angle = torch.cat(angles, -1)
    return (torch.stack([angle.cos(), angle.sin()], -1) * size).float()


def _table_own(s):
    import paper_2510_08431_b200 as aj
    case = s["case"]
    scaling = None if case["scaling"] == "none" else case["scaling"]
    return aj.rotary_table(s["positions"], _dims(case), base=10000.0, scaling=scaling, factor=case["factor"],
                           original_length=ORIGINAL_LENGTH if scaling == "yarn" else None)


# ---------------------------------------------------------------------------------------------------------------
# rotary, plain
# ---------------------------------------------------------------------------------------------------------------
def _turn(x, cos, sin, layout):
    """The first R channels rotated by pairs, the others as they are."""
    R = 2 * cos.shape[-1]
    r, rest = x[..., :R], x[..., R:]
    if layout == "half":
        a, b = r[..., :R // 2], r[..., R // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _head_norm(x, kind):
    if kind == "none":
        return x, None
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    r = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * r, r


def _head_norm_tangent(n, r, t, kind):
    if kind == "none":
        return t
    c = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    return r * (c - n * (n * c).mean(-1, keepdim=True))


def _rotary_plain(s):
    case = s["case"]
    norm, layout = case["norm"], case["layout"]
    cs = s["table"] if s["index"] is None else s["table"][s["index"].long()]
    cos, sin = (t.unsqueeze(-2) for t in cs.unbind(-1))              # [..., 1 (heads), R / 2]
    out = {}
    for n in "qk":
        if s[n] is None:
            continue
        w = 1.0 if s[n + "w"] is None else s[n + "w"]
        b = 0.0 if s[n + "b"] is None else s[n + "b"]
        h, r = _head_norm(s[n].float(), norm)
        out[n] = _turn(h * w + b, cos, sin, layout).to(torch.bfloat16)
        if case["direction"] == "jvp":
            out["t" + n] = _turn(_head_norm_tangent(h, r, s["t" + n].float(), norm) * w, cos, sin, layout).to(torch.bfloat16)
        if case["direction"] == "train":
            du = _turn(s["d" + n].float(), cos, -sin, layout)
            out["d" + n] = _head_norm_tangent(h, r, du * w, norm).to(torch.bfloat16)
            if s[n + "w"] is not None:
                out["d" + n + "w"] = (du * h).sum((0, 1, 2))
            if s[n + "b"] is not None:
                out["d" + n + "b"] = du.sum((0, 1, 2))
    return out


def _rotary_own(s):
    import paper_2510_08431_b200 as aj
    case = s["case"]
    args = dict(index=s["index"], norm=None if case["norm"] == "none" else case["norm"], layout=case["layout"], eps=EPS,
                q_weight=s["qw"], k_weight=s["kw"], q_bias=s["qb"], k_bias=s["kb"])
    jvp = case["direction"] == "jvp"
    q, k, tq, tk = aj.qk_rotary_jvp(s["q"], s["k"], s["table"], **args, tq=s["tq"] if jvp else None, tk=s["tk"] if jvp else None)
    out = dict(q=q, k=k, tq=tq, tk=tk)
    if case["direction"] == "train":
        d = aj.qk_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["table"], **args)
        out.update(dq=d.q, dk=d.k, dqw=d.q_weight, dkw=d.k_weight, dqb=d.q_bias, dkb=d.k_bias)
    order = [n for c in "qk" for n in (c, "t" + c, "d" + c, "d" + c + "w", "d" + c + "b")]
    return {n: out[n] for n in order if out.get(n) is not None}


# ---------------------------------------------------------------------------------------------------------------
# attention, plain
# ---------------------------------------------------------------------------------------------------------------
def _attention_plain(s):
    case = s["case"]
    B, H, Hk, Lq, Lk, D = (case[k] for k in ("B", "H", "Hk", "Lq", "Lk", "D"))
    scale = 1 / math.sqrt(D)

    def heads(x, n):                                                 # [B][L][H][D] -> [B][H][L][D], shared heads repeated
        return x.float().transpose(1, 2).repeat_interleave(n, 1)

    q, k, v = heads(s["q"], 1), heads(s["k"], H // Hk), heads(s["v"], H // Hk)
    train = case["direction"] == "train"
    do = heads(s["do"], 1) if train else None
    kt, vt = k.transpose(-1, -2), v.transpose(-1, -2)
    key = torch.arange(Lk, device=q.device)
    length = torch.full((B,), Lk, device=q.device) if s["lengths"] is None else s["lengths"]
    hidden = (key >= length.view(B, 1, 1, 1))
    o, lse = torch.empty_like(q), torch.empty(B, H, Lq, device=q.device)
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v)) if train else (None,) * 3
    step = max(1, (1 << 28) // (B * H * Lk))
    for i in range(0, Lq, step):
        rows = slice(i, min(Lq, i + step))
        S = (q[:, :, rows] @ kt).mul_(scale)
        masked = hidden
        if case["causal"]:
            masked = hidden | (key > torch.arange(rows.start, rows.stop, device=q.device)[:, None] + (Lk - Lq))
        S.masked_fill_(masked, NEG)
        m = S.amax(-1, keepdim=True)
        m = torch.where(m == NEG, 0.0, m)
        P = S.sub_(m).exp_()
        l = P.sum(-1, keepdim=True)
        lse[:, :, rows] = (m + l.log())[..., 0]
        P.div_(torch.where(l == 0, 1.0, l))
        o[:, :, rows] = P @ v
        if train:
            d = do[:, :, rows]
            dv += P.transpose(-1, -2) @ d
            dS = (d @ vt).sub_((d * o[:, :, rows]).sum(-1, keepdim=True)).mul_(P).mul_(scale)
            dq[:, :, rows] = dS @ k
            dk += dS.transpose(-1, -2) @ q[:, :, rows]

    def tokens(x, n):                                                # and back, summed over the heads that share one
        return x.unflatten(1, (-1, n)).sum(2).transpose(1, 2).to(torch.bfloat16).contiguous()

    out = dict(o=tokens(o, 1), lse=lse)
    if train:
        out.update(dq=tokens(dq, 1), dk=tokens(dk, H // Hk), dv=tokens(dv, H // Hk))
    return out


def _attention_own(s):
    import paper_2510_08431_b200 as aj
    case = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    masks = dict(causal=case["causal"], k_lengths=s["lengths"])
    o, _, lse = aj.attention_jvp(q, k, v, fwd_only=True, **masks)
    out = dict(o=o, lse=lse)
    if case["direction"] == "train":
        out["dq"], out["dk"], out["dv"] = aj.attention_backward(s["do"], q, k, v, o, lse, **masks)
    return out


def run(state):
    plain, mine = {"table": (_table_plain, _table_own), "rotary": (_rotary_plain, _rotary_own),
                   "attention": (_attention_plain, _attention_own)}[state["case"]["op"]]
    return mine(state) if own else plain(state)


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "table":
        dims = _dims(case)
        return dict(bytes=case["L"] * 4 * (len(dims) + sum(dims)), flops=case["L"] * 20 * sum(dims))
    if case["op"] == "rotary":
        B, L, D, R = (case[k] for k in ("B", "L", "D", "R"))
        cells = B * L * (case["H"] + case["Hk"]) * D
        table = 4 * R * (B * L if case["index"] else L)
        flops = 8 * cells
        if case["direction"] == "forward":
            return dict(bytes=4 * cells + table, flops=flops)
        if case["direction"] == "jvp":
            return dict(bytes=8 * cells + table, flops=18 * cells)
        return dict(bytes=8 * cells + table, flops=24 * cells)
    B, H, Hk, Lq, Lk, D = (case[k] for k in ("B", "H", "Hk", "Lq", "Lk", "D"))
    lengths = [int(n) for n in case["lengths"].split(",")] if case["lengths"] else [Lk] * B
    if case["causal"]:
        # query i sees the keys up to i + Lk - Lq: the first n of them within a length
        off = Lk - Lq + 1
        pairs = sum(min(n, max(0, i + off)) for n in lengths for i in range(Lq))
    else:
        pairs = Lq * sum(lengths)
    q_bytes, k_bytes = 2 * B * H * Lq * D, 2 * sum(lengths) * Hk * D
    fwd = 2 * q_bytes + 2 * k_bytes + 4 * B * H * Lq
    if case["direction"] == "forward":
        return dict(bytes=fwd, flops=4 * D * H * pairs)
    return dict(bytes=fwd + 2 * q_bytes + 4 * B * Lk * Hk * D, flops=14 * D * H * pairs)


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_table(s):
    case = s["case"]
    dims, f = _dims(case), case["factor"]
    theta, axis = [], []
    for a, d in enumerate(dims):
        for i in range(d // 2):
            base = 10000.0
            if case["scaling"] == "ntk":
                base *= math.pow(f, d / (d - 2))
            t = math.pow(base, -2.0 * i / d)
            if case["scaling"] == "linear":
                t /= f
            if case["scaling"] == "yarn":
                ramp = min(1.0, max(0.0, (ORIGINAL_LENGTH * t / (2 * math.pi) - 1) / (32 - 1)))
                t = (1 - ramp) * t / f + ramp * t
            theta.append(t)
            axis.append(a)
    pos = s["positions"].double().reshape(case["L"], len(dims))[:, axis]
    z = torch.polar(torch.ones_like(pos), pos * torch.tensor(theta, dtype=torch.float64, device=pos.device))
    size = 0.1 * math.log(f) + 1 if case["scaling"] == "yarn" else 1.0
    return torch.view_as_real(z) * size


def _exact_rotary(s):
    case = s["case"]
    R, D = case["R"], case["D"]
    table = s["table"].double()
    if s["index"] is not None:
        table = table[s["index"].long()]
    z = torch.view_as_complex(table).unsqueeze(-2)

    def head(x, w, b):
        if case["norm"] == "layer":
            x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
        elif case["norm"] == "rms":
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
        x = x * w + b
        if case["layout"] == "half":
            pairs = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * z
            turned = torch.cat([pairs.real, pairs.imag], -1)
        else:
            pairs = torch.complex(x[..., 0:R:2], x[..., 1:R:2]) * z
            turned = torch.view_as_real(pairs).flatten(-2)
        return torch.cat([turned, x[..., R:]], -1)

    out = {}
    for n in "qk":
        if s[n] is None:
            continue
        one = torch.ones(D, dtype=torch.float64, device="cuda")
        x = s[n].double()
        w = one if s[n + "w"] is None else s[n + "w"].double()
        b = 0 * one if s[n + "b"] is None else s[n + "b"].double()
        if case["direction"] == "jvp":
            out[n], out["t" + n] = torch.func.jvp(lambda t: head(t, w, b), (x,), (s["t" + n].double(),))
        elif case["direction"] == "train":
            args = [t.clone().requires_grad_() for t in (x, w, b)]
            with torch.enable_grad():
                y = head(*args)
                dx, dw, db = torch.autograd.grad(y, args, s["d" + n].double())
            out[n], out["d" + n] = y.detach(), dx
            if s[n + "w"] is not None:
                out["d" + n + "w"] = dw
            if s[n + "b"] is not None:
                out["d" + n + "b"] = db
        else:
            out[n] = head(x, w, b)
    return out


def _exact_attention(s):
    """Head by head of every batch, over the keys that its length leaves."""
    case = s["case"]
    B, H, Hk, Lq, Lk, D = (case[k] for k in ("B", "H", "Hk", "Lq", "Lk", "D"))
    train = case["direction"] == "train"
    q, k, v = (s[n].double() for n in "qkv")
    o, lse = torch.zeros_like(q), torch.full((B, H, Lq), NEG, dtype=torch.float64, device=q.device)
    dq, dk, dv = (torch.zeros(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
    lengths = [Lk] * B if s["lengths"] is None else s["lengths"].tolist()
    for b in range(B):
        n = lengths[b]
        if n == 0:
            continue
        j = torch.arange(n, device=q.device)
        step = max(128, (1 << 27) // n)
        for h in range(H):
            K, V = k[b, :n, h * Hk // H], v[b, :n, h * Hk // H]
            for i in range(0, Lq, step):
                rows = torch.arange(i, min(Lq, i + step), device=q.device)
                Q = q[b, rows, h]
                S = Q @ K.T / math.sqrt(D)
                if case["causal"]:
                    S = torch.where(j <= rows[:, None] + (Lk - Lq), S, NEG)
                L = torch.logsumexp(S, -1)
                P = torch.where(L[:, None] == NEG, 0.0, torch.exp(S - L[:, None]))
                o[b, rows, h], lse[b, h, rows] = P @ V, L
                if train:
                    d = s["do"][b, rows, h].double()
                    dP = d @ V.T
                    dS = P * (dP - (P * dP).sum(-1, keepdim=True)) / math.sqrt(D)
                    dq[b, rows, h] = dS @ K
                    dk[b, :n, h * Hk // H] += dS.T @ Q
                    dv[b, :n, h * Hk // H] += P.T @ d
    out = dict(o=o, lse=lse)
    if train:
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"table": _exact_table, "rotary": _exact_rotary, "attention": _exact_attention}[case["op"]](s)
