"""What stands around the attention of a block, measured through the library's own entry points: rotary
positions of projected queries and keys, cross attention of a map's queries to an encoder's states, and the
norms on both sides of a block with its gate and residual scale.

`run` computes a pass in its plain form (elementary torch operations in 32 bits, rounded once at the end) or,
where `own` is true, by the calls a user makes.  `exact` says what comes out in 64 bits; its gradients come
from automatic differentiation of the definition, apart from the formulas of the plain form.
"""
import math

import torch

own = False


# ---------------------------------------------------------------- cases
def _rope(name, B, N, heads, kv_heads, head_dim, rot_dim, layout, axes=1, width=0, far=0, scaling="none", factor=1.0,
          given=False, dtype="bf16", train=False):
    """given: positions come as a tensor; far: about where in its context a sequence starts."""
    return _named(name, dict(op="rope", B=B, N=N, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot_dim=rot_dim,
                             layout=layout, axes=axes, width=width, far=far, scaling=scaling, factor=factor,
                             given=given, dtype=dtype, train=train))


def _cross(name, B, Nq, Nk, heads, kv_heads, head_dim, ragged=False, masked=False, fused=False, dtype="bf16", train=False):
    """ragged: every image has its own number of keys; masked: some keys are hidden; fused: K and V are the
    halves of one projection's output."""
    return _named(name, dict(op="cross", B=B, Nq=Nq, Nk=Nk, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                             ragged=ragged, masked=masked, fused=fused, dtype=dtype, train=train))


def _norm(name, B, N, C, pre, post="none", gate="none", per_image=False, alpha=1.0, dtype="bf16", train=False):
    """per_image: weight and bias of the norm before the next block are [B, C] (modulated by a condition)."""
    return _named(name, dict(op="norm", B=B, N=N, C=C, pre=pre, post=post, gate=gate, per_image=per_image, alpha=alpha,
                             dtype=dtype, train=train))


def _named(name, case):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # a step of generation with a few sequences, each at its own far position
        _rope("rope-decode", 16, 1, 12, 12, 64, 64, "half", far=100000, given=True),
        # first stage at 224 x 224, positions by row and column; forward and the gradients' rotation back
        _rope("rope-stage1-train", 64, 3136, 2, 2, 32, 32, "interleaved", axes=2, width=56, train=True),
        # one long sequence, a part of each head, shared key heads, a context stretched eight times, single precision
        _rope("rope-long-fp32", 1, 65537, 12, 4, 128, 64, "half", scaling="parts", factor=8.0, dtype="f32"),
        # a step of generation: one token of each sequence against its encoder's states
        _cross("cross-decode", 16, 1, 2048, 16, 4, 64, ragged=True),
        # third stage (14 x 14 maps) attending to a short, padded text
        _cross("cross-stage3-train", 64, 196, 100, 8, 8, 32, ragged=True, train=True),
        # plain vision transformer, 32 x 32 maps attending to another encoder's 32 x 32, K and V from one projection
        _cross("cross-vit-train", 16, 1024, 1024, 12, 12, 64, fused=True, train=True),
        # a dense-prediction map of 128 x 128 tokens against a long state sequence, shared key heads, some states hidden
        _cross("cross-long", 2, 16384, 4099, 8, 2, 128, masked=True),
        # second stage (28 x 28) in single precision
        _cross("cross-stage2-fp32-train", 16, 784, 196, 4, 4, 32, dtype="f32", train=True),
        # one token through one norm
        _norm("norm-one-token", 1, 1, 768, "rms"),
        # first stage: norm, gate and residual after the attention, norm before the next block
        _norm("norm-stage1-train", 64, 3136, 64, "layer", post="layer", gate="channel", train=True),
        # plain vision transformer whose norms and gates are modulated for each image
        _norm("norm-vit-train", 16, 1024, 768, "layer", gate="image", per_image=True, train=True),
        # a wide stream of an odd width, post-norm and a residual scale, single precision
        _norm("norm-wide-fp32", 8, 1024, 5001, "rms", post="rms", alpha=0.7, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    lo, hi = max(1, lo), max(1, lo, hi)
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["rope", "cross", "cross", "norm"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    train = rng.random() < 0.5
    if op == "rope":
        head_dim, kv_heads, group = rng.choice([32, 64, 128]), _log_int(rng, 1, 12), rng.choice([1, 1, 2, 3, 4])
        heads, axes = kv_heads * group, rng.choice([1, 1, 2])
        rot_dim = rng.choice([head_dim, head_dim, head_dim // 2, 3 * head_dim // 4, head_dim - 4 * axes])
        B = _log_int(rng, 1, 64)
        # tokens x channels of the largest listed case at most, a training step half of it
        room = 65537 * 16 * 128 // (2 if train else 1) // (B * (heads + kv_heads) * head_dim)
        N = _log_int(rng, 1, min(70000, room))
        scaling = rng.choice(["none", "linear", "base", "parts"]) if axes == 1 else "none"
        return _rope(None, B, N, heads, kv_heads, head_dim, rot_dim, rng.choice(["interleaved", "half"]), axes,
                     rng.randint(1, max(1, N)) if axes == 2 else 0, rng.choice([0, 0, 5000, 1000000]) if axes == 1 else 0, scaling,
                     1.0 if scaling == "none" else rng.choice([2.0, 4.0, 16.0]), rng.random() < 0.5, dtype, train)
    if op == "cross":
        head_dim, kv_heads, group = rng.choice([32, 64, 128]), _log_int(rng, 1, 12), rng.choice([1, 1, 2, 3, 4])
        heads = kv_heads * group
        # at most the products of the largest listed case; single precision a sixteenth, a training step a quarter of it
        room = 2 * 16384 * 4099 * 8 * 128 // (16 if dtype == "f32" else 1) // (4 if train else 1) // (heads * head_dim)
        B = _log_int(rng, 1, 64)
        Nk = _log_int(rng, 16, min(8192, room // B))
        Nq = _log_int(rng, 1, min(16384, room // B // Nk)) if rng.random() < 0.8 else 1
        return _cross(None, B, Nq, Nk, heads, kv_heads, head_dim, rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3,
                      dtype, train)
    C = _log_int(rng, 48, 8192)
    if rng.random() < 0.75:
        C = max(8, C // 8 * 8)
    room = 8 * 1024 * 5001 // (2 if train else 1) // C
    B = _log_int(rng, 1, min(64, room))
    return _norm(None, B, _log_int(rng, 1, room // B), C, rng.choice(["rms", "layer"]), rng.choice(["none", "none", "rms", "layer"]),
                 rng.choice(["none", "channel", "image"]), rng.random() < 0.3, rng.choice([1.0, 1.0, 0.7]), dtype, train)


# ---------------------------------------------------------------- inputs
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _data(case, seed):
    """The inputs alone, from the seed."""
    gen, t, B = _generator(seed), _type(case), case["B"]

    def normal(*shape, mean=0.0, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std + mean

    d = {}
    if case["op"] == "rope":
        N, D = case["N"], case["head_dim"]
        d["Q"], d["K"] = (normal(B, N, case[h] * D).to(t) for h in ("heads", "kv_heads"))
        if case["train"]:
            d["dQ"], d["dK"] = (normal(B, N, case[h] * D).to(t) for h in ("heads", "kv_heads"))
        d["positions"] = None
        if case["given"]:
            if case["axes"] == 2:
                d["positions"] = torch.randint(0, 512, (B, N, 2), device="cuda", generator=gen, dtype=torch.int32)
            else:   # every sequence starts somewhere else
                start = torch.randint(0, case["far"] + 4096, (B, 1), device="cuda", generator=gen, dtype=torch.int32)
                d["positions"] = (start + torch.arange(N, device="cuda", dtype=torch.int32))[..., None].contiguous()
    elif case["op"] == "cross":
        Nq, Nk, C, Ck = case["Nq"], case["Nk"], case["heads"] * case["head_dim"], case["kv_heads"] * case["head_dim"]
        d["Q"] = normal(B, Nq, C).to(t)
        if case["fused"]:
            kv = normal(B, Nk, 2 * Ck).to(t)
            d["K"], d["V"] = kv[..., :Ck], kv[..., Ck:]
        else:
            d["K"], d["V"] = normal(B, Nk, Ck).to(t), normal(B, Nk, Ck).to(t)
        if case["train"]:
            d["dO"] = normal(B, Nq, C).to(t)
        d["key_len"] = d["key_mask"] = None
        if case["ragged"]:
            d["key_len"] = torch.randint(max(2, Nk // 2), Nk + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
        if case["masked"]:
            d["key_mask"] = torch.rand(B, Nk, device="cuda", generator=gen) < 0.9
            d["key_mask"][:, :2] = True
    else:
        N, C = case["N"], case["C"]
        d["x"], d["y"] = normal(B, N, C, std=1.5, mean=0.1).to(t), normal(B, N, C).to(t)
        d["gate"] = None if case["gate"] == "none" else normal(*((B, C) if case["gate"] == "image" else (C,)), std=0.3, mean=0.5)
        of = (B, C) if case["per_image"] else (C,)
        d["w"], d["b"] = normal(*of, std=0.1, mean=1.0), normal(*of, std=0.1)
        d["post_w"], d["post_b"] = (normal(C, std=0.1, mean=1.0), normal(C, std=0.1)) if case["post"] != "none" else (None, None)
        if case["pre"] == "rms":
            d["b"] = None
        if case["post"] == "rms":
            d["post_b"] = None
        if case["train"]:
            d["dh"], d["dn"] = normal(B, N, C).to(t), normal(B, N, C).to(t)
    return d


def _frequencies(case, like=None):
    """Rotations per position of each pair of a block, in 64 bits."""
    n = case["rot_dim"] // case["axes"]
    i = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    base, factor = 10000.0, case["factor"]
    if case["scaling"] == "base" and n > 2:
        base *= factor ** (n / (n - 2))
    f = base ** (-2 * i / n)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        keep = ((4096 * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


def prepare(case, seed):
    """The inputs, and what a program keeps between calls: the problem statement, frequencies, scratch."""
    st = _data(case, seed)
    st["case"] = case
    if case["op"] == "rope":
        st["freq"] = _frequencies(case)
    if own:
        import paper_2303_08810_b200 as bra
        t = case["dtype"]
        if case["op"] == "rope":
            st["p"] = bra.make_rope_problem(case["B"], case["N"], case["heads"], case["head_dim"], kv_heads=case["kv_heads"],
                                            rot_dim=case["rot_dim"], layout=case["layout"], axes=case["axes"],
                                            width=case["width"], first=0 if case["given"] else case["far"], dtype=t)
            st["freq"] = bra.rope_frequencies(case["rot_dim"], axes=case["axes"], scaling=case["scaling"],
                                              factor=case["factor"], original_length=4096, low=1.0, high=32.0)
        elif case["op"] == "cross":
            stride = 2 * case["kv_heads"] * case["head_dim"] if case["fused"] else 0
            st["p"] = bra.make_cross_problem(case["B"], case["Nq"], case["Nk"], case["heads"], case["head_dim"],
                                             kv_heads=case["kv_heads"], dtype=t, k_stride=stride, v_stride=stride)
            st["ws"] = bra.cross_workspace(st["p"])
        else:
            st["p"] = bra.make_norm_problem(case["B"], case["N"], case["C"], pre=case["pre"], post=case["post"],
                                            gate=case["gate"], per_image=case["per_image"], alpha=case["alpha"], eps=1e-6, dtype=t)
            st["ws"] = bra.norm_workspace(st["p"])
    return st


# ---------------------------------------------------------------- plain forms
def _angles(case, positions, freq):
    """[B, N, axes, pairs] in 64 bits, then the cosine and sine in 32."""
    B, N = case["B"], case["N"]
    if positions is not None:
        pos = positions.double()
    elif case["axes"] == 2:
        n = torch.arange(N, device="cuda")
        pos = torch.stack((n // case["width"], n % case["width"]), -1).double()[None]
    else:
        pos = (case["far"] + torch.arange(N, device="cuda")).double()[None, :, None]
    angle = pos[..., None] * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rotate(case, x, cos, sin):
    B, N, D, r, axes = case["B"], case["N"], case["head_dim"], case["rot_dim"], case["axes"]
    n = r // axes
    f = x.float().reshape(B, N, -1, D)
    turn, rest = f[..., :r].reshape(B, N, -1, axes, n), f[..., r:]
    cos, sin = cos[:, :, None], sin[:, :, None]
    if case["layout"] == "interleaved":
        u, v = turn[..., 0::2], turn[..., 1::2]
        out = torch.stack((u * cos - v * sin, u * sin + v * cos), -1)
    else:
        u, v = turn[..., : n // 2], turn[..., n // 2:]
        out = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    out = out.reshape(B, N, -1, r)
    return torch.cat((out, rest), -1).reshape(x.shape).to(x.dtype)


def _plain_rope(st):
    case = st["case"]
    cos, sin = _angles(case, st["positions"], st["freq"])
    out = {"Q": _rotate(case, st["Q"], cos, sin), "K": _rotate(case, st["K"], cos, sin)}
    if case["train"]:
        out["dQ"], out["dK"] = _rotate(case, st["dQ"], cos, -sin), _rotate(case, st["dK"], cos, -sin)
    return out


def _visible(case, st):
    B, Nk = case["B"], case["Nk"]
    see = torch.ones(B, Nk, dtype=torch.bool, device="cuda")
    if st["key_len"] is not None:
        see = see & (torch.arange(Nk, device="cuda")[None] < st["key_len"][:, None])
    if st["key_mask"] is not None:
        see = see & st["key_mask"]
    return see


def _by_kv_head(case, x):
    """[B, Nq, heads * D] as [B, kv_heads, group * Nq, D] in 32 bits."""
    B, kv, D = case["B"], case["kv_heads"], case["head_dim"]
    return x.float().reshape(B, case["Nq"], kv, -1, D).permute(0, 2, 3, 1, 4).reshape(B, kv, -1, D)


def _by_token(case, x, like):
    B, kv, D = case["B"], case["kv_heads"], case["head_dim"]
    return x.reshape(B, kv, -1, case["Nq"], D).permute(0, 3, 1, 2, 4).reshape(like.shape).to(like.dtype)


def _plain_cross(st):
    case = st["case"]
    B, Nk, kv, D = case["B"], case["Nk"], case["kv_heads"], case["head_dim"]
    see = _visible(case, st)[:, None, None, :]
    scale = 1 / math.sqrt(D)
    q = _by_kv_head(case, st["Q"])
    k, v = (st[n].float().reshape(B, Nk, kv, D).transpose(1, 2) for n in ("K", "V"))
    s = torch.where(see, q @ k.transpose(2, 3) * scale, -math.inf)
    most = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = torch.exp(s - most)
    total = p.sum(-1, keepdim=True)
    p = p / total.clamp_min(1e-30)
    out = {"O": _by_token(case, p @ v, st["Q"])}
    if case["train"]:
        out["lse"] = (most + torch.log(total)).reshape(B, case["heads"], case["Nq"])
        do = _by_kv_head(case, st["dO"])
        dp = do @ v.transpose(2, 3)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        out["dQ"] = _by_token(case, ds @ k, st["Q"])
        out["dK"] = (ds.transpose(2, 3) @ q).transpose(1, 2).reshape(B, Nk, kv * D).to(st["K"].dtype)
        out["dV"] = (p.transpose(2, 3) @ do).transpose(1, 2).reshape(B, Nk, kv * D).to(st["V"].dtype)
    return out


def _normed(kind, x):
    """The normalised rows and one over their spread."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    return x * r, r


def _norm_back(kind, hat, r, g):
    """Gradient of the row from the gradient g of its normalised form."""
    back = g - hat * (g * hat).mean(-1, keepdim=True)
    if kind == "layer":
        back = back - g.mean(-1, keepdim=True)
    return back * r


def _rows(v):
    """A [C] or [B, C] vector against [B, N, C]."""
    return v[:, None] if v.dim() == 2 else v


def _plain_norm(st):
    case = st["case"]
    x, y = st["x"].float(), st["y"].float()
    yy = y
    if case["post"] != "none":
        yhat, yr = _normed(case["post"], y)
        yy = yhat * st["post_w"] + (st["post_b"] if st["post_b"] is not None else 0)
    gate = 1.0 if st["gate"] is None else _rows(st["gate"])
    h = case["alpha"] * x + gate * yy
    hat, r = _normed(case["pre"], h)
    n = hat * _rows(st["w"]) + (_rows(st["b"]) if st["b"] is not None else 0)
    t = st["x"].dtype
    out = {"h": h.to(t), "n": n.to(t)}
    if case["train"]:
        dn = st["dn"].float()
        over = (1,) if case["per_image"] else (0, 1)
        out["dw"] = (dn * hat).sum(over)
        if st["b"] is not None:
            out["db"] = dn.sum(over)
        dH = st["dh"].float() + _norm_back(case["pre"], hat, r, dn * _rows(st["w"]))
        out["dx"] = (case["alpha"] * dH).to(t)
        if st["gate"] is not None:
            out["dgate"] = (dH * yy).sum((1,) if case["gate"] == "image" else (0, 1))
        dy = gate * dH
        if case["post"] != "none":
            out["d_post_w"] = (dy * yhat).sum((0, 1))
            if st["post_b"] is not None:
                out["d_post_b"] = dy.sum((0, 1))
            dy = _norm_back(case["post"], yhat, yr, dy * st["post_w"])
        out["dy"] = dy.to(t)
    return out


# ---------------------------------------------------------------- the library's calls
def _own_rope(st):
    import paper_2303_08810_b200 as bra
    out = dict(zip(("Q", "K"), bra.bra_rope(st["p"], st["Q"], st["K"], st["freq"], st["positions"])))
    if st["case"]["train"]:
        out["dQ"], out["dK"] = bra.bra_rope(st["p"], st["dQ"], st["dK"], st["freq"], st["positions"], inverse=True)
    return out


def _own_cross(st):
    import paper_2303_08810_b200 as bra
    train = st["case"]["train"]
    O, lse = bra.bra_cross_attend(st["p"], st["Q"], st["K"], st["V"], st["key_len"], st["key_mask"], ws=st["ws"], want_lse=train)
    if not train:
        return {"O": O}
    dQ, dK, dV = bra.bra_cross_backward(st["p"], st["Q"], st["K"], st["V"], O, lse, st["dO"], st["key_len"], st["key_mask"],
                                        ws=st["ws"])
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}


def _own_norm(st):
    import paper_2303_08810_b200 as bra
    args = (st["p"], st["x"], st["y"])
    weights = {n: st[n] for n in ("gate", "post_w", "post_b", "w", "b")}
    h, n = bra.bra_residual_norm(*args, **weights)
    out = {"h": h, "n": n}
    if st["case"]["train"]:
        out.update(bra.bra_residual_norm_backward(*args, st["dh"], st["dn"], **weights, ws=st["ws"]))
    return out


def run(st):
    op = st["case"]["op"]
    if own:
        return {"rope": _own_rope, "cross": _own_cross, "norm": _own_norm}[op](st)
    return {"rope": _plain_rope, "cross": _plain_cross, "norm": _plain_norm}[op](st)


# ---------------------------------------------------------------- floors
def work(case):
    """Every input read once, every output written once, and the products and sums of the definition."""
    size, twice = (2 if case["dtype"] == "bf16" else 4), (2 if case["train"] else 1)
    B = case["B"]
    if case["op"] == "rope":
        rows = B * case["N"]
        heads = case["heads"] + case["kv_heads"]
        nbytes = rows * heads * case["head_dim"] * 2 * size + (4 * rows * case["axes"] if case["given"] else 0)
        return {"bytes": nbytes * twice, "flops": 3 * rows * heads * case["rot_dim"] * twice}
    if case["op"] == "cross":
        seen = case["Nk"] * (0.75 if case["ragged"] else 1.0)
        q, kv = B * case["Nq"] * case["heads"] * case["head_dim"], B * seen * case["kv_heads"] * case["head_dim"]
        pairs = B * case["heads"] * case["Nq"] * seen * (0.9 if case["masked"] else 1.0)
        nbytes, flops = size * (2 * q + 2 * kv), 4 * pairs * case["head_dim"]
        if case["train"]:
            every = B * case["Nk"] * case["kv_heads"] * case["head_dim"]     # gradients of hidden keys are zeros, written too
            nbytes += size * (4 * q + 2 * kv + 2 * every) + 8 * B * case["heads"] * case["Nq"]
            flops += 10 * pairs * case["head_dim"]
        return {"bytes": nbytes, "flops": flops}
    rows, C = B * case["N"], case["C"]
    nbytes = 4 * rows * C * size
    flops = rows * C * (10 + (6 if case["post"] != "none" else 0))
    if case["train"]:
        nbytes += 6 * rows * C * size
        flops += rows * C * (20 + (12 if case["post"] != "none" else 0))
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------- in 64 bits
def _exact_rope(case, st):
    B, N, D, r = case["B"], case["N"], case["head_dim"], case["rot_dim"]
    n = r // case["axes"]
    # rotation of channel c: partner, sign, coordinate and pair
    c = torch.arange(r, device="cuda")
    axis, at = c // n, c % n
    if case["layout"] == "interleaved":
        pair, second = at // 2, at % 2 == 1
        partner = torch.where(second, c - 1, c + 1)
    else:
        pair, second = at % (n // 2), at >= n // 2
        partner = torch.where(second, c - n // 2, c + n // 2)
    token = torch.arange(N, device="cuda", dtype=torch.float64)
    if st["positions"] is not None:
        place = st["positions"].double()
    elif case["axes"] == 2:
        place = torch.stack((torch.floor(token / case["width"]), torch.remainder(token, case["width"])), 1).expand(B, N, 2)
    else:
        place = (token + case["far"])[:, None].expand(B, N, 1)
    angle = place[:, :, axis] * _frequencies(case)[pair]
    out = {}
    for name, way in (("Q", 1.0), ("K", 1.0), ("dQ", -1.0), ("dK", -1.0)):
        if name in st:
            x = st[name].double().view(B, N, -1, D)
            sign = torch.where(second, way, -way)
            z = x.clone()
            z[..., :r] = x[..., :r] * angle.cos()[:, :, None] + x[..., partner] * (sign * angle.sin())[:, :, None]
            out[name] = z.view(B, N, -1)
    return out


def _exact_cross(case, st):
    group, D = case["heads"] // case["kv_heads"], case["head_dim"]
    names = ["O"] + (["lse", "dQ", "dK", "dV"] if case["train"] else [])
    parts = {n: [] for n in names}
    see = _visible(case, st)
    for b in range(case["B"]):
        q, k, v = (st[n][b].double().requires_grad_(case["train"]) for n in ("Q", "K", "V"))
        with torch.set_grad_enabled(case["train"]):
            heads = [q.view(case["Nq"], -1, D).transpose(0, 1)]
            heads += [x.view(case["Nk"], -1, D)[see[b]].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v)]
            s = torch.einsum("hid,hjd->hij", heads[0], heads[1]) / math.sqrt(D)
            lse = torch.logsumexp(s, -1)
            O = torch.einsum("hij,hjd->ihd", torch.exp(s - lse[..., None]), heads[2]).reshape(case["Nq"], -1)
        parts["O"].append(O.detach())
        if case["train"]:
            parts["lse"].append(lse.detach())
            for n, g in zip(("dQ", "dK", "dV"), torch.autograd.grad(O, (q, k, v), st["dO"][b].double())):
                parts[n].append(g)
    return {n: torch.stack(v) for n, v in parts.items()}


def _exact_norm(case, st):
    names = [n for n in ("x", "y", "gate", "post_w", "post_b", "w", "b") if st.get(n) is not None]
    a = {n: st[n].double().requires_grad_(case["train"]) for n in names}

    def norm(kind, v):
        centred = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        return centred / torch.sqrt(centred.square().mean(-1, keepdim=True) + 1e-6)

    def wide(v):
        return v.unsqueeze(1) if v.dim() == 2 else v

    with torch.set_grad_enabled(case["train"]):
        y = a["y"]
        if case["post"] != "none":
            y = norm(case["post"], y) * a["post_w"] + a.get("post_b", 0.0)
        h = case["alpha"] * a["x"] + (y * wide(a["gate"]) if "gate" in a else y)
        n = norm(case["pre"], h) * wide(a["w"]) + (wide(a["b"]) if "b" in a else 0.0)
    out = {"h": h.detach(), "n": n.detach()}
    if case["train"]:
        grads = torch.autograd.grad((h, n), [a[k] for k in names], (st["dh"].double(), st["dn"].double()))
        out.update({("d_" if k.startswith("post") else "d") + k: g for k, g in zip(names, grads)})
    return out


def exact(case, seed):
    st = _data(case, seed)
    return {"rope": _exact_rope, "cross": _exact_cross, "norm": _exact_norm}[case["op"]](case, st)
