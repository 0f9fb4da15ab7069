"""Rotary positions, cross attention and residual norms on the GPU, through the public calls, against their definitions in 64 bits.

Tolerances are bounds, derived here before any run: u is half a step of the outputs' type (2^-8 for bf16, 2^-24 for fp32), every
fp32 sum of n terms is off by at most n 2^-24 of the sum of their magnitudes, and in bf16 problems P and dS are rounded once to
bf16 before the products that contract over them.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def bra():
    import paper_2303_08810_b200 as pkg
    from paper_2303_08810_b200 import build
    build.build_library()
    pkg.load_library()
    return pkg


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else E


def torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def randn(seed, *shape, dtype="bf16", std=1.0, mean=0.0):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(*shape, device="cuda", generator=gen) * std + mean).to(torch_type(dtype))


def within(got, ref, bound, what):
    """|got - ref| <= bound everywhere; infinities have to be the same ones."""
    import torch
    got = got.double()
    finite = torch.isfinite(ref)
    assert torch.equal(got[~finite], ref[~finite]), what
    off = (got - ref)[finite].abs() / bound[finite].clamp_min(1e-300)
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times its bound"         # a NaN fails this too


# ---------------------------------------------------------------- rotary positions
def rope_ref(x, positions, freq, rot, layout, axes, D, sign=1.0, magnitude=1.0):
    """The definition, pair by pair; also |u| + |v| of each channel's pair."""
    import torch
    B, N, C = x.shape
    y = x.double().reshape(B, N, C // D, D).clone()
    size = torch.zeros_like(y)
    n = rot // axes
    for a in range(axes):
        for i in range(n // 2):
            c0 = a * n + (2 * i if layout == "interleaved" else i)
            c1 = c0 + (1 if layout == "interleaved" else n // 2)
            angle = positions[..., a].double() * float(freq[i])
            c, s = magnitude * torch.cos(angle)[..., None], sign * magnitude * torch.sin(angle)[..., None]
            u, v = y[..., c0].clone(), y[..., c1].clone()
            y[..., c0], y[..., c1] = u * c - v * s, u * s + v * c
            size[..., c0] = size[..., c1] = (u.abs() + v.abs()) * magnitude
    return y.reshape(B, N, C), size.reshape(B, N, C)


ROPE = [
    # B, N, heads, kv, D, rot, layout, axes, given
    (1, 1, 1, 1, 2, 2, "interleaved", 1, False),
    (1, 1, 1, 0, 8, 8, "half", 1, False),
    (16, 1, 12, 12, 64, 64, "half", 1, True),
    (2, 49, 2, 2, 32, 32, "interleaved", 2, False),
    (3, 35, 3, 1, 32, 32, "half", 2, False),
    (2, 77, 4, 2, 64, 28, "half", 1, False),                     # halves of 14 channels
    (2, 77, 4, 2, 64, 28, "interleaved", 1, False),              # a part of a 16-byte unit
    (1, 130, 5, 3, 20, 12, "half", 2, True),                     # rows that start on 8 bytes
    (1, 33, 3, 2, 7, 6, "interleaved", 1, False),                # odd head dim
    (1, 33, 3, 2, 7, 6, "half", 1, True),
    (1, 2049, 8, 2, 128, 64, "half", 1, False),
    (2, 700, 2, 2, 96, 96, "interleaved", 2, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope(bra, case, dtype):
    import torch
    B, N, heads, kv, D, rot, layout, axes, given = case
    first, width = 0 if axes == 2 else 11, 7
    p = bra.make_rope_problem(B, N, heads, D, kv_heads=kv, rot_dim=rot, layout=layout, axes=axes, width=width, first=first, dtype=dtype,
                              magnitude=1.25)
    freq = bra.rope_frequencies(rot, axes=axes)
    n = torch.arange(N, device="cuda")
    pos = (torch.stack((n // width, n % width), -1) if axes == 2 else (n + first)[:, None]).expand(B, N, axes)
    positions = None
    if given:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        positions = torch.randint(0, 2 ** 20, (B, N, axes), device="cuda", generator=gen, dtype=torch.int32)
        pos = positions
    Q = randn(1, B, N, heads * D, dtype=dtype)
    K = randn(2, B, N, kv * D, dtype=dtype) if kv else None
    for inverse in (False, True):
        Qo, Ko = bra.bra_rope(p, Q, K, freq, positions, inverse=inverse)
        assert bra.last_launch_count() == 1
        for x, got in ((Q, Qo), (K, Ko)):
            if x is None:
                assert got is None
                continue
            ref, size = rope_ref(x, pos, freq, rot, layout, axes, D, -1.0 if inverse else 1.0, 1.25)
            # the angle's turns go to 32 bits (2^-25 turns = 2^-22.3), sine and cosine are off by 2^-23, two products and a sum
            within(got, ref, half_step(dtype) * ref.abs() + 2.0 ** -20 * size, "rope")
            assert torch.equal(got.view(B, N, -1, D)[..., rot:], x.view(B, N, -1, D)[..., rot:])
    # in place, to the same bits
    again = bra.bra_rope(p, Q, K, freq, positions)
    q, k = Q.clone(), None if K is None else K.clone()
    bra.bra_rope(p, q, k, freq, positions, Qo=q, Ko=k)
    assert torch.equal(q, again[0]) and (k is None or torch.equal(k, again[1]))


def test_rope_far_positions(bra):
    """Angles are formed in 64 bits: positions near 2^31 turn as exactly as near ones."""
    import torch
    p = bra.make_rope_problem(1, 64, 1, 32, dtype="f32")
    freq = bra.rope_frequencies(32)
    pos = (2 ** 31 - 1 - 12345 * torch.arange(64, device="cuda", dtype=torch.int64)).to(torch.int32).view(1, 64, 1)
    Q, K = randn(1, 1, 64, 32, dtype="f32"), randn(2, 1, 64, 32, dtype="f32")
    Qo, _ = bra.bra_rope(p, Q, K, freq, pos)
    ref, size = rope_ref(Q, pos, freq, 32, "interleaved", 1, 32)
    # the product of a position and a frequency in 64 bits is off by 2^-53 of up to 2^31 radians
    within(Qo, ref, (2.0 ** -20 + 2.0 ** -22) * size, "far")


def test_rope_on_slices_of_a_fused_projection(bra):
    """Q and K inside one [B, N, (heads + 2 kv) D] tensor, rotated in place; V and the rest stay as they are."""
    import torch
    B, N, heads, kv, D = 2, 75, 4, 2, 32
    fused = randn(5, B, N, (heads + 2 * kv) * D)
    before = fused.clone()
    stride = fused.shape[-1]
    p = bra.make_rope_problem(B, N, heads, D, kv_heads=kv, q_stride=stride, k_stride=stride)
    Q, K = fused[..., :heads * D], fused[..., heads * D:(heads + kv) * D]
    freq = bra.rope_frequencies(D)
    dense = bra.make_rope_problem(B, N, heads, D, kv_heads=kv)
    want = bra.bra_rope(dense, Q.contiguous(), K.contiguous(), freq)
    new = bra.bra_rope(p, Q, K, freq)
    assert torch.equal(new[0], want[0]) and torch.equal(new[1], want[1]) and torch.equal(fused, before)
    bra.bra_rope(p, Q, K, freq, Qo=Q, Ko=K)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1])
    assert torch.equal(fused[..., (heads + kv) * D:], before[..., (heads + kv) * D:])


def test_rope_infinities_stay_in_their_pair(bra):
    import torch
    p = bra.make_rope_problem(1, 3, 1, 16, kv_heads=0, rot_dim=12)
    Q = randn(1, 1, 3, 16)
    clean = bra.bra_rope(p, Q, None, bra.rope_frequencies(12))[0]
    Q[0, 1, 2], Q[0, 1, 13] = math.inf, math.nan
    got = bra.bra_rope(p, Q, None, bra.rope_frequencies(12))[0]
    touched = torch.zeros(16, dtype=torch.bool, device="cuda")
    touched[[2, 3, 13]] = True
    assert torch.equal(got[0, 1][~touched], clean[0, 1][~touched]) and not torch.isfinite(got[0, 1][touched]).any()
    assert torch.equal(got[0, [0, 2]], clean[0, [0, 2]])


# ---------------------------------------------------------------- cross attention
def cross_ref(Q, K, V, dO, see, heads, kv, D, scale, dtype, O_used=None):
    """Outputs and gradients in 64 bits, head by head, each with its bound."""
    import torch
    B, Nq, Nk, g = Q.shape[0], Q.shape[1], K.shape[1], heads // kv
    u, up = half_step(dtype), (2.0 ** -8 if dtype == "bf16" else 0.0)
    out = {n: torch.zeros(B, Nq, heads, D, dtype=torch.float64, device="cuda") for n in ("O", "O_", "dQ", "dQ_")}
    out |= {n: torch.zeros(B, Nk, kv, D, dtype=torch.float64, device="cuda") for n in ("dK", "dK_", "dV", "dV_")}
    out |= {n: torch.zeros(B, heads, Nq, dtype=torch.float64, device="cuda") for n in ("lse", "lse_")}
    q4, d4 = Q.double().reshape(B, Nq, heads, D), dO.double().reshape(B, Nq, heads, D)
    k4, v4 = K.double().reshape(B, Nk, kv, D), V.double().reshape(B, Nk, kv, D)
    for b in range(B):
        at = see[b].nonzero()[:, 0]
        for h in range(heads):
            q, do, k, v = q4[b, :, h], d4[b, :, h], k4[b, at, h // g], v4[b, at, h // g]
            if not len(at):
                out["lse"][b, h] = -math.inf
                continue
            s = q @ k.T * scale
            lse = torch.logsumexp(s, -1)
            P = torch.exp(s - lse[:, None])
            O = P @ v
            e_s = (D + 4) * E * scale * (q.abs() @ k.abs().T)                    # of a score
            e_p = 2 * e_s.amax(-1, keepdim=True) + 2.0 ** -20 + len(at) * E     # of P, relative
            O_ = u * O.abs() + (e_p + up) * (P @ v.abs())
            out["O"][b, :, h], out["O_"][b, :, h] = O, O_
            out["lse"][b, h], out["lse_"][b, h] = lse, e_s.amax(-1) + 2.0 ** -20 + len(at) * E + 4 * E * lse.abs()
            dP = do @ v.T
            delta = (do * O).sum(-1, keepdim=True)
            dS = P * (dP - delta)
            e_dp = (D + 4) * E * (do.abs() @ v.abs().T)
            e_delta = (do.abs() * O_).sum(-1, keepdim=True) + (D + 4) * E * (do.abs() * O.abs()).sum(-1, keepdim=True)
            e_p = e_p + out["lse_"][b, h][:, None]
            e_ds = P * (e_dp + e_delta) + (e_p + up) * dS.abs()
            out["dQ"][b, :, h] = scale * dS @ k
            out["dQ_"][b, :, h] = scale * (e_ds + len(at) * E * dS.abs()) @ k.abs()
            out["dK"][b, at, h // g] += scale * dS.T @ q
            out["dK_"][b, at, h // g] += scale * (e_ds + g * Nq * E * dS.abs()).T @ q.abs()
            out["dV"][b, at, h // g] += P.T @ do
            out["dV_"][b, at, h // g] += ((e_p + up + g * Nq * E) * P).T @ do.abs()
    for n in ("dQ", "dK", "dV"):
        out[n + "_"] += u * out[n].abs()
    for n in ("O", "dQ", "dK", "dV"):
        out[n], out[n + "_"] = (out[m].reshape(B, out[m].shape[1], -1) for m in (n, n + "_"))
    return out


CROSS = [
    # B, Nq, Nk, heads, kv, D, lens, mask
    (1, 1, 1, 1, 1, 16, None, False),
    (1, 1, 1, 1, 1, 128, None, False),
    (2, 1, 300, 8, 2, 64, None, False),                      # a step of generation, keys split over CTAs
    (3, 1, 515, 4, 4, 32, [515, 0, 129], False),
    (2, 3, 2050, 5, 1, 128, None, True),                     # 15 rows of one key head
    (2, 4, 140, 12, 3, 16, [1, 140], True),
    (2, 65, 63, 2, 2, 32, None, False),
    (2, 64, 64, 3, 3, 64, None, False),
    (2, 129, 127, 2, 1, 128, [127, 65], False),
    (3, 196, 100, 8, 8, 32, [100, 57, 0], False),
    (2, 130, 260, 6, 2, 64, None, True),
    (1, 1100, 33, 2, 2, 16, None, False),                    # few keys: queries split over CTAs
    (1, 900, 40, 4, 2, 128, [40], True),
    (1, 40, 900, 2, 2, 64, None, True),                      # few queries: keys split over CTAs
    (1, 257, 513, 3, 1, 32, [400], True),                    # a group that is no power of two
]


# Where the tcgen05 kernels run: more than 64 rows a key head, more than a block of keys (or many tiles)
CROSS_WIDE = [
    (2, 300, 400, 4, 4, 32, [400, 129], True),
    (2, 257, 640, 6, 2, 64, [0, 640], False),                # a group of three: 126 of a tile's 128 rows
    (1, 700, 700, 5, 1, 128, None, True),                    # a group of five
    (20, 100, 130, 8, 8, 64, None, False),                   # more tiles than SMs, one of a pair
    (24, 140, 90, 8, 8, 32, [(11 * i) % 91 for i in range(24)], False),     # one block of keys
    (19, 300, 300, 8, 8, 32, [300 - 16 * i for i in range(19)], True),      # CTAs with several pairs of different lengths
    (11, 260, 257, 8, 8, 128, None, False),
    (1, 3000, 200, 1, 1, 64, [150], False),                  # walks over the queries are split
    (1, 130, 3000, 1, 1, 128, [2900], True),                 # walks over the keys are split
    (1, 300, 1300, 2, 2, 32, [257], False),                  # and most parts have nothing to do
    (1, 3, 300, 100, 1, 32, None, False),                    # a group of a hundred: a token a tile
    (1, 2, 300, 128, 1, 64, None, True),
    (1, 2, 300, 130, 1, 32, None, False),                    # a group larger than a tile
]


def cross_problem(bra, case, dtype, seed=0, **kw):
    import torch
    B, Nq, Nk, heads, kv, D, lens, masked = case
    Q, dO = randn(seed + 1, B, Nq, heads * D, dtype=dtype), randn(seed + 2, B, Nq, heads * D, dtype=dtype)
    K, V = randn(seed + 3, B, Nk, kv * D, dtype=dtype), randn(seed + 4, B, Nk, kv * D, dtype=dtype)
    key_len = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    see = torch.ones(B, Nk, dtype=torch.bool, device="cuda")
    key_mask = None
    if masked:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed + 5)
        key_mask = torch.rand(B, Nk, device="cuda", generator=gen) < 0.7
        see &= key_mask
    if lens is not None:
        see &= torch.arange(Nk, device="cuda")[None] < key_len[:, None]
    p = bra.make_cross_problem(B, Nq, Nk, heads, D, kv_heads=kv, dtype=dtype, **kw)
    return p, Q, K, V, dO, key_len, key_mask, see


def check_cross(bra, p, Q, K, V, dO, key_len, key_mask, see, dtype, ws=None):
    B, Nq, Nk, heads, kv, D = p.B, p.Nq, p.Nk, p.heads, p.kv_heads, p.head_dim
    scale = p.scale if p.scale > 0 else 1 / math.sqrt(D)
    ws = bra.cross_workspace(p) if ws is None else ws
    O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask, ws=ws)
    dQ, dK, dV = bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask, ws=ws)
    ref = cross_ref(Q, K, V, dO, see, heads, kv, D, scale, dtype)
    got = {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}
    for n, v in got.items():
        within(v.reshape(ref[n].shape), ref[n], ref[n + "_"], n)
    assert (ws[:2048 * 4] == 0).all()                        # the counters are left as they were found
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CROSS, ids=str)
def test_cross(bra, case, dtype):
    check_cross(bra, *cross_problem(bra, case, dtype), dtype)


@pytest.mark.parametrize("case", CROSS_WIDE, ids=str)
def test_cross_wide(bra, case):
    check_cross(bra, *cross_problem(bra, case, "bf16"), "bf16")


@pytest.mark.parametrize("D", [32, 64, 128])
def test_cross_wide_many_launches(bra, D):
    """Long walks of many tiles, again and again, forward and backward: the same bits, no wait that gives up."""
    import torch
    p, Q, K, V, dO, _, _, _ = cross_problem(bra, (4, 1000, 1100, 20, 10, D, None, False), "bf16")
    ws = bra.cross_workspace(p)
    first = None
    for _ in range(10):
        O, lse = bra.bra_cross_attend(p, Q, K, V, ws=ws)
        got = (O, lse) + bra.bra_cross_backward(p, Q, K, V, O, lse, dO, ws=ws)
        first = got if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    assert bra.bra_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("Nq,Nk", [(1, 2), (16, 17), (17, 31), (63, 33), (64, 65), (66, 128), (128, 129), (255, 257)])
def test_cross_sizes_around_tiles(bra, Nq, Nk, D, dtype):
    check_cross(bra, *cross_problem(bra, (2, Nq, Nk, 2, 1, D, [Nk, Nk // 2], False), dtype), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_on_slices_and_with_a_scale(bra, dtype):
    """Q, K and V inside wider tensors; gradients of the same layout; what lies between stays as it was."""
    import torch
    B, Nq, Nk, heads, kv, D = 2, 70, 90, 4, 2, 32
    wide_q, wide_kv = randn(1, B, Nq, heads * D + 64, dtype=dtype), randn(2, B, Nk, 2 * kv * D, dtype=dtype)
    p = bra.make_cross_problem(B, Nq, Nk, heads, D, kv_heads=kv, dtype=dtype, scale=0.3, q_stride=wide_q.shape[-1],
                               k_stride=wide_kv.shape[-1], v_stride=wide_kv.shape[-1])
    Q, K, V = wide_q[..., :heads * D], wide_kv[..., :kv * D], wide_kv[..., kv * D:]
    dO = randn(3, B, Nq, heads * D, dtype=dtype)
    see = torch.ones(B, Nk, dtype=torch.bool, device="cuda")
    check_cross(bra, p, Q, K, V, dO, None, None, see, dtype)
    O, lse = bra.bra_cross_attend(p, Q, K, V)
    d_kv, d_q = torch.full_like(wide_kv, 7.0), torch.full_like(wide_q, 7.0)
    dQ, dK, dV = bra.bra_cross_backward(p, Q, K, V, O, lse, dO)
    bra.bra_cross_backward(p, Q, K, V, O, lse, dO, dQ=d_q[..., :heads * D], dK=d_kv[..., :kv * D], dV=d_kv[..., kv * D:])
    assert torch.equal(d_kv[..., :kv * D], dK) and torch.equal(d_kv[..., kv * D:], dV) and torch.equal(d_q[..., :heads * D], dQ)
    assert (d_q[..., heads * D:] == 7.0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(2, 1, 300, 4, 2, 64, [300, 170], True), (2, 80, 200, 4, 2, 32, [200, 0], True),
                                  (2, 200, 70, 2, 2, 128, [33, 70], True), (1, 300, 400, 2, 2, 64, [257], False),
                                  (3, 200, 300, 6, 2, 32, [300, 0, 130], True), (2, 300, 520, 2, 2, 128, [520, 300], True),
                                  (1, 2000, 140, 2, 1, 64, [129], True)], ids=str)
def test_cross_hidden_keys_reach_nothing(bra, case, dtype, bad):
    """Outputs and gradients to the same bits, whatever stands in hidden keys and values."""
    import torch
    p, Q, K, V, dO, key_len, key_mask, see = cross_problem(bra, case, dtype)
    clean = check_cross(bra, p, Q, K, V, dO, key_len, key_mask, see, dtype)
    K[~see], V[~see] = bad, bad
    O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask)
    dQ, dK, dV = bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask)
    for n, v in (("O", O), ("lse", lse), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        assert torch.equal(v, clean[n]), n
    assert (dK[~see] == 0).all() and (dV[~see] == 0).all()


def test_cross_lengths_outside_the_range_and_masks_of_bytes(bra):
    import torch
    case = (3, 40, 50, 2, 2, 32, [-5, 1000, 50], False)
    p, Q, K, V, dO, key_len, _, _ = cross_problem(bra, case, "bf16")
    see = torch.ones(3, 50, dtype=torch.bool, device="cuda")
    see[0] = False
    check_cross(bra, p, Q, K, V, dO, key_len, None, see, "bf16")
    see = torch.rand(3, 50, device="cuda") < 0.5
    check_cross(bra, p, Q, K, V, dO, None, see.to(torch.uint8) * 200, see, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_large_scores(bra, dtype):
    """Scores of several hundred, growing along the keys: the running maximum moves in every tile."""
    import torch
    B, Nq, Nk, D = 1, 100, 700, 64
    Q, K = randn(1, B, Nq, D, dtype=dtype), randn(2, B, Nk, D, dtype=dtype)
    K = (K.float() + Q[:, :1].float() * (torch.arange(Nk, device="cuda")[None, :, None] / 100)).to(K.dtype)
    V, dO = randn(3, B, Nk, D, dtype=dtype), randn(4, B, Nq, D, dtype=dtype)
    p = bra.make_cross_problem(B, Nq, Nk, 1, D, dtype=dtype, scale=1.0)
    check_cross(bra, p, Q, K, V, dO, None, None, torch.ones(B, Nk, dtype=torch.bool, device="cuda"), dtype)


def test_cross_is_the_same_every_time_and_on_other_streams(bra):
    import torch
    for case in (CROSS[2], CROSS[11], CROSS[13], CROSS_WIDE[1], CROSS_WIDE[7], CROSS_WIDE[8]):
        p, Q, K, V, dO, key_len, key_mask, _ = cross_problem(bra, case, "bf16")
        ws = bra.cross_workspace(p)
        O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask, ws=ws)
        want = (O, lse) + bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask, ws=ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            with torch.cuda.stream(side):
                O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask, ws=ws)
                got = (O, lse) + bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask, ws=ws)
            side.synchronize()
            for a, b in zip(want, got):
                assert torch.equal(a, b)


def test_cross_problems_share_a_scratch(bra):
    """Problems of different sizes, types and kernels in turn in the scratch of the one that needs most; two streams with one each."""
    import torch
    runs = [cross_problem(bra, c, t, seed=9) for c, t in ((CROSS[12], "bf16"), (CROSS_WIDE[8], "bf16"), (CROSS_WIDE[7], "bf16"), (CROSS[2], "f32"),
                                                          (CROSS[11], "bf16"), (CROSS_WIDE[5], "bf16"), (CROSS[12], "f32"))]

    def run(i, ws):
        p, Q, K, V, dO, key_len, key_mask, _ = runs[i]
        O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask, ws=ws)
        return (O, lse) + bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask, ws=ws)

    want = [run(i, bra.cross_workspace(r[0])) for i, r in enumerate(runs)]
    most = max(bra.cross_workspace_bytes(r[0]) for r in runs)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.zeros(most, device="cuda", dtype=torch.uint8) for _ in streams]
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(len(runs)):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(run(len(runs) - 1 - i if k else i, ws[k]))
    for k, st in enumerate(streams):
        assert bra.bra_device_status(ws[k], stream=st.cuda_stream) == 0
        for a, b in zip(want, got[k][::-1] if k else got[k]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_cross_gradients_by_differences(bra):
    """d(sum O o dO) along a direction of Q, K and V against central differences of the fp32 forward."""
    import torch
    p, Q, K, V, dO, key_len, key_mask, _ = cross_problem(bra, (2, 33, 45, 4, 2, 32, [45, 20], True), "f32")
    O, lse = bra.bra_cross_attend(p, Q, K, V, key_len, key_mask)
    grads = bra.bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask)
    for i, g in enumerate(grads):
        way = randn(50 + i, *g.shape, dtype="f32")
        step = 2.0 ** -8
        def value(sign):
            args = [Q, K, V]
            args[i] = args[i] + sign * step * way
            return float((bra.bra_cross_attend(p, *args, key_len, key_mask)[0].double() * dO.double()).sum())
        slope = (value(1) - value(-1)) / (2 * step)
        want = float((g.double() * way.double()).sum())
        # third-order term of the difference: step^2 / 6 of a third derivative of the order of the slope's own scale
        scale = float(g.double().norm() * way.double().norm() / math.sqrt(g.numel()))
        assert abs(slope - want) <= 0.02 * scale + 0.02 * abs(want)


# ---------------------------------------------------------------- residual norms
NORM = [
    # B, N, C, pre, post, gate, per_image, alpha
    (1, 1, 1, "layer", "none", "none", False, 1.0),
    (1, 1, 768, "rms", "none", "none", False, 1.0),
    (1, 1, 8, "rms", "rms", "channel", False, 0.5),
    (2, 3, 7, "layer", "rms", "image", True, 1.0),
    (2, 50, 64, "layer", "layer", "channel", False, 1.0),
    (3, 49, 96, "layer", "none", "image", True, 1.0),
    (5, 37, 100, "rms", "layer", "channel", True, 0.7),
    (2, 300, 256, "rms", "rms", "image", False, 1.0),
    (2, 40, 257, "layer", "layer", "channel", False, 1.0),
    (3, 33, 768, "layer", "none", "image", True, 1.0),
    (700, 1, 128, "rms", "none", "image", True, 1.0),
    (2, 9, 1024, "layer", "rms", "none", False, 1.0),
    (2, 30, 1032, "layer", "rms", "image", True, 1.0),
    (2, 11, 2050, "rms", "layer", "channel", True, 1.0),
    (1, 20, 4096, "layer", "layer", "channel", False, 1.0),
    (2, 7, 5001, "rms", "rms", "image", False, 0.7),
    (1, 5, 8192, "layer", "layer", "channel", False, 1.0),
    (4, 6, 48, "none", "rms", "channel", False, 1.0),
]


def norm_inputs(case, dtype, seed=0):
    B, N, C, pre, post, gate, per_image, alpha = case
    x, y = randn(seed + 1, B, N, C, dtype=dtype, std=1.5, mean=0.3), randn(seed + 2, B, N, C, dtype=dtype)
    f = lambda s, *shape, **kw: randn(seed + s, *shape, dtype="f32", **kw)                          # noqa: E731
    w = {"gate": None if gate == "none" else f(3, *((B, C) if gate == "image" else (C,)), std=0.5)}
    w["post_w"], w["post_b"] = (f(4, C, std=0.2, mean=1.0), f(5, C, std=0.2)) if post != "none" else (None, None)
    of = (B, C) if per_image else (C,)
    w["w"], w["b"] = (f(6, *of, std=0.2, mean=1.0), f(7, *of, std=0.2)) if pre != "none" else (None, None)
    return x, y, randn(seed + 8, B, N, C, dtype=dtype), randn(seed + 9, B, N, C, dtype=dtype) if pre != "none" else None, w


def norm_forward_ref(case, a, eps):
    import torch
    B, N, C, pre, post, gate, per_image, alpha = case
    def norm(kind, v):
        m = v.mean(-1, keepdim=True) if kind == "layer" else 0.0
        r = torch.rsqrt((v - m).square().mean(-1, keepdim=True) + eps)
        return (v - m) * r, r
    wide = lambda v: v[:, None] if v.dim() == 2 else v                                              # noqa: E731
    y, yhat, ry = a["y"], None, None
    if post != "none":
        yhat, ry = norm(post, y)
        y = yhat * a["post_w"] + a["post_b"]
    h = alpha * a["x"] + (y * wide(a["gate"]) if "gate" in a else y)
    if pre == "none":
        return h, None, (y, yhat, ry, None, None)
    hat, r = norm(pre, h)
    return h, hat * wide(a["w"]) + wide(a["b"]), (y, yhat, ry, hat, r)


def check_norm(bra, case, dtype, eps=1e-6):
    import torch
    B, N, C, pre, post, gate, per_image, alpha = case
    u = half_step(dtype)
    x, y, dh, dn, w = norm_inputs(case, dtype)
    p = bra.make_norm_problem(B, N, C, pre=pre, post=post, gate=gate, per_image=per_image, alpha=alpha, eps=eps, dtype=dtype)
    h, n = bra.bra_residual_norm(p, x, y, **w)
    out = bra.bra_residual_norm_backward(p, x, y, dh, dn, **w)
    a = {k: v.double().requires_grad_() for k, v in dict(x=x, y=y, **w).items() if v is not None}
    H, Nn, (yy, yhat, ry, hat, r) = norm_forward_ref(case, a, eps)
    wide = lambda v: v[:, None] if v.dim() == 2 else v                                              # noqa: E731
    g = wide(a["gate"]).detach() if "gate" in a else torch.ones((), dtype=torch.float64, device="cuda")
    with torch.no_grad():
        # a normalised value: its mean's sum and its own subtraction, relative to the row's magnitude; the factor
        def spread(kind, v, r):
            big = v.abs() + (v.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0)
            return 2.0 ** -18 * r * big
        e_y = 2.0 ** -22 * yy.abs() if post == "none" else a["post_w"].abs() * spread(post, a["y"], ry) + 2.0 ** -22 * yy.abs()
        e_h = g.abs() * e_y + 2.0 ** -22 * ((alpha * a["x"]).abs() + (g * yy).abs())
        within(h, H, u * H.abs() + e_h, "h")
        if pre != "none":
            e_hat = spread(pre, H, r) + r * (e_h + e_h.mean(-1, keepdim=True)) + hat.abs() * r * (e_h * hat.abs()).mean(-1, keepdim=True)
            W = wide(a["w"])
            within(n, Nn, u * Nn.abs() + W.abs() * e_hat + 2.0 ** -22 * ((hat * W).abs() + wide(a["b"]).abs()), "n")
    grads_of = (H, Nn) if pre != "none" else (H,)
    grads = torch.autograd.grad(grads_of, list(a.values()), (dh.double(), dn.double()) if pre != "none" else (dh.double(),))
    ref = dict(zip(a, grads))
    with torch.no_grad():
        # magnitudes of the terms that make dH and dy; their relative error is that of normalised values and of sums over a row
        rel = 2.0 ** -15
        T = dh.double().abs()
        if pre != "none":
            G = (dn.double() * W).abs()
            T = T + r * (G + (hat.abs() + e_hat / rel) * (G * hat.abs()).mean(-1, keepdim=True) + G.mean(-1, keepdim=True))
            T = T + r * (e_hat / rel) * G.mean(-1, keepdim=True)
        within(out["dx"], ref["x"], u * ref["x"].abs() + rel * abs(alpha) * T, "dx")
        Ty = g.abs() * T
        if post != "none":
            Gy = Ty * a["post_w"].abs()
            Ty2 = ry * (Gy + (yhat.abs() + spread(post, a["y"], ry) / rel) * (Gy * (yhat.abs() + 2.0 ** -18)).mean(-1, keepdim=True) + Gy.mean(-1, keepdim=True))
        else:
            Ty2 = Ty
        within(out["dy"], ref["y"], u * ref["y"].abs() + rel * Ty2, "dy")
        over = (0, 1)
        # sums over tokens: at most rows 2^-24 of their terms, and the terms' own error
        own = rel + B * N * E
        if "gate" in a:
            dims = (1,) if gate == "image" else over
            within(out["dgate"], ref["gate"], own * (T * (yy.abs() + e_y / rel)).sum(dims), "dgate")
        if post != "none":
            within(out["d_post_w"], ref["post_w"], own * (Ty * (yhat.abs() + spread(post, a["y"], ry) / rel)).sum(over), "d_post_w")
            within(out["d_post_b"], ref["post_b"], own * Ty.sum(over), "d_post_b")
        if pre != "none":
            dims = (1,) if per_image else over
            within(out["dw"], ref["w"], own * (dn.double().abs() * (hat.abs() + e_hat / rel)).sum(dims), "dw")
            within(out["db"], ref["b"], own * dn.double().abs().sum(dims), "db")
    return h, n, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", NORM, ids=str)
def test_norm(bra, case, dtype):
    check_norm(bra, case, dtype)


# Rows of a CTA of their own, in each size that such CTAs have; many rows a CTA, images that begin inside its run
NORM_LONG = [
    (3, 411, 520, "layer", "rms", "image", True, 1.0),
    (2, 900, 1304, "layer", "layer", "image", True, 0.7),
    (3, 401, 1777, "rms", "rms", "channel", False, 1.0),
    (2, 500, 2504, "layer", "none", "channel", False, 1.0),
    (2, 301, 3333, "layer", "rms", "image", True, 1.0),
    (1, 700, 4500, "rms", "layer", "channel", False, 1.0),
    (2, 333, 5000, "layer", "none", "image", False, 1.0),
    (1, 500, 7001, "rms", "rms", "channel", False, 1.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", NORM_LONG, ids=str)
def test_norm_long_rows(bra, case, dtype):
    check_norm(bra, case, dtype)


# Without a post-norm, channels that do not come by eight: in each size of kernel, the first and last widths of a number of warps
ODD = [257, 513, 1023, 1025, 1027, 1111, 1119, 1279, 1281, 1343, 1535, 1537, 1567, 1791, 1793, 2049, 3333, 4095, 4097, 5001, 7001, 8191]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", ODD)
def test_norm_odd_widths(bra, C, dtype):
    check_norm(bra, (2, 37, C, "layer", "none", "channel", False, 1.0), dtype)
    check_norm(bra, (3, 5, C, "rms", "none", "image", True, 0.7), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "channel", "image"])
@pytest.mark.parametrize("C", ODD)
def test_norm_odd_widths_keep_to_their_rows(bra, C, gate, dtype):
    """What lies behind inputs and weights (NaN) reaches nothing, what lies behind h and n stays, with rows of many CTAs and of one."""
    import torch
    for N in (3, 700):
        behind = lambda t: torch.cat([t.flatten(), torch.full((256,), math.nan, device="cuda", dtype=t.dtype)])[:t.numel()].view(t.shape)      # noqa: E731
        B = 2 if N == 3 else 1
        x, y, _, _, w = norm_inputs((B, N, C, "layer", "none", gate, gate == "image", 1.0), dtype)
        x, y, w = behind(x), behind(y), {k: None if v is None else behind(v) for k, v in w.items()}
        p = bra.make_norm_problem(B, N, C, pre="layer", gate=gate, per_image=gate == "image", dtype=dtype)
        want = bra.bra_residual_norm(p, x, y, **w)
        guard = [torch.full((x.numel() + 256,), 3.0, device="cuda", dtype=x.dtype) for _ in range(2)]
        h, n = (g[:x.numel()].view(x.shape) for g in guard)
        bra.bra_residual_norm(p, x, y, h=h, n=n, **w)
        assert torch.equal(h, want[0]) and torch.equal(n, want[1])
        assert all(bool((g[x.numel():] == 3.0).all()) for g in guard)
        X, Y = x.double(), y.double()
        g = 1.0 if gate == "none" else w["gate"].double()[:, None] if gate == "image" else w["gate"].double()
        H = X + g * Y
        # an fma of two roundings and the output's own
        within(h, H, half_step(dtype) * H.abs() + 2.0 ** -22 * (X.abs() + (g * Y).abs()), "h")
        assert bool(torch.isfinite(n).all())


@pytest.mark.parametrize("C", [64, 768, 1304, 1777, 4096, 5001])
def test_norm_gradients_of_some_weights(bra, C):
    """A sum that is not wanted leaves the others' bits as they are; weights that are not given are ones and zeros."""
    import torch
    x, y, dh, dn, w = norm_inputs((2, 150, C, "layer", "rms", "channel", False, 1.0), "bf16")
    p = bra.make_norm_problem(2, 150, C, pre="layer", post="rms", gate="channel")
    w["w"], w["post_w"] = torch.ones_like(w["w"]), torch.ones_like(w["post_w"])
    full = bra.bra_residual_norm_backward(p, x, y, dh, dn, **w)
    some = {k: w[k] if k in ("gate", "b") else None for k in w}
    some["post_b"] = w["post_b"]
    part = bra.bra_residual_norm_backward(p, x, y, dh, dn, **some)
    assert set(part) == {"dx", "dy", "dgate", "db", "d_post_b"}
    assert all(torch.equal(part[k], full[k]) for k in part)


def test_norm_without_a_block_or_weights(bra):
    """The first norm of a network: h = alpha x, no y; missing weights are ones and zeros; in place into x."""
    import torch
    B, N, C = 2, 21, 72
    x = randn(1, B, N, C)
    p = bra.make_norm_problem(B, N, C, pre="rms", alpha=2.0)
    h, n = bra.bra_residual_norm(p, x)
    H = 2.0 * x.double()
    within(h, H, 2.0 ** -8 * H.abs(), "h")
    ref = H * torch.rsqrt(H.square().mean(-1, keepdim=True) + 1e-6)
    within(n, ref, (2.0 ** -8 + 2.0 ** -18) * ref.abs(), "n")
    assert bra.bra_residual_norm(p, x, want_h=False)[0] is None
    dn = randn(2, B, N, C)
    out = bra.bra_residual_norm_backward(p, x, None, None, dn)
    assert set(out) == {"dx"}
    a = x.double().requires_grad_()
    H = 2.0 * a
    (want,) = torch.autograd.grad(H * torch.rsqrt(H.square().mean(-1, keepdim=True) + 1e-6), a, dn.double())
    r = torch.rsqrt((2 * x.double()).square().mean(-1, keepdim=True) + 1e-6)
    within(out["dx"], want, 2.0 ** -8 * want.abs() + 2.0 ** -15 * 2 * r * (dn.double().abs() + (x.double().abs() * r * 2) * (dn.double() * x.double() * 2 * r).abs().mean(-1, keepdim=True)), "dx")
    y = randn(3, B, N, C)
    p = bra.make_norm_problem(B, N, C, pre="layer")
    want = bra.bra_residual_norm(p, x, y)
    again = x.clone()
    got = bra.bra_residual_norm(p, again, y, h=again)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0] is again


def test_norm_large_means_and_constant_rows(bra):
    """The variance is a sum of squared distances from the mean: a mean of a thousand times the spread costs it little; a
    constant row has zero variance and gives the bias."""
    import torch
    B, N, C = 1, 9, 640
    x = randn(1, B, N, C, dtype="f32", mean=1000.0)
    x[0, 4] = 7.0
    b = randn(2, C, dtype="f32")
    p = bra.make_norm_problem(B, N, C, pre="layer", dtype="f32")
    _, n = bra.bra_residual_norm(p, x, b=b)
    X = x.double()
    m = X.mean(-1, keepdim=True)
    r = torch.rsqrt((X - m).square().mean(-1, keepdim=True) + 1e-6)
    # the mean of 640 numbers near 1000, fp32: a chain of 8, 5 exchanges and 5 more, each 2^-24 of 1000, and a division
    bound = r * 1000 * 20 * E * (1 + ((X - m) * r).abs()) + 2.0 ** -20 * (((X - m) * r).abs() + b.double().abs())
    within(n, (X - m) * r + b.double(), bound, "n")
    assert torch.equal(n[0, 4], b)


def test_norm_nan_stays_in_its_token(bra):
    import torch
    B, N, C = 2, 30, 64
    x, y = randn(1, B, N, C), randn(2, B, N, C)
    p = bra.make_norm_problem(B, N, C, pre="layer", post="rms")
    clean = bra.bra_residual_norm(p, x, y)
    x[1, 7, 3], y[0, 29, 5] = math.nan, math.inf
    got = bra.bra_residual_norm(p, x, y)
    touched = torch.zeros(B, N, dtype=torch.bool, device="cuda")
    touched[1, 7] = touched[0, 29] = True
    for c, g in zip(clean, got):
        assert torch.equal(c[~touched], g[~touched])
    assert torch.isnan(got[1][1, 7]).all()


def test_norm_is_the_same_every_time(bra):
    import torch
    for case in (NORM[4], NORM[9], NORM[13]):
        x, y, dh, dn, w = norm_inputs(case, "bf16")
        B, N, C, pre, post, gate, per_image, alpha = case
        p = bra.make_norm_problem(B, N, C, pre=pre, post=post, gate=gate, per_image=per_image, alpha=alpha)
        ws = bra.norm_workspace(p)
        first = bra.bra_residual_norm_backward(p, x, y, dh, dn, **w, ws=ws)
        ws.fill_(255)                                        # the scratch needs no initial value
        again = bra.bra_residual_norm_backward(p, x, y, dh, dn, **w, ws=ws)
        assert set(first) == set(again) and all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [24, 64, 250, 765, 1024, 5001, 8192])
@pytest.mark.parametrize("onto", ["x", "y"])
def test_norm_over_its_input(bra, C, dtype, onto):
    """h in the place of x or y: the same bits, rows read ahead or not, and what lies behind the last row stays."""
    import torch
    N = 700
    full = randn(5, N * C + 64, dtype=dtype), randn(6, N * C + 64, dtype=dtype)
    gate, w = randn(7, C, dtype="f32"), randn(8, C, dtype="f32")
    p = bra.make_norm_problem(1, N, C, pre="layer", post="rms", gate="channel", dtype=dtype)
    x, y = (t[:N * C].view(1, N, C) for t in full)
    h, n = bra.bra_residual_norm(p, x, y, gate=gate, w=w)
    tail = [t[N * C:].clone() for t in full]
    h2, n2 = bra.bra_residual_norm(p, x, y, gate=gate, w=w, h=x if onto == "x" else y)
    assert torch.equal(h, h2) and torch.equal(n, n2)
    assert all(torch.equal(t[N * C:], u) for t, u in zip(full, tail))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("D", [6, 32])
def test_rope_frequencies_that_are_no_numbers(bra, D, layout, dtype):
    """A pair whose frequency is NaN or infinite has no angle: it comes out NaN (at coordinate 0 too), the others as they were."""
    import torch
    x = randn(40, 2, 5, 3 * D, dtype=dtype)
    p = bra.make_rope_problem(2, 5, 3, D, kv_heads=0, layout=layout, dtype=dtype)
    good = bra.rope_frequencies(D)
    want = bra.bra_rope(p, x, None, good)[0].view(2, 5, 3, D)
    for value in (math.nan, math.inf, -math.inf):
        for pair in (0, D // 2 - 1):
            freq = good.clone()
            freq[pair] = value
            mine = torch.zeros(D, dtype=torch.bool, device="cuda")
            mine[[2 * pair, 2 * pair + 1] if layout == "interleaved" else [pair, pair + D // 2]] = True
            for inverse in (False, True):
                got = bra.bra_rope(p, x, None, freq, inverse=inverse)[0].view(2, 5, 3, D)
                assert bool(torch.isnan(got[..., mine]).all())
                if not inverse:
                    assert torch.equal(got[..., ~mine], want[..., ~mine])


# ---------------------------------------------------------------- another stream
def test_calls_on_a_stream_while_the_current_one_is_busy(bra):
    """Outputs and scratch that the calls make themselves, on a stream given as an object and as a handle, behind nothing of the current
    stream: the results are there while that one still sleeps, with sums that are split (counters in scratch) and the routed calls too."""
    import torch
    # one token on many keys (parts joined by a counter), tiles on tcgen05 whose walks are split
    crosses = [cross_problem(bra, (2, 1, 3000, 4, 2, 64, None, False), d) for d in ("bf16", "f32")] + \
        [cross_problem(bra, (1, 100, 1500, 4, 2, 64, None, False), "bf16")]
    r, freq = bra.make_rope_problem(2, 50, 4, 32), bra.rope_frequencies(32)
    nc = (2, 60, 96, "layer", "rms", "image", False, 1.0)
    x, y, dh, dn, w = norm_inputs(nc, "bf16")
    n = bra.make_norm_problem(2, 60, 96, pre="layer", post="rms", gate="image")
    qr = randn(21, 2, 50, 128)
    m = [randn(30 + i, 2, 16, 16, 64) for i in range(4)]
    lce = randn(35, 64, 5, 5, dtype="f32")
    p = bra.make_problem(2, 16, 16, 64, heads=2, S=4, topk=2)

    def all_of(**k):
        out = []
        for c, Q, K, V, dO, *_ in crosses:
            O, lse = bra.bra_cross_attend(c, Q, K, V, **k)
            out += [O, lse, *bra.bra_cross_backward(c, Q, K, V, O, lse, dO, **k)]
        out += bra.bra_rope(r, qr, qr, freq, **k)
        out += bra.bra_residual_norm(n, x, y, **w, **k)
        out += [v for _, v in sorted(bra.bra_residual_norm_backward(n, x, y, dh, dn, **w, **k).items())]
        O, index, lse = bra.bra_forward(p, *m[:3], lce, **k)
        out += [O, index, lse, *[t for t in bra.bra_backward(p, *m[:3], index, lce, lse, m[3], **k) if t is not None]]
        return out

    want = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for given in (side, side.cuda_stream):
        all_of(stream=given)                                 # what a first call loads and sets is done
        torch.cuda.synchronize()
        for _ in range(3):
            slept = torch.cuda.Event()
            torch.cuda._sleep(600_000_000)                   # 0.3 s
            slept.record()
            got = all_of(stream=given)
            side.synchronize()
            early = not slept.query()
            with torch.cuda.stream(side):
                same = all(torch.equal(a, b) for a, b in zip(want, got))
            assert same and early and len(want) == len(got)
            torch.cuda.synchronize()


# ---------------------------------------------------------------- together
def block(bra, t, st):
    """Two branches of a block around projected tensors: positions, routed attention, norm, cross attention, norm; and back."""
    q, k = bra.bra_rope(st["rope"], t["q"], t["k"], st["freq"])
    o1, index, lse1 = bra.bra_forward(st["bra"], q, k, t["v"], t["lce"], ws=st["ws_bra"])
    h1, n1 = bra.bra_residual_norm(st["norm"], t["x"], o1, gate=t["g1"], w=t["w1"], b=t["b1"])
    o2, lse2 = bra.bra_cross_attend(st["cross"], n1, t["ek"], t["ev"], t["len"], ws=st["ws_cross"])
    h2, n2 = bra.bra_residual_norm(st["norm"], h1, o2, gate=t["g2"], w=t["w2"], b=t["b2"])
    b2 = bra.bra_residual_norm_backward(st["norm"], h1, o2, t["dh"], t["dn"], gate=t["g2"], w=t["w2"], b=t["b2"], ws=st["ws_norm"])
    dn1, dek, dev = bra.bra_cross_backward(st["cross"], n1, t["ek"], t["ev"], o2, lse2, b2["dy"], t["len"], ws=st["ws_cross"])
    b1 = bra.bra_residual_norm_backward(st["norm"], t["x"], o1, b2["dx"], dn1, gate=t["g1"], w=t["w1"], b=t["b1"], ws=st["ws_norm"])
    dq, dk, dv, dlce, _ = bra.bra_backward(st["bra"], q, k, t["v"], index, t["lce"], lse1, b1["dy"], ws=st["ws_bra"])
    dq, dk = bra.bra_rope(st["rope"], dq, dk, st["freq"], inverse=True)
    return dict(h2=h2, n2=n2, dx=b1["dx"], dq=dq, dk=dk, dv=dv, dek=dek, dev=dev, dlce=dlce, dg1=b1["dgate"], dw2=b2["dw"], dg2=b2["dgate"]), index


def block_setup(bra, dtype, seed=0):
    import torch
    B, H, W, heads, D, S, topk, Nk = 2, 16, 16, 2, 32, 4, 4, 45
    C, N = heads * D, H * W
    st = {"rope": bra.make_rope_problem(B, N, heads, D, axes=2, width=W, dtype=dtype), "freq": bra.rope_frequencies(D, axes=2),
          "bra": bra.make_problem(B, H, W, C, heads, S, topk, dtype), "norm": bra.make_norm_problem(B, N, C, gate="channel", dtype=dtype),
          "cross": bra.make_cross_problem(B, N, Nk, heads, D, dtype=dtype)}
    st |= {"ws_bra": bra.workspace(st["bra"]), "ws_cross": bra.cross_workspace(st["cross"]), "ws_norm": bra.norm_workspace(st["norm"])}
    t = {n: randn(seed + i, B, H, W, C, dtype=dtype) for i, n in enumerate(("x", "q", "k", "v", "dh", "dn"))}
    t |= {n: randn(seed + 10 + i, B, Nk, C, dtype=dtype) for i, n in enumerate(("ek", "ev"))}
    t |= {n: randn(seed + 20 + i, C, dtype="f32", std=0.1, mean=0.0 if n[0] == "b" else 1.0) for i, n in enumerate(("g1", "w1", "b1", "g2", "w2", "b2"))}
    t["lce"] = randn(seed + 30, C, 5, 5, dtype="f32", std=0.02)
    t["len"] = torch.tensor([Nk, 30], device="cuda", dtype=torch.int32)
    return st, t


def test_block_together_against_autograd(bra):
    """The whole chain in fp32 against automatic differentiation of its definition in 64 bits (on the library's routing index)."""
    import torch
    st, t = block_setup(bra, "f32")
    got, index = block(bra, t, st)
    B, H, W, C = t["x"].shape
    heads, D, S, N = 2, 32, 4, H * W
    names = ("x", "q", "k", "v", "ek", "ev", "lce", "g1", "w2", "g2")
    a = {n: t[n].double().requires_grad_(n in names) for n in t if n not in ("len",)}

    n_ = torch.arange(N, device="cuda")
    freq = [10000.0 ** (-i / 8) for i in range(8)]
    def turn(x):
        y = x.reshape(B, N, heads, 2, 8, 2)
        place = torch.stack((n_ // W, n_ % W), -1).double()
        angle = place[:, :, None] * torch.tensor(freq, device="cuda", dtype=torch.float64)
        c, s = angle.cos()[None, :, None], angle.sin()[None, :, None]
        return torch.stack((y[..., 0] * c - y[..., 1] * s, y[..., 0] * s + y[..., 1] * c), -1).reshape(B, N, heads, D)
    q, k, v = turn(a["q"]), turn(a["k"]), a["v"].reshape(B, N, heads, D)
    region = ((n_ // W) // (H // S)) * S + (n_ % W) // (W // S)
    routed = torch.zeros(B, heads, S * S, S * S, dtype=torch.bool, device="cuda").scatter_(3, index.long(), True)
    see = routed[:, :, region][:, :, :, region]
    s = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(D)
    P = torch.softmax(s.masked_fill(~see, -math.inf), -1)
    o1 = torch.einsum("bhij,bjhd->bihd", P, v).reshape(B, H, W, C)
    vm = a["v"].permute(0, 3, 1, 2)
    o1 = o1 + torch.nn.functional.conv2d(vm, a["lce"][:, None], padding=2, groups=C).permute(0, 2, 3, 1)
    def norm(h, w, b):
        m = h.mean(-1, keepdim=True)
        return (h - m) * torch.rsqrt((h - m).square().mean(-1, keepdim=True) + 1e-6) * w + b
    h1 = a["x"] + a["g1"] * o1
    n1 = norm(h1, a["w1"], a["b1"])
    s2 = torch.einsum("bihd,bjhd->bhij", n1.reshape(B, N, heads, D), a["ek"].reshape(B, -1, heads, D)) / math.sqrt(D)
    hidden = torch.arange(s2.shape[-1], device="cuda")[None] >= t["len"][:, None]
    o2 = torch.einsum("bhij,bjhd->bihd", torch.softmax(s2.masked_fill(hidden[:, None, None], -math.inf), -1), a["ev"].reshape(B, -1, heads, D))
    h2 = h1 + a["g2"] * o2.reshape(B, H, W, C)
    n2 = norm(h2, a["w2"], a["b2"])
    ref = dict(zip(["d" + n for n in names], torch.autograd.grad((h2, n2), [a[n] for n in names], (a["dh"], a["dn"]))))
    ref |= {"h2": h2.detach(), "n2": n2.detach()}
    for n, v in got.items():
        r = ref[n].reshape(v.shape)
        # a chain of about ten fp32 steps, each off by some 2^-20 of its operands (sums of up to 512 terms)
        assert float((v.double() - r).abs().max()) <= 2.0 ** -14 * float(r.abs().max()), n


def test_block_captured_and_replayed(bra):
    """The chain in a CUDA graph: replays on new inputs give what the calls give, also with a second graph of the same scratch."""
    import torch
    st, t = block_setup(bra, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(bra, t, st)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, index = block(bra, t, st)
        graphs.append((g, out))
    for seed in (100, 200):
        new = block_setup(bra, "bf16", seed)[1]
        for n in t:
            t[n].copy_(new[n])
        want, _ = block(bra, t, st)
        for g, out in graphs:
            for v in out.values():
                v.fill_(3.0)
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for n in want:
                assert torch.equal(out[n], want[n]), n


def test_calls_refuse_wrong_tensors(bra):
    """Element type, size, order in memory and device are checked before anything is launched."""
    import torch
    p = bra.make_cross_problem(1, 4, 6, 2, 32)
    Q, K, V = randn(1, 1, 4, 64), randn(2, 1, 6, 64), randn(3, 1, 6, 64)
    bra.bra_cross_attend(p, Q, K, V)
    for bad in (Q.float(), Q[:, :3], randn(1, 1, 64, 4).transpose(1, 2), None):
        with pytest.raises(bra.binding.BraError):
            bra.bra_cross_attend(p, bad, K, V)
    with pytest.raises(ValueError):
        bra.bra_cross_attend(p, Q.cpu(), K, V)
    with pytest.raises(bra.binding.BraError):
        bra.bra_cross_attend(p, Q, K, V, key_len=torch.ones(1, device="cuda", dtype=torch.int64))
    with pytest.raises(bra.binding.BraError):
        bra.bra_cross_attend(p, Q, K, V, key_mask=torch.ones(1, 5, device="cuda", dtype=torch.bool))
    with pytest.raises(bra.binding.BraError):
        bra.bra_cross_attend(p, Q, randn(2, 1, 6, 128)[..., :64], V)             # a slice, but the problem says dense
    with pytest.raises(bra.binding.BraError):
        bra.bra_cross_attend(p, Q, K, V, ws=torch.zeros(256, device="cuda", dtype=torch.uint8))
    r = bra.make_rope_problem(1, 4, 2, 32)
    freq = bra.rope_frequencies(32)
    with pytest.raises(bra.binding.BraError):
        bra.bra_rope(r, Q, Q, freq.float())
    with pytest.raises(bra.binding.BraError):
        bra.bra_rope(r, Q, Q, freq, positions=torch.zeros(1, 4, device="cuda", dtype=torch.int64))
    with pytest.raises(bra.binding.BraError):
        bra.bra_rope(r, Q, None, freq)
    n = bra.make_norm_problem(1, 4, 64, gate="image")
    with pytest.raises(bra.binding.BraError):
        bra.bra_residual_norm(n, Q, Q)                                            # no gate
    with pytest.raises(bra.binding.BraError):
        bra.bra_residual_norm(n, Q, Q, gate=torch.ones(2, 64, device="cuda"))
