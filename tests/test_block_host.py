"""Rotary positions, cross attention and residual norms at the C boundary without a GPU: refusals, frequencies, scratch sizes."""
import ctypes
import math

import pytest

A = 0x10000  # a fake, aligned, never dereferenced device address
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 4, 5, 6, 7


@pytest.fixture(scope="module")
def bra():
    import paper_2303_08810_b200 as pkg
    from paper_2303_08810_b200 import build
    build.build_library()
    pkg.load_library()
    return pkg


def with_fields(p, kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


# ---------------------------------------------------------------- rotary positions
def rope(bra, kw=None, Q=A, K=A, positions=None, freq=A, Qo=A, Ko=A):
    p = with_fields(bra.make_rope_problem(2, 5, 4, 32, kv_heads=2), kw or {})
    return bra.load_library().bra_rope(ctypes.byref(p), Q, K, positions, freq, 0, Qo, Ko, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(N=-1), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=-1), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(rot_dim=0), SHAPE), (dict(rot_dim=33), SHAPE), (dict(rot_dim=34), SHAPE), (dict(rot_dim=31), SHAPE),
    (dict(axes=0), SHAPE), (dict(axes=3), SHAPE), (dict(axes=2), SHAPE), (dict(axes=2, rot_dim=30, width=5), SHAPE),
    (dict(first=-1), SHAPE), (dict(first=2 ** 31 - 3), SHAPE), (dict(q_stride=127), SHAPE), (dict(k_stride=63), SHAPE),
    (dict(B=2 ** 30, N=2 ** 30), SHAPE), (dict(dtype=5), DTYPE), (dict(layout=2), UNSUPPORTED),
    (dict(head_dim=2 ** 24, rot_dim=32), SHAPE),
])
def test_rope_refuses_bad_problems(bra, kw, code):
    assert rope(bra, kw) == code
    assert bra.last_launch_count() == 0


def test_rope_refuses_bad_pointers(bra):
    assert rope(bra, Q=None) == NULL and rope(bra, K=None) == NULL and rope(bra, Ko=None) == NULL and rope(bra, freq=None) == NULL
    assert rope(bra, dict(kv_heads=0)) == NULL                      # K given, but no heads of it
    assert rope(bra, Q=A + 8) == ALIGN and rope(bra, Ko=A + 2) == ALIGN and rope(bra, freq=A + 4) == ALIGN
    assert rope(bra, positions=A + 2) == ALIGN
    assert bra.load_library().bra_rope(None, A, A, None, A, 0, A, A, None) == NULL


def frequencies(bra, n, axes=1, base=10000.0, scaling=0, factor=1.0, length=0.0, low=1.0, high=32.0):
    out = (ctypes.c_double * max(1, n // axes // 2))()
    code = bra.load_library().bra_rope_frequencies(n, axes, base, scaling, factor, length, low, high, out)
    return code, list(out)


def test_rope_frequencies(bra):
    code, plain = frequencies(bra, 64)
    assert code == 0
    assert plain == pytest.approx([10000 ** (-i / 32) for i in range(32)], rel=1e-14)
    assert frequencies(bra, 64, axes=2)[1] == pytest.approx(plain[::2], rel=1e-14)
    assert frequencies(bra, 64, scaling=1, factor=4.0)[1] == pytest.approx([f / 4 for f in plain], rel=1e-14)
    changed = frequencies(bra, 64, scaling=2, factor=8.0)[1]
    assert changed[0] == 1.0 and changed[-1] == pytest.approx(plain[-1] / 8, rel=1e-12)
    parts = frequencies(bra, 64, scaling=3, factor=8.0, length=4096.0)[1]
    for f, g in zip(plain, parts):
        turns = 4096 * f / (2 * math.pi)
        if turns >= 32:
            assert g == f
        elif turns <= 1:
            assert g == pytest.approx(f / 8, rel=1e-14)
        else:
            assert f / 8 < g < f


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), SHAPE), (dict(n=7), SHAPE), (dict(n=6, axes=2), SHAPE), (dict(n=8, axes=3), SHAPE), (dict(n=8, base=0.0), SHAPE),
    (dict(n=8, base=math.nan), SHAPE), (dict(n=8, scaling=4), UNSUPPORTED), (dict(n=8, scaling=1, factor=0.0), SHAPE),
    (dict(n=2, scaling=2, factor=2.0), SHAPE), (dict(n=8, scaling=3, factor=2.0), SHAPE),
    (dict(n=8, scaling=3, factor=2.0, length=10.0, low=2.0, high=2.0), SHAPE),
])
def test_rope_frequencies_refuses(bra, kw, code):
    assert frequencies(bra, **kw)[0] == code


# ---------------------------------------------------------------- cross attention
def cross(bra, kw=None, ws=A, ws_bytes=1 << 40, mask=None, length=None, back=False, **at):
    p = with_fields(bra.make_cross_problem(2, 40, 24, 4, 32, kv_heads=2), kw or {})
    get = lambda n: at.get(n, A)                                                                # noqa: E731
    lib = bra.load_library()
    if back:
        return lib.bra_cross_backward(ctypes.byref(p), get("Q"), get("K"), get("V"), length, mask, get("O"), get("lse"), get("dO"),
                                      get("dQ"), get("dK"), get("dV"), ws, ws_bytes, None)
    return lib.bra_cross_attend(ctypes.byref(p), get("Q"), get("K"), get("V"), length, mask, get("O"), get("lse"), ws, ws_bytes, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(Nq=0), SHAPE), (dict(Nk=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(kv_heads=3), SHAPE), (dict(kv_heads=8), SHAPE), (dict(head_dim=-32), SHAPE), (dict(dtype=2), DTYPE),
    (dict(head_dim=24), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(q_stride=120), SHAPE), (dict(k_stride=60), SHAPE),
    (dict(v_stride=8), SHAPE), (dict(q_stride=130), ALIGN), (dict(k_stride=68), ALIGN), (dict(v_stride=65), ALIGN),
    (dict(Nq=2 ** 30, heads=4), SHAPE), (dict(B=2 ** 20, Nk=2 ** 25), SHAPE), (dict(k_stride=2 ** 40), SHAPE),
])
def test_cross_refuses_bad_problems(bra, kw, code, back):
    assert cross(bra, kw, back=back) == code
    assert bra.last_launch_count() == 0
    p = with_fields(bra.make_cross_problem(2, 40, 24, 4, 32, kv_heads=2), kw)
    assert bra.cross_workspace_bytes(p) == 0


def test_cross_refuses_bad_pointers(bra):
    for n in ("Q", "K", "V", "O"):
        assert cross(bra, **{n: None}) == NULL and cross(bra, **{n: A + 8}) == ALIGN
    for n in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV"):
        assert cross(bra, back=True, **{n: None}) == NULL and cross(bra, back=True, **{n: A + 4}) == ALIGN
    assert cross(bra, back=True, lse=None) == NULL and cross(bra, lse=A + 2) == ALIGN and cross(bra, length=A + 1) == ALIGN
    for back in (False, True):
        assert cross(bra, ws=None, back=back) == NULL and cross(bra, ws=A + 128, back=back) == ALIGN
        need = bra.cross_workspace_bytes(bra.make_cross_problem(2, 40, 24, 4, 32, kv_heads=2))
        assert cross(bra, ws_bytes=need - 1, back=back) == WORKSPACE
        assert cross(bra, dict(Nk=2 ** 19 + 1), mask=A, back=back) == UNSUPPORTED      # bits of a mask are held in shared memory


def test_cross_scratch_covers_split_sums(bra):
    """Where output tiles are few the sums are split, and the scratch holds every part."""
    few = bra.make_cross_problem(1, 1, 8192, 8, 64, kv_heads=1)
    many = bra.make_cross_problem(64, 512, 8192, 8, 64, kv_heads=1)
    assert bra.cross_workspace_bytes(few) > 8192 * 4                # more than counters and statistics
    stats = 64 * 4096 * 8
    assert stats < bra.cross_workspace_bytes(many) <= stats + 16384 + 4096


# ---------------------------------------------------------------- residual norms
def norm(bra, kw=None, back=False, ws=A, ws_bytes=1 << 40, **at):
    p = with_fields(bra.make_norm_problem(2, 5, 64, pre="layer", post="rms", gate="channel"), kw or {})
    B = A + (1 << 20)
    base = dict(x=A, y=A, gate=A, post_w=A, post_b=None, w=A, b=A, h=B, n=2 * B, dh=A, dn=A, dx=3 * B, dy=4 * B, dg=B, dpw=B, dpb=None, dw=B, db=B)
    base.update(at)
    g = base.get
    lib = bra.load_library()
    if back:
        return lib.bra_residual_norm_backward(ctypes.byref(p), g("x"), g("y"), g("gate"), g("post_w"), g("post_b"), g("w"), g("dh"), g("dn"),
                                              g("dx"), g("dy"), g("dg"), g("dpw"), g("dpb"), g("dw"), g("db"), ws, ws_bytes, None)
    return lib.bra_residual_norm(ctypes.byref(p), g("x"), g("y"), g("gate"), g("post_w"), g("post_b"), g("w"), g("b"), g("h"), g("n"), None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(N=0), SHAPE), (dict(C=0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=math.nan), SHAPE),
    (dict(B=2 ** 20, N=2 ** 20), SHAPE), (dict(dtype=9), DTYPE), (dict(pre=3), UNSUPPORTED), (dict(post=-1), UNSUPPORTED),
    (dict(B=1, N=2 ** 30 + 1, C=8), SHAPE), (dict(B=2, N=2 ** 30 - 60, C=8), SHAPE),      # rows asked for ahead pass 32 bits
    (dict(gate=3), UNSUPPORTED), (dict(C=8200), UNSUPPORTED),
])
def test_norm_refuses_bad_problems(bra, kw, code, back):
    assert norm(bra, kw, back=back) == code
    assert bra.last_launch_count() == 0
    p = with_fields(bra.make_norm_problem(2, 5, 64), kw)
    assert bra.norm_workspace_bytes(p) == 0


def test_norm_refuses_bad_pointers(bra):
    assert norm(bra, x=None) == NULL and norm(bra, n=None) == NULL and norm(bra, gate=None) == NULL
    assert norm(bra, y=None) == NULL                                 # a gate and a norm of nothing
    assert norm(bra, dict(pre=0)) == NULL                            # n is given, but there is no norm
    assert norm(bra, dict(pre=0), n=None, h=None) == NULL            # nothing to write
    assert norm(bra, dict(gate=0)) == NULL
    assert norm(bra, n=A) == UNSUPPORTED                             # n over x
    for n in ("x", "y", "gate", "post_w", "post_b", "w", "b", "h", "n"):
        assert norm(bra, **{n: A + 4}) == ALIGN
    assert norm(bra, back=True, dx=None) == NULL and norm(bra, back=True, dn=None) == NULL and norm(bra, back=True, dy=None) == NULL
    assert norm(bra, dict(pre=0), back=True, dn=None, dh=None, dw=None, db=None) == NULL
    assert norm(bra, dict(post=0), back=True) == UNSUPPORTED         # a gradient of weights that do not exist
    assert norm(bra, dict(gate=0), back=True, gate=None) == UNSUPPORTED
    assert norm(bra, dict(pre=0), back=True, dn=None) == UNSUPPORTED
    B = A + (1 << 20)
    assert norm(bra, back=True, dy=3 * B) == UNSUPPORTED and norm(bra, back=True, dx=A) == UNSUPPORTED
    assert norm(bra, back=True, ws=None) == NULL and norm(bra, back=True, ws=A + 16) == ALIGN
    need = bra.norm_workspace_bytes(bra.make_norm_problem(2, 5, 64, pre="layer", post="rms", gate="channel"))
    assert norm(bra, back=True, ws_bytes=need - 1) == WORKSPACE


def test_norm_refuses_outputs_that_overlap(bra):
    """Any bytes in common, not only the same address: rows are read ahead of the ones written."""
    B = A + (1 << 20)
    size = 2 * 5 * 64 * 2                                            # of a tensor in bytes
    for off in (16, size // 2, size - 16):
        for n in (A - off, A + off, B - off, B + off):               # n over x (and y) or h
            assert norm(bra, n=n) == UNSUPPORTED
        for h in (A - off, A + off):
            assert norm(bra, h=h, n=8 * B) == UNSUPPORTED
            assert norm(bra, h=h, x=32 * B, n=8 * B) == UNSUPPORTED
        for at in (A - off, A + off):                                # dx or dy over x, y, dh, dn
            for first in (dict(x=at), dict(y=at), dict(dh=at), dict(dn=at)):
                for out in ("dx", "dy"):
                    far = dict(x=32 * B, y=32 * B, dh=32 * B, dn=32 * B, dx=64 * B, dy=128 * B)
                    assert norm(bra, back=True, **{**far, **first, out: A}) == UNSUPPORTED
        assert norm(bra, back=True, dx=64 * B, dy=64 * B + off) == UNSUPPORTED
    # next to one another is apart: refused for want of scratch only
    apart = dict(x=64 * B, y=64 * B + size, dh=64 * B + 2 * size, dn=64 * B + 3 * size, dx=64 * B + 4 * size, dy=64 * B + 5 * size)
    assert norm(bra, back=True, ws=None, **apart) == NULL


COLUMNS = r"""
#include <stdio.h>
#include <vector>
#include "norm_cols.h"
using namespace bra;
static std::vector<int> seen;
template <bool VECD, bool FULL, bool QUADS> bool each_once(int C, int group) {
    seen.assign(C, 0);
    for (int t = 0; t < group; ++t) {
        const NormCols<VECD, FULL, QUADS> c(t, group, C);
        for (int j = 0; j < NORM_E; ++j)
            if (c.has(j)) {
                if (c.at(j) < 0 || c.at(j) >= C) return false;
                ++seen[c.at(j)];
            }
    }
    for (int n : seen) if (n != 1) return false;
    return true;
}
int main() {
    int bad = 0;
    for (int C = 1; C <= NORM_MAX_C; ++C)
        for (int backward = 0; backward < 2; ++backward)
            for (int post = 0; post < 2; ++post) {
                const int group = norm_group(C);
                const NormKernel k = norm_kernel(group, backward, post);
                const bool wide = norm_wide(C), full = wide && k.full;
                bool ok = !wide || (group <= k.threads && k.threads <= 1024);
                if (C % NORM_E == 0) ok = ok && each_once<true, false, false>(C, group) && each_once<true, false, true>(C, group);
                else ok = ok && (full ? each_once<false, true, false>(C, group) : each_once<false, false, false>(C, group));
                if (!ok && ++bad <= 5) printf("C %d backward %d post %d threads %d of %d\n", C, backward, post, group, k.threads);
            }
    printf("%d", bad);
    return 0;
}
"""


def test_norm_threads_have_each_channel_once():
    """Every width, direction and kernel: the threads of a row have all its channels, each once, and none behind the row."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "s.cpp"), os.path.join(d, "s")
        with open(src, "w") as f:
            f.write(COLUMNS)
        subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(root, "paper_2303_08810_b200", "csrc"), "-o", exe, src], check=True)
        assert subprocess.run([exe], capture_output=True, text=True, check=True).stdout == "0"


# ---------------------------------------------------------------- streams
class OnStreams:
    """torch whose allocations and whose current stream are written down (tensors are the host's)."""

    def __init__(self):
        import contextlib
        import types
        import torch
        self.real, self.current, self.made = torch, 5, []

        class Stream:
            def __init__(self, handle):
                self.cuda_stream = handle

        @contextlib.contextmanager
        def stream(s):
            before, self.current = self.current, s.cuda_stream
            yield
            self.current = before

        self.cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=Stream, stream=stream, default_stream=lambda: Stream(0))

    def __getattr__(self, name):
        real = getattr(self.real, name)
        if name not in ("empty", "zeros", "empty_like"):
            return real

        def make(*args, **kw):
            self.made.append((name, self.current))
            return real(*args, **kw)
        return make


@pytest.mark.parametrize("as_object", [True, False])
@pytest.mark.parametrize("handle", [0, 0x7000])
def test_what_a_call_makes_belongs_to_its_stream(bra, monkeypatch, handle, as_object):
    """Outputs, scratch and its zeros, of every call that is given a stream other than the current one."""
    import torch
    from paper_2303_08810_b200 import binding

    fake, ran_on = OnStreams(), []

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *args: 512
            return lambda *args: (ran_on.append((name, args[-1])), 0)[1]

    monkeypatch.setattr(binding, "_TORCH", fake)
    monkeypatch.setattr(binding, "_LIB", Lib())
    monkeypatch.setattr(binding, "_RAW_STREAM", lambda: fake.current)
    monkeypatch.setattr(binding, "_GET_DEVICE", lambda: -1)
    stream = fake.cuda.Stream(handle) if as_object else handle

    p = bra.make_problem(1, 8, 8, 64, heads=2, S=2, topk=1, dtype="f32")
    m = torch.zeros(1, 8, 8, 64)
    idx = torch.zeros(1, 2, 4, 1, dtype=torch.int32)
    r = bra.make_rope_problem(1, 64, 2, 32, dtype="f32")
    c = bra.make_cross_problem(1, 64, 64, 2, 32, dtype="f32")
    n = bra.make_norm_problem(1, 64, 64, gate="channel", dtype="f32")
    t, w = torch.zeros(1, 64, 64), torch.ones(64)
    lse = torch.zeros(1, 2, 64)
    calls = [
        lambda **k: bra.bra_route(p, m, m, **k), lambda **k: bra.bra_route_static(p, m, m, **k), lambda **k: bra.bra_attend(p, m, m, m, idx, **k),
        lambda **k: bra.bra_forward(p, m, m, m, **k), lambda **k: bra.bra_backward(p, m, m, m, idx, w, lse, m, **k),
        lambda **k: bra.bra_rope(r, t, t, torch.ones(16, dtype=torch.float64), **k),
        lambda **k: bra.bra_cross_attend(c, t, t, t, **k), lambda **k: bra.bra_cross_backward(c, t, t, t, t, lse, t, **k),
        lambda **k: bra.bra_residual_norm(n, t, t, gate=w, w=w, **k), lambda **k: bra.bra_residual_norm_backward(n, t, t, t, t, gate=w, w=w, **k),
    ]
    for call in calls:
        for where, given in ((handle, dict(stream=stream)), (5, {})):
            fake.made.clear()
            ran_on.clear()
            call(**given)
            assert len(ran_on) == 1 and ran_on[0][1] == where
            assert fake.made and all(at == where for _, at in fake.made), ran_on
            assert fake.current == 5


def test_a_call_that_makes_nothing_leaves_the_current_stream(host, monkeypatch):
    """With all outputs and scratch given, and what is not wanted left out, a stream is only passed on."""
    from paper_2303_08810_b200 import binding
    bra, z, torch = host.bra, host.zeros, host.torch
    monkeypatch.setattr(binding, "_on", lambda stream: pytest.fail("entered"))
    p = bra.make_problem(1, 8, 8, 64, heads=2, S=2, topk=1, dtype="f32", lce=False)
    m, idx, ws, lse = z(1, 8, 8, 64), z(1, 2, 4, 1, dtype=torch.int32), z(512, dtype=torch.uint8), z(1, 2, 64)
    r = bra.make_rope_problem(1, 64, 2, 32, kv_heads=0, dtype="f32")
    c = bra.make_cross_problem(1, 64, 64, 2, 32, dtype="f32")
    n = bra.make_norm_problem(1, 64, 64, pre="none", dtype="f32")
    t = z(1, 64, 64)
    bra.bra_route(p, m, m, index=idx, ws=ws, want_means=False, stream=7)
    bra.bra_route_static(p, m, m, index=idx, stream=7)
    bra.bra_attend(p, m, m, m, idx, O=m, ws=ws, want_lse=False, stream=7)
    bra.bra_forward(p, m, m, m, O=m, ws=ws, want_index=False, want_lse=False, stream=7)
    bra.bra_backward(p, m, m, m, idx, None, lse, m, dQ=m, dK=m, dV=m, ws=ws, stream=7)
    bra.bra_rope(r, t, None, z(16, dtype=torch.float64), Qo=t, stream=7)
    bra.bra_cross_attend(c, t, t, t, O=t, ws=ws, want_lse=False, stream=7)
    bra.bra_cross_backward(c, t, t, t, t, lse, t, dQ=t, dK=t, dV=t, ws=ws, stream=7)
    bra.bra_residual_norm(n, t, t, h=t, stream=7)


# ---------------------------------------------------------------- shapes
@pytest.fixture
def host(bra, monkeypatch):
    """The binding over a library that answers 0 and tensors of the host."""
    import types
    import torch
    from paper_2303_08810_b200 import binding

    class Lib:
        def __getattr__(self, name):
            return lambda *args: 512 if name.endswith("_bytes") else b"refused" if name == "bra_status_string" else 0

    monkeypatch.setattr(binding, "_TORCH", torch)
    monkeypatch.setattr(binding, "_LIB", Lib())
    monkeypatch.setattr(binding, "_RAW_STREAM", lambda: 5)
    monkeypatch.setattr(binding, "_GET_DEVICE", lambda: -1)
    return types.SimpleNamespace(torch=torch, bra=bra, zeros=lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype))


@pytest.mark.parametrize("shape,axes,yes", [
    ((2, 30, 4, 8), (2, 30, 4, 8), True), ((2, 30, 32), (2, 30, 4, 8), True), ((60, 32), (2, 30, 4, 8), True), ((1920,), (2, 30, 4, 8), True),
    ((2, 5, 6, 32), (2, 30, 4, 8), True), ((2, 1, 5, 6, 2, 2, 8), (2, 30, 4, 8), True), ((60, 4, 2, 4, 1), (2, 30, 4, 8), True),
    ((2, 960), (2, 30, 4, 8), True), ((2, 4, 30, 8), (2, 30, 4, 8), False), ((30, 2, 32), (2, 30, 4, 8), False),
    ((2, 30, 8, 4), (2, 30, 4, 8), False), ((4, 2, 30, 8), (2, 30, 4, 8), False), ((2, 32, 30), (2, 30, 4, 8), False),
    ((20, 96), (2, 30, 4, 8), False), ((2, 30, 31), (2, 30, 4, 8), False), ((7, 3, 1), (3, 7, 1), False), ((3, 7), (3, 7, 1), True),
    ((2, 30, 32, 2), (2, 30, 4, 8), False), ((0, 32), (2, 30, 4, 8), False), ((), (1, 1), True),
])
def test_shapes_that_lay_out_axes(shape, axes, yes):
    from paper_2303_08810_b200.binding import _lays_out
    assert _lays_out(shape, axes) is yes


def test_calls_refuse_axes_in_another_order(host):
    """As many elements as the problem has, in another order: refused, with the name of the tensor; nothing of it is remembered."""
    bra, z, torch = host.bra, host.zeros, host.torch
    i32, f64 = torch.int32, torch.float64
    r = bra.make_rope_problem(2, 10, 4, 32, dtype="f32")
    c = bra.make_cross_problem(2, 10, 12, 4, 32, kv_heads=2, dtype="f32")
    n = bra.make_norm_problem(2, 10, 64, gate="image", per_image=True, dtype="f32")
    free = bra.make_norm_problem(2, 10, 64, dtype="f32")
    q, kv, lse, x = z(2, 10, 4, 32), z(2, 12, 64), z(2, 4, 10), z(2, 10, 64)
    freq, w = z(16, dtype=f64), z(2, 64)
    rope = dict(p=r, Q=q, K=q, freq=freq, positions=z(2, 10, dtype=i32))
    attend = dict(p=c, Q=q, K=kv, V=kv, key_len=z(2, dtype=i32), key_mask=z(2, 12, dtype=torch.bool), lse=lse)
    back = dict(p=c, Q=q, K=kv, V=kv, O=q, lse=lse, dO=q)
    norm, norm_back = dict(p=n, x=x, y=x, gate=w, w=w), dict(p=n, x=x, y=x, dh=x, dn=x, gate=w, w=w)
    heads_first, wrong_kv = z(2, 4, 10, 32), z(2, 2, 12, 32)
    for call, good, bad in (
            (bra.bra_rope, rope, dict(Q=heads_first, K=heads_first, Qo=heads_first, Ko=heads_first, positions=z(10, 2, 1, dtype=i32))),
            (bra.bra_cross_attend, attend, dict(Q=heads_first, K=wrong_kv, V=wrong_kv, O=heads_first, lse=z(2, 10, 4), key_mask=z(12, 2, dtype=torch.bool))),
            (bra.bra_cross_backward, back, dict(dO=heads_first, O=heads_first, lse=z(10, 2, 4), dQ=heads_first, dK=wrong_kv, dV=wrong_kv)),
            (bra.bra_residual_norm, norm, dict(x=z(10, 2, 64), y=z(2, 64, 10), gate=z(64, 2), w=z(64, 2), h=z(10, 2, 64), n=z(10, 2, 64))),
            (bra.bra_residual_norm_backward, norm_back, dict(dh=z(10, 2, 64), dn=z(2, 64, 10), dx=z(10, 2, 64), dy=z(10, 2, 64)))):
        call(**good)
        for name, t in bad.items():
            for _ in range(2):
                with pytest.raises(bra.BraError, match=f": {name} is") as e:
                    call(**{**good, name: t})
                assert e.value.code == SHAPE
        call(**good)
    # axes merged and split; without weights of images any order of tokens is one
    bra.bra_rope(r, z(20, 128), z(2, 2, 5, 128), freq, positions=z(2, 2, 5, 1, dtype=i32))
    bra.bra_cross_attend(c, z(2, 5, 2, 128), z(24, 64), z(2, 12, 2, 32), key_mask=z(2, 1, 1, 12, dtype=torch.uint8))
    bra.bra_residual_norm(n, z(2, 2, 5, 64), z(20, 64), gate=z(2, 1, 64), w=z(2, 64))
    bra.bra_residual_norm(free, z(10, 2, 64))


def test_problem_structures_match_the_header(bra):
    """Sizes as a C compiler lays the structures out."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = '#include <stdio.h>\n#include "bra.h"\nint main(void){printf("%zu %zu %zu %zu",sizeof(bra_problem),sizeof(bra_rope_problem),' \
           'sizeof(bra_cross_problem),sizeof(bra_norm_problem));return 0;}\n'
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        with open(src, "w") as f:
            f.write(code)
        subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", exe, src], check=True)
        sizes = [int(v) for v in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [ctypes.sizeof(t) for t in (bra.BraProblem, bra.BraRopeProblem, bra.BraCrossProblem, bra.BraNormProblem)]
