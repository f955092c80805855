"""The layer norm's forward and backward pass on the GPU against the 64-bit formula.

Tolerances, per value, from the arithmetic (u = 2^-24, sums over F in chains of at most K = F / 64 + 16
additions, over rows in chains of at most KB = B / 64 + 600):
  mean: K u mean|h|;  the squares around it, and so rstd, relatively (K + 4) u and what the mean is off,
  squared and so below the rest;  xh: the mean's error times rstd, and |xh| times rstd's;
  dH: rstd times the two sums' errors, K u of their terms' magnitudes, and 4 u of what is subtracted;
  dweight, dbias: (KB + 6) u of their terms' magnitudes;
and half a step of the stored type.
"""
import numpy as np
import pytest

import train_ref as ref
from gpu_helpers import say

pytestmark = pytest.mark.gpu
U = ref.U32


@pytest.fixture(scope="module")
def hs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    import paper_2606_01117_amd as m
    return m


def _dt(name):
    import torch
    return torch.float32 if name == "f32" else torch.bfloat16


def _half(name):
    return ref.U32 if name == "f32" else ref.U16


def _code(hs, name):
    return hs.HASTE_DTYPE_F32 if name == "f32" else hs.HASTE_DTYPE_BF16


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _check(name, got, want, tol):
    off = np.abs(got - want)
    assert got.shape == want.shape
    worst = float((off / tol).max()) if off.size else 0.0
    say(f"    {name:<8s} largest error {float(off.max()) if off.size else 0:.3e}, {worst:.3f} of its tolerance")
    assert np.all(off <= tol), name


class Case:
    def __init__(self, B, F, h, x, seed=0, rows=1, affine=True, shift=0.3, eps=1e-5, first=0, pad=0):
        """rows: H's rows are that many times F + pad apart, starting `first` values in."""
        import torch
        g = torch.Generator().manual_seed(seed + 7919 * F + B)
        self.B, self.F, self.h, self.x, self.eps = B, F, h, x, eps
        self.ld = rows * F + pad
        self.store = (torch.randn(first + B * self.ld + F, generator=g) * 1.5 + shift).to(_dt(h)).cuda()
        self.H = self.store[first:first + B * self.ld].view(B, self.ld)[:, :F] if B else self.store[:0].view(0, F)
        self.w = (torch.randn(F, generator=g) * 0.2 + 1).cuda() if affine else None
        self.b = torch.randn(F, generator=g).cuda() if affine else None
        self.dX = (torch.randn((B, F), generator=g) * 0.1).to(_dt(x)).cuda()

    def forward(self, hs, X=None, stats=True, stream=None):
        import torch
        X = torch.full((self.B, self.F), 7.0, dtype=_dt(self.x), device="cuda") if X is None else X
        mean, rstd = (torch.full((self.B,), 7.0, device="cuda") if stats else None for _ in range(2))
        if stream is not None:
            torch.cuda.synchronize()
        hs.haste_layer_norm_fwd(self.B, self.F, _code(hs, self.h), self.H, self.w, self.b, self.eps, _code(hs, self.x), X,
                                mean, rstd, stream)
        return X, mean, rstd

    def reference(self):
        h = _host(self.H)
        out, mean, rstd = ref.layer_norm(h, None if self.w is None else _host(self.w),
                                         None if self.b is None else _host(self.b), self.eps)
        K = self.F / 64 + 16
        xh = (h - mean) * rstd
        tm = K * U * np.abs(h).mean(1, keepdims=True) + U * np.abs(mean)
        # the mean's own rounding moves every difference alike; to second order that enters the spread
        tr = ((K + 6) * U + (tm * rstd) ** 2) * rstd
        w = 1.0 if self.w is None else np.abs(_host(self.w))
        tx = w * (tm * rstd + np.abs(xh) * (tr / rstd + 4 * U)) + 2 * U * np.abs(out)
        return out, mean, rstd, tx * (1 + _half(self.x)) + np.abs(out) * _half(self.x) + 1e-40, tm, tr

    def check_forward(self, X, mean, rstd):
        out, mu, rs, tx, tm, tr = self.reference()
        _check("X", _host(X), out, tx)
        if mean is not None:
            _check("mean", _host(mean), mu[:, 0], tm[:, 0] + 1e-40)
            _check("rstd", _host(rstd), rs[:, 0], tr[:, 0])

    def stats(self):
        """mean and rstd as the forward call leaves them: 64 bits, rounded to fp32."""
        import torch
        _, mu, rs = ref.layer_norm(_host(self.H), None, None, self.eps)
        return torch.from_numpy(mu[:, 0]).float().cuda(), torch.from_numpy(rs[:, 0]).float().cuda()

    def backward(self, hs, mean, rstd, dH="new", dw="new", db="new", beta=0, stream=None, dX=None, ws=None, sync=True):
        import torch
        new = {"dH": lambda: torch.full((self.B, self.F), 7.0, dtype=_dt(self.h), device="cuda"),
               "dw": lambda: torch.full((self.F,), 0.5, device="cuda")}
        dH = new["dH"]() if isinstance(dH, str) else dH
        dw, db = (new["dw"]() if isinstance(t, str) else t for t in (dw, db))
        ws = hs.workspace(hs.haste_layer_norm_workspace_bytes(self.B, self.F)) if ws is None else ws
        if stream is not None and sync:
            torch.cuda.synchronize()
        hs.haste_layer_norm_bwd(self.B, self.F, _code(hs, self.h), self.H, self.w, mean, rstd, _code(hs, self.x),
                                self.dX if dX is None else dX, dH, dw, db, beta, ws, stream)
        return dH, dw, db

    def check_backward(self, mean, rstd, dH, dw, db, old=0.0):
        h, d = _host(self.H), _host(self.dX)
        mu, rs = _host(mean)[:, None], _host(rstd)[:, None]
        w = np.ones(self.F) if self.w is None else _host(self.w)
        gh, gw, gb = ref.layer_norm_grads(h, w, mu, rs, d)
        K, KB = self.F / 64 + 16, self.B / 64 + 600
        xh = (h - mu) * rs
        q = d * w
        s, t = np.abs(q).mean(1, keepdims=True), np.abs(q * xh).mean(1, keepdims=True)
        if dH is not None:
            tol = rs * ((K + 4) * U * (s + np.abs(xh) * t) + 5 * U * (np.abs(q) + s + np.abs(xh) * t))
            _check("dH", _host(dH), gh, tol * (1 + _half(self.h)) + np.abs(gh) * _half(self.h) + 1e-40)
        if dw is not None:
            _check("dweight", _host(dw), gw + old, (KB + 6) * U * np.abs(d * xh).sum(0) + 2 * U * abs(old) + 1e-40)
        if db is not None:
            _check("dbias", _host(db), gb + old, (KB + 6) * U * np.abs(d).sum(0) + 2 * U * abs(old) + 1e-40)


SIZES = [(1, 1), (1, 768), (3, 2), (5, 63), (7, 64), (2, 65), (33, 100), (512, 768), (77, 500), (129, 1003), (40, 1024),
         (17, 1030), (9, 2048), (6, 2049), (5, 4096), (3, 8191), (4, 8192), (2, 8200), (2, 20001), (1500, 96),
         (4100, 256), (6, 300), (5, 384), (4, 385), (5, 1025), (4, 1300), (3, 1536), (3, 2500), (2, 4097), (2, 5000),
         (2, 6144), (2, 9000), (2, 12289), (2, 16384), (2, 16385)]


@pytest.mark.parametrize("B,F", SIZES)
@pytest.mark.parametrize("h,x", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_forward_and_backward(hs, B, F, h, x):
    say(f"[layer norm] B={B} F={F} {h} -> {x}")
    c = Case(B, F, h, x)
    c.check_forward(*c.forward(hs))
    mean, rstd = c.stats()
    c.check_backward(mean, rstd, *c.backward(hs, mean, rstd))


@pytest.mark.parametrize("B,F", [(20000, 128), (20001, 131), (9000, 768), (8999, 769), (5000, 500), (3000, 2048),
                                 (2999, 1027), (2500, 4096), (2100, 2051), (1300, 8192), (20000, 301), (5000, 1026),
                                 (4000, 1500), (2000, 5001), (700, 9001), (600, 16000)])
@pytest.mark.parametrize("h,x", [("bf16", "f32"), ("f32", "bf16")])
def test_many_rows(hs, B, F, h, x):
    """Workgroups of several teams, each of several rows."""
    test_forward_and_backward(hs, B, F, h, x)


@pytest.mark.parametrize("B,F,h,x,kw", [
    (12, 768, "f32", "bf16", dict(rows=5)), (12, 768, "bf16", "f32", dict(rows=3, first=768)),
    (9, 768, "bf16", "bf16", dict(first=1, pad=1)), (9, 768, "f32", "f32", dict(first=3, pad=5)),
    (9, 770, "bf16", "bf16", dict(first=2, pad=2)), (7, 101, "bf16", "f32", dict(first=5, pad=6)),
    (3, 9000, "bf16", "bf16", dict(first=1, pad=3)), (5, 1500, "f32", "bf16", dict(pad=2)), (6, 1002, "bf16", "f32", {}),
    (64, 256, "bf16", "bf16", dict(affine=False)), (9, 333, "f32", "f32", dict(affine=False)),
])
def test_strides_alignment_and_no_weight(hs, B, F, h, x, kw):
    say(f"[layer norm] B={B} F={F} {h} -> {x} {kw}")
    c = Case(B, F, h, x, **kw)
    c.check_forward(*c.forward(hs))
    mean, rstd = c.stats()
    c.check_backward(mean, rstd, *c.backward(hs, mean, rstd))
    X, none, _ = c.forward(hs, stats=False)
    assert none is None
    c.check_forward(X, None, None)


@pytest.mark.parametrize("F", [100, 768, 9001])
def test_weight_or_bias_alone(hs, F):
    for drop in ("w", "b"):
        c = Case(11, F, "bf16", "f32")
        setattr(c, drop, None)
        c.check_forward(*c.forward(hs))
        mean, rstd = c.stats()
        c.check_backward(mean, rstd, *c.backward(hs, mean, rstd))


def test_two_streams_at_once(hs):
    """Calls that overlap, each with a workspace of its own."""
    import torch
    cases = [Case(3000 + 7 * k, 768, "bf16", "f32", seed=k) for k in range(4)]
    stats = [c.stats() for c in cases]
    alone = [c.backward(hs, *s) for c, s in zip(cases, stats)]
    ws = [hs.workspace(hs.haste_layer_norm_workspace_bytes(c.B, c.F)) for c in cases]
    out = [[torch.zeros_like(t) for t in a] for a in alone]
    side = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [c.backward(hs, *s, *o, stream=q, ws=w, sync=False) for c, s, o, q, w in zip(cases, stats, out, side, ws)]
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("B,F", [(33, 768), (5, 99), (3, 4104), (2, 9001)])
def test_views_as_outputs_leave_the_rest(hs, B, F):
    """X and dH as the first rows of wider sequences: what lies between their rows stays as it was."""
    import torch
    c = Case(B, F, "f32", "f32")
    for kind in ("f", "b"):
        big = torch.full((B + 1, 3, F + 5), 3.0, device="cuda")
        out = big[:B, 1, 2:2 + F]
        mean, rstd = c.stats()
        if kind == "f":
            X, m, r = c.forward(hs, X=out)
            c.check_forward(X, m, r)
        else:
            c.check_backward(mean, rstd, *c.backward(hs, mean, rstd, dH=out))
        out.fill_(3.0)
        assert bool((big == 3.0).all())


@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("F", [768, 301, 3000, 9001])
def test_in_place(hs, h, F):
    import torch
    c = Case(21, F, h, h)
    X, mean, rstd = c.forward(hs)
    dH, dw, db = c.backward(hs, mean, rstd)
    d = c.dX.clone()
    c.backward(hs, mean, rstd, dH=d, dX=d)
    assert torch.equal(d, dH)
    keep = c.H.clone()
    hs.haste_layer_norm_fwd(21, F, _code(hs, h), keep, c.w, c.b, c.eps, _code(hs, h), keep, None, None)
    assert torch.equal(keep, X)


def test_skipped_outputs_accumulation_and_repeats(hs):
    import torch
    for B, F in ((700, 768), (90, 1003), (3, 8200)):
        c = Case(B, F, "bf16", "f32")
        mean, rstd = c.stats()
        dH, dw, db = c.backward(hs, mean, rstd)
        again = c.backward(hs, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip((dH, dw, db), again)), "the same call gives the same bits"
        assert torch.equal(c.backward(hs, mean, rstd, dw=None, db=None)[0], dH)
        _, w2, none = c.backward(hs, mean, rstd, dH=None, db=None)
        assert torch.equal(w2, dw)
        _, none, b2 = c.backward(hs, mean, rstd, dH=None, dw=None)
        assert torch.equal(b2, db)
        c.check_backward(mean, rstd, *c.backward(hs, mean, rstd, beta=1), old=0.5)


def test_no_rows(hs):
    import torch
    c = Case(0, 40, "bf16", "f32")
    c.forward(hs)
    e = torch.empty(0, device="cuda")
    _, dw, db = c.backward(hs, e, e, beta=1)
    assert bool((dw == 0.5).all()) and bool((db == 0.5).all())
    _, dw, db = c.backward(hs, e, e)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("F", [64, 500, 768, 3000])
def test_rows_that_are_not_ordinary(hs, F):
    """Equal values (their spread is rounding alone), a large offset, an infinity and a NaN in rows of their own."""
    import torch
    c = Case(8, F, "f32", "f32")
    c.H[0], c.H[2] = 0.0, 4.0
    c.H[4] += 1000.0
    c.H[5, F // 2] = float("inf")
    c.H[6, 0] = float("nan")
    X, mean, rstd = c.forward(hs)
    dH, dw, db = c.backward(hs, mean, rstd)
    ok = [0, 1, 2, 3, 4, 7]
    assert bool(torch.isnan(X[[5, 6]]).all()) and bool(torch.isnan(dH[[5, 6]]).all())
    assert bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())
    out, mu, rs, tx, tm, tr = (a[ok] for a in c.reference())
    # rows of equal powers of two and zeros are exact sums: the spread is eps's root
    _check("X", _host(X)[ok], out, tx)
    assert bool((X[0] == c.b).all()) and bool((X[2] == c.b).all())
    assert bool(torch.isfinite(dH[ok]).all())


def test_gradient_against_differences(hs):
    """The directional derivative of sum(dX * X) by the forward call's own values: D(e) = (f(h + e d) - f(h - e d)) / 2e,
    (4 D(e) - D(2e)) / 3.  Error: that of each f (the forward call's tolerances, and half a step of every input) 3/2 over
    e; and the fifth derivative's, a few times (2e)^4 of the sum's magnitude."""
    import torch
    for B, F in ((6, 64), (4, 301), (3, 2500)):
        c = Case(B, F, "f32", "f32", seed=5)
        mean, rstd = c.stats()
        dH, dw, db = c.backward(hs, mean, rstd)
        d, base, e = torch.randn_like(c.H), c.H.clone(), 2.0 ** -6

        def f(s):
            c.H.copy_(base + s * d)
            return float((c.forward(hs)[0].double() * c.dX.double()).sum())

        D = lambda e: (f(e) - f(-e)) / (2 * e)
        got = (4 * D(e) - D(2 * e)) / 3
        c.H.copy_(base)
        want = float((dH.double() * d.double()).sum())
        _, _, _, tx, _, _ = c.reference()
        fwd = float((tx * np.abs(_host(c.dX))).sum())
        tol = 1.5 / e * (fwd + U * float((np.abs(_host(dH)) * (np.abs(_host(base)) + 2 * e * np.abs(_host(d)))).sum()))
        tol += 40 * (2 * e) ** 4 * float((np.abs(_host(dH)) * np.abs(_host(d))).sum())
        say(f"    differences: {got:.6f}, gradient {want:.6f}, tolerance {tol:.2e}")
        assert abs(got - want) <= tol
        # X is linear in weight and bias; chains of at most 600 + 10 additions
        lin = float((dw.double() * c.w.double()).sum() + (db.double() * c.b.double()).sum())
        size = np.abs(_host(c.dX)) * (np.abs(_host(c.forward(hs)[0])) + 2 * np.abs(_host(c.b)))
        assert abs(lin - f(0.0)) <= fwd + 610 * U * float(size.sum())


def test_other_stream_and_large_row_count(hs):
    import torch
    c = Case(70001, 65, "bf16", "bf16")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    X, mean, rstd = c.forward(hs, stream=side)
    dH, dw, db = c.backward(hs, mean, rstd, stream=side.cuda_stream)
    side.synchronize()
    c.check_forward(X, mean, rstd)
    c.check_backward(mean, rstd, dH, dw, db)


def test_offsets_past_32_bits(hs):
    """Rows whose last starts more than 2^32 values behind the first."""
    import torch
    B, F, ld = 3, 768, (1 << 31) + 8
    big = torch.empty(2 * ld + F, dtype=torch.bfloat16, device="cuda")
    H = torch.as_strided(big, (B, F), (ld, 1))
    c = Case(B, F, "bf16", "bf16")
    H.copy_(c.H)
    c.H = H
    X, mean, rstd = c.forward(hs)
    c.check_forward(X, mean, rstd)
    c.check_backward(mean, rstd, *c.backward(hs, mean, rstd))


def test_captured_and_replayed(hs):
    import torch
    c = Case(300, 768, "bf16", "f32")
    X = torch.empty((300, 768), device="cuda")
    mean, rstd, dw, db = (torch.empty(n, device="cuda") for n in (300, 300, 768, 768))
    dH = torch.empty((300, 768), dtype=torch.bfloat16, device="cuda")
    ws = hs.workspace(hs.haste_layer_norm_workspace_bytes(300, 768))

    def run():
        hs.haste_layer_norm_fwd(300, 768, 1, c.H, c.w, c.b, 1e-5, 0, X, mean, rstd)
        hs.haste_layer_norm_bwd(300, 768, 1, c.H, c.w, mean, rstd, 0, c.dX, dH, dw, db, 0, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(3):
        c.H.normal_()
        c.dX.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (X, mean, rstd, dH, dw, db)]
        for t in (X, mean, rstd, dH, dw, db):
            t.fill_(9.0)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (X, mean, rstd, dH, dw, db))), f"replay {k}"


def test_binding_refuses(hs):
    import torch
    x = torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError, match="dtype"):
        hs.haste_layer_norm_fwd(4, 8, hs.HASTE_DTYPE_BF16, x, None, None, 1e-5, hs.HASTE_DTYPE_F32, x)
    with pytest.raises(ValueError, match="weight"):
        hs.haste_layer_norm_fwd(4, 8, 0, x, x[0, :7], None, 1e-5, 0, x)
    with pytest.raises(hs.HasteError, match="workspace"):
        hs.haste_layer_norm_bwd(4, 8, 0, x, None, x[0, :4].contiguous(), x[1, :4].contiguous(), 0, x,
                                None, torch.zeros(8, device="cuda"))
