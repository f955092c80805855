"""The gradient norm and the AdamW step on the GPU, against plain implementations (train_ref).

The moments are defined by their fp32 operations, in either width, and are compared for equality.  The
weights: the update is formed with a reciprocal and five roundings, so it is off by at most 8 u of its terms'
magnitudes (u = 2^-24); the result by u of its own, and by half a step of bf16 where it is stored so.
The norm is a 64-bit sum, rounded once to fp32: 1.01 u; its factor by one division more.
"""
import math

import numpy as np
import pytest

import train_ref as ref
from gpu_helpers import say

pytestmark = pytest.mark.gpu
U = ref.U32
OPTS = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=7, seed=12345)


@pytest.fixture(scope="module")
def hs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    import paper_2606_01117_amd as m
    return m


def _np(t):
    import torch
    if t.dtype in (torch.bfloat16, torch.float32):
        return t.detach().float().cpu().numpy()
    return t.detach().cpu().numpy()


class Tensors:
    """A list of tensors side by side in arrays of their own kind, with words between them that nothing may touch."""

    GUARD = 64

    def __init__(self, hs, sizes, w="f32", g="f32", bits=32, master=False, seed=0, edge=False, lr_scale=None, decay=None):
        import torch
        rng = np.random.default_rng(seed + 31 * len(sizes) + sizes[0])
        self.hs, self.sizes, self.bits, self.w, self.master = hs, sizes, bits, w, master
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}
        self.at, at = [], self.GUARD
        for n in sizes:
            self.at.append(at)
            at += -(-n // self.GUARD) * self.GUARD + self.GUARD
        self.total = at
        live = np.zeros(at, bool)
        for n, a in zip(sizes, self.at):
            live[a:a + n] = True
        self.live = torch.from_numpy(live).cuda()

        def mk(x, d):
            return torch.from_numpy(x.astype(np.float32)).cuda().to(d)

        grad = rng.standard_normal(at) * 10.0 ** rng.uniform(-4, 0, at)
        if edge:
            grad[rng.random(at) < 0.2] = 0.0
            grad[rng.random(at) < 0.02] = 1e-42          # below fp32's normal range
            grad[rng.random(at) < 0.02] = 3e12
        weight = rng.standard_normal(at)
        self.grad, self.W = mk(grad, dt[g]), mk(weight, dt[w])
        self.W32 = mk(weight, torch.float32) if master else None
        m = rng.standard_normal(at) * 0.05
        r = np.abs(rng.standard_normal(at)) * 10.0 ** rng.uniform(-3, 0, at)
        if edge:
            z = rng.random(at) < 0.3
            m[z] = r[z] = 0.0
            for a in self.at[::3]:
                m[a:a + 64] = r[a:a + 64] = 0.0
        if bits == 8:
            d = rng.integers(0, 65536, at)
            m, sm = ref._store(m.astype(np.float32), d, False)
            v, sv = ref._store(r.astype(np.float32), d, True)
            self.m, self.v = torch.from_numpy(m).cuda(), torch.from_numpy(v).cuda()
            self.scale = torch.from_numpy(np.stack([sm, sv], 1)).cuda()
        else:
            self.m, self.v, self.scale = mk(m, torch.float32), mk(r * r, torch.float32), None
        self.lr_scale = lr_scale or [1.0 + 0.5 * (k % 3) for k in range(len(sizes))]
        self.decay = decay or [0.1 * (k % 2) for k in range(len(sizes))]
        made = []
        for k, (n, a) in enumerate(zip(sizes, self.at)):
            cut = lambda t: None if t is None else t[a:a + n]
            made.append(hs.param(self.W[a:a + n], self.grad[a:a + n], self.m[a:a + n], self.v[a:a + n],
                                 None if self.scale is None else self.scale[a // 32:a // 32 + (n + 31) // 32],
                                 cut(self.W32), self.lr_scale[k], self.decay[k]))
        self.params = hs.param_list(made)

    def arrays(self):
        return {k: t for k, t in (("W", self.W), ("W32", self.W32), ("m", self.m), ("v", self.v), ("scale", self.scale))
                if t is not None}

    def snapshot(self):
        return {k: t.clone() for k, t in self.arrays().items()}

    def check(self, before, opts, gs=1.0, equal_states=True):
        import torch
        grad = _np(self.grad)
        now = {k: _np(t) for k, t in self.arrays().items()}
        old = {k: _np(t) for k, t in before.items()}
        for k, (n, a) in enumerate(zip(self.sizes, self.at)):
            part = slice(a, a + n)
            blocks = slice(a // 32, a // 32 + (n + 31) // 32)
            w, step, m, v, scale = ref.adamw(old["W32" if self.master else "W"][part], grad[part], old["m"][part],
                                             old["v"][part], None if self.scale is None else old["scale"][blocks], opts, k,
                                             self.lr_scale[k], self.decay[k], gs)
            if self.scale is None:
                np.testing.assert_array_equal(now["m"][part], m, err_msg=f"m of tensor {k}")
                np.testing.assert_array_equal(now["v"][part], v, err_msg=f"v of tensor {k}")
            else:
                np.testing.assert_array_equal(now["scale"][blocks], scale, err_msg=f"scales of tensor {k}")
                np.testing.assert_array_equal(now["m"][part], m, err_msg=f"m of tensor {k}")
                np.testing.assert_array_equal(now["v"][part], v, err_msg=f"v of tensor {k}")
            for name, half in (("W", ref.U16 if self.w == "bf16" else U), ("W32", U)):
                if name not in now:
                    continue
                tol = 8 * U * step + 2 * U * np.abs(w)
                tol = tol * (1 + half) + half * np.abs(w)
                off = np.abs(now[name][part] - w)
                bad = ~(off <= tol) & ~(np.isnan(w) & np.isnan(now[name][part]))
                assert not bad.any(), f"{name} of tensor {k}: {off[bad][:3]} over {tol[bad][:3]}"
        # what lies between the tensors
        for k, t in self.arrays().items():
            live = self.live if k != "scale" else self.live.view(-1, 32).any(1)
            assert torch.equal(t[~live].view(torch.uint8), before[k][~live].view(torch.uint8)), f"{k} beside the tensors"


def _step(hs, t, opts, stream=None, **dev):
    import torch
    before = t.snapshot()
    torch.cuda.synchronize()                     # the call may go to another stream
    hs.haste_adamw(t.params, hs.adamw_opts(**opts, **dev), stream)
    torch.cuda.synchronize()
    return before


SIZES = {"one": [1], "few": [5, 31, 32, 33, 64, 1], "odd": [2047, 2049, 8193, 4096, 7, 100003],
         "empty": [1, 1, 333, 1], "many": [1 + 37 * k % 211 for k in range(170)]}


@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("w,g,bits,master", [
    ("f32", "f32", 32, False), ("bf16", "f32", 32, False), ("bf16", "bf16", 32, True), ("f32", "bf16", 32, False),
    ("bf16", "bf16", 32, False), ("bf16", "f32", 32, True), ("f32", "f32", 8, False), ("bf16", "f32", 8, False),
    ("bf16", "bf16", 8, True), ("f32", "bf16", 8, False), ("bf16", "bf16", 8, False), ("bf16", "f32", 8, True)])
def test_step(hs, name, w, g, bits, master):
    say(f"[adamw] {name} w={w} g={g} bits={bits} master={master}")
    t = Tensors(hs, SIZES[name], w, g, bits, master, edge=name != "odd")
    for step in (1, 2, 1000):
        o = dict(OPTS, step=step)
        t.check(_step(hs, t, o), o)


@pytest.mark.parametrize("bits", [32, 8])
def test_mixed_list_with_empty_tensors(hs, bits):
    """One list of all kinds, tensors of no values among them (their numbers count for the draws)."""
    import torch
    kinds = [("f32", "f32", 32, False), ("bf16", "f32", bits, True), ("bf16", "bf16", bits, False), ("f32", "bf16", 40 - bits, False)]
    ts = [Tensors(hs, [100 + 64 * j], *kind, seed=j) for j, kind in enumerate(kinds * 20)]
    entries, number = [], []
    for j, t in enumerate(ts):
        if j % 7 == 3:
            entries.append(hs.haste_param_t(n=0))
        number.append(len(entries))
        entries.append(t.params[0])
    lst = hs.param_list(entries)
    before = [t.snapshot() for t in ts]
    hs.haste_adamw(lst, hs.adamw_opts(**OPTS))
    torch.cuda.synchronize()
    for t, b, k in zip(ts, before, number):
        plain = ref.adamw
        try:
            ref.adamw = lambda *a, _k=k, **kw: plain(*a[:6], _k, *a[7:], **kw)
            t.check(b, OPTS)
        finally:
            ref.adamw = plain


@pytest.mark.parametrize("w,g,bits,master", [("f32", "f32", 32, False), ("bf16", "f32", 32, False), ("bf16", "bf16", 32, True),
                                             ("f32", "bf16", 8, False), ("bf16", "bf16", 8, False), ("bf16", "f32", 8, True)])
def test_long_lists_give_the_same_bits(hs, w, g, bits, master):
    """Lists of more than 128 MB of weights take the accesses past the caches: the same tensors behind a large one and
    behind an empty one of the same number."""
    import torch
    n = 70_000_000
    z = lambda dt: torch.zeros(n, dtype=dt, device="cuda")
    big = hs.param(z(torch.bfloat16), z(torch.bfloat16), z(torch.uint8), z(torch.uint8),
                   torch.zeros((n + 31) // 32, 2, dtype=torch.uint8, device="cuda"))
    got = []
    for head in (hs.haste_param_t(n=0), big):
        t = Tensors(hs, [1000, 33, 2048, 5], w, g, bits, master, edge=True)
        before = t.snapshot()
        hs.haste_adamw(hs.param_list([head, *t.params]), hs.adamw_opts(**OPTS))
        torch.cuda.synchronize()
        assert not torch.equal(before["W"], t.W)
        got.append(t.snapshot())
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])
    assert not bool(big.keep[0].any()) and not bool(big.keep[2].any()) and not bool(big.keep[3].any())


def test_offsets_past_32_bits(hs):
    """A tensor of more than 2^32 values: the step and the norm reach its end, its moments and draws go by the place."""
    import torch
    n = (1 << 32) + 32 * 7 + 5
    W, G = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    scale = torch.zeros(((n + 31) // 32, 2), dtype=torch.uint8, device="cuda")
    places = [0, 1 << 31, (1 << 32) - 64, (1 << 32) + 32 * 6]
    ends = [p + 64 for p in places[:3]] + [n]
    for p, e in zip(places, ends):
        G[p:e] = torch.randn(e - p, device="cuda").bfloat16()
        W[p:e] = torch.randn(e - p, device="cuda").bfloat16()
    params = hs.param_list([hs.param(W, G, m, v, scale, weight_decay=0.1)])
    old = [_np(W[p:e]) for p, e in zip(places, ends)]
    out = torch.zeros(2, device="cuda")
    hs.haste_grad_norm(params, 1e9, out, hs.workspace(hs.haste_grad_norm_workspace_bytes(params)))
    hs.haste_adamw(params, hs.adamw_opts(**OPTS))
    torch.cuda.synchronize()
    total = math.sqrt(sum(float((G[p:e].double() ** 2).sum()) for p, e in zip(places, ends)))
    assert abs(float(out[0]) - total) <= 1.01 * U * total
    for p, e, w in zip(places, ends, old):
        zero = np.zeros(e - p, np.uint8)
        new, step, rm, rv, rs = ref.adamw(w, _np(G[p:e]), zero, zero, np.zeros(((e - p + 31) // 32, 2), np.uint8), OPTS, 0, 1.0,
                                          0.1, 1.0, p)
        np.testing.assert_array_equal(_np(m[p:e]), rm)
        np.testing.assert_array_equal(_np(v[p:e]), rv)
        np.testing.assert_array_equal(_np(scale[p // 32:(e + 31) // 32]), rs)
        tol = 8 * U * step + 2 * U * np.abs(new)
        assert np.all(np.abs(_np(W[p:e]) - new) <= tol * (1 + ref.U16) + ref.U16 * np.abs(new))
    for lo in range(0, n, 1 << 30):               # the rest stays zero
        hi = min(n, lo + (1 << 30))
        rest = torch.ones(hi - lo, dtype=torch.bool, device="cuda")
        for p, e in zip(places, ends):
            rest[max(p - lo, 0):max(e - lo, 0)] = False
        assert not bool((m[lo:hi] != 0)[rest].any()) and not bool((W[lo:hi] != 0)[rest].any())


@pytest.mark.parametrize("bits", [32, 8])
def test_options_on_the_device_and_the_factor(hs, bits):
    import torch
    t = Tensors(hs, [1000, 50, 4097], "bf16", "f32", bits, True)
    lr, step, gs = torch.tensor([3e-3], device="cuda"), torch.tensor([41], device="cuda"), torch.tensor([0.37], device="cuda")
    o = dict(OPTS, lr=float(np.float32(3e-3)), step=41)
    before = _step(hs, t, dict(OPTS, lr=0.5, step=1), lr_dev=lr, step_dev=step, grad_scale=gs)
    t.check(before, o, gs=np.float32(0.37))
    # the values, not the pointers, are what counts; and the host's way gives the same bits but for beta^step's last ones
    for s in (1, 2, 3, 1000, 123456789):
        step.fill_(s)
        gs.fill_(1.0)
        t.check(_step(hs, t, dict(OPTS, step=1), step_dev=step, lr_dev=lr, grad_scale=gs), dict(o, step=s))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gs", [float("nan"), float("inf"), float("-inf")])
def test_a_factor_that_is_not_finite_changes_nothing(hs, bits, gs):
    import torch
    t = Tensors(hs, [1000, 50], "bf16", "f32", bits, True)
    before = _step(hs, t, OPTS, grad_scale=torch.full((1,), gs, device="cuda"))
    assert all(torch.equal(before[k], v) for k, v in t.arrays().items())


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite_reach_their_own_weights(hs, bits):
    import torch
    t = Tensors(hs, [500], "f32", "f32", bits)
    a = t.at[0]
    t.grad[a + 3], t.grad[a + 40], t.grad[a + 41], t.grad[a + 499] = float("nan"), float("inf"), float("-inf"), 3e30
    before = _step(hs, t, OPTS)
    hit = torch.zeros(500, dtype=torch.bool, device="cuda")
    hit[[3, 40, 41]] = True
    assert bool(torch.isnan(t.W[a:a + 500])[[3, 40, 41]].all()) and bool(torch.isfinite(t.W[a:a + 500][~hit]).all())
    if bits == 8:
        code = t.m[a:a + 500].view(torch.float8_e4m3fn).float()
        assert bool(torch.isnan(code)[[3, 40, 41]].all()) and bool(torch.isfinite(code[~hit]).all())
    clean = {k: v.clone() for k, v in before.items()}
    # the others as if those gradients had been zero: their blocks' scales go by finite values alone
    for j in (3, 40, 41):
        t.grad[a + j] = 0.0
    got = t.snapshot()
    for k, v in t.arrays().items():
        v.copy_(clean[k])
    _step(hs, t, OPTS)
    for k in ("W", "m", "v"):
        x, y = got[k][a:a + 500], t.arrays()[k][a:a + 500]
        same = (x.view(torch.uint8).view(500, -1) == y.view(torch.uint8).view(500, -1)).all(1)
        quiet = torch.ones(500, dtype=torch.bool, device="cuda")
        quiet[:64] = bits == 32                  # those blocks' largest value may have been one of the three
        assert bool(same[quiet & ~hit].all()), k


def test_rounding_is_right_in_the_mean(hs):
    """beta1 = 0 stores m = grad: over many draws the stored value's mean is the value, within five standard
    errors of the two neighbours' distance; the roots of v likewise."""
    import torch
    n = 1 << 18
    W, m, v = torch.zeros(n, device="cuda"), *(torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    scale = torch.zeros((n // 32, 2), dtype=torch.uint8, device="cuda")
    g = torch.full((n,), 1.0, device="cuda")
    g[::32] = 100.0                              # the block's largest
    p = hs.param_list([hs.param(W, g, m, v, scale)])
    for x in (1.0 + 1 / 32, 0.77, 3.3e-3):
        g.view(-1, 32)[:, 1:] = x
        hs.haste_adamw(p, hs.adamw_opts(0.0, 0.0, 0.0, step=1, seed=int(x * 1e6)))
        torch.cuda.synchronize()
        for q, s, sign in ((m, 0, 1), (v, 1, 1)):
            val = (q.view(torch.float8_e4m3fn).double() * torch.exp2(scale[:, s].double() - 127).repeat_interleave(32))
            val = val.view(-1, 32)[:, 1:].reshape(-1)
            near = torch.unique(val).cpu().numpy()
            assert len(near) <= 2, near
            gap = near[-1] - near[0] if len(near) == 2 else 0.0
            mean, want = float(val.mean()), float(np.float32(x))
            err = 5 * max(gap, abs(want) * 2 ** -22) / 2 / math.sqrt(val.numel()) + gap / 65536 + abs(want) * 2 * U
            say(f"    {x}: stored as {near}, mean {mean:.8g}, off by {abs(mean - want):.2e}, tolerance {err:.2e}")
            assert abs(mean - want) <= err


def test_zero_bytes_are_zero_moments_and_draws_follow_seed_and_step(hs):
    import torch
    n = 4000
    g = torch.randn(n, device="cuda")
    got = []
    for seed, step in ((1, 1), (1, 1), (1, 2), (2, 1)):
        W, m, v = torch.zeros(n, device="cuda"), *(torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
        s = torch.zeros((n // 32, 2), dtype=torch.uint8, device="cuda")
        hs.haste_adamw(hs.param_list([hs.param(W, g, m, v, s)]), hs.adamw_opts(1e-3, step=step, seed=seed))
        got.append((W, m, v, s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[0], got[1]))
    assert torch.equal(got[2][1], got[3][1]), "seed + step is what counts"
    assert not torch.equal(got[0][1], got[2][1])
    assert torch.equal(got[0][0], got[3][0]), "the weights take the moments before they are rounded"
    # the first step's moments over their corrections are g and g^2: the step is lr g / (|g| + eps), which is lr's sign
    # only where eps is small beside |g|
    first = 1e-3 * g.double() / (g.double().abs() + 1e-8)
    assert float((got[0][0].double() + first).abs().max()) < 1e-3 * 1e-4


def test_8bit_moments_follow_32bit_ones(hs):
    """300 steps with gradients of a fixed size and random sign: sqrt(v) stays at the 32-bit one's but for the
    rounding's noise.  Step k moves the root by 1 / 2k of itself at most and rounds it between neighbours at most 1/8
    apart: a relative variance of move times distance, 1 / 16k.  At the end, an error of step k counts k / T times, so
    the variance is at most sum (k / T)^2 / 16k = 1/32 (a standard deviation of 0.177); v takes the variance itself
    on, at most sum (k / T) / 16k = 1/16, its root half of that, less half the variance: -0.016 .. 0.032."""
    import torch
    n = 1 << 15
    out = {}
    for bits in (32, 8):
        gen = torch.Generator(device="cuda").manual_seed(3)
        W = torch.zeros(n, device="cuda")
        dt = torch.float32 if bits == 32 else torch.uint8
        m, v = (torch.zeros(n, dtype=dt, device="cuda") for _ in range(2))
        s = torch.zeros((n // 32, 2), dtype=torch.uint8, device="cuda") if bits == 8 else None
        g = torch.empty(n, device="cuda")
        p = hs.param_list([hs.param(W, g, m, v, s)])
        o = hs.adamw_opts(1e-3, seed=5)
        for k in range(300):
            g.copy_((torch.rand(n, device="cuda", generator=gen) < 0.5).float() * 2 - 1)
            o.step = k + 1
            hs.haste_adamw(p, o)
        torch.cuda.synchronize()
        out[bits] = v.sqrt() if bits == 32 else (v.view(torch.float8_e4m3fn).float()
                                                 * torch.exp2(s[:, 1].float() - 127).repeat_interleave(32))
    ratio = (out[8] / out[32]).double()
    say(f"    sqrt(v), 8 bits over 32: mean {float(ratio.mean()):.4f}, standard deviation {float(ratio.std()):.4f}")
    assert -0.017 < float(ratio.mean()) - 1 < 0.033 and float(ratio.std()) < 0.18


@pytest.mark.parametrize("bits", [32, 8])
def test_other_stream_and_repeat(hs, bits):
    import torch
    t = Tensors(hs, [70000, 33], "bf16", "bf16", bits)
    start = t.snapshot()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = _step(hs, t, OPTS, side)
    t.check(before, OPTS)
    first = t.snapshot()
    for k, v in t.arrays().items():
        v.copy_(start[k])
    _step(hs, t, OPTS)
    assert all(torch.equal(first[k], v) for k, v in t.arrays().items())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_norm_and_step_follow_device_options(hs, bits):
    """The norm's factor feeds the step inside one graph; the step's number is counted in it too."""
    import torch
    # more tensors than one launch takes
    t, e = (Tensors(hs, [3000, 17, 64] * 30, "bf16", "f32", bits, True) for _ in range(2))
    steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2)]
    lr = torch.full((1,), 1e-2, device="cuda")
    outs = [torch.zeros(2, device="cuda") for _ in range(2)]
    ws = [hs.workspace(hs.haste_grad_norm_workspace_bytes(x.params)) for x in (t, e)]
    opts = [hs.adamw_opts(0.0, seed=9, lr_dev=lr, step_dev=steps[j], grad_scale=outs[j][1:]) for j in range(2)]

    def run(j, x):
        steps[j].add_(1)
        hs.haste_grad_norm(x.params, 0.5, outs[j], ws[j])
        hs.haste_adamw(x.params, opts[j])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(0, t)
    for k in range(4):
        g = torch.randn_like(t.grad)
        if k == 2:
            g[t.at[1]] = float("inf")            # this step is passed over
        t.grad.copy_(g)
        e.grad.copy_(g)
        lr.mul_(0.7)
        graph.replay()
        before = e.snapshot()
        run(1, e)
        torch.cuda.synchronize()
        assert int(steps[0]) == k + 1
        assert all(torch.equal(a, b) for a, b in zip(t.arrays().values(), e.arrays().values())), f"replay {k}"
        assert torch.equal(torch.nan_to_num(outs[0], 5.0), torch.nan_to_num(outs[1], 5.0))
        if k == 2:
            assert all(torch.equal(before[n], v) for n, v in e.arrays().items())
        else:
            e.check(before, dict(OPTS, lr=float(lr), step=k + 1, seed=9), gs=float(outs[1][1]))


# ---- the norm ---------------------------------------------------------------------------------
def _norm(hs, grads, max_norm, stream=None):
    import torch
    p = hs.param_list([hs.param(grad=g) for g in grads])
    out = torch.full((2,), -1.0, device="cuda")
    ws = hs.workspace(hs.haste_grad_norm_workspace_bytes(p))
    torch.cuda.synchronize()                     # the call may go to another stream
    hs.haste_grad_norm(p, max_norm, out, ws, stream)
    torch.cuda.synchronize()
    return [float(x) for x in out.cpu()]


@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [8191, 8192, 8193], [100003, 1], [1 + 53 * k % 999 for k in range(150)],
                                   [1 + 71 * k % 501 for k in range(400)],
                                   [3_000_001, 70_000], [255, 256, 257, 1023, 1025, 16385, 32769, 65537]])
@pytest.mark.parametrize("dt", ["f32", "bf16", "both"])
def test_norm(hs, sizes, dt):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "both": [torch.float32, torch.bfloat16]}[dt]
    grads = [torch.randn(n, device="cuda", generator=gen).to(kinds[k % len(kinds)]) for k, n in enumerate(sizes)]
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    for max_norm in (1.0, 1e9, float("inf")):
        norm, factor = _norm(hs, grads, max_norm)
        say(f"    norm {norm}, factor {factor}, want {want}")
        assert abs(norm - want) <= 1.01 * U * want
        scale = min(1.0, max_norm / want)
        assert abs(factor - scale) <= 1.01 * U * scale
    assert _norm(hs, grads, 1.0) == _norm(hs, grads, 1.0)


def test_norm_of_nothing_of_large_and_of_not_finite_values(hs):
    import torch
    assert _norm(hs, [], 1.0) == [0.0, 1.0]
    assert _norm(hs, [torch.zeros(0, device="cuda")], 1.0) == [0.0, 1.0]
    assert _norm(hs, [torch.zeros(77, device="cuda")], 1.0) == [0.0, 1.0]
    n, f = _norm(hs, [torch.full((1000,), 1e30, device="cuda")], 1.0)      # squares beyond fp32
    assert abs(n / (1e30 * math.sqrt(1000)) - 1) < 4 * U and f > 0
    n, f = _norm(hs, [torch.full((1000,), 3e38, device="cuda")], 1e10)     # the norm beyond fp32, its factor not
    assert n == math.inf and abs(f / (1e10 / (3e38 * math.sqrt(1000))) - 1) < 4 * U
    n, f = _norm(hs, [torch.full((1000,), 1e-40, device="cuda")], 1.0)     # squares below fp32
    assert abs(n / (float(np.float32(1e-40)) * math.sqrt(1000)) - 1) < 1e-6 and f == 1.0
    for bad in (float("inf"), float("-inf"), float("nan")):
        for dt in (torch.float32, torch.bfloat16):
            g = torch.ones(20000, device="cuda", dtype=dt)
            g[19999] = bad
            n, f = _norm(hs, [g], 1.0)
            assert not math.isfinite(n) and math.isnan(f)


def test_norm_reads_the_list_alone_and_on_another_stream(hs):
    import torch
    big = torch.full((4096,), float("nan"), device="cuda")
    big[64:64 + 1001] = 2.0
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    n, f = _norm(hs, [big[64:64 + 1001]], 1.0, side)
    assert abs(n - 2 * math.sqrt(1001)) <= 1.01 * U * n


def test_binding_refuses(hs):
    import torch
    x = torch.zeros(100, device="cuda")
    b = torch.zeros(100, dtype=torch.uint8, device="cuda")
    for bad in (lambda: hs.param(x, x[:99], x, x), lambda: hs.param(x, x.half(), x, x), lambda: hs.param(x, x, b, x),
                lambda: hs.param(x, x, b, b), lambda: hs.param(x, x, b, b, b[:6]), lambda: hs.param(x, x, x.bfloat16(), x),
                lambda: hs.param(x.bfloat16(), x, x, x, W32=x.bfloat16()), lambda: hs.param(x[::2], x[:50], x[:50], x[:50])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(hs.HasteError, match="twice"):
        hs.haste_adamw(hs.param_list([hs.param(x, x.clone(), x.clone(), x)]), hs.adamw_opts(1e-3))
    with pytest.raises(hs.HasteError, match="aligned"):
        hs.haste_adamw(hs.param_list([hs.param(x[1:], x[1:].clone(), x[1:].clone(), x[1:].clone())]), hs.adamw_opts(1e-3))
