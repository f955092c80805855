"""A training step as a program makes it: layer norm of the encoder's first tokens, tail and head with the loss
gradient, the norm's backward pass, the norm of all gradients and the AdamW step; each call's outputs feed the next.

Against 64 bits: every stage's reference is computed from the values that stage really read, so each is held to its own
rounding (the layer's to the framework's measure, largest error over the largest value: 1e-5 in fp32, 2e-2 in bf16),
and the gradient at the encoder's output is held to the whole pass in 64 bits from the start.
"""
import numpy as np
import pytest

import oracle
import synth
import train_ref as ref
from gpu_helpers import TOL, host_f32, oracle_fwd_bce, out_tensor, rel_err, say, to_dev

pytestmark = pytest.mark.gpu
F32, BF16 = synth.DT_F32, synth.DT_BF16


@pytest.fixture(scope="module")
def hs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    import paper_2606_01117_amd as m
    return m


@pytest.fixture(scope="module")
def orc():
    return oracle.get()


class Step:
    """One model: buffers, parameter list, and the calls of a step."""

    def __init__(self, hs, dt, bits, B=48, T=3, F_s=256, L=2048, G=32, F_in=64, H=96, P=4, max_norm=0.5):
        import torch
        self.hs, self.dt, self.bits = hs, dt, bits
        self.B, self.F_s, self.L, self.H, self.max_norm, self.P = B, F_s, L, H, max_norm, P
        self.wl = synth.small("chain", B=B, F_s=F_s, L=L, G=G, F_in=F_in, H=H, dtype=dt, wid=950)
        self.desc = hs.make_desc(B, F_s, L, G, F_in, dt)
        gen = torch.Generator(device="cuda").manual_seed(7)
        td = torch.float32 if dt == F32 else torch.bfloat16
        self.tokens = torch.randn((B, T, F_s), device="cuda", generator=gen) * 2 + 0.5
        self.H_in = self.tokens[:, 0]
        self.idx = to_dev(synth.draw_idx(self.wl))
        self.pos, self.pos_h = (torch.randint(0, n, (B, P), device="cuda", dtype=torch.int32, generator=gen) for n in (L, H))
        w = lambda a: to_dev(a).view(td) if dt == BF16 else to_dev(a)
        self.p = {"weight": torch.ones(F_s, device="cuda"), "bias": torch.zeros(F_s, device="cuda"),
                  "W": w(synth.draw_W(self.wl)), "b": torch.zeros(L, device="cuda"),
                  "W_h": w(synth.draw_W_head(self.wl)), "b_h": torch.zeros(H, device="cuda")}
        self.g = {k: torch.zeros(v.shape, device="cuda") for k, v in self.p.items()}
        self.m, self.v, self.scale, made = {}, {}, {}, []
        for k, v in self.p.items():
            n = v.numel()
            eight = bits == 8 and n >= 4096
            st = lambda: torch.zeros(n, dtype=torch.uint8 if eight else torch.float32, device="cuda")
            self.m[k], self.v[k] = st(), st()
            self.scale[k] = torch.zeros(((n + 31) // 32, 2), dtype=torch.uint8, device="cuda") if eight else None
            made.append(hs.param(v, self.g[k], self.m[k], self.v[k], self.scale[k],
                                 weight_decay=0.01 if v.dim() == 2 else 0.0))
        self.names = list(self.p)
        self.params = hs.param_list(made)
        self.X, self.dY, self.dY_h = (torch.zeros(s, dtype=td, device="cuda") for s in ((B, F_s), (B, L), (B, H)))
        self.mean, self.rstd = (torch.zeros(B, device="cuda") for _ in range(2))
        self.dX, self.dH = (torch.zeros((B, F_s), device="cuda") for _ in range(2))
        self.norm, self.step = torch.zeros(2, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        self.opts = hs.adamw_opts(1e-2, seed=3, step_dev=self.step, grad_scale=self.norm[1:])
        wsn = hs.workspace
        self.ws = wsn(hs.haste_workspace_bytes(self.desc, hs.HASTE_OP_TAIL_STEP))
        self.ws_h = wsn(hs.haste_head_workspace_bytes(B, F_s, H, dt))
        self.ws_n = wsn(hs.haste_layer_norm_workspace_bytes(B, F_s))
        self.ws_g = wsn(hs.haste_grad_norm_workspace_bytes(self.params))

    def run(self):
        hs, p, g, B, F_s, H = self.hs, self.p, self.g, self.B, self.F_s, self.H
        hs.haste_layer_norm_fwd(B, F_s, F32, self.H_in, p["weight"], p["bias"], 1e-5, self.dt, self.X, self.mean, self.rstd)
        hs.haste_tail_step(self.desc, self.X, self.idx, p["W"], p["b"], self.pos, self.dY, g["W"], g["b"], 0, self.dX, 0,
                           self.ws)
        hs.haste_head_fwd_bce(B, F_s, H, self.dt, self.X, p["W_h"], p["b_h"], self.pos_h, self.dY_h)
        hs.haste_head_bwd(B, F_s, H, self.dt, self.X, p["W_h"], self.dY_h, g["W_h"], self.dX, 1, self.ws_h)
        g["b_h"].copy_(self.dY_h.float().sum(0))
        hs.haste_layer_norm_bwd(B, F_s, F32, self.H_in, p["weight"], self.mean, self.rstd, F32, self.dX, self.dH, g["weight"],
                                g["bias"], 0, self.ws_n)
        hs.haste_grad_norm(self.params, self.max_norm, self.norm, self.ws_g)
        self.step.add_(1)
        hs.haste_adamw(self.params, self.opts)

    def all(self):
        out = {"X": self.X, "dX": self.dX, "dH": self.dH, "norm": self.norm}
        for n in self.names:
            out |= {n: self.p[n], "g." + n: self.g[n], "m." + n: self.m[n], "v." + n: self.v[n]}
        return out


def _np(t):
    import torch
    t = t.detach()
    return (t.float() if t.is_floating_point() else t).cpu().numpy()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
def test_training_step(hs, orc, dt, bits):
    import torch
    s = Step(hs, dt, bits)
    for it in range(1, 4):
        old = {k: (_np(s.p[k]), _np(s.m[k]), _np(s.v[k]), None if s.scale[k] is None else _np(s.scale[k])) for k in s.names}
        raw = {k: s.p[k].clone() for k in ("W", "W_h")}
        s.run()
        torch.cuda.synchronize()
        say(f"[chain] dtype={dt} bits={bits} step {it}: gradient norm {float(s.norm[0]):.4f}, factor {float(s.norm[1]):.4f}")
        # layer norm
        h = _np(s.H_in).astype(np.float64)
        X, mean, rstd = ref.layer_norm(h, old["weight"][0].astype(np.float64), old["bias"][0].astype(np.float64), 1e-5)
        half = ref.U16 if dt == BF16 else ref.U32
        assert np.all(np.abs(_np(s.X) - X) <= np.abs(X) * half * 1.01 + 40 * ref.U32 * (1 + np.abs(X)))
        # the layer, on the features that it read
        bits_of = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16) if dt == BF16 else _np(t)
        Xs, Ws, Whs, idx = bits_of(s.X), bits_of(raw["W"]), bits_of(raw["W_h"]), s.idx.cpu().numpy()
        dY, dW, db = oracle_fwd_bce(orc, Xs, idx, Ws, old["b"][0], s.pos.cpu().numpy(), 32, 64, dt)
        zh = orc.head_fwd(Xs, Whs, old["b_h"][0], dt)
        dYh = orc.bce_grad(zh, s.pos_h.cpu().numpy())
        dYs, dYhs = bits_of(s.dY), bits_of(s.dY_h)
        dX = orc.bwd_x(idx, Ws, dYs, 32, s.F_s, dt) + orc.head_bwd_x(Whs, dYhs, dt)
        for name, got, want in (("dY", _np(s.dY), dY), ("dW", _np(s.g["W"]), dW), ("db", _np(s.g["b"]), db),
                                ("dY_h", _np(s.dY_h), dYh), ("dW_h", _np(s.g["W_h"]), orc.head_bwd_w(Xs, dYhs, dt)),
                                ("dX", _np(s.dX), dX)):
            e = rel_err(got, want)
            assert e <= TOL[dt], f"{name}: {e:.2e}"
        # the norm's backward pass, on the dX that it read; and on the whole pass's
        w = old["weight"][0]
        mu, rs = _np(s.mean).astype(np.float64)[:, None], _np(s.rstd).astype(np.float64)[:, None]
        for dx, tol in ((_np(s.dX), 1e-6), (dX, TOL[dt])):
            dH, dw, dbn = ref.layer_norm_grads(h, w, mu, rs, dx)
            for name, got, want in (("dH", s.dH, dH), ("dweight", s.g["weight"], dw), ("dbias", s.g["bias"], dbn)):
                e = rel_err(_np(got), want)
                assert e <= tol, f"{name}: {e:.2e} > {tol}"
        # norm and step, on the gradients that they read
        grads = {k: _np(s.g[k]).reshape(-1) for k in s.names}
        norm = np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads.values()))
        scale = min(1.0, s.max_norm / norm)
        assert abs(float(s.norm[0]) - norm) <= 1.01 * ref.U32 * norm and abs(float(s.norm[1]) - scale) <= 1.01 * ref.U32 * scale
        o = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=it, seed=3)
        for k, name in enumerate(s.names):
            pw, pm, pv, ps = old[name]
            new, move, m, v, sc = ref.adamw(pw.reshape(-1), grads[name], pm, pv, ps, o, k, 1.0,
                                            0.01 if s.p[name].dim() == 2 else 0.0, float(s.norm[1]))
            np.testing.assert_array_equal(_np(s.m[name]), m, err_msg=name)
            np.testing.assert_array_equal(_np(s.v[name]), v, err_msg=name)
            if sc is not None:
                np.testing.assert_array_equal(_np(s.scale[name]), sc, err_msg=name)
            hw = ref.U16 if s.p[name].dtype == torch.bfloat16 else ref.U32
            off = np.abs(_np(s.p[name]).reshape(-1) - new)
            assert np.all(off <= (8 * ref.U32 * move + 2 * ref.U32 * np.abs(new)) * (1 + hw) + hw * np.abs(new)), name


def test_captured_step_replays_as_eager(hs):
    """The whole step in one graph, replayed over changing inputs with the program's own work between the replays: every
    replay equals the eager step bit for bit, also where a step is passed over because a gradient is not finite."""
    import torch
    a, b = Step(hs, BF16, 8), Step(hs, BF16, 8)
    b.run()                                       # warm: every kernel has been loaded before the capture
    torch.cuda.synchronize()
    b = Step(hs, BF16, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for k in range(4):
        x = torch.randn_like(a.tokens)
        if k == 2:
            x[5, 0, 7] = float("inf")
        a.tokens.copy_(x)
        b.tokens.copy_(x)
        before = {n: a.p[n].clone() for n in a.names}
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for n, (u, v) in {n: (a.all()[n], b.all()[n]) for n in a.all()}.items():
            assert torch.equal(torch.nan_to_num(u.float(), 7.0), torch.nan_to_num(v.float(), 7.0)), f"replay {k}: {n}"
        same = all(torch.equal(before[n], a.p[n]) for n in a.names)
        assert same == (k == 2), f"replay {k}"


def test_step_goes_down_the_gradient(hs):
    """A step along AdamW's direction: the directional derivative of the loss along the change of the weights, from the
    step's own gradients, is negative."""
    import torch
    s = Step(hs, F32, 32)
    before = {n: s.p[n].clone() for n in s.names}
    s.run()
    torch.cuda.synchronize()
    slope = sum(float((s.g[n].double() * (s.p[n] - before[n]).double()).sum()) for n in s.names)
    assert slope < 0
