"""Host-side checks of the layer norm, gradient norm and AdamW entry points: what they refuse, before any
launch (no GPU needed), and the plain implementations that their GPU tests compare with."""
import ctypes

import numpy as np
import pytest

import train_ref as ref

FAKE = 1 << 20
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def hs():
    import paper_2606_01117_amd as m
    return m


def _fwd(hs, **kw):
    a = dict(B=4, F=8, dh=BF16, H=FAKE, ldh=8, w=FAKE, b=FAKE, eps=1e-5, dx=BF16, X=2 * FAKE, ldx=8, mean=FAKE, rstd=FAKE)
    a.update(kw)
    return hs.lib.haste_layer_norm_fwd(a["B"], a["F"], a["dh"], a["H"], a["ldh"], a["w"], a["b"], a["eps"], a["dx"], a["X"],
                                       a["ldx"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("kw,what", [
    (dict(dh=2), "dtype"), (dict(dx=-1), "dtype"), (dict(B=-1), "B must"), (dict(B=1 << 31), "B must"),
    (dict(F=0), "F must"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(mean=None), "together"),
    (dict(rstd=None), "together"), (dict(H=None), "H is NULL"), (dict(X=None), "X is NULL"), (dict(H=FAKE + 1), "aligned"),
    (dict(dx=F32, X=FAKE + 2), "aligned"), (dict(w=FAKE + 4), "weight"), (dict(b=FAKE + 8), "bias"), (dict(ldh=7), "rows"),
    (dict(ldx=7), "rows"), (dict(X=FAKE, ldx=16), "place"), (dict(X=FAKE, dx=F32), "place"),
])
def test_layer_norm_fwd_refuses(hs, kw, what):
    assert _fwd(hs, **kw) == 1
    assert what in hs.haste_last_error()


def test_layer_norm_width_limit(hs):
    n = (1 << 24) + 1
    assert _fwd(hs, F=n, ldh=n, ldx=n) == 2 and "2^24" in hs.haste_last_error()
    assert _bwd(hs, F=n, ldh=n, lddx=n, lddh=n) == 2
    assert hs.haste_layer_norm_workspace_bytes(4, n) == 0


def _bwd(hs, **kw):
    a = dict(B=4, F=8, dh=F32, H=FAKE, ldh=8, w=FAKE, mean=FAKE, rstd=FAKE, dd=F32, dX=2 * FAKE, lddx=8, dH=3 * FAKE, lddh=8,
             dw=FAKE, db=2 * FAKE, beta=0, ws=FAKE, n=1 << 30)
    a.update(kw)
    return hs.lib.haste_layer_norm_bwd(a["B"], a["F"], a["dh"], a["H"], a["ldh"], a["w"], a["mean"], a["rstd"], a["dd"],
                                       a["dX"], a["lddx"], a["dH"], a["lddh"], a["dw"], a["db"], a["beta"], a["ws"], a["n"],
                                       None)


@pytest.mark.parametrize("kw,code,what", [
    (dict(dd=7), 1, "dtype"), (dict(F=0), 1, "F must"), (dict(beta=2), 1, "beta"), (dict(H=None), 1, "H is NULL"),
    (dict(dX=None), 1, "dX is NULL"), (dict(mean=None), 1, "mean"), (dict(rstd=None), 1, "rstd"), (dict(lddx=5), 1, "rows"),
    (dict(lddh=5), 1, "rows"), (dict(dH=3 * FAKE + 2), 1, "aligned"), (dict(dw=FAKE + 4), 1, "dweight"),
    (dict(db=FAKE + 4), 1, "dbias"), (dict(db=FAKE), 1, "same array"), (dict(dH=FAKE), 1, "H's place"),
    (dict(dH=2 * FAKE, lddh=16), 1, "place"), (dict(ws=None), 3, "workspace"), (dict(n=8), 3, "workspace"),
    (dict(ws=FAKE + 4), 1, "ws"),
])
def test_layer_norm_bwd_refuses(hs, kw, code, what):
    assert _bwd(hs, **kw) == code
    assert what in hs.haste_last_error()


def test_layer_norm_calls_that_have_nothing_to_do(hs):
    assert _fwd(hs, B=0, H=None, X=None) == 0
    assert _bwd(hs, dH=None, dw=None, db=None, H=None) == 0
    assert _bwd(hs, B=0, beta=1, H=None, dX=None) == 0
    assert hs.haste_layer_norm_workspace_bytes(0, 8) == 0
    assert hs.haste_layer_norm_workspace_bytes(4, 0) == 0
    assert hs.haste_layer_norm_workspace_bytes(4, 8) >= 2 * 8 * 4


def _list(hs, *kws):
    made = []
    for j, kw in enumerate(kws):
        a = dict(W=(8 * j + 1) * FAKE, grad=(8 * j + 2) * FAKE, m=(8 * j + 3) * FAKE, v=(8 * j + 4) * FAKE, n=64, lr_scale=1.0,
                 dtype=F32, grad_dtype=F32, state_bits=32)
        a.update(kw)
        made.append(hs.haste_param_t(**a))
    return (hs.haste_param_t * len(made))(*made)


def _adamw(hs, params, **kw):
    o = hs.adamw_opts(1e-3)
    for k, v in kw.items():
        setattr(o, k, v)
    return hs.lib.haste_adamw(params, len(params), ctypes.byref(o), None)


@pytest.mark.parametrize("kw,code,what", [
    (dict(n=-1), 1, "n must"), (dict(n=(1 << 33) + 1), 2, "2^33"), (dict(dtype=2), 1, "dtype"), (dict(grad_dtype=3), 1, "grad_dtype"),
    (dict(state_bits=16), 1, "state_bits"), (dict(state_bits=8), 1, "scale is NULL"),
    (dict(state_bits=8, scale=FAKE + 1), 1, "scale is not"), (dict(W32=7 * FAKE), 1, "W32"),
    (dict(W=None), 1, "W is NULL"), (dict(grad=None), 1, "grad is NULL"), (dict(m=FAKE + 4), 1, "m is not"),
    (dict(v=FAKE + 8), 1, "v is not"), (dict(grad=FAKE + 4), 1, "grad is not"), (dict(reserved=1), 1, "reserved"),
    (dict(lr_scale=float("inf")), 1, "lr_scale"), (dict(weight_decay=-0.1), 1, "weight_decay"),
    (dict(weight_decay=float("nan")), 1, "weight_decay"), (dict(m=9 * FAKE), 1, "twice"),
    (dict(v=FAKE), 1, "twice"),
])
def test_adamw_refuses_a_tensor(hs, kw, code, what):
    """As the second of two tensors, whose first has its weights at FAKE."""
    assert _adamw(hs, _list(hs, {}, kw)) == code
    assert what in hs.haste_last_error() and (what == "n_params" or "tensor 1" in hs.haste_last_error())


def test_adamw_refuses_the_same_weights_far_apart(hs):
    kws = [{} for _ in range(1500)]
    kws[1400] = dict(W=FAKE)                       # the first tensor's
    assert _adamw(hs, _list(hs, *kws)) == 1
    assert "tensor 1400" in hs.haste_last_error()
    kws[1400] = dict(W=None, n=0)                  # an empty tensor's arrays are not looked at; the last one's gradient is not there
    kws[1499] = dict(grad=None)
    assert _adamw(hs, _list(hs, *kws)) == 1
    assert "tensor 1499: grad" in hs.haste_last_error()


@pytest.mark.parametrize("kw,what", [
    (dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"), (dict(lr=float("inf")), "lr"), (dict(beta1=1.0), "beta"),
    (dict(beta2=-0.1), "beta"), (dict(beta2=float("nan")), "beta"), (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"),
    (dict(step=0), "step"), (dict(lr_dev=FAKE + 2), "lr_dev"), (dict(step_dev=FAKE + 4), "step_dev"),
    (dict(grad_scale=FAKE + 1), "grad_scale"),
])
def test_adamw_refuses_options(hs, kw, what):
    assert _adamw(hs, _list(hs, {}), **kw) == 1
    assert what in hs.haste_last_error()


def test_adamw_and_norm_refuse_lists(hs):
    o = hs.adamw_opts(1e-3)
    one = _list(hs, {})
    assert hs.lib.haste_adamw(None, 1, ctypes.byref(o), None) == 1
    assert hs.lib.haste_adamw(one, -1, ctypes.byref(o), None) == 1
    assert hs.lib.haste_adamw(one, (1 << 16) + 1, ctypes.byref(o), None) == 2
    assert hs.lib.haste_adamw(one, 1, None, None) == 1
    assert hs.lib.haste_adamw(None, 0, ctypes.byref(o), None) == 0
    need = hs.haste_grad_norm_workspace_bytes(one)
    assert need > 0
    norm = hs.lib.haste_grad_norm
    assert norm(one, 1, 0.0, FAKE, FAKE, need, None) == 1 and "max_norm" in hs.haste_last_error()
    assert norm(one, 1, float("nan"), FAKE, FAKE, need, None) == 1
    assert norm(one, 1, 1.0, None, FAKE, need, None) == 1 and "out" in hs.haste_last_error()
    assert norm(one, 1, 1.0, FAKE + 2, FAKE, need, None) == 1
    assert norm(one, 1, 1.0, FAKE, None, 0, None) == 3
    assert norm(one, 1, 1.0, FAKE, FAKE, need - 1, None) == 3 and str(need) in hs.haste_last_error()
    assert norm(_list(hs, dict(grad=None)), 1, 1.0, FAKE, FAKE, need, None) == 1 and "grad" in hs.haste_last_error()
    assert norm(_list(hs, dict(grad_dtype=5)), 1, 1.0, FAKE, FAKE, need, None) == 1
    assert hs.haste_grad_norm_workspace_bytes(_list(hs, dict(n=-5))) == 0


def test_binding_refuses_host_tensors(hs):
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        hs.haste_layer_norm_fwd(4, 8, F32, x, None, None, 1e-5, F32, x)
    with pytest.raises(ValueError, match=r"\[4, 9\]"):
        hs.haste_layer_norm_fwd(4, 9, F32, x, None, None, 1e-5, F32, x)
    for bad in (torch.float16, torch.float64, torch.bfloat16):
        with pytest.raises(ValueError, match="dtype"):
            hs.haste_layer_norm_fwd(4, 8, F32 if bad == torch.bfloat16 else BF16, x.to(bad), None, None, 1e-5, F32, x)
    with pytest.raises(ValueError, match="next to each other"):
        hs.haste_layer_norm_fwd(8, 4, F32, x.t(), None, None, 1e-5, F32, x)
    with pytest.raises(ValueError, match="overlap"):
        hs.haste_layer_norm_fwd(4, 8, F32, torch.zeros(8).expand(4, 8), None, None, 1e-5, F32, x)
    with pytest.raises(ValueError, match="GPU"):
        hs.param(grad=x)
    with pytest.raises(ValueError, match="must be one value"):
        hs.adamw_opts(1e-3, step_dev=torch.zeros(1))


# ---- the plain implementations -----------------------------------------------------------------------
def test_e4m3_values():
    import torch
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.e4m3(code), want)


def test_plain_store_keeps_what_is_exact_and_rounds_both_ways():
    rng = np.random.default_rng(1)
    code = rng.integers(0, 120, 32 * 50).astype(np.uint8)
    code[::32] = 112 + rng.integers(0, 8, 50)              # the block's largest in [128, 256)
    code[np.arange(0, 32 * 50, 7)] |= 128
    exps = rng.integers(30, 200, 50)
    x = (ref.e4m3(code) * np.repeat(2.0 ** (exps - 127.0), 32)).astype(np.float32)
    for d in (0, 1, 40000, 65535):
        q, s = ref._store(x, np.full(len(x), d), False)
        np.testing.assert_array_equal(s, exps)
        np.testing.assert_array_equal(ref.e4m3(q), ref.e4m3(code))
    # a value 0.3 of the way between two: up for the largest 0.3 of the draws
    x = np.full(32, 128 + 0.3 * 16, np.float32)
    d = np.arange(0, 65536, 2048)
    q, _ = ref._store(x, d, False)
    assert np.array_equal(ref.e4m3(q), np.where(d / 65536 >= 0.7 - 1e-6, 144, 128))
    # nothing but what is above zero is kept above it
    q, _ = ref._store(np.array([1.0, 1e-30, 0.0], np.float32), np.zeros(3, int), True)
    assert list(q[1:]) == [1, 0]


def test_plain_adamw_first_step_is_the_sign_of_the_gradient():
    """Without decay and with a small eps, the first step from zero moments moves by lr against each sign."""
    g = np.array([3.0, -2e-3, 0.5, -7.0], np.float32)
    o = dict(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-12, step=1, seed=3)
    w, _, m, v, _ = ref.adamw(np.zeros(4, np.float32), g, np.zeros(4, np.float32), np.zeros(4, np.float32), None, o)
    np.testing.assert_allclose(w, -0.1 * np.sign(g), rtol=1e-5)
    np.testing.assert_allclose(m, 0.1 * g, rtol=1e-6)


def test_plain_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(2)
    h, w, b, dx = rng.standard_normal((3, 17)), rng.standard_normal(17), rng.standard_normal(17), rng.standard_normal((3, 17))
    _, mean, rstd = ref.layer_norm(h, w, b, 1e-5)
    dh, dw, db = ref.layer_norm_grads(h, w, mean, rstd, dx)
    f = lambda h, w, b: float((ref.layer_norm(h, w, b, 1e-5)[0] * dx).sum())
    for a, grad, at in ((h, dh, 0), (w, dw, 1), (b, db, 2)):
        for _ in range(3):
            e = rng.standard_normal(a.shape) * 1e-5
            args = lambda s: [x + s * e if j == at else x for j, x in enumerate((h, w, b))]
            np.testing.assert_allclose((f(*args(1)) - f(*args(-1))) / 2, float((grad * e).sum()), rtol=1e-6, atol=1e-11)
