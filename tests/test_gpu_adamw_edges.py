"""The gradient norm and the AdamW step on the GPU where the other tests do not go: lists that change, lists on both
sides of the sizes at which the kernels change, values at the ends of their range, and long runs."""
import math

import numpy as np
import pytest

import train_ref as ref
from gpu_helpers import say
from test_gpu_adamw import OPTS, Tensors, U, _norm, _np, _step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    import paper_2606_01117_amd as m
    return m


@pytest.mark.parametrize("bits", [32, 8])
def test_new_gradients_every_step(hs, bits):
    """A list that is pointed at new gradients, fp32 and then bf16, does what a new list of them does; the old gradients
    may be overwritten by then."""
    import torch
    a, b = (Tensors(hs, [1000, 33, 5], "f32", "f32", bits) for _ in range(2))
    old = a.grad
    norms = torch.zeros((2, 2), device="cuda")
    for step, dt in ((1, torch.float32), (2, torch.bfloat16)):
        gen = torch.Generator(device="cuda").manual_seed(step)
        grads = [torch.randn(n, device="cuda", generator=gen).to(dt) for n in a.sizes]
        hs.set_grads(a.params, grads)
        entries = [hs.param(*(b.params[k].keep[j] if j != 1 else g for j in range(5)), lr_scale=b.lr_scale[k],
                            weight_decay=b.decay[k]) for k, g in enumerate(grads)]
        old.fill_(float("nan"))
        for row, params in enumerate((a.params, hs.param_list(entries))):
            hs.haste_grad_norm(params, 1.0, norms[row], hs.workspace(hs.haste_grad_norm_workspace_bytes(params)))
            hs.haste_adamw(params, hs.adamw_opts(**dict(OPTS, step=step), grad_scale=norms[row][1:]))
        torch.cuda.synchronize()
        assert torch.equal(norms[0], norms[1]) and bool(torch.isfinite(norms).all())
        assert all(torch.equal(x, y) for x, y in zip(a.arrays().values(), b.arrays().values()))
    with pytest.raises(ValueError, match="is on cpu"):
        hs.set_grads(a.params, [torch.zeros(1000), None, None])


def test_8bit_second_moments_settle_where_the_rounding_puts_them(hs):
    """6000 steps of normally distributed gradients from v = sigma^2, sigma over 12 binades of each block.

    A step moves the root by (c / 2) (g^2 - v) / r, c = 1 - beta2, and rounds it between neighbours D apart, with a
    variance of |move| D less the move's square.  v takes that on and forgets c of it a step, so it settles above
    sigma^2 by E|g^2 - v| / 2v times D / r, which is between 1/16 and 1/8 (no root is below 2^-13 of its block's
    largest).  E|x^2 - 1| is 0.968 for a normal x, and 1.01 where v varies by 0.3 around 1.05; the squares take c / 4
    E(x^2 - 1)^2 = 0.0005 off.  So 0.0298 .. 0.0632, and 0.003 for five standard errors of the mean.
    The root's own deviation decays by 1 - c a step: a variance of 0.968 / 4 D / r, a standard deviation of 0.123 .. 0.174,
    v's twice that and a little for its curvature: 0.24 .. 0.37."""
    import torch
    n = 1 << 18
    gen = torch.Generator(device="cuda").manual_seed(11)
    sigma = torch.exp2(-12 * torch.rand(n, device="cuda", generator=gen))
    sigma[::32] = 1.0
    host = sigma.cpu().numpy()
    q, s = ref._store(host, np.random.default_rng(12).integers(0, 65536, n), True)
    got = {}
    grad, W = torch.empty(n, device="cuda"), torch.zeros(n, device="cuda")
    m8, v8, scale = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.from_numpy(q).cuda(), torch.zeros((n // 32, 2), dtype=torch.uint8, device="cuda")
    scale[:, 1] = torch.from_numpy(s).cuda()
    m32, v32 = torch.zeros(n, device="cuda"), sigma ** 2
    lists = [hs.param_list([hs.param(W, grad, m8, v8, scale)]), hs.param_list([hs.param(W.clone(), grad, m32, v32)])]
    opts = hs.adamw_opts(1e-3, seed=13)
    for k in range(6000):
        torch.randn(n, device="cuda", generator=gen, out=grad)
        grad.mul_(sigma)
        opts.step = 1000 + k
        for p in lists:
            hs.haste_adamw(p, opts)
    r = v8.view(torch.float8_e4m3fn).double() * torch.exp2(scale[:, 1].double() - 127).repeat_interleave(32)
    ratio = (r / sigma.double()) ** 2
    bias = float(ratio.mean() / (v32.double() / sigma.double() ** 2).mean()) - 1
    say(f"    v, 8 bits over 32: {bias:+.4f}, varies by {float(ratio.std()):.4f}")
    assert 0.0268 < bias < 0.0662 and 0.24 < float(ratio.std()) < 0.37


@pytest.mark.parametrize("bits", [32, 8])
def test_finite_gradients_whose_squares_overflow(hs, bits):
    """(c2 g) g beyond fp32, from |g| = 5.8e20 at beta2 = 0.999 on: v is an infinity.  In 32 bits the weight moves by
    its decay alone from then on; in 8 bits v is stored as a NaN, and the next step's weight is one.  Neither
    reaches its neighbours, and just below the overflow nothing of the kind happens."""
    import torch
    t = Tensors(hs, [96], "f32", "f32", bits, decay=[0.0])
    a = t.at[0]
    t.grad[a + 40], t.grad[a + 90] = 6.0e20, 5.0e20
    before = _step(hs, t, OPTS)
    W = t.W[a:a + 96].clone()
    assert bool(torch.isfinite(W).all()) and float(W[40]) == float(before["W"][a + 40])
    if bits == 8:
        assert int(t.v[a + 40]) == 0x7f and bool((t.m[a:a + 96] & 0x7f != 0x7f).all())
    else:
        assert math.isinf(float(t.v[a + 40])) and math.isfinite(float(t.v[a + 90]))
    t.grad[a + 40] = t.grad[a + 90] = 1.0
    for step in (8, 9, 10):
        _step(hs, t, dict(OPTS, step=step))
    now = t.W[a:a + 96]
    others = torch.arange(96, device="cuda") != 40
    assert bool(torch.isfinite(now[others]).all())
    assert math.isnan(float(now[40])) if bits == 8 else float(now[40]) == float(W[40])


def _over_roots(hs, v, slow=None):
    """1 / sqrt(v / 2) as the step forms it, for each v: m = 1 over the root in the update of a weight of zero.  slow:
    the value of that number in each run of 256, a wave's, is one that sends its wave to the C library's sqrtf."""
    import torch
    v = v.clone()
    if slow is not None:
        v[slow::256] = 2.0 ** -99
    W, grad, m = torch.zeros_like(v), torch.zeros_like(v), torch.full_like(v, 2.0)
    hs.haste_adamw(hs.param_list([hs.param(W, grad, m, v)]), hs.adamw_opts(1.0, 0.5, 0.5, 1.2e-38, step=10000))
    return W.neg_()


@pytest.mark.parametrize("name,lo,count", [("all of [1, 4)", 2.0, 1 << 24), ("from 2^-90", 2.0 ** -89, 1 << 20),
                                           ("from 2^126", 2.0 ** 127, 1 << 23)])
def test_roots_are_those_of_sqrtf(hs, name, lo, count):
    """Every fp32 value of two binades, the lowest ones of the range that the short way takes, and the largest ones that
    half of a finite v can be: the same bits as from sqrtf, which rounds correctly.  A root that were one unit off
    would show in its reciprocal always up to root 1.41 and every other time up to 2."""
    import torch
    start = int(np.float32(lo).view(np.int32))
    v = torch.arange(start, start + count, dtype=torch.int32, device="cuda").view(torch.float32)
    short = _over_roots(hs, v)
    assert bool(torch.isfinite(v).all()) and int(v.numel()) % 256 == 0
    for slow in (0, 1):
        same = short.view(torch.int32) == _over_roots(hs, v, slow).view(torch.int32)
        same[slow::256] = True
        assert bool(same.all()), f"{int((~same).sum())} of {count}, the first for v = {float(v[~same][0]) / 2!r}"
    # and what they are: the reciprocal is the hardware's, to one unit
    want = 1 / (v.double() / 2).sqrt()
    assert float(((short.double() - want).abs() / want).max()) <= 2.5 * 2.0 ** -23


# lists of up to 2^22 values and of more take chunks of 4096 and of 16384 values; a round of loads takes 4096 fp32 or 8192 bf16
@pytest.mark.parametrize("sizes", [[4194305, 16383, 8191, 8193], [16384 + 4096 + 8, 4 << 20, 7, 2047, 12289],
                                   [4095, 4096, 4097, 8, 9, 7, 1], [2048, 2049, 2055, 2056, 1023, 6150, 3, 4104]])
@pytest.mark.parametrize("dt", ["f32", "bf16", "both"])
def test_norm_counts_every_value_once(hs, sizes, dt):
    """Random values to rounding, and ones at a few hundred places, the ends of chunks, rounds and loads among them: one
    that were left out or read twice would move the norm by a thousandth."""
    import torch
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "both": [torch.float32, torch.bfloat16]}[dt]
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    grads = [torch.randn(n, device="cuda", generator=gen).to(kinds[k % len(kinds)]) for k, n in enumerate(sizes)]
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    norm, factor = _norm(hs, grads, 1.0)
    assert abs(norm - want) <= 1.01 * U * want and abs(factor * want - 1) <= 1.01 * U
    rng = np.random.default_rng(sum(sizes))
    edges = [e + j for e in range(0, max(sizes) + 1, 1024) for j in (-8, -5, -4, -1, 0, 3, 4, 7)]
    for _ in range(4):
        total = 0
        for g, n in zip(grads, sizes):
            at = [int(x) for x in rng.integers(0, n, 40)] + [0, n - 1, max(0, n - 4), max(0, n - 9), n // 8 * 8 - 1, n // 4 * 4 - 1]
            at += [int(x) for x in rng.choice(edges, 60)]
            at = sorted({p for p in at if 0 <= p < n})
            g.zero_()
            g[torch.tensor(at, device="cuda")] = 1.0
            total += len(at)
        norm, _ = _norm(hs, grads, math.inf)
        assert norm == float(np.float32(math.sqrt(total))), (norm ** 2, total)


KINDS = [("f32", "f32", 32, False), ("bf16", "f32", 32, True), ("bf16", "bf16", 32, False), ("bf16", "bf16", 8, False),
         ("f32", "f32", 8, False), ("bf16", "f32", 8, True)]


@pytest.mark.parametrize("w,g,bits,master", KINDS)
def test_step_of_lists_beyond_two_million_values(hs, w, g, bits, master):
    """Lists of more than 2^21 values a launch take whole chunks of 1024 values a workgroup, a lane's second run among
    them, with the weights through the caches: ragged tensors, partial last blocks, against the plain form."""
    t = Tensors(hs, [1_000_003, 1024, 1023, 31, 1_300_001, 1025 + 512, 33], w, g, bits, master)
    for step in (1, 500):
        o = dict(OPTS, step=step)
        t.check(_step(hs, t, o), o)


@pytest.mark.parametrize("w,g,bits,master", KINDS)
def test_the_same_bits_on_both_sides_of_a_chunks_size(hs, w, g, bits, master):
    """2^21 values a launch are the last in chunks of 512, one value more makes them 1024: the tensors in front come out
    the same."""
    import torch
    n = 1 << 21
    front = [5000, 2048 + 512 + 33, 1]
    got = []
    for rest in (n - sum(front), n - sum(front) + 1):
        t = Tensors(hs, front, w, g, bits, master, edge=True)
        last = Tensors(hs, [rest], "bf16", "bf16", 8, seed=1)
        hs.haste_adamw(hs.param_list([*t.params, last.params[0]]), hs.adamw_opts(**OPTS))
        torch.cuda.synchronize()
        got.append(t.snapshot())
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])
    before = Tensors(hs, front, w, g, bits, master, edge=True)
    t.check(before.snapshot(), OPTS)
