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
