"""The layer norm on the GPU at the shapes where its kernels change and where they use most of a CU, against the 64-bit
formula with the tolerances of its other tests."""
import pytest

from gpu_helpers import say
from test_gpu_norm import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    import paper_2606_01117_amd as m
    return m


def _both(hs, B, F, h, x):
    say(f"[layer norm] B={B} F={F} {h} -> {x}")
    c = Case(B, F, h, x)
    c.check_forward(*c.forward(hs))
    mean, rstd = c.stats()
    c.check_backward(mean, rstd, *c.backward(hs, mean, rstd))


# in one launch and in two
@pytest.mark.parametrize("B,F", [(512, 3072), (512, 3073), (512, 4096), (512, 4097), (300, 7168), (180, 7168), (160, 8192),
                                 (161, 8192), (17, 8192), (80, 16384), (130, 12289), (512, 16384), (513, 768), (512, 1)])
@pytest.mark.parametrize("h,x", [("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_few_rows(hs, B, F, h, x):
    _both(hs, B, F, h, x)


# 64 KB of LDS: 64 teams of a row of up to 256 values, 16 of a row of up to 1024
@pytest.mark.parametrize("B,F", [(32769, 256), (40001, 193), (8193, 1024), (9001, 1001), (32768, 256), (8192, 1024)])
@pytest.mark.parametrize("h,x", [("bf16", "f32"), ("f32", "bf16")])
def test_workgroups_that_add_up_the_most_teams(hs, B, F, h, x):
    _both(hs, B, F, h, x)
