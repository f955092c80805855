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
@pytest.mark.parametrize("B,F", [(512, 3040), (512, 3073), (512, 4096), (512, 4097), (300, 7168), (180, 7168), (160, 8192),
                                 (161, 8192), (17, 8192), (80, 16384), (130, 12289), (512, 16384), (513, 768), (512, 1)])
@pytest.mark.parametrize("h,x", [("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_few_rows(hs, B, F, h, x):
    _both(hs, B, F, h, x)


# 64 KB of LDS: 64 teams of a row of up to 256 values, 16 of a row of up to 1024
@pytest.mark.parametrize("B,F", [(32769, 256), (40001, 193), (8193, 1024), (9001, 1001), (32768, 256), (8192, 1024)])
@pytest.mark.parametrize("h,x", [("bf16", "f32"), ("f32", "bf16")])
def test_workgroups_that_add_up_the_most_teams(hs, B, F, h, x):
    _both(hs, B, F, h, x)


@pytest.mark.parametrize("F", [3, 64, 768, 3000, 9001, 16385])
def test_rows_beyond_the_range_of_their_squares(hs, F):
    """Differences from the mean of 2^64 and more have squares beyond fp32: rstd is 0 and X the bias.  A sum beyond fp32
    makes its row NaN.  Neither reaches another row, nor dH of theirs."""
    import torch
    c = Case(4, F, "f32", "f32")
    c.H[1] = 0.0
    c.H[1, 0] = 2.0 ** 100                       # its sum, mean and difference are exact powers or near
    c.H[2] = 3e38
    X, mean, rstd = c.forward(hs)
    assert float(rstd[1]) == 0.0 and torch.equal(X[1], c.b)
    assert bool(torch.isnan(X[2]).all())
    out, mu, rs, tx, tm, tr = c.reference()
    for k in (0, 3):
        assert (abs(X[k].cpu().numpy() - out[k]) <= tx[k]).all()
    dH = c.backward(hs, mean, rstd, dw=None, db=None)[0]
    assert bool((dH[1] == 0).all()) and bool(torch.isfinite(dH[[0, 3]]).all())


@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("B,F,rows", [(20001, 131, 1), (9001, 768, 1), (8999, 769, 2), (3000, 2050, 1), (2500, 4096, 1),
                                      (700, 9001, 1), (600, 16000, 1), (3000, 20001, 1)])
def test_in_place_over_many_rows(hs, h, B, F, rows):
    """Teams of several rows, each asked for before the one in front of it is stored."""
    import torch
    c = Case(B, F, h, h, rows=rows)
    X, mean, rstd = c.forward(hs)
    few = c.backward(hs, mean, rstd)
    d = c.dX.clone()
    got = c.backward(hs, mean, rstd, dH=d, dX=d)
    assert all(torch.equal(a, b) for a, b in zip(few, got))
    between = c.store.clone()
    c.forward(hs, X=c.H)
    assert torch.equal(c.H, X)
    c.H.copy_(between[:B * c.ld].view(B, c.ld)[:, :F])
    assert torch.equal(c.store, between), "what lies between the rows"


def test_two_graphs_share_a_workspace(hs):
    """Backward passes of more rows than one launch takes, captured one by one over the same workspace and replayed in
    turn, with eager calls over it in between."""
    import torch
    cases = [Case(2000, 768, "bf16", "f32"), Case(700, 1003, "f32", "bf16"), Case(9000, 100, "bf16", "bf16")]
    stats = [c.stats() for c in cases]
    ws = hs.workspace(max(hs.haste_layer_norm_workspace_bytes(c.B, c.F) for c in cases))
    outs = [c.backward(hs, *s, ws=ws) for c, s in zip(cases, stats)]
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for c, s, o in zip(cases, stats, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            c.backward(hs, *s, *o, ws=ws)
    for _ in range(3):
        for c in cases:
            c.dX.normal_()
        for g in (*graphs, graphs[0]):
            g.replay()
        torch.cuda.synchronize()
        for c, s, o in zip(cases, stats, outs):
            got = [t.clone() for t in o]
            for t in o:
                t.fill_(9.0)
            c.backward(hs, *s, *o, ws=ws)
            assert all(torch.equal(a, b) for a, b in zip(got, o))
