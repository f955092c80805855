"""The binding's lists of tensors: what they keep alive, and what they and the calls refuse (no GPU needed)."""
import gc
import weakref

import pytest


@pytest.fixture(scope="module")
def hs():
    import paper_2606_01117_amd as m
    return m


class Thing:
    """In a tensor's place, where only its life counts."""


def _entry(hs, n=1, device=0):
    p = hs.haste_param_t(n=n)
    thing = Thing()
    p.keep, p.device = (thing,), device
    return p, weakref.ref(thing)


def test_entries_taken_out_of_a_list_keep_their_tensors(hs):
    (a, ra), (b, rb) = _entry(hs, 5), _entry(hs, 7)
    first = hs.param_list([a, b])
    second = hs.param_list([first[1], *first[:1]])
    del a, b, first
    gc.collect()
    assert [p.n for p in second] == [7, 5]
    assert ra() is not None and rb() is not None
    del second
    gc.collect()
    assert ra() is None and rb() is None


def test_an_entry_put_into_a_list_takes_its_tensors_along(hs):
    (a, ra), (b, rb) = _entry(hs, 5), _entry(hs, 7)
    params = hs.param_list([a])
    params[0] = b
    del a, b
    gc.collect()
    assert params[0].n == 7 and params[-1].n == 7 and rb() is not None
    assert ra() is None, "nothing names it any more"
    with pytest.raises(TypeError):
        params[:] = [params[0]]


def test_lists_know_their_device_wherever_their_entries_come_from(hs):
    here, there = hs.param_list([_entry(hs, device=0)[0]]), hs.param_list([_entry(hs, device=1)[0]])
    assert (here.device, there.device) == (0, 1)
    assert hs.param_list(there[:]).device == 1
    with pytest.raises(ValueError, match="one GPU"):
        hs.param_list([here[0], there[0]])
    with pytest.raises(ValueError, match="one GPU"):
        here[0] = there[0]
    empty = hs.param_list([hs.haste_param_t(n=0), here[0]])
    assert empty.device == 0 and empty[0].device is None
    assert len(hs.param_list([])) == 0


def test_an_entry_written_in_place_is_the_lists(hs):
    params = hs.param_list([hs.haste_param_t(n=3), hs.haste_param_t(n=4)])
    params[1].weight_decay = 0.25
    assert params[1].weight_decay == 0.25 and [p.n for p in params] == [3, 4]
    assert hs.haste_grad_norm_workspace_bytes(params) > 0


# ---- new gradients ------------------------------------------------------------------------------------
@pytest.fixture
def on_host(hs, monkeypatch):
    """Lets the binding make lists of host tensors, for what it checks and keeps itself (their device is -1)."""
    monkeypatch.setattr(hs, "_here", lambda t, name: t.get_device())


def _host_list(hs, sizes=(5, 8), bits=32):
    import torch
    return hs.param_list([hs.param(torch.zeros(n), torch.ones(n), torch.zeros(n), torch.zeros(n)) for n in sizes])


def test_new_gradients_are_kept_and_the_old_ones_let_go(hs, on_host):
    import torch
    params = _host_list(hs)
    old, weights = [weakref.ref(p.keep[1]) for p in params], [p.W for p in params]
    fresh = torch.full((2, 4), 2.0).bfloat16()
    new = weakref.ref(fresh)
    hs.set_grads(params, [None, fresh])
    assert params[1].grad == fresh.data_ptr() and params[1].grad_dtype == hs.HASTE_DTYPE_BF16
    assert params[0].grad_dtype == hs.HASTE_DTYPE_F32 and params[0].grad == old[0]().data_ptr()
    del fresh
    gc.collect()
    assert new() is not None and old[0]() is not None and old[1]() is None
    assert [p.W for p in params] == weights and all(t is not None for p in params for t in p.keep[:4])


def test_new_gradients_that_do_not_fit_change_nothing(hs, on_host):
    import torch
    params = _host_list(hs)
    before = [(p.grad, p.grad_dtype) for p in params]
    good = torch.ones(5)
    for bad, what in ((torch.ones(9), "8 contiguous"), (torch.ones(8, 2)[:, 0], "8 contiguous"), (torch.ones(8).half(), "float32")):
        with pytest.raises(ValueError, match=what):
            hs.set_grads(params, [good, bad])
    params.device = 0                            # a list on a GPU takes no host tensor
    with pytest.raises(ValueError, match="is on cpu, the list on cuda:0"):
        hs.set_grads(params, [good, None])
    with pytest.raises(ValueError, match="1 gradients for a list of 2"):
        hs.set_grads(params, [good])
    assert [(p.grad, p.grad_dtype) for p in params] == before


def test_new_gradients_for_entries_without_tensors(hs, on_host):
    import torch
    params = hs.param_list([hs.haste_param_t(n=4)])
    g = torch.ones(4)
    hs.set_grads(params, [g])
    assert params[0].grad == g.data_ptr() and params[0].keep[1] is g and params.device == -1


# ---- entries ------------------------------------------------------------------------------------------
def test_moments_of_other_8_bit_types_are_refused(hs, on_host):
    """Those of E4M3 without negative zero and of E5M2, and truth values, would be taken for other values."""
    import torch
    x, q, s = torch.zeros(64), torch.zeros(64, dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    for good in (torch.uint8, torch.int8, torch.float8_e4m3fn):
        for exponents in (torch.uint8, torch.int8, torch.float8_e8m0fnu):
            assert hs.param(x, x, q.view(good), q.view(good), s.view(exponents)).state_bits == 8
    for bad in (torch.float8_e4m3fnuz, torch.float8_e5m2, torch.float8_e5m2fnuz, torch.bool):
        for m, v in ((q.view(bad), q), (q, q.view(bad))):
            with pytest.raises(ValueError, match="must be uint8 or float8_e4m3fn"):
                hs.param(x, x, m, v, s)
    with pytest.raises(ValueError, match="need scale"):
        hs.param(x, x, q, q, s.view(torch.float8_e4m3fn))


def test_missing_tensors_are_named(hs, on_host, monkeypatch):
    import torch
    x, v = torch.zeros(4, 8), torch.zeros(4)
    with pytest.raises(ValueError, match="needs grad, or W"):
        hs.param()
    monkeypatch.undo()
    for H, X, name in ((None, x, "H"), (None, None, "H")):
        with pytest.raises(ValueError, match=f"{name} is missing"):
            hs.haste_layer_norm_fwd(4, 8, 0, H, None, None, 1e-5, 0, X)
    with pytest.raises(ValueError, match="H is missing"):
        hs.haste_layer_norm_bwd(4, 8, 0, None, None, v, v, 0, x)
    with pytest.raises(ValueError, match="out is missing"):
        hs.haste_grad_norm(hs.param_list([]), 1.0, None)
    monkeypatch.setattr(hs, "_here", lambda t, name: -1)
    with pytest.raises(ValueError, match="X is missing"):
        hs.haste_layer_norm_fwd(4, 8, 0, x, None, None, 1e-5, 0, None)


def test_options_and_lists_made_on_another_device_are_refused(hs, on_host, monkeypatch):
    """Refused before the call: the lists are empty, and the options wrong, so that nothing could be launched."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(hs, "_here", lambda t, name: 0)
    empty = hs.param_list([])
    for name, dtype in (("lr_dev", torch.float32), ("step_dev", torch.int64), ("grad_scale", torch.float32)):
        opts = hs.adamw_opts(1e-3, **{name: torch.zeros(1, dtype=dtype)})
        with pytest.raises(ValueError, match="options' tensors are on cuda:0, not on the current device cuda:1"):
            hs.haste_adamw(empty, opts)
    opts = hs.adamw_opts(-1.0)                   # no tensors: the call itself refuses it
    with pytest.raises(hs.HasteError, match="lr"):
        hs.haste_adamw(empty, opts, stream=0)
    empty.device = 0
    for call in (lambda: hs.haste_adamw(empty, opts), lambda: hs.haste_grad_norm(empty, 1.0, torch.zeros(2))):
        with pytest.raises(ValueError, match="list's tensors are on cuda:0"):
            call()


def test_the_check_for_arrays_named_twice_takes_its_time_by_tensor(hs):
    """Lists of 2048 and of 65536 tensors, the last one of which names the weights of the one before.  Going through the
    list once for every 512 tensors looks at 2 and at 64 of those runs on average for each tensor, 32 times as much
    (measured 21 times the time); looking each up once, at one (2 to 3 times, for the larger table).  The processor's time of
    this thread, the least of many."""
    import ctypes
    import time
    lists, took = {}, {}
    for n in (2048, 65536):
        params = lists[n] = (hs.haste_param_t * n)()
        for j, p in enumerate(params):
            p.W, p.grad, p.m, p.v, p.n, p.state_bits = *((8 * j + i) << 20 for i in (1, 2, 3, 4)), 64, 32
        params[n - 1].v = params[n - 2].W
    opts = hs.adamw_opts(1e-3)
    for _ in range(15):
        for n, params in lists.items():
            start = time.thread_time_ns()
            assert hs.lib.haste_adamw(params, n, ctypes.byref(opts), None) == 1
            took[n] = min(took.get(n, 1e12), (time.thread_time_ns() - start) / n)
            assert f"tensor {n - 1}:" in hs.haste_last_error() and "twice" in hs.haste_last_error()
    assert took[65536] < 10 * took[2048], took
