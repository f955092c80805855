"""Which kernels the layer norm's backward pass takes (no GPU needed: the rule is a host function of the library).
Each shape was measured in one launch and in two; the figures are those on MI355X, us a call in a graph, and of the calls
that the host bounds, us a call in a loop."""
import ctypes

import pytest

F32, BF16 = 0, 1


@pytest.mark.parametrize("B,F,dtype,one,us", [
    (512, 768, BF16, True, (5.3, 6.4)), (512, 768, F32, True, (5.7, 6.4)), (16, 64, BF16, True, (2.6, 4.8)),
    (512, 2048, BF16, True, (8.1, 9.0)), (512, 4096, BF16, False, (15.7, 12.2)), (512, 4096, F32, False, (15.9, 13.3)),
    (256, 4096, F32, True, (10.7, 11.6)), (512, 8192, BF16, False, (30.1, 18.8)), (512, 8192, F32, False, (32.7, 21.8)),
    (256, 8192, BF16, False, (18.5, 16.1)), (16, 8192, BF16, True, (9.5, 11.8)), (64, 8192, BF16, True, (10.3, 12.0)), (512, 12000, BF16, False, (39.6, 22.8)),
    (512, 16384, BF16, False, (51.1, 26.7)), (512, 16384, F32, False, (62.8, 33.7)),
    (64, 16384, BF16, True, (17.4, 20.0)), (128, 16384, F32, False, (22.6, 18.4)), (1, 12000, F32, True, (9.4, 12.0)),
    (300, 5000, BF16, True, (11.1, 14.2)), (512, 6144, BF16, False, (20.1, 16.0)), (200, 6144, BF16, True, (9.9, 13.3)),
    (200, 5000, F32, True, (12.4, 13.5)), (400, 5000, F32, False, (17.4, 15.5)), (512, 6144, F32, False, (26.8, 17.9)),
    (64, 7000, F32, True, (8.7, 9.9)), (512, 7000, BF16, False, (26.6, 18.6)), (512, 3500, BF16, False, (13.2, 11.7)),
    (513, 768, BF16, False, None), (100, 3, F32, False, None), (1, 16385, F32, False, None),
])
def test_few_rows_go_in_one_launch_where_that_is_faster(B, F, dtype, one, us):
    from paper_2606_01117_amd import lib
    fn = lib._ZN5haste10ln_bwd_fewElli
    fn.restype, fn.argtypes = ctypes.c_bool, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32]
    assert fn(B, F, dtype) == one
    assert us is None or one == (us[0] < us[1])


def _teams(F, backward, bf16):
    """The team that takes a row, and its runs of four values a thread."""
    runs = lambda team: -(-F // (4 * team))
    limits = ((256, 16), (1024, 64), (2048, 256), (4096, 512)) if backward else ((256, 16), (1024, 64), (4096, 256))
    team = next((t for most, t in limits if F <= most), 1024)
    small = {1024: 256, 512: 256, 256: 64, 64: 16}.get(team)
    if bf16 and small and 4 * F <= 3 * 4 * team * runs(team) and runs(small) <= 6:
        team = small
    return team, runs(team)


def test_no_kernel_is_built_that_no_width_takes():
    import re
    import subprocess

    from paper_2606_01117_amd import LIB_PATH
    out = subprocess.run(["nm", "-C", LIB_PATH], capture_output=True, text=True, check=True).stdout
    built = set(re.findall(r"__device_stub__(k_ln_\w+)<(.*?)>\(", out))
    types = {"float": False, "__hip_bfloat16": True, "unsigned short": True}
    names = {n for _, args in built for n in args.split(", ")[:2]}
    assert names <= set(types), names
    want = set()
    for F in range(4, 16385):
        for a in names:
            for b in names:
                fwd, bwd = _teams(F, False, types[a] or types[b]), _teams(F, True, types[a])
                want.add(("k_ln_fwd", f"{a}, {b}, {fwd[0]}, {fwd[1]}"))
                want.add(("k_ln_bwd_few", f"{a}, {b}, {bwd[0]}, {bwd[1]}"))
                want |= {("k_ln_bwd", f"{a}, {b}, {bwd[0]}, {bwd[1]}, {stream}") for stream in ("false", "true")}
    held = {k for k in built if k[0] in ("k_ln_fwd", "k_ln_bwd", "k_ln_bwd_few")}
    assert held == want, (sorted(held - want)[:5], sorted(want - held)[:5])
