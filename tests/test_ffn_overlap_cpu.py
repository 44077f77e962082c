"""Outputs of the feed-forward block that share memory with inputs or with one another are refused by the
C entry points before any CUDA call (a product writes what a later one still reads)."""
import ctypes

import pytest

from test_ffn_cpu import desc, kdn  # noqa: F401

ROWS, D, F = 20, 64, 96
STEP = 1 << 20  # between the pointers, which nothing dereferences: every call here is refused
FWD = ("x", "wg", "wu", "wd", "g", "u", "h", "y", "workspace")
BWD = ("x", "wg", "wu", "wd", "g", "u", "h", "dy", "dx", "dwg", "dwu", "dwd", "workspace")
OUT = {"fwd": ("g", "u", "h", "y", "workspace"), "bwd": ("dx", "dwg", "dwu", "dwd", "workspace")}


def size(name, dtype, dw_dtype, workspace):
    es = 4 if (dw_dtype if name in ("dwg", "dwu", "dwd") else dtype) == 0 else 2
    n = {"workspace": workspace, "x": ROWS * D, "y": ROWS * D, "dx": ROWS * D, "dy": ROWS * D}
    return workspace if name == "workspace" else n.get(name, D * F if "w" in name else ROWS * F) * es


@pytest.mark.parametrize("way", ["fwd", "bwd"])
@pytest.mark.parametrize("dtype,dw_dtype", [(1, 1), (1, 0), (0, 0)])
def test_refuses_shared_memory(kdn, way, dtype, dw_dtype):  # noqa: F811
    d = desc(kdn, rows=ROWS, D=D, F=F, dtype=dtype, dw_dtype=dtype if way == "fwd" else dw_dtype)
    L, names = kdn.lib(), FWD if way == "fwd" else BWD
    call = L.kdn_ffn_fwd if way == "fwd" else L.kdn_ffn_bwd
    need = (L.kdn_ffn_fwd_workspace_bytes if way == "fwd" else L.kdn_ffn_bwd_workspace_bytes)(ctypes.byref(d))
    assert need <= STEP
    n = {name: size(name, dtype, d.dw_dtype, need) for name in names}
    for out in OUT[way]:
        for other in names:
            if other == out:
                continue
            # the same place, the other's last 256 bytes, and a start before it that reaches into it
            for shift in (0, (n[other] - 1) // 256 * 256, -((n[out] - 1) // 256 * 256)):
                at = {name: (i + 1) * STEP for i, name in enumerate(names)}
                at[out] = at[other] + shift
                st = call(ctypes.byref(d), *[ctypes.c_void_p(at[name]) for name in names], need, None)
                assert st == kdn.KDN_ERR_INVALID_ARG, (out, other, shift)


def test_refuses_weights_that_are_their_gradients_without_rows(kdn):  # noqa: F811
    d, p = desc(kdn, rows=0), ctypes.c_void_p
    at = [p(STEP * (i + 1)) for i in range(4)]
    for i in range(3):
        w = [None] * 3
        w[i] = at[i]
        assert kdn.lib().kdn_ffn_bwd(ctypes.byref(d), None, *w, *[None] * 5, *at, 256, None) == kdn.KDN_ERR_INVALID_ARG
