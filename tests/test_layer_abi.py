"""The layer operators' part of the C ABI: exports, sizes, refusals (no GPU needed)."""
import ctypes
import os
import re

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def layer():
    from paper_2204_10562_amd import build, layer
    if not os.path.exists(build.LIB_PATH):
        build.build_libpp()
    layer.lib()
    return layer


def test_every_declared_symbol_is_exported(layer):
    text = open(os.path.join(ROOT, "include", "pp_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(pp_[a-z_]+)\s*\(", text)))
    assert sorted(layer.EXPORTS) == names
    for name in names:
        assert getattr(layer.lib(), name) is not None


def test_constants_are_the_headers(layer):
    text = open(os.path.join(ROOT, "include", "pp_layer.h")).read()
    for name, value in re.findall(r"#define (PP_[A-Z0-9_]+) ([0-9(][0-9<() ]*)", text):
        assert getattr(layer, name) == eval(value), name


def test_workspace_sizes(layer):
    import torch
    for call in (0, 1, 2):
        for dtype in (torch.bfloat16, torch.float16, torch.float32):
            for rows, k, n in [(0, 1, 1), (1, 1, 1), (1, 4096, 16384), (333, 4100, 5000), (32771, 520, 1000), (8192, 4096, 16384)]:
                b = layer.pp_linear_workspace_bytes(call, dtype, rows, k, n)
                assert b > 0 and b % 256 == 0
        assert layer.pp_linear_workspace_bytes(call, torch.float64, 4, 4, 4) == 0
        assert layer.pp_linear_workspace_bytes(call, torch.float32, -1, 4, 4) == 0
        assert layer.pp_linear_workspace_bytes(call, torch.float32, 4, 0, 4) == 0
        assert layer.pp_linear_workspace_bytes(call, torch.float32, 4, 4, (1 << 22) + 1) == 0
        assert layer.pp_linear_workspace_bytes(call, torch.float32, (1 << 30) + 1, 4, 4) == 0
    assert layer.pp_linear_workspace_bytes(3, torch.float32, 4, 4, 4) == 0
    assert layer.pp_linear_workspace_bytes(-1, torch.float32, 4, 4, 4) == 0


# pointers that are never read: every call below is refused by the host
Z, P, ODD = None, ctypes.c_void_p(4096), ctypes.c_void_p(4097)
BIG = 1 << 40


def test_pack_refusals(layer):
    L = layer.lib()
    ok = [0, 2, 4, 64, P, 64, P, P, Z]
    for at, bad in [(0, 2), (0, -1), (1, 3), (1, -1), (2, -1), (2, (1 << 30) + 1), (3, 0), (3, (1 << 22) + 1), (4, Z), (4, ODD),
                    (5, 63), (6, Z), (6, ctypes.c_void_p(4104)), (7, Z), (7, ctypes.c_void_p(4104))]:
        a = list(ok)
        a[at] = bad
        assert L.pp_pack(*a) == -1, (at, bad)
        if at in (4, 5):     # src and ld stand behind codes and scales in pp_unpack
            b = [ok[0], ok[1], ok[2], ok[3], P, P, bad if at == 4 else P, bad if at == 5 else 64, Z]
        elif at in (6, 7):
            b = [ok[0], ok[1], ok[2], ok[3], bad if at == 6 else P, bad if at == 7 else P, P, 64, Z]
        else:
            b = a[:4] + [P, P, P, 64, Z]
        assert L.pp_unpack(*b) == -1, (at, bad)
    # no rows: nothing to do, whatever the pointers
    assert L.pp_pack(0, 2, 0, 64, Z, 64, Z, Z, Z) == 0
    assert L.pp_unpack(1, 0, 0, 64, Z, Z, Z, 64, Z) == 0


def test_act_refusals(layer):
    L = layer.lib()
    ok = [0, 1, 4, 64, P, 64, P, 64, P, 64, P, P, P, P, Z]
    for at, bad in [(0, 3), (0, -1), (1, 7), (2, -2), (3, 0), (4, Z), (4, ODD), (5, 63), (6, ODD), (7, 1), (8, Z), (9, 3),
                    (10, Z), (11, Z), (10, ODD), (12, Z), (13, Z), (13, ODD)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_act_forward(*a) == -1, (at, bad)
    a = list(ok)
    a[6] = Z                       # u's checkpoint without u
    assert L.pp_act_forward(*a) == -1
    ok = [0, 1, 4, 64, P, 64, P, P, P, P, P, 64, P, 64, Z]
    for at, bad in [(0, 3), (1, -1), (2, -2), (3, 0), (4, Z), (4, ODD), (5, 63), (6, Z), (7, Z), (8, Z), (9, Z), (9, ODD), (10, Z),
                    (11, 63), (12, Z), (13, 63)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_act_backward(*a) == -1, (at, bad)
    assert L.pp_act_forward(0, 1, 0, 64, Z, 64, Z, 0, Z, 64, Z, Z, Z, Z, Z) == 0
    assert L.pp_act_backward(0, 1, 0, 64, Z, 64, Z, Z, Z, Z, Z, 64, Z, 0, Z) == 0


def test_linear_refusals(layer):
    L = layer.lib()
    ok = [2, 4, 64, 96, P, 64, P, P, P, P, 96, P, P, P, BIG, Z]
    for at, bad in [(0, 3), (1, -1), (2, 0), (3, 0), (3, (1 << 22) + 1), (4, Z), (4, ODD), (5, 63), (6, Z), (7, Z), (6, ODD), (8, ODD),
                    (9, Z), (10, 95), (11, Z), (12, Z), (12, ODD)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_forward(*a) == -1, (at, bad)
    for at, bad in [(13, Z), (13, ctypes.c_void_p(4104)), (14, 16)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_forward(*a) == -2, (at, bad)
    ok = [2, 4, 64, 96, P, 96, P, P, P, 64, P, BIG, Z]
    for at, bad in [(0, -1), (1, -1), (2, 0), (3, 0), (4, Z), (4, ODD), (5, 95), (6, Z), (7, Z), (7, ODD), (8, Z), (9, 63)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_backward_input(*a) == -1, (at, bad)
    for at, bad in [(10, Z), (10, ctypes.c_void_p(4104)), (11, 16)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_backward_input(*a) == -2, (at, bad)
    ok = [2, 4, 64, 96, P, 96, P, P, P, P, 64, P, P, BIG, Z]
    for at, bad in [(0, -1), (1, -1), (2, 0), (3, 0), (4, Z), (4, ODD), (5, 95), (6, Z), (7, Z), (6, ODD), (8, ODD), (9, Z), (10, 63), (11, ODD)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_backward_weight(*a) == -1, (at, bad)
    for at, bad in [(12, Z), (12, ctypes.c_void_p(4104)), (13, 16)]:
        a = list(ok)
        a[at] = bad
        assert L.pp_linear_backward_weight(*a) == -2, (at, bad)


def test_binding_refuses_tensors_of_the_host(layer):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    p = layer.empty_packed(layer.PP_PACK_INT8, 4, 64, device="cpu")
    with pytest.raises(ValueError):
        layer.pp_pack(layer.PP_PACK_INT8, x, p)
    with pytest.raises(ValueError):
        layer.pp_pack(layer.PP_PACK_INT8, x.double(), p)
    with pytest.raises(ValueError):
        layer.pp_unpack(layer.PP_PACK_INT8, p, x[0])


def test_packed_bytes(layer):
    assert layer.packed_bytes(layer.PP_PACK_INT8, 2048, 4096) == 2048 * 4096 + 2048 * 128
    assert layer.packed_bytes(layer.PP_PACK_FP4, 3, 129) == 3 * 2 * 68
