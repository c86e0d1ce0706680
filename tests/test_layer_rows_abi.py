"""Norms, scans and losses: what the C entry points refuse before anything is enqueued, and the sizes they say (no GPU needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def layer():
    from paper_2204_10562_amd import build, layer
    if not os.path.exists(build.LIB_PATH):
        build.build_libpp()
    layer.lib()
    return layer


# pointers that are never read: every call below is refused by the host
Z, P, ODD, OFF8 = None, ctypes.c_void_p(4096), ctypes.c_void_p(4097), ctypes.c_void_p(4104)
BIG = 1 << 40


def refused(call, ok, bad, code=-1):
    for at, value in bad:
        a = list(ok)
        a[at] = value
        assert call(*a) == code, (at, value)


def test_norm(layer):
    L = layer.lib()
    ok = [2, 4, 64, P, 64, P, 64, P, 1e-5, P, 64, P, 64, P, P, P, P, P, Z]
    nan = float("nan")
    refused(L.pp_norm_forward, ok, [(0, 3), (0, -1), (1, -1), (1, (1 << 30) + 1), (2, 0), (2, (1 << 22) + 1), (3, Z), (3, ODD), (4, 63), (5, ODD), (6, 63),
                                    (7, ODD), (8, 0.0), (8, -1.0), (8, nan), (8, 1e39), (8, 1e-40), (9, ODD), (10, 63), (11, ODD), (12, 63), (13, Z),
                                    (14, Z), (13, OFF8), (15, Z), (16, Z), (16, OFF8), (17, ODD)])
    a = list(ok)
    a[11] = a[13] = a[14] = Z                      # no output of the norm
    assert L.pp_norm_forward(*a) == -1
    assert L.pp_norm_forward(*([2, 0, 64, Z, 64, Z, 0, Z, 1e-5, Z, 0, Z, 0] + [Z] * 6)) == 0
    ok = [2, 4, 64, P, 64, P, 64, Z, Z, P, P, P, 64, P, 64, P, P, P, BIG, Z]
    refused(L.pp_norm_backward, ok, [(0, 7), (1, -1), (2, 0), (3, Z), (3, ODD), (4, 63), (5, Z), (5, ODD), (6, 63), (7, P), (8, P), (9, Z), (9, ODD), (10, ODD),
                                     (11, ODD), (12, 63), (13, Z), (14, 63), (15, ODD), (16, ODD), (16, Z)])
    refused(L.pp_norm_backward, ok, [(17, Z), (17, OFF8), (18, 16)], -2)
    a = list(ok)
    a[7] = a[8] = P                                # the sum both ways
    assert L.pp_norm_backward(*a) == -1
    for dtype, rows, cols in (("float32", 8192, 4096), ("bfloat16", 1, 1), ("float16", 3, 1 << 22)):
        import torch
        t = getattr(torch, dtype)
        b = layer.pp_norm_workspace_bytes(t, rows, cols)
        assert b > 0 and b % 256 == 0 and layer.pp_norm_workspace_bytes(t, max(1, rows // 3), cols) <= b
    assert layer.pp_norm_workspace_bytes(torch.float64, 4, 4) == layer.pp_norm_workspace_bytes(torch.float32, -1, 4) == 0


def test_scan(layer):
    import torch
    L = layer.lib()
    ok = [1, 40, 64, P, 64, P, 64, 3, P, P, P, 64, P, P, P, BIG, Z]
    sizes = [(0, 3), (1, -1), (2, 0), (7, -1), (7, (1 << 30) + 1)]
    refused(L.pp_scan_forward, ok, sizes + [(3, Z), (3, ODD), (4, 63), (5, Z), (6, 63), (8, ODD), (8, Z), (9, ODD), (10, Z), (11, 63), (12, ODD), (13, ODD)])
    refused(L.pp_scan_forward, ok, [(14, Z), (14, OFF8), (15, 16)], -2)
    a = list(ok)
    a[1], a[2], a[4], a[6], a[11] = 1 << 30, 64 * 3, 192, 192, 192    # too many tiles for a launch
    assert L.pp_scan_forward(*a) == -1
    ok = [1, 40, 64, P, 64, P, 64, P, 64, 3, P, P, P, P, P, 64, P, 64, P, P, BIG, Z]
    refused(L.pp_scan_backward, ok, [(0, -1), (1, -1), (2, 0), (3, Z), (4, 63), (5, Z), (6, 63), (7, ODD), (8, 63), (9, -1), (10, Z), (10, ODD), (11, ODD), (12, Z),
                                     (12, ODD), (13, ODD), (14, Z), (15, 63), (16, Z), (17, 63), (18, ODD)])
    refused(L.pp_scan_backward, ok, [(19, Z), (20, 16)], -2)
    assert L.pp_scan_forward(1, 40, 64, P, 64, P, 64, 0, P, Z, P, 64, Z, Z, P, BIG, Z) == 0       # no sequences
    ok = [0, 4, 64, P, 64, P, 64, 9, P, P, P, 64, Z]
    refused(L.pp_scan_step, ok, [(0, 3), (1, -1), (2, 0), (3, Z), (4, 63), (5, ODD), (6, 1), (7, -1), (8, ODD), (9, Z), (9, ODD), (10, Z), (11, 63)])
    a = list(ok)
    a[7], a[8] = 3, Z                              # fewer slots than rows, one to each
    assert L.pp_scan_step(*a) == -1
    assert L.pp_scan_step(0, 0, 64, Z, 0, Z, 0, 0, Z, Z, Z, 0, Z) == 0
    assert layer.pp_scan_kept_rows(torch.bfloat16, 0, 5) == 0 and layer.pp_scan_kept_rows(torch.bfloat16, 1, 5) == 1
    assert layer.pp_scan_kept_rows(torch.float64, 1, 5) == -1 and layer.pp_scan_kept_rows(torch.float32, 1, 0) == -1
    for call in (0, 1):
        for rows, cols in ((0, 1), (1, 1), (128, 64), (129, 65), (65536, 2048)):
            b = layer.pp_scan_workspace_bytes(call, torch.float16, rows, cols)
            assert b > 0 and b % 256 == 0 and b <= layer.pp_scan_workspace_bytes(call, torch.float16, rows + 130, cols)
    assert layer.pp_scan_workspace_bytes(2, torch.float16, 4, 4) == 0


def test_logprob(layer):
    import torch
    L = layer.lib()
    nan = float("nan")
    ok = [2, 4, 1 << 20, P, 1 << 20, 1.0, P, P, P, P, 5, P, P, P, BIG, Z]
    refused(L.pp_logprob_forward, ok, [(0, 3), (1, -1), (2, 0), (3, Z), (3, ODD), (4, 5), (5, 0.0), (5, -1.0), (5, nan), (5, 1e7), (6, ODD), (6, Z), (7, ODD), (8, ODD),
                                       (9, ODD), (9, ctypes.c_void_p(4100)), (10, -1), (10, 129), (11, Z), (11, ODD), (12, Z), (12, ODD)])
    refused(L.pp_logprob_forward, ok, [(13, Z), (13, OFF8), (14, 16)], -2)
    assert L.pp_logprob_forward(2, 0, 64, Z, 64, 1.0, Z, Z, Z, Z, 0, Z, Z, Z, 0, Z) == 0
    ok = [2, 4, 64, P, 64, 1.0, P, P, P, P, P, P, 64, Z]
    refused(L.pp_logprob_backward, ok, [(0, 3), (1, -1), (2, 0), (3, Z), (4, 5), (5, 0.0), (5, nan), (6, ODD), (6, Z), (7, Z), (7, ODD), (8, ODD), (9, Z), (9, ODD),
                                        (10, ODD), (11, Z), (11, ODD), (12, 63)])
    for t in (torch.bfloat16, torch.float32):
        for cols in (1, 5000, 131072, 1 << 22):
            sizes = [layer.pp_logprob_workspace_bytes(t, rows, cols, 20) for rows in (1, 2, 7, 16, 100, 1000, 5000)]
            assert sizes == sorted(sizes) and sizes[0] > 0 and all(b % 256 == 0 for b in sizes)
            assert layer.pp_logprob_workspace_bytes(t, 7, cols, 3) <= layer.pp_logprob_workspace_bytes(t, 7, cols, 128)
    assert layer.pp_logprob_workspace_bytes(torch.float32, 4, 4, 129) == layer.pp_logprob_workspace_bytes(torch.float64, 4, 4, 1) == 0


def test_distill(layer):
    import torch
    L = layer.lib()
    nan = float("nan")
    ok = [1, 2, 4, 64, P, 64, 1.0, 5, P, P, P, P, P, 64, P, BIG, Z]
    refused(L.pp_distill_loss, ok, [(0, 2), (0, -1), (1, 3), (2, -1), (3, 0), (4, Z), (4, ODD), (5, 63), (6, 0.0), (6, nan), (6, 1e8), (7, 0), (7, 129), (8, Z),
                                    (8, ODD), (9, Z), (9, ODD), (10, ODD), (11, Z), (11, ODD), (12, ODD), (13, 63)])
    refused(L.pp_distill_loss, ok, [(14, Z), (14, OFF8), (15, 16)], -2)
    assert L.pp_distill_loss(0, 2, 0, 64, Z, 64, 1.0, 1, Z, Z, Z, Z, Z, 0, Z, 0, Z) == 0
    for t in (torch.bfloat16, torch.float32):
        for cols in (1, 5000, 131072, 262144, 1 << 22):
            sizes = [layer.pp_distill_workspace_bytes(t, rows, cols, 20) for rows in (1, 2, 7, 16, 100, 1000, 5000)]
            assert sizes == sorted(sizes) and sizes[0] > 0 and all(b % 256 == 0 for b in sizes)
    assert layer.pp_distill_workspace_bytes(torch.float32, 4, 4, 0) == layer.pp_distill_workspace_bytes(torch.float32, 4, 4, 129) == 0
