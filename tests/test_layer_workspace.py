"""A workspace sized for some number of rows serves every smaller number."""
import os
import random
import shutil
import sys

import pytest

from conftest import ROOT
from layer_helpers import torch_type
from layer_plans import FORWARD, INPUT, TYPES, WEIGHT, Plans

# call, type, rows of the workspace, fewer rows that want more bytes, n_in, n_out
WANTING = [(INPUT, "bf16", 2048, 1300, 4096, 16384), (INPUT, "bf16", 300, 205, 256, 520), (INPUT, "f16", 1874, 993, 1409, 606), (INPUT, "f32", 293, 222, 5595, 1237),
           (FORWARD, "f16", 267, 202, 3864, 2958), (FORWARD, "f32", 161, 135, 3391, 3656), (FORWARD, "bf16", 95, 82, 8014, 1588),
           (WEIGHT, "f16", 9300, 9200, 300, 520), (WEIGHT, "bf16", 902, 819, 1342, 128), (WEIGHT, "f32", 3886, 3616, 297, 280)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    return Plans(str(tmp_path_factory.mktemp("plans")))


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


def first_bytes(call, t, rows, n_in, n_out):
    """What a call cannot do without: x in 4 bits, or dy's planes."""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    if call == FORWARD:
        g = -(-n_in // 128)
        return 256 + up(rows * g * 64) + up(rows * g * 4)
    return 256 + up((3 - TYPES[t]) * rows * (-(-n_out // 8) * 8) * 2)


def test_partial_sums_fit_the_room_they_get(plans):
    rng = random.Random(5)
    several = 0
    for _ in range(3000):
        call, t = rng.randrange(3), rng.choice(list(TYPES))
        rows, n_in, n_out = (int(2 ** rng.uniform(0, 14)) for _ in range(3))
        whole = plans.divide(call, t, rows, n_in, n_out)
        several += whole["pieces"] > 1
        for room in (0, whole["bytes"] // 2, whole["bytes"] - 1 if whole["bytes"] else 0, whole["bytes"], 2 * whole["bytes"]):
            p = plans.divide(call, t, rows, n_in, n_out, room)
            assert p["bytes"] <= room and 1 <= p["pieces"]
            assert room < whole["bytes"] or p == whole
            assert p["per"] * p["pieces"] >= p["steps"] > p["per"] * (p["pieces"] - 1)
    assert several > 500


def test_bytes_asked_for(plans, pp):
    """The library's bytes are those of its own division; what is indispensable grows with the rows."""
    rng = random.Random(6)
    wanting = 0
    for _ in range(2000):
        call, t = rng.randrange(3), rng.choice(list(TYPES))
        n_in, n_out = (int(2 ** rng.uniform(3, 14)) for _ in range(2))
        rows = int(2 ** rng.uniform(5.1, 14))
        fewer = rng.randrange(33, rows + 1)
        asked, less = (pp.pp_linear_workspace_bytes(call, torch_type(t), r, n_in, n_out) for r in (rows, fewer))
        need = max(first_bytes(call, q, rows, n_in, n_out) + plans.divide(call, q, rows, n_in, n_out)["bytes"] for q in TYPES if TYPES[q] >= TYPES[t])
        assert asked == need
        assert asked >= first_bytes(call, t, fewer, n_in, n_out)
        wanting += less > asked
    assert wanting > 20


@pytest.mark.gpu
@pytest.mark.parametrize("call, t, more, rows, n_in, n_out", WANTING)
def test_fewer_rows_than_the_workspace_is_for(pp, call, t, more, rows, n_in, n_out):
    """Small whole numbers, so the results do not depend on how the sum is divided."""
    import torch
    n = pp.pp_linear_workspace_bytes(call, torch_type(t), more, n_in, n_out)
    print("[case]", call, t, more, rows, n_in, n_out, n, pp.pp_linear_workspace_bytes(call, torch_type(t), rows, n_in, n_out), flush=True)
    assert n < pp.pp_linear_workspace_bytes(call, torch_type(t), rows, n_in, n_out)
    room = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(81)

    def whole(r, c, most):
        return torch.randint(-most, most + 1, (r, c), generator=g, device="cuda").float()
    x, w, dy = whole(rows, n_in, 4), whole(n_out, n_in, 4), whole(rows, n_out, 2).to(torch_type(t))
    x[:, ::32] = w[:, ::32] = 4.0
    wp, kept = pp.empty_packed(pp.PP_PACK_FP4, n_out, n_in), pp.empty_packed(pp.PP_PACK_INT8, rows, n_in)
    pp.pp_pack(pp.PP_PACK_FP4, w, wp)
    pp.pp_pack(pp.PP_PACK_INT8, x, kept)
    if call == FORWARD:
        y = torch.empty(rows, n_out, dtype=dy.dtype, device="cuda")
        pp.pp_linear_forward(x.to(y.dtype), wp, None, y, None, room[:n])
        assert torch.equal(y, (x.double() @ w.double().t().contiguous()).to(y.dtype))
    elif call == INPUT:
        dx = torch.empty(rows, n_in, dtype=dy.dtype, device="cuda")
        pp.pp_linear_backward_input(dy, wp, dx, room[:n])
        assert torch.equal(dx, (dy.double() @ w.double()).to(dy.dtype))
    else:
        dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
        pp.pp_linear_backward_weight(dy, kept, None, dw, db, room[:n])
        d = dy.double().t().contiguous()
        assert torch.equal(dw.double(), d @ x.double()) and torch.equal(db.double(), d.sum(1))
    assert (room[n:] == 255).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows, fewer, t", [(300, 205, "bf16"), (300, 77, "f32"), (300, 1, "f16")])
def test_block_takes_a_smaller_microbatch(rows, fewer, t):
    """The example's block, built for `rows`: a last microbatch of fewer gives what a block of its own size gives."""
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import packed_stage as example
    finally:
        sys.path.pop(0)
    dtype = torch_type(t)
    own, block = (example.PackedBlock(256, 520, r, dtype, seed=3) for r in (fewer, rows))
    g = torch.Generator(device="cuda").manual_seed(82)
    x, dy = (torch.randn(fewer, 256, generator=g, device="cuda").to(dtype) for _ in range(2))
    found = []
    for b in (own, block):
        y, kept = b.forward(x)
        found.append([y, b.backward(dy, kept)] + [l.grad for l in b.layers] + [l.bias_grad for l in b.layers])
    for a, b in zip(*found):
        # at most 520 terms to a sum, added in another order: three products one after the other, and the type's rounding
        assert (a.double() - b.double()).norm() <= 4 * {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -16}[t] * a.double().norm()
