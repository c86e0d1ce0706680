"""Norms of more rows than a launch has workgroups, where several waves have a row (marker gpu).  Bounds as in the norms' other tests; the
gain's gradient has an addition for every row of a part, of which there are 512."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_forward_and_backward():
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols, step = (1 << 20) + 300, 2050, 1 << 16
    print("[case] norm", rows, cols, flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for at in range(0, rows, step):
        for m in (x, dy):
            m[at:at + step] = torch.randn(x[at:at + step].shape, generator=g, device="cuda")
    gain = 1 + torch.randn(cols, generator=g, device="cuda") * 0.2
    y, dx, inv, dgain = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
    pp.pp_norm_forward(x, None, gain, 1e-5, None, y, None, None, inv)
    ws = torch.full((pp.pp_norm_workspace_bytes(x.dtype, rows, cols),), 255, dtype=torch.uint8, device="cuda")
    pp.pp_norm_backward(dy, x, inv, gain, None, dx, None, dgain, ws)
    total, terms = (torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2))

    def near(got, want, bound):
        return bool(((got.double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound) + 2.0 ** -133).all())
    for at in range(0, rows, step):
        part = slice(at, at + step)
        s, d, r = x[part].double(), dy[part].double(), inv[part].double()[:, None]
        z = s * ((s * s).mean(1, keepdim=True) + 1e-5).rsqrt()
        want = z * gain.double()
        assert near(y[part], want, 64 * U * want.abs()), at
        z, gd = s * r, d * gain.double()
        want = r * (gd - z * (gd * z).mean(1, keepdim=True))
        assert near(dx[part], want, r * (6 * U * gd.abs() + z.abs() * 70 * U * (gd * z).abs().mean(1, keepdim=True)) + 2 * U * want.abs()), at
        total += (d * z).sum(0)
        terms += (d * z).abs().sum(0)
    assert ((dgain - total).abs() <= (rows // 512 + 160) * U * terms).all()
    del x, dy, y, dx, ws
    torch.cuda.empty_cache()
