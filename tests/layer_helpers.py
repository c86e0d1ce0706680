"""Inputs, guards and bounds that the layer operators' GPU tests share."""
import numpy as np

TYPES = ("bf16", "f16", "f32")


def torch_type(t):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[t]


def on_gpu(values, t, pad=0, off=0):
    """A float64 array as a GPU matrix of type t whose rows lie cols + pad apart and start `off` values
    behind an allocation's start, and the values it holds after rounding to t."""
    import torch
    rows, cols = values.shape
    room = torch.full((rows * (cols + pad) + off + 8,), float("nan"), dtype=torch_type(t), device="cuda")
    m = room[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.from_numpy(values).to(torch_type(t)))
    return m, m.double().cpu().numpy()


class Guarded:
    """An output matrix with marked room in front, behind and between its rows, which has to stay as it is."""

    def __init__(self, rows, cols, t, pad=0, off=0):
        import torch
        self.room = torch.full((off + rows * (cols + pad) + 64,), 77.0, dtype=torch_type(t), device="cuda")
        self.rows, self.cols, self.pad, self.off = rows, cols, pad, off
        self.m = self.room[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def values(self):
        n = self.rows * (self.cols + self.pad)
        room = self.room.double().cpu().numpy()
        assert (room[:self.off] == 77).all() and (room[self.off + n:] == 77).all()
        body = room[self.off:self.off + n].reshape(self.rows, self.cols + self.pad)
        assert (body[:, self.cols:] == 77).all()
        return body[:, :self.cols]


def packed_guarded(fmt, rows, cols):
    """Room for a packed matrix, filled with 7s, and a function that checks that 64 bytes behind stay so."""
    import torch
    from paper_2204_10562_amd import layer
    dtype, width = layer._CODES[fmt]
    g = -(-cols // 128)
    c = torch.full((rows * g * width + 64,), 7, dtype=dtype, device="cuda")
    s = torch.full((rows * g * 4 + 64,), 7, dtype=torch.uint8, device="cuda")
    pair = (c[:rows * g * width].view(rows, g, width), s[:rows * g * 4].view(rows, g, 4))

    def check():
        assert (c[rows * g * width:] == 7).all() and (s[rows * g * 4:] == 7).all()
        return pair[0].cpu().numpy(), pair[1].cpu().numpy()
    return pair, check


def half_step(t, v):
    """Half the spacing of type t at the size of v: what rounding to nearest may add."""
    bits, low = {"bf16": (8, -133), "f16": (11, -24), "f32": (24, -149)}[t]
    e = np.where(v != 0, np.frexp(v)[1], low)
    return np.ldexp(0.5, np.maximum(e - bits, low))


def assert_within(got, want, bound, t):
    """|got - want| <= bound (of the computation) and the rounding of what it gave to type t."""
    lim = bound + half_step(t, np.abs(want) + bound)
    far = ~(np.abs(got - want) <= lim)
    assert not far.any(), (np.argwhere(far)[:4], got[far][:4], want[far][:4], lim[far][:4])
