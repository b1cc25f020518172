"""Inputs, layouts and error bounds shared by the tests of the operators around the layers."""
import numpy as np
import torch

import paper_1803_07289_amd as fx

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24        # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest_half(dtype):
    """Half the spacing of the type's subnormals."""
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def chain(terms, lanes=16):
    """Roundings that one value goes through in a sum of so many terms by at least `lanes` partial sums that are then added, plus
    those of the handful of operations around it."""
    return (terms / lanes + 32) * U


def to_positions(t, layout):
    """[B,C,N] / [B,N,C] tensor -> float64 numpy [B*N, C]."""
    t = t.detach().double()
    t = t.transpose(1, 2) if layout == fx.BCN else t
    return t.reshape(-1, t.shape[2]).cpu().numpy()


def laid_out(rows, B, layout, dtype, offset=0, row=None):
    """numpy [B*N, C] -> device tensor in the layout and type, `offset` elements into its storage, rows of `row` elements (point-major: of
    scores; channel-major: of points), the rest NaN."""
    N, C = rows.shape[0] // B, rows.shape[1]
    t = torch.from_numpy(np.ascontiguousarray(rows)).to(dtype).view(B, N, C)
    t = t.transpose(1, 2).contiguous() if layout == fx.BCN else t
    b, r, w = t.shape
    row = row or w
    store = torch.full((offset + b * r * row,), float("nan"), dtype=dtype, device="cuda")
    view = store[offset:].view(b, r, row)[:, :, :w]
    view.copy_(t)
    return view


def within(got, ref, bound, what):
    """|got - ref| <= bound, elementwise; infinities and NaN where the reference has them."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    finite = np.isfinite(ref)
    assert np.array_equal(got[~finite], ref[~finite], equal_nan=True), what
    off = np.abs(got - ref)[finite] - np.broadcast_to(bound, ref.shape)[finite]
    assert off.size == 0 or (np.all(np.isfinite(got[finite])) and off.max() <= 0), (what, off.max(), int(off.argmax()))
