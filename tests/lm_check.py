"""Comparisons of the language-model operators with plain forms in 64 bits."""
import torch

U32 = 2.0 ** -24                                      # unit roundoff of fp32: 24 significant bits
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def within(got, want, size, roundings, what):
    """Each element of got lies within `roundings` fp32 roundings of terms that add up to `size`, and one
    rounding to got's own type, of the 64-bit value want."""
    g = got.detach().double().cpu()
    want, size = want.double().cpu(), torch.as_tensor(size).double().cpu()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    assert bool(torch.isfinite(g).all()), f"{what}: not finite"
    room = roundings * U32 * size
    room = room + UNIT[got.dtype] * (want.abs() + room) + 1e-37
    bad = ((g - want).abs() > room).nonzero()
    if len(bad):
        i = tuple(bad[0].tolist())
        raise AssertionError(f"{what}: {len(bad)} of {g.numel()} outside; at {i} {g[i].item()!r}, want "
                             f"{want[i].item()!r}, room {(room.expand_as(g))[i].item()!r}")


def slope(f, x, v, h):
    """The derivative of f at x along v by a central difference of 64-bit values."""
    return (f(x + h * v) - f(x - h * v)) / (2 * h)
