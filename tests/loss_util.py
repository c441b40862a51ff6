"""Inputs and bounds shared by the GPU tests of the losses.

Bounds.  An exponential exp(x - m) is off by the roundings of x - m and of its product with log2 e, both relative to an argument of at most `span` that
matters (beyond 90 it is zero in float32): 2 * 90 * 2^-24, and 4 * 2^-24 of its own; a sum of C of them by at most C / 64 additions in one lane and
some 20 across lanes, 2^-24 each.  REL(C) is that, for p, log p (per unit) and what is linear in them; a product of a few such factors
stays within 4 REL.  Stored gradients are rounded once: half a step, 2^-8 (bf16) or 2^-24 of the value."""
import numpy as np


def rel(C):
    return (180 + 4 + C / 64 + 20) * 2.0 ** -24


def half_step(bf16):
    return 2.0 ** -8 if bf16 else 2.0 ** -24


def round_to(x, bf16):
    """float64 values as the device stores them."""
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16 if bf16 else torch.float32)


class Rows:
    """A matrix on the device whose rows lie `stride` apart, `skip` elements behind an aligned address; what lies between and around holds `fill`."""

    def __init__(self, rows, C, bf16, stride=None, skip=0, fill=-3.0):
        import torch
        self.rows, self.C, self.stride, self.skip, self.fill = rows, C, stride or C, skip, fill
        self.dtype = torch.bfloat16 if bf16 else torch.float32
        self.flat = torch.full((skip + (rows - 1) * self.stride + C + 64,), fill, dtype=self.dtype, device="cuda")
        self.view = self.flat[skip:].as_strided((rows, C), (self.stride, 1), skip)

    def put(self, values):
        self.view.copy_(values.to(self.dtype))
        return self

    def ptr(self):
        return self.flat.data_ptr() + self.skip * self.flat.element_size()

    def host(self):
        return self.view.double().cpu().numpy()

    def untouched(self):
        """Whether everything outside the rows still holds the fill."""
        mark = self.flat.clone()
        mark[self.skip:].as_strided((self.rows, self.C), (self.stride, 1), self.skip).fill_(self.fill)
        return bool((mark == self.fill).all())


def dev(v, dtype=np.float32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(v, dtype)).cuda()


def close(got, want, tolerance, what):
    """Every element within its tolerance; infinities and NaN in the same places."""
    got, want, tolerance = (np.asarray(v, np.float64) for v in (got, want, tolerance))
    tolerance = np.broadcast_to(tolerance, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    bad = ~(np.abs(got - want)[fine] <= tolerance[fine])
    assert not bad.any(), "%s: %d of %d off, the worst %.3g with %.3g allowed" % (
        what, bad.sum(), bad.size, np.abs(got - want)[fine][bad].max(), tolerance[fine][bad].min())
