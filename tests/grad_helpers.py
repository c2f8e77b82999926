"""Helpers of the gradient operators' GPU tests: strided device matrices with guarded surroundings."""
import numpy as np

import paper_2607_19331_amd as iso

GUARD = 7.25


def code(dtype):
    return iso.BF16 if dtype == "bf16" else iso.F32


def ttype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def unit(dtype):
    """Largest relative error of one rounding to nearest."""
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


class Mat:
    """A rows x cols view (row stride cols + gap) of a device buffer whose other elements hold GUARD."""

    def __init__(self, rows, cols, dtype, gap=0, values=None):
        import torch
        self.rows, self.cols, self.ld, self.dtype = rows, cols, cols + gap, dtype
        self.buf = torch.full((rows * self.ld + 64,), GUARD, dtype=ttype(dtype), device="cuda")
        self.view = self.buf[:rows * self.ld].view(rows, self.ld)[:, :cols]
        if values is not None:
            self.view.copy_(torch.as_tensor(np.ascontiguousarray(values), dtype=torch.float64).to(ttype(dtype)))

    def host(self):
        """Values in binary64; asserts that the guards are untouched."""
        a = self.buf.double().cpu().numpy()
        rows = a[:self.rows * self.ld].reshape(self.rows, self.ld)
        assert (rows[:, self.cols:] == GUARD).all() and (a[self.rows * self.ld:] == GUARD).all()
        return rows[:, :self.cols].copy()

    def unchanged_guards(self):
        self.host()


def close(got, want, tol):
    """|got - want| <= tol where want is finite, the same non-finite values elsewhere."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    off = np.abs(got - want)[fine] - np.broadcast_to(tol, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, off.max()
