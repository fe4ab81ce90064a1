"""Helpers of the tests of the operators on rows: tensors with any row stride and start, stored values, error bounds."""
import numpy as np

from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod

EPS32 = 2.0 ** -24                                             # half a unit in the last place of fp32, relative
ROUND = {wl.F32: 2.0 ** -24, wl.F16: 2.0 ** -11, wl.BF16: 2.0 ** -8}   # one rounding to the storage type, relative
TINY = {wl.F32: 2.0 ** -149, wl.F16: 2.0 ** -25, wl.BF16: 2.0 ** -134}  # ... and absolute, among its denormal numbers


def torch_type(dtype):
    torch = torch_mod()
    return {wl.F32: torch.float32, wl.F16: torch.float16, wl.BF16: torch.bfloat16}[dtype]


def stored(x, dtype):
    """float array -> float64 array of the values that the storage type holds."""
    with np.errstate(over="ignore", invalid="ignore"):
        return wl.storage_to_f64(wl.to_storage(np.asarray(x, dtype=np.float32), dtype), dtype)


class Rows:
    """A rows x cols tensor on the GPU with the row stride `ld`, starting `start` elements into its memory.  What lies between
    the rows is filled with `fill`, so that what is read there shows, and so does what is written (see untouched())."""

    def __init__(self, rows, cols, ttype, ld=None, start=0, fill=0):
        torch = torch_mod()
        self.rows, self.cols, self.ld, self.fill = rows, cols, cols if ld is None else ld, fill
        self.flat = torch.full((start + rows * self.ld + 64,), fill, dtype=ttype, device="cuda")
        self.view = self.flat[start:start + rows * self.ld].view(rows, self.ld)[:, :cols]
        self.start = start

    @property
    def ptr(self):
        return self.view.data_ptr() if self.rows else self.flat[self.start:].data_ptr()

    def set(self, x64):
        torch = torch_mod()
        self.view.copy_(torch.from_numpy(np.ascontiguousarray(x64)).to(self.view.dtype))
        return self

    def host(self):
        return self.view.double().cpu().numpy() if self.view.dtype.is_floating_point else self.view.cpu().numpy()

    def untouched(self, written=None):
        """Whether everything outside the first `written` (default: cols) columns still holds the fill."""
        torch = torch_mod()
        m = torch.ones_like(self.flat, dtype=torch.bool)
        if self.rows:
            m[self.start:self.start + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols if written is None else written] = False
        rest = self.flat[m]
        same = torch.isnan(rest) if self.fill != self.fill else rest == self.fill
        return bool(same.all())


def vec(x, fill=None):
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def nan_vec(n):
    return torch_mod().full((n,), float("nan"), dtype=torch_mod().float32, device="cuda")


def assert_close(got, want, tol, what):
    """Elementwise |got - want| <= tol; values that are not finite have to be the same."""
    got, want, tol = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64), np.broadcast_to(tol, np.shape(want))
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), "%s: NaN in other places" % what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), "%s: infinities differ" % what
    off = np.abs(got[fine] - want[fine])
    bad = off > tol[fine]
    assert not bad.any(), "%s: %d of %d elements off, worst %.3g where %.3g is allowed" % (
        what, int(bad.sum()), bad.size, float(off[bad].max()), float(tol[fine][bad][np.argmax(off[bad])]))
