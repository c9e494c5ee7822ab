"""Helpers for the tests of the operators of include/gemm_layer.h: matrices of 8-bit and other integers inside larger buffers, and the
operators' definitions in 64 bits (numpy, on the host)."""
import numpy as np
import torch

from ops_util import DT, LEAST, UNIT

SCALE_FLOOR = np.float32(2.0 ** -96)
F32 = 1e-5       # relative: f32 sums of up to 20001 terms, at most 32 in a row in a lane and 22 sums of those (54 * 2^-24 = 3.3e-6), and a few operations


class Ints:
    """A (batch x) rows x cols matrix of integers on the device in a larger buffer, `ld` elements a row, `offset` elements from its start.  Around an operand lie
    values that would change any sum; an output (no values given) is a canary, which has to stay around it."""

    def __init__(self, dtype, rows, cols, ld=None, offset=0, values=None, batch=1):
        self.rows, self.cols, self.batch, self.offset = rows, cols, batch, offset
        self.ld = cols if ld is None else ld
        self.stride = rows * self.ld
        self.host = torch.full((offset + batch * self.stride + 16,), 85, dtype=dtype)
        if values is not None and rows and cols:
            self._view(self.host).copy_(torch.as_tensor(np.asarray(values)).reshape(batch, rows, cols).to(dtype))
        self.dev = self.host.clone().cuda()

    def _view(self, t):
        return t.as_strided((self.batch, self.rows, self.cols), (self.stride, self.ld, 1), self.offset)

    @property
    def ptr(self):
        return self.dev.data_ptr() + self.offset * self.dev.element_size()

    def values(self):
        v = self._view(self.host).numpy().astype(np.int64)
        return v if self.batch > 1 else v[0]

    def fetch(self):
        back = self.dev.cpu()
        v = self._view(back).numpy().astype(np.int64)
        around, before = back.clone(), self.host.clone()
        for t in (around, before):
            if self.rows and self.cols:
                self._view(t).zero_()
        assert torch.equal(around, before), "memory outside the result was written"
        return v if self.batch > 1 else v[0]


def rounded(x, kind):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DT[kind]).double().numpy()


def row_scales(y):
    """Of exactly known values: to the bit, as f32 has them; NaN of a row that is not finite."""
    most = np.maximum(np.abs(y).max(1).astype(np.float32), SCALE_FLOOR)
    return np.where(np.isfinite(most), most * (np.float32(1) / np.float32(127)), np.float32(np.nan))


def quantized(y):
    """Elements and scales of rows whose values are exactly known (numpy rounds ties to even; a quotient of 24 bits by 24 bits is never
    nearer than 2^-49 of itself to a border without being on it, so 53 bits tell)."""
    s = row_scales(y)
    finite = np.isfinite(s)
    return np.where(finite[:, None], np.rint(np.where(finite[:, None], y, 0) / np.where(finite, s, 1).astype(np.float64)[:, None]), 0), s


def layer_norm(h, gamma, beta, eps):
    """mean, rstd, y and y's bound in f32 (without a rounding of y itself), from the stored h."""
    mean = h.mean(1, keepdims=True)
    d = h - mean
    rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    y = d * rstd * gamma + beta
    # the mean is off by F32 of the mean magnitude, the difference by its rounding, rstd by F32 of itself
    off = np.abs(gamma) * rstd * (F32 * np.abs(d) + F32 * np.abs(h).mean(1, keepdims=True) + 2.0 ** -23 * (np.abs(h) + np.abs(mean))) + 2.0 ** -23 * (np.abs(gamma * d * rstd) + np.abs(beta))
    return mean, rstd, y, off


def rounding(want, off, kind):
    return off + (np.abs(want) + off) * UNIT[kind] + LEAST[kind]


def order(expert, E):
    """offsets, source and place of choices (T x k), by a stable sort."""
    flat = np.where((expert >= 0) & (expert < E), expert, E).astype(np.int64).ravel()
    by = np.argsort(flat, kind="stable")
    valid = flat[by] < E
    k = expert.shape[1] if expert.ndim == 2 else 1
    source = np.where(valid, by // max(k, 1), -1)
    place = np.empty(flat.size, dtype=np.int64)
    place[by] = np.where(valid, np.arange(flat.size), -1)
    return np.searchsorted(flat[by], np.arange(E + 1)), source, place.reshape(expert.shape)
