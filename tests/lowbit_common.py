"""Helpers of the low-bit GPU tests: tensors to and from float64, guard bands."""

import numpy as np
import torch

from paper_2607_20940_amd import mssa

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_ULP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # of rounding to nearest, relative


def f64(t):
    return t.double().cpu().numpy()


def cuda(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda").to(TORCH[dtype])


class Banded:
    """A tensor between two bands of a byte pattern, to see writes past its ends."""

    PAD = 4096

    def __init__(self, shape, dtype, fill=None):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.raw = torch.full((n + 2 * self.PAD,), 0xA5, dtype=torch.uint8, device="cuda")
        self.t = self.raw[self.PAD: self.PAD + n].view(dtype).reshape(shape)
        if fill is not None:
            self.t.fill_(fill)

    def intact(self):
        return bool((self.raw[: self.PAD] == 0xA5).all()) and bool((self.raw[-self.PAD:] == 0xA5).all())


def quantize(x, dtype="f32"):
    """(codes, scales) device tensors of a [rows, cols] tensor, by the library."""
    codes, scales = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in mssa.mx_shapes(*x.shape))
    mssa.mssa_mx_quantize(x.shape[0], x.shape[1], dtype, x, codes, scales, x_stride=x.stride(0))
    return codes, scales
