"""GPU arrays whose surroundings are watched."""

import numpy as np

from .gpu_run import torch_cuda


class Framed:
    """A GPU array of matrices whose rows lie `pad` apart, in an allocation that holds 7
    wherever the array does not."""

    def __init__(self, shape, dtype, pad, ahead=1):
        torch = torch_cuda()
        *count, rows, cols = shape
        n = int(np.prod(count, dtype=np.int64)) if count else 1
        self.flat = torch.full((ahead + n * rows * (cols + pad) + 64,), 7.0, device="cuda").to(dtype)
        body = self.flat[ahead:ahead + n * rows * (cols + pad)]
        self.view = body.view(*count, rows, cols + pad)[..., :cols]
        self.inside = torch.zeros_like(self.flat, dtype=torch.bool)
        self.inside[ahead:ahead + n * rows * (cols + pad)].view(*count, rows, cols + pad)[..., :cols] = True

    def check(self):
        assert (self.flat[~self.inside] == 7.0).all(), "written past the array"
