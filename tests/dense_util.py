"""Helpers of the tests of the dense operators: plain float64 forms and views with guard bands."""
import math

import torch

DEV = "cuda:0"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U32 = 2.0 ** -24                        # half a step of fp32, relative


def half_step(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Guarded:
    """A [rows, cols] view at column `left` of a larger matrix whose other elements must stay as they are."""

    def __init__(self, rows, cols, dtype, left=0, right=0, fill=float("nan")):
        self.whole = torch.full((rows + 2, left + cols + right), fill, dtype=dtype, device=DEV)
        self.t = self.whole[1:rows + 1, left:left + cols]
        self.left, self.cols, self.fill = left, cols, fill

    def check(self):
        w = self.whole.clone()
        w[1:-1, self.left:self.left + self.cols] = self.fill
        same = torch.isnan(w) if math.isnan(self.fill) else w == self.fill
        assert bool(same.all()), "written outside the matrix"


def strided(t, left, right):
    """The values of t as a view with its own row stride and first column."""
    g = Guarded(t.shape[0], t.shape[1], t.dtype, left, right)
    g.t.copy_(t)
    return g.t


def act64(z, act):
    if act == 1:
        return torch.relu(z)
    if act == 2:
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == 3:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == 4 else z


def slope64(z, act):
    if act == 1:
        return (z > 0).double()
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act64(z, act).sum(), z)[0]


def norm64(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * rstd
    y = h * (1 if gamma is None else gamma.double()) + (0 if beta is None else beta.double())
    return y, mean[:, 0], rstd[:, 0], h


def norm64_bwd(dy, h, rstd, gamma):
    dy = dy.double()
    a = dy if gamma is None else dy * gamma.double()
    dx = rstd[:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)
