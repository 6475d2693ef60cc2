"""The operators of a training step from their formulas, in 64 bits on the CPU: what the GPU tests compare with."""
import math

import numpy as np
import torch

RELU, LEAKY, NONE = 0, 1, 2
SLOPE = 0.01
EPS32 = 2.0 ** -24                                  # half a step of fp32
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}   # step of the numbers below the normal ones


def taps(nbhd, delay):
    reach = {10: 1, 12: 2}[nbhd]
    out = [(-2, d) for d in range(-2, reach + 1)] + [(-1, d) for d in range(-2, reach + 1)] + [(0, -2), (0, -1)]
    if delay == 1:
        out = [(-1, 0) if t in ((-2, 2), (-1, 1), (-1, 2)) else t for t in out]
    return out


def contexts(img, nbhd, delay):
    n, h, w, _ = img.shape
    out = np.zeros((n, h, w, nbhd, 3))
    for j, (dr, dc) in enumerate(taps(nbhd, delay)):
        for r in range(max(0, -dr), h):
            for c in range(w):
                if 0 <= c + dc < w:
                    out[:, r, c, j] = img[:, r + dr, c + dc] / 256.0
    return out.reshape(n * h * w, 3 * nbhd)


def activate(z, act):
    return z if act == NONE else torch.where(z < 0, (0.0 if act == RELU else SLOPE) * z, z)


def derivative(x, act):
    return torch.ones_like(x) if act == NONE else torch.where(x > 0, 1.0, 0.0 if act == RELU else SLOPE).to(x.dtype)


def linear(x, w, bias, offsets, act):
    """(y, how far a sum in fp32 may be off) of rows of groups; other rows are NaN in y."""
    x, w = x.double().cpu(), w.double().cpu()
    y = torch.full((x.shape[0], w.shape[1]), float("nan"), dtype=torch.float64)
    bound = torch.zeros_like(y)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        b = bias[g].double().cpu() if bias is not None else torch.zeros(w.shape[1], dtype=torch.float64)
        z = x[lo:hi] @ w[g].T + b
        y[lo:hi] = activate(z, act)
        bound[lo:hi] = (x.shape[1] + 3) * EPS32 * (x[lo:hi].abs() @ w[g].abs().T + b.abs())
    return y, bound


def linear_grad(dz, x, w, offsets, x_act):
    """dx, dw, db and how far sums in fp32 may be off."""
    dz, x, w = dz.double().cpu(), x.double().cpu(), w.double().cpu()
    dx, dx_bound = torch.full_like(x, float("nan")), torch.zeros_like(x)
    dw, db = torch.zeros_like(w), torch.zeros(w.shape[:2], dtype=torch.float64)
    dw_bound, db_bound = torch.zeros_like(dw), torch.zeros_like(db)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        a, b = dz[lo:hi], x[lo:hi]
        slope = derivative(b, x_act)
        dx[lo:hi] = (a @ w[g]) * slope
        dx_bound[lo:hi] = (w.shape[1] + 2) * EPS32 * (a.abs() @ w[g].abs()) * slope
        dw[g], db[g] = a.T @ b, a.sum(0)
        dw_bound[g], db_bound[g] = (hi - lo + 2) * EPS32 * (a.abs().T @ b.abs()), (hi - lo + 2) * EPS32 * a.abs().sum(0)
    return (dx, dx_bound), (dw, dw_bound), (db, db_bound)


def assert_near(got, want, bound, what):
    """Each value within `bound` (of the sum in fp32) and half a step of its type of the formula's."""
    dtype = got.dtype
    got = got.detach().double().cpu()
    there = ~torch.isnan(want)
    tol = bound * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype]
    off = (got - want).abs()[there]
    worst = (off / tol[there]).max().item() if off.numel() else 0.0
    assert torch.isfinite(got[there]).all(), what
    assert worst <= 1.0, "%s: off by %.3g of the tolerance" % (what, worst)


def mixture(params, rgb, k, dist):
    """Per pixel and channel: pi, distance of the level's borders from each mean in widths, width, of the formula."""
    o, x = params.double().cpu(), rgb.double().cpu()
    out = []
    for c in range(3):
        logit, mean, ls = (o[:, 3 * k * c + k * i:3 * k * c + k * (i + 1)] for i in range(3))
        if c == 1:
            mean = mean + o[:, 9 * k:10 * k] * x[:, :1] / 256
        if c == 2:
            mean = mean + o[:, 10 * k:11 * k] * x[:, :1] / 256 + o[:, 11 * k:] * x[:, 1:2] / 256
        ls = torch.where(torch.isnan(ls), torch.full_like(ls, -8.0), ls)
        sigma = torch.exp(ls.clamp(-8.0, 4.0))
        out.append((torch.softmax(logit, 1), ((x[:, c:c + 1] - 0.5) / 256 - mean) / sigma, ((x[:, c:c + 1] + 0.5) / 256 - mean) / sigma, sigma))
    return out


def tail(z, dist):
    return 0.5 * torch.special.erfc(z / math.sqrt(2.0)) if dist == 0 else torch.sigmoid(-z)


def density(z, dist):
    return torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi) if dist == 0 else torch.sigmoid(z) * torch.sigmoid(-z)


def code_length(params, rgb, k, dist):
    """bits [count] of the formula; differentiable."""
    x = rgb.double().cpu()
    total = torch.zeros(len(x), dtype=torch.float64)
    for c, (pi, a, b, _) in enumerate(mixture(params, rgb, k, dist)):
        level = x[:, c:c + 1]
        left = a + b > 0                             # the nearer tail's difference
        q = torch.where(left, tail(a, dist) - tail(b, dist), tail(-b, dist) - tail(-a, dist))
        q = torch.where(level == 0, tail(-b, dist), q)
        q = torch.where(level == 255, tail(a, dist), q)
        total = total - torch.log2((65280 * (pi * q).sum(1) + 1) / 65536)
    return total


def loss_gradient(params, rgb, k, dist, scale, weight=None):
    """(gradient [count, 12 K] by the formula, size of the terms that it is the difference of)."""
    x = rgb.double().cpu()
    count = len(x)
    grad, size = torch.zeros(count, 12 * k, dtype=torch.float64), torch.zeros(count, 12 * k, dtype=torch.float64)
    factor = torch.full((count, 1), float(scale), dtype=torch.float64)
    if weight is not None:
        factor = factor * weight.double().cpu()[:, None]
    for c, (pi, a, b, sigma) in enumerate(mixture(params, rgb, k, dist)):
        level = x[:, c:c + 1]
        zero = torch.zeros((), dtype=torch.float64)
        fa = torch.where(level == 0, zero, density(a, dist))
        fb = torch.where(level == 255, zero, density(b, dist))
        left = a + b > 0
        q = torch.where(left, tail(a, dist) - tail(b, dist), tail(-b, dist) - tail(-a, dist))
        q = torch.where(level == 0, tail(-b, dist), q)
        q = torch.where(level == 255, tail(a, dist), q)
        p = (pi * q).sum(1, keepdim=True)
        outer = -65280 * factor / ((65280 * p + 1) * math.log(2.0))
        ls = params[:, 3 * k * c + 2 * k:3 * k * (c + 1)].double().cpu()
        inside = (ls >= -8) & (ls <= 4)
        at = 3 * k * c
        grad[:, at:at + k] = outer * pi * (q - p)
        size[:, at:at + k] = outer.abs() * pi * (q + p)
        d_mu, s_mu = outer * pi * (fa - fb) / sigma, outer.abs() * pi * (fa + fb) / sigma
        grad[:, at + k:at + 2 * k], size[:, at + k:at + 2 * k] = d_mu, s_mu
        afa, bfb = torch.where(level == 0, zero, a * fa), torch.where(level == 255, zero, b * fb)
        grad[:, at + 2 * k:at + 3 * k] = torch.where(inside, outer * pi * (afa - bfb), zero)
        size[:, at + 2 * k:at + 3 * k] = torch.where(inside, outer.abs() * pi * (afa.abs() + bfb.abs()), zero)
        if c == 1:
            grad[:, 9 * k:10 * k], size[:, 9 * k:10 * k] = d_mu * x[:, :1] / 256, s_mu * x[:, :1] / 256
        if c == 2:
            grad[:, 10 * k:11 * k], size[:, 10 * k:11 * k] = d_mu * x[:, :1] / 256, s_mu * x[:, :1] / 256
            grad[:, 11 * k:], size[:, 11 * k:] = d_mu * x[:, 1:2] / 256, s_mu * x[:, 1:2] / 256
    return grad, size


# ---- AdamW in numpy, operation by operation in fp32 as include/pcc.h defines it ----

def dither(t):
    low = np.uint64(0xFFFFFFFF)
    mul = lambda a, b: (a * np.uint64(b)) & low  # noqa: E731
    h = (mul(np.arange(256, dtype=np.uint64), 0x9E3779B9) + mul(np.uint64(t), 0xB7E15163)) & low
    h ^= h >> np.uint64(15)
    h = mul(h, 0x6A09E667)
    h ^= h >> np.uint64(13)
    h = mul(h, 0x9E3779B9)
    h ^= h >> np.uint64(16)
    return (h >> np.uint64(12)).astype(np.int64), (mul(h, 0xB7E15163) >> np.uint64(12)).astype(np.int64)


CODES = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()


def decode(codes, scale):
    return CODES[codes] * np.repeat(scale, 256)[:len(codes)]


def encode(x, part, positive):
    """(codes, scales) of fp32 x in blocks of 256."""
    n, blocks = len(x), -(-len(x) // 256)
    y = np.zeros(blocks * 256, np.float32)
    y[:n] = x
    y = y.reshape(-1, 256)
    scale = np.abs(y).max(1) * np.float32(1 / 448)
    with np.errstate(divide="ignore", over="ignore"):
        inverse = np.where(scale >= np.float32(2.0 ** -100), np.float32(1) / scale, np.float32(0)).astype(np.float32)
    a = np.abs(y) * inverse[:, None]
    normal = ((a.view(np.int32).astype(np.int64) + part) >> 20) - 960
    small = (a * np.float32(512) + part.astype(np.float32) * np.float32(2.0 ** -20)).astype(np.float32).astype(np.int64)
    code = np.minimum(np.where(a >= np.float32(2.0 ** -6), normal, small), 0x7E)
    code = np.where((y > 0) & (code == 0), 1, code) if positive else code + (y < 0) * 128
    return code.reshape(-1)[:n].astype(np.uint8), scale.astype(np.float32)


class AdamW:
    """One tensor."""

    def __init__(self, param, bits, lr, betas, eps, weight_decay):
        self.p, self.bits = param.astype(np.float32).copy(), bits
        self.lr, self.betas, self.eps, self.wd, self.t = lr, betas, eps, weight_decay, 0
        n = len(param)
        if bits == 32:
            self.m, self.v = np.zeros(n, np.float32), np.zeros(n, np.float32)
        else:
            self.m, self.v = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
            self.ms, self.vs = np.zeros(-(-n // 256), np.float32), np.zeros(-(-n // 256), np.float32)

    def step(self, g):
        f = np.float32
        self.t += 1
        (b1, b2), t = self.betas, self.t
        m = self.m if self.bits == 32 else decode(self.m, self.ms)
        v = self.v if self.bits == 32 else np.square(decode(self.v, self.vs))
        m = f(b1) * m + f(1 - b1) * g
        v = f(b2) * v + (f(1 - b2) * g) * g
        root = np.sqrt(v)
        rate, scale = f(self.lr / (1 - b1 ** t)), f(1 / math.sqrt(1 - b2 ** t))
        self.p = self.p * f(1 - self.lr * self.wd) - rate * (m / (root * scale + f(self.eps)))
        if self.bits == 32:
            self.m, self.v = m, v
        else:
            pm, pv = dither(t)
            self.m, self.ms = encode(m, pm, False)
            self.v, self.vs = encode(root, pv, True)
