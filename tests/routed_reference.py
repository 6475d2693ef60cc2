"""The operators round the grouped products from their formulas, in 64 bits on the CPU, and how far arithmetic in fp32 may be off."""
import math

import numpy as np
import torch

U = 2.0 ** -24          # half a step of fp32, relative
# Additions that one value goes through in a sum over a row: at most 64 in a lane, 6 over a wave's lanes, 16 over waves, rounded up.
DEPTH = 100


def groups_of(rows, offsets):
    """Each row's group, -1 for none."""
    g = np.full(rows, -1)
    for i, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        g[lo:hi] = i
    return torch.from_numpy(g)


def _per_row(t, g, fill, rows, features):
    if t is None:
        return torch.full((rows, features), fill, dtype=torch.float64)
    return t.double().cpu()[g.clamp_min(0)]


def layer_norm(x, gamma, beta, offsets, eps):
    """((y, bound), (stats, bound)); rows of no group are NaN."""
    x = x.double().cpu()
    rows, features = x.shape
    g = groups_of(rows, offsets)
    gm, bt = _per_row(gamma, g, 1.0, rows, features), _per_row(beta, g, 0.0, rows, features)
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    s = (var + eps) ** -0.5
    h = d * s
    y = gm * h + bt
    # the mean: a sum of DEPTH roundings, divided (as a product with 1 / features: two roundings)
    e_mean = (DEPTH + 2) * U * x.abs().mean(1, keepdim=True)
    e_var = (DEPTH + 6) * U * var + 2 * d.abs().mean(1, keepdim=True) * e_mean + e_mean ** 2
    # 1 / sqrt(v): half of v's relative error (and of its second order), eps in fp32, an addition, a root, a quotient
    low = (var + eps - e_var).clamp_min(eps / 2)
    e_s = s * (e_var / (2 * low) + 5 * U)
    e_h = s * e_mean + 3 * U * h.abs() + (d.abs() + e_mean) * e_s
    e_y = gm.abs() * e_h + 2 * U * (y.abs() + (gm * h).abs())
    there = (g >= 0)[:, None]
    nan = torch.full((), float("nan"), dtype=torch.float64)
    stats, e_stats = torch.cat([mean, s], 1), torch.cat([e_mean, e_s], 1)
    return (torch.where(there, y, nan), e_y), (torch.where(there, stats, nan), e_stats)


def layer_norm_grad(dy, x, stats, gamma, offsets):
    """(dx, bound), (dgamma, bound), (dbeta, bound) with the given statistics."""
    dy, x, stats = dy.double().cpu(), x.double().cpu(), stats.double().cpu()
    rows, features = x.shape
    g = groups_of(rows, offsets)
    gm = _per_row(gamma, g, 1.0, rows, features)
    mean, s = stats[:, :1], stats[:, 1:]
    h, u = (x - mean) * s, dy * gm
    a, b = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    dx = s * (u - a - h * b)
    e_h = 2 * U * h.abs()
    e_a = (DEPTH + 3) * U * u.abs().mean(1, keepdim=True)
    e_b = (DEPTH + 7) * U * (u * h).abs().mean(1, keepdim=True)
    e_dx = s.abs() * (U * u.abs() + e_a + h.abs() * e_b + (e_h + 2 * U * h.abs()) * (b.abs() + e_b) + 4 * U * (u.abs() + a.abs() + (h * b).abs()))
    there = (g >= 0)[:, None]
    dx = torch.where(there, dx, torch.full((), float("nan"), dtype=torch.float64))
    groups = len(offsets) - 1
    out = torch.zeros(4, groups, features, dtype=torch.float64)
    for i, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        p = dy[lo:hi] * h[lo:hi]
        out[0, i], out[1, i] = p.sum(0), (hi - lo + 8) * U * p.abs().sum(0)
        out[2, i], out[3, i] = dy[lo:hi].sum(0), (hi - lo + 4) * U * dy[lo:hi].abs().sum(0)
    return (dx, e_dx), (out[0], out[1]), (out[2], out[3])


def route(logits, k, over_all):
    """(expert, (weight, bound)), token by token."""
    l = logits.double().cpu()
    tokens, experts = l.shape
    expert = torch.full((tokens, k), -1, dtype=torch.int32)
    weight, bound = torch.zeros(tokens, k, dtype=torch.float64), torch.full((tokens, k), 2.0 ** -126, dtype=torch.float64)
    for t in range(tokens):
        row = l[t].tolist()
        order = sorted(range(experts), key=lambda i: (0 if math.isnan(row[i]) else 1, 0.0 if math.isnan(row[i]) else -row[i], i))
        chosen = [i for i in order[:k] if row[i] != -math.inf]
        summed = [row[i] for i in (range(experts) if over_all else chosen)]
        if not chosen:
            continue
        expert[t, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
        if any(math.isnan(v) or v == math.inf for v in summed):
            weight[t, :len(chosen)] = float("nan")
            continue
        top = max(summed)
        total = sum(math.exp(v - top) for v in summed)
        for j, i in enumerate(chosen):
            w = math.exp(row[i] - top) / total
            weight[t, j] = w
            # e^v of a v that is rounded once: v's size in roundings, and 6 of its own; the sum's terms have |v| e^v < 1
            bound[t, j] += w * U * (top - row[i] + 6 + 8 + DEPTH + 2)
    return expert, (weight, bound)


def route_grad(dweight, logits, expert, k, over_all):
    """(gradient, bound) from the softmax's derivative, for finite or masked logits and given choices."""
    l, dw, expert = logits.double().cpu(), dweight.double().cpu(), expert.long().cpu()
    tokens, experts = l.shape
    taken = expert >= 0
    chosen = torch.zeros(tokens, experts, dtype=torch.bool)
    grad = torch.zeros(tokens, experts, dtype=torch.float64)
    for j in range(k):
        rows = torch.nonzero(taken[:, j])[:, 0]
        chosen[rows, expert[rows, j]] = True
        grad[rows, expert[rows, j]] = dw[rows, j]
    inside = (l > -math.inf) & (chosen if not over_all else True)
    top = torch.where(inside, l, torch.full_like(l, -math.inf)).amax(1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    e = torch.where(inside, torch.exp(l - top), torch.zeros_like(l))
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total > 0, total, torch.ones_like(total))
    along = (p * grad).sum(1, keepdim=True)
    size = p * (grad.abs() + (p * grad.abs()).sum(1, keepdim=True))
    away = torch.where(inside, top - l, torch.zeros_like(l))
    # each p is off by what `route` says of a weight; so is each term of the sum along
    worst = (away * p).amax(1, keepdim=True) / p.clamp_min(1e-300)
    bound = size * U * (away + torch.minimum(worst, torch.full_like(worst, 200.0)) + 2 * DEPTH + 40) + 2.0 ** -120
    return p * (grad - along), bound


def sort(expert, experts):
    """(offsets, place) by running through the entries."""
    flat = expert.cpu().reshape(-1).tolist()
    lists = [[] for _ in range(experts)]
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            lists[e].append(i)
    place, offsets = [-1] * len(flat), [0]
    for entries in lists:
        for i in entries:
            place[i] = offsets[-1] + entries.index(i) if len(entries) < 50 else -2
        if len(entries) >= 50:
            for n, i in enumerate(entries):
                place[i] = offsets[-1] + n
        offsets.append(offsets[-1] + len(entries))
    return torch.tensor(offsets), torch.tensor(place, dtype=torch.int32).view(expert.shape)


def join(z, place, weight, rows):
    z, place = z.double().cpu(), place.long().cpu()
    tokens, k = place.shape
    w = weight.double().cpu() if weight is not None else torch.ones(tokens, k, dtype=torch.float64)
    y, bound = torch.zeros(tokens, z.shape[1], dtype=torch.float64), torch.zeros(tokens, z.shape[1], dtype=torch.float64)
    for j in range(k):
        there = (place[:, j] >= 0) & (place[:, j] < rows)
        part = z[place[there, j]] * w[there, j, None]
        y[there] += part
        bound[there] += (k + 1) * U * part.abs()
    return y, bound


def join_grad(dy, z, place, weight, rows):
    """(dz, bound), (dweight, bound); rows that no choice has are NaN in dz."""
    dy, z, place = dy.double().cpu(), z.double().cpu(), place.long().cpu()
    tokens, k = place.shape
    w = weight.double().cpu() if weight is not None else torch.ones(tokens, k, dtype=torch.float64)
    dz = torch.full(z.shape, float("nan"), dtype=torch.float64)
    dw, bound = torch.zeros(tokens, k, dtype=torch.float64), torch.zeros(tokens, k, dtype=torch.float64)
    for j in range(k):
        there = (place[:, j] >= 0) & (place[:, j] < rows)
        at = place[there, j]
        dz[at] = dy[there] * w[there, j, None]
        dw[there, j] = (dy[there] * z[at]).sum(1)
        bound[there, j] = (z.shape[1] + 2) * U * (dy[there] * z[at]).abs().sum(1)
    return (dz, U * dz.abs()), (dw, bound)


# ---------------------------------------------------------------------------------------------------- dropout

def philox(counter, key):
    """Philox4x32 with ten rounds on Python integers: counter of four words, key of two."""
    c, (k0, k1) = list(counter), key
    for i in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ ((k0 + i * 0x9E3779B9) % 2 ** 32), b % 2 ** 32, (a >> 32) ^ c[3] ^ ((k1 + i * 0xBB67AE85) % 2 ** 32), a % 2 ** 32]
    return c


def drop_bits(rows, features, seed, step, columns=None):
    """The 16 bits of each element of the given rows (whole numbers), [rows, features]."""
    out = np.zeros((len(rows), -(-features // 8) * 8), dtype=np.int64)
    for i, r in enumerate(rows):
        for chunk in range(-(-features // 8)):
            words = philox((chunk | (r >> 32) << 16, r % 2 ** 32, step % 2 ** 32, (step % 2 ** 64) >> 32), (seed % 2 ** 32, seed >> 32))
            out[i, 8 * chunk:8 * chunk + 8] = [(w >> s) & 0xFFFF for w in words for s in (0, 16)]
    return torch.from_numpy(out[:, :features])


def dropout(x, p, residual, bits):
    """(y, bound) for given bits."""
    border = int(math.floor(p * 65536 + 0.5))
    kept = bits >= border
    x = x.double().cpu()
    v = torch.where(kept, x * (65536.0 / (65536 - border) if border < 65536 else 0.0), torch.zeros_like(x))
    y = v + residual.double().cpu() if residual is not None else v
    return y, 2 * U * v.abs() + U * y.abs()
