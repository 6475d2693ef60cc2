"""The work of a training step of coding networks, as cases that can be timed one by one.

A case names one of four operators: the causal contexts of all pixels as rows (`contexts`), the product of rows with the
weights of their network, several networks at once (`linear`) and its backward pass (`linear_grad`), the code length of
pixels with its gradient (`loss`), and the AdamW step over many tensors (`adamw`).  `listed()` gives the cases that are
always looked at, `draw()` others of the same ranges, `prepare()` what the program has in hand before the call, `run()` the
call: with `own` the framework's entry points, else the operator written with elementary torch operations.  `exact()` is
the operator's definition once more, in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
RELU, LEAKY, NONE = 0, 1, 2          # activation ids: the first two are the weight blob's
ACTS = {"relu": RELU, "leaky": LEAKY, "none": NONE}
SLOPE = 0.01
BLOCK = 256                          # elements of an 8-bit state that share a scale

# Weight and bias sizes of the nine networks that the codec takes: layer widths.
NETWORKS = [(30, 160, 160, 128, 60), (36, 128, 128, 128, 128, 36), (36, 128, 128, 128, 36), (36, 64, 64, 64, 64, 36),
            (36, 128, 128, 128, 128, 60), (36, 128, 128, 128, 128, 84), (36, 128, 128, 128, 128, 128, 36), (36, 192, 192, 192, 192, 36)]

# A drawn case stays within the largest listed ones.
MOST_PIXELS, MOST_FLOPS, MOST_BYTES, MOST_LOSS, MOST_ELEMENTS = 24 * 768 * 512, 6.8e10, 3.7e8, 2048 * 1365, 1 << 25


def _contexts(name, n, h, w, nbhd, delay):
    return {"name": name, "op": "contexts", "n": n, "h": h, "w": w, "nbhd": nbhd, "delay": delay}


def _linear(name, op, rows, groups, fan_in, fan_out, act, dtype="bf16", y="same", spread=0.0, empty=False, tail=0, dx=True):
    return {"name": name, "op": op, "rows": rows, "groups": groups, "in": fan_in, "out": fan_out, "act": act, "dtype": dtype, "y": y,
            "spread": spread, "empty": empty, "tail": tail, "dx": dx}


def _loss(name, count, k, dist, grad, masked):
    return {"name": name, "op": "loss", "count": count, "k": k, "dist": dist, "grad": grad, "masked": masked}


def _adamw(name, tensors, elements, bits, grad="fp32", copy="bf16"):
    return {"name": name, "op": "adamw", "tensors": tensors, "elements": elements, "bits": bits, "grad": grad, "copy": copy}


def listed():
    return [
        # one small crop, as in a step on a few crops: latency is all there is
        _contexts("contexts 64x64", 1, 64, 64, 10, 2),
        # the inputs of an epoch's chunk: a batch of photographs, the order with copied neighbours
        _contexts("contexts 24 of 768x512 diagonal", 24, 512, 768, 12, 1),
        # three networks, one of them without a pixel in this step, the others with a handful: the smallest call
        _linear("linear 7 pixels, 3 networks", "linear", 7, 3, 32, 160, "relu", spread=1.0, empty=True, tail=2),
        # a hidden layer of the measured workloads' network on all pixels of a photograph
        _linear("linear 768x512, 160 to 160", "linear", 768 * 512, 1, 160, 160, "relu"),
        # sixteen wide experts with ragged shares of 8,192 rows
        _linear("linear 16 experts, 1024 to 4096", "linear", 8192, 16, 1024, 4096, "none", spread=0.3, tail=100),
        # the head of four networks of the paper's shape that train on a few crops each
        _linear("linear grad 4 networks, 128 to 36", "linear_grad", 4 * 64 * 64, 4, 128, 36, "leaky", spread=0.5),
        # a hidden layer on all pixels of a photograph
        _linear("linear grad 768x512, 160 to 160", "linear_grad", 768 * 512, 1, 160, 160, "relu"),
        # sixteen wide experts, half precision
        _linear("linear grad 16 experts, 1024 to 2048", "linear_grad", 8192, 16, 1024, 2048, "relu", dtype="fp16", spread=0.3, tail=100),
        # one crop, padded to its rectangle, the ablation's other distribution, gradients for a backward pass in 32 bits
        _loss("loss 64x64 logistic, padded", 64 * 64, 3, "logistic", "fp32", True),
        # a large picture, gradients for the backward pass above
        _loss("loss 2048x1365", 2048 * 1365, 5, "gaussian", "bf16", False),
        # all tensors of the networks that the codec takes, trained side by side with small states
        _adamw("adamw 8 networks, 8 bits", 0, 0, 8),
        # many tensors of very different sizes, states in 32 bits
        _adamw("adamw 300 tensors, 32 bits", 300, 1 << 25, 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["contexts", "linear", "linear", "linear_grad", "linear_grad", "loss", "loss", "adamw", "adamw"])
    if op == "contexts":
        h, w = _log_int(rng, 1, 2160), _log_int(rng, 1, 4096)
        nbhd, delay = rng.choice([(10, 2), (12, 3), (12, 1)])
        return {k: v for k, v in _contexts("", min(MOST_PIXELS // (h * w), _log_int(rng, 1, 24)), h, w, nbhd, delay).items() if k != "name"}
    if op in ("linear", "linear_grad"):
        if rng.random() < 0.5:
            dims = rng.choice(NETWORKS)
            at = rng.randrange(len(dims) - 1)
            fan_in, fan_out = dims[at], dims[at + 1]
            if at == 0 and rng.random() < 0.7:
                fan_in = -(-fan_in // 8) * 8         # the contexts' rows as the trainer lays them out
        else:
            fan_in, fan_out = _log_int(rng, 8, 2048), _log_int(rng, 8, 2048)
            if rng.random() < 0.7:
                fan_in, fan_out = -(-fan_in // 8) * 8, -(-fan_out // 8) * 8
        groups = _log_int(rng, 1, 64)
        most = min(MOST_FLOPS / (2 * fan_in * fan_out * (2 if op == "linear_grad" else 1)), MOST_BYTES / (2 * (2 * fan_in + 2 * fan_out)), 400000)
        rows = _log_int(rng, 1, max(1, int(most)))
        act = rng.choice(["relu", "leaky", "none"])
        c = _linear("", op, rows, groups, fan_in, fan_out, act, rng.choice(["bf16", "bf16", "fp16"]),
                    rng.choice(["same", "same", "fp32"]) if op == "linear" else "same", rng.choice([0.0, 0.3, 0.6]),
                    groups > 1 and rng.random() < 0.3, rng.choice([0, 0, 1, 77]), op == "linear" or rng.random() < 0.8)
    elif op == "loss":
        c = _loss("", _log_int(rng, 1, MOST_LOSS), rng.choice([3, 5, 7]), rng.choice(["gaussian", "gaussian", "logistic"]),
                  rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.4)
    else:
        elements = _log_int(rng, 1000, MOST_ELEMENTS)
        c = _adamw("", _log_int(rng, 1, min(400, elements)), elements, rng.choice([8, 32]), rng.choice(["fp32", "fp32", "bf16"]),
                   rng.choice(["bf16", "bf16", "fp16", "none"]))
    return {k: v for k, v in c.items() if k != "name"}


# ---------------------------------------------------------------------------------------------------- inputs

def _pictures(gen, n, h, w):
    """Smooth pictures with some noise: neighbouring pixels are near each other, as in photographs."""
    dev = torch.device("cuda")
    y = torch.linspace(0, 1, h, device=dev).view(1, h, 1, 1)
    x = torch.linspace(0, 1, w, device=dev).view(1, 1, w, 1)
    f = torch.rand(4, n, 1, 1, 3, generator=gen, device=dev)
    img = 128 + 90 * torch.sin(12 * f[0] * x + 6 * f[1]) * torch.cos(9 * f[2] * y + 6 * f[3])
    img = img + 3 * torch.randn(n, h, w, 3, generator=gen, device=dev)
    return img.round_().clamp_(0, 255).to(torch.uint8)


def _lengths(case, seed):
    """Rows of each group: equal shares, or shares whose logarithm is spread."""
    rng, groups, rows = np.random.RandomState(seed % (1 << 31)), case["groups"], case["rows"]
    share = np.exp(case["spread"] * rng.randn(groups))
    if case["empty"]:
        share[1] = 0.0
    at = np.floor(np.cumsum(share) / share.sum() * rows + 0.5).astype(np.int64)
    at[-1] = rows
    return np.diff(np.concatenate([[0], at]))


def _activated(x, act):
    return torch.where(x < 0, x * (0.0 if act == RELU else SLOPE), x) if act != NONE else x


def _tensor_sizes(case):
    if case["tensors"] == 0:
        return [s for d in NETWORKS for i, o in zip(d[:-1], d[1:]) for s in (i * o, o)]
    rng = np.random.RandomState(1000 + case["tensors"])
    share = np.exp(2.0 * rng.randn(case["tensors"]))
    return [max(1, int(s)) for s in np.floor(share / share.sum() * case["elements"])]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 7919 + 17)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev)  # noqa: E731
    s = {"case": dict(case)}
    if case["op"] == "contexts":
        s["img"] = _pictures(gen, case["n"], case["h"], case["w"])
        s["width"] = -(-3 * case["nbhd"] // 8) * 8
    elif case["op"] in ("linear", "linear_grad"):
        lengths = _lengths(case, int(seed))
        dt, act = DTYPES[case["dtype"]], ACTS[case["act"]]
        rows, fan_in, fan_out = case["rows"] + case["tail"], case["in"], case["out"]
        s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)])).to(dev)
        s["longest"] = int(lengths.max())            # the program that dealt out the rows knows it
        s["w"] = (normal(case["groups"], fan_out, fan_in) * math.sqrt(2.0 / fan_in)).to(dt)
        if case["op"] == "linear":
            s["x"] = normal(rows, fan_in).to(dt)
            s["bias"] = normal(case["groups"], fan_out) * 0.1
            s["y"] = torch.zeros(rows, fan_out, dtype=torch.float32 if case["y"] == "fp32" else dt, device=dev)
        else:
            s["x"] = _activated(normal(rows, fan_in), act).to(dt)
            s["dz"] = (normal(rows, fan_out) * 0.01).to(dt)
            s["dx"] = torch.zeros(rows, fan_in, dtype=dt, device=dev) if case["dx"] else None
    elif case["op"] == "loss":
        count, k = case["count"], case["k"]
        side = max(1, int(math.sqrt(count)))
        s["rgb"] = _pictures(gen, 1, -(-count // side), side).reshape(-1, 3)[:count].contiguous()
        # what a network under training answers: means near the pixel and further off, widths from a fraction of a
        # level to the whole range, some beyond the clamp; coupling coefficients around zero
        mean = s["rgb"].float()[:, :, None] / 256 + 0.1 * normal(count, 3, k)
        log_sigma = normal(count, 3, k) * 1.5 - 3.5
        head = torch.stack([normal(count, 3, k), mean, log_sigma], 2).reshape(count, 9 * k)
        s["params"] = torch.cat([head, 0.1 * normal(count, 3 * k)], 1).contiguous()
        s["scale"] = 1.0 / 64 if case["grad"] == "fp16" else 1.0 / count      # half precision: the program scales its loss
        s["weight"] = None
        if case["masked"]:                           # pixels of the padding: weight zero, and whatever the network made of them
            keep = torch.rand(count, generator=gen, device=dev) < 0.8
            s["weight"] = torch.where(keep, 0.5 + torch.rand(count, generator=gen, device=dev), torch.zeros((), device=dev))
            s["params"][~keep] = float("nan")
    else:
        sizes = _tensor_sizes(case)
        starts = np.concatenate([[0], np.cumsum([-(-n // BLOCK) * BLOCK for n in sizes])])
        total = int(starts[-1])
        spans = [(int(a), int(n)) for a, n in zip(starts[:-1], sizes)]
        inside = torch.zeros(total + 1, device=dev)
        at = torch.tensor([a for a, _ in spans], device=dev)
        inside.index_add_(0, at, torch.ones(len(spans), device=dev))
        inside.index_add_(0, at + torch.tensor(sizes, device=dev), -torch.ones(len(spans), device=dev))
        inside = inside.cumsum(0)[:total] > 0.5      # one flat buffer for all tensors, each from a multiple of 256 on
        flat = lambda v: torch.where(inside, v, torch.zeros((), device=dev))  # noqa: E731
        s["hyper"] = {"lr": 1e-3, "betas": (0.9, 0.999), "eps": 1e-8, "weight_decay": 0.01}
        s["param"] = flat(0.1 * normal(total))
        s["grad"] = flat(1e-3 * torch.exp(normal(total)) * normal(total)).to(DTYPES[case["grad"]])
        s["copy"] = s["param"].to(DTYPES[case["copy"]]) if case["copy"] != "none" else None
        s["step"] = torch.full((1,), 10, dtype=torch.int64, device=dev)
        m, u = flat(3e-4 * normal(total)), flat(1e-3 * torch.exp(normal(total)))
        if case["bits"] == 32:
            s["m"], s["v"] = m, u * u
        else:                                        # codes of earlier steps
            for name, x in (("m", m), ("v", u)):
                scale = x.abs().view(-1, BLOCK).amax(1) * (1.0 / 448.0)
                code = (x.view(-1, BLOCK) / scale[:, None].clamp_min(1e-30)).clamp(-448, 448).to(torch.float8_e4m3fn)
                s[name], s[name + "_scale"] = code.view(-1), scale
        if own:
            from paper_2212_01185_amd import binding
            part = lambda t: [t[a:a + n] for a, n in spans] if t is not None else None  # noqa: E731
            blocks = lambda t: [t[a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in spans] if t is not None else None  # noqa: E731
            s["optimizer"] = binding.AdamW(part(s["param"]), part(s["grad"]), copies=part(s["copy"]), state_bits=case["bits"], step=s["step"],
                                           m=part(s["m"]), v=part(s["v"]), m_scale=blocks(s.get("m_scale")), v_scale=blocks(s.get("v_scale")),
                                           **s["hyper"])
    return s


# ---------------------------------------------------------------------------------------------------- one pass

def _shifted(img, dr, dc):
    """img[:, r + dr, c + dc], 0 outside, for dr <= 0."""
    n, h, w, _ = img.shape
    p = torch.zeros(n, h - dr, w + 4, 3, dtype=img.dtype, device=img.device)
    p[:, -dr if dr else 0:, 2:2 + w] = img
    return p[:, :h, 2 + dc:2 + dc + w]


def _taps(nbhd, delay):
    reach = 1 if nbhd == 10 else 2
    taps = [(dr, dc) for dr in (-2, -1) for dc in range(-2, reach + 1)] + [(0, -2), (0, -1)]
    # diagonal order: what is not decoded yet is read as the pixel above
    return [(-1, 0) if delay == 1 and t in ((-2, 2), (-1, 1), (-1, 2)) else t for t in taps]


def _plain_contexts(s):
    img = s["img"]
    taps = [_shifted(img, dr, dc) for dr, dc in _taps(s["case"]["nbhd"], s["case"]["delay"])]
    x = torch.cat(taps, 3).reshape(-1, 3 * len(taps)).float() / 256
    return torch.nn.functional.pad(x, (0, s["width"] - x.shape[1])).to(torch.bfloat16)


def _by_group(s, x):
    """(rows of each group side by side [G, longest, .] in 32 bits, zeros behind the last; which places hold a row; their row)."""
    off = s["offsets"]
    row = off[:-1, None] + torch.arange(s["longest"], device=off.device)
    there = row < off[1:, None]
    row = torch.where(there, row, torch.zeros_like(row))
    return torch.where(there[:, :, None], x[row].float(), torch.zeros((), device=off.device)), there, row


def _plain_linear(s):
    x, there, row = _by_group(s, s["x"])
    y = torch.bmm(x, s["w"].float().transpose(1, 2).contiguous()) + s["bias"][:, None]
    s["y"][row[there]] = _activated(y, ACTS[s["case"]["act"]])[there].to(s["y"].dtype)
    return s["y"]


def _plain_linear_grad(s):
    act = ACTS[s["case"]["act"]]
    x, there, row = _by_group(s, s["x"])
    dz, _, _ = _by_group(s, s["dz"])
    if s["dx"] is not None:
        dx = torch.bmm(dz, s["w"].float())
        if act != NONE:
            dx = torch.where(x > 0, dx, dx * (0.0 if act == RELU else SLOPE))
        s["dx"][row[there]] = dx[there].to(s["dx"].dtype)
    dw = torch.bmm(dz.transpose(1, 2).contiguous(), x)
    out = {"dw": dw, "db": dz.sum(1)}
    return dict(out, dx=s["dx"]) if s["dx"] is not None else out


def _plain_loss(s):
    # in 64 bits: a probability is the difference of the distribution's values at neighbouring borders, which 32 bits
    # cannot hold against the one count of 65,536 that every level has at least
    k, dist = s["case"]["k"], s["case"]["dist"]
    o, x = s["params"].double(), s["rgb"].double()[:, :, None]
    head, coef = o[:, :9 * k].view(-1, 3, 3, k), o[:, 9 * k:].view(-1, 3, k)
    r, g, none = x[:, 0:1] / 256, x[:, 1:2] / 256, torch.zeros_like(coef[:, 0:1])
    mu = head[:, :, 1] + torch.cat([none, coef[:, 0:1] * r, coef[:, 1:2] * r + coef[:, 2:3] * g], 1)
    ls = head[:, :, 2]
    sigma = torch.exp(ls.clamp(-8, 4))
    a, b = ((x - 0.5) / 256 - mu) / sigma, ((x + 0.5) / 256 - mu) / sigma
    first, last = x == 0, x == 255
    zero = torch.zeros((), dtype=o.dtype, device=o.device)
    if dist == "gaussian":
        low, high = (0.5 * torch.special.erfc(z * -math.sqrt(0.5)) for z in (a, b))
        fa, fb = (torch.exp(z * z * -0.5) * (1 / math.sqrt(2 * math.pi)) for z in (a, b))
    else:
        low, high = torch.sigmoid(a), torch.sigmoid(b)
        fa, fb = low * (1 - low), high * (1 - high)
    q = torch.where(last, zero + 1, high) - torch.where(first, zero, low)
    fa, fb = torch.where(first, zero, fa), torch.where(last, zero, fb)
    pi = torch.softmax(head[:, :, 0], 2)
    p = (pi * q).sum(2, keepdim=True)
    bits = -torch.log2((65280 * p + 1) / 65536).sum((1, 2))
    outer = -65280 / ((65280 * p + 1) * math.log(2)) * s["scale"]
    if s["weight"] is not None:
        outer = outer * s["weight"].double()[:, None, None]
    d_logit = outer * pi * (q - p)
    d_mu = outer * pi * (fa - fb) / sigma
    d_ls = torch.where((ls < -8) | (ls > 4), zero, outer * pi * (a * fa - b * fb))
    grad = torch.cat([torch.stack([d_logit, d_mu, d_ls], 2).reshape(-1, 9 * k), (d_mu[:, 1:2] * r).view(-1, k),
                      (d_mu[:, 2:3] * r).view(-1, k), (d_mu[:, 2:3] * g).view(-1, k)], 1)
    if s["weight"] is not None:
        used = s["weight"] != 0
        bits, grad = torch.where(used, bits, zero), torch.where(used[:, None], grad, zero)
    return {"bits": bits.float(), "grad": grad.to(DTYPES[s["case"]["grad"]])}


def _dither(step, which):
    """20 bits for each place of a block, fixed by the place and the step's number: how much of a code's step is added before
    the value is cut to its code.  Over the steps every place sees all amounts, so a moment that changes by less than a step
    of its code moves all the same."""
    low = 0xFFFFFFFF
    h = (torch.arange(BLOCK, device=step.device) * 0x9E3779B9 + step * 0xB7E15163) & low
    h = h ^ (h >> 15)
    h = (h * 0x6A09E667) & low
    h = h ^ (h >> 13)
    h = (h * 0x9E3779B9) & low
    h = h ^ (h >> 16)
    return ((h if which == "m" else (h * 0xB7E15163) & low) >> 12).to(torch.int32)


def _to_codes(x, step, which):
    """Blocks of 256 as e4m3 codes and a scale each.  A second moment above zero never gets the code of zero: the step divides by it."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) * (1.0 / 448.0)
    inverse = torch.where(scale >= 2.0 ** -100, (1 / scale.double()).float(), torch.zeros_like(scale))
    y, d = x.abs() * inverse[:, None], _dither(step, which)
    code = torch.where(y >= 2.0 ** -6, ((y.view(torch.int32) + d) >> 20) - (120 << 3), (y * 512 + d.float() * 2.0 ** -20).to(torch.int32))
    code = code.clamp_max(0x7E)
    code = torch.where((x > 0) & (code == 0), torch.ones_like(code), code) if which == "v" else code + (x < 0).to(torch.int32) * 128
    return code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1), scale


def _from_codes(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _plain_adamw(s):
    (b1, b2), lr = s["hyper"]["betas"], s["hyper"]["lr"]
    small = s["case"]["bits"] == 8
    s["step"] += 1
    t = s["step"].double()
    correct1, correct2 = 1 - b1 ** t, 1 - b2 ** t
    g = s["grad"].float()
    m = _from_codes(s["m"], s["m_scale"]) if small else s["m"]
    v = _from_codes(s["v"], s["v_scale"]).square() if small else s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * (1 - b2)) * g
    root = torch.sqrt(v.double()).float()
    denom = root * (1 / torch.sqrt(correct2)).float() + s["hyper"]["eps"]
    s["param"].copy_(s["param"] * (1 - lr * s["hyper"]["weight_decay"]) - (lr / correct1).float() * (m / denom))
    if small:
        for name, x in (("m", m), ("v", root)):
            code, scale = _to_codes(x, s["step"], name)
            s[name].view(torch.uint8).copy_(code.view(torch.uint8))
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(s["param"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("param", "copy", "m", "v", "m_scale", "v_scale", "step") if s.get(k) is not None}


def _own(s):
    from paper_2212_01185_amd import binding
    case = s["case"]
    if case["op"] == "contexts":
        return binding.pcc_contexts(s["img"], case["nbhd"], case["delay"], s["width"])
    if case["op"] == "linear":
        return binding.pcc_grouped_linear(s["x"], s["w"], s["bias"], s["offsets"], ACTS[case["act"]], out=s["y"])
    if case["op"] == "linear_grad":
        dx, dw, db = binding.pcc_grouped_linear_grad(s["dz"], s["x"], s["w"], s["offsets"], ACTS[case["act"]], dx=s["dx"], want_dx=case["dx"])
        return {"dw": dw, "db": db, "dx": dx} if case["dx"] else {"dw": dw, "db": db}
    if case["op"] == "loss":
        bits, grad = binding.pcc_mixture_loss(s["params"], s["rgb"], 0 if case["dist"] == "gaussian" else 1, s["scale"], weight=s["weight"],
                                              grad_dtype=DTYPES[case["grad"]])
        return {"bits": bits, "grad": grad}
    s["optimizer"].pcc_adamw_step()
    return _adamw_outputs(s)


def run(state):
    if own:
        return _own(state)
    return {"contexts": _plain_contexts, "linear": _plain_linear, "linear_grad": _plain_linear_grad, "loss": _plain_loss,
            "adamw": _plain_adamw}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------- 64 bits

def _exact_loss(s):
    """Code length by logarithms of the distribution's two tails, gradients by automatic differentiation."""
    k, dist = s["case"]["k"], s["case"]["dist"]
    used = torch.ones(len(s["rgb"]), dtype=torch.bool, device="cuda") if s["weight"] is None else s["weight"] != 0
    o = torch.where(used[:, None], s["params"], torch.zeros((), device="cuda")).double().requires_grad_(True)
    level = s["rgb"].double()
    total = 0.0
    tail = (lambda z: 0.5 * torch.special.erfc(z / math.sqrt(2.0))) if dist == "gaussian" else (lambda z: torch.sigmoid(-z))
    for c in range(3):
        logit, mean, ls = (o[:, 3 * k * c + k * i:3 * k * c + k * (i + 1)] for i in range(3))
        if c == 1:
            mean = mean + o[:, 9 * k:10 * k] * level[:, 0:1] / 256
        if c == 2:
            mean = mean + o[:, 10 * k:11 * k] * level[:, 0:1] / 256 + o[:, 11 * k:] * level[:, 1:2] / 256
        x = level[:, c:c + 1]
        inverse = torch.exp(-torch.clamp(ls, -8.0, 4.0))
        mid = (x / 256 - mean) * inverse
        half = inverse / 512
        side = torch.where(mid < 0, -1.0, 1.0)       # mass between two borders as a difference of the nearer tail
        near, far = side * mid - half, side * mid + half
        lowest, highest = x == 0, x == 255
        open_near = torch.where(side > 0, lowest, highest)
        open_far = torch.where(side > 0, highest, lowest)
        mass = torch.where(open_near, torch.ones_like(near), tail(near)) - torch.where(open_far, torch.zeros_like(far), tail(far))
        p = (torch.exp(logit - torch.logsumexp(logit, 1, keepdim=True)) * mass).sum(1)
        total = total + 16.0 - torch.log(65280.0 * p + 1.0) / math.log(2.0)
    weight = torch.ones_like(total) if s["weight"] is None else s["weight"].double()
    (grad,) = torch.autograd.grad((total * weight).sum() * s["scale"], o)
    keep = used.double()
    return {"bits": total.detach() * keep, "grad": grad * keep[:, None]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "contexts":
        n, h, w, _ = s["img"].shape
        r, c = torch.arange(h, device="cuda")[:, None], torch.arange(w, device="cuda")[None]
        out = torch.zeros(n, h, w, s["width"], dtype=torch.float32, device="cuda")      # eight bits: exact in any type
        for j, (dr, dc) in enumerate(_taps(case["nbhd"], case["delay"])):
            ok = (r + dr >= 0) & (c + dc >= 0) & (c + dc < w)
            out[..., 3 * j:3 * j + 3] = s["img"][:, (r + dr).clamp(0, h - 1), (c + dc).clamp(0, w - 1)] * ok[..., None] / 256.0
        return out.view(-1, s["width"])
    if case["op"] in ("linear", "linear_grad"):
        off, act = s["offsets"].tolist(), ACTS[case["act"]]
        x, w = s["x"].double(), s["w"].double()
        slope = {RELU: 0.0, LEAKY: SLOPE, NONE: 1.0}[act]
        if case["op"] == "linear":
            y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
            for g, (lo, hi) in enumerate(zip(off, off[1:])):
                z = x[lo:hi] @ w[g].T + s["bias"][g].double()
                y[lo:hi] = torch.maximum(z, torch.zeros_like(z)) + slope * torch.minimum(z, torch.zeros_like(z))
            return y
        dz, dw, dx = s["dz"].double(), torch.zeros_like(w), torch.zeros_like(x)
        db = torch.zeros(w.shape[:2], dtype=torch.float64, device="cuda")
        for g, (lo, hi) in enumerate(zip(off, off[1:])):
            dw[g], db[g] = dz[lo:hi].T @ x[lo:hi], dz[lo:hi].sum(0)
            dx[lo:hi] = (dz[lo:hi] @ w[g]) * ((x[lo:hi] > 0).double() * (1 - slope) + slope)
        return {"dw": dw, "db": db, "dx": dx} if case["dx"] else {"dw": dw, "db": db}
    if case["op"] == "loss":
        return _exact_loss(s)
    (b1, b2), lr, t = s["hyper"]["betas"], s["hyper"]["lr"], 11
    g = s["grad"].double()
    if case["bits"] == 8:
        m = (s["m"].double().view(-1, BLOCK) * s["m_scale"].double()[:, None]).view(-1)
        v = (s["v"].double().view(-1, BLOCK) * s["v_scale"].double()[:, None]).view(-1) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = s["param"].double()
    p = p - lr * s["hyper"]["weight_decay"] * p - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + s["hyper"]["eps"])
    out = {"param": p, "copy": p if s["copy"] is not None else None, "step": s["step"] + 1}
    if case["bits"] == 32:
        return dict(out, m=m, v=v)
    return dict(out, m=None, v=None, m_scale=None, v_scale=None)     # a code is defined by its rounding, not by a value in 64 bits


def work(case):
    if case["op"] == "contexts":
        pixels = case["n"] * case["h"] * case["w"]
        return {"bytes": pixels * (3 + 2 * (-(-3 * case["nbhd"] // 8) * 8)), "flops": 0}
    if case["op"] in ("linear", "linear_grad"):
        rows, a, b, g = case["rows"], case["in"], case["out"], case["groups"]
        if case["op"] == "linear":
            return {"bytes": rows * (2 * a + (4 if case["y"] == "fp32" else 2) * b) + g * b * (2 * a + 4), "flops": 2 * rows * a * b}
        return {"bytes": rows * 2 * (a + b + (a if case["dx"] else 0)) + g * b * (4 * a + 4 + (2 * a if case["dx"] else 0)),
                "flops": (4 if case["dx"] else 2) * rows * a * b}
    if case["op"] == "loss":
        outputs = 12 * case["k"]
        return {"bytes": case["count"] * (4 * outputs + 3 + 4 + outputs * (4 if case["grad"] == "fp32" else 2) + (4 if case["masked"] else 0)),
                "flops": case["count"] * 3 * case["k"] * 100}
    n = sum(_tensor_sizes(case))
    each = 8 + (4 if case["grad"] == "fp32" else 2) + (0 if case["copy"] == "none" else 2) + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": n * each, "flops": n * 15}
