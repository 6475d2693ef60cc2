"""Training of the codec's networks on pictures (the loss Eq. (5)).

A ``Trainer`` holds several networks of one shape, each trained on its own pictures: one per class of pictures, or the candidates of
a sweep.  Every layer of all of them is one product over the pixels of all pictures (``binding.pcc_grouped_linear`` and its backward
pass), the loss and its gradient one call, and one AdamW step moves all tensors.  Weights are kept in fp32 and used, handed
out and stored as bf16, which is what a weight blob holds; activations are rounded to bf16 between layers, the head's outputs are
fp32.

    python -m paper_2212_01185_amd.train pictures.npy --steps 1000 --out model.blob

trains one network on the uint8 pictures [n, H, W, 3] of a NumPy file.
"""
from __future__ import annotations

import argparse
import struct

import numpy as np
import torch

from . import binding, synth


def parse_blob(blob: bytes):
    """(layers [(W[out, in], b[out])], K, neighbourhood size, delay, activation, distribution) of a weight blob."""
    if len(blob) < 64:
        raise ValueError("a weight blob has a header of 64 bytes")
    words = struct.unpack("<16I", blob[:64])
    n = words[2]
    if words[0] != synth.BLOB_MAGIC or words[1] != synth.BLOB_VERSION or not 1 <= n <= 7:
        raise ValueError("not a weight blob")
    dims, at, layers = words[3:4 + n], 64, []
    if len(blob) != 64 + 4 * synth.param_count(dims):
        raise ValueError("a weight blob of %d bytes where its header says %d" % (len(blob), 64 + 4 * synth.param_count(dims)))
    for fan_in, fan_out in zip(dims[:-1], dims[1:]):
        w = np.frombuffer(blob, "<f4", fan_in * fan_out, at).reshape(fan_out, fan_in)
        b = np.frombuffer(blob, "<f4", fan_out, at + 4 * w.size)
        layers.append((w, b))
        at += 4 * (w.size + b.size)
    return (layers,) + tuple(words[11:16])


class Trainer:
    """Networks of one shape under training.  ``blobs``: the weight blobs they start from, one a network."""

    def __init__(self, blobs, device: int = 0, lr: float = 1e-4, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                 state_bits: int = 32, lr_tensor=None):
        blobs = [blobs] if isinstance(blobs, (bytes, bytearray)) else list(blobs)
        parsed = [parse_blob(bytes(b)) for b in blobs]
        if not parsed or any(p[1:] != parsed[0][1:] or [w.shape for w, _ in p[0]] != [w.shape for w, _ in parsed[0][0]] for p in parsed):
            raise ValueError("blobs must be one or more networks of one shape")
        if not eps > 0:
            raise ValueError("eps must be above 0: padded inputs and networks without pictures have moments of 0")
        self.k, self.nbhd, self.delay, self.act, self.dist = parsed[0][1:]
        self.groups, self.device = len(parsed), torch.device("cuda", device)
        self.dims = [parsed[0][0][0][0].shape[1]] + [w.shape[0] for w, _ in parsed[0][0]]
        if self.dims[0] != 3 * self.nbhd or self.dims[-1] != 12 * self.k:
            raise ValueError("a network has 3 inputs a neighbour and 12 outputs a component")
        # inputs are padded with zeros to a multiple of eight; their weights start as zeros and have zero gradients
        self.width = -(-self.dims[0] // 8) * 8
        self.w, self.b, self.w16, self.dw, self.db = [], [], [], [], []
        for layer in range(len(self.dims) - 1):
            w = np.stack([p[0][layer][0] for p in parsed])
            if layer == 0:
                w = np.pad(w, ((0, 0), (0, 0), (0, self.width - self.dims[0])))
            self.w.append(torch.tensor(w, dtype=torch.float32, device=self.device))
            self.b.append(torch.tensor(np.stack([p[0][layer][1] for p in parsed]), dtype=torch.float32, device=self.device))
            self.w16.append(self.w[-1].to(torch.bfloat16))
            self.dw.append(torch.zeros_like(self.w[-1]))
            self.db.append(torch.zeros_like(self.b[-1]))
        # 8-bit states have one scale for 256 elements of a tensor: where a network's share is not whole blocks it is a tensor of its
        # own, so that no network's states hang on another's
        def shares(t):
            return list(t.unbind(0)) if state_bits == 8 and t[0].numel() % binding.STATE_BLOCK else [t]

        lists = [[], [], []]
        for row in list(zip(self.w, self.dw, self.w16)) + [(b, db, None) for b, db in zip(self.b, self.db)]:
            parts = [shares(t) if t is not None else None for t in row]
            for own, part in zip(lists, parts):
                own.extend(part if part is not None else [None] * len(parts[0]))
        self.optimizer = binding.AdamW(lists[0], lists[1], copies=lists[2], state_bits=state_bits, lr=lr, betas=betas, eps=eps,
                                       weight_decay=weight_decay, lr_tensor=lr_tensor)

    def gradients(self, pictures) -> torch.Tensor:
        """Forward and backward pass; the gradients of each network's mean code length are left in ``dw`` and ``db``.

        pictures: for every network a uint8 tensor [n, H, W, 3] or a list of them (either may be empty).  Returns the mean
        bits per sub-pixel of each network's pictures, fp64 [networks] (0 for a network without any)."""
        if self.groups == 1 and isinstance(pictures, torch.Tensor):
            pictures = [pictures]
        pictures = [[p for p in ([own] if isinstance(own, torch.Tensor) else own) if p.numel()] for own in pictures]
        if len(pictures) != self.groups or not any(pictures):
            raise ValueError("pictures must be given for each network, and some for one of them")
        lengths = [sum(int(p.shape[0] * p.shape[1] * p.shape[2]) for p in own) for own in pictures]
        every = [p for own in pictures for p in own]
        rows = sum(lengths)
        x = torch.empty((rows, self.width), dtype=torch.bfloat16, device=self.device)
        at = 0
        for p in every:
            n = int(p.shape[0] * p.shape[1] * p.shape[2])
            binding.pcc_contexts(p, self.nbhd, self.delay, self.width, out=x[at:at + n])
            at += n
        rgb = every[0].reshape(-1, 3) if len(every) == 1 else torch.cat([p.reshape(-1, 3) for p in every])
        counts = torch.tensor(lengths, dtype=torch.int64, device=self.device)
        offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0))
        layers = len(self.w16)
        h = [x]
        for layer in range(layers):
            last = layer + 1 == layers
            h.append(binding.pcc_grouped_linear(h[-1], self.w16[layer], self.b[layer], offsets, binding.PCC_ACT_NONE if last else self.act,
                                                out_dtype=torch.float32 if last else torch.bfloat16))
        weight = torch.repeat_interleave(1.0 / counts.clamp_min(1).to(torch.float32), counts, output_size=rows) if self.groups > 1 else None
        bits, dz = binding.pcc_mixture_loss(h.pop(), rgb, self.dist, 1.0 if self.groups > 1 else 1.0 / rows, weight=weight, grad_dtype=torch.bfloat16)
        for layer in reversed(range(layers)):
            dz, _, _ = binding.pcc_grouped_linear_grad(dz, h.pop(), self.w16[layer], offsets, self.act if layer else binding.PCC_ACT_NONE,
                                                       want_dx=layer > 0, dw=self.dw[layer], db=self.db[layer])
        total = torch.segment_reduce(bits.double(), "sum", lengths=counts)
        return total / (3 * counts.clamp_min(1))

    def step(self, pictures) -> torch.Tensor:
        """One step of the optimizer on these pictures; returns what ``gradients`` does.  (A network without pictures has zero gradients, and
        moves on by what its moments hold.)"""
        bits = self.gradients(pictures)
        self.optimizer.pcc_adamw_step()
        return bits

    def blob(self, network: int = 0) -> bytes:
        """The weight blob of a network as it stands: what ``binding.Codec`` takes."""
        layers = []
        for layer, (w, b) in enumerate(zip(self.w16, self.b)):
            layers.append((w[network, :, :self.dims[layer]].float().cpu().numpy(), b[network].cpu().numpy()))
        return synth.pack_blob(layers, k=self.k, nbhd=self.nbhd, delay=self.delay, act=self.act, dist=self.dist)


def main(argv=None) -> None:
    p = argparse.ArgumentParser(description="Train a coding network on the uint8 pictures [n, H, W, 3] of a NumPy file.")
    p.add_argument("pictures")
    p.add_argument("--out", required=True, help="weight blob to write")
    p.add_argument("--blob", help="weight blob to start from (default: He-initialised)")
    p.add_argument("--network", choices=["workload", "paper", "diagonal"], default="workload")
    p.add_argument("--steps", type=int, default=1000)
    p.add_argument("--batch", type=int, default=64, help="crops a step")
    p.add_argument("--crop", type=int, default=64, help="their height and width at most")
    p.add_argument("--lr", type=float, default=1e-3)
    p.add_argument("--state-bits", type=int, choices=[8, 32], default=32)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    pictures = np.load(a.pictures, allow_pickle=False)
    if pictures.dtype != np.uint8 or pictures.ndim != 4 or pictures.shape[3] != 3 or not pictures.size:
        raise SystemExit("the pictures must be uint8 [n, H, W, 3]")
    if a.blob:
        with open(a.blob, "rb") as f:
            start = f.read()
    else:
        start = {"workload": synth.make_blob, "paper": synth.make_paper_blob, "diagonal": synth.make_diagonal_blob}[a.network](a.seed)
    trainer = Trainer(start, lr=a.lr, state_bits=a.state_bits)
    rng = np.random.default_rng(a.seed)
    n, h, w, _ = pictures.shape
    ch, cw = min(a.crop, h), min(a.crop, w)
    for step in range(a.steps):
        crops = []
        for _ in range(a.batch):
            i, r, c = rng.integers(n), rng.integers(h - ch + 1), rng.integers(w - cw + 1)
            crops.append(pictures[i, r:r + ch, c:c + cw])
        bits = trainer.step(torch.from_numpy(np.stack(crops)).to(trainer.device))
        if step % 100 == 0 or step + 1 == a.steps:
            print("step %d: %.4f bits per sub-pixel" % (step, bits.item()), flush=True)
    with open(a.out, "wb") as f:
        f.write(trainer.blob())


if __name__ == "__main__":
    main()
