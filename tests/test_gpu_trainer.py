"""Training steps of the codec's networks as a user takes them.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding, synth, train

pytestmark = pytest.mark.gpu

BLOBS = {"workload": lambda s: synth.make_blob(s), "paper": lambda s: synth.make_paper_blob(s), "diagonal": lambda s: synth.make_diagonal_blob(s),
         "logistic": lambda s: synth.make_blob(s, dist=synth.DIST_LOGISTIC)}
BLOBS.update({name: (lambda shape: lambda s: synth.make_ablation_blob(*shape, seed=s))(shape) for name, shape in synth.ABLATION_SHAPES.items()})


def _picture(seed, h=40, w=33, n=1):
    return np.stack([synth.make_image(seed + i, synth.ImageSpec(w, h, 4, 3.0, 12.0)) for i in range(n)])


def _bf16(x):
    return x.to(torch.bfloat16).to(x.dtype)


def _reference(blob, img):
    """Gradients of the mean code length in 64 bits, rounded to bf16 where the trainer rounds: activations and the gradients before them."""
    layers, k, nbhd, delay, act, dist = train.parse_blob(blob)
    h = [torch.from_numpy(ref.contexts(img, nbhd, delay))]
    for i, (w, b) in enumerate(layers):
        z = h[-1] @ torch.from_numpy(w.astype(np.float64)).T + torch.from_numpy(b.astype(np.float64))
        h.append(z if i + 1 == len(layers) else _bf16(ref.activate(z, act)))
    rgb = torch.from_numpy(img.reshape(-1, 3))
    bits = ref.code_length(h[-1], rgb, k, dist)
    dz, _ = ref.loss_gradient(h[-1], rgb, k, dist, 1.0 / len(rgb))
    dz = _bf16(dz)
    out = []
    for i in reversed(range(len(layers))):
        out.append((dz.T @ h[i], dz.sum(0)))
        dz = _bf16((dz @ torch.from_numpy(layers[i][0].astype(np.float64))) * ref.derivative(h[i], act if i else ref.NONE))
    return bits.mean().item() / 3, out[::-1]


# The trainer's sums are in fp32, so a value next to a border of bf16 may be rounded to the other side: one in a few hundred (a sum of 200
# products is off by some 2^-22 of its size, a step is 2^-8), and each such value is off by 2^-8.  As independent errors that is
# 2^-8 * sqrt(1 / 300) = 2.3e-4 of a layer's values, and six layers of it are 6e-4 of a gradient's norm; 2e-3 leaves a factor of three.
NEAR = 2e-3


@pytest.mark.parametrize("name", sorted(BLOBS))
def test_gradients_of_each_network(name):
    blob = BLOBS[name](3)
    img = _picture(5)
    trainer = train.Trainer(blob)
    bits = trainer.gradients(torch.from_numpy(img).cuda())
    want_bits, want = _reference(blob, img)
    assert abs(bits.item() - want_bits) <= NEAR * want_bits
    for i, (dw, db) in enumerate(want):
        got = trainer.dw[i][0].double().cpu()
        assert (got[:, dw.shape[1]:] == 0).all()
        assert (got[:, :dw.shape[1]] - dw).norm() <= NEAR * dw.norm(), i
        assert (trainer.db[i][0].double().cpu() - db).norm() <= NEAR * db.norm(), i
    assert trainer.blob() == blob                    # nothing has moved, and a blob comes back as it was


def test_gradient_along_its_direction_against_differences():
    """The loss a small step along the head's bias gradient and against it, with the codec's own network evaluation in 64 bits."""
    blob = synth.make_blob(4)
    img = _picture(8)
    trainer = train.Trainer(blob)
    trainer.gradients(torch.from_numpy(img).cuda())
    layers, k, nbhd, delay, act, dist = train.parse_blob(blob)
    d = trainer.db[-1][0].double().cpu()
    h = torch.from_numpy(ref.contexts(img, nbhd, delay))
    for i, (w, b) in enumerate(layers[:-1]):
        h = _bf16(ref.activate(h @ torch.from_numpy(w.astype(np.float64)).T + torch.from_numpy(b.astype(np.float64)), act))
    z = h @ torch.from_numpy(layers[-1][0].astype(np.float64)).T + torch.from_numpy(layers[-1][1].astype(np.float64))
    rgb = torch.from_numpy(img.reshape(-1, 3))
    e = 1e-6 / d.norm()
    slope = (ref.code_length(z + e * d, rgb, k, dist).mean() - ref.code_length(z - e * d, rgb, k, dist).mean()) / (2 * e)
    assert abs(slope.item() / (d * d).sum().item() - 1) <= 2 * NEAR       # d itself is within NEAR, and so is d . d


@pytest.mark.parametrize("state_bits", [32, 8])
def test_networks_side_by_side(state_bits):
    """Three networks, one of them without pictures this time: each has the gradients that it has alone, and moves by them."""
    blobs = [synth.make_blob(s) for s in (1, 2, 3)]
    pictures = [torch.from_numpy(_picture(20, 50, 30, 2)).cuda(), [], [torch.from_numpy(_picture(30, 17, 23)).cuda(), torch.from_numpy(_picture(31, 9, 64)).cuda()]]
    together = train.Trainer(blobs, state_bits=state_bits, lr=1e-3)
    bits = together.gradients(pictures)
    assert bits[1] == 0 and all((d[1] == 0).all() for d in together.dw + together.db)
    for g in (0, 2):
        alone = train.Trainer(blobs[g], state_bits=state_bits, lr=1e-3)
        own = alone.gradients([pictures[g]])
        # the loss's gradient is scaled by a weight or a factor before it is rounded to bf16, and sums have other chunks
        assert abs(own.item() / bits[g].item() - 1) <= 1e-6
        for a, b in zip(alone.dw + alone.db, together.dw + together.db):
            assert (a[0] - b[g]).norm() <= NEAR * a[0].norm()
    before = [w.clone() for w in together.w]
    together.step(pictures)
    for old, new, copy in zip(before, together.w, together.w16):
        assert not torch.equal(old[0], new[0]) and torch.equal(old[1], new[1]) and not torch.equal(old[2], new[2])
        assert torch.equal(copy, new.to(torch.bfloat16))
    assert (together.w[0][:, :, 30:] == 0).all()


def test_a_trained_network_codes():
    """What a few steps make is a blob that the codec takes, codes with and decodes."""
    trainer = train.Trainer([synth.make_blob(1), synth.make_blob(2)], lr=1e-3)
    img = _picture(40, 64, 64, 2)
    for _ in range(5):
        bits = trainer.step([torch.from_numpy(img[:1]).cuda(), torch.from_numpy(img[1:]).cuda()])
    assert bits.shape == (2,) and torch.isfinite(bits).all()
    for g in range(2):
        codec = binding.Codec(trainer.blob(g), 0)
        d = torch.from_numpy(img).cuda()
        out = codec.pcc_decode(codec.pcc_encode(d), 2, 64, 64)
        torch.cuda.synchronize()
        assert torch.equal(out, d)
        codec.close()


def test_the_command(tmp_path):
    np.save(tmp_path / "p.npy", _picture(50, 24, 24, 3))
    train.main([str(tmp_path / "p.npy"), "--out", str(tmp_path / "m.blob"), "--steps", "3", "--batch", "4", "--crop", "16", "--network", "paper", "--state-bits", "8"])
    blob = (tmp_path / "m.blob").read_bytes()
    assert len(train.parse_blob(blob)[0]) == 5
    binding.Codec(blob, 0).close()
    with pytest.raises(SystemExit):
        np.save(tmp_path / "q.npy", np.zeros((2, 3), np.float32))
        train.main([str(tmp_path / "q.npy"), "--out", str(tmp_path / "m.blob")])


def test_refusals():
    with pytest.raises(ValueError):
        train.Trainer([])
    with pytest.raises(ValueError):
        train.Trainer([synth.make_blob(0), synth.make_paper_blob(0)])
    with pytest.raises(ValueError):
        train.Trainer(synth.make_blob(0)[:-4])
    trainer = train.Trainer([synth.make_blob(0), synth.make_blob(1)])
    with pytest.raises(ValueError):
        trainer.gradients([torch.zeros(1, 4, 4, 3, dtype=torch.uint8, device="cuda")])
    with pytest.raises(ValueError):
        trainer.gradients([[], []])
    with pytest.raises(ValueError):
        trainer.gradients([torch.zeros(1, 4, 4, 3, dtype=torch.uint8), []])
