"""The trainer's dropout: shares that it refuses, seeds of the command's masks.  On the CPU."""
import numpy as np
import pytest

from paper_2212_01185_amd import synth, train


@pytest.mark.parametrize("dropout", [1 - 2.0 ** -17, 0.999995, 1 - 2.0 ** -40, 1 - 2.0 ** -53])
def test_a_share_that_would_be_rounded_to_1_is_refused(dropout):
    with pytest.raises(ValueError, match="dropout"):
        train.Trainer(synth.make_blob(0), dropout=dropout)


@pytest.mark.parametrize("dropout", [0.0, 0.5, 1 - 2.0 ** -16, 1 - 2.0 ** -17 - 2.0 ** -40])
def test_a_share_that_leaves_something_is_taken(dropout, monkeypatch):
    class Taken(Exception):
        pass

    def device(*_):
        raise Taken

    monkeypatch.setattr(train.torch, "device", device)      # what comes behind the checks
    with pytest.raises(Taken):
        train.Trainer(synth.make_blob(0), dropout=dropout)


def _seed_of_the_command(monkeypatch, tmp_path, number):
    class Taken(Exception):
        pass

    def trainer(*args, **kw):
        raise Taken(kw["seed"])

    monkeypatch.setattr(train, "Trainer", trainer)
    np.save(tmp_path / "p.npy", np.zeros((1, 8, 8, 3), dtype=np.uint8))
    with pytest.raises(Taken) as taken:
        train.main([str(tmp_path / "p.npy"), "--out", str(tmp_path / "m.blob"), "--dropout", "0.1", "--seed", str(number)])
    return taken.value.args[0]


def test_runs_of_neighbouring_numbers_share_no_masks(monkeypatch, tmp_path):
    """A hidden layer's masks have the key seed + layer: no two of some runs' keys are the same."""
    seeds = [_seed_of_the_command(monkeypatch, tmp_path, n) for n in list(range(8)) + [100]]
    keys = [(s + layer) % (1 << 64) for s in seeds for layer in range(64)]
    assert all(0 <= s < 1 << 64 for s in seeds) and len(set(keys)) == len(keys)


def test_seeds_of_masks_are_far_apart():
    """mask_seed is linear, so two runs' seeds are as far apart as that of their numbers' difference is from 0; the least of those stand at the
    denominators of the best approximations to its factor's share of 2^64, which the continued fraction gives."""
    far = lambda n: min(train.mask_seed(n), train.mask_seed(-n))  # noqa: E731
    n = np.arange(1, 1 << 20, dtype=np.uint64)
    seeds = n * np.uint64(train.mask_seed(1))
    assert [int(v) for v in seeds[[0, 5, -1]]] == [train.mask_seed(int(v)) for v in n[[0, 5, -1]]]
    assert int(np.minimum(seeds, -seeds).min()) > 1 << 20
    best, (a, b), (q, before) = [], (train.mask_seed(1), 1 << 64), (1, 0)
    while b:
        t = a // b
        a, b, q, before = b, a - t * b, t * q + before if best else 1, q if best else 0
        best.append(q)
    assert any(1 << 33 < q < 1 << 64 for q in best)         # it goes on beyond the differences that are looked at
    assert min(far(q) for q in best if q <= 1 << 33) > 1 << 20
