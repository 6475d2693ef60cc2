"""The trainer's dropout: shares that it refuses.  On the CPU."""
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
