"""The encoder's choice of mixer and optimiser (no GPU is needed)."""
import pytest

pytest.importorskip("torch")

from paper_2608_02168_amd import encoder


def test_mixers():
    assert encoder.EncoderConfig().mixer == "attention" and encoder.EncoderConfig().params == encoder.PARAMS
    assert encoder.EncoderConfig(mixer="recurrence").params == encoder.RECURRENT_PARAMS
    with pytest.raises(ValueError, match="mixer"):
        encoder.EncoderConfig(mixer="state")


def test_optimizers():
    with pytest.raises(ValueError, match="optimizer"):
        encoder.train(encoder.EncoderConfig(), 1, optimizer="sgd")


@pytest.mark.parametrize("mixer", ["attention", "recurrence"])
def test_weights_have_their_names(mixer):
    cfg = encoder.EncoderConfig(mixer=mixer, blocks=3)
    params = encoder.make_params(cfg, 1, device="cpu")
    assert len(params) == 3 and all(tuple(p) == cfg.params for p in params)
    assert len({p[n].data_ptr() for p in params for n in p}) == 3 * len(cfg.params)
