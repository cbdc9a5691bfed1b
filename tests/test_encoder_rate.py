"""Rates of the recurrence's gates that its operator or its first weights do not take
are refused where the configuration is made (no GPU is needed)."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2608_02168_amd.encoder import EncoderConfig, make_params


@pytest.mark.parametrize("rate", [0.0, -8.0, 1e-5, math.inf, math.nan])
def test_refused(rate):
    with pytest.raises(ValueError, match="rate"):
        EncoderConfig(mixer="recurrence", rate=rate)


@pytest.mark.parametrize("rate", [1e-3, 0.1, 8.0, 1e6])
def test_first_factors(rate):
    """At r = 0 a channel's factor is what it was made for, from 0.9 to 0.999."""
    cfg = EncoderConfig(mixer="recurrence", rate=rate, blocks=1)
    decay = make_params(cfg, 0, device="cpu")[0]["decay"].double()
    a = torch.exp(-rate * torch.logaddexp(decay, torch.zeros(1).double()) / 2)
    # (decay, up to 211 in size, is rounded to 2^-17 of 1, and log a = -rate softplus(decay) / 2 by rate / 2 times that;
    # where rate is large, softplus(decay) is about exp(decay), off by 2^-20 of itself)
    assert torch.allclose(a, torch.linspace(0.9, 0.999, cfg.d).double(), rtol=0, atol=1e-5)
