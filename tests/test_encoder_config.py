"""Widths that the sequence encoder's operators do not take are refused where the
configuration is made (no GPU is needed)."""
import pytest

pytest.importorskip("torch")

from paper_2608_02168_amd.encoder import EncoderConfig


@pytest.mark.parametrize("kw", [dict(d=66), dict(heads=3, kv_heads=1), dict(heads=4, kv_heads=3), dict(d=48),
                                dict(d=1088), dict(heads=0), dict(kv_heads=0), dict(f=0), dict(blocks=-1), dict(n_pos=-1)])
def test_refused(kw):
    with pytest.raises(ValueError):
        EncoderConfig(**kw)


@pytest.mark.parametrize("kw", [dict(), dict(d=512, heads=4, kv_heads=1), dict(d=8, heads=1, kv_heads=1, f=1, blocks=0)])
def test_taken(kw):
    assert EncoderConfig(**kw).d_head % 8 == 0
