"""The sequence encoder (paper_2608_02168_amd/encoder.py) where a batch holds
nothing: no sequences, no tokens, no rows to serve, and sequences of length zero
among others."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_02168_amd import encoder

pytestmark = pytest.mark.gpu


def model(dtype):
    cfg = encoder.EncoderConfig(dtype=dtype)
    return cfg, encoder.make_params(cfg, 3), encoder.make_plan(cfg)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,t", [(0, 5), (3, 0), (0, 0)])
def test_no_sequences_or_no_tokens(b, t, dtype):
    cfg, params, plan = model(dtype)
    x = torch.zeros(b, t, cfg.d, dtype=dtype, device="cuda")
    pos = torch.zeros(b, t, dtype=torch.int32, device="cuda")
    z, saved, states = encoder.forward(cfg, params, plan, x, pos)
    assert z.shape == (b, t, cfg.d)
    for s in states:
        assert s.shape == (b, cfg.heads, cfg.d_head, cfg.d_head) and not s.any()
    dx, grads = encoder.backward(cfg, params, plan, saved, torch.zeros_like(z))
    assert dx.shape == x.shape
    assert all(not g[n].any() for g in grads for n in encoder.PARAMS)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows_to_serve(dtype):
    cfg, params, plan = model(dtype)
    held = [torch.full((4, cfg.heads, cfg.d_head, cfg.d_head), 2.0, device="cuda") for _ in params]
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    z = encoder.step(cfg, params, plan, torch.zeros(0, cfg.d, dtype=dtype, device="cuda"), none, held, none)
    assert z.shape == (0, cfg.d) and all(torch.all(s == 2) for s in held)


def test_a_sequence_of_no_tokens_changes_no_other():
    cfg, params, plan = model(torch.float32)
    x, pos, _, _ = encoder.make_histories(1, 3, 20, cfg.d)
    lens = torch.tensor([20, 0, 7], dtype=torch.int32, device="cuda")
    z, _, states = encoder.forward(cfg, params, plan, x, pos, lens)
    alone, _, only = encoder.forward(cfg, params, plan, x[2:, :7].contiguous(), pos[2:, :7].contiguous())
    assert torch.allclose(z[2, :7], alone[0], rtol=1e-4, atol=1e-4)
    for s, o in zip(states, only):
        assert not s[1].any() and torch.allclose(s[2], o[0], rtol=1e-4, atol=1e-4)
