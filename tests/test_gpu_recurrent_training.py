"""Training steps of the sequence encoder (encoder.train) against the oracle: the
gradients of both blocks and of the head from the same weights and histories, and
every update of a weight from its own gradient and moments, by the optimiser and
at the rate that are its own.

Bars: losses and gradients as of the two blocks, 1e-3 and 2e-3.  A matrix's
update: X is off by at most 485 2^-21 of its norm, which is at most 1.21
sqrt(min(rows, cols)), and W is rounded once.  Adam's: some ten roundings of a
step of about lr, and one of the weight."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import objective
from oracle import recurrent as rec
from paper_2608_02168_amd import api, encoder
from tests.helpers import parity_err
from tests.test_gpu_recurrent_encoder import host, oracle_backward, oracle_forward

pytestmark = pytest.mark.gpu
LR = 1e-2


def watched(monkeypatch, cfg, optimizer, steps):
    """encoder.train with the updates that it makes: (operator, weight, gradient, moments before, weight after)."""
    seen = []

    def watch(name, call):
        def update(w, g, *moments, **k):
            tensors = [t.clone() for t in moments if torch.is_tensor(t)]
            before = w.clone()
            call(w, g, *moments, **k)
            seen.append((name, before, g.clone(), tensors, w.clone()))
        return update

    monkeypatch.setattr(api, "hg_adam_step", watch("adam", api.hg_adam_step))
    monkeypatch.setattr(api, "hg_muon_step", watch("muon", api.hg_muon_step))
    losses, params, head, _ = encoder.train(cfg, steps, batch=32, t=40, lr=LR, optimizer=optimizer)
    return losses, params, head, seen


@pytest.mark.parametrize("mixer", ["attention", "recurrence"])
@pytest.mark.parametrize("optimizer", ["adam", "muon"])
def test_updates(monkeypatch, mixer, optimizer):
    cfg = encoder.EncoderConfig(mixer=mixer)
    _, params, head, seen = watched(monkeypatch, cfg, optimizer, 2)
    names = [(i, n) for i in range(cfg.blocks) for n in cfg.params] + [(None, n) for n in head]
    assert len(seen) == 2 * len(names)
    for k, (name, before, g, moments, after) in enumerate(seen):
        block, what = names[k % len(names)]
        t = k // len(names) + 1
        matrix = block is not None and before.dim() == 2
        assert name == ("muon" if optimizer == "muon" and matrix else "adam"), (block, what)
        w, d, m = host(before), host(g), [host(v) for v in moments]
        if name == "muon":
            # weights are [in, out]: the root of outputs over inputs, where there are more
            scale = max(1.0, w.shape[1] / w.shape[0]) ** 0.5
            want, _ = rec.muon_step(w, d, m[0], LR, scale=scale)
            bar = LR * scale * 1.21 * min(w.shape) ** 0.5 * 485 * 2.0 ** -21 + 2.0 ** -23 * np.linalg.norm(want)
            assert np.linalg.norm(host(after) - want) < bar, (block, what)
        else:
            want, _, _ = objective.adam_step(w, d, m[0], m[1], t, lr=LR)
            assert (np.abs(host(after) - want) < 1e-5 * LR + 2.0 ** -23 * np.abs(want)).all(), (block, what)
    final = {(i, n): p[n] for i, p in enumerate(params) for n in cfg.params} | {(None, n): w for n, w in head.items()}
    for (_, _, _, _, after), key in zip(seen[len(names):], names):
        assert torch.equal(final[key], after)


def test_first_gradients(monkeypatch):
    cfg = encoder.EncoderConfig(mixer="recurrence")
    losses, _, head, seen = watched(monkeypatch, cfg, "muon", 1)
    x, _, lens, label = encoder.make_histories(11, 32, 40, cfg.d)
    lens_h = lens.cpu().numpy()
    z, saved, _ = oracle_forward(cfg, encoder.make_params(cfg, 0), host(x), lens_h)
    rows = np.arange(32)
    w = dict(zip(head, (host(v[1]) for v in seen[-len(head):])))
    loss, dlast, *dhead, _ = objective.mlp_bce(z[rows, lens_h - 1], w["W1"], w["b1"], w["W2"], w["b2"], label.cpu().numpy())
    dz = np.zeros_like(z)
    dz[rows, lens_h - 1] = dlast
    _, grads = oracle_backward(cfg, saved, dz, lens_h)
    assert abs(losses[0] - loss) < 1e-3 * abs(loss)
    want = [g[n] for g in grads for n in cfg.params] + dhead
    for (_, _, g, _, _), r in zip(seen, want):
        assert np.linalg.norm(r) > 0 and parity_err(host(g), np.reshape(r, g.shape)) <= 2e-3
