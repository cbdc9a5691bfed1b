"""Which layouts of rows the recurrence and the group norm take as apart, against
the addresses themselves, listed one by one (no GPU is needed: a call is refused
for its workspace, or for an overlap, before any device work)."""
import itertools
import os
import random

import pytest

pytest.importorskip("torch")

from paper_2608_02168_amd import api

P, BIG = 0x100000, 1 << 40
ARG, CAPACITY = api.HG_ERR_ARG, api.HG_ERR_CAPACITY


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        pytest.skip("libhg.so not built")
    return api.lib()


def far(k, b, t, w):
    return api._pack_heads(k * P, t * w, w, 0)


def gradients(L, b, t, w, starts, sb, st, dtype=1):
    """The answer to dx, dr, di from these values on, all with these strides, without a workspace."""
    d, e = api._pack_recur(t, b, w, dtype, 8.0), 2 if dtype else 4
    rows = [api._pack_heads(9 * P + e * s, sb, st, 0) for s in starts]
    return L.hg_recur_bwd(d, far(1, b, t, w), far(2, b, t, w), far(3, b, t, w), 4 * P, None, None, far(5, b, t, w),
                          far(6, b, t, w), None, *rows, 7 * P, None, 0, None, 0, None)


def norm(L, b, t, w, x, y):
    """The same of a group norm's x and y: (start, batch stride, token stride) each."""
    d = api._pack_group_norm(t, b, w, 1, 1, 0, 1e-5)
    at = [api._pack_heads(9 * P + 2 * s, sb, st, 0) for s, sb, st in (x, y)]
    return L.hg_group_norm_bwd(d, far(1, b, t, w), None, None, None, 5 * P, at[0], at[1], None, None, 0, None, 0, None)


def addresses(b, t, w, start, sb, st):
    return {start + i * sb + k * st + c for i in range(b) for k in range(t) for c in range(w)}


def test_columns_of_packed_buffers(L):
    b, t, w = 2, 20, 16
    # [batch, t, 3 w], [t, batch, 3 w], and three planes of one buffer, inside a sequence, inside a token, or whole
    for sb, st, step in ((3 * t * w, 3 * w, w), (3 * w, 3 * b * w, w), (3 * t * w, w, t * w), (w, 3 * b * w, b * w),
                         (t * w, w, b * t * w), (w, b * w, b * t * w)):
        assert gradients(L, b, t, w, (0, step, 2 * step), sb, st) == CAPACITY, (sb, st)
        assert gradients(L, b, t, w, (2 * step, step, 0), sb, st) == CAPACITY, (sb, st)
        assert gradients(L, b, t, w, (0, step - 1, 2 * step), sb, st) == ARG, (sb, st)
        assert gradients(L, b, t, w, (0, step, step + 1), sb, st) == ARG, (sb, st)
    # float32, one sequence, one token
    assert gradients(L, 5, 7, 8, (0, 8, 16), 24, 120, dtype=0) == CAPACITY
    assert gradients(L, 1, 20, 16, (0, 16, 32), 0, 48) == gradients(L, 20, 1, 16, (0, 16, 32), 48, 0) == CAPACITY
    assert gradients(L, 1, 20, 16, (0, 16, 31), 0, 48) == gradients(L, 20, 1, 16, (0, 16, 31), 48, 0) == ARG


def test_random_layouts(L):
    """Same strides: exactly those that share an address are refused.  Others: none that does is taken."""
    rng, seen = random.Random(5), set()
    for _ in range(4000):
        b, t, w = rng.randint(1, 4), rng.randint(1, 4), rng.randint(4, 9)
        tokens_inside = rng.random() < 0.5
        s1 = w + rng.randint(0, 3 * w)
        s2 = ((t if tokens_inside else b) - 1) * s1 + w + rng.randint(0, 4 * w)
        sb, st = (s2, s1) if tokens_inside else (s1, s2)
        y = (rng.randint(0, 200), sb, st)
        x = (rng.randint(0, 200), sb, st)
        meet = bool(addresses(b, t, w, *x) & addresses(b, t, w, *y))
        assert norm(L, b, t, w, x, y) == (ARG if meet else CAPACITY), (b, t, w, x, y)
        seen.add((meet, abs(x[0] - y[0]) < min(sb, st)))
        z = (x[0], sb + rng.choice([0, 1, w]), st + rng.choice([0, 1, w]))
        if norm(L, b, t, w, z, y) == CAPACITY:
            assert not addresses(b, t, w, *z) & addresses(b, t, w, *y), (b, t, w, z, y)
    assert seen == set(itertools.product((False, True), (False, True)))


def test_a_repeated_input(L):
    """An input that is one row for every token (strides of zero) inside and outside an output's memory."""
    for sb, st in ((0, 0), (0, 8), (8, 0)):
        inside = norm(L, 3, 4, 8, (8, sb, st), (0, 32, 8))
        assert inside == ARG and norm(L, 3, 4, 8, (200, sb, st), (0, 32, 8)) == CAPACITY
