"""The C ABI of the recurrent block's operators on the host: descriptors as the
binding packs them, workspace sizes, and the refusal of invalid arguments before
any device work (no GPU is needed for any of these)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2608_02168_amd import api
from tests.test_api_encoder_places import no_launch  # noqa: F401

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hg.h")
P = 0x100000  # never dereferenced: validation fails first
BIG = 1 << 40
ARG, UNSUPPORTED, CAPACITY, OK = api.HG_ERR_ARG, api.HG_ERR_UNSUPPORTED, api.HG_ERR_CAPACITY, api.HG_OK


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        pytest.skip("libhg.so not built")
    return api.lib()


STRUCTS = {"hg_recur_desc": (api.RecurDesc, api._pack_recur, (1, 2, 3, 4, 5.0)),
           "hg_group_norm_desc": (api.GroupNormDesc, api._pack_group_norm, (1, 2, 3, 4, 5, 6, 7.0)),
           "hg_muon_desc": (api.MuonDesc, api._pack_muon, (1, 2, 3, 4, 5, 6, 7.0, 8.0, 9.0, 10.0, 11.0, 12))}


def test_structs_match_the_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not available")
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void) {"]
    for cname, (py, _, _) in STRUCTS.items():
        lines.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out if x.strip()}
    for cname, (py, pack, vals) in STRUCTS.items():
        assert got[(cname, "size")] == C.sizeof(py), cname
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)
        assert pack(*vals) == bytes(py(*vals)), cname


def rows(i, batch=20 * 16, token=16, shift=0):
    return api._pack_heads(i * P + shift, batch, token, 0)


def test_recur_refusals(L):
    def d(t=20, b=2, w=16, dtype=1, rate=8.0):
        return api._pack_recur(t, b, w, dtype, rate)

    def fwd(desc, x=rows(1), r=rows(2), i=rows(3), g=4 * P, s=5 * P, h=rows(6), so=7 * P, ws=8 * P, n=BIG):
        return L.hg_recur_fwd(desc, x, r, i, g, None, s, h, so, ws, n, None)

    def bwd(desc, x=rows(1), dx=rows(9), dr=rows(10), di=rows(11), g=4 * P, dg=12 * P, s=5 * P, dso=13 * P, ds=14 * P, acc=0,
            ws=15 * P, n=BIG):
        return L.hg_recur_bwd(desc, x, rows(2), rows(3), g, None, s, rows(6), rows(8), dso, dx, dr, di, dg, ds, acc, ws, n,
                              None)

    for kw, code in ((dict(t=-1), ARG), (dict(b=-1), ARG), (dict(w=0), ARG), (dict(dtype=2), ARG), (dict(rate=0.0), ARG),
                     (dict(rate=-1.0), ARG), (dict(rate=float("nan")), ARG), (dict(rate=float("inf")), ARG),
                     (dict(w=3), UNSUPPORTED), (dict(w=(1 << 20) + 1), UNSUPPORTED), (dict(b=1 << 22), UNSUPPORTED),
                     (dict(t=(1 << 40) + 1), UNSUPPORTED)):
        assert fwd(d(**kw)) == bwd(d(**kw)) == code, kw
        assert len(api.last_error_detail()) > 0
    assert fwd(None) == bwd(None) == ARG
    assert fwd(d(), x=None) == fwd(d(), r=rows(0)) == fwd(d(), g=None) == fwd(d(), h=None) == ARG
    assert fwd(d(), x=rows(1, shift=1)) == fwd(d(), x=rows(1, token=-1)) == fwd(d(), x=rows(1, batch=1 << 41)) == ARG
    assert fwd(d(), h=rows(1)) == fwd(d(), h=rows(2, shift=2)) == fwd(d(), h=rows(3, token=17)) == ARG   # overlap inputs
    assert fwd(d(), x=rows(1, batch=1 << 30, token=(1 << 21) + 1)) == UNSUPPORTED
    assert fwd(d(), h=rows(6, token=15)) == fwd(d(), h=rows(6, batch=300)) == fwd(d(), so=5 * P) == ARG
    assert bwd(d(), dx=rows(9), dr=rows(9)) == bwd(d(), di=rows(6)) == bwd(d(), dx=rows(8)) == ARG
    assert bwd(d(), ds=13 * P) == bwd(d(), ds=5 * P) == bwd(d(), dg=4 * P) == bwd(d(), acc=2) == ARG
    assert bwd(d(), ws=None) == bwd(d(), n=L.hg_recur_bwd_workspace_size(d()) - 1) == CAPACITY
    assert bwd(d(), ws=15 * P + 8) == fwd(d(t=1 << 16, b=1), x=rows(1), ws=8 * P + 8) == ARG
    assert fwd(d(b=0)) == OK

    def step(desc, s=5 * P, slots=None, n=2, h=rows(6)):
        return L.hg_recur_step(desc, rows(1), rows(2), rows(3), 4 * P, s, slots, n, h, None)

    assert step(d()) == ARG                                            # more than one token
    assert step(d(t=1), n=1) == step(d(t=1), n=-1) == step(d(t=1), s=None) == step(d(t=1), h=rows(2)) == ARG
    assert step(d(t=1, b=0)) == OK


def test_interleaved_outputs_are_taken_apart(L):
    """Columns of one packed buffer do not overlap; columns that do are refused."""
    d = api._pack_recur(20, 2, 16, 1, 8.0)

    def bwd(starts, ws):  # dx, dr, di as columns of [2, 20, 48] values of two bytes
        packed = [api._pack_heads(9 * P + 2 * c, 20 * 48, 48, 0) for c in starts]
        return L.hg_recur_bwd(d, rows(1), rows(2), rows(3), 4 * P, None, None, rows(6), rows(8), None, *packed, 12 * P, None,
                              0, ws, BIG, None)

    # refused for its workspace alone, after the overlaps were looked at
    assert bwd((0, 16, 32), None) == CAPACITY
    assert bwd((0, 15, 32), None) == bwd((0, 16, 33), None) == bwd((0, 0, 16), None) == ARG


def test_group_norm_refusals(L):
    def d(t=20, b=2, w=16, g=4, dtype=1, act=2, eps=1e-5):
        return api._pack_group_norm(t, b, w, g, dtype, act, eps)

    def fwd(desc, x=rows(1), y=rows(2), ws=8 * P, n=BIG):
        return L.hg_group_norm_fwd(desc, x, 3 * P, 4 * P, None, y, 5 * P, ws, n, None)

    def bwd(desc, x=rows(1), st=5 * P, dy=rows(2), dx=rows(6), dw=7 * P, db=9 * P, acc=0, ws=8 * P, n=BIG):
        return L.hg_group_norm_bwd(desc, x, 3 * P, 4 * P, None, st, dy, dx, dw, db, acc, ws, n, None)

    for kw, code in ((dict(t=-1), ARG), (dict(b=-1), ARG), (dict(w=0), ARG), (dict(g=0), ARG), (dict(g=3), ARG),
                     (dict(dtype=-1), ARG), (dict(act=4), ARG), (dict(act=-1), ARG), (dict(eps=0.0), ARG),
                     (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(w=1025, g=1), UNSUPPORTED),
                     (dict(w=8200, g=1), UNSUPPORTED), (dict(w=4100, g=1, dtype=0), UNSUPPORTED),
                     (dict(t=1 << 41), UNSUPPORTED), (dict(t=1 << 30, b=64), UNSUPPORTED)):
        assert fwd(d(**kw)) == bwd(d(**kw)) == code, kw
    assert fwd(None) == fwd(d(), x=None) == fwd(d(), x=rows(1, shift=1)) == fwd(d(), y=rows(2, token=8)) == ARG
    assert fwd(d(), y=rows(1)) == fwd(d(), y=rows(1, shift=32)) == ARG
    assert bwd(d(), st=None) == bwd(d(), dx=rows(2)) == bwd(d(), dx=rows(1)) == bwd(d(), acc=-1) == ARG
    assert bwd(d(), dw=9 * P) == bwd(d(), dw=3 * P) == bwd(d(), db=4 * P) == ARG
    assert bwd(d(), ws=None) == bwd(d(), n=L.hg_group_norm_bwd_workspace_size(d()) - 1) == CAPACITY
    assert bwd(d(), ws=8 * P + 8) == ARG
    long = d(t=1 << 20, b=1)
    assert L.hg_group_norm_fwd_workspace_size(long) > 0 == L.hg_group_norm_fwd_workspace_size(d())
    assert fwd(long, y=rows(200), ws=None, n=0) == CAPACITY
    assert fwd(long, ws=None, n=0) == ARG                                # y inside x's stretch
    assert fwd(d(b=0)) == OK


def test_states_and_gradients_that_share_part_of_a_buffer(L):
    """Refused as well as the same buffer: another block may read what one wrote."""
    d = api._pack_recur(20, 2, 16, 1, 8.0)
    state = 2 * 16 * 4

    def fwd(so, ws):
        return L.hg_recur_fwd(d, rows(1), rows(2), rows(3), 4 * P, None, 5 * P, rows(6), so, ws, BIG, None)

    def bwd(dg, ds):  # (refused for its workspace alone where nothing overlaps)
        return L.hg_recur_bwd(d, rows(1), rows(2), rows(3), 4 * P, None, 5 * P, rows(6), rows(8), 13 * P, rows(9), rows(10),
                              rows(11), dg, ds, 0, None, 0, None)

    assert fwd(5 * P + state - 4, None) == fwd(5 * P - state + 4, None) == ARG
    assert bwd(12 * P, 5 * P + state) == bwd(4 * P + 64, 14 * P) == CAPACITY
    assert bwd(12 * P, 5 * P + state - 4) == bwd(12 * P, 13 * P - 4) == bwd(4 * P + 60, 14 * P) == ARG
    g = api._pack_group_norm(20, 2, 16, 4, 1, 2, 1e-5)

    def norm(dw, db):
        return L.hg_group_norm_bwd(g, rows(1), 3 * P, 4 * P, None, 5 * P, rows(2), rows(6), dw, db, 0, None, 0, None)

    assert norm(7 * P, 7 * P + 64) == norm(3 * P + 64, 9 * P) == CAPACITY
    assert norm(7 * P, 7 * P + 60) == norm(3 * P + 60, 9 * P) == norm(7 * P, 4 * P - 60) == ARG


def test_grids_stay_launchable(L):
    """Single channels a thread in slabs of 64, 256 threads each: fewer than 2^32 threads a launch."""
    def bwd(batch):
        w = 1021 * 1024  # 16336 slabs
        d = api._pack_group_norm(3, batch, w, 1024, 0, 0, 1e-5)
        x = [api._pack_heads(k << 42, 3 * w, w, 0) for k in (1, 2, 3)]
        return L.hg_group_norm_bwd(d, x[0], None, None, None, 5 * P, x[1], x[2], None, None, 0, None, 0, None)

    assert bwd(1) == bwd(1027) == CAPACITY
    assert bwd(1028) == bwd(4000) == UNSUPPORTED


def test_muon_refusals(L):
    def d(c=2, m=16, n=24, dtype=0, steps=5, nes=1, lr=0.1, mu=0.9, wd=0.0, scale=1.0, eps=1e-7):
        return api._pack_muon(c, m, n, dtype, steps, nes, lr, mu, wd, scale, eps, 0)

    def step(desc, W=P, G=2 * P, M=3 * P, ws=4 * P, n=BIG):
        return L.hg_muon_step(desc, W, G, M, ws, n, None)

    inf, nan = float("inf"), float("nan")
    for kw, code in ((dict(c=-1), ARG), (dict(m=0), ARG), (dict(n=0), ARG), (dict(dtype=2), ARG), (dict(steps=-1), ARG),
                     (dict(steps=33), ARG), (dict(nes=2), ARG), (dict(lr=nan), ARG), (dict(mu=inf), ARG),
                     (dict(wd=nan), ARG), (dict(scale=inf), ARG), (dict(eps=0.0), ARG), (dict(eps=nan), ARG),
                     (dict(m=(1 << 15) + 1), UNSUPPORTED), (dict(n=(1 << 15) + 1), UNSUPPORTED),
                     (dict(c=1 << 16), UNSUPPORTED), (dict(c=8, m=1 << 15, n=1 << 15), UNSUPPORTED)):
        assert step(d(**kw)) == code, kw
    assert step(None) == step(d(), W=None) == step(d(), G=None) == step(d(), M=None) == ARG
    assert step(d(), W=P + 2) == step(d(), G=2 * P + 1) == step(d(), M=3 * P + 2) == step(d(), ws=4 * P + 8) == ARG
    assert step(d(), G=P) == step(d(), M=P + 1024) == step(d(), M=2 * P - 16) == ARG
    large = d(m=200, n=300)  # small matrices need no workspace
    need = L.hg_muon_workspace_size(large)
    assert L.hg_muon_workspace_size(d()) == 0 < need
    assert step(large, M=9 * P, n=need - 1) == step(large, M=9 * P, ws=None) == CAPACITY
    assert step(d(c=0)) == OK


def test_host_tensors_are_refused(no_launch):  # noqa: F811
    x, v, s = torch.randn(2, 3, 8), torch.randn(8), torch.randn(2, 8)
    m = torch.randn(4, 8)
    for call in (lambda: api.hg_recur_fwd(x, x, x, v), lambda: api.hg_recur_bwd(x, x, x, v, x, x),
                 lambda: api.hg_recur_step(s, s, s, v, s), lambda: api.hg_group_norm_fwd(x, 2, v, v),
                 lambda: api.hg_group_norm_bwd(x, 2, v, v, torch.zeros(2, 2, 2), x),
                 lambda: api.hg_muon_step(m, m, m, 0.1)):
        with pytest.raises(TypeError, match="GPU"):
            call()


def test_shapes_are_checked():
    """Before the library is asked anything."""
    m = torch.randn(4, 8)
    with pytest.raises(ValueError, match="accumulate"):
        api.hg_recur_bwd(*[torch.randn(2, 3, 8)] * 3, torch.randn(8), *[torch.randn(2, 3, 8)] * 2, accumulate=True)
    with pytest.raises(ValueError, match="matrices"):
        api.hg_muon_step(torch.randn(8), torch.randn(8), torch.randn(8), 0.1)
    for t, shape in ((torch.randn(3, 2, 8), (2, 3, 8)), (torch.randn(2, 3, 16)[..., ::2], (2, 3, 8))):
        with pytest.raises(ValueError, match="expected x"):
            api._channels("call", "x", t, shape)
    assert api._channels("call", "x", torch.randn(1, 1, 8), (1, 1, 8))[8:24] == bytes(16)  # strides never walked
