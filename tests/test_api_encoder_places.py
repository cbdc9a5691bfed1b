"""Where the tensors of the sequence encoder's calls lie (no GPU is needed): host
tensors, whose addresses would fault in a kernel, and workspaces on another
device, with gaps or not aligned are refused before anything reaches the library."""
import pytest

torch = pytest.importorskip("torch")

import os

from paper_2608_02168_amd import api

P = 0x10000  # never dereferenced: validation fails first


class Library:
    """Answers the workspace sizes and fails a test that launches."""

    def __getattr__(self, name):
        if name.endswith("_workspace_size"):
            return lambda *a: 4096
        return lambda *a: pytest.fail(f"{name} was called")


@pytest.fixture
def no_launch(monkeypatch):
    monkeypatch.setattr(api, "lib", Library)
    monkeypatch.setattr(api, "_current_raw", lambda device: 0)


def calls():
    x, W, b, y = torch.randn(3, 8), torch.randn(8, 16), torch.randn(16), torch.randn(3, 16)
    q, k, one = torch.randn(3, 2, 8), torch.randn(3, 1, 8), torch.ones(8)
    table, pos = torch.randn(5, 8), torch.zeros(3, dtype=torch.int32)
    q4, k4, g, S = torch.randn(2, 3, 2, 8), torch.randn(2, 3, 1, 8), torch.zeros(2), torch.zeros(3, 2, 8, 8)
    return {
        "linear_fwd": lambda: api.hg_linear_fwd(x, W, bias=b),
        "linear_bwd": lambda: api.hg_linear_bwd(x, W, b, y),
        "glu_fwd": lambda: api.hg_glu_fwd(x, W, bias=b),
        "glu_bwd": lambda: api.hg_glu_bwd(x, W, b, y[:, :8].contiguous()),
        "table": lambda: api.hg_rope_table(5, 8, device="cpu"),
        "given table": lambda: api.hg_rope_table(5, 8, table=table),
        "rope_fwd": lambda: api.hg_qk_norm_rope_fwd(q, k, one, one, table, pos),
        "rope_bwd": lambda: api.hg_qk_norm_rope_bwd(q, k, one, one, table, pos, q, k),
        "linattn_fwd": lambda: api.hg_linattn_fwd(q4, k4, k4, g),
        "linattn_bwd": lambda: api.hg_linattn_bwd(q4, k4, k4, g, q4),
        "linattn_step": lambda: api.hg_linattn_step(q, k, k, g, S),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_host_tensors_are_refused(no_launch, name):
    with pytest.raises(TypeError, match="GPU"):
        calls()[name]()


class OnDevice:
    """What the workspace check asks of a tensor, as if it lay on a device."""
    dtype, device = torch.uint8, "cuda:0"

    def __init__(self, index, contiguous=True, n=64, size=1):
        self.get_device, self.is_contiguous = lambda: index, lambda: contiguous
        self.numel, self.element_size, self.data_ptr, self.stride = (lambda: n), (lambda: size), (lambda: P), (lambda: (1,))


def test_workspaces_of_other_places_are_refused():
    like = OnDevice(0)
    assert api._workspace("call", OnDevice(0), 64, like)[1:] == (P, 64)
    assert api._workspace("call", OnDevice(0, size=4), 64, like)[1:] == (P, 256)  # its size in bytes
    assert api._workspace("call", None, 0, like) == (None, None, 0)
    for ws in (torch.empty(64, dtype=torch.uint8), OnDevice(1), OnDevice(0, contiguous=False)):
        with pytest.raises(ValueError, match="call"):
            api._workspace("call", ws, 64, like)


@pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libhg.so not built")
def test_unaligned_workspaces_are_refused():
    L = api.lib()
    ws, big = 9 * P + 8, 1 << 40
    linear = api._pack_linear(20, 23, 31, 1, 2, 23, 31, 23)
    glu = api._pack_glu(20, 23, 31, 1, 2, 23, 31, 23)
    rope = api._pack_rope(10, 50, 4, 2, 16, 16, 0, 1, 1e-6, 0)
    attn = api._pack_linattn(4096, 1, 4, 2, 16, 1, 1.0)
    heads = [api._pack_heads(i * P, 1 << 20, 160, 16) for i in range(1, 8)]
    X, W, b, Y, dX, dW, db = (i * P for i in range(1, 8))
    got = [L.hg_linear_fwd(linear, X, W, b, None, Y, ws, big, None),
           L.hg_linear_bwd(linear, X, W, b, Y, dX, dW, db, 0, ws, big, None),
           L.hg_glu_fwd(glu, X, W, b, Y, ws, big, None),
           L.hg_glu_bwd(glu, X, W, b, Y, dX, dW, db, 0, ws, big, None),
           L.hg_qk_norm_rope_bwd(rope, *heads[:2], P, P, P, P, *heads[2:4], *heads[4:6], P, P, 0, ws, big, None),
           L.hg_linattn_fwd(attn, *heads[:3], P, None, None, heads[3], None, ws, big, None),
           L.hg_linattn_bwd(attn, *heads[:3], P, None, None, heads[3], None, *heads[4:7], None, ws, big, None)]
    assert got == [api.HG_ERR_ARG] * 7


@pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libhg.so not built")
def test_calls_of_too_many_threads_are_refused():
    """A grid of 2^32 threads cannot be launched: refused like every size before any device work."""
    L, big = api.lib(), 1 << 62
    X, W, b, Y, dX, dW, db = (i << 56 for i in range(1, 8))

    def linear(n, d, m, dtype=1, act=2, ld_x=None, ld_y=None):
        return api._pack_linear(n, d, m, dtype, act, ld_x or d, ld_y or m, m), \
            api._pack_linear(n, d, m, dtype, act, ld_x or d, ld_y or m, d)

    # 2^24 tiles; X to be copied into padded rows; only the backward's tiles
    for n, d, m, ld_x in ((1 << 30, 8, 8, 8), ((1 << 31) - 64, 17, 16, 17), (1 << 26, 513, 8, 513)):
        fwd, bwd = linear(n, d, m, ld_x=ld_x)
        assert L.hg_linear_fwd(fwd, X, W, b, None, Y, 1 << 48, big, None) == api.HG_ERR_UNSUPPORTED
        assert L.hg_linear_bwd(bwd, X, W, b, Y, dX, dW, db, 0, 1 << 48, big, None) == api.HG_ERR_UNSUPPORTED
        assert L.hg_linear_fwd_workspace_size(fwd) == L.hg_linear_bwd_workspace_size(bwd) == 0
    # the forward's tiles are few, those of dX too many
    _, bwd = linear(1 << 24, 1 << 14, 8)
    assert L.hg_linear_bwd(bwd, X, W, b, Y, dX, dW, db, 0, 1 << 48, big, None) == api.HG_ERR_UNSUPPORTED
    glu = api._pack_glu(1 << 30, 8, 8, 0, 2, 8, 8, 8)
    assert L.hg_glu_fwd(glu, X, W, b, Y, 1 << 48, big, None) == api.HG_ERR_UNSUPPORTED
    assert L.hg_glu_bwd(glu, X, W, b, Y, dX, dW, db, 0, 1 << 48, big, None) == api.HG_ERR_UNSUPPORTED
    # what can be launched has a workspace still
    fwd, bwd = linear((1 << 29) - 64, 8, 8)
    assert L.hg_linear_bwd_workspace_size(bwd) > 0 == L.hg_linear_fwd_workspace_size(fwd)
    rope = api._pack_rope(1 << 31, 50, 4, 4, 64, 64, 0, 1, 1e-6, 0)
    heads = [api._pack_heads(i << 56, 0, 512, 64) for i in range(1, 5)]
    assert L.hg_qk_norm_rope_fwd(rope, *heads[:2], P, P, P, P, *heads[2:], None) == api.HG_ERR_UNSUPPORTED
    assert L.hg_rope_table(1 << 30, 16, 1e4, 1.0, P, None) == api.HG_ERR_UNSUPPORTED
    assert L.hg_rope_table(1 << 30, 0, 1e4, 1.0, P, None) == api.HG_OK


@pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libhg.so not built")
def test_a_step_does_not_write_its_inputs():
    L = api.lib()
    A = api._pack_linattn(1, 2, 4, 2, 16, 1, 1.0)
    q, k, v = (api._pack_heads(i * P, 160, 0, 16) for i in (1, 2, 3))
    for o in (q, k, v):
        assert L.hg_linattn_step(A, q, k, v, 4 * P, 5 * P, None, 2, o, None) == api.HG_ERR_ARG
        assert "o is an input" in api.last_error_detail()


@pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libhg.so not built")
def test_a_product_does_not_write_its_bias():
    L = api.lib()
    X, W, Y = P, 2 * P, 4 * P
    for at in (0, 60, 20 * 32 * 2 - 4):
        assert L.hg_linear_fwd(api._pack_linear(20, 24, 32, 1, 0, 24, 32, 32), X, W, Y + at, None, Y, None, 0, None) == api.HG_ERR_ARG
        assert "overlaps" in api.last_error_detail()
    assert L.hg_glu_fwd(api._pack_glu(20, 24, 16, 1, 2, 24, 16, 24), X, W, Y - 64, Y, None, 0, None) == api.HG_ERR_ARG
    assert "overlaps" in api.last_error_detail()
