"""What the calls of the loss and of the optimiser refuse, on the host, before anything is launched (no GPU)."""
import os

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2204_00595_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        from paper_2204_00595_amd import build
        build.build()
    return b


P = 4096  # never dereferenced


def test_loss_forward(binding):
    L = binding.lib()
    need = binding.monarch_xent_fwd_workspace_bytes(8, 50, 64, 1)
    assert need > 0

    def call(x=P, W=P, t=P, loss=P, lse=P, rows=8, vocab=50, width=64, dtype=1, ws=P, ws_bytes=need, flags=0):
        return L.monarch_xent_fwd(x, W, t, loss, lse, rows, vocab, width, -100, dtype, None, ws, ws_bytes, flags)

    assert call(rows=0) == binding.MONARCH_OK
    assert call(rows=0, x=None, t=None, loss=None, lse=None, ws=None) == binding.MONARCH_OK
    for key in ("x", "W", "t", "loss", "lse"):
        assert call(**{key: None}) == binding.MONARCH_ERR_INVALID
    assert call(x=P + 2) == binding.MONARCH_ERR_INVALID
    assert call(W=P + 8) == binding.MONARCH_ERR_INVALID
    assert call(t=P + 4) == binding.MONARCH_ERR_INVALID
    assert call(rows=-1) == binding.MONARCH_ERR_INVALID
    assert call(vocab=0) == binding.MONARCH_ERR_INVALID
    assert call(width=-3) == binding.MONARCH_ERR_INVALID
    assert call(dtype=5) == binding.MONARCH_ERR_INVALID
    assert call(flags=binding.MONARCH_FLAG_WGRAD_F32) == binding.MONARCH_ERR_INVALID
    assert call(ws=None) == binding.MONARCH_ERR_WORKSPACE
    assert call(ws=P + 64) == binding.MONARCH_ERR_WORKSPACE
    assert call(ws_bytes=need - 1) == binding.MONARCH_ERR_WORKSPACE
    for key, most in (("rows", 1 << 20), ("vocab", 1 << 20), ("width", 1 << 16)):
        assert call(**{key: most + 1}) == binding.MONARCH_ERR_UNSUPPORTED
        assert binding.monarch_xent_fwd_workspace_bytes(*[{"rows": 8, "vocab": 50, "width": 64, key: most + 1}[k] for k in ("rows", "vocab", "width")], 1) == 0


def test_loss_backward(binding):
    L = binding.lib()
    need = binding.monarch_xent_bwd_workspace_bytes(8, 50, 64, 0)
    assert need > 0

    def call(x=P, W=P, t=P, lse=P, dloss=P, stride=1, divisor=None, dx=P, dW=P, rows=8, vocab=50, width=64, dtype=0, ws=P, ws_bytes=need, flags=0):
        return L.monarch_xent_bwd(x, W, t, lse, dloss, stride, divisor, dx, dW, rows, vocab, width, -100, dtype, None, ws, ws_bytes, flags)

    assert call(rows=0, dW=None) == binding.MONARCH_OK
    assert call(dx=None, dW=None) == binding.MONARCH_OK
    for key in ("x", "W", "t", "lse", "dloss"):
        assert call(**{key: None}) == binding.MONARCH_ERR_INVALID
    assert call(stride=2) == binding.MONARCH_ERR_INVALID
    assert call(dx=P + 4) == binding.MONARCH_ERR_INVALID
    assert call(dW=P + 8) == binding.MONARCH_ERR_INVALID
    assert call(divisor=P + 2) == binding.MONARCH_ERR_INVALID
    assert call(flags=binding.MONARCH_FLAG_PERM_B) == binding.MONARCH_ERR_INVALID
    assert call(ws=None) == binding.MONARCH_ERR_WORKSPACE
    assert call(ws_bytes=1024) == binding.MONARCH_ERR_WORKSPACE
    assert call(rows=(1 << 20) + 1) == binding.MONARCH_ERR_UNSUPPORTED


def test_loss_total(binding):
    L = binding.lib()
    assert L.monarch_xent_total(P, P, None, 3, -100, 1, None) == binding.MONARCH_ERR_INVALID
    assert L.monarch_xent_total(None, P, P, 3, -100, 1, None) == binding.MONARCH_ERR_INVALID
    assert L.monarch_xent_total(P, P, P, -3, -100, 1, None) == binding.MONARCH_ERR_INVALID
