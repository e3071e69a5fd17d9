"""Host-side checks of the vocabulary loss and the orthogonalised update that need no GPU: sizes, refusals, workspaces."""
import pytest

import __graft_entry__ as entry
from paper_2204_00595_b200 import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return B.lib()


def addresses(n, step=1 << 28):
    """Distinct 256-byte aligned addresses, never dereferenced: every call below fails before it launches."""
    return [(i + 1) * step for i in range(n)]


def test_loss_refusals(lib):
    x, W, y, loss, lse, ws = addresses(6)
    f = lambda **k: lib.monarch_xent_fwd(*[{**dict(x=x, W=W, y=y, loss=loss, lse=lse, T=10, d=64, V=100, ign=-100, dt=1, ws=ws, nb=BIG,  # noqa: E731
                                                   s=None), **k}[a] for a in ("x", "W", "y", "loss", "lse", "T", "d", "V", "ign", "dt", "ws", "nb", "s")])
    for name in ("x", "W", "y", "loss", "lse"):
        assert f(**{name: None}) == INVALID, name
    for bad in (dict(T=-1), dict(d=0), dict(V=0), dict(dt=2), dict(dt=-1), dict(x=x + 8), dict(W=W + 8), dict(y=y + 4), dict(loss=loss + 2),
                dict(loss=x), dict(lse=loss), dict(loss=loss, lse=loss + 36), dict(lse=ws), dict(x=ws + 4096)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(T=(1 << 24) + 1), dict(d=65537), dict(V=(1 << 24) + 1)):
        assert f(**bad) == UNSUPPORTED, bad
    need = B.monarch_xent_workspace_bytes(10, 64, 100, B.BF16)
    for bad in (dict(ws=None), dict(ws=ws + 16), dict(nb=need - 1)):
        assert f(**bad) == WORKSPACE, bad
    # no tokens: nothing to read or write, nothing launched
    assert f(T=0, x=None, y=None, loss=None, lse=None) == OK


def test_loss_gradient_refusals(lib):
    names = ("x", "W", "y", "lse", "dl", "dx", "dW", "acc", "T", "d", "V", "ign", "dt", "ws", "nb", "s")
    x, W, y, lse, dl, dx, dW, ws = addresses(8)
    base = dict(x=x, W=W, y=y, lse=lse, dl=dl, dx=dx, dW=dW, acc=0, T=10, d=64, V=100, ign=-100, dt=0, ws=ws, nb=BIG, s=None)
    f = lambda **k: lib.monarch_xent_bwd(*[{**base, **k}[a] for a in names])  # noqa: E731
    for name in ("x", "W", "y", "lse", "dl", "dx", "dW"):
        assert f(**{name: None}) == INVALID, name
    for bad in (dict(acc=2), dict(acc=-1), dict(T=-1), dict(d=-3), dict(V=0), dict(dt=7), dict(dx=x), dict(dW=W), dict(dx=dW), dict(dx=dx + 4),
                dict(dW=dW + 8), dict(lse=lse + 1), dict(dl=dl + 2), dict(dW=ws)):
        assert f(**bad) == INVALID, bad
    need = B.monarch_xent_bwd_workspace_bytes(10, 64, 100, B.F32)
    for bad in (dict(ws=None), dict(ws=ws + 128), dict(nb=need - 1)):
        assert f(**bad) == WORKSPACE, bad


def test_update_refusals(lib):
    G, O, V, ws = addresses(4)
    f = lambda *a: lib.monarch_orthogonalize(*a)  # noqa: E731
    assert f(None, O, 2, 8, 8, 5, 0, ws, BIG, None) == INVALID
    assert f(G, G, 2, 8, 8, 5, 0, ws, BIG, None) == INVALID
    assert f(G, G + 256, 2, 8, 8, 5, 0, ws, BIG, None) == INVALID
    assert f(G, O + 4, 2, 8, 8, 5, 0, ws, BIG, None) == INVALID
    for sizes in ((-1, 8, 8, 5), (2, 0, 8, 5), (2, 8, -1, 5), (2, 8, 8, 0)):
        assert f(G, O, *sizes, 0, ws, BIG, None) == INVALID, sizes
    for sizes in ((2, 32769, 8, 5), (2, 8, 32769, 5), ((1 << 20) + 1, 8, 8, 5), (2, 8, 8, 33)):
        assert f(G, O, *sizes, 0, ws, BIG, None) == UNSUPPORTED, sizes
    assert f(G, O, 2, 8, 8, 5, 3, ws, BIG, None) == INVALID
    assert f(G, O, 2, 8, 8, 5, 0, None, BIG, None) == WORKSPACE
    assert f(G, O, 2, 300, 300, 5, 0, ws, 4096, None) == WORKSPACE
    assert f(None, None, 0, 8, 8, 5, 0, ws, BIG, None) == OK
    m = lib.monarch_muon_step
    good = (2, 8, 8, 0.1, 0.0, 0.9, 1, 1.0, 5, 1, ws, BIG, None)
    assert m(G, None, V, *good) == INVALID
    assert m(G, G, V, *good) == INVALID
    assert m(G, O, G, *good) == INVALID
    assert m(G, O, V, 2, 8, 8, 0.1, 0.0, 0.9, 2, 1.0, 5, 1, ws, BIG, None) == INVALID
    for bad in (float("nan"), float("inf")):
        for at in (3, 4, 5, 7):
            a = list(good)
            a[at] = bad
            assert m(G, O, V, *a) == INVALID, (bad, at)


def test_workspaces(lib):
    for q in (B.monarch_xent_workspace_bytes, B.monarch_xent_bwd_workspace_bytes):
        assert q(1, 1, 1, B.F32) >= 256 and q(0, 8, 8, B.BF16) >= 256
        assert q(-1, 8, 8, B.BF16) == 0 and q(1, 0, 8, B.BF16) == 0 and q(1, 8, 0, B.BF16) == 0 and q(1, 8, 8, 9) == 0
    # the point of the operators: far less than the logits (4 bytes each) of a large batch
    T, d, V = 8192, 1024, 50257
    assert B.monarch_xent_workspace_bytes(T, d, V, B.BF16) < T * V * 4 / 16
    assert B.monarch_xent_bwd_workspace_bytes(T, d, V, B.BF16) < T * V * 4 / 2
    assert B.monarch_ortho_workspace_bytes(64, 64, 64, B.BF16) >= 256
    assert B.monarch_ortho_workspace_bytes(4, 1024, 1024, B.F32) > 0
    assert B.monarch_ortho_workspace_bytes(0, 1024, 1024, B.F32) >= 256 and B.monarch_ortho_workspace_bytes(0, 8, 8, B.F32) >= 256
    assert B.monarch_ortho_workspace_bytes(4, 0, 1024, B.F32) == 0 and B.monarch_ortho_workspace_bytes(4, 8, 8, 5) == 0


def test_binding_checks_sizes_types_and_layout():
    import torch
    T, d, V = 4, 16, 32
    x, W, y = torch.zeros(T, d), torch.zeros(V, d), torch.zeros(T, dtype=torch.int64)
    loss, lse = torch.zeros(T), torch.zeros(T)
    ws = (256, 1 << 30)
    with pytest.raises(ValueError, match="W must have at least"):
        B.monarch_xent_fwd(x, W[:-1], y, loss, lse, T, d, V, -100, ws, 0)
    with pytest.raises(ValueError, match="loss must have at least"):
        B.monarch_xent_fwd(x, W, y, loss[:2], lse, T, d, V, -100, ws, 0)
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        B.monarch_xent_fwd(x, W, y, loss, lse, T, d, V, -100, ws, 0)
    G = torch.zeros(2, 8, 8)
    with pytest.raises(ValueError, match="O must have at least"):
        B.monarch_orthogonalize(G, G[:1], 2, 8, 8, 5, ws, 0)
    with pytest.raises(ValueError, match="V must have at least"):
        B.monarch_muon_step(G, G, G[:1], 2, 8, 8, 0.1, 0.0, 0.9, 1, 1.0, 5, ws, 0)
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        B.monarch_muon_step(G, G, G, 2, 8, 8, 0.1, 0.0, 0.9, 1, 1.0, 5, ws, 0)
