"""A workspace that was asked for with some number of tokens or blocks serves every smaller one: on the host alone.  The calls below are
given outputs that overlap, which is found behind the check of the workspace and before anything is launched."""
import random

import pytest

import __graft_entry__ as entry
from paper_2204_00595_b200 import binding as B

INVALID, WORKSPACE = 1, 3
ADDRESS = [(i + 1) << 44 for i in range(8)]      # distinct, far apart, never dereferenced


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return B.lib()


def loss(lib, T, d, V, code, nbytes):
    x, W, y, out, ws = ADDRESS[:5]
    return lib.monarch_xent_fwd(x, W, y, out, out, T, d, V, -100, code, ws, nbytes, None)


def gradient(lib, T, d, V, code, nbytes):
    x, W, y, lse, dl, out, ws = ADDRESS[:7]
    return lib.monarch_xent_bwd(x, W, y, lse, dl, out, out, 0, T, d, V, -100, code, ws, nbytes, None)


def log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


KNOWN = [  # call, dtype, d, vocab, smaller, larger number of tokens: where the smaller one alone is given more
    ("gradient", B.BF16, 1024, 50257, 4096, 5000), ("gradient", B.BF16, 2048, 32000, 7452, 8192), ("gradient", B.F32, 1024, 50257, 1000, 2048),
    ("gradient", B.F32, 4096, 32768, 2048, 8192), ("gradient", B.BF16, 1018, 50257, 1024, 2048), ("loss", B.F32, 4096, 131072, 64, 1024),
]


@pytest.mark.parametrize("call,code,d,V,t,T", KNOWN)
def test_fewer_tokens_with_the_workspace_of_more(lib, call, code, d, V, t, T):
    need = B.monarch_xent_workspace_bytes if call == "loss" else B.monarch_xent_bwd_workspace_bytes
    assert need(t, d, V, code) > need(T, d, V, code)
    run = loss if call == "loss" else gradient
    assert run(lib, t, d, V, code, need(T, d, V, code)) == INVALID


@pytest.mark.parametrize("call", ["loss", "gradient"])
def test_fewer_tokens_with_the_workspace_of_more_at_any_sizes(lib, call):
    rng = random.Random(7)
    need = B.monarch_xent_workspace_bytes if call == "loss" else B.monarch_xent_bwd_workspace_bytes
    run = loss if call == "loss" else gradient
    more = 0
    for _ in range(4000):
        code, d, V = rng.choice([B.F32, B.BF16]), log_int(rng, 1, 16384), log_int(rng, 1, 300000)
        d = d if rng.random() < 0.5 else (d + 7) // 8 * 8
        T = log_int(rng, 1, 100000)
        t = max(1, rng.choice([rng.randint(1, T), log_int(rng, 1, T), T - 1, (T - 1) // 256 * 256, min(T, rng.choice([16, 17, 32, 48, 128, 129, 512]))]))
        large = need(T, d, V, code)
        more += need(t, d, V, code) > large
        assert run(lib, t, d, V, code, large) == INVALID, (code, d, V, t, T)
        assert run(lib, t, d, V, code, 1 << 16) == WORKSPACE
    assert more > 20                             # the sizes met are not all of the plain kind


def update(lib, blocks, rows, cols, code, nbytes):
    out, ws = ADDRESS[:2]
    return lib.monarch_orthogonalize(out, out, blocks, rows, cols, 5, code, ws, nbytes, None)


@pytest.mark.parametrize("code,rows,cols,few,many", [(B.BF16, 63, 897, 12, 16), (B.F32, 512, 512, 4, 5), (B.F32, 512, 512, 4, 6)])
def test_fewer_blocks_with_the_workspace_of_more(lib, code, rows, cols, few, many):
    need = B.monarch_ortho_workspace_bytes
    assert need(few, rows, cols, code) > need(many, rows, cols, code)
    assert update(lib, few, rows, cols, code, need(many, rows, cols, code)) == INVALID


def test_fewer_blocks_with_the_workspace_of_more_at_any_sizes(lib):
    rng = random.Random(8)
    more = 0
    for _ in range(4000):
        code, rows, cols = rng.choice([B.F32, B.BF16]), log_int(rng, 1, 4096), log_int(rng, 1, 4096)
        most = log_int(rng, 1, 300)
        blocks = rng.randint(1, most)
        large = B.monarch_ortho_workspace_bytes(most, rows, cols, code)
        more += B.monarch_ortho_workspace_bytes(blocks, rows, cols, code) > large
        assert update(lib, blocks, rows, cols, code, large) == INVALID, (code, rows, cols, blocks, most)
        assert update(lib, blocks, rows, cols, code, 128) == WORKSPACE
    assert more > 20
