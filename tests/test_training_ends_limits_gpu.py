"""The vocabulary loss and the orthogonalised update at the ends of the ranges that their documentation allows: values near the ends
of the types' range, tokens without any word left, several host threads, workspaces of other sizes, waits that run out, and the
precision that the results are promised up to 128 tokens."""

import pytest
import torch

import paper_2204_00595_b200 as P
from tests.test_training_ends_gpu import backward, exact, make, near, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ values near the ends of the range
def scaled(got, want, err, power, what):
    """within, of values so small or large that its absolute allowance would hide or not cover them: times an exact power of two"""
    within(got.double() * 2.0 ** power, want * 2.0 ** power, err * 2.0 ** power, what)


@pytest.mark.parametrize("T", [129, 700])
def test_large_rows_of_x(T):
    """Rows of x up to 3e38 beside a small W: moderate logits, finite gradients."""
    d, V = 96, 700
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=40)
    big = 2.0 ** 116                                       # largest values of a row: 2^117 to 2^119
    x = (x.double() * big).to(x.dtype)
    x[5] = (x[5].double() * 2.0 ** 9).to(x.dtype)          # and one above 2^126
    W = (W.double() / big).to(W.dtype)
    W[:, :8] = 0.0
    dloss = dloss / 1024                                   # sums of some hundred tokens stay in range
    e = exact(x, W, y, dloss)
    assert float(e["dW"].abs().max()) < 1e38
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    assert torch.isfinite(dx).all()
    scaled(dW, e["dW"], e["dW_err"], -100, "dW")


@pytest.mark.parametrize("T", [129, 700])
def test_small_rows_of_x(T):
    """Rows of x around 1e-36: dW keeps the bits that it is promised."""
    d, V = 96, 700
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=41)
    x = (x.double() * 2.0 ** -120).to(x.dtype)
    dloss = dloss * 1e6
    e = exact(x, W, y, dloss)
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    scaled(dW, e["dW"], e["dW_err"], 110, "dW")


@pytest.mark.parametrize("power", [104, -100])
def test_large_and_small_weights_of_tokens(power):
    T, d, V = 300, 96, 700
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=42)
    dloss = (dloss.double() * 2.0 ** power).float()
    e = exact(x, W, y, dloss)
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    scaled(dx, e["dx"], e["dx_err"], -power, "dx")
    scaled(dW, e["dW"], e["dW_err"], -power, "dW")


def test_weights_and_rows_at_opposite_ends():
    """Tokens of large x and small weight beside tokens of small x and large weight: what they add to dW is of one size."""
    T, d, V = 400, 64, 500
    x, W, y, dloss = make(T, d, V, "bf16", 0.0, seed=43)
    s = torch.where(torch.arange(T, device="cuda") % 2 == 0, 2.0 ** 100, 2.0 ** -100).double()
    x = (x.double() * s[:, None]).to(x.dtype)
    dloss = (dloss.double() / s).float()
    W = (W.double() * 2.0 ** -100).to(W.dtype)
    e = exact(x, W, y, dloss)
    _, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dW, e["dW"], e["dW_err"], "dW")
