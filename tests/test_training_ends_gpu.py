"""The vocabulary loss with its gradient and the orthogonalised update against plain float64 forms on the GPU.

Tolerances of the loss are bounds, computed per element from the operands (``acc``): a sum of K products on the tensor cores is
off by at most (steps) * 2^-23 of the sum of their absolute values, a step being 16 products of one plane pair and a run at most
96 steps before it is added up to nearest; exponentials, logarithms and their arguments add 2^-20 relative.  Half a step of bf16
is 2^-8 of the value, so one, two or three parts leave 2^-8, 2^-16 or 2^-24: g is held to three in fp32 and for up to 64 tokens,
else dW takes two fp16 parts (2^-11 each: 2^-22, and x, in fp16, is off by at most 2^-25 of its row's largest), a bf16 dx one; fp32 operands in three parts (2^-24 each) leave out two products of 2^-8 2^-16 as well, 2^-22 in
all; a bf16 result is off by 2^-8.
The orthogonalised update is compared normwise per block.  To first order an error of X grows by at most max |p'| = 3.9 a step
(p(s) = a s + b s^3 + c s^5 on [0, 1.2]) while X itself grows from norm 1 to 0.9 sqrt(k), and each step adds its own rounding, some
30 units (a + 2 |b| s^2 + 3 c s^4): 30 (1 + 3.9 + 15) units over the last three steps, in which nearly all of the norm is there.
With a unit of 2^-24 that is 3.6e-5 at the very worst for fp32 (random errors: 1e-6); the float32 bound of the other calls,
1e-5, is asked for, and by the same growth 3.9 times that for each step beyond five.  bf16: 2^-8 for the rounding of the result and 2^-11 for 16-bit products.
"""
import math

import numpy as np
import pytest
import torch

import paper_2204_00595_b200 as P

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, P.F32), "bf16": (torch.bfloat16, P.BF16)}
IGNORE = -100
CANARY = 4096.0


def acc(k, planes=1):
    """Relative error of a sum of k products (of absolute values) in runs of at most 96 steps."""
    steps = min(96.0, planes * math.ceil(k / 16) + 1)
    return (steps + planes * k / 512 + 2) * 2.0 ** -23


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def guarded(n, dtype):
    """n values with a band behind them that no call may touch."""
    buf = torch.full((n + 256,), CANARY, dtype=dtype, device="cuda")
    return buf, buf[:n]


def untouched(buf, n):
    return bool((buf[n:] == CANARY).all())


def make(T, d, V, dtype, ignored, seed=0, scale=2.0):
    g = gen(seed)
    dt = DT[dtype][0]
    x = torch.randn(T, d, generator=g, device="cuda").to(dt)
    W = (torch.randn(V, d, generator=g, device="cuda") * (scale / math.sqrt(d))).to(dt)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    out = torch.rand(T, generator=g, device="cuda") < ignored
    return x, W, torch.where(out, IGNORE, y), torch.rand(T, generator=g, device="cuda") + 0.1


def forward(x, W, y, ignore=IGNORE, stream=None, ws=None):
    (T, d), V = x.shape, W.shape[0]
    code = P.F32 if x.dtype == torch.float32 else P.BF16
    ws = ws or P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, code))
    lb, loss = guarded(T, torch.float32)
    sb, lse = guarded(T, torch.float32)
    P.monarch_xent_fwd(x, W, y, loss, lse, T, d, V, ignore, ws, stream)
    torch.cuda.synchronize()
    assert P.monarch_last_device_status(ws) == 0
    assert untouched(lb, T) and untouched(sb, T)
    return loss, lse


def backward(x, W, y, lse, dloss, ignore=IGNORE, dW0=None, ws=None):
    (T, d), V = x.shape, W.shape[0]
    code = P.F32 if x.dtype == torch.float32 else P.BF16
    ws = ws or P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, code))
    xb, dx = guarded(T * d, x.dtype)
    wb, dW = guarded(V * d, torch.float32)
    dx.fill_(float("nan"))
    if dW0 is None:
        dW.fill_(float("nan"))
    else:
        dW.copy_(dW0.reshape(-1))
    P.monarch_xent_bwd(x, W, y, lse, dloss, dx, dW, dW0 is not None, T, d, V, ignore, ws)
    torch.cuda.synchronize()
    assert P.monarch_last_device_status(ws) == 0
    assert untouched(xb, T * d) and untouched(wb, V * d)
    return dx.view(T, d), dW.view(V, d)


def exact(x, W, y, dloss=None, ignore=IGNORE):
    """loss, lse, dx, dW in float64 and bounds on the errors of each."""
    dtype = "f32" if x.dtype == torch.float32 else "bf16"
    f32 = dtype == "f32"
    keep = y != ignore
    rows = torch.nonzero(keep)[:, 0]
    xk, Wd, yk = x[rows].double(), W.double(), y[rows]
    d, V = x.shape[1], W.shape[0]
    z = xk @ Wd.T
    mag = xk.abs() @ Wd.abs().T
    dz = mag * (acc(d, 6 if f32 else 1) + (2.0 ** -22 if f32 else 0.0))
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    # an error of a logit enters lse with its probability; the exponentials' own errors enter relative to the sum
    dlse = (p * dz).sum(1) + 2.0 ** -20 * (1.0 + lse.abs())
    loss = lse - z.gather(1, yk[:, None])[:, 0]
    dloss_err = dlse + dz.gather(1, yk[:, None])[:, 0] + 2.0 ** -23 * loss.abs()
    full = lambda v: torch.zeros(x.shape[0], *v.shape[1:], dtype=torch.float64, device="cuda").index_copy_(0, rows, v)  # noqa: E731
    out = {"loss": full(loss), "lse": full(lse), "loss_err": full(dloss_err), "lse_err": full(dlse)}
    if dloss is None:
        return out
    given = lse.float().double()                          # the lse that the backward pass is given
    p = torch.exp(z - given[:, None])
    w = dloss[rows].double()[:, None]
    onehot = torch.zeros_like(p).scatter_(1, yk[:, None], 1.0)
    gr = w * (p - onehot)
    three = f32 or x.shape[0] <= 64
    dg = w * p * (dz + 2.0 ** -20 * (1.0 + z.abs() / 16)) + gr.abs() * ((2.0 ** -24 if three else 2.0 ** -22) + 2.0 ** -23)
    dg1 = dg if f32 else dg + gr.abs() * 2.0 ** -8
    xa, Wa = xk.abs(), Wd.abs()
    w_planes = 2.0 ** -22 if f32 else 0.0
    out["dx"] = full(gr @ Wd)
    out["dx_err"] = full(dg1 @ Wa + (gr.abs() @ Wa) * ((acc(V, 6) if f32 else V / 16 * 2.0 ** -23 + 2.0 ** -20) + w_planes)
                         + (gr @ Wd).abs() * (2.0 ** -23 if f32 else 2.0 ** -8))
    out["dW"] = gr.T @ xk
    T = rows.numel()
    if not three:                                          # x in fp16, and g' = g 2^(a - E + 13) below 2^14 to 2^-25 of its unit
        top = xa.amax(1, keepdim=True)
        big = float((top[:, 0] * w[:, 0].abs()).max())
        extra = gr.abs().T @ (top * 2.0 ** -24).expand_as(xk) + 2.0 ** -37 * big * rows.numel()
    else:
        extra = 0.0
    out["dW_err"] = extra + dg.T @ xa + (gr.abs().T @ xa) * (acc(T, 6 if f32 else 3) + w_planes) + out["dW"].abs() * 2.0 ** -23
    return out


def within(got, want, err, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - err - 1e-30
    assert float(over.max()) <= 0.0, f"{what}: off by {float((got - want).abs().max()):.3e}, over its bound by {float(over.max()):.3e}"


SIZES = [
    # tokens, d, vocab, ignored
    (1, 8, 1, 0.0), (1, 16, 7, 0.0), (1, 1024, 1000, 0.0), (2, 64, 256, 0.5), (7, 72, 255, 0.0), (63, 128, 257, 0.3),
    (64, 8, 512, 0.0), (127, 256, 1000, 0.1), (128, 200, 128, 0.9), (129, 1, 300, 0.0), (255, 67, 1001, 0.2), (256, 64, 2048, 0.0),
    (3, 512, 5000, 0.0), (8, 40, 16, 0.5), (9, 2048, 1500, 0.2), (16, 136, 999, 0.0), (17, 64, 2000, 0.3), (32, 1024, 3000, 0.1), (33, 1024, 3000, 0.0),
    (257, 136, 4099, 0.5), (300, 1032, 777, 0.0), (600, 250, 511, 0.1), (1000, 96, 20000, 0.2),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V,ignored", SIZES)
def test_loss_and_gradient(T, d, V, ignored, dtype):
    x, W, y, dloss = make(T, d, V, dtype, ignored, seed=T + d)
    e = exact(x, W, y, dloss)
    loss, lse = forward(x, W, y)
    within(loss, e["loss"], e["loss_err"], "loss")
    within(lse, e["lse"], e["lse_err"], "lse")
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")


@pytest.mark.parametrize("T,d,V", [(17, 1024, 3001), (32, 520, 999), (33, 520, 999), (47, 72, 5000), (48, 128, 257), (49, 128, 257), (8, 4096, 600),
                                   (9, 4096, 600), (24, 4096, 600), (25, 4096, 600), (16, 2048, 600), (40, 2048, 600),
                                   (15, 104, 261), (45, 104, 261), (16, 110, 50), (8, 512, 90), (8, 576, 90)])
def test_loss_of_few_fp32_tokens(T, d, V):
    """one, two or three launches of few tokens each, the first sizes beyond them, and shared memory of just under 48 KB"""
    x, W, y, _ = make(T, d, V, "f32", 0.1, seed=T + d)
    e = exact(x, W, y)
    loss, lse = forward(x, W, y)
    within(loss, e["loss"], e["loss_err"], "loss")
    within(lse, e["lse"], e["lse_err"], "lse")
    dloss = torch.rand(T, generator=gen(T), device="cuda")
    b = exact(x, W, y, dloss)
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, b["dx"], b["dx_err"], "dx")
    within(dW, b["dW"], b["dW_err"], "dW")
    for t in range(0, T, 5):                               # a token's result does not depend on its neighbours' launch
        alone, _ = forward(x[t:t + 1].clone(), W, y[t:t + 1])            # rows of x need not be 16 bytes aligned, a call's x is
        within(alone, e["loss"][t:t + 1], e["loss_err"][t:t + 1], "loss of one")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ignored_rows_may_hold_anything(dtype):
    T, d, V = 200, 96, 700
    x, W, y, dloss = make(T, d, V, dtype, 0.4, seed=3)
    e = exact(x, W, y, dloss)
    out = y == IGNORE
    lse_in = e["lse"].float()
    x[out] = float("nan")
    x[torch.nonzero(out)[0, 0]] = float("inf")
    dloss = torch.where(out, float("nan"), dloss)
    lse_in = torch.where(out, float("inf"), lse_in)
    loss, lse = forward(x, W, y)
    within(loss, e["loss"], e["loss_err"], "loss")
    within(lse, e["lse"], e["lse_err"], "lse")
    assert (loss[out] == 0).all() and (lse[out] == 0).all()
    dx, dW = backward(x, W, y, lse_in, dloss)
    assert (dx[out] == 0).all()
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")


def test_every_token_ignored_and_no_tokens():
    T, d, V = 70, 64, 300
    x, W, y, dloss = make(T, d, V, "bf16", 1.1, seed=4)
    loss, lse = forward(x, W, y)
    assert (loss == 0).all() and (lse == 0).all()
    dx, dW = backward(x, W, y, lse, dloss)
    assert (dx == 0).all() and (dW == 0).all()
    before = torch.randn(V, d, device="cuda")
    _, dW = backward(x, W, y, lse, dloss, dW0=before)
    assert torch.equal(dW, before)
    empty = x[:0]
    loss, lse = forward(empty, W, y[:0])
    assert loss.numel() == 0
    _, dW = backward(empty, W, y[:0], lse, dloss[:0])
    assert (dW == 0).all()
    _, dW = backward(empty, W, y[:0], lse, dloss[:0], dW0=before)
    assert torch.equal(dW, before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(1, 8, 1), (1, 520, 70), (3, 136, 4097), (8, 1024, 3001), (9, 1032, 600), (13, 40, 20000), (16, 64, 63), (16, 2048, 900),
                                   (1, 1, 1), (1, 313, 3001), (2, 7, 40), (5, 1018, 700), (8, 129, 9), (8, 33, 2000), (9, 65, 1000), (16, 1001, 300), (12, 4, 77)])
def test_gradient_of_few_tokens(T, d, V, dtype):
    """Up to 16 tokens: masked rows that are not numbers, targets out of range, added to what is there, the same bits again and replayed."""
    x, W, y, dloss = make(T, d, V, dtype, 0.3, seed=T * d)
    e = exact(x, W, y, dloss)
    got, lse = forward(x, W, y)
    within(got, e["loss"], e["loss_err"], "loss")
    within(lse, e["lse"], e["lse_err"], "lse")
    lse = e["lse"].float()
    out = y == IGNORE
    x[out] = float("nan")
    dloss[out] = float("inf")
    lse[out] = float("nan")
    before = torch.randn(V, d, device="cuda")
    dx, dW = backward(x, W, y, lse, dloss, dW0=before)
    within(dx, e["dx"], e["dx_err"], "dx")
    assert (dx[out] == 0).all()
    within(dW, e["dW"] + before.double(), e["dW_err"] + (before.double().abs() + e["dW"].abs()) * 2.0 ** -23, "dW")
    dx, dW = backward(x, W, y, lse, dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")
    ws = P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, DT[dtype][1]))
    gx, gw = torch.zeros_like(x), torch.zeros(V, d, device="cuda")
    ys = torch.full_like(y, IGNORE)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.monarch_xent_bwd(x, W, ys, lse, dloss, gx, gw, 0, T, d, V, IGNORE, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.monarch_xent_bwd(x, W, ys, lse, dloss, gx, gw, 0, T, d, V, IGNORE, ws)
    graph.replay()
    assert (gw == 0).all() and (gx == 0).all()
    ys.copy_(y)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(gx, dx) and torch.equal(gw, dW)
    keep = torch.nonzero(~out)[:, 0]
    if keep.numel() > 1:
        y[keep[0]] = V
        dx, dW = backward(x, W, y, lse, dloss)
        assert torch.isnan(dx[keep[0]]).all() and torch.isnan(dW).all()
        within(dx[keep[1:]], e["dx"][keep[1:]], e["dx_err"][keep[1:]], "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V,ignored", [(4704, 491, 65, 0.0), (1024, 64, 10, 0.0), (1023, 64, 10, 0.0), (3000, 300, 700, 0.9), (2500, 136, 1, 0.0), (5000, 33, 257, 1.1)])
def test_gradient_of_a_small_vocabulary(T, d, V, ignored, dtype):
    """dW in parts of the tokens (1024 of them and more): few tiles, most or all tokens left out, added to what is there."""
    x, W, y, dloss = make(T, d, V, dtype, ignored, seed=T + V)
    before = torch.randn(V, d, device="cuda")
    if ignored > 1.0:
        dx, dW = backward(x, W, y, torch.zeros(T, device="cuda"), dloss)
        assert (dx == 0).all() and (dW == 0).all()
        _, dW = backward(x, W, y, torch.zeros(T, device="cuda"), dloss, dW0=before)
        assert torch.equal(dW, before)
        return
    e = exact(x, W, y, dloss)
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")
    _, again = backward(x, W, y, e["lse"].float(), dloss)
    assert torch.equal(dW, again)
    _, dW = backward(x, W, y, e["lse"].float(), dloss, dW0=before)
    within(dW, e["dW"] + before.double(), e["dW_err"] + (before.double().abs() + e["dW"].abs()) * 2.0 ** -23, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accumulate_adds(dtype):
    T, d, V = 150, 80, 900
    x, W, y, dloss = make(T, d, V, dtype, 0.0, seed=5)
    e = exact(x, W, y, dloss)
    before = torch.randn(V, d, device="cuda")
    _, dW = backward(x, W, y, e["lse"].float(), dloss, dW0=before)
    within(dW, e["dW"] + before.double(), e["dW_err"] + (before.double().abs() + e["dW"].abs()) * 2.0 ** -23, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_of_very_different_size(dtype):
    """Rows of x from 1e-12 to 1e6, zero rows, weights of tokens from 0 to 1e8 and down to 1e-30: each token has its own scale on the way."""
    T, d, V = 200, 96, 700
    x, W, y, dloss = make(T, d, V, dtype, 0.1, seed=13)
    g = gen(14)
    s = 10.0 ** (torch.rand(T, 1, generator=g, device="cuda") * 18 - 12)
    x = (x.double() * s.double()).to(x.dtype)
    x[7] = 0.0
    x[9, 1:] = 0.0
    W = (W.double() * 1e-6).to(W.dtype)                    # logits stay moderate
    dloss = (dloss.double() * 10.0 ** (torch.rand(T, generator=g, device="cuda").double() * 38 - 30)).float()
    dloss[3] = 0.0
    e = exact(x, W, y, dloss)
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")
    _, dW = backward(x, W, y, e["lse"].float(), torch.zeros_like(dloss))
    assert (dW == 0).all()


def test_targets_out_of_range_and_any_ignore_index():
    T, d, V = 40, 64, 300
    x, W, y, dloss = make(T, d, V, "bf16", 0.0, seed=6)
    bad = y.clone()
    bad[3], bad[17], bad[20] = V, -1, 1 << 40
    e = exact(x, W, y, dloss)
    loss, lse = forward(x, W, bad)
    at = torch.tensor([3, 17, 20], device="cuda")
    assert torch.isnan(loss[at]).all()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[at] = False
    within(loss[rest], e["loss"][rest], e["loss_err"][rest], "loss")
    within(lse, e["lse"], e["lse_err"], "lse")
    dx, dW = backward(x, W, bad, e["lse"].float(), dloss)
    assert torch.isnan(dx[at]).all() and torch.isfinite(dx[rest]).all() and torch.isnan(dW).any()
    # an ignore_index inside the vocabulary, and one of 40 bits
    y[:10] = 7
    e7 = exact(x, W, y, dloss, ignore=7)
    loss, _ = forward(x, W, y, ignore=7)
    within(loss, e7["loss"], e7["loss_err"], "loss")
    y[:10] = 1 << 40
    loss, _ = forward(x, W, y, ignore=1 << 40)
    assert (loss[:10] == 0).all() and torch.isfinite(loss).all()


def test_large_and_masked_logits():
    """Logits of hundreds (the maximum is taken off), entries masked by the lowest value of the type, and rows that are not finite."""
    T, d, V = 64, 64, 600
    x, W, y, dloss = make(T, d, V, "f32", 0.0, seed=7, scale=200.0)
    e = exact(x, W, y, dloss)
    loss, lse = forward(x, W, y)
    within(loss, e["loss"], e["loss_err"], "loss")
    x[:, 0] = 1.0
    W[:300, 0] = torch.finfo(torch.float32).min            # the first tiles of every row: masked out
    y = y.clamp(min=300)
    W[300:, 1:] *= 0.01
    x.clamp_(min=0.0, max=1e-3)
    x[:, 0] = 1.0
    W[:300, 1:] = 0.0
    keep = W[300:].double()
    want = torch.logsumexp(x.double() @ keep.T, 1)
    loss, lse = forward(x, W, y)
    assert torch.allclose(lse.double(), want, rtol=1e-5, atol=1e-5)
    x[5, 3] = float("nan")
    loss, lse = forward(x, W, y)
    assert torch.isnan(loss[5]) and torch.isnan(lse[5])
    rest = torch.arange(T, device="cuda") != 5
    assert torch.isfinite(loss[rest]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 5, 12])
def test_masked_logits_of_few_tokens(T, dtype):
    """Entries masked by the lowest value of the type have no part in the loss nor in dx, and dW = 0; a token that is not a number keeps to itself."""
    d, V = 64, 500
    x, W, y, dloss = make(T, d, V, dtype, 0.0, seed=17 + T)
    y = y.clamp(min=200)
    x[:, 0] = 1.0
    W[:, 0] = 0.0
    live = exact(x, W[200:].contiguous(), y - 200, dloss)
    W[:200, 0] = torch.finfo(W.dtype).min
    loss, lse = forward(x, W, y)
    within(loss, live["loss"], live["loss_err"], "loss")
    within(lse, live["lse"], live["lse_err"], "lse")
    dx, dW = backward(x, W, y, live["lse"].float(), dloss)
    within(dx[:, 1:], live["dx"][:, 1:], live["dx_err"][:, 1:], "dx")
    assert (dW[:200] == 0).all()
    within(dW[200:], live["dW"], live["dW_err"], "dW")
    x[0, 3] = float("nan")
    loss, lse = forward(x, W, y)
    assert torch.isnan(loss[0]) and torch.isnan(lse[0])
    if T > 1:
        within(loss[1:], live["loss"][1:], live["loss_err"][1:], "loss of the others")
        dx, _ = backward(x, W, y, live["lse"].float(), dloss)
        assert torch.isnan(dx[0]).all()
        within(dx[1:, 1:], live["dx"][1:, 1:], live["dx_err"][1:, 1:], "dx of the others")


def test_shifted_labels_in_place_and_other_stream():
    """targets[1:] (8 bytes off a 16-byte boundary) and per-token outputs at odd offsets; a stream that is not the current one."""
    T, d, V = 90, 64, 500
    x, W, y, dloss = make(T + 1, d, V, "bf16", 0.0, seed=8)
    e = exact(x[:T], W, y[1:])
    s = torch.cuda.Stream()
    ws = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, P.BF16))
    out = torch.zeros(T + 1, device="cuda")
    lse = torch.zeros(T + 1, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    P.monarch_xent_fwd(x[:T], W, y[1:], out[1:], lse[1:], T, d, V, IGNORE, ws, s)
    s.synchronize()
    within(out[1:], e["loss"], e["loss_err"], "loss")
    assert out[0] == 0 and lse[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_every_run_and_in_a_graph(dtype):
    T, d, V = 333, 136, 3001
    x, W, y, dloss = make(T, d, V, dtype, 0.2, seed=9)
    loss, lse = forward(x, W, y)
    dx, dW = backward(x, W, y, lse, dloss)
    loss2, lse2 = forward(x, W, y)
    dx2, dW2 = backward(x, W, y, lse, dloss)
    for a, b in ((loss, loss2), (lse, lse2), (dx, dx2), (dW, dW2)):
        assert torch.equal(a, b)
    code = DT[dtype][1]
    fws = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, code))
    bws = P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, code))
    gl, gs = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    gx, gw = torch.zeros_like(x), torch.zeros(V, d, device="cuda")
    xs, ys = torch.zeros_like(x), torch.full_like(y, IGNORE)

    def step():
        P.monarch_xent_fwd(xs, W, ys, gl, gs, T, d, V, IGNORE, fws)
        P.monarch_xent_bwd(xs, W, ys, gs, dloss, gx, gw, 0, T, d, V, IGNORE, bws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    # captured with every token left out; replayed with other tokens and another number of them
    xs.copy_(x)
    ys.copy_(y)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in ((loss, gl), (lse, gs), (dx, gx), (dW, gw)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [5, 20, 100])
def test_one_workspace_for_calls_that_follow_one_another(T):
    """A workspace large enough for all may serve every call of the library in turn: none leaves anything there that another minds."""
    d, V, m, rows = 128, 700, 128, 300
    big = max(P.monarch_xent_workspace_bytes(T, d, V, P.BF16), P.monarch_xent_bwd_workspace_bytes(T, d, V, P.BF16),
              P.monarch_workspace_bytes(P.OP_FWD, rows, m * m, m, P.BF16), P.monarch_workspace_bytes(P.OP_BWD, rows, m * m, m, P.BF16),
              P.monarch_ortho_workspace_bytes(1, 200, 200, P.BF16), P.monarch_workspace_bytes(P.OP_FWD, 500, 256, 16, P.F32))
    ws = P.Workspace(big)
    g = gen(3)
    r = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    a, L, R = r(rows, m * m), r(m, m, m) / 12, r(m, m, m) / 12
    f, Lf, Rf = r(500, 256, dt=torch.float32), r(16, 16, 16, dt=torch.float32), r(16, 16, 16, dt=torch.float32)
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=1)
    G = gradient(1, 200, 200, 9).bfloat16()

    def everything():
        out = [torch.empty_like(a), torch.empty_like(f), torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x),
               torch.empty(V, d, device="cuda"), torch.empty_like(G), torch.empty_like(G[:, :128, :128].contiguous())]
        P.monarch_fwd(a, L, R, out[0], rows, m * m, m, ws)
        P.monarch_xent_fwd(x, W, y, out[2], out[3], T, d, V, IGNORE, ws)
        P.monarch_fwd(f, Lf, Rf, out[1], 500, 256, 16, ws)
        P.monarch_xent_bwd(x, W, y, out[3], dloss, out[4], out[5], 0, T, d, V, IGNORE, ws)
        P.monarch_orthogonalize(G, out[6], 1, 200, 200, 5, ws)
        P.monarch_orthogonalize(G[:, :128, :128].contiguous(), out[7], 1, 128, 128, 5, ws)
        torch.cuda.synchronize()
        assert P.monarch_last_device_status(ws) == 0
        return out

    first = everything()
    for _ in range(2):
        for p, q in zip(first, everything()):
            assert torch.equal(p, q)
    fresh = torch.empty_like(a)
    P.monarch_fwd(a, L, R, fresh, rows, m * m, m, P.Workspace.for_op(P.OP_FWD, rows, m, P.BF16))
    assert torch.equal(fresh, first[0])


def test_pieces_of_the_vocabulary_and_token_chunks():
    """Sizes that take several pieces in the backward pass, and more tokens than one chunk of partial sums."""
    T, d, V = 33000, 16, 9000
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=10)
    e = exact(x, W, y, dloss)
    loss, lse = forward(x, W, y)
    within(loss, e["loss"], e["loss_err"], "loss")
    dx, dW = backward(x, W, y, e["lse"].float(), dloss)
    within(dx, e["dx"], e["dx_err"], "dx")
    within(dW, e["dW"], e["dW_err"], "dW")


def test_gradient_against_differences():
    """<dx, u> and <dW, w> against central differences of the float64 loss along u and w."""
    T, d, V = 60, 48, 400
    x, W, y, dloss = make(T, d, V, "f32", 0.1, seed=11)
    _, lse = forward(x, W, y)
    dx, dW = backward(x, W, y, lse, dloss)
    g = gen(1)
    u = torch.randn(T, d, generator=g, device="cuda").double()
    w = torch.randn(V, d, generator=g, device="cuda").double() / math.sqrt(d)
    keep = y != IGNORE

    def total(h, k):
        z = (x.double() + h * u) @ (W.double() + k * w).T
        z = z[keep]
        return float((dloss.double()[keep] * (torch.logsumexp(z, 1) - z.gather(1, y[keep][:, None])[:, 0])).sum())

    h = 1e-4                                               # truncation h^2 f''' / 6 is some 1e-8 of f'
    for got, want in ((float((dx.double() * u).sum()), (total(h, 0) - total(-h, 0)) / (2 * h)),
                      (float((dW.double() * w).sum()), (total(0, h) - total(0, -h)) / (2 * h))):
        assert abs(got - want) <= 1e-5 * max(1.0, abs(want))


# ------------------------------------------------------------------------------------------------ orthogonalisation
A, B, C = 3.4445, -4.7750, 2.0315


def newton_schulz(u, steps=5):
    x = u / (torch.linalg.vector_norm(u, dim=(1, 2), keepdim=True) + 1e-7)
    for _ in range(steps):
        s = x @ x.mT if x.shape[1] <= x.shape[2] else x.mT @ x
        p = B * s + C * (s @ s)
        x = A * x + (p @ x if x.shape[1] <= x.shape[2] else x @ p)
    return x


def gradient(blocks, rows, cols, seed, scale=1e-2):
    g = gen(seed)
    k = max(1, min(rows, cols) // 4)
    low = torch.randn(blocks, rows, k, generator=g, device="cuda") @ torch.randn(blocks, k, cols, generator=g, device="cuda")
    return scale * (low + 0.1 * torch.randn(blocks, rows, cols, generator=g, device="cuda"))


def near(got, want, dtype, what, steps=5):
    got, want = got.double(), want.double()
    tol = 1e-5 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -11
    tol *= 3.9 ** max(0, steps - 5)
    off = torch.linalg.vector_norm(got - want, dim=(1, 2))
    size = torch.linalg.vector_norm(want, dim=(1, 2))
    assert torch.isfinite(got).all(), what
    assert bool((off <= tol * size).all()), f"{what}: {float((off / size.clamp(min=1e-300)).max()):.3e} of the norm"


def ortho(G, steps=5, ws=None):
    blocks, rows, cols = G.shape
    code = P.F32 if G.dtype == torch.float32 else P.BF16
    ws = ws or P.Workspace(P.monarch_ortho_workspace_bytes(blocks, rows, cols, code))
    buf, O = guarded(G.numel(), G.dtype)
    O.fill_(float("nan"))
    P.monarch_orthogonalize(G, O, blocks, rows, cols, steps, ws)
    torch.cuda.synchronize()
    assert P.monarch_last_device_status(ws) == 0
    assert untouched(buf, G.numel())
    return O.view_as(G)


BLOCKS = [
    (1, 1, 1), (5, 1, 9), (5, 9, 1), (3, 2, 2), (7, 3, 5), (4, 16, 16), (33, 8, 12), (3, 17, 15), (2, 31, 33), (6, 32, 32), (3, 33, 80),
    (2, 64, 64), (5, 63, 65), (2, 64, 20), (2, 100, 127), (2, 128, 128), (1, 127, 128), (2, 128, 64), (3, 4, 1000), (3, 1000, 4), (1, 129, 129),
    (2, 130, 256), (2, 256, 130), (1, 200, 301), (1, 301, 200), (2, 256, 256), (1, 512, 640), (1, 65, 2000), (1, 2000, 65), (1, 1030, 1031),
    (2, 1, 20000), (1, 20000, 2), (3, 64, 200), (2, 200, 40), (5, 32, 256), (2, 257, 32), (200, 33, 64), (150, 5, 6), (2, 64, 129), (90, 130, 131),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blocks,rows,cols", BLOCKS)
def test_orthogonalize(blocks, rows, cols, dtype):
    G = gradient(blocks, rows, cols, seed=rows * 7 + cols).to(DT[dtype][0])
    near(ortho(G), newton_schulz(G.double()), dtype, "O")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blocks,rows,cols", [(132, 5, 251), (3, 251, 5), (2, 16, 256), (300, 16, 129), (1, 1, 200), (2, 17, 256), (2, 16, 257), (2, 16, 128),
                                              (2, 9, 65), (2, 33, 256), (2, 48, 130), (2, 64, 256), (2, 65, 256), (2, 32, 257), (2, 4, 1528), (2, 4, 1525)])
def test_orthogonalize_sides_where_the_kernels_change(blocks, rows, cols, dtype):
    """Both sides of the rules that choose a kernel and its padding; 16 x 256 has one column tile per warp and one buffer of X, 4 x 1528
    48 KB of shared memory beside the static ones."""
    G = gradient(blocks, rows, cols, seed=rows * 7 + cols).to(DT[dtype][0])
    near(ortho(G), newton_schulz(G.double()), dtype, "O")


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
@pytest.mark.parametrize("blocks,rows,cols", [(3, 24, 40), (2, 150, 140)])
def test_other_numbers_of_steps(blocks, rows, cols, steps):
    G = gradient(blocks, rows, cols, seed=steps)
    near(ortho(G, steps), newton_schulz(G.double(), steps), "f32", "O", steps)


@pytest.mark.parametrize("rows,cols", [(16, 16), (64, 64), (40, 60), (128, 128), (160, 200)])
def test_blocks_stand_alone(rows, cols):
    """Zeros give zeros; NaN and infinity stay in their block; norms beyond the range of fp32 squares, and tiny ones."""
    G = gradient(8, rows, cols, seed=2)
    G[1] = 0.0
    G[2, 3, 5] = float("nan")
    G[3, 0, 0] = float("inf")
    G[4] *= 1e30
    G[5] *= 1e-30                                          # below the 1e-7 that keeps off a division by zero
    G[6] *= 1e-6
    O = ortho(G)
    assert (O[1] == 0).all()
    assert torch.isnan(O[2]).all() and torch.isnan(O[3]).all()
    fine = [0, 4, 6, 7]
    near(O[fine], newton_schulz(G[fine].double()), "f32", "O")
    want = newton_schulz(G[5:6].double())                  # about a^5 U / 1e-7
    near(O[5:6], want, "f32", "O")


def test_two_streams_at_once():
    """Calls that overlap on the GPU, each with a workspace of its own; the stacks of large blocks are launches whose CTAs wait for
    one another."""
    T, d, V = 700, 256, 5000
    x, W, y, dloss = make(T, d, V, "bf16", 0.1, seed=30)
    G = [gradient(3, 300, 520, 31 + i).to(dt) for i, dt in enumerate((torch.bfloat16, torch.float32))]
    want = [ortho(g) for g in G]
    loss, lse = forward(x, W, y)
    dx, dW = backward(x, W, y, lse, dloss)
    ws = [P.Workspace(P.monarch_ortho_workspace_bytes(3, 300, 520, c)) for c in (P.BF16, P.F32)]
    wf, wb = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, P.BF16)), P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, P.BF16))
    out = [torch.empty_like(g) for g in G]
    l2, s2, dx2, dW2 = torch.empty_like(loss), torch.empty_like(lse), torch.empty_like(dx), torch.empty_like(dW)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            P.monarch_orthogonalize(G[i], out[i], 3, 300, 520, 5, ws[i], streams[i])
        P.monarch_xent_fwd(x, W, y, l2, s2, T, d, V, IGNORE, wf, streams[2])
        P.monarch_xent_bwd(x, W, y, s2, dloss, dx2, dW2, 0, T, d, V, IGNORE, wb, streams[2])
    torch.cuda.synchronize()
    for w in ws + [wf, wb]:
        assert P.monarch_last_device_status(w) == 0
    for a, b in zip(want + [loss, lse, dx, dW], out + [l2, s2, dx2, dW2]):
        assert torch.equal(a.view(-1), b.view(-1))


def test_result_is_nearly_orthogonal():
    G = gradient(4, 64, 64, seed=12)
    s = torch.linalg.svdvals(ortho(G).double())
    u = torch.linalg.svdvals(G.double())
    strong = u > 0.02 * torch.linalg.vector_norm(u, dim=1, keepdim=True)
    assert float(s.max()) < 1.3 and float(s[strong].min()) > 0.6


def muon(W, dW, V, lr, wd, beta, nesterov, scale, steps=5):
    blocks, rows, cols = W.shape
    code = P.F32 if W.dtype == torch.float32 else P.BF16
    ws = P.Workspace(P.monarch_ortho_workspace_bytes(blocks, rows, cols, code))
    P.monarch_muon_step(W, dW, V, blocks, rows, cols, lr, wd, beta, nesterov, scale, steps, ws)
    torch.cuda.synchronize()
    assert P.monarch_last_device_status(ws) == 0


@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blocks,rows,cols", [(1, 1, 1), (16, 16, 16), (3, 33, 80), (64, 64, 64), (2, 128, 128), (3, 90, 20), (2, 140, 260),
                                              (2, 260, 140), (1, 300, 300)])
def test_muon_step(blocks, rows, cols, dtype, nesterov):
    g = gen(rows)
    W = (torch.randn(blocks, rows, cols, generator=g, device="cuda") / math.sqrt(cols)).to(DT[dtype][0])
    dW, V = gradient(blocks, rows, cols, 3), gradient(blocks, rows, cols, 4, 0.1)
    lr, wd, beta, scale = 0.3, 0.1, 0.9, 1.5
    v = beta * V.double() + dW.double()
    o = newton_schulz(dW.double() + beta * v if nesterov else v)
    w = (1 - lr * wd) * W.double() - lr * scale * o
    kept = dW.clone()
    muon(W, dW, V, lr, wd, beta, nesterov, scale)
    assert torch.equal(dW, kept)
    # V: one product and one sum, each to nearest
    assert bool(((V.double() - v).abs() <= 2.0 ** -23 * (v.abs() + kept.double().abs() + 1e-30)).all())
    off = torch.linalg.vector_norm(W.double() - w, dim=(1, 2))
    part = lr * scale * torch.linalg.vector_norm(o, dim=(1, 2))
    unit = 2.0 ** -23 if dtype == "f32" else 2.0 ** -8
    tol = unit * torch.linalg.vector_norm(w, dim=(1, 2)) + (1e-5 if dtype == "f32" else 2.0 ** -11) * part + 2.0 ** -23 * part
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("rows,cols", [(64, 64), (150, 200)])
def test_muon_step_in_a_graph_and_without_blocks(rows, cols):
    W = torch.randn(3, rows, cols, device="cuda") / math.sqrt(cols)
    dW, V = gradient(3, rows, cols, 5), torch.zeros(3, rows, cols, device="cuda")
    W1, V1 = W.clone(), V.clone()
    for _ in range(3):
        muon(W1, dW, V1, 0.02, 0.1, 0.95, 1, 1.0)
    ws = P.Workspace(P.monarch_ortho_workspace_bytes(3, rows, cols, P.F32))
    W2, V2 = W.clone(), V.clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.monarch_muon_step(W2, dW, V2, 3, rows, cols, 0.02, 0.1, 0.95, 1, 1.0, 5, ws)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        P.monarch_muon_step(W2, dW, V2, 3, rows, cols, 0.02, 0.1, 0.95, 1, 1.0, 5, ws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(W1, W2) and torch.equal(V1, V2)
    none = W[:0]
    P.monarch_muon_step(none, dW[:0], V[:0], 0, rows, cols, 0.02, 0.1, 0.95, 1, 1.0, 5, ws)
    P.monarch_orthogonalize(none, none.clone(), 0, rows, cols, 5, ws)


# ------------------------------------------------------------------------------------------------ together
def dense(L, R):
    """M[l*m+j][k*m+i] = L[j][l][k] R[k][j][i], differentiable."""
    m = L.shape[0]
    return torch.einsum("jlk,kji->ljki", L, R).reshape(m * m, m * m)


def test_training_step():
    """Feed-forward block -> vocabulary loss -> its gradient -> the block's gradients -> updates of the factors, fp32, against
    float64 automatic differentiation of the dense form."""
    m, T, V = 16, 48, 300
    n = m * m
    g = gen(21)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, head = r(T, n), 2.0 / math.sqrt(n) * r(V, n)
    f = {k: r(m, m, m) / math.sqrt(m) for k in ("L1", "R1", "L2", "R2")}
    b1, b2 = 0.1 * r(n), 0.1 * r(n)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[::7] = IGNORE
    count = int((y != IGNORE).sum())
    dloss = torch.full((T,), 1.0 / count, device="cuda")

    h, dh, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dhead = torch.empty(V, n, device="cuda")
    grads = {k: torch.empty(m, m, m, device="cuda") for k in f}
    db1, db2 = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    w1, w2 = P.Workspace.for_op(P.OP_MLP_FWD, T, m, P.F32), P.Workspace.for_op(P.OP_MLP_BWD, T, m, P.F32)
    w3 = P.Workspace(P.monarch_xent_workspace_bytes(T, n, V, P.F32))
    w4 = P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, n, V, P.F32))
    w5 = P.Workspace(P.monarch_ortho_workspace_bytes(m, m, m, P.F32))
    P.monarch_mlp_fwd(x, f["L1"], f["R1"], b1, f["L2"], f["R2"], b2, h, T, n, m, w1)
    P.monarch_xent_fwd(h, head, y, loss, lse, T, n, V, IGNORE, w3)
    P.monarch_xent_bwd(h, head, y, lse, dloss, dh, dhead, 0, T, n, V, IGNORE, w4)
    P.monarch_mlp_bwd(x, dh, f["L1"], f["R1"], b1, f["L2"], f["R2"], dx, grads["L1"], grads["R1"], db1, grads["L2"], grads["R2"], db2, 0,
                      T, n, m, w2)
    new = {k: v.clone() for k, v in f.items()}
    mom = {k: torch.zeros_like(v) for k, v in f.items()}
    for k in f:
        P.monarch_muon_step(new[k], grads[k], mom[k], m, m, m, 0.02, 0.1, 0.95, 1, 1.0, 5, w5)

    p = {k: v.double().requires_grad_() for k, v in f.items()}
    hd = head.double().requires_grad_()
    a = torch.nn.functional.gelu(x.double() @ dense(p["L1"], p["R1"]).T + b1.double())
    z = (a @ dense(p["L2"], p["R2"]).T + b2.double()) @ hd.T
    keep = y != IGNORE
    want = torch.where(keep, torch.logsumexp(z, 1) - z.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    (want * dloss.double()).sum().backward()
    want = want.detach()
    assert float((loss.double() - want).abs().max()) < 1e-5 * float(want.max())
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(dhead, hd.grad) < 2e-5
    for k in f:
        assert rel(grads[k], p[k].grad) < 2e-5, k
        o = newton_schulz(1.95 * grads[k].double())          # V = g, U = g + 0.95 V, of the gradients that the update was given
        w = (1 - 0.02 * 0.1) * f[k].double() - 0.02 * o
        assert rel(new[k], w) < 1e-6, k
