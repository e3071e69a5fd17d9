"""The vocabulary loss and the orthogonalised update at the ends of the ranges that their documentation allows: values near the ends
of the types' range, tokens without any word left, several host threads, workspaces of other sizes, waits that run out, and the
precision that the results are promised up to 128 tokens."""
import ctypes
import subprocess
import time

import pytest
import torch

import paper_2204_00595_b200 as P
from tests.test_training_ends_gpu import DT, IGNORE, acc, backward, exact, forward, gen, gradient, make, near, newton_schulz, ortho, within

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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 40, 300])
def test_rows_whose_mask_leaves_nothing(T, dtype):
    """Tokens all of whose words are masked by the type's lowest value: finite results, and nothing of them reaches the others."""
    d, V = 64, 500
    x, W, y, _ = make(T, d, V, dtype, 0.0, seed=44)
    lowest = torch.finfo(W.dtype).min
    masked = torch.arange(T, device="cuda") % 2 == 0
    x[:, 0] = 0.0
    W[:, 0] = 0.0
    e = exact(x, W, y)
    x[masked] = 0.0
    x[masked, 0] = 1.0
    W[:, 0] = lowest
    loss, lse = forward(x, W, y)
    within(loss[~masked], e["loss"][~masked], e["loss_err"][~masked], "loss of the others")
    within(lse[~masked], e["lse"][~masked], e["lse_err"][~masked], "lse of the others")
    # z = lowest for every word: lse = lowest + log V, which is lowest in float32 (half a step of it is 1e31)
    assert torch.isfinite(loss[masked]).all() and torch.isfinite(lse[masked]).all()
    assert bool(((lse[masked].double() - lowest).abs() <= 2.0 ** -22 * -lowest).all())
    assert bool((loss[masked].double().abs() <= 2.0 ** -22 * -lowest).all())
    # exp(z - lse) = 1 for the lse that is given: g = dloss (1 - [v == target]), of the others as it was
    dloss = torch.full((T,), 2.0 ** -20, device="cuda")
    given = torch.where(masked, torch.full_like(lse, lowest), e["lse"].float())
    xo = torch.where(masked[:, None], torch.zeros_like(x), x)
    o = exact(xo, torch.cat([torch.zeros_like(W[:, :1]), W[:, 1:]], 1), torch.where(masked, IGNORE, y), dloss)
    dx, dW = backward(x, W, y, given, dloss)
    within(dx[~masked][:, 1:], o["dx"][~masked][:, 1:], o["dx_err"][~masked][:, 1:], "dx of the others")
    assert torch.isfinite(dx).all()
    within(dW[:, 1:], o["dW"][:, 1:], o["dW_err"][:, 1:] + 2.0 ** -37 * 2.0 ** -19 * T, "dW")
    hits = torch.bincount(y[masked], minlength=V).double()
    within(dW[:, 0], 2.0 ** -20 * (float(masked.sum()) - hits), torch.full((V,), 2.0 ** -20 * T * 2.0 ** -20, device="cuda", dtype=torch.float64), "dW of the mask")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 200])
def test_logits_of_3e38(T, dtype):
    d, V = 64, 300
    x, W, y, _ = make(T, d, V, dtype, 0.0, seed=45)
    x[:, 0] = 0.0
    W[:, 0] = 0.0
    e = exact(x, W, y)
    top = float(torch.tensor(3e38).to(W.dtype))
    x[1] = 0.0
    x[1, 0] = 1.0
    W[7, 0] = top
    W[8, 0] = -top
    for target, want in ((7, 0.0), (9, top)):
        y[1] = target
        loss, lse = forward(x, W, y)
        assert float(lse[1]) == pytest.approx(top, rel=2.0 ** -22) and float(loss[1]) == pytest.approx(want, rel=2.0 ** -22)
        rest = torch.arange(T, device="cuda") != 1
        within(loss[rest], e["loss"][rest], e["loss_err"][rest], "loss of the others")


# ------------------------------------------------------------------------------------------------ several host threads
HAMMER = r"""
#include <pthread.h>
#include <stdint.h>
#include <stddef.h>
typedef int (*fwd_fn)(const void *, const void *, const int64_t *, float *, float *, int64_t, int32_t, int32_t, int64_t, int, void *, size_t, void *);
struct job { fwd_fn fn; void *p[7]; int64_t tokens; int64_t d, vocab; size_t bytes; int calls, status; };
static void *work(void *arg)
{
    struct job *j = arg;
    for (int i = 0; i < j->calls && j->status == 0; ++i)
        j->status = j->fn(j->p[0], j->p[1], j->p[2], j->p[3], j->p[4], j->tokens, j->d, j->vocab, -100, 0, j->p[5], j->bytes, j->p[6]);
    return 0;
}
int hammer(struct job *jobs, int n)
{
    pthread_t t[8];
    for (int i = 0; i < n; ++i) if (pthread_create(&t[i], 0, work, &jobs[i])) return -1;
    for (int i = 0; i < n; ++i) pthread_join(t[i], 0);
    return 0;
}
"""


class Job(ctypes.Structure):
    _fields_ = [("fn", ctypes.c_void_p), ("p", ctypes.c_void_p * 7), ("tokens", ctypes.c_int64), ("d", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("bytes", ctypes.c_size_t), ("calls", ctypes.c_int), ("status", ctypes.c_int)]


def test_host_threads_with_calls_of_different_size(tmp_path):
    """Host threads, each with its stream, tensors and workspace, whose calls take different amounts of shared memory of one kernel:
    none lowers the limit under another's launch.  Threads of C: those of Python take turns."""
    src, so = tmp_path / "hammer.c", tmp_path / "hammer.so"
    src.write_text(HAMMER)
    subprocess.run(["gcc", "-O2", "-shared", "-fPIC", "-pthread", "-o", str(so), str(src)], check=True)
    V, T = 40, 6
    jobs, keep = (Job * 4)(), []
    for j, d in zip(jobs, (1032, 4096, 1536, 3200)):
        x, W, y, _ = make(T, d, V, "f32", 0.0, seed=d)
        loss, lse = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
        ws = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, P.F32))
        stream = torch.cuda.Stream()
        j.fn = ctypes.cast(P.lib().monarch_xent_fwd, ctypes.c_void_p).value
        for i, p in enumerate((x.data_ptr(), W.data_ptr(), y.data_ptr(), loss.data_ptr(), lse.data_ptr(), ws.ptr, stream.cuda_stream)):
            j.p[i] = p
        j.tokens, j.d, j.vocab, j.bytes, j.calls = T, d, V, ws.nbytes, 20000
        keep.append((x, W, y, loss, lse, ws, stream))
    torch.cuda.synchronize()
    hammer = ctypes.CDLL(str(so)).hammer
    hammer.argtypes = [ctypes.POINTER(Job), ctypes.c_int]
    assert hammer(jobs, 4) == 0
    torch.cuda.synchronize()
    assert [j.status for j in jobs] == [0, 0, 0, 0]
    for x, W, y, loss, lse, _, _ in keep:
        e = exact(x, W, y)
        within(loss, e["loss"], e["loss_err"], "loss")


# ------------------------------------------------------------------------------------------------ the choice of kernels
@pytest.mark.parametrize("d,V,most,limit", [(4096, 600, 8, 3), (8192, 600, 4, 3), (1024, 600, 16, 2), (1024, 22000, 16, 3)])
def test_fp32_loss_of_few_tokens_reads_the_vocabulary_while_that_takes_less(d, V, most, limit):
    """Launches of few tokens (`most` at these sizes) read all of W each: beyond `limit` of them the tile kernels take less time."""
    def launches(T):
        x, W, y, _ = make(T, d, V, "f32", 0.0, seed=T)
        e = exact(x, W, y)
        before = P.monarch_launch_count()
        loss, _ = forward(x, W, y)
        count = P.monarch_launch_count() - before
        within(loss, e["loss"], e["loss_err"], "loss")
        return count

    tiles = launches(64)
    for n in range(1, min(6, 64 // most) + 1):
        assert launches(n * most) == (n if n <= limit else tiles), n
    assert launches(limit * most + 1) == tiles


# ------------------------------------------------------------------------------------------------ waits that run out
def after_a_time_out(ws, call, outputs, must=True):
    """The call under a limit of 1 us gives up instead of hanging and says so; the workspace, made anew, then serves the same call as before."""
    def run():
        for t in outputs:
            t.zero_()
        call()
        torch.cuda.synchronize()
        return [t.clone() for t in outputs]

    want = run()
    assert P.monarch_last_device_status(ws) == 0
    P.monarch_debug_set_wait_limit(ws, 1)
    t0 = time.perf_counter()
    run()
    assert time.perf_counter() - t0 < 5.0
    status = P.monarch_last_device_status(ws)
    assert status == 5 if must else status in (0, 5)       # MONARCH_ERR_TIMEOUT
    P.monarch_workspace_init(ws)
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
    assert P.monarch_last_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks,rows,cols", [(1, 300, 520), (3, 520, 300), (1, 1024, 1024)])
def test_waits_of_large_blocks_run_out(blocks, rows, cols, dtype):
    """Products wait for the ones before them, several microseconds each: every pair gives up at one place or another."""
    G = gradient(blocks, rows, cols, 60).to(DT[dtype][0])
    O = torch.empty_like(G)
    ws = P.Workspace(P.monarch_ortho_workspace_bytes(blocks, rows, cols, DT[dtype][1]))
    after_a_time_out(ws, lambda: P.monarch_orthogonalize(G, O, blocks, rows, cols, 5, ws), [O])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_short_waits_of_the_other_kernels(dtype):
    """Whether a wait on chip takes longer than a microsecond is up to the device: where one does, the call ends all the same."""
    G = gradient(4, 100, 120, 61).to(DT[dtype][0])
    O = torch.empty_like(G)
    ws = P.Workspace(P.monarch_ortho_workspace_bytes(4, 100, 120, DT[dtype][1]))
    after_a_time_out(ws, lambda: P.monarch_orthogonalize(G, O, 4, 100, 120, 5, ws), [O], must=False)
    T, d, V = 300, 512, 3000
    x, W, y, dloss = make(T, d, V, dtype, 0.1, seed=62)
    loss, lse, dx, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty(V, d, device="cuda")
    ws = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, DT[dtype][1]))
    after_a_time_out(ws, lambda: P.monarch_xent_fwd(x, W, y, loss, lse, T, d, V, IGNORE, ws), [loss, lse], must=False)
    given = lse.clone()
    ws = P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, DT[dtype][1]))
    after_a_time_out(ws, lambda: P.monarch_xent_bwd(x, W, y, given, dloss, dx, dW, 0, T, d, V, IGNORE, ws), [dx, dW], must=False)


# ------------------------------------------------------------------------------------------------ workspaces of other sizes
def least(refused, most):
    """The smallest workspace that a call is not refused for (tests/test_training_ends_workspaces.py: nothing is launched)."""
    low, high = 0, most
    while high - low > 1:
        mid = (low + high) // 2
        low, high = (mid, high) if refused(mid) else (low, mid)
    return high


class Guarded(P.Workspace):
    """A workspace of exactly n bytes with a band behind it that no call may touch."""

    def __init__(self, n):
        super().__init__(n + 65536)
        at = self.ptr - self.buf.data_ptr() + n
        self.nbytes, self.band = n, self.buf[at:at + 65536]
        self.band.fill_(0x5A)

    def untouched(self):
        return bool((self.band == 0x5A).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(300, 136, 5000), (129, 250, 3000), (2100, 64, 700), (200, 520, 257), (50, 1000, 20000)])
def test_loss_and_gradient_within_less_memory(T, d, V, dtype):
    """From the workspace that the query reports down to the least that is taken: pieces of the vocabulary, results within their bounds."""
    x, W, y, dloss = make(T, d, V, dtype, 0.1, seed=70)
    e = exact(x, W, y, dloss)
    code = DT[dtype][1]
    need = P.monarch_xent_workspace_bytes(T, d, V, code)
    p = [(i + 1) << 44 for i in range(8)]                  # never dereferenced: overlapping outputs are refused behind the workspace
    low = least(lambda n: P.lib().monarch_xent_fwd(p[0], p[1], p[2], p[3], p[3], T, d, V, IGNORE, code, p[4], n, None) == 3, need)
    for n in sorted({low, (low + need) // 2, max(low, need - 1), need, 2 * need}):
        ws = Guarded(n)
        loss, lse = forward(x, W, y, ws=ws)
        within(loss, e["loss"], e["loss_err"], "loss")
        within(lse, e["lse"], e["lse_err"], "lse")
        assert ws.untouched(), n
    need = P.monarch_xent_bwd_workspace_bytes(T, d, V, code)
    low = least(lambda n: P.lib().monarch_xent_bwd(*p[:5], p[5], p[5], 0, T, d, V, IGNORE, code, p[6], n, None) == 3, need)
    assert low < need or V != 5000
    for n in sorted({low, low + (need - low) // 8, (low + need) // 2, max(low, need - 1), need, 2 * need}):
        ws = Guarded(n)
        dx, dW = backward(x, W, y, e["lse"].float(), dloss, ws=ws)
        within(dx, e["dx"], e["dx_err"], "dx")
        within(dW, e["dW"], e["dW_err"], "dW")
        assert ws.untouched(), n
        again, dW2 = backward(x, W, y, e["lse"].float(), dloss, ws=ws)
        assert torch.equal(dx, again) and torch.equal(dW, dW2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks,rows,cols", [(2, 1030, 260), (1, 1024, 1024), (12, 63, 897), (1, 200, 3000)])
def test_update_within_less_memory(blocks, rows, cols, dtype):
    G = gradient(blocks, rows, cols, 71).to(DT[dtype][0])
    want = newton_schulz(G.double())
    need = P.monarch_ortho_workspace_bytes(blocks, rows, cols, DT[dtype][1])
    p = [1 << 44, 2 << 44]
    low = least(lambda n: P.lib().monarch_orthogonalize(p[0], p[0], blocks, rows, cols, 5, DT[dtype][1], p[1], n, None) == 3, need)
    assert low < need
    for n in (low, low + (need - low) // 3, need - 1, need, 2 * need):
        ws = Guarded(n)
        near(ortho(G, ws=ws), want, dtype, "O")
        assert ws.untouched(), n


# ------------------------------------------------------------------------------------------------ what is promised of the precision
@pytest.mark.parametrize("T", [9, 17, 40, 65, 100, 128])
def test_gradients_of_up_to_128_bf16_tokens_are_as_exact_as_their_types(T):
    """g in three parts in dW and two in dx (2^-24 and 2^-16 of a term).  The words share a component 16 times as large as what tells them
    apart: the sum of a token's g is zero, so in dx that component cancels, and what g loses does not."""
    d, V = 64, 5000
    g = gen(80 + T)
    W = ((torch.randn(1, d, generator=g, device="cuda") * 16 + torch.randn(V, d, generator=g, device="cuda")) / 64).bfloat16()
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    dloss = torch.rand(T, generator=g, device="cuda") + 0.1
    xd, Wd, w = x.double(), W.double(), dloss.double()[:, None]
    z = xd @ Wd.T
    lse = torch.logsumexp(z, 1).float()
    p = torch.exp(z - lse.double()[:, None])
    gr = w * (p - torch.zeros_like(p).scatter_(1, y[:, None], 1.0))
    dz = (xd.abs() @ Wd.abs().T) * acc(d)
    dg = w * p * (dz + 2.0 ** -20 * (1.0 + z.abs() / 16)) + gr.abs() * (2.0 ** -24 + 2.0 ** -23)
    dx, dW = backward(x, W, y, lse, dloss)
    want = gr.T @ xd
    within(dW, want, dg.T @ xd.abs() + (gr.abs().T @ xd.abs()) * acc(T, 3) + want.abs() * 2.0 ** -23, "dW")
    want = gr @ Wd
    err = (dg + gr.abs() * 2.0 ** -16) @ Wd.abs() + (gr.abs() @ Wd.abs()) * acc(V, 2)
    within(dx, want, err + want.abs() * 2.0 ** -8, "dx")
    # one part alone could be off by 2^-8 of every term: twenty times the bound
    assert float(((gr.abs() * 2.0 ** -8) @ Wd.abs()).mean()) > 20 * float((err + want.abs() * 2.0 ** -8).mean())


@pytest.mark.parametrize("T", [129, 300])
def test_masked_logits_and_tokens_that_are_not_numbers_among_many(T):
    """The fp16 parts of dW: words masked by the lowest value of the type have no part in anything, a token that is not a number keeps
    to itself in dx and makes dW NaN."""
    d, V = 64, 500
    x, W, y, dloss = make(T, d, V, "bf16", 0.0, seed=81 + T)
    y = y.clamp(min=200)
    x[:, 0] = 1.0
    W[:, 0] = 0.0
    live = exact(x, W[200:].contiguous(), y - 200, dloss)
    W[:200, 0] = torch.finfo(W.dtype).min
    loss, lse = forward(x, W, y)
    within(loss, live["loss"], live["loss_err"], "loss")
    within(lse, live["lse"], live["lse_err"], "lse")
    given = live["lse"].float()
    dx, dW = backward(x, W, y, given, dloss)
    within(dx[:, 1:], live["dx"][:, 1:], live["dx_err"][:, 1:], "dx")
    assert (dW[:200] == 0).all()
    within(dW[200:], live["dW"], live["dW_err"], "dW")
    rest = torch.arange(T, device="cuda") != 3
    for bad in (float("nan"), float("inf")):
        xb = x.clone()
        xb[3, 5] = bad
        loss, lse = forward(xb, W, y)
        assert torch.isnan(loss[3]) and torch.isnan(lse[3])
        within(loss[rest], live["loss"][rest], live["loss_err"][rest], "loss of the others")
        dx, dW = backward(xb, W, y, lse, dloss)
        assert torch.isnan(dx[3]).all() and torch.isnan(dW).all()
    w = dloss.clone()
    w[3] = float("nan")
    dx, dW = backward(x, W, y, given, w)
    assert torch.isnan(dx[3]).all() and torch.isnan(dW).all()
    within(dx[rest][:, 1:], live["dx"][rest][:, 1:], live["dx_err"][rest][:, 1:], "dx of the others")


@pytest.mark.parametrize("rows,cols", [(16, 16), (64, 64), (40, 60), (30, 200), (60, 200), (128, 128), (90, 128), (160, 200), (8, 600)])
def test_bf16_blocks_stand_alone(rows, cols):
    """Zeros give zeros; NaN and infinity stay in their block; norms beyond the range of fp32 squares, and tiny ones."""
    G = gradient(8, rows, cols, seed=82)
    G[1] = 0.0
    G[2, 3, 5] = float("nan")
    G[3, 0, 0] = float("inf")
    G[4] *= 1e30
    G[5] *= 1e-30
    G[6] *= 1e-6
    G = G.bfloat16()
    O = ortho(G)
    assert (O[1] == 0).all()
    assert torch.isnan(O[2]).all() and torch.isnan(O[3]).all()
    fine = [0, 4, 6, 7]
    near(O[fine], newton_schulz(G[fine].double()), "bf16", "O")
    near(O[5:6], newton_schulz(G[5:6].double()), "bf16", "O")


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
@pytest.mark.parametrize("blocks,rows,cols", [(3, 24, 40), (3, 60, 60), (2, 100, 120), (2, 8, 500), (2, 150, 140)])
def test_other_numbers_of_steps_in_bf16(blocks, rows, cols, steps):
    G = gradient(blocks, rows, cols, seed=83 + steps).bfloat16()
    near(ortho(G, steps), newton_schulz(G.double(), steps), "bf16", "O", steps)
