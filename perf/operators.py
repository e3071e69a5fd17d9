"""Timed cases of the two ends of a training step around Monarch layers: the loss over the vocabulary and the update.

A case is a dict of plain values.  ``kind`` names the operator, the other keys its sizes:

  xent_fwd  loss[t] = log sum_v exp(x[t] . W[v]) - x[t] . W[target[t]]   (training loss, scoring of a text)
  xent_bwd  dx, dW of sum_t dloss[t] loss[t] from the saved log sums       (the loss in a training step)
  ortho     O = orthogonalised G for each block of a stack, five quintic Newton-Schulz steps
  muon      momentum, orthogonalised update and weight decay of a stack of blocks, in place

Hidden states have unit variance (the output of a last normalisation); the rows of W are scaled for logits of standard
deviation 2.  ``ignored`` is the share of tokens that carry no loss (prompts, padding).  Gradients of weights are a few
strong directions and noise, as sums over the tokens of a batch are.
"""
import math

import torch

own = False

DTYPES = {"bf16": (torch.bfloat16, 2), "f32": (torch.float32, 4)}
IGNORE = -100
A, B, C, EPS = 3.4445, -4.7750, 2.0315, 1e-7      # the quintic's coefficients; kept away from a division by zero
STEPS = 5
LR, DECAY, BETA = 0.02, 0.1, 0.95


def listed():
    return [
        # Scoring one token against a whole vocabulary: the smallest call, bound by reading W once.
        {"name": "xent_fwd_bf16_t1", "kind": "xent_fwd", "dtype": "bf16", "tokens": 1, "d": 1024, "vocab": 50257, "ignored": 0.0},
        # The loss of a training batch of eight sequences of 1024 tokens, some of them padded.
        {"name": "xent_fwd_bf16_t8192", "kind": "xent_fwd", "dtype": "bf16", "tokens": 8192, "d": 1024, "vocab": 50257,
         "ignored": 0.1},
        # Single precision, a short text, a small vocabulary and no size that fits a tile.
        {"name": "xent_fwd_f32_t777", "kind": "xent_fwd", "dtype": "f32", "tokens": 777, "d": 1000, "vocab": 4999, "ignored": 0.0},
        # The loss in a fine-tuning step: a third of the tokens are prompts.
        {"name": "xent_bwd_bf16_t4096", "kind": "xent_bwd", "dtype": "bf16", "tokens": 4096, "d": 1024, "vocab": 50257,
         "ignored": 0.3},
        # The loss in a pre-training step of the widest hidden state: the largest case.
        {"name": "xent_bwd_bf16_t8192_d4096", "kind": "xent_bwd", "dtype": "bf16", "tokens": 8192, "d": 4096, "vocab": 32768,
         "ignored": 0.0},
        # A small single-precision model, rows of x and W that are not 16-byte multiples.
        {"name": "xent_bwd_f32_t511", "kind": "xent_bwd", "dtype": "f32", "tokens": 511, "d": 250, "vocab": 8191, "ignored": 0.1},
        # Both factors of the smallest layer (m = 16): the latency of a call.
        {"name": "ortho_f32_32x16", "kind": "ortho", "dtype": "f32", "blocks": 32, "rows": 16, "cols": 16},
        # Four large blocks, as the paper's language and vision models use them.
        {"name": "ortho_bf16_4x1024", "kind": "ortho", "dtype": "bf16", "blocks": 4, "rows": 1024, "cols": 1024},
        # Blocks of a rectangular layer, no power of two.
        {"name": "ortho_f32_96x33x80", "kind": "ortho", "dtype": "f32", "blocks": 96, "rows": 33, "cols": 80},
        # The update of both factors of an ordinary layer (m = 64) held as one tensor.
        {"name": "muon_bf16_128x64", "kind": "muon", "dtype": "bf16", "blocks": 128, "rows": 64, "cols": 64},
        # The update of one factor of the widest layer (m = 128).
        {"name": "muon_bf16_128x128", "kind": "muon", "dtype": "bf16", "blocks": 128, "rows": 128, "cols": 128},
        # A dense weight in the dense phase of training, before it is projected.
        {"name": "muon_f32_1024x4096", "kind": "muon", "dtype": "f32", "blocks": 1, "rows": 1024, "cols": 4096},
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["xent_fwd", "xent_bwd", "ortho", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("xent"):
        d = log_int(rng, 16, 4096)
        d = d if rng.random() < 0.3 else 8 * (-(-d // 8))
        vocab = log_int(rng, 64, 131072)
        # products of one pass: at most those of the largest listed case, an eighth in fp32; logits of the plain form: 2 GB
        most = (1 << 40) if dtype == "bf16" else (1 << 37)
        tokens = log_int(rng, 1, max(1, min(16384, (1 << 29) // vocab, most // (vocab * d))))
        return {"kind": kind, "dtype": dtype, "tokens": tokens, "d": d, "vocab": vocab,
                "ignored": rng.choice([0.0, 0.0, 0.1, 0.5, 0.9])}
    family = rng.choice(["square", "slices", "rect", "large"])
    if family == "square":                       # both factors of a layer, n = m * m
        m = rng.choice([16, 32, 64, 128])
        rows = cols = m
        blocks = m * rng.choice([1, 2, 4])
    elif family == "slices":                     # a factor of the general class
        rows, cols = log_int(rng, 2, 256), log_int(rng, 2, 256)
        blocks = log_int(rng, 1, max(1, min(4096, (1 << 22) // (rows * cols))))
    elif family == "rect":                       # few large blocks
        rows, cols = 8 * log_int(rng, 16, 128), 8 * log_int(rng, 16, 128)
        blocks = rng.choice([1, 2, 4, 8])
    else:                                        # one dense weight
        rows, cols = log_int(rng, 256, 4096), log_int(rng, 256, 4096)
        blocks = 1
    return {"kind": kind, "dtype": dtype, "blocks": blocks, "rows": rows, "cols": cols}


def _gradient(gen, blocks, rows, cols, scale):
    k = max(1, min(rows, cols) // 4)
    strong = torch.matmul(torch.randn(blocks, rows, k, generator=gen, device="cuda"),
                          torch.randn(blocks, k, cols, generator=gen, device="cuda")) / math.sqrt(k)
    return scale * (strong + 0.1 * torch.randn(blocks, rows, cols, generator=gen, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]][0]
    s = {"kind": case["kind"], "ws": None}
    if case["kind"].startswith("xent"):
        T, d, V = case["tokens"], case["d"], case["vocab"]
        s["x"] = torch.randn(T, d, generator=gen, device="cuda").to(dt)
        s["W"] = (torch.randn(V, d, generator=gen, device="cuda") * (2.0 / math.sqrt(d))).to(dt)
        targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
        left_out = torch.rand(T, generator=gen, device="cuda") < case["ignored"]
        s["targets"] = torch.where(left_out, IGNORE, targets)
        s["lse"] = torch.empty(T, device="cuda")
        if case["kind"] == "xent_fwd":
            s["loss"] = torch.empty(T, device="cuda")
        else:
            # what the forward pass saved, and the weights of a mean over the tokens that count
            piece = max(1, (1 << 27) // V)
            torch.cat([torch.logsumexp(torch.matmul(s["x"][t:t + piece].float(), s["W"].float().T).double(), 1)
                       for t in range(0, T, piece)], out=(lse := torch.empty(T, device="cuda", dtype=torch.float64)))
            s["lse"] = torch.where(left_out, 0.0, lse).float()
            s["dloss"] = (0.5 + torch.rand(T, generator=gen, device="cuda")) / max(1, T - int(case["ignored"] * T))
            s["dx"] = torch.empty_like(s["x"])
            s["dW"] = torch.empty(V, d, device="cuda")
        return s
    blocks, rows, cols = case["blocks"], case["rows"], case["cols"]
    if case["kind"] == "ortho":
        s["G"] = _gradient(gen, blocks, rows, cols, 1e-2).to(dt)
        s["O"] = torch.empty_like(s["G"])
    else:
        s["W"] = (torch.randn(blocks, rows, cols, generator=gen, device="cuda") / math.sqrt(cols)).to(dt)
        s["dW"] = _gradient(gen, blocks, rows, cols, 1e-2)
        s["V"] = _gradient(gen, blocks, rows, cols, 1e-1)
    return s


def _scale(rows, cols):
    return math.sqrt(max(1.0, rows / cols))


def _plain_xent(s):
    x, W, keep = s["x"].float(), s["W"].float(), s["targets"] != IGNORE
    at = torch.where(keep, s["targets"], 0)[:, None]
    logits = torch.matmul(x, W.T)
    if s["kind"] == "xent_fwd":
        top = logits.amax(1, keepdim=True)
        lse = torch.log(torch.exp(logits - top).sum(1)) + top[:, 0]
        return torch.where(keep, lse - logits.gather(1, at)[:, 0], 0.0), torch.where(keep, lse, 0.0)
    g = torch.exp(logits - s["lse"][:, None])
    g.scatter_add_(1, at, torch.full_like(s["lse"], -1.0)[:, None])
    g.mul_(torch.where(keep, s["dloss"], 0.0)[:, None])
    return torch.matmul(g, W).to(s["x"].dtype), torch.matmul(g.T, x)


def _plain_newton_schulz(u):
    x = u / (torch.sqrt(torch.square(u).sum((1, 2), keepdim=True)) + EPS)
    wide = x.shape[1] <= x.shape[2]
    for _ in range(STEPS):
        g = torch.matmul(x, x.mT) if wide else torch.matmul(x.mT, x)
        p = B * g + C * torch.matmul(g, g)
        x = A * x + (torch.matmul(p, x) if wide else torch.matmul(x, p))
    return x


def run(s):
    if own:
        return _run_own(s)
    if s["kind"].startswith("xent"):
        return _plain_xent(s)
    if s["kind"] == "ortho":
        return _plain_newton_schulz(s["G"].float()).to(s["G"].dtype)
    rows, cols = s["W"].shape[1:]
    s["V"].mul_(BETA).add_(s["dW"])
    o = _plain_newton_schulz(s["dW"] + BETA * s["V"])
    s["W"].copy_((1.0 - LR * DECAY) * s["W"].float() - LR * _scale(rows, cols) * o)
    return s["W"], s["V"]


def _run_own(s):
    import paper_2204_00595_b200 as P
    if s["kind"].startswith("xent"):
        (T, d), V = s["x"].shape, s["W"].shape[0]
        if s["kind"] == "xent_fwd":
            if s["ws"] is None:
                s["ws"] = P.Workspace(P.monarch_xent_workspace_bytes(T, d, V, P.F32 if s["x"].dtype == torch.float32 else P.BF16))
            P.monarch_xent_fwd(s["x"], s["W"], s["targets"], s["loss"], s["lse"], T, d, V, IGNORE, s["ws"])
            return s["loss"], s["lse"]
        if s["ws"] is None:
            s["ws"] = P.Workspace(P.monarch_xent_bwd_workspace_bytes(T, d, V, P.F32 if s["x"].dtype == torch.float32 else P.BF16))
        P.monarch_xent_bwd(s["x"], s["W"], s["targets"], s["lse"], s["dloss"], s["dx"], s["dW"], 0, T, d, V, IGNORE, s["ws"])
        return s["dx"], s["dW"]
    blocks, rows, cols = (s["G"] if s["kind"] == "ortho" else s["W"]).shape
    if s["ws"] is None:
        dt = (s["G"] if s["kind"] == "ortho" else s["W"]).dtype
        s["ws"] = P.Workspace(P.monarch_ortho_workspace_bytes(blocks, rows, cols, P.F32 if dt == torch.float32 else P.BF16))
    if s["kind"] == "ortho":
        P.monarch_orthogonalize(s["G"], s["O"], blocks, rows, cols, STEPS, s["ws"])
        return s["O"]
    P.monarch_muon_step(s["W"], s["dW"], s["V"], blocks, rows, cols, LR, DECAY, BETA, 1, _scale(rows, cols), STEPS, s["ws"])
    return s["W"], s["V"]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("xent"):
        T, V = case["tokens"], case["vocab"]
        W, labels = s["W"].double(), s["targets"]
        piece = max(1, (1 << 27) // V)
        loss, lses, dxs = [], [], []
        dW = None if case["kind"] == "xent_fwd" else torch.zeros_like(W)
        for t in range(0, T, piece):
            x, y = s["x"][t:t + piece].double(), labels[t:t + piece]
            z = x @ W.T
            counts = y.ne(IGNORE)
            rows = torch.nonzero(counts)[:, 0]
            if dW is None:
                lse = torch.logsumexp(z, 1)
                lses.append(lse.masked_fill(~counts, 0.0))
                picked = torch.zeros_like(lse)
                picked[rows] = lse[rows] - z[rows, y[rows]]
                loss.append(picked)
                continue
            p = torch.exp(z - s["lse"][t:t + piece].double()[:, None])
            p[rows, y[rows]] -= 1.0
            p *= (s["dloss"][t:t + piece].double() * counts)[:, None]
            dxs.append(p @ W)
            dW += p.T @ x
        return (torch.cat(loss), torch.cat(lses)) if dW is None else (torch.cat(dxs), dW)
    blocks, rows, cols = case["blocks"], case["rows"], case["cols"]
    if case["kind"] == "ortho":
        u = s["G"].double()
    else:
        v = BETA * s["V"].double() + s["dW"].double()
        u = s["dW"].double() + BETA * v
    # the polynomial on the smaller side's Gram matrix, from the definition: X <- X (a + b X'X + c (X'X)^2)
    tall = u if rows >= cols else u.transpose(1, 2)
    x = tall / (torch.linalg.vector_norm(tall, dim=(1, 2), keepdim=True) + EPS)
    eye = torch.eye(x.shape[2], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        g = x.transpose(1, 2) @ x
        x = x @ (A * eye + B * g + C * (g @ g))
    o = x if rows >= cols else x.transpose(1, 2)
    if case["kind"] == "ortho":
        return o.contiguous()
    return s["W"].double() * (1.0 - LR * DECAY) - LR * _scale(rows, cols) * o, v


def work(case):
    es = DTYPES[case["dtype"]][1]
    if case["kind"].startswith("xent"):
        T, d, V = case["tokens"], case["d"], case["vocab"]
        counts = T * (1.0 - case["ignored"])
        read = counts * d * es + V * d * es + 8 * T
        if case["kind"] == "xent_fwd":
            return {"bytes": read + 8 * T, "flops": 2.0 * counts * V * d}
        # the logits again, then dx and dW
        return {"bytes": read + 8 * T + T * d * es + 4.0 * V * d, "flops": 6.0 * counts * V * d}
    blocks, rows, cols = case["blocks"], case["rows"], case["cols"]
    k, n = min(rows, cols), max(rows, cols)
    size = blocks * rows * cols
    # a Gram matrix and its square are symmetric: half of each product is enough
    flops = blocks * STEPS * (k * k * n + k ** 3 + 2.0 * k * k * n)
    return {"bytes": size * (2 * es if case["kind"] == "ortho" else 2 * es + 12), "flops": flops}
