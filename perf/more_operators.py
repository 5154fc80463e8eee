"""The operators between a model's last block and its optimizer step, as cases that can be timed and compared: dropout onto
the residual stream, layer norm with its gradient, and the head's token log-probabilities and cross entropy without logits.

One pass is one operator as a training or serving program calls it.  `op` names it:

  dropout     dropout whose mask comes from a counter-based generator, with the residual that it is added to or without one
              (the backward pass) (gs_dropout)
  norm        layer norm of rows (gs_layer_norm)
  norm_grad   its gradient in the rows, the scale and the shift (gs_layer_norm_grad)
  score       log-probability of one given token per hidden state under the head's weights (gs_head_logp)
  loss        cross entropy of the head with its gradient in the hidden states, the weights and the bias (gs_head_cross_entropy)

Rows of hidden states are the tokens of `seqs` sequences of different lengths, one after another.  `prompt`: the first
quarter of each sequence is a prompt, whose rows have no target and take no part.  Where `own` is false, `run` computes the
same in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
_MOST_LOGITS = 1 << 30             # rows x vocabulary of the largest case
_MOST_WEIGHTS = 1 << 29            # vocabulary x hidden
_MOST_VALUES = 1 << 27             # rows x columns of the largest case of dropout and norm


def listed():
    return [
        # one short sequence's activations on their way back
        dict(name="dropout_257x1024", op="dropout", rows=257, cols=1024, dtype="bf16", residual=False, p=0.1, offset=0),
        # activations in 32 bits, an odd width, one part of a tensor that others hold the rest of
        dict(name="dropout_4095x5003_f32", op="dropout", rows=4095, cols=5003, dtype="f32", residual=True, p=0.2, offset=20_487_293),
        # eight sequences of 2048 tokens in the widest layer's stream
        dict(name="dropout_16384x8192", op="dropout", rows=16384, cols=8192, dtype="bf16", residual=True, p=0.1, offset=0),
        # serving: the one token of a decoding step
        dict(name="norm_1x8192", op="norm", rows=1, cols=8192, dtype="bf16", weights="bf16"),
        # eight sequences of 2048 tokens
        dict(name="norm_16384x8192", op="norm", rows=16384, cols=8192, dtype="bf16", weights="bf16"),
        # a small model's short batch, everything in 32 bits, odd width
        dict(name="norm_grad_1023x1001_f32", op="norm_grad", rows=1023, cols=1001, dtype="f32", weights="f32"),
        # eight sequences of 2048 tokens
        dict(name="norm_grad_16384x8192", op="norm_grad", rows=16384, cols=8192, dtype="bf16", weights="bf16"),
        # serving: the log-probability of the one token that was drawn, a large vocabulary
        dict(name="score_1x4096x131072", op="score", rows=1, hidden=4096, vocab=131072, bias=False, seqs=1, prompt=False, temperature=0.7),
        # scoring long prompts with a frozen model
        dict(name="score_8192x2048x50304", op="score", rows=8192, hidden=2048, vocab=50304, bias=False, seqs=8, prompt=False, temperature=1.0),
        # a small step: a few short completions
        dict(name="loss_64x4096x32000", op="loss", rows=64, hidden=4096, vocab=32000, bias=False, seqs=4, prompt=False, temperature=1.0),
        # an ordinary micro-batch with prompts in it, odd vocabulary, with a bias
        dict(name="loss_4095x2048x50001", op="loss", rows=4095, hidden=2048, vocab=50001, bias=True, seqs=13, prompt=True, temperature=1.0),
        # the largest: long sequences, a large vocabulary
        dict(name="loss_8192x4096x131072", op="loss", rows=8192, hidden=4096, vocab=131072, bias=False, seqs=4, prompt=False, temperature=1.0),
    ]


def draw(rng):
    def span(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["dropout", "norm", "norm_grad", "score", "loss", "loss"])
    if op in ("dropout", "norm", "norm_grad"):
        cols = span(256, 16384)
        if rng.random() < 0.6:
            cols = cols // 64 * 64                              # most widths are whole tiles
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = span(1, min(65536, _MOST_VALUES // cols // (2 if dtype == "f32" else 1)))
        if op == "dropout":
            return dict(op=op, rows=rows, cols=cols, dtype=dtype, residual=rng.random() < 0.5, p=rng.choice([0.05, 0.1, 0.2, 0.5]),
                        offset=rng.choice([0, 0, rng.randrange(1 << 34)]))
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, weights=dtype if rng.random() < 0.7 else "f32")
    hidden = span(256, 8192)
    if rng.random() < 0.8:
        hidden = hidden // 64 * 64                              # most widths are whole tiles
    vocab = min(span(1000, 160_000), _MOST_WEIGHTS // hidden)
    if rng.random() < 0.5:
        vocab = vocab // 128 * 128                              # half of the vocabularies are padded to whole tiles
    rows = min(span(1, 16384), _MOST_LOGITS // vocab, (1 << 42) // (hidden * vocab))
    return dict(op=op, rows=rows, hidden=hidden, vocab=vocab, bias=rng.random() < 0.3, seqs=max(1, min(rng.randint(1, 16), rows // 2)),
                prompt=rng.random() < 0.5 and rows >= 8, temperature=rng.choice([1.0, 1.0, 0.7]))


# ---- what a program has in hand ------------------------------------------------------------------------------------

def _ends(case):
    """First row of each sequence, and the number of rows: uneven lengths."""
    rows, seqs = case["rows"], case["seqs"]
    parts = [2 + (5 * i) % 7 for i in range(seqs)]
    at, out = 0, [0]
    for p in parts:
        at += p
        out.append(rows * at // sum(parts))
    return out


def _prompts(case):
    """[(first, end)] of the rows without a target."""
    ends = _ends(case)
    return [(a, a + (b - a) // 4) for a, b in zip(ends, ends[1:])] if case["prompt"] else []


def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + what * 7919 + 29) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(seed, what, *shape):
    return torch.randn(*shape, generator=_gen(seed, what), device=DEV, dtype=torch.float32)


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "dropout":
        shape, dt = (case["rows"], case["cols"]), DTYPES[case["dtype"]]
        s["x"] = _randn(seed, 1, *shape).to(dt)
        s["residual"] = _randn(seed, 2, *shape).mul_(2.0).to(dt) if case["residual"] else None
        s["out"] = torch.empty_like(s["x"])
        s["seed"] = (int(seed) * 0x9E3779B97F4A7C15 + 0x1234567) & 0x7FFFFFFFFFFFFFFF
        s["step"] = torch.tensor([int(seed) % 1000 + 5], dtype=torch.int64, device=DEV)      # of training
        return s
    if case["op"] in ("norm", "norm_grad"):
        rows, cols, dt, wt = case["rows"], case["cols"], DTYPES[case["dtype"]], DTYPES[case["weights"]]
        # a residual stream: columns with a mean of their own, a few of them large, rows of different size
        size = torch.where(torch.rand(cols, generator=_gen(seed, 3), device=DEV) < 0.01, 12.0, 1.0)
        x = _randn(seed, 4, rows, cols).add_(_randn(seed, 5, cols).mul_(0.4)).mul_(size).mul_(_randn(seed, 6, rows, 1).mul_(0.3).exp_())
        s["x"] = x.to(dt)
        s["gamma"] = _randn(seed, 7, cols).mul_(0.2).add_(1.0).to(wt)
        s["beta"] = _randn(seed, 8, cols).mul_(0.1).to(wt)
        s["stats"] = torch.empty(rows, 2, dtype=torch.float32, device=DEV)
        if case["op"] == "norm":
            s["y"] = torch.empty_like(s["x"])
            return s
        del x
        s["dy"] = _randn(seed, 9, rows, cols).mul_(1e-3).to(dt)
        # of the forward pass
        wide = s["x"].double()
        mean = wide.mean(1)
        s["stats"][:, 0] = mean
        s["stats"][:, 1] = wide.sub_(mean[:, None]).square_().mean(1).add_(EPS).rsqrt_()
        del wide
        s.update(dx=torch.empty_like(s["x"]), dgamma=torch.empty_like(s["gamma"]), dbeta=torch.empty_like(s["beta"]))
        return s
    rows, hidden, vocab = case["rows"], case["hidden"], case["vocab"]
    bf16 = torch.bfloat16
    w = _randn(seed, 10, vocab, hidden).mul_(2.5 * hidden ** -0.5).to(bf16)
    target = torch.randint(0, vocab, (rows,), generator=_gen(seed, 11), device=DEV)
    # a trained model's rows: most targets stand out, some do not
    lift = torch.where(torch.rand(rows, generator=_gen(seed, 12), device=DEV) < 0.7, 9.0 / 6.25, 0.0)
    x = _randn(seed, 13, rows, hidden).add_(w[target].float().mul_(lift[:, None])).to(bf16)
    live = torch.ones(rows, dtype=torch.bool, device=DEV)
    for a, b in _prompts(case):
        live[a:b] = False
    target[~live] = -1
    s.update(x=x, w=w, target=target, logp=torch.zeros(rows, dtype=torch.float32, device=DEV),
             bias=_randn(seed, 14, vocab).to(bf16) if case["bias"] else None)
    if case["op"] == "loss":
        s["weights"] = live.float() / live.sum()
        s.update(dx=torch.empty_like(x), dw=torch.empty_like(w), dbias=torch.empty_like(s["bias"]) if case["bias"] else None,
                 loss=torch.zeros(1, dtype=torch.float32, device=DEV))
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------

_M32 = 0xFFFFFFFF


def _plain_words(block, step, seed):
    """Philox4x32-10 of the counters (block, step) under the key `seed`, in 64-bit whole numbers: four words each."""
    c0, c1 = block & _M32, block >> 32
    c2, c3 = (step & _M32).expand_as(block), (step >> 32).expand_as(block)
    k0, k1 = seed & _M32, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57               # wraps, with the right 64 bits
        c0, c1, c2, c3 = ((b >> 32) & _M32) ^ c1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ c3 ^ k1, a & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return torch.stack([c0, c1, c2, c3], dim=1)


def _plain_dropout(s):
    case = s["case"]
    n, first = case["rows"] * case["cols"], case["offset"]
    words = _plain_words(torch.arange(first // 8, (first + n + 7) // 8, device=DEV), s["step"], s["seed"])
    drawn = torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)[first % 8:first % 8 + n].reshape(case["rows"], case["cols"])
    least = round(case["p"] * 65536)
    out = torch.where(drawn >= least, s["x"].float() * (65536.0 / (65536 - least)), 0.0)
    if case["residual"]:
        out = out + s["residual"].float()
    return {"out": out.to(s["x"].dtype)}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1.0 / ((x * x).mean(1, keepdim=True) + EPS).sqrt()
    y = x * rstd * s["gamma"].float() + s["beta"].float()
    return {"y": y.to(s["x"].dtype), "stats": torch.cat([mean, rstd], dim=1)}


def _plain_norm_grad(s):
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    dy, xhat = s["dy"].float(), (s["x"].float() - mean) * rstd
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    dt, wt = s["x"].dtype, s["gamma"].dtype
    return {"dx": dx.to(dt), "dgamma": (dy * xhat).sum(0).to(wt), "dbeta": dy.sum(0).to(wt)}


def _plain_head(s):
    case, it, target = s["case"], 1.0 / s["case"]["temperature"], s["target"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if case["bias"]:
        z = z + s["bias"].float()
    z = (z - z.amax(1, keepdim=True)) * it
    live, at = target >= 0, target.clamp(min=0)[:, None]
    picked = z.gather(1, at)[:, 0]
    e = z.exp_()
    total = e.sum(1, keepdim=True)
    logp = torch.where(live, picked - total[:, 0].log(), 0.0)
    if case["op"] == "score":
        return {"logp": logp}
    weights = torch.where(live, s["weights"], 0.0)
    dz = e.mul_((it * weights)[:, None] / total)
    dz.scatter_add_(1, at, (-it * weights)[:, None])
    out = {"loss": -(weights * logp).sum().reshape(1), "logp": logp, "dx": (dz @ w).to(s["x"].dtype), "dw": (dz.t() @ x).to(s["w"].dtype)}
    if case["bias"]:
        out["dbias"] = dz.sum(0).to(s["w"].dtype)
    return out


_PLAIN = {"dropout": _plain_dropout, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "score": _plain_head, "loss": _plain_head}


# ---- the framework's operators -------------------------------------------------------------------------------------

def _workspace(s, size):
    """A program asks for the size once and keeps the memory."""
    if "ws" not in s:
        s["ws"] = torch.empty(size(), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own(s):
    from paper_2512_17570_amd import gs

    case = s["case"]
    if case["op"] == "dropout":
        gs.gs_dropout(s["x"], s["residual"], s["out"], case["p"], s["seed"], case["offset"], d_step=s["step"])
        return {"out": s["out"]}
    if case["op"] == "norm":
        gs.gs_layer_norm(s["x"], s["gamma"], s["beta"], s["y"], s["stats"], eps=EPS)
        return {"y": s["y"], "stats": s["stats"]}
    if case["op"] == "norm_grad":
        ws = _workspace(s, lambda: gs.gs_layer_norm_workspace_bytes(case["rows"], case["cols"]))
        gs.gs_layer_norm_grad(s["dy"], s["x"], s["gamma"], s["stats"], s["dx"], s["dgamma"], s["dbeta"], ws)
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    grad = case["op"] == "loss"
    ws = _workspace(s, lambda: gs.gs_head_workspace_bytes(case["rows"], case["hidden"], case["vocab"], gradient=grad))
    if not grad:
        gs.gs_head_logp(s["x"], s["w"], s["bias"], s["target"], s["logp"], temperature=case["temperature"], d_workspace=ws)
        return {"logp": s["logp"]}
    gs.gs_head_cross_entropy(s["x"], s["w"], s["bias"], s["target"], s["weights"], s["logp"], s["dx"], s["dw"], s["dbias"], s["loss"], ws,
                             temperature=case["temperature"])
    out = {"loss": s["loss"], "logp": s["logp"], "dx": s["dx"], "dw": s["dw"]}
    return out | ({"dbias": s["dbias"]} if case["bias"] else {})


def run(s):
    return _own(s) if own else _PLAIN[s["case"]["op"]](s)


def work(case):
    """Inputs once, outputs once; rows without a target need no product, and their gradients are zeros that are written."""
    if "cols" in case:
        rows, cols, size = case["rows"], case["cols"], 2 if case["dtype"] == "bf16" else 4
        n = rows * cols
        if case["op"] == "dropout":
            return {"bytes": (3 if case["residual"] else 2) * n * size, "flops": 2 * n}
        vectors = cols * (2 if case["weights"] == "bf16" else 4)
        if case["op"] == "norm":
            return {"bytes": 2 * n * size + 2 * vectors + 8 * rows, "flops": 7 * n}
        return {"bytes": 3 * n * size + 3 * vectors + 8 * rows, "flops": 13 * n}
    rows, hidden, vocab = case["rows"], case["hidden"], case["vocab"]
    live = rows - sum(b - a for a, b in _prompts(case))
    weights = 2 * vocab * (hidden + (1 if case["bias"] else 0))
    if case["op"] == "score":
        return {"bytes": weights + 2 * live * hidden + 12 * rows, "flops": 2 * live * vocab * hidden}
    return {"bytes": 2 * weights + 2 * (live + rows) * hidden + 16 * rows, "flops": 6 * live * vocab * hidden}


# ---- 64 bits -------------------------------------------------------------------------------------------------------

def _exact_kept(case, seed, step):
    """Which elements stay, from the published generator in numpy's unsigned whole numbers."""
    n, first, u = case["rows"] * case["cols"], case["offset"], np.uint64
    kept, mask = np.empty(n, dtype=bool), u(_M32)
    least = round(case["p"] * 65536)
    for a in range(0, n, 1 << 23):
        b = min(n, a + (1 << 23))
        blocks = np.arange((first + a) // 8, (first + b + 7) // 8, dtype=u)
        x = [blocks & mask, blocks >> u(32), np.full_like(blocks, step & _M32), np.full_like(blocks, step >> 32)]
        for r in range(10):
            key = ((seed & _M32) + r * 0x9E3779B9) & _M32, ((seed >> 32) + r * 0xBB67AE85) & _M32
            left, right = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
            x = [(right >> u(32)) ^ x[1] ^ u(key[0]), right & mask, (left >> u(32)) ^ x[3] ^ u(key[1]), left & mask]
        halves = np.stack(x, axis=1).astype(np.uint32).view(np.uint16).reshape(-1)
        skip = (first + a) % 8
        kept[a:b] = halves[skip:skip + b - a] >= least
    return torch.from_numpy(kept).to(DEV).reshape(case["rows"], case["cols"])


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "dropout":
        least = round(case["p"] * 65536)
        out = s["x"].to(f64) / (1.0 - least / 65536.0) * _exact_kept(case, s["seed"], int(s["step"]))
        return {"out": out if s["residual"] is None else out + s["residual"].to(f64)}
    if case["op"] in ("norm", "norm_grad"):
        x, gamma = s["x"].to(f64), s["gamma"].to(f64)
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).rsqrt()
        hat = (x - mean[:, None]) * rstd[:, None]
        if case["op"] == "norm":
            return {"y": torch.addcmul(s["beta"].to(f64), hat, gamma), "stats": torch.stack([mean, rstd], dim=1)}
        del x
        dy = s["dy"].to(f64)
        out = {"dgamma": torch.einsum("rc,rc->c", dy, hat), "dbeta": dy.sum(0)}
        g = dy * gamma
        out["dx"] = (g - (g.sum(1) / case["cols"])[:, None] - hat * (torch.einsum("rc,rc->r", g, hat) / case["cols"])[:, None]) * rstd[:, None]
        return out
    rows, vocab, temp = case["rows"], case["vocab"], case["temperature"]
    w = s["w"].to(f64)
    live, at = s["target"] >= 0, s["target"].clamp(min=0)[:, None]
    logp, dx = torch.zeros(rows, dtype=f64, device=DEV), torch.zeros(rows, case["hidden"], dtype=f64, device=DEV)
    grad = case["op"] == "loss"
    dw = torch.zeros_like(w) if grad else None
    db = torch.zeros(vocab, dtype=f64, device=DEV)
    step = max(1, (1 << 28) // vocab)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        x = s["x"][a:b].to(f64)
        z = x @ w.t()
        ls = torch.log_softmax((z if s["bias"] is None else z + s["bias"].to(f64)) / temp, dim=1)
        logp[a:b] = torch.where(live[a:b], ls.gather(1, at[a:b])[:, 0], 0.0)
        if grad:
            d = ls.exp_()
            d.scatter_add_(1, at[a:b], torch.full((b - a, 1), -1.0, dtype=f64, device=DEV))
            d.mul_((torch.where(live[a:b], s["weights"][a:b].to(f64), 0.0) / temp)[:, None])
            dx[a:b] = d @ w
            dw.addmm_(d.t(), x)
            db += d.sum(0)
    if not grad:
        return {"logp": logp}
    out = {"loss": -(logp * s["weights"].to(f64))[live].sum().reshape(1), "logp": logp, "dx": dx, "dw": dw}
    return out | ({"dbias": db} if case["bias"] else {})
