"""The loss, norm and clip operators that a post-training program uses around the optimizer step, as cases that can be
timed and compared.

One pass is one operator as such a program calls it.  `op` names it:

  logp        log-probability of one given token per row of logits (gs_token_logp): scoring a prompt, or the one
              token that was just drawn
  policy      clipped policy loss with a KL term over rows of logits, with its gradient in the logits (gs_policy_loss)
  preference  preference loss over pairs of sequences: token log-probabilities, the loss of the paired log ratios, and
              the gradient in the logits (gs_token_logp, gs_preference_loss, gs_token_logp_grad)
  clip        global norm over the gradients of many tensors, and the gradients scaled to it (gs_grads_sqnorm,
              gs_grads_clip), into buffers of their own

Rows of logits are the tokens of `seqs` sequences of different lengths, one after another.  `prompt`: the first quarter
of each sequence is a prompt, whose rows have no target and take no part.  Where `own` is false, `run` computes the
same in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_MOST = 1 << 30                    # logits of the largest case
_WORKSPACE = 4 << 20               # bytes of device workspace that the program brings


def listed():
    return [
        # serving: the log-probability of the one token that was drawn, a large vocabulary
        dict(name="logp_1x131072", op="logp", rows=1, vocab=131072, dtype="bf16", seqs=1, prompt=False, temperature=0.7),
        # scoring long prompts with a frozen model, for the old or the reference log-probabilities
        dict(name="logp_16384x32000", op="logp", rows=16384, vocab=32000, dtype="bf16", seqs=8, prompt=False, temperature=1.0),
        # a small step: a few short completions
        dict(name="policy_64x32000", op="policy", rows=64, vocab=32000, dtype="bf16", seqs=4, prompt=False, temperature=1.0),
        # an ordinary micro-batch with prompts in it, odd vocabulary: rows start on any element
        dict(name="policy_4095x50001", op="policy", rows=4095, vocab=50001, dtype="bf16", seqs=13, prompt=True, temperature=1.0),
        # logits kept in 32 bits
        dict(name="policy_2048x32003_f32", op="policy", rows=2048, vocab=32003, dtype="f32", seqs=8, prompt=False, temperature=0.7),
        # the largest: long completions under a large vocabulary
        dict(name="policy_8192x131072", op="policy", rows=8192, vocab=131072, dtype="bf16", seqs=4, prompt=False, temperature=1.0),
        # two short pairs
        dict(name="preference_301x32000", op="preference", rows=301, vocab=32000, dtype="bf16", seqs=4, prompt=True, temperature=1.0),
        # pairs of uneven length with prompts, odd vocabulary, logits in 32 bits
        dict(name="preference_3001x50001_f32", op="preference", rows=3001, vocab=50001, dtype="f32", seqs=10, prompt=True, temperature=1.0),
        # sixteen long pairs
        dict(name="preference_16000x65536", op="preference", rows=16000, vocab=65536, dtype="bf16", seqs=32, prompt=True, temperature=1.0),
        # only the vectors of a model (biases, LayerNorm) as the gradients of an adapter-sized program
        dict(name="clip_vectors_h2048", op="clip", h=2048, layers=6, dtype="bf16", vectors=True),
        # four small layers: matrices in bf16, vectors in 32 bits, 48 tensors
        dict(name="clip_4layers_h2048_mixed", op="clip", h=2048, layers=4, dtype="mixed", vectors=False),
        # one GPT-65B-shaped layer's full-precision gradients
        dict(name="clip_layer_h8192_f32", op="clip", h=8192, layers=1, dtype="f32", vectors=False),
    ]


def draw(rng):
    def span(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["logp", "policy", "policy", "preference", "clip", "clip"])
    if op == "clip":
        dtype = rng.choice(["bf16", "f32", "mixed"])
        vectors = rng.random() < 0.25
        h = span(100, 6500)
        if h in (768, 1024, 3072):
            h += 1
        most = 700_000_000 if dtype == "f32" else 1_000_000_000
        layers = rng.randint(1, 12)
        if not vectors:
            layers = max(1, min(layers, most // (12 * h * h + 13 * h)))
        return dict(op=op, h=h, layers=layers, dtype=dtype, vectors=vectors)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    vocab = span(2000, 160_000)
    if rng.random() < 0.5:
        vocab = vocab // 128 * 128 + 128                      # half of the vocabularies are padded to whole tiles
    most = (_MOST if dtype == "bf16" else _MOST // 2) // vocab
    rows = min(span(1, 16384) if op == "logp" else span(16, 16384), most)
    seqs = max(1, min(rng.randint(1, 16), rows // 2))
    if op == "preference":
        seqs = 2 * ((seqs + 1) // 2)
    vocab, rows = vocab + (vocab == 3072), rows - (rows == 3072)
    return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, seqs=seqs, prompt=rng.random() < 0.5,
                temperature=1.0 if op == "preference" else rng.choice([1.0, 1.0, 0.7]))


# ---- what a program has in hand ------------------------------------------------------------------------------------

CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.05
MAX_NORM = 1.0


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
    g.manual_seed((int(seed) * 1000003 + what * 7919 + 17) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(n, seed, what):
    return torch.randn(n, generator=_gen(seed, what), device=DEV, dtype=torch.float32)


def _row_chunks(rows, vocab):
    step = max(1, (1 << 26) // vocab)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


def _layer_tensors(case):
    """Elements of each tensor of the layers, and whether it is a vector."""
    h = case["h"]
    layer = [(h, True), (h, True), (3 * h * h, False), (3 * h, True), (h * h, False), (h, True), (h, True), (h, True),
             (4 * h * h, False), (4 * h, True), (4 * h * h, False), (h, True)]
    return [(n, v) for n, v in layer * case["layers"] if v or not case["vectors"]]


def _arenas(case):
    """Elements of each of the flat buffers that the tensors lie in one after another, by type."""
    sizes = {}
    for n, vector in _layer_tensors(case):
        kind = case["dtype"] if case["dtype"] != "mixed" else "f32" if vector else "bf16"
        sizes[kind] = sizes.get(kind, 0) + n
    return sizes


def _prepare_clip(case, seed):
    flat, outs = {}, {}
    for i, (kind, n) in enumerate(sorted(_arenas(case).items())):
        flat[kind] = torch.empty(n, dtype=DTYPES[kind], device=DEV)
        g = _gen(seed, 30 + i)
        for a in range(0, n, 1 << 26):
            b = min(n, a + (1 << 26))
            flat[kind][a:b] = torch.randn(b - a, generator=g, device=DEV) * 2e-2
        outs[kind] = torch.empty_like(flat[kind])
    at, tensors, into = dict.fromkeys(flat, 0), [], []
    for n, vector in _layer_tensors(case):
        kind = case["dtype"] if case["dtype"] != "mixed" else "f32" if vector else "bf16"
        tensors.append(flat[kind][at[kind]:at[kind] + n])
        into.append(outs[kind][at[kind]:at[kind] + n])
        at[kind] += n
    return {"flat": flat, "outs": outs, "tensors": tensors, "into": into,
            "sq": torch.zeros(1, dtype=torch.float64, device=DEV), "norm": torch.zeros(1, dtype=torch.float32, device=DEV)}


def prepare(case, seed):
    s = {"case": case, "ws": torch.empty(_WORKSPACE, dtype=torch.uint8, device=DEV)}
    if case["op"] == "clip":
        s.update(_prepare_clip(case, seed))
        return s
    rows, vocab, it = case["rows"], case["vocab"], 1.0 / case["temperature"]
    target = torch.randint(0, vocab, (rows,), generator=_gen(seed, 1), device=DEV)
    # a trained model's rows: most targets stand out, some do not
    lift = torch.where(torch.rand(rows, generator=_gen(seed, 2), device=DEV) < 0.7, 9.0, 0.0)
    logits = torch.empty(rows, vocab, dtype=DTYPES[case["dtype"]], device=DEV)
    logp = torch.empty(rows, dtype=torch.float32, device=DEV)
    g = _gen(seed, 3)
    for a, b in _row_chunks(rows, vocab):
        z = torch.randn(b - a, vocab, generator=g, device=DEV).mul_(2.5)
        z.scatter_add_(1, target[a:b, None], lift[a:b, None])
        logits[a:b] = z
        z = logits[a:b].float()
        logp[a:b] = (z.gather(1, target[a:b, None])[:, 0] - z.amax(1)) * it - ((z - z.amax(1, keepdim=True)) * it).exp_().sum(1).log()
    live = torch.ones(rows, dtype=torch.bool, device=DEV)
    for a, b in _prompts(case):
        live[a:b] = False
    target[~live] = -1
    logp[~live] = 0.0
    f32 = lambda: torch.zeros(rows, dtype=torch.float32, device=DEV)  # noqa: E731
    s.update(logits=logits, target=target, logp=f32())
    if case["op"] == "logp":
        return s
    s["dlogits"] = torch.empty_like(logits)
    ends = _ends(case)
    lengths = torch.tensor([b - a for a, b in zip(ends, ends[1:])], device=DEV)
    if case["op"] == "policy":
        # the policy has moved a little since the tokens were drawn; no ratio lies on the edge of the clipped range
        delta = _randn(rows, seed, 4) * 0.15
        for edge in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
            delta = torch.where((delta - edge).abs() < 2e-3, delta + 0.01, delta)
        s["old"] = logp - delta
        s["ref"] = logp + _randn(rows, seed, 5) * 0.3
        s["adv"] = _randn(len(lengths), seed, 6).repeat_interleave(lengths, output_size=rows)
        s["weights"] = live.float() / live.sum()
        s["stats"] = torch.zeros(4, dtype=torch.float32, device=DEV)
    else:
        s["ref"] = torch.where(live, logp + _randn(rows, seed, 5) * 0.3, 0.0)
        s["weights"] = live.float()
        s["offsets"] = torch.tensor(ends, dtype=torch.int64, device=DEV)
        s["row_stats"] = torch.zeros(rows, 2, dtype=torch.float32, device=DEV)
        s["dlogp"] = f32()
        s["margins"] = torch.zeros(len(lengths) // 2, dtype=torch.float32, device=DEV)
        s["loss"] = torch.zeros(1, dtype=torch.float32, device=DEV)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _plain_softmax(s):
    """Token log-probabilities and each row's probabilities, 32 bits."""
    it, target = 1.0 / s["case"]["temperature"], s["target"]
    x = s["logits"].float()
    x = (x - x.amax(1, keepdim=True)) * it
    live = target >= 0
    at = target.clamp(min=0)[:, None]
    picked = x.gather(1, at)[:, 0]
    e = x.exp_()
    total = e.sum(1, keepdim=True)
    logp = torch.where(live, picked - total[:, 0].log(), 0.0)
    return logp, e, total, at


def _plain_dlogits(s, dlogp, e, total, at):
    it = 1.0 / s["case"]["temperature"]
    d = e.mul_(-it * dlogp[:, None] / total)
    d.scatter_add_(1, at, (dlogp * it)[:, None])
    return torch.where(dlogp[:, None] == 0, 0.0, d).to(s["logits"].dtype)


def _plain(s):
    case = s["case"]
    if case["op"] == "clip":
        wide = {k: x.float() for k, x in s["flat"].items()}
        norm = sum((x * x).sum() for x in wide.values()).sqrt()
        c = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
        return {"norm": norm.reshape(1), "out": {k: (x * c).to(s["flat"][k].dtype) for k, x in wide.items()}}
    logp, e, total, at = _plain_softmax(s)
    if case["op"] == "logp":
        return {"logp": logp}
    if case["op"] == "policy":
        live = (s["weights"] != 0) & (s["target"] >= 0)
        r = (logp - s["old"]).exp()
        plain, held = r * s["adv"], r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * s["adv"]
        clipped = held < plain
        d = s["ref"] - logp
        pg, kl = -torch.minimum(plain, held), d.exp() - d - 1.0
        slope = torch.where(clipped, 0.0, -plain) + KL_COEF * (1.0 - d.exp())
        w = torch.where(live, s["weights"], 0.0)
        dlogp = w * slope
        stats = torch.stack([(w * (pg + KL_COEF * kl)).sum(), (w * pg).sum(), (w * kl).sum(), (w * clipped).sum()])
        return {"stats": stats, "logp": torch.where(live, logp, 0.0), "dlogits": _plain_dlogits(s, dlogp, e, total, at)}
    ends, w = s["offsets"], s["weights"]
    run = torch.where(w != 0, w * (logp - s["ref"]), 0.0)
    which = torch.bucketize(torch.arange(case["rows"], device=DEV), ends[1:], right=True)
    sums = torch.zeros(case["seqs"], device=DEV).index_add_(0, which, run)
    pairs = case["seqs"] // 2
    h = BETA * (sums[:pairs] - sums[pairs:])
    soft = lambda x: x.clamp(min=0) + (-x.abs()).exp().log1p()  # noqa: E731  ln(1 + exp(x))
    loss = ((1.0 - SMOOTHING) * soft(-h) + SMOOTHING * soft(h)).sum() / pairs
    up = 1.0 / (1.0 + (-h).exp())
    dh = (SMOOTHING * up - (1.0 - SMOOTHING) * (1.0 - up)) / pairs * BETA
    dlogp = torch.cat([dh, -dh])[which] * w
    return {"loss": loss.reshape(1), "margins": h, "logp": logp, "dlogp": dlogp, "dlogits": _plain_dlogits(s, dlogp, e, total, at)}


# ---- the framework's operators -------------------------------------------------------------------------------------

def _own(s):
    from paper_2512_17570_amd import gs

    case = s["case"]
    if case["op"] == "clip":
        gs.gs_grads_sqnorm(s["tensors"], s["sq"], s["ws"])
        gs.gs_grads_clip(s["tensors"], s["sq"], MAX_NORM, s["norm"], outs=s["into"])
        return {"norm": s["norm"], "out": s["outs"]}
    if case["op"] == "logp":
        gs.gs_token_logp(s["logits"], s["target"], s["logp"], temperature=case["temperature"], d_workspace=s["ws"])
        return {"logp": s["logp"]}
    if case["op"] == "policy":
        hp = gs.PolicyHParams(temperature=case["temperature"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF)
        gs.gs_policy_loss(s["logits"], s["target"], s["old"], s["ref"], s["adv"], s["weights"], hp, s["logp"], s["dlogits"], s["stats"], s["ws"])
        return {"stats": s["stats"], "logp": s["logp"], "dlogits": s["dlogits"]}
    hp = gs.PreferenceHParams(beta=BETA, label_smoothing=SMOOTHING, scale=2.0 / case["seqs"])
    gs.gs_token_logp(s["logits"], s["target"], s["logp"], s["row_stats"], d_workspace=s["ws"])
    gs.gs_preference_loss(s["logp"], s["ref"], s["weights"], s["offsets"], hp, s["margins"], s["dlogp"], s["loss"], s["ws"])
    gs.gs_token_logp_grad(s["logits"], s["target"], s["row_stats"], s["dlogp"], s["dlogits"])
    return {"loss": s["loss"], "margins": s["margins"], "logp": s["logp"], "dlogp": s["dlogp"], "dlogits": s["dlogits"]}


def run(s):
    return _own(s) if own else _plain(s)


def work(case):
    """Inputs once, outputs once; rows without a target are not read, and their gradients are zeros that are written."""
    if case["op"] == "clip":
        sizes = _arenas(case)
        n = sum(sizes.values())
        return {"bytes": 2 * sum(k * (2 if d == "bf16" else 4) for d, k in sizes.items()), "flops": 3 * n}
    rows, vocab, size = case["rows"], case["vocab"], 2 if case["dtype"] == "bf16" else 4
    live = rows - sum(b - a for a, b in _prompts(case))
    if case["op"] == "logp":
        return {"bytes": live * vocab * size + rows * 12, "flops": 4 * live * vocab}
    return {"bytes": (live + rows) * vocab * size + rows * (28 if case["op"] == "policy" else 24), "flops": 7 * live * vocab}


# ---- 64 bits -------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "clip":
        total = 0.0
        for x in s["flat"].values():
            for a in range(0, x.numel(), 1 << 26):
                total += float(x[a:a + (1 << 26)].to(f64).square().sum())
        norm = math.sqrt(total)
        c = min(1.0, MAX_NORM / (norm + 1e-6))
        return {"norm": torch.tensor([norm], dtype=f64), "out": {k: x.to(f64) * c for k, x in s["flat"].items()}}
    rows, vocab, temp = case["rows"], case["vocab"], case["temperature"]
    live = s["target"] >= 0
    at = s["target"].clamp(min=0)[:, None]

    def chunks():
        for a, b in _row_chunks(rows, 4 * vocab):
            yield a, b, torch.log_softmax(s["logits"][a:b].to(f64) / temp, dim=1)

    logp = torch.zeros(rows, dtype=f64, device=DEV)
    for a, b, ls in chunks():
        logp[a:b] = torch.where(live[a:b], ls.gather(1, at[a:b])[:, 0], 0.0)
    if case["op"] == "logp":
        return {"logp": logp}
    var = logp.clone().requires_grad_(True)
    if case["op"] == "policy":
        w, adv = s["weights"].to(f64), s["adv"].to(f64)
        ratio = torch.exp(var - s["old"].to(f64))
        a_free, a_held = ratio * adv, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
        pg = -torch.where(a_held < a_free, a_held, a_free)
        log_ratio = s["ref"].to(f64) - var
        kl = torch.expm1(log_ratio) - log_ratio
        sums = [(w * (pg + KL_COEF * kl))[live].sum(), (w * pg)[live].sum(), (w * kl)[live].sum(), (w * (a_held < a_free))[live].sum()]
        loss, out = sums[0], {"stats": torch.stack(sums).detach()}
    else:
        ends, pairs = _ends(case), case["seqs"] // 2
        ref, w = s["ref"].to(f64), s["weights"].to(f64)
        sums = torch.stack([((var[a:b] - ref[a:b]) * w[a:b]).sum() for a, b in zip(ends, ends[1:])])
        h = BETA * (sums[:pairs] - sums[pairs:])
        loss = -((1 - SMOOTHING) * torch.nn.functional.logsigmoid(h) + SMOOTHING * torch.nn.functional.logsigmoid(-h)).mean()
        out = {"loss": loss.detach().reshape(1), "margins": h.detach()}
    (dlogp,) = torch.autograd.grad(loss, var)
    dlogp = torch.where(live, dlogp, 0.0)
    grad = torch.empty(rows, vocab, dtype=f64, device=DEV)
    for a, b, ls in chunks():
        d = ls.exp().mul_(-dlogp[a:b, None])
        d.scatter_add_(1, at[a:b], dlogp[a:b, None])
        grad[a:b] = d / temp
    out.update(logp=logp, dlogits=grad)
    if case["op"] == "preference":
        out["dlogp"] = dlogp
    return out
