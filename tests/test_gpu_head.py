"""A linear head without its logits on the GPU (gs_head_logp, gs_head_logp_grad, gs_head_cross_entropy) against the definitions in 64 bits, at the sizes,
strides and masks where they can go wrong.  The bounds are derived in head_oracle.py."""
from __future__ import annotations

import pytest
import torch

from paper_2512_17570_amd import gs
from tests.head_oracle import F64, check, oracle

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


def rows_of(rows, cols, stride, gen, scale=1.0, shift=0):
    """(rows, cols) bf16 values whose rows lie `stride` apart, `shift` elements into their memory; what lies between is NaN."""
    flat = torch.full((shift + max(rows, 1) * stride,), float("nan"), dtype=BF16, device=DEV)
    m = flat[shift:].view(max(rows, 1), stride)[:rows, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * scale)
    return m


class Case:
    def __init__(self, rows, hidden, vocab, seed=0, bias=False, x_stride=None, w_stride=None, shift=0, prompt=False, weights="mean"):
        g = torch.Generator(device=DEV).manual_seed(seed * 1000 + rows * 31 + hidden * 7 + vocab)
        self.rows, self.hidden, self.vocab = rows, hidden, vocab
        self.x = rows_of(rows, hidden, x_stride or hidden, g, shift=shift)
        self.w = rows_of(vocab, hidden, w_stride or hidden, g, 2.0 * hidden ** -0.5, shift)
        self.bias = torch.randn(vocab, generator=g, device=DEV).to(BF16) if bias else None
        self.targets = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
        if prompt:
            self.targets[: rows // 3] = -1
            self.targets[rows // 2] = vocab
            self.targets[-1:] = -100
        if weights == "mean":
            self.weights = torch.full((rows,), 1.0 / max(rows, 1), device=DEV)
        else:
            self.weights = torch.rand(rows, generator=g, device=DEV) / max(rows, 1)
        self.logp = torch.full((rows,), float("nan"), device=DEV)
        self.stats = torch.full((rows, 2), float("nan"), device=DEV)
        self.loss = torch.full((1,), float("nan"), device=DEV)
        self.dx = rows_of(rows, hidden, x_stride or hidden, g, shift=shift)
        self.dw = rows_of(vocab, hidden, w_stride or hidden, g, shift=shift)
        self.db = torch.full((vocab,), float("nan"), dtype=BF16, device=DEV)

    def workspace(self, gradient=True):
        return torch.full((gs.gs_head_workspace_bytes(self.rows, self.hidden, self.vocab, gradient),), 0xFF, dtype=torch.uint8, device=DEV)

    def score(self, temperature=1.0):
        gs.gs_head_logp(self.x, self.w, self.bias, self.targets, self.logp, self.stats, temperature, self.workspace(False))
        return {"logp": self.logp, "M": self.stats[:, 0], "S": self.stats[:, 1]}

    def cross_entropy(self, temperature=1.0, **more):
        gs.gs_head_cross_entropy(self.x, self.w, self.bias, self.targets, self.weights, self.logp, self.dx, self.dw, self.db, self.loss, self.workspace(),
                                 temperature, **more)
        return {"logp": self.logp, "dx": self.dx, "dw": self.dw, "db": self.db}

    def check_loss(self, temperature=1.0):
        got = self.cross_entropy(temperature)
        out, bound = oracle(self.x, self.w, self.bias, self.targets, None if self.weights is None else -self.weights, temperature)
        check(got, out, bound, ["logp", "dx", "dw", "db"])
        w = self.weights.to(F64)
        want = -(torch.where(w != 0, w, 0.0) * out["logp"]).sum()
        if bool(want.isfinite()):
            off = float((w.abs() * bound["logp"]).sum()) + abs(float(want)) * 2.0 ** -23
            assert abs(float(self.loss) - float(want)) <= off, (float(self.loss), float(want), off)
        return out


SIZES = [(1, 1, 1), (1, 64, 1), (1, 64, 2), (2, 8, 255), (3, 64, 256), (15, 72, 257), (16, 128, 1000), (17, 100, 513), (33, 512, 300), (64, 7, 999), (65, 192, 1031),
         (255, 64, 511), (256, 256, 512), (257, 264, 513), (300, 1000, 777), (513, 320, 1025), (700, 63, 90), (128, 448, 1500), (129, 128, 255), (1500, 128, 40_100)]


@pytest.mark.parametrize("rows, hidden, vocab", SIZES)
def test_scores(rows, hidden, vocab):
    c = Case(rows, hidden, vocab, prompt=rows > 4, bias=vocab % 2 == 1)
    got = c.score(0.7)
    out, bound = oracle(c.x, c.w, c.bias, c.targets, None, 0.7, gradient=False)
    check(got, out, bound, ["logp", "M", "S"])


@pytest.mark.parametrize("hidden", [8, 100, 504, 512, 2048, 2056, 4096, 4104, 8192, 8200])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9, 16, 17])
def test_scores_of_few_rows(rows, hidden):
    """Both sides of the lines between the kernels for few rows."""
    for vocab, bias in ((700, False), (65, True)):
        c = Case(rows, hidden, vocab, bias=bias, prompt=rows > 4)
        got = c.score(1.3)
        out, bound = oracle(c.x, c.w, c.bias, c.targets, None, 1.3, gradient=False)
        check(got, out, bound, ["logp", "M", "S"])


@pytest.mark.parametrize("rows, hidden, vocab", SIZES)
def test_cross_entropy(rows, hidden, vocab):
    Case(rows, hidden, vocab, prompt=rows > 4, bias=vocab % 2 == 0).check_loss(1.0 if rows % 2 else 1.5)


@pytest.mark.parametrize("rows, hidden, vocab", [(5, 64, 300), (40, 128, 257), (300, 192, 700)])
@pytest.mark.parametrize("x_pad, w_pad, shift", [(8, 64, 0), (1, 8, 0), (8, 3, 0), (0, 0, 1), (5, 7, 3)])
def test_any_stride_and_alignment(rows, hidden, vocab, x_pad, w_pad, shift):
    c = Case(rows, hidden, vocab, x_stride=hidden + x_pad, w_stride=hidden + w_pad, shift=shift, weights="uneven", bias=True)
    before = [t._base.clone() for t in (c.dx, c.dw)]
    c.check_loss()
    got = c.score(2.0)
    out, bound = oracle(c.x, c.w, c.bias, c.targets, None, 2.0, gradient=False)
    check(got, out, bound, ["logp", "M", "S"])
    for t, old, pad in ((c.dx, before[0], x_pad), (c.dw, before[1], w_pad)):       # nothing between the rows is written
        mine = torch.zeros_like(old, dtype=torch.bool)
        mine[shift:].view(-1, hidden + pad)[:, :hidden] = True
        assert torch.equal(t._base.view(torch.int16)[~mine], old.view(torch.int16)[~mine])


@pytest.mark.parametrize("rows", [3, 70, 300])
def test_rows_that_do_not_count_may_hold_anything(rows):
    c = Case(rows, 128, 400, prompt=True, weights="uneven", bias=True)
    c.weights[1] = 0.0
    dead = (c.targets < 0) | (c.targets >= c.vocab) | (c.weights == 0)
    c.x[dead] = torch.tensor([float("nan"), float("inf")], dtype=BF16, device=DEV).repeat(64)
    c.weights[dead & (c.weights != 0)] = float("nan")
    c.weights[-1] = float("inf")
    got = c.cross_entropy()
    w = torch.where(dead, 0.0, c.weights)
    out, bound = oracle(c.x, c.w, c.bias, c.targets, -w)
    check(got, out, bound, ["logp", "dx", "dw", "db"])
    assert not bool(c.dx[dead].view(torch.int16).any()) and not bool(c.logp[dead].view(torch.int32).any())        # +0
    c.score()
    assert bool((c.stats[(c.targets < 0) | (c.targets >= c.vocab)] == torch.tensor([0.0, 1.0], device=DEV)).all())


@pytest.mark.parametrize("rows", [0, 1, 5, 300])
def test_nothing_counts(rows):
    c = Case(rows, 64, 300)
    c.targets.fill_(-1)
    got = c.cross_entropy()
    for name, t in got.items():
        assert not bool(t.view(torch.int16 if t.dtype == BF16 else torch.int32).any()), name
    assert float(c.loss) == 0.0
    c.loss.fill_(3.5)
    c.cross_entropy(accumulate=True)
    assert float(c.loss) == 3.5


@pytest.mark.parametrize("rows", [2, 40, 260])
def test_excluded_words(rows):
    c = Case(rows, 64, 700, bias=True)
    c.bias[::3] = float("-inf")
    c.bias[256:512] = float("-inf")              # a whole tile of words
    c.bias[5] = torch.finfo(BF16).min            # the type's lowest value
    c.targets.fill_(1)
    c.targets[0] = 0                             # an excluded one: its log-probability is -inf
    c.weights[0] = 0.0
    c.check_loss()
    assert float(c.score()["logp"][0]) == float("-inf")
    c.bias.fill_(float("-inf"))                  # nothing is left
    assert bool(c.score()["logp"].isnan().all())


def test_nan_and_infinity_in_a_row_stay_there():
    c = Case(300, 64, 500)
    c.x[7, 3] = float("nan")
    c.x[9, 3] = float("inf")
    logp = c.score()["logp"]
    assert bool(logp[[7, 9]].isnan().all()) and int(logp.isnan().sum()) == 2
    c.cross_entropy()
    assert bool(c.dx[[7, 9]].isnan().all())
    rest = torch.ones(300, dtype=torch.bool, device=DEV)
    rest[[7, 9]] = False
    assert not bool(c.dx[rest].isnan().any())


@pytest.mark.parametrize("rows, hidden, vocab, bias", [(8192, 64, 40_000, True), (20_000, 72, 9_000, False), (3, 64, 300_000, True), (5, 8, 4_400_000, True), (1100, 512, 20_000, True),
                                                       (20, 8200, 10_000, True), (300, 8200, 9_000, False)])
def test_many_pieces_and_tiles(rows, hidden, vocab, bias):
    """More words than a piece has, with z kept and made again, weights packed in pieces of their own, more rows than a group of tiles."""
    Case(rows, hidden, vocab, prompt=True, bias=bias).check_loss()


@pytest.mark.parametrize("rows, hidden, vocab", [(256, 136, 32_768), (250, 136, 32_769), (700, 1000, 11_003), (600, 264, 17_001), (40, 1000, 8_300), (40, 1000, 8_100),
                                                 (70, 128, 20_000), (300, 129, 17_000)])
def test_large_and_small_tiles(rows, hidden, vocab):
    """Both sides of the numbers of tiles from which they are large: of the statistics and dz, of the sums to the rows, of those to the weights."""
    Case(rows, hidden, vocab, prompt=True, bias=vocab % 2 == 1).check_loss()


@pytest.mark.parametrize("rows, hidden, vocab", [(40, 1000, 16_384), (40, 264, 16_385), (33, 100, 17_003), (64, 600, 20_001), (17, 64, 33_000)])
def test_narrow_tiles(rows, hidden, vocab):
    """Up to 64 rows, both sides of the number of words from which their tiles are of 128."""
    c = Case(rows, hidden, vocab, prompt=True, bias=vocab % 2 == 1)
    got = c.score(0.7)
    out, bound = oracle(c.x, c.w, c.bias, c.targets, None, 0.7, gradient=False)
    check(got, out, bound, ["logp", "M", "S"])
    c.check_loss(0.7)


@pytest.mark.parametrize("rows, hidden, vocab", [(4, 64, 500), (30, 256, 700), (400, 128, 600)])
def test_gradient_from_logp(rows, hidden, vocab):
    """Any gradient in the log-probabilities, statistics from gs_head_logp; the parts that nobody needs left out."""
    c = Case(rows, hidden, vocab, bias=True, prompt=rows > 4)
    c.score(0.8)
    dlogp = torch.randn(rows, device=DEV)
    dlogp[2] = 0.0
    out, bound = oracle(c.x, c.w, c.bias, c.targets, dlogp, 0.8)
    for parts in ("dx", "dw", "db", "dx dw", "dx dw db"):
        c.dx.fill_(7.0), c.dw.fill_(7.0), c.db.fill_(7.0)
        gs.gs_head_logp_grad(c.x, c.w, c.bias, c.targets, c.stats, dlogp, *[t if n in parts.split() else None for n, t in (("dx", c.dx), ("dw", c.dw), ("db", c.db))],
                             c.workspace(), temperature=0.8)
        check({"dx": c.dx, "dw": c.dw, "db": c.db}, out, bound, parts.split())
        for n, t in (("dx", c.dx), ("dw", c.dw), ("db", c.db)):
            assert n in parts.split() or bool((t == 7.0).all())


def test_gradients_against_differences():
    c = Case(37, 128, 300, bias=True, prompt=True)
    c.check_loss()
    w64 = [t.to(F64) for t in (c.x, c.w, c.bias)]
    live = (c.targets >= 0) & (c.targets < c.vocab)

    def loss(x, w, b):
        ls = torch.log_softmax(x @ w.t() + b, 1)
        return -(c.weights.to(F64) * ls.gather(1, c.targets.clamp(0, c.vocab - 1)[:, None])[:, 0])[live].sum()

    g = torch.Generator(device=DEV).manual_seed(5)
    for i, grad in enumerate((c.dx, c.dw, c.db)):
        way = torch.randn(grad.shape, generator=g, device=DEV, dtype=F64)
        step = 1e-5
        ends = [loss(*[t + (s * step * way if j == i else 0) for j, t in enumerate(w64)]) for s in (1, -1)]
        slope = float((ends[0] - ends[1]) / (2 * step))
        _, bound = oracle(c.x, c.w, c.bias, c.targets, -c.weights)
        off = float((bound[("dx", "dw", "db")[i]] * way.abs()).sum()) + 1e-7
        assert abs(slope - float((grad.to(F64) * way).sum())) <= off


def test_without_weights_or_gradient_and_accumulated():
    c = Case(100, 64, 300, prompt=True)
    c.weights = torch.ones(100, device=DEV)
    got = {k: v.clone() for k, v in c.cross_entropy().items()}
    first = c.loss.clone()
    c.weights = None
    c.dx.fill_(0), c.dw.fill_(0), c.loss.fill_(2.0)
    again = c.cross_entropy(accumulate=True)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    assert float(c.loss) == pytest.approx(float(first) + 2.0, rel=2.0 ** -23)
    gs.gs_head_cross_entropy(c.x, c.w, None, c.targets, None, c.logp, None, None, None, c.loss, c.workspace(False))
    assert torch.equal(c.loss, first) and torch.equal(c.logp, got["logp"])


@pytest.mark.parametrize("rows", [1, 9, 64, 500])
def test_same_bits_from_call_to_call_on_any_stream_and_from_a_graph(rows):
    c, d = Case(rows, 256, 900, bias=True, prompt=rows > 8), Case(rows, 256, 900, seed=1, bias=True, prompt=rows > 8)
    want = []
    for q in (c, d):
        want.append({k: v.clone() for k, v in q.cross_entropy().items()} | {"loss": q.loss.clone()})
    side = torch.cuda.Stream()
    spaces = [c.workspace(), d.workspace()]

    def call(q, ws):
        gs.gs_head_cross_entropy(q.x, q.w, q.bias, q.targets, q.weights, q.logp, q.dx, q.dw, q.db, q.loss, ws)

    def check_all(q, k):
        for name, t in {"logp": q.logp, "dx": q.dx, "dw": q.dw, "db": q.db, "loss": q.loss}.items():
            assert torch.equal(t.view(torch.uint8) if t.is_contiguous() else t, want[k][name].view(torch.uint8) if t.is_contiguous() else want[k][name]), name

    def spoil(q):
        for t in (q.logp, q.dx, q.dw, q.db, q.loss):
            t.fill_(9.0)

    spoil(c)
    side.wait_stream(torch.cuda.current_stream())
    gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, c.dx, c.dw, c.db, c.loss, spaces[0], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check_all(c, 0)
    graphs = []
    for q, ws in ((c, spaces[0]), (d, spaces[1])):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(q, ws)
        graphs.append(graph)
    for _ in range(3):
        for k, q in enumerate((c, d)):
            spoil(q)
            graphs[k].replay()
            torch.cuda.synchronize()
            check_all(q, k)
    for k, q in enumerate((c, d)):                # both on the way at once
        spoil(q)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, graph in zip(streams, graphs):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    check_all(c, 0), check_all(d, 1)


@pytest.mark.parametrize("rows", [3, 50, 400])
def test_on_some_of_the_cus(rows):
    """A stream that has 16 of the CUs: the same bits."""
    c = Case(rows, 512, 1500, bias=True, prompt=rows > 4)
    want = {k: v.clone() for k, v in c.cross_entropy().items()}
    ws = c.workspace()
    stream = gs.gs_cu_stream_create(16)
    try:
        for t in (c.logp, c.dx, c.dw, c.db):
            t.fill_(8.0)
        torch.cuda.synchronize()
        gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, c.dx, c.dw, c.db, c.loss, ws, stream=stream)
        torch.cuda.synchronize()
        for k, v in {"logp": c.logp, "dx": c.dx, "dw": c.dw, "db": c.db}.items():
            assert torch.equal(v, want[k]), k
    finally:
        gs.gs_cu_stream_destroy(stream)


def test_two_calls_at_once_with_workspaces_of_their_own():
    c, d = Case(300, 256, 2000), Case(90, 256, 2000, seed=3)
    want = [{k: v.clone() for k, v in q.cross_entropy().items()} for q in (c, d)]
    spaces, streams = [c.workspace(), d.workspace()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for q, ws, s in zip((c, d), spaces, streams):
            gs.gs_head_cross_entropy(q.x, q.w, q.bias, q.targets, q.weights, q.logp, q.dx, q.dw, q.db, q.loss, ws, stream=s)
    torch.cuda.synchronize()
    for q, w in zip((c, d), want):
        for k, v in {"logp": q.logp, "dx": q.dx, "dw": q.dw, "db": q.db}.items():
            assert torch.equal(v, w[k]), k


def test_weights_beyond_32_bits_of_offsets():
    """2^32 and more elements of weights and of their gradient: the last words' results are those of the last words alone."""
    hidden, vocab, rows = 8192, (1 << 19) + 300, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    w = torch.zeros(vocab, hidden, dtype=BF16, device=DEV)
    tail = torch.randn(600, hidden, generator=g, device=DEV) * hidden ** -0.5
    w[-600:] = tail
    bias = torch.full((vocab,), float("-inf"), dtype=BF16, device=DEV)
    bias[-600:] = 0.25
    x = torch.randn(rows, hidden, generator=g, device=DEV).to(BF16)
    targets = torch.arange(rows, device=DEV) * 119 + vocab - 600
    c = Case(1, 8, 8)
    c.__dict__.update(rows=rows, hidden=hidden, vocab=vocab, x=x, w=w, bias=bias, targets=targets, weights=torch.full((rows,), 0.2, device=DEV),
                      logp=torch.empty(rows, device=DEV), stats=torch.empty(rows, 2, device=DEV), dx=torch.empty_like(x), dw=torch.full_like(w, 3.0),
                      db=torch.empty_like(bias), loss=torch.empty(1, device=DEV))
    got = c.cross_entropy()
    out, bound = oracle(x, w[-600:], bias[-600:], targets - (vocab - 600), -c.weights)
    assert not bool(got["dw"][:-600].any()) and not bool(got["db"][:-600].any())
    check({"logp": got["logp"], "dx": got["dx"], "dw": got["dw"][-600:], "db": got["db"][-600:]}, out, bound, ["logp", "dx", "dw", "db"])
    check(c.score(), out, bound, ["logp", "M", "S"])


def test_preference_loss_without_logits():
    """Token log-probabilities, the loss of pairs, and its gradient in the head: the three calls as a program makes them."""
    c = Case(90, 128, 400, bias=True)
    offsets = torch.tensor([0, 20, 45, 60, 90], device=DEV)
    ref, weights = torch.randn(90, device=DEV) * 0.2 - 5.0, torch.ones(90, device=DEV)
    weights[:5] = 0.0
    ws, small = c.workspace(), torch.empty(gs.gs_sqnorm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    margins, dlogp, loss = torch.empty(2, device=DEV), torch.empty(90, device=DEV), torch.empty(1, device=DEV)
    gs.gs_head_logp(c.x, c.w, c.bias, c.targets, c.logp, c.stats, d_workspace=ws)
    gs.gs_preference_loss(c.logp, ref, weights, offsets, gs.PreferenceHParams(beta=0.3, scale=0.5), margins, dlogp, loss, small)
    gs.gs_head_logp_grad(c.x, c.w, c.bias, c.targets, c.stats, dlogp, c.dx, c.dw, c.db, ws)
    out, bound = oracle(c.x, c.w, c.bias, c.targets, dlogp)
    check({"dx": c.dx, "dw": c.dw, "db": c.db}, out, bound, ["dx", "dw", "db"])


def test_native_and_general_reading_agree():
    """A raw stream and workspace bytes by name are read natively too, a NumPy-like temperature or a raw address is not: the same results."""
    c = Case(70, 64, 300, bias=True, prompt=True)
    want = {k: v.clone() for k, v in c.cross_entropy().items()}
    ws = c.workspace()
    for t in (c.logp, c.dx, c.dw, c.db):
        t.fill_(8.0)
    gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, c.dx, c.dw, c.db, c.loss, ws.data_ptr(), 1, workspace_bytes=ws.numel(),
                             stream=torch.cuda.current_stream().cuda_stream)
    for k, v in {"logp": c.logp, "dx": c.dx, "dw": c.dw, "db": c.db}.items():
        assert torch.equal(v, want[k]), k
    c.score(0.5)
    one = c.logp.clone(), c.stats.clone()
    gs.gs_head_logp(c.x, c.w, c.bias, c.targets, c.logp.fill_(0), c.stats, 0.5, ws.data_ptr(), workspace_bytes=ws.numel())
    assert torch.equal(c.logp, one[0]) and torch.equal(c.stats, one[1])


def test_binding_refuses():
    c = Case(10, 64, 100)
    ws = c.workspace()
    call = lambda **k: gs.gs_head_logp(k.get("x", c.x), k.get("w", c.w), k.get("bias"), k.get("targets", c.targets), k.get("logp", c.logp), d_workspace=k.get("ws", ws))  # noqa: E731
    for kind, bad in ((TypeError, dict(x=c.x.float())), (ValueError, dict(x=c.x[:, :32])), (ValueError, dict(x=c.x.cpu())), (TypeError, dict(targets=c.targets.int())),
                      (ValueError, dict(logp=c.logp[:5])), (ValueError, dict(bias=torch.zeros(99, dtype=BF16, device=DEV))), (ValueError, dict(x=c.x.t())),
                      (gs.GsError, dict(ws=ws[: 256])), (gs.GsError, dict(ws=None)), (gs.GsError, dict(ws=ws[8:]))):
        with pytest.raises(kind):
            call(**bad)
