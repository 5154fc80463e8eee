"""Layer norm, its gradient and dropout on the GPU against their definitions in 64 bits.

Bounds.  u = 2^-24 is half a step in 32 bits, t that of the output's type (2^-8 or 2^-24).  A sum of n values in 32 bits is off by at most n u sum |values|.
    mean  (n + 1) u mean |x|                                                             e_m
    rstd  relative: half of what the variance is off by, relative: (n + 8) u / 2 + the mean's share e_m |..|, which enters squared (the sum
          of the deviations is 0): (e_m rstd)^2 / 2; and 3 u                             e_r
    xhat  e_m rstd + |xhat| (e_r + 3 u);  y: |gamma| e_xhat + u (2 |xhat gamma| + |y|) + t |y|
    dx    the two means are off by (n + 6) u mean |g| and (n + 8) u mean |g xhat| + mean |g| e_xhat; xhat's own error meets the second mean
    dgamma, dbeta: (rows + 6) u sum |dy xhat| + sum |dy| e_xhat, (rows + 1) u sum |dy|; and t of themselves
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2512_17570_amd import gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = 2.0 ** -24
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def rows_of(rows, cols, stride, dtype, gen, shift=0, scale=1.0, base=0.0):
    flat = torch.full((shift + max(rows, 1) * stride,), float("nan"), dtype=dtype, device=DEV)
    m = flat[shift:].view(max(rows, 1), stride)[:rows, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * scale + base)
    return m


def norm_bounds(x, eps):
    n = x.shape[1]
    mean, var = x.mean(1, keepdim=True), x.var(1, correction=0, keepdim=True)
    rstd = (var + eps).rsqrt()
    hat = (x - mean) * rstd
    e_m = (n + 1) * U * x.abs().mean(1, keepdim=True)
    e_r = (n + 8) * U / 2 + (e_m * rstd) ** 2 / 2 + 3 * U
    e_hat = e_m * rstd + hat.abs() * (e_r + 3 * U) + 2 * U * x.abs().amax(1, keepdim=True) * rstd
    return mean, rstd, hat, e_m, e_r, e_hat


def within(got, want, bound, what):
    got = got.to(F64)
    ok = (got - want).abs() <= bound + 1e-38
    if not bool(ok.all()):
        i = int((~ok).flatten().nonzero()[0])
        raise AssertionError(f"{what}[{i}]: {got.flatten()[i].item()} for {want.flatten()[i].item()}, bound {(bound + 0 * want).flatten()[i].item()}, {int((~ok).sum())} of {ok.numel()}")


COLS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1001, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 20000, 32768, 32769, 70001]
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)]


def run_norm(rows, cols, dtype, wtype, pads=(0, 0, 0), shift=0, eps=1e-5, base=0.5, vectors=True, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + rows * 131 + cols)
    x = rows_of(rows, cols, cols + pads[0], dtype, g, shift, 2.0, base)
    gamma = (torch.randn(cols, generator=g, device=DEV) * 0.3 + 1.0).to(wtype) if vectors else None
    beta = torch.randn(cols, generator=g, device=DEV).to(wtype) if vectors else None
    y = rows_of(rows, cols, cols + pads[1], dtype, g, shift)
    stats = torch.full((rows, 2), float("nan"), device=DEV)
    gs.gs_layer_norm(x, gamma, beta, y, stats, eps)
    wide, one = x.to(F64), torch.ones(cols, dtype=F64, device=DEV)
    mean, rstd, hat, e_m, e_r, e_hat = norm_bounds(wide, eps)
    gm, bt = (gamma.to(F64), beta.to(F64)) if vectors else (one, 0 * one)
    want = hat * gm + bt
    within(stats[:, :1], mean, e_m, "mean")
    within(stats[:, 1:], rstd, rstd * e_r, "rstd")
    within(y, want, gm.abs() * e_hat + U * (2 * (hat * gm).abs() + want.abs()) + HALF[dtype] * want.abs() * 1.001, "y")
    # the gradient, its statistics from the call above
    dy = rows_of(rows, cols, cols + pads[2], dtype, g, shift, 1e-2)
    dx = rows_of(rows, cols, cols + pads[1], dtype, g, shift)
    before = dx._base.clone()
    dgamma, dbeta = (torch.full((cols,), float("nan"), dtype=wtype, device=DEV) for _ in range(2))
    ws = torch.full((gs.gs_layer_norm_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device=DEV)
    gs.gs_layer_norm_grad(dy, x, gamma, stats, dx, dgamma, dbeta, ws)
    d = dy.to(F64)
    gr = d * gm
    a, b = gr.mean(1, keepdim=True), (gr * hat).mean(1, keepdim=True)
    want = rstd * (gr - a - hat * b)
    abs_g = gr.abs().mean(1, keepdim=True)
    e_b = (cols + 8) * U * (gr * hat).abs().mean(1, keepdim=True) + (gr.abs() * e_hat).mean(1, keepdim=True)
    inner = gr.abs() + a.abs() + (hat * b).abs()
    e_dx = rstd * ((cols + 6) * U * abs_g + hat.abs() * e_b + e_hat * b.abs() + 8 * U * inner + (e_r + 2 * U) * inner)
    within(dx, want, e_dx + HALF[dtype] * want.abs() * 1.001, "dx")
    e_dg = (rows + 6) * U * (d * hat).abs().sum(0) + (d.abs() * e_hat).sum(0)
    dg, db = (d * hat).sum(0), d.sum(0)
    within(dgamma, dg, e_dg + HALF[wtype] * dg.abs() * 1.001, "dgamma")
    within(dbeta, db, (rows + 1) * U * d.abs().sum(0) + HALF[wtype] * db.abs() * 1.001, "dbeta")
    mine = torch.zeros(before.shape, dtype=torch.bool, device=DEV)                   # nothing between the rows is written
    mine[shift:].view(-1, cols + pads[1])[:rows, :cols] = True
    assert bool(dx._base[~mine].isnan().all())
    return x, gamma, beta, y, stats, dy, dx, dgamma, dbeta, ws


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype, wtype", TYPES)
def test_norm_at_any_width(cols, dtype, wtype):
    for rows in (1, 5) if cols > 9000 else (1, 7, 600):
        run_norm(rows, cols, dtype, wtype)


@pytest.mark.parametrize("dtype, wtype", TYPES)
@pytest.mark.parametrize("pads, shift", [((1, 3, 5), 0), ((8, 0, 16), 0), ((0, 0, 0), 1), ((7, 2, 0), 3)])
def test_norm_at_any_stride_and_alignment(dtype, wtype, pads, shift):
    for cols in (9, 640, 1000, 4099, 17000):
        run_norm(13, cols, dtype, wtype, pads, shift)


@pytest.mark.parametrize("rows, cols", [(5000, 256), (3001, 1000), (2500, 3000 + 71), (1500, 8192), (700, 17001)])
def test_norm_of_many_rows(rows, cols):
    """More rows than a gradient has workgroups: columns are added up over several rows, then over workgroups."""
    run_norm(rows, cols, BF16, F32)
    run_norm(rows, cols, F32, F32, vectors=False)


@pytest.mark.parametrize("rows", [256, 257])
@pytest.mark.parametrize("cols", [1000, 2052, 8192])
def test_norm_of_few_and_many_rows(rows, cols):
    """Both sides of the number of rows from which workgroups stay."""
    run_norm(rows, cols, BF16, BF16)
    run_norm(rows, cols, F32, BF16, vectors=False)


def test_norm_in_place():
    g = torch.Generator(device=DEV).manual_seed(0)
    for cols in (100, 1000, 5000, 40000):
        x, gamma, beta, y, stats, dy, dx, dgamma, dbeta, ws = run_norm(9, cols, BF16, BF16)
        inplace = x.clone()
        gs.gs_layer_norm(inplace, gamma, beta, inplace)
        assert torch.equal(inplace, y)
        d = dy.clone()
        dg, db = torch.empty_like(dgamma), torch.empty_like(dbeta)
        gs.gs_layer_norm_grad(d, x, gamma, stats, d, dg, db, ws)
        assert torch.equal(d, dx) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)
        d = dy.clone()
        gs.gs_layer_norm_grad(d, x, gamma, stats, d, None, None)
        assert torch.equal(d, dx)


def test_norm_rows_of_one_value_and_not_finite():
    x = torch.full((4, 300), 3.25, dtype=BF16, device=DEV)
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    y, stats = torch.empty_like(x), torch.empty(4, 2, device=DEV)
    gs.gs_layer_norm(x, None, None, y, stats, 1e-5)
    assert not bool(y[[0, 3]].any()) and bool(y[1:3].isnan().all()) and float(stats[0, 0]) == 3.25
    big = torch.tensor([[1e4, 1e4 + 1.0, 1e4 - 1.0, 1e4]], device=DEV)          # the squares only after the mean
    y = torch.empty_like(big)
    gs.gs_layer_norm(big, None, None, y, None, 0.0)
    assert torch.allclose(y.to(F64), torch.tensor([[0.0, 2.0 ** 0.5, -(2.0 ** 0.5), 0.0]], dtype=F64, device=DEV), atol=1e-5)


def test_norm_without_rows():
    x = torch.empty(0, 64, dtype=BF16, device=DEV)
    gs.gs_layer_norm(x, None, None, x)
    dg, db = torch.full((64,), 5.0, device=DEV), torch.full((64,), 5.0, device=DEV)
    gs.gs_layer_norm_grad(x, x, None, torch.empty(0, 2, device=DEV), x, dg, db, torch.empty(gs.gs_layer_norm_workspace_bytes(0, 64), dtype=torch.uint8, device=DEV))
    assert not bool(dg.any()) and not bool(db.any())


def test_norm_gradients_against_differences():
    x, gamma, beta, y, stats, dy, dx, dgamma, dbeta, ws = run_norm(6, 130, F32, F32)
    d, eps = dy.to(F64), 1e-5

    def loss(x, gamma, beta):
        m = x - x.mean(1, keepdim=True)
        return ((m / (m.square().mean(1, keepdim=True) + eps).sqrt() * gamma + beta) * d).sum()

    at = [t.to(F64) for t in (x, gamma, beta)]
    for i, grad in enumerate((dx, dgamma, dbeta)):
        way = torch.randn(grad.shape, dtype=F64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(i))
        ends = [loss(*[t + (s * 1e-5 * way if j == i else 0) for j, t in enumerate(at)]) for s in (1, -1)]
        assert float((ends[0] - ends[1]) / 2e-5) == pytest.approx(float((grad.to(F64) * way).sum()), rel=1e-5, abs=1e-6)


def test_norm_from_graphs_and_streams():
    x, gamma, beta, y, stats, dy, dx, dgamma, dbeta, ws = run_norm(900, 2048, BF16, BF16)
    want = [t.clone() for t in (y, stats, dx, dgamma, dbeta)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_layer_norm(x, gamma, beta, y, stats)
        gs.gs_layer_norm_grad(dy, x, gamma, stats, dx, dgamma, dbeta, ws)
    for _ in range(3):
        for t in (y, stats, dx, dgamma, dbeta):
            t.fill_(4.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((y, stats, dx, dgamma, dbeta), want):
            assert torch.equal(t, w)
    y.fill_(0)
    torch.cuda.synchronize()
    gs.gs_layer_norm(x, gamma, beta, y, stats, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])


def test_norm_beyond_32_bits_of_offsets():
    rows, cols = (1 << 20) + 3, 4099            # 2^32 elements and more
    x = torch.empty(rows, cols, dtype=BF16, device=DEV)
    x[:] = (torch.arange(rows, device=DEV) % 97).to(BF16)[:, None]
    x[:, ::2] += 3
    y = torch.empty_like(x)
    gs.gs_layer_norm(x, None, None, y)
    tail = torch.empty(5, cols, dtype=BF16, device=DEV)
    gs.gs_layer_norm(x[-5:].clone(), None, None, tail)
    assert torch.equal(y[-5:], tail) and torch.equal(y[97 * 10000], y[0])


# ---- dropout -----------------------------------------------------------------------------------------------------------

def kept(n, p, seed, offset, step):
    """The mask, from the published generator (Philox4x32-10) in whole numbers."""
    least = int(np.floor(p * 65536 + 0.5))
    m, u = np.uint64(0xFFFFFFFF), np.uint64
    with np.errstate(over="ignore"):
        blocks = u(offset // 8) + np.arange((n + offset % 8 + 7) // 8, dtype=u)
        c = [blocks & m, blocks >> u(32), np.full_like(blocks, step & 0xFFFFFFFF), np.full_like(blocks, step >> 32)]
        k0, k1 = seed & 0xFFFFFFFF, seed >> 32
        for _ in range(10):
            a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
            c = [(b >> u(32)) ^ c[1] ^ u(k0), b & m, (a >> u(32)) ^ c[3] ^ u(k1), a & m]
            k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    bits = np.stack(c, 1).astype(np.uint32).view(np.uint16).reshape(-1)[offset % 8: offset % 8 + n]
    return torch.from_numpy(bits.astype(np.int64) >= least).to(DEV), 65536.0 / (65536 - least) if least < 65536 else 0.0


def test_the_oracles_generator_is_the_published_one():
    """Known answers of Philox4x32-10: counter and key all zeros, and all ones."""
    def words(counter, key):
        c, k = list(counter), list(key)
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        return c
    assert words([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def run_dropout(n, dtype, p, seed, offset, step, residual, shift=0):
    g = torch.Generator(device=DEV).manual_seed(n)
    flat = lambda: torch.randn(n + shift, generator=g, device=DEV).to(dtype)[shift:]  # noqa: E731
    x, res = flat(), flat() if residual else None
    out = torch.full((n + shift + 9,), float("nan"), dtype=dtype, device=DEV)
    mask, scale = kept(n, p, seed, offset, step)
    x[~mask] = float("nan")                        # what is dropped does not count
    at = torch.tensor([step], dtype=torch.int64, device=DEV) if step else None
    gs.gs_dropout(x, res, out[shift:shift + n], p, seed, offset, at)
    want = torch.where(mask, x.to(F64) * scale, 0.0)
    size = want.abs()
    if residual:
        want = want + res.to(F64)
    within(out[shift:shift + n], want, 2 * U * size + U * want.abs() + HALF[dtype] * want.abs() * 1.001, "out")
    assert bool(out[:shift].isnan().all()) and bool(out[shift + n:].isnan().all())
    return x, res, out[shift:shift + n]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 1000, 2048, 2049, 100_003])
def test_dropout(n, dtype, residual):
    for offset, shift in ((0, 0), (3, 1), (8, 3), ((1 << 35) + 5, 0)):
        run_dropout(n, dtype, 0.1, 12345678901234567, offset, 7, residual, shift)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 0.25, 0.5, 0.9999, 1.0])
def test_dropout_of_any_share(p):
    x, res, out = run_dropout(5000, F32, p, 3, 0, 0, True)
    if p in (0.0, 1.0):
        assert torch.equal(out, res if p else x + res)


def test_dropout_numbers_at_their_limits():
    run_dropout(1000, F32, 0.3, (1 << 64) - 1, (1 << 64) - 1000, (1 << 63) - 1, False)


def test_dropout_mask_is_of_elements_and_not_of_calls():
    """Any part alone, in place or onto the residual, forward or backward: the same elements."""
    n, seed = 50_001, 99
    x, res = torch.randn(n, device=DEV).to(BF16), torch.randn(n, device=DEV).to(BF16)
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    gs.gs_dropout(x, res, whole, 0.2, seed, 1000)
    for a, b in ((0, 1), (1, 17), (17, 20_000), (20_000, 20_003), (20_003, n)):
        gs.gs_dropout(x[a:b], res[a:b], parts[a:b], 0.2, seed, 1000 + a)
    assert torch.equal(whole, parts)
    onto = res.clone()
    gs.gs_dropout(x, onto, onto, 0.2, seed, 1000)
    assert torch.equal(onto, whole)
    inplace = x.clone()
    gs.gs_dropout(inplace, res, inplace, 0.2, seed, 1000)
    assert torch.equal(inplace, whole)
    twice = x.clone()
    gs.gs_dropout(twice, twice, twice, 0.2, seed, 1000)
    ones, back = torch.ones_like(x), torch.empty_like(x)
    gs.gs_dropout(ones, None, back, 0.2, seed, 1000)
    mask, scale = kept(n, 0.2, seed, 1000, 0)
    assert torch.equal(back != 0, mask)
    assert torch.equal(twice, (torch.where(mask, x.float() * scale, 0.0) + x.float()).to(BF16))
    other = torch.empty_like(x)
    gs.gs_dropout(ones, None, other, 0.2, seed + 1, 1000)
    assert not torch.equal(other, back)


def test_dropout_in_a_graph_draws_anew():
    n = 3000
    x, out, step = torch.ones(n, device=DEV), torch.empty(n, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_dropout(x, None, out, 0.5, 11, 0, step)
        step.add_(1)
    step.zero_()
    for s in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out != 0, kept(n, 0.5, 11, 0, s)[0])


def test_dropout_share_that_stays():
    """16 M elements: the share kept is within five deviations of 1 - P, and neighbours' fates do not follow each other."""
    n, p = 1 << 24, 0.1
    out = torch.empty(n, device=DEV)
    gs.gs_dropout(torch.ones(n, device=DEV), None, out, p, 2024)
    k = (out != 0).to(F64)
    keep = 1 - int(p * 65536 + 0.5) / 65536
    assert abs(float(k.mean()) - keep) < 5 * (keep * (1 - keep) / n) ** 0.5
    for lag in (1, 2, 7, 8, 64):
        c = float(((k[lag:] - keep) * (k[:-lag] - keep)).mean()) / (keep * (1 - keep))
        assert abs(c) < 5 / n ** 0.5, lag


def test_dropout_beyond_32_bits_of_offsets():
    n = (1 << 32) + 21
    x = torch.ones(n, dtype=BF16, device=DEV)
    gs.gs_dropout(x, None, x, 0.5, 5, 40)
    tail = torch.ones(1000, dtype=BF16, device=DEV)
    gs.gs_dropout(tail, None, tail, 0.5, 5, 40 + n - 1000)
    assert torch.equal(x[-1000:], tail)


def test_native_and_general_reading_agree():
    x, gamma, beta, y, stats, dy, dx, dgamma, dbeta, ws = run_norm(9, 300, F32, BF16)
    want = [t.clone() for t in (y, stats, dx, dgamma, dbeta)]
    for t in (y, stats, dx, dgamma, dbeta):
        t.fill_(3.0)

    class Stream:
        cuda_stream = torch.cuda.current_stream().cuda_stream

    gs.gs_layer_norm(torch.nn.Parameter(x, requires_grad=False), gamma, beta, y, stats, np.float64(1e-5), stream=Stream())
    gs.gs_layer_norm_grad(dy, x, gamma, stats, dx, dgamma, dbeta, ws.data_ptr(), ws.numel())
    for t, w in zip((y, stats, dx, dgamma, dbeta), want):
        assert torch.equal(t, w)
    a, b = torch.empty_like(x), torch.empty_like(x)
    gs.gs_dropout(x, None, a, 0.5, (1 << 64) - 5, 3)
    gs.gs_dropout(x, None, b, np.float64(0.5), (1 << 64) - 5, 3)
    assert torch.equal(a, b) and bool((a == 0).any())


def test_binding_refuses():
    x = torch.zeros(4, 64, dtype=BF16, device=DEV)
    w = torch.zeros(64, device=DEV)
    for kind, call in ((TypeError, lambda: gs.gs_layer_norm(x, w, w.to(BF16), x)), (ValueError, lambda: gs.gs_layer_norm(x, w[:63], None, x)),
                       (ValueError, lambda: gs.gs_layer_norm(x, None, None, x[:3])), (TypeError, lambda: gs.gs_layer_norm(x, None, None, x.float())),
                       (ValueError, lambda: gs.gs_layer_norm(x.t(), None, None, x.t())), (gs.GsError, lambda: gs.gs_layer_norm(x, None, None, x, eps=-1.0)),
                       (gs.GsError, lambda: gs.gs_layer_norm_grad(x, x, None, torch.zeros(4, 2, device=DEV), x.clone(), w, w.clone())),
                       (ValueError, lambda: gs.gs_dropout(x, None, x[:2], 0.1, 1)), (ValueError, lambda: gs.gs_dropout(x, None, x, 0.1, -1)),
                       (gs.GsError, lambda: gs.gs_dropout(x, None, x, 1.5, 1)), (gs.GsError, lambda: gs.gs_dropout(x, None, x, float("nan"), 1)),
                       (ValueError, lambda: gs.gs_dropout(x.cpu(), None, x, 0.1, 1))):
        with pytest.raises(kind):
            call()
