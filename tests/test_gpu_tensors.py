"""GPU tests of norm and clip over many tensors: against sums in 64 bits and the clip's definition, for lists of any
length, tensors of any size and alignment, in place and into other buffers."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV, gs

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def workspace():
    return torch.full((gs.gs_sqnorm_workspace_bytes(),), 0xFF, dtype=torch.uint8, device=DEV)


def make(sizes, kinds, seed=0, lead=0, sigma=0.02):
    """Tensors of these sizes back to back in one buffer of each type, the first `lead` elements behind a 512-byte boundary."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    total = {k: lead + sum(n for n, q in zip(sizes, kinds) if q == k) for k in (BF16, F32)}
    flat = {k: (torch.randn(n + 64, generator=g, device=DEV) * sigma).to(k) for k, n in total.items()}
    at, out = {k: lead for k in flat}, []
    for n, k in zip(sizes, kinds):
        out.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    return flat, out


def want_sqnorm(tensors):
    return sum(float(t.double().square().sum()) for t in tensors)


def sqnorm(tensors, **kw):
    sq = torch.full((1,), float("nan"), dtype=torch.float64, device=DEV)
    gs.gs_grads_sqnorm(tensors, sq, workspace(), **kw)
    return sq


def want_clip(t, S, max_norm):
    """c g, each product rounded once to fp32 and, in bf16, once more: the same operations in torch."""
    norm = np.float32(math.sqrt(S))
    c = np.float32(max_norm) / (norm + np.float32(1e-6))
    c = float(c) if c < 1 else 1.0
    return (t.float() * c).to(t.dtype)


def same_bits(a, b):
    view = torch.int16 if a.dtype == BF16 else torch.int32
    return torch.equal(a.view(view), b.view(view))


LISTS = {
    "one element": [1],
    "nothing and little": [0, 3, 0, 0, 1, 7, 0],
    "one": [100_003],
    "a layer": [64, 64, 64 * 192, 192, 64 * 64, 64, 64, 64, 64 * 256, 256, 256 * 64, 64],
    "lengths around a vector": list(range(1, 40)),
    "around a tile": [2047, 2048, 2049, 8191, 8192, 8193, 16383, 16384, 16385, 16391, 32768, 65537],
    "a short table": [33] * 16,
    "and one more": [33] * 17,
    "a full table": [33] * 128,
    "and one more again": [33] * 129,
    "many": [(i * 37) % 301 for i in range(1000)],
    "one long among short": [5] * 64 + [3_000_001] + [6] * 64,
    "long": [40_000_003, 11],
}


def kinds_of(sizes, kind):
    return [kind] * len(sizes) if kind != "mixed" else [F32 if i % 3 == 0 else BF16 for i in range(len(sizes))]


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("kind", [BF16, F32, "mixed"])
@pytest.mark.parametrize("lead", [0, 1, 5])
def test_norm_and_clip(name, kind, lead):
    sizes = LISTS[name]
    flat, tensors = make(sizes, kinds_of(sizes, kind), lead=lead)
    before = {k: v.clone() for k, v in flat.items()}
    S = want_sqnorm(tensors)
    sq = sqnorm(tensors)
    # fp64 sums of exact squares: n roundings of 2^-53 at worst
    assert abs(float(sq) - S) <= 1e-15 * (1 + sum(sizes) ** 0.5) * S
    S = float(sq)
    max_norm = 0.3 * math.sqrt(S)
    want = [want_clip(t, S, max_norm) for t in tensors]
    norm = torch.full((1,), float("nan"), dtype=F32, device=DEV)
    # into buffers of the same and of another alignment
    for shift in (lead, lead + 1, 0):
        outs, into = make(sizes, kinds_of(sizes, kind), seed=9, lead=shift)
        kept = {k: v.clone() for k, v in outs.items()}
        gs.gs_grads_clip(tensors, sq, max_norm, norm, outs=into)
        assert float(norm) == np.float32(math.sqrt(S))
        assert all(same_bits(a, b) for a, b in zip(into, want))
        assert all(torch.equal(flat[k], before[k]) for k in flat)
        for k, t in outs.items():
            n = shift + sum(a for a, q in zip(sizes, kinds_of(sizes, kind)) if q == k)
            assert torch.equal(t[:shift], kept[k][:shift]) and torch.equal(t[n:], kept[k][n:])
    gs.gs_grads_clip(tensors, sq, max_norm)
    assert all(same_bits(a, b) for a, b in zip(tensors, want))
    for k, t in flat.items():
        n = lead + sum(a for a, q in zip(sizes, kinds_of(sizes, kind)) if q == k)
        assert torch.equal(t[:lead], before[k][:lead]) and torch.equal(t[n:], before[k][n:])


def test_norm_accumulates_and_equals_the_flat_norms():
    sizes = [1000, 77, 40_001, 8]
    _, tensors = make(sizes, [BF16] * 4)
    sq = sqnorm(tensors)
    parts = torch.zeros(1, dtype=torch.float64, device=DEV)
    for i, t in enumerate(tensors):
        gs.gs_grads_sqnorm([t], parts, workspace(), accumulate=i > 0)
    assert float(parts) == pytest.approx(float(sq), rel=1e-14)
    flat = torch.cat([torch.nn.functional.pad(t, (0, -t.numel() % 8)) for t in tensors])
    ref = torch.zeros(1, dtype=torch.float64, device=DEV)
    gs.gs_grad_sqnorm([flat], 0, flat.numel(), ref, workspace())
    assert float(ref) == pytest.approx(float(sq), rel=1e-14)
    gs.gs_grads_sqnorm([], parts, workspace(), accumulate=True)
    assert float(parts) == pytest.approx(float(sq), rel=1e-14)
    gs.gs_grads_sqnorm([], parts, workspace())
    assert float(parts) == 0.0


@pytest.mark.parametrize("count", [1, 2, 63, 64, 65, 128, 129, 255, 256, 257])
def test_norm_of_any_number_of_workgroups(count):
    """One tensor a workgroup: up to 256 of them finish by themselves, in one launch or two; more take another launch."""
    _, tensors = make([50] * count, [F32] * count, seed=count)
    S = want_sqnorm(tensors)
    for _ in range(3):
        assert float(sqnorm(tensors)) == pytest.approx(S, rel=1e-14)
    sq = torch.full((1,), 5.0, dtype=torch.float64, device=DEV)
    for i in range(3):
        gs.gs_grads_sqnorm(tensors, sq, workspace(), accumulate=True)
        assert float(sq) == pytest.approx(5.0 + (i + 1) * S, rel=1e-14)


def test_a_graph_of_small_norms():
    _, tensors = make([70_001], [BF16], lead=1)
    ws, sq = workspace(), torch.zeros(1, dtype=torch.float64, device=DEV)
    gs.gs_grads_sqnorm(tensors, sq, ws)
    want = float(sq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_grads_sqnorm(tensors, sq, ws)
        gs.gs_grads_sqnorm(tensors, sq, ws, accumulate=True)
    for i in range(5):
        sq.fill_(-1.0)
        if i == 3:
            tensors[0].mul_(2.0)
            want *= 4.0
        graph.replay()
        torch.cuda.synchronize()
        assert float(sq) == 2 * want
        gs.gs_grads_sqnorm(tensors, sq, ws)
        assert float(sq) == want


def test_nothing_to_clip_still_gives_the_norm():
    sq = torch.full((1,), 9.0, dtype=torch.float64, device=DEV)
    norm = torch.zeros(1, dtype=F32, device=DEV)
    gs.gs_grads_clip([], sq, 1.0, norm)
    assert float(norm) == 3.0
    gs.gs_grads_clip([torch.empty(0, device=DEV)], sq, 1.0, norm.zero_())
    assert float(norm) == 3.0
    gs.gs_grads_clip([], sq, 1.0)


@pytest.mark.parametrize("S", [0.25, 0.0, float("nan"), float("inf")])
def test_coefficient_at_its_ends(S):
    """No clipping below the bound and for a NaN norm; 0 for an infinite one, which is NaN where a gradient is infinite."""
    sizes = [1000, 33]
    _, tensors = make(sizes, [BF16, F32], seed=2)
    tensors[0][5], tensors[1][6], tensors[0][7] = float("inf"), float("-inf"), float("nan")
    sq = torch.full((1,), S, dtype=torch.float64, device=DEV)
    _, into = make(sizes, [BF16, F32], seed=3)
    want = [t.clone() if S != float("inf") else t * 0.0 for t in tensors]
    gs.gs_grads_clip(tensors, sq, 1.0, outs=into)
    for a, b in zip(into, want):
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0))
    bits = [t.view(torch.int16 if t.dtype == BF16 else torch.int32).clone() for t in tensors]
    gs.gs_grads_clip(tensors, sq, 1.0)
    for a, b, q in zip(tensors, want, bits):
        if S != float("inf"):
            assert torch.equal(a.view(q.dtype), q)                  # not a bit
        else:
            assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0))


def test_non_finite_gradients_reach_the_norm():
    for bad, test in ((float("nan"), math.isnan), (float("inf"), lambda v: v == math.inf)):
        for at in (0, 3, 999, 1000 + 32):
            flat, tensors = make([1000, 33], [F32, F32], seed=2)
            flat[F32][at] = bad
            assert test(float(sqnorm(tensors)))


def test_mixed_in_place_and_elsewhere():
    sizes = [500, 600, 700]
    _, tensors = make(sizes, [BF16, F32, BF16], seed=4)
    _, into = make(sizes, [BF16, F32, BF16], seed=5)
    sq = sqnorm(tensors)
    want = [want_clip(t, float(sq), 0.1) for t in tensors]
    untouched = [t.clone() for t in tensors]
    gs.gs_grads_clip(tensors, sq, 0.1, outs=[None, into[1], tensors[2]])
    assert same_bits(tensors[0], want[0]) and same_bits(into[1], want[1]) and same_bits(tensors[2], want[2])
    assert same_bits(tensors[1], untouched[1])


def test_same_bits_on_another_stream_and_from_a_graph():
    sizes = [5] * 130 + [1_000_003]
    _, tensors = make(sizes, kinds_of(sizes, "mixed"), lead=3)
    _, into = make(sizes, kinds_of(sizes, "mixed"), seed=6, lead=3)
    ws, sq, norm = workspace(), torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1, dtype=F32, device=DEV)

    def run(stream=None):
        gs.gs_grads_sqnorm(tensors, sq, ws, stream=stream)
        gs.gs_grads_clip(tensors, sq, 0.5, norm, outs=into, stream=stream)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in [sq, norm, *into]]

    def same():
        torch.cuda.synchronize()
        for a, b in zip([sq, norm, *into], want):
            assert torch.equal(a, b)
            a.fill_(2.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(side)
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        graph.replay()
        same()
        torch.randn(1000, device=DEV).sum().item()


def test_more_elements_than_32_bits_count():
    n = (1 << 32) + 12_345
    t = torch.zeros(n, dtype=BF16, device=DEV)
    at = [0, 1, (1 << 31) - 1, 1 << 31, (1 << 32) - 1, 1 << 32, n - 1]
    t[at] = 3.0
    sq = sqnorm([t[1:], t[:1]])
    assert float(sq) == 9.0 * len(at)
    gs.gs_grads_clip([t[1:], t[:1]], sq, 0.5 * math.sqrt(9.0 * len(at)))
    c = want_clip(torch.tensor([3.0], dtype=BF16), float(sq), 0.5 * math.sqrt(9.0 * len(at)))
    assert t[at].tolist() == c.tolist() * len(at) and int((t != 0).sum()) == len(at)


def test_many_tensors_share_the_workspace():
    """More tensors than a launch takes and more tiles than the workspace holds at the usual size of a tile."""
    n = 65_536
    flat = torch.ones(n * 2, dtype=F32, device=DEV)
    tensors = [flat[2 * i:2 * i + 2] for i in range(n)]
    assert float(sqnorm(tensors)) == 2.0 * n
    with pytest.raises(gs.GsError):
        sqnorm(tensors + [flat[:1]])


def test_native_and_general_reading_agree(monkeypatch):
    sizes = [10, 20_000, 0, 31]
    _, tensors = make(sizes, kinds_of(sizes, "mixed"))
    _, into = make(sizes, kinds_of(sizes, "mixed"), seed=7)
    got, taken = [], []

    class Counting:
        def __init__(self, call):
            self.call = call

        def __getattr__(self, name):
            def f(*a):
                st = getattr(self.call, name)(*a)
                taken.append((name, st))
                return st
            return f

    class General:
        def __getattr__(self, name):
            return lambda *a: None

    for call in (Counting(gs._call), General()):
        with monkeypatch.context() as mp:
            mp.setattr(gs, "_call", call)
            sq = sqnorm(tensors)
            norm = torch.zeros(1, dtype=F32, device=DEV)
            gs.gs_grads_clip(tensors, sq, 0.5, norm, outs=into)
            got.append([t.clone() for t in [sq, norm, *into]])
    assert taken == [("grads_sqnorm", 0), ("grads_clip", 0)]
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_wrong_tensors_are_refused():
    sq, ws = torch.zeros(1, dtype=torch.float64, device=DEV), workspace()
    t = torch.zeros(100, device=DEV)
    with pytest.raises(TypeError):
        gs.gs_grads_sqnorm(t, sq, ws)
    with pytest.raises(TypeError):
        gs.gs_grads_sqnorm([t.half()], sq, ws)
    with pytest.raises(ValueError):
        gs.gs_grads_sqnorm([t.cpu()], sq, ws)
    with pytest.raises(ValueError):
        gs.gs_grads_sqnorm([t[::2]], sq, ws)
    with pytest.raises(TypeError):
        gs.gs_grads_sqnorm([t], sq.float(), ws)
    with pytest.raises(gs.GsError):
        gs.gs_grads_sqnorm([t], sq, ws[:1000])
    for outs in ([t[:99]], [t.bfloat16()], [t, t]):
        with pytest.raises((TypeError, ValueError)):
            gs.gs_grads_clip([t], sq, 1.0, outs=outs)
    u = torch.zeros(1000, device=DEV)
    for tensors, outs in (([t, t], None), ([u[:100]], [u[50:150]]), ([u[:100], u[200:300]], [u[300:400], u[350:450]]),
                          ([u[:100], u[100:200]], [u[100:200], u[:100]]), ([u[:600]] + [u[600 + i:601 + i] for i in range(40)], [None] + [u[599:600]] + [None] * 39)):
        with pytest.raises(gs.GsError):
            gs.gs_grads_clip(tensors, sq, 1.0, outs=outs)
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(gs.GsError):
            gs.gs_grads_clip([t], sq, bad)
    gs.gs_grads_clip([u[:100], u[100:200]], sq, 1.0, outs=[u[200:300], u[300:400]])        # side by side is fine
    assert ctypes.sizeof(gs.gs_tensor) == 32


@pytest.mark.parametrize("count", [15, 16, 17, 159, 160, 161, 239, 240, 241, 320, 321, 480, 481])
def test_lists_at_the_lines_between_launches(count):
    """Norm and clip of lists as long as a launch takes, and one tensor longer, with empty tensors among them; all in place, all elsewhere,
    and one of many elsewhere."""
    sizes = [(i * 29) % 77 + 1 for i in range(count)]
    sizes = [n for i, n in enumerate(sizes) for n in ([n, 0] if i % 50 == 7 else [n])]
    kinds = kinds_of(sizes, "mixed")
    _, tensors = make(sizes, kinds, seed=count, lead=1)
    S = want_sqnorm(tensors)
    sq = sqnorm(tensors)
    assert float(sq) == pytest.approx(S, rel=1e-14)
    max_norm = 0.3 * math.sqrt(S)
    want = [want_clip(t, float(sq), max_norm) for t in tensors]
    _, into = make(sizes, kinds, seed=9, lead=1)
    gs.gs_grads_clip(tensors, sq, max_norm, outs=into)
    assert all(same_bits(a, b) for a, b in zip(into, want))
    copies = [t.clone() for t in tensors]
    gs.gs_grads_clip(copies, sq, max_norm)
    assert all(same_bits(a, b) for a, b in zip(copies, want))
    into[3].fill_(7.0)
    gs.gs_grads_clip(tensors, sq, max_norm, outs=[into[3] if i == 3 else None for i in range(len(tensors))])
    assert all(same_bits(into[3] if i == 3 else t, want[i]) for i, t in enumerate(tensors))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tensors_longer_than_a_piece(dtype):
    """More than 2^31 elements, from an odd one on: the norm is its parts', the clip that of short tensors over the same elements."""
    n = 2 ** 31 + 12_345
    flat = torch.full((n + 64,), 2.0 ** -10, dtype=dtype, device=DEV)
    ends = [3, 4, 2 ** 31 + 2, 2 ** 31 + 3, 2 ** 31 + 4, n + 2]
    flat[torch.tensor(ends, device=DEV)] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0], device=DEV).to(dtype)
    flat[2], flat[n + 3] = 9.0, 9.0
    t = flat[3:n + 3]
    S = (n - 6) * 2.0 ** -20 + 1 + 4 + 9 + 16 + 25 + 36
    sq = sqnorm([t])
    assert float(sq) == pytest.approx(S, rel=1e-12)
    gs.gs_grads_clip([t], sq, 0.25 * math.sqrt(S))
    want = want_clip(torch.tensor([2.0 ** -10, 1.0, 2.0, 3.0, 4.0, 5.0, 6.0], device=DEV).to(dtype), float(sq), 0.25 * math.sqrt(S))
    assert same_bits(flat[torch.tensor(ends, device=DEV)], want[1:]) and float(flat[2]) == float(flat[n + 3]) == 9.0
    flat[torch.tensor(ends, device=DEV)] = want[0].to(dtype)
    for a in range(3, n + 3, 1 << 28):
        assert bool((flat[a:min(a + (1 << 28), n + 3)] == want[0]).all())
