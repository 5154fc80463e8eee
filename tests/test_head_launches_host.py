"""How the calls of a head without its logits choose, size and place their launches, on the CPU: the launchers are compiled for the host only
against a HIP runtime that records launches and the memory that each reads and writes (hipmock/head_recorder.cpp).  Each launch is one the runtime
accepts, the launches of a call take the vocabulary exactly once, everything in the workspace lies inside it and apart from what is
still to be read there, and the tiles that have rows that count are dealt to all dies."""
from __future__ import annotations

import ctypes
import os
import random
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_17570_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

vp, i64, f32, sz, u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_uint64
A = [(1 << 60) + i * (1 << 54) for i in range(16)]        # far-apart addresses that are never dereferenced
X, W, BIAS, TARGETS, LOGP, STATS, DX, DW, DB, LOSS, WEIGHTS, WS = A[:12]


class Launch(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_char * 256), *[(n, u64) for n in ("grid", "grid_y", "block")],
                *[(n, i64) for n in ("word0", "words", "steps", "splits", "first", "rows", "hidden")], ("rows_workgroups", u64), ("status", ctypes.c_int32), ("pad", ctypes.c_int32)]

    @property
    def name(self):
        return self.kernel.decode()

    def is_a(self, *kernels):
        return re.match(r"\w+", self.name)[0] in kernels

    @property
    def tile(self):
        return [int(x) for x in re.search(r"Tile<(\d+), (\d+)", self.name).groups()]


class Span(ctypes.Structure):
    _fields_ = [("role_", ctypes.c_char * 24), ("lo", u64), ("bytes", u64), ("write", ctypes.c_int32), ("launch", ctypes.c_int32)]

    @property
    def role(self):
        return self.role_.decode()

    @property
    def hi(self):
        return self.lo + self.bytes


class Head(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("x", "w", "bias")] + [(n, i64) for n in ("rows", "hidden", "vocab", "x_stride", "w_stride")]


class Grads(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("dx", "dw", "dbias")] + [(n, i64) for n in ("dx_stride", "dw_stride")]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("head"))
    o, so = os.path.join(out, "head.o"), os.path.join(out, "libhead.so")
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-fuse-cuid=none", "-std=c++17", "-O1", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(ROOT, "tests", "hipmock", "head_recorder.cpp"), "-o", o],
                   check=True, capture_output=True, text=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,defs", "-Wl,-z,muldefs", o, "-o", so], check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(so)
    lib.gs_head_workspace_bytes.argtypes, lib.gs_head_workspace_bytes.restype = [i64, i64, i64, ctypes.c_int], sz
    lib.gs_head_logp_grad_workspace_bytes.argtypes, lib.gs_head_logp_grad_workspace_bytes.restype = [i64, i64, i64], sz
    lib.gs_head_logp.argtypes = [vp, vp, f32, vp, vp, vp, sz, vp]
    lib.gs_head_logp_grad.argtypes = [vp, vp, f32, vp, vp, vp, vp, sz, vp]
    lib.gs_head_cross_entropy.argtypes = [vp, vp, vp, f32, vp, vp, vp, ctypes.c_int, vp, sz, vp]
    return lib


REACHED = set()


class Call:
    """One call's launches, in a workspace of just the size that is asked for."""

    def __init__(self, lib, what, rows, hidden, vocab, parts="dx dw db", w_pad=0, w_shift=0):
        self.rows, self.hidden, self.vocab, self.what = rows, hidden, vocab, what
        h = Head(X, W + w_shift, BIAS, rows, hidden, vocab, hidden, hidden + w_pad)
        g = Grads(*[a if n in parts.split() else None for n, a in (("dx", DX), ("dw", DW), ("db", DB))], hidden, hidden)
        h, g, t = ctypes.byref(h), ctypes.byref(g), f32(1.0)
        self.w = W + w_shift, W + w_shift + 2 * ((vocab - 1) * (hidden + w_pad) + hidden)
        if what == "logp_grad":
            self.bytes = lib.gs_head_logp_grad_workspace_bytes(rows, hidden, vocab)
        else:
            self.bytes = lib.gs_head_workspace_bytes(rows, hidden, vocab, what == "loss")
        call = {"logp": lambda: lib.gs_head_logp(h, TARGETS, t, LOGP, STATS, WS, self.bytes, None),
                "logp_grad": lambda: lib.gs_head_logp_grad(h, TARGETS, t, STATS, LOGP, g, WS, self.bytes, None),
                "evaluation": lambda: lib.gs_head_cross_entropy(h, TARGETS, WEIGHTS, t, LOGP, None, LOSS, 0, WS, self.bytes, None),
                "loss": lambda: lib.gs_head_cross_entropy(h, TARGETS, WEIGHTS, t, LOGP, g, LOSS, 0, WS, self.bytes, None)}[what]
        lib.rec_reset()
        assert call() == 0
        self.launches, self.spans = [Launch() for _ in range(lib.rec_count())], [Span() for _ in range(lib.rec_spans())]
        for i, l in enumerate(self.launches):
            lib.rec_get(i, ctypes.byref(l))
            assert l.status == 0, l.name
            REACHED.add(l.name)
        for i, s in enumerate(self.spans):
            lib.rec_span(i, ctypes.byref(s))

    def of(self, *kernels):
        return [l for l in self.launches if l.is_a(*kernels)]

    def check(self):
        inside = [s for s in self.spans if s.role not in ("dx", "dw", "db", "bias", "w") and not (s.role == "w read" and self.w[0] <= s.lo < self.w[1])]
        for s in inside:
            assert WS <= s.lo and s.hi <= WS + self.bytes, (s.role, self.launches[s.launch].name)
        for s in self.spans:
            if s.role in ("w", "w read") and s not in inside:
                assert self.w[0] <= s.lo and s.hi <= self.w[1], s.role
        # each kind of thing has a place of its own, whose parts are all there is of it
        places = {}
        for s in inside:
            role = {"w read": "w packed", "place": "list", "index": "list", "token": "list", "count": "list"}.get(s.role, s.role)
            lo, hi = places.get(role, (s.lo, s.hi))
            places[role] = min(lo, s.lo), max(hi, s.hi)
        order = sorted((lo, hi, role) for role, (lo, hi) in places.items())
        for a, b in zip(order, order[1:]):
            assert a[1] <= b[0], (a, b)
        # what is read there was written by an earlier launch
        written = {}
        for s in inside:
            if s.write:
                written.setdefault(s.role, s.launch)
            elif s.role in ("z", "dz", "sum", "partials", "row", "x packed"):
                assert written.get(s.role, 1 << 30) < s.launch or self.launches[s.launch].is_a("k_head_dx_dw"), (s.role, self.launches[s.launch].name)
        passes = [self.of(k) for k in ("k_head_stats", "k_head_dw", "k_head_db")] + [self.of("k_head_dz", "k_head_dz_kept"), self.of("k_head_dx", "k_head_dx_dw")]
        for ls in passes:
            assert not ls or sum(l.words for l in ls) == self.vocab
            at = 0
            for l in ls:
                if l.is_a("k_head_stats", "k_head_dz", "k_head_dz_kept", "k_head_dw"):
                    assert l.word0 == at
                at += l.words
        for ls in (self.of("k_head_dx", "k_head_dx_dw"),):
            assert [bool(l.first) for l in ls] == [i == 0 for i in range(len(ls))]
        return self


SIZES = [(0, 64, 100), (1, 1, 1), (1, 4096, 131_072), (4, 8192, 32_000), (5, 100, 700), (16, 2048, 50_304), (17, 512, 300), (64, 4096, 32_000), (64, 4096, 16_000), (65, 1000, 9_001),
         (128, 4096, 50_304), (300, 8192, 10_000), (1000, 2048, 32_000), (1354, 320, 39_296), (4095, 2048, 50_001), (8192, 64, 40_000), (8192, 4096, 131_072), (20_000, 72, 9_000),
         (1 << 20, 8, 257), (3, 64, 300_000), (5, 8, 4_400_000), (2, 8200, 1 << 20), (1, 64, 1 << 30), (1, 1 << 17, 5)]


@pytest.mark.parametrize("what", ["logp", "logp_grad", "evaluation", "loss"])
@pytest.mark.parametrize("rows, hidden, vocab", SIZES)
def test_launches_lie_in_the_workspace(lib, what, rows, hidden, vocab):
    if what == "logp" and rows == 0:
        return
    for w_pad, w_shift in ((0, 0), (3, 0), (8, 2)):
        Call(lib, what, rows, hidden, vocab, w_pad=w_pad, w_shift=w_shift).check()


def test_launches_of_drawn_sizes(lib):
    rng = random.Random(3)
    for _ in range(400):
        rows, hidden, vocab = int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 13.5)), int(2 ** rng.uniform(0, 19))
        if rng.random() < 0.5:
            hidden = -(-hidden // 64) * 64
        what, parts = rng.choice(["logp", "logp_grad", "evaluation", "loss"]), rng.choice(["dx dw db", "dx dw", "dx", "dw", "db", "dw db", ""])
        Call(lib, what, rows, hidden, vocab, parts, rng.choice([0, 0, 8, 1]), rng.choice([0, 0, 16, 2])).check()


def test_every_kernel_is_reached(lib):
    for rows, hidden, vocab in SIZES[1:] + [(r, h, 700) for r in (1, 4) for h in (504, 512, 1024, 2048, 4096, 8192)] + [(40, 64, 700), (200, 64, 700), (200, 1000, 700)]:
        for what in ("logp", "loss", "logp_grad"):
            for parts in ("dx dw db", "dx"):
                for w_pad in (0, 3):
                    Call(lib, what, rows, hidden, vocab, parts, w_pad=w_pad)
    buffer = ctypes.create_string_buffer(1 << 16)
    lib.rec_kernels(buffer, len(buffer))
    assert {n for n in buffer.value.decode().split("\n") if n.startswith("k_")} - REACHED <= {n for n in buffer.value.decode().split("\n") if "<false>" in n and ("gather" in n or "pack" in n)}


@pytest.mark.parametrize("rows, hidden, vocab", SIZES + [(1024, 4096, 131_072), (1024, 512, 131_072), (1024, 448, 131_072), (1025, 512, 131_072), (2, 512, 1 << 21)])
def test_a_gradient_asks_for_no_memory_that_only_a_loss_uses(lib, rows, hidden, vocab):
    """A loss keeps z, in 32 bits, of up to 2^27 values and of states that are wide enough; gs_head_logp_grad never does, and all that it asks for is
    read or written where weights have to be packed, but for alignment and for the rest of a tile of 256 packed words."""
    padded, words = max(64, -(-rows // 64) * 64), -(-vocab // 256) * 256
    more = lib.gs_head_workspace_bytes(rows, hidden, vocab, 1) - lib.gs_head_logp_grad_workspace_bytes(rows, hidden, vocab)
    kept = any(s.role == "z" for s in Call(lib, "loss", rows, hidden, vocab).spans)
    assert kept == (more > 0) and more <= 1 << 29
    if kept:
        assert padded * words * 4 <= more and hidden > 448
    assert lib.gs_head_workspace_bytes(rows, hidden, vocab, 0) <= lib.gs_head_logp_grad_workspace_bytes(rows, hidden, vocab)
    c = Call(lib, "logp_grad", rows, hidden, vocab, w_shift=2)
    used = max(s.hi for s in c.spans if WS <= s.lo < WS + (1 << 50)) - WS
    assert c.bytes - used < 256 + 255 * 2 * -(-hidden // 64) * 64 and not any(s.role == "z" for s in c.spans)


def test_sizes_and_workspaces_that_are_refused(lib):
    size = lib.gs_head_logp_grad_workspace_bytes
    assert size(-1, 64, 64) == size((1 << 20) + 1, 64, 64) == size(1, 0, 64) == size(1, (1 << 17) + 1, 64) == size(1, 64, 0) == size(1, 64, (1 << 30) + 1) == 0
    rows, hidden, vocab = 1000, 2048, 32_000                # a loss would keep z
    h, g = Head(X, W, BIAS, rows, hidden, vocab, hidden, hidden), Grads(DX, DW, DB, hidden, hidden)
    lib.rec_reset()
    for ws, n in ((WS, size(rows, hidden, vocab) - 1), (WS + 8, 1 << 40), (None, 1 << 40)):
        assert lib.gs_head_logp_grad(ctypes.byref(h), TARGETS, 1.0, STATS, LOGP, ctypes.byref(g), ws, n, None) == -2
    assert lib.gs_head_cross_entropy(ctypes.byref(h), TARGETS, WEIGHTS, 1.0, LOGP, ctypes.byref(g), LOSS, 0, WS, size(rows, hidden, vocab), None) == -2
    assert lib.rec_count() == 0


@pytest.mark.parametrize("rows, hidden, vocab, pieces", [(40, 1000, 16_384, 1), (40, 1000, 200_000, 4), (300, 5000, 30_000, 3), (3000, 520, 40_000, 1)])
def test_weights_are_packed_where_they_are_read(lib, rows, hidden, vocab, pieces):
    """A loss that kept z reads the weights for the hidden states' gradient only; packed as one piece they are there from the forward pass."""
    def packed(what, parts):
        c = Call(lib, what, rows, hidden, vocab, parts, w_pad=3).check()
        return sum(s.role == "w packed" and s.write for s in c.spans), sum(l.is_a("k_head_dw") for l in c.launches)

    assert packed("evaluation", "")[0] == pieces
    for parts in ("dw", "db", "dw db", ""):
        assert packed("loss", parts) == (pieces, "dw" in parts)
    assert packed("loss", "dx dw db")[0] == packed("loss", "dx")[0] == (1 if pieces == 1 else 2 * pieces)
    assert packed("logp_grad", "dw")[0] == pieces


# ---- tiles and dies -------------------------------------------------------------------------------------------------------

def dies_work(lib, tile, of_rows, workgroups, across, rows, count):
    """Tiles of each of the 8 dies, to which a launch's workgroups go in turn; each tile that has a row that counts is taken exactly once."""
    a, b, seen, dies = ctypes.c_uint32(), ctypes.c_uint32(), set(), [0] * 8
    for i in range(workgroups):
        there = lib.rec_tile(*tile, int(of_rows), ctypes.c_uint32(i), i64(across), i64(rows), count, ctypes.byref(a), ctypes.byref(b))
        assert there >= 0
        if there:
            row, other = (a.value, b.value) if of_rows else (b.value, a.value)
            assert row * tile[1] < count and other * tile[0] < across
            assert (row, other) not in seen
            seen.add((row, other))
            dies[i % 8] += 1
    assert len(seen) == -(-count // tile[1]) * -(-across // tile[0])
    return dies


@pytest.mark.parametrize("rows, hidden, vocab", [(8192, 4096, 131_072), (8192, 2048, 4_000), (4095, 2048, 50_001), (1000, 640, 20_000), (128, 4096, 50_304), (64, 4096, 16_000), (1354, 320, 39_296)])
def test_rows_that_count_are_dealt_to_all_dies(lib, rows, hidden, vocab):
    """Rows that count lie in front of those that do not: of whatever part of a batch counts, no die has more than its share of tiles (rounded up)."""
    c = Call(lib, "loss", rows, hidden, vocab)
    kinds = {}
    for l in c.of("k_head_stats", "k_head_dz"):
        kinds[l.name] = l.tile, False, l.grid, l.words, l.rows
    for l in c.of("k_head_dx", "k_head_dx_dw"):
        kinds[l.name] = l.tile, True, l.rows_workgroups, l.hidden, l.rows
    assert len(kinds) >= 2
    for tile, of_rows, workgroups, across, packed in kinds.values():
        for count in {0, 1, rows // 8, rows // 4, rows // 3, rows // 2, 3 * rows // 4, rows - 1, rows}:
            dies = dies_work(lib, tile, of_rows, workgroups, across, packed, count)
            assert max(dies) <= -(-sum(dies) // 8), (tile, of_rows, count, dies)
