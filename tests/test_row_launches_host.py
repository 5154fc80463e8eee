"""Every rule by which the losses and the norm and clip over many tensors choose and size their launches, on the CPU: the launchers are
compiled for the host only against a HIP runtime that records launches (hipmock/row_recorder.cpp).  Each launch is one the runtime
accepts, the launches of a call take its rows, pairs and tensors exactly once, a kernel that holds a row has room for it, and what is left
in the workspace lies inside it, apart from what is still to be read there."""
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

vp, i64, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float
BF16, F32 = 0, 1
SIZE = {BF16: 2, F32: 4}
PARTIALS, SLICES = 262_144, 128
WS_BYTES = 8 * (PARTIALS + SLICES)
A = [(1 << 60) + i * (1 << 54) for i in range(16)]        # far-apart addresses that are never dereferenced
WS = A[15]


class Launch(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_char * 512), *[(n, ctypes.c_uint64) for n in ("grid", "block")],
                *[(n, i64) for n in ("row0", "rows", "parts", "len", "runs", "count")], ("partials", ctypes.c_uint64), ("slots", ctypes.c_uint64),
                ("slot0", i64), ("meet", i64), ("tag", ctypes.c_uint64), *[(n, i64) for n in ("words", "tiles", "tile_runs", "nv", "keep_tile")],
                ("out", ctypes.c_uint64), *[(n, ctypes.c_int32) for n in ("accumulate", "ends", "status")]]

    @property
    def name(self):
        return self.kernel.decode()

    def is_a(self, kernel):
        return re.match(r"[\w]+", self.name)[0] == kernel

    @property
    def targs(self):
        return [x.strip() for x in self.name[self.name.index("<") + 1:-1].split(",")]


class Tensor(ctypes.Structure):
    _fields_ = [("launch", ctypes.c_int32), *[(n, ctypes.c_uint64) for n in ("inp", "out", "numel")], ("dtype", ctypes.c_int32), ("first", ctypes.c_uint32)]


class Logits(ctypes.Structure):
    _fields_ = [("data", vp), ("rows", i64), ("vocab", i64), ("stride", i64), ("dtype", ctypes.c_int32)]


class GsTensor(ctypes.Structure):
    _fields_ = [("data", vp), ("out", vp), ("numel", i64), ("dtype", ctypes.c_int32)]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rows"))
    o, so = os.path.join(out, "rows.o"), os.path.join(out, "librows.so")
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-fuse-cuid=none", "-std=c++17", "-O1", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(ROOT, "tests", "hipmock", "row_recorder.cpp"), "-o", o],
                   check=True, capture_output=True, text=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,defs", "-Wl,-z,muldefs", o, "-o", so], check=True, capture_output=True, text=True)
    return ctypes.CDLL(so)


REACHED = set()


def launches(lib, call):
    lib.rec_reset()
    assert call() == 0
    out = []
    for i in range(lib.rec_count()):
        l = Launch()
        lib.rec_get(i, ctypes.byref(l))
        assert l.status == 0, (l.name, l.grid, l.block)
        REACHED.add(l.name)
        out.append(l)
    return out


def in_workspace(lo, words):
    assert WS <= lo and lo + 8 * words <= WS + WS_BYTES


def apart(a, b):
    assert a[1] <= b[0] or b[1] <= a[0]


class Batch:
    def __init__(self, rows, vocab, dtype, offset=0, gap=0):
        self.rows, self.vocab, self.dtype = rows, vocab, dtype
        self.x = Logits(A[0] + offset * SIZE[dtype], rows, vocab, vocab + gap, dtype)
        self.per = 16 // SIZE[dtype]

    def cuts(self):
        """(vectors of a row's first line that are not its own, vectors): of every way in which its rows lie."""
        for r in range(min(self.rows, 128 // SIZE[self.dtype])):
            a = self.x.data + r * self.x.stride * SIZE[self.dtype]
            head = min(self.vocab, (-a % 16) // SIZE[self.dtype])
            yield (a + head * SIZE[self.dtype]) // 16 % 8, (self.vocab - head) // self.per

    def check_held(self, l):
        """The row fits the workgroup's registers, and what it loads without asking lies in every row."""
        e, block, nv, lo, keep, policy = l.targs
        block, nv, lo = int(block), int(nv), int(lo)
        assert e == ("gs::Bf16" if self.dtype == BF16 else "gs::F32") and l.block == block
        for skip, vecs in self.cuts():
            assert skip + vecs <= block * nv and block * lo <= skip + vecs, (l.name, self.vocab, skip, vecs)


def tile(rows, ls):
    """The launches take the rows one after another."""
    at = 0
    for l in ls:
        assert l.row0 == at and l.rows > 0
        at += l.rows
    assert at == rows


def check_sums(ls, rows, words, out, accumulate):
    l, = ls
    assert l.count == rows and l.out == out and l.accumulate == accumulate and l.meet == l.grid <= 128 and l.words == words
    in_workspace(l.slots, l.meet * l.words)


def token_logp(lib, b, stats):
    return launches(lib, lambda: lib.gs_token_logp(ctypes.byref(b.x), vp(A[2]), f32(1.0), vp(A[3]), vp(A[4] if stats else 0), vp(WS), ctypes.c_size_t(WS_BYTES), None))


def token_logp_grad(lib, b, in_place=False):
    out, stride = (b.x.data, b.x.stride) if in_place else (A[5], b.vocab)
    return launches(lib, lambda: lib.gs_token_logp_grad(ctypes.byref(b.x), vp(A[2]), f32(1.0), vp(A[4]), vp(A[3]), vp(out), i64(stride), None))


def policy_loss(lib, b, gradient, accumulate):
    hp = (f32 * 4)(1.0, 0.2, 0.2, 0.1)
    return launches(lib, lambda: lib.gs_policy_loss(ctypes.byref(b.x), vp(A[2]), hp, vp(A[6]), vp(A[7]), vp(A[8]), vp(A[9]), vp(A[3]),
                                                    vp(A[5] if gradient else 0), i64(b.vocab), vp(A[10]), accumulate, vp(WS), ctypes.c_size_t(WS_BYTES), None))


def check_scored(b, ls):
    tile(b.rows, ls)
    for l in ls:
        if l.is_a("k_held"):
            assert l.targs[5] == "false" and l.meet == 0
            b.check_held(l)
        else:
            assert l.is_a("k_part") and l.targs[1] == "true" and l.meet == l.parts <= 64
            in_workspace(l.slots, l.rows * l.parts * l.words)


def check_policy(b, ls, gradient, accumulate):
    held = [l for l in ls if l.is_a("k_held")]
    sums = [l for l in ls if l.is_a("k_policy_sums")]
    meeting = []
    if held:
        tile(b.rows, held)
        for l in held:
            assert l.targs[5] == "true"
            b.check_held(l)
        meeting = held
        rest = ls[len(held):]
    else:
        rest, at = ls, 0
        while rest and rest[0].is_a("k_part"):
            part = rest[0]
            assert part.row0 == at and part.targs[1] == "false" and part.partials == WS and part.parts <= 64
            in_workspace(part.partials, part.rows * (part.parts + 1))
            used = WS, WS + 8 * part.rows * (part.parts + 1)
            n = 1
            while at < part.row0 + part.rows:
                l = rest[n]
                assert l.row0 == at and l.rows > 0 and l.parts == part.parts
                assert l.partials == WS + 8 * (at - part.row0) * (l.parts + 1)
                if gradient:
                    assert l.is_a("k_grad") and l.targs[1] == "true" and l.grid == l.rows * l.runs
                    assert l.runs * 512 >= b.vocab // b.per + 7
                    meeting.append(l)
                    if l.meet:
                        apart(used, (l.slots, l.slots + 8 * l.meet * l.words))
                else:
                    assert l.is_a("k_join")
                at += l.rows
                n += 1
            assert at == part.row0 + part.rows
            rest = rest[n:]
        assert at == b.rows
    assert rest == sums
    if sums:
        assert all(l.meet == 0 for l in meeting)
        check_sums(sums, b.rows, 8, A[10], accumulate)
    else:
        assert meeting and all(l.meet == b.rows <= 128 and l.words == 5 for l in meeting)
        in_workspace(meeting[0].slots, b.rows * 5)


def check_grad(b, ls):
    tile(b.rows, ls[::-1])
    for l in ls:
        assert l.is_a("k_grad") and l.targs[1] == "false" and l.grid == l.rows * l.runs and l.meet == 0 and l.runs * 512 >= b.vocab // b.per + 7


def check_batch(lib, b, accumulate=0):
    for stats in (False, True):
        check_scored(b, token_logp(lib, b, stats))
    for gradient in (False, True):
        check_policy(b, policy_loss(lib, b, gradient, accumulate), gradient, accumulate)
    for in_place in (False, True):
        check_grad(b, token_logp_grad(lib, b, in_place))


HELD_LINES = [256, 512, 1024, 2048, 3072, 4096, 6144, 8192, 12288, 16384, 20480, 24576]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_vocabularies_at_the_lines_between_kernels(lib, dtype):
    per = 16 // SIZE[dtype]
    for vecs in HELD_LINES:
        for d in (-8 * per, -7 * per - 1, -7 * per, -7 * per + 1, -6 * per, -1, 0, 1, per - 1, per, per + 1, 8 * per):
            for offset, gap in ((0, 0), (0, 64), (1, 0), (3, 5), (per, 1), (128 // SIZE[dtype] - 1, 7)):
                for rows in (1, 2, 65, 129, 300):
                    check_batch(lib, Batch(rows, vecs * per + d, dtype, offset, gap))


# (type, vocabulary, rows, rows in parts faster) where one is ahead by 5 % and more
SCORED = [(F32, 20_480, 1, 0), (F32, 20_480, 32, 0), (F32, 24_576, 16, 0), (F32, 32_768, 16, 1), (F32, 65_536, 64, 1), (F32, 57_344, 128, 1), (F32, 57_344, 192, 0),
          (F32, 81_920, 96, 1), (F32, 81_920, 256, 0), (BF16, 40_960, 24, 1), (BF16, 40_960, 128, 0), (BF16, 81_920, 96, 1), (BF16, 114_688, 192, 0),
          (BF16, 131_072, 128, 1), (BF16, 163_840, 256, 0), (BF16, 16_000, 1, 0)]
POLICY = [(F32, 20_480, 1, 0), (F32, 32_768, 1, 0), (F32, 32_768, 16, 0), (F32, 49_152, 4, 1), (F32, 49_152, 48, 0), (F32, 65_536, 32, 1), (F32, 65_536, 64, 0),
          (F32, 98_000, 32, 1), (F32, 98_000, 64, 0), (BF16, 40_960, 4, 0), (BF16, 57_344, 16, 1), (BF16, 57_344, 64, 0), (BF16, 131_072, 48, 1),
          (BF16, 131_072, 96, 0), (BF16, 180_000, 64, 1)]


def test_rows_go_in_parts_where_that_is_faster(lib):
    for dtype, vocab, rows, parts in SCORED:
        assert token_logp(lib, Batch(rows, vocab, dtype), False)[0].is_a("k_part" if parts else "k_held"), (dtype, vocab, rows)
    for dtype, vocab, rows, parts in POLICY:
        assert policy_loss(lib, Batch(rows, vocab, dtype), True, 0)[0].is_a("k_part" if parts else "k_held"), (dtype, vocab, rows)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_numbers_of_rows_at_their_lines(lib, dtype):
    for rows in (1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 2048, 2049, 3971, 3972, 4096, 4097, 50_000):
        for vocab in (1, 5, 20_000, 40_001, 98_310, 131_072, 196_609, 262_144, 524_300, 1 << 22):
            check_batch(lib, Batch(rows, vocab, dtype, rows % 3, vocab % 5), accumulate=rows % 2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_batches_of_more_rows_than_a_launch_takes(lib, dtype):
    """Work items of 2^32 and more; rows in parts beyond what the workspace holds, and gradients of so long rows that a launch takes fewer
    than that."""
    for rows, vocab in ((1 << 26, 1), ((1 << 26) - 1, 3), (1 << 27, 900), (5_000_000, 30_000), (20_000_000, 131_072), (9000, 300_000), (2048, 1 << 25), (2049, 1 << 25),
                        (1024, 1 << 25), (40, 1 << 30), (31, 1 << 30), (32, (1 << 30) - 1), (130, 1 << 30), (1 << 34, 200)):
        check_batch(lib, Batch(rows, vocab, dtype))


@pytest.mark.parametrize("seed", range(4))
def test_any_batch(lib, seed):
    rng = random.Random(seed)
    for _ in range(1500):
        dtype = rng.randrange(2)
        rows, vocab = int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 22))
        check_batch(lib, Batch(rows, vocab, dtype, rng.randrange(64), rng.choice([0, 0, 1, rng.randrange(200)])), rng.randrange(2))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_beside_their_logits(lib, dtype):
    """Rows of logits and of gradients in turn in one buffer do not overlap, from either side; an element further they do."""
    vocab, size, hp = 1000, SIZE[dtype], (f32 * 4)(1.0, 0.2, 0.2, 0.1)
    for rows, stride, at, good in ((5, 2000, 1000, True), (5, 2000, -1000, True), (5, 2000, 999, False), (5, 2000, 1001, False), (5, 2000, -1001, False), (5, 2000, -999, False),
                                   (5, 2007, 1000, True), (5, 2007, 1007, True), (5, 2007, 1008, False), (5, 2007, 3 * 2007 + 1003, True), (5, 2007, 3 * 2007 + 3, False),
                                   (5, 1999, 1000, False), (1, 2000, 1000, True), (1, 2000, 999, False), (5, 2000, 0, True), (5, 2000, 9000, True), (5, 2000, 2000, False)):
        x = Logits(A[0], rows, vocab, stride, dtype)
        out = A[0] + at * size
        got = [lib.gs_token_logp_grad(ctypes.byref(x), vp(A[2]), f32(1.0), vp(A[4]), vp(A[3]), vp(out), i64(stride), None),
               lib.gs_policy_loss(ctypes.byref(x), vp(A[2]), hp, vp(A[6]), vp(A[7]), vp(A[8]), vp(A[9]), vp(A[3]), vp(out), i64(stride), vp(A[10]), 0, vp(WS),
                                  ctypes.c_size_t(WS_BYTES), None)]
        assert got == ([0, 0] if good else [-1, -1]), (rows, stride, at)
    x = Logits(A[0], 5, vocab, 2000, dtype)                # rows of another distance do
    assert lib.gs_token_logp_grad(ctypes.byref(x), vp(A[2]), f32(1.0), vp(A[4]), vp(A[3]), vp(A[0] + 1000 * size), i64(4000), None) == -1


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("pairs", [0, 1, 64, 127, 128, 129, 512, 513, 32_768, 65_537, 262_143, 262_144, 262_145, 600_000, 8_388_607])
def test_pairs(lib, pairs, accumulate):
    hp = (f32 * 3)(0.1, 0.0, 1.0)
    ls = launches(lib, lambda: lib.gs_preference_loss(vp(A[0]), vp(A[1]), vp(A[2]), i64(1 << 35), vp(A[3]), i64(pairs), hp, vp(A[4]), vp(A[5]), vp(A[6]), accumulate, vp(WS),
                                                      ctypes.c_size_t(WS_BYTES), None))
    if pairs == 0:
        assert ls.pop(0).is_a("k_zero")
        assert not ls if accumulate else ls[0].is_a("k_pair_sums") and ls[0].count == 0 and ls[0].out == A[6]
        return
    work, sums = [l for l in ls if l.is_a("k_pairs")], [l for l in ls if l.is_a("k_pair_sums")]
    at = 0
    for i, l in enumerate(work):
        assert l.grid == l.rows and l.row0 == A[3] + 8 * at and l.out == A[4] + 4 * at
        assert l.ends == (1 if i == 0 else 0) + (2 if i == len(work) - 1 else 0)
        at += l.rows
    assert at == pairs
    if pairs <= 128:
        assert not sums and len(work) == 1 and work[0].meet == pairs and work[0].slots == WS
        return
    assert [l.is_a("k_pairs") for l in ls] == [True, False] * len(work)
    for i, (w, s) in enumerate(zip(work, sums)):
        last = i == len(work) - 1
        assert w.meet == 0 and w.partials == s.partials == WS and s.count == w.rows and s.row0 == w.out
        assert s.meet == s.grid <= 64
        in_workspace(s.slots, s.meet * s.words)
        so_far = WS + 8 * (PARTIALS - 1)
        assert WS + 8 * w.rows <= so_far and so_far + 8 <= s.slots
        assert s.out == (A[6] if last else so_far) and s.accumulate == (accumulate if last else i > 0)
        assert s.len == (so_far if last and i else 0)


# ---- lists of tensors ------------------------------------------------------------------------------------

PIECE = 1 << 31


def lists(rng, count, most):
    at, out, ts = 1 << 60, 1 << 61, []
    for _ in range(count):
        dtype = rng.randrange(2)
        n = 0 if rng.random() < 0.1 else int(2 ** rng.uniform(0, most))
        at += 16 * rng.randrange(1, 9) + SIZE[dtype] * rng.randrange(8)
        at, out = -(-at // SIZE[dtype]) * SIZE[dtype], -(-out // SIZE[dtype]) * SIZE[dtype]
        ts.append((at, out, n, dtype))
        at += n * SIZE[dtype]
        out += n * SIZE[dtype] + rng.randrange(3) * 16
    return ts


def pieces(ts):
    return [(a + k * SIZE[d], o + k * SIZE[d] if o else a + k * SIZE[d], min(PIECE, n - k), d) for a, o, n, d in ts for k in range(0, n, PIECE)]


def tiles(t, per_tile):
    """Tiles of a tensor, whose vectors are counted from the start of the first one's line."""
    a, _, n, d = t
    head = min(n, (-a % 16) // SIZE[d])
    vecs = (n - head) // (16 // SIZE[d])
    return -(-((a + 15) // 16 % 8 + vecs) // per_tile)


def recorded(lib):
    """The tables of the launches: [(tensor, its first tile)] by launch."""
    t, out = Tensor(), {}
    for i in range(lib.rec_tensors()):
        lib.rec_tensor(i, ctypes.byref(t))
        out.setdefault(t.launch, []).append(((t.inp, t.out, t.numel, t.dtype), t.first))
    return out


def check_tables(lib, work, want, back, outs):
    tables, chunks = recorded(lib), []
    for i, l in work:
        entries = tables[i]
        assert l.count == len(entries) > 0 and l.grid == l.tiles <= 1 << 23
        per_tile = 256 * l.nv * l.tile_runs
        ends = [f for _, f in entries[1:]] + [l.tiles]
        for (t, first), end in zip(entries, ends):
            assert end - first >= max(1, tiles(t, per_tile)), (l.name, t)
        assert entries[0][1] == 0
        chunks.append([t for t, _ in entries])
    got = [t for es in (reversed(chunks) if back else chunks) for t in es]
    keep = (lambda t: t) if outs else (lambda t: (t[0], *t[2:]))         # the norm looks at no output
    assert list(map(keep, got)) == list(map(keep, want))


def check_list(lib, ts, in_place, accumulate=0):
    table = (GsTensor * max(1, len(ts)))(*[GsTensor(a, None if in_place else o, n, d) for a, o, n, d in ts])
    want = pieces([(a, None if in_place else o, n, d) for a, o, n, d in ts])
    ls = launches(lib, lambda: lib.gs_grads_sqnorm(table, i64(len(ts)), vp(A[1]), accumulate, vp(WS), ctypes.c_size_t(WS_BYTES), None))
    work = [(i, l) for i, l in enumerate(ls) if l.is_a("k_tensors_sqnorm")]
    check_tables(lib, work, want, False, False)
    total = sum(l.tiles for _, l in work)
    fold = ls[len(work):]
    if 0 < total <= 256:
        at = 0
        for _, l in work:
            assert l.meet == total and l.slot0 == at and l.slots == WS and l.out == A[1] and l.accumulate == accumulate
            at += l.tiles
        assert not fold and len({l.tag for _, l in work}) == 1
    elif total == 0 and accumulate:
        assert not ls
    else:
        at = 0
        for _, l in work:
            assert l.meet == 0 and l.partials == WS + 8 * at
            at += l.tiles
        assert total <= PARTIALS
        f, = fold
        assert f.is_a("k_tensors_fold") and f.count == total and f.partials == WS and f.out == A[1] and f.accumulate == accumulate and f.meet == f.grid <= 64
        in_workspace(f.slots, f.meet * f.words)
        assert f.slots >= WS + 8 * total
    ls = launches(lib, lambda: lib.gs_grads_clip(table, i64(len(ts)), vp(A[1]), f32(1.0), vp(A[2]), None))
    if not want:
        l, = ls
        assert l.grid == 1 and l.count == 0 and l.out == A[2]
        return
    check_tables(lib, list(enumerate(ls)), want, True, True)
    assert [l.out for l in ls] == [A[2]] + [0] * (len(ls) - 1)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(3))
def test_any_list_of_tensors(lib, seed, in_place):
    rng = random.Random(seed)
    for count in (0, 1, 2, 15, 16, 17, 100, 159, 160, 161, 239, 240, 241, 255, 256, 257, 320, 321, 480, 481, 1000, 5000):
        for most in (2, 12, 22, 30):
            check_list(lib, lists(rng, count, most), in_place, rng.randrange(2))


@pytest.mark.parametrize("in_place", [False, True])
def test_longest_lists_and_tensors(lib, in_place):
    rng = random.Random(7)
    check_list(lib, lists(rng, 65_536, 3), in_place)
    check_list(lib, lists(rng, 65_536, 20), in_place)
    for n in (PIECE - 1, PIECE, PIECE + 1, 3 * PIECE, (1 << 34) + 5, 1 << 44):
        for dtype in (BF16, F32):
            check_list(lib, [((1 << 50) + SIZE[dtype], 1 << 52, n, dtype)], in_place)
    check_list(lib, [((1 << 48) + (i << 36), (1 << 55) + (i << 36), (1 << 33) + i, i % 2) for i in range(400)], in_place)


def test_every_kernel_is_reached(lib):
    """None is built that no call takes."""
    REACHED.clear()
    for dtype in (BF16, F32):
        test_vocabularies_at_the_lines_between_kernels(lib, dtype)
        test_numbers_of_rows_at_their_lines(lib, dtype)
    for pairs in (0, 1, 300, 300_000):
        test_pairs(lib, pairs, 0)
    for in_place in (False, True):
        test_any_list_of_tensors(lib, 0, in_place)
    buf = ctypes.create_string_buffer(1 << 16)
    lib.rec_kernels(buf, len(buf))
    assert set(buf.value.decode().split("\n")[:-1]) == REACHED
