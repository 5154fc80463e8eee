"""A head without its logits, layer norm and dropout, on the CPU: what is refused before any HIP call, the structs as C has them, the workspaces' sizes, and
what the compiler makes of the kernels."""
from __future__ import annotations

import ctypes
import os
import re
import subprocess

import pytest

from paper_2512_17570_amd import build as B
from paper_2512_17570_amd import gs

BAD, WS, OK = gs.GS_ERR_INVALID_ARG, gs.GS_ERR_WORKSPACE, gs.GS_OK
L = gs._lib
# distinct, far apart addresses that no refused call follows
X, W, BIAS, T, LOGP, STATS, DX, DW, DB, LOSS, SPACE, WEIGHTS = ((i + 1) << 32 for i in range(12))
ROWS, HIDDEN, VOCAB = 100, 64, 1000
BYTES = gs.gs_head_workspace_bytes(ROWS, HIDDEN, VOCAB)


def head(**k):
    a = dict(x=X, w=W, bias=BIAS, rows=ROWS, hidden=HIDDEN, vocab=VOCAB, x_stride=HIDDEN, w_stride=HIDDEN) | k
    return gs.gs_head(*[a[n] for n, _ in gs.gs_head._fields_])


def grads(**k):
    a = dict(dx=DX, dw=DW, dbias=DB, dx_stride=HIDDEN, dw_stride=HIDDEN) | k
    return gs.gs_head_grads(*[a[n] for n, _ in gs.gs_head_grads._fields_])


def ref(s):
    return None if s is None else ctypes.byref(s)


def logp(h, targets=T, temperature=1.0, out=LOGP, stats=STATS, ws=SPACE, size=BYTES):
    return L.gs_head_logp(ref(h), targets, temperature, out, stats, ws, size, None)


def grad(h, targets=T, temperature=1.0, stats=STATS, dlogp=LOGP, g=None, ws=SPACE, size=BYTES):
    return L.gs_head_logp_grad(ref(h), targets, temperature, stats, dlogp, ref(g), ws, size, None)


def entropy(h, targets=T, weights=WEIGHTS, temperature=1.0, out=LOGP, g=None, loss=LOSS, ws=SPACE, size=BYTES):
    return L.gs_head_cross_entropy(ref(h), targets, weights, temperature, out, ref(g), loss, 0, ws, size, None)


BAD_HEADS = [None, dict(rows=-1), dict(rows=(1 << 20) + 1), dict(hidden=0), dict(hidden=(1 << 17) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(x=None), dict(w=None),
             dict(x=X + 1), dict(w=W + 1), dict(bias=BIAS + 1), dict(x_stride=HIDDEN - 1), dict(w_stride=HIDDEN - 1), dict(w_stride=1 << 60), dict(x_stride=1 << 60)]


@pytest.mark.parametrize("bad", BAD_HEADS)
def test_heads_that_are_refused(bad):
    h = None if bad is None else head(**bad)
    huge = 1 << 50
    assert logp(h, size=huge) == BAD
    assert grad(h, g=grads(), size=huge) == BAD
    assert entropy(h, g=grads(), size=huge) == BAD


@pytest.mark.parametrize("temperature", [0.0, -1.0, float("nan"), float("inf"), 1e-5, 1e5])
def test_temperatures_that_are_refused(temperature):
    assert logp(head(), temperature=temperature) == BAD
    assert grad(head(), temperature=temperature, g=grads()) == BAD
    assert entropy(head(), temperature=temperature, g=grads()) == BAD


@pytest.mark.parametrize("bad", [dict(targets=None), dict(targets=T + 4), dict(out=None), dict(out=LOGP + 2), dict(stats=STATS + 1)])
def test_arrays_of_log_probabilities_that_are_refused(bad):
    assert logp(head(), **bad) == BAD


@pytest.mark.parametrize("bad", [dict(targets=None), dict(stats=None), dict(stats=STATS + 2), dict(dlogp=None), dict(dlogp=LOGP + 1), dict(g=None),
                                 dict(g=grads(dx=DX + 1)), dict(g=grads(dw=DW + 1)), dict(g=grads(dbias=DB + 1)), dict(g=grads(dx_stride=63)),
                                 dict(g=grads(dw_stride=63)), dict(g=grads(dw_stride=1 << 60))])
def test_gradients_that_are_refused(bad):
    assert grad(head(), **({"g": grads()} | bad)) == BAD


@pytest.mark.parametrize("bad", [dict(weights=WEIGHTS + 2), dict(out=None), dict(loss=None), dict(loss=LOSS + 2), dict(targets=T + 1), dict(g=grads(dx=DX + 1))])
def test_losses_that_are_refused(bad):
    assert entropy(head(), **({"g": grads()} | bad)) == BAD


@pytest.mark.parametrize("ws, size", [(None, BYTES), (SPACE + 8, BYTES), (SPACE, BYTES - 1), (SPACE, 0)])
def test_workspaces_that_are_refused(ws, size):
    assert grad(head(), g=grads(), ws=ws, size=size) == WS
    assert entropy(head(), g=grads(), ws=ws, size=size) == WS
    assert logp(head(), ws=ws, size=size if size != BYTES - 1 else gs.gs_head_workspace_bytes(ROWS, HIDDEN, VOCAB, False) - 1) == WS


def test_overlaps_are_refused():
    n = HIDDEN * 2
    assert logp(head(), out=X + 4) == BAD
    assert logp(head(), out=W + VOCAB * n - 4) == BAD
    assert logp(head(), out=STATS + 4) == BAD
    assert logp(head(), stats=T) == BAD
    assert logp(head(w=SPACE)) == BAD
    for g in (grads(dx=X), grads(dw=W), grads(dbias=BIAS), grads(dx=DW), grads(dbias=DX + 2), grads(dw=SPACE), grads(dx=T), grads(dw=LOGP)):
        assert grad(head(), g=g) == BAD
        assert entropy(head(), g=g) == BAD
    assert entropy(head(), g=grads(dx=WEIGHTS)) == BAD
    assert entropy(head(), g=grads(), loss=LOGP) == BAD


def test_an_empty_batch_of_scores_is_a_no_op():
    size = gs.gs_head_workspace_bytes(0, HIDDEN, VOCAB, False)
    assert logp(head(rows=0, x=None), targets=None, out=None, stats=None, size=size) == OK


def test_workspace_sizes():
    assert gs.gs_head_workspace_bytes(-1, 64, 64) == gs.gs_head_workspace_bytes(1, 0, 64) == gs.gs_head_workspace_bytes(1, 64, 0) == 0
    assert gs.gs_head_workspace_bytes((1 << 20) + 1, 64, 64) == gs.gs_head_workspace_bytes(1, (1 << 17) + 1, 64) == gs.gs_head_workspace_bytes(1, 64, (1 << 30) + 1) == 0
    for rows in (0, 1, 100, 8192, 1 << 20):
        for hidden in (1, 100, 4096):
            for vocab in (1, 50_001, 131_072):
                assert 0 < gs.gs_head_workspace_bytes(rows, hidden, vocab, False) <= gs.gs_head_workspace_bytes(rows, hidden, vocab, True)
    # nothing of the size of the logits: 8192 x 131072 are 2.1 GB in bf16
    assert gs.gs_head_workspace_bytes(8192, 4096, 131_072) < 1 << 30
    assert gs.gs_layer_norm_workspace_bytes(-1, 5) == gs.gs_layer_norm_workspace_bytes(5, 0) == gs.gs_layer_norm_workspace_bytes(5, (1 << 24) + 1) == 0
    assert gs.gs_layer_norm_workspace_bytes(0, 5) > 0


# ---- layer norm and dropout ---------------------------------------------------------------------------------------------

NBYTES = gs.gs_layer_norm_workspace_bytes(ROWS, HIDDEN)


def matrix(**k):
    a = dict(data=X, rows=ROWS, cols=HIDDEN, row_stride=HIDDEN, dtype=gs.GS_BF16) | k
    return gs.gs_matrix(*[a[n] for n, _ in gs.gs_matrix._fields_])


def norm(m, gamma=W, beta=BIAS, wt=gs.GS_F32, eps=1e-5, y=DX, stride=HIDDEN, stats=STATS):
    return L.gs_layer_norm(ref(m), gamma, beta, wt, eps, y, stride, stats, None)


def norm_grad(m, gamma=W, wt=gs.GS_F32, stats=STATS, dy=T, dys=HIDDEN, dx=DX, dxs=HIDDEN, dg=DW, db=DB, ws=SPACE, size=NBYTES):
    return L.gs_layer_norm_grad(ref(m), gamma, wt, stats, dy, dys, dx, dxs, dg, db, ws, size, None)


@pytest.mark.parametrize("bad", [None, dict(data=None), dict(data=X + 1), dict(rows=-1), dict(rows=(1 << 31) + 1), dict(cols=0), dict(cols=(1 << 24) + 1), dict(row_stride=63),
                                 dict(row_stride=1 << 61), dict(dtype=2), dict(dtype=-1)])
def test_matrices_that_are_refused(bad):
    m = None if bad is None else matrix(**bad)
    assert norm(m) == BAD
    assert norm_grad(m, size=1 << 50) == BAD


@pytest.mark.parametrize("bad", [dict(gamma=W + 2), dict(beta=BIAS + 1), dict(wt=5), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=None), dict(y=DX + 1),
                                 dict(stride=63), dict(stats=STATS + 2), dict(y=X + 2), dict(y=W), dict(stats=X), dict(y=X, stride=65), dict(beta=DX)])
def test_norms_that_are_refused(bad):
    assert norm(matrix(), **bad) == BAD


@pytest.mark.parametrize("bad", [dict(gamma=W + 2), dict(wt=3), dict(stats=None), dict(dy=None), dict(dx=None), dict(dy=T + 1), dict(dys=63), dict(dxs=63), dict(dg=None), dict(db=None),
                                 dict(dg=DW + 1), dict(dx=X), dict(dx=T, dxs=65), dict(dx=T + 2), dict(dg=DB), dict(dg=W), dict(dg=SPACE), dict(dx=STATS)])
def test_norm_gradients_that_are_refused(bad):
    assert norm_grad(matrix(), **bad) == BAD


@pytest.mark.parametrize("ws, size", [(None, NBYTES), (SPACE + 4, NBYTES), (SPACE, NBYTES - 1)])
def test_norm_workspaces_that_are_refused(ws, size):
    assert norm_grad(matrix(), ws=ws, size=size) == WS


def test_empty_norms_are_no_ops():
    assert norm(matrix(rows=0, data=None), y=None, stats=None) == OK
    assert norm_grad(matrix(rows=0, data=None), dy=None, dx=None, stats=None, dg=None, db=None, ws=None, size=0) == OK


def dropout(x=X, res=W, out=DX, n=1000, dtype=gs.GS_BF16, p=0.1, seed=1, offset=0, step=T):
    return L.gs_dropout(x, res, out, n, dtype, p, seed, offset, step, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(x=X + 1), dict(res=W + 1), dict(out=DX + 1), dict(n=-1), dict(n=(1 << 40) + 1), dict(dtype=7), dict(p=-0.1), dict(p=1.1),
                                 dict(p=float("nan")), dict(step=T + 4), dict(offset=(1 << 64) - 999), dict(out=X + 2), dict(out=W - 2), dict(out=T - 8),
                                 dict(dtype=gs.GS_F32, x=X + 2)])
def test_dropouts_that_are_refused(bad):
    assert dropout(**bad) == BAD


def test_no_dropout_of_nothing():
    assert dropout(n=0, x=None, res=None, out=None) == OK


# ---- structs, assembly -----------------------------------------------------------------------------------------------------

def test_structs_as_c_has_them(tmp_path):
    names = {"gs_head": gs.gs_head, "gs_head_grads": gs.gs_head_grads, "gs_matrix": gs.gs_matrix}
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"gs.h\"\nint main(void){\n"
    for n, s in names.items():
        src += f'printf("{n} %zu\\n", sizeof({n}));\n' + "".join(f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));\n' for f, _ in s._fields_)
    (tmp_path / "s.c").write_text(src + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(B.ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    said = dict(l.split() for l in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.splitlines())
    for n, s in names.items():
        assert int(said[n]) == ctypes.sizeof(s)
        for f, _ in s._fields_:
            assert int(said[f"{n}.{f}"]) == getattr(s, f).offset


@pytest.fixture(scope="module", params=["gs_head.hip", "gs_norm.hip"])
def kernels(request, tmp_path_factory):
    """{name: (registers of a lane, scratch, LDS, lanes of a workgroup, assembly)}"""
    out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
    flags = [f for f in B.FLAGS if f != "-shared"]
    subprocess.run([B.HIPCC, *flags, "--offload-device-only", "-S", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, os.path.join(B.CSRC, request.param),
                    "-o", out], check=True, capture_output=True, text=True)
    text = open(out).read()
    found, kernels = {}, {re.search(r"\.name: +(\S+)", b)[1]: b for b in text.split("\n  - .agpr_count:")[1:]}
    for name, block in re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", text, re.S):
        number = lambda key: int(re.search(rf"{key} (\d+)", block)[1])  # noqa: E731
        start = text.index(f"\n{name}:")
        lanes = int(re.search(r"\.max_flat_workgroup_size: (\d+)", kernels[name])[1])
        found[name] = number("next_free_vgpr"), number("private_segment_fixed_size"), number("group_segment_fixed_size"), lanes, text[start:text.index(".section", start)]
    assert found
    return found


def test_no_scratch_memory_and_room_for_a_workgroup(kernels):
    for name, (registers, scratch, lds, lanes, code) in kernels.items():
        assert scratch == 0 and not re.search(r"\b(scratch|buffer)_(load|store)", code), name
        assert lds <= 160 * 1024, name
        assert registers <= 512 // max(1, -(-lanes // 256)), name


def test_no_packed_fp32(kernels):
    for name, (*_, code) in kernels.items():
        assert not re.search(r"v_pk_(add|mul|fma)_f32", code), name


def test_products_wait_for_loads_once_a_step(kernels):
    """In the loop over k of a product, loads to LDS are waited for at the step's barrier only (the compiler's own wait in front of a transposing read
    would end the overlap), and it has as many products as two parts of a tile need."""
    found = 0
    for name, (*_, code) in kernels.items():
        if "global_load_lds" not in code:
            continue
        lines = code.split("\n")
        labels = {l.split(":")[0]: i for i, l in enumerate(lines) if re.match(r"\.LBB\d+_\d+:", l)}
        loops = []
        for i, l in enumerate(lines):
            m = re.search(r"s_cbranch_\w+ (\.LBB\d+_\d+)", l)
            if m and labels.get(m[1], i) < i:
                body = lines[labels[m[1]]:i]
                if any("v_mfma" in x for x in body) and any("global_load_lds" in x for x in body):
                    loops.append(body)
        assert len(loops) == (2 if "dx_dw" in name else 1), name        # a kernel of two products has a loop for each
        found += 1
        for body in loops:
            assert sum("s_waitcnt" in x and "vmcnt" in x for x in body) == 1 == sum("s_barrier" in x for x in body), name
    assert found or not any("head" in n for n in kernels)
