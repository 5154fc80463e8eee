"""What the losses' and the tensors' entry points refuse before any HIP call, on the CPU, with addresses that are never
dereferenced."""
from __future__ import annotations

import ctypes

import pytest

from paper_2512_17570_amd import gs

A = [(1 << 40) + i * (1 << 36) for i in range(16)]        # far-apart addresses
BAD, WORK = gs.GS_ERR_INVALID_ARG, gs.GS_ERR_WORKSPACE
WS = gs.gs_sqnorm_workspace_bytes()
NAN, INF = float("nan"), float("inf")


def x(data=A[0], rows=4, vocab=100, stride=100, dtype=gs.GS_BF16):
    return gs.gs_logits(data, rows, vocab, stride, dtype)


WRONG_LOGITS = [x(None), x(A[0] + 1), x(A[0] + 2, dtype=gs.GS_F32), x(rows=-1), x(vocab=0), x(vocab=-5), x(vocab=(1 << 30) + 1, stride=1 << 31), x(stride=99),
                x(stride=0), x(stride=-100), x(dtype=2), x(dtype=-1), x(rows=1 << 40, stride=1 << 40), x(rows=(1 << 40) + 1)]


def logp(lg=None, targets=A[1], out=A[2], stats=A[3], temperature=1.0, ws=A[4], bytes_=WS):
    return gs.gs_token_logp(lg or x(), targets, out, stats, temperature, ws, bytes_, stream=0, check=False)


def test_token_logp():
    for lg in WRONG_LOGITS:
        assert logp(lg) == BAD
    for kw in ({"targets": 0}, {"targets": A[1] + 4}, {"out": 0}, {"out": A[2] + 2}, {"stats": A[3] + 1}, {"out": A[0] + 16}, {"out": A[1] + 8}, {"stats": A[2]},
               {"out": A[4] + 64}, {"stats": A[0] + 792}, *({"temperature": t} for t in (0.0, -1.0, NAN, INF, 9e-5, 1.1e4))):
        assert logp(**kw) == BAD, kw
    for kw in ({"ws": 0}, {"ws": A[4] + 4}, {"bytes_": WS - 1}):
        assert logp(**kw) == WORK, kw
    assert logp(x(None, rows=0), 0, 0, 0) == gs.GS_OK
    assert gs._lib.gs_token_logp(None, A[1], 1.0, A[2], None, A[4], WS, None) == BAD


def grad(lg=None, targets=A[1], stats=A[2], dlogp=A[3], out=A[4], stride=100, temperature=1.0):
    lg = lg or x()
    return gs._lib.gs_token_logp_grad(ctypes.byref(lg), targets, temperature, stats, dlogp, out, stride, None)


def test_token_logp_grad():
    for lg in WRONG_LOGITS:
        assert grad(lg) == BAD
    for kw in ({"targets": 0}, {"targets": A[1] + 1}, {"stats": 0}, {"stats": A[2] + 2}, {"dlogp": 0}, {"dlogp": A[3] + 1}, {"out": 0}, {"out": A[4] + 1}, {"stride": 99},
               {"stride": -100}, {"out": A[0], "stride": 101}, {"out": A[0] + 2}, {"out": A[0] + 798}, {"out": A[1] + 16}, {"out": A[2] - 2}, {"out": A[3]},
               {"stride": 1 << 61}, {"temperature": 0.0}, {"temperature": NAN}):
        assert grad(**kw) == BAD, kw
    assert grad(x(None, rows=0), 0, 0, 0, 0) == gs.GS_OK


def policy(lg=None, targets=A[1], hp=None, old=A[2], ref=A[3], adv=A[4], w=A[5], logp=A[6], out=A[7], stride=100, stats=A[8], acc=0, ws=A[9], bytes_=WS):
    lg = lg or x()
    hp = hp or gs.PolicyHParams()
    return gs._lib.gs_policy_loss(ctypes.byref(lg), targets, ctypes.byref(hp.c_struct()), old, ref, adv, w, logp, out, stride, stats, acc, ws, bytes_, None)


def test_policy_loss():
    for lg in WRONG_LOGITS:
        assert policy(lg) == BAD
    for name, a in (("targets", A[1]), ("old", A[2]), ("adv", A[4]), ("logp", A[6]), ("stats", A[8])):
        assert policy(**{name: 0}) == BAD and policy(**{name: a + 2}) == BAD, name
    for kw in ({"ref": A[3] + 1}, {"w": A[5] + 2}, {"out": A[7] + 1}, {"stride": 99}, {"out": A[0] + 4}, {"out": A[0], "stride": 200}, {"out": A[2] + 4}, {"logp": A[2]},
               {"logp": A[7] + 100}, {"stats": A[6] + 12}, {"stats": A[9] + 8}, {"logp": A[0] + 400}):
        assert policy(**kw) == BAD, kw
    for hp in (gs.PolicyHParams(temperature=0.0), gs.PolicyHParams(clip_low=-0.1), gs.PolicyHParams(clip_low=1.5), gs.PolicyHParams(clip_low=NAN),
               gs.PolicyHParams(clip_high=-0.1), gs.PolicyHParams(clip_high=INF), gs.PolicyHParams(kl_coef=-1.0), gs.PolicyHParams(kl_coef=NAN)):
        assert policy(hp=hp) == BAD, hp
    for kw in ({"ws": 0}, {"ws": A[9] + 4}, {"bytes_": WS - 1}):
        assert policy(**kw) == WORK, kw
    assert policy(x(None, rows=0), 0, None, 0, 0, 0, 0, 0, 0, acc=1) == gs.GS_OK
    assert gs._lib.gs_policy_loss(ctypes.byref(x()), A[1], None, A[2], A[3], A[4], A[5], A[6], A[7], 100, A[8], 0, A[9], WS, None) == BAD


def preference(logp=A[0], ref=A[1], w=A[2], tokens=100, offsets=A[3], pairs=2, hp=None, margins=A[4], dlogp=A[5], loss=A[6], acc=0, ws=A[7], bytes_=WS):
    hp = hp or gs.PreferenceHParams()
    return gs._lib.gs_preference_loss(logp, ref, w, tokens, offsets, pairs, ctypes.byref(hp.c_struct()), margins, dlogp, loss, acc, ws, bytes_, None)


def test_preference_loss():
    for name, a in (("logp", A[0]), ("offsets", A[3]), ("margins", A[4]), ("dlogp", A[5]), ("loss", A[6])):
        assert preference(**{name: 0}) == BAD and preference(**{name: a + 2}) == BAD, name
    for kw in ({"ref": A[1] + 1}, {"w": A[2] + 3}, {"tokens": -1}, {"pairs": -1}, {"pairs": 1 << 31}, {"tokens": 1 << 41}, {"dlogp": A[0]}, {"dlogp": A[1] + 4}, {"dlogp": A[2]},
               {"dlogp": A[3] + 36}, {"margins": A[5] + 396}, {"loss": A[4]}, {"loss": A[7] + 8}, {"margins": A[3] + 8}):
        assert preference(**kw) == BAD, kw
    for hp in (gs.PreferenceHParams(beta=0.0), gs.PreferenceHParams(beta=-1.0), gs.PreferenceHParams(beta=NAN), gs.PreferenceHParams(beta=INF),
               gs.PreferenceHParams(label_smoothing=-0.1), gs.PreferenceHParams(label_smoothing=1.0), gs.PreferenceHParams(label_smoothing=NAN),
               gs.PreferenceHParams(scale=NAN), gs.PreferenceHParams(scale=INF)):
        assert preference(hp=hp) == BAD, hp
    for kw in ({"ws": 0}, {"ws": A[7] + 4}, {"bytes_": WS - 1}):
        assert preference(**kw) == WORK, kw
    assert preference(0, 0, 0, 0, 0, 0, None, 0, 0, acc=1) == gs.GS_OK
    assert gs._lib.gs_preference_loss(A[0], A[1], A[2], 100, A[3], 2, None, A[4], A[5], A[6], 0, A[7], WS, None) == BAD


def tensors(*t):
    return (gs.gs_tensor * max(1, len(t)))(*[gs.gs_tensor(*v) for v in t]), len(t)


GOOD = (A[0], None, 100, gs.GS_F32)
WRONG_TENSORS = [(None, None, 100, gs.GS_F32), (A[0] + 2, None, 100, gs.GS_F32), (A[0] + 1, None, 100, gs.GS_BF16), (A[0], None, -1, gs.GS_F32), (A[0], None, 100, 2),
                 (A[0], None, (1 << 44) + 1, gs.GS_BF16)]


def test_grads_sqnorm():
    call = lambda t, n, sq=A[5], acc=0, ws=A[6], b=WS: gs._lib.gs_grads_sqnorm(t, n, sq, acc, ws, b, None)  # noqa: E731
    for t in WRONG_TENSORS:
        assert call(*tensors(GOOD, t)) == BAD, t
    many = (A[0], None, 1 << 43, gs.GS_BF16)
    assert call(*tensors(many, many, many)) == BAD
    assert call(None, 1) == BAD and call(tensors(GOOD)[0], -1) == BAD and call(tensors(GOOD)[0], gs.GS_MAX_TENSORS + 1) == BAD
    for kw in ({"sq": 0}, {"sq": A[5] + 4}):
        assert call(*tensors(GOOD), **kw) == BAD
    for kw in ({"ws": 0}, {"ws": A[6] + 4}, {"b": WS - 1}):
        assert call(*tensors(GOOD), **kw) == WORK
    for kw in ({"sq": A[0] + 392}, {"ws": A[0] + 8}, {"sq": A[6] + 64}, {"ws": A[0] - WS + 8}):
        assert call(*tensors(GOOD), **kw) == BAD, kw
    assert call(None, 0, acc=1) == gs.GS_OK and call(*tensors((None, None, 0, gs.GS_BF16)), acc=1) == gs.GS_OK


def test_grads_clip():
    call = lambda t, n, sq=A[5], most=1.0, norm=A[6]: gs._lib.gs_grads_clip(t, n, sq, most, norm, None)  # noqa: E731
    for t in WRONG_TENSORS:
        assert call(*tensors(GOOD, t)) == BAD, t
    for kw in ({"sq": 0}, {"sq": A[5] + 4}, {"norm": A[6] + 2}, {"most": 0.0}, {"most": -1.0}, {"most": NAN},
               {"sq": A[0] + 392}, {"norm": A[0] + 396}, {"norm": A[5] + 4}):
        assert call(*tensors(GOOD), **kw) == BAD, kw
    overlaps = [
        [GOOD, GOOD],                                                               # twice
        [(A[0], A[0] + 4, 100, gs.GS_F32)], [(A[0], A[0] + 396, 100, gs.GS_F32)],   # an output in its own input
        [(A[0], A[1], 100, gs.GS_F32), (A[2], A[1] + 396, 100, gs.GS_F32)],         # two outputs
        [(A[0], A[1], 100, gs.GS_F32), (A[1], A[2], 100, gs.GS_F32)],               # an output over another's input
        [(A[1], A[2], 100, gs.GS_F32), (A[0], A[1], 100, gs.GS_F32)],
        [(A[0], None, 100, gs.GS_F32), (A[0] + 200, None, 100, gs.GS_BF16)],        # two in place
        [(A[0], None, 1000, gs.GS_F32), (A[1], None, 5, gs.GS_F32), (A[0] + 4, A[2], 1, gs.GS_F32)],  # an input inside an output
        [(A[0], A[3], 1000, gs.GS_F32), (A[0] + 40, A[0] + 44, 1, gs.GS_F32)],      # an output inside a long input
    ]
    for rest in ([], [(A[7] + 64 * i, None, 8, gs.GS_F32) for i in range(50)]):     # short lists, and those that are sorted elsewhere
        for t in overlaps:
            assert call(*tensors(*t, *rest)) == BAD, (t, len(rest))
            assert call(*tensors(*rest, *t)) == BAD, (t, len(rest))
    assert call(None, 0, norm=0) == gs.GS_OK


def test_structs_as_the_header_has_them(tmp_path):
    import subprocess

    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "gs.h"\nint main(void) { printf("%zu %zu %zu %zu %d %d %d\\n", sizeof(gs_logits), sizeof(gs_policy_hparams),\n'
                   'sizeof(gs_preference_hparams), sizeof(gs_tensor), GS_BF16, GS_F32, GS_MAX_TENSORS); return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == [*(ctypes.sizeof(c) for c in (gs.gs_logits, gs.gs_policy_hparams, gs.gs_preference_hparams, gs.gs_tensor)),
                                     gs.GS_BF16, gs.GS_F32, gs.GS_MAX_TENSORS]


@pytest.mark.parametrize("n", [0, 1])
def test_a_stacked_tensor_is_no_list(n):
    import torch
    with pytest.raises(TypeError):
        gs.gs_grads_sqnorm(torch.zeros(n + 1, 4), 0, 0)
