"""Arrays of no elements overlap nothing, wherever their addresses lie: calls that launch nothing, on the CPU, with addresses
that are never dereferenced."""
from __future__ import annotations

import ctypes

import pytest

from paper_2512_17570_amd import gs

A = [(1 << 40) + i * (1 << 36) for i in range(8)]         # far-apart addresses
WS = gs.gs_sqnorm_workspace_bytes()


@pytest.mark.parametrize("inside", [A[1] + 8, A[1], A[1] + WS - 8, A[1] + WS, A[2] + 4, A[2]])
def test_norm_of_empty_tensors_in_the_workspace_or_the_result(inside):
    table = (gs.gs_tensor * 2)(gs.gs_tensor(inside, None, 0, gs.GS_F32), gs.gs_tensor(inside, inside, 0, gs.GS_BF16))
    assert gs._lib.gs_grads_sqnorm(table, 2, A[2], 1, A[1], WS, None) == gs.GS_OK


@pytest.mark.parametrize("inside", [A[1] + 8, A[2] + 4])
def test_clip_of_empty_tensors_in_the_norm(inside):
    table = (gs.gs_tensor * 1)(gs.gs_tensor(inside, inside, 0, gs.GS_F32))
    assert gs._lib.gs_grads_clip(table, 1, A[2], 1.0, None, None) == gs.GS_OK


def preference(**at):
    p = {"logp": A[0], "ref": A[0], "w": A[0], "offsets": A[0], "margins": A[0], "dlogp": A[0], "loss": A[2], "ws": A[1], **at}
    hp = gs.PreferenceHParams().c_struct()
    return gs._lib.gs_preference_loss(p["logp"], p["ref"], p["w"], 0, p["offsets"], 0, ctypes.byref(hp), p["margins"], p["dlogp"], p["loss"], 1,
                                      p["ws"], WS, None)


@pytest.mark.parametrize("name", ["logp", "ref", "w", "offsets", "margins", "dlogp"])
@pytest.mark.parametrize("inside", [A[1] + 8, A[1], A[1] + WS - 8])
def test_preference_loss_of_no_tokens(name, inside):
    assert preference(**{name: inside}) == gs.GS_OK


def test_arrays_that_hold_something_still_overlap():
    table = (gs.gs_tensor * 2)(gs.gs_tensor(A[1] + 8, None, 0, gs.GS_F32), gs.gs_tensor(A[1] + 8, None, 1, gs.GS_F32))
    assert gs._lib.gs_grads_sqnorm(table, 2, A[2], 1, A[1], WS, None) == gs.GS_ERR_INVALID_ARG
    assert preference(loss=A[1] + 8) == gs.GS_ERR_INVALID_ARG
