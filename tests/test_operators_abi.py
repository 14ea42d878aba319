"""CPU tests of the argument checks of the few-token forward, the policy and
preference losses and the clipping: refused before any device work."""
import ctypes
import os

import pytest

from paper_2606_19528_gb300 import build, lora

P = 256         # an address that is aligned to everything, never read
WS = (None, 0)  # no workspace: arguments that pass the other checks end at this one, so no call here can launch


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(lora._LIB_PATH):
        build.build_cuda()
    return lora.library()


def code(fn, *args):
    try:
        fn(*args)
    except lora.LoraError as e:
        return e.code
    return lora.LORA_OK


def passed(want):
    """What a call without a workspace returns for arguments whose check gives `want`."""
    return want or lora.LORA_EWORKSPACE


def proj(T=1, K=64, N=1, r=4, s=1.0, **kw):
    a = dict(x=P, A=P, B=P, y=P, Wq=lora.make_q4(P, P))
    a.update(kw)
    return lora.make_projs([lora.make_proj(lora.make_shape(T, K, N, r, s), **a)])


@pytest.mark.parametrize("kw,want", [
    ({"T": 0}, lora.LORA_EINVAL), ({"T": 17}, lora.LORA_EINVAL), ({"K": 32}, lora.LORA_EINVAL),
    ({"K": 96}, lora.LORA_EINVAL), ({"K": 0}, lora.LORA_EINVAL), ({"N": 0}, lora.LORA_EINVAL),
    ({"N": (1 << 20) + 1}, lora.LORA_EINVAL), ({"r": -1}, lora.LORA_EINVAL), ({"r": 129}, lora.LORA_EINVAL),
    ({"s": float("nan")}, lora.LORA_EINVAL)])
def test_decode_shapes(kw, want):
    assert code(lora.lora_decode_workspace_size, proj(**kw)) == want
    assert code(lora.lora_decode_q4, proj(**kw), *WS, 0) == want


@pytest.mark.parametrize("kw,want", [
    ({"x": None}, lora.LORA_ENULL), ({"y": None}, lora.LORA_ENULL), ({"A": None}, lora.LORA_ENULL),
    ({"B": None}, lora.LORA_ENULL), ({"Wq": None}, lora.LORA_ENULL), ({"Wq": lora.make_q4(P, None)}, lora.LORA_ENULL),
    ({"W": P}, lora.LORA_EINVAL), ({"x": P + 8}, lora.LORA_EALIGN), ({"y": P + 2}, lora.LORA_EALIGN),
    ({"Wq": lora.make_q4(P + 8, P)}, lora.LORA_EALIGN), ({"Wq": lora.make_q4(P, P + 4)}, lora.LORA_EALIGN),
    ({"B": P + 2}, lora.LORA_EALIGN)])
def test_decode_pointers(kw, want):
    assert code(lora.lora_decode_q4, proj(**kw), *WS, 0) == want


def test_decode_workspace():
    assert lora.lora_decode_workspace_size(proj(T=16, r=128)) >= 16 * 128 * 4
    assert lora.lora_decode_workspace_size(proj(r=0, A=None, B=None)) == 0
    assert code(lora.lora_decode_q4, proj(), None, 0, 0) == lora.LORA_EWORKSPACE
    assert code(lora.lora_decode_q4, proj(), P, 16, 0) == lora.LORA_EWORKSPACE
    assert code(lora.lora_decode_q4, proj(), P + 16, 1 << 20, 0) == lora.LORA_EALIGN
    n = ctypes.c_size_t(0)
    assert lora.library().lora_decode_workspace_size(None, 1, ctypes.byref(n)) == lora.LORA_ENULL
    assert lora.library().lora_decode_workspace_size(proj(), 0, ctypes.byref(n)) == lora.LORA_EINVAL
    assert lora.library().lora_decode_workspace_size(proj(), 65, ctypes.byref(n)) == lora.LORA_EINVAL
    assert lora.library().lora_decode_workspace_size(proj(), 1, None) == lora.LORA_ENULL


def policy(**kw):
    a = dict(T=10, S=2, d=64, offsets=P, nll=P, old_nll=P, advantage=P, loss=P, dh_nll=P, dh=P)
    a.update(kw)
    return lora.make_policy_args(**a)


@pytest.mark.parametrize("kw,want", [
    ({"T": 0}, lora.LORA_EINVAL), ({"T": (1 << 24) + 1}, lora.LORA_EINVAL), ({"S": 0}, lora.LORA_EINVAL),
    ({"d": 12}, lora.LORA_EINVAL), ({"d": 0}, lora.LORA_EINVAL), ({"reduction": 3}, lora.LORA_EINVAL),
    ({"reduction": -1}, lora.LORA_EINVAL), ({"clip_low": -0.1}, lora.LORA_EINVAL),
    ({"clip_low": 1.1}, lora.LORA_EINVAL), ({"clip_high": float("inf")}, lora.LORA_EINVAL),
    ({"clip_high": -0.1}, lora.LORA_EINVAL), ({"beta": float("nan")}, lora.LORA_EINVAL),
    ({"scale": float("inf")}, lora.LORA_EINVAL), ({"nll": None}, lora.LORA_ENULL),
    ({"old_nll": None}, lora.LORA_ENULL), ({"advantage": None}, lora.LORA_ENULL), ({"loss": None}, lora.LORA_ENULL),
    ({"offsets": None}, lora.LORA_ENULL), ({"dh_nll": None}, lora.LORA_ENULL), ({"nll": P + 2}, lora.LORA_EALIGN),
    ({"dh": P + 8}, lora.LORA_EALIGN), ({"stats": P + 1}, lora.LORA_EALIGN), ({"nll": P + 4}, lora.LORA_OK),
    ({"dh": None}, lora.LORA_OK), ({"clip_low": 1.0}, lora.LORA_OK), ({"mask": P + 1}, lora.LORA_OK)])
def test_policy_arguments(kw, want):
    assert code(lora.lora_policy_workspace_size, policy(**kw)) == want
    assert code(lora.lora_policy_fwd_bwd, policy(**kw), *WS, 0) == passed(want)


def pref(**kw):
    a = dict(T=10, P=1, d=64, offsets=P, nll=P, loss=P, dh_nll=P, dh=P)
    a.update(kw)
    return lora.make_pref_args(**a)


@pytest.mark.parametrize("kw,want", [
    ({"T": 0}, lora.LORA_EINVAL), ({"P": 0}, lora.LORA_EINVAL), ({"P": (1 << 23) + 1}, lora.LORA_EINVAL),
    ({"d": 4}, lora.LORA_EINVAL), ({"kind": 3}, lora.LORA_EINVAL), ({"kind": -1}, lora.LORA_EINVAL),
    ({"beta": 0.0}, lora.LORA_EINVAL), ({"beta": float("nan")}, lora.LORA_EINVAL),
    ({"margin": float("inf")}, lora.LORA_EINVAL), ({"label_smoothing": 1.5}, lora.LORA_EINVAL),
    ({"label_smoothing": -0.5}, lora.LORA_EINVAL), ({"nll": None}, lora.LORA_ENULL), ({"loss": None}, lora.LORA_ENULL),
    ({"offsets": None}, lora.LORA_ENULL), ({"dh_nll": None}, lora.LORA_ENULL), ({"rewards": P + 2}, lora.LORA_EALIGN),
    ({"dh_nll": P + 4}, lora.LORA_EALIGN), ({"label_smoothing": 7.0, "kind": 1}, lora.LORA_OK)])
def test_pref_arguments(kw, want):
    assert code(lora.lora_pref_workspace_size, pref(**kw)) == want
    assert code(lora.lora_pref_fwd_bwd, pref(**kw), *WS, 0) == passed(want)


def test_loss_workspaces():
    for fn, size, args in ((lora.lora_policy_fwd_bwd, lora.lora_policy_workspace_size, policy()),
                           (lora.lora_pref_fwd_bwd, lora.lora_pref_workspace_size, pref())):
        n = size(args)
        assert n >= 10 * 4
        assert code(fn, args, P, n - 1, 0) == lora.LORA_EWORKSPACE
        assert code(fn, args, None, n, 0) == lora.LORA_EWORKSPACE
        assert code(fn, args, P + 16, n, 0) == lora.LORA_EALIGN
    assert lora.library().lora_policy_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == lora.LORA_ENULL
    assert lora.library().lora_pref_fwd_bwd(None, None, 0, None) == lora.LORA_ENULL


def grads(*entries):
    arr = (lora.lora_grad * len(entries))()
    for g, e in zip(arr, entries):
        g.src, g.dst, g.n, g.dtype = e
    return arr


@pytest.mark.parametrize("entry,want", [
    ((P, P, -1, 0), lora.LORA_EINVAL), ((P, P, 5, 2), lora.LORA_EINVAL), ((P, P, 1 << 39, 0), lora.LORA_EINVAL),
    ((None, P, 5, 0), lora.LORA_ENULL), ((P + 2, P, 5, 0), lora.LORA_EALIGN), ((P, P + 2, 5, 0), lora.LORA_EALIGN),
    ((P, P + 1, 5, 1), lora.LORA_EALIGN), ((P + 2, P, 5, 1), lora.LORA_OK), ((P, None, 5, 0), lora.LORA_OK),
    ((None, None, 0, 0), lora.LORA_OK)])
def test_clip_tensors(entry, want):
    arr = grads((P, P, 3, 0), entry)
    assert code(lora.lora_clip_grads, arr, 1.0, P, P, *WS, 0) == passed(want)


def test_clip_arguments():
    arr = grads((P, P, 100, 0))
    n = lora.lora_clip_workspace_size(arr)
    assert code(lora.lora_clip_grads, arr, -1.0, P, P, *WS, 0) == lora.LORA_EINVAL
    assert code(lora.lora_clip_grads, arr, float("nan"), P, P, *WS, 0) == lora.LORA_EINVAL
    assert code(lora.lora_clip_grads, arr, float("inf"), P, None, *WS, 0) == lora.LORA_EWORKSPACE
    assert code(lora.lora_clip_grads, arr, 1.0, None, P, *WS, 0) == lora.LORA_ENULL
    assert code(lora.lora_clip_grads, arr, 1.0, P + 2, P, *WS, 0) == lora.LORA_EALIGN
    assert code(lora.lora_clip_grads, arr, 1.0, P, P, P, n - 1, 0) == lora.LORA_EWORKSPACE
    m = ctypes.c_size_t(0)
    assert lora.library().lora_clip_workspace_size(arr, 0, ctypes.byref(m)) == lora.LORA_EINVAL
    assert lora.library().lora_clip_workspace_size(None, 1, ctypes.byref(m)) == lora.LORA_ENULL
    assert lora.library().lora_clip_workspace_size(arr, 65537, ctypes.byref(m)) == lora.LORA_EINVAL


def test_grads_are_of_one_size_and_type():
    import torch
    a = torch.zeros(4)
    with pytest.raises(TypeError):
        lora.make_grads([(a.double(), None)])
    for other in (torch.zeros(5), torch.zeros(4, dtype=torch.bfloat16), torch.zeros(8)[::2]):
        with pytest.raises(ValueError):
            lora.make_grads([(a, other)])
    with pytest.raises(ValueError):
        lora.make_grads([(torch.zeros(4, 4).t(), None)])
