"""Refusals of the training-side entry points: rejected on the host before any CUDA call (no GPU)."""
import ctypes
import math

import pytest

from paper_2606_00395_gb300 import binding as B
from paper_2606_00395_gb300 import build

P = ctypes.c_void_p(256)
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 6


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


def policy(lib, dm, **change):
    names = ("logits", "target", "weight", "advantage", "logp_old", "logp_ref", "loss", "logp", "entropy", "grad",
             "workspace")
    a = dict.fromkeys(names, P)
    a.update(change)
    size = a.pop("ws_bytes", 1 << 20)
    status = a.pop("status", None)
    return lib.pr2_policy_loss(ctypes.byref(dm), *[a[n] for n in names], ctypes.c_size_t(size), status, None)


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(V=0), dict(ld_logits=99), dict(ld_grad=99), dict(inv_temp=0.0), dict(inv_temp=-1.0),
    dict(inv_temp=math.nan), dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(kl_coef=-1.0),
    dict(kl_coef=math.inf), dict(grad_scale=math.nan), dict(flags=B.PR2_F_DELTA_LOSS)])
def test_policy_dims(lib, kw):
    dm = B.policy_dims(**{**dict(T=4, V=100), **kw})
    assert B.pr2_policy_loss_workspace_bytes(dm) == 0 and policy(lib, dm) == INVALID


def test_policy_arguments(lib):
    dm = B.policy_dims(4, 100)
    for n in ("logits", "target", "advantage", "loss"):
        assert policy(lib, dm, **{n: None}) == INVALID, n
    assert policy(lib, B.policy_dims(4, 100, kl_coef=0.1), logp_ref=None) == INVALID
    assert policy(lib, dm, logits=ctypes.c_void_p(257)) == INVALID
    assert policy(lib, B.policy_dims(4, 100, "fp32"), grad=ctypes.c_void_p(258)) == INVALID
    assert policy(lib, dm, target=ctypes.c_void_p(258)) == INVALID
    assert policy(lib, B.policy_dims(4, 100, flags=B.PR2_F_SYNC_STATUS)) == INVALID
    assert policy(lib, B.policy_dims(4, 100, ld_grad=101), grad=P, logits=P) == INVALID
    other = B.policy_dims(4, 100)
    other.dtype = 5
    assert policy(lib, other) == INVALID
    assert policy(lib, B.policy_dims(4, (1 << 30) + 1)) == UNSUPPORTED
    far = ctypes.c_void_p(1 << 20)
    for kw in (dict(workspace=None), dict(workspace=ctypes.c_void_p(128)), dict(ws_bytes=8)):
        assert policy(lib, dm, grad=far, **kw) == WORKSPACE
    with pytest.raises(B.Pr2Error):
        B.alloc_policy_workspace(B.policy_dims(4, 0))


@pytest.mark.parametrize("kw,code", [(dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(k=0), INVALID),
                                     (dict(k=17), INVALID), (dict(flags=0x80), INVALID), (dict(N=512), UNSUPPORTED),
                                     (dict(N=64, k=33), UNSUPPORTED), (dict(T=1 << 30), UNSUPPORTED)])
def test_token_dims(lib, kw, code):
    a = {**dict(T=4, d=64, N=16, k=2, m=1), **kw}
    dm = ctypes.byref(B.dims(**a))
    assert lib.pr2_token_sort_workspace_bytes(dm) == 0
    assert lib.pr2_token_sort(dm, P, P, P, P, P, P, P, ctypes.c_size_t(1 << 30), None, None) == code
    assert lib.pr2_token_sort_backward(dm, P, P, P, None) == code
    assert lib.pr2_token_unsort(dm, P, P, P, P, None) == code
    assert lib.pr2_token_unsort_backward(dm, P, P, P, P, P, P, P, None) == code
    assert lib.pr2_replay_gates_backward(dm, P, P, P, P, None, None) == code


def test_token_arguments(lib):
    d = B.dims(4, 63, 16, 2, 1)  # widths need not be even
    dm, big = ctypes.byref(d), ctypes.c_size_t(1 << 30)
    need = B.pr2_token_sort_workspace_bytes(d)
    assert need > 0
    sort = lambda *a, ws=P, size=big, status=None: lib.pr2_token_sort(dm, *a, ws, size, status, None)  # noqa: E731
    assert sort(P, P, None, P, P, P) == INVALID          # h without x
    assert sort(None, P, P, P, P, P) == INVALID
    assert sort(None, None, None, P, P, P) == INVALID    # neither a plan nor rows to make
    assert sort(P, P, P, None, P, P) == INVALID
    assert sort(P, P, P, P, None, P) == INVALID          # a plan that is made needs perm
    assert sort(P, P, P, P, P, None) == INVALID
    assert sort(ctypes.c_void_p(257), P, P, P, P, P) == INVALID
    assert sort(P, P, P, P, P, P, ws=None) == WORKSPACE
    assert sort(P, P, P, P, P, P, size=ctypes.c_size_t(need - 1)) == WORKSPACE
    assert sort(P, P, P, P, P, P, ws=ctypes.c_void_p(128)) == WORKSPACE
    for i in range(3):
        a = [P, P, P]
        a[i] = None
        assert lib.pr2_token_sort_backward(dm, *a, None) == INVALID
    for i in range(4):
        a = [P] * 4
        a[i] = None
        assert lib.pr2_token_unsort(dm, *a, None) == INVALID
        assert lib.pr2_replay_gates_backward(dm, *a, None, None) == INVALID
    for i in range(7):
        a = [P] * 7
        a[i] = None
        assert lib.pr2_token_unsort_backward(dm, *a, None) == INVALID
    with pytest.raises(B.Pr2Error):
        B.alloc_token_workspace(B.dims(4, 0, 16, 2, 1))
    sync = ctypes.byref(B.dims(4, 63, 16, 2, 1, flags=B.PR2_F_SYNC_STATUS))
    assert lib.pr2_token_sort(sync, P, P, P, P, P, P, P, big, None, None) == INVALID
    assert lib.pr2_replay_gates_backward(sync, P, P, P, P, None, None) == INVALID


@pytest.mark.parametrize("kw,code", [(dict(rows=-1), INVALID), (dict(m=0), INVALID), (dict(ld=63), INVALID),
                                     (dict(m=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED)])
def test_activation_dims(lib, kw, code):
    a = {**dict(rows=4, m=64, ld=64), **kw}
    dm = ctypes.byref(B.act_dims(a["rows"], a["m"], "bf16", a["ld"]))
    assert lib.pr2_swiglu_checkpoint(dm, P, P, P, P, P, None) == code
    assert lib.pr2_swiglu_checkpoint_backward(dm, P, P, P, P, P, P, None) == code


def test_activation_arguments(lib):
    dm = ctypes.byref(B.act_dims(4, 63))
    for i in range(5):
        a = [P] * 5
        a[i] = None
        assert lib.pr2_swiglu_checkpoint(dm, *a, None) == INVALID
        assert lib.pr2_swiglu_checkpoint_backward(dm, *a, P, None) == INVALID
    odd = ctypes.c_void_p(257)
    assert lib.pr2_swiglu_checkpoint(dm, odd, P, P, P, P, None) == INVALID
    assert lib.pr2_swiglu_checkpoint_backward(dm, P, P, P, P, P, odd, None) == INVALID


def test_empty_calls_do_nothing(lib):
    dm = ctypes.byref(B.dims(0, 64, 16, 2, 1))
    assert lib.pr2_token_sort_backward(dm, None, None, None, None) == 0
    assert lib.pr2_token_unsort(dm, None, None, None, None, None) == 0
    assert lib.pr2_token_unsort_backward(dm, *[None] * 7, None) == 0
    assert lib.pr2_replay_gates_backward(dm, *[None] * 4, None, None) == 0
    act = ctypes.byref(B.act_dims(0, 64))
    assert lib.pr2_swiglu_checkpoint(act, *[None] * 5, None) == 0
    assert lib.pr2_swiglu_checkpoint_backward(act, *[None] * 6, None) == 0
    assert lib.pr2_token_sort(dm, *[None] * 7, ctypes.c_size_t(0), None, None) == 1  # offsets are still written
