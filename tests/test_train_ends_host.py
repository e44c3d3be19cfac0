"""Refusals of the loss, norm and clipping calls: each returns its status before anything touches a GPU
(device pointers are made up and never read)."""
import ctypes

import pytest

from paper_2609_08189_amd import hero as H
from tests.test_abi_host import FAKE, good_dims

GB = 1 << 30
V, T = 1000, 37


def at(i):
    return FAKE + i * 8 * GB


def size(f, *a):
    n = ctypes.c_size_t(0)
    return getattr(H.lib(), f)(*a, ctypes.byref(n)), n.value


def loss(dims=None, vocab=V, T=T, x=at(1), w=at(2), w_t=at(3), y=at(4), red=H.HERO_LOSS_MEAN, scale=1.0, loss=at(5),
         token=at(6), dx=at(7), dw=at(8), ws=at(9), ws_bytes=None, head=True, out=True):
    dims = dims or good_dims()
    if ws_bytes is None:
        ws_bytes = size("hero_lm_loss_workspace_size", ctypes.byref(dims), vocab, T, int(dx is not None), int(dw is not None))[1]
    return H.hero_lm_loss(dims, vocab, T, x, H.hero_lm_head(w, w_t) if head else None, y, red, scale,
                          H.hero_lm_loss_out(loss, token, dx, dw) if out else None, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(vocab=0), H.HERO_E_DIM), (dict(T=0), H.HERO_E_DIM), (dict(T=-3), H.HERO_E_DIM),
    (dict(vocab=64), H.HERO_E_UNSUPPORTED), (dict(vocab=4194241), H.HERO_E_UNSUPPORTED),
    (dict(T=(1 << 24) + 1), H.HERO_E_UNSUPPORTED), (dict(T=1 << 23), H.HERO_E_UNSUPPORTED),   # x spans 8 GiB
    (dict(dims=good_dims(d=8192), vocab=262144), H.HERO_E_UNSUPPORTED),                     # w_t spans 4 GiB
    (dict(red=2), H.HERO_E_RANGE), (dict(red=-1), H.HERO_E_RANGE),
    (dict(scale=float("nan")), H.HERO_E_RANGE), (dict(scale=float("inf")), H.HERO_E_RANGE),
    (dict(x=None), H.HERO_E_NULL), (dict(w=None), H.HERO_E_NULL), (dict(w_t=None), H.HERO_E_NULL),
    (dict(y=None), H.HERO_E_NULL), (dict(loss=None), H.HERO_E_NULL), (dict(head=False), H.HERO_E_NULL),
    (dict(out=False), H.HERO_E_NULL),
    (dict(x=at(1) + 8), H.HERO_E_ALIGN), (dict(y=at(4) + 4), H.HERO_E_ALIGN), (dict(dw=at(8) + 2), H.HERO_E_ALIGN),
    (dict(token=at(6) + 4), H.HERO_E_ALIGN), (dict(ws=at(9) + 8), H.HERO_E_ALIGN),
    (dict(ws=None), H.HERO_E_WORKSPACE), (dict(ws_bytes=1000), H.HERO_E_WORKSPACE),
    (dict(dx=at(1)), H.HERO_E_ALIAS), (dict(dw=at(2)), H.HERO_E_ALIAS), (dict(token=at(4)), H.HERO_E_ALIAS),
    (dict(ws=at(3)), H.HERO_E_ALIAS), (dict(dx=at(9) + 4096), H.HERO_E_ALIAS), (dict(dx=at(8)), H.HERO_E_ALIAS),
    (dict(dims=good_dims(dtype=5)), H.HERO_E_DTYPE),
])
def test_loss_refusals(change, status):
    assert loss(**change) == status


def test_loss_takes_what_it_documents_up_to_the_device_check():
    """The widest calls pass every host check: on a machine without a GPU they end at the device."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up pointers stay off a GPU")
    for change in [dict(), dict(dx=None, w_t=None), dict(dw=None), dict(dx=None, dw=None, token=None, w_t=None), dict(vocab=65),
                   dict(dims=good_dims(H.HERO_F32), vocab=3), dict(dims=good_dims(d=8192), vocab=300000, dx=None),
                   dict(red=H.HERO_LOSS_SUM, scale=0.0), dict(T=100000)]:
        assert loss(**change) == H.HERO_E_DEVICE, change


def test_loss_workspace_sizes():
    d = good_dims(d=4096)
    get = lambda *a: size("hero_lm_loss_workspace_size", ctypes.byref(d), *a)  # noqa: E731
    sizes = {k: get(128256, 4096, *k) for k in [(0, 0), (1, 0), (0, 1), (1, 1)]}
    assert all(st == H.HERO_OK for st, _ in sizes.values())
    assert sizes[0, 0][1] < sizes[1, 0][1] < sizes[1, 1][1] and sizes[0, 0][1] < sizes[0, 1][1] < sizes[1, 1][1]
    # the logits of the call are 2 GiB in fp32: no form of it keeps them, or half as many
    assert sizes[1, 1][1] < 4096 * 128256 * 2
    assert get(128256, 4096, 1, 0)[1] <= (7 << 27) and get(0, 4096, 1, 0)[0] == H.HERO_E_DIM
    assert H.lib().hero_lm_loss_workspace_size(ctypes.byref(d), 1000, 5, 1, 1, None) == H.HERO_E_NULL


@pytest.mark.parametrize("change,status", [
    (dict(vocab=-1), H.HERO_E_DIM), (dict(w=None), H.HERO_E_NULL), (dict(w_t=None), H.HERO_E_NULL),
    (dict(w_t=at(2) + 4), H.HERO_E_ALIGN), (dict(w_t=at(1) + 1024), H.HERO_E_ALIAS), (dict(vocab=1), H.HERO_E_UNSUPPORTED),
])
def test_head_weights_refusals(change, status):
    a = {**dict(vocab=V, w=at(1), w_t=at(2)), **change}
    assert H.hero_lm_head_weights_make(good_dims(), a["vocab"], a["w"], a["w_t"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=0), H.HERO_E_DIM), (dict(h=None), H.HERO_E_NULL), (dict(w=None), H.HERO_E_NULL), (dict(x=None), H.HERO_E_NULL),
    (dict(h=at(1) + 2), H.HERO_E_ALIGN), (dict(x=at(1) + 16), H.HERO_E_ALIAS), (dict(x=at(2)), H.HERO_E_ALIAS),
    (dict(dims=good_dims(d=33024)), H.HERO_E_UNSUPPORTED), (dict(dims=good_dims(d=640)), H.HERO_E_UNSUPPORTED),
])
def test_final_norm_refusals(change, status):
    a = {**dict(dims=good_dims(), T=T, h=at(1), w=at(2), x=at(3)), **change}
    assert H.hero_final_norm(a["dims"], a["T"], a["h"], a["w"], a["x"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=0), H.HERO_E_DIM), (dict(dx=None), H.HERO_E_NULL), (dict(dh=None), H.HERO_E_NULL), (dict(ws=None), H.HERO_E_WORKSPACE),
    (dict(n=16), H.HERO_E_WORKSPACE), (dict(dw=at(5) + 4), H.HERO_E_ALIGN), (dict(dh=at(2)), H.HERO_E_ALIAS),
    (dict(dh=at(1)), H.HERO_E_ALIAS), (dict(ws=at(4)), H.HERO_E_ALIAS), (dict(dw=at(6)), H.HERO_E_ALIAS),
    (dict(dims=good_dims(d=33024)), H.HERO_E_UNSUPPORTED),
])
def test_final_norm_backward_refusals(change, status):
    a = {**dict(dims=good_dims(), T=T, h=at(1), dx=at(2), w=at(3), dh=at(4), dw=at(5), ws=at(6), n=1 << 24), **change}
    assert H.hero_final_norm_backward(a["dims"], a["T"], a["h"], a["dx"], a["w"], a["dh"], a["dw"], a["ws"], a["n"],
                                      None) == status


def test_most_tokens():
    """The limit on the tokens, where the spans of the arrays allow more."""
    most, f32 = 4194240, good_dims(H.HERO_F32)
    assert loss(dims=good_dims(d=256), T=most + 1) == loss(dims=f32, T=most + 1) == H.HERO_E_UNSUPPORTED
    assert size("hero_lm_loss_workspace_size", ctypes.byref(f32), V, most, 1, 1)[0] == H.HERO_OK
    assert size("hero_lm_loss_workspace_size", ctypes.byref(good_dims(d=256)), V, most, 1, 1)[0] == H.HERO_OK
    assert size("hero_final_norm_backward_workspace_size", ctypes.byref(f32), most + 1)[0] == H.HERO_E_UNSUPPORTED
    assert H.hero_final_norm(f32, most + 1, at(1), at(2), at(3), None) == H.HERO_E_UNSUPPORTED


F, B = H.HERO_F32, H.HERO_BF16


@pytest.mark.parametrize("items,change,status", [
    ([], {}, H.HERO_E_DIM),
    (4097 * [(at(1), at(1), 0, F)], {}, H.HERO_E_UNSUPPORTED),
    ([(at(1), at(1), (1 << 36) + 1, F)], {}, H.HERO_E_UNSUPPORTED),
    ([(at(1), at(1), 5, 2)], {}, H.HERO_E_DTYPE),
    ([(None, at(1), 5, F)], {}, H.HERO_E_NULL), ([(at(1), None, 5, F)], {}, H.HERO_E_NULL),
    ([(at(1) + 2, at(2), 5, F)], {}, H.HERO_E_ALIGN), ([(at(1), at(2) + 1, 5, B)], {}, H.HERO_E_ALIGN),
    ([(at(1), at(1), 5, F)], dict(max_norm=-1.0), H.HERO_E_RANGE), ([(at(1), at(1), 5, F)], dict(max_norm=float("nan")), H.HERO_E_RANGE),
    ([(at(1), at(1), 5, F)], dict(norm=None), H.HERO_E_NULL), ([(at(1), at(1), 5, F)], dict(norm=at(20) + 4), H.HERO_E_ALIGN),
    ([(at(1), at(1), 5, F)], dict(ws=None), H.HERO_E_WORKSPACE), ([(at(1), at(1), 5, F)], dict(n=100), H.HERO_E_WORKSPACE),
    ([(at(1), at(1) + 16, 5, F)], {}, H.HERO_E_ALIAS),                              # half over itself
    ([(at(1), at(1), 5, F), (at(1), at(2), 5, F)], {}, H.HERO_E_ALIAS),             # read while it is scaled
    ([(at(1), at(1), 5, F), (at(2), at(2), 5, F), (at(1), at(1), 5, F)], {}, H.HERO_E_ALIAS),   # scaled twice
    ([(at(1), at(2), 100, F), (at(3), at(2) + 396, 100, B)], {}, H.HERO_E_ALIAS),
    ([(at(1), at(20), 100, F)], {}, H.HERO_E_ALIAS), ([(at(21), at(2), 100, F)], {}, H.HERO_E_ALIAS),
])
def test_clip_refusals(items, change, status):
    a = {**dict(max_norm=1.0, norm=at(20), ws=at(21), n=1 << 20), **change}
    assert H.hero_grad_clip(H.hero_grad_tensors(items), a["max_norm"], a["norm"], a["ws"], a["n"], None) == status


def test_clip_and_norm_take_what_they_document_up_to_the_device_check():
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up pointers stay off a GPU")
    ok = [[(at(1), at(1), 5, F), (at(1) + 20, at(1) + 20, 3, B)], [(at(1), at(2), 7, F), (at(1), at(3), 7, F)],
          [(None, None, 0, F), (at(1) + 4, at(2) + 12, 9, F)], [(at(1) + 4 * i, at(1) + 4 * i, 1, F) for i in range(4096)]]
    for items in ok:
        t = H.hero_grad_tensors(items)
        n = H.hero_grad_norm_workspace_size(t)
        assert H.hero_grad_clip(t, 1.0, at(20), at(21), n, None) == H.HERO_E_DEVICE
        assert H.hero_grad_norm(t, at(20), at(21), n, None) == H.HERO_E_DEVICE
    same = H.hero_grad_tensors(2 * [(at(1), None, 5, F)])   # read twice, written nowhere
    assert H.hero_grad_norm(same, at(20), at(21), 1 << 20, None) == H.HERO_E_DEVICE
    assert H.hero_grad_norm(same, at(1), at(21), 1 << 20, None) == H.HERO_E_ALIAS
