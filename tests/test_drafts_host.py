"""Host side of the drafted step's operators (no GPU): every refusal, which comes before any HIP
call; and their oracle against differences and brute force."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import drafts as ref
from oracle import rotary
from paper_2606_03077_amd import libra

INVAL, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 4096  # an aligned address that nothing here reads


def status(name, *args):
    return getattr(libra.load(), name)(*args)


@pytest.fixture()
def handles():
    lay = libra.libra_kv_layout_create(P, P, 10, 2)
    rot = libra.libra_rotary_create()
    yield lay, rot
    libra.libra_rotary_destroy(rot)
    libra.libra_kv_layout_destroy(lay)


MAP = dict(batch=3, prior=P, new=P, held=P, table=P, stride=4, free=P, capacity=9, num_free=P, depths=P,
           rows=5, slots=P, positions=P, starts=P, held_out=P, num_out=P, refused=P, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(batch=-1), INVAL), (dict(stride=-1), INVAL), (dict(capacity=-1), INVAL), (dict(rows=-1), INVAL),
    (dict(rows=2 ** 31), UNSUPPORTED), (dict(capacity=2 ** 31), UNSUPPORTED),
    (dict(batch=2 ** 30 + 1), UNSUPPORTED),
    *[({k: None}, INVAL) for k in ("prior", "new", "held", "table", "free", "num_free", "slots", "positions",
                                   "starts", "held_out", "num_out", "refused")],
    *[({k: P + 2}, INVAL) for k in ("prior", "new", "held", "table", "free", "num_free", "depths",
                                    "positions", "starts", "held_out", "num_out", "refused")],
    (dict(slots=P + 4), INVAL)])
def test_map_refuses(change, want):
    assert status("libra_kv_map", *dict(MAP, **change).values()) == want


ACCEPT = dict(layout=None, batch=3, prior=P, accepted=P, most=4, counts=P, table=P, stride=4, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(layout=0), INVAL), (dict(batch=-1), INVAL), (dict(most=-1), INVAL), (dict(stride=-1), INVAL),
    (dict(batch=2 ** 30), UNSUPPORTED), (dict(most=2 ** 30 + 1), UNSUPPORTED),
    *[({k: None}, INVAL) for k in ("prior", "accepted", "counts", "table")],
    *[({k: P + 2}, INVAL) for k in ("prior", "accepted", "counts", "table")],
    (dict(batch=0), 0), (dict(most=0), 0)])
def test_accept_refuses(handles, change, want):
    a = dict(dict(ACCEPT, layout=handles[0]), **change)
    assert status("libra_kv_accept", *a.values()) == want


HEADS = dict(x=P, x_row_stride=1024, x_head_stride=128, num_heads=4, weight=P, out=2 * P,
             out_row_stride=512, out_head_stride=128, grad=P, grad_row_stride=512, grad_head_stride=128,
             weight_grad=P)
NORM = dict(rotary=None, dtype=0, weight_dtype=0, eps=1e-6, positions=P, rows=5, dim=128)


def norm_status(handles, backward, change={}, q={}, k={}, ws=P, ws_bytes=1 << 30):
    a = dict(dict(NORM, rotary=handles[1]), **change)
    tensors = [None if t is None else ctypes.byref(libra.NormHeads(**dict(HEADS, weight_grad=g, **t)))
               for t, g in ((q, P), (k, 2 * P))]
    if backward:
        return status("libra_qk_norm_rotary_backward", *a.values(), *tensors, ws, ws_bytes, None)
    return status("libra_qk_norm_rotary", *a.values(), *tensors, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("change,want", [
    (dict(rotary=None), INVAL), (dict(dim=64), INVAL), (dict(dtype=3), UNSUPPORTED),
    (dict(weight_dtype=-1), UNSUPPORTED), (dict(eps=0.0), INVAL), (dict(eps=1e-39), INVAL), (dict(eps=-1.0), INVAL),
    (dict(eps=float("nan")), INVAL), (dict(eps=float("inf")), INVAL), (dict(rows=-1), INVAL),
    (dict(rows=2 ** 31), UNSUPPORTED), (dict(positions=None), INVAL)])
def test_norm_refuses(handles, backward, change, want):
    assert norm_status(handles, backward, change) == want


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("change,want", [
    (dict(num_heads=-1), INVAL), (dict(num_heads=65536), UNSUPPORTED), (dict(x=None), INVAL),
    (dict(out=None), INVAL), (dict(weight=None), INVAL), (dict(x=P + 1), INVAL), (dict(out=P + 1), INVAL),
    (dict(weight=P + 1), INVAL), (dict(x_row_stride=-1), INVAL), (dict(x_head_stride=-1), INVAL),
    (dict(out_row_stride=511), INVAL), (dict(out_head_stride=127), INVAL), (dict(out_row_stride=0), INVAL),
    (dict(x_row_stride=2 ** 60), INVAL), (dict(out=P), INVAL)])  # in place, other strides
def test_norm_refuses_tensors(handles, backward, which, change, want):
    assert norm_status(handles, backward, **{which: change}) == want


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("change,want", [
    (dict(grad=None), INVAL), (dict(grad=P + 1), INVAL), (dict(grad_row_stride=-1), INVAL),
    (dict(out=P, grad=P, x=3 * P, grad_row_stride=1024), INVAL)])
def test_norm_gradient_refuses_tensors(handles, which, change, want):
    assert norm_status(handles, True, **{which: change}) == want


def test_norm_gradient_refuses_workspaces(handles):
    need = libra.libra_qk_norm_rotary_workspace_bytes(5, 4, 4, 128)
    assert need > 0
    assert norm_status(handles, True, ws=None) == INVAL
    assert norm_status(handles, True, ws=P + 8) == INVAL
    assert norm_status(handles, True, ws_bytes=need - 1) == WORKSPACE
    same = [ctypes.byref(libra.NormHeads(**HEADS)) for _ in range(2)]
    assert status("libra_qk_norm_rotary_backward", *dict(NORM, rotary=handles[1]).values(), *same, P, need,
                  None) == INVAL


@pytest.mark.parametrize("backward", [False, True])
def test_norm_of_nothing(handles, backward):
    assert norm_status(handles, backward, q=None, k=None) == 0
    none = dict(num_heads=0, x=None, out=None, weight=None)
    assert norm_status(handles, backward, q=none, k=none) == 0
    if not backward:
        assert norm_status(handles, backward, dict(rows=0, positions=None)) == 0


APPEND = dict(layout=None, rotary=None, weight_dtype=0, eps=1e-6, positions=P, slots=P, rows=5, q=P,
              q_row=1024, hq=4, q_weight=P, k=P, k_row=1024, k_weight=P, v=P, v_row=1024, hkv=2,
              q_out=2 * P, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(layout=None), INVAL), (dict(rotary=None), INVAL), (dict(weight_dtype=9), UNSUPPORTED),
    (dict(eps=0.0), INVAL), (dict(eps=1e-39), INVAL), (dict(rows=-1), INVAL), (dict(rows=2 ** 31), UNSUPPORTED),
    (dict(q=None), INVAL), (dict(q_out=None), INVAL), (dict(q_weight=None), INVAL),
    (dict(k_weight=None), INVAL), (dict(k_weight=P + 1), INVAL), (dict(hkv=4), INVAL),
    (dict(slots=None), INVAL), (dict(positions=None), INVAL), (dict(k=None), INVAL), (dict(v=P + 8), INVAL),
    (dict(k_row=255), INVAL), (dict(v_row=128), INVAL), (dict(hq=0), INVAL), (dict(hq=65536), INVAL),
    (dict(q_row=511), INVAL), (dict(q_out=P + 8), INVAL), (dict(q_out=P), INVAL), (dict(rows=0), 0)])
def test_append_refuses(handles, change, want):
    a = dict(dict(APPEND, layout=handles[0], rotary=handles[1]), **change)
    assert status("libra_kv_append_norm", *a.values()) == want


def test_append_refuses_other_head_sizes(handles):
    rot = libra.libra_rotary_create(head_dim=64)
    a = dict(APPEND, layout=handles[0], rotary=rot)
    assert status("libra_kv_append_norm", *a.values()) == INVAL
    libra.libra_rotary_destroy(rot)


TREE = dict(layout=None, q=P, rows=5, prior=P, starts=P, mask=P, words=1, table=P, stride=4, batch=3, hq=4,
            scale=0.1, ws=P, ws_bytes=1 << 30, out=2 * P, lse=P, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(layout=None), INVAL), (dict(rows=-1), INVAL), (dict(batch=-1), INVAL), (dict(hq=0), INVAL),
    (dict(hq=5), INVAL), (dict(hq=34), UNSUPPORTED), (dict(rows=2 ** 30), UNSUPPORTED),
    (dict(scale=0.0), INVAL), (dict(scale=float("nan")), INVAL), (dict(scale=float("inf")), INVAL),
    (dict(words=0), INVAL), (dict(words=9), UNSUPPORTED), (dict(mask=None), INVAL), (dict(q=None), INVAL),
    (dict(out=None), INVAL), (dict(q=P + 8), INVAL), (dict(out=P + 8), INVAL), (dict(prior=None), INVAL),
    (dict(starts=None), INVAL), (dict(table=None), INVAL), (dict(stride=0), INVAL), (dict(ws=None), INVAL),
    (dict(ws=P + 128), INVAL), (dict(ws_bytes=1 << 20), WORKSPACE), (dict(rows=0), 0), (dict(batch=0), 0),
    (dict(out=P), INVAL), (dict(batch=2 ** 30 + 1), UNSUPPORTED),
    *[({k: P + 2}, INVAL) for k in ("prior", "starts", "mask", "table", "lse")]])
def test_tree_refuses(handles, change, want):
    a = dict(dict(TREE, layout=handles[0]), **change)
    assert status("libra_tree_attn", *a.values()) == want


def test_workspace_sizes_of_bad_arguments():
    assert libra.libra_tree_attn_workspace_bytes(1, 1, 5, 2) == 0
    assert libra.libra_tree_attn_workspace_bytes(-1, 1, 4, 2) == 0
    assert libra.libra_tree_attn_workspace_bytes(0, 0, 4, 2) > 0
    assert libra.libra_qk_norm_rotary_workspace_bytes(-1, 1, 1, 128) == 0


def test_tensors_of_other_devices_are_refused(handles, monkeypatch):
    """Before anything of them is used: on the CPU, theirs is not the current device."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    lay, rot = handles
    i = torch.zeros(4, dtype=torch.int32)
    x, w = torch.zeros((4, 2, 128), dtype=torch.bfloat16), torch.zeros(128, dtype=torch.bfloat16)
    for bad in (lambda: libra.libra_kv_map(i, i, i, i, 1, i, i[:1], None, i.long(), i, i, i, i[:1], i),
                lambda: libra.libra_kv_accept(lay, i, i[:, None], i, i, 1),
                lambda: libra.libra_qk_norm_rotary(rot, x, None, w, None, 1e-6, i, x, None),
                lambda: libra.libra_qk_norm_rotary_backward(rot, x, None, x, None, w, None, 1e-6, i, x, None,
                                                            None, None, None),
                lambda: libra.libra_kv_append_norm(lay, rot, i, i.long(), None, x, x, None, w, 1e-6, None),
                lambda: libra.libra_tree_attn(lay, x, i, i, None, i, 1, 2, 0.1, i, x)):
        with pytest.raises(ValueError, match="current device"):
            bad()


# --- the oracle ------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(interleaved=True, amplitude=1.25)])
def test_oracle_gradient_against_differences(kw):
    rng = np.random.default_rng(3)
    x, dy, w = rng.standard_normal((2, 3, 12)), rng.standard_normal((2, 3, 12)), rng.standard_normal(12)
    theta, pos = rotary.frequencies(8), [5, 900]
    dx, dw, _ = ref.norm_turn_grad(x, w, 1e-3, pos, theta, dy, **kw)
    loss = lambda x, w: float((ref.norm_turn(x, w, 1e-3, pos, theta, **kw)[0] * dy).sum())
    h = 1e-5  # central differences: error h^2 times a third derivative of order 1, rounding 1e-15 / h
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-7
    for i in range(12):
        e = np.zeros(12)
        e[i] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i]) < 1e-7


def test_oracle_attention_of_one_key_and_none():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 2, 8)), rng.standard_normal((2, 1, 8)), rng.standard_normal((2, 1, 8))
    out, lse, _, _ = ref.tree_attention(q, k, v, 0, np.array([[1, 0], [0, 0]], bool), 0.5)
    assert np.allclose(out[0], v[0]) and np.allclose(lse[0], 0.5 * q[0] @ k[0, 0])
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all()


def test_oracle_map_by_hand():
    out = ref.kv_map(prior=[16, 40, 0], new=[1, 0, 17], held=[1, 4, 0], rows=20, num_free=1,
                     table=[[5, 0, 0, 0], [6, 7, 8, 9], [0, 0, 0, 0]], free=[3, 0, 0, 0])
    assert out["refused"].tolist() == [0, 0, 1]      # 9 comes back; one page each for 0 and none for 2
    assert out["table"][0].tolist() == [5, 9, 0, 0] and out["num_free"] == 1
    assert out["held"].tolist() == [2, 3, 0] and out["starts"].tolist() == [0, 1, 1, 18]
    assert out["slots"].tolist() == [9 * 16] + [-1] * 19
    assert out["positions"].tolist() == [16] + list(range(17)) + [0, 0]
