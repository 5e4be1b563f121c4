"""Pins of the token losses' oracle (closed forms, finite differences, autograd) and the refusals of their binding that
need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub


def problem(seed=0, N=11, H=6, V=16, K=2, n_top=5):
    rng = np.random.default_rng(seed)
    cu = np.array([0, 3, 3, 8, N])
    return dict(hidden=rng.normal(size=(N, H)), W=[rng.normal(size=(V, H)) for _ in range(K)], cu_seqlens=cu,
                inv_role=np.array([0, 1, 1, 0]), role_model=np.array([0, K - 1]), target=rng.integers(0, V, N),
                tok_mask=(np.arange(N) % 4 != 2).astype(np.uint8), tok_weight=rng.normal(size=N)), rng


VARIANTS = [dict(), dict(label_smoothing=0.2), dict(z_loss=0.05), dict(label_smoothing=0.1, z_loss=0.01, inv_temperature=0.7),
            dict(kd=True), dict(kd=True, hard_coef=0.5, inv_temperature=1.3), dict(kd=True, logits=False, kd_coef=2.0)]


def run(p, kw, teacher):
    kw = {k: v for k, v in kw.items() if k not in ("kd", "logits")}
    return orc.token_loss_fwd_bwd(**p, teacher=teacher, **kw)


def teacher_of(p, kw, rng, V=16, n_top=5):
    if not kw.get("kd"):
        return None
    N = p["hidden"].shape[0]
    ids = rng.integers(-2, V, (N, n_top))
    ids[1] = -1
    vals = rng.normal(size=(N, n_top)) - (0 if kw.get("logits", True) else 2.5)
    return orc.teacher_rows(ids, vals, V, kw.get("logits", True), kw.get("inv_temperature", 1.0))


@pytest.mark.parametrize("kw", VARIANTS)
def test_gradients_match_differences_and_autograd(kw):
    p, rng = problem()
    q = teacher_of(p, kw, rng)
    o = run(p, kw, q)
    # differences of the summed losses, direction by direction
    for _ in range(4):
        dh, dw = rng.normal(size=p["hidden"].shape), [rng.normal(size=w.shape) for w in p["W"]]
        e = 1e-5
        hi = run({**p, "hidden": p["hidden"] + e * dh, "W": [w + e * d for w, d in zip(p["W"], dw)]}, kw, q)
        lo = run({**p, "hidden": p["hidden"] - e * dh, "W": [w - e * d for w, d in zip(p["W"], dw)]}, kw, q)
        want = (o["dHidden"] * dh).sum() + sum((a * b).sum() for a, b in zip(o["dW"], dw))
        assert abs((hi["loss"].sum() - lo["loss"].sum()) / (2 * e) - want) <= 1e-6 * (1 + abs(want))
    # autograd of torch's own log-softmax
    h = torch.tensor(p["hidden"], requires_grad=True)
    W = [torch.tensor(w, requires_grad=True) for w in p["W"]]
    total = 0.0
    for i in np.nonzero(o["on"])[0]:
        k = o["tok_model"][i]
        z = kw.get("inv_temperature", 1.0) * (W[k] @ h[i])
        lp, lse = torch.log_softmax(z, 0), torch.logsumexp(z, 0)
        y = int(p["target"][i])
        if q is None:
            eps = kw.get("label_smoothing", 0.0)
            l = torch.nn.functional.cross_entropy(z[None], torch.tensor([y]), label_smoothing=eps) + kw.get("z_loss", 0.0) * lse ** 2
        else:
            t = torch.tensor(q[i])
            l = kw.get("kd_coef", 1.0) * torch.nn.functional.kl_div(lp, t, reduction="sum") - kw.get("hard_coef", 0.0) * lp[y]
        assert abs(l.item() - o["tok_loss"][i]) <= 1e-12 * (1 + abs(l.item()))
        total = total + p["tok_weight"][i] * l / o["M"][k]
    total.backward()
    assert np.abs(h.grad.numpy() - o["dHidden"]).max() <= 1e-12
    assert all(np.abs(w.grad.numpy() - d).max() <= 1e-12 for w, d in zip(W, o["dW"]))


def test_closed_forms():
    p, _ = problem()
    p["W"] = [np.zeros_like(w) for w in p["W"]]
    o = run(p, dict(label_smoothing=0.3), None)
    assert np.allclose(o["tok_loss"][o["on"]], math.log(16), atol=1e-14)        # uniform model: log V whatever the smoothing
    assert np.all(o["tok_loss"][~o["on"]] == 0) and np.all(o["dHidden"][~o["on"]] == 0)
    p, rng = problem()
    own = orc.token_loss_fwd_bwd(**p)                                            # a teacher equal to the model: no loss, no gradient
    q = np.zeros_like(own["G"])
    for i in np.nonzero(own["on"])[0]:
        z = p["W"][own["tok_model"][i]] @ p["hidden"][i]
        q[i] = np.exp(z - own["lse"][i])
    o = orc.token_loss_fwd_bwd(**p, teacher=q)
    assert np.abs(o["tok_loss"]).max() < 1e-13 and np.abs(o["dHidden"]).max() < 1e-13


def test_teacher_rows():
    ids = np.array([[3, 1, 3, -1], [-1, -5, -1, -1], [0, 2, 5, 99], [4, 0, 1, 2]])
    vals = np.array([[0.0, 1.0, 2.0, 9.0], [1.0] * 4, [0.0, -np.inf, 1.0, 7.0], [-np.inf] * 4])
    q = orc.teacher_rows(ids, vals, 6, True)
    e = np.exp([0.0, 1.0, 2.0])
    assert np.allclose(q[0], [0, e[1] / e.sum(), 0, (e[0] + e[2]) / e.sum(), 0, 0])
    assert np.all(q[1] == 0) and np.all(q[3] == 0) and q[2, 2] == 0 and abs(q[2].sum() - 1) < 1e-15
    q = orc.teacher_rows(ids, np.log([[0.1, 0.2, 0.3, 1.0]] * 4), 6, False)
    assert np.allclose(q[0], [0, 0.2, 0, 0.4, 0, 0]) and abs(q[2].sum() - 0.6) < 1e-15


# ---------------------------------------------------------------------------- host side

def host_call(op="ce", **change):
    N, H, V, K, n_top = 5, 64, 16, 2, 3
    b16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    a = dict(hidden=torch.zeros(N, H, dtype=b16), W=[torch.zeros(V, H, dtype=b16)] * K, cu_seqlens=torch.tensor([0, 2, N]),
             inv_role=torch.zeros(2, dtype=i32), role_model=[0, 1], target=torch.zeros(N, dtype=i32),
             tok_mask=torch.ones(N, dtype=torch.uint8), inv_temperature=1.0, norm=None, accumulate_dW=False,
             tok_weight=torch.ones(N), loss=torch.zeros(K), tok_loss=torch.zeros(N), lse=torch.zeros(N),
             dHidden=torch.zeros(N, H, dtype=b16), dW=[torch.zeros(V, H, dtype=b16)] * K)
    if op == "ce":
        a.update(label_smoothing=0.0, z_loss=0.0)
    else:
        a.update(top_ids=torch.zeros(N, n_top, dtype=i32), top_vals=torch.zeros(N, n_top), teacher_mode=ub.TEACHER_LOGITS,
                 kd_coef=1.0, hard_coef=0.0)
    a.update(change)
    (ub.unity_cross_entropy_fwd_bwd if op == "ce" else ub.unity_distill_fwd_bwd)(None, **a)


@pytest.mark.parametrize("change,error", [
    (dict(target=torch.zeros(4, dtype=torch.int32)), ValueError), (dict(target=torch.zeros(5, dtype=torch.int64)), TypeError),
    (dict(tok_mask=torch.ones(6, dtype=torch.uint8)), ValueError), (dict(loss=torch.zeros(3)), ValueError),
    (dict(loss=None), ValueError), (dict(tok_weight=torch.ones(5, dtype=torch.float64)), TypeError),
    (dict(dW=[torch.zeros(16, 64)]), ValueError), (dict(dW=[torch.zeros(16, 64, dtype=torch.float16)] * 2), TypeError),
    (dict(dW=[torch.zeros(16, 64), torch.zeros(16, 64, dtype=torch.bfloat16)]), TypeError),
    (dict(dHidden=torch.zeros(5, 64)), TypeError), (dict(norm=[1.0]), ValueError), (dict(W=[]), ValueError),
    (dict(W=[torch.zeros(16, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)]), ValueError),
    (dict(cu_seqlens=torch.tensor([0, 5])), ValueError), (dict(hidden=torch.zeros(5, dtype=torch.bfloat16)), ValueError),
    (dict(), ValueError)])                                             # the last: CPU tensors
def test_binding_refuses(change, error):
    with pytest.raises(error):
        host_call("ce", **change)
    with pytest.raises(error):
        host_call("kd", **change)


@pytest.mark.parametrize("change,error", [
    (dict(top_ids=torch.zeros(5, 3, dtype=torch.int64)), TypeError), (dict(top_vals=torch.zeros(5, 4)), ValueError),
    (dict(top_ids=torch.zeros(4, 3, dtype=torch.int32)), ValueError), (dict(top_ids=torch.zeros(15, dtype=torch.int32)), ValueError)])
def test_distill_binding_refuses(change, error):
    with pytest.raises(error):
        host_call("kd", **change)


def test_null_context_and_workspace_queries():
    lib = ub.load_library()
    null = ctypes.c_void_p(None)
    assert lib.unity_cross_entropy_fwd_bwd(None, None, None, null, null, null, null, null, None) == -1
    assert lib.unity_distill_fwd_bwd(None, None, None, null, null, null, null, null, null, null, None) == -1
    size = ub.unity_token_loss_workspace_bytes
    assert 0 < size(1000, 256, 4096, 1, 0, False) < size(1000, 256, 4096, 1, 20, False) < size(1000, 256, 4096, 1, 20, True)
    assert size(-1, 256, 4096, 1) == 0 and size(10, 256, 4096, 1, 129) == 0 and size(10, 256, 4096, 1, -1) == 0
    assert size(1_000_000, 3584, 152064, 2) < 40 * 2 ** 30                       # bounded blocks whatever the batch
