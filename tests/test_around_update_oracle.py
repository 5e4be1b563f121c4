"""The oracle's final norm, clipping and sampling, pinned by differences, invariants and library special cases; host-side checks
of the calls that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub


def test_norm_backward_is_the_gradient_of_the_forward():
    rng = np.random.default_rng(1)
    cu, role, rm, mask = [0, 2, 2, 5], [0, 1, 1], [1, 0], np.array([1, 1, 0, 1, 1], np.uint8)
    x, w, res = rng.normal(size=(5, 6)), [rng.normal(size=6) for _ in range(2)], rng.normal(size=(5, 6))
    dy, dres = rng.normal(size=(5, 6)), rng.normal(size=(5, 6))

    def value(x, w):
        y, r = orc.rms_norm_fwd(x, res, w, cu, role, rm, mask, 1e-3)
        return (y * dy).sum() + (r * dres).sum()

    _, r = orc.rms_norm_fwd(x, res, w, cu, role, rm, mask, 1e-3)
    dx, dg, _, _ = orc.rms_norm_bwd(r, w, cu, role, rm, mask, 1e-3, dy, dres)
    h = 1e-6
    for i, j in ((0, 0), (1, 5), (2, 3), (3, 1), (4, 4)):
        up, down = x.copy(), x.copy()
        up[i, j] += h
        down[i, j] -= h
        assert abs((value(up, w) - value(down, w)) / (2 * h) - dx[i, j]) < 1e-7
    for k in range(2):
        up, down = [a.copy() for a in w], [a.copy() for a in w]
        up[k][2] += h
        down[k][2] -= h
        assert abs((value(x, up) - value(x, down)) / (2 * h) - dg[k][2]) < 1e-7


def test_norm_against_torch():
    x = torch.randn(4, 64, dtype=torch.float64)
    w = torch.randn(64, dtype=torch.float64)
    y, r = orc.rms_norm_fwd(x.numpy(), None, [w.numpy()], [0, 4], [0], [0], None, 1e-5)
    assert np.allclose(y, torch.nn.functional.rms_norm(x, (64,), w, 1e-5).numpy(), atol=1e-12) and np.array_equal(r, x.numpy())


def test_clip_against_torch():
    g = [torch.randn(7, 3), torch.randn(5), torch.randn(2)]
    p = [torch.zeros_like(t, requires_grad=True) for t in g]
    for a, b in zip(p, g):
        a.grad = b.clone()
    total = torch.nn.utils.clip_grad_norm_(p, 0.5)
    norm, coef, out = orc.clip_grad_norm([t.numpy() for t in g], [0, 0, 0], 2, [0.5, 1.0])
    assert abs(norm[0] - float(total)) < 1e-6 and norm[1] == 0 and coef[1] == 1
    for a, b in zip(p, out):
        assert np.allclose(a.grad.numpy(), b, atol=1e-6)


def test_sampling_frequencies_and_limits():
    z = np.log(np.array([0.1, 0.4, 0.05, 0.3, 0.15]))
    us = (np.arange(2000) + 0.5) / 2000
    got = np.bincount([orc.sample_row(z, 1.0, 0, 1.0, 0.0, u)[0] for u in us], minlength=5) / 2000
    assert np.allclose(got, np.exp(z), atol=1e-3)
    assert {orc.sample_row(z, 1.0, 0, 0.69, 0.0, u)[0] for u in us} == {1, 3}            # 0.4 + 0.3 reach 0.69
    assert {orc.sample_row(z, 1.0, 3, 1.0, 0.0, u)[0] for u in us} == {1, 3, 4}
    assert {orc.sample_row(z, 1.0, 0, 1.0, 0.35, u)[0] for u in us} == {1, 3, 4}         # 0.35 * 0.4 = 0.14
    t, lp, lk, n = orc.sample_row(z, 0.0, 0, 1.0, 0.0, 0.7)
    assert (t, n, lk) == (1, 1, 0.0) and abs(lp - np.log(0.4)) < 1e-12
    assert orc.sample_row(np.zeros(4), 1.0, 2, 1.0, 0.0, 0.6)[0] == 1                    # equal logits: by index
    assert orc.sample_row(np.array([np.nan, 0.0]), 1.0, 0, 1.0, 0.0, 0.6)[0] == -1


def test_workspace_sizes_and_null_contexts():
    lib = ub.load_library()
    assert 0 < ub.unity_rms_norm_workspace_bytes(1, 64, 1) < ub.unity_rms_norm_workspace_bytes(5000, 3584, 2) < 2 ** 26
    assert ub.unity_rms_norm_workspace_bytes(5000, 63, 2) == 0 and ub.unity_rms_norm_workspace_bytes(-1, 64, 2) == 0
    assert 0 < ub.unity_clip_grad_norm_workspace_bytes(0, 1) <= ub.unity_clip_grad_norm_workspace_bytes(5000, 16) < 2 ** 24
    assert ub.unity_clip_grad_norm_workspace_bytes(1, 17) == 0
    assert lib.unity_rms_norm_fwd(None, None, None, None, 0, None, None) == -1
    assert lib.unity_rms_norm_bwd(None, None, None, 0, None, None, None, None, 0) == -1
    assert lib.unity_clip_grad_norm(None, 0, None, 1, None, None, None) == -1
    assert lib.unity_sample(None, 0, 1, None, 0, 1, 1, None, None, None, None, None, None, None, None) == -1
    assert ctypes.sizeof(ub.unity_tensor) == 32 and ctypes.sizeof(ub.unity_sampling_rule) == 16


def test_python_layer_refuses_tensors_of_the_host():
    t = torch.zeros(4, 64, dtype=torch.bfloat16)
    cu, role = torch.tensor([0, 4]), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        ub.unity_rms_norm_fwd(None, t, [torch.ones(64)], cu, role, [0], None, 1e-6, t.clone())
    with pytest.raises(ValueError):
        ub.GradTensors([t], [0])
    with pytest.raises(ValueError):
        ub.GradTensors([t], [0, 1])
    with pytest.raises(TypeError):
        ub.GradTensors([t.half()], [0])
    with pytest.raises(ValueError):
        ub.unity_sample(None, torch.zeros(2, 8), [(1, 0, 1, 0)], torch.zeros(2), torch.zeros(2, dtype=torch.int32))
