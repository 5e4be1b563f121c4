"""GPU parity of the per-model gradient norm and clipping against the fp64 oracle.

Tolerances, derived.  u = 2^-24.  Eight squares are added in fp32 (one rounding of each product's sum: at most 8 u of the sum), all
else is fp64; the norm is the root of that (4 u) rounded to fp32 (u), the factor a quotient of the fp64 norm (4 u + u), an output one
product (u) rounded to its type (bf16 2^-8)."""
import numpy as np
import pytest
import torch

import parity_harness as pu
from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
F32, B16 = torch.float32, torch.bfloat16


def bits(t):
    return pu.bf16_bits(t) if t.dtype == B16 else t.cpu().numpy()


def clip(grads, models, K, max_norm, outs=None, ctx=None):
    ctx = ctx or ub.Context(0, ub.unity_clip_grad_norm_workspace_bytes(len(grads), K))
    ctx.workspace.fill_(0xff)
    norm, coef = torch.full((K,), 7.0, device="cuda"), torch.full((K,), 7.0, device="cuda")
    ctx.clip_grad_norm(ub.GradTensors(grads, models, outs), max_norm, norm, coef)
    ctx.check_status()
    return norm.double().cpu().numpy(), coef.double().cpu().numpy()


def check(before, models, K, max_norm, norm, coef, after):
    wn, wc, wo = orc.clip_grad_norm([bits(g) for g in before], models, K, max_norm)
    assert np.all(np.abs(norm - wn) <= 5.1 * U * wn), np.max(np.abs(norm / wn - 1)) / U
    assert np.all(np.abs(coef - wc) <= 5.1 * U * wc)
    for g, o, k, w in zip(before, after, models, wo):
        got = o.double().cpu().numpy()
        assert np.all(np.abs(got - w) <= (6.2 * U + (B * (1 + U * 8) if o.dtype == B16 else 0)) * np.abs(w) + 2.0 ** -133 * (o.dtype == B16)
                      + 2.0 ** -149), k
        if wc[k] == 1 and o.dtype == g.dtype:
            assert torch.equal(o, g)


def views(sizes, dtype, seed, gap=0, scale=1e-3):
    """Tensors behind one another in one bucket, `gap` elements apart: most of them at odd places."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(sum(sizes) + gap * len(sizes) + 1, generator=g, device="cuda").mul_(scale).to(dtype)
    at, out = 0, []
    for s in sizes:
        at += gap
        out.append(flat[at:at + s])
        at += s
    return flat, out


SIZES = [[1], [7, 8, 9], [0, 5, 0, 0, 8191, 8192, 8193, 0], [33, 65537, 1, 300001, 12, 16384], [3, 1000003, 257 * 129]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("dtype,out", [(F32, None), (B16, None), (F32, F32), (F32, B16), (B16, B16)])
@pytest.mark.parametrize("gap,out_gap", [(0, 0), (1, 0), (3, 2)])
def test_lists_of_ragged_tensors(sizes, dtype, out, gap, out_gap):
    K = 2
    flat, grads = views(sizes, dtype, 1, gap)
    before, whole = [g.clone() for g in grads], flat.clone()
    models = [i % 2 for i in range(len(sizes))]
    max_norm = [2e-4 * sum(sizes) ** 0.5, 1e3]
    outs = None
    if out is not None:
        bucket, outs = views(sizes, out, 2, out_gap)
        untouched = bucket.clone()
    norm, coef = clip(grads, models, K, max_norm, outs)
    check(before, models, K, max_norm, norm, coef, grads if outs is None else outs)
    # nothing outside the tensors is written
    marks = torch.ones_like(whole if outs is None else untouched, dtype=torch.bool)
    base = flat if outs is None else bucket
    for v in (grads if outs is None else outs):
        off = (v.data_ptr() - base.data_ptr()) // base.element_size()
        marks[off:off + v.numel()] = False
    assert torch.equal(base[marks], (whole if outs is None else untouched)[marks])
    if outs is not None:
        assert torch.equal(flat, whole)


def test_norms_only_write_nothing_else_and_models_without_tensors_have_none():
    flat, grads = views([100, 2000], F32, 3)
    whole = flat.clone()
    norm, coef = clip(grads, [2, 0], 4, None)
    assert torch.equal(flat, whole) and np.all(coef == 1) and norm[1] == 0 and norm[3] == 0
    wn, _, _ = orc.clip_grad_norm([bits(g) for g in grads], [2, 0], 4)
    assert np.all(np.abs(norm - wn) <= 5.1 * U * wn)
    norm, coef = clip([], [], 2, [1.0, 0.0])
    assert not norm.any() and np.all(coef == 1)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("scale", [1e-30, 1e-42, 3e30])
def test_tiny_and_huge_gradients(dtype, scale):
    g = (torch.randn(20011, dtype=torch.float64, generator=torch.Generator().manual_seed(1)) * scale).to(dtype).cuda()
    g[:4000] = 0
    before = g.clone()
    bound = [1e-3 * scale if scale > 1e-40 else 0.0]
    norm, coef = clip([g], [0], 1, bound)
    wn, wc, wo = orc.clip_grad_norm([bits(before)], [0], 1, bound)
    assert abs(norm[0] - wn[0]) <= 5.1 * U * wn[0] + 2.0 ** -149
    assert abs(coef[0] - wc[0]) <= 5.1 * U * wc[0]
    tol = (6.2 * U + (B if dtype == B16 else 0)) * np.abs(wo[0]) + 2.0 ** (-149 if dtype == F32 else -133)
    assert np.all(np.abs(g.double().cpu().numpy() - wo[0]) <= tol)


def test_mixed_sizes_within_a_vector():
    """A huge element among tiny ones, and the other way round: what fp32 squares would lose does not count, or is kept."""
    g = torch.full((64,), 1e-25, device="cuda")
    norm, _ = clip([g], [0], 1, None)
    assert abs(norm[0] - 8e-25) <= 8e-25 * 8 * U
    g[5] = 1e25
    norm, _ = clip([g], [0], 1, None)
    assert abs(norm[0] - 1e25) <= 1e25 * 6 * U


def test_norms_that_are_not_finite():
    g = torch.ones(1000, device="cuda")
    g[3] = float("inf")
    h = torch.ones(1000, device="cuda")
    h[999] = float("nan")
    ok = torch.ones(1000, device="cuda")
    norm, coef = clip([g, h, ok], [0, 1, 2], 3, [1.0, 1.0, 1.0])
    assert norm[0] == np.inf and coef[0] == 0 and np.isnan(norm[1]) and np.isnan(coef[1]) and abs(coef[2] - 1000 ** -0.5) < 1e-7
    assert torch.isnan(h).all() and torch.isnan(g[3]) and not g[4:].any() and torch.isfinite(ok).all()


def test_a_bound_of_zero_and_of_infinity():
    g, h = torch.randn(513, device="cuda"), torch.randn(513, device="cuda")
    keep = h.clone()
    norm, coef = clip([g, h], [0, 1], 2, [0.0, float("inf")])
    assert not g.any() and torch.equal(h, keep) and coef[0] == 0 and coef[1] == 1


@pytest.mark.parametrize("n", [64, 65, 800, 801, 1700])
def test_many_tensors(n):
    """One launch's table holds 64 or 800 tensors; the norm is over all launches."""
    rng = np.random.default_rng(n)
    sizes = [int(s) for s in rng.integers(0, 600, n)]
    _, grads = views(sizes, B16, n, 1)
    before = [g.clone() for g in grads]
    models = [int(m) for m in rng.integers(0, 3, n)]
    bound = [0.001 * 300 ** 0.5, 1e-4, 1e4]
    norm, coef = clip(grads, models, 3, bound)
    wn, wc, wo = orc.clip_grad_norm([bits(g) for g in before], models, 3, bound)
    assert np.all(np.abs(norm - wn) <= 5.1 * U * wn) and np.all(np.abs(coef - wc) <= 5.1 * U * wc)
    for g, w in zip(grads, wo):
        assert np.all(np.abs(g.double().cpu().numpy() - w) <= (B + 8 * U) * np.abs(w) + 2.0 ** -133)


def test_refusals():
    ctx = ub.Context(0, ub.unity_clip_grad_norm_workspace_bytes(3, 2))
    flat = torch.randn(1000, device="cuda")
    other = torch.randn(1000, device="cuda")
    norm = torch.zeros(2, device="cuda")

    def code(grads, models, bound, outs=None, norm=norm):
        with pytest.raises(ub.UnityError) as e:
            ctx.clip_grad_norm(ub.GradTensors(grads, models, outs), bound, norm)
        return e.value.code

    keep = flat.clone()
    assert code([flat, flat], [0, 0], [1.0, 1.0]) == -1                                 # the same tensor twice
    assert code([flat[:600], flat[500:]], [0, 1], [1.0, 1.0]) == -1                     # overlapping tensors
    assert code([flat[:500], flat[500:]], [0, 1], [1.0, 1.0], [None, flat[100:600]]) == -1
    assert code([flat[:500], flat[500:]], [0, 1], [1.0, 1.0], [other[:500], other[499:999]]) == -1
    assert code([flat], [2], [1.0, 1.0]) == -1
    assert code([flat], [0], [-1.0, 1.0]) == -1
    assert code([flat], [0], [float("nan"), 1.0]) == -1
    b = torch.randn(10, device="cuda").to(B16)
    assert code([b], [0], [1.0, 1.0], [torch.empty(10, device="cuda")]) == -1           # bf16 to f32
    assert code([flat] * 1000, [0] * 1000, None) == -4
    assert code([flat], [0], [1.0] * 17, norm=torch.zeros(17, device="cuda")) == -2
    assert torch.equal(flat, keep)
    # the same tensor twice is no fault where nothing is written, nor is one input with two outputs
    ctx.clip_grad_norm(ub.GradTensors([flat, flat], [0, 0]), None, norm)
    ctx.clip_grad_norm(ub.GradTensors([flat, flat], [0, 1], [other, torch.empty_like(flat)]), [1.0, 1.0], norm)
    ctx.check_status()
    for bad in (lambda: ub.GradTensors([flat[::2]], [0]), lambda: ub.GradTensors([flat.cpu()], [0]), lambda: ub.GradTensors([flat], [0, 1]),
                lambda: ctx.clip_grad_norm(ub.GradTensors([flat], [0]), [1.0], norm)):
        with pytest.raises((ValueError, TypeError)):
            bad()


def test_captured_and_replayed():
    st = torch.cuda.Stream()
    ctx = ub.Context(0, ub.unity_clip_grad_norm_workspace_bytes(70, 2), st)
    _, grads = views([1 + 997 * i for i in range(70)], F32, 4, 1)
    outs = [torch.empty_like(g) for g in grads]
    models = [i % 2 for i in range(70)]
    norm, coef = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    handle = ub.GradTensors(grads, models, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.clip_grad_norm(handle, [0.1, 1e9], norm, coef)
    for scale in (1.0, 3.0):
        for g in grads:
            g.mul_(scale)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(grads, models, 2, [0.1, 1e9], norm.double().cpu().numpy(), coef.double().cpu().numpy(), outs)


def test_more_than_32_bits_of_elements():
    n = 2 ** 31 + 4099
    g = torch.full((n,), 2.0 ** -10, dtype=B16, device="cuda")
    g[-1] = 3.0
    norm, coef = clip([g], [0], 1, [1.0])
    want = np.sqrt((n - 1) * 2.0 ** -20 + 9.0)
    assert abs(norm[0] - want) <= 5.1 * U * want and abs(coef[0] * want - 1) <= 6 * U
    for i, v in ((0, 2.0 ** -10), (2 ** 31 + 5, 2.0 ** -10), (n - 1, 3.0)):
        assert abs(g[i].item() - v / want) <= B * v / want
