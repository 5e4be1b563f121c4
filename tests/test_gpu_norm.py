"""GPU parity of the final RMS norm (forward and backward) against the fp64 oracle, element by element.

Tolerances, derived.  u = 2^-24 and b = 2^-8 are the largest relative errors of one rounding to fp32 and bf16.
  r      one fp32 addition: u |r|, and the rounding of its type
  s      a sum of squares is at most 64 additions in a lane, 5 in a warp and 16 of warps, of terms with 3 roundings: 88 u, half of
         that in the root, 4 u for mean, root and quotient: 48 u
  y      s, r and two products: 52 u |y|, then b |y|
  dx     a mean of products has 90 u of its terms' magnitudes, s^3 144 u, and the sums 4 u: 256 u of the magnitudes that dx adds
         up (oracle), then b |dx| where dx is bf16
  dgamma terms within 52 u; a block adds at most n / min(n, 592) + 1 rows in turn, the blocks' shares 592 / 16 + 17 in turn
"""
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
    return None if t is None else pu.bf16_bits(t) if t.dtype == B16 else t.cpu().numpy()


class Rows:
    def __init__(self, n, H, K=1, n_inv=3, res=B16, gamma=B16, mask=0.2, seed=0, x_scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.n, self.H, self.K = n, H, K
        cuts = torch.randint(0, n + 1, (n_inv - 1,), generator=g).sort().values
        self.cu = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])])
        self.role_model = list(range(K - 1, -1, -1)) + [0]
        self.role = torch.randint(0, K + 1, (n_inv,), generator=g).to(torch.int32)
        self.mask = (torch.rand(n, generator=g) >= mask).to(torch.uint8)
        scale = x_scale * (0.1 + 3 * torch.rand(n, 1, generator=g))
        self.x = (torch.randn(n, H, generator=g) * scale).to(B16)
        self.res = None if res is None else (torch.randn(n, H, generator=g) * scale * 2).to(res)
        self.dy = (torch.randn(n, H, generator=g) * 1e-2).to(B16)
        self.dres = (torch.randn(n, H, generator=g) * 1e-2).to(res or B16)
        self.gamma = [(1 + 0.5 * torch.randn(H, generator=g)).to(gamma) for _ in range(K)]
        self.eps = 1e-6

    def head(self):
        return ([w.cuda() for w in self.gamma], self.cu.cuda(), self.role.cuda(), self.role_model,
                None if self.mask is None else self.mask.cuda(), self.eps)

    def table(self):
        return (self.cu.numpy(), self.role.numpy(), self.role_model, None if self.mask is None else self.mask.numpy())


def check_fwd(p, y, r, want=None):
    wy, wr = want or orc.rms_norm_fwd(bits(p.x), bits(p.res), [bits(w) for w in p.gamma], *p.table(), float(np.float32(p.eps)))
    got = y.double().cpu().numpy()
    tol = (B + 53 * U) * np.abs(wy) + 1e-38
    assert np.all(np.abs(got - wy) <= tol), np.max(np.abs(got - wy) / tol)
    if r is not None:
        got = r.double().cpu().numpy()
        assert np.all(np.abs(got - wr) <= (U + (B if r.dtype == B16 else 0)) * (1 + U) * np.abs(wr) + 1e-38)


def check_bwd(p, r, dx, dgamma, dres=True, base=None):
    wx, wg, mx, mg = orc.rms_norm_bwd(bits(r), [bits(w) for w in p.gamma], *p.table(), float(np.float32(p.eps)), bits(p.dy),
                                      bits(p.dres) if dres else None)
    got = dx.double().cpu().numpy()
    tol = 256 * U * mx + (B if dx.dtype == B16 else U) * np.abs(wx) * (1 + 256 * U) + 1e-38
    assert np.all(np.abs(got - wx) <= tol), np.max(np.abs(got - wx) / tol)
    if dgamma is not None:
        chain = p.n / min(p.n, 592) + 592 / 16 + 18
        for k in range(p.K):
            old = 0.0 if base is None else base[k].double().cpu().numpy()
            tol = (52 + chain) * U * (mg[k] + np.abs(old)) + 1e-40
            err = np.abs(dgamma[k].double().cpu().numpy() - (wg[k] + old))
            assert np.all(err <= tol), (k, np.max(err / tol))


def junk(shape, dtype):
    return torch.full(shape, 7.0, dtype=dtype, device="cuda")


SIZES = [(1, 64), (1, 3584), (3, 16384), (5, 192), (37, 256), (64, 896), (130, 1536), (333, 2112), (700, 3584), (61, 5120),
         (29, 8256), (2001, 128)]


@pytest.mark.parametrize("n,H", SIZES)
@pytest.mark.parametrize("res,gamma", [(None, F32), (B16, B16), (F32, F32), (F32, B16)])
def test_forward(n, H, res, gamma):
    p = Rows(n, H, K=1 + n % 3, n_inv=1 + n % 9, res=res, gamma=gamma, seed=n + H)
    y, out = junk((n, H), B16), None if res is None else junk((n, H), res)
    ctx = ub.Context(0, 256)
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, None if res is None else p.res.cuda(), out)
    check_fwd(p, y, out)
    ctx.check_status()


@pytest.mark.parametrize("n,H", SIZES)
@pytest.mark.parametrize("res,gamma,dres", [(B16, F32, False), (B16, B16, True), (F32, B16, True)])
def test_backward(n, H, res, gamma, dres):
    K = 1 + n % 3
    p = Rows(n, H, K=K, n_inv=1 + n % 9, res=res, gamma=gamma, seed=n + H)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, K))
    ctx.workspace.fill_(0xff)
    dx, dg = junk((n, H), res), [junk((H,), F32) for _ in range(K)]
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda() if dres else None, dg)
    check_bwd(p, p.res, dx, dg, dres)
    # adding to what is there, and the frozen norm
    base = [w.clone() for w in dg]
    dx2 = junk((n, H), res)
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx2, p.dres.cuda() if dres else None, dg, True)
    check_bwd(p, p.res, dx2, dg, dres, base)
    frozen = junk((n, H), res)
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), frozen, p.dres.cuda() if dres else None)
    assert torch.equal(dx, dx2) and torch.equal(dx, frozen)
    ctx.check_status()


def test_many_short_invocations_change_the_model_within_a_block():
    n, H, K = 4001, 256, 5
    p = Rows(n, H, K=K, n_inv=1500, res=B16, seed=5)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, K))
    dx, dg = junk((n, H), B16), [junk((H,), F32) for _ in range(K)]
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), dg)
    check_bwd(p, p.res, dx, dg)
    again = [junk((H,), F32) for _ in range(K)]
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), again)
    assert all(torch.equal(a, b) for a, b in zip(dg, again))
    # a smaller workspace: fewer blocks, the same sums in another order
    small = ub.Context(0, ub.unity_rms_norm_workspace_bytes(7, H, K))
    small.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), again)
    wg = orc.rms_norm_bwd(bits(p.res), [bits(w) for w in p.gamma], *p.table(), 1e-6, bits(p.dy), bits(p.dres))
    for k in range(K):
        assert np.all(np.abs(again[k].double().cpu().numpy() - wg[1][k]) <= (52 + n) * U * wg[3][k])


def test_masked_rows_are_not_read_and_no_mask_is_all_rows():
    p = Rows(40, 320, K=2, res=F32, mask=0.5, seed=3)
    for t in (p.x, p.res, p.dy, p.dres):
        t[p.mask == 0] = float("nan")
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(40, 320, 2))
    y, r, dx, dg = junk((40, 320), B16), junk((40, 320), F32), junk((40, 320), F32), [junk((320,), F32) for _ in range(2)]
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, p.res.cuda(), r)
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), dg)
    off = (p.mask == 0).cuda()
    for t in (y, r, dx):
        assert torch.isfinite(t).all() and (t[off] == 0).all() and (t[~off] != 0).any()
    assert all(torch.isfinite(t).all() for t in dg)
    q = Rows(40, 320, K=2, res=F32, seed=3)
    q.mask = None
    ctx.rms_norm_fwd(q.x.cuda(), *q.head(), y, q.res.cuda(), r)
    check_fwd(q, y, r)
    # every row masked
    q.mask = torch.zeros(40, dtype=torch.uint8)
    ctx.rms_norm_fwd(q.x.cuda(), *q.head(), y, q.res.cuda(), r)
    ctx.rms_norm_bwd(q.res.cuda(), *q.head(), q.dy.cuda(), dx, q.dres.cuda(), dg)
    assert not y.any() and not r.any() and not dx.any() and not any(t.any() for t in dg)


def test_roles_out_of_range_are_flagged_and_masked():
    p = Rows(50, 128, K=2, n_inv=6, res=B16, seed=8)
    p.cu = torch.tensor([0, 10, 20, 20, 30, 41, 50])
    p.role = torch.tensor([0, 99, -5, 1, -1, 2], dtype=torch.int32)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(50, 128, 2))
    y, dx, dg = junk((50, 128), B16), junk((50, 128), B16), [junk((128,), F32) for _ in range(2)]
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, p.res.cuda())
    with pytest.raises(ub.UnityError) as e:
        ctx.check_status()
    assert e.value.code == -7
    check_fwd(p, y, None)
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), dg)
    with pytest.raises(ub.UnityError):
        ctx.check_status()
    check_bwd(p, p.res, dx, dg)


def test_outputs_may_be_the_inputs():
    p = Rows(70, 1088, K=2, res=B16, seed=4)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(70, 1088, 2))
    y, r = junk((70, 1088), B16), junk((70, 1088), B16)
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, p.res.cuda(), r)
    x, res = p.x.cuda(), p.res.cuda()
    ctx.rms_norm_fwd(x, *p.head(), x, res, res)
    assert torch.equal(x, y) and torch.equal(res, r)
    dx, dg = junk((70, 1088), B16), [junk((1088,), F32) for _ in range(2)]
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), dg)
    for which in range(3):
        ins = [p.res.cuda(), p.dy.cuda(), p.dres.cuda()]
        dg2 = [junk((1088,), F32) for _ in range(2)]
        ctx.rms_norm_bwd(ins[0], *p.head(), ins[1], ins[which], ins[2], dg2)
        assert torch.equal(ins[which], dx) and all(torch.equal(a, b) for a, b in zip(dg, dg2))


def test_zero_rows_large_values_and_no_tokens():
    p = Rows(6, 256, res=F32, seed=2, mask=0.0)
    p.x[0] = 0
    p.res[0] = 0
    p.res[1] = 3e17
    p.x[2] = float("inf")
    y, r = junk((6, 256), B16), junk((6, 256), F32)
    ctx = ub.Context(0, 1 << 20)
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, p.res.cuda(), r)
    assert not y[0].any() and torch.isnan(y[2]).any()
    p.x[2] = 0
    ctx.rms_norm_fwd(p.x.cuda(), *p.head(), y, p.res.cuda(), r)
    check_fwd(p, y, r)
    e = torch.empty(0, 256, dtype=B16, device="cuda")
    dg = [junk((256,), F32)]
    none = (torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), [0], None, 1e-6)
    ctx.rms_norm_fwd(e, p.head()[0], *none, e)
    ctx.rms_norm_bwd(e, p.head()[0], *none, e, e, None, dg, True)
    assert (dg[0] == 7).all()
    ctx.rms_norm_bwd(e, p.head()[0], *none, e, e, None, dg)
    assert not dg[0].any()


def test_refusals():
    p = Rows(8, 128, K=2, res=B16)
    ctx = ub.Context(0, 256)
    x, y = p.x.cuda(), junk((8, 128), B16)
    head = p.head()

    def code(fn, *a):
        with pytest.raises(ub.UnityError) as e:
            fn(*a)
        return e.value.code

    assert code(ctx.rms_norm_fwd, x, *head, y, None, y.clone()) == -1                   # res_out without residual
    assert code(ctx.rms_norm_fwd, x, *head[:3], [0, 5], *head[4:], y) == -1
    assert code(ctx.rms_norm_fwd, x, *head[:5], -1.0, y) == -1
    assert code(ctx.rms_norm_fwd, x, *head[:5], float("nan"), y) == -1
    assert code(ctx.rms_norm_fwd, x[:, :96].contiguous(), [w[:96].contiguous() for w in head[0]], *head[1:], y[:, :96].contiguous()) == -2
    off = torch.zeros(8 * 128 + 1, dtype=B16, device="cuda")[1:].view(8, 128)
    assert code(ctx.rms_norm_fwd, off, *head, y) == -3
    dg = [junk((128,), F32) for _ in range(2)]
    assert code(ctx.rms_norm_bwd, x, *head, x, y, None, dg) == -4                       # workspace of 256 bytes
    assert code(ctx.rms_norm_bwd, x, *head, x, y, None, [dg[0], dg[0]]) == -1
    for bad in (lambda: ctx.rms_norm_fwd(x.float(), *head, y), lambda: ctx.rms_norm_fwd(x, *head, y[:4]),
                lambda: ctx.rms_norm_fwd(x, [head[0][0], head[0][1].float()], *head[1:], y),
                lambda: ctx.rms_norm_fwd(x, *head, y, x.half()), lambda: ctx.rms_norm_bwd(x, *head, x, y.float()),
                lambda: ctx.rms_norm_bwd(x, *head, x, y, None, dg[:1]), lambda: ctx.rms_norm_fwd(x.t(), *head, y)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    ctx.rms_norm_fwd(x, *head, y)
    ctx.check_status()


def test_captured_and_replayed_on_a_stream_of_its_own():
    n, H, K = 90, 512, 2
    p, q = Rows(n, H, K=K, res=B16, seed=1), Rows(n, H, K=K, res=B16, seed=2)
    st = torch.cuda.Stream()
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, K), st)
    x, res, dy, head = p.x.cuda(), p.res.cuda(), p.dy.cuda(), p.head()
    y, r, dx, dg = junk((n, H), B16), junk((n, H), B16), junk((n, H), B16), [junk((H,), F32) for _ in range(K)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.rms_norm_fwd(x, *head, y, res, r)
        ctx.rms_norm_bwd(r, *head, dy, dx, None, dg)
    for w in (p, q):
        for a, b in zip((x, res, dy, head[1], head[2], head[4]), (w.x, w.res, w.dy, w.cu, w.role, w.mask)):
            a.copy_(b)
        for a, b in zip(head[0], w.gamma):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_fwd(w, y, r)
        check_bwd(w, r, dx, dg, False)


def test_offsets_beyond_32_bits():
    """n_tok * H above 2^31 elements: the last rows against the oracle."""
    H = 16384
    n = 2 ** 31 // H + 33
    cu = torch.tensor([0, n - 20, n], device="cuda")
    x = torch.randn(64, H, device="cuda").to(B16).repeat(n // 64 + 1, 1)[:n].contiguous()
    p = Rows(20, H, seed=6, mask=0.0)
    x[-20:] = p.x.cuda()
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[-20:] = 1
    y = torch.empty_like(x)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, 1))
    ctx.rms_norm_fwd(x, [p.gamma[0].cuda()], cu, torch.zeros(2, dtype=torch.int32, device="cuda"), [0], mask, 1e-6, y)
    p.cu, p.role, p.mask, p.res = torch.tensor([0, 20]), torch.zeros(1, dtype=torch.int32), None, None
    p.role_model = [0]
    check_fwd(p, y[-20:], None)
    assert not y[:64].any() and not y[-84:-20].any()
    y[-20:] = p.dy.cuda()
    dg = [junk((H,), F32)]
    ctx.rms_norm_bwd(x, [p.gamma[0].cuda()], cu, torch.zeros(2, dtype=torch.int32, device="cuda"), [0], mask, 1e-6, y, y, None, dg)
    check_bwd(p, p.x, y[-20:], None, False)
    wg = orc.rms_norm_bwd(bits(p.x), [bits(p.gamma[0])], *p.table(), 1e-6, bits(p.dy))
    assert np.all(np.abs(dg[0].double().cpu().numpy() - wg[1][0]) <= 200 * U * wg[3][0])
