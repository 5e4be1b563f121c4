"""Calls at the ends of what the norm, the clipping and the sampling accept: rows far from zero, contexts of several host threads,
captured calls of different sizes."""
import threading

import numpy as np
import pytest
import torch

import test_gpu_norm as tn
import test_gpu_sample as ts
from paper_2605_26646_b200 import binding as ub

pytestmark = pytest.mark.gpu

F32, B16 = torch.float32, torch.bfloat16


# ------------------------------------------------------------------------------------------------
# Rows whose largest logit is so far from zero that its share of an octave has no digits left, or none of its octaves: a mask that refuses
# everything leaves such a row.  Tokens, numbers of kept entries and log-probabilities (tolerance of test_gpu_sample.py).
# ------------------------------------------------------------------------------------------------
def far_rows(V, dtype, n):
    """n rows, one kind after another."""
    lowest, largest = torch.finfo(dtype).min, torch.finfo(dtype).max
    g = torch.Generator(device="cuda").manual_seed(V)
    rows = []
    for i in range(n):
        kind = i % 9
        if kind < 5:
            row = torch.full((V,), (-1e9, lowest, 1e9, largest, -1e30)[kind], device="cuda")
        elif kind == 5:                                              # some entries are not allowed at all
            row = torch.full((V,), lowest, device="cuda")
            row[torch.rand(V, generator=g, device="cuda") < 0.3] = -float("inf")
            row[V // 2] = lowest
        elif kind == 6:                                              # the largest stands alone
            row = torch.full((V,), -1e9, device="cuda")
            row[V // 3] = 1e9
        elif kind == 7:                                              # a few equal ones above ordinary logits
            row = torch.randn(V, generator=g, device="cuda") * 3
            row[::1 + V // 3] = 2e9
        else:                                                        # neighbours of one another around 2^20 octaves
            row = 726817.0 + torch.randn(V, generator=g, device="cuda").mul_(3).round_()
        rows.append(row)
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("V,n", [(1, 27), (7, 27), (64, 700), (513, 27), (20481, 18), (20481, 297), (151936, 9), (262144, 9), (151936, 45)])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_greedy_rows_far_from_zero(V, n, dtype):
    z = far_rows(V, dtype, n)
    u = torch.rand(n, generator=torch.Generator().manual_seed(n)).cuda()
    ctx = ub.Context(0, 256)
    rule = (0.0, 0, 1.0, 0.0)
    got = ts.draw(z, [rule], u, None, None, ctx)
    assert np.all(got[2] == 0) and np.all(got[3] == 1)
    ts.check(z, [rule], u, None, got)
    ctx.check_status()


@pytest.mark.parametrize("V,n", [(7, 72), (513, 72), (20481, 72), (20481, 297), (151936, 36)])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_every_rule_on_rows_far_from_zero(V, n, dtype):
    rules = [(0.0, 0, 1.0, 0.0), ts.OFF, (0.7, 20, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.02), (1.0, 700, 0.5, 0.0), (1e-6, 0, 0.9, 0.0),
             (1e6, 5, 1.0, 0.1)]
    z = far_rows(V, dtype, n)
    role = torch.arange(n, dtype=torch.int32) // 9 % len(rules)
    u = torch.rand(n, generator=torch.Generator().manual_seed(n)).cuda()
    ctx = ub.Context(0, 256)
    ts.check(z, rules, u, role, ts.draw(z, rules, u, role.cuda(), None, ctx))
    ctx.check_status()


# ------------------------------------------------------------------------------------------------
# Norm backward: s and its powers lie far from 1, all that the definition gives lies within fp32 (tolerances of test_gpu_norm.py).
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H", [64, 896, 3584])
@pytest.mark.parametrize("res", [F32, B16])
@pytest.mark.parametrize("x_scale,eps", [(2e16, 1e-6), (2e16, 0.0), (1e13, 1e-6), (1e8, 0.0), (1e-9, 0.0), (1e-14, 0.0), (1e-17, 0.0), (1e-14, 1e-30)])
@pytest.mark.parametrize("dy_scale", [1.0, 1e-8])
def test_backward_of_large_and_of_tiny_rows(H, res, x_scale, eps, dy_scale):
    n = 40
    p = tn.Rows(n, H, K=2, n_inv=5, res=res, gamma=F32, seed=H, x_scale=x_scale)
    p.eps = eps
    p.dy = (p.dy.float() * dy_scale).to(B16)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, 2))
    dx, dg = tn.junk((n, H), res), [tn.junk((H,), F32) for _ in range(2)]
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, None, dg)
    assert torch.isfinite(dx.float()).all()
    tn.check_bwd(p, p.res, dx, dg, False)
    ctx.check_status()


# ------------------------------------------------------------------------------------------------
# Contexts of several host threads share nothing: calls of one size do not change what another's may ask for.
# ------------------------------------------------------------------------------------------------
def norm_bwd_call(n, H, res, dres, stream):
    p = tn.Rows(n, H, K=2, n_inv=3, res=res, seed=n)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, 2), stream)
    r, head, dy, more = p.res.cuda(), p.head(), p.dy.cuda(), p.dres.cuda() if dres else None
    dx, dg = tn.junk((n, H), res), [tn.junk((H,), F32) for _ in range(2)]
    return ctx, lambda: ctx.rms_norm_bwd(r, *head, dy, dx, more, dg), [dx, *dg]


def sample_call(n, V, stream):
    ctx = ub.Context(0, 256, stream)
    z, u = ts.logits(n, V, "peaked", F32, V), torch.rand(n, generator=torch.Generator().manual_seed(V)).cuda()
    token, logp = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    return ctx, lambda: ctx.sample(z, [(0.9, 40, 0.9, 0.0)], u, token, None, None, logp), [token, logp]


PAIRS = {"norm": (lambda st: norm_bwd_call(8, 3584, F32, True, st), lambda st: norm_bwd_call(8, 3584, F32, False, st)),
         "sample": (lambda st: sample_call(1, 152064, st), lambda st: sample_call(1, 4096, st))}


class Tape:
    """The library with its last call kept, so that a loop can make it again without the interpreter between two calls."""

    def __init__(self, lib):
        self.lib = lib

    def __getattr__(self, name):
        fn = getattr(self.lib, name)

        def call(*args):
            self.last = (fn, args)
            return fn(*args)
        return call


@pytest.mark.parametrize("which", PAIRS)
def test_host_threads_with_calls_of_different_sizes(which, monkeypatch):
    """A thread's calls give the same whatever the other threads ask for, and none is refused."""
    work, failed = [make(torch.cuda.Stream()) for make in 2 * PAIRS[which]], []
    tape = Tape(ub.load_library())
    monkeypatch.setattr(ub, "load_library", lambda: tape)
    torch.cuda.synchronize()
    want, calls = [], []
    for _, call, out in work:
        call()
        torch.cuda.synchronize()
        calls.append(tape.last)
        want.append([t.clone() for t in out])
        for t in out:
            t.zero_()
    torch.cuda.synchronize()
    monkeypatch.undo()
    start = threading.Barrier(len(work))

    def loop(ctx, fn, args):                                         # (no interpreter in between: calls overlap)
        start.wait(60)
        for i in range(5000):
            code = fn(*args)
            if code:
                failed.append((code, ub.load_library().unity_last_error(ctx.ctx).decode()))
                return

    threads = [threading.Thread(target=loop, args=(w[0], *c)) for w, c in zip(work, calls)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    torch.cuda.synchronize()
    assert not failed, failed
    for (ctx, _, out), w in zip(work, want):
        ctx.check_status()
        assert all(torch.equal(a, b) for a, b in zip(out, w))


@pytest.mark.parametrize("which", PAIRS)
def test_a_large_call_is_captured_before_a_small_one(which):
    st = torch.cuda.Stream()
    work = [make(st) for make in PAIRS[which]]
    torch.cuda.synchronize()
    want = []
    for _, call, out in work:
        call()
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
        for t in out:
            t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        for _, call, _ in work:
            call()
    work[1][1]()                                                     # (the smaller one comes last before the replay, too)
    torch.cuda.synchronize()
    for _, _, out in work:
        for t in out:
            t.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    for (ctx, _, out), w in zip(work, want):
        ctx.check_status()
        assert all(torch.equal(a, b) for a, b in zip(out, w))


@pytest.mark.parametrize("H", [64, 256, 448, 512])
@pytest.mark.parametrize("res", [F32, B16])
def test_rows_of_one_warp_take_their_places_in_the_ring_in_turn(H, res):
    """Many rows per block, one warp each: the place of a row that was read takes the next one.  Of 12001 rows on all blocks dx against the
    formula in 64 bits, with the tolerance of test_gpu_norm.py; 601 rows on a few blocks as there."""
    n, K = 12001, 2
    p = tn.Rows(n, H, K=K, n_inv=5, res=res, seed=H, mask=0.1)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(n, H, K))
    r, head, dy, more = p.res.cuda(), p.head(), p.dy.cuda(), p.dres.cuda()
    dx, dg = tn.junk((n, H), res), [tn.junk((H,), F32) for _ in range(K)]
    ctx.rms_norm_bwd(r, *head, dy, dx, more, dg)
    role = torch.repeat_interleave(p.role.long(), p.cu[1:] - p.cu[:-1])
    model = torch.tensor(p.role_model)[role].cuda()
    x, g = r.double(), dy.double() * torch.stack(head[0]).double()[model]
    s = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + float(np.float32(p.eps)))
    want = s * g - x * s ** 3 * (g * x).mean(1, keepdim=True) + more.double()
    size = (s * g).abs() + x.abs() * s ** 3 * (g * x).abs().mean(1, keepdim=True) + more.double().abs()
    on = (p.mask != 0).cuda().unsqueeze(1)
    want, size = torch.where(on, want, 0.0), torch.where(on, size, 0.0)
    tol = 256 * tn.U * size + (tn.B if res == B16 else tn.U) * want.abs() * (1 + 256 * tn.U) + 1e-38
    assert ((dx.double() - want).abs() <= tol).all()
    for _ in range(20):
        dx2, dg2 = tn.junk((n, H), res), [tn.junk((H,), F32) for _ in range(K)]
        ctx.rms_norm_bwd(r, *head, dy, dx2, more, dg2)
        assert torch.equal(dx, dx2) and all(torch.equal(a, b) for a, b in zip(dg, dg2))
    ctx.check_status()
    p = tn.Rows(601, H, K=K, n_inv=5, res=res, seed=H, mask=0.1)
    ctx = ub.Context(0, ub.unity_rms_norm_workspace_bytes(7, H, K))
    dx = tn.junk((601, H), res)
    ctx.rms_norm_bwd(p.res.cuda(), *p.head(), p.dy.cuda(), dx, p.dres.cuda(), dg)
    tn.check_bwd(p, p.res, dx, None)
    ctx.check_status()


def test_a_captured_update_writes_every_output_again():
    """Norm, sampling, policy loss, norm backward and clipping of two models in one graph: before the replay every output holds something
    else, behind it what the calls gave one by one."""
    N, H, V, K, eps = 200, 256, 4096, 2, 1e-6
    g = torch.Generator().manual_seed(9)
    cu, role = torch.tensor([0, 60, 60, 140, 200]).cuda(), torch.tensor([0, 1, 2, 1], dtype=torch.int32).cuda()
    role_model, T = [0, 1, 1], 0.8
    tok_role = torch.repeat_interleave(role, cu[1:] - cu[:-1])
    mask = (torch.rand(N, generator=g) < 0.85).to(torch.uint8).cuda()
    x, residual = torch.randn(N, H, generator=g).to(B16).cuda(), (torch.randn(N, H, generator=g) * 3).cuda()
    gamma = [(1 + 0.2 * torch.randn(H, generator=g)).to(B16).cuda() for _ in range(K)]
    W = [(torch.randn(V, H, generator=g) * 0.15).to(B16).cuda() for _ in range(K)]
    u, adv, z = torch.rand(N, generator=g).cuda(), torch.randn(N, generator=g).cuda(), (torch.randn(N, V, generator=g) * 3).cuda()
    rules = [(T, 0, 1.0, 0.0), (T, 50, 0.95, 0.0), (0.0, 0, 1.0, 0.0)]
    new = lambda *s, t=F32: torch.empty(s, dtype=t, device="cuda")
    o = dict(y=new(N, H, t=B16), r=new(N, H), token=new(N, t=torch.int32), logp=new(N), logk=new(N), kept=new(N, t=torch.int32), old=new(N),
             loss=new(K), dh=new(N, H, t=B16), dx=new(N, H), norm=new(K), coef=new(K))
    lists = dict(dW=[new(V, H) for _ in range(K)], dg=[new(H) for _ in range(K)], out=[new(V, H, t=B16) for _ in range(K)] + [new(H) for _ in range(K)])
    outputs = list(o.values()) + [t for v in lists.values() for t in v]
    st = torch.cuda.Stream()
    ctx = ub.Context(0, max(ub.unity_workspace_bytes(N, H, V, K, 4), ub.unity_rms_norm_workspace_bytes(N, H, K),
                            ub.unity_clip_grad_norm_workspace_bytes(4, K)), st)
    handle, route = ub.GradTensors(lists["dW"] + lists["dg"], [0, 1, 0, 1], lists["out"]), (cu, role, role_model)
    target = torch.empty_like(o["token"])

    def step():
        ctx.rms_norm_fwd(x, gamma, *route, mask, eps, o["y"], residual, o["r"])
        ctx.sample(z, rules, u, o["token"], tok_role, mask, o["logp"], o["logk"], o["kept"])
        torch.clamp(o["token"], min=0, out=target)
        ctx.logprob_fwd(o["y"], W, *route, target, mask, 1 / T, o["old"])
        ctx.ppo_loss_fwd_bwd(o["y"], W, *route, target, mask, 1 / T, 0.2, 0.2, 0.01, 3, 0.0, None, False, o["old"], o["old"], adv, o["loss"],
                             None, None, None, None, o["dh"], lists["dW"])
        ctx.rms_norm_bwd(o["r"], gamma, *route, mask, eps, o["dh"], o["dx"], residual, lists["dg"])
        ctx.clip_grad_norm(handle, [1e-3, 1e3], o["norm"], o["coef"])

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    for _ in range(2):
        for t in outputs:
            t.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(outputs, want):
            assert torch.equal(t, w)
        ctx.check_status()


def test_a_list_of_tensors_keeps_its_memory():
    """A listed tensor that is given other memory: what was listed stays what it was, and nobody else's memory is written."""
    n = 1 << 20
    g = torch.full((n,), 2.0, device="cuda")
    out = torch.empty(n, device="cuda")
    handle = ub.GradTensors([g, torch.ones(5, device="cuda")], [0, 0], [None, None])
    other = ub.GradTensors([torch.ones(n, device="cuda")], [0], [out])
    ctx = ub.Context(0, 1 << 16)
    norm = torch.zeros(1, device="cuda")
    with torch.no_grad():
        g.set_(torch.full((n,), 3.0, device="cuda"))
        out.set_(torch.full((n,), 3.0, device="cuda"))
    later = [torch.full((n,), 7.0, device="cuda") for _ in range(8)]
    ctx.clip_grad_norm(handle, [1.0], norm)
    assert abs(norm.item() - (4.0 * n + 5) ** 0.5) <= 5.1 * 2.0 ** -24 * (4.0 * n + 5) ** 0.5
    ctx.clip_grad_norm(other, [1.0], norm)
    ctx.check_status()
    assert (g == 3).all() and (out == 3).all() and all((t == 7).all() for t in later)
