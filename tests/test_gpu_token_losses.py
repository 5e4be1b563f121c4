"""GPU parity of the token losses (cross entropy, distillation) against the fp64 oracle, element by element.

Tolerances, derived.  u = 2^-24 and b = 2^-8 are the largest relative errors of one rounding to fp32 and bf16.
  logits     the tensor core adds H products to an fp32 accumulator, 16 per step, and may cut instead of round: a logit is
             off by at most (H/16 + 2) * 2u * tau * sum_j |h_j W_vj|; `ez` below is the largest such bound of a row
  lse        ez, plus V additions in chunks and exponentials of relative error 2^-21: 2^-17 in all on log s, plus 2u |lse|
  l          as many times the sum of its terms' weights as it has lse and z: 2 (ez + 2^-17) * mass, plus u times the terms
  G = dL/dz  p is off by a factor of e^(2 ez + 2^-17); G is written in bf16 (b; up to 64 tokens in two
             halves, b^2), a block that was kept between the two sweeps
             in steps of 2^-9 octaves (half a step: ln2 2^-10): relative to the terms that make G up,
             eg = b + 2^-10 + 2 ez + 2^-16, and a kept logit 64 octaves or more below the row's maximum may count as
             64: at most 2^-64 of the row's coefficient
  dHidden    eg sum_v |G||W|, plus fp32 sums and the output's rounding: b |dHidden|
  dW         eg sum_i |G||h|, the same; f32: without the output's rounding
The fp32 sums of the products are covered by 2^-12 of the sums of magnitudes (V/16 steps of 2u).
"""
import ctypes

import numpy as np
import pytest
import torch

import parity_harness as pu
from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub

pytestmark = pytest.mark.gpu

B, U = 2.0 ** -8, 2.0 ** -24


class Problem:
    def __init__(self, N, H, V, K=1, R=None, n_inv=None, n_top=0, seed=0, mask=0.2, spread=4.0, short_lists=True):
        rng = np.random.default_rng(seed)
        R = R or K
        self.N, self.H, self.V, self.K = N, H, V, K
        n_inv = n_inv or max(1, min(N, 7))
        cuts = np.sort(rng.integers(0, N + 1, n_inv - 1))
        self.cu = torch.from_numpy(np.concatenate([[0], cuts, [N]]))
        self.inv_role = torch.from_numpy(rng.integers(0, R, n_inv).astype(np.int32))
        self.role_model = [r % K for r in range(R)]
        self.mask = torch.from_numpy((rng.random(N) >= mask).astype(np.uint8))
        self.target = torch.from_numpy(rng.integers(0, V, N).astype(np.int32))
        self.weight = torch.from_numpy(rng.normal(size=N).astype(np.float32))
        W = [rng.normal(size=(V, H)).astype(np.float32) / np.sqrt(H) for _ in range(K)]
        model = np.asarray(self.role_model)[np.repeat(self.inv_role.numpy(), np.diff(self.cu.numpy()))]
        hidden = rng.normal(size=(N, H)).astype(np.float32)
        for k in range(K):         # from hopeless to sure predictions
            hidden += (model == k)[:, None] * rng.random((N, 1)).astype(np.float32) * 3 * spread * W[k][self.target.numpy()]
        self.W = [torch.from_numpy(w).to(torch.bfloat16) for w in W]
        self.hidden = torch.from_numpy(hidden).to(torch.bfloat16)
        self.n_top = n_top
        if n_top:
            ids = np.stack([rng.choice(V, n_top, replace=n_top > V) for _ in range(N)]).reshape(N, n_top)
            take = rng.random(N) < 0.7
            ids[take, rng.integers(0, n_top)] = self.target.numpy()[take]
            if short_lists:
                ids[rng.random((N, n_top)) < 0.2] = -7
                ids[::9] = -1                                    # rows without a list
                ids[4::11] = ids[4::11, :1]                      # one id many times
            self.top_ids = torch.from_numpy(ids.astype(np.int32))
            self.top_vals = torch.from_numpy((rng.normal(size=(N, n_top)) * 2).astype(np.float32))

    def gpu(self):
        for name in ("cu", "inv_role", "mask", "target", "weight", "hidden", "top_ids", "top_vals"):
            if hasattr(self, name):
                setattr(self, "d_" + name, getattr(self, name).cuda())
        self.d_W = [w.cuda() for w in self.W]
        return self


def call(ctx, p, op, grads="all", dw=torch.bfloat16, weight=True, norm=None, accumulate=False, dW=None, dH=None, tau=1.0,
         smoothing=0.0, z_loss=0.0, mode=ub.TEACHER_LOGITS, kd=1.0, hard=0.0, mask=True, target=True):
    junk = dict(device="cuda")
    o = dict(loss=torch.full((p.K,), 7.0, **junk), tok_loss=torch.full((p.N,), 7.0, **junk), lse=torch.full((p.N,), 7.0, **junk))
    o["dHidden"] = None if grads in ("none", "head") else dH if dH is not None else torch.full((p.N, p.H), 7.0, dtype=torch.bfloat16, **junk)
    o["dW"] = None if grads in ("none", "hidden") else dW if dW is not None else [torch.full((p.V, p.H), 7.0, dtype=dw, **junk) for _ in range(p.K)]
    head = (p.d_hidden, p.d_W, p.d_cu, p.d_inv_role, p.role_model, p.d_target if target else None, p.d_mask if mask else None, tau)
    outs = (norm, accumulate, p.d_weight if weight else None, o["loss"], o["tok_loss"], o["lse"], o["dHidden"], o["dW"])
    if op == "ce":
        ctx.cross_entropy_fwd_bwd(*head, smoothing, z_loss, *outs)
    else:
        ctx.distill_fwd_bwd(*head, p.d_top_ids, p.d_top_vals, mode, kd, hard, *outs)
    return o


def oracle(p, op, weight=True, norm=None, tau=1.0, smoothing=0.0, z_loss=0.0, mode=ub.TEACHER_LOGITS, kd=1.0, hard=0.0, mask=True):
    t32 = float(np.float32(tau))
    q = None if op == "ce" else orc.teacher_rows(p.top_ids.numpy(), p.top_vals.numpy(), p.V, mode == ub.TEACHER_LOGITS, t32)
    bits = pu.bf16_bits
    o = orc.token_loss_fwd_bwd(bits(p.hidden), [bits(w) for w in p.W], p.cu.numpy(), p.inv_role.numpy(), np.asarray(p.role_model),
                               p.target.numpy(), p.mask.numpy() if mask else None, p.weight.numpy() if weight else None, norm, t32,
                               float(np.float32(smoothing)), float(np.float32(z_loss)), q, float(np.float32(kd)), float(np.float32(hard)))
    # bounds of the module docstring
    N = p.N
    ez, terms, mass = np.zeros(N), np.zeros((N, p.V)), np.zeros(N)
    for k in range(p.K):
        i = np.nonzero(o["on"] & (o["tok_model"] == k))[0]
        h, W = orc.to_f64(bits(p.hidden[i])), orc.to_f64(bits(p.W[k]))
        if not i.size:
            continue
        ez[i] = (p.H / 16 + 2) * 2 * U * t32 * (np.abs(h) @ np.abs(W).T).max(1)
        P = np.exp(t32 * (h @ W.T) - o["lse"][i][:, None])
        c = t32 * (p.weight.numpy().astype(float)[i] if weight else np.ones(i.size)) / o["M"][k]
        if q is None:
            cp, own = 1 + 2 * z_loss * np.abs(o["lse"][i]), np.full((i.size, p.V), smoothing / p.V)
            own[np.arange(i.size), p.target.numpy()[i]] += 1
            mass[i] = 1 + 2 * z_loss * np.abs(o["lse"][i])
        else:
            cp, own = kd * q[i].sum(1) + hard, kd * q[i]
            if hard > 0:
                own[np.arange(i.size), p.target.numpy()[i]] += hard
            mass[i] = cp
        terms[i] = np.abs(c)[:, None] * (cp[:, None] * P + own)
        o.setdefault("floor", np.zeros(N))[i] = np.abs(c) * cp * 2.0 ** -64
    big = np.abs(o["lse"]) + np.abs(o["tok_loss"])
    o["tol_lse"] = ez + 2.0 ** -17 + 2 * U * np.abs(o["lse"])
    o["tol_l"] = (2 * ez + 2.0 ** -16) * mass + 8 * U * (1 + big * (1 + mass) + (z_loss * o["lse"] ** 2 if q is None else 0))
    # a sure row's G is a small difference of p and its target: p's own error counts, not G's
    eg = 2.0 ** -10 + 2 * ez[:, None] + 2.0 ** -16
    rounding = B * (1 + B) if N > 64 else B * B
    o["dG"] = rounding * np.abs(o["G"]) + eg * terms + (o["floor"][:, None] if "floor" in o else 0)
    return o


def check(p, g, o, k_only=None, base=None):
    on = o["on"]
    for key, tol in (("lse", "tol_lse"), ("tok_loss", "tol_l")):
        got = g[key].double().cpu().numpy()
        assert np.all(got[~on] == 0), key
        assert np.all(np.abs(got - o[key]) <= o[tol]), (key, np.max(np.abs(got - o[key]) / np.maximum(o[tol], 1e-300)))
    loss = g["loss"].double().cpu().numpy()
    for k in range(p.K):
        i = on & (o["tok_model"] == k)
        w = np.abs(p.weight.numpy().astype(float)) if g.get("weight", True) else np.ones(p.N)
        tol = (w * (o["tol_l"] + 16 * U * np.abs(o["tok_loss"])))[i].sum() / o["M"][k] + 4 * U * abs(o["loss"][k])
        assert abs(loss[k] - o["loss"][k]) <= tol, (k, loss[k], o["loss"][k], tol)
    if g["dHidden"] is not None:
        got = g["dHidden"].double().cpu().numpy()
        assert np.all(got[~on] == 0)
        for k in range(p.K):
            i = np.nonzero(on & (o["tok_model"] == k))[0]
            W = np.abs(orc.to_f64(pu.bf16_bits(p.W[k])))
            tol = (o["dG"][i] + 2.0 ** -12 * np.abs(o["G"][i])) @ W + B * np.abs(o["dHidden"][i]) * (1 + B) + 1e-38
            err = np.abs(got[i] - o["dHidden"][i])
            assert np.all(err <= tol), (k, (err / tol).max())
    if g["dW"] is not None:
        for k in range(p.K):
            i = np.nonzero(on & (o["tok_model"] == k))[0]
            h = np.abs(orc.to_f64(pu.bf16_bits(p.hidden[i])))
            want = o["dW"][k] + (0 if base is None else base[k])
            tol = (o["dG"][i] + 2.0 ** -12 * np.abs(o["G"][i])).T @ h + 1e-38 + 4 * U * np.abs(want)
            if g["dW"][k].dtype == torch.bfloat16:
                tol = tol * (1 + B) + B * np.abs(want)
            err = np.abs(g["dW"][k].double().cpu().numpy() - want)
            assert np.all(err <= tol), (k, (err / tol).max())


def context(p, op, backward=True, n_tok=None):
    return ub.Context(0, ub.unity_token_loss_workspace_bytes(n_tok or p.N, p.H, p.V, p.K, p.n_top if op == "kd" else 0, backward))


CE = [dict(), dict(smoothing=0.1), dict(z_loss=1e-2, tau=0.7), dict(smoothing=0.3, z_loss=1e-3, weight=False, tau=1.5)]
KD = [dict(), dict(hard=0.5), dict(mode=ub.TEACHER_LOGPROBS, tau=0.5), dict(mode=ub.TEACHER_LOGPROBS, hard=1.25, kd=0.3, weight=False, tau=2.0)]


@pytest.mark.parametrize("kw", CE)
@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,V,K,R", [(1, 64, 8, 1, 1), (130, 64, 264, 1, 1), (300, 192, 1000, 2, 3), (517, 128, 4104, 3, 5)])
def test_cross_entropy(N, H, V, K, R, dw, kw):
    p = Problem(N, H, V, K, R, seed=N).gpu()
    ctx = context(p, "ce")
    g = call(ctx, p, "ce", dw=dw, **kw)
    ctx.check_status()
    g["weight"] = kw.get("weight", True)
    check(p, g, oracle(p, "ce", **kw))
    ctx.close()


@pytest.mark.parametrize("kw", KD)
@pytest.mark.parametrize("N,H,V,K,R,n_top", [(1, 64, 8, 1, 1, 1), (130, 64, 264, 1, 1, 5), (300, 192, 1000, 2, 3, 64),
                                             (517, 128, 4104, 3, 5, 128), (65, 64, 16, 1, 1, 33)])
def test_distill(N, H, V, K, R, n_top, kw):
    p = Problem(N, H, V, K, R, n_top=n_top, seed=N + n_top).gpu()
    ctx = context(p, "kd")
    g = call(ctx, p, "kd", target=kw.get("hard", 0) > 0, **kw)
    ctx.check_status()
    g["weight"] = kw.get("weight", True)
    check(p, g, oracle(p, "kd", **kw))
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("grads", ["none", "hidden", "head"])
def test_forms_agree_with_the_whole_call(op, grads):
    p = Problem(333, 128, 2056, 2, 2, n_top=17, seed=3).gpu()
    ctx = context(p, op)
    whole, part = call(ctx, p, op), call(ctx, p, op, grads)
    ctx.check_status()
    for key in ("loss", "tok_loss", "lse", "dHidden"):
        assert part[key] is None or torch.equal(part[key], whole[key]), key
    assert part["dW"] is None or all(torch.equal(a, b) for a, b in zip(part["dW"], whole["dW"]))
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N", [1, 40, 64, 65, 128])
@pytest.mark.parametrize("H,V", [(64, 2000), (320, 1000), (1344, 520), (1920, 20000)])
def test_few_rows_in_every_form(N, H, V, op):
    """Both gradients in one launch, or one of them, or added to an old dW, of either type; the first rows may be all masked."""
    p = Problem(N, H, V, 1, 1, n_top=6, seed=N + V, mask=0.3 if N > 1 else 0.0).gpu()
    ctx = context(p, op)
    o = oracle(p, op)
    for dw in (torch.bfloat16, torch.float32):
        check(p, call(ctx, p, op, dw=dw), o)
        check(p, call(ctx, p, op, "head", dw=dw), o)
        old = [torch.full((V, H), 0.5, device="cuda", dtype=dw)]
        check(p, call(ctx, p, op, accumulate=True, dW=old), o, base=[np.full((V, H), 0.5)])
    check(p, call(ctx, p, op, "hidden"), o)
    ctx.check_status()
    p.mask.zero_()
    p.d_mask = p.mask.cuda()
    g = call(ctx, p, op)
    assert g["loss"][0] == 0 and g["dW"][0].abs().max() == 0 and g["dHidden"].abs().max() == 0
    ctx.check_status()
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V,K", [(129, 64, 264, 1), (300, 576, 3000, 1), (1024, 256, 1000, 4), (700, 1088, 2504, 3), (1024, 128, 60000, 1)])
def test_small_problems_gradients_side_by_side(N, H, V, K, op):
    """Both gradients of all models share a launch: each type of dW, added to or not, a model without rows among them."""
    p = Problem(N, H, V, K, K, n_top=6, seed=N + V, mask=0.2).gpu()
    ctx = context(p, op)
    o = oracle(p, op)
    for dw in (torch.bfloat16, torch.float32):
        g = call(ctx, p, op, dw=dw)
        check(p, g, o)
        again = call(ctx, p, op, dw=dw)
        assert torch.equal(g["dHidden"], again["dHidden"]) and all(torch.equal(a, b) for a, b in zip(g["dW"], again["dW"]))
        old = [torch.full((V, H), 0.5, device="cuda", dtype=dw) for _ in range(K)]
        check(p, call(ctx, p, op, accumulate=True, dW=old), o, base=[np.full((V, H), 0.5)] * K)
    ctx.check_status()
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [200, 3000])
def test_accumulation_and_norm(N, op, dw):
    p = Problem(N, 64, 520, 2, 2, n_top=9, seed=5).gpu()
    ctx = context(p, op)
    torch.manual_seed(1)
    old = [torch.randn(p.V, p.H, device="cuda").to(dw) * 0.01 for _ in range(p.K)]
    base = [x.double().cpu().numpy() for x in old]
    g = call(ctx, p, op, norm=[123.0, 7.5], accumulate=True, dW=old)
    ctx.check_status()
    check(p, g, oracle(p, op, norm=[123.0, 7.5]), base=base)
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
def test_every_workspace_down_to_the_least_gives_the_same_answer(op):
    """Smaller workspaces take smaller blocks of rows, then pieces of the vocabulary whose logits are recomputed."""
    p = Problem(4500, 64, 6000, 1, 1, n_top=6, seed=9, n_inv=3).gpu()
    o = oracle(p, op)
    size = ub.unity_token_loss_workspace_bytes(p.N, p.H, p.V, p.K, p.n_top if op == "kd" else 0)
    for dw in (torch.bfloat16, torch.float32):
        now, ways = size, set()
        while True:
            ctx = ub.Context(0, now)
            try:
                g = call(ctx, p, op, dw=dw)
            except ub.UnityError as e:
                assert e.code == -4
                ctx.close()
                break
            ctx.check_status()
            ways.add(ctx.launch_count)
            check(p, g, o)
            ctx.close()
            now = now * 4 // 5 // 256 * 256
        # one block, blocks of kept logits, and the least: pieces of 1024 entries for blocks of at most 1024 rows
        assert len(ways) >= 4 and max(ways) > 60 and now < size // 4, (ways, now, size)


@pytest.mark.parametrize("op", ["ce", "kd"])
def test_few_rows_of_many_models_in_smaller_workspaces(op):
    """Sixteen models' rows in one block, then a block of each in turn, then pieces of the vocabulary."""
    p = Problem(100, 64, 4104, 16, 16, n_inv=40, n_top=6, seed=19).gpu()
    o = oracle(p, op)
    now, ways = ub.unity_token_loss_workspace_bytes(p.N, p.H, p.V, p.K, p.n_top if op == "kd" else 0), set()
    while True:
        ctx = ub.Context(0, now)
        try:
            g = call(ctx, p, op)
        except ub.UnityError as e:
            assert e.code == -4
            ctx.close()
            break
        ctx.check_status()
        ways.add(ctx.launch_count)
        check(p, g, o)
        ctx.close()
        now = now * 31 // 32 // 256 * 256      # (most of it is a buffer that all ways need)
    assert len(ways) >= 3, ways


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V,K,n_inv", [
    (64, 192, 2000, 3, 9), (63, 64, 264, 1, 2), (127, 320, 248, 3, 5), (128, 64, 256, 2, 5), (129, 64, 512, 2, 5),        # one row tile of one CTA, and just more
    (1024, 64, 136, 2, 3000), (1025, 64, 136, 3, 900),                        # routed with the packing or by a block of its own,
    (8192, 64, 72, 1, 1500), (8193, 64, 72, 2, 40),                           # or by several; boundaries staged or searched
    (10, 128, 20000, 1, 3), (40, 1344, 6000, 2, 4),                           # few rows: a contraction in many parts
    (700, 896, 3000, 1, 9), (2600, 192, 1000, 2, 6),
    (90, 64, 4104, 4, 9), (900, 640, 3000, 4, 9), (60, 64, 520, 5, 9),        # models side by side in a launch, and one too many
    (6000, 256, 1024, 1, 9), (5000, 576, 600, 3, 9)])                         # many rows of a small head: dW in parts
def test_sizes_where_the_way_of_working_changes(N, H, V, K, n_inv, op):
    p = Problem(N, H, V, K, K, n_inv=n_inv, n_top=7, seed=N + H).gpu()
    ctx = context(p, op)
    g = call(ctx, p, op, tau=0.9)
    ctx.check_status()
    check(p, g, oracle(p, op, tau=0.9))
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
def test_more_rows_than_one_block(op, dw):
    """Over 18432 rows per model: several blocks, whose dW adds up in fp32."""
    p = Problem(24000, 64, 200, 2, 2, n_inv=50, n_top=5, seed=6, mask=0.1)
    p.inv_role[:] = 0
    p.inv_role[7] = 1
    p.gpu()
    ctx = context(p, op)
    torch.manual_seed(2)
    old = [torch.randn(p.V, p.H, device="cuda").to(dw) * 0.01 for _ in range(p.K)]
    base = [x.double().cpu().numpy() for x in old]
    o = oracle(p, op)
    check(p, call(ctx, p, op, dw=dw), o)
    check(p, call(ctx, p, op, accumulate=True, dW=old), o, base=base)
    ctx.check_status()
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("options", [[(0, 1), (1, 1), (2, 1), (3, 1)], [(11, 0)], [(9, 0), (10, 0)], [(29, 0)]])
def test_options_of_the_gemms(op, options):
    """CTAs per tile, tiles one block wide, no rendezvous, no tail launch."""
    p = Problem(2300, 640, 1400, 1, 1, n_top=9, seed=12).gpu()
    ctx = context(p, op)
    for option, value in options:
        ctx.set_option(option, value)
    g = call(ctx, p, op)
    ctx.check_status()
    check(p, g, oracle(p, op))
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
def test_rows_that_leave_nothing(op):
    p = Problem(150, 64, 136, 2, 2, n_top=4, seed=11).gpu()
    ctx = context(p, op)
    for what in ("all", "one model"):
        mask = torch.zeros(p.N, dtype=torch.uint8)
        if what == "one model":
            tok_model = torch.repeat_interleave(p.inv_role, p.cu[1:] - p.cu[:-1]) % 2
            mask[tok_model == 1] = 1
        p.mask, p.d_mask = mask, mask.cuda()
        p.d_weight = torch.where(p.d_mask == 0, torch.nan, p.weight.cuda())               # nothing of a masked row is read
        p.d_hidden = torch.where(p.d_mask[:, None] == 0, torch.nan, p.hidden.cuda())
        p.d_target = torch.where(p.d_mask == 0, -5, p.target.cuda())
        if op == "kd":
            p.d_top_vals = torch.where(p.d_mask[:, None] == 0, torch.nan, p.top_vals.cuda())
        g = call(ctx, p, op)
        ctx.check_status()
        o = oracle(p, op)
        check(p, g, o)
        assert g["loss"][0] == 0 and g["dW"][0].abs().max() == 0
        old = [torch.full((p.V, p.H), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        call(ctx, p, op, accumulate=True, dW=old)
        assert torch.all(old[0] == 3.0)
    ctx.close()


def test_lists_without_probability_and_places_that_are_not_read():
    p = Problem(40, 64, 200, 1, 1, n_top=4, seed=2, short_lists=False).gpu()
    p.top_ids[0] = -1
    p.top_vals[1] = -torch.inf
    p.top_vals[2, 1:] = -torch.inf
    p.top_ids[3, 1], p.top_vals[3, 1] = -1, torch.nan
    p.top_ids[5, 1], p.top_vals[5, 1] = -1, torch.inf
    p.top_vals[6] = torch.finfo(torch.float32).min
    p.gpu()
    ctx = context(p, "kd")
    for mode in (ub.TEACHER_LOGITS, ub.TEACHER_LOGPROBS):
        g = call(ctx, p, "kd", mode=mode, target=False)
        ctx.check_status()
        check(p, g, oracle(p, "kd", mode=mode))
        for i in (0, 1):
            assert g["tok_loss"][i] == 0 and g["dHidden"][i].abs().max() == 0
    ctx.close()


def test_bad_indexes_are_reported_and_left_out():
    p = Problem(60, 64, 104, 1, 1, n_top=3, seed=4, mask=0.0).gpu()
    ctx = context(p, "kd")
    p.d_target[7] = p.V
    p.d_target[8] = -1
    g = call(ctx, p, "ce")
    with pytest.raises(ub.UnityError) as e:
        ctx.check_status()
    assert e.value.code == -7
    p.mask[7:9] = 0
    check(p, g, oracle(p, "ce"))
    p.gpu()
    p.d_top_ids[3, 2] = p.V
    p.d_top_ids[4, 0] = 2 ** 31 - 1
    g = call(ctx, p, "kd", target=False)
    with pytest.raises(ub.UnityError):
        ctx.check_status()
    p.top_ids[3, 2] = p.top_ids[4, 0] = -1
    check(p, g, oracle(p, "kd"))
    ctx.close()


def test_refusals():
    p = Problem(10, 64, 104, 1, 1, n_top=3, seed=4).gpu()
    ctx = context(p, "kd")
    bad = [("ce", dict(smoothing=1.0), -1), ("ce", dict(smoothing=-0.1), -1), ("ce", dict(smoothing=float("nan")), -1),
           ("ce", dict(z_loss=-1.0), -1), ("ce", dict(z_loss=float("inf")), -1), ("kd", dict(kd=-1.0), -1),
           ("kd", dict(hard=float("nan")), -1), ("kd", dict(mode=2), -1), ("kd", dict(hard=1.0, target=False), -1),
           ("ce", dict(target=False), -1), ("ce", dict(tau=0.0), -1), ("kd", dict(tau=float("nan")), -1), ("ce", dict(norm=[0.0]), -1),
           ("kd", dict(norm=[-1.0]), -1)]
    for op, kw, code in bad:
        with pytest.raises(ub.UnityError) as e:
            call(ctx, p, op, **kw)
        assert e.value.code == code, (op, kw)
    wide = Problem(4, 64, 200, 1, 1, n_top=129, seed=1).gpu()
    with pytest.raises(ub.UnityError) as e:
        call(ctx, wide, "kd", target=False)
    assert e.value.code == -2
    for H, V in ((32, 64), (96, 64), (64, 12)):
        with pytest.raises(ub.UnityError) as e:
            call(ctx, Problem(4, H, V).gpu(), "ce")
        assert e.value.code == -2
    off = torch.zeros(p.V * p.H + 8, dtype=torch.bfloat16, device="cuda")[1:1 + p.V * p.H].view(p.V, p.H)
    with pytest.raises(ub.UnityError) as e:
        call(ctx, p, "ce", dW=[off])
    assert e.value.code == -3
    two = Problem(40, 64, 104, 2, 2, n_top=3, seed=4).gpu()
    same = torch.zeros(two.V, two.H, device="cuda")
    for op in ("ce", "kd"):
        with pytest.raises(ub.UnityError) as e:
            call(ctx, two, op, accumulate=True, dW=[same, same])
        assert e.value.code == -1 and "same" in str(e.value)
    small = ub.Context(0, 1 << 16)
    with pytest.raises(ub.UnityError) as e:
        call(small, p, "ce")
    assert e.value.code == -4 and "bytes" in str(e.value)
    small.close()
    lib = ub.load_library()
    assert lib.unity_cross_entropy_fwd_bwd(ctx.ctx, None, None, None, None, None, None, None, None) == -1
    g = call(ctx, p, "ce")                        # the context still works
    ctx.check_status()
    check(p, g, oracle(p, "ce"))
    ctx.close()


def test_no_tokens():
    p = Problem(3, 64, 16, 2, 2, n_top=2).gpu()
    ctx = context(p, "kd")
    p.N = 0
    for name in ("hidden", "target", "mask", "weight", "top_ids", "top_vals"):
        setattr(p, "d_" + name, getattr(p, "d_" + name)[:0])
    p.d_cu, p.d_inv_role = p.d_cu[:1] * 0, p.d_inv_role[:0]
    for op in ("ce", "kd"):
        g = call(ctx, p, op)
        ctx.check_status()
        assert torch.all(g["loss"] == 0) and all(torch.all(w == 0) for w in g["dW"])
        old = [torch.full((p.V, p.H), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        call(ctx, p, op, accumulate=True, dW=old)
        assert all(torch.all(w == 3.0) for w in old)
    ctx.close()


def test_results_repeat_bit_by_bit_on_streams_and_in_graphs():
    p = Problem(400, 128, 5000, 2, 2, n_top=20, seed=8).gpu()
    size = ub.unity_token_loss_workspace_bytes(p.N, p.H, p.V, p.K, p.n_top)
    first = {}
    ctx = ub.Context(0, size)
    for op in ("ce", "kd"):
        first[op] = call(ctx, p, op)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = ub.Context(0, size, side)
        again = {op: call(other, p, op) for op in ("ce", "kd")}
        other.check_status()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kept = {op: call(other, p, op) for op in ("ce", "kd")}
        for _ in range(2):
            for g in kept.values():
                for t in (g["loss"], g["tok_loss"], g["dHidden"], *g["dW"]):
                    t.fill_(9.0)
            graph.replay()
        side.synchronize()
    other.check_status()
    ctx.check_status()
    for g in (again, kept):
        for op in ("ce", "kd"):
            for key in ("loss", "tok_loss", "lse", "dHidden"):
                assert torch.equal(g[op][key], first[op][key]), (op, key)
            assert all(torch.equal(a, b) for a, b in zip(g[op]["dW"], first[op]["dW"]))
    del graph
    other.close()
    ctx.close()


def test_extreme_logits():
    """Rows whose logits reach hundreds: sure tokens' losses keep their digits, far entries vanish."""
    p = Problem(96, 64, 512, 1, 1, n_top=8, seed=21, spread=4.0)
    p.hidden = (p.hidden.float() * torch.linspace(0.01, 40, 96)[:, None]).to(torch.bfloat16)
    p.gpu()
    ctx = context(p, "kd")
    for op in ("ce", "kd"):
        g = call(ctx, p, op)
        ctx.check_status()
        check(p, g, oracle(p, op))
    ctx.close()


def test_step_of_both_losses_and_the_policy_update_on_one_context():
    """As a trainer uses them: cross entropy, distillation and the policy loss one after the other on the same rows, heads and
    workspace, the heads' gradients added up."""
    p = Problem(260, 128, 1032, 2, 3, n_top=10, seed=17).gpu()
    ctx = ub.Context(0, max(ub.unity_token_loss_workspace_bytes(p.N, p.H, p.V, p.K, p.n_top),
                            ub.unity_workspace_bytes(p.N, p.H, p.V, p.K, int(p.inv_role.numel()))))
    f = torch.float32
    dW = [torch.zeros(p.V, p.H, device="cuda", dtype=f) for _ in range(p.K)]
    logp, ent, lse = (torch.zeros(p.N, device="cuda") for _ in range(3))
    ctx.logprob_fwd(p.d_hidden, p.d_W, p.d_cu, p.d_inv_role, p.role_model, p.d_target, p.d_mask, 1.0, logp, ent, lse)
    ce = call(ctx, p, "ce", accumulate=True, dW=dW)
    kd = call(ctx, p, "kd", accumulate=True, dW=dW, hard=0.25)
    ppo_dW = [torch.zeros(p.V, p.H, device="cuda", dtype=f) for _ in range(p.K)]
    loss, dH = torch.zeros(p.K, device="cuda"), torch.zeros_like(p.d_hidden)
    adv = torch.randn(p.N, device="cuda")

    def ppo(out, accumulate):
        ctx.ppo_loss_fwd_bwd(p.d_hidden, p.d_W, p.d_cu, p.d_inv_role, p.role_model, p.d_target, p.d_mask, 1.0, 0.2, 0.2, 0.0, 3,
                             0.0, None, accumulate, logp, logp, adv, loss, None, None, None, None, dH, out)
    ppo(ppo_dW, False)
    ppo(dW, True)
    ctx.check_status()
    # the policy update's log-probabilities and the cross entropy are the same quantity from two kernels
    o = oracle(p, "ce")
    on = torch.from_numpy(o["on"]).cuda()
    tol = torch.from_numpy(o["tol_l"]).cuda() + 2.0 ** -15
    assert torch.all((ce["tok_loss"] + logp).abs()[on] <= 2 * tol[on])
    k = oracle(p, "kd", hard=0.25)
    for m in range(p.K):
        part = [call(ctx, p, op, dw=f, **kw)["dW"][m] for op, kw in (("ce", {}), ("kd", dict(hard=0.25)))]
        want = part[0].double() + part[1].double() + ppo_dW[m].double()
        scale = part[0].double().abs() + part[1].double().abs() + ppo_dW[m].double().abs()
        assert torch.all((dW[m].double() - want).abs() <= 4 * U * scale + 1e-30)
    check(p, {**ce, "dW": None}, o)
    check(p, {**kd, "dW": None}, k)
    ctx.close()


def test_outputs_between_guards():
    """Rows before the first and behind the last token, and entries before and behind the heads' gradients, stay as they were."""
    p = Problem(77, 64, 264, 1, 1, n_top=6, seed=14).gpu()
    ctx = context(p, "kd")
    for op in ("ce", "kd"):
        o = oracle(p, op)
        dH = torch.full((p.N + 16, p.H), 5.0, dtype=torch.bfloat16, device="cuda")
        per = {k: torch.full((p.N + 8,), 5.0, device="cuda") for k in ("tok_loss", "lse")}
        dW = torch.full((p.V + 16, p.H), 5.0, dtype=torch.bfloat16, device="cuda")
        loss = torch.full((5,), 5.0, device="cuda")
        head = (p.d_hidden, p.d_W, p.d_cu, p.d_inv_role, p.role_model, p.d_target, p.d_mask, 1.0)
        outs = (None, False, p.d_weight, loss[2:3], per["tok_loss"][4:-4], per["lse"][4:-4], dH[8:-8], [dW[8:-8]])
        if op == "ce":
            ctx.cross_entropy_fwd_bwd(*head, 0.0, 0.0, *outs)
        else:
            ctx.distill_fwd_bwd(*head, p.d_top_ids, p.d_top_vals, ub.TEACHER_LOGITS, 1.0, 0.0, *outs)
        ctx.check_status()
        check(p, dict(loss=outs[3], tok_loss=outs[4], lse=outs[5], dHidden=outs[6], dW=outs[7]), o)
        for t, w in ((dH, 8), (dW, 8), (per["tok_loss"], 4), (per["lse"], 4), (loss, 2)):
            assert torch.all(t[:w] == 5.0) and torch.all(t[-w:] == 5.0)
    ctx.close()


def test_two_contexts_at_once():
    """Calls on two streams, each with its own context and workspace, overlap without touching one another."""
    p, q = Problem(300, 128, 3000, 1, 1, n_top=6, seed=1).gpu(), Problem(90, 192, 2000, 2, 2, n_top=6, seed=2).gpu()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    ctxs, got = [], [[], []]
    for s, x in zip(streams, (p, q)):
        with torch.cuda.stream(s):
            ctxs.append(ub.Context(0, ub.unity_token_loss_workspace_bytes(x.N, x.H, x.V, x.K, x.n_top), s))
    for _ in range(4):
        for i, x in enumerate((p, q)):
            with torch.cuda.stream(streams[i]):
                got[i] += [call(ctxs[i], x, "ce"), call(ctxs[i], x, "kd")]
    torch.cuda.synchronize()
    for i, x in enumerate((p, q)):
        ctxs[i].check_status()
        want = [oracle(x, "ce"), oracle(x, "kd")]
        for j, g in enumerate(got[i]):
            check(x, g, want[j % 2])
            assert torch.equal(g["dHidden"], got[i][j % 2]["dHidden"])
        ctxs[i].close()


def test_current_device_and_default_arguments_stay():
    p = Problem(20, 64, 104, 1, 1, n_top=3, seed=4, mask=0.0).gpu()
    ctx = context(p, "ce")
    before = torch.cuda.current_device()
    g = call(ctx, p, "ce", mask=False, weight=False)
    assert torch.cuda.current_device() == before
    ctx.check_status()
    g["weight"] = False
    check(p, g, oracle(p, "ce", mask=False, weight=False))
    ctx.close()


@pytest.mark.parametrize("N", [87, 150, 333, 1500])
def test_targets_of_unsure_rows_are_not_rounded_together(N):
    """Without weights dL/dz / (tau/M) is p - 1 at the target: at most p away from -1, which bf16 holds.  tau/M itself, which it does
    not hold, comes in fp32.  So the target's entry is off by at most p (and its own error), the others' p by b and eg of them."""
    p = Problem(N, 64, 4096, 1, 1, seed=N, mask=0.0, spread=0.0).gpu()
    ctx = context(p, "ce")
    g = call(ctx, p, "ce", dw=torch.float32, weight=False)
    ctx.check_status()
    h, W, y, at = p.d_hidden.double(), p.d_W[0].double(), p.d_target.long(), torch.arange(N, device="cuda")
    ez = (p.H / 16 + 2) * 2 * U * (h.abs() @ W.abs().T).max(1).values[:, None]
    P = torch.softmax(h @ W.T, 1)
    tol = (B * (1 + B) + 2.0 ** -10 + 2 * ez + 2.0 ** -16) * P
    tol[at, y] = P[at, y] * (1 + 2 * ez[:, 0] + 2.0 ** -16) + 4 * U
    G = P.clone()
    G[at, y] -= 1
    want = G.T @ h / N
    sums = ((N / 16 + 2) * 2 * U * G.abs()).T @ h.abs()
    assert torch.all((g["dW"][0].double() - want).abs() <= (tol.T @ h.abs() + sums) / N + 4 * U * want.abs())
    ctx.close()


def test_offsets_beyond_32_bits():
    """16500 rows of 152064 kept logits: more than 2^31 of them.  Reference: the formulas in 64 bits on the device, 500 rows at a
    time; tolerances as in oracle(), with a bound of |h| |W| that holds for every entry."""
    N, H, V = 16500, 64, 152064
    g = torch.Generator(device="cuda").manual_seed(5)
    W = (torch.randn(V, H, generator=g, device="cuda") / 8).to(torch.bfloat16)
    h = torch.randn(N, H, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    target[-1], target[-2] = V - 1, 0
    mask = (torch.rand(N, generator=g, device="cuda") < 0.99).to(torch.uint8)
    mask[-3:] = 1
    cu = torch.tensor([0, N], device="cuda")
    role = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = ub.Context(0, ub.unity_token_loss_workspace_bytes(N, H, V, 1, 0))
    loss, tl, lse = torch.empty(1, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    dH = torch.empty_like(h)
    dW = torch.empty(V, H, device="cuda")
    ctx.cross_entropy_fwd_bwd(h, [W], cu, role, [0], target, mask, 1.0, 0.0, 0.0, None, False, None, loss, tl, lse, dH, [dW])
    ctx.check_status()
    on = mask.bool()
    M, Wd = int(on.sum()), W.double()
    want_W, tol_W = torch.zeros(V, H, device="cuda", dtype=torch.float64), torch.zeros(V, H, device="cuda", dtype=torch.float64)
    total = 0.0
    for i in range(0, N, 500):
        rows, y = h[i:i + 500].double(), target[i:i + 500].long()
        c = on[i:i + 500].double()[:, None] / M
        z = rows @ Wd.T
        want_lse = torch.logsumexp(z, 1)
        at = torch.arange(rows.shape[0], device="cuda")
        want_l = want_lse - z[at, y]
        keep = on[i:i + 500]
        ez = (H / 16 + 2) * 2 * U * rows.abs().sum(1) * Wd.abs().max()
        assert torch.all(((lse[i:i + 500] - want_lse).abs() <= ez + 2.0 ** -17 + 2 * U * want_lse.abs())[keep])
        assert torch.all(((tl[i:i + 500] - want_l).abs() <= 2 * ez + 2.0 ** -16 + 8 * U * (1 + 2 * (want_lse.abs() + want_l.abs())))[keep])
        assert torch.all(tl[i:i + 500][~keep] == 0) and torch.all(dH[i:i + 500][~keep] == 0)
        total += float((want_l * keep).sum())
        P = torch.exp(z - want_lse[:, None])
        terms = P.clone()
        terms[at, y] += 1
        P[at, y] -= 1
        G = P * c
        dG = B * (1 + B) * G.abs() + (2.0 ** -10 + 2 * ez[:, None] + 2.0 ** -16) * terms * c + c * 2.0 ** -64
        dG += 2.0 ** -12 * G.abs()
        want = G @ Wd
        assert torch.all((dH[i:i + 500].double() - want).abs() <= dG @ Wd.abs() + B * (1 + B) * want.abs() + 1e-38), i
        want_W += G.T @ rows
        tol_W += dG.T @ rows.abs()
    assert abs(float(loss) - total / M) <= 1e-5 * abs(total / M)
    assert torch.all((dW.double() - want_W).abs() <= tol_W + 4 * U * want_W.abs() + 1e-38)
    ctx.close()
