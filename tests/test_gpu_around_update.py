"""The calls around the update in a row with the update itself, on one context: final norm -> logits -> sampled answers ->
log-probabilities of the samples -> policy loss and its gradients -> norm backward -> clipping per model.

Each link is held against the fp64 oracle fed with the link's own inputs; the whole chain against the oracle's chain within the parity
contract (2e-2 of the gradients' norm, 1e-2 per log-probability)."""
import numpy as np
import pytest
import torch

import parity_harness as pu
from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub

pytestmark = pytest.mark.gpu

F32, B16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("captured", [False, True])
def test_rollout_and_update_of_two_models(captured):
    N, H, V, K, eps = 300, 256, 4096, 2, 1e-6
    g = torch.Generator().manual_seed(5)
    cu = torch.tensor([0, 40, 40, 133, 201, 300])
    role = torch.tensor([0, 1, 2, 1, 0], dtype=torch.int32)
    role_model, T = [0, 1, 1], 0.8
    mask = (torch.rand(N, generator=g) < 0.85).to(torch.uint8)
    x, residual = torch.randn(N, H, generator=g).to(B16), torch.randn(N, H, generator=g) * 3
    gamma = [(1 + 0.2 * torch.randn(H, generator=g)).to(B16) for _ in range(K)]
    W = [(torch.randn(V, H, generator=g) * 0.15).to(B16) for _ in range(K)]
    u, adv = torch.rand(N, generator=g), torch.randn(N, generator=g)
    rules = [(T, 0, 1.0, 0.0), (T, 50, 0.95, 0.0), (T, 0, 1.0, 0.02)]
    tok_role = torch.repeat_interleave(role.long(), cu[1:] - cu[:-1])
    tok_model = torch.tensor(role_model)[tok_role]

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = ub.Context(0, max(ub.unity_workspace_bytes(N, H, V, K, 5), ub.unity_rms_norm_workspace_bytes(N, H, K)), st)
        d = {k: v.cuda() for k, v in dict(cu=cu, role=role, mask=mask, x=x, res=residual, u=u, adv=adv, row_role=tok_role.to(torch.int32),
                                          pick=(tok_model == 1)).items()}
        gm, Wd = [w.cuda() for w in gamma], [w.cuda() for w in W]
        new = lambda *s, t=F32: torch.full(s, 7.0, device="cuda").to(t)
        y, r, dh, dx = new(N, H, t=B16), new(N, H), new(N, H, t=B16), new(N, H)
        token, logp, logk, kept = new(N, t=torch.int32), new(N), new(N), new(N, t=torch.int32)
        logits, old, loss = new(N, V), new(N), new(K)
        dW, dg = [new(V, H) for _ in range(K)], [new(H) for _ in range(K)]
        out = [new(V, H, t=B16) for _ in range(K)] + [new(H) for _ in range(K)]
        norm, coef = new(K), new(K)
        handle = ub.GradTensors(dW + dg, [0, 1, 0, 1], out)
        route = (d["cu"], d["role"], role_model)

        def step():
            ctx.rms_norm_fwd(d["x"], gm, *route, d["mask"], eps, y, d["res"], r)
            a, b = torch.mm(y.float(), Wd[0].float().T), torch.mm(y.float(), Wd[1].float().T)
            torch.where(d["pick"].unsqueeze(1), b, a, out=logits)
            ctx.sample(logits, rules, d["u"], token, d["row_role"], d["mask"], logp, logk, kept)
            token.clamp_(min=0)                                   # (finished rows are masked out from here on)
            ctx.logprob_fwd(y, Wd, *route, token, d["mask"], 1 / T, old)
            ctx.ppo_loss_fwd_bwd(y, Wd, *route, token, d["mask"], 1 / T, 0.2, 0.2, 0.01, 3, 0.0, None, False, old, old, d["adv"], loss,
                                 None, None, None, None, dh, dW)
            ctx.rms_norm_bwd(r, gm, *route, d["mask"], eps, dh, dx, None, dg)
            ctx.clip_grad_norm(handle, [1e-3, 1e3], norm, coef)

        step()
        torch.cuda.synchronize()
        if captured:
            before = [t.clone() for t in (y, token, loss, dx, norm, *dg, *out)]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                step()
            for t in (y, token, dx, norm, *dg, *out):
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(before, (y, token, loss, dx, norm, *dg, *out)))
            return
    ctx.check_status()
    on = mask.numpy() != 0
    # sampled tokens are the oracle's on the same logits, and their log-probabilities those of stage 2
    z, lp = logits.cpu().numpy(), logp.cpu().numpy()
    for i in np.nonzero(on)[0]:
        t, want, _, n = orc.sample_row(z[i], *rules[int(tok_role[i])], u[i].item())
        assert int(token[i]) == t and int(kept[i]) == n and abs(lp[i] - want) <= 1e-5
    assert np.abs(lp - old.cpu().numpy())[on].max() <= pu.TOL_LOGP
    # the chain in fp64
    table = (cu.numpy(), role.numpy(), role_model, mask.numpy(), eps)
    oy, orr = orc.rms_norm_fwd(pu.bf16_bits(x), residual.numpy(), [pu.bf16_bits(w) for w in gamma], *table)
    o = orc.ppo_loss_fwd_bwd(oy, [pu.bf16_bits(w) for w in W], cu.numpy(), role.numpy(), np.asarray(role_model), token.cpu().numpy(), mask.numpy(),
                             old.cpu().numpy(), old.cpu().numpy(), adv.numpy(), clip_lo=0.2, clip_hi=0.2, kl_coef=0.01, kl_mode=3, ent_coef=0.0,
                             inv_temperature=float(np.float32(1 / T)))
    wx, wg, _, _ = orc.rms_norm_bwd(orr, [pu.bf16_bits(w) for w in gamma], *table, o["dHidden"])
    assert pu.rel_fro(dx.cpu().numpy(), wx) <= pu.TOL_GRAD
    for k in range(K):
        assert pu.rel_fro(dg[k].cpu().numpy(), wg[k]) <= pu.TOL_GRAD
    wn, wc, wo = orc.clip_grad_norm(o["dW"] + list(wg), [0, 1, 0, 1], K, [1e-3, 1e3])
    assert np.all(np.abs(norm.cpu().numpy() - wn) <= pu.TOL_GRAD * wn) and wc[0] < 1 and wc[1] == 1 and coef[1].item() == 1
    for a, b in zip(out, wo):
        assert pu.rel_fro(a.float().cpu().numpy(), b) <= 2 * pu.TOL_GRAD


def test_contexts_on_two_streams_at_once():
    """The same three calls on two contexts whose kernels overlap give what each gives alone."""
    work = []
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        st = torch.cuda.Stream()
        n, H, V = 700, 1536, 33000
        d = dict(st=st, x=torch.randn(n, H, generator=g, device="cuda").to(B16), gamma=[torch.randn(H, generator=g, device="cuda") for _ in range(2)],
                 cu=torch.tensor([0, 300, n], device="cuda"), role=torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                 z=torch.randn(300, V, generator=g, device="cuda") * 3, u=torch.rand(300, generator=g, device="cuda"),
                 grads=[torch.randn(300001, generator=g, device="cuda"), torch.randn(4097, generator=g, device="cuda").to(B16)])
        d["ctx"] = ub.Context(0, max(ub.unity_rms_norm_workspace_bytes(n, H, 2), ub.unity_clip_grad_norm_workspace_bytes(2, 2)), st)
        d["o"] = lambda d=d, n=n, H=H: dict(
            y=torch.zeros(n, H, dtype=B16, device="cuda"), dx=torch.zeros(n, H, dtype=B16, device="cuda"),
            dg=[torch.zeros(H, device="cuda") for _ in range(2)], token=torch.zeros(300, dtype=torch.int32, device="cuda"),
            logp=torch.zeros(300, device="cuda"), norm=torch.zeros(2, device="cuda"), out=[torch.zeros_like(t) for t in d["grads"]])
        work.append(d)
    torch.cuda.synchronize()

    def go(d, o):
        route = (d["cu"], d["role"], [0, 1], None, 1e-6)
        d["ctx"].rms_norm_fwd(d["x"], d["gamma"], *route, o["y"])
        d["ctx"].sample(d["z"], [(0.9, 30, 0.9, 0.0)], d["u"], o["token"], None, None, o["logp"])
        d["ctx"].rms_norm_bwd(d["x"], d["gamma"], *route, o["y"], o["dx"], None, o["dg"])
        d["ctx"].clip_grad_norm(ub.GradTensors(d["grads"], [0, 1], o["out"]), [1.0, 1e9], o["norm"])

    def flat(o):
        return [t for v in o.values() for t in (v if isinstance(v, list) else [v])]

    alone = []
    for d in work:
        o = d["o"]()
        torch.cuda.synchronize()
        go(d, o)
        torch.cuda.synchronize()
        alone.append(flat(o))
    for _ in range(5):
        outs = [d["o"]() for d in work]
        torch.cuda.synchronize()
        for d, o in zip(work, outs):
            go(d, o)
        torch.cuda.synchronize()
        for o, want in zip(outs, alone):
            assert all(torch.equal(a, b) for a, b in zip(flat(o), want))
    for d in work:
        d["ctx"].check_status()
