"""Token losses over a large vocabulary, with their gradients: the cases they are measured on.

Two operators on the rows that the policy update works on (hidden rows of response tokens, K output heads W, tokens
routed to a head by the role of their invocation):

  cross_entropy   supervised warm start of a role: label smoothing, z-loss, token weights
  distill         learning from a teacher's listed logits (its top entries per token), optionally mixed with the
                  cross entropy of the recorded token

With z = inv_temperature * W_k h_i over the V entries of the vocabulary, lse = log sum_v exp z_v, p = exp(z - lse):

  cross entropy   l_i = lse - (1 - eps) z_y - eps/V sum_v z_v + lam lse^2
  distillation    l_i = kd sum_v q_v (log q_v - z_v + lse) + hard (lse - z_y)
                  q: softmax of the listed teacher logits (mode "logits"), or exp of listed log-probabilities as they are
                  (mode "logprobs"); entries with a negative id are empty places; equal ids add up
  loss_k = 1/M_k sum over valid tokens i of model k of w_i l_i,  M_k = max(number of valid tokens, 1)

``run`` computes them in plain torch operations in 32 bits, or, where ``own`` is true, by this package's calls.
"""
import math

import torch

own = False

# (H, V) of the repository's configurations
TINY, RAG_QA, SEARCH, CODE, STRESS = (256, 4096), (896, 151936), (1536, 151936), (3584, 152064), (5120, 152064)


def _ce(name, hv, n_tok, n_inv, models, grads, eps, lam, masked):
    return {"name": name, "op": "cross_entropy", "H": hv[0], "V": hv[1], "n_tok": n_tok, "n_inv": n_inv, "models": models,
            "grads": grads, "smoothing": eps, "z_loss": lam, "masked": masked, "inv_temperature": 1.0}


def _kd(name, hv, n_tok, n_inv, models, grads, n_top, mode, hard, inv_t, masked):
    return {"name": name, "op": "distill", "H": hv[0], "V": hv[1], "n_tok": n_tok, "n_inv": n_inv, "models": models,
            "grads": grads, "n_top": n_top, "mode": mode, "hard": hard, "inv_temperature": inv_t, "masked": masked}


def listed():
    return [
        # a unit-test sized head: every launch counts, nothing else does
        _ce("ce eval tiny", TINY, 64, 4, 1, "none", 0.0, 0.0, 0.0),
        # one micro-batch of the smallest model, forward and backward: latency again, now of the whole chain
        _ce("ce train tiny", TINY, 333, 9, 2, "all", 0.0, 1e-4, 0.2),
        # validation loss of held-out answers of the question-answering roles; odd number of rows
        _ce("ce eval rag_qa", RAG_QA, 1001, 25, 1, "none", 0.0, 0.0, 0.2),
        # a single short demonstration on the largest head that is trained: the weights' traffic decides
        _ce("ce train few rows", CODE, 96, 1, 1, "all", 0.0, 0.0, 0.1),
        # supervised warm start of the search roles, two models, with smoothing and z-loss
        _ce("ce train search", SEARCH, 5000, 40, 2, "all", 0.1, 1e-4, 0.2),
        # the same for the coding roles: a full micro-batch of long answers for two models
        _ce("ce train code", CODE, 8000, 12, 2, "all", 0.0, 1e-4, 0.2),
        # scoring a few tokens against a teacher on the unit-test head
        _kd("distill eval tiny", TINY, 37, 3, 1, "none", 8, "logits", 0.0, 1.0, 0.0),
        # one token of one answer: a monitor that follows the distance to the teacher while it decodes
        _kd("distill eval one token", SEARCH, 1, 1, 1, "none", 20, "logprobs", 0.0, 1.0, 0.0),
        # two small role models learn from the entries that a serving engine returns by default
        _kd("distill train rag_qa", RAG_QA, 3001, 70, 2, "all", 20, "logprobs", 0.0, 1.0, 0.2),
        # the head is frozen, only the hidden rows' gradient is wanted
        _kd("distill frozen head", SEARCH, 2050, 17, 1, "hidden", 50, "logits", 0.0, 0.5, 0.2),
        # temperature 2, mixed with the recorded tokens' cross entropy
        _kd("distill train code", CODE, 4100, 6, 1, "all", 64, "logits", 0.5, 0.5, 0.2),
        # the largest head with a long list per token
        _kd("distill train stress", STRESS, 6000, 30, 1, "all", 100, "logits", 0.0, 1.0, 0.2),
    ]


def _size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    H, V = rng.choice([TINY, RAG_QA, SEARCH, CODE, STRESS, (64 * _size(rng, 1, 80), 8 * _size(rng, 125, 19000))])
    grads = rng.choice(["none", "hidden", "all", "all"])
    models = rng.choice([1, 1, 2, 3])
    masked = rng.choice([0.0, 0.1, 0.2, 0.5])
    # the most that a listed case costs, in multiply-adds of the plain form, bounds the number of tokens
    most = 6000 * 5120 * 152064 / (H * V) / {"none": 1, "hidden": 2, "all": 3}[grads] * 3
    n_tok = _size(rng, 1, max(1, min(16000, int(0.8 * most))))
    n_inv = max(1, min(n_tok, _size(rng, 1, 64)))
    if rng.random() < 0.5:
        c = _ce("", (H, V), n_tok, n_inv, models, grads, rng.choice([0.0, 0.1, 0.05]), rng.choice([0.0, 1e-4]), masked)
    else:
        c = _kd("", (H, V), n_tok, n_inv, models, grads, _size(rng, 1, 128), rng.choice(["logits", "logprobs"]),
                rng.choice([0.0, 0.3]), rng.choice([1.0, 0.5, 0.8]), masked)
    del c["name"]
    return c


def _valid(case):
    return case["n_tok"] - int(case["masked"] * case["n_tok"])


def work(case):
    H, V, n, K = case["H"], case["V"], case["n_tok"], case["models"]
    m = _valid(case)
    heads = min(K, m)
    by = m * H * 2 + heads * V * H * 2 + n * (1 + 4 + 4) + n * 4 * 2
    fl = 2.0 * m * H * V
    if case["op"] == "distill":
        by += m * case["n_top"] * 8
    if case["grads"] != "none":
        by += n * H * 2
        fl += 2.0 * m * H * V
    if case["grads"] == "all":
        by += K * V * H * 2
        fl += 2.0 * m * H * V
    return {"bytes": by, "flops": fl}


def prepare(case, seed):
    H, V, n, K, S = case["H"], case["V"], case["n_tok"], case["models"], case["n_inv"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda")

    # ragged answers, one of them empty where there are a few; every role is served by the model of its number
    cuts = torch.randint(0, n + 1, (S - 1,), generator=c).sort().values
    if S > 3:
        cuts[1] = cuts[0]
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])])
    role = torch.randint(0, K, (S,), generator=c)
    model = torch.repeat_interleave(role, cu[1:] - cu[:-1]).cuda()
    mask = torch.ones(n, dtype=torch.uint8)
    mask[torch.randperm(n, generator=c)[:n - _valid(case)]] = 0      # tool output and prompts inside the answers
    st = {"case": case, "cu_seqlens": cu.cuda(), "inv_role": role.to(torch.int32).cuda(), "tok_mask": mask.cuda()}
    # heads and hidden rows as the repository draws them, with a part of each hidden row pointing at its token, so that
    # some tokens are predicted surely and some hardly at all
    st["W"] = [(normal(V, H) * 0.02).to(torch.bfloat16) for _ in range(K)]
    target = ints(0, V, n)
    unit = 1.0 / (H * 0.02 * 0.02)
    aims = [target]
    if case["op"] == "distill":
        k = case["n_top"]
        step = max(1, V // k)
        ids = (ints(0, V, n, 1) + ints(1, step + 1, n, k).cumsum(1)) % V
        ids[:, 0] = torch.where(ints(0, 5, n) > 0, target, ids[:, 0])
        vals = 9.0 - 1.5 * torch.log1p(torch.arange(k, device="cuda", dtype=torch.float32)) + 0.3 * normal(n, k)
        if case["mode"] == "logprobs":
            vals = vals - vals.exp().sum(1, keepdim=True).log() - 0.1
        order = torch.argsort(torch.rand(n, k, generator=g, device="cuda"), 1)
        aims += [ids[:, j] for j in range(1, min(k, 4))]
        ids, vals = ids.gather(1, order), vals.gather(1, order)
        gone = torch.arange(k, device="cuda") >= ints(k // 2, k + 1, n, 1)      # places that the engine left empty
        st["top_ids"] = torch.where(gone, -1, ids).to(torch.int32)
        st["top_vals"] = torch.where(gone, 0.0, vals).contiguous()
    hidden = normal(n, H)
    for j, a in enumerate(aims):
        gain = torch.rand(n, 1, generator=g, device="cuda") * (14.0 - 3.0 * j) * unit
        for k in range(K):
            hidden += gain * st["W"][k][a].float() * (model == k).unsqueeze(1)
    st["hidden"] = hidden.to(torch.bfloat16)
    st["target"] = target.to(torch.int32)
    st["tok_weight"] = 0.5 + torch.rand(n, generator=g, device="cuda")
    f32, b16 = torch.float32, torch.bfloat16
    st["out"] = {"loss": torch.empty(K, dtype=f32, device="cuda"), "tok_loss": torch.empty(n, dtype=f32, device="cuda"),
                 "lse": torch.empty(n, dtype=f32, device="cuda"),
                 "dHidden": torch.empty(n, H, dtype=b16, device="cuda") if case["grads"] != "none" else None,
                 "dW": [torch.empty(V, H, dtype=b16, device="cuda") for _ in range(K)] if case["grads"] == "all" else None}
    if own:
        from paper_2605_26646_b200 import binding as ub
        st["ctx"] = ub.Context(0, ub.unity_token_loss_workspace_bytes(n, H, V, K, case.get("n_top", 0),
                                                                      case["grads"] != "none"))
        st["mode"] = {"logits": ub.TEACHER_LOGITS, "logprobs": ub.TEACHER_LOGPROBS}[case.get("mode", "logits")]
    return st


def _run_own(st):
    case, o = st["case"], st["out"]
    roles = list(range(case["models"]))
    head = (st["hidden"], st["W"], st["cu_seqlens"], st["inv_role"], roles, st["target"], st["tok_mask"],
            case["inv_temperature"])
    outs = (o["loss"], o["tok_loss"], o["lse"], o["dHidden"], o["dW"])
    if case["op"] == "cross_entropy":
        st["ctx"].cross_entropy_fwd_bwd(*head, case["smoothing"], case["z_loss"], None, False, st["tok_weight"], *outs)
    else:
        st["ctx"].distill_fwd_bwd(*head, st["top_ids"], st["top_vals"], st["mode"], 1.0, case["hard"], None, False,
                                  st["tok_weight"], *outs)
    return {k: v for k, v in o.items() if v is not None}


def _plain_model(st, k, tok_model):
    """The rows of model k: their indexes, l, lse and the gradients, in 32 bits."""
    case = st["case"]
    rows = torch.nonzero((tok_model == k) & (st["tok_mask"] != 0)).squeeze(1)
    tau, V = case["inv_temperature"], case["V"]
    h, W = st["hidden"][rows].float(), st["W"][k].float()
    y, w = st["target"][rows].long().unsqueeze(1), st["tok_weight"][rows]
    z = (h @ W.T) * tau
    top = z.amax(1, keepdim=True)
    p = (z - top).exp()
    s = p.sum(1, keepdim=True)
    lse = (top + s.log()).squeeze(1)
    zy = z.gather(1, y).squeeze(1)
    if case["op"] == "cross_entropy":
        eps, lam = case["smoothing"], case["z_loss"]
        l = lse - (1 - eps) * zy + lam * lse * lse
        if eps:
            l = l - eps * z.mean(1)
        cp, ct, cu, ids, q = 1 + 2 * lam * lse, 1 - eps, eps / V, None, None
    else:
        ids = st["top_ids"][rows].long()
        on = ids >= 0
        t = st["top_vals"][rows]
        if case["mode"] == "logits":
            e = torch.where(on, (torch.where(on, t * tau, -math.inf) - torch.where(on, t * tau, -1e30).amax(1, keepdim=True)).exp(), 0.0)
            q = e / e.sum(1, keepdim=True).clamp_min(1e-30)
        else:
            q = torch.where(on, t.exp(), 0.0)
        ids = ids.clamp_min(0)
        if case["n_top"] > 1:                                   # equal ids add up
            same = (ids.unsqueeze(2) == ids.unsqueeze(1)) & on.unsqueeze(1)
            whole = (same * q.unsqueeze(1)).sum(2)
        else:
            whole = q
        Q = q.sum(1)
        l = (q * torch.where(q > 0, whole.clamp_min(1e-38).log(), 0.0)).sum(1) - (q * z.gather(1, ids)).sum(1) + Q * lse
        l = l + case["hard"] * (lse - zy)
        cp, ct, cu = Q + case["hard"], case["hard"], 0.0
    M = max(int(rows.numel()), 1)
    loss = (w * l).sum() / M
    if case["grads"] == "none":
        return rows, l, lse, loss, None, None
    del z
    p *= (cp / s.squeeze(1)).unsqueeze(1)
    if cu:
        p -= cu
    if q is not None:
        p.scatter_add_(1, ids, -q)
    if ct:
        p.scatter_add_(1, y, torch.full_like(y, -ct, dtype=torch.float32))
    p *= (w * (tau / M)).unsqueeze(1)
    dH = (p @ W).to(torch.bfloat16)
    dW = (p.T @ h).to(torch.bfloat16) if case["grads"] == "all" else None
    return rows, l, lse, loss, dH, dW


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    lens = state["cu_seqlens"][1:] - state["cu_seqlens"][:-1]
    tok_model = torch.repeat_interleave(state["inv_role"].long(), lens)
    parts = [_plain_model(state, k, tok_model) for k in range(case["models"])]
    at = torch.cat([p[0] for p in parts])
    o = {"loss": torch.stack([p[3] for p in parts]),
         "tok_loss": state["hidden"].new_zeros(case["n_tok"], dtype=torch.float32).index_copy_(0, at, torch.cat([p[1] for p in parts])),
         "lse": state["hidden"].new_zeros(case["n_tok"], dtype=torch.float32).index_copy_(0, at, torch.cat([p[2] for p in parts]))}
    if case["grads"] != "none":
        o["dHidden"] = torch.zeros_like(state["hidden"]).index_copy_(0, at, torch.cat([p[4] for p in parts]))
    if case["grads"] == "all":
        o["dW"] = [p[5] for p in parts]
    return o


def exact(case, seed):
    """The same in 64 bits: the loss as a sum of -target log p, its gradients by automatic differentiation."""
    st = prepare(case, seed)
    n, H, V, K = case["n_tok"], case["H"], case["V"], case["models"]
    tau, f64 = case["inv_temperature"], torch.float64
    bounds = st["cu_seqlens"].cpu()
    tok_model = torch.empty(n, dtype=torch.int64)
    for s, r in enumerate(st["inv_role"].cpu().tolist()):
        tok_model[int(bounds[s]):int(bounds[s + 1])] = r
    on = st["tok_mask"].cpu() != 0
    out = {"loss": torch.zeros(K, dtype=f64), "tok_loss": torch.zeros(n, dtype=f64, device="cuda"),
           "lse": torch.zeros(n, dtype=f64, device="cuda")}
    want_h, want_w = case["grads"] != "none", case["grads"] == "all"
    if want_h:
        out["dHidden"] = torch.zeros(n, H, dtype=f64, device="cuda")
    if want_w:
        out["dW"] = []
    for k in range(K):
        rows = torch.nonzero((tok_model == k) & on).squeeze(1).cuda()
        W = st["W"][k].to(f64).requires_grad_(want_w)
        total = 0.0
        for r0 in range(0, rows.numel(), 1024):
            r = rows[r0:r0 + 1024]
            h = st["hidden"][r].to(f64).requires_grad_(want_h)
            with torch.set_grad_enabled(want_h):
                z = tau * (h @ W.t())
                lse = torch.logsumexp(z, 1)
                hard = z.gather(1, st["target"][r].long().unsqueeze(1)).squeeze(1) - lse
                if case["op"] == "cross_entropy":
                    eps = case["smoothing"]
                    l = -(1 - eps) * hard - eps * (z - lse.unsqueeze(1)).mean(1) + case["z_loss"] * lse.square()
                else:
                    ids, t = st["top_ids"][r].long(), st["top_vals"][r].to(f64)
                    t = torch.where(ids >= 0, t * (tau if case["mode"] == "logits" else 1.0), -math.inf)
                    none = (ids < 0).all(1, keepdim=True)
                    q = torch.softmax(torch.where(none, 0.0, t), 1) if case["mode"] == "logits" else t.exp()
                    q = torch.where(none | (ids < 0), 0.0, q)
                    dense = torch.zeros(r.numel(), V, dtype=f64, device="cuda").scatter_add_(1, ids.clamp_min(0), q)
                    l = (torch.xlogy(dense, dense).sum(1) - (dense * (z - lse.unsqueeze(1))).sum(1)) - case["hard"] * hard
                loss = (st["tok_weight"][r].to(f64) * l).sum() / max(rows.numel(), 1)
            if want_h:
                loss.backward()
                out["dHidden"][r] = h.grad
            out["tok_loss"][r], out["lse"][r] = l.detach(), lse.detach()
            total += float(loss)
        out["loss"][k] = total
        if want_w:
            out["dW"].append(W.grad if W.grad is not None else torch.zeros(V, H, dtype=f64, device="cuda"))
    return out
