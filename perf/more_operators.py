"""What stands around the policy computation on a role model's answers, and the cases it is measured on.

  norm_fwd   final root-mean-square norm with the residual's addition, one weight vector per model:
             r = x + residual, s = 1 / sqrt(mean(r^2) + eps), y = gamma_k * r * s; it makes the rows the heads read
  norm_bwd   its backward from dy, the gradient of those rows: with g = dy * gamma_k,
             dr = s * g - r * s^3 * mean(g * r) + dres (what else arrives on r), dgamma_k = sum over the model's tokens of dy * r * s
  clip       norm_k = sqrt(sum of squares of all gradients of model k), out = gradient * min(1, max_k / norm_k)
  sample     next tokens from logits and given uniform numbers u, with a rule per role: temperature T, top_k, top_p, min_p.
             In the order of falling logits (equal ones by index) an entry is allowed if its rank is < top_k and its
             probability at least min_p times the largest; it is kept if the allowed mass before it is < top_p of the whole
             allowed mass.  The token is the first kept index, ascending, whose running mass is > u times the kept mass.
             Also log p of the token in the whole distribution at T and among the kept entries, and their number.
             T = 0 takes the largest logit (log p at T = 1, and 0 among the kept).

Rows that are masked out read nothing and have zeros as outputs (sample: token -1).  ``run`` computes them in plain torch
operations, or, where ``own`` is true, by this package's calls.
"""
import math

import torch

own = False

# (H, V) of the repository's configurations
TINY, RAG_QA, SEARCH, CODE, STRESS = (256, 4096), (896, 151936), (1536, 151936), (3584, 152064), (5120, 152064)
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, op, H, n_tok, n_inv, models, residual, gamma, masked):
    return {"name": name, "op": op, "H": H, "n_tok": n_tok, "n_inv": n_inv, "models": models, "residual": residual,
            "gamma": gamma, "masked": masked}


def _clip(name, hv, models, blocks, odd, grad, out, tight):
    """models x (a head [V, H], `blocks` layers of four [H, H] matrices and two [H] vectors, `odd` values of another tensor)."""
    return {"name": name, "op": "clip", "H": hv[0], "V": hv[1], "models": models, "blocks": blocks, "odd": odd, "grad": grad,
            "out": out, "tight": tight}


def _sample(name, n_rows, V, logits, rules, spread, masked):
    """rules: "T,top_k,top_p,min_p" of each role, between semicolons; spread: standard deviation of the logits."""
    return {"name": name, "op": "sample", "n_rows": n_rows, "V": V, "logits": logits, "rules": rules, "spread": spread,
            "masked": masked}


def listed():
    return [
        # the next token of one answer while it is decoded: latency
        _norm("norm fwd one token", "norm_fwd", CODE[0], 1, 1, 1, "bf16", "bf16", 0.0),
        # a unit-test sized batch without residual
        _norm("norm fwd tiny", "norm_fwd", TINY[0], 333, 9, 2, "none", "f32", 0.2),
        # hidden rows of a full micro-batch of two coding roles, prompts and tool output masked
        _norm("norm fwd code", "norm_fwd", CODE[0], 20001, 40, 2, "bf16", "bf16", 0.2),
        # four separate models, residual stream kept in 32 bits
        _norm("norm fwd stress", "norm_fwd", STRESS[0], 32768, 512, 4, "f32", "bf16", 0.1),
        # the same rows on the way back: the search roles' micro-batch, nothing else arrives on the residual stream
        _norm("norm bwd search", "norm_bwd", SEARCH[0], 5000, 40, 2, "bf16", "bf16", 0.2),
        # many long answers, with a gradient that arrives on the residual stream in 32 bits
        _norm("norm bwd code", "norm_bwd", CODE[0], 40001, 60, 2, "f32", "f32", 0.2),
        # the unit-test sized head with its layers: launches count
        _clip("clip tiny", TINY, 1, 2, 77, "f32", "f32", 0.6),
        # the search models' bf16 gradients in several hundred tensors, one model clipped and one not
        _clip("clip search", SEARCH, 2, 24, 0, "bf16", "bf16", 0.6),
        # fp32 gradients of the coding heads, summed over micro-batches, handed on in bf16
        _clip("clip code", CODE, 2, 0, 1, "f32", "bf16", 0.7),
        # one answer that is decoded alone
        _sample("sample one token", 1, CODE[1], "f32", "0.8,50,0.95,0", 3.0, 0.0),
        # a rollout step of 64 groups x 8 samples from the unchanged distribution
        _sample("sample rollout", 512, SEARCH[1], "f32", "1,0,1,0", 2.5, 0.0),
        # four roles with rules of their own on bf16 logits, some answers already finished
        _sample("sample roles", 301, STRESS[1], "bf16", "0.7,20,0.8,0;1,0,0.95,0;0,0,1,0;1.2,0,1,0.05", 3.0, 0.1),
    ]


def _size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "clip", "sample"])
    if op in ("norm_fwd", "norm_bwd"):
        H = rng.choice([TINY[0], RAG_QA[0], SEARCH[0], CODE[0], STRESS[0], 64 * _size(rng, 1, 128)])
        n_tok = _size(rng, 1, 100_000_000 // H)
        c = _norm("", op, H, n_tok, max(1, min(n_tok, _size(rng, 1, 500))), rng.choice([1, 1, 2, 3, 4]),
                  rng.choice(["none", "bf16", "f32"] if op == "norm_fwd" else ["bf16", "f32"]), rng.choice(["bf16", "f32"]),
                  rng.choice([0.0, 0.1, 0.2, 0.5]))
    elif op == "clip":
        hv = rng.choice([TINY, RAG_QA, SEARCH, (64 * _size(rng, 1, 40), 8 * _size(rng, 125, 19000))])
        grad = rng.choice(["f32", "bf16"])
        c = _clip("", hv, rng.choice([1, 2, 3]), rng.choice([0, 1, 6, 24]), rng.choice([0, 1, 77, 1001]), grad,
                  rng.choice(["f32", "bf16"]) if grad == "f32" else "bf16", rng.choice([0.1, 0.6, 2.0]))
        c["models"] = max(1, min(c["models"], 700_000_000 // sum(_shapes(c))))
    else:
        V = rng.choice([TINY[1], RAG_QA[1], CODE[1], _size(rng, 2, 200_000)])
        rules = [rng.choice([0.3, 0.7, 1.0, 1.0, 1.3, 0.0]) for _ in range(rng.choice([1, 2, 4]))]
        rules = ";".join("%g,%d,%g,%g" % (t, rng.choice([0, 0, 1, 20, 50, 1000]), rng.choice([1, 1, 0.8, 0.95, 0.99]),
                                          rng.choice([0, 0, 0.05, 0.001])) for t in rules)
        c = _sample("", _size(rng, 1, min(512, 70_000_000 // V)), V, rng.choice(["f32", "bf16"]), rules,
                    rng.choice([1.0, 2.5, 4.0]), rng.choice([0.0, 0.1]))
    del c["name"]
    return c


def _valid(n, masked):
    return n - int(masked * n)


def _width(t):
    return {"none": 0, "f32": 4, "bf16": 2}[t]


def _shapes(case):
    """Elements of the tensors of one model."""
    H = case["H"]
    return [H * case["V"], H] + ([case["odd"]] if case["odd"] else []) + [H * H, H * H, H * H, H * H, H, H] * case["blocks"]


def work(case):
    if case["op"] in ("norm_fwd", "norm_bwd"):
        H, n, K = case["H"], case["n_tok"], case["models"]
        m, w = _valid(n, case["masked"]), _width(case["residual"])
        by = n + K * H * _width(case["gamma"])
        if case["op"] == "norm_fwd":
            return {"bytes": by + (m + n) * H * (2 + w), "flops": 5.0 * m * H}
        return {"bytes": by + m * H * (2 + 2 * w) + n * H * w + K * H * 4, "flops": 10.0 * m * H}
    if case["op"] == "clip":
        n = case["models"] * sum(_shapes(case))
        return {"bytes": n * (_width(case["grad"]) + _width(case["out"])), "flops": 3.0 * n}
    n = _valid(case["n_rows"], case["masked"])
    return {"bytes": n * case["V"] * _width(case["logits"]) + case["n_rows"] * 25, "flops": 4.0 * n * case["V"]}


def _mask(n, masked, c):
    mask = torch.ones(n, dtype=torch.uint8)
    mask[torch.randperm(n, generator=c)[:n - _valid(n, masked)]] = 0
    return mask.cuda()


def _prepare_norm(case, g, c):
    H, n, K, S = case["H"], case["n_tok"], case["models"], case["n_inv"]
    # ragged answers, one of them empty where there are a few; every role is served by the model of its number
    cuts = torch.randint(0, n + 1, (S - 1,), generator=c).sort().values
    if S > 3:
        cuts[1] = cuts[0]
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])])
    role = torch.randint(0, K, (S,), generator=c)
    st = {"cu_seqlens": cu.cuda(), "inv_role": role.to(torch.int32).cuda(), "tok_mask": _mask(n, case["masked"], c)}

    def normal(dtype, scale):
        # rows of different sizes, as residual streams have
        t = torch.randn(n, H, generator=g, device="cuda")
        t *= scale * (0.25 + 2 * torch.rand(n, 1, generator=g, device="cuda"))
        return t.to(dtype)

    st["gamma"] = [(1 + 0.3 * torch.randn(H, generator=g, device="cuda")).to(TYPES[case["gamma"]]) for _ in range(K)]
    kind = TYPES.get(case["residual"])
    if case["op"] == "norm_fwd":
        st["x"] = normal(torch.bfloat16, 1.0)
        st["residual"] = normal(kind, 4.0) if kind else None
        st["y"], st["res_out"] = torch.empty_like(st["x"]), torch.empty(n, H, dtype=kind, device="cuda") if kind else None
    else:
        st["res"], st["dy"] = normal(kind, 4.0), normal(torch.bfloat16, 1e-3)
        st["dres"] = normal(kind, 1e-3) if kind == torch.float32 else None
        st["dx"] = torch.empty(n, H, dtype=kind, device="cuda")
        st["dgamma"] = [torch.empty(H, device="cuda") for _ in range(K)]
    if own:
        from paper_2605_26646_b200 import binding as ub
        st["ctx"] = ub.Context(0, max(256, ub.unity_rms_norm_workspace_bytes(n, H, K)))
    return st


def _prepare_clip(case, g, c):
    K, sizes = case["models"], _shapes(case)
    st = {"buckets": [], "outs": [], "max_norm": []}
    tensors, outs, models = [], [], []
    for k in range(K):
        # all gradients of a model sit behind one another in one bucket
        b = torch.randn(sum(sizes), generator=g, device="cuda")
        b *= 1e-3 * (1 + k)
        st["max_norm"].append((case["tight"] if k == 0 else 2.0) * 1e-3 * (1 + k) * math.sqrt(sum(sizes)))
        st["buckets"].append(b.to(TYPES[case["grad"]]))
        del b
        st["outs"].append(torch.empty(sum(sizes), dtype=TYPES[case["out"]], device="cuda"))
        tensors += torch.split(st["buckets"][k], sizes)
        outs += torch.split(st["outs"][k], sizes)
        models += [k] * len(sizes)
    st["norm"], st["coef"] = torch.empty(K, device="cuda"), torch.empty(K, device="cuda")
    if own:
        from paper_2605_26646_b200 import binding as ub
        st["grads"] = ub.GradTensors(tensors, models, outs)
        st["ctx"] = ub.Context(0, ub.unity_clip_grad_norm_workspace_bytes(len(tensors), K))
    return st


def _rules(case):
    return [tuple(float(x) for x in r.split(",")) for r in case["rules"].split(";")]


def _prepare_sample(case, g, c):
    n, V, rules = case["n_rows"], case["V"], _rules(case)
    z = torch.randn(n, V, generator=g, device="cuda")
    z *= case["spread"]
    # what the answer goes on with: a few entries stand out, more in some rows than in others
    gain = (3 + 9 * torch.rand(n, 8, generator=g, device="cuda")) * torch.rand(n, 1, generator=g, device="cuda")
    at = torch.randint(0, V, (n, 8), generator=g, device="cuda")
    rows = torch.arange(n, device="cuda")
    for j in range(8):                                             # (one after another: a place may come twice)
        z[rows, at[:, j]] += gain[:, j]
    if V > 64:                                                     # entries behind the tokenizer's last token
        z[:, V - V // 64:] = -math.inf
    role = torch.randint(0, len(rules), (n,), generator=c).to(torch.int32)
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    st = {"logits": z.to(TYPES[case["logits"]]), "role": role.cuda(), "mask": _mask(n, case["masked"], c),
          "u": torch.rand(n, generator=g, device="cuda"), "rules": [(t, int(k), p, m) for t, k, p, m in rules],
          "token": torch.empty(n, **i32), "n_kept": torch.empty(n, **i32), "logp": torch.empty(n, **f32),
          "logp_kept": torch.empty(n, **f32)}
    if own:
        from paper_2605_26646_b200 import binding as ub
        st["ctx"] = ub.Context(0, 256)
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.Generator().manual_seed(seed)
    make = {"clip": _prepare_clip, "sample": _prepare_sample}.get(case["op"], _prepare_norm)
    return {"case": case, **make(case, g, c)}


def _run_own(st):
    case = st["case"]
    op = case["op"]
    roles = list(range(case.get("models", 0)))
    if op == "norm_fwd":
        st["ctx"].rms_norm_fwd(st["x"], st["gamma"], st["cu_seqlens"], st["inv_role"], roles, st["tok_mask"], EPS, st["y"],
                               residual=st["residual"], res_out=st["res_out"])
        return [t for t in (st["y"], st["res_out"]) if t is not None]
    if op == "norm_bwd":
        st["ctx"].rms_norm_bwd(st["res"], st["gamma"], st["cu_seqlens"], st["inv_role"], roles, st["tok_mask"], EPS, st["dy"],
                               st["dx"], dres=st["dres"], dgamma=st["dgamma"])
        return [st["dx"], st["dgamma"]]
    if op == "clip":
        st["ctx"].clip_grad_norm(st["grads"], st["max_norm"], st["norm"], st["coef"])
        return [st["norm"], st["coef"], st["outs"]]
    st["ctx"].sample(st["logits"], st["rules"], st["u"], st["token"], row_role=st["role"], row_mask=st["mask"], logp=st["logp"],
                     logp_kept=st["logp_kept"], n_kept=st["n_kept"])
    return [st["token"], st["logp"], st["logp_kept"], st["n_kept"]]


def _plain_norm(st):
    case = st["case"]
    n, H, K = case["n_tok"], case["H"], case["models"]
    lens = st["cu_seqlens"][1:] - st["cu_seqlens"][:-1]
    model = torch.repeat_interleave(st["inv_role"].long(), lens)
    on = (st["tok_mask"] != 0).unsqueeze(1)
    gamma = torch.stack([w.float() for w in st["gamma"]])[model]
    if case["op"] == "norm_fwd":
        r = st["x"].float()
        if st["residual"] is not None:
            r = r + st["residual"].float()
        s = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)
        y = torch.where(on, gamma * r * s, 0.0).to(torch.bfloat16)
        return [y] if st["residual"] is None else [y, torch.where(on, r, 0.0).to(st["residual"].dtype)]
    r, dy = st["res"].float(), st["dy"].float()
    s = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)
    gr = dy * gamma
    dr = s * gr - r * s * s * s * (gr * r).mean(1, keepdim=True)
    if st["dres"] is not None:
        dr = dr + st["dres"].float()
    share = torch.where(on, dy * r * s, 0.0)
    return [torch.where(on, dr, 0.0).to(st["res"].dtype), [(share * (model == k).unsqueeze(1)).sum(0) for k in range(K)]]


def _plain_clip(st):
    norm = [torch.sqrt(sum((part.float() ** 2).sum(dtype=torch.float64) for part in torch.split(b, 1 << 28))).float() for b in st["buckets"]]
    coef = [torch.where(v > m, m / v, 1.0) for v, m in zip(norm, st["max_norm"])]
    return [torch.stack(norm), torch.stack(coef), [(b.float() * f).to(o.dtype) for b, f, o in zip(st["buckets"], coef, st["outs"])]]


def _plain_sample(st):
    z = st["logits"].double()                                     # 64 bits: u * mass may lie next to a running sum
    n, V = z.shape
    rule = torch.tensor(st["rules"], dtype=torch.float64).to(torch.float32).cuda()[st["role"].long()]     # parameters are 32-bit numbers
    T, k, top_p, min_p = rule.double().unsqueeze(2).unbind(1)
    greedy = T == 0
    z = z / torch.where(greedy, 1.0, T)
    order = torch.sort(z, dim=1, descending=True, stable=True)
    x = order.values - order.values[:, :1]
    del z
    e = x.exp()
    rank = torch.arange(V, device=x.device).unsqueeze(0)
    ok = ((k <= 0) | (rank < k)) & ((min_p <= 0) | (x >= torch.log(min_p))) & (x > -math.inf)
    part = torch.where(ok, e, 0.0)
    run = part.cumsum(1)
    ok &= (top_p >= 1) | (run - part < top_p * run[:, -1:])
    ok &= ~greedy | (rank == 0)
    del run, part
    lse = torch.log(e.sum(1))
    held = torch.zeros_like(e).scatter_(1, order.indices, torch.where(ok, e, 0.0))
    run = held.cumsum(1)
    total = run[:, -1:]
    hit = (run > st["u"].double().unsqueeze(1) * total) & (held > 0)
    token = torch.where(hit, rank, V).amin(1, keepdim=True)
    last = torch.where(held > 0, rank, 0).amax(1, keepdim=True)
    token = torch.where(token == V, last, token)
    own_e = held.gather(1, token)
    on = st["mask"] != 0
    logp = torch.where(on, (torch.log(own_e.squeeze(1)) - lse), 0.0)
    logk = torch.where(on, torch.log(own_e / total).squeeze(1), 0.0)
    return [torch.where(on, token.squeeze(1), -1).to(torch.int32), logp.float(), logk.float(),
            torch.where(on, ok.sum(1), 0).to(torch.int32)]


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    return _plain_clip(state) if op == "clip" else _plain_sample(state) if op == "sample" else _plain_norm(state)


def _exact_norm(case, st):
    """Automatic differentiation of the forward formula, in blocks of rows of one answer."""
    f64, n, H = torch.float64, case["n_tok"], case["H"]
    gamma = [w.to(f64).requires_grad_(True) for w in st["gamma"]]
    back = case["op"] == "norm_bwd"
    base = st["res"] if back else st["x"]
    first = torch.zeros(n, H, dtype=f64, device="cuda")
    second = torch.zeros(n, H, dtype=f64, device="cuda") if not back and st["residual"] is not None else None
    bounds, roles = st["cu_seqlens"].tolist(), st["inv_role"].tolist()
    for s, k in enumerate(roles):
        for a in range(bounds[s], bounds[s + 1], 4096):
            b = min(a + 4096, bounds[s + 1])
            rows = a + torch.nonzero(st["tok_mask"][a:b]).squeeze(1)
            if not rows.numel():
                continue
            r = base[rows].to(f64)
            if not back and st["residual"] is not None:
                r = r + st["residual"][rows].to(f64)
            r.requires_grad_(back)
            y = r * (r.square().mean(1, keepdim=True) + EPS).rsqrt() * gamma[k]
            if not back:
                first[rows] = y.detach()
                if second is not None:
                    second[rows] = r
                continue
            y.backward(st["dy"][rows].to(f64))
            first[rows] = r.grad if st["dres"] is None else r.grad + st["dres"][rows].to(f64)
    if back:
        return [first, [torch.zeros(H, dtype=f64, device="cuda") if w.grad is None else w.grad for w in gamma]]
    return [first] if second is None else [first, second]


def _exact_clip(case, st):
    norms, coefs, outs = [], [], []
    for b, most in zip(st["buckets"], st["max_norm"]):
        d = b.double()
        norms.append(torch.linalg.vector_norm(d))
        # the bound is a 32-bit number
        coefs.append(torch.clamp(torch.tensor(most, dtype=torch.float32).double().cuda() / norms[-1], max=1.0))
        outs.append(d.mul_(coefs[-1]))
    return [torch.stack(norms), torch.stack(coefs), outs]


def _exact_sample(case, st):
    """Row by row: a softmax, entries taken from the likeliest down, then a search among the kept."""
    out = []
    rules = torch.tensor(st["rules"], dtype=torch.float64).to(torch.float32).tolist()
    for i in range(case["n_rows"]):
        if not st["mask"][i]:
            out.append((-1, 0.0, 0.0, 0))
            continue
        T, k, top_p, min_p = rules[int(st["role"][i])]
        row = st["logits"][i].double()
        p = torch.softmax(row / (T or 1.0), 0)
        by = torch.argsort(row, descending=True, stable=True)
        by = by[row[by] > -math.inf]
        if T == 0:
            by = by[:1]
        if k > 0:
            by = by[:int(k)]
        q = p[by]
        if min_p > 0:
            q = q[q >= min_p * q[0]]
        if top_p < 1:
            done = torch.cumsum(q, 0)
            q = q[:1 + int((done[:-1] < top_p * done[-1]).sum())]
        by = by[:q.numel()].sort().values
        q = p[by]
        done = torch.cumsum(q, 0)
        j = min(int((done <= float(st["u"][i]) * float(done[-1])).sum()), q.numel() - 1)
        out.append((int(by[j]), math.log(float(q[j])), math.log(float(q[j] / done[-1])), q.numel()))
    cols = list(zip(*out))
    return [torch.tensor(cols[0], dtype=torch.int32), torch.tensor(cols[1], dtype=torch.float64),
            torch.tensor(cols[2], dtype=torch.float64), torch.tensor(cols[3], dtype=torch.int32)]


def exact(case, seed):
    st = prepare(case, seed)
    return {"clip": _exact_clip, "sample": _exact_sample}.get(case["op"], _exact_norm)(case, st)
