"""GPU: forms of the token losses at the edges - gradients of the head added to old values where a warp's rows end inside the
vocabulary's last tile, few tokens in workspaces that do not hold all their logits, values that are not finite or stand for masks."""
import numpy as np
import pytest
import torch

from paper_2605_26646_b200 import binding as ub
from test_gpu_token_losses import B, U, Problem, call, check, context, oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V,K", [(50, 64, 8, 1), (100, 320, 1000, 1), (300, 192, 136, 2), (700, 1088, 2504, 1), (1500, 576, 4120, 1),
                                     (1200, 128, 40000, 2)])
def test_adding_to_the_heads_gradients_at_ragged_vocabularies(N, H, V, K, op, dw):
    """V ends 8, 16 or 24 entries into a warp's 32 rows of dW: the others of the warp neither read nor write."""
    p = Problem(N, H, V, K, K, n_top=5, seed=N + V).gpu()
    ctx = context(p, op)
    guard = 64
    torch.manual_seed(V)
    whole = [torch.randn((V + 2 * guard) * H, device="cuda").to(dw) * 0.01 for _ in range(K)]
    before = [w.clone() for w in whole]
    old = [w[guard * H:-guard * H].view(V, H) for w in whole]
    base = [x.double().cpu().numpy() for x in old]
    g = call(ctx, p, op, accumulate=True, dW=old)
    ctx.check_status()
    check(p, g, oracle(p, op), base=base)
    for w, b in zip(whole, before):
        assert torch.equal(w[:guard * H], b[:guard * H]) and torch.equal(w[-guard * H:], b[-guard * H:])
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V,K", [(40, 64, 4104, 16), (64, 192, 20000, 1), (1, 64, 60000, 1), (33, 128, 10000, 3)])
def test_up_to_64_tokens_in_smaller_workspaces(N, H, V, K, op):
    """The low halves of dL/dz exist where one block holds all models' rows and their logits.  A workspace without room for that
    takes the other forms, whose dL/dz is rounded to bf16 once: b of it in place of b^2."""
    p = Problem(N, H, V, K, K, n_inv=min(N, 40), n_top=6, seed=N + V).gpu()
    o = oracle(p, op)
    loose = dict(o, dG=o["dG"] + (B * (1 + B) - B * B) * np.abs(o["G"]))
    full = ub.unity_token_loss_workspace_bytes(p.N, p.H, p.V, p.K, p.n_top if op == "kd" else 0)
    now, ways = full, set()
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
        check(p, g, o if now == full else loose)
        ctx.close()
        now = now * 15 // 16 // 256 * 256
    assert len(ways) >= 2, ways


def rows_of(p, k):
    """The valid rows of model k."""
    role = np.repeat(p.inv_role.numpy(), np.diff(p.cu.numpy()))
    return np.nonzero((np.asarray(p.role_model)[role] == k) & (p.mask.numpy() != 0))[0]


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("N,H,V", [(40, 64, 520), (100, 320, 1000), (400, 64, 4104), (1600, 128, 1000)])
def test_hidden_rows_that_are_not_finite_stay_by_themselves(N, H, V, bad, op):
    """A valid row with a NaN or an infinity: its loss, lse and gradient are NaN (as its model's loss and dW, which sum over it); the
    other rows and the other model come out bit for bit as they do without it."""
    p = Problem(N, H, V, 2, 2, n_top=5, seed=N, short_lists=False).gpu()
    ctx = context(p, op)
    clean = call(ctx, p, op, dw=torch.float32)
    own = rows_of(p, 0)
    hit = own[[0, len(own) // 2, -1]]
    p.d_hidden = p.d_hidden.clone()
    p.d_hidden[torch.from_numpy(hit).cuda(), H // 2] = bad
    g = call(ctx, p, op, dw=torch.float32)
    ctx.check_status()
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[torch.from_numpy(hit).cuda()] = False
    for key in ("tok_loss", "lse", "dHidden"):
        assert torch.all(torch.isnan(g[key][~keep])), key
        assert torch.equal(g[key][keep], clean[key][keep]), key
    assert torch.isnan(g["loss"][0]) and torch.equal(g["loss"][1], clean["loss"][1])
    assert torch.all(torch.isnan(g["dW"][0])) and torch.equal(g["dW"][1], clean["dW"][1])
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V", [(40, 64, 520), (100, 320, 1000), (400, 64, 4104), (1600, 128, 1000)])
def test_masked_rows_may_hold_anything(N, H, V, op):
    """Hidden values, weights, targets and lists of masked tokens are not read."""
    p = Problem(N, H, V, 2, 2, n_top=5, seed=N + 1).gpu()
    ctx = context(p, op)
    clean = call(ctx, p, op, hard=0.5) if op == "kd" else call(ctx, p, op)
    off = p.d_mask == 0
    assert int(off.sum()) > 2
    for name, what in (("d_hidden", float("nan")), ("d_weight", float("inf")), ("d_target", V + 7), ("d_top_ids", V), ("d_top_vals", float("nan"))):
        t = getattr(p, name).clone()
        t[off] = what
        setattr(p, name, t)
    g = call(ctx, p, op, hard=0.5) if op == "kd" else call(ctx, p, op)
    ctx.check_status()
    for key in ("loss", "tok_loss", "lse", "dHidden"):
        assert torch.equal(g[key], clean[key]), key
    assert all(torch.equal(a, b) for a, b in zip(g["dW"], clean["dW"]))
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("first", [0, 300, 700])
@pytest.mark.parametrize("N", [30, 100, 400])
def test_entries_of_the_vocabulary_that_are_masked_by_the_lowest_value(N, first, op):
    """Rows of the head at the type's lowest value (logits of -1e38 and less, to -inf), whole column tiles of them: they have probability 0,
    and the others' losses and gradients are those of a head without them."""
    H, V, n_off = 64, 1320, 600
    p = Problem(N, H, V, 1, 1, n_top=6, seed=N + first, spread=1.0)
    off = np.arange(first, first + n_off)
    on = np.setdiff1d(np.arange(V), off)
    rng = np.random.default_rng(N)
    hidden = p.hidden.float()
    hidden[:, 0] = torch.from_numpy(rng.random(N).astype(np.float32)) + 0.5
    hidden[::3, 0] *= 2
    W = p.W[0].clone()
    W[:, 0] = 0
    p.hidden, p.target = hidden.to(torch.bfloat16), torch.from_numpy(rng.choice(on, N).astype(np.int32))
    p.top_ids = torch.from_numpy(np.where(p.top_ids.numpy() < 0, -1, rng.choice(on, p.top_ids.shape)).astype(np.int32))
    q = Problem(N, H, V, 1, 1, n_top=6, seed=N + first, spread=1.0)      # the same rows over the entries that are left
    where = np.full(V + 1, -1)
    where[on] = np.arange(on.size)
    q.hidden, q.V, q.W = p.hidden, on.size, [W[on]]
    q.target = torch.from_numpy(where[p.target.numpy()].astype(np.int32))
    q.top_ids = torch.from_numpy(where[p.top_ids.numpy()].astype(np.int32))
    W[off] = 0
    W[off, 0] = torch.finfo(torch.bfloat16).min
    p.W = [W]
    p.gpu()
    ctx = context(p, op)
    g = call(ctx, p, op)
    ctx.check_status()
    assert torch.all(g["dW"][0][torch.from_numpy(off).cuda()] == 0)
    g["dW"] = [g["dW"][0][torch.from_numpy(on).cuda()]]
    check(q, g, oracle(q, op))
    ctx.close()


@pytest.mark.parametrize("N", [20, 300])
def test_logits_of_minus_infinity(N):
    """Evaluation: an entry at -inf has no share in lse; a target at -inf costs inf; a row of nothing else has lse -inf and no loss."""
    H, V = 64, 520
    p = Problem(N, H, V, 1, 1, seed=N, mask=0.0)
    h = p.hidden.float()
    h[:, 0] = 0
    h[1, 0], h[2, 0] = 1, 1
    p.hidden = h.to(torch.bfloat16)
    W = p.W[0].clone()
    W[:, 0] = 0
    p.W = [W]
    p.gpu()
    ctx = context(p, "ce")
    base = call(ctx, p, "ce", grads="none")
    # rows 1 and 2 see -inf at some entries (0 x inf would be NaN in the others, so they get a head of their own)
    q = Problem(2, H, V, 1, 1, seed=N, mask=0.0)
    q.hidden, q.target = p.hidden[1:3], torch.tensor([p.target[1], 11], dtype=torch.int32)
    if int(q.target[0]) in (11, 300, 519):
        q.target[0] = 12
    q.weight = q.weight * 0 + 1
    Wq = W.clone()
    Wq[[11, 300, 519], 0] = float("-inf")
    q.W = [Wq]
    q.gpu()
    g = call(ctx, q, "ce", grads="none")
    ctx.check_status()
    z = q.hidden.double() @ Wq.double().T
    want = torch.logsumexp(z, 1)
    got = g["lse"].double().cpu()
    ez = (H / 16 + 2) * 2 * U * (q.hidden.double().abs() @ torch.where(torch.isinf(Wq), 0, Wq).double().abs().T).max(1).values
    assert torch.all((got - want).abs() <= ez + 2.0 ** -17 + 2 * U * want.abs())
    assert torch.isfinite(g["tok_loss"][0]) and float(g["tok_loss"][1]) == float("inf") and torch.all(torch.isfinite(base["lse"]))
    q.d_W = [torch.where(torch.arange(H, device="cuda") == 0, float("-inf"), q.d_W[0].float()).to(torch.bfloat16)]
    g = call(ctx, q, "ce", grads="none")
    ctx.check_status()
    assert torch.all(g["lse"] == float("-inf")) and torch.all(torch.isnan(g["tok_loss"])) and torch.all(torch.isnan(g["loss"]))
    ctx.close()


@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("H,V,cuts", [(64, 520, [30, 70]), (128, 264, [1, 64, 65]), (320, 2000, [10, 240, 50]), (1344, 20000, [5, 700]),
                                      (64, 40000, [64, 200, 3]), (256, 1000, [2, 900, 40, 60, 0]), (576, 30000, [20, 100])])
def test_models_of_few_rows_beside_others(H, V, cuts, op, dw):
    """Up to 64 rows of a model take the low halves of dL/dz however many rows the other models have (in a batch of up to 1024): their
    gradients are off by b^2 of G in place of b."""
    N = sum(cuts)
    p = Problem(N, H, V, len(cuts), len(cuts), n_inv=len(cuts), n_top=6, seed=N + V, mask=0.0)
    p.cu = torch.from_numpy(np.concatenate([[0], np.cumsum(cuts)]))
    p.inv_role = torch.arange(len(cuts), dtype=torch.int32)
    p.gpu()
    ctx = context(p, op)
    o = oracle(p, op)
    if N > 64:
        few = np.asarray(cuts)[o["tok_model"]] <= 64
        o["dG"][few] -= (B * (1 + B) - B * B) * np.abs(o["G"][few])
    g = call(ctx, p, op, dw=dw)
    ctx.check_status()
    check(p, g, o)
    again = call(ctx, p, op, dw=dw)
    assert torch.equal(g["dHidden"], again["dHidden"]) and all(torch.equal(a, b) for a, b in zip(g["dW"], again["dW"]))
    old = [torch.full((V, H), 0.5, device="cuda", dtype=dw) for _ in cuts]
    check(p, call(ctx, p, op, accumulate=True, dW=old), o, base=[np.full((V, H), 0.5)] * len(cuts))
    ctx.check_status()
    ctx.close()


@pytest.mark.parametrize("op", ["ce", "kd"])
@pytest.mark.parametrize("N,H,V", [(100, 64, 520), (300, 1344, 30000), (1024, 128, 2000)])
def test_batches_with_few_valid_rows(N, H, V, op):
    """The same for a batch of which the mask leaves at most 64 rows."""
    p = Problem(N, H, V, 1, 1, n_top=6, seed=N, mask=0.95)
    assert 0 < int(p.mask.sum()) <= 64
    p.gpu()
    ctx = context(p, op)
    o = oracle(p, op)
    o["dG"] -= (B * (1 + B) - B * B) * np.abs(o["G"])
    for dw in (torch.bfloat16, torch.float32):
        check(p, call(ctx, p, op, dw=dw), o)
    ctx.check_status()
    ctx.close()
