"""GPU: forms of the token losses at the edges - gradients of the head added to old values where a warp's rows end inside the
vocabulary's last tile, few tokens in workspaces that do not hold all their logits, entries masked by the lowest value."""
import numpy as np
import pytest
import torch

from paper_2605_26646_b200 import binding as ub
from test_gpu_token_losses import B, Problem, call, check, context, oracle

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
