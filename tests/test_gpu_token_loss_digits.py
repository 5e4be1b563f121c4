"""GPU: digits of the token losses that the bounds of test_gpu_token_losses.py cannot see - losses and target gradients of
sure tokens, the logits' scale, logits that are not finite, and few rows in workspaces that do not hold them all."""
import numpy as np
import pytest
import torch

from paper_2605_26646_b200 import binding as ub
from test_gpu_token_losses import B, U, Problem, call, check, context, oracle

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ sure tokens
class Sure:
    """Rows whose logits are exact in fp32 (two products each): z_y rises from 12 to 30 (14 to 28 and the target's own background) over a background within +-2.

    Hidden channel 1 times a multiple of 1/16 is the background, channel 2 + t is switched on for the t-th target alone."""

    def __init__(self, N, V, seed):
        rng = np.random.default_rng(seed)
        H, spots = 64, sorted({0, 7, V // 3, V // 2, V - 1} | ({255, 256} if V > 256 else set()))
        W, h = np.zeros((V, H), np.float32), np.zeros((N, H), np.float32)
        W[:, 1] = rng.integers(-32, 33, V) / 16
        W[spots, 2 + np.arange(len(spots))] = 1
        t = rng.integers(0, len(spots), N)
        h[:, 1] = 1
        h[np.arange(N), 2 + t] = np.round(np.linspace(14, 28, N) * 8) / 8          # bf16 holds them
        self.N, self.V, self.H, self.K = N, V, H, 1
        self.y = np.asarray(spots)[t]
        z = h.astype(np.float64) @ W.astype(np.float64).T
        at = np.arange(N)
        self.z, zy = z, z[at, self.y]
        e = np.exp(z - zy[:, None])
        e[at, self.y] = 0
        self.dy = np.log1p(e.sum(1))                                               # lse - z_y
        self.h = h.astype(np.float64)
        cuda = dict(device="cuda")
        self.d_hidden = torch.tensor(h, **cuda).to(torch.bfloat16)
        self.d_W = [torch.tensor(W, **cuda).to(torch.bfloat16)]
        assert torch.equal(self.d_hidden.float().cpu(), torch.from_numpy(h)) and torch.equal(self.d_W[0].float().cpu(), torch.from_numpy(W))
        self.d_cu = torch.tensor([0, N], **cuda)
        self.d_inv_role = torch.zeros(1, dtype=torch.int32, **cuda)
        self.role_model = [0]
        self.d_target = torch.tensor(self.y, dtype=torch.int32, **cuda)
        self.d_mask = torch.ones(N, dtype=torch.uint8, **cuda)
        self.d_weight = torch.ones(N, **cuda)
        self.n_top = 1
        self.d_top_ids = self.d_target[:, None].contiguous()
        self.d_top_vals = torch.zeros(N, 1, **cuda)
        # relative error of dy: exponents of up to 45 octaves whose reference, scale, constant and product are rounded (4 u of
        # the exponent), the logits' scale (H/16 * 1.6e-8 + 4e-8 of the logit), sums of 32 + 8 + V/256 + 148 terms, and
        # exponentials, the quotient and its logarithm of 2^-21 in all
        self.tol = 45 * 4 * U * np.log(2) + 32 * (H / 16 * 1.6e-8 + 4e-8) + (40 + V / 256 + 148) * U + 2.0 ** -21


@pytest.mark.parametrize("form", ["ce", "hard", "list"])
@pytest.mark.parametrize("N,V,grads", [(1, 520, "all"), (40, 4104, "all"), (100, 520, "none"), (300, 4104, "all"), (1500, 1000, "all"),
                                       (64, 8, "all"), (33, 40000, "none")])
def test_sure_tokens_keep_their_digits(N, V, grads, form):
    """A loss far below one, relative to itself: cross entropy, the targets' part of a distillation, a teacher as sure as the model."""
    p = Sure(N, V, seed=N + V)
    ctx = context(p, "kd")
    op, kw = ("ce", {}) if form == "ce" else ("kd", dict(kd=0.0, hard=0.5) if form == "hard" else {})
    g = call(ctx, p, op, grads=grads, target=form != "list", **kw)
    ctx.check_status()
    f = 0.5 if form == "hard" else 1.0
    got = g["tok_loss"].double().cpu().numpy()
    assert np.all(np.abs(got - f * p.dy) <= (p.tol + 2 * U) * f * p.dy), np.max(np.abs(got / (f * p.dy) - 1))
    want = f * p.dy.sum() / N
    assert abs(float(g["loss"][0]) - want) <= (p.tol + 16 * U) * want
    ctx.close()


@pytest.mark.parametrize("form", ["ce", "hard", "list"])
@pytest.mark.parametrize("N", [1, 300])
@pytest.mark.parametrize("V", [520, 4104])
def test_sure_tokens_keep_their_targets_gradient(N, V, form):
    """fp32 dW at the targets' rows: channel 2 + t is switched on in the t-th target's rows alone, which makes dW there a sum of
    terms of one sign, (p_y - 1) h / N."""
    p = Sure(N, V, seed=3 * N + V)
    ctx = context(p, "kd")
    op, kw = ("ce", {}) if form == "ce" else ("kd", dict(kd=0.0, hard=0.5) if form == "hard" else {})
    g = call(ctx, p, op, dw=torch.float32, target=form != "list", **kw)
    ctx.check_status()
    f = 0.5 if form == "hard" else 1.0
    dW = g["dW"][0].double().cpu().numpy()
    for y in np.unique(p.y):
        i = np.nonzero(p.y == y)[0]
        t = int(np.nonzero(p.h[i[0], 2:])[0][0]) + 2
        want = f * (np.expm1(-p.dy[i]) * p.h[i, t]).sum() / N
        # G's rounding to bf16, the fp32 sums over at most 300 rows
        assert abs(dW[y, t] - want) <= (B * (1 + B) + p.tol + (N / 16 + 8) * 2 * U) * abs(want), (y, dW[y, t] / want - 1)
    ctx.close()


# ------------------------------------------------------------------------------------------------ the logits' scale
def scale_excess(H):
    """What the logits' scale adds to the temperature: the tensor core's mean cut on sums of products of both signs."""
    return 1.6e-8 * (H // 16) + 4e-8


def one_target(h, w, V=264, y=5):
    """Rows `h` whose one large logit is h w at `y` (the others are 0), and what cross entropy's lse says of them, relative."""
    N, H = h.shape
    W = torch.zeros(V, H, dtype=torch.bfloat16)
    W[y] = w
    z = (h.double() @ W[y].double()).numpy()
    cuda = dict(device="cuda")
    ctx = ub.Context(0, ub.unity_token_loss_workspace_bytes(N, H, V, 1, 0, False))
    loss, lse = torch.empty(1, **cuda), torch.empty(N, **cuda)
    ctx.cross_entropy_fwd_bwd(h.cuda(), [W.cuda()], torch.tensor([0, N], **cuda), torch.zeros(1, dtype=torch.int32, **cuda), [0],
                              torch.full((N,), y, dtype=torch.int32, **cuda), None, 1.0, 0.0, 0.0, None, False, None, loss, None, lse)
    ctx.check_status()
    ctx.close()
    want = z + np.log1p((V - 1) * np.exp(-z))
    return (lse.double().cpu().numpy() - want) / want


@pytest.mark.parametrize("noise", [1, 3, 8])
@pytest.mark.parametrize("H", [256, 896, 1536, 3584])
def test_scale_takes_back_the_mean_cut_of_products_of_both_signs(H, noise):
    """Left out or taken twice, the excess would leave a mean of about minus or plus itself; half of it is the bound (the cut was
    measured between 0.92 and 1.34 of it on such rows).  Logits from 33 to 60: their row's reference is the logit itself, so lse has no
    more roundings than scale, product and sum (3 u)."""
    g = torch.Generator().manual_seed(100 * H + noise)
    w = (torch.randn(H, generator=g) / H ** 0.5).to(torch.bfloat16)
    h = 46 * w.float() + noise * torch.randn(400, H, generator=g)
    h = (h * (torch.linspace(35, 58, 400) / (h.double() @ w.double()).float())[:, None]).to(torch.bfloat16)
    err = one_target(h, w)
    assert abs(err.mean()) <= scale_excess(H) / 2 + 3 * U, (err.mean(), scale_excess(H))


@pytest.mark.parametrize("N", [100, 600])
@pytest.mark.parametrize("H", [896, 1536, 3584])
def test_scale_of_products_of_one_sign(H, N):
    """No mean is taken back here: 16 products and the sum so far are cut to the largest one's grid, and products of one sign lose on the
    same side (0.4 to 2.8 times the excess, the more the wider).  What holds is the accumulator's bound: a step cuts at most 2 u of the
    sum so far, H/16 + 2 steps, all downwards, and then the excess and 3 u."""
    g = torch.Generator().manual_seed(H + N)
    w = (torch.rand(H, generator=g) + 0.5).to(torch.bfloat16)
    h = torch.rand(N, H, generator=g) + 0.5
    h = (h * (torch.linspace(34, 59, N) / (h.double() @ w.double()).float())[:, None]).to(torch.bfloat16)
    err = one_target(h, w)
    assert np.all(err <= scale_excess(H) + 3 * U) and np.all(err >= scale_excess(H) - (H / 16 + 2) * 2 * U - 3 * U), (err.min(), err.max())


@pytest.mark.parametrize("where", [0, 17, -1])
@pytest.mark.parametrize("H", [64, 896, 3584])
def test_scale_of_rows_that_sit_in_one_channel(H, where):
    """Their logits are exact in the tensor core, so the excess stands in lse as it is, to the roundings of scale, product and sum."""
    h = torch.zeros(112, H, dtype=torch.bfloat16)
    h[:, where] = torch.arange(112) / 4 + 33                   # up to 60.75: bf16 holds them
    w = torch.zeros(H, dtype=torch.bfloat16)
    w[where] = 1
    err = one_target(h, w)
    assert np.all(np.abs(err - scale_excess(H)) <= 3 * U), (err.min(), err.max(), scale_excess(H))
