"""GPU parity of sampling against the fp64 oracle: tokens and numbers of kept entries are equal.

Tolerances, derived.  A log-probability is x - log(mass): x in fp64, the mass of fp32 exponentials within 2^-19 of itself (ex2 2^-22,
the roundings of its argument 1.5e-6 under the distribution, sums of four 1.8e-7), so 2^-19 in all, and the rounding of the result."""
import numpy as np
import pytest
import torch

from oracle import unity_oracle as orc
from paper_2605_26646_b200 import binding as ub

pytestmark = pytest.mark.gpu

F32, B16 = torch.float32, torch.bfloat16
OFF = (1.0, 0, 1.0, 0.0)
RULES = [OFF, (0.0, 0, 1.0, 0.0), (0.7, 20, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.02), (0.8, 50, 0.95, 0.001),
         (1.0, 1, 0.5, 1.0), (0.05, 1000, 0.999, 0.0), (1.0, 700, 0.5, 0.0), (1e-6, 5, 0.7, 0.0), (1e6, 0, 0.3, 0.0), (1.0, 0, 1e-6, 0.0),
         (1.0, 10 ** 9, 1.0, 0.0), (2.0, -1, 0.99999994, 0.0)]


def draw(z, rules, u, role=None, mask=None, ctx=None):
    n = z.shape[0]
    ctx = ctx or ub.Context(0, 256)
    o = [torch.full((n,), 7, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda"),
         torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7, dtype=torch.int32, device="cuda")]
    ctx.sample(z, rules, u, o[0], role, mask, o[1], o[2], o[3])
    return [t.cpu().numpy() for t in o]


def check(z, rules, u, role, got):
    zs, us = z.float().cpu().numpy(), u.cpu().numpy()
    for i in range(z.shape[0]):
        rule = rules[0 if role is None else int(role[i])]
        t, lp, lk, n = orc.sample_row(zs[i], *rule, us[i])
        at = (i, rule, us[i], [g[i] for g in got], (t, lp, lk, n))
        assert got[0][i] == t and got[3][i] == n, at
        for v, w in ((got[1][i], lp), (got[2][i], lk)):
            assert (np.isnan(v) and np.isnan(w)) or abs(v - w) <= 2.0 ** -19 * 1.01 + 2.0 ** -23 * abs(w) + 1e-12, at


def logits(n, V, kind, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(n, V, generator=g, device="cuda")
    if kind == "peaked":
        z = z * 2
        for j in range(6):
            z[torch.arange(n), torch.randint(0, V, (n,), generator=g, device="cuda")] += 10.0 + j
    elif kind == "wide":
        z = z * 4
    elif kind == "ties":
        z = (z * 2).round() / 2
    elif kind == "masked":
        z = torch.where(torch.rand(n, V, generator=g, device="cuda") < 0.7, -float("inf"), z * 3)
        z[:, V // 2] = 1.0
    elif kind == "lowest":
        z = torch.where(torch.rand(n, V, generator=g, device="cuda") < 0.9, torch.finfo(dtype).min, z * 3)
        z[:, V // 3] = 0.0
    elif kind == "negative":
        z = z * 0.1 - 1e4
    elif kind == "equal":
        z = torch.full_like(z, -3.25)
    elif kind == "signed zeros":
        z = torch.where(z > 0, 0.0, -0.0)
    return z.to(dtype)


KINDS = ["normal", "peaked", "wide", "ties", "masked", "lowest", "negative", "equal", "signed zeros"]


@pytest.mark.parametrize("V", [1, 2, 7, 64, 513, 4096, 20000, 20481, 70001, 151936, 262144])
@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("kind", KINDS)
def test_every_rule(V, dtype, kind):
    n = 2 * len(RULES)
    z = logits(n, V, kind, dtype, V)
    role = torch.arange(n, dtype=torch.int32) % len(RULES)
    u = torch.rand(n, generator=torch.Generator().manual_seed(V)).cuda()
    check(z, RULES, u, role, draw(z, RULES, u, role.cuda()))


@pytest.mark.parametrize("V,dtype", [(4096, F32), (151936, F32), (152064, B16)])
def test_uniform_numbers_at_the_ends_and_next_to_running_masses(V, dtype):
    z = logits(1, V, "peaked", dtype, 3)[0]
    e = np.exp(z.double().cpu().numpy() - z.double().max().item())
    run = np.cumsum(e) / e.sum()
    ends = [0.0, 2.0 ** -149, 2.0 ** -24, 1 - 2.0 ** -24, 0.5]
    at = np.argsort(-e)[:10]
    near = np.concatenate([run[at], run[at] - e[at] / e.sum()]).astype(np.float32)
    us = [np.float32(v) for v in ends] + list(near) + list(np.nextafter(near, np.float32(0))) + list(np.nextafter(near, np.float32(1)))
    us = np.array([v for v in us if 0 <= v < 1], np.float32)
    n = len(us)
    zz = z.unsqueeze(0).repeat(n, 1)
    u = torch.from_numpy(us).cuda()
    for rules in ([OFF], [(1.0, 12, 1.0, 0.0)], [(1.0, 0, 0.9, 0.0)]):
        check(zz, rules, u, None, draw(zz, rules, u))


def test_shares_next_to_running_masses():
    """top_p exactly at, just below and just above the mass of the first entries."""
    z = logits(1, 5000, "normal", F32, 9)[0] * 3
    e = np.sort(np.exp(z.double().cpu().numpy() - z.double().max().item()))[::-1]
    run = (np.cumsum(e) / e.sum())[:30].astype(np.float32)
    rules = [(1.0, 0, float(v), 0.0) for p in run for v in (p, np.nextafter(p, np.float32(0)))][:60]
    n = len(rules)
    zz, u, role = z.unsqueeze(0).repeat(n, 1), torch.rand(n).cuda(), torch.arange(n, dtype=torch.int32)
    check(zz, rules, u, role, draw(zz, rules, u, role.cuda()))


def test_uniform_distribution_takes_64_bits():
    V = 152064
    z = torch.zeros(24, V, device="cuda")
    z += 1e-6 * torch.randn(24, V, device="cuda")
    u = torch.rand(24).cuda()
    check(z, [OFF], u, None, draw(z, [OFF], u))
    check(z, [(1.0, 0, 0.5, 0.0)], u, None, draw(z, [(1.0, 0, 0.5, 0.0)], u))


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("V", [300, 4096, 151936])
@pytest.mark.parametrize("rule", [OFF, (0.0, 0, 1.0, 0.0), (1.0, 40, 1.0, 0.0), (1.0, 0, 0.9999999, 0.0), (1.0, 0, 1.0, 1e-9), (0.5, 200, 0.99, 0.0),
                                  (1.0, 100000, 0.999999, 0.0)])
def test_sure_tokens_keep_their_digits(V, dtype, rule):
    """log p of an entry with nearly all of the mass is what the others have, relative to itself: each weight is off by 2^-22 and by two
    roundings of an exponent of at most 40 octaves (2 * 40 * ln2 * 2^-24 = 3.3e-6), both sides of the quotient: 7.2e-6 and the output's
    rounding.  The others' mass is a difference of fp64 sums of about 1 (5 + 3 + 4 lanes, warps and blocks, and the share that is taken
    off: 13 additions of at most 2^-53): 2^-49 absolute.  One entry alone has log p = 0."""
    n = 12
    z = logits(n, V, "normal", dtype, V).float()
    z[torch.arange(n), torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(V))] = torch.linspace(12, 27, n, device="cuda") + np.log(V) / 2
    z = z.to(dtype)
    u = torch.full((n,), 0.5, device="cuda")
    got = draw(z, [rule], u)
    check(z, [rule], u, None, got)
    zs = z.double().cpu().numpy()
    for i in range(n):
        t, lp, lk, k = orc.sample_row(zs[i], *rule, 0.5)
        T = float(np.float32(rule[0])) or 1.0
        x = (zs[i] - zs[i].max()) / T
        order = np.argsort(-zs[i], kind="stable")
        if t != order[0]:
            continue
        rest = np.exp(np.delete(x, t)).sum()
        rest_kept = np.exp(x[order[1:k]]).sum()
        for v, w in ((got[1][i], -np.log1p(rest)), (got[2][i], -np.log1p(rest_kept))):
            assert abs(v - w) <= 7.4e-6 * abs(w) + 2.0 ** -49, (i, v, w)


def test_rows_without_a_distribution_and_masked_rows():
    z = logits(8, 3001, "peaked", F32, 1)
    z[1, 2000] = float("nan")
    z[2, 5] = float("inf")
    z[3] = -float("inf")
    z[4] = float("nan")
    z[6, :3000] = -float("inf")
    u = torch.rand(8).cuda()
    mask = torch.ones(8, dtype=torch.uint8).cuda()
    mask[4] = 0
    ctx = ub.Context(0, 256)
    for rule in RULES:
        got = draw(z, [rule], u, None, mask, ctx)
        assert [got[k][4] for k in range(4)] == [-1, 0, 0, 0]
        ok = torch.arange(8) != 4
        check(z[ok.cuda()], [rule], u[ok.cuda()], None, [g[ok.numpy()] for g in got])
        assert got[0][6] == 3000
    ctx.check_status()


def test_bad_roles_and_uniform_numbers_are_flagged():
    z = logits(6, 100, "normal", F32, 1)
    u = torch.tensor([0.5, 1.0, -0.1, float("nan"), 0.2, 0.3]).cuda()
    role = torch.tensor([0, 0, 0, 0, 5, -1], dtype=torch.int32).cuda()
    ctx = ub.Context(0, 256)
    got = draw(z, [OFF], u, role, None, ctx)
    with pytest.raises(ub.UnityError) as e:
        ctx.check_status()
    assert e.value.code == -7
    assert got[0][0] >= 0 and np.all(got[0][1:] == -1) and not got[1][1:].any() and not got[3][1:].any()


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("V,ld,off", [(1000, 1003, 0), (1000, 1001, 1), (4096, 4104, 8), (20483, 20483, 3), (151936, 152064, 0), (4096, 4097, 2)])
def test_pitches_and_alignments(dtype, V, ld, off):
    n = 6
    flat = torch.full((n * ld + off + 8,), float("nan"), dtype=dtype, device="cuda")
    z = flat[off:off + n * ld].view(n, ld)[:, :V]
    z.copy_(logits(n, V, "peaked", dtype, ld))
    u = torch.rand(n).cuda()
    for rule in (OFF, (0.9, 40, 0.9, 0.0)):
        check(z, [rule], u, None, draw(z, [rule], u))


def test_optional_outputs_no_rows_and_two_calls_in_a_row():
    z = logits(5, 5000, "normal", B16, 2)
    u = torch.rand(5).cuda()
    ctx = ub.Context(0, 256)
    want = draw(z, [OFF], u, None, None, ctx)
    token = torch.zeros(5, dtype=torch.int32, device="cuda")
    ctx.sample(z, [OFF], u, token)
    assert np.array_equal(token.cpu().numpy(), want[0])
    ctx.sample(z[:0], [OFF], u[:0], token[:0])
    again = draw(z, [OFF], u, None, None, ctx)
    assert all(np.array_equal(a, b) for a, b in zip(want, again))


def test_more_rows_than_the_machine_holds():
    n, V = 700, 33001
    z = logits(n, V, "peaked", F32, 12)
    rules = RULES[:6]
    role = torch.randint(0, 6, (n,), dtype=torch.int32)
    u = torch.rand(n).cuda()
    check(z, rules, u, role, draw(z, rules, u, role.cuda()))


def test_offsets_beyond_32_bits():
    V, ld = 4096, 2 ** 28 + 16
    flat = torch.zeros(8 * ld + V, dtype=B16, device="cuda")
    z = torch.as_strided(flat, (9, V), (ld, 1))
    z.copy_(logits(9, V, "peaked", B16, 4))
    u = torch.rand(9).cuda()
    check(z, [OFF], u, None, draw(z, [OFF], u))


def test_refusals():
    ctx = ub.Context(0, 256)
    z, u, t = torch.zeros(2, 64, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def code(rules, z=z):
        with pytest.raises(ub.UnityError) as e:
            ctx.sample(z, rules, u, t)
        return e.value.code

    for rule in ((-1.0, 0, 1.0, 0.0), (1e-7, 0, 1.0, 0.0), (float("inf"), 0, 1.0, 0.0), (float("nan"), 0, 1.0, 0.0), (1.0, 0, 0.0, 0.0),
                 (1.0, 0, 1.1, 0.0), (1.0, 0, float("nan"), 0.0), (1.0, 0, 1.0, -0.1), (1.0, 0, 1.0, 1.5), (1.0, 0, 1.0, float("nan"))):
        assert code([rule]) == -1
    assert code([]) == -2 and code([OFF] * 65) == -2
    assert code([OFF], torch.zeros(2, 262145, device="cuda")) == -2
    assert code([OFF], z[:1].expand(2, 64)) == -2
    for bad in (lambda: ctx.sample(z.half(), [OFF], u, t), lambda: ctx.sample(z.t(), [OFF], u, t), lambda: ctx.sample(z, [OFF], u[:1], t),
                lambda: ctx.sample(z, [OFF], u, t.long()), lambda: ctx.sample(z, [OFF], u.cpu(), t)):
        with pytest.raises((TypeError, ValueError)):
            bad()


def test_captured_and_replayed():
    st = torch.cuda.Stream()
    ctx = ub.Context(0, 256, st)
    z, u = logits(4, 30000, "peaked", F32, 5), torch.rand(4).cuda()
    o = [torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"),
         torch.zeros(4, dtype=torch.int32, device="cuda")]
    rules = [(0.9, 40, 0.9, 0.0)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.sample(z, rules, u, o[0], None, None, *o[1:])
    for seed in (6, 7):
        z.copy_(logits(4, 30000, "peaked", F32, seed))
        u.uniform_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(z, rules, u, None, [t.cpu().numpy() for t in o])


# Calls whose rows the machine does not hold at once take one pass over all rows first and search only what a short list leaves open.
@pytest.mark.parametrize("V,n,kinds", [(513, 640, KINDS), (20481, 300, KINDS), (151936, 42, ["peaked", "wide", "ties", "masked"])])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_every_rule_in_calls_of_many_rows(V, n, kinds, dtype):
    for kind in kinds:
        z = logits(n, V, kind, dtype, V)
        role = torch.arange(n, dtype=torch.int32) % len(RULES)
        u = torch.rand(n, generator=torch.Generator().manual_seed(V)).cuda()
        check(z, RULES, u, role, draw(z, RULES, u, role.cuda()))


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("left", [1, 30, 1000, 1100, 10000])
def test_many_rows_with_most_of_the_vocabulary_masked(left, dtype):
    n, V = 300, 20481
    z = logits(n, V, "normal", dtype, left)
    z[:, left:] = -float("inf")
    z[::2] = z[::2].flip(1)
    rules = [(1.0, 40, 1.0, 0.0), (0.7, 0, 1.0, 0.1), (1.0, 0, 0.7, 0.0), (1.0, 30, 0.9, 0.01)]
    role = torch.arange(n, dtype=torch.int32) % 4
    u = torch.rand(n).cuda()
    check(z, rules, u, role, draw(z, rules, u, role.cuda()))


def test_list_sizes_of_many_rows():
    n, V = 300, 20481
    z = logits(n, V, "normal", F32, 77) * 2
    rules = [(1.0, k, p, m) for k in (1, 2, 255, 256, 383, 384, 385, 1000) for p, m in ((1.0, 0.0), (0.8, 0.0), (1.0, 0.002))] + [(1.0, 0, 1.0, 1e-5)]
    role = torch.arange(n, dtype=torch.int32) % len(rules)
    u = torch.rand(n).cuda()
    check(z, rules, u, role, draw(z, rules, u, role.cuda()))


def test_many_rows_without_a_distribution_at_odd_pitches():
    n, V = 640, 3001
    for ld, off, dtype in ((3001, 0, F32), (3007, 3, B16)):
        flat = torch.full((n * ld + off,), float("nan"), dtype=dtype, device="cuda")
        z = torch.as_strided(flat, (n, V), (ld, 1), off)
        z.copy_(logits(n, V, "peaked", dtype, ld))
        for i, v in ((1, float("nan")), (2, float("inf")), (3, -float("inf"))):
            z[i::9, i * 700] = v
        z[5::9] = -float("inf")
        z[6::9] = float("nan")
        mask = torch.ones(n, dtype=torch.uint8)
        mask[7::9] = 0
        rules = [(1.0, 20, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (1.0, 700, 1.0, 0.0), OFF]
        role = torch.arange(n, dtype=torch.int32) % 5
        u = torch.rand(n).cuda()
        ctx = ub.Context(0, 256)
        got = draw(z, rules, u, role.cuda(), mask.cuda(), ctx)
        on = mask.bool()
        check(z[on.cuda()], rules, u[on.cuda()], role[on], [g[on.numpy()] for g in got])
        assert all((g[7::9] == w).all() for g, w in zip(got, (-1, 0, 0, 0)))
        ctx.check_status()


@pytest.mark.parametrize("rule", [(1.0, 40, 1.0, 0.0), (1.0, 0, 0.99, 0.0), (1.0, 0, 1.0, 1e-9), (0.5, 200, 0.99, 0.0)])
def test_sure_tokens_of_many_rows_keep_their_digits(rule):
    """As in calls of few rows: 7.4e-6 relative and 2^-49; here the others' mass is added up by itself."""
    n, V = 300, 20481
    z = logits(n, V, "normal", F32, 5)
    z[torch.arange(n), torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(V))] = torch.linspace(12, 27, n, device="cuda") + np.log(V) / 2
    u = torch.full((n,), 0.5, device="cuda")
    got = draw(z, [rule], u)
    check(z, [rule], u, None, got)
    zs = z.double().cpu().numpy()
    for i in range(n):
        t, lp, lk, k = orc.sample_row(zs[i], *rule, 0.5)
        x = (zs[i] - zs[i].max()) / rule[0]
        order = np.argsort(-zs[i], kind="stable")
        if t != order[0]:
            continue
        for v, rest in ((got[1][i], np.exp(np.delete(x, t)).sum()), (got[2][i], np.exp(x[order[1:k]]).sum())):
            assert abs(v + np.log1p(rest)) <= 7.4e-6 * np.log1p(rest) + 2.0 ** -49, (i, v, rest)


def test_many_rows_captured_and_replayed_give_the_same_twice():
    n, V = 640, 4097
    st = torch.cuda.Stream()
    ctx = ub.Context(0, 256, st)
    z, u = logits(n, V, "peaked", B16, 5), torch.rand(n).cuda()
    o = [torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"),
         torch.zeros(n, dtype=torch.int32, device="cuda")]
    role = (torch.arange(n, dtype=torch.int32) % 6)
    dev = role.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.sample(z, RULES[:6], u, o[0], dev, None, *o[1:])
        ctx.sample(z, RULES[:6], u, o[0], dev, None, *o[1:])
    for seed in (6, 7):
        z.copy_(logits(n, V, "peaked", B16, seed))
        u.uniform_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in o]
        check(z, RULES[:6], u, role, got)
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a, t.cpu().numpy()) for a, t in zip(got, o))


@pytest.mark.parametrize("V", [1, 2, 7, 64])
def test_many_rows_of_short_vocabularies(V):
    n = 40 * len(RULES) + 41
    z = torch.cat([logits(n // 3, V, kind, F32, V) for kind in ("normal", "ties", "masked")])
    role = torch.arange(len(z), dtype=torch.int32) % len(RULES)
    u = torch.rand(len(z)).cuda()
    check(z, RULES, u, role, draw(z, RULES, u, role.cuda()))
