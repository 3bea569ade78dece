"""Drawing tokens on the GPU against the fp64 oracle: every filter, ties, borders, absent elements, odd sizes, streams
and graphs.  Tokens and counts have to be equal."""
import itertools
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF, NAN = float("inf"), float("nan")


def check(scores, uniforms, probabilities=False, **filters):
    """scores [rows, V] on the GPU; filters: lists of a value for each row, or None."""
    rows = scores.shape[0]
    u = torch.tensor(uniforms, dtype=torch.float32).cuda()
    given = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32).cuda()
             for n, v in filters.items() if v is not None}
    token, prob, kept = (t.cpu().numpy() for t in knn.sample(scores, u, probabilities=probabilities, **given))
    x, u = scores.double().cpu().numpy(), u.double().cpu().numpy()
    given = {n: t.double().cpu().numpy() for n, t in given.items()}
    for r in range(rows):
        want = lm.sample(x[r], u[r], probabilities, **{n: v[r] for n, v in given.items()})
        where = (r, {n: v[r] for n, v in given.items()}, want, token[r], prob[r], kept[r])
        assert (token[r], kept[r]) == (want[0], want[2]), where
        # half a step of fp32, and the weights' sum in units of 2^-46 of the largest at worst (V <= 2^17)
        assert abs(float(prob[r]) - want[1]) <= 2.0 ** -24 * want[1] + 1e-9 * want[1] + 2.0 ** -149, where
    return token, prob, kept


def rows_of(n, V, dtype, form, seed, sigma=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g) * sigma
    if form == "probs":
        x = torch.softmax(x, 1)
    return x.to(TYPES[dtype]).cuda(), torch.rand(n, generator=g).tolist()


@pytest.mark.parametrize("form,dtype", [("logits", "f32"), ("logits", "bf16"), ("logits", "f16"), ("probs", "f32"),
                                        ("probs", "bf16")])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 1000, 1023, 4097, 32000, 50257])
def test_every_filter(form, dtype, V):
    n = 12
    x, u = rows_of(n, V, dtype, form, V)
    t = [0.7, 1.0, 1.3, 0.0, 2.0, 0.3, 1.0, 1.0, 5.0, 0.9, 1.0, 1.1]
    k = [0, 1, 5, 50, V, V + 1, -3, max(1, V - 1), V // 2, 7, 2, 1000]
    p = [0.9, 1.0, 0.5, 0.1, 0.999, 2.0, 0.0, 0.95, 0.99, 0.7, -1.0, 0.3]
    m = [0.0, 0.05, 0.2, 1.0, 0.001, 2.0, -1.0, 0.5, 0.01, 0.0, 0.1, 1e-6]
    probs = form == "probs"
    check(x, u, probs)
    check(x, u, probs, temperature=t)
    check(x, u, probs, top_k=k)
    check(x, u, probs, top_p=p)
    check(x, u, probs, min_p=m)
    check(x, u, probs, temperature=t, top_k=k, top_p=p, min_p=m)
    check(x, u, probs, temperature=t, top_p=p)
    check(x, u, probs, top_k=k, min_p=m)


def test_large_vocabulary_and_many_rows():
    x, u = rows_of(40, 131072, "f32", "logits", 1)
    check(x, u, temperature=[0.5 + 0.02 * i for i in range(40)], top_p=[0.5 + 0.0125 * i for i in range(40)])
    check(x, u, temperature=[1.0] * 40)
    check(x, u, top_k=[1 + 200 * i for i in range(40)], top_p=[0.9] * 40)
    x, u = rows_of(300, 777, "f16", "logits", 2)
    check(x, u, top_p=[0.9] * 300)


def test_ties_go_to_the_lower_token():
    V = 3000
    g = torch.Generator().manual_seed(3)
    x = torch.randint(-2, 3, (16, V), generator=g).float().cuda()  # five values: hundreds of ties at every cut
    u = torch.rand(16, generator=g).tolist()
    check(x, u, top_k=[1, 2, 3, 100, 599, 600, 601, 1200, 2999, 3000, 5, 6, 7, 8, 9, 10])
    check(x, u, top_p=[0.1 + 0.05 * i for i in range(16)])
    check(x, u, top_k=[40 * i + 1 for i in range(16)], top_p=[0.8] * 16)
    check(x, u, temperature=[0.0] * 16)
    same = torch.full((8, V), 0.25, device="cuda")
    for form in (False, True):
        check(same, [0.0, 0.1, 0.25, 0.5, 0.75, 0.9, 0.99, 0.999999], form, top_p=[0.5, 0.25, 0.9, 0.1, 1.0, 0.001, 0.7, 0.3])
        check(same, [0.0, 0.1, 0.25, 0.5, 0.75, 0.9, 0.99, 0.999999], form, top_k=[1, 2, 3, 4, 0, 2999, 1500, 64])


def test_uniforms_at_their_ends():
    x, _ = rows_of(6, 500, "f32", "logits", 4)
    u = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, NAN]
    check(x, u)
    check(x, u, top_p=[0.9] * 6)
    # the first and the last token carry all the weight there is
    y = torch.full((6, 500), -INF, device="cuda")
    y[:, 3], y[:, 496] = 0.0, 0.0
    token, _, kept = check(y, u)
    assert token.tolist() == [3, 496, 496, 496, 3, 3] and (kept == 2).all()


def test_absent_elements_and_empty_rows():
    V = 400
    x, u = rows_of(8, V, "f32", "logits", 5)
    x[0, :] = -INF
    x[1, :] = NAN
    x[2, ::2] = NAN
    x[3, 1:] = -INF
    x[4, 100:] = torch.finfo(torch.float32).min
    x[5, :] = torch.finfo(torch.float32).min
    x[6, 7] = INF
    x[6, 9] = INF
    x[7, :-1] = NAN
    for filters in ({}, dict(top_k=[3] * 8), dict(top_p=[0.5] * 8), dict(min_p=[0.1] * 8), dict(temperature=[0.0] * 8),
                    dict(temperature=[1e-30] * 8, top_p=[0.9] * 8), dict(temperature=[INF] * 8), dict(top_k=[150] * 8)):
        token, prob, kept = check(x, u, **filters)
        assert token[0] == token[1] == -1 and prob[0] == 0 and kept[0] == 0
    p = torch.softmax(x.nan_to_num(0.0, 0.0, -1e9), 1)
    p[0] = 0.0
    p[1] = -1.0
    p[2, ::3] = NAN
    p[3] = 0.0
    p[3, 17] = 1e-40
    p[4, 5] = INF
    for filters in ({}, dict(top_k=[3] * 8), dict(top_p=[0.5] * 8), dict(min_p=[0.1] * 8), dict(temperature=[0.5] * 8),
                    dict(temperature=[0.0] * 8)):
        check(p, u, True, **filters)


def test_half_types_lowest_values():
    for dtype in ("bf16", "f16"):
        t = TYPES[dtype]
        x = torch.full((4, 100), torch.finfo(t).min, dtype=t, device="cuda")
        x[1, 50:] = 0
        x[2, 99] = torch.finfo(t).max
        x[3, :] = -INF
        check(x, [0.3, 0.6, 0.9, 0.5])
        check(x, [0.3, 0.6, 0.9, 0.5], top_p=[0.5] * 4)


def test_signed_zeros_are_equal():
    x = torch.zeros(2, 64, device="cuda")
    x[0, ::2] = -0.0
    token, _, kept = check(x, [0.5, 0.5], top_k=[10, 10])
    assert token[0] == token[1]


def test_peaked_and_wide_rows():
    V = 32000
    x = torch.zeros(6, V, device="cuda")
    x[0, 12345] = 100.0
    x[1] = torch.linspace(-1e30, 1e30, V)
    x[2] = torch.linspace(0, 1e-3, V)
    x[3] = torch.linspace(-80, 0, V)
    x[4] = -torch.arange(V).float()
    x[5] = torch.arange(V).float() * 1e-30
    u = [0.5, 0.1, 0.7, 0.3, 0.9, 0.2]
    for filters in ({}, dict(top_p=[0.9] * 6), dict(top_k=[1000] * 6), dict(min_p=[0.01] * 6),
                    dict(temperature=[2.0] * 6, top_p=[0.99] * 6)):
        check(x, u, **filters)


def test_frequencies_follow_the_weights():
    # 4,000 evenly spread uniforms draw each token as often as its share says, to within one draw
    g = torch.Generator().manual_seed(6)
    x = torch.randn(1, 50, generator=g).cuda().repeat(4000, 1)
    u = (torch.arange(4000) + 0.5) / 4000
    token, _, _ = knn.sample(x, u.cuda())
    share = torch.softmax(x[0].double(), 0).cpu() * 4000
    assert ((torch.bincount(token.cpu(), minlength=50) - share).abs() <= 1.0).all()


def test_strides_and_views():
    x, u = rows_of(5, 1001, "f32", "logits", 7)
    wide = torch.full((5, 1100), 50.0, device="cuda")
    wide[:, 37:1038] = x
    a = check(wide[:, 37:1038], u, top_p=[0.9] * 5)
    b = check(x, u, top_p=[0.9] * 5)
    assert all(np.array_equal(i, j) for i, j in zip(a, b))
    one = x[:1].expand(4, 1001)  # one row of logits, several draws
    check(one, u[:4], top_k=[20] * 4)
    h = x.bfloat16()
    for off in range(1, 4):
        check(h[:, off:], u, top_p=[0.8] * 5)


def test_streams_graphs_and_repeats():
    x, u = rows_of(32, 32000, "bf16", "logits", 8)
    u = torch.tensor(u).cuda()
    k = torch.full((32,), 40, dtype=torch.int32, device="cuda")
    p = torch.full((32,), 0.9, device="cuda")
    call = knn.Sampler(x, u, top_k=k, top_p=p)
    first = [t.clone() for t in call.run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = knn.Sampler(x, u, top_k=k, top_p=p)
    for _ in range(3):
        a, b = call.run(), other.run(stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(i, j) and torch.equal(i, l) for i, j, l in zip(first, a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    for i in range(4):
        x.normal_()
        u.uniform_()
        k.fill_(1 + 10 * i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (call.token, call.prob, call.kept)]
        for t in (call.token, call.prob, call.kept):
            t.zero_()
        assert all(torch.equal(i, j) for i, j in zip(got, call.run()))
        torch.cuda.synchronize()


def test_refusals():
    x, u = rows_of(3, 100, "f32", "logits", 9)
    u = torch.tensor(u).cuda()
    f = torch.ones(3, device="cuda")
    for bad in (dict(uniforms=u[:2]), dict(uniforms=u.double()), dict(uniforms=u.cpu()), dict(scores=x[0]),
                dict(scores=x.t()), dict(temperature=f[:2]), dict(top_k=f), dict(top_p=f.half()), dict(min_p=f.cpu()),
                dict(scores=x.double())):
        with pytest.raises((ValueError, TypeError)):
            knn.sample(**dict(dict(scores=x, uniforms=u), **bad))


def test_small_k_and_min_p_of_ordered_rows():
    V = 20000
    down = -torch.arange(V).float() * 0.001
    x = torch.stack([down, down.flip(0), (torch.arange(V) % 7).float(), torch.full((V,), -1e30), down, down]).cuda()
    x[3, ::97] = 0.5 + torch.arange(len(range(0, V, 97))).float().cuda() * 0.01  # few that are not masked
    x[4, 1:] = float("-inf")
    x[5, 300:] = float("nan")
    u = [0.0, 0.3, 0.5, 0.77, 0.9, 0.999]
    for k in (1, 2, 255, 256, 257, 1023):
        check(x, u, top_k=[k] * 6)
        check(x, u, temperature=[1e-3, 0.1, 1.0, 2.0, 50.0, 1e4], top_k=[k] * 6, top_p=[0.9, 0.5, 0.99, 0.8, 0.3, 0.7])
        check(x, u, top_k=[k] * 6, top_p=[0.9] * 6, min_p=[0.5, 0.1, 0.9, 0.97, 0.01, 1.0])
    check(x, u, min_p=[0.9, 0.5, 1.0, 0.97, 0.01, 0.999])
    check(x, u, temperature=[1e-3, 0.1, 1.0, 2.0, 50.0, 1e4], min_p=[0.9, 0.5, 1.0, 0.97, 0.01, 0.999])


def test_infinite_elements_under_every_filter():
    x = torch.randn(4, 5000, generator=torch.Generator().manual_seed(9)).cuda()
    x[0, 77] = x[1, 5] = x[1, 4999] = float("inf")
    x[2, :400] = float("inf")
    x[3, 10:] = float("-inf")
    u = [0.5, 0.6, 0.4, 0.9]
    for form in (False, True):
        for f in ({}, dict(top_k=[3] * 4), dict(top_p=[0.6] * 4), dict(min_p=[0.2] * 4),
                  dict(top_k=[300] * 4, top_p=[0.7] * 4, min_p=[0.1] * 4, temperature=[0.5] * 4)):
            check(x, u, form, **f)


def test_a_row_of_millions():
    V = (1 << 22) + 4321
    # Weights in units of 2^-39 of the largest, their sum above 1000 of it, and errors of either sign: 2^11 2^-40 / 1000
    # = 2e-12 is what to expect of the sum, far within check()'s 1e-9.
    x = torch.randn(2, V, generator=torch.Generator().manual_seed(11)).mul_(2).half().cuda()
    check(x, [0.3, 0.98], temperature=[0.9, 1.2])
    check(x, [0.3, 0.98], top_p=[0.7, 0.4], top_k=[0, 100000])
    check(x, [0.7, 0.1], min_p=[0.3, 0.001], top_k=[40, 0])


def test_min_p_above_one_keeps_the_first_alone():
    """No weight reaches it, those of elements equal to the largest neither."""
    x = torch.randn(8, 3000, generator=torch.Generator().manual_seed(12)).cuda()
    x[0, :3] = torch.tensor([9.0, 9.0, 8.0])
    x[1, 5::7] = 9.0                   # hundreds of equal ones
    x[2, 3:] = 9.0
    x[3, 40] = x[3, 2999] = INF
    x[4, 1:] = INF
    x[5, 700] = 9.0                    # alone
    x[6, 100:] = -INF
    x[6, 50] = x[6, 60] = 9.0
    x[7, 10] = x[7, 20] = 9.0          # min-p of 1 itself: the equal ones stay
    u = [0.9, 0.999, 0.5, 0.9, 0.99, 0.0, 0.99, 0.6]
    m = [2.0, 1.0 + 2.0 ** -23, 1e30, 2.0, INF, 3.0, 1.5, 1.0]
    for probs in (False, True):
        _, prob, kept = check(x, u, probs, min_p=m)
        assert (kept[:7] == 1).all() and kept[7] == 2 and (prob[:7] == 1.0).all()
        check(x, u, probs, min_p=m, top_p=[0.9] * 8)
        check(x, u, probs, min_p=m, top_k=[100] * 8)
        check(x, u, probs, min_p=m, top_k=[1000] * 8, top_p=[0.7] * 8, temperature=[0.5] * 8)
    check(torch.tensor([[1.0, 1.0, 0.0]], device="cuda"), [0.9], min_p=[2.0])


@pytest.mark.parametrize("first,second,t,u", [
    (2.0335712280772356e-10, 2.0255402910507314e-10, 0.013835875317454338, 0.42898452281951904),
    (2.6456388191320457e-09, 2.6005610997970052e-09, 0.020649559795856476, 0.3031722903251648)])
def test_small_probabilities_at_a_low_temperature(first, second, t, u):
    """The share w / (1 + w) of the second, w = (x / max)^(1 / T), lies 2^-45.3 or 2^-46.6 from the uniform.  w is right to
    2^-51 / T of itself, which moves the share by w / (1 + w)^2 < 1 / 4 of that: 2^-46.8 and 2^-47.6.  A logarithm in one
    number, of -32 and -28, is off by up to 2^-48 in either, 8 times as much."""
    with localcontext() as c:
        c.prec = 60
        w = ((Decimal(second) / Decimal(first)).ln() / Decimal(t)).exp()
        share = w / (1 + w)
        assert 2.0 ** -47 < abs(share - Decimal(u)) < 2.0 ** -45
        want = 0 if share > Decimal(u) else 1
    x = torch.tensor([[second, first]], device="cuda")
    token, _, kept = knn.sample(x, torch.tensor([u], device="cuda"), probabilities=True,
                                temperature=torch.tensor([t], device="cuda"))
    assert (int(token[0]), int(kept[0])) == (want, 2)


def test_small_probabilities_with_every_filter():
    x, u = rows_of(8, 4097, "f32", "probs", 13)
    x *= 1e-6 / x.max(1, keepdim=True).values
    t = [0.01, 0.02, 0.05, 0.1, 0.3, 1.0, 1.5, 0.015]
    check(x, u, True, temperature=t)
    check(x, u, True, temperature=t, top_p=[0.9, 0.5, 0.99, 0.7, 0.9, 0.3, 0.9, 0.999])
    check(x, u, True, temperature=t, top_k=[3, 50, 300, 7, 1000, 2, 64, 9], min_p=[0.0, 1e-4, 0.01, 0.5, 0.001, 0.2, 0.05, 1e-6])
    check(x * 1e-30, u, True, temperature=t, top_p=[0.9] * 8)  # into the numbers below fp32's normal range
