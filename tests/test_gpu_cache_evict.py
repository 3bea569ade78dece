"""Eviction on the GPU against the oracle, every place of the caches and the ledger equal: budgets, lengths from zero on,
ties, protected tokens, masses that are no numbers, pages, and what has to stay as it was."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def batch(lens, Hk=2, d=64, page=16, dtype="bf16", seed=0, width=None, masses="spread"):
    g = torch.Generator().manual_seed(seed)
    need = [max(1, -(-n // page)) for n in lens]
    width = width or max(need)
    n_pages = sum(need) + 2
    order = torch.randperm(n_pages, generator=g)
    pages = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        pages[s, :n] = order[at:at + n].int()
        at += n
    shape = (n_pages, Hk, page)
    # every place has elements of its own: whole numbers that the type holds
    k = torch.randint(0, 256, (*shape, d), generator=g).to(TYPES[dtype])
    mass = torch.randn(shape, generator=g).exp() if masses == "spread" else torch.randint(0, 3, shape, generator=g).float()
    return {"k_cache": k.cuda(), "v_cache": (255 - k).flip(3).cuda(), "mass": mass.cuda(), "pages": pages.cuda(),
            "key_positions": torch.randint(0, 10 * max(1, max(lens)), shape, generator=g, dtype=torch.int32).cuda(),
            "cache_lens": torch.tensor(lens, dtype=torch.int32).cuda()}


def ints(t):
    return None if t is None else t.cpu().numpy()


def bits(t):
    return None if t is None else t.cpu().view({2: torch.int16, 4: torch.int32}[t.element_size()]).numpy()


def check(x, budgets, next_positions=None, sinks=0, recent=0, max_keys=None, out=False, positions=True):
    """Runs the eviction and compares all that it writes with the oracle, bit by bit."""
    x = dict(x)
    if not positions:
        x["key_positions"] = None
    budgets = torch.tensor(budgets, dtype=torch.int32).cuda()
    nxt = None if next_positions is None else torch.tensor(next_positions, dtype=torch.int32).cuda()
    outs = {}
    if out:
        outs["mass_out"] = torch.full_like(x["mass"], -3.0)
        if positions:
            outs["positions_out"] = torch.full_like(x["key_positions"], -4)
    limit = max_keys if max_keys is not None else max(1, min(int(x["cache_lens"].max()), x["pages"].numel()
                                                             // len(x["pages"]) * x["k_cache"].shape[2]))
    # the caches as bit patterns, the masses as the numbers that order like them
    want = lm.evict(bits(x["k_cache"]), bits(x["v_cache"]), x["mass"].cpu().numpy(), ints(x["key_positions"]),
                    ints(x["pages"]), ints(x["cache_lens"]), ints(budgets), ints(nxt), sinks, recent, limit,
                    *(ints(outs.get(n)) for n in ("mass_out", "positions_out")))
    before = {n: t.clone() for n, t in x.items() if t is not None}
    got = knn.cache_evict(x["k_cache"], x["v_cache"], x["mass"], x["pages"], x["cache_lens"], budgets, max_keys,
                          key_positions=x["key_positions"], next_positions=nxt, sinks=sinks, recent=recent, **outs)
    torch.cuda.synchronize()
    assert np.array_equal(ints(got), want[4])
    assert np.array_equal(bits(x["k_cache"]), want[0]) and np.array_equal(bits(x["v_cache"]), want[1])
    assert np.array_equal(bits(outs.get("mass_out", x["mass"])), want[2].view(np.int32))
    if positions:
        assert np.array_equal(ints(outs.get("positions_out", x["key_positions"])), want[3])
    for n in ("pages", "cache_lens") + (("mass", "key_positions") if out and positions else ()):
        assert np.array_equal(bits(before[n]), bits(x[n]))
    return got


@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("masses", ["spread", "even"])
def test_lengths_and_budgets(out, positions, masses):
    lens = [0, 1, 2, 15, 16, 17, 64, 65, 200, 333]
    budgets = [0, 0, 1, 7, 15, 17, 1, 64, 100, 0]
    x = batch(lens, masses=masses, seed=len(masses))
    check(x, budgets, next_positions=[3000] * 10, sinks=30, recent=300, out=out, positions=positions)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("Hk,d", [(1, 64), (5, 128), (2, 256), (3, 80), (2, 33), (1, 1), (2, 1024)])
def test_heads_pages_and_sizes(dtype, page, Hk, d):
    check(batch([100, 300, 5], Hk, d, page, dtype, seed=d), [50, 290, 4], recent=3, positions=False)


@pytest.mark.parametrize("n,budget", [(1025, 1024), (1024, 1023), (4105, 4096), (5000, 100), (20000, 19999), (20000, 7000),
                                      (40000, 3), (70001, 65536), (140000, 30000)])
def test_long_lengths(n, budget):
    for masses in ("spread", "even"):
        check(batch([n, n // 3 + 1], 2, 64, 64, seed=n, masses=masses), [budget, budget], [10 * n, 10 * n], sinks=5,
              recent=n // 2, out=masses == "even")


def test_more_protected_tokens_than_the_budget():
    x = batch([300, 300, 300], seed=1)
    for budgets in ([100, 1, 299], [0, 200, 150]):
        check({n: t.clone() for n, t in x.items()}, budgets, sinks=120, recent=110, positions=False)
        check({n: t.clone() for n, t in x.items()}, budgets, [3000] * 3, sinks=1000, recent=1500)


def test_protected_positions_at_the_ends_of_32_bits():
    x = batch([100, 60, 50], seed=2)
    top = 2 ** 31 - 1
    x["key_positions"][::2] = top
    x["key_positions"][1::3] = -(2 ** 31)
    for sinks, recent, nxt in ((top, 5, top), (3, top, -(2 ** 31)), (0, 0, top), (0, 1, top), (0, top, top)):
        check({n: t.clone() for n, t in x.items()}, [50, 10, 49], [nxt] * 3, sinks, recent)


def test_masses_that_are_no_numbers():
    x = batch([200, 200, 90], seed=3)
    m = x["mass"].flatten()
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0, -1.0, 1e-45, -1e-45, 3.4e38)):
        m[i::23] = v
    for budgets in ([100, 30, 89], [180, 3, 1], [1, 199, 45]):
        check({n: t.clone() for n, t in x.items()}, budgets)
        check({n: t.clone() for n, t in x.items()}, budgets, sinks=40, recent=30, positions=False)
    for v in (float("nan"), 0.0, float("-inf")):
        x["mass"][:] = v
        check({n: t.clone() for n, t in x.items()}, [100, 30, 89], sinks=4, recent=10, positions=False)
    x["mass"][:] = torch.where(torch.rand_like(x["mass"]) < 0.5, 0.0, -0.0)  # equal, whatever their sign
    check(x, [100, 30, 89])


def test_sequences_that_are_left_as_they_are():
    x = batch([100, 100, 100, 100, 100], width=8, seed=4)
    x["pages"][1, 3] = -1
    x["pages"][2, 6] = x["k_cache"].shape[0]
    x["cache_lens"][3] = 8 * 16 + 1  # longer than its table
    x["cache_lens"][4] = -5
    for out in (False, True):
        check({n: t.clone() for n, t in x.items()}, [100, 50, 50, 50, 50], out=out, max_keys=128)
        check({n: t.clone() for n, t in x.items()}, [-1, -(2 ** 31), 99, 4, 0], out=out, max_keys=128)
    x = batch([100, 90, 20], seed=5)
    check(x, [10, 20, 10], max_keys=95, out=True)  # longer than the hint


def test_far_pages_of_a_large_cache():
    """Offsets past 2^32 bytes of keys, and past 2^31 elements."""
    x = batch([300, 700], 2, 128, 256, seed=6)
    n = 40000
    move = n - x["k_cache"].shape[0]
    big = {name: torch.zeros((n, *x[name].shape[1:]), dtype=x[name].dtype, device="cuda")
           for name in ("k_cache", "v_cache", "mass", "key_positions")}
    for name, t in big.items():
        t[move:] = x[name]
    pages = torch.where(x["pages"] >= 0, x["pages"] + move, x["pages"])
    knn.cache_evict(big["k_cache"], big["v_cache"], big["mass"], pages, x["cache_lens"],
                    torch.tensor([100, 650], dtype=torch.int32).cuda(), key_positions=big["key_positions"])
    check(x, [100, 650])
    for name, t in big.items():
        assert torch.equal(t[move:], x[name]) and float(t[:move].abs().max()) == 0


def test_step_after_step_in_a_graph():
    """One token more each step, and one evicted; the graph is replayed on the lengths that it wrote."""
    x = batch([80, 80], Hk=2, width=8, seed=7)  # pages for more than the 64 tokens that are there
    x["cache_lens"][:] = 64
    budgets = torch.tensor([64, 40], dtype=torch.int32).cuda()
    nxt = torch.tensor([640, 640], dtype=torch.int32).cuda()
    call = knn.CacheEvict(x["k_cache"], x["v_cache"], x["mass"], x["pages"], x["cache_lens"], budgets, 80,
                          key_positions=x["key_positions"], next_positions=nxt, sinks=3, recent=10)

    def step():
        x["cache_lens"].add_(1)
        nxt.add_(1)
        call.run()
        x["cache_lens"].copy_(call.new_lens)

    kept = {n: t.clone() for n, t in dict(x, nxt=nxt).items()}

    def back():
        for n, t in kept.items():
            (nxt if n == "nxt" else x[n]).copy_(t)

    want = []
    for _ in range(4):
        step()
        want.append({n: x[n].clone() for n in ("k_cache", "v_cache", "mass", "key_positions", "cache_lens")})
    back()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    back()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for n, t in w.items():
            assert torch.equal(x[n], t), n
    assert x["cache_lens"].tolist() == [64, 40]


def test_argument_checks():
    x = batch([100])
    args = dict(k_cache=x["k_cache"], v_cache=x["v_cache"], mass=x["mass"], pages=x["pages"], cache_lens=x["cache_lens"],
                budgets=torch.tensor([50], dtype=torch.int32).cuda())
    for over in (dict(mass=x["mass"].half()), dict(mass=x["mass"][:1]), dict(key_positions=x["mass"]),
                 dict(positions_out=x["key_positions"]), dict(budgets=args["budgets"].long()),
                 dict(mass_out=x["mass"].cpu()), dict(v_cache=x["v_cache"][:, :1]), dict(next_positions=x["pages"])):
        with pytest.raises(ValueError):
            knn.cache_evict(**dict(args, **over))
    for over in (dict(sinks=-1), dict(v_cache=x["k_cache"]), dict(max_keys=1 << 20), dict(max_keys=0)):
        with pytest.raises(knn.KnnError):
            knn.cache_evict(**dict(args, **over))


LONG = [20000, 9000, 5, 0, 8193, 12345]


def shaped(x, kind, n):
    """Masses of all places in some shape that samples may misjudge."""
    g = torch.Generator().manual_seed(n)
    m = x["mass"].cpu()
    if kind == "equal":
        m[:] = 0.3
    elif kind == "zero but few":
        m[:] = torch.where(torch.rand(m.shape, generator=g) < 0.01, torch.rand(m.shape, generator=g), torch.zeros(1))
    elif kind == "by pages":  # neighbours are alike
        m[:] = torch.rand((m.shape[0], 1, 1), generator=g)
    elif kind == "two":
        m[:] = torch.where(torch.rand(m.shape, generator=g) < 0.3, 1.0, 1.0 + 2.0 ** -23)
    elif kind == "narrow":
        m[:] = 1.0 + torch.rand(m.shape, generator=g) * 2.0 ** -12
    elif kind == "wide":
        m[:] = torch.exp(torch.randn(m.shape, generator=g) * 25)
    elif kind == "signed":
        m[:] = torch.randn(m.shape, generator=g) * 10.0 ** torch.randint(-30, 30, m.shape, generator=g)
    elif kind == "one outlier":
        m[:] = 1e-3 * torch.rand(m.shape, generator=g)
        m[0] = 3e38
    elif kind == "nan":
        m[:] = torch.where(torch.rand(m.shape, generator=g) < 0.6, float("nan"), 1.0)
    x["mass"] = m.cuda()
    return x


@pytest.mark.parametrize("kind", ["equal", "zero but few", "by pages", "two", "narrow", "wide", "signed", "one outlier", "nan",
                                  "spread"])
def test_long_heads_of_any_shape(kind):
    for budgets in ([2500, 8000, 4, 0, 8192, 12344], [19999, 1, 0, 0, 1, 6000]):
        check(shaped(batch(LONG, 1, 64, 64, seed=8), kind, budgets[0]), budgets, [10 * n for n in LONG], sinks=4, recent=64,
              out=budgets[1] == 1)
    check(shaped(batch([8192, 100, 4097, 33], 2, 64, 16, seed=9), kind, 5), [4096, 50, 4096, 32], sinks=3, recent=9,
          positions=False)


def test_long_heads_with_more_protected_tokens_than_the_budget():
    x = batch(LONG, 1, 64, 64, seed=10)
    check({n: t.clone() for n, t in x.items()}, [2500, 800, 4, 0, 100, 12344], sinks=1500, recent=1200, positions=False)
    check(x, [2500, 800, 4, 0, 100, 12344], [10 * n for n in LONG], sinks=30000, recent=40000, out=True)


def test_long_heads_that_are_left_as_they_are():
    x = batch(LONG, 2, 64, 16, width=1300, seed=11)
    x["pages"][0, 700] = -1
    x["pages"][1, 3] = x["k_cache"].shape[0]
    x["cache_lens"][5] = 1300 * 16 + 1
    for out in (False, True):
        for budgets in ([100, 0, -1, 0, 100, 7], [0, 8999, 5, 3, 8193, 0]):
            check({n: t.clone() for n, t in x.items()}, budgets, out=out, max_keys=20800)


def test_ledgers_off_16_bytes_and_caches_off_them():
    for lens, budgets in (([100, 333, 16], [50, 332, 1]), ([9000, 50], [3000, 20])):
        x = batch(lens, 2, 64, 16, seed=12)
        for n in ("mass", "key_positions"):
            wide = torch.zeros(x[n].numel() + 1, dtype=x[n].dtype, device="cuda")
            wide[1:] = x[n].flatten()
            x[n] = wide[1:].view(x[n].shape)
        for n in ("k_cache", "v_cache"):
            wide = torch.zeros(x[n].numel() + 1, dtype=x[n].dtype, device="cuda")
            wide[1:] = x[n].flatten()
            x[n] = wide[1:].view(x[n].shape)
        check({n: t.clone() if t.data_ptr() % 16 == 0 else t for n, t in x.items()}, budgets, sinks=2, recent=5)


def test_one_ledger_in_place_and_one_apart():
    for lens, budget in (([200, 33], [150, 10]), ([9000, 33], [4000, 10])):
        x = batch(lens, 2, 64, 32, seed=16)
        want = lm.evict(bits(x["k_cache"]), bits(x["v_cache"]), x["mass"].cpu().numpy(), ints(x["key_positions"]),
                        ints(x["pages"]), lens, budget, recent=5)
        apart = {n: torch.zeros_like(x[n]) for n in ("mass", "key_positions")}
        for n, other in (("mass", "key_positions"), ("key_positions", "mass")):
            y = {m: t.clone() for m, t in x.items()}
            out = {"mass_out" if n == "mass" else "positions_out": apart[n]}
            knn.cache_evict(y["k_cache"], y["v_cache"], y["mass"], y["pages"], y["cache_lens"],
                            torch.tensor(budget, dtype=torch.int32).cuda(), key_positions=y["key_positions"], recent=5, **out)
            assert np.array_equal(bits(y["k_cache"]), want[0]) and torch.equal(y[n], x[n])
            assert np.array_equal(ints(y[other]), want[3] if other == "key_positions" else want[2])
            for s in range(2):
                for c in range(budget[s]):
                    page, slot = lm.place(ints(x["pages"]), s, c, len(x["mass"]), 32)
                    ledger = want[2] if n == "mass" else want[3]
                    assert np.array_equal(ints(apart[n])[page, :, slot], ledger[page, :, slot])


def test_many_short_heads():
    n = np.random.RandomState(5).randint(0, 60, 300).tolist()
    check(batch(n, 3, 64, 16, seed=13), [max(0, v - 3) for v in n], sinks=1, recent=2, positions=False)


def test_on_another_stream_and_two_calls_at_once():
    a, b = (batch([9000, 700], 2, 64, 64, seed=s) for s in (14, 15))
    want = []
    for x in (a, b):
        y = {n: t.clone() for n, t in x.items()}
        check(y, [4000, 600])
        want.append(y)
    budgets = torch.tensor([4000, 600], dtype=torch.int32).cuda()
    calls = [knn.CacheEvict(x["k_cache"], x["v_cache"], x["mass"], x["pages"], x["cache_lens"], budgets, 9000,
                            key_positions=x["key_positions"]) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for c, s in zip(calls, streams):
        c.run(s)
    torch.cuda.synchronize()
    for x, y in zip((a, b), want):
        for n in ("k_cache", "v_cache", "mass", "key_positions"):
            assert torch.equal(x[n], y[n])


def test_the_longest_head():
    """2^31 - 1 tokens, whose keys and values are their indices; weights of 24 bits in no order, many of them alike."""
    n, page, piece = 2 ** 31 - 1, 65536, 2 ** 28
    pages = torch.arange(2 ** 31 // page, dtype=torch.int32).cuda()[None]
    shape = (pages.numel(), 1, page)
    index = torch.empty(2 ** 31, dtype=torch.int32, device="cuda")
    mass = torch.empty(2 ** 31, dtype=torch.float32, device="cuda")
    for j in range(0, 2 ** 31, piece):
        index[j:j + piece] = torch.arange(j, j + piece, dtype=torch.int64, device="cuda").int()
        mass[j:j + piece] = ((torch.arange(j, j + piece, dtype=torch.int64, device="cuda") * 2654435761 >> 8) & 0xffffff).float()
    border = float(7 << 20)
    over = sum(int((mass[j:min(n, j + piece)] > border).sum()) for j in range(0, n, piece))
    even = sum(int((mass[j:min(n, j + piece)] == border).sum()) for j in range(0, n, piece))
    keep = over + even // 2
    assert even > 3 and 2 ** 30 < keep < n
    # who stays, and from where the places that are given up are filled
    gone, come, left = [], [], even // 2
    for j in range(0, n, piece):
        m = mass[j:min(n, j + piece)]
        equal = m == border
        stays = (m > border) | (equal & (equal.long().cumsum(0) <= left))
        left = max(0, left - int(equal.sum()))
        here = max(0, min(keep - j, len(m)))
        gone.append((~stays[:here]).nonzero()[:, 0].add_(j).int())
        come.append(stays[here:].nonzero()[:, 0].add_(j + here).int())
    del m, equal, stays
    gone, come = torch.cat(gone), torch.cat(come)
    assert gone.numel() == come.numel()
    want = index.clone()
    for i in range(0, gone.numel(), piece):
        want[gone[i:i + piece].long()] = come[i:i + piece]
    del gone, come
    k, v = index.clone(), index.clone()
    lens, budget = (torch.tensor([x], dtype=torch.int32).cuda() for x in (n, keep))
    new = knn.cache_evict(k.view(torch.bfloat16).view(*shape, 2), v.view(torch.bfloat16).view(*shape, 2), mass.view(shape),
                          pages, lens, budget, max_keys=n)
    assert new.tolist() == [keep]
    assert torch.equal(k, want) and torch.equal(v, want)
    for j in range(0, keep, piece):  # and each weight went with its token
        w = want[j:min(keep, j + piece)].long()
        assert torch.equal(mass[j:j + len(w)], ((w * 2654435761 >> 8) & 0xffffff).float())


def test_sequences_longer_than_the_hint_keep_their_whole_ledger():
    """Left as they are, with a ledger apart up to their lengths (or as far as their tables go), not up to max_keys."""
    for lens, width, budgets, max_keys in (([100, 90, 20, 95, 200], None, [10, 20, 10, 0, 199], 95),
                                           ([5000, 30, 3000], None, [10, 20, 10], 2500),
                                           ([20000, 9000, 5, 12345, 70001], 1100, [2500, 800, 4, 12344, 0], 9000)):
        x = batch(lens, 2, 64, 64 if width else 16, width=width, seed=17)
        if width:
            x["pages"][0, 250] = -1  # behind the hint: passed over
            x["cache_lens"][4] = 1100 * 64 + 7  # longer than its table, whose last entries are no pages
        for positions in (False, True):
            kept = {n: t.clone() for n, t in x.items()}
            new = check(kept, budgets, out=True, positions=positions, max_keys=max_keys)
            assert int(new[0]) == lens[0] and torch.equal(kept["mass"], x["mass"])


WIDE = 1 << 20  # of a table: a segment is two chunks of 8,192 tokens


@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("kind", ["equal", "two", "by pages", "spread"])
def test_segments_of_several_chunks(kind, positions, out):
    lens = [40000, 20000, 9000, 5, 0, 16385, 16384]
    x = shaped(batch(lens, 2, 64, 64, width=WIDE // 64, seed=18), kind, 18)
    for budgets in ([20000, 16383, 100, 4, 0, 8193, 16383], [39999, 8192, 8999, 0, 0, 1, 8191]):
        y = {n: t.clone() for n, t in x.items()}
        check(y, budgets, [10 * n for n in lens] if positions else None, sinks=4, recent=64, max_keys=WIDE, out=out,
              positions=positions)
        if out:
            assert torch.equal(y["mass"].view(torch.int32), x["mass"].view(torch.int32))


@pytest.mark.parametrize("out", [False, True])
def test_segments_of_several_chunks_with_many_protected_tokens_or_no_page(out):
    lens = [40000, 20000, 16390]
    x = batch(lens, 2, 64, 64, width=WIDE // 64, seed=19, masses="even")
    for recent in (20000 - 30, 17000, 30000):  # just the budget of the first sequence; more than others'; more than all
        check({n: t.clone() for n, t in x.items()}, [20000, 10000, 16389], sinks=30, recent=recent, max_keys=WIDE, out=out,
              positions=False)
    x["pages"][0, 500] = -1                      # in the last chunk
    x["pages"][1, 128] = x["k_cache"].shape[0]   # the first one of the second chunk
    for positions in (False, True):
        check({n: t.clone() for n, t in x.items()}, [30000, 100, 16000], sinks=4, recent=64, max_keys=WIDE, out=out,
              positions=positions)


@pytest.mark.parametrize("max_keys", [None, 40000, WIDE])
@pytest.mark.parametrize("n,budget", [(300, 100), (5000, 4000), (20000, 2500), (20000, 19999), (16385, 16384), (20000, 5)])
def test_a_window_that_is_the_whole_budget(n, budget, max_keys):
    """The first tokens and the last ones stay, whatever the masses; and one more, or one less, than these."""
    for off in (0, 1, -1):
        x = batch([n, n // 2, 30], 2, 64, 64, seed=20, masses="even", width=None if max_keys is None else max_keys // 64)
        check(x, [budget, min(budget, n // 2 - 1), 29], sinks=4, recent=budget - 4 + off, max_keys=max_keys, positions=False)
