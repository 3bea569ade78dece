"""A long run of decoding on a cache with a budget, as the calls are made together: rows are appended at positions of their
own, attend, give the keys they saw their weight, the keys of least weight leave; a token is drawn from scores with
penalties.  Once step by step against the oracle, once with a tree of drafts, once captured and replayed."""
import os

import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

S, H, HK, D, PAGE, WIDTH, V, MODEL = 2, 8, 2, 64, 16, 6, 301, 128
BUDGET, SINKS, RECENT = 40, 2, 8


def host(t):
    return t.detach().double().cpu().numpy()


def ints(t):
    return t.cpu().numpy()


class Run:
    """The state of a run and one step of it."""

    def __init__(self, rows, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.w_qkv = (torch.randn(MODEL, (H + 2 * HK) * D, generator=g) / MODEL ** 0.5 * 1.5).cuda()
        self.w_out = (torch.randn(H * D, V, generator=g) / (H * D) ** 0.5 * 4).cuda()
        self.embed = torch.randn(V, MODEL, generator=g).cuda()
        shape = (S * WIDTH + 1, HK, PAGE, D)
        dev = dict(device="cuda")
        self.k, self.v = (torch.zeros(shape, dtype=torch.bfloat16, **dev) for _ in range(2))
        self.mass = torch.zeros(shape[:3], **dev)
        self.where = torch.zeros(shape[:3], dtype=torch.int32, **dev)
        self.pages = torch.randperm(S * WIDTH + 1, generator=g)[:S * WIDTH].view(S, WIDTH).int().cuda()
        self.lens = torch.zeros(S, dtype=torch.int32, **dev)
        self.next = torch.zeros(S, dtype=torch.int32, **dev)  # positions
        self.budgets = torch.full((S,), BUDGET, dtype=torch.int32, **dev)
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2).float() / D)).cuda()
        self.rows = rows
        self.offsets = torch.arange(S + 1, dtype=torch.int64, **dev) * rows
        self.tokens = torch.randint(0, V, (S * rows,), generator=g).int().cuda()
        self.uniforms = torch.rand(S, generator=g).cuda()
        self.history = torch.zeros(S, 400, dtype=torch.int32, **dev)
        self.history_lens = torch.zeros(S, dtype=torch.int32, **dev)
        self.theta, self.alpha = torch.full((S,), 1.3, **dev), torch.full((S,), 0.4, **dev)
        self.allowed = torch.randint(-(2 ** 31), 2 ** 31, (S, (V + 31) // 32), generator=g, dtype=torch.int32).cuda()
        self.at = torch.arange(rows, dtype=torch.int32, **dev).repeat(S)
        self.qkv = torch.zeros(S * rows, H + 2 * HK, D, dtype=torch.bfloat16, **dev)
        self.positions = torch.zeros(S * rows, dtype=torch.int32, **dev)
        self.logits = torch.zeros(S, V, **dev)
        paged = dict(pages=self.pages, row_offsets=self.offsets, cache_lens=self.lens)
        q, k, v = self.qkv[:, :H], self.qkv[:, H:H + HK], self.qkv[:, H + HK:]
        self.append = knn.KVAppend(k, v, self.k, self.v, q=q, inv_freq=self.inv_freq, positions=self.positions, **paged)
        self.attend = knn.TreeAttention(self.append.q_out, self.k, self.v, want_lse=True, **paged)
        self.weigh = knn.KeyWeights(self.append.q_out, self.attend.lse, self.k, mass=self.mass, key_positions=self.where,
                                    positions=self.positions, decay=0.9, **paged)
        self.evict = knn.CacheEvict(self.k, self.v, self.mass, self.pages, self.lens, self.budgets, key_positions=self.where,
                                    next_positions=self.next, sinks=SINKS, recent=RECENT)
        self.adjust = knn.ScoreAdjuster(self.logits, history=self.history, history_lens=self.history_lens,
                                        repetition=self.theta, presence=self.alpha, allowed=self.allowed)
        self.draw = knn.Sampler(self.adjust.out, self.uniforms)

    def state(self):
        return [self.k, self.v, self.mass, self.where, self.lens, self.next, self.history, self.history_lens, self.tokens]

    def project(self):
        x = self.embed[self.tokens.long()] @ self.w_qkv
        self.qkv.copy_(x.view(S * self.rows, -1, D))
        self.positions.copy_(self.next.repeat_interleave(self.rows) + self.at)

    def close(self):
        """After the rows are in the cache and weighed: the lengths, the eviction."""
        self.lens.add_(self.rows)
        self.next.add_(self.rows)
        self.evict.run()
        self.lens.copy_(self.evict.new_lens)

    def answer(self, out):
        self.logits.copy_(out.view(S, self.rows, -1)[:, -1].float() @ self.w_out)
        self.adjust.run()
        token, _, _ = self.draw.run()
        self.history.scatter_(1, self.history_lens.long()[:, None], token[:, None])
        self.history_lens.add_(1)
        self.tokens.copy_(torch.cat([self.tokens.view(S, -1)[:, 1:], token[:, None]], 1).flatten())
        self.uniforms.copy_((self.uniforms * 7.3 + 0.17) % 1.0)

    def step(self):
        self.project()
        self.append.run()
        out = self.attend.run()
        self.weigh.run()
        self.close()
        self.answer(out)


def check_weights(before, run, tree=None, source=None, q=None, lse=None, offsets=None):
    """mass and positions against the oracle from what the GPU has; before: (mass, where) of before the call."""
    q = run.append.q_out if q is None else q
    lse = run.attend.lse if lse is None else lse
    offsets = run.offsets if offsets is None else offsets
    rows = int(offsets[-1])
    want, where, terms = lm.key_weights(host(q), host(lse), host(run.k), ints(run.pages), ints(offsets), ints(run.lens),
                                        host(before[0]), D ** -0.5, 0.9, tree, source, ints(before[1]),
                                        ints(run.positions)[:rows])
    # as in the operator's own tests: the scores' and sums' roundings in 32 bits
    assert (np.abs(host(run.mass) - want) <= 2.0 ** -22 * terms + 64 * 2.0 ** -24 * np.abs(want) + 1e-30).all()
    assert np.array_equal(ints(run.where), where)


def check_eviction(before, run):
    """Everything that the eviction moved, to the bit; before: (k, v, mass, where, lens)."""
    words = [t.cpu().view(torch.int16).numpy() for t in before[:2]]
    want = lm.evict(*words, before[2].cpu().numpy(), ints(before[3]), ints(run.pages), ints(before[4]), ints(run.budgets),
                    ints(run.next), SINKS, RECENT, WIDTH * PAGE)
    for got, w in ((run.k.view(torch.int16), want[0]), (run.v.view(torch.int16), want[1]), (run.mass, want[2]),
                   (run.where, want[3]), (run.lens, want[4])):
        assert np.array_equal(ints(got), w)


def test_steps_against_the_oracle():
    run = Run(1)
    sees = lambda: (run.k.clone(), run.v.clone(), run.mass.clone(), run.where.clone())  # noqa: E731
    for i in range(60):
        run.project()
        run.append.run()
        out = run.attend.run()
        before = run.mass.clone(), run.where.clone()
        run.weigh.run()
        torch.cuda.synchronize()
        if i % 7 == 0 or i > 50:
            want, lse = lm.attend(host(run.append.q_out), host(run.k), host(run.v), ints(run.pages), ints(run.offsets),
                                  ints(run.lens), D ** -0.5)
            big, _ = lm.attend(host(run.append.q_out), host(run.k), np.abs(host(run.v)), ints(run.pages), ints(run.offsets),
                               ints(run.lens), D ** -0.5)
            # half a step for the result and for each weight (numerator and sum); 1e-4 covers the 32-bit scores
            assert (np.abs(host(out) - want) <= 2.0 ** -8 * (2 * np.abs(want) + big) + 1e-4 * big).all()
            # the weights are summed as they are rounded to bf16: 2^-9 of the sum, and the 32-bit scores
            assert (np.abs(host(run.attend.lse) - lse) <= 2.0 ** -8).all()
            check_weights(before, run)
            # what a row's weights are: they add up to its heads' ones, to what its sum's rounding is
            new = host(run.mass) - 0.9 * host(before[0])
            at = [[lm.place(ints(run.pages), s, c, S * WIDTH + 1, PAGE) for c in range(int(run.lens[s]) + 1)] for s in range(S)]
            for s in range(S):
                for h in range(HK):
                    last = at[s][-1]
                    total = sum(new[p, h, slot] for p, slot in at[s][:-1]) + host(run.mass)[last[0], h, last[1]]
                    assert abs(total - H // HK) <= 2.0 ** -7 * (H // HK)
        held = (*sees(), (run.lens + 1).clone())
        run.close()
        torch.cuda.synchronize()
        check_eviction(held, run)
        run.answer(out)
        torch.cuda.synchronize()
        for s in range(S):
            n = int(run.history_lens[s]) - 1
            adjusted = lm.adjust(host(run.logits)[s], output=ints(run.history)[s, :n], repetition=float(run.theta[s]),
                                 presence=float(run.alpha[s]),
                                 allowed=np.unpackbits(ints(run.allowed)[s].view(np.uint8), bitorder="little")[:V])
            got = host(run.adjust.out)[s]
            assert np.array_equal(np.isinf(got), np.isinf(adjusted))
            fine = np.isfinite(adjusted)
            # a product or quotient and a difference in 32 bits
            assert (np.abs(got - adjusted)[fine] <= 2.0 ** -23 * (np.abs(adjusted[fine]) * 2 + 1)).all()
            assert fine[int(run.history[s, n])]  # a token that the grammar allows
    assert run.lens.tolist() == [BUDGET, BUDGET] and run.next.tolist() == [60, 60]
    # each head keeps tokens of its own, the first and the last ones among them
    for s in range(S):
        for h in range(HK):
            kept = sorted(int(run.where[p, h, slot]) for p, slot in (
                lm.place(ints(run.pages), s, c, S * WIDTH + 1, PAGE) for c in range(BUDGET)))
            assert len(set(kept)) == BUDGET and kept[:SINKS] == [0, 1] and kept[-RECENT:] == list(range(52, 60))


def test_a_tree_is_accepted_and_weighed():
    """A prompt, then a tree of drafts for each sequence, of which a path stays: its rows are appended over the drafts and
    weighed by their sums, with the positions of the path."""
    run = Run(20, seed=3)
    run.step()  # the prompts
    assert run.lens.tolist() == [20, 20]
    parents = [-1, 0, 1, 1, 3, 2, 0, 6]
    paths = [[0, 1, 3, 4], [0, 6, 7]]
    n = len(parents)
    mask = torch.cat([knn.tree_words(parents, "cuda")] * S)
    depth = []
    for a in parents:
        depth.append(0 if a < 0 else depth[a] + 1)
    offsets = torch.arange(S + 1, dtype=torch.int64, device="cuda") * n
    positions = run.next.repeat_interleave(n) + torch.tensor(depth * S, dtype=torch.int32, device="cuda")
    drafts = torch.randint(0, V, (S * n,), device="cuda")
    qkv = (run.embed[drafts] @ run.w_qkv).bfloat16().view(S * n, -1, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:]
    cache = dict(pages=run.pages, row_offsets=offsets, cache_lens=run.lens)
    turned = knn.kv_append(k, v, run.k, run.v, q=q, inv_freq=run.inv_freq, positions=positions, **cache)
    _, lse = knn.tree_attention(turned, run.k, run.v, tree_mask=mask, want_lse=True, **cache)
    scores = torch.zeros(S * n, V, device="cuda")
    got = knn.adjust_scores(scores, row_offsets=offsets, row_tokens=drafts.int(), tree_mask=mask,
                            frequency=torch.ones(S * n, device="cuda"))
    for t in range(S * n):  # each row counts the drafts that it hangs under
        want, i = np.zeros(V), t % n
        while i >= 0:
            want[int(drafts[t - t % n + i])] -= 1
            i = parents[i]
        assert np.array_equal(host(got)[t], want)
    source = torch.tensor(sum(([s * n + i for i in p] for s, p in enumerate(paths)), []), dtype=torch.int32, device="cuda")
    kept = torch.tensor([0, len(paths[0]), len(paths[0]) + len(paths[1])], dtype=torch.int64, device="cuda")
    cache["row_offsets"] = kept
    run.positions[:len(source)] = positions[source.long()]
    path_positions = run.positions[:len(source)].clone()
    knn.kv_append(k, v, run.k, run.v, inv_freq=run.inv_freq, positions=path_positions, source_rows=source, **cache)
    before = run.mass.clone(), run.where.clone()
    knn.key_weights(turned, lse, run.k, mass=run.mass, key_positions=run.where, positions=path_positions, source_rows=source,
                    decay=0.9, **cache)
    torch.cuda.synchronize()
    check_weights(before, run, source=ints(source), q=turned, lse=lse, offsets=kept)
    # the path's rows saw what they see now, so that their weights add up to one a head
    for s in range(S):
        rows = len(paths[s])
        total = 0.0
        for c in range(20 + rows):
            p, slot = lm.place(ints(run.pages), s, c, S * WIDTH + 1, PAGE)
            total += host(run.mass)[p, :, slot].sum() - (0.9 * host(before[0])[p, :, slot].sum() if c < 20 else 0.0)
        assert abs(total - rows * H) <= 2.0 ** -7 * rows * H


def test_steps_in_a_graph():
    """Steps captured once and replayed, with eager steps of another run between: the same state to the bit."""
    a, b = Run(1, seed=5), Run(1, seed=5)
    for r in (a, b):
        for _ in range(45):  # until the budget is reached
            r.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step()
    torch.cuda.current_stream().wait_stream(side)
    a.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(8):
        graph.replay()
        a.step()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)
    assert a.lens.tolist() == [BUDGET, BUDGET]


def test_the_example_of_the_readme():
    """Its lines as they stand there, step after step: the first tokens and the last ones are never evicted."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        block = next(b for b in f.read().split("```")[1::2] if "knn.CacheEvict" in b)
    setup, step = block.removeprefix("python\n").rstrip("\n").rsplit("\n", 1)
    assert "evict.run()" in step
    n, per, budget, page, width = 290, 8, 300, 64, 128
    g = torch.Generator().manual_seed(5)
    dev = dict(device="cuda")
    shape = (S * width, HK, page, D)
    x = {"knn": knn, "added": per, "table": torch.arange(S * width, dtype=torch.int32, **dev).view(S, width),
         "lens": torch.full((S,), n, dtype=torch.int32, **dev), "budgets": torch.full((S,), budget, dtype=torch.int32, **dev),
         "next_positions": torch.full((S,), n, dtype=torch.int32, **dev),
         "depths": torch.zeros(S * per, dtype=torch.int32, **dev), "mass": torch.full(shape[:3], 5.0, **dev),
         "where": torch.arange(width * page, dtype=torch.int32, **dev).view(1, width, 1, page).expand(
             S, width, HK, page).reshape(shape[:3]).contiguous(),
         "p_m": torch.softmax(torch.randn(S, V, generator=g), 1).cuda(),
         "history": torch.randint(0, V, (S, 50), generator=g, dtype=torch.int32).cuda(),
         "history_lens": torch.full((S,), 50, dtype=torch.int32, **dev), "prompt_lens": torch.full((S,), 9, dtype=torch.int32, **dev),
         "penalty": torch.full((S,), 1.2, **dev), "grammar": torch.full((S, (V + 31) // 32), -1, dtype=torch.int32, **dev)}
    x["where"].masked_fill_(x["where"] >= n, -1)
    x["mass"].masked_fill_((x["where"] >= 0) & (x["where"] < 4), 0.0)  # the first tokens have drawn least
    x["k_cache"], x["v_cache"] = (torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    x["rows"] = dict(pages=x["table"], row_offsets=torch.arange(S + 1, dtype=torch.int64, **dev) * per, cache_lens=x["lens"])
    q, k, v = (torch.randn(S * per, h, D, generator=g).to(torch.bfloat16).cuda() for h in (H, HK, HK))
    x["append"] = knn.KVAppend(k, v, x["k_cache"], x["v_cache"], q=q, positions=x["depths"], **x["rows"])
    x["attend"] = knn.TreeAttention(x["append"].q_out, x["k_cache"], x["v_cache"], max_rows=16, max_keys=8192, want_lse=True,
                                    **x["rows"])
    exec(setup, x)
    at = n
    for _ in range(12):
        x["depths"].copy_(torch.arange(at, at + per, dtype=torch.int32, **dev).repeat(S))
        x["append"].run()
        x["attend"].run()
        exec(step, x)
        at += per
        assert x["lens"].tolist() == [min(budget, at)] * S and x["scores"].shape == (S, V)
        places = x["where"].view(S, width, HK, page).permute(0, 2, 1, 3).reshape(S, HK, -1)[:, :, :min(budget, at)]
        for kept in places.reshape(S * HK, -1).tolist():
            assert len(set(kept)) == len(kept) and {0, 1, 2, 3, *range(at - 256, at)} <= set(kept)
