"""The calls together, as a step of speculation makes them: a draft tree's rows go into the cache, attend over it, give
logits, the mixture and a drawn token; the accepted path is appended once more and decoding goes on from there."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().double().cpu().numpy()


class Layer:
    """One attention layer with random weights, its logits, and the same in fp64 from the rounded tensors."""

    def __init__(self, d_model=256, heads=8, kv_heads=2, d=64, V=999, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.d, self.V = heads, kv_heads, d, V
        self.w_qkv = (torch.randn(d_model, (heads + 2 * kv_heads) * d, generator=g) / d_model ** 0.5).bfloat16().cuda()
        self.w_out = (torch.randn(heads * d, V, generator=g) / (heads * d) ** 0.5 * 3).bfloat16().cuda()
        self.embed = torch.randn(V, d_model, generator=g).bfloat16().cuda()
        self.inv_freq = (10000.0 ** (-torch.arange(0, d, 2).float() / d)).cuda()

    def qkv(self, tokens):
        x = (self.embed[tokens].float() @ self.w_qkv.float()).bfloat16().view(len(tokens), -1, self.d)
        return x[:, :self.heads], x[:, self.heads:self.heads + self.kv_heads], x[:, self.heads + self.kv_heads:]

    def logits(self, out):
        return out.flatten(1).float() @ self.w_out.float()


class Sequence:
    """The caches of two sequences and the same in the oracle's hands."""

    def __init__(self, layer, n_pages=40, page=16, width=12):
        shape = (n_pages, layer.kv_heads, page, layer.d)
        self.layer = layer
        self.k, self.v = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.pages = torch.randperm(n_pages)[:2 * width].view(2, width).int().cuda()
        self.lens = torch.zeros(2, dtype=torch.int32, device="cuda")

    def step(self, tokens, offsets, positions=None, mask=None, source=None):
        """Appends the rows and attends; (out, q) checked against the oracle on the cache as it is."""
        la = self.layer
        q, k, v = la.qkv(tokens)
        off = torch.tensor(offsets, dtype=torch.int64, device="cuda")
        before_k, before_v = host(self.k), host(self.v)
        turned = knn.kv_append(k, v, self.k, self.v, self.pages, off, self.lens, q=q, positions=positions,
                               inv_freq=la.inv_freq, source_rows=source)
        pages, o, lens = self.pages.cpu().numpy(), off.cpu().numpy(), self.lens.cpu().numpy()
        want_q, want_k, want_v = lm.append(
            host(q), host(k), host(v), before_k, before_v, pages, o, lens, turned.shape[0], q_out=host(turned),
            positions=None if positions is None else positions.cpu().numpy(), inv_freq=la.inv_freq.cpu().numpy(),
            source_rows=None if source is None else source.cpu().numpy())
        for got, want in ((turned, want_q), (self.k, want_k), (self.v, want_v)):
            got = host(got)
            assert np.array_equal(np.isnan(got), np.isnan(want))
            err = np.nan_to_num(np.abs(got - want))
            assert (err <= np.nan_to_num(2.0 ** -8 * np.abs(want)) + 5e-6).all()
        if source is not None:
            return None
        out = knn.tree_attention(turned, self.k, self.v, self.pages, off, self.lens, tree_mask=mask)
        torch.cuda.synchronize()
        sees = None
        if mask is not None:
            sees = np.unpackbits(mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
        kk, vv = np.nan_to_num(host(self.k)), np.nan_to_num(host(self.v))
        want, _ = lm.attend(host(turned), kk, vv, pages, o, lens, la.d ** -0.5, sees)
        mass, _ = lm.attend(host(turned), kk, np.abs(vv), pages, o, lens, la.d ** -0.5, sees)
        # half a step for the result and for each weight (numerator and sum); 1e-4 of the mass covers the 32-bit scores
        assert (np.abs(host(out) - want) <= 2.0 ** -8 * (2 * np.abs(want) + mass) + 1e-4 * mass).all()
        return out


def test_a_tree_is_drafted_verified_kept_and_decoded_on():
    torch.manual_seed(0)
    layer = Layer()
    seq = Sequence(layer)
    # the prompts, as chains
    prompts = [37, 90]
    tokens = torch.randint(0, layer.V, (sum(prompts),), device="cuda")
    out = seq.step(tokens, [0, 37, 127])
    assert torch.isfinite(out.float()).all()
    seq.lens += torch.tensor(prompts, dtype=torch.int32, device="cuda")

    # a tree for the first sequence (two spans with a common beginning), a chain for the second
    parents = [[-1, 0, 1, 1, 3, 2], [-1, 0, 1, 2]]
    mask = torch.cat([knn.tree_words(p, "cuda") for p in parents])
    depth = []
    for p in parents:
        d = []
        for a in p:
            d.append(0 if a < 0 else d[a] + 1)
        depth.append(d)
    at = torch.cat([seq.lens[s].item() + torch.tensor(depth[s]) for s in range(2)]).int().cuda()
    drafts = torch.randint(0, layer.V, (10,), device="cuda")
    out = seq.step(drafts, [0, 6, 10], positions=at, mask=mask)
    logits = layer.logits(out)

    # p_LM, the mixture with retrieved neighbours, and a token of each row from p_M
    p_lm = torch.softmax(logits, 1)
    keys = torch.randn(500, 128, device="cuda")
    queries = torch.randn(10, 128, device="cuda")
    values = torch.randint(0, layer.V, (500,), dtype=torch.int32, device="cuda")
    prob = knn.MixtureProblem(queries, keys, values, torch.tensor([0, 500], device="cuda"),
                              torch.tensor([0, 10], device="cuda"), p_lm, 32)
    step = prob.run_nest(0.3, 0.1, 0.5, draft_tokens=drafts.int())
    uniforms = torch.rand(10, device="cuda")
    top_p = torch.full((10,), 0.9, device="cuda")
    token, share, kept = knn.sample(step["p_m"], uniforms, probabilities=True, top_p=top_p)
    torch.cuda.synchronize()
    p_m = host(step["p_m"])
    for r in range(10):
        want = lm.sample(p_m[r], float(uniforms[r]), True, top_p=float(top_p[r]))
        assert (int(token[r]), int(kept[r])) == (want[0], want[2]) and abs(float(share[r]) - want[1]) < 1e-6
    # T = 0 is the step's own greedy token
    greedy, _, _ = knn.sample(step["p_m"], uniforms, probabilities=True, temperature=torch.zeros(10, device="cuda"))
    assert torch.equal(greedy, step["next_token"])
    # the chain through relaxed verification
    offs = torch.tensor([6, 10], dtype=torch.int64, device="cuda")
    accepted, _ = knn.spec_verify(step["p_max"], step["p_draft"], step["next_token"], offs, 1.0)
    assert 0 <= int(accepted[0]) <= 4

    # keep the branch 0, 1, 3, 4 of the tree and two of the chain: once more, over the drafts, at their depths
    path = torch.tensor([0, 1, 3, 4, 6, 7], dtype=torch.int32, device="cuda")
    seq.step(drafts, [0, 4, 6], source=path)
    seq.lens += torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    # one more token each: as if the kept tokens had been fed one after the other
    last = torch.randint(0, layer.V, (2,), device="cuda")
    after = seq.step(last, [0, 1, 2]).clone()

    other = Sequence(layer)
    all_tokens = [torch.cat([tokens[:37], drafts[[0, 1, 3, 4]], last[:1]]), torch.cat([tokens[37:], drafts[6:8], last[1:]])]
    fed = other.step(torch.cat(all_tokens), [0, 42, 42 + 93])
    # the caches hold the same bits, so either side is off by half a step of the result and of its weights, of which the
    # mass is at most the largest value's, 1e-4 of it for the 32-bit scores
    most = float(np.nan_to_num(np.abs(host(seq.v))).max())
    want = host(fed[[41, 134]])
    assert (np.abs(host(after) - want) <= 2 * (2.0 ** -8 * (2 * np.abs(want) + most) + 1e-4 * most) + 1e-6).all()


def test_two_calls_at_once_and_a_graph_of_all():
    """Objects of their own on two streams at the same time, and one graph of append, attention and draw, replayed on
    new lengths: the bits of the same calls one after the other."""
    S, n, heads, kv_heads, d, page, V = 3, 4, 8, 2, 128, 32, 4001
    shape = (64, kv_heads, page, d)
    off = torch.arange(0, S * n + 1, n, dtype=torch.int64).cuda()
    inv_freq = (10000.0 ** (-torch.arange(0, d, 2).float() / d)).cuda()

    class Program:
        def __init__(self, seed):
            r = torch.Generator().manual_seed(seed)
            self.q, self.k, self.v = (torch.randn(S * n, h, d, generator=r).bfloat16().cuda()
                                      for h in (heads, kv_heads, kv_heads))
            self.cache = [torch.randn(shape, generator=r).bfloat16().cuda() for _ in range(2)]
            self.first = [c.clone() for c in self.cache]
            self.pages = torch.randperm(64, generator=r)[:60].view(S, 20).int().cuda()
            self.lens = torch.zeros(S, dtype=torch.int32, device="cuda")
            rows = (*self.cache, self.pages, off, self.lens)
            self.append = knn.KVAppend(self.k, self.v, *rows, q=self.q, inv_freq=inv_freq)
            self.attend = knn.TreeAttention(self.append.q_out, *rows, max_rows=n, max_keys=640, want_lse=True)
            logits = (torch.randn(S * n, V, generator=r) * 3).bfloat16().cuda()
            self.draw = knn.Sampler(logits, torch.rand(S * n, generator=r).cuda(),
                                    top_p=torch.full((S * n,), 0.9, device="cuda"))

        def reset(self, lens):
            self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
            for c, f in zip(self.cache, self.first):
                c.copy_(f)

        def run(self):
            self.append.run()
            self.attend.run()
            self.draw.run()

        def results(self):
            return [t.clone() for t in (*self.cache, self.append.q_out, self.attend.out, self.attend.lse,
                                        self.draw.token, self.draw.prob, self.draw.kept)]

    both = [Program(1), Program(2)]
    lengths = [[600, 17, 0], [1, 636, 300], [255, 256, 257]]
    want = {}
    for i, lens in enumerate(lengths):
        for j, p in enumerate(both):
            p.reset(lens)
            p.run()
            want[i, j] = p.results()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for i, lens in enumerate(lengths):
        for p in both:
            p.reset(lens)
        torch.cuda.synchronize()
        for _ in range(3):  # the same rows at the same indices again
            for p, s in zip(both, streams):
                with torch.cuda.stream(s):
                    p.run()
        torch.cuda.synchronize()
        for j, p in enumerate(both):
            assert all(torch.equal(a, b) for a, b in zip(p.results(), want[i, j])), (i, j)
    p = both[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for i, lens in enumerate(lengths * 2):
        p.reset(lens)
        graph.replay()
        got = p.results()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i % 3, 0])), i
        p.run()  # the program's own work between the replays
        torch.cuda.synchronize()


def test_outputs_on_another_stream_wait_for_the_memory_they_took():
    """A block that the current stream still reads is freed; the next outputs get it, and are written on another stream."""
    S, heads, d, page = 2048, 64, 128, 16
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(64, 8, page, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(S, heads, d, generator=g).bfloat16().cuda()  # 32 MiB, as the outputs: a block of its own
    pages = (torch.arange(S, dtype=torch.int32) % 64).view(S, 1).cuda()
    off, lens = torch.arange(S + 1).cuda(), torch.full((S,), 7, dtype=torch.int32, device="cuda")
    rows = dict(max_rows=1, max_keys=8)
    want = knn.tree_attention(q, k, v, pages, off, lens, **rows)
    x = torch.randn(4096, 4096, generator=g).bfloat16().cuda()
    side = torch.cuda.Stream()
    y = x @ x
    torch.cuda.synchronize()
    torch.cuda.empty_cache()  # no other free block of that size
    first = torch.full_like(q, 3.0)
    for _ in range(40):
        y = x @ x
    second = first.clone()  # behind the products
    at = first.data_ptr()
    del first
    out = knn.tree_attention(q, k, v, pages, off, lens, stream=side, **rows)
    torch.cuda.synchronize()
    if out.data_ptr() != at:
        pytest.skip("the allocator gave the outputs another block")
    assert (second == 3.0).all() and torch.equal(out, want)
