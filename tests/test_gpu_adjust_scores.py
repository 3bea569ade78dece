"""Adjusted scores on the GPU against the fp64 oracle: penalties, biases, masks, on logits and probabilities, trees of
drafts, odd sizes and strides, in place, and what has to stay as it was."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PARAMETERS = ("repetition", "presence", "frequency")


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def batch(rows, V, dtype="f32", probs=False, S=None, width=40, seed=0, bias=0, grammar=False, drafts=None, tree=False,
          prompt=True, extra=0):
    """drafts: the rows of each sequence."""
    g = torch.Generator().manual_seed(seed)
    S = rows if drafts is None else len(drafts)
    x = torch.randn(rows, V, generator=g) * 3
    if probs:
        x = torch.softmax(x, 1) * (torch.rand(rows, V, generator=g) < 0.9)

    def tokens(*shape):  # among few, so that they repeat, and some that are none
        return torch.randint(-2, min(V, 30) + 1, shape, generator=g, dtype=torch.int32)

    def some(lo, hi):
        return (lo + (hi - lo) * torch.rand(rows, generator=g)).float()

    c = {"scores": x.to(TYPES[dtype]), "history": tokens(S, width), "probabilities": probs,
         "history_lens": torch.randint(0, width + 1, (S,), generator=g, dtype=torch.int32),
         "repetition": some(0.7, 1.5), "presence": some(-1, 1), "frequency": some(-0.5, 0.5)}
    c["history"][:, -1] = V - 1
    if prompt:
        c["prompt_lens"] = torch.randint(0, width // 2 + 1, (S,), generator=g, dtype=torch.int32)
    if drafts is not None:
        c["row_offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(drafts)]), dtype=torch.int64)
        c["row_tokens"] = tokens(rows)
        if tree:
            masks = [knn.tree_words([int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)], "cpu")
                     for n in drafts]
            words = max(1, max(m.shape[1] for m in masks))
            c["tree_mask"] = torch.cat([torch.nn.functional.pad(m, (0, words - m.shape[1])) for m in masks] + [
                torch.full((rows - sum(drafts), words), -1, dtype=torch.int32)])
    if bias:
        c["bias_tokens"] = tokens(S, bias)
        c["bias_values"] = torch.randn(S, bias, generator=g) * 5
    if grammar:
        c["allowed"] = torch.randint(-(2 ** 31), 2 ** 31, (rows, (V + 31) // 32), generator=g, dtype=torch.int32)
    return {n: t.cuda() if torch.is_tensor(t) else t for n, t in c.items()}


def want_of(c):
    """The oracle's scores of the rows that belong to a sequence; NaN for the others."""
    scores = host(c["scores"])
    rows, V = scores.shape
    want = np.full((rows, V), np.nan)
    h = {n: t.cpu().numpy() for n, t in c.items() if torch.is_tensor(t) and n != "scores"}
    off = h.get("row_offsets", np.arange(rows + 1))
    for t in range(rows):
        s = lm.sequence_of(off, t)
        if s < 0:
            continue
        prompt, output = [], []
        if "history" in h:
            n = min(max(int(h["history_lens"][s]), 0), h["history"].shape[1])
            p = min(max(int(h["prompt_lens"][s]), 0), n) if "prompt_lens" in h else 0
            prompt, output = h["history"][s, :p].tolist(), h["history"][s, p:n].tolist()
        if "row_tokens" in h:
            for j in range(int(off[s]), int(off[s + 1])):
                i = j - int(off[s])
                seen = j <= t
                if "tree_mask" in h:
                    seen = i < 32 * h["tree_mask"].shape[1] and (int(h["tree_mask"][t, i // 32]) >> (i % 32)) & 1
                if seen:
                    output.append(int(h["row_tokens"][j]))
        bias = list(zip(h["bias_tokens"][s].tolist(), h["bias_values"][s].tolist())) if "bias_tokens" in h else ()
        allowed = None
        if "allowed" in h:
            allowed = np.unpackbits(h["allowed"][t].view(np.uint8), bitorder="little")[:V]
        want[t] = lm.adjust(scores[t], c["probabilities"], prompt, output, *(
            float(h[n][t]) if n in h else off for n, off in zip(PARAMETERS, (1.0, 0.0, 0.0))), bias, allowed)
    return want


def compare(c, want, got, before):
    """Within half a step of the type and the arithmetic before it; untouched scores to the bit, rows of nobody as they
    were."""
    t = c["scores"].dtype
    g, x = host(got), host(c["scores"]) if got is not c["scores"] else before
    mine = ~np.isnan(want) | np.isnan(x)
    nobody = np.isnan(want).all(1) & ~np.isnan(x).all(1)
    assert np.array_equal(g[nobody], before[nobody], equal_nan=True)
    mine[nobody] = False
    w, g = want[mine], g[mine]
    assert np.array_equal(np.isnan(w), np.isnan(g))
    # Logits: a quotient or product, two differences, the product with the count and a sum, each a rounding to 2^-24 of what
    # is there then, at most |y| + 2 (|presence| + |frequency| c + |bias|); with the type's own half step.  Probabilities:
    # 64 bits (2^-40 is ample), then 32, then the type's.
    logits, count = not c["probabilities"], 64.0
    rel = 8 * 2.0 ** -24 if logits else 2.0 ** -40 if t == torch.float32 else 2.0 ** -24
    rel += torch.finfo(t).eps / 2 * (1 + 2.0 ** -20)
    size = 8 * 2.0 ** -24 * (1 + count * 0.5 + 25) if logits else 0.0
    tiny = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[t] / 2
    with np.errstate(invalid="ignore"):
        over = np.abs(w) > float(torch.finfo(t).max) * (1 + torch.finfo(t).eps / 4)  # rounds to infinity
        assert np.array_equal(np.isinf(g), np.isinf(w) | over)
        ok = (np.abs(g - w) <= rel * np.abs(w) + size + tiny) | np.isnan(g)  # (where w is one too)
    assert (ok | np.isinf(g)).all() and np.array_equal(np.sign(g[np.isinf(g)]), np.sign(w[np.isinf(g)]))


def check(c, out=None, **over):
    c = dict(c, **over)
    want = want_of(c)
    out = torch.randn(c["scores"].shape, device="cuda").to(c["scores"].dtype) if out is None else out
    before = host(out)
    kept = c["scores"].clone()
    got = knn.adjust_scores(out=out, **c)
    torch.cuda.synchronize()
    assert got is out
    if out.data_ptr() != c["scores"].data_ptr():
        assert torch.equal(kept.view(torch.uint8), c["scores"].view(torch.uint8)) if kept.is_contiguous() else True
    compare(c, want, got, before)
    return got


@pytest.mark.parametrize("dtype,probs", [("f32", False), ("bf16", False), ("f16", False), ("f32", True), ("bf16", True),
                                         ("f16", True)])
@pytest.mark.parametrize("V", [1, 5, 31, 33, 1000, 8192, 8193, 20011])
def test_types_and_vocabularies(dtype, probs, V):
    check(batch(3, V, dtype, probs, seed=V, bias=9, grammar=True))
    check(batch(2, V, dtype, probs, seed=V + 1, bias=1))
    check(batch(2, V, dtype, probs, seed=V + 2))


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_of_drafts(probs, tree):
    c = batch(50, 997, "f32", probs, drafts=[1, 0, 40, 7], tree=tree, seed=1, bias=5, grammar=True)  # two rows of nobody
    check(c)
    check({n: t for n, t in c.items() if n not in ("history", "history_lens", "prompt_lens")})
    check({n: t for n, t in c.items() if n not in ("row_tokens", "tree_mask")})


def test_a_mask_that_names_rows_of_no_sequence():
    c = batch(6, 200, drafts=[3, 3], tree=True, seed=2)
    c["tree_mask"][:] = -1  # every bit: those past the sequence's rows name nobody
    check(c)


def test_each_step_alone():
    for seed, dtype in enumerate(("f32", "bf16")):
        c = batch(4, 3001, dtype, seed=seed, bias=20, grammar=True)
        for keep in ((), ("bias_tokens", "bias_values"), ("allowed",), *((n, "history", "history_lens") for n in PARAMETERS),
                     ("history", "history_lens", "repetition", "prompt_lens")):
            got = check({n: t for n, t in c.items() if n in ("scores", "probabilities") + keep})
            if keep == ():
                assert torch.equal(got, c["scores"])


def test_parameters_that_are_off():
    c = batch(6, 500, seed=4)
    c["repetition"][:5] = torch.tensor([0.0, -1.0, float("nan"), float("inf"), -float("inf")])
    c["presence"][:3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    c["frequency"][3:] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    check(c)


@pytest.mark.parametrize("probs", [False, True])
def test_scores_that_are_no_numbers(probs):
    c = batch(3, 400, probs=probs, seed=5, bias=10, grammar=True)
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, 3e38, -1.0)):
        c["scores"][:, i::13] = v
    check(c)


def test_probabilities_small_and_large():
    """Powers of what fp32 just holds, and biases whose factors alone pass fp32."""
    c = batch(2, 64, probs=True, seed=6, bias=30)
    c["scores"][0, :40] = torch.logspace(-45, 38, 40, device="cuda")
    c["repetition"][:], c["presence"][:], c["frequency"][:] = 1.2, 0.0, 0.0
    c["bias_values"] *= 40
    check(c)


def test_biases_that_are_infinite_or_named_twice():
    c = batch(3, 100, seed=7, bias=12)
    c["bias_tokens"][:] = torch.tensor([5, 6, 5, 7, 8, 5, 9, 9, -1, 100, 2 ** 31 - 1, -(2 ** 31)], dtype=torch.int32)
    c["bias_values"][:, 5] = -float("inf")
    c["bias_values"][:, 3] = float("inf")
    check(c)
    check(dict(c, probabilities=True, scores=c["scores"].abs()))


def test_masks_that_allow_nothing_or_everything():
    c = batch(3, 70, "bf16", seed=8, grammar=True)
    c["allowed"][0], c["allowed"][1] = 0, -1
    got = check(c)
    assert torch.isinf(got[0]).all()
    tokens, _, kept = knn.sample(got, torch.full((3,), 0.5, device="cuda"))
    assert tokens[0].item() == -1 and kept[0].item() == 0


@pytest.mark.parametrize("lens", [[0, 0, 0], [-4, 1 << 30, 40], [1, 2, 3]])
def test_lengths_of_histories(lens):
    c = batch(3, 90, seed=9)
    c["history_lens"][:] = torch.tensor(lens, dtype=torch.int32)
    c["prompt_lens"][:] = torch.tensor([5, 1 << 30, -3], dtype=torch.int32)
    check(c)


@pytest.mark.parametrize("tokens", [3, 50])
def test_long_histories_of_the_same_tokens(tokens):
    """Counts of thousands: 30,000 tokens of which few differ (biases of nothing, so that fp32 holds the steps)."""
    c = batch(2, 9000, width=30000, seed=10, prompt=False)
    c["history"][:] = torch.randint(0, tokens, (2, 30000), dtype=torch.int32) * 179
    c["history_lens"][:] = torch.tensor([30000, 29999], dtype=torch.int32)
    c["frequency"][:] = 2.0 ** -12   # a power of two: the counts' products are whole multiples of it
    c["presence"][:] = 0.5
    want, got = want_of(c), host(knn.adjust_scores(**c))
    # a rounding of the product or quotient of |x| <= 16 and two of differences under 32
    assert (np.abs(got - want) <= 2.0 ** -24 * (np.abs(host(c["scores"])) * 2 + 64)).all()


def test_strides_and_in_place():
    for dtype in ("f32", "bf16"):
        for V, stride in ((1000, 1003), (37, 38), (8200, 8200), (4096, 4104)):
            c = batch(5, V, dtype, seed=V, bias=3, grammar=V < 5000)
            wide = torch.zeros(5, stride, dtype=TYPES[dtype], device="cuda")
            wide[:, :V] = c["scores"]
            view = wide[:, :V]
            a = check(c)
            b = check(c, scores=view)
            assert torch.equal(a, b)
            into = torch.full((5, stride + 1), 7.0, dtype=TYPES[dtype], device="cuda")
            check(c, scores=view, out=into[:, 1:V + 1])
            assert torch.equal(into[:, 1:V + 1], a) and (into[:, 0] == 7).all() and (into[:, V + 1:] == 7).all()
            knn.adjust_scores(**dict(c, scores=view, out=view))
            assert torch.equal(view, a) and (wide[:, V:] == 0).all()
    one = batch(4, 100, seed=11)
    same = one["scores"][:1].expand(4, 100)  # one row of scores, read four times
    check(one, scores=same)


def test_replays_of_a_graph():
    c = batch(20, 5000, "bf16", drafts=[5, 8, 7], tree=True, seed=12, bias=6, grammar=True)
    call = knn.ScoreAdjuster(**c)
    want = call.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    for shift in range(3):
        call.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, want)
        c["history_lens"].add_(1).clamp_(max=40)
        c["row_tokens"].add_(1)
        want = knn.adjust_scores(**c)


def test_argument_checks():
    c = batch(4, 100, drafts=[1, 3], bias=3, grammar=True)
    for over in (dict(history=c["history"].long()), dict(history_lens=c["history_lens"][:1]), dict(bias_values=c["presence"]),
                 dict(allowed=c["allowed"][:, :2]), dict(out=c["scores"].half()), dict(out=c["scores"][:3]),
                 dict(scores=c["scores"].t()), dict(repetition=c["repetition"].double()), dict(row_offsets=c["history_lens"]),
                 dict(row_tokens=c["row_tokens"].cpu())):
        with pytest.raises(ValueError):
            knn.adjust_scores(**dict(c, **over))
    with pytest.raises(TypeError):
        knn.adjust_scores(c["scores"].double())
    with pytest.raises(knn.KnnError):
        knn.adjust_scores(c["scores"], repetition=c["repetition"])
    with pytest.raises(knn.KnnError):
        knn.adjust_scores(c["scores"], out=c["scores"].view(-1).as_strided((4, 100), (50, 1)))


@pytest.mark.parametrize("V,rows", [(2048, 2), (2047, 1), (8192, 200), (8190, 200)])
@pytest.mark.parametrize("probs", [False, True])
def test_every_token_is_touched(V, rows, probs):
    """A whole slice's tokens in the history, of either kind of workgroup, and with biases besides."""
    c = batch(rows, V, probs=probs, seed=13, width=V + 5, bias=4)
    c["history"][:, :V] = torch.arange(V, dtype=torch.int32).flip(0)
    c["history_lens"][:] = V
    c["bias_tokens"][:, 0] = V - 1
    check(c)


def test_histories_longer_than_a_pass_and_many_drafts():
    c = batch(1200, 300, "bf16", drafts=[1000, 200], seed=14, width=9000)
    c["history_lens"][:] = torch.tensor([9000, 8193], dtype=torch.int32)
    c["prompt_lens"][:] = torch.tensor([8500, 8192], dtype=torch.int32)
    c["frequency"][:] = 2.0 ** -10
    want, got = want_of(c), host(knn.adjust_scores(**c))
    # half a step of bf16, and before it the fp32 steps' roundings of numbers under 64
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16).all()


def test_on_another_stream():
    c = batch(20, 5000, "bf16", seed=15, bias=6, grammar=True)
    want = knn.adjust_scores(**c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = knn.ScoreAdjuster(**c)
    call.run(side)
    side.synchronize()
    assert torch.equal(call.out, want)


@pytest.mark.parametrize("rows,probs", [((1 << 18) + 9, False), ((1 << 20) + 33, True)])
def test_more_rows_than_a_row_of_the_grid(rows, probs):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.rand(rows, 5, generator=g, device="cuda") + 0.1
    history = torch.randint(0, 5, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
    allowed = torch.randint(0, 32, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
    presence = torch.rand(rows, generator=g, device="cuda")
    got = knn.adjust_scores(x, history, torch.ones(rows, dtype=torch.int32, device="cuda"), presence=presence,
                            allowed=allowed, probabilities=probs)
    off = torch.zeros(rows, 5, dtype=torch.float64, device="cuda").scatter_(1, history.long(), presence.double()[:, None])
    want = x.double() * torch.exp(-off) if probs else x.double() - off
    seen = (allowed >> torch.arange(5, device="cuda", dtype=torch.int32) & 1) != 0
    want = torch.where(seen, want, 0.0 if probs else float("-inf"))
    # one rounding to 32 bits, of a value of at most 1.1
    assert ((got - want).abs()[seen] <= 2.0 ** -24 * 1.1 + 1e-12).all() and torch.equal(got[~seen].double(), want[~seen])


@pytest.mark.parametrize("probs", [False, True])
def test_histories_and_biases_of_no_entries(probs):
    """Tables without columns are none at all, as a program has them that has drawn nothing yet."""
    c = batch(6, 500, probs=probs, drafts=[4, 2], bias=3, grammar=True, seed=16)
    none = dict(history=c["history"][:, :0], bias_tokens=c["bias_tokens"][:, :0], bias_values=c["bias_values"][:, :0])
    for some in (("history",), ("bias_tokens", "bias_values"), tuple(none)):
        check(dict(c, **{n: none[n] for n in some}))
    no_drafts = {n: t for n, t in c.items() if n not in ("row_tokens", "tree_mask")}
    check(dict(no_drafts, history=torch.empty(2, 0, dtype=torch.int32, device="cuda")))
    got = knn.adjust_scores(**dict({n: t for n, t in no_drafts.items() if n != "allowed"}, **none))
    assert torch.equal(got, c["scores"])
    with pytest.raises(ValueError):
        knn.adjust_scores(**dict(c, history=none["history"], history_lens=c["history_lens"][:1]))
    with pytest.raises((ValueError, knn.KnnError)):
        knn.adjust_scores(c["scores"], history=c["history"], row_offsets=c["row_offsets"])
