"""Attention of drafts over the paged cache on the GPU against the fp64 oracle: lengths, pages, head layouts, trees,
rows that see nothing, what lies in unseen places, ranges joined, streams and graphs."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def batch(dtype, rows_of, lens, heads, d, page, seed=0, tree=False, width=None, sharp=1.5, pad_rows=0, junk=None):
    """A cache that holds the sequences' tokens and their new rows; `junk` fills every slot that no sequence uses."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.RandomState(seed)
    T, (H, Hk), t = sum(rows_of) + pad_rows, heads, TYPES[dtype]
    need = [max(1, -(-(r + n) // page)) for r, n in zip(rows_of, lens)]
    n_pages = sum(need) + 2
    order = rng.permutation(n_pages)
    pages = np.full((len(lens), width or max(need)), -1, np.int32)
    k = torch.randn(n_pages, Hk, page, d, generator=g)
    v = torch.randn(n_pages, Hk, page, d, generator=g)
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    at = 0
    for s, n in enumerate(need):
        pages[s, :n] = order[at:at + n]
        for c in range(rows_of[s] + lens[s]):
            used[pages[s, c // page], c % page] = True
        at += n
    if junk is not None:
        for x in (k, v):
            x.masked_fill_(~used[:, None, :, None], junk)
    words = (max(rows_of) + 31) // 32
    sees, mask = None, None
    if tree:
        sees = np.zeros((T, 32 * words), bool)
        mask = torch.zeros(T, words, dtype=torch.int32)
        r = 0
        for n in rows_of:
            parents = [int(rng.randint(-1, i)) if rng.rand() < 0.5 else i - 1 for i in range(n)]
            if n:
                w = knn.tree_words(parents, "cpu")
                mask[r:r + n, :w.shape[1]] = w
            r += n
        sees = np.unpackbits(mask.numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
    x = {"q": (torch.randn(T, H, d, generator=g) * sharp).to(t).cuda(), "k_cache": k.to(t).cuda(), "v_cache": v.to(t).cuda(),
         "pages": torch.from_numpy(pages).cuda(),
         "row_offsets": torch.tensor(np.concatenate([[0], np.cumsum(rows_of)]), dtype=torch.int64).cuda(),
         "cache_lens": torch.tensor(lens, dtype=torch.int32).cuda()}
    return x, (None if mask is None else mask.cuda()), sees


NAMES = ("q", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens")


def host(t):
    return t.detach().double().cpu().numpy()


def compare(x, out, lse, sees, scale):
    """Checks out and lse [rows, heads]; returns the oracle's out."""
    q, k, v = (np.nan_to_num(host(x[n]), nan=0.0, posinf=0.0, neginf=0.0) for n in ("q", "k_cache", "v_cache"))
    pages, off, lens = (x[n].cpu().numpy() for n in ("pages", "row_offsets", "cache_lens"))
    want, want_lse = lm.attend(q, k, v, pages, off, lens, scale, sees)
    mass, _ = lm.attend(q, k, np.abs(v), pages, off, lens, scale, sees)  # sum of weight |v|
    live = int(off[-1])
    n = int(max(lens + np.diff(off)))
    # Per element: half a step of the type for the result and, through numerator and sum, for each weight; a score's
    # 32-bit sum of d products is off by (d + 4) 2^-23 |q| |k| scale at most, which scales the weights (twice: numerator
    # and sum), the exponential by 2^-21; sums of n terms by n 2^-23.  Below f16's normal range half a step is 2^-25.
    e = torch.finfo(x["q"].dtype).eps / 2
    d = q.shape[2]
    delta = (d + 4) * 2.0 ** -23 * abs(scale) * np.linalg.norm(q, axis=2).max() * np.linalg.norm(k, axis=3).max() + 2.0 ** -21
    tol = e * (2 * np.abs(want) + mass) + mass * (2 * delta + n * 2.0 ** -23) + 2.0 ** -25
    err = np.abs(host(out) - want)[:live]
    assert np.isfinite(err).all()
    assert (err <= tol[:live]).all(), float((err - tol[:live]).max())
    if lse is not None:
        a, b = host(lse)[:live], want_lse[:live]
        empty = np.isneginf(b)
        assert np.array_equal(empty, np.isneginf(a))
        assert (np.abs(a - b)[~empty] <= e + delta + n * 2.0 ** -23 + 2.0 ** -20 * (1 + np.abs(b[~empty]))).all()
    return want


def check(x, mask=None, sees=None, scale=None, **hints):
    s = 1.0 / x["q"].shape[2] ** 0.5 if scale is None else scale
    out, lse = knn.tree_attention(*[x[n] for n in NAMES], tree_mask=mask, scale=scale, want_lse=True, **hints)
    torch.cuda.synchronize()
    compare(x, out, lse, sees, s)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (6, 2), (4, 4)])
@pytest.mark.parametrize("tree", [False, True])
def test_head_layouts(dtype, d, heads, tree):
    x, mask, sees = batch(dtype, [3, 1, 9, 4], [0, 40, 17, 130], heads, d, 16, seed=d + heads[0], tree=tree)
    check(x, mask, sees)


@pytest.mark.parametrize("length", [0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 63, 127, 128, 129, 255, 256, 257, 511, 700])
@pytest.mark.parametrize("page", [16, 64])
def test_lengths(length, page):
    x, mask, sees = batch("bf16", [1, 2], [length, max(0, length - 1)], (4, 2), 128, page, seed=length)
    check(x)


@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 40, 64, 65, 100, 160])
def test_rows_and_column_tiles(rows):
    for tree in (False, True):
        x, mask, sees = batch("f16", [rows, 1, rows], [50, 3, 0], (8, 2), 64, 32, seed=rows, tree=tree)
        check(x, mask, sees)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 4096])
def test_pages(page):
    x, mask, sees = batch("bf16", [6, 0, 3], [100, 9, 600], (4, 2), 128, page, seed=page, tree=True)
    check(x, mask, sees)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (128, "bf16"), (256, "bf16")])
def test_long_caches_in_ranges(d, dtype):
    # few sequences: many ranges, joined; a sequence far shorter than the bound has ranges without a key
    x, mask, sees = batch(dtype, [5, 2, 1], [5000, 37, 2048], (4, 2), d, 64, seed=d, tree=True)
    check(x, mask, sees)
    x, mask, sees = batch(dtype, [1], [6001], (2, 1), d, 16, seed=d + 1)
    check(x)
    check(x, max_keys=x["pages"].shape[1] * 16)


def test_sharp_and_flat_scores():
    for sharp, scale in ((40.0, None), (0.0, None), (1.0, 0.0), (2.0, -0.5), (8.0, 1.0)):
        x, mask, sees = batch("bf16", [4, 2], [300, 90], (4, 2), 128, 16, seed=7, sharp=sharp)
        check(x, scale=scale)


def test_growing_scores_move_the_reference():
    # the scores rise along the cache, by far more than the slack of the running reference
    x, _, _ = batch("f16", [3], [900], (2, 1), 64, 16, seed=8)
    q = torch.ones_like(x["q"])
    ramp = torch.linspace(-3, 3, 903)
    pages = x["pages"].cpu()
    for c in range(903):
        x["k_cache"][pages[0, c // 16], 0, c % 16] = ramp[c].half()
    x["q"] = q
    check(x, scale=1.0)
    x["k_cache"].neg_()
    check(x, scale=1.0)


def test_rows_that_see_nothing_and_odd_masks():
    x, mask, sees = batch("bf16", [5, 3], [0, 20], (4, 2), 128, 16, seed=9, tree=True)
    mask[0] = 0          # no cached token and no draft: empty
    mask[2] = 0b00011    # not itself
    mask[3] = 0b11111    # later drafts too
    mask[6] = 0          # the cached tokens only
    mask[7] = -1         # bits past the sequence's rows say nothing
    sees = np.unpackbits(mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
    out = check(x, mask, sees)
    assert (out[0] == 0).all()


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), 3e4])
def test_unused_slots_may_hold_anything(junk):
    for lens in ([0, 13], [100, 31], [47, 1000]):
        x, mask, sees = batch("f16", [5, 3], lens, (4, 2), 128, 32, seed=10, tree=True, junk=junk)
        check(x, mask, sees)
        x, mask, sees = batch("bf16", [1, 1], lens, (4, 2), 64, 64, seed=11, junk=junk)
        check(x)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_masked_drafts_may_hold_anything(bad):
    x, mask, sees = batch("bf16", [6], [40], (4, 2), 128, 16, seed=12, tree=True)
    words = knn.tree_words([-1, 0, -1, 2, 0, 3], "cuda")   # 2, 3 and 5 are a branch of their own
    sees = np.unpackbits(words.cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
    page = int(x["pages"][0, 42 // 16])
    for cache in ("k_cache", "v_cache"):
        y = dict(x)
        y[cache] = x[cache].clone()
        y[cache][page, :, 42 % 16, 5] = bad                # draft 2
        out, lse = knn.tree_attention(*[y[n] for n in NAMES], tree_mask=words, want_lse=True)
        clean, lse0 = knn.tree_attention(*[x[n] for n in NAMES], tree_mask=words, want_lse=True)
        torch.cuda.synchronize()
        for r in (0, 1, 4):
            assert torch.equal(out[r], clean[r]) and torch.equal(lse[r], lse0[r])
        if cache == "v_cache":
            for r in (2, 3, 5):
                assert not torch.isfinite(out[r, :, 5]).any()
                assert torch.equal(out[r, :, :5], clean[r, :, :5]) and torch.equal(out[r, :, 6:], clean[r, :, 6:])


def test_entries_that_are_no_page():
    x, mask, sees = batch("bf16", [4, 2], [100, 40], (4, 2), 64, 16, seed=13, tree=True)
    pages = x["pages"].clone()
    pages[0, 2] = -1
    pages[1, 0] = x["k_cache"].shape[0]
    pages[0, 5] = 1 << 30
    x["pages"] = pages
    check(x, mask, sees)
    pages[:] = -1        # no key at all
    out = check(x, mask, sees)
    assert (out == 0).all()


@pytest.mark.parametrize("S", [63, 64, 65, 130, 200])
@pytest.mark.parametrize("most", [60, 1500])
def test_many_sequences(S, most):
    rng = np.random.RandomState(S + most)
    lens = [int(x) for x in rng.randint(0, most, S)]
    rows = [int(x) for x in rng.choice([0, 1, 1, 2, 5], S)]
    rows[0] = rows[-1] = 0
    lens[S // 2] = most * 3
    x, mask, sees = batch("bf16", rows, lens, (4, 2), 64, 32, seed=S, tree=True)
    check(x, mask, sees)


def test_bounds_on_either_side_of_parting():
    # a head of up to 256 keys has one workgroup, a longer one parts of several; the bound decides, not the lengths
    x, mask, sees = batch("f16", [9, 2], [247, 100], (8, 2), 128, 32, seed=40, tree=True, width=40)
    a = check(x, mask, sees, max_keys=256)
    b = check(x, mask, sees, max_keys=288)
    assert (a - b).abs().max() < 0.02
    for keys in (255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2049):
        x, mask, sees = batch("bf16", [1, 3], [keys - 1, 5], (4, 4), 64, 64, seed=keys)
        check(x)


def test_strides_of_queries():
    x, _, _ = batch("bf16", [3, 2], [40, 100], (8, 2), 128, 16, seed=14)
    want = check(x)
    wide = torch.zeros(5, 12, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10] = x["q"]
    assert torch.equal(check(dict(x, q=wide[:, 2:10])), want)
    assert torch.equal(check(dict(x, q=x["q"].transpose(0, 1).contiguous().transpose(0, 1))), want)


def test_rows_behind_the_last_sequence_stay():
    x, _, _ = batch("f16", [3, 0, 2], [40, 5, 3000], (4, 2), 64, 16, seed=15, pad_rows=4)
    out = torch.full_like(x["q"], 7.0)
    lse = torch.full((9, 4), 5.0, device="cuda")
    knn.tree_attention(*[x[n] for n in NAMES], max_rows=3, max_keys=3002, out=out, lse=lse)
    torch.cuda.synchronize()
    compare(x, out, lse, None, 1 / 8)
    assert (out[5:] == 7.0).all() and (lse[5:] == 5.0).all()


def test_repeats_are_the_same_bits_on_any_stream():
    x, mask, _ = batch("bf16", [16, 3, 9], [4000, 100, 777], (8, 2), 128, 16, seed=16, tree=True)
    call = knn.TreeAttention(*[x[n] for n in NAMES], tree_mask=mask)
    first = call.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = knn.TreeAttention(*[x[n] for n in NAMES], tree_mask=mask)
    for _ in range(3):  # two calls at once, each with its workspace
        a = call.run()
        b = other.run(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(a, first) and torch.equal(b, first)


def test_graph_replays_on_new_lengths():
    x, mask, _ = batch("bf16", [4, 4], [3000, 2500], (4, 2), 128, 64, seed=17, tree=True)
    call = knn.TreeAttention(*[x[n] for n in NAMES], max_keys=3004, tree_mask=mask)
    call.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    for lens in ([3000, 1], [0, 2999], [63, 64], [1200, 700]):
        x["cache_lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        x["q"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = call.out.clone()
        call.out.zero_()
        assert torch.equal(call.run(), got)
        torch.cuda.synchronize()
    sees = np.unpackbits(mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
    compare(x, call.out, None, sees, 128 ** -0.5)


def test_cache_past_32_bit_offsets():
    page, d, Hk = 64, 128, 8
    n_pages = (5 << 30) // (Hk * page * d * 2)  # 5 GiB a cache
    x, _, _ = batch("bf16", [3, 1], [200, 60], (8, 8), d, page, seed=18)
    small_k, small_v, pages = x["k_cache"], x["v_cache"], x["pages"].clone()
    n = small_k.shape[0]
    k, v = (torch.empty(n_pages, Hk, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[-n:], v[-n:] = small_k, small_v
    want = check(x)
    got = knn.tree_attention(x["q"], k, v, torch.where(pages >= 0, pages + (n_pages - n), pages), x["row_offsets"],
                             x["cache_lens"])
    torch.cuda.synchronize()
    assert torch.equal(want, got)


def test_refusals():
    x, mask, _ = batch("bf16", [2, 2], [10, 40], (4, 2), 128, 16, seed=19, tree=True)
    args = dict((n, x[n]) for n in NAMES)
    for bad in (dict(q=x["q"].float()), dict(q=x["q"][:, :, :64]), dict(pages=x["pages"].long()),
                dict(cache_lens=x["cache_lens"][:1]), dict(q=x["q"].cpu()), dict(v_cache=x["v_cache"].half()),
                dict(tree_mask=mask.long()), dict(tree_mask=mask[:2]), dict(out=x["q"].half()),
                dict(lse=torch.zeros(3, 4, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            knn.tree_attention(**dict(args, **bad))
    for bad in (dict(q=x["q"][:, :3]), dict(max_rows=5), dict(max_keys=10 ** 6), dict(scale=float("nan")),
                dict(max_rows=0), dict(max_keys=0)):
        with pytest.raises(knn.KnnError):
            knn.tree_attention(**dict(args, **bad))
    odd = torch.zeros(4, 4, 136, dtype=torch.bfloat16, device="cuda")[:, :, 4:132]
    with pytest.raises(knn.KnnError):
        knn.tree_attention(**dict(args, q=odd))


@pytest.mark.parametrize("length", [3, 300])
def test_scores_far_below_zero(length):
    """Equal scores of -64 * 1e32 / 8: the weights are equal however low they are, and the mean is exact (of ones)."""
    x, _, _ = batch("bf16", [1], [length], (2, 1), 64, 16, seed=3)
    x["q"].fill_(1e16)
    x["k_cache"].fill_(-1e16)
    x["v_cache"].fill_(1.0)
    out, lse = knn.tree_attention(*[x[n] for n in NAMES], want_lse=True)
    assert (out == 1.0).all()
    score = -64 * float(torch.tensor(1e16).bfloat16()) ** 2 / 8
    assert (lse.double() / score - 1).abs().max() < 70 * 2.0 ** -23  # a 32-bit sum of 64 products


@pytest.mark.parametrize("heads", [(4, 2), (32, 2)])
def test_hints_that_are_too_low_leave_out(heads):
    """Sequence 0 has more rows and keys than the hints say: its first rows see the first keys, its others stay."""
    x, _, _ = batch("f16", [5, 3], [100, 40], heads, 64, 16, seed=12)
    out = torch.full((x["q"].shape[0], heads[0], 64), 7.0, dtype=torch.float16, device="cuda")
    knn.tree_attention(*[x[n] for n in NAMES], max_rows=4, max_keys=64, out=out)
    short = dict(x, cache_lens=torch.tensor([64, 40], dtype=torch.int32, device="cuda"))
    none = torch.zeros(8, 1, dtype=torch.int32, device="cuda")  # of sequence 0 no draft is seen, so 64 keys are
    none[5:] = knn.tree_words([-1, 0, 1], "cuda")
    want = knn.tree_attention(*[short[n] for n in NAMES], tree_mask=none)
    live = [0, 1, 2, 3, 5, 6, 7]
    # the same sums in another order: half a step for each result and its weights, twice
    assert ((out - want).float()[live].abs() <= 4 * 2.0 ** -11 * (1 + want.float()[live].abs().max())).all()
    assert (out[4] == 7.0).all()


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("length", [200, 3001])
@pytest.mark.parametrize("heads,rows,d", [((2, 1), 3, 64), ((16, 2), 3, 128), ((32, 2), 3, 128), ((32, 1), 4, 64),
                                          ((8, 2), 3, 256), ((32, 2), 5, 256)])
def test_values_that_are_not_finite_make_nan_what_sees_them(bad, dtype, length, heads, rows, d):
    """Of heavy keys and of such as weigh nothing, in tiles that every row sees and in the last ones, and of a draft that
    only the last row sees; every other element is what it was."""
    x, _, _ = batch(dtype, [rows], [length], heads, d, 16, seed=21)
    pages = x["pages"].cpu()

    def slot(c):
        return int(pages[0, c // 16]), slice(None), c % 16

    x["q"] = x["q"].abs()
    light = [37, length - 2]
    for c in light:
        x["k_cache"][slot(c)] = -200.0  # scores under -200 for positive q of this size: weights of 0
    cells = {40: 5, length - 3: 6, light[0]: 7, light[1]: 40, length + rows - 1: 60}  # key: the element of its value
    clean, lse0 = knn.tree_attention(*[x[n] for n in NAMES], want_lse=True)
    for c, e in cells.items():
        x["v_cache"][slot(c) + (e,)] = bad
    out, lse = knn.tree_attention(*[x[n] for n in NAMES], want_lse=True)
    torch.cuda.synchronize()
    want = torch.zeros_like(out, dtype=torch.bool)
    for c, e in cells.items():
        want[max(0, c - length):, :, e] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want], clean[~want]) and torch.equal(lse, lse0)


@pytest.mark.parametrize("rows,heads", [(1, (8, 8)), (5, (64, 8))])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_long_flat_tail_behind_one_heavy_key(rows, heads, dtype):
    """The first key's score is 17, those of the 32,767 behind it are 0: each weighs 2^-24.5 of the first.  f16 holds them
    to 2^-32 of the largest, so that all together are off by 2^-17; half a step of the type for each weight and the result
    and the 32-bit sums (2^-23 a term, of a mass of 2^-9) come on top.

    The weights' own sum lies between 1 and 2, where a step of fp32 is 2^-23, and grows by 32 keys at a time, a wave's
    quarter of the keys at one row and all of them at 40 columns: 256 and 1,024 sums that are each off by up to a step,
    which the logarithm of a number over 1 takes on as they are."""
    S, n, d, page = 64, 32768, 64, 128
    k = torch.zeros(2, heads[1], page, d, dtype=TYPES[dtype], device="cuda")
    v = torch.ones_like(k)
    k[0, :, 0], v[0, :, 0] = 2.125, 0.0
    q = torch.ones(S * rows, heads[0], d, dtype=k.dtype, device="cuda")
    pages = torch.ones(S, n // page + 1, dtype=torch.int32, device="cuda")
    pages[:, 0] = 0                                    # a page of ones and zeros is all the others
    off = torch.arange(S + 1, device="cuda") * rows
    lens = torch.full((S,), n, dtype=torch.int32, device="cuda")
    none = torch.zeros(S * rows, 1, dtype=torch.int32, device="cuda")
    out, lse = knn.tree_attention(q, k, v, pages, off, lens, tree_mask=none, want_lse=True)
    mass = (n - 1) * np.exp(-17.0)
    want, e = mass / (1 + mass), torch.finfo(k.dtype).eps / 2
    assert (out.double() - want).abs().max() <= 3 * e * want + 2.0 ** -16
    sums = n // 32 // (4 if rows == 1 else 1)
    assert (lse.double() - 17.0 - np.log1p(mass)).abs().max() <= e * mass + 2.0 ** -16 + 18 * 2.0 ** -22 + sums * 2.0 ** -23


@pytest.mark.parametrize("tree", [False, True])
def test_calls_without_hints_follow_lengths_and_rows(tree):
    """One object, made when the sequences were short, on the tensors' contents of later steps: longer caches, and rows that
    went from one sequence to the other."""
    x, mask, sees = batch("bf16", [2, 2], [30, 40], (4, 2), 64, 16, seed=22, width=8, tree=tree)
    g = torch.Generator().manual_seed(1)
    x["k_cache"], x["v_cache"] = (torch.randn(16, 2, 16, 64, generator=g).bfloat16().cuda() for _ in range(2))
    x["pages"] = torch.randperm(16, generator=g).view(2, 8).int().cuda()
    call = knn.TreeAttention(*[x[n] for n in NAMES], tree_mask=mask, want_lse=True)
    for lens, off in (([30, 40], [0, 2, 4]), ([31, 41], [0, 2, 4]), ([126, 3], [0, 2, 4]), ([5, 125], [0, 1, 4]),
                      ([70, 80], [0, 4, 4]), ([124, 0], [0, 4, 4]), ([0, 0], [0, 0, 4])):
        x["cache_lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        x["row_offsets"].copy_(torch.tensor(off))
        call.run()
        torch.cuda.synchronize()
        compare(x, call.out, call.lse, sees, 1 / 8)


@pytest.mark.parametrize("rows,heads,strides", [(1, (4, 2), (333, 64)), (3, (1, 1), (64, 77)), (1, (1, 1), (13, 7))])
def test_strides_of_a_single_row_or_head_say_nothing(rows, heads, strides):
    x, _, _ = batch("bf16", [rows], [90], heads, 64, 16, seed=23)
    want = check(x)
    q = torch.zeros(2000, dtype=torch.bfloat16, device="cuda").as_strided((rows, heads[0], 64), (*strides, 1))
    q.copy_(x["q"])
    assert torch.equal(check(dict(x, q=q)), want)


def some_rows(x, out, lse, rows, scale):
    """Chains: these rows alone against the oracle, each as a sequence of its own on the tokens before it."""
    off, lens = x["row_offsets"].cpu(), x["cache_lens"].cpu()
    seq = torch.searchsorted(off, torch.tensor(rows), right=True) - 1
    at = torch.tensor(rows)
    y = dict(x, q=x["q"][rows], pages=x["pages"][seq.cuda()], row_offsets=torch.arange(len(rows) + 1),
             cache_lens=(lens[seq] + at - off[seq]).int())
    compare(y, out[rows], lse[rows], None, scale)


@pytest.mark.parametrize("dtype,rows,lens,heads,d", [
    ("bf16", [1100], [0], (64, 1), 128),            # 550 column tiles on one key head: parts in two launches
    ("f16", [1030, 40, 0], [10, 700, 3], (64, 1), 128),
    ("bf16", [1, 1, 1020, 2, 1, 1, 1, 1, 1], [9000, 7, 100, 30, 0, 63, 64, 65, 900], (64, 1), 128),
    ("bf16", [600], [301], (64, 1), 128),           # parts in one
    ("f16", [2100], [0], (16, 1), 256),             # the same at 64 columns
    ("bf16", [1100, 7], [0, 40], (64, 2), 64),
    ("bf16", [3, 520, 1, 0, 270, 1, 1, 2], [900, 0, 64, 5, 300, 0, 7, 3000], (64, 1), 128),  # eight heads: none parted
    ("bf16", [1] * 40 + [505] + [2] * 30, [77] * 71, (64, 1), 128),
    ("bf16", [2000], [0], (8, 8), 128),
    ("f16", [1500, 700], [0, 1000], (8, 2), 128),
    ("bf16", [1030], [1000], (64, 8), 64),
    ("f16", [1030, 1], [0, 200], (64, 4), 256)])
def test_prompts(dtype, rows, lens, heads, d):
    x, _, _ = batch(dtype, rows, lens, heads, d, 64, seed=sum(rows))
    out, lse = torch.full_like(x["q"], 7.0), torch.full((sum(rows), heads[0]), 5.0, device="cuda")
    knn.tree_attention(*[x[n] for n in NAMES], out=out, lse=lse)
    torch.cuda.synchronize()
    T = sum(rows)
    some_rows(x, out, lse, sorted({int(i) for i in np.linspace(0, T - 1, 17)} | {T // 2 - 1, T // 2 + 1}), d ** -0.5)
    # every row was written: its largest weighted value is none of the constants
    assert torch.isfinite(lse).all() and not (out == 7.0).all(2).any() and not (lse == 5.0).any()


@pytest.mark.parametrize("most", [60, 700])
def test_rows_that_cannot_fill_what_max_rows_asks_for(most):
    """Many sequences of few rows and no bound on them: a head is not parted then, whatever its keys."""
    S = 200
    rng = np.random.RandomState(most)
    lens = [int(n) for n in rng.randint(0, most, S)]
    rows = [int(n) for n in rng.choice([0, 1, 1, 2, 3], S)]
    lens[S // 2], rows[7] = most * 3, 150
    x, mask, sees = batch("bf16", rows, lens, (8, 4), 64, 32, seed=S + most, tree=True)
    call = knn.TreeAttention(*[x[n] for n in NAMES], tree_mask=mask, want_lse=True)
    assert call.workspace.numel() == 256
    call.run()
    torch.cuda.synchronize()
    compare(x, call.out, call.lse, sees, 1 / 8)
