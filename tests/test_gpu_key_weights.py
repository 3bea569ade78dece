"""Weights of cached keys on the GPU against the fp64 oracle: head layouts, ragged rows and lengths, trees, accepted paths,
strides, pages, rows that see nothing, and what has to stay as it was."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def ints(t):
    return None if t is None else t.cpu().numpy()


def offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int64).cuda()


def batch(dtype, rows_of, lens, heads, d, page, seed=0, width=None, tree=False, path=False, extra_rows=0):
    """The tensors of a call: caches whose unused places hold NaN, and sums as attention gives them (from the oracle)."""
    g = torch.Generator().manual_seed(seed)
    T, (H, Hk) = sum(rows_of), heads
    need = [max(1, -(-(r + n) // page)) for r, n in zip(rows_of, lens)]
    width = width or max(need)
    n_pages = sum(need) + 2
    order = torch.randperm(n_pages, generator=g)
    pages = torch.full((len(lens), width), -7, dtype=torch.int32)
    k = torch.full((n_pages, Hk, page, d), float("nan"))
    at = 0
    for s, n in enumerate(need):
        pages[s, :n] = order[at:at + n].int()
        at += n
        for c in range(rows_of[s] + lens[s]):
            k[int(pages[s, c // page]), :, c % page] = torch.randn(Hk, d, generator=g)
    source = 2 * T + 3 if path else T + extra_rows
    x = {"q": (1.5 * torch.randn(source, H, d, generator=g)).to(TYPES[dtype]).cuda(), "k_cache": k.to(TYPES[dtype]).cuda(),
         "pages": pages.cuda(), "row_offsets": offsets(rows_of), "cache_lens": torch.tensor(lens, dtype=torch.int32).cuda(),
         "mass": torch.rand(n_pages, Hk, page, generator=g).cuda(), "tree_mask": None, "source_rows": None,
         "key_positions": torch.randint(0, 99, (n_pages, Hk, page), generator=g, dtype=torch.int32).cuda(),
         "positions": torch.randint(0, 10 ** 6, (T + (0 if path else extra_rows),), generator=g, dtype=torch.int32).cuda(),
         "lse": torch.randn(source, H, generator=g).cuda()}
    if tree:
        masks = [knn.tree_words([int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)], "cpu")
                 for n in rows_of]
        words = max(1, max(m.shape[1] for m in masks))
        x["tree_mask"] = torch.cat([torch.nn.functional.pad(m, (0, words - m.shape[1])) for m in masks] + [
            torch.full((0 if path else extra_rows, words), -1, dtype=torch.int32)]).cuda()
    if path:
        x["source_rows"] = torch.randperm(source, generator=g)[:T].int().cuda()
    # what attention says of these rows, from the rows as they are read
    rows = host(x["q"]) if not path else host(x["q"])[ints(x["source_rows"])]
    _, lse = lm.attend(rows, np.nan_to_num(host(x["k_cache"])), np.zeros(k.shape), ints(x["pages"]),
                       ints(x["row_offsets"]), ints(x["cache_lens"]), d ** -0.5, sees(x))
    if T:
        where = torch.arange(T) if not path else x["source_rows"].cpu().long()
        x["lse"][where.cuda()] = torch.from_numpy(lse[:T]).float().cuda()
    return x


def sees(x):
    if x["tree_mask"] is None:
        return None
    return np.unpackbits(ints(x["tree_mask"]).view(np.uint8), axis=1, bitorder="little").astype(bool)


def want_of(x, scale=None, decay=1.0, source_rows=None):
    """The oracle's (mass, key_positions) and how far mass may be off."""
    d = x["q"].shape[2]
    mass, where, terms = lm.key_weights(
        host(x["q"]), host(x["lse"]), host(x["k_cache"]), ints(x["pages"]), ints(x["row_offsets"]), ints(x["cache_lens"]),
        host(x["mass"]), d ** -0.5 if scale is None else scale, decay, sees(x), ints(x["source_rows"]),
        ints(x["key_positions"]), ints(x["positions"]))
    # Of a weight exp(x - lse): the sum of d products in 32 bits is off by at most d 2^-23 sum |q k| whatever its order
    # and whether its steps round or cut; x, lse, the change to powers of two and their difference by 4 roundings of |x| +
    # |lse|; exp2 by 2^-22.  A sum of n weights, and the share of the mass before, by n 2^-24 and 2^-23 of it.
    n = x["row_offsets"].diff().max().item() * (x["q"].shape[1] // x["k_cache"].shape[1]) + 4
    return mass, where, 2.0 ** -22 * terms + (n * 2.0 ** -24 + 2.0 ** -22) * np.abs(mass) + 1e-30


def check(x, decay=1.0, scale=None, hints=True, **over):
    x = dict(x, **over)
    want, where, tol = want_of(x, scale, decay)
    more = {}
    if hints:
        count = x["row_offsets"].diff()
        more = dict(max_rows=max(1, int(count.max())), max_keys=max(1, int((x["cache_lens"] + count).max())))
    got = knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"],
                          key_positions=x["key_positions"], positions=x["positions"], source_rows=x["source_rows"],
                          tree_mask=x["tree_mask"], scale=scale, decay=decay, **more)
    torch.cuda.synchronize()
    assert got is x["mass"]
    err = np.abs(host(got) - want)
    assert (err <= tol).all(), float(np.nanmax(err - tol))  # (a NaN is no less)
    assert np.array_equal(ints(x["key_positions"]), where)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (8, 2), (16, 1), (10, 2)])
def test_decoding_over_ragged_lengths(dtype, d, heads):
    check(batch(dtype, [1, 1, 1, 1, 1], [0, 1, 15, 300, 77], heads, d, 16, seed=d))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("form", ["chain", "tree", "path", "tree path"])
def test_rows_of_drafts(dtype, page, form):
    x = batch(dtype, [3, 0, 17, 40, 1], [0, 33, 100, 250, 511], (8, 2), 128, page, seed=page, tree="tree" in form,
              path="path" in form)
    check(x, decay=0.75)


@pytest.mark.parametrize("heads,rows", [((64, 8), [64, 5]), ((32, 1), [9, 70]), ((6, 3), [130, 1])])
def test_many_columns(heads, rows):
    check(batch("bf16", rows, [500, 9], heads, 128, 16, seed=7))
    check(batch("f16", rows, [31, 257], heads, 64, 32, seed=8, tree=True))


def test_long_lengths():
    check(batch("bf16", [2, 1], [5000, 1], (4, 1), 64, 64, seed=3), decay=0.5)


def test_without_hints_and_a_wide_table():
    check(batch("bf16", [2, 5], [40, 3], (4, 2), 64, 16, seed=4, width=60), hints=False)
    check(batch("bf16", [2, 5], [40, 3], (4, 2), 64, 16, seed=4, width=60, tree=True), hints=False)


def test_rows_behind_the_last_sequence_and_sequences_without_rows():
    x = batch("bf16", [2, 0, 3], [40, 50, 0], (4, 2), 64, 16, seed=5, extra_rows=4)
    x["q"][5:] = float("nan")
    check(x)


def test_decay_of_zero_reads_no_mass():
    x = batch("f16", [1, 2], [40, 60], (4, 2), 64, 16, seed=6)
    used = torch.zeros_like(x["mass"], dtype=torch.bool)
    for s, n in enumerate((41, 62)):
        for c in range(n):
            used[int(x["pages"][s, c // 16]), :, c % 16] = True
    x["mass"][used] = float("nan")
    check(x, decay=0.0)
    y = batch("f16", [1, 2], [40, 60], (4, 2), 64, 16, seed=6)
    for s, (n, r) in enumerate(((40, 1), (60, 2))):  # the rows' own places are set, whatever they held
        for c in range(n, n + r):
            y["mass"][int(y["pages"][s, c // 16]), :, c % 16] = float("nan")
    check(y)


def test_scales():
    for scale in (0.0, -0.2, 1.0):
        x = batch("bf16", [2, 1], [40, 60], (4, 2), 64, 16, seed=9)
        _, lse = lm.attend(host(x["q"]), np.nan_to_num(host(x["k_cache"])), np.zeros(x["k_cache"].shape), ints(x["pages"]),
                           ints(x["row_offsets"]), ints(x["cache_lens"]), scale)
        x["lse"].copy_(torch.from_numpy(lse).float())
        check(x, scale=scale)


def test_rows_that_saw_nothing_or_are_left_out_add_nothing():
    x = batch("bf16", [3, 2], [40, 0], (4, 2), 64, 16, seed=10)
    x["lse"][0, :] = float("-inf")
    x["lse"][1, 2] = float("nan")
    x["lse"][3, 1] = float("inf")
    x["q"][0] = float("nan")
    want = want_of(dict(x, q=torch.nan_to_num(x["q"])))
    knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"])
    assert (np.abs(host(x["mass"]) - want[0]) <= want[2]).all()
    x = batch("bf16", [3, 2], [40, 0], (4, 2), 64, 16, seed=11, path=True)
    x["source_rows"][:] = torch.tensor([-1, 4, x["q"].shape[0], 1 << 30, -(1 << 31)], dtype=torch.int32)
    check(x, decay=0.5)


def test_masked_drafts_may_hold_anything():
    """Rows that see neither their own key nor each other's: those keys hold NaN and get the weight of nobody."""
    x = batch("bf16", [4, 33], [40, 5], (4, 2), 64, 16, seed=12, tree=True)
    x["tree_mask"][:] = 0
    x["tree_mask"][1, 0] = 0b0001  # one row sees the first draft
    for s, (n, r) in enumerate(((40, 4), (5, 33))):
        for c in range(n + (s == 0), n + r):
            x["k_cache"][int(x["pages"][s, c // 16]), :, c % 16] = float("nan")
    k = torch.nan_to_num(x["k_cache"])
    want, where, tol = want_of(dict(x, k_cache=k))
    knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"],
                    tree_mask=x["tree_mask"])
    assert (np.abs(host(x["mass"]) - want) <= tol).all()


def test_a_sequence_with_no_tokens_but_masked_ones():
    x = batch("bf16", [1, 3], [0, 0], (4, 2), 64, 16, seed=13, tree=True)
    x["tree_mask"][:] = 0
    x["lse"][:] = float("-inf")
    check(x)
    assert x["mass"][int(x["pages"][0, 0]), :, 0].abs().max() == 0


def test_entries_that_are_no_page():
    x = batch("bf16", [2, 20], [40, 100], (4, 2), 64, 16, seed=14)
    x["pages"][0, 1], x["pages"][1, 2], x["pages"][1, 7] = -1, x["k_cache"].shape[0], 1 << 30
    check(x)


def test_strides_of_projections():
    x = batch("bf16", [2, 7], [40, 100], (4, 2), 64, 16, seed=15)
    wide = torch.full((9, 4 + 5, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:7] = x["q"]
    check(x, q=wide[:, 3:7])
    x = batch("bf16", [2, 7], [40, 100], (4, 2), 64, 16, seed=15)
    turned = x["q"].transpose(0, 1).contiguous().transpose(0, 1)  # heads outside, rows inside
    check(x, q=turned)
    x = batch("bf16", [1], [40], (4, 2), 64, 16, seed=16)
    check(x, q=torch.as_strided(x["q"], (1, 4, 64), (4 * 64 + 3, 64, 1)))  # the stride of a single row says nothing


def test_far_pages_of_a_large_cache():
    """Offsets past 2^32 bytes of keys, and past 2^31 elements."""
    n_pages, Hk, page, d = 40000, 2, 256, 128  # 2.6e9 elements
    x = batch("bf16", [2, 1], [300, 700], (4, Hk), d, page, seed=17)
    k = torch.zeros(n_pages, Hk, page, d, dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros(n_pages, Hk, page, device="cuda")
    move = n_pages - x["k_cache"].shape[0]
    k[move:], mass[move:] = x["k_cache"], x["mass"]
    want, _, tol = want_of(x)
    pages = torch.where(x["pages"] >= 0, x["pages"] + move, x["pages"])
    knn.key_weights(x["q"], x["lse"], k, pages, x["row_offsets"], x["cache_lens"], mass, max_rows=2, max_keys=701)
    assert (np.abs(host(mass[move:]) - want) <= tol).all() and float(mass[:move].abs().max()) == 0


def test_hints_that_are_too_low_leave_keys_out_and_stay_inside():
    x = batch("bf16", [2, 7], [40, 100], (4, 2), 64, 16, seed=18)
    before = x["mass"].clone()
    knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"], max_rows=3,
                    max_keys=50)
    torch.cuda.synchronize()
    for c in range(50, 107):
        at = (int(x["pages"][1, c // 16]), slice(None), c % 16)
        assert torch.equal(x["mass"][at], before[at])


def test_the_same_bits_every_time_and_in_a_graph():
    x = batch("bf16", [5, 1, 9], [400, 30, 1000], (16, 2), 128, 64, seed=19)
    first = x["mass"].clone()
    call = knn.KeyWeights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"],
                          decay=0.5)
    want = []
    for _ in range(3):
        call.run()
        want.append(x["mass"].clone())
    x["mass"].copy_(first)
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call.run()
    x["mass"].copy_(first)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x["mass"], want[i])
    # other lengths in the same buffers
    x["cache_lens"].sub_(7)
    expect, _, tol = want_of(dict(x, key_positions=None, positions=None), decay=0.5)
    graph.replay()
    assert (np.abs(host(x["mass"]) - expect) <= tol).all()


def test_argument_checks():
    x = batch("bf16", [2], [40], (4, 2), 64, 16)
    args = dict(q=x["q"], lse=x["lse"], k_cache=x["k_cache"], pages=x["pages"], row_offsets=x["row_offsets"],
                cache_lens=x["cache_lens"], mass=x["mass"])
    for over in (dict(lse=x["lse"].double()), dict(lse=x["lse"][:1]), dict(mass=x["mass"][:1]), dict(q=x["q"].half()),
                 dict(positions=x["positions"]), dict(key_positions=x["mass"]), dict(pages=x["pages"][0]),
                 dict(source_rows=x["positions"].long()), dict(mass=x["mass"].cpu()), dict(tree_mask=x["pages"][:, :1])):
        with pytest.raises(ValueError):
            knn.key_weights(**dict(args, **over))
    with pytest.raises(knn.KnnError):
        knn.key_weights(**dict(args, decay=-1.0))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_column_counts_of_every_kernel(dtype, d):
    """1 to 16, 32, 96 columns by waves of their own, then four, eight and sixteen waves a workgroup; more columns than LDS
    holds in rounds."""
    for rows, heads in (([2, 5], (8, 2)), ([4, 1], (16, 2)), ([12, 7], (16, 2)), ([13], (16, 2)), ([31, 2], (8, 2)),
                        ([50, 9], (16, 2)), ([70, 3], (16, 2)), ([150], (16, 2))):
        check(batch(dtype, rows, [300, 77][:len(rows)], heads, d, 32, seed=d + rows[0]), decay=0.5)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("tree", [False, True])
def test_column_counts_under_high_hints(d, tree):
    """As many columns in calls that may have many tiles, which waves do not share."""
    for rows, heads in (([13], (16, 2)), ([31, 2], (8, 2)), ([50, 9], (16, 2)), ([70, 3], (16, 2)), ([150], (16, 2))):
        x = batch("bf16", rows, [300, 77][:len(rows)], heads, d, 32, seed=d + rows[0], width=30000, tree=tree)
        check(x, decay=0.5, hints=False)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_whose_columns_waves_share(d):
    """More tiles than workgroups, from one a workgroup to more than it has waves."""
    check(batch("bf16", [40] * 9, [1300, 1700, 60, 1999, 1111, 900, 1500, 2, 1700], (32, 2), d, 16, seed=d), decay=0.5)
    check(batch("f16", [64, 3], [4000, 0], (12, 1), d, 64, seed=d + 1, tree=True))
    x = batch("bf16", [40] * 5, [700, 900, 1, 500, 300], (64, 8), d, 16, seed=d + 2, path=True)
    x["pages"][1, 20] = x["pages"][3, 0] = -1
    check(x)


def test_many_sequences():
    """More than a wave's lanes and than a workgroup's threads, some without rows or tokens."""
    g = np.random.RandomState(3)
    for n, rows in ((150, 2), (700, 1), (300, 20)):
        lens = g.randint(0, 40, n).tolist()
        rows_of = g.randint(0, rows + 1, n).tolist()
        rows_of[-1] = rows
        check(batch("bf16", rows_of, lens, (8, 2), 64, 16, seed=n))


def test_keys_that_are_not_finite_and_seen():
    """An infinite element of a cached key: its own mass is no number, every other key's is as it would be."""
    for rows, heads in (([1, 2], (4, 2)), ([40, 3], (16, 2))):
        x = batch("bf16", rows, [100, 60], heads, 64, 16, seed=20)
        want, _, tol = want_of(x)
        at = (int(x["pages"][0, 3]), 1, 5)  # cache index 53 of the first sequence
        x["k_cache"][at] = float("nan")
        knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"])
        got = host(x["mass"])
        assert np.isnan(got[at])
        want[at] = got[at] = 0.0
        assert (np.abs(got - want) <= tol).all()


def test_nobody_adds_to_keys_that_are_not_finite():
    """Rows whose sums are not finite add nothing, also to keys that are not."""
    for rows, heads in (([1, 2], (4, 2)), ([40, 3], (16, 2))):
        x = batch("f16", rows, [100, 60], heads, 64, 16, seed=21)
        x["lse"][:] = float("-inf")
        x["k_cache"][:] = float("inf")
        check(x, decay=0.5)


def test_on_another_stream():
    x = batch("bf16", [2, 5], [400, 100], (8, 2), 128, 16, seed=22)
    want, _, tol = want_of(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = knn.KeyWeights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"])
    call.run(side)
    side.synchronize()
    assert (np.abs(host(x["mass"]) - want) <= tol).all()


@pytest.mark.parametrize("heads", [(1, 1), (112, 1)])
def test_the_longest_length(heads):
    """2^31 - 1 keys, all but the last page's of two pages that the table names again and again."""
    page, total, H = 1024, 2 ** 31 - 1, heads[0]
    g = torch.Generator().manual_seed(21)
    k = torch.randn(3, 1, page, 64, generator=g).bfloat16().cuda()
    q = torch.randn(1, H, 64, generator=g).bfloat16().cuda()
    lse = (torch.rand(1, H, generator=g) + 3.0).cuda()
    pages = torch.zeros(1, total // page + 1, dtype=torch.int32).cuda()
    pages[:, 1::2] = 1
    pages[:, -1] = 2
    mass = torch.rand(3, 1, page, generator=g).cuda()
    before = mass.clone()
    positions = torch.full((3, 1, page), -5, dtype=torch.int32).cuda()
    knn.key_weights(q, lse, k, pages, offsets([1]), torch.tensor([total - 1], dtype=torch.int32).cuda(), mass, max_rows=1,
                    max_keys=total, key_positions=positions, decay=0.0)
    x, size = host(k)[:, 0] @ host(q)[0].T / 8.0, np.abs(host(k)[:, 0]) @ np.abs(host(q)[0]).T / 8.0  # [pages, page, heads]
    weights = np.exp(x - host(lse)[0])
    want = weights.sum(-1)
    # (as in want_of)
    off = (weights * (64 * 2.0 ** -23 * size + 2.0 ** -22 * (np.abs(x) + np.abs(host(lse)[0]) + 1))).sum(-1)
    off += (H + 4) * 2.0 ** -24 * want
    assert np.all(np.abs(host(mass)[:2, 0] - want[:2]) <= off[:2])
    assert np.all(np.abs(host(mass)[2, 0, :-1] - want[2, :-1]) <= off[2, :-1])
    assert float(mass[2, 0, -1]) == float(before[2, 0, -1])
    assert int(positions[2, 0, -2]) == total - 1 and int((positions == -5).sum()) == 3 * page - 1


def test_masks_without_words_are_refused():
    """A mask with no bit for any row is none, where the call without one would be a chain's."""
    x = batch("bf16", [2, 1], [40, 5], (4, 2), 64, 16)
    none = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    rows = dict(pages=x["pages"], row_offsets=x["row_offsets"], cache_lens=x["cache_lens"], tree_mask=none, max_rows=2,
                max_keys=64)
    before = x["mass"].clone()
    with pytest.raises(ValueError):
        knn.key_weights(x["q"], x["lse"], x["k_cache"], mass=x["mass"], **rows)
    with pytest.raises(ValueError):
        knn.tree_attention(x["q"], x["k_cache"], x["k_cache"].clone(), **rows)
    with pytest.raises(ValueError):
        knn.adjust_scores(torch.zeros(3, 10, device="cuda"), row_offsets=x["row_offsets"], tree_mask=none,
                          row_tokens=torch.zeros(3, dtype=torch.int32, device="cuda"),
                          presence=torch.ones(3, device="cuda"))
    assert torch.equal(x["mass"], before)


@pytest.mark.parametrize("heads,rows", [((8, 2), [1, 2]), ((64, 1), [9, 3])])
def test_a_page_that_two_sequences_share(heads, rows):
    """What its places get is not said; all others have what the oracle says."""
    x = batch("bf16", rows, [40, 500], heads, 64, 16, seed=17)
    x["pages"][1, 0] = x["pages"][0, 0]
    want, where, tol = want_of(x, decay=0.5)
    knn.key_weights(x["q"], x["lse"], x["k_cache"], x["pages"], x["row_offsets"], x["cache_lens"], x["mass"],
                    key_positions=x["key_positions"], positions=x["positions"], decay=0.5)
    torch.cuda.synchronize()
    err = np.abs(host(x["mass"]) - want) <= tol
    assert np.delete(err, int(x["pages"][0, 0]), 0).all() and np.array_equal(ints(x["key_positions"]), where)
