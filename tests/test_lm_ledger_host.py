"""Host-side checks of the weights of cached keys, eviction and adjusted scores (no GPU needed): bad arguments are refused
before anything is enqueued; the oracle's forms on cases worked out by hand."""
import math

import numpy as np
import pytest

from oracle import lm
from paper_2405_19325_amd import _lib

OK, INVALID, _, UNSUPPORTED, WORKSPACE, HIP = range(6)
MB = 1 << 20  # the buffers of each call lie some megabytes apart; none is ever followed


def apart(names, **more):
    return dict({n: (2 + 2 * i) * MB for i, n in enumerate(names)}, **more)


WEIGH = apart(("q", "lse", "k_cache", "pages", "row_offsets", "cache_lens", "positions", "source_rows", "tree_mask"), rows=32,
              source_count=40, S=2, q_heads=8, kv_heads=2, head_dim=128, q_row=1024, q_head=128, n_pages=100, page_size=16,
              table_width=40, mask_words=1, max_rows=16, max_keys=640, dtype=1, scale=0.1, decay=1.0, mass=40 * MB,
              key_positions=42 * MB, stream=None)
EVICT = apart(("k_cache", "v_cache", "mass", "key_positions", "pages", "cache_lens", "budgets", "next_positions"), S=2,
              kv_heads=2, head_dim=128, n_pages=100, page_size=16, table_width=40, max_keys=640, sinks=4, recent=16, dtype=1,
              mass_out=40 * MB, positions_out=42 * MB, new_lens=44 * MB, workspace=46 * MB, workspace_bytes=1 << 30,
              stream=None)
ADJUST = apart(("scores", "history", "history_lens", "prompt_lens", "row_offsets", "row_tokens", "tree_mask", "repetition",
                "presence", "frequency", "bias_tokens", "bias_values", "allowed"), rows=4, V=1000, S=2, row_stride=1000,
               history_width=50, mask_words=1, bias_width=7, out_stride=1000, probabilities=0, dtype=0, out=40 * MB,
               stream=None)
CALLS = {"weigh": ("knn_key_weights", WEIGH), "evict": ("knn_cache_evict", EVICT), "adjust": ("knn_adjust_scores", ADJUST)}


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def call(lib, which, **over):
    name, args = CALLS[which]
    assert not set(over) - set(args)
    return getattr(lib, name)(*dict(args, **over).values())


@pytest.mark.parametrize("over,expect", [(dict([(n, None)]), INVALID) for n in (
    "q", "lse", "k_cache", "pages", "row_offsets", "cache_lens", "mass", "key_positions")] + [
    (dict(rows=0), INVALID), (dict(source_count=0), INVALID), (dict(source_rows=None, source_count=31), INVALID),
    (dict(S=0), INVALID), (dict(q_heads=9), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(page_size=48), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(max_rows=0), INVALID),
    (dict(max_rows=33), INVALID), (dict(mask_words=0), INVALID), (dict(max_keys=0), INVALID), (dict(max_keys=641), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(decay=-0.5), INVALID),
    (dict(decay=math.inf), INVALID), (dict(decay=math.nan), INVALID), (dict(q_row=-8), INVALID),
    (dict(q_row=1025), UNSUPPORTED), (dict(q_head=130), UNSUPPORTED), (dict(q=2 * MB + 2), UNSUPPORTED),
    (dict(k_cache=6 * MB + 8), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED), (dict(dtype=9), INVALID),
    (dict(dtype=0x101), INVALID), (dict(source_count=1 << 31), UNSUPPORTED),
    (dict(rows=1 << 20, max_rows=1 << 17, mask_words=1 << 12, source_count=1 << 20), UNSUPPORTED),
    (dict(n_pages=1 << 31, kv_heads=1024, q_heads=1024, page_size=65536), UNSUPPORTED)])
def test_key_weights_refuses(lib, over, expect):
    assert call(lib, "weigh", **over) == expect


@pytest.mark.parametrize("over,expect", [(dict([(n, None)]), INVALID) for n in (
    "k_cache", "v_cache", "mass", "key_positions", "pages", "cache_lens", "budgets", "mass_out", "positions_out",
    "new_lens")] + [
    (dict(S=0), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(n_pages=0), INVALID),
    (dict(page_size=17), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(table_width=0), INVALID),
    (dict(max_keys=0), INVALID), (dict(max_keys=641), INVALID), (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID),
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(dtype=0x101), INVALID), (dict(head_dim=1025), UNSUPPORTED),
    (dict(kv_heads=1025), UNSUPPORTED), (dict(S=1 << 31), UNSUPPORTED), (dict(S=1 << 30, kv_heads=4), UNSUPPORTED),
    (dict(workspace=None), WORKSPACE), (dict(workspace=46 * MB + 16), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE)])
def test_evict_refuses(lib, over, expect):
    assert call(lib, "evict", **over) == expect


def test_evict_workspace_size(lib):
    size = lib.knn_cache_evict_workspace_size
    for keys in (1, 2, 31, 4096, 131072, 0x7fffffff):
        assert size(2, 8, keys) > 0 and size(2, 8, keys) % 256 == 0
    assert size((1 << 31) - 1, 1, (1 << 31) - 1) == 0  # 2^64 bytes
    assert size(1 << 20, 32, (1 << 31) - 1) > 1 << 57
    assert size(0, 8, 100) == 0 and size(2, 0, 100) == 0 and size(2, 8, 0) == 0 and size(2, 8, 1 << 31) == 0


@pytest.mark.parametrize("over,expect", [
    (dict(scores=None), INVALID), (dict(out=None), INVALID), (dict(rows=0), INVALID), (dict(V=0), INVALID),
    (dict(S=0), INVALID), (dict(row_offsets=None), INVALID), (dict(row_stride=-1), INVALID), (dict(out_stride=999), INVALID),
    (dict(history=None), INVALID), (dict(history_lens=None), INVALID), (dict(history_width=0), INVALID),
    (dict(history=None, history_lens=None), INVALID), (dict(row_tokens=None), INVALID), (dict(mask_words=0), INVALID),
    (dict(history=None, history_lens=None, prompt_lens=None, row_tokens=None, tree_mask=None), INVALID),
    (dict(bias_tokens=None), INVALID), (dict(bias_values=None), INVALID), (dict(bias_width=0), INVALID),
    (dict(dtype=4), INVALID), (dict(dtype=0x101), INVALID), (dict(V=(1 << 24) + 1), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(history_width=(1 << 30) + 1), UNSUPPORTED),
    (dict(bias_width=(1 << 30) + 1), UNSUPPORTED), (dict(scores=2 * MB + 2), UNSUPPORTED), (dict(out=40 * MB + 1), UNSUPPORTED)])
def test_adjust_refuses(lib, over, expect):
    assert call(lib, "adjust", **over) == expect


@pytest.mark.parametrize("which,output,other,off", [
    ("weigh", o, n, 0) for o in ("mass", "key_positions") for n in (
        "q", "lse", "k_cache", "pages", "row_offsets", "cache_lens", "positions", "source_rows", "tree_mask")] + [
    ("weigh", "mass", "key_positions", 12796), ("weigh", "mass", "lse", 40 * 8 * 4 - 4), ("weigh", "lse", "mass", -4)] + [
    ("evict", o, n, 0) for o in ("k_cache", "v_cache", "mass_out", "positions_out", "new_lens", "workspace") for n in (
        "mass", "key_positions", "pages", "cache_lens", "budgets", "next_positions")
    if (o, n) not in (("mass_out", "mass"), ("positions_out", "key_positions"))] + [
    ("evict", "k_cache", "v_cache", 100 * 2 * 16 * 256 - 2), ("evict", "mass_out", "mass", 4),
    ("evict", "positions_out", "key_positions", -4), ("evict", "mass_out", "positions_out", 0),
    ("evict", "new_lens", "workspace", 0), ("evict", "new_lens", "cache_lens", 4), ("evict", "workspace", "k_cache", 256)] + [
    ("adjust", "out", n, 0) for n in ("history", "history_lens", "prompt_lens", "row_offsets", "row_tokens", "tree_mask",
                                      "repetition", "presence", "frequency", "bias_tokens", "bias_values", "allowed")] + [
    ("adjust", "out", "scores", 4), ("adjust", "out", "scores", -(4 * 1000 - 1) * 4),
    ("adjust", "allowed", "out", 4 * 1000 * 4 - 4)])
def test_outputs_apart_from_all_that_is_read(lib, which, output, other, off):
    """An output that lies on an input, at its first byte or on the last, or on another output, is refused."""
    assert call(lib, which, **{output: CALLS[which][1][other] + off}) == INVALID


def test_adjust_in_place_needs_the_same_stride(lib):
    assert call(lib, "adjust", out=ADJUST["scores"], out_stride=1008) == INVALID
    assert call(lib, "adjust", out=ADJUST["scores"], row_stride=0) == INVALID


def test_oracle_key_weights_by_hand():
    """One sequence of two cached tokens and two rows, one head of one element: scores 1 and 2 with these sums."""
    k = np.array([1.0, 2.0, 3.0, 4.0] + [np.nan] * 12).reshape(1, 1, 16, 1)
    q, lse = np.array([1.0, 0.5]).reshape(2, 1, 1), np.array([3.0, 2.0]).reshape(2, 1)
    args = (k, np.array([[0]]), [0, 2], [2], np.full((1, 1, 16), 10.0), 1.0)
    mass, where, _ = lm.key_weights(q, lse, *args, decay=0.5, key_positions=np.zeros((1, 1, 16), int))
    e = math.exp
    want = [5 + e(1 - 3) + e(0.5 - 2), 5 + e(2 - 3) + e(1 - 2), e(3 - 3) + e(1.5 - 2), e(2 - 2)]
    assert np.allclose(mass[0, 0, :4], want) and (mass[0, 0, 4:] == 10).all()
    assert where[0, 0, :5].tolist() == [0, 0, 2, 3, 0]
    tree = np.array([[False, True], [False, False]])
    mass, where, _ = lm.key_weights(q, lse, *args, tree=tree, source_rows=[1, -1], key_positions=where, positions=[70, 80])
    assert np.allclose(mass[0, 0, :4], [10 + e(0.5 - 2), 10 + e(1 - 2), 0.0, e(2 - 2)])
    assert where[0, 0, :5].tolist() == [0, 0, 70, 80, 0]
    lse[:] = [[-np.inf], [np.nan]]
    assert lm.key_weights(q, lse, *args)[0][0, 0, :5].tolist() == [10, 10, 0, 0, 10]


def test_oracle_evict_by_hand():
    k = np.arange(16.0).reshape(1, 1, 16, 1)
    mass = np.array([5.0, 1, 4, 4, 9, 4, 0, np.nan] + [99.0] * 8).reshape(1, 1, 16)
    out = lm.evict(k, -k, mass, None, np.array([[0]]), [8], [4])
    # 4 and 0 lead; of the three of 4 the first two stay; 4 moves to the place of 1
    assert out[0].flatten()[:8].tolist() == [0, 4, 2, 3, 4, 5, 6, 7] and out[4].tolist() == [4]
    assert out[1].flatten()[1] == -4 and out[2].flatten()[:5].tolist() == [5, 9, 4, 4, 9]
    out = lm.evict(k, -k, mass, None, np.array([[0]]), [8], [4], sinks=2, recent=1)   # 0, 1 and 7 stay, then 4
    assert out[0].flatten()[:4].tolist() == [0, 1, 4, 7]
    out = lm.evict(k, -k, mass, None, np.array([[0]]), [8], [2], sinks=2, recent=6)   # all are protected
    assert out[0].flatten()[:3].tolist() == [0, 4, 2]
    where = np.arange(16)[::-1].reshape(1, 1, 16)
    out = lm.evict(k, -k, mass, where, np.array([[0]]), [8], [1], next_positions=[16], recent=1)  # position 15: index 0
    assert out[0].flatten()[0] == 0 and out[3].flatten()[0] == 15
    for budgets, lens, pages, max_keys in (([8], [8], [[0]], None), ([-1], [8], [[0]], None), ([2], [8], [[1]], None),
                                           ([2], [8], [[0]], 7), ([2], [17], [[0]], None)):
        out = lm.evict(k, -k, mass, None, np.array(pages), lens, budgets, max_keys=max_keys)
        assert np.array_equal(out[0], k) and out[4].tolist() == lens


def test_oracle_adjust_by_hand():
    x = [2.0, -2.0, 0.0, 1.0, 3.0]
    got = lm.adjust(x, prompt=[0, 1, 9], output=[1, 1, 3, -1], repetition=2.0, presence=0.5, frequency=0.25,
                    bias=[(3, 7.0), (4, 1.0), (3, -1.0), (5, 2.0)], allowed=[1, 1, 0, 1, 1])
    assert got.tolist() == [1.0, -4.0 - 0.5 - 0.5, -math.inf, 0.5 - 0.5 - 0.25 - 1.0, 4.0]
    got = lm.adjust([0.25, 0.0, 0.5, 4.0], probabilities=True, output=[0, 1, 3], repetition=2.0, presence=math.log(2),
                    bias=[(1, 5.0)], allowed=[1, 1, 0, 1])
    assert np.allclose(got, [0.25 ** 2 / 2, 0.0, 0.0, 1.0])
    assert lm.adjust(x, output=[0], repetition=math.nan, presence=math.inf, frequency=math.nan).tolist() == x
    assert lm.adjust(x, output=[0], repetition=-1.0).tolist() == x


@pytest.mark.parametrize("words", [(1 << 28) + 1, 1 << 31, (1 << 31) + 100, 1 << 58, 1 << 59, (1 << 59) + 1, (1 << 63) - 1])
def test_masks_that_are_too_wide(lib, words):
    assert call(lib, "weigh", mask_words=words) == UNSUPPORTED
    assert call(lib, "adjust", mask_words=words) == UNSUPPORTED


def test_masks_of_fewer_bits_than_rows(lib):
    for rows, words, expect in ((33, 1, INVALID), (33, 0, INVALID), (64, 1, INVALID), (33, -1, INVALID), (33, -(1 << 62), INVALID),
                                (33, (1 << 28) + 1, UNSUPPORTED)):
        assert call(lib, "weigh", rows=64, source_count=64, max_rows=rows, mask_words=words) == expect


def test_adjust_refuses_more_than_its_counts_hold(lib):
    """Occurrences have 30 bits beside two flags: of histories and of drafts 2^28 at most."""
    over = (1 << 28) + 1
    for name in ("history_width", "bias_width", "mask_words"):
        assert call(lib, "adjust", **{name: over}) == UNSUPPORTED
        assert call(lib, "adjust", **{name: over - 1}) == INVALID  # (such a buffer lies on the output here)
    rows = dict(rows=over, V=10, row_stride=10, out_stride=10)
    assert call(lib, "adjust", **rows) == UNSUPPORTED
    assert call(lib, "adjust", row_tokens=None, tree_mask=None, **rows) == INVALID
