"""Host-side checks of the calls around the mixture (no GPU needed): bad arguments are refused before anything is
enqueued."""
import pytest

from paper_2405_19325_amd import _lib

OK, INVALID, _, UNSUPPORTED, WORKSPACE, HIP = range(6)
FAKE = 1 << 20  # a non-null pointer value; it is never followed

APPEND = dict(q=FAKE, k=FAKE, v=FAKE, row_offsets=FAKE, cache_lens=FAKE, pages=FAKE, positions=None, inv_freq=FAKE,
              source_rows=None, rows=4, source_count=4, S=2, q_heads=8, kv_heads=2, head_dim=128, rot_dim=128,
              interleaved=0, q_row=1024, q_head=128, k_row=256, k_head=128, v_row=256, v_head=128, n_pages=10,
              page_size=16, table_width=5, dtype=1, q_out=FAKE, k_cache=FAKE, v_cache=FAKE, stream=None)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


@pytest.mark.parametrize("over,expect", [(dict([(n, None)]), INVALID) for n in (
    "k", "v", "row_offsets", "cache_lens", "pages", "k_cache", "v_cache", "q", "q_out", "inv_freq")] + [
    (dict(rows=0), INVALID), (dict(rows=-1), INVALID), (dict(source_count=3), INVALID),
    (dict(source_rows=FAKE, source_count=0), INVALID), (dict(S=0), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=-1), INVALID), (dict(q=None, q_out=None), INVALID), (dict(kv_heads=0), INVALID),
    (dict(head_dim=0), INVALID), (dict(rot_dim=-2), INVALID), (dict(rot_dim=130), INVALID),
    (dict(rot_dim=127), INVALID), (dict(rot_dim=0), INVALID), (dict(q_row=-1), INVALID), (dict(v_head=-8), INVALID),
    (dict(n_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(page_size=24), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=131072), UNSUPPORTED), (dict(table_width=0), INVALID),
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(dtype=0x101), INVALID),
    (dict(head_dim=1026, rot_dim=64), UNSUPPORTED), (dict(kv_heads=1025), UNSUPPORTED),
    (dict(q_heads=1025), UNSUPPORTED), (dict(rows=1 << 31, source_count=1 << 31), UNSUPPORTED),
    (dict(n_pages=1 << 32), UNSUPPORTED)])
def test_append_refuses(lib, over, expect):
    assert lib.knn_kv_append(*dict(APPEND, **over).values()) == expect


ATTEND = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, pages=FAKE, row_offsets=FAKE, cache_lens=FAKE, tree_mask=FAKE, rows=32,
              S=2, q_heads=8, kv_heads=2, head_dim=128, q_row=1024, q_head=128, n_pages=100, page_size=16,
              table_width=40, mask_words=1, max_rows=16, max_keys=640, dtype=1, scale=0.1, out=FAKE, lse=None,
              workspace=FAKE, workspace_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("over,expect", [(dict([(n, None)]), INVALID) for n in (
    "q", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens", "out")] + [
    (dict(rows=0), INVALID), (dict(S=0), INVALID), (dict(q_heads=0), INVALID), (dict(q_heads=9), INVALID),
    (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(page_size=48), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(max_rows=0), INVALID),
    (dict(max_rows=33), INVALID), (dict(mask_words=0), INVALID), (dict(max_rows=32, rows=33, mask_words=0), INVALID),
    (dict(max_keys=0), INVALID), (dict(max_keys=641), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(q_row=-8), INVALID), (dict(q_row=1025), UNSUPPORTED),
    (dict(q_head=130), UNSUPPORTED), (dict(q=FAKE + 2), UNSUPPORTED), (dict(out=FAKE + 8), UNSUPPORTED),
    (dict(k_cache=FAKE + 8), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED), (dict(dtype=9), INVALID),
    (dict(workspace=None), WORKSPACE), (dict(workspace=FAKE + 16), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE),
    (dict(rows=1 << 20, max_rows=1 << 17, mask_words=1 << 12), UNSUPPORTED)])
def test_attention_refuses(lib, over, expect):
    assert lib.knn_tree_attention(*dict(ATTEND, **over).values()) == expect


def test_attention_workspace_size(lib):
    size = lib.knn_tree_attention_workspace_size
    assert size(32, 2, 8, 2, 128, 16, 640) >= 256
    assert size(32, 2, 9, 2, 128, 16, 640) == 0 and size(32, 2, 8, 2, 96, 16, 640) == 0
    assert size(0, 2, 8, 2, 128, 16, 640) == 0
    for keys in (1, 31, 4096, 131072, 0x7fffffff):  # every size gets a workspace that is a multiple of its alignment
        assert size(64, 64, 32, 8, 128, 1, keys) % 256 == 0 and size(64, 64, 32, 8, 128, 1, keys) > 0
