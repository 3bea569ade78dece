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


SAMPLE = dict(scores=FAKE, uniforms=FAKE, temperature=None, top_k=None, top_p=None, min_p=None, rows=4, V=1000,
              row_stride=1000, probabilities=0, dtype=0, token=FAKE, prob=None, kept=None, workspace=FAKE,
              workspace_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(scores=None), INVALID), (dict(uniforms=None), INVALID), (dict(token=None), INVALID), (dict(rows=0), INVALID),
    (dict(V=0), INVALID), (dict(row_stride=-1), INVALID), (dict(dtype=4), INVALID), (dict(dtype=0x101), INVALID),
    (dict(V=(1 << 24) + 1), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(workspace=None), WORKSPACE),
    (dict(workspace=FAKE + 4), WORKSPACE), (dict(workspace_bytes=0), WORKSPACE)])
def test_sample_refuses(lib, over, expect):
    assert lib.knn_sample(*dict(SAMPLE, **over).values()) == expect


def test_sample_workspace_size(lib):
    assert lib.knn_sample_workspace_size(1, 1, 0) > 0 and lib.knn_sample_workspace_size(256, 131072, 2) > 0
    assert lib.knn_sample_workspace_size(0, 1, 0) == 0 and lib.knn_sample_workspace_size(1, 1, 5) == 0


def test_oracle_sample_by_hand():
    """The oracle's draw on rows worked out by hand."""
    import math

    from oracle import lm

    x = [math.log(0.1), math.log(0.4), math.log(0.2), math.log(0.3)]
    assert [lm.sample(x, u, False)[0] for u in (0.0, 0.05, 0.15, 0.55, 0.65, 0.75, 0.99)] == [0, 0, 1, 2, 2, 3, 3]
    assert lm.sample(x, 0.5, False, top_k=2)[::2] == (1, 2)          # 0.4 and 0.3 stay: 4/7 > 0.5
    assert lm.sample(x, 0.6, False, top_k=2)[::2] == (3, 2)
    assert lm.sample(x, 0.6, False, top_p=0.39)[::2] == (1, 1)
    assert lm.sample(x, 0.99, False, top_p=0.75)[::2] == (3, 3)      # 0.4, 0.3, 0.2: 0.7 lies before the third
    assert lm.sample(x, 0.99, False, min_p=0.6)[::2] == (3, 2)
    assert abs(lm.sample(x, 0.0, False, temperature=0.5)[1] - 0.01 / 0.30) < 1e-12
    assert lm.sample([0.25] * 4, 0.5, True, top_k=3)[::2] == (1, 3)  # running 1/3, 2/3: the first over a half
    assert lm.sample([0.0, -1.0], 0.5, True) == (-1, 0.0, 0)
    assert lm.sample(x, 0.9, False, temperature=0.0) == (1, 1.0, 1)


def test_outputs_apart_from_their_inputs(lib):
    """A call whose output would overwrite what it still reads is refused (q ends 4 * 1024 and 32 * 1024 elements on)."""
    for q_out in (FAKE + 16, FAKE + 8 * 1024 - 2, FAKE - 8 * 1024 + 16):
        assert lib.knn_kv_append(*dict(APPEND, q_out=q_out).values()) == INVALID
    assert lib.knn_kv_append(*dict(APPEND, source_rows=FAKE).values()) == INVALID  # q_out is q, and rows change places
    assert lib.knn_kv_append(*dict(APPEND, q_row=1032).values()) == INVALID        # q_out is q, with other strides
    for out in (FAKE, FAKE + 64 * 1024 - 16, FAKE - 64 * 1024 + 16):
        assert lib.knn_tree_attention(*dict(ATTEND, out=out).values()) == INVALID


def test_limits_of_lengths_and_alignment(lib):
    longest = dict(out=FAKE * 64, max_keys=1 << 31, table_width=1 << 20, page_size=65536)
    assert lib.knn_tree_attention(*dict(ATTEND, **longest).values()) == UNSUPPORTED
    assert lib.knn_tree_attention_workspace_size(32, 2, 8, 2, 128, 16, (1 << 31) - 1) > 0
    assert lib.knn_tree_attention_workspace_size(32, 2, 8, 2, 128, 16, 1 << 31) == 0
    assert lib.knn_sample(*dict(SAMPLE, scores=FAKE + 1).values()) == UNSUPPORTED


MB = 1 << 20
# the buffers of each call a megabyte and more apart
APART = {"append": dict(APPEND, **{n: (2 + i) * MB for i, n in enumerate((
             "q", "k", "v", "row_offsets", "cache_lens", "pages", "positions", "inv_freq", "source_rows", "q_out",
             "k_cache", "v_cache"))}),
         "attend": dict(ATTEND, **{n: (2 + 2 * i) * MB for i, n in enumerate((
             "q", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens", "tree_mask", "out", "lse", "workspace"))}),
         "sample": dict(SAMPLE, **{n: (2 + i) * MB for i, n in enumerate((
             "scores", "uniforms", "temperature", "top_k", "top_p", "min_p", "token", "prob", "kept", "workspace"))})}
NAMES = {"append": "knn_kv_append", "attend": "knn_tree_attention", "sample": "knn_sample"}


@pytest.mark.parametrize("call,output,other,off", [
    ("append", "q_out", n, 0) for n in ("q", "k", "v", "row_offsets", "cache_lens", "pages", "positions", "inv_freq",
                                        "source_rows", "k_cache", "v_cache")] + [
    ("append", c, n, 0) for c in ("k_cache", "v_cache") for n in ("q", "k", "v", "row_offsets", "cache_lens", "pages",
                                                                  "positions", "inv_freq", "source_rows")] + [
    ("append", "k_cache", "k", 3 * 256 * 2 + 254), ("append", "k_cache", "v", -10 * 2 * 16 * 128 * 2 + 2)] + [
    ("attend", o, n, 0) for o in ("out", "lse", "workspace") for n in (
        "q", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens", "tree_mask")] + [
    ("attend", "out", "lse", 0), ("attend", "lse", "workspace", 0), ("attend", "workspace", "out", 256)] + [
    ("sample", o, "scores", (4 * 1000 - 1) * 4) for o in ("token", "prob", "kept")] + [
    ("sample", "token", "prob", 12), ("sample", "prob", "kept", -12), ("sample", "kept", "token", 0)])
def test_outputs_apart_from_all_that_is_read(lib, call, output, other, off):
    """An output that lies on an input, at its first byte or on the last, or on another output, is refused."""
    args = APART[call]
    assert getattr(lib, NAMES[call])(*dict(args, **{output: args[other] + off}).values()) == INVALID


@pytest.mark.parametrize("home,stream", [(0, 7), (5, 7), (5, 0)])
def test_another_stream_waits_once_for_where_the_buffers_came_from(monkeypatch, home, stream):
    """The order of things on streams that only write down what they are asked for."""
    from paper_2405_19325_amd import lm

    log = []

    class Stream:
        def __init__(self, handle=0):
            self.cuda_stream = handle

        def wait_stream(self, other):
            log.append(("wait", self.cuda_stream, other.cuda_stream))

    class Buffer:
        def record_stream(self, s):
            log.append(("record", s.cuda_stream))

    for name, fake in (("current_device", lambda: 0), ("is_current_stream_capturing", lambda: False),
                       ("ExternalStream", Stream), ("default_stream", Stream)):
        monkeypatch.setattr(lm.torch.cuda, name, fake)
    monkeypatch.setattr(lm, "_stream", lambda s=None: home if s is None else s)

    class Library:
        @staticmethod
        def call(*args):
            log.append(("run", args[-1]))
            return OK

    Library.call.argtypes = []
    monkeypatch.setattr(lm, "load", lambda: Library)
    c = lm._Call()
    c._keep(0, "call", (), (), (Buffer(),))
    c._call(None)
    assert log == [("run", home)]
    del log[:]
    c._call(stream)
    c._call(stream)
    assert log == [("wait", stream, home), ("record", stream), ("run", stream), ("run", stream)]


def test_attention_workspace_is_bounded(lib):
    """Two parts a workgroup, of column tiles that are worked off so many at a time that 512 MiB hold them; none where no
    head is parted."""
    size = lib.knn_tree_attention_workspace_size
    for rows in (1, 64, 1000, 8000, 32000, 65535):
        for S in (1, 4, 64):
            for heads, kv in ((8, 1), (64, 1), (1024, 1), (64, 8), (32, 32), (1024, 16)):
                for d in (64, 128, 256):
                    for keys in (rows, 4 * rows, 1 << 20):
                        assert 0 < size(rows * S, S, heads, kv, d, rows, keys) <= 512 << 20
    assert size(8000, 1, 64, 8, 128, 8000, 9000) == 256   # eight heads in eight runs
    assert size(64, 4, 64, 8, 128, 64, 131136) > 1 << 20  # parts all the same where heads lie in several runs


def test_caches_whose_offsets_pass_64_bits(lib):
    """2^62 elements are 2^63 bytes; the limits of each size alone allow 2^67."""
    for over in (dict(n_pages=1 << 31, kv_heads=1024, q_heads=1024, page_size=65536),
                 dict(n_pages=1 << 31, kv_heads=512, q_heads=512, page_size=65536)):
        assert lib.knn_kv_append(*dict(APART["append"], **over).values()) == UNSUPPORTED
        assert lib.knn_tree_attention(*dict(APART["attend"], **over).values()) == UNSUPPORTED
