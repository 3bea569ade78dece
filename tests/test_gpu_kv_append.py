"""Cache append on the GPU against the fp64 oracle: rotation forms, head layouts, strides, pages, positions, rows left
out, and what has to stay as it was."""
import numpy as np
import pytest
import torch

import paper_2405_19325_amd as knn
from oracle import lm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def batch(dtype, rows_of, lens, heads, d, page, rot, seed=0, extra_pages=2, width=None, scale=1.0):
    """The tensors of an append on `rows_of` new rows of each sequence, caches filled with other values."""
    g = torch.Generator().manual_seed(seed)
    T, (H, Hk) = sum(rows_of), heads
    need = [max(1, -(-(r + n) // page)) for r, n in zip(rows_of, lens)]
    width = width or max(need)
    n_pages = sum(need) + extra_pages
    order = torch.randperm(n_pages, generator=g)
    pages = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        pages[s, :n] = order[at:at + n].int()
        at += n
    t = TYPES[dtype]
    x = {"q": torch.randn(T, H, d, generator=g) * scale, "k": torch.randn(T, Hk, d, generator=g) * scale,
         "v": torch.randn(T, Hk, d, generator=g), "k_cache": torch.randn(n_pages, Hk, page, d, generator=g),
         "v_cache": torch.randn(n_pages, Hk, page, d, generator=g), "q_out": torch.randn(T, H, d, generator=g)}
    x = {n: v.to(t).cuda() for n, v in x.items()}
    x["pages"] = pages.cuda()
    x["row_offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(rows_of)]), dtype=torch.int64).cuda()
    x["cache_lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    x["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2).float() / max(rot, 1))).cuda() if rot else None
    return x


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check(x, rows=None, **more):
    """Runs the append and compares q_out and both caches with the oracle, cell by cell."""
    names = ("q", "k", "v", "k_cache", "v_cache", "q_out")
    h = {n: host(x[n]) for n in names}
    rows = x["q_out"].shape[0] if rows is None else rows
    extra = {n: (v.cpu().numpy() if torch.is_tensor(v) else v) for n, v in more.items()}
    freq = x["inv_freq"]
    want = lm.append(h["q"], h["k"], h["v"], h["k_cache"], h["v_cache"], x["pages"].cpu().numpy(),
                     x["row_offsets"].cpu().numpy(), x["cache_lens"].cpu().numpy(), rows, q_out=h["q_out"],
                     inv_freq=None if freq is None else freq.cpu().numpy(), **extra)
    got = knn.kv_append(x["k"], x["v"], x["k_cache"], x["v_cache"], x["pages"], x["row_offsets"], x["cache_lens"],
                        q=x["q"], q_out=x["q_out"], inv_freq=freq, **more)
    torch.cuda.synchronize()
    assert got is x["q_out"]
    # Half a step of the element type, and the 32-bit arithmetic before it: the sine and cosine are off by at most
    # 2.1e-7 (the angle's rounding in turns, 2^-25 * 2 pi, and 2^-24 of the functions'), the product by 2^-23 of
    # |a| + |b| <= 2 * 6; 12 * 3.3e-7 < 4e-6.  Half a step of f16 below its normal range is 2^-25.
    eps = torch.finfo(x["k"].dtype).eps / 2
    for name, w, g in (("q_out", want[0], x["q_out"]), ("k_cache", want[1], x["k_cache"])):
        err = np.abs(host(g) - w)
        tol = eps * np.abs(w) + 4e-6 + 2.0 ** -25
        assert (err <= tol).all(), (name, float((err - tol).max()))
    assert np.array_equal(host(x["v_cache"]), want[2])
    return want


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 64), (256, 256), (128, 0), (80, 80), (96, 32), (40, 20),
                                   (33, 6), (1, 0)])
def test_rotation_forms_and_head_sizes(dtype, interleaved, d, rot):
    x = batch(dtype, [3, 1, 5], [0, 40, 17], (4, 2), d, 16, rot, seed=d + rot)
    check(x, interleaved=interleaved)


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("heads", [(1, 1), (32, 32), (8, 1), (5, 5)])
def test_pages_and_heads(page, heads):
    x = batch("bf16", [1, 0, 20, 2], [15, 9, 250, 0], heads, 64, page, 64, seed=page)
    check(x)


def test_one_token():
    check(batch("bf16", [1], [777], (32, 32), 128, 16, 128, seed=3))


def test_many_tokens_share_workgroups():
    # few heads and many rows: several tokens of a workgroup, the last one not full
    check(batch("f16", [1500, 2, 607], [3, 0, 90], (2, 1), 64, 64, 64, seed=4))


def test_positions_apart_from_the_index_and_far_ones():
    x = batch("bf16", [6, 4], [3, 30], (4, 4), 128, 16, 128, seed=5)
    pos = torch.tensor([0, 1, 1, 2, 2, 1, 1 << 20, (1 << 31) - 1, 1000003, 131071], dtype=torch.int32).cuda()
    check(x, positions=pos)


def test_parts_of_one_projection_and_other_orders():
    # views of one [T, (q + 2 kv) d] projection
    x = batch("bf16", [7, 9], [5, 100], (8, 2), 128, 32, 128, seed=6)
    qkv = torch.cat([x["q"], x["k"], x["v"]], dim=1).contiguous()
    x["q"], x["k"], x["v"] = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    check(x)
    # heads before rows
    x = batch("f16", [7, 9], [5, 100], (8, 2), 64, 32, 64, seed=7)
    for n in ("q", "k", "v"):
        x[n] = x[n].transpose(0, 1).contiguous().transpose(0, 1)
    check(x)
    # rows that start off a 16-byte boundary
    x = batch("bf16", [7, 9], [5, 100], (8, 2), 64, 32, 64, seed=8)
    for n in ("q", "k", "v"):
        t = torch.zeros(x[n].shape[0], x[n].shape[1], 67, dtype=x[n].dtype, device="cuda")
        t[:, :, 3:] = x[n]
        x[n] = t[:, :, 3:]
    check(x)


def test_in_place_queries_and_no_queries():
    x = batch("bf16", [4, 4], [10, 20], (4, 2), 128, 16, 128, seed=9)
    y = dict(x, q=x["q"].clone())
    want = check(dict(x, q_out=torch.zeros_like(x["q"])))
    k0, v0 = x["k_cache"].clone(), x["v_cache"].clone()
    got = knn.kv_append(x["k"], x["v"], x["k_cache"], x["v_cache"], x["pages"], x["row_offsets"], x["cache_lens"],
                        q=y["q"], q_out=y["q"], inv_freq=x["inv_freq"])
    assert got is y["q"] and np.abs(host(got) - want[0]).max() <= 2.0 ** -8 * 6
    assert torch.equal(x["k_cache"], k0) and torch.equal(x["v_cache"], v0)
    assert knn.kv_append(x["k"], x["v"], x["k_cache"], x["v_cache"], x["pages"], x["row_offsets"], x["cache_lens"],
                         inv_freq=x["inv_freq"]) is None
    assert torch.equal(x["k_cache"], k0) and torch.equal(x["v_cache"], v0)


def test_source_rows_leave_out_and_repeat():
    x = batch("f16", [4, 3, 2], [10, 33, 5], (4, 2), 64, 16, 64, seed=10)
    src = torch.tensor([8, 8, -1, 0, 3, 9, 1 << 30, 2, -(1 << 31)], dtype=torch.int32).cuda()
    check(x, source_rows=src)
    # more source rows than rows: an accepted path out of a draft
    x = batch("bf16", [12], [10], (4, 2), 64, 16, 64, seed=11)
    x["row_offsets"] = torch.tensor([0, 3], dtype=torch.int64).cuda()
    x["q_out"] = x["q_out"][:3].contiguous()
    check(x, source_rows=torch.tensor([0, 5, 11], dtype=torch.int32).cuda())


def test_rows_behind_the_last_sequence_stay():
    x = batch("bf16", [4, 3, 9], [10, 33, 5], (4, 2), 64, 16, 64, seed=12)
    x["row_offsets"] = torch.tensor([0, 4, 4, 7], dtype=torch.int64).cuda()
    check(x)
    x["row_offsets"] = torch.tensor([0, 0, 0, 0], dtype=torch.int64).cuda()
    check(x)


def test_no_page_and_past_the_table():
    x = batch("bf16", [20, 20, 20], [10, 60, 0], (2, 2), 64, 16, 64, seed=13)
    n = x["k_cache"].shape[0]
    pages = x["pages"].clone()
    pages[0, 1] = -1          # the second page of the first sequence is none
    pages[2, 0] = n           # nor is the first of the third
    x["pages"] = pages
    check(x)
    # indices past the table's width and before the cache
    x = batch("bf16", [20, 20], [30, 50], (2, 2), 64, 16, 64, seed=14)
    x["pages"] = x["pages"][:, :3].contiguous()
    check(x)
    x["cache_lens"] = torch.tensor([-5, (1 << 31) - 3], dtype=torch.int32).cuda()
    check(x)


def test_graph_replays_on_new_lengths_and_tables():
    x = batch("bf16", [2, 2], [10, 40], (4, 2), 128, 16, 128, seed=15, width=4)
    call = knn.KVAppend(x["k"], x["v"], x["k_cache"], x["v_cache"], x["pages"], x["row_offsets"], x["cache_lens"],
                        q=x["q"], q_out=x["q_out"], inv_freq=x["inv_freq"])
    call.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    n = x["k_cache"].shape[0]
    for step in range(4):
        x["cache_lens"].copy_(torch.tensor([11 + 7 * step, 2 * step], dtype=torch.int32))
        x["pages"].copy_(torch.randperm(n)[:8].view(2, 4).int() if n >= 8 else x["pages"])
        x["k"].normal_()
        k0, v0 = x["k_cache"].clone(), x["v_cache"].clone()
        graph.replay()
        torch.cuda.synchronize()
        got = x["k_cache"].clone(), x["v_cache"].clone(), x["q_out"].clone()
        x["k_cache"].copy_(k0), x["v_cache"].copy_(v0)
        call.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (x["k_cache"], x["v_cache"], x["q_out"])))


def test_another_stream_and_refusals():
    x = batch("bf16", [2, 2], [10, 40], (4, 2), 128, 16, 128, seed=16)
    args = [x[n] for n in ("k", "v", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens")]
    here = knn.kv_append(*args, q=x["q"], inv_freq=x["inv_freq"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = knn.kv_append(*args, q=x["q"], inv_freq=x["inv_freq"], stream=side)
    side.synchronize()
    assert torch.equal(here, there)
    bad = [dict(k=x["k"].float()), dict(v=x["v"][:, :1]), dict(pages=x["pages"].long()),
           dict(cache_lens=x["cache_lens"][:1]), dict(k=x["k"].cpu()), dict(v_cache=x["v_cache"][:, :, ::2]),
           dict(row_offsets=x["row_offsets"].int()), dict(k=x["k"].transpose(1, 2).contiguous().transpose(1, 2))]
    for b in bad:
        y = dict(x, **b)
        with pytest.raises((ValueError, TypeError)):
            knn.kv_append(*[y[n] for n in ("k", "v", "k_cache", "v_cache", "pages", "row_offsets", "cache_lens")])
    with pytest.raises(ValueError):
        knn.kv_append(*args, q=x["q"], positions=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        knn.kv_append(*args, q_out=x["q_out"])
    f = [t.float() if t.is_floating_point() else t for t in args]
    with pytest.raises(knn.KnnError):
        knn.kv_append(*f)


def test_one_row_or_head_in_place():
    """Dense to torch, whatever the stride of a dimension of one: a decoding token's part of a projection, a single head."""
    x = batch("bf16", [1], [10], (4, 2), 128, 16, 128, seed=17)
    want = check(dict(x, q_out=torch.zeros_like(x["q"])))[0]
    qkv = torch.cat([x["q"], x["k"], x["v"]], dim=1)
    q = qkv[:, :4]
    names = ("k_cache", "v_cache", "pages", "row_offsets", "cache_lens")
    got = knn.kv_append(qkv[:, 4:6], qkv[:, 6:], *[x[n] for n in names], q=q, q_out=q, inv_freq=x["inv_freq"])
    assert got is q and (np.abs(host(got) - want) <= 2.0 ** -8 * np.abs(want) + 4e-6).all()
    assert torch.equal(qkv[:, 4:6], x["k"]) and torch.equal(qkv[:, 6:], x["v"])
    x = batch("f16", [3], [10], (1, 1), 64, 16, 64, seed=18)
    want = check(dict(x, q_out=torch.zeros_like(x["q"])))[0]
    q = x["q"].as_strided((3, 1, 64), (64, 999, 1))
    got = knn.kv_append(x["k"], x["v"], *[x[n] for n in names], q=q, q_out=q, inv_freq=x["inv_freq"])
    assert got is q and (np.abs(host(got) - want) <= 2.0 ** -11 * np.abs(want) + 4e-6 + 2.0 ** -25).all()
