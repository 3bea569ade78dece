"""What a language model's own step needs around the mixture, as cases that can be timed and compared.

A decoding step of nearest-neighbour speculation runs the language model over
each sequence's next rows: one token while decoding, the 5 to 35 tokens of a
proposed span, or a tree of several spans that share their beginnings.  In
every layer the rows' keys and values go into a paged cache with their position
rotation ("append"), then the rows attend over that cache ("attend"); at the
end a token is drawn from the model's logits or from the mixture ("sample").

`run` computes each of them in plain torch operations, or, where `own` is true,
by the calls that a program makes of this package.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# The fields of a case.
# "append": `seqs` sequences of rows_lo..rows_hi new rows on caches of len_lo..len_hi tokens; q_heads, kv_heads,
#   d (head size), rot (rotated elements of a head), interleaved (pairs 2i, 2i+1 instead of i, i + rot/2), page
#   (tokens a page), tree (positions by depth in a tree of drafts, not by index), kept (the rows of an accepted path
#   are appended once more, out of the rows of the whole draft).
# "attend": the same sizes; tree: the rows are a tree with ancestor masks, else a chain.
# "sample": rows, V, form ("logits" or "probs"), dtype, and which of the filters the rows have.


def _rows(kind, name, dtype, seqs, rows, length, heads, d, page, **more):
    c = {"kind": kind, "dtype": dtype, "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "len_lo": length[0],
         "len_hi": length[1], "q_heads": heads[0], "kv_heads": heads[1], "d": d, "page": page}
    c.update(more)
    return dict(c, name=name) if name else c


def _append(name, dtype, seqs, rows, length, heads, d, page, rot=None, interleaved=False, tree=False, kept=False):
    return _rows("append", name, dtype, seqs, rows, length, heads, d, page, rot=rot or d, interleaved=interleaved,
                 tree=tree, kept=kept)


def _attend(name, dtype, seqs, rows, length, heads, d, page, tree=False):
    return _rows("attend", name, dtype, seqs, rows, length, heads, d, page, tree=tree)


def _sample(name, form, dtype, rows, V, temperature=True, top_k=0, top_p=False, min_p=False):
    c = {"kind": "sample", "form": form, "dtype": dtype, "rows": rows, "V": V, "temperature": temperature,
         "top_k": top_k, "top_p": top_p, "min_p": min_p}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One sequence decoding with a small model: one token of one layer; latency only.
        _append("append_one", "bf16", 1, (1, 1), (777, 777), (32, 32), 128, 16),
        # The accepted paths of drafted trees, written over the drafts; pairs side by side, half of each head rotated.
        _append("append_kept", "f16", 32, (1, 9), (500, 4000), (32, 8), 128, 32, rot=64, interleaved=True, tree=True,
                kept=True),
        # The prompts of a batch: inputs with 40 retrieved passages.
        _append("append_prompts", "bf16", 4, (4000, 8000), (0, 0), (32, 32), 128, 64),
        # One token over a short context: latency only.
        _attend("decode_one", "bf16", 1, (1, 1), (1000, 1000), (32, 32), 128, 16),
        # A proposed span of 16 tokens over an input with 40 passages, one head of keys a query head.
        _attend("verify_span", "bf16", 1, (16, 16), (7437, 7437), (32, 32), 128, 64),
        # A serving batch decoding over ragged contexts with grouped heads.
        _attend("decode_batch", "f16", 64, (1, 1), (2000, 16000), (32, 8), 128, 16),
        # Trees of drafts over 8 sequences of 128 long passages with a large model's grouped heads: the most key bytes.
        _attend("verify_trees", "bf16", 8, (16, 16), (65536, 131072), (64, 8), 128, 64, tree=True),
        # Wide trees over long contexts: the most arithmetic.
        _attend("wide_trees", "bf16", 4, (64, 64), (131072, 131072), (64, 8), 128, 64, tree=True),
        # One row of the mixture, its nucleus: latency only.
        _sample("sample_one", "probs", "f32", 1, 32000, temperature=False, top_p=True),
        # A serving batch's logits with every filter.
        _sample("sample_batch", "logits", "bf16", 64, 32000, top_k=50, top_p=True, min_p=True),
        # The rows of drafts, drawn from the whole mixture.
        _sample("sample_drafts", "probs", "f32", 128, 50257, min_p=True),
        # A large batch over a large vocabulary, nucleus over all of it: the most bytes.
        _sample("sample_large", "logits", "f32", 256, 131072, top_p=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32), (40, 40), (64, 8), (64, 8), (32, 8), (16, 2)]
MOST_BYTES = 2 << 30     # of a drawn "attend" case: the largest listed ones' keys and values
MOST_FLOPS = 1 << 40     # and the largest one's arithmetic (its 64 rows on 131072 tokens)
MOST_APPEND = 250 << 20  # bytes of the new rows of a drawn "append" case


def draw(rng):
    pick = rng.random()
    if pick < 0.3:
        form = rng.choice(["logits", "logits", "probs"])
        dtype = "f32" if form == "probs" else rng.choice(["f32", "bf16", "f16"])
        V = rng.choice([32000, 32000, 32001, 50257, 65536, 131072, _log(rng, 1000, 131072)])
        some = rng.random() < 0.7
        return _sample(None, form, dtype, _log(rng, 1, 256), V, temperature=rng.random() < 0.6,
                       top_k=_log(rng, 1, min(V, 2000)) if some and rng.random() < 0.5 else 0,
                       top_p=some and rng.random() < 0.6, min_p=some and rng.random() < 0.4)
    dtype, heads = rng.choice(["bf16", "bf16", "f16"]), rng.choice(HEADS)
    d, page = rng.choice([128, 128, 128, 64, 256]), rng.choice([16, 16, 32, 64, 64, 128, 256])
    use = rng.random()
    if use < 0.3:  # decoding
        rows = (1, 1)
    elif use < 0.9:  # spans and trees
        lo = rng.randint(1, 40)
        rows = (lo, min(64, lo + rng.randint(0, 24)))
    else:  # a piece of a prompt
        lo = rng.randint(65, 400)
        rows = (lo, lo + rng.randint(0, 112))
    tree = 1 < rows[1] <= 64 and rng.random() < 0.6
    if pick < 0.5:
        if use >= 0.9:  # whole prompts
            hi = _log(rng, 512, 8000)
            rows = (int(hi * rng.uniform(0.3, 1.0)), hi)
        most = MOST_APPEND // (4 * rows[1] * (heads[0] + 2 * heads[1]) * d)
        seqs = _log(rng, 1, max(1, min(64, most)))
        hi = _log(rng, 1, 8000)
        return _append(None, dtype, seqs, rows, (int(hi * rng.uniform(0.2, 1.0)), hi), heads, d, page,
                       rot=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3, tree=tree,
                       kept=tree and rng.random() < 0.3)
    seqs = _log(rng, 1, 64 if rows[1] <= 64 else 4)
    most = min(MOST_BYTES // (4 * seqs * heads[1] * d), MOST_FLOPS // (4 * seqs * rows[1] * heads[0] * d))
    hi = _log(rng, 1 if rng.random() < 0.15 else 64, max(64, min(131072, most - 512)))
    lo = hi if rng.random() < 0.3 else int(hi * rng.uniform(0.1, 1.0))
    return _attend(None, dtype, seqs, rows, (lo, hi), heads, d, page, tree=tree)


def _spread(lo, hi, n, phase):
    """n sizes over lo..hi in no order, the largest among them: the same for every seed."""
    at = [(phase + i * 0.6180339887) % 1.0 for i in range(n)]
    at[at.index(max(at))] = 1.0
    return [lo + int(round((hi - lo) * x)) for x in at]


def _sizes(case):
    """New rows and cached tokens of each sequence."""
    return (_spread(case["rows_lo"], case["rows_hi"], case["seqs"], 0.6),
            _spread(case["len_lo"], case["len_hi"], case["seqs"], 0.25))


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["V"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + 32 * case["rows"], "flops": 3 * n}
    rows, lens = _sizes(case)
    T, H, Hk, d = sum(rows), case["q_heads"], case["kv_heads"], case["d"]
    if case["kind"] == "append":
        return {"bytes": 4 * T * (H + 2 * Hk) * d, "flops": 3 * T * (H + Hk) * case["rot"]}
    keys = sum(r + n for r, n in zip(rows, lens))
    seen = sum(r * (n + (r + 1) / 2) for r, n in zip(rows, lens))
    return {"bytes": 4 * keys * Hk * d + 4 * T * H * d, "flops": 4 * d * H * seen}


def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + n)
    return g


def _device(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype)).cuda()


def _trees(rows, width, seed):
    """Ancestor masks (each node sees itself) as words of 32 bits, and depths, of one random tree for each sequence: a
    node hangs under the node before it (a span goes on) more often than under an earlier one (a span that branches)."""
    rng = np.random.RandomState(int(seed) % (1 << 31))
    sees, depth = np.zeros((sum(rows), 32 * width), bool), np.zeros(sum(rows), np.int64)
    at = 0
    for n in rows:
        for i in range(n):
            parent = i - 1 if rng.rand() < 0.6 else rng.randint(-1, i) if i else -1
            if parent >= 0:
                sees[at + i] = sees[at + parent]
                depth[at + i] = depth[at + parent] + 1
            sees[at + i, i] = True
        at += n
    return np.packbits(sees, axis=1, bitorder="little").view(np.int32), depth


def _cache(case, seed, rows, lens, filled):
    """Pages in no order, the table that names them, and the caches: [pages, kv_heads, page, d]."""
    page, shape = case["page"], (case["kv_heads"], case["page"], case["d"])
    need = [-(-(r + n) // page) for r, n in zip(rows, lens)]
    total, g = sum(need) + 3, _gen(seed, 1)
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    starts = np.concatenate([[0], np.cumsum(need)])[:-1]
    at = starts[:, None] + np.minimum(np.arange(max(need))[None], np.asarray(need)[:, None] - 1)
    dtype = DTYPES[case["dtype"]]
    k = torch.empty((total, *shape), dtype=dtype, device="cuda").normal_(0.0, filled, generator=g)
    v = torch.empty((total, *shape), dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)
    return k, v, ids[_device(at, np.int64)].contiguous()


def _prepare_append(case, seed):
    rows, lens = _sizes(case)
    g, dtype, d = _gen(seed, 2), DTYPES[case["dtype"]], case["d"]
    T, H, Hk = sum(rows), case["q_heads"], case["kv_heads"]
    k_cache, v_cache, pages = _cache(case, seed, rows, lens, 1.0)
    # the projections' output: queries, keys and values of a token side by side; of a tree's draft, four times the rows kept
    source = T * 4 if case["kept"] else T
    qkv = torch.empty(source, H + 2 * Hk, d, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)
    at = np.concatenate([np.arange(n) for n in rows])
    depth = _trees(rows, -(-max(rows) // 32), seed)[1] if case["tree"] and not case["kept"] else at
    s = {"kind": "append", "q": qkv[:, :H], "k": qkv[:, H:H + Hk], "v": qkv[:, H + Hk:], "k_cache": k_cache,
         "v_cache": v_cache, "pages": pages, "row_offsets": _device(np.concatenate([[0], np.cumsum(rows)]), np.int64),
         "cache_lens": _device(lens, np.int32), "positions": None, "source_rows": None,
         "interleaved": case["interleaved"],
         # as a model keeps it: inverse frequencies of base 10000 in 32 bits
         "inv_freq": (1.0 / 10000.0 ** (torch.arange(0, case["rot"], 2, device="cuda").float() / case["rot"])),
         "q_out": torch.zeros(T, H, d, dtype=dtype, device="cuda")}
    if case["tree"]:
        s["positions"] = _device(np.repeat(lens, rows) + depth, np.int32)
    if case["kept"]:
        s["source_rows"] = _device(4 * np.arange(T), np.int32) + torch.randint(0, 4, (T,), generator=g, device="cuda",
                                                                               dtype=torch.int32)
    return s


def _prepare_attend(case, seed):
    rows, lens = _sizes(case)
    k_cache, v_cache, pages = _cache(case, seed, rows, lens, 1.0)
    T, d = sum(rows), case["d"]
    q = torch.empty(T, case["q_heads"], d, dtype=DTYPES[case["dtype"]], device="cuda")
    q.normal_(0.0, 1.5, generator=_gen(seed, 2))  # scores of a deviation of 1.5: a few keys in a hundred carry the weight
    s = {"kind": "attend", "q": q, "k_cache": k_cache, "v_cache": v_cache, "pages": pages, "scale": 1.0 / math.sqrt(d),
         "row_offsets": _device(np.concatenate([[0], np.cumsum(rows)]), np.int64),
         "cache_lens": _device(lens, np.int32), "max_rows": max(rows), "tree_mask": None,
         "max_keys": max(r + n for r, n in zip(rows, lens))}
    if case["tree"]:
        s["tree_mask"] = torch.from_numpy(_trees(rows, -(-max(rows) // 32), seed)[0]).cuda()
    return s


def _prepare_sample(case, seed):
    rows, V, g = case["rows"], case["V"], _gen(seed, 1)
    x = torch.randn(rows, V, generator=g, device="cuda") * 3.0
    if case["form"] == "probs":  # the mixture: the model's distribution and the weights of some retrieved tokens
        near = torch.randint(0, V, (rows, min(V, 300)), generator=g, device="cuda")
        w = torch.rand(near.shape, generator=g, device="cuda") ** 4
        x = torch.softmax(x, dim=1).mul_(0.3).scatter_add_(1, near, w * (0.7 / w.sum(1, keepdim=True)))

    def each(lo, hi, off):
        """A value for each row, and `off` for one row in eight."""
        t = lo + (hi - lo) * torch.rand(rows, generator=g, device="cuda")
        return torch.where(torch.rand(rows, generator=g, device="cuda") < 0.125, torch.full_like(t, off), t)

    s = {"kind": "sample", "form": case["form"], "scores": x.to(DTYPES[case["dtype"]]).contiguous(),
         "uniforms": torch.rand(rows, generator=g, device="cuda"), "temperature": None, "top_k": None, "top_p": None,
         "min_p": None}
    if case["temperature"]:
        s["temperature"] = each(0.5, 1.3, 0.0)
    if case["top_k"]:
        s["top_k"] = each(1 + case["top_k"] // 2, case["top_k"] + 1, 0.0).to(torch.int32)
    if case["top_p"]:
        s["top_p"] = each(0.5, 0.98, 1.0)
    if case["min_p"]:
        s["min_p"] = each(0.001, 0.1, 0.0)
    return s


def prepare(case, seed):
    return {"append": _prepare_append, "attend": _prepare_attend, "sample": _prepare_sample}[case["kind"]](case, seed)


def run(state):
    return {"append": _run_append, "attend": _run_attend, "sample": _run_sample}[state["kind"]](state)


def _call(state, make):
    """The object that a program keeps for its calls on these buffers."""
    if "call" not in state:
        import paper_2405_19325_amd as knn
        state["call"] = make(knn)
    return state["call"]


def _rotated(x, cos, sin, interleaved):
    """Rows [T, heads, d] with their first 2 * cos.shape[1] elements rotated, in 32 bits."""
    half = cos.shape[1]
    x = x.float()
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    c, s = cos[:, None], sin[:, None]
    pair = (a * c - b * s, b * c + a * s)
    out = torch.stack(pair, dim=-1).flatten(-2) if interleaved else torch.cat(pair, dim=-1)
    return torch.cat([out, x[..., 2 * half:]], dim=-1)


def _run_append(s):
    if own:
        call = _call(s, lambda knn: knn.KVAppend(
            s["k"], s["v"], s["k_cache"], s["v_cache"], s["pages"], s["row_offsets"], s["cache_lens"], q=s["q"],
            q_out=s["q_out"], positions=s["positions"], inv_freq=s["inv_freq"], interleaved=s["interleaved"],
            source_rows=s["source_rows"]))
        call.run()
        return s["q_out"], s["k_cache"], s["v_cache"]
    q, k, v = s["q"], s["k"], s["v"]
    if s["source_rows"] is not None:
        at = s["source_rows"].long()
        q, k, v = q[at], k[at], v[at]
    row = torch.arange(q.shape[0], device=q.device)
    seq = torch.searchsorted(s["row_offsets"], row, right=True) - 1
    index = s["cache_lens"][seq].long() + row - s["row_offsets"][seq]
    pos = index if s["positions"] is None else s["positions"].long()
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    page_size = s["k_cache"].shape[2]
    page, slot = s["pages"][seq, index // page_size].long(), index % page_size
    s["k_cache"][page, :, slot] = _rotated(k, cos, sin, s["interleaved"]).to(k.dtype)
    s["v_cache"][page, :, slot] = v
    s["q_out"].copy_(_rotated(q, cos, sin, s["interleaved"]))
    return s["q_out"], s["k_cache"], s["v_cache"]


def _run_attend(s):
    if own:
        return _call(s, lambda knn: knn.TreeAttention(
            s["q"], s["k_cache"], s["v_cache"], s["pages"], s["row_offsets"], s["cache_lens"], s["max_rows"],
            s["max_keys"], tree_mask=s["tree_mask"], scale=s["scale"])).run()
    q, k_cache, n, keys = s["q"], s["k_cache"], s["max_rows"], s["max_keys"]
    (T, H, d), (_, Hk, page, _) = q.shape, k_cache.shape
    first, lens, S = s["row_offsets"][:-1], s["cache_lens"].long(), s["pages"].shape[0]
    count = s["row_offsets"][1:] - first
    i = torch.arange(n, device=q.device)
    held = i < count[:, None]                                         # [S, n]: padded rows are no rows
    row = (first[:, None] + i).clamp_(max=T - 1)
    # what each row sees: the cached tokens, and the drafts that its mask names
    at = torch.arange(keys, device=q.device)
    draft = at - lens[:, None]                                        # [S, keys]
    if s["tree_mask"] is None:
        sees = draft[:, None] <= i[:, None]
    else:
        j = draft.clamp(0, n - 1)
        words = s["tree_mask"][row]                                   # [S, n, words]
        word = words.gather(2, (j // 32)[:, None].expand(S, n, keys))
        sees = (((word >> (j % 32)[:, None].int()) & 1) == 1) | (draft < 0)[:, None]
    sees = sees & (draft < count[:, None])[:, None]                   # [S, n, keys]

    def whole(cache):
        pages = s["pages"][:, :-(-keys // page)].long()
        return cache[pages].transpose(1, 2).reshape(S, Hk, -1, d)[:, :, :keys].float()

    x = q[row].float().view(S, n, Hk, H // Hk, d).permute(0, 2, 1, 3, 4).reshape(S, Hk, -1, d)
    x = torch.matmul(x, whole(k_cache).transpose(2, 3).contiguous()).mul_(s["scale"])
    x = x.view(S, Hk, n, H // Hk, keys).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)  # rows that see nothing: no NaN
    x = x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    out = torch.matmul(x.view(S, Hk, -1, keys), whole(s["v_cache"])).view(S, Hk, n, H // Hk, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out)).permute(0, 2, 1, 3, 4).reshape(S, n, H, d)
    return out[held].to(q.dtype)


def _run_sample(s):
    if own:
        return _call(s, lambda knn: knn.Sampler(
            s["scores"], s["uniforms"], probabilities=s["form"] == "probs", temperature=s["temperature"],
            top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])).run()
    x = s["scores"].double()  # 64 bits: the sums decide which token is drawn
    rows, V = x.shape
    order = torch.sort(x, dim=1, descending=True, stable=True)  # equal values: the lower token first
    best, column = order.values[:, :1], torch.arange(V, device=x.device)

    def each(name, value):
        t = s[name]
        return torch.full((rows, 1), value, dtype=torch.float64, device=x.device) if t is None else t.double()[:, None]

    t = each("temperature", 1.0)
    w = (order.values / best).pow(1.0 / t) if s["form"] == "probs" else ((order.values - best) / t).exp()
    w = torch.where(t > 0, w, (column == 0).double())
    k = each("top_k", 0)
    w = torch.where((k <= 0) | (column < k), w, 0.0)
    before = w.cumsum(1) - w
    p = each("top_p", 1.0)
    keep = (p >= 1) | (before < p * w.sum(1, keepdim=True)) | (column == 0)
    keep &= (w >= each("min_p", 0.0)) & (w > 0)
    w = torch.where(keep, w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order.indices, w)  # by token
    mass = w.cumsum(1)
    total = mass[:, -1:]
    last = (mass < total).sum(1).clamp_(max=V - 1)  # the last token that carries weight
    token = torch.minimum((mass <= s["uniforms"].double()[:, None] * total).sum(1), last)
    prob = (w.gather(1, token[:, None]) / total).flatten().float()
    return token.int(), prob, keep.sum(1).int()


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](prepare(case, seed))


def _exact_append(s):
    """Pairs as complex numbers times exp(i angle), each sequence's tokens put where its table says."""
    T = s["q_out"].shape[0]
    source = torch.arange(T, device="cuda") if s["source_rows"] is None else s["source_rows"].long()
    half, page_size = s["inv_freq"].numel(), s["k_cache"].shape[2]
    q, k, v = (s[n][source].double() for n in ("q", "k", "v"))
    k_out, v_out = s["k_cache"].double(), s["v_cache"].double()
    offsets, lens = s["row_offsets"].tolist(), s["cache_lens"].tolist()
    for b, length in enumerate(lens):
        r0, r1 = offsets[b], offsets[b + 1]
        at = torch.arange(length, length + r1 - r0, device="cuda")
        pos = (at if s["positions"] is None else s["positions"][r0:r1]).double()
        turn = torch.polar(torch.ones(r1 - r0, half, dtype=torch.float64, device="cuda"),
                           pos[:, None] * s["inv_freq"].double()[None])[:, None]
        for x in (q, k):
            part = x[r0:r1, :, :2 * half]
            if s["interleaved"]:
                z = torch.view_as_complex(part.unflatten(2, (half, 2)).contiguous()) * turn
                x[r0:r1, :, :2 * half] = torch.view_as_real(z).flatten(2)
            else:
                z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * turn
                x[r0:r1, :, :2 * half] = torch.cat([z.real, z.imag], 2)
        slot = s["pages"][b].long()[at // page_size] * page_size + at % page_size
        for x, out in ((k, k_out), (v, v_out)):
            flat = out.transpose(1, 2).contiguous()  # [pages, slots, heads, d]
            flat.view(-1, *x.shape[1:])[slot] = x[r0:r1]
            out.copy_(flat.transpose(1, 2))
    return q, k_out, v_out


def _exact_attend(s):
    """One sequence and one head of keys after the other, tokens gathered one by one."""
    q, page, n_words = s["q"].double(), s["k_cache"].shape[2], 0 if s["tree_mask"] is None else s["tree_mask"].shape[1]
    Hk = s["k_cache"].shape[1]
    g = q.shape[1] // Hk
    out, offsets = torch.zeros_like(q), s["row_offsets"].tolist()
    for b, length in enumerate(s["cache_lens"].tolist()):
        r0, r1 = offsets[b], offsets[b + 1]
        n = r1 - r0
        at = torch.arange(length + n, device="cuda")
        where = s["pages"][b].long()[at // page]
        hidden = torch.zeros(n, length + n, dtype=torch.bool, device="cuda")
        if n_words == 0:
            hidden[:, length:] = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        else:
            bits = torch.from_numpy(np.unpackbits(s["tree_mask"][r0:r1].cpu().numpy().view(np.uint8), axis=1,
                                                  bitorder="little"))
            hidden[:, length:] = bits[:, :n].cuda() == 0
        for h in range(Hk):
            k, v = (s[c][where, h, at % page].double() for c in ("k_cache", "v_cache"))
            for a in range(h * g, (h + 1) * g):
                score = (q[r0:r1, a] * s["scale"]) @ k.t()
                out[r0:r1, a] = torch.softmax(score.masked_fill(hidden, -math.inf), dim=1).nan_to_num(0.0) @ v
    return out


def _exact_sample(s):
    """One row after the other on the host."""
    x, u = s["scores"].double().cpu().numpy(), s["uniforms"].double().cpu().numpy()
    rows, V = x.shape
    p = {n: None if s[n] is None else s[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p")}
    token, prob, kept = np.zeros(rows, np.int32), np.zeros(rows), np.zeros(rows, np.int32)
    for b in range(rows):
        order = np.argsort(-x[b], kind="stable")
        t = 1.0 if p["temperature"] is None else p["temperature"][b]
        if not t > 0:
            token[b], prob[b], kept[b] = order[0], 1.0, 1
            continue
        first = x[b, order[0]]
        w = np.exp(np.log(x[b] / first) / t) if s["form"] == "probs" else np.exp((x[b] - first) / t)
        n = V
        if p["top_k"] is not None and p["top_k"][b] > 0:
            n = min(n, int(p["top_k"][b]))
        if p["top_p"] is not None and p["top_p"][b] < 1:
            mass = np.cumsum(w[order[:n]])
            n = 1 + int(np.searchsorted(mass[:-1], p["top_p"][b] * mass[-1], side="left"))
        if p["min_p"] is not None:
            n = int(np.sum(w[order[:n]] >= p["min_p"][b]))
        some = np.sort(order[:n])
        mass = np.cumsum(w[some])
        i = min(n - 1, int(np.searchsorted(mass, u[b] * mass[-1], side="right")))
        token[b], prob[b], kept[b] = some[i], w[some[i]] / mass[-1], n
    return torch.from_numpy(token), torch.from_numpy(prob), torch.from_numpy(kept)
