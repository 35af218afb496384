"""Measured cases of the operators that serve many sequences at once: the paged
key-value cache's append with the rotation on the way, the attention of one
new token per row over that cache, and the penalties, biases and grammar masks
between the logits and the next token.

The model sizes are those of this repository's synthetic decoder (16 heads of
128, vocabulary 50,304) and generic ones with fewer key than query heads.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32,
          "e4m3": torch.float8_e4m3fn}
ITEM = {"bf16": 2, "fp16": 2, "f32": 4, "e4m3": 1}
E4M3_MAX = 448.0
ROPE_BASE = 10000.0


# ---------------------------------------------------------------- cases
def _append(name, tokens, seqs, heads, kv_heads, dim, page, dtype="bf16", cache=None, rotary=None,
            interleaved=False, start=0):
    """`tokens` new tokens over `seqs` sequences; each sequence has about `start` tokens already."""
    return dict(name=name, kind="append", tokens=tokens, seqs=seqs, heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, dtype=dtype, cache=cache or dtype, rotary=rotary or dim,
                interleaved=interleaved, start=start)


def _attend(name, rows, heads, kv_heads, dim, page, shortest, longest, dtype="bf16", cache=None,
            window=0):
    return dict(name=name, kind="attend", rows=rows, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, shortest=shortest, longest=longest, dtype=dtype, cache=cache or dtype,
                window=window)


def _logits(name, rows, vocab, history, dtype="f32", biases=0, masked=False):
    return dict(name=name, kind="logits", rows=rows, vocab=vocab, history=history, dtype=dtype,
                biases=biases, masked=masked)


def listed():
    return [
        # One sequence of this repository's decoder, in the middle of a request.
        _append("append_1", 1, 1, 16, 16, 128, 16, start=302),
        # A decode batch over an 8-bit cache, far into its sequences.
        _append("append_61_e4m3", 61, 61, 32, 8, 128, 32, cache="e4m3", start=20000),
        # Ragged prompts of five requests at once; a quarter of each head is
        # rotated, neighbouring dimensions paired.
        _append("append_7919_prompts", 7919, 5, 32, 8, 128, 16, dtype="fp16", rotary=32,
                interleaved=True),
        # The decoder's attention in the middle of a request: latency.
        _attend("attend_1x302", 1, 16, 16, 128, 16, 302, 302),
        # A small decode batch of requests of very different ages.
        _attend("attend_16_ragged", 16, 32, 8, 128, 16, 1, 4096),
        # One long document: all parallelism comes from the cache's length.
        _attend("attend_1x131072", 1, 32, 8, 128, 64, 131072, 131072),
        # A large batch over an 8-bit cache.
        _attend("attend_128_e4m3", 128, 64, 8, 128, 32, 64, 16384, cache="e4m3"),
        # A sliding window, five query heads to a key head, pages of 8 slots,
        # some rows of the batch empty.
        _attend("attend_47_window", 47, 20, 4, 64, 8, 0, 6000, dtype="fp16", window=1024),
        # One request of the decoder: latency.
        _logits("logits_1", 1, 50304, 302),
        # A decode batch, some requests with biases and grammars.
        _logits("logits_64", 64, 50304, 2000, biases=300, masked=True),
        # A large batch and vocabulary in 16 bits.
        _logits("logits_256_bf16", 256, 131072, 1000, dtype="bf16", masked=True),
        # Long histories, a vocabulary that nothing divides.
        _logits("logits_19_long", 19, 49999, 32000, biases=20),
    ]


HEADS = [(16, 16), (8, 8), (32, 8), (64, 8), (20, 4), (28, 4), (8, 1), (48, 2)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "logits"])
    if kind == "logits":
        case = _logits("", _log_int(rng, 1, 256), _log_int(rng, 1000, 131072),
                       _log_int(rng, 1, 16000), dtype=rng.choice(["f32", "bf16", "fp16"]),
                       biases=rng.choice([0, 0, _log_int(rng, 1, 300)]),
                       masked=rng.random() < 0.5)
    else:
        heads, kv_heads = rng.choice(HEADS)
        dim = rng.choice([64, 128, 128, 256])
        page = rng.choice([8, 16, 32, 64, 128])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        cache = rng.choice([dtype, dtype, "e4m3"])
        if kind == "append":
            tokens = _log_int(rng, 1, 4000)
            case = _append("", tokens, rng.randint(1, min(tokens, 100)), heads, kv_heads, dim, page,
                           dtype, cache, rng.choice([dim, dim, dim // 2, 32]), rng.random() < 0.5,
                           rng.choice([0, _log_int(rng, 1, 200000)]))
        else:
            longest = _log_int(rng, 1, 65536)
            # About half a gigabyte of cache at most.
            most = 2**29 // (longest * kv_heads * dim * 2 * ITEM[cache])
            rows = _log_int(rng, 1, max(1, min(300, most)))
            case = _attend("", rows, heads, kv_heads, dim, page, rng.choice([0, 1, longest]),
                           longest, dtype, cache, rng.choice([0, 0, 0, _log_int(rng, 1, longest)]))
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs
def _lengths(case, r):
    lo, hi = case["shortest"], case["longest"]
    n = np.exp(r.uniform(math.log(lo + 1), math.log(hi + 1), case["rows"])).astype(np.int64) - 1
    n = np.clip(n, lo, hi)
    # Half of the rows anywhere in the range, so that the batch is not all short.
    n = np.where(r.random(case["rows"]) < 0.5, n, r.integers(lo, hi + 1, case["rows"]))
    n[0] = hi
    return n


def _append_rows(case, r):
    """Sequence and position of every token, sequence after sequence, positions ascending; each
    sequence's first new position and the one after its last."""
    n, s = case["tokens"], case["seqs"]
    cuts = np.sort(r.choice(np.arange(1, n), s - 1, replace=False)) if s > 1 else np.array([], int)
    counts = np.diff(np.concatenate([[0], cuts, [n]])).astype(int)
    first = r.integers(case["start"] // 2, case["start"] + 1, s) if case["start"] else np.zeros(s, int)
    if s == 1:
        first[:] = case["start"]
    seq = np.repeat(np.arange(s), counts)
    pos = np.concatenate([np.arange(f, f + c) for f, c in zip(first, counts)])
    return seq, pos, first, first + counts


def _tables(r, first, ends, page):
    """Page tables of sequences whose positions first .. end - 1 have pages, shuffled over the
    pool; the other entries are -1 (pages given back behind a window, or not needed yet)."""
    at = np.arange(max(1, -(-int(ends.max()) // page)))[None, :]
    has = (at >= first[:, None] // page) & (at < -(-ends[:, None] // page))
    ids = r.permutation(int(has.sum()) + 3).astype(np.int32)
    table = np.full(has.shape, -1, np.int32)
    table[has] = ids[:int(has.sum())]
    return table, len(ids)


def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(dtype)


def _pages(g, case, pages):
    """A cache full of keys and values, in the values that its type stores."""
    shape = (pages, case["page"], case["kv_heads"], case["dim"])
    dt = DTYPES[case["cache"]]
    if case["cache"] != "e4m3":
        values = lambda: torch.randn(shape, device="cuda", generator=g, dtype=dt)
        return values(), values(), None, None
    scale = 0.02 + 0.03 * torch.rand(2, case["kv_heads"], device="cuda", generator=g)
    stored = lambda s: (torch.randn(shape, device="cuda", generator=g, dtype=torch.float16)
                        / s[:, None].half()).to(dt)
    return stored(scale[0]), stored(scale[1]), scale[0], scale[1]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = np.random.default_rng([seed, 77])
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    st = dict(case=case)
    if case["kind"] == "logits":
        _prepare_logits(st, case, g, r, dev)
        return st
    dt = DTYPES[case["dtype"]]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        seq, pos, first, ends = _append_rows(case, r)
        table, _ = _tables(r, first, ends, case["page"])
        pages = case["tokens"] // case["page"] + 2 * case["seqs"] + 3  # enough for any split
        # q, k and v as the fused projection leaves them: parts of one row.
        row = _normal(g, case["tokens"], (H + 2 * Hk) * D, dtype=dt)
        st["q"], st["k"], st["v"] = (x.unflatten(1, (-1, D)) for x in
                                     row.split([H * D, Hk * D, Hk * D], 1))
        st["q_out"] = torch.empty(case["tokens"], H, D, device="cuda", dtype=dt)
        st["seqs"], st["positions"] = dev(seq.astype(np.int32)), dev(pos.astype(np.int32))
        R = case["rotary"]
        st["inv_freq"] = dev(ROPE_BASE ** (-2.0 * np.arange(R // 2) / R))
    else:
        n = _lengths(case, r)
        table, pages = _tables(r, np.zeros_like(n), n, case["page"])
        st["q"] = _normal(g, case["rows"], H, D, dtype=dt)
        st["out"] = torch.empty_like(st["q"])
        st["lengths"] = dev(n.astype(np.int32))
    st["table"] = dev(table)
    st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"] = _pages(g, case, pages)
    if own:
        from paper_2608_15383_amd import api
        st["kv"] = api.PagedKV(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        if case["kind"] == "attend":
            st["workspace"] = torch.zeros(
                api.paged_attention_workspace_bytes(st["kv"], case["rows"], H, case["longest"]),
                dtype=torch.uint8, device="cuda")
    return st


def _prepare_logits(st, case, g, r, dev):
    B, V, L = case["rows"], case["vocab"], case["history"]
    st["logits"] = _normal(g, B, V, dtype=DTYPES[case["dtype"]]) * 3
    st["out"] = torch.empty_like(st["logits"])
    st["next_token"] = torch.empty(B, dtype=torch.int32, device="cuda")
    # Token ids with a natural text's skew, so that some repeat often.
    ids = np.minimum(r.zipf(1.2, (B, L)) - 1, 10**9) * 7919 % V
    n = r.integers(max(1, L // 2), L + 1, B)
    ids[np.arange(L)[None, :] >= n[:, None]] = -1
    st["history"], st["history_lengths"] = dev(ids.astype(np.int32)), dev(n.astype(np.int32))
    st["prompt_lengths"] = dev((n * r.random(B)).astype(np.int32))
    st["repetition"] = dev((1 + 0.3 * r.random(B)).astype(np.float32))
    st["presence"] = dev(r.random(B).astype(np.float32))
    st["frequency"] = dev((0.5 * r.random(B)).astype(np.float32))
    st["bias_ids"] = st["bias_values"] = st["bias_counts"] = None
    if case["biases"]:
        m = min(case["biases"], V)
        st["bias_ids"] = dev(np.stack([r.permutation(V)[:m] for _ in range(B)]).astype(np.int32))
        st["bias_values"] = dev(r.normal(0, 4, (B, m)).astype(np.float32))
        st["bias_counts"] = dev(r.integers(0, m + 1, B).astype(np.int32))
    st["mask"] = None
    if case["masked"]:
        words = r.integers(0, 2**32, (B, -(-V // 32)), dtype=np.uint32)
        words[::2] = 2**32 - 1  # every other request has no grammar
        st["mask"] = dev(words.view(np.int32))
    if own:
        from paper_2608_15383_amd import api
        st["workspace"] = torch.zeros(api.process_logits_workspace_bytes(B, V), dtype=torch.uint8,
                                      device="cuda")


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        return _run_own(st, case)
    return {"append": _plain_append, "attend": _plain_attend, "logits": _plain_logits}[case["kind"]](
        st, case)


def _run_own(st, case):
    from paper_2608_15383_amd import api
    if case["kind"] == "append":
        api.paged_append(st["kv"], st["q"], st["k"], st["v"], st["positions"], st["table"],
                         st["inv_freq"], seqs=st["seqs"], q_out=st["q_out"],
                         interleaved=case["interleaved"])
        return st["q_out"], st["k_pages"], st["v_pages"]
    if case["kind"] == "attend":
        api.paged_attention(st["kv"], st["q"], st["table"], st["lengths"], st["out"],
                            st["workspace"], case["longest"], window=case["window"])
        return st["out"]
    api.process_logits(st["logits"], st["out"], st["workspace"], history=st["history"],
                       history_lengths=st["history_lengths"], prompt_lengths=st["prompt_lengths"],
                       repetition=st["repetition"], presence=st["presence"],
                       frequency=st["frequency"], bias_ids=st["bias_ids"],
                       bias_values=st["bias_values"], bias_counts=st["bias_counts"],
                       mask=st["mask"], next_token=st["next_token"])
    return st["out"], st["next_token"]


def _rotate(x, angle, interleaved):
    """x [N][h][D] in 32 bits; angle [N][R/2] in 64 bits; dimensions from R on stay."""
    half = angle.shape[1]
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([r, rest], -1)


def _bits(pages):
    """A view to index: the 8-bit type goes by its bytes."""
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _store(pages, page, slot, x, scale):
    if scale is not None:
        x = (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    _bits(pages)[page, slot] = _bits(x.to(pages.dtype))


def _plain_append(st, case):
    pos = st["positions"].long()
    angle = pos[:, None].double() * st["inv_freq"][None, :]
    page = st["table"][st["seqs"].long(), pos // case["page"]].long()
    slot = pos % case["page"]
    st["q_out"].copy_(_rotate(st["q"].float(), angle, case["interleaved"]))
    _store(st["k_pages"], page, slot, _rotate(st["k"].float(), angle, case["interleaved"]),
           st["k_scale"])
    _store(st["v_pages"], page, slot, st["v"].float(), st["v_scale"])
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_attend(st, case):
    B, H, Hk, D = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    G = H // Hk
    page = st["table"].clamp(min=0).long()
    keys = torch.arange(page.shape[1] * case["page"], device="cuda")
    n = st["lengths"].long()[:, None]
    seen = keys < n
    if case["window"]:
        seen = seen & (keys >= n - case["window"])
    seen = seen[:, None, None, :]                                   # [B][1][1][L]
    k = _bits(st["k_pages"])[page].view(st["k_pages"].dtype).flatten(1, 2).float().permute(0, 2, 3, 1).contiguous()  # [B][Hk][D][L]
    q = st["q"].float().view(B, Hk, G, D)
    scale = torch.full((Hk,), 1.0 / math.sqrt(D), device="cuda")
    if st["k_scale"] is not None:
        scale = scale * st["k_scale"]
    s = (torch.matmul(q, k) * scale[:, None, None]).masked_fill(~seen, -math.inf)
    del k
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = _bits(st["v_pages"])[page].view(st["v_pages"].dtype).flatten(1, 2).float().permute(0, 2, 1, 3).contiguous()  # [B][Hk][L][D]
    v = torch.where(seen.transpose(-1, -2), v, 0.0)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    if st["v_scale"] is not None:
        o = o * st["v_scale"][:, None, None]
    st["out"].copy_(o.reshape(B, H, D))
    return st["out"]


def _counts(st, case, from_prompt_end):
    """How often each token id is in the history of each row, [B][V]."""
    h = st["history"].long()
    at = torch.arange(h.shape[1], device="cuda")
    here = (at < st["history_lengths"].long()[:, None]) & (h >= 0) & (h < case["vocab"])
    if from_prompt_end:
        here = here & (at >= st["prompt_lengths"].long()[:, None])
    out = torch.zeros(case["rows"], case["vocab"], dtype=torch.int32, device="cuda")
    return out.scatter_add_(1, torch.where(here, h, 0), here.int())


def _plain_logits(st, case):
    V = case["vocab"]
    x = st["logits"].float()
    rep = st["repetition"][:, None]
    x = torch.where(_counts(st, case, False) > 0, torch.where(x > 0, x / rep, x * rep), x)
    made = _counts(st, case, True)
    x = x - st["frequency"][:, None] * made.float()
    x = x - st["presence"][:, None] * (made > 0).float()
    if st["bias_ids"] is not None:
        m = st["bias_ids"].shape[1]
        given = torch.arange(m, device="cuda") < st["bias_counts"].long()[:, None]
        bias = torch.zeros(case["rows"], V + 1, device="cuda")
        bias.scatter_(1, torch.where(given, st["bias_ids"].long(), V), st["bias_values"])
        x = x + bias[:, :V]
    ids = torch.arange(V, device="cuda")
    if st["mask"] is not None:
        allowed = (st["mask"][:, ids >> 5] >> (ids & 31).int()) & 1
        x = x.masked_fill(allowed == 0, -math.inf)
    top = x.amax(1, keepdim=True)
    first = torch.where(x == top, ids, V).amin(1)
    st["next_token"].copy_(torch.where(top[:, 0] == -math.inf, -1, first))
    st["out"].copy_(x)
    return st["out"], st["next_token"]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "logits":
        n = case["rows"] * case["vocab"]
        hist = case["rows"] * case["history"] * 3 // 4
        return {"bytes": 2 * n * ITEM[case["dtype"]] + 4 * hist
                + (n // 8 if case["masked"] else 0) + 4 * case["rows"] * case["biases"],
                "flops": 6 * n}
    item, kept = ITEM[case["dtype"]], ITEM[case["cache"]]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        n = case["tokens"]
        return {"bytes": n * D * (2 * H * item + 2 * Hk * (item + kept)),
                "flops": 3 * n * (H + Hk) * case["rotary"]}
    lo, hi = case["shortest"], case["longest"]
    # The mean length: half of the rows spread over the logarithm, half evenly.
    log_mean = (hi - lo) / max(1e-9, math.log(hi + 1) - math.log(lo + 1)) if hi > lo else hi
    mean = (log_mean + (lo + hi) / 2) / 2
    keys = hi + (case["rows"] - 1) * mean
    if case["window"]:
        keys = min(keys, case["rows"] * min(case["window"], hi))
    keys = int(keys)
    return {"bytes": 2 * keys * Hk * D * kept + 2 * case["rows"] * H * D * item,
            "flops": 4 * keys * H * D}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(st, case)
    if case["kind"] == "attend":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        for row, n in enumerate(st["lengths"].tolist()):
            first = max(0, n - case["window"]) if case["window"] else 0
            if first < n:
                out[row] = _exact_row(st, case, row, first, n)
        return out
    x = st["logits"].double().cpu().numpy()
    host = {k: v.cpu().numpy() for k, v in st.items() if isinstance(v, torch.Tensor)
            and k not in ("logits", "out", "workspace")}
    token = np.empty(case["rows"], np.int64)
    for b in range(case["rows"]):
        _exact_logits_row(x[b], host, b)
        token[b] = x[b].argmax() if x[b].max() > -np.inf else -1
    return torch.from_numpy(x), torch.from_numpy(token)


def _exact_append(st, case):
    R, half = case["rotary"], case["rotary"] // 2
    freq = torch.tensor([ROPE_BASE ** (-2.0 * i / R) for i in range(half)], dtype=torch.float64,
                        device="cuda")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(case["tokens"], half),
                       st["positions"].double()[:, None] * freq)[:, None, :]
    if case["interleaved"]:
        ia, ib = torch.arange(0, R, 2, device="cuda"), torch.arange(1, R, 2, device="cuda")
    else:
        ia, ib = torch.arange(half, device="cuda"), torch.arange(half, R, device="cuda")

    def turned(x):
        x = x.double().clone()
        z = torch.complex(x[..., ia], x[..., ib]) * turn
        x[..., ia], x[..., ib] = z.real, z.imag
        return x

    q, k, v = turned(st["q"]), turned(st["k"]), st["v"].double()
    kp, vp = st["k_pages"].double(), st["v_pages"].double()
    if st["k_scale"] is not None:
        k = (k / st["k_scale"].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        v = (v / st["v_scale"].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    seq, pos, table = (st[x].cpu().numpy() for x in ("seqs", "positions", "table"))
    at = torch.from_numpy(table[seq, pos // case["page"]].astype(np.int64) * case["page"]
                          + pos % case["page"]).cuda()
    kp.flatten(0, 1)[at] = k
    vp.flatten(0, 1)[at] = v
    return q, kp, vp


def _exact_row(st, case, row, first, n):
    """One row's attention over the keys first .. n - 1, [H][D]."""
    ps, Hk = case["page"], case["kv_heads"]
    pages = st["table"][row, first // ps:(n - 1) // ps + 1].long()
    part = slice(first % ps, first % ps + n - first)

    def values(which):
        x = _bits(st[which + "_pages"])[pages].view(st[which + "_pages"].dtype)
        x = x.flatten(0, 1)[part].double()                              # [keys][Hk][D]
        s = st[which + "_scale"]
        return x if s is None else x * s.double()[:, None]

    q = st["q"][row].double().view(Hk, -1, case["dim"])                 # [Hk][G][D]
    k = values("k").permute(1, 2, 0).contiguous()
    w = torch.softmax(torch.matmul(q, k) / math.sqrt(case["dim"]), -1)
    return torch.matmul(w, values("v").permute(1, 0, 2).contiguous()).flatten(0, 1)


def _exact_logits_row(row, host, b):
    past = host["history"][b, :host["history_lengths"][b]]
    seen = np.unique(past)
    rep = float(host["repetition"][b])
    row[seen] = np.where(row[seen] > 0, row[seen] / rep, row[seen] * rep)
    made, times = np.unique(past[host["prompt_lengths"][b]:], return_counts=True)
    row[made] -= float(host["frequency"][b]) * times + float(host["presence"][b])
    if "bias_ids" in host:
        m = host["bias_counts"][b]
        row[host["bias_ids"][b, :m]] += host["bias_values"][b, :m].astype(np.float64)
    if "mask" in host:
        bits = np.unpackbits(host["mask"][b].view(np.uint8), bitorder="little")[:len(row)]
        row[bits == 0] = -np.inf
