"""Attention of a transformer with its positions and its cache, as cases that can be timed and compared: the plain forms in
torch, or, with `own` set, the calls of the library's binding.

A case is one of five kinds:

  rope       rotary positions on a tensor of heads, half or interleaved pairs, a part of the head, forward or backward
  append     the keys and values of new tokens of a ragged batch into the pages of a cache
  attention  fused attention of whole sequences: causal, window, document and prefix masks, capped scores, distance bias
  train      the same with its backward pass
  cache      attention of the newest tokens of every sequence (one, or a chunk) over a paged cache

The rows of `starts` behind the last sequence stand for a serving batch that is padded to a fixed number of tokens: their
outputs are left as they were.  Lengths follow from the case alone, in an order that follows from the seed.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _rope(name, dtype, batch, heads, seq, dim, rotary, interleaved=False, inverse=False, factor=1.0, far=0):
    return dict(name=name, kind="rope", dtype=dtype, batch=batch, heads=heads, seq=seq, dim=dim, rotary=rotary,
                interleaved=interleaved, inverse=inverse, factor=factor, far=far)


def _append(name, dtype, seqs, new_low, new_high, old_high, heads, dim, page):
    return dict(name=name, kind="append", dtype=dtype, seqs=seqs, new_low=new_low, new_high=new_high, old_high=old_high,
                heads=heads, dim=dim, page=page)


def _attention(name, kind, dtype, batch, heads, kv_heads, seq, keys, dim, causal=True, window=0, softcap=0.0, slopes=False,
               documents=0, prefix=0):
    return dict(name=name, kind=kind, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, seq=seq, keys=keys, dim=dim,
                causal=causal, window=window, softcap=softcap, slopes=slopes, documents=documents, prefix=prefix)


def _cache(name, dtype, seqs, new_low, new_high, old_low, old_high, heads, kv_heads, dim, page, window=0, softcap=0.0,
           slopes=False):
    return dict(name=name, kind="cache", dtype=dtype, seqs=seqs, new_low=new_low, new_high=new_high, old_low=old_low,
                old_high=old_high, heads=heads, kv_heads=kv_heads, dim=dim, page=page, window=window, softcap=softcap,
                slopes=slopes)


def listed():
    return [
        # the query and key heads of one decoding step of 32 sequences at far positions: latency
        _rope("rope_decode", "bf16", 1, 40, 32, 128, 128, far=100000),
        # the same heads of a long prompt whose frequencies are scaled for it: memory
        _rope("rope_prompt_scaled", "bf16", 1, 40, 16384, 128, 128, factor=8.0),
        # the gradient of interleaved pairs in half of the head, fp32, odd length
        _rope("rope_backward_f32", "f32", 4, 12, 1021, 64, 32, interleaved=True, inverse=True),
        # one token of each of 128 sequences into pages of 16
        _append("append_decode", "bf16", 128, 1, 1, 4000, 8, 128, 16),
        # prompts of unequal lengths, some behind a cached beginning, into pages of 64
        _append("append_prompts", "f16", 24, 1, 4001, 700, 12, 64, 64),
        # the heads of BERT-base at its short sequence length, no mask: latency
        _attention("attention_encoder", "attention", "f16", 1, 12, 12, 128, 128, 64, causal=False),
        # a prompt with grouped heads and capped scores
        _attention("attention_prompt_capped", "attention", "bf16", 1, 32, 8, 4096, 4096, 128, softcap=50.0),
        # a training step of packed documents of unequal lengths
        _attention("train_documents", "train", "bf16", 2, 16, 4, 4096, 4096, 128, documents=7),
        # a training step with a bidirectional prefix and a bias by distance, odd length
        _attention("train_prefix_slopes", "train", "f16", 3, 12, 12, 1021, 1021, 64, slopes=True, prefix=200),
        # one decoding step of 64 sequences of unequal lengths: memory
        _cache("cache_decode", "bf16", 64, 1, 1, 100, 8000, 32, 8, 128, 16),
        # one decoding step of one long sequence: the keys are all there is to split
        _cache("cache_decode_long", "f16", 1, 1, 1, 131000, 131000, 16, 2, 128, 64, slopes=True),
        # chunks of four prompts over what is cached of them, with a window and capped scores
        _cache("cache_chunks_window", "bf16", 4, 37, 512, 1000, 15000, 32, 8, 128, 32, window=4096, softcap=30.0),
    ]


def _log(rng, low, high):
    """A whole number between `low` and `high`, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("rope", "append", "attention", "attention", "train", "train", "cache", "cache", "cache"))
    if kind == "rope":
        dim = 8 * rng.randint(4, 16)
        heads, batch = rng.randint(1, 48), rng.randint(1, 4)
        return dict(kind=kind, dtype=rng.choice(("f32", "f16", "bf16")), batch=batch, heads=heads,
                    seq=_log(rng, 1, max(2, 60000000 // (heads * batch * dim))), dim=dim,
                    rotary=dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2), interleaved=rng.random() < 0.5,
                    inverse=rng.random() < 0.5, factor=rng.choice((1.0, 4.0, 32.0)), far=_log(rng, 1, 1000000))
    if kind == "append":
        seqs, heads, dim = _log(rng, 1, 256), rng.randint(1, 16), 8 * rng.randint(4, 16)
        return dict(kind=kind, dtype=rng.choice(("f16", "bf16", "f32")), seqs=seqs, new_low=1,
                    new_high=_log(rng, 1, max(2, 30000000 // (seqs * heads * dim))), old_high=_log(rng, 1, 3000), heads=heads,
                    dim=dim, page=rng.choice((1, 8, 16, 24, 64, 256)))
    group, kv_heads = rng.choice((1, 1, 2, 4, 7, 8)), rng.choice((1, 2, 3, 4, 8))
    dim = rng.choice((64, 64, 128, 128, 40, 80, 96, 112))
    softcap, slopes = rng.choice((0.0, 0.0, 20.0, 50.0)), rng.random() < 0.3
    if kind == "cache":
        seqs = _log(rng, 1, 64)
        chunk = rng.random() < 0.4
        old = _log(rng, 16, min(130000, (50000 if chunk else 250000) // seqs))
        new = rng.choice((1, 1, 1, 2, 4))
        if chunk:
            new = _log(rng, 2, max(3, min(1024, 300000000 // (seqs * old * group * kv_heads), 30000 // seqs)))
        return dict(kind=kind, dtype=rng.choice(("f16", "bf16")), seqs=seqs, new_low=rng.randint(1, new), new_high=new,
                    old_low=rng.randint(0, old), old_high=old, heads=group * kv_heads, kv_heads=kv_heads, dim=dim,
                    page=rng.choice((8, 16, 32, 64, 100, 256)), window=rng.choice((0, 0, _log(rng, 1, 2 * old))),
                    softcap=softcap, slopes=slopes)
    mask = rng.choice(("full", "causal", "causal", "window", "documents", "prefix"))
    heads = group * kv_heads
    batch = rng.randint(1, 4)
    most = int(math.sqrt((2.5e8 if kind == "train" else 5e8) / (heads * batch)))
    seq = _log(rng, 1, min(8192, most))
    keys = seq
    if kind == "attention" and mask not in ("documents", "prefix") and rng.random() < 0.4:
        keys = seq + _log(rng, 1, max(1, most - seq) + 1)
    causal = mask in ("causal", "prefix") or (mask != "full" and rng.random() < 0.5)
    return dict(kind=kind, dtype=rng.choice(("f16", "bf16")), batch=batch, heads=heads, kv_heads=kv_heads, seq=seq, keys=keys,
                dim=dim, causal=causal, window=_log(rng, 1, keys) if mask == "window" else 0, softcap=softcap, slopes=slopes,
                documents=rng.randint(1, min(9, seq)) if mask == "documents" else 0,
                prefix=_log(rng, 1, keys) if mask == "prefix" else 0)


def _spread(count, low, high):
    """`count` lengths from `low` to `high`."""
    return [high - (high - low) * i // max(1, count - 1) for i in range(count)]


def _document_lengths(case):
    """Lengths of the documents of a row, in the proportions 1 : 2 : ... and at least one token each."""
    n, seq = case["documents"], case["seq"]
    cuts = [max(i, seq * i * (i + 1) // (n * (n + 1))) for i in range(n)] + [seq]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _slope_values(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _lengths(case):
    """(new tokens, tokens in the cache with them) of every sequence of an append or cache case."""
    new = _spread(case["seqs"], case["new_low"], case["new_high"])
    old = _spread(case["seqs"], case.get("old_low", 0), case["old_high"])
    return [(n, n + o) for n, o in zip(new, reversed(old))]


def _shuffled(values, seed):
    order = torch.randperm(len(values), generator=torch.Generator().manual_seed(seed)).tolist()
    return [values[i] for i in order]


def prepare(case, seed):
    device, dtype = torch.device("cuda"), DTYPES[case["dtype"]]
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device, dtype=torch.float32).to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=device)

    s = dict(case=case)
    if case["kind"] == "rope":
        # tokens of a projection's output, [batch][token][head][dim], seen as [batch][head][token][dim]
        x = normal(case["batch"], case["seq"], case["heads"], case["dim"])
        s["x"], s["y"] = x.transpose(1, 2), torch.empty_like(x).transpose(1, 2)
        at = torch.randint(0, max(1, case["far"]), (case["batch"], 1), generator=g, device=device)
        s["positions"] = (at + torch.arange(case["seq"], device=device)).to(torch.int32)
        pair = torch.arange(case["rotary"] // 2, device=device, dtype=torch.float64)
        s["frequencies"] = 10000.0 ** (-2.0 * pair / case["rotary"]) / case["factor"]
        s["amplitude"] = 0.1 * math.log(case["factor"]) + 1.0
        return s
    if case["kind"] in ("append", "cache"):
        lengths = _shuffled(_lengths(case), seed)
        total, page, dim = sum(n for n, _ in lengths), case["page"], case["dim"]
        tokens = total + total % 3  # (a batch padded by up to two tokens)
        kv_heads = case.get("kv_heads", case["heads"])
        used = [-(-length // page) for _, length in lengths]
        width, pages = max(used), sum(used) + 3
        s["k_pages"], s["v_pages"] = normal(pages, page, kv_heads, dim), normal(pages, page, kv_heads, dim)
        taken = torch.randperm(pages, generator=torch.Generator().manual_seed(seed + 1))
        tables = torch.full((case["seqs"], width), -1, dtype=torch.int32)
        at = 0
        for row, n in enumerate(used):
            tables[row, :n] = taken[at:at + n]
            at += n
        s["tables"], s["lengths"] = tables.to(device), ints([length for _, length in lengths])
        starts = [0]
        for n, _ in lengths:
            starts.append(starts[-1] + n)
        s["starts"], s["total"], s["max_new"] = ints(starts), total, max(n for n, _ in lengths)
        # of every new token: its sequence, its place among the sequence's new tokens, its position
        token = torch.arange(total, device=device)
        s["sequence"] = torch.searchsorted(s["starts"][1:].contiguous(), token.to(torch.int32), right=True)
        s["place"] = token - s["starts"][s["sequence"]]
        s["position"] = s["lengths"][s["sequence"]] - (s["starts"][1:] - s["starts"][:-1])[s["sequence"]] + s["place"]
        if case["kind"] == "append":
            s["k"], s["v"] = normal(tokens, kv_heads, dim), normal(tokens, kv_heads, dim)
        else:
            s["q"] = normal(tokens, case["heads"], dim)
            s["out"] = torch.zeros_like(s["q"])
            s["slopes"] = torch.tensor(_slope_values(case["heads"]), device=device) if case["slopes"] else None
        return s
    b, h, hk, n, m, d = (case[x] for x in ("batch", "heads", "kv_heads", "seq", "keys", "dim"))
    # projections' outputs, [batch][token][head][dim], seen as [batch][head][token][dim]
    s["q"], s["k"], s["v"] = (normal(b, t, u, d).transpose(1, 2) for t, u in ((n, h), (m, hk), (m, hk)))
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((b, h, n), device=device)
    s["slopes"] = torch.tensor(_slope_values(h), device=device) if case["slopes"] else None
    s["documents"] = s["prefix"] = None
    if case["documents"]:
        rows = [_shuffled(_document_lengths(case), seed + i) for i in range(b)]
        s["documents"] = ints([[i for i, length in enumerate(row) for _ in range(length)] for row in rows])
    if case["prefix"]:
        s["prefix"] = ints(_shuffled(_spread(b, max(1, case["prefix"] // 2), case["prefix"]), seed))
    if s["documents"] is not None or s["prefix"] is not None:
        s["ranges"] = torch.empty((b, n, 2), dtype=torch.int32, device=device)
    if case["kind"] == "train":
        s["grad_out"] = normal(b, n, h, d).transpose(1, 2)
        s["grad_q"], s["grad_k"], s["grad_v"] = (torch.empty_like(s[x]) for x in ("q", "k", "v"))
    return s


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["kind"] == "rope":
        return _plain_rope(state, case)
    if case["kind"] == "append":
        page = state["position"] // case["page"]
        slot = state["tables"][state["sequence"], page].long() * case["page"] + state["position"] % case["page"]
        state["k_pages"].flatten(0, 1)[slot] = state["k"][:state["total"]]
        state["v_pages"].flatten(0, 1)[slot] = state["v"][:state["total"]]
        return state["k_pages"], state["v_pages"]
    if case["kind"] == "cache":
        return _plain_cache(state, case)
    return _plain_attention(state, case)


def _run_own(s, case):
    from paper_2210_09603_amd import binding as hb

    if case["kind"] == "rope":
        hb.hidet_rope(s["x"], s["y"], s["frequencies"], positions=s["positions"], interleaved=case["interleaved"],
                      inverse=case["inverse"], amplitude=s["amplitude"])
        return s["y"]
    if case["kind"] in ("append", "cache"):
        if "cache" not in s:  # the cache's descriptor and the workspace, which a serving loop keeps
            s["cache"] = hb.make_cache(s["k_pages"], s["v_pages"], s["tables"], s["lengths"])
            if case["kind"] == "cache":
                size = hb.hidet_cache_attention_workspace_bytes(s["cache"], s["q"], s["max_new"])
                s["workspace"] = torch.empty(size, dtype=torch.uint8, device=s["q"].device)
        if case["kind"] == "append":
            hb.hidet_cache_append(s["cache"], s["k"], s["v"], s["starts"], s["max_new"])
            return s["k_pages"], s["v_pages"]
        hb.hidet_cache_attention(s["cache"], s["q"], s["out"], s["starts"], s["max_new"], window=case["window"],
                                 softcap=case["softcap"], slopes=s["slopes"], workspace=s["workspace"])
        return s["out"]
    train = case["kind"] == "train"
    if "workspace" not in s:
        size = hb.hidet_attention_workspace_bytes(s["q"], s["k"])
        if train:
            size = max(size, hb.hidet_attention_backward_workspace_bytes(s["q"], s["k"]))
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=s["q"].device)
    mask = dict(causal=case["causal"], window=case["window"])
    if "ranges" in s:
        hb.hidet_attention_ranges(s["ranges"], keys=case["keys"], documents=s["documents"], prefix=s["prefix"], **mask)
        mask = dict(ranges=s["ranges"])
    mask.update(softcap=case["softcap"], slopes=s["slopes"], workspace=s["workspace"])
    hb.hidet_attention(s["q"], s["k"], s["v"], s["out"], lse=s["lse"], **mask)
    if not train:
        return s["out"], s["lse"]
    hb.hidet_attention_backward(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["grad_q"], s["grad_k"],
                                s["grad_v"], **mask)
    return s["out"], s["lse"], s["grad_q"], s["grad_k"], s["grad_v"]


def _plain_rope(s, case):
    # far positions lose their angle in 32 bits
    angle = s["positions"].double()[:, None, :, None] * s["frequencies"]
    if case["inverse"]:
        angle = -angle
    cos, sin = (angle.cos() * s["amplitude"]).float(), (angle.sin() * s["amplitude"]).float()
    x, r = s["x"].float(), case["rotary"]
    y = x.clone()
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    return y.to(s["x"].dtype)


def _visible(s, case, device):
    """[batch or 1][1][query][key]: which keys a query sees."""
    at = torch.arange(case["keys"] - case["seq"], case["keys"], device=device)[:, None]
    key = torch.arange(case["keys"], device=device)[None, :]
    see = (key <= at) if case["causal"] else torch.ones((case["seq"], case["keys"]), dtype=torch.bool, device=device)
    if case["window"]:
        see = see & ((at - key).abs() < case["window"])
    see = see[None]
    if s["prefix"] is not None:
        see = see | (key[None] < s["prefix"][:, None, None])
    if s["documents"] is not None:
        of = s["documents"]
        see = see & (of[:, -case["seq"]:, None] == of[:, None, :])
    return see[:, None], (at - key).abs().float()


def _plain_attention(s, case):
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = torch.matmul(q, k.transpose(2, 3)) * scale
    if case["softcap"]:
        t = torch.tanh(x / case["softcap"])
        x = t * case["softcap"]
    see, distance = _visible(s, case, x.device)
    if s["slopes"] is not None:
        x = x - s["slopes"][:, None, None] * distance
    x = x.masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, v)
    if case["kind"] == "attention":
        return out.to(s["q"].dtype), lse
    dout = s["grad_out"].float()
    dv = torch.matmul(p.transpose(2, 3), dout)
    dx = p * (torch.matmul(dout, v.transpose(2, 3)) - (dout * out).sum(-1, keepdim=True))
    if case["softcap"]:
        dx = dx * (1 - t * t)
    dq = torch.matmul(dx, k) * scale
    dk = torch.matmul(dx.transpose(2, 3), q) * scale
    dk, dv = (x.unflatten(1, (case["kv_heads"], group)).sum(2) for x in (dk, dv))
    out, dq, dk, dv = (x.to(s["q"].dtype) for x in (out, dq, dk, dv))
    return out, lse, dq, dk, dv


def _plain_cache(s, case):
    group, scale, seqs = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"]), case["seqs"]
    tables = s["tables"].clamp(min=0).long()
    k, v = (x[tables].flatten(1, 2).transpose(1, 2).float() for x in (s["k_pages"], s["v_pages"]))  # [seq][head][position][dim]
    q = torch.zeros((seqs, s["max_new"], case["heads"], case["dim"]), device=k.device)
    q[s["sequence"], s["place"]] = s["q"][:s["total"]].float()
    q = q.unflatten(2, (case["kv_heads"], group)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [seq][kv head][group * place][dim]
    x = torch.matmul(q, k.transpose(2, 3)).unflatten(2, (group, s["max_new"])) * scale
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    new = s["starts"][1:] - s["starts"][:-1]
    at = (s["lengths"] - new)[:, None] + torch.arange(s["max_new"], device=k.device)
    gap = at[:, :, None] - torch.arange(k.shape[2], device=k.device)  # [seq][place][key]
    see = gap >= 0
    if case["window"]:
        see = see & (gap < case["window"])
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, case["kv_heads"], group, 1, 1) * gap[:, None, None].float()
    p = torch.softmax(x.masked_fill(~see[:, None, None], -math.inf), -1)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (group, s["max_new"]))
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)  # [seq][place][head][dim]
    s["out"][:s["total"]] = out[s["sequence"], s["place"]].to(s["q"].dtype)
    return s["out"]


def _pairs(case):
    """Visible (query, key) pairs of one head, over the batch or over all sequences."""
    if case["kind"] == "cache":
        pairs = 0
        for n, length in _lengths(case):
            for at in range(length - n, length):
                pairs += min(at + 1, case["window"]) if case["window"] else at + 1
        return pairs
    n, m = case["seq"], case["keys"]
    if case["documents"]:
        return case["batch"] * sum(x * (x + 1) // 2 if case["causal"] else x * x for x in _document_lengths(case))
    if case["prefix"]:
        return sum(max(min(p, m), m - n + i + 1) for p in _spread(case["batch"], max(1, case["prefix"] // 2), case["prefix"]) for i in range(n))
    pairs = 0
    for at in range(m - n, m):
        w = case["window"] or m
        pairs += at + 1 - max(0, at + 1 - w) + (0 if case["causal"] else min(m, at + w) - at - 1)
    return case["batch"] * pairs


def work(case):
    e, kind = BYTES[case["dtype"]], case["kind"]
    if kind == "rope":
        n = case["batch"] * case["heads"] * case["seq"] * case["dim"]
        return {"bytes": 2 * n * e + 4 * case["batch"] * case["seq"], "flops": 3 * n}
    if kind == "append":
        return {"bytes": 4 * sum(n for n, _ in _lengths(case)) * case["heads"] * case["dim"] * e, "flops": 0}
    if kind == "cache":
        tokens = sum(n for n, _ in _lengths(case))
        seen = sum(min(length, n - 1 + case["window"]) if case["window"] else length for n, length in _lengths(case))
        return {"bytes": (2 * seen * case["kv_heads"] + 2 * tokens * case["heads"]) * case["dim"] * e,
                "flops": 4 * _pairs(case) * case["heads"] * case["dim"]}
    rows, keys = case["batch"] * case["heads"] * case["seq"], case["batch"] * case["kv_heads"] * case["keys"]
    pairs = _pairs(case) * case["heads"]
    size = (2 * rows + 2 * keys) * case["dim"] * e + 4 * rows
    if kind == "attention":
        return {"bytes": size, "flops": 4 * pairs * case["dim"]}
    return {"bytes": size + (2 * rows + 2 * keys) * case["dim"] * e, "flops": 14 * pairs * case["dim"]}


# ---- the definitions, in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(s, case)
    if case["kind"] == "append":
        return _exact_append(s, case)
    if case["kind"] == "cache":
        return _exact_cache(s, case)
    return _exact_attention(s, case)


def _exact_rope(s, case):
    """Every pair as a complex number times amplitude * exp(i * angle)."""
    x, half = s["x"].double(), case["rotary"] // 2
    y = x.clone()
    for j in range(half):
        angle = s["positions"].double() * s["frequencies"][j] * (-1.0 if case["inverse"] else 1.0)
        turn = torch.polar(torch.full_like(angle, s["amplitude"]), angle)[:, None]
        first, second = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + half)
        z = torch.complex(x[..., first], x[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(s, case):
    k, v = s["k_pages"].double(), s["v_pages"].double()
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    tables = s["tables"].tolist()
    for row, length in enumerate(lengths):
        n, done = starts[row + 1] - starts[row], 0
        while done < n:
            at = length - n + done
            page, slot = divmod(at, case["page"])
            count = min(case["page"] - slot, n - done)
            token = starts[row] + done
            k[tables[row][page], slot:slot + count] = s["k"][token:token + count].double()
            v[tables[row][page], slot:slot + count] = s["v"][token:token + count].double()
            done += count
    return k, v


def _exact_rows(case, q, k, v, see, distance, slope):
    """One head in 64 bits: (probabilities, derivative of the cap, log of the sum, output); rows that see nothing are zero."""
    x = q @ k.T / math.sqrt(case["dim"])
    cap = torch.ones_like(x)
    if case["softcap"]:
        t = torch.tanh(x / case["softcap"])
        x, cap = case["softcap"] * t, 1 - t * t
    if slope is not None:
        x = x - slope * distance
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, 1)
    p = torch.where(see, torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None]), torch.zeros_like(x))
    return p, cap, lse, p @ v


def _exact_cache(s, case):
    out = s["out"].double()
    starts, lengths, group = s["starts"].tolist(), s["lengths"].tolist(), case["heads"] // case["kv_heads"]
    for row, length in enumerate(lengths):
        first, last = starts[row], starts[row + 1]
        pages = s["tables"][row, :-(-length // case["page"])].long()
        at = torch.arange(length - (last - first), length, device=out.device)[:, None]
        gap = at - torch.arange(length, device=out.device)[None]
        see = (gap >= 0) & ((gap < case["window"]) if case["window"] else True)
        for kv in range(case["kv_heads"]):
            k = s["k_pages"][pages, :, kv].flatten(0, 1)[:length].double()
            v = s["v_pages"][pages, :, kv].flatten(0, 1)[:length].double()
            for h in range(kv * group, (kv + 1) * group):
                slope = float(s["slopes"][h]) if case["slopes"] else None
                out[first:last, h] = _exact_rows(case, s["q"][first:last, h].double(), k, v, see, gap.double(), slope)[3]
    return out


def _exact_attention(s, case):
    n, m, group = case["seq"], case["keys"], case["heads"] // case["kv_heads"]
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device), s["lse"].double()
    dq, dk, dv = torch.zeros_like(out), torch.zeros(s["k"].shape, dtype=torch.float64, device=out.device), None
    dv = torch.zeros_like(dk)
    at = torch.arange(m - n, m, device=out.device)[:, None]
    key = torch.arange(m, device=out.device)[None]
    for b in range(case["batch"]):
        see = (at - key >= 0) if case["causal"] else torch.ones((n, m), dtype=torch.bool, device=out.device)
        if case["window"]:
            see = see & (at - key < case["window"]) & (key - at < case["window"])
        if case["prefix"]:
            see = see | (key < s["prefix"][b])
        if case["documents"]:
            see = see & (s["documents"][b][:, None] == s["documents"][b][None])
        for h in range(case["heads"]):
            q, k, v = s["q"][b, h].double(), s["k"][b, h // group].double(), s["v"][b, h // group].double()
            slope = float(s["slopes"][h]) if case["slopes"] else None
            p, cap, lse[b, h], out[b, h] = _exact_rows(case, q, k, v, see, (at - key).abs().double(), slope)
            if case["kind"] == "train":
                g = s["grad_out"][b, h].double()
                dx = p * (g @ v.T - (g * out[b, h]).sum(1, keepdim=True)) * cap / math.sqrt(case["dim"])
                dq[b, h] = dx @ k
                dk[b, h // group] += dx.T @ q
                dv[b, h // group] += p.T @ g
    return (out, lse) if case["kind"] == "attention" else (out, lse, dq, dk, dv)
