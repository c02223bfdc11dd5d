"""Performance cases of the operators around a key/value cache: what makes its rows and what keeps it small.

Four operators, all through the public entry points of `binding`:

  rope   swaa_qk_norm_rope: RMS norms of the heads of queries and keys, and the position rotation, in one pass; while
         serving, the keys and values go straight into the (paged) cache that the attention calls read
  grad   swaa_qk_norm_rope_bwd: from the gradients that swaa_attn_bwd returns to those of the projections and the norms
  weigh  swaa_attn_key_weights: the attention weight that each cached key has got from the query rows of a call
  evict  swaa_cache_evict: the lightest rows of a cache leave it, the others close up

A case is a dict of plain values.  Sequence lengths of a batch are drawn from the case's own `lengths` number, so that
work(case) knows them without the inputs.  Where `own` is false, run() computes the operators in plain torch operations.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16  # tokens per page of a paged cache
EPS = 1e-6
BASE = 1e6  # of the rotation's frequencies


def listed():
    """The listed cases."""
    return [
        # one new token of each of 64 sequences (the paper serves batches of 64), into a paged cache whose sequences have lost
        # tokens before: positions are not rows.  A small launch in every layer of every step
        dict(name="rope_decode", kind="rope", form="paged", B=64, rows=1, shortest=30, longest=2000, lengths=1, gone=100000,
             Hq=32, Hkv=8, D=128, rot=128, norm=True, adjacent=False, fp16=False),
        # continuous batching: chunks of prompts of odd lengths packed into one tensor; half of the dimensions rotate
        dict(name="rope_packed", kind="rope", form="packed", B=9, rows=0, shortest=50, longest=1500, lengths=2, gone=0,
             Hq=40, Hkv=8, D=128, rot=64, norm=True, adjacent=False, fp16=True),
        # the prompt of a training step or a prefill, projections in [B, N, H, D] order
        dict(name="rope_prompt", kind="rope", form="prompt", B=1, rows=16384, shortest=0, longest=0, lengths=0, gone=0,
             Hq=32, Hkv=8, D=128, rot=128, norm=True, adjacent=False, fp16=False),
        # backward of a small layer: head dimension 64, an odd length, neighbours as pairs
        dict(name="grad_small", kind="grad", B=3, rows=1021, Hq=8, Hkv=2, D=64, rot=64, norm=True, adjacent=True, fp16=False),
        # backward of the prompt above
        dict(name="grad_prompt", kind="grad", B=1, rows=16384, Hq=32, Hkv=8, D=128, rot=128, norm=True, adjacent=False,
             fp16=False),
        # weights that one new token gives a cache of 128k tokens: a read of the keys
        dict(name="weigh_decode_128k", kind="weigh", form="dense", B=1, rows=1, shortest=131072, longest=131072, lengths=0,
             Hq=32, Hkv=8, D=128, window=131072, n_sink=4, decay=1.0, fp16=False),
        # a serving batch of sequences of very different lengths, paged cache, weights summed up over the steps
        dict(name="weigh_decode_batch", kind="weigh", form="paged", B=16, rows=1, shortest=200, longest=16384, lengths=3,
             Hq=40, Hkv=8, D=128, window=131072, n_sink=4, decay=1.0, fp16=True),
        # the last 64 tokens of a long prompt judge its keys
        dict(name="weigh_last_rows", kind="weigh", form="dense", B=1, rows=64, shortest=32768, longest=32768, lengths=0,
             Hq=32, Hkv=8, D=128, window=131072, n_sink=4, decay=0.0, fp16=False),
        # every row of a prompt counts: a sliding-window layer of the benchmark's mid-sized workload
        dict(name="weigh_prompt", kind="weigh", form="dense", B=1, rows=16384, shortest=16384, longest=16384, lengths=0,
             Hq=32, Hkv=8, D=128, window=2048, n_sink=4, decay=0.0, fp16=False),
        # the same of a full-attention layer, an odd length, five query heads per KV head
        dict(name="weigh_prompt_full", kind="weigh", form="dense", B=1, rows=8001, shortest=8001, longest=8001, lengths=0,
             Hq=40, Hkv=8, D=128, window=131072, n_sink=0, decay=0.0, fp16=False),
        # a decode batch whose sequences are cut back to their budget now and then, a few rows each
        dict(name="evict_step", kind="evict", form="paged", B=16, shortest=900, longest=1152, lengths=5, Hkv=8, D=128, keep=1024,
             n_sink=4, recent=128, fp16=True),
        # a long prompt's cache is cut to a quarter behind the prefill
        dict(name="evict_prompt", kind="evict", form="dense", B=1, shortest=65536, longest=65536, lengths=0, Hkv=8, D=128,
             keep=16384, n_sink=4, recent=1024, fp16=False),
    ]


#: No drawn case needs more operations or bytes than this.
MOST_FLOPS, MOST_BYTES = 1.2e12, 6.5e8


def draw(rng: random.Random):
    """One more case of the ranges that the listed ones stand for."""
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _log(rng, lo, hi):
    """A whole number of [lo, hi], its logarithm uniform; every third one a multiple of 64."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    return max(64, n // 64 * 64) if rng.randrange(3) == 0 and lo >= 64 else n


def _draw(rng):
    kind = rng.choice(("rope", "grad", "weigh", "weigh", "evict"))
    Hq, Hkv = rng.choice(((32, 8), (40, 8), (16, 4), (8, 8), (8, 2)))
    case = dict(kind=kind, Hq=Hq, Hkv=Hkv, D=rng.choice((128, 128, 64)), fp16=rng.random() < 0.4)
    if kind in ("rope", "grad"):
        case.update(rot=rng.choice((case["D"], case["D"], case["D"] // 2)), norm=rng.random() < 0.8, adjacent=rng.random() < 0.3)
    if kind == "rope":
        case.update(form=rng.choice(("paged", "packed", "prompt")), B=rng.choice((1, 2, 7, 32, 96)), rows=rng.choice((1, 1, 2, 5)),
                    shortest=_log(rng, 20, 300), longest=_log(rng, 300, 3500), lengths=rng.randrange(10 ** 6), gone=rng.choice((0, 90000)))
        if case["form"] == "prompt":
            case.update(B=rng.choice((1, 2, 3)), rows=_log(rng, 64, 16384), shortest=0, longest=0, lengths=0, gone=0)
        elif case["form"] == "packed":
            case.update(B=rng.randint(2, 14), rows=0, gone=0)
    elif kind == "grad":
        case.update(B=rng.choice((1, 2, 3)), rows=_log(rng, 64, 16384))
    elif kind == "weigh":
        case.update(D=128, form=rng.choice(("dense", "paged")), decay=rng.choice((0.0, 1.0, 0.9)), n_sink=rng.choice((0, 4, 100)),
                    window=rng.choice((1024, 2048, 131072, 131072)), lengths=rng.randrange(10 ** 6))
        style = rng.choice(("decode", "decode", "last", "prompt"))
        if style == "prompt":
            n = _log(rng, 100, 12000)
            case.update(form="dense", B=rng.choice((1, 1, 2)), rows=n, shortest=n, longest=n, D=rng.choice((128, 64)))
        elif style == "last":
            n = _log(rng, 1000, 40000)
            case.update(form="dense", B=rng.choice((1, 2)), rows=rng.choice((16, 33, 64, 200)), shortest=n, longest=n)
        else:
            case.update(B=rng.choice((1, 2, 8, 31)), rows=rng.choice((1, 1, 1, 4)), shortest=_log(rng, 100, 1000),
                        longest=_log(rng, 1000, 65536))
            if case["form"] == "dense":
                case["shortest"] = case["longest"]
    else:
        case.update(form=rng.choice(("dense", "paged")), B=rng.choice((1, 2, 5, 24)), longest=_log(rng, 300, 65536),
                    lengths=rng.randrange(10 ** 6), n_sink=rng.choice((0, 4, 100)))
        case["shortest"] = case["longest"] if case["form"] == "dense" else max(200, case["longest"] // rng.choice((2, 10)))
        case["recent"] = _log(rng, 8, max(9, case["longest"] // 8))
        case["keep"] = min(case["longest"], case["n_sink"] + case["recent"] + _log(rng, 16, max(17, case["longest"] // 2)))
        case.pop("Hq")
    return case


# ---- sizes ------------------------------------------------------------------------------------------------
def _lengths(case):
    """Cached tokens of each sequence, from [shortest, longest], their logarithms uniform; the longest is there."""
    rng = random.Random(case["lengths"])
    lo, hi = case["shortest"], case["longest"]
    n = [int(round(lo * (hi / lo) ** rng.random())) for _ in range(case["B"])]
    n[-1] = hi
    return n


def _chunks(case):
    """Of packed sequences: how many of the cached tokens are new."""
    rng = random.Random(case["lengths"] + 1)
    return [rng.choice((1, n, n // 2 + 1)) for n in _lengths(case)]


def _pairs(rows, n, window, n_sink):
    """Visible (query, key) pairs of a head: the newest `rows` of n tokens."""
    pos = np.arange(n - rows, n, dtype=np.int64)
    first = np.maximum(pos - window + 1, 0)
    return int((pos + 1 - first + np.minimum(first, n_sink)).sum())


def work(case):
    """Bytes and operations that one pass cannot do without."""
    Hkv, D, kind = case["Hkv"], case["D"], case["kind"]
    if kind in ("rope", "grad"):
        Hq = case["Hq"]
        tokens = sum(_chunks(case)) if case.get("form") == "packed" else case["B"] * case["rows"]
        heads = Hq + Hkv + (Hkv if case.get("form", "prompt") != "prompt" else 0)
        sides = 2 if kind == "rope" else 3
        return {"bytes": tokens * heads * D * 2 * sides, "flops": tokens * (Hq + Hkv) * D * (10 if kind == "rope" else 20)}
    if kind == "weigh":
        Hq, rows = case["Hq"], case["rows"]
        data = flops = 0
        for n in _lengths(case):
            keys = n if rows + case["window"] >= n else min(n, rows + case["window"] - 1 + case["n_sink"])
            data += rows * Hq * (D * 2 + 4) + keys * Hkv * D * 2 + n * Hkv * (8 if case["decay"] else 4)
            flops += Hq * _pairs(rows, n, case["window"], case["n_sink"]) * (2 * D + 3)
        return {"bytes": data, "flops": flops}
    data = 0
    for n in _lengths(case):
        if n > case["keep"]:  # nearly every kept row behind the first few stands behind one that has left
            data += Hkv * (8 * n + 4 * case["keep"] + (case["keep"] - case["n_sink"]) * D * 2 * 2 * 2)
        else:
            data += Hkv * 4 * case["keep"]
    return {"bytes": data, "flops": data // 8}


# ---- inputs -----------------------------------------------------------------------------------------------
def _cache(case, lens, dtype, g):
    """K and V of a cache [B, Hkv, Nk, D], or of pages [pages, Hkv, PAGE, D] in random order with their table."""
    Hkv, D, longest = case["Hkv"], case["D"], max(lens)
    if case["form"] == "dense":
        return [torch.randn(len(lens), Hkv, longest, D, device="cuda", generator=g).to(dtype) for _ in range(2)] + [None]
    per = -(-longest // PAGE)
    count = [-(-n // PAGE) for n in lens]
    pages = sum(count)
    k, v = (torch.randn(pages, Hkv, PAGE, D, device="cuda", generator=g).to(dtype) for _ in range(2))
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(lens), per, dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(count):
        table[b, :c] = order[at:at + c]
        at += c
    return k, v, table


def prepare(case, seed):
    """What a user's program has in hand before the call."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = torch.float16 if case["fp16"] else torch.bfloat16
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    Hkv, D, kind = case["Hkv"], case["D"], case["kind"]
    s = dict(case)
    if kind in ("rope", "grad"):
        Hq, R = case["Hq"], case["rot"]
        s["inv_freq"] = (BASE ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).to(torch.float32).cuda()
        s["q_weight"], s["k_weight"] = [1.0 + 0.2 * rand(D) for _ in range(2)] if case["norm"] else (None, None)
        s["positions"] = None
    if kind == "grad" or (kind == "rope" and case["form"] == "prompt"):
        # one projection's output, [B, N, heads, D]; values are handed to the attention as they are
        qkv = (rand(case["B"], case["rows"], Hq + 2 * Hkv, D) * 1.5).to(dtype)
        s["q"], s["k"] = (t.permute(0, 2, 1, 3) for t in (qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]))
        if kind == "grad":
            s["dq_out"], s["dk_out"] = (rand(case["B"], H, case["rows"], D).to(dtype) for H in (Hq, Hkv))
        return s
    lens = _lengths(case)
    s["lens"] = lens
    if kind == "rope":
        s["k_cache"], s["v_cache"], s["table"] = _cache(dict(case, form="paged"), lens, dtype, g)
        new = _chunks(case) if case["form"] == "packed" else [case["rows"]] * case["B"]
        s["new"] = new
        qkv = (rand(sum(new), Hq + 2 * Hkv, D) * 1.5).to(dtype)
        parts = [t.permute(1, 0, 2) for t in (qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:])]
        if case["form"] == "packed":
            s["cu_q"], s["cu_k"] = (ints([0] + list(np.cumsum(x))) for x in (new, lens))
        else:  # [H, B rows, D] -> [B, H, rows, D]
            parts = [t.unflatten(1, (case["B"], case["rows"])).permute(1, 0, 2, 3) for t in parts]
            s["seq_lens"] = ints(lens)
            if case["gone"]:
                s["positions"] = ints([[case["gone"] * (b + 1) // case["B"] + n - case["rows"] + r for r in range(case["rows"])]
                                       for b, n in enumerate(lens)])
        s["q"], s["k"], s["v"] = parts
        return s
    if kind == "weigh":
        Hq, rows = case["Hq"], case["rows"]
        s["k"], _, s["table"] = _cache(case, lens, dtype, g)
        s["q"] = rand(case["B"], Hq, rows, D).to(dtype)
        s["scale"] = 1.0 / math.sqrt(D)
        s["seq_lens"] = ints(lens) if case["form"] == "paged" else None
        s["lse"] = torch.empty(case["B"], Hq, rows, device="cuda")
        for b, h, r0, _, scores in _scores(s):
            s["lse"][b, h, r0:r0 + scores.shape[1]] = torch.logsumexp(scores, -1)
        s["weights"] = rand(case["B"], Hkv, max(lens)).exp() if case["decay"] else torch.zeros(case["B"], Hkv, max(lens), device="cuda")
        return s
    s["k"], s["v"], s["table"] = _cache(case, lens, dtype, g)
    s["seq_lens"] = ints(lens) if case["form"] == "paged" else None
    # few keys get most of the weight, some none at all
    weights = (2.0 * rand(case["B"], Hkv, max(lens))).exp()
    s["weights"] = torch.where(rand(*weights.shape) < -1.5, torch.zeros_like(weights), weights)
    return s


# ---- the operators in plain operations --------------------------------------------------------------------
def _rows_of(cache, table, b, n):
    """The first n rows of sequence b, [Hkv, n, D]."""
    if table is None:
        return cache[b, :, :n]
    t = torch.arange(n, device="cuda")
    return cache[table[b].long()[t // PAGE], :, t % PAGE].permute(1, 0, 2)


def _angles(s, pos):
    a = pos.double()[..., None] * s["inv_freq"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _halves(s, x):
    R = s["rot"]
    return (x[..., 0:R:2], x[..., 1:R:2]) if s["adjacent"] else (x[..., :R // 2], x[..., R // 2:R])


def _joined(s, x1, x2, rest):
    turned = torch.stack((x1, x2), -1).flatten(-2) if s["adjacent"] else torch.cat((x1, x2), -1)
    return torch.cat((turned, rest), -1)


def _norm_rope(s, x, w, cos, sin):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    x1, x2 = _halves(s, x)
    return _joined(s, x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., s["rot"]:])


def _norm_rope_grad(s, dy, x, w, cos, sin):
    x, dy = x.float(), dy.float()
    d1, d2 = _halves(s, dy)
    g = _joined(s, d1 * cos + d2 * sin, d2 * cos - d1 * sin, dy[..., s["rot"]:])
    if w is None:
        return g, None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n, wg = x * r, g * w
    return r * (wg - n * (n * wg).mean(-1, keepdim=True)), (g * n).double().sum((0, 1, 2)).float()


def _scores(s, most=1 << 27):
    """(b, heads, first row, sequence's keys, masked scores [heads of the group, rows, keys]) in 32 bits."""
    rows, G = s["rows"], s["Hq"] // s["Hkv"]
    for b, n in enumerate(s["lens"]):
        keys = _rows_of(s["k"], s["table"], b, n).float()
        step = max(1, most // (G * n))
        for kvh in range(s["Hkv"]):
            heads = slice(kvh * G, kvh * G + G)
            for r0 in range(0, rows, step):
                q = s["q"][b, heads, r0:r0 + step].float()
                end = n - rows + min(r0 + step, rows)  # no row of this part sees a key from here on
                pos = torch.arange(end - q.shape[1], end, device="cuda")[:, None]
                j = torch.arange(end, device="cuda")
                seen = (j <= pos) & ((j > pos - s["window"]) | (j < s["n_sink"]))
                scores = torch.matmul(q, keys[kvh, :end].t()) * s["scale"]
                yield b, heads, r0, kvh, scores.masked_fill_(~seen, -math.inf)


def _plain_rope(s):
    dtype = s["q"].dtype
    if s["form"] == "prompt":
        cos, sin = _angles(s, torch.arange(s["rows"], device="cuda"))
        return [_norm_rope(s, x, w, cos, sin).to(dtype).contiguous() for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"]))]
    packed = s["form"] == "packed"
    row = torch.cat([torch.arange(n - m, n) for n, m in zip(s["lens"], s["new"])]).cuda()
    seq = torch.repeat_interleave(torch.arange(s["B"]), torch.tensor(s["new"])).cuda()
    pos = row if s["positions"] is None else s["positions"].flatten()
    flat = (lambda x: x) if packed else (lambda x: x.permute(1, 0, 2, 3).flatten(1, 2))  # [H, tokens, D]
    cos, sin = _angles(s, pos)
    q, k = (_norm_rope(s, flat(x), w, cos, sin).to(dtype) for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])))
    page, at = s["table"][seq, row // PAGE].long(), row % PAGE
    s["k_cache"][page, :, at] = k.permute(1, 0, 2)
    s["v_cache"][page, :, at] = flat(s["v"]).permute(1, 0, 2)
    return [q if packed else q.unflatten(1, (s["B"], s["rows"])).permute(1, 0, 2, 3).contiguous(), s["k_cache"], s["v_cache"]]


def _plain_grad(s):
    cos, sin = _angles(s, torch.arange(s["rows"], device="cuda"))
    dq, dqw = _norm_rope_grad(s, s["dq_out"], s["q"], s["q_weight"], cos, sin)
    dk, dkw = _norm_rope_grad(s, s["dk_out"], s["k"], s["k_weight"], cos, sin)
    return [dq.to(s["q"].dtype), dk.to(s["k"].dtype)] + ([dqw, dkw] if s["norm"] else [])


def _plain_weigh(s):
    w = s["weights"]
    for b, n in enumerate(s["lens"]):
        w[b, :, :n] = w[b, :, :n] * s["decay"] if s["decay"] else 0.0
    for b, heads, r0, kvh, scores in _scores(s):
        lse = s["lse"][b, heads, r0:r0 + scores.shape[1], None]
        w[b, kvh, :scores.shape[2]] += torch.exp(scores - lse).sum((0, 1))
    return w


def _plain_evict(s):
    keep, n_sink, recent = s["keep"], s["n_sink"], s["recent"]
    w = s["weights"].clone()  # (a program's weights go on from where the call leaves them; here each pass cuts the same ones)
    kept = torch.full((s["B"], s["Hkv"], keep), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(s["lens"]):
        if n <= keep:
            kept[b, :, :n] = torch.arange(n, device="cuda")
            continue
        judged = w[b, :, :n].clone()
        judged[:, :n_sink] = math.inf
        judged[:, n - recent:] = math.inf
        rows = torch.sort(judged, dim=-1, descending=True, stable=True).indices[:, :keep].sort(-1).values
        kept[b] = rows
        heads = torch.arange(s["Hkv"], device="cuda")[:, None]
        w[b, :, :keep] = w[b].gather(1, rows)
        w[b, :, keep:n] = 0
        t = torch.arange(keep, device="cuda")
        for c in (s["k"], s["v"]):
            if s["table"] is None:
                c[b, :, :keep] = c[b][heads, rows]
            else:
                page = s["table"][b].long()
                c[page[t // PAGE], :, t % PAGE] = c[page[rows // PAGE], heads, rows % PAGE].permute(1, 0, 2)
    lens = torch.tensor(s["lens"], dtype=torch.int32, device="cuda").clamp(max=keep)
    return [kept, lens, w, s["k"], s["v"]]


def run(s):
    """One pass through an operator, as a user's program calls it."""
    kind = s["kind"]
    if not own:
        return {"rope": _plain_rope, "grad": _plain_grad, "weigh": _plain_weigh, "evict": _plain_evict}[kind](s)
    from paper_2512_10411_amd import binding
    if kind == "rope":
        how = dict(positions=s["positions"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=s["adjacent"])
        if s["form"] == "prompt":
            return list(binding.swaa_qk_norm_rope(s["q"], s["k"], s["inv_freq"], **how))[:2]
        if s["form"] == "packed":
            how.update(cu_seqlens_q=s["cu_q"], cu_seqlens_k=s["cu_k"], max_seqlen_q=max(s["new"]))
        else:
            how.update(seq_lens=s["seq_lens"])
        return list(binding.swaa_qk_norm_rope(s["q"], s["k"], s["inv_freq"], v=s["v"], k_out=s["k_cache"], v_out=s["v_cache"],
                                              block_table=s["table"], max_seqlen_k=max(s["lens"]), **how))
    if kind == "grad":
        out = binding.swaa_qk_norm_rope_bwd(s["dq_out"], s["dk_out"], s["q"], s["k"], s["inv_freq"], q_weight=s["q_weight"],
                                            k_weight=s["k_weight"], eps=EPS, interleaved=s["adjacent"])
        return list(out if s["norm"] else out[:2])
    if kind == "weigh":
        return binding.swaa_attn_key_weights(s["q"], s["k"], s["lse"], s["window"], s["n_sink"], scale=s["scale"], weights=s["weights"],
                                             decay=s["decay"], seq_lens=s["seq_lens"], block_table=s["table"],
                                             max_seqlen_k=max(s["lens"]))
    w = s["weights"].clone()  # (as in the plain form)
    kept, lens = binding.swaa_cache_evict(s["k"], s["v"], w, s["keep"], s["n_sink"], s["recent"], seq_lens=s["seq_lens"],
                                          block_table=s["table"], max_seqlen_k=max(s["lens"]))
    return [kept, lens, w, s["k"], s["v"]]


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def _turn(s, pos):
    """The rotation of each position as matrices' entries: cos and sin over all D dimensions, and each dimension's partner and sign."""
    D, R = s["D"], s["rot"]
    freq = s["inv_freq"].double()
    which = torch.zeros(D, dtype=torch.long)
    partner, sign = torch.arange(D), torch.zeros(D, dtype=torch.float64)
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if s["adjacent"] else (i, i + R // 2)
        which[a] = which[b] = i
        partner[a], partner[b], sign[a], sign[b] = b, a, -1.0, 1.0
    angle = pos.double()[..., None] * freq[which.cuda()] * (torch.arange(D, device="cuda") * 0 + sign.abs().cuda())
    return angle.cos(), angle.sin(), partner.cuda(), sign.cuda()


def _exact_rope(s, x, w, pos):
    x = x.double()
    cos, sin, partner, sign = _turn(s, pos)
    if w is not None:
        x = x / (x.square().sum(-1, keepdim=True) / s["D"] + EPS).sqrt() * w.double()
    return x * cos + sign * x[..., partner] * sin


def _exact_grad(s, dy, x, w, pos):
    dy, x = dy.double(), x.double()
    cos, sin, partner, sign = _turn(s, pos)
    g = dy * cos - sign * dy[..., partner] * sin  # the transposed rotation
    if w is None:
        return g, None
    norm = (x.square().sum(-1, keepdim=True) / s["D"] + EPS).sqrt()
    gw = g * w.double()
    dx = gw / norm - x * (x * gw).sum(-1, keepdim=True) / (s["D"] * norm ** 3)
    return dx, (g * x / norm).flatten(0, -2).sum(0)


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "grad":
        pos = torch.arange(case["rows"], device="cuda")
        (dq, a), (dk, b) = (_exact_grad(s, s[d], s[x], s[w], pos) for d, x, w in (("dq_out", "q", "q_weight"), ("dk_out", "k", "k_weight")))
        return [dq, dk] + ([a, b] if case["norm"] else [])
    if kind == "rope":
        if case["form"] == "prompt":
            pos = torch.arange(case["rows"], device="cuda")
            return [_exact_rope(s, s[x], s[w], pos) for x, w in (("q", "q_weight"), ("k", "k_weight"))]
        out, at = [], 0
        caches = [s["k_cache"].double(), s["v_cache"].double()]
        for b, (n, m) in enumerate(zip(s["lens"], s["new"])):
            rows = torch.arange(n - m, n, device="cuda")
            pos = rows if s["positions"] is None else s["positions"][b]
            q, k, v = (s[x][:, at:at + m] if case["form"] == "packed" else s[x][b] for x in ("q", "k", "v"))
            at += m
            out.append(_exact_rope(s, q, s["q_weight"], pos))
            for cache, new in zip(caches, (_exact_rope(s, k, s["k_weight"], pos), v.double())):
                for p in range((n - m) // PAGE, (n - 1) // PAGE + 1):  # page by page
                    lo, hi = max(n - m, p * PAGE), min(n, (p + 1) * PAGE)
                    cache[int(s["table"][b, p]), :, lo - p * PAGE:hi - p * PAGE] = new[:, lo - (n - m):hi - (n - m)]
        return [torch.cat(out, 1) if case["form"] == "packed" else torch.stack(out)] + caches
    if kind == "weigh":
        G, rows = case["Hq"] // case["Hkv"], case["rows"]
        w = s["weights"].double() * (case["decay"] or 0.0)
        for b, n in enumerate(s["lens"]):
            w[b, :, n:] = s["weights"][b, :, n:].double()
            for h in range(case["Hq"]):
                keys = _rows_of(s["k"], s["table"], b, n)[h // G].double()
                step = max(1, (1 << 26) // n)
                for r0 in range(0, rows, step):
                    q = s["q"][b, h, r0:r0 + step].double()
                    pos = n - rows + r0 + torch.arange(q.shape[0], device="cuda")[:, None]
                    back = pos - torch.arange(n, device="cuda")  # how far behind the row a key stands
                    p = (q @ keys.t() * s["scale"] - s["lse"][b, h, r0:r0 + step, None].double()).exp()
                    hidden = (back < 0) | ((back >= case["window"]) & (torch.arange(n, device="cuda") >= case["n_sink"]))
                    w[b, h // G, :n] += p.masked_fill(hidden, 0.0).sum(0)
        return w
    keep, judged = case["keep"], s["weights"].cpu().numpy().astype(np.float64)
    kept = np.full((case["B"], case["Hkv"], keep), -1, dtype=np.int32)
    new = judged.copy()
    k, v = s["k"].clone(), s["v"].clone()
    for b, n in enumerate(s["lens"]):
        for h in range(case["Hkv"]):
            if n <= keep:
                kept[b, h, :n] = np.arange(n)
                continue
            middle = np.arange(case["n_sink"], n - case["recent"])
            by_weight = middle[np.lexsort((middle, -judged[b, h, middle]))]
            rows = np.concatenate((np.arange(case["n_sink"]), np.sort(by_weight[:keep - case["n_sink"] - case["recent"]]),
                                   np.arange(n - case["recent"], n)))
            kept[b, h] = rows
            new[b, h, :n] = np.concatenate((judged[b, h, rows], np.zeros(n - keep)))
            rows = torch.from_numpy(rows).cuda()
            for old, c in ((s["k"], k), (s["v"], v)):
                if s["table"] is None:
                    c[b, h, :keep] = old[b, h].index_select(0, rows)
                else:
                    pages = s["table"][b].long()
                    all_rows = old[pages, h].flatten(0, 1)  # [tokens, D]
                    whole = all_rows.clone()
                    whole[:keep] = all_rows.index_select(0, rows)
                    mine = -(-n // PAGE)  # (what follows in the table is not this sequence's)
                    c[pages[:mine], h] = whole.unflatten(0, (-1, PAGE))[:mine]
    lens = torch.tensor([min(n, keep) for n in s["lens"]], dtype=torch.int32, device="cuda")
    return [torch.from_numpy(kept), lens, torch.from_numpy(new), k, v]
