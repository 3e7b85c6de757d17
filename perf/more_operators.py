"""Performance cases of the operators for long and shared contexts, and for drafts drawn at random.

Misses that come together often begin alike (one system prompt, one set of examples), their contexts outgrow the cache, and
a draft model that samples needs its drafts verified by chance. A case is one pass through an operator:

  shared  attention of the new tokens of every sequence, where groups of sequences hold their first positions in common
  weigh   the attention weight that each cached token got from the new tokens, added to what it got before
  evict   the tokens of largest weight (and the last ones) kept, in order, and copied to other pages
  verify  drafts accepted against the target's probabilities by given random numbers, and the next token drawn

Plain forms are elementary torch operations in fp32 (fp64 for cumulative probabilities). The cache's pages are
[page, kv head, slot, dim]; a sequence's pages are named by its row of an int32 table; an 8-bit row is codes times one fp32
scale (its largest magnitude / 448 or 127).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
POOL = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}
POOL_LIMIT = 1 << 28      # elements of K (or V) that a drawn case may hold ...
MAC_LIMIT = 15 * 10 ** 9  # ... its products of q with K ...
SCORE_LIMIT = 1 << 27     # ... and its scores
PROB_LIMIT = 1 << 27      # probabilities of the target that a drawn case may hold


def _shared(name, fmt, dtype, seqs, groups, prefix, least, most, q_heads, kv_heads, head_dim, **kw):
    """`prefix`: the longest group's common positions; each sequence has `least` to `most` of its own behind them."""
    case = {"op": "shared", "fmt": fmt, "dtype": dtype, "seqs": seqs, "groups": groups, "prefix": prefix, "least": least,
            "most": most, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": 16, "new": 1, "window": 0,
            "start": 0}
    case.update(kw)
    return {"name": name, **case} if name else case


def _weigh(name, fmt, dtype, seqs, least, most, q_heads, kv_heads, head_dim, **kw):
    case = {"op": "weigh", "fmt": fmt, "dtype": dtype, "seqs": seqs, "least": least, "most": most, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": 16, "new": 1, "window": 0, "start": 0, "decay": 1.0}
    case.update(kw)
    return {"name": name, **case} if name else case


def _evict(name, fmt, seqs, least, most, keep, recent, kv_heads, head_dim, **kw):
    case = {"op": "evict", "fmt": fmt, "seqs": seqs, "least": least, "most": most, "keep": keep, "recent": recent,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": 16, "start": 0}
    case.update(kw)
    return {"name": name, **case} if name else case


def _verify(name, seqs, drafts, vocab, **kw):
    """`sampled`: drafts were drawn from the draft model's probabilities, else they are its likeliest tokens."""
    case = {"op": "verify", "seqs": seqs, "drafts": drafts, "vocab": vocab, "sampled": True, "served": False, "ragged": False}
    case.update(kw)
    return {"name": name, **case} if name else case


def listed():
    return [
        # two questions behind one short instruction, a small draft model: nothing but latency
        _shared("shared-pair", "bf16", "bf16", 2, 1, 300, 9, 40, 8, 8, 64),
        # a batch of misses decoding behind one system prompt with its examples
        _shared("shared-batch", "bf16", "bf16", 64, 1, 6000, 1, 700, 32, 8, 128),
        # three tenants' prompts, the target verifying 16 drafts and the token before them; the prompts end inside a page
        _shared("shared-verify", "f16", "f16", 24, 3, 3001, 17, 900, 16, 4, 128, new=17, page=32),
        # a full batch asking about one long document, on a quantised cache
        _shared("shared-document", "e4m3", "bf16", 128, 1, 30_011, 20, 500, 32, 8, 128, page=64),
        # the weights of one user's prefix in a small draft model: latency
        _weigh("weigh-one", "bf16", "bf16", 1, 700, 700, 8, 8, 64),
        # a decode step of a serving batch on a quantised cache, old weights fading
        _weigh("weigh-batch", "e4m3", "bf16", 64, 500, 16_384, 32, 8, 128, page=64, decay=0.95),
        # the last 512 tokens of prompts being read in: many rows a key
        _weigh("weigh-prompt", "bf16", "bf16", 4, 512, 4000, 32, 8, 128, new=512),
        # one short context cut to a quarter
        _evict("evict-one", "bf16", 1, 500, 500, 128, 32, 4, 64),
        # a batch of long contexts on a quantised cache, each cut to 4,096 tokens
        _evict("evict-batch", "e4m3", 24, 3000, 40_000, 4096, 512, 8, 128, page=64),
        # one query's four drafts
        _verify("verify-one", 1, 4, 32_000),
        # a batch of misses, 16 drafts each (some fewer, some queries served by the cache), an odd vocabulary
        _verify("verify-batch", 64, 16, 100_003, served=True, ragged=True),
        # drafts that are the draft model's likeliest tokens
        _verify("verify-likeliest", 32, 8, 50_000, sampled=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["shared", "shared", "weigh", "evict", "verify"])
    if op == "verify":
        seqs, drafts = _log(rng, 1, 128), _log(rng, 1, 24)
        vocab = _log(rng, 500, max(500, min(200_000, PROB_LIMIT // (seqs * (drafts + 1)))))
        return _verify("", seqs, drafts, vocab, sampled=rng.random() < 0.6, served=rng.random() < 0.5, ragged=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "f16"])
    fmt = rng.choice([dtype, "e4m3", "int8"])
    head_dim = rng.choice([64, 80, 96, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
    page = rng.choice([16, 32, 48, 64, 128])
    row = kv_heads * head_dim

    def start(most):   # (padding that leaves the longest sequence most of its tokens)
        return rng.choice([0, 0, rng.randint(1, min(40, max(1, most // 6)))]) if most > 5 else 0

    if op == "evict":
        seqs = _log(rng, 1, 64)
        most = _log(rng, 1, max(2, min(150_000, POOL_LIMIT // (seqs * row))))
        keep = _log(rng, 1, most)
        # codes that are whole numbers stand for values only with their scales: the kept formats are the floating ones
        return _evict("", rng.choice([dtype, "e4m3"]), seqs, _log(rng, 1, most), most, keep, rng.randint(0, keep), kv_heads,
                      head_dim, page=page, start=start(most))
    if op == "weigh":
        seqs, new = _log(rng, 1, 128), rng.choice([1, 1, 1, 5, 17, 160, 512])
        held = min(POOL_LIMIT // row, MAC_LIMIT // (new * q_heads * head_dim), SCORE_LIMIT // (new * q_heads))
        most = _log(rng, 1, max(2, min(100_000, held // seqs)))
        return _weigh("", fmt, dtype, seqs, _log(rng, 1, most), most, q_heads, kv_heads, head_dim, page=page, new=new,
                      window=rng.choice([0, 0, 0, _log(rng, 1, most)]), start=start(most), decay=rng.choice([1.0, 0.9]))
    seqs, new = _log(rng, 2, 256), rng.choice([1, 1, 1, 2, 5, 17])
    groups = rng.choice([1, 1, 1, min(seqs, 2), min(seqs, 5)])
    held = min(MAC_LIMIT // (new * q_heads * head_dim), SCORE_LIMIT // (new * q_heads)) // seqs
    most = _log(rng, 1, max(2, min(1500, held // 4, POOL_LIMIT // (4 * seqs * row))))
    prefix = _log(rng, 1, max(2, min(60_000, held * 3 // 4, POOL_LIMIT // (2 * groups * row))))
    return _shared("", fmt, dtype, seqs, groups, prefix, _log(rng, 1, most), most, q_heads, kv_heads, head_dim, page=page,
                   new=new, window=rng.choice([0, 0, 0, _log(rng, 1, prefix + most)]), start=start(most))


# ---------------------------------------------------------------------------------------------------------------------
# what a case means
# ---------------------------------------------------------------------------------------------------------------------
def _spread(n, least, most):
    """n lengths over [least, most]: the longest, the shortest, then the golden ratio's multiples."""
    rest = [least + int((most - least + 1) * math.modf(i * 0.6180339887498949)[0]) for i in range(1, n)]
    return ([most, least] + rest)[:n]


def _starts(case):
    return [(case["start"] * (1 + i % 3)) if case["start"] else 0 for i in range(case["seqs"])]


def _bounds(case):
    """Where the groups begin and end: group i of g has a share of i + 1 parts, one sequence at least."""
    n, g = case["seqs"], case["groups"]
    sizes, left = [], n - g
    for i in range(g):
        extra = left * (i + 1) * 2 // (g * (g + 1)) if i + 1 < g else left - sum(s - 1 for s in sizes)
        sizes.append(1 + extra)
    out = [0]
    for s in sizes:
        out.append(out[-1] + s)
    return out


def _prefixes(case):
    g = case["groups"]
    return [max(1, case["prefix"] * (g - i) // g) for i in range(g)]


def _lengths(case):
    own_part = _spread(case["seqs"], case["least"], case["most"])
    if case["op"] != "shared":
        return own_part
    b, p = _bounds(case), _prefixes(case)
    return [n + p[i] for i in range(case["groups"]) for n in own_part[b[i]:b[i + 1]]]


def _width(case):
    return max(1, -(-max(_lengths(case)) // case["page"]))


def _row_bytes(case):
    return case["head_dim"] * (1 if case["fmt"] in TOP else 2) + (4 if case["fmt"] in TOP else 0)


def work(case):
    op = case["op"]
    if op == "verify":
        B, k, V = case["seqs"], case["drafts"], case["vocab"]
        rows = 2 if case["sampled"] else 1           # of the position where the window ends
        return {"bytes": B * (4 * rows * V + 16 * k + 12), "flops": B * V * (rows + 1)}
    D, H, row = case["head_dim"], case["kv_heads"], _row_bytes(case)
    lengths, starts = _lengths(case), _starts(case)
    if op == "evict":
        held = [max(0, n - s) for n, s in zip(lengths, starts)]
        kept = sum(min(case["keep"], n) for n in held)
        return {"bytes": H * (4 * sum(held) + kept * (4 * row + 8)), "flops": H * sum(held)}
    T, pairs, seen = case["new"], 0, 0
    for n, s in zip(lengths, starts):
        w = case["window"] or n
        pairs += sum(max(0, p + 1 - max(s, p - w + 1, 0)) for p in range(n - T, n) if p >= 0)
    rows = case["seqs"] * T * case["q_heads"]
    first = [max(s, n - T - (case["window"] or n) + 1, 0) for n, s in zip(lengths, starts)]   # the first position that is seen
    if op == "weigh":
        seen = sum(max(0, n - f) for n, f in zip(lengths, first))
        return {"bytes": seen * H * row + 8 * H * sum(lengths) + rows * (2 * D + 4), "flops": 2 * pairs * case["q_heads"] * D}
    b, p = _bounds(case), _prefixes(case)
    for g in range(case["groups"]):
        of = range(b[g], b[g + 1])
        seen += max(0, p[g] - min(first[s] for s in of))
        seen += sum(max(0, lengths[s] - max(first[s], p[g])) for s in of)
    return {"bytes": 2 * seen * H * row + rows * (4 * D + 4), "flops": 4 * pairs * case["q_heads"] * D}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _heads(gen, n, heads, D, dtype, scale=1.0):
    """[n x heads x D] rows as a projection gives them: unequal channels, unequal tokens."""
    x = torch.randn(n, heads, D, generator=gen, device=DEV)
    x *= scale * (0.5 + torch.rand(1, heads, D, generator=gen, device=DEV)) * (0.5 + torch.rand(n, 1, 1, generator=gen, device=DEV))
    return x.to(dtype)


def _quantise(x, fmt):
    """Rows of x (last axis, fp32) in the cache's format: (values, scales or None)."""
    if fmt not in TOP:
        return x.to(POOL[fmt]), None
    top = TOP[fmt]
    scale = x.abs().amax(-1) / top
    code = (x / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(-1)).clamp(-top, top)
    return (code.round() if fmt == "int8" else code).to(POOL[fmt]), scale


def _pool(gen, case, pages):
    """One of K or V, filled: ([pages x heads x page x D] values, [pages x heads x page] scales or None)."""
    shape = (pages, case["kv_heads"], case["page"])
    out = torch.empty(*shape, case["head_dim"], dtype=POOL[case["fmt"]], device=DEV)
    scales = torch.empty(shape, device=DEV) if case["fmt"] in TOP else None
    step = max(1, (1 << 27) // (shape[1] * shape[2] * case["head_dim"]))
    for a in range(0, pages, step):
        b = min(pages, a + step)
        x = _heads(gen, (b - a) * case["page"], case["kv_heads"], case["head_dim"], torch.float32)
        out[a:b], s = _quantise(x.view(b - a, case["page"], case["kv_heads"], -1).transpose(1, 2), case["fmt"])
        if s is not None:
            scales[a:b] = s
    return out, scales


def _table(gen, case):
    """(table, pages): the common pages of a group under every one of its sequences, then their own. A page that the common
    part ends in is each sequence's own, with a copy of that part."""
    page, lengths = case["page"], _lengths(case)
    b, p = (_bounds(case), _prefixes(case)) if case["op"] == "shared" else ([0, len(lengths)], [0])
    rows, used = [], 0
    for g in range(len(p)):
        common = list(range(used, used + p[g] // page))
        used += len(common)
        for s in range(b[g], b[g + 1]):
            mine = max(0, -(-lengths[s] // page) - len(common))
            rows.append(common + list(range(used, used + mine)))
            used += mine
    used = max(used, 1)
    order = torch.randperm(used, generator=gen, device=DEV).to(torch.int32)
    flat = torch.tensor([r + [0] * (_width(case) - len(r)) for r in rows], device=DEV)
    return order[flat].contiguous(), used


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    if case["op"] == "verify":
        return _drafted(gen, case)
    x, D, B = {}, case["head_dim"], case["seqs"]
    x["table"], pages = _table(gen, case)
    x["pages"] = pages
    x["k"], x["ks"] = _pool(gen, case, pages)
    x["v"], x["vs"] = _pool(gen, case, pages)
    x["lengths"], x["starts"] = _ints(_lengths(case)), _ints(_starts(case))
    if case["op"] == "evict":
        # weights as they gather: a few tokens have most of them, some have none
        w = torch.rand(B, case["kv_heads"], _width(case) * case["page"], generator=gen, device=DEV)
        x["weights"] = torch.where(w < 0.05, torch.zeros_like(w), (w ** 6) * 50)
        wide = -(-case["keep"] // case["page"])
        x["to"] = pages + torch.randperm(B * wide, generator=gen, device=DEV).to(torch.int32).view(B, wide)
        return x
    x["q"] = _heads(gen, B * case["new"], case["q_heads"], D, DTYPES[case["dtype"]])
    if case["op"] == "shared":
        x["bounds"], x["shared"] = _ints(_bounds(case)), _ints(_prefixes(case))
        b, p = _bounds(case), _prefixes(case)
        for g in range(case["groups"]):
            at, rest = p[g] // case["page"], p[g] % case["page"]
            if rest:
                ids = x["table"][b[g]:b[g + 1], at].long()
                for name in ("k", "ks", "v", "vs"):
                    if x[name] is not None:
                        x[name][ids[1:], :, :rest] = x[name][ids[:1], :, :rest].clone()
    else:
        x["weights"] = torch.rand(B, case["kv_heads"], _width(case) * case["page"], generator=gen, device=DEV) ** 4 * 20
        score = _scores(case, x)
        x["lse"] = torch.logsumexp(score, -1).permute(0, 2, 1, 3).reshape(B * case["new"], case["q_heads"]).contiguous()
    return x


def _drafted(gen, case):
    """A target's and a draft model's next-token probabilities, which agree in the main, and drafts of the second."""
    B, k, V = case["seqs"], case["drafts"], case["vocab"]
    target, draft = torch.empty(B, k + 1, V, device=DEV), torch.empty(B, k, V, device=DEV)
    drafts = torch.empty(B, k, dtype=torch.int32, device=DEV)
    for b in range(B):
        logits = torch.randn(k + 1, V, generator=gen, device=DEV) * 2.5
        near = logits[:k] + torch.randn(k, V, generator=gen, device=DEV) * 0.4
        target[b], draft[b] = torch.softmax(logits, -1), torch.softmax(near, -1)
        drafts[b] = torch.multinomial(draft[b], 1, generator=gen).view(-1) if case["sampled"] else draft[b].argmax(-1)
    if not case["sampled"]:
        # likeliest drafts are accepted when the target is as sure: half of its rows are
        boost = torch.rand(B, k, 1, generator=gen, device=DEV).round()
        at = drafts.long().unsqueeze(-1)
        head = target[:, :k].gather(-1, at)
        top = head + boost * (0.9 - head)
        target[:, :k] *= (1 - top) / (1 - head)
        target[:, :k].scatter_(-1, at, top)
    if case["ragged"]:
        for b in range(4, B, 5):
            drafts[b, k // 2:] = -1               # a shorter window
    status = torch.zeros(B, dtype=torch.uint8, device=DEV)
    if case["served"]:
        status[3::8] = 1                          # served by the cache: nothing to verify
    return {"p_target": target, "p_draft": draft if case["sampled"] else None, "drafts": drafts, "status": status,
            "u": torch.rand(B, k + 1, generator=gen, device=DEV)}


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    B = case["seqs"]
    if case["op"] == "verify":
        s["accepted"] = torch.empty(B, dtype=torch.int32, device=DEV)
        s["token"] = torch.empty(B, dtype=torch.int32, device=DEV)
        return s
    H, D, pages = case["kv_heads"], case["head_dim"], s["pages"]
    total = pages + (s["to"].numel() if case["op"] == "evict" else 0)
    if own:
        from paper_2608_01718_gb300 import lacache as L
        s["kv"] = L.KVCache(kv_heads=H, head_dim=D, pages=total, page_size=case["page"], format=case["fmt"],
                            device=torch.cuda.current_device())
        pool = s["kv"].pool(0)
    else:
        pool = {n: torch.empty(total, *s[n].shape[1:], dtype=s[n].dtype, device=DEV) for n in ("k", "v", "ks", "vs")
                if s[n] is not None}
    for name, t in pool.items():
        t[:pages].copy_(s.pop(name))
        t[pages:].zero_()
        s[name] = t
    if case["op"] == "shared":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], device=DEV)
    elif case["op"] == "weigh":
        s["out"] = torch.zeros_like(s["weights"])
    else:
        s["kept"] = torch.empty(B, H, case["keep"], dtype=torch.int32, device=DEV)
        s["new_lengths"] = torch.empty(B, dtype=torch.int32, device=DEV)
        s["new_weights"] = torch.zeros(B, H, case["keep"], device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)(state["case"]["op"], state)


def _evicted(s):
    """What an eviction leaves: the kept tokens' pages, and the outputs beside them."""
    got = {n: s[n][s["pages"]:] for n in ("k", "v", "ks", "vs") if s.get(n) is not None}
    return {**got, "kept": s["kept"], "lengths": s["new_lengths"], "weights": s["new_weights"]}


def _own(op, s):
    case = s["case"]
    if op == "verify":
        from paper_2608_01718_gb300 import lacache as L
        L.lacache_verify_sample(s["p_target"], s["p_draft"], s["drafts"], s["u"], s["accepted"], s["token"],
                                status=s["status"] if case["served"] else None)
        return {"accepted": s["accepted"], "token": s["token"]}
    kv, starts = s["kv"], s["starts"] if case["start"] else None
    if op == "shared":
        kv.attend_shared(s["q"], s["table"], s["lengths"], s["shared"], bounds=s["bounds"], new_tokens=case["new"],
                         window=case["window"], starts=starts, out=s["out"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "weigh":
        kv.weigh(s["q"], s["table"], s["lengths"], s["lse"], weights=s["weights"], decay=case["decay"], out=s["out"],
                 new_tokens=case["new"], window=case["window"], starts=starts)
        return s["out"]
    kv.evict(s["table"], s["lengths"], s["weights"], case["keep"], s["to"], recent=case["recent"], starts=starts,
             kept=s["kept"], new_lengths=s["new_lengths"], new_weights=s["new_weights"])
    return _evicted(s)


def _rows(x, name, page, slot):
    """fp32 values of the cached rows at page ids and slots (of any one shape): [..., heads, D]."""
    v = x[name][page, :, slot].float()
    return v if x.get(name + "s") is None else v * x[name + "s"][page, :, slot].unsqueeze(-1)


def _at(case, table, first, last):
    """Page ids [rows x n] and slots [n] of positions [first, last) of some rows of the table."""
    j = torch.arange(first, last, device=DEV)
    return table.long()[:, j // case["page"]], j % case["page"]


def _by_head(x, T, H):
    """[B * T x heads x D] as [B x H x T * G x D]."""
    n, heads, D = x.shape
    return x.view(n // T, T, H, heads // H, D).permute(0, 2, 1, 3, 4).reshape(n // T, H, T * (heads // H), D)


def _seen(case, lengths, starts, first, last):
    """[B x 1 x T x 1 x n]: which of the positions [first, last) each new token sees."""
    T = case["new"]
    j = torch.arange(first, last, device=DEV)
    p = (lengths.unsqueeze(1) - T + torch.arange(T, device=DEV)).view(-1, 1, T, 1, 1)
    seen = (j <= p) & (j >= starts.view(-1, 1, 1, 1, 1))
    return seen & (j > p - case["window"]) if case["window"] else seen


def _scores(case, x):
    """[B x H x T x G x positions], -inf where not seen."""
    B, T, H = case["seqs"], case["new"], case["kv_heads"]
    page, slot = _at(case, x["table"], 0, _width(case) * case["page"])
    k = _rows(x, "k", page, slot.expand_as(page)).permute(0, 2, 3, 1)
    score = (_by_head(x["q"].float(), T, H) @ k).view(B, H, T, case["q_heads"] // H, -1) / math.sqrt(case["head_dim"])
    return score.masked_fill_(~_seen(case, x["lengths"], x["starts"], 0, k.shape[-1]), -math.inf)


def _plain(op, s):
    case = s["case"]
    return {"shared": _plain_shared, "weigh": _plain_weigh, "evict": _plain_evict, "verify": _plain_verify}[op](case, s)


def _plain_shared(case, s):
    T, H, G, D = case["new"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]
    lengths, b, p = _lengths(case), _bounds(case), _prefixes(case)
    for g in range(case["groups"]):
        of, n = slice(b[g], b[g + 1]), b[g + 1] - b[g]
        last = max(lengths[of])
        q = _by_head(s["q"][b[g] * T:b[g + 1] * T].float(), T, H)
        # the common positions once, from the first sequence's pages; each sequence's own
        page, slot = _at(case, s["table"][b[g]:b[g] + 1], 0, p[g])
        k0, v0 = (_rows(s, name, page[0], slot).transpose(0, 1) for name in ("k", "v"))         # [H x P x D]
        page, slot = _at(case, s["table"][of], p[g], last)
        k1, v1 = (_rows(s, name, page, slot.expand_as(page)).transpose(1, 2) for name in ("k", "v"))
        together = q.transpose(0, 1).reshape(H, n * T * G, D)
        score = torch.cat(((together @ k0.transpose(-1, -2)).view(H, n, T * G, -1).transpose(0, 1), q @ k1.transpose(-1, -2)), -1)
        score = score.view(n, H, T, G, -1) / math.sqrt(D)
        score = score.masked_fill(~_seen(case, s["lengths"][of], s["starts"][of], 0, last), -math.inf)
        top = score.amax(-1, keepdim=True)
        weight = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = weight.sum(-1, keepdim=True)
        weight = (weight / torch.where(total > 0, total, torch.ones_like(total))).view(n, H, T * G, -1)
        w0 = weight[..., :p[g]].transpose(0, 1).reshape(H, n * T * G, -1)
        out = (w0 @ v0).view(H, n, T * G, D).transpose(0, 1) + weight[..., p[g]:] @ v1
        rows = slice(b[g] * T, b[g + 1] * T)
        s["out"][rows] = out.view(n, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(n * T, H * G, D).to(s["out"].dtype)
        s["lse"][rows] = (top + torch.log(total)).view(n, H, T, G).permute(0, 2, 1, 3).reshape(n * T, H * G)
    return {"out": s["out"], "lse": s["lse"]}


def _plain_weigh(case, s):
    B, T, H, G = case["seqs"], case["new"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    lse = s["lse"].view(B, T, H, G).permute(0, 2, 1, 3).unsqueeze(-1)
    got = torch.exp(_scores(case, s) - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)).sum((2, 3))
    j, n = torch.arange(got.shape[-1], device=DEV), s["lengths"].view(B, 1, 1)
    before = torch.where(j < n - T, s["weights"] * case["decay"], torch.zeros_like(got))
    s["out"].copy_(torch.where(j < n, before + got, s["out"]))
    return s["out"]


def _plain_evict(case, s):
    B, H, keep, recent = case["seqs"], case["kv_heads"], case["keep"], case["recent"]
    s["new_lengths"].copy_((s["lengths"] - s["starts"]).clamp(0, keep))
    s["kept"].fill_(-1)
    j = torch.arange(s["weights"].shape[-1], device=DEV)
    n, first = s["lengths"].view(B, 1, 1), s["starts"].view(B, 1, 1)
    w = torch.where(j >= n - recent, torch.full_like(s["weights"], math.inf), s["weights"])
    w = torch.where((j < first) | (j >= n), torch.full_like(w, -math.inf), w)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]    # the largest, of equal ones the first
    cols = torch.arange(order.shape[-1], device=DEV)
    there = (cols < s["new_lengths"].view(B, 1, 1)).expand(B, H, -1)
    order = torch.where(there, order, torch.full_like(order, 1 << 40)).sort(-1).values
    seq, head, col = torch.nonzero(there, as_tuple=True)
    pos = order[seq, head, col]
    s["kept"][seq, head, col] = pos.to(torch.int32)
    s["new_weights"][seq, head, col] = s["weights"][seq, head, pos]
    frm = s["table"][seq, pos // case["page"]].long(), head, pos % case["page"]
    to = s["to"][seq, col // case["page"]].long(), head, col % case["page"]
    for name in ("k", "v", "ks", "vs"):
        if s.get(name) is not None:
            x = s[name].view(torch.uint8) if s[name].dtype == torch.float8_e4m3fn else s[name]
            x[to] = x[frm]
    return _evicted(s)


def _plain_verify(case, s):
    B, k, V = case["seqs"], case["drafts"], case["vocab"]
    x = s["drafts"].long()
    there = (x >= 0) & (x < V)
    at = torch.where(there, x, torch.zeros_like(x)).unsqueeze(-1)
    p = s["p_target"][:, :k].gather(-1, at).squeeze(-1).double()
    q = s["p_draft"].gather(-1, at).squeeze(-1).double() if case["sampled"] else torch.ones_like(p)
    go = there & (s["u"][:, :k].double() * q < p)
    n = go.long().cumprod(-1).sum(-1)
    row, b = s["p_target"][torch.arange(B, device=DEV), n], torch.arange(B, device=DEV)
    at_end = torch.cat((x, torch.full((B, 1), -1, device=DEV)), 1)[b, n]          # the draft that was refused, -1 for none
    refused = (at_end >= 0) & (at_end < V)
    if case["sampled"]:
        take = s["p_draft"][b, n.clamp(max=k - 1)].double()
    else:
        take = (torch.arange(V, device=DEV) == at_end.unsqueeze(1)).double()
    rest = (row.double() - take).clamp(min=0.0)
    weight = torch.where(refused.unsqueeze(1) & (rest.sum(-1, keepdim=True) > 0), rest, row.double())
    upto = weight.cumsum(-1)
    token = (upto <= s["u"][:, k:].double() * upto[:, -1:]).sum(-1)
    last = torch.where(weight > 0, torch.arange(V, device=DEV), torch.zeros_like(weight, dtype=torch.long)).amax(-1)
    token = torch.minimum(token, last)
    if case["served"]:
        served = s["status"] == 1
        n, token = torch.where(served, torch.full_like(n, -1), n), torch.where(served, torch.full_like(n, -1), token)
    s["accepted"].copy_(n)
    s["token"].copy_(token)
    return {"accepted": s["accepted"], "token": s["token"]}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "verify":
        return _exact_verify(case, x)
    if case["op"] == "evict":
        return _exact_evict(case, x)
    T, H, G, D = case["new"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]
    lengths, starts = _lengths(case), _starts(case)

    def rows64(name, seq, lo, n):   # cached tokens [lo, n) of a sequence: [heads x n - lo x D]
        first = lo // case["page"]
        pages = x["table"][seq, first: max(first + 1, -(-n // case["page"]))].long()
        z = x[name][pages].double()
        if x[name + "s"] is not None:
            z = z * x[name + "s"][pages].double().unsqueeze(-1)
        z = z.permute(1, 0, 2, 3).reshape(H, -1, D)
        return z[:, lo - first * case["page"]: n - first * case["page"]]

    outs, lses = [], []
    got = torch.zeros_like(x["weights"], dtype=torch.float64) if case["op"] == "weigh" else None
    for b, (n, start) in enumerate(zip(lengths, starts)):
        q = x["q"][b * T:(b + 1) * T].double().view(T, H, G, D)
        lo = min(n, max(start, n - T - case["window"] + 1 if case["window"] else 0, 0))
        p = torch.arange(n - T, n, device=DEV).view(1, T, 1, 1)
        j = torch.arange(lo, n, device=DEV)
        seen = (j <= p) & (j >= start)
        if case["window"]:
            seen = seen & (j > p - case["window"])
        score = torch.einsum("thgd,hjd->htgj", q, rows64("k", b, lo, n)) * D ** -0.5
        if case["op"] == "weigh":
            lse = x["lse"][b * T:(b + 1) * T].double().view(T, H, G).permute(1, 0, 2).unsqueeze(-1)
            w = torch.where(seen, torch.exp(score - lse), torch.zeros_like(score)).sum((1, 2))
            got[b, :, :max(0, n - T)] = x["weights"][b, :, :max(0, n - T)].double() * case["decay"]
            got[b, :, lo:n] += w
            continue
        score = torch.where(seen, score, torch.full_like(score, -math.inf))
        lse = torch.logsumexp(score, -1) if n > lo else torch.full((H, T, G), -math.inf, dtype=torch.float64, device=DEV)
        some = torch.isfinite(lse).unsqueeze(-1)
        w = torch.where(some, torch.exp(score - torch.where(some, lse.unsqueeze(-1), torch.zeros_like(some, dtype=torch.float64))),
                        torch.zeros_like(score))
        outs.append(torch.einsum("htgj,hjd->thgd", w, rows64("v", b, lo, n)).reshape(T, H * G, D))
        lses.append(lse.permute(1, 0, 2).reshape(T, H * G))
    return got if got is not None else {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_evict(case, x):
    B, H, keep, page = case["seqs"], case["kv_heads"], case["keep"], case["page"]
    names = [n for n in ("k", "v", "ks", "vs") if x[n] is not None]
    got = {n: torch.zeros(x["to"].numel(), *x[n].shape[1:], dtype=torch.float64, device=DEV) for n in names}
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device=DEV)
    weights = torch.zeros(B, H, keep, dtype=torch.float64, device=DEV)
    counts = []
    for b, (n, start) in enumerate(zip(_lengths(case), _starts(case))):
        count = min(keep, max(0, n - start))
        counts.append(count)
        if count == 0:
            continue
        free = max(start, n - min(case["recent"], keep))           # tokens from here on stay in any case
        for h in range(H):
            w = x["weights"][b, h, start:free].double()
            must = n - free
            want = count - must
            # a token stays if fewer than `want` come before it: those of more weight, and of its own weight the earlier ones
            value = w.sort(descending=True).values[want - 1] if want > 0 else None
            if value is None:
                stay = torch.zeros_like(w, dtype=torch.bool)
            else:
                equal = w == value
                stay = (w > value) | (equal & (equal.cumsum(0) <= want - (w > value).sum()))
            pos = torch.cat((torch.nonzero(stay).view(-1) + start, torch.arange(free, n, device=DEV)))
            kept[b, h, :count] = pos.to(torch.int32)
            weights[b, h, :count] = x["weights"][b, h, pos].double()
            col = torch.arange(count, device=DEV)
            to, frm = x["to"][b, col // page].long() - x["pages"], x["table"][b, pos // page].long()
            for name in names:
                got[name][to, h, col % page] = x[name][frm, h, pos % page].double()
    return {**got, "kept": kept, "lengths": _ints(counts), "weights": weights}


def _exact_verify(case, x):
    B, k, V = case["seqs"], case["drafts"], case["vocab"]
    drafts, u, status = x["drafts"].tolist(), x["u"].double().cpu(), x["status"].tolist()
    accepted, token = [], []
    for b in range(B):
        if case["served"] and status[b] == 1:
            accepted.append(-1)
            token.append(-1)
            continue
        n, refused = 0, None
        while n < k and 0 <= drafts[b][n] < V:
            d = drafts[b][n]
            q = x["p_draft"][b, n, d].double().item() if case["sampled"] else 1.0
            if not u[b, n].item() * q < x["p_target"][b, n, d].double().item():
                refused = d
                break
            n += 1
        weight = x["p_target"][b, n].double()
        if refused is not None:
            less = weight.clone()
            if case["sampled"]:
                less -= x["p_draft"][b, n].double()
            else:
                less[refused] -= 1.0
            less = torch.relu(less)
            if less.sum() > 0:
                weight = less
        upto = torch.cumsum(weight, 0)
        past = torch.nonzero(upto > u[b, k].item() * upto[-1])
        accepted.append(n)
        token.append(int(past[0]) if len(past) else int(torch.nonzero(weight)[-1]))
    return {"accepted": _ints(accepted), "token": _ints(token)}
