"""Performance cases of the decoding operators: what a miss costs after the lookup.

A query that is not served is decoded: a draft model produces its lookahead prefix token by token, and the target model
verifies the k drafts in one pass. Both work on a paged key-value cache. A case is one pass through an operator:

  attend  attention of the new tokens of every sequence (one, or a draft window) over the paged cache
  write   rotary positions applied to q and k, and k and v written into the cache (quantised or as they are)
  read    cached tokens read back, as rows of a 16-bit type
  rotate  rotary positions of a tensor of heads, or their gradient

Plain forms are elementary torch operations in fp32. The cache's pages are [page, kv head, slot, dim]; a sequence's pages
are named by its row of an int32 table; an 8-bit row is codes times one fp32 scale (its largest magnitude / 448 or 127).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
POOL = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}
KV_LIMIT = 1 << 28                       # elements of K (or V) that a drawn attend case may hold, padded ...
MAC_LIMIT = 1 << 31                      # ... and their products with its rows of q
ROW_LIMIT = 16384 * 32 * 128             # elements that a drawn rotate case may hold
BASE = 10000.0


def _attend(name, fmt, dtype, seqs, least, most, q_heads, kv_heads, head_dim, **kw):
    case = {"op": "attend", "fmt": fmt, "dtype": dtype, "seqs": seqs, "least": least, "most": most, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": 16, "new": 1, "window": 0, "start": 0}
    case.update(kw)
    return {"name": name, **case} if name else case


def _write(name, fmt, dtype, seqs, tokens, first, q_heads, kv_heads, head_dim, rot, **kw):
    case = {"op": "write", "fmt": fmt, "dtype": dtype, "seqs": seqs, "tokens": tokens, "first": first, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "rot": rot, "layout": "half", "factor": 1.0, "page": 16}
    case.update(kw)
    return {"name": name, **case} if name else case


def _read(name, fmt, dtype, seqs, tokens, kv_heads, head_dim, **kw):
    case = {"op": "read", "fmt": fmt, "dtype": dtype, "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": 16}
    case.update(kw)
    return {"name": name, **case} if name else case


def _rotate(name, dtype, tokens, first, heads, head_dim, rot, **kw):
    case = {"op": "rotate", "dtype": dtype, "tokens": tokens, "first": first, "heads": heads, "head_dim": head_dim,
            "rot": rot, "layout": "half", "factor": 1.0, "gradient": False}
    case.update(kw)
    return {"name": name, **case} if name else case


def listed():
    return [
        # a small draft model decoding one user's prefix: nothing but latency
        _attend("attend-one", "bf16", "bf16", 1, 100, 100, 8, 8, 64),
        # a batch of misses decoding together, grouped heads, lengths all over (one sequence still empty)
        _attend("attend-batch", "bf16", "bf16", 32, 0, 4096, 32, 8, 128),
        # one long context: few rows, all of the work along one axis
        _attend("attend-long", "bf16", "bf16", 1, 200_003, 200_003, 32, 8, 128),
        # a full serving batch on a quantised cache
        _attend("attend-e4m3", "e4m3", "bf16", 64, 500, 16384, 32, 8, 128, page=64),
        # the target model verifying a window of 16 drafts and the token before them
        _attend("attend-verify", "bf16", "bf16", 16, 300, 3000, 32, 4, 128, new=17),
        # sliding-window layers, left-padded prompts, wide heads, an int8 cache and a short draft window
        _attend("attend-window", "int8", "f16", 48, 3, 20_001, 16, 4, 256, new=4, window=1024, start=7, page=32),
        # one decode step of 32 sequences
        _write("write-step", "e4m3", "bf16", 32, 32, 1900, 32, 8, 128, 128),
        # prompts of a batch of misses written at once, rotary on half of each head, stretched positions
        _write("write-prompts", "e4m3", "bf16", 7, 12_001, 0, 32, 8, 128, 64, layout="interleaved", factor=4.0, page=64),
        # one short prefix taken out of the cache (to hand it to another worker)
        _read("read-prefix", "e4m3", "bf16", 1, 333, 8, 128),
        # a batch of prompts read back to attend over them in 16 bits
        _read("read-prompts", "int8", "f16", 16, 60_000, 8, 128, page=32),
        # rotary positions of one new token's queries
        _rotate("rotate-token", "bf16", 1, 5000, 32, 128, 128),
        # the gradient of the rotation in a training step
        _rotate("rotate-gradient", "bf16", 16_384, 0, 32, 128, 128, gradient=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "write", "read", "rotate"])
    dtype = rng.choice(["bf16", "f16"])
    fmt = rng.choice([dtype, "e4m3", "int8"])
    head_dim = rng.choice([64, 80, 96, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
    page = rng.choice([16, 32, 48, 64, 128])
    layout = rng.choice(["half", "interleaved"])
    factor = rng.choice([1.0, 2.5, 8.0])
    rot = rng.choice([head_dim, max(16, head_dim // 32 * 16)])
    first = _log(rng, 1, 100_000)
    if op == "attend":
        seqs = _log(rng, 1, 256)
        new = rng.choice([1, 1, 1, 2, 5, 9, 17])
        held = min(KV_LIMIT, MAC_LIMIT * kv_heads // (new * q_heads))
        most = _log(rng, 1, max(2, min(150_000, held // (seqs * kv_heads * head_dim))))
        return _attend("", fmt, dtype, seqs, _log(rng, 1, most), most, q_heads, kv_heads, head_dim, page=page, new=new,
                       window=rng.choice([0, 0, 0, _log(rng, 1, most)]), start=rng.choice([0, 0, rng.randint(1, 40)]))
    if op == "write":
        tokens = _log(rng, 1, 12_000)
        # a cache held in whole numbers comes back as values only through read(): written formats are the floating ones
        return _write("", rng.choice([dtype, "e4m3"]), dtype, min(tokens, _log(rng, 1, 64)), tokens, first, q_heads, kv_heads,
                      head_dim, rot, layout=layout, factor=factor, page=page)
    if op == "read":
        tokens = _log(rng, 1, 60_000)
        return _read("", fmt, dtype, min(tokens, _log(rng, 1, 64)), tokens, kv_heads, head_dim, page=page)
    heads = _log(rng, 1, 64)
    return _rotate("", dtype, _log(rng, 1, max(2, min(30_000, ROW_LIMIT // (heads * head_dim)))), first, heads, head_dim, rot,
                   layout=layout, factor=factor, gradient=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------------------------
# what a case means
# ---------------------------------------------------------------------------------------------------------------------
def _spread(n, least, most):
    """n lengths over [least, most]: the longest, the shortest, then the golden ratio's multiples."""
    rest = [least + int((most - least + 1) * math.modf(i * 0.6180339887498949)[0]) for i in range(1, n)]
    return ([most, least] + rest)[:n]


def _starts(case):
    return [(case["start"] * (1 + i % 3)) if case["start"] else 0 for i in range(case["seqs"])]


def _lengths(case):
    if case["op"] == "attend":
        return _spread(case["seqs"], case["least"], case["most"])
    each = [case["tokens"] // case["seqs"]] * case["seqs"]     # tokens written or read, a sequence
    for i in range(case["tokens"] % case["seqs"]):
        each[i] += 1
    return each


def _places(case):
    """(sequence, position) of each token of a write or read, in order."""
    n = np.array(_lengths(case))
    seq = np.repeat(np.arange(case["seqs"]), n)
    pos = np.arange(case["tokens"]) - np.repeat(np.cumsum(n) - n, n)
    return seq.astype(np.int32), pos.astype(np.int32)


def _width(case):
    return max(1, -(-max(_lengths(case)) // case["page"]))


def _turns(case):
    """Angular frequency of each rotated pair: positions divided by `factor`."""
    i = np.arange(case["rot"] // 2, dtype=np.float64)
    return BASE ** (-2.0 * i / case["rot"]) / case["factor"]


def work(case):
    D, op = case["head_dim"], case["op"]
    if op == "rotate":
        n = case["tokens"] * case["heads"] * D
        return {"bytes": 4 * n + 4 * case["tokens"], "flops": 3 * n}
    item = 1 if case["fmt"] in TOP else 2
    row = D * item + (4 if case["fmt"] in TOP else 0)          # one cached row, its scale with it
    H = case["kv_heads"]
    if op == "read":
        return {"bytes": 2 * case["tokens"] * H * (row + 2 * D) + 8 * case["tokens"], "flops": 2 * case["tokens"] * H * D}
    if op == "write":
        q, kv = case["tokens"] * case["q_heads"] * D, case["tokens"] * H * D
        return {"bytes": 4 * q + 4 * kv + 2 * case["tokens"] * H * row + 8 * case["tokens"], "flops": 3 * (q + kv) + 2 * kv}
    T, seen, pairs = case["new"], 0, 0
    for n, s in zip(_lengths(case), _starts(case)):
        w = case["window"] or n
        seen += max(0, n - max(s, n - T - w + 1, 0))
        pairs += sum(max(0, p + 1 - max(s, p - w + 1, 0)) for p in range(n - T, n) if p >= 0)
    rows = case["seqs"] * T * case["q_heads"]
    return {"bytes": 2 * seen * H * row + 4 * rows * D + 4 * rows + 4 * case["seqs"] * (_width(case) + 2),
            "flops": 4 * pairs * case["q_heads"] * D}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
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
    code = x / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(-1)
    code = code.clamp(-top, top)
    return (code.round() if fmt == "int8" else code).to(POOL[fmt]), scale


def _pool(gen, case, pages, dtype):
    """One of K or V, filled: ([pages x heads x page x D] values, [pages x heads x page] scales or None)."""
    shape = (pages, case["kv_heads"], case["page"])
    out = torch.empty(*shape, case["head_dim"], dtype=POOL[case["fmt"]], device=DEV)
    scales = torch.empty(shape, device=DEV) if case["fmt"] in TOP else None
    step = max(1, (1 << 27) // (shape[1] * shape[2] * case["head_dim"]))
    for a in range(0, pages, step):
        b = min(pages, a + step)
        x = _heads(gen, (b - a) * case["page"], case["kv_heads"], case["head_dim"], dtype)
        v, s = _quantise(x.view(b - a, case["page"], case["kv_heads"], -1).transpose(1, 2).float(), case["fmt"])
        out[a:b] = v
        if s is not None:
            scales[a:b] = s
    return out, scales


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dtype, D = DTYPES[case["dtype"]], case["head_dim"]
    x = {}
    if case["op"] == "rotate":
        x["x"] = _heads(gen, case["tokens"], case["heads"], D, dtype)
        x["pos"] = torch.arange(case["first"], case["first"] + case["tokens"], dtype=torch.int32, device=DEV)
        return x
    width = _width(case)
    pages = case["seqs"] * width
    x["table"] = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32).view(case["seqs"], width)
    if case["op"] == "attend":
        x["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
        x["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device=DEV)
        x["q"] = _heads(gen, case["seqs"] * case["new"], case["q_heads"], D, dtype)
    else:
        seq, pos = _places(case)
        x["seq"], x["slot"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
    if case["op"] == "write":
        heads = case["q_heads"] + 2 * case["kv_heads"]
        x["qkv"] = _heads(gen, case["tokens"], heads, D, dtype)          # one fused projection: q, k and v are slices of it
        x["pos"] = x["slot"] + case["first"]
    else:
        x["k"], x["ks"] = _pool(gen, case, pages, dtype)
        x["v"], x["vs"] = _pool(gen, case, pages, dtype)
    return x


def _split(case, qkv):
    a, b = case["q_heads"], case["q_heads"] + case["kv_heads"]
    return qkv[:, :a], qkv[:, a:b], qkv[:, b:]


def prepare(case, seed):
    x = _inputs(case, seed)
    s = {"case": case, **x}
    dtype, D, op = DTYPES[case["dtype"]], case["head_dim"], case["op"]
    if op in ("rotate", "write"):
        if own:
            from paper_2608_01718_gb300 import lacache as L
            s["rope"] = L.Rope(case["rot"], base=BASE, interleaved=case["layout"] == "interleaved",
                               scaling="linear" if case["factor"] != 1.0 else None, factor=case["factor"])
        else:
            # the tables of cosines and sines that a program keeps, by position
            p = torch.arange(case["first"] + case["tokens"], dtype=torch.float64, device=DEV)
            a = p.unsqueeze(1) * torch.from_numpy(_turns(case)).to(DEV)
            s["cos"], s["sin"] = a.cos().float(), a.sin().float()
    if op == "rotate":
        s["out"] = torch.empty_like(s["x"])
        return s
    if own:
        from paper_2608_01718_gb300 import lacache as L
        kv = L.KVCache(kv_heads=case["kv_heads"], head_dim=D, pages=s["table"].numel(), page_size=case["page"],
                       format=case["fmt"], device=torch.cuda.current_device())
        s["kv"], pool = kv, kv.pool(0)
        for name in ("k", "v", "ks", "vs"):
            if s.get(name) is not None:
                pool[name].copy_(s.pop(name))
            elif pool.get(name) is not None:
                pool[name].zero_()
        s["pool"] = pool
    elif op == "write":
        shape = (s["table"].numel(), case["kv_heads"], case["page"])
        for name in ("k", "v"):
            s[name] = torch.zeros(*shape, D, dtype=POOL[case["fmt"]], device=DEV)
            s[name + "s"] = torch.zeros(shape, device=DEV) if case["fmt"] in TOP else None
    if op == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], device=DEV)
    elif op == "write":
        s["q_out"] = torch.empty(case["tokens"], case["q_heads"], D, dtype=dtype, device=DEV)
    elif op == "read":
        s["k_out"] = torch.empty(case["tokens"], case["kv_heads"], D, dtype=dtype, device=DEV)
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)(state["case"]["op"], state)


def _own(op, s):
    case = s["case"]
    if op == "rotate":
        return s["rope"].apply(s["x"], s["pos"], inverse=case["gradient"], out=s["out"])
    kv = s["kv"]
    if op == "attend":
        kv.attend(s["q"], s["table"], s["lengths"], new_tokens=case["new"], window=case["window"],
                  starts=s["starts"] if case["start"] else None, out=s["out"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "write":
        q, k, v = _split(case, s["qkv"])
        kv.append(k, v, s["seq"], s["slot"], s["table"], rope=s["rope"], rope_pos=s["pos"], q=q, q_out=s["q_out"])
        return {"q": s["q_out"], **s["pool"]}
    kv.read(s["seq"], s["slot"], s["table"], k_out=s["k_out"], v_out=s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _rotated(case, x, cos, sin):
    """x [n x heads x D] fp32 with its first `rot` dimensions rotated; cos and sin [n x 1 x rot/2]."""
    r, h = case["rot"], case["rot"] // 2
    if case["layout"] == "interleaved":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:r]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., r:]), -1)


def _dequantised(values, scales):
    return values.float() if scales is None else values.float() * scales.unsqueeze(-1)


def _plain(op, s):
    case = s["case"]
    if op in ("rotate", "write"):
        at = s["pos"].long()
        cos, sin = s["cos"][at].unsqueeze(1), s["sin"][at].unsqueeze(1)
        if op == "rotate":
            return _rotated(case, s["x"].float(), cos, -sin if case["gradient"] else sin).to(s["x"].dtype)
        q, k, v = _split(case, s["qkv"])
        page = s["table"][s["seq"].long(), s["slot"].long() // case["page"]].long()
        slot = s["slot"].long() % case["page"]
        s["q_out"] = _rotated(case, q.float(), cos, sin).to(q.dtype)
        for name, x in (("k", _rotated(case, k.float(), cos, sin)), ("v", v.float())):
            values, scales = _quantise(x, case["fmt"])
            s[name][page, :, slot] = values
            if scales is not None:
                s[name + "s"][page, :, slot] = scales
        return {"q": s["q_out"], **{n: s[n] for n in ("k", "v", "ks", "vs") if s[n] is not None}}
    if op == "read":
        page = s["table"][s["seq"].long(), s["slot"].long() // case["page"]].long()
        slot = s["slot"].long() % case["page"]
        dtype = s["k_out"].dtype
        k = _dequantised(s["k"][page, :, slot], None if s["ks"] is None else s["ks"][page, :, slot])
        v = _dequantised(s["v"][page, :, slot], None if s["vs"] is None else s["vs"][page, :, slot])
        return {"k": k.to(dtype), "v": v.to(dtype)}
    B, T, H, D = case["seqs"], case["new"], case["kv_heads"], case["head_dim"]
    G, table = case["q_heads"] // H, s["table"].long()

    def cached(name):   # [B x H x keys x D] fp32
        x = _dequantised(s[name][table], None if s[name + "s"] is None else s[name + "s"][table])
        return x.transpose(1, 2).reshape(B, H, -1, D)

    k, v = cached("k"), cached("v")
    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    score = (q @ k.transpose(-1, -2)).view(B, H, T, G, -1) / math.sqrt(D)
    j = torch.arange(k.shape[2], device=DEV)
    p = (s["lengths"].unsqueeze(1) - T + torch.arange(T, device=DEV)).view(B, 1, T, 1, 1)
    seen = (j <= p) & (j >= s["starts"].view(B, 1, 1, 1, 1))
    if case["window"]:
        seen = seen & (j > p - case["window"])
    score = torch.where(seen, score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(B, H, T * G, -1) @ v) / torch.where(total > 0, total, torch.ones_like(total)).view(B, H, T * G, 1)
    out = out.view(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B * T, H * G, D).to(s["q"].dtype)
    lse = (top + torch.log(total)).view(B, H, T, G).permute(0, 2, 1, 3).reshape(B * T, H * G)
    return {"out": out, "lse": torch.where(torch.isnan(lse), torch.full_like(lse, -math.inf), lse)}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------
def _turned64(case, x, pos, sign):
    z, h = x.double().clone(), case["rot"] // 2
    angle = pos.double().view(-1, 1, 1) * torch.from_numpy(_turns(case)).to(DEV) * sign
    first = slice(0, 2 * h, 2) if case["layout"] == "interleaved" else slice(0, h)
    second = slice(1, 2 * h, 2) if case["layout"] == "interleaved" else slice(h, 2 * h)
    w = torch.complex(z[..., first], z[..., second]) * torch.polar(torch.ones_like(angle), angle)
    z[..., first], z[..., second] = w.real, w.imag
    return z


def _stored64(z, fmt):
    """Rows in the cache's 8-bit floating format: (codes, scales); 16-bit formats hold z itself."""
    if fmt != "e4m3":
        return z, None
    scale = z.abs().amax(-1) / 448.0
    u = torch.where(scale.unsqueeze(-1) > 0, z / scale.unsqueeze(-1), torch.zeros_like(z))
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))).clamp(max=8.0) - 3.0)
    return (torch.round(u / step) * step).clamp(-448.0, 448.0), scale


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "rotate":
        return _turned64(case, x["x"], x["pos"], -1.0 if case["gradient"] else 1.0)
    if case["op"] == "write":
        q, k, v = _split(case, x["qkv"])
        page = x["table"].cpu().numpy()[x["seq"].cpu().numpy(), x["slot"].cpu().numpy() // case["page"]]
        page, slot = torch.from_numpy(page).long().to(DEV), x["slot"].long() % case["page"]
        got = {"q": _turned64(case, q, x["pos"], 1.0)}
        for name, rows in (("k", _turned64(case, k, x["pos"], 1.0)), ("v", v.double())):
            values, scales = _stored64(rows, case["fmt"])
            shape = (x["table"].numel(), case["kv_heads"], case["page"])
            got[name] = torch.zeros(*shape, case["head_dim"], dtype=torch.float64, device=DEV)
            got[name][page, :, slot] = values
            if scales is not None:
                got[name + "s"] = torch.zeros(shape, dtype=torch.float64, device=DEV)
                got[name + "s"][page, :, slot] = scales
        return got

    def rows64(name, seq, n):   # the first n cached tokens of a sequence: [heads x n x D]
        pages = x["table"][seq, : -(-n // case["page"])].long()
        z = x[name][pages].double()
        if x[name + "s"] is not None:
            z = z * x[name + "s"][pages].double().unsqueeze(-1)
        return z.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, case["head_dim"])[:, :n]

    if case["op"] == "read":
        return {n: torch.cat([rows64(n, b, m).transpose(0, 1) for b, m in enumerate(_lengths(case))]) for n in ("k", "v")}
    T, H, G = case["new"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    outs, lses = [], []
    for b, (n, start) in enumerate(zip(_lengths(case), _starts(case))):
        q = x["q"][b * T:(b + 1) * T].double().view(T, H, G, -1)
        lo = max(start, n - T - case["window"] + 1 if case["window"] else 0, 0)
        k, v = rows64("k", b, n)[:, lo:], rows64("v", b, n)[:, lo:]
        out = torch.zeros(T, H * G, case["head_dim"], dtype=torch.float64, device=DEV)
        lse = torch.full((T, H * G), -math.inf, dtype=torch.float64, device=DEV)
        for t in range(T):
            p = n - T + t
            a, e = max(start, p - case["window"] + 1 if case["window"] else 0, 0) - lo, p + 1 - lo
            if e <= a or p < 0:
                continue
            score = torch.einsum("hgd,hjd->hgj", q[t], k[:, a:e]) * case["head_dim"] ** -0.5
            out[t] = torch.einsum("hgj,hjd->hgd", torch.softmax(score, -1), v[:, a:e]).reshape(H * G, -1)
            lse[t] = torch.logsumexp(score, -1).reshape(-1)
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
