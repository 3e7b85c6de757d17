"""Seeded caches for the tests of the decoding operators: a filled cache whose every unused slot and table entry holds what a
kernel must not use, with the fp64 values it stands for."""
import numpy as np
import torch

from paper_2608_01718_gb300 import lacache as L

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


class Filled:
    """A cache with `lengths` tokens a sequence, written through append."""

    def __init__(self, fmt, lengths, kv_heads, head_dim, page=16, dtype=None, seed=0, spread=1.0, layers=1, layer=0,
                 spare=3):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.lengths, self.page, self.layer = list(lengths), page, layer
        dtype = TORCH[dtype or (fmt if fmt in TORCH else "bf16")]
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + spare
        self.kv = L.KVCache(kv_heads, head_dim, pages, page, fmt, layers=layers)
        for i in range(layers):
            self.poison(i)
        width = max(used + [1]) + 1
        table = np.full((len(lengths), width), 1 << 29, dtype=np.int32)      # never to be read past a sequence's own
        order = rng.permutation(pages)
        at = 0
        for s, u in enumerate(used):
            table[s, :u] = order[at:at + u]
            at += u
        self.host_table = table
        self.table = torch.from_numpy(table).cuda()
        n = sum(lengths)
        self.seq = torch.from_numpy(np.repeat(np.arange(len(lengths)), lengths).astype(np.int32)).cuda()
        self.pos = torch.from_numpy(np.concatenate([np.arange(m) for m in lengths] + [np.zeros(0)]).astype(np.int32)).cuda()
        k = (torch.randn(n, kv_heads, head_dim, generator=gen, device="cuda") * spread).to(dtype)
        v = torch.randn(n, kv_heads, head_dim, generator=gen, device="cuda").to(dtype)
        v *= torch.exp2(torch.randint(-6, 7, (n, kv_heads, 1), generator=gen, device="cuda")).to(dtype)
        self.k_rows, self.v_rows = k, v
        self.kv.append(k, v, self.seq, self.pos, self.table, layer=layer)
        self.len_dev = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def poison(self, layer):
        """NaN everywhere: in 16-bit values, or in codes and scales."""
        pool = self.kv.pool(layer)
        for name, t in pool.items():
            if t.dtype == torch.int8:
                t.fill_(-128)
            elif t.dtype == torch.float8_e4m3fn:
                t.view(torch.uint8).fill_(0x7f)
            else:
                t.fill_(float("nan"))

    def values(self):
        """Per sequence ([tokens x kv_heads x d] k, the same of v) as fp64."""
        pool = self.kv.pool(self.layer)
        out = []
        for name in ("k", "v"):
            x = pool[name].double()
            if name + "s" in pool:
                x = x * pool[name + "s"].double().unsqueeze(-1)
            x = x.cpu().numpy()
            rows = []
            for s, n in enumerate(self.lengths):
                pages = self.host_table[s, : -(-n // self.page)]
                rows.append(x[pages].transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:n])
            out.append(rows)
        return out


def bounds(want, mass, span, lse, q, k, scale, dtype):
    """Error bounds of an attention's outputs, elementwise, from its arithmetic. The products of 16-bit values are exact in
    fp32 and summed in fp32: a score is off by at most delta = 2^-19 of the sum of |q k| * scale (256 terms, each step
    rounding within 2^-24 of at most that sum, then the scale, the base-2 exponent and the shift), and by what a q scaled
    into f16 loses below 2^-24 of its row's largest magnitude against any key. exp turns that into a relative error
    2 delta of numerator and denominator; weights are held to 2^-11 or better of themselves (or, below 2^-14 of the largest,
    2^-25 of it, for at most 2^13 keys a partial); the output is rounded once."""
    q_top = np.abs(q).max(-1)
    k_sum = max([np.abs(x).sum(-1).max() if x.size else 0.0 for x in k] + [0.0])
    delta = 2.0 ** -19 * span + 2.0 ** -24 * q_top * k_sum * abs(scale)
    out = {"bf16": 2.0 ** -8, "f16": 2.0 ** -10}[dtype] * np.abs(want) + (2.0 ** -10 + 4 * delta)[..., None] * mass + 2.0 ** -24
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return out, 2 * delta + 2.0 ** -19 * (1 + finite)
