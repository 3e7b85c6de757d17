"""Queries behind one system prompt, decoded on one copy of its keys and values, on small random models.

    python examples/decode_shared.py

The prompt's full pages are in every query's row of the table; the page that it ends in is copied. A draft model samples k tokens a
query; the target model reads them in one pass over the shared prefix and accepts or replaces them by given random numbers, so that
what is decoded is distributed as its own tokens. Then it goes on token by token, each cached token gathering the attention weight
that it gets, until every context is cut to the tokens of the largest weights and the last ones, and decoding continues on those.
The models are one attention layer between an embedding and its transpose; their products are torch's.
"""
from __future__ import annotations

import os
import sys

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]

import torch  # noqa: E402

from decode_miss import HEAD_DIM, K, VOCAB, WIDTH, Model, ints  # noqa: E402
from paper_2608_01718_gb300 import lacache as L  # noqa: E402


class SharedModel(Model):
    """A model whose sequences have a prompt's full pages in common: row s of the table starts with row 0's."""

    def __init__(self, prompt, *args, **kw):
        super().__init__(*args, **kw)
        self.prompt, self.common = prompt, ints([prompt.numel()])
        n, full = prompt.numel(), prompt.numel() // self.kv.cfg.page_size
        self.table[:, :full] = self.table[:1, :full].clone()
        zeros, pos = ints([0] * n), ints(range(n))
        _, _, k, v = self.project(prompt)          # (with one layer, the prompt's keys and values need no attention)
        self.kv.append(k, v, zeros, pos, self.table, rope=self.rope)
        rest, others = pos[full * self.kv.cfg.page_size:], self.seqs - 1
        if rest.numel() and others:
            k, v = self.kv.read(zeros[:rest.numel()], rest, self.table)
            seq = ints(range(1, self.seqs)).repeat_interleave(rest.numel())
            self.kv.append(k.repeat(others, 1, 1), v.repeat(others, 1, 1), seq, rest.repeat(others), self.table)

    def project(self, tokens):
        x = self.embed[tokens.long()]
        qkv = (x @ self.w_in).view(-1, self.q_heads + 2 * self.kv_heads, HEAD_DIM)
        return x, *qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)

    def forward(self, tokens, seq, pos, lengths, new_tokens, lse=None):
        """As Model.forward, the prompt read once for all sequences; also returns the rotated queries."""
        x, q, k, v = self.project(tokens)
        q = self.kv.append(k, v, seq, pos, self.table, rope=self.rope, q=q)
        out = self.kv.attend_shared(q, self.table, lengths, self.common, new_tokens=new_tokens, lse=lse)
        return self.logits(x, out), q

    def logits(self, x, out):
        return (x + out.flatten(1) @ self.w_out).float() @ self.embed.float().T / WIDTH ** 0.5

    def window(self, tokens, first):
        """New tokens [sequences x n] at positions first (int32 [sequences]) and on: their logits [sequences x n x vocabulary]."""
        n = tokens.shape[1]
        seq = ints(range(self.seqs)).repeat_interleave(n)
        pos = (first.unsqueeze(1) + ints(range(n))).reshape(-1)
        return self.forward(tokens.reshape(-1), seq, pos, first + n, n)[0].view(self.seqs, n, VOCAB)


def draft(model, last, first, k=K):
    """k tokens a sequence, sampled from the model's probabilities, which come with them [sequences x k x vocabulary]."""
    drafts, probs = [], []
    for i in range(k):
        p = torch.softmax(model.window(last, first + i)[:, 0], -1)
        last = torch.multinomial(p, 1).int()
        drafts.append(last)
        probs.append(p)
    return torch.cat(drafts, 1), torch.stack(probs, 1)


def verify(model, last, drafts, p_draft, first, u):
    """The target's probabilities of the window in one pass, how many drafts of each sequence are accepted, and its next token."""
    p = torch.softmax(model.window(torch.cat((last, drafts), 1), first), -1)
    accepted, token = (torch.empty(model.seqs, dtype=torch.int32, device="cuda") for _ in range(2))
    L.lacache_verify_sample(p, p_draft, drafts.contiguous(), u, accepted, token)
    return p, accepted, token


def decode(model, token, lengths, steps, weights, decay=0.9):
    """Greedy tokens behind contexts of `lengths`, the cached tokens' weights gathered in place. Returns tokens and lengths."""
    seq, lse = ints(range(model.seqs)), torch.empty(model.seqs, model.q_heads, device="cuda")
    for _ in range(steps):
        logits, q = model.forward(token, seq, lengths, lengths + 1, 1, lse)
        lengths = lengths + 1
        model.kv.weigh(q, model.table, lengths, lse, weights=weights, decay=decay)
        token = logits.argmax(-1).int()
    return token, lengths


def decode_cut(model, token, positions, to, lengths, steps):
    """Greedy tokens on contexts that were cut: a token is rotated by its position and written behind what is kept."""
    seq, tokens = ints(range(model.seqs)), []
    for i in range(steps):
        x, q, k, v = model.project(token)
        q = model.kv.append(k, v, seq, lengths + i, to, rope=model.rope, rope_pos=positions + i, q=q)
        out = model.kv.attend(q, to, lengths + i + 1)
        token = model.logits(x, out).argmax(-1).int()
        tokens.append(token)
    return torch.stack(tokens, 1)


def main(queries=4, prompt_tokens=150, question_tokens=20, steps=12, keep=96, recent=16):
    torch.manual_seed(0)
    prompt = torch.randint(0, VOCAB, (prompt_tokens,), device="cuda")
    questions = torch.randint(0, VOCAB, (queries, question_tokens), device="cuda").int()
    reach, page = prompt_tokens + question_tokens + K + 1 + steps, 16
    used, spare = -(-reach // page), -(-(keep + steps) // page)
    small = SharedModel(prompt, 1, 4, 4, "e4m3", queries, reach, page)
    target = SharedModel(prompt, 2, 8, 2, "bf16", queries, (used + spare) * page, page, embed=small.embed)
    first = ints([prompt_tokens] * queries)
    for model in (small, target):
        model.window(questions[:, :-1], first)
    first, last = first + question_tokens - 1, questions[:, -1:]
    drafts, p_draft = draft(small, last, first)
    p_target, accepted, token = verify(target, last, drafts, p_draft, first, torch.rand(queries, K + 1, device="cuda"))

    lengths = first + 1 + accepted                       # the window's token before the drafts, and those accepted
    weights = torch.zeros(queries, target.kv_heads, used * page, device="cuda")
    token, lengths = decode(target, token, lengths, steps, weights)
    to = target.table[:, used:].contiguous()             # the pages behind the contexts
    cut, kept, _ = target.kv.evict(target.table, lengths, weights, keep, to, recent=recent)
    more = decode_cut(target, token, lengths, to, cut, steps)
    small.kv.sync()
    target.kv.sync()
    print("accepted drafts:", accepted.tolist(), "contexts:", lengths.tolist(), "cut to:", cut.tolist())
    return accepted, lengths, cut, kept, more


if __name__ == "__main__":
    main()
