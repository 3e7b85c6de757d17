"""A miss from lookup to verification, on small random models: the lookup, then the decoding calls together.

    python examples/decode_miss.py

Queries are looked up; those that are not served are decoded. A draft model writes k tokens one at a time on a paged e4m3
cache (append and attend, captured once into a CUDA graph), the target model verifies them in one pass of k + 1 new tokens on
a bf16 cache, and the accepted part is put behind another prompt: its keys are read back, turned back to position 0, and
written to their new positions. The models are one attention layer between an embedding and its transpose; their products
are torch's.
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2608_01718_gb300 import lacache as L  # noqa: E402

VOCAB, WIDTH, HEAD_DIM, K = 512, 256, 64, 16


def ints(values):
    return torch.as_tensor(values, dtype=torch.int32, device="cuda")


class Model:
    """Embedding, one layer of grouped attention over its own paged cache, logits. Sequence s owns row s of the table."""

    def __init__(self, seed, q_heads, kv_heads, fmt, seqs, reach, page=16, embed=None):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device="cuda") / rows ** 0.5).to(torch.bfloat16)

        self.q_heads, self.kv_heads, self.seqs = q_heads, kv_heads, seqs
        self.embed = torch.randn(VOCAB, WIDTH, generator=gen, device="cuda").to(torch.bfloat16) if embed is None else embed
        self.w_in = matrix(WIDTH, (q_heads + 2 * kv_heads) * HEAD_DIM)
        self.w_out = matrix(q_heads * HEAD_DIM, WIDTH)
        width = -(-reach // page)
        self.kv = L.KVCache(kv_heads, HEAD_DIM, seqs * width, page, fmt)
        self.table = torch.randperm(seqs * width, generator=gen, device="cuda").to(torch.int32).view(seqs, width)
        self.rope = L.Rope(HEAD_DIM)

    def forward(self, tokens, seq, pos, lengths, new_tokens):
        """Logits [tokens x vocabulary] of new tokens (int32), new_tokens a sequence, at their positions; the cache gets them.
        ``lengths`` counts them in."""
        x = self.embed[tokens.long()]
        qkv = (x @ self.w_in).view(-1, self.q_heads + 2 * self.kv_heads, HEAD_DIM)
        q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        q = self.kv.append(k, v, seq, pos, self.table, rope=self.rope, q=q)
        out = self.kv.attend(q, self.table, lengths, new_tokens=new_tokens)
        x = x + out.flatten(1) @ self.w_out
        return x.float() @ self.embed.float().T / WIDTH ** 0.5

    def prefill(self, prompts):
        """Prompts of one length [sequences x n], all but the last token: that one starts the decoding."""
        n = prompts.shape[1] - 1
        seq = torch.arange(self.seqs, device="cuda").repeat_interleave(n).int()
        pos = torch.arange(n, device="cuda").repeat(self.seqs).int()
        self.forward(prompts[:, :-1].reshape(-1).int(), seq, pos, ints([n] * self.seqs), n)


def draft_prefix(model, prompts, k=K):
    """k greedy tokens a sequence, and the model's probabilities of them: one captured step, replayed."""
    n, seqs = prompts.shape[1], model.seqs
    model.prefill(prompts)
    tokens, pos, lengths = prompts[:, -1].int().contiguous(), ints([n - 1] * seqs), ints([n] * seqs)
    seq, p = ints(range(seqs)), torch.empty(seqs, device="cuda")
    start = [t.clone() for t in (tokens, pos, lengths)]

    def step():
        top = torch.softmax(model.forward(tokens, seq, pos, lengths, 1), -1).max(-1)
        p.copy_(top.values)
        tokens.copy_(top.indices)
        pos.add_(1)
        lengths.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                            # warm-up; then back to the start
        for t, was in zip((tokens, pos, lengths), start):
            t.copy_(was)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    drafts, probs = [], []
    for _ in range(k):
        graph.replay()
        drafts.append(tokens.clone())
        probs.append(p.clone())
    return torch.stack(drafts, 1), torch.stack(probs, 1)


def verify(model, prompts, drafts, p_draft, status):
    """The target's probabilities of the drafts, in one pass, and how many of each sequence's it accepts."""
    n, k, seqs = prompts.shape[1], drafts.shape[1], model.seqs
    model.prefill(prompts)
    window = torch.cat((prompts[:, -1:].int(), drafts), 1)               # the token before them, and the drafts
    seq = torch.arange(seqs, device="cuda").repeat_interleave(k + 1).int()
    pos = torch.arange(n - 1, n + k, device="cuda").repeat(seqs).int()
    logits = model.forward(window.reshape(-1), seq, pos, ints([n + k] * seqs), k + 1).view(seqs, k + 1, VOCAB)
    p = torch.softmax(logits[:, :k], -1).gather(-1, drafts.long().unsqueeze(-1)).squeeze(-1).contiguous()
    accepted = torch.empty(seqs, dtype=torch.int32, device="cuda")
    L.lacache_verify_draft(p, p_draft.contiguous(), status, accepted)
    return p, accepted


def move(model, frm, first, count, to, at):
    """Cached tokens [first, first + count) of sequence frm become tokens at, at + 1, ... of sequence to (the same model's):
    their keys are turned back by their old positions and written with their new ones. Values carry no position."""
    old = torch.arange(first, first + count, device="cuda").int()
    k, v = model.kv.read(ints([frm] * count), old, model.table)
    bare = model.rope.apply(k, old, inverse=True)
    model.kv.append(bare, v, ints([to] * count), torch.arange(at, at + count, device="cuda").int(), model.table, rope=model.rope)
    return bare, v


def main():
    torch.manual_seed(0)
    queries, n = 4, 40
    q_emb = torch.nn.functional.normalize(torch.randn(queries, 64, device="cuda"), dim=-1).to(torch.bfloat16)
    prompts = torch.randint(0, VOCAB, (queries, n), device="cuda")
    draft = Model(1, 4, 4, "e4m3", queries, n + K)
    target = Model(2, 8, 2, "bf16", queries, 2 * (n + K), embed=draft.embed)

    drafts, p_draft = draft_prefix(draft, prompts)
    q_prefix = torch.nn.functional.normalize(draft.embed[drafts.long()].float().mean(1)[:, :64], dim=-1).to(torch.bfloat16)
    cache = L.LaCache(d=64, k=K, capacity=64, tau_c=0.9, tau_a=0.8, top_c=2, max_batch=queries)
    cache.insert(q_emb[:1], q_prefix[:1], drafts[:1].contiguous())       # the first query has been answered before
    found = cache.lookup(q_emb, q_prefix, drafts.contiguous())

    p_target, accepted = verify(target, prompts, drafts, p_draft, found["status"])
    cache.append_misses(q_emb, q_prefix, drafts.contiguous(), found["status"])
    count = int(accepted.max())
    if count > 0:                                                        # the longest accepted part, behind prompt 0
        move(target, int(accepted.argmax()), n, count, 0, n + K)
    draft.kv.sync()
    target.kv.sync()
    print("served:", (found["status"] == L.LACACHE_HIT).tolist(), "accepted drafts:", accepted.tolist(), "entries:", cache.size)
    return found, accepted


if __name__ == "__main__":
    main()
