"""examples/decode_shared.py: shared prefixes, sampled verification, gathered weights and eviction together."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_shared.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decode_shared", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("kw", [{}, dict(queries=1, prompt_tokens=160), dict(queries=3, prompt_tokens=7, question_tokens=2)])
def test_it_runs(ex, capsys, kw):
    accepted, lengths, cut, kept, more = ex.main(**kw)
    prompt, question = kw.get("prompt_tokens", 150), kw.get("question_tokens", 20)
    assert all(0 <= a <= ex.K for a in accepted.tolist())
    assert lengths.tolist() == [prompt + question + a + 12 for a in accepted.tolist()]
    assert cut.tolist() == [min(96, n) for n in lengths.tolist()]
    for s, n in enumerate(lengths.tolist()):
        for row in kept[s].tolist():
            held = row[:int(cut[s])]
            assert held == sorted(set(held)) and set(range(max(0, n - 16), n)) <= set(held) <= set(range(n))
    assert ((more >= 0) & (more < ex.VOCAB)).all()
    assert "accepted drafts" in capsys.readouterr().out


def test_nothing_is_cut_from_short_contexts(ex):
    """With room for the whole contexts, decoding goes on as if they had not been cut."""
    prompt = torch.randint(0, ex.VOCAB, (37,), device="cuda", generator=torch.Generator("cuda").manual_seed(8))
    questions = torch.randint(0, ex.VOCAB, (2, 5), device="cuda", generator=torch.Generator("cuda").manual_seed(9)).int()
    tokens = []
    for cut in (False, True):
        m = ex.SharedModel(prompt, 3, 4, 2, "bf16", 2, 200)
        first = ex.ints([37, 37])
        logits = m.window(questions, first)
        token, lengths = logits[:, -1].argmax(-1).int(), first + 5
        weights = torch.zeros(2, 2, 208, device="cuda")
        token, lengths = ex.decode(m, token, lengths, 4, weights)
        to = m.table[:, 6:10].contiguous()
        if cut:
            lengths2, kept, _ = m.kv.evict(m.table, lengths, weights, 56, to)
            assert lengths2.tolist() == lengths.tolist() == [46, 46]
            tokens.append(ex.decode_cut(m, token, lengths, to, lengths2, 6))
        else:
            tokens.append(ex.decode_cut(m, token, lengths, m.table, lengths, 6))
        m.kv.sync()
    assert torch.equal(tokens[0], tokens[1])
