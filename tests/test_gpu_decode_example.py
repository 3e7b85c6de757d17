"""examples/decode_miss.py: the decoding calls together."""
import importlib.util
import os

import pytest
import torch

from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_miss.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decode_miss", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_it_runs(ex, capsys):
    found, accepted = ex.main()
    status = found["status"].tolist()
    assert status[0] == L.LACACHE_HIT and all(s != L.LACACHE_HIT for s in status[1:])
    assert accepted[0] == -1 and all(0 <= a <= ex.K for a in accepted[1:].tolist())
    assert "served" in capsys.readouterr().out


def test_graph_steps_equal_eager_steps(ex):
    prompts = torch.randint(0, ex.VOCAB, (3, 21), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    drafts, p = ex.draft_prefix(ex.Model(1, 4, 2, "int8", 3, 40), prompts, 8)
    m = ex.Model(1, 4, 2, "int8", 3, 40)
    m.prefill(prompts)
    tokens = prompts[:, -1].int()
    for i in range(8):
        top = torch.softmax(m.forward(tokens.contiguous(), ex.ints(range(3)), ex.ints([20 + i] * 3), ex.ints([21 + i] * 3), 1), -1).max(-1)
        tokens = top.indices.int()
        assert torch.equal(tokens, drafts[:, i]) and torch.equal(top.values, p[:, i])


def test_verification_is_the_acceptance_rule(ex):
    prompts = torch.randint(0, ex.VOCAB, (4, 30), device="cuda", generator=torch.Generator("cuda").manual_seed(6))
    drafts, p_draft = ex.draft_prefix(ex.Model(1, 4, 4, "e4m3", 4, 46), prompts)
    p, accepted = ex.verify(ex.Model(2, 8, 2, "bf16", 4, 46), prompts, drafts, p_draft, None)
    want = (p >= p_draft).int().cumprod(1).sum(1)
    assert torch.equal(accepted.long(), want.long())


def test_moved_keys(ex):
    """A key turned back and turned again: the second turn is rope.apply's, bit for bit; the way back and forth rounds to bf16
    three times (each within 2^-8 of a component, so of the pair's norm), the products of other rows once more."""
    prompts = torch.randint(0, ex.VOCAB, (2, 50), device="cuda", generator=torch.Generator("cuda").manual_seed(7))
    m = ex.Model(3, 4, 2, "bf16", 2, 96)
    m.prefill(prompts)
    bare, v = ex.move(m, 0, 10, 17, 1, 60)
    fresh = (m.embed[prompts[0, 10:27]] @ m.w_in).view(17, -1, ex.HEAD_DIM)[:, 4:6].double()
    h = ex.HEAD_DIM // 2
    norm = torch.hypot(fresh[..., :h], fresh[..., h:]).repeat(1, 1, 2)
    assert ((bare.double() - fresh).abs() <= 4 * 2 ** -8 * norm * (1 + 2 ** -6)).all()
    at = ex.ints(range(60, 77))
    k2, v2 = m.kv.read(ex.ints([1] * 17), at, m.table)
    assert torch.equal(k2, m.rope.apply(bare, at)) and torch.equal(v2, v)
