"""The example of sampling with drafted tokens: what it hands over and what it keeps."""
import os
import sys

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_prefill_returns_the_keys_that_its_last_step_used(monkeypatch):
    import draft_decode
    seen = []
    step = wise.WiseAttention.step

    def record(self, t, Q, K, V, O, stream=None):
        seen.append((t, Q.clone(), K.clone(), V.clone()))
        step(self, t, Q, K, V, O, stream)

    monkeypatch.setattr(wise.WiseAttention, "step", record)
    torch.manual_seed(0)
    model = draft_decode.StandIn(101, 4, 2, 64, 0)
    K, V = draft_decode.prefill(model, torch.arange(64, device="cuda") % 101, steps=4, discovery=2)
    assert [t for t, *_ in seen] == [0, 1, 2, 3]
    assert torch.equal(K, seen[-1][2]) and torch.equal(V, seen[-1][3])
    for (_, Q0, K0, _), (_, Q1, K1, _) in zip(seen, seen[1:]):
        assert not torch.equal(Q0, Q1) and not torch.equal(K0, K1)   # every step has its own


def test_a_pool_that_runs_out_costs_no_token_of_the_prompt(monkeypatch):
    """Samples that are granted nothing in a round keep what they hold; the shortage is reported."""
    import draft_decode
    made = []

    class Small(serve.PagedCache):
        def __init__(self, n_layers, n_pages, *a, **kw):
            super().__init__(n_layers, 10, *a, **kw)   # 8 for the prompt's 255 tokens, one copy, one more
            made.append(self)

    def refuse_all(p, q, drafted, *rest):
        accepted = torch.zeros(p.shape[0], dtype=torch.int32, device="cuda")
        return accepted, torch.zeros(p.shape[:2], dtype=torch.int32, device="cuda")

    monkeypatch.setattr(serve, "PagedCache", Small)
    monkeypatch.setattr(serve, "verify_draft", refuse_all)
    lens = []
    drop = Small.drop
    monkeypatch.setattr(Small, "drop", lambda self, *a, **kw: (drop(self, *a, **kw), lens.append(self.lens.tolist()))[0])
    with pytest.raises(RuntimeError, match="free pages"):
        draft_decode.run(samples=4, rounds=3, draft=3, prompt_len=256, vocab=331)
    assert made and len(lens) >= 3
    for x in lens[:3]:
        assert min(x) >= 255, lens
