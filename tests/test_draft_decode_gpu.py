"""The example of sampling with drafted tokens: what it hands over and what it keeps."""
import os
import sys

import pytest
import torch

from paper_2609_27373_gb300 import wise

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
