"""Attention over caches in 8 or 4 bits when a wait has run out: the call ends within its limit, whatever the others of a
CTA were at, and the next call is right."""
import pytest
import torch

from paper_2609_27373_gb300 import wise
from quant_helpers import build
from serve_helpers import u32
from test_quant_attn_gpu import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_heads,tokens", [(16, 700), (16, 1500), (16, 2600), (80, 1500)])
def test_a_call_whose_wait_has_run_out_ends_soon(bits, n_heads, tokens):
    """Ordinary bounded waits with a limit of 1 ns give up at many places, between the two ends of a CTA's work among them
    (16 heads: two teams for V, an end for each); none of the waits for copies in flight may then last the default 2 s."""
    lens = [tokens + 37 * i % 500 for i in range(160)]
    cache, twin, slots, gen = build(bits, lens, 64, 4, 128, torch.bfloat16, n_heads + tokens)
    Q = torch.randn((160, n_heads, 1, 128), generator=gen, device="cuda").bfloat16()
    O, s, longest, ran_out = torch.empty_like(Q), u32(slots), 0.0, False
    cache.attend(0, Q, O, s)
    torch.cuda.synchronize()
    wise.wise_set_wait_limit_ns(1)
    try:
        for i in range(100):
            s.copy_(u32(slots[i % 7:] + slots[:i % 7]))
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            cache.attend(0, Q, O, s)
            b.record()
            ran_out |= wise.wise_get_status() == wise.WISE_ERR_TIMEOUT
            longest = max(longest, a.elapsed_time(b))
            if longest >= 1000.0:
                break
    finally:
        wise.wise_set_wait_limit_ns(0)
    assert ran_out and longest < 1000.0, longest
    run(cache, twin, slots, gen, n_heads, 1)
    assert wise.wise_get_status() == wise.WISE_OK
