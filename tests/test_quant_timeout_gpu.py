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
@pytest.mark.parametrize("n_heads", [4, 20])
def test_a_call_whose_wait_has_run_out_ends_soon(bits, n_heads):
    """An item a CTA, of a length at which the first wait to run out (the hardware holds one for some microseconds before
    its limit is looked at) does so next to the end of the CTA's work, between the two ends that the teams of V get among
    other places.  None of the waits for copies in flight may then last the default 2 s."""
    B = torch.cuda.get_device_properties(0).multi_processor_count
    cache, twin, slots, gen = build(bits, [1700] * B, 64, 1, 128, torch.bfloat16, n_heads)
    Q = torch.randn((B, n_heads, 1, 128), generator=gen, device="cuda").bfloat16()
    O, s, longest, ran_out = torch.empty_like(Q), u32(slots), 0.0, 0
    cache.attend(0, Q, O, s)
    torch.cuda.synchronize()
    wise.wise_set_wait_limit_ns(1)
    try:
        for tokens in range(600, 1700, 20):
            cache.lens.fill_(tokens)
            for _ in range(10):
                a, b = torch.cuda.Event(True), torch.cuda.Event(True)
                a.record()
                cache.attend(0, Q, O, s)
                b.record()
                ran_out += wise.wise_get_status() == wise.WISE_ERR_TIMEOUT
                longest = max(longest, a.elapsed_time(b))
            if longest >= 1000.0:
                break
    finally:
        wise.wise_set_wait_limit_ns(0)
    assert ran_out > 100 and longest < 1000.0, (ran_out, longest)
    cache.lens.fill_(1700)
    run(cache, twin, slots, gen, n_heads, 1)
    assert wise.wise_get_status() == wise.WISE_OK
