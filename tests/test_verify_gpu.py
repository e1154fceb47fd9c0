"""Verification of drafted tokens against the rule in Python integers (every comparison is exact)."""
import numpy as np
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import u32, verify

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def case(B, K, V, dtype, seed, near=0.4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.randn((B, K + 1, V), generator=g, device="cuda") * 2
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :K] + near * torch.randn((B, K, V), generator=g, device="cuda"), -1)
    draft = torch.multinomial(q.reshape(B * K, V), 1, generator=g).reshape(B, K).int() if K else u32([]).reshape(B, 0)
    return (p.to(dtype), q.to(dtype), draft, torch.rand((B, K), generator=g, device="cuda"),
            torch.rand((B,), generator=g, device="cuda"))


def both(p, q, draft, n_draft, ua, us):
    acc, tok = serve.verify_draft(p, q, draft, None if n_draft is None else u32(n_draft), ua, us)
    want = verify(p.float().cpu().numpy(), q.float().cpu().numpy(), draft.tolist(), n_draft, ua.cpu().numpy(),
                  us.cpu().numpy())
    assert acc.tolist() == want[0]
    assert tok.tolist() == want[1]
    return want


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 2, 2), (2, 4, 31), (5, 3, 33), (4, 5, 1000), (3, 4, 4099), (2, 2, 32000),
                                   (2, 1, 131075), (1, 1, 1 << 18), (2, 40, 257)])
def test_rule(dtype, B, K, V):
    p, q, draft, ua, us = case(B, K, V, dtype, seed=B * 1000 + V)
    both(p, q, draft, None, ua, us)
    both(p, q, draft, [(3 * b) % (K + 1) for b in range(B)], ua, us)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("dtype", TYPES)
def test_edges_of_the_random_numbers(dtype):
    """u = 0 accepts what has mass and takes the first token with weight; u next to 1 takes the last one."""
    p, q, draft, ua, us = case(8, 3, 500, dtype, seed=5)
    for a in (0.0, 1.0 - 2.0 ** -24, 1.0):
        for s in (0.0, 2.0 ** -24, 0.5, 1.0 - 2.0 ** -24, 1.0, float("nan"), -1.0):
            if s != s:
                continue
            both(p, q, draft, None, torch.full_like(ua, a), torch.full_like(us, s))


def test_no_residual_falls_back_to_the_target():
    """p == q with a refused token (u = 1): the residual is empty everywhere, so the target row is sampled."""
    p, q, draft, ua, us = case(6, 2, 700, torch.float32, seed=9)
    q = p[:, :2].clone()
    want = both(p, q, draft, None, torch.ones_like(ua), us)
    assert want[0] == [0] * 6 and all(t[0] >= 0 for t in want[1])


def test_one_token_has_all_the_mass_and_ties_take_the_lowest():
    V = 300
    p = torch.zeros((2, 2, V), device="cuda")
    q = torch.full((2, 1, V), 1.0 / V, device="cuda")
    p[0, :, 123] = 1.0
    p[1, :, 7] = 0.5
    p[1, :, 299] = 0.5
    draft = u32([[5], [5]])
    for us, last in ((0.0, 7), (0.49, 7), (0.51, 299)):
        want = both(p, q, draft, None, torch.full((2, 1), 0.5, device="cuda"), torch.full((2,), us, device="cuda"))
        assert want[1] == [[123, -1], [last, -1]]


def test_rows_without_mass_nan_and_infinities():
    V = 200
    p = torch.zeros((4, 2, V), device="cuda")
    q = torch.zeros((4, 1, V), device="cuda")
    p[1] = float("nan")
    p[2, :, 5] = float("inf")
    p[3, :, 9] = 2.0 ** -41          # below the resolution of the weights
    q[2, 0, 5] = float("inf")
    ua, us = torch.full((4, 1), 0.25, device="cuda"), torch.full((4,), 0.75, device="cuda")
    acc, tok = serve.verify_draft(p, q, u32([[0], [0], [5], [9]]), None, ua, us)
    # Row 2: inf * 0.25 < inf is false, the residual inf - inf counts as 0, the target row samples token 5.
    assert acc.tolist() == [0, 0, 0, 1]
    assert tok.tolist() == [[-1, -1], [-1, -1], [5, -1], [9, -1]]


def test_drafted_tokens_out_of_range_are_refused():
    p, q, draft, ua, us = case(3, 3, 100, torch.float32, seed=3, near=0.0)
    draft[0, 0], draft[1, 1], draft[2, 2] = 100, -5, 1 << 30
    ua.zero_()
    want = both(p, q, draft, None, ua, us)
    assert want[0] == [0, 1, 2]
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    both(p, q, draft, [0, 1, 2], ua, us)   # never reached: not a fault
    assert wise.wise_get_status() == wise.WISE_OK


def test_counts_out_of_range_are_clamped_and_reported():
    p, q, draft, ua, us = case(2, 2, 50, torch.float32, seed=4)
    both(p, q, draft, [-1, 3], ua, us)
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE


def test_without_drafts_it_samples_the_target():
    p, q, draft, ua, us = case(5, 0, 777, torch.bfloat16, seed=11)
    acc, tok = serve.verify_draft(p, None, None, None, None, us)
    want = verify(p.float().cpu().numpy(), np.zeros((5, 0, 777), np.float32), [[]] * 5, None, np.zeros((5, 0)),
                  us.cpu().numpy())
    assert acc.tolist() == want[0] and tok.tolist() == want[1]


def test_repeats_are_equal():
    p, q, draft, ua, us = case(64, 4, 50001, torch.bfloat16, seed=21)
    first = serve.verify_draft(p, q, draft, None, ua, us)
    for _ in range(5):
        again = serve.verify_draft(p, q, draft, None, ua, us)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_refusals_of_the_binding():
    p, q, draft, ua, us = case(2, 2, 50, torch.float32, seed=4)
    for bad in ((p, q.half(), draft, None, ua, us), (p, q[:, :1], draft, None, ua, us),
                (p, q, draft.long(), None, ua, us), (p, q, draft, None, ua.double(), us), (p, None, draft, None, ua, us),
                (p.transpose(0, 1), q, draft, None, ua, us)):
        with pytest.raises(ValueError):
            serve.verify_draft(*bad)
