"""Verification of full batches over the largest vocabulary, and of random numbers that are none (every comparison is
exact)."""
import numpy as np
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import u32, verify

pytestmark = pytest.mark.gpu


def rule(p, q, draft, ua, us):
    """The rule of wise_verify_draft for rows without faults, in 64-bit integers row by row; p, q as fp32 arrays."""
    accepted, tokens = [], []
    for b in range(p.shape[0]):
        k, n = q.shape[1], 0
        while n < k and np.float32(ua[b, n]) * q[b, n, draft[b, n]] < p[b, n, draft[b, n]]:
            n += 1
        r = p[b, n] if n == k else np.maximum(p[b, n] - q[b, n], np.float32(0))
        w = np.floor(np.clip(r.astype(np.float64), 0.0, 1.0) * 2.0 ** 40).astype(np.int64)
        if not w.any():
            w = np.floor(np.clip(p[b, n].astype(np.float64), 0.0, 1.0) * 2.0 ** 40).astype(np.int64)
        cum = np.cumsum(w)   # below 2^58
        u = 0.0 if np.isnan(us[b]) else min(max(float(us[b]), 0.0), 1.0 - 2.0 ** -24)
        t = int(cum[-1]) * int(u * 2 ** 24) >> 24
        accepted.append(n)
        tokens.append([int(x) for x in draft[b, :n]] + [int(np.searchsorted(cum, t, side="right")) if cum[-1] else -1] +
                      [-1] * (k - n))
    return accepted, tokens


@pytest.mark.parametrize("B,V,dtype", [(130, 1 << 18, torch.bfloat16), (101, (1 << 18) - 1, torch.float16),
                                       (110, 131075, torch.float32)])
def test_full_batches(B, V, dtype):
    """More requests than one wave of the largest clusters holds; rows of every kind, weights of 1.0 everywhere among
    them, which fill the lanes' 32-bit sums."""
    g = torch.Generator(device="cuda").manual_seed(B)
    logits = torch.randn((B, 2, V), generator=g, device="cuda") * 2
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :1] + 0.5 * torch.randn((B, 1, V), generator=g, device="cuda"), -1)
    p[0], p[1, 0], q[1] = 1.0, 1.0, 0.0
    p[2], q[2] = 0.0, 1.0
    p[3] = 0.0
    p[3, :, V - 1] = 1.0
    p, q = p.to(dtype), q.to(dtype)
    draft = torch.randint(0, V, (B, 1), generator=g, device="cuda").int()
    ua, us = torch.rand((B, 1), generator=g, device="cuda"), torch.rand((B,), generator=g, device="cuda")
    ua[1] = 1.0
    us[0], us[4] = 1.0 - 2.0 ** -24, 0.0
    acc, tok = serve.verify_draft(p, q, draft, None, ua, us)
    want = rule(p.float().cpu().numpy(), q.float().cpu().numpy(), draft.cpu().numpy(), ua.cpu().numpy(),
                us.cpu().numpy())
    assert acc.tolist() == want[0]
    assert tok.tolist() == want[1]
    assert wise.wise_get_status() == wise.WISE_OK


def test_a_random_number_that_is_none_counts_as_zero():
    """u_sample NaN takes the first token with weight; u_accept NaN refuses, since no comparison with it holds."""
    g = torch.Generator(device="cuda").manual_seed(1)
    p = torch.softmax(torch.randn((4, 2, 500), generator=g, device="cuda"), -1)
    p[:, :, :3] = 0.0
    q = p[:, :1].clone()
    q[:, :, 100:] *= 0.5
    draft, nan = u32([[200]] * 4), float("nan")
    ua = torch.tensor([[0.5], [nan], [0.5], [nan]], device="cuda")
    us = torch.tensor([nan, nan, 0.25, 0.25], device="cuda")
    acc, tok = serve.verify_draft(p, q, draft, None, ua, us)
    zero = torch.nan_to_num(us, 0.0)
    want = verify(p.cpu().numpy(), q.cpu().numpy(), draft.tolist(), None, ua.cpu().numpy(), zero.cpu().numpy())
    assert acc.tolist() == want[0] == [1, 0, 1, 0]
    assert tok.tolist() == want[1]
    assert want[1][0] == [200, 3] and want[1][1][0] == 100
