"""Samples several answers to one prompt with drafted tokens: the prompt's recurrent steps run through WiseAttention,
its last step's keys and values go into a paged cache, the samples are forks of it, and every round drafts, verifies
and drops.

    python examples/draft_decode.py --samples 8 --rounds 12 --draft 4

The model is a stand-in (random embeddings and projections, one attention layer, a draft that is the model with noise on
its logits): it shows the calls in their order of use, not language.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_27373_gb300 import serve, wise  # noqa: E402


class StandIn:
    """Embeddings, projections to Q, K and V, and logits from the attention's output."""

    def __init__(self, vocab, n_heads, n_kv_heads, head_dim, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=g, device="cuda") / shape[0] ** 0.5).bfloat16()

        self.n_heads, self.n_kv_heads, self.head_dim, width = n_heads, n_kv_heads, head_dim, n_heads * head_dim
        self.emb = torch.randn((vocab, width), generator=g, device="cuda").bfloat16()
        self.wq, self.wk = weight(width, width), weight(width, n_kv_heads * head_dim)
        self.wv, self.out = weight(width, n_kv_heads * head_dim), weight(width, vocab)

    def qkv(self, tokens):
        """Q, K, V as [batch, heads, tokens, head_dim] for tokens [batch, n]."""
        x = self.emb[tokens]
        return [(x @ w).unflatten(2, (-1, self.head_dim)).transpose(1, 2).contiguous()
                for w in (self.wq, self.wk, self.wv)]

    def probabilities(self, O, temperature=1.0, noise=None):
        logits = O.transpose(1, 2).flatten(2).float() @ self.out.float() / temperature
        return torch.softmax(logits if noise is None else logits + noise, -1)


def prefill(model, prompt, steps=4, discovery=2):
    """The prompt's recurrent steps (here: with drifting Q and K) through the dense, selecting and sparse calls;
    returns the last step's K and V."""
    Q, K, V = model.qkv(prompt[None])
    n = prompt.shape[0]
    shape = wise.Shape(1, n, model.n_heads, model.n_kv_heads, model.head_dim, 64)
    sel = wise.Select(1, 1, wise.WISE_SEL_TOPK, 2, 0.0, 4)
    layer, O = wise.WiseAttention(shape, sel, discovery), torch.empty_like(Q)
    for t in range(steps):
        if t > 0:
            Q, K = Q + 0.01 * torch.randn_like(Q), K + 0.01 * torch.randn_like(K)
        layer.step(t, Q, K, V, O)
    return K, V


def run(samples=8, rounds=12, draft=4, prompt_len=512, vocab=997, share=True, seed=0):
    """Returns each sample's tokens, and the cache."""
    torch.manual_seed(seed)
    model = StandIn(vocab, 8, 2, 64, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    prompt = torch.randint(0, vocab, (prompt_len,), generator=g, device="cuda")
    page = 32
    pages_each = -(-(draft + 1) * (rounds + 1) // page) + 1
    cache = serve.PagedCache(n_layers=1, n_pages=prompt_len // page + 2 + samples * pages_each, n_kv_heads=2, page=page,
                             head_dim=64, n_slots=samples + 1, max_pages=prompt_len // page + pages_each + 1)
    i32 = dict(dtype=torch.int32, device="cuda")

    # The prompt (all but its last token, which every sample feeds itself) into slot 0, then a fork per sample.
    K, V = prefill(model, prompt)
    first = torch.zeros(1, **i32)
    granted = cache.extend(first, torch.full((1,), prompt_len - 1, **i32))
    cache.write(0, first, granted, K[:, :, :-1].contiguous(), V[:, :, :-1].contiguous())
    slots = torch.arange(1, samples + 1, **i32)
    cache.fork(torch.zeros(samples, **i32), slots)
    groups = (torch.tensor([0, samples], **i32), torch.full((1,), prompt_len - 1, **i32)) if share else (None, None)

    answers = [[] for _ in range(samples)]
    last = prompt[-1].repeat(samples)
    feed = torch.full((samples,), draft + 1, **i32)
    for _ in range(rounds):
        # A draft for every sample (here: unrelated tokens with a flat distribution, often refused).
        drafted = torch.randint(0, vocab, (samples, draft), generator=g, device="cuda")
        q = torch.full((samples, draft, vocab), 1.0 / vocab, device="cuda")
        Q, K, V = model.qkv(torch.cat([last[:, None], drafted], 1))
        O = torch.empty_like(Q)
        granted = cache.extend(slots, feed)
        cache.write(0, slots, granted, K, V)
        cache.attend(0, Q, O, slots, granted, *groups)
        p = model.probabilities(O)
        u = torch.rand((samples, draft), generator=g, device="cuda")
        us = torch.rand((samples,), generator=g, device="cuda")
        accepted, tokens = serve.verify_draft(p, q, drafted.int(), None, u, us)
        # What stays of the granted tokens: the fed one and the accepted ones.  The next token is fed in the next round.
        cache.drop(slots, (granted - 1 - accepted).clamp(min=0))
        last = tokens.gather(1, accepted[:, None].long())[:, 0].long()
        for s, (n, row) in enumerate(zip(accepted.tolist(), tokens.tolist())):
            answers[s] += row[:n + 1]
    status = wise.wise_get_status()
    if status != wise.WISE_OK:
        raise RuntimeError(wise.status_string(status))
    # The first half of the samples ends; what is left moves to the front of the pool.
    ended = slots[: samples // 2]
    cache.drop(ended, torch.full_like(ended, 1 << 30))
    _, n_live = cache.compact()
    return answers, cache, int(n_live)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--rounds", type=int, default=12)
    ap.add_argument("--draft", type=int, default=4)
    args = ap.parse_args()
    answers, cache, n_live = run(args.samples, args.rounds, args.draft)
    for s, a in enumerate(answers):
        print(f"sample {s}: {len(a)} tokens: {' '.join(map(str, a[:16]))} ...")
    print(f"{n_live} of {cache.n_pages} pages in use after half of the samples ended")
