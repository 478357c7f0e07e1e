"""A long prompt in chunks, then beams, on one paged cache of fixed size: the operators for long contexts as a serving loop uses them.

A toy decoder of two attention blocks with random weights: every block's queries and keys are turned by positions scaled for long contexts
(`rope_append`), attention sees a window and a few first positions (`window_attention`), pages that slid out of the window are handed out
again (`pages_advance`), the beams share the prompt's pages and part from them page by page (`pages_reorder`), and at the end the pages in use
move together (`pages_compact`).  The cache holds a fraction of the positions that pass through it.

    python examples/windowed_beams.py [--tokens 2000] [--beams 4] [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_18396_b200 import pages_advance, pages_compact, pages_reorder, rope_append, rope_frequencies, window_attention  # noqa: E402

LAYERS, D, HQ, HKV, DH, VOCAB, PAGE = 2, 256, 8, 2, 64, 512, 16


class Model:
    def __init__(self, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g) / s[0] ** 0.5).to(torch.bfloat16).to(device)  # noqa: E731
        self.embed = w(VOCAB, D) * VOCAB ** 0.5
        self.qkv = [w(D, (HQ + 2 * HKV) * DH) for _ in range(LAYERS)]
        self.out = [w(HQ * DH, D) for _ in range(LAYERS)]
        self.head = w(D, VOCAB)
        # four times the positions that the frequencies were made for
        self.inv_freq, self.scale = rope_frequencies(DH, 10000.0, "ramp", factor=4.0, original_context=1024)
        self.inv_freq = self.inv_freq.to(device)


class Cache:
    """Pool, page table, lengths and reference counts of `seqs` sequences; `grow` and `become` keep the state before in a second set.

    What goes wrong on the device stays in `failed` until somebody looks: rotary positions and attention write it only when something is wrong,
    but the pages' calls answer every time, so they have a word of their own that is taken over behind each."""

    def __init__(self, seqs, pages, positions, device="cuda"):
        i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device=device)  # noqa: E731
        self.pool = torch.full((LAYERS, pages, 2, HKV, PAGE, DH), float("nan"), dtype=torch.bfloat16, device=device)
        self.state = [i32(seqs, -(-positions // PAGE), v=-1), i32(seqs), i32(pages)]
        self.other = [torch.empty_like(t) for t in self.state]
        self.status, self.failed = i32(1), i32(1)

    table, lens, refs = (property(lambda self, k=k: self.state[k]) for k in range(3))

    def grow(self, n_new, window, sinks):
        pages_advance(*self.state, n_new, *self.state, self.status, page_size=PAGE, window=window, sinks=sinks)
        torch.minimum(self.failed, self.status, out=self.failed)

    def become(self, parents):
        pages_reorder(self.pool, *self.state, parents, *self.other, self.status)
        torch.minimum(self.failed, self.status, out=self.failed)
        self.state, self.other = self.other, self.state


def forward(model, cache, tokens, positions, seqs, q_start, max_q, window, sinks):
    """Hidden rows of `tokens`, which stand at `positions` of `seqs` (their last ones); the cache has grown by them already."""
    x = model.embed[tokens]
    q_out = torch.empty(len(tokens), HQ, DH, dtype=torch.bfloat16, device=x.device)
    o = torch.empty_like(q_out)
    for layer in range(LAYERS):
        q, k, v = ((x @ model.qkv[layer]).split([HQ * DH, HKV * DH, HKV * DH], -1))
        q, k, v = (t.unflatten(-1, (-1, DH)) for t in (q, k, v))
        rope_append(q, k, v, positions, seqs, model.inv_freq, cache.pool, layer + 1, cache.table, q_out, scale=model.scale, status=cache.failed)
        window_attention(q_out, o, q_start, cache.pool, layer + 1, cache.table, cache.lens, window=window, sinks=sinks, max_q=max_q, status=cache.failed)
        x = x + o.flatten(1) @ model.out[layer]
    return x


def run(model, prompt, *, beams, steps, chunk=256, window=300, sinks=4, pages=None, device="cuda"):
    """-> (tokens of every beam [beams, steps], log-probabilities [beams], last hidden rows [beams, D], cache)."""
    n = len(prompt)
    # what a window, the sinks, a chunk in flight and the beams' own pages take - not what the context is long
    pages = pages or -(-(window + chunk) // PAGE) + 2 + -(-sinks // PAGE) + beams * (min(-(-(window + steps) // PAGE), -(-steps // PAGE) + 2) + 2)
    cache = Cache(beams, pages, n + steps, device)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
    only_first = lambda m: i32([m] + [0] * (beams - 1))  # noqa: E731
    for at in range(0, n, chunk):
        part = prompt[at:at + chunk]
        m = len(part)
        cache.grow(only_first(m), window, sinks)
        x = forward(model, cache, part, torch.arange(at, at + m, dtype=torch.int32, device=device), i32([0] * m), i32([0] + [m] * beams), m, window, sinks)
    logp = torch.log_softmax((x[-1:] @ model.head).float(), -1)
    score, token = logp[0].topk(beams)
    cache.become(i32([0] * beams))
    said = token[:, None]
    every, one = torch.arange(beams, dtype=torch.int32, device=device), i32([1] * beams)
    q_start = torch.arange(beams + 1, dtype=torch.int32, device=device)
    for _ in range(steps - 1):
        cache.grow(one, window, sinks)
        x = forward(model, cache, said[:, -1], cache.lens - 1, every, q_start, 1, window, sinks)
        logp = torch.log_softmax((x @ model.head).float(), -1) + score[:, None]
        score, flat = logp.flatten().topk(beams)
        parent = flat // VOCAB
        cache.become(parent.int())
        said, x = torch.cat((said[parent], (flat % VOCAB)[:, None]), 1), x[parent]
    if cache.failed.item():
        raise RuntimeError(f"a call on the cache failed: {cache.failed.item()}")
    return said, score, x, cache


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tokens", 2000), ("beams", 4), ("steps", 40), ("window", 300), ("sinks", 4), ("chunk", 256)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    model = Model()
    prompt = torch.randint(0, VOCAB, (a.tokens,), generator=torch.Generator().manual_seed(1)).cuda()
    said, score, _, cache = run(model, prompt, beams=a.beams, steps=a.steps, chunk=a.chunk, window=a.window, sinks=a.sinks)
    remap, n_used = torch.empty_like(cache.refs), torch.zeros(1, dtype=torch.int32, device="cuda")
    pages_compact(cache.pool, cache.table, cache.refs, cache.table, cache.refs, remap, n_used)
    for b in range(a.beams):
        print(f"beam {b}: log-probability {score[b].item():.3f}, {said[b, :8].tolist()} ..")
    print(f"{a.tokens} + {a.beams} x {a.steps} positions through {cache.pool.shape[1]} pages of {PAGE}; {n_used.item()} in use at the end, now the first ones")


if __name__ == "__main__":
    main()
