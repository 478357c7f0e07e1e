"""Questions behind one long instruction, on one paged cache: the operators for requests that share prefixes as a serving loop uses them.

The toy decoder of `windowed_beams.py`.  The instruction is computed once, in sequence 0; every question is admitted as a request that begins like it
(`pages_admit`: whole pages are shared, the rest is computed), the new tokens' places come from the lengths (`pages_slots`), and attention reads the
shared positions once for all (`prefix_groups`, `prefix_attention`).  When a question has its answer, the next one takes its place.

    python examples/shared_prompts.py [--instruction 1500] [--questions 12] [--places 5] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from windowed_beams import DH, HKV, HQ, LAYERS, PAGE, VOCAB, Model  # noqa: E402  (it finds the package)
from paper_2604_18396_b200 import pages_admit, pages_advance, pages_slots, prefix_attention, prefix_groups, rope_append  # noqa: E402


class Requests:
    """The cache of `seqs` sequences and the batch in hand: the rows of its new tokens, and which of its sequences share their first pages."""

    def __init__(self, seqs, pages, positions, device="cuda"):
        i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device=device)  # noqa: E731
        self.pool = torch.full((LAYERS, pages, 2, HKV, PAGE, DH), float("nan"), dtype=torch.bfloat16, device=device)
        self.state = [i32(seqs, -(-positions // PAGE), v=-1), i32(seqs), i32(pages)]
        self.other = [torch.empty_like(t) for t in self.state]
        self.n_new, self.q_start, self.lead, self.shared = i32(seqs), i32(seqs + 1), i32(seqs), i32(seqs)
        self.status, self.failed = i32(1), i32(1)

    table, lens, refs = (property(lambda self, k=k: self.state[k]) for k in range(3))

    def admit(self, like, begin, total):
        """Sequence i becomes a request of total[i] positions that begins with the first begin[i] of sequence like[i]."""
        pages_admit(*self.state, like, begin, total, *self.other, self.n_new, self.status, page_size=PAGE)
        torch.minimum(self.failed, self.status, out=self.failed)
        self.state, self.other = self.other, self.state

    def grow(self, n_new):
        self.n_new = n_new
        pages_advance(*self.state, n_new, *self.state, self.status, page_size=PAGE)
        torch.minimum(self.failed, self.status, out=self.failed)

    def rows(self, tokens):
        """Positions, sequences and slots of up to `tokens` new tokens (a fixed number of rows; those behind the last are padding)."""
        p, s = (torch.empty(tokens, dtype=torch.int32, device=self.pool.device) for _ in range(2))
        slots = torch.empty(tokens, dtype=torch.int64, device=self.pool.device)
        pages_slots(self.table, self.lens, self.n_new, self.q_start, p, s, slots, page_size=PAGE, status=self.failed)
        prefix_groups(self.table, self.lens, self.q_start, self.lead, self.shared, page_size=PAGE)
        return p, s, slots


def forward(model, r, tokens, positions, seqs, max_q, max_own):
    """Hidden rows of `tokens` (padding rows hold anything)."""
    x = model.embed[tokens]
    q_out = torch.empty(len(tokens), HQ, DH, dtype=torch.bfloat16, device=x.device)
    o = torch.zeros_like(q_out)
    for layer in range(LAYERS):
        q, k, v = (t.unflatten(-1, (-1, DH)) for t in (x @ model.qkv[layer]).split([HQ * DH, HKV * DH, HKV * DH], -1))
        rope_append(q, k, v, positions, seqs, model.inv_freq, r.pool, layer + 1, r.table, q_out, scale=model.scale, status=r.failed)
        prefix_attention(q_out, o, r.q_start, r.pool, layer + 1, r.table, r.lens, r.lead, r.shared, max_q=max_q, max_own=max_own, status=r.failed)
        x = x + o.flatten(1) @ model.out[layer]
    return x


def run(model, instruction, questions, *, places=5, steps=20, pages=None, device="cuda"):
    """-> (answers [questions][steps], the last hidden row of each, requests): greedy answers to each question behind the instruction."""
    n, longest = len(instruction), max(len(q) for q in questions)
    whole, tail = n // PAGE * PAGE, n % PAGE  # what is shared, and what each request computes again
    seqs, width = 1 + places, n + longest + steps
    r = Requests(seqs, pages or -(-n // PAGE) + places * (-(-(tail + longest + steps) // PAGE) + 1), width, device)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
    text = torch.zeros(seqs, width, dtype=torch.long, device=device)  # every sequence's tokens
    text[:, :n] = instruction
    # the instruction by itself
    r.admit(i32([-1] * seqs), i32([0] * seqs), i32([n] + [0] * places))
    p, s, _ = r.rows(n)
    forward(model, r, text[0, :n], p, s, n, n)
    answers, last, waiting, busy = [None] * len(questions), [None] * len(questions), list(range(len(questions))), [-1] * seqs
    left = [0] * seqs
    while waiting or any(b >= 0 for b in busy):
        # questions that are answered leave, the next ones take their places
        arrived = []
        for i in range(1, seqs):
            if busy[i] >= 0 and left[i] == 0:
                busy[i] = -1
            if busy[i] < 0 and waiting:
                busy[i], left[i] = waiting.pop(0), steps
                arrived.append(i)
                text[i, n:n + len(questions[busy[i]])] = questions[busy[i]]
                answers[busy[i]] = []
        going = [i for i in range(1, seqs) if busy[i] >= 0]
        if not going:
            break
        if arrived:
            # the new ones begin like the instruction, the others go on by a token, the empty ones hold nothing
            new = set(arrived)
            lens = [n if i == 0 else n + len(questions[busy[i]]) + (0 if i in new else len(answers[busy[i]])) if busy[i] >= 0 else 0 for i in range(seqs)]
            r.admit(i32([0 if i in new or i == 0 else i if busy[i] >= 0 else -1 for i in range(seqs)]), i32([n if i in new or i == 0 else lens[i] for i in range(seqs)]), i32(lens))
            tokens, max_q = len(arrived) * (tail + longest) + len(going), tail + longest
        else:
            r.grow(i32([1 if i in going else 0 for i in range(seqs)]))
            tokens, max_q = len(going), 1
        p, s, _ = r.rows(tokens)
        x = forward(model, r, text[s.clamp(min=0).long(), p.clamp(min=0).long()], p, s, max_q, tail + longest + steps)
        rows = x[(r.q_start[1:] - 1).clamp(min=0).long()]  # each sequence's last row
        said = (rows @ model.head).float().argmax(-1)
        for i in going:
            q = busy[i]
            text[i, n + len(questions[q]) + len(answers[q])] = said[i]
            answers[q].append(said[i])
            last[q] = rows[i]
            left[i] -= 1
    if r.failed.item():
        raise RuntimeError(f"a call on the cache failed: {r.failed.item()}")
    return torch.stack([torch.stack(a) for a in answers]), torch.stack(last), r


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("instruction", 1500), ("questions", 12), ("places", 5), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    draw = lambda n: torch.randint(0, VOCAB, (n,), generator=g).cuda()  # noqa: E731
    said, _, r = run(Model(), draw(a.instruction), [draw(5 + 7 * i % 40) for i in range(a.questions)], places=a.places, steps=a.steps)
    for i in range(min(4, a.questions)):
        print(f"question {i}: {said[i, :8].tolist()} ..")
    alone = a.questions * -(-(a.instruction + 45 + a.steps) // PAGE)
    print(f"{a.questions} questions behind {a.instruction} positions through {r.pool.shape[1]} pages of {PAGE}; by themselves they would hold {alone}")


if __name__ == "__main__":
    main()
