"""The example of questions behind one instruction against a dense statement of the same decoder (needs a B200)."""
import importlib.util
import os

import pytest
import torch

from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("shared_prompts", os.path.join(ROOT, "examples", "shared_prompts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(ex, model, tokens):
    """Last hidden row of `tokens`, every position computed, in 64 bits but for the roundings to bf16 that the decoder has."""
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    n = len(tokens)
    x = model.embed[tokens].double()
    pos = torch.arange(n, device=tokens.device)
    seen = pos[:, None] >= pos
    for layer in range(ex.LAYERS):
        q, k, v = (t.unflatten(-1, (-1, ex.DH)) for t in bf(x @ model.qkv[layer].double()).split([ex.HQ * ex.DH, ex.HKV * ex.DH, ex.HKV * ex.DH], -1))
        q, k = (bf(ref.rope(t, pos, model.inv_freq, False, model.scale)) for t in (q, k))
        o = torch.empty_like(q)
        for h in range(ex.HQ):
            s = (q[:, h] @ k[:, h * ex.HKV // ex.HQ].T / ex.DH ** 0.5).masked_fill(~seen, -float("inf"))
            o[:, h] = torch.softmax(s, -1) @ v[:, h * ex.HKV // ex.HQ]
        x = bf(x + bf(bf(o).flatten(1) @ model.out[layer].double()))
    return x[-1]


@pytest.mark.parametrize("n,questions,places,steps", [(1500, 7, 3, 9), (320, 5, 5, 4), (37, 4, 2, 20), (5, 3, 3, 3)])
def test_answers_are_those_of_a_dense_decoder(ex, n, questions, places, steps):
    model = ex.Model(seed=n)
    g = torch.Generator().manual_seed(2)
    draw = lambda k: torch.randint(0, ex.VOCAB, (k,), generator=g).cuda()  # noqa: E731
    instruction, asked = draw(n), [draw(1 + 11 * i % 29) for i in range(questions)]
    said, x, r = ex.run(model, instruction, asked, places=places, steps=steps)
    assert said.shape == (questions, steps)
    for i in range(questions):
        # the rows that chose the last token: a handful of bf16 roundings apart (2^-9 of values of a few units, some ten of them)
        want = dense(ex, model, torch.cat((instruction, asked[i], said[i, :-1])))
        err = (x[i].double() - want).abs().max().item()
        assert err <= 2.0 ** -9 * 10 * want.abs().max().item(), (i, err)
    # every page is held by as many table entries as its count says, and the instruction's whole pages by all who are behind it
    count = torch.bincount(r.table[r.table >= 0].long().flatten(), minlength=r.refs.numel())
    assert torch.equal(count.int(), r.refs)
    assert (r.refs > 1).sum().item() == n // ex.PAGE


def test_the_command_runs(ex, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["shared_prompts.py", "--instruction", "200", "--questions", "3", "--steps", "4"])
    ex.main()
    assert "by themselves" in capsys.readouterr().out
