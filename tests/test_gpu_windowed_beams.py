"""The example of windowed beams against a dense statement of the same decoder (needs a B200)."""
import importlib.util
import os

import pytest
import torch

from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("windowed_beams", os.path.join(ROOT, "examples", "windowed_beams.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(ex, model, tokens, window, sinks):
    """Last hidden row of `tokens`, every position computed, in 64 bits but for the roundings to bf16 that the decoder has."""
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    n = len(tokens)
    x = model.embed[tokens].double()
    pos = torch.arange(n, device=tokens.device)
    seen = ref.visible(n, n, window, sinks, tokens.device)
    for layer in range(ex.LAYERS):
        q, k, v = (t.unflatten(-1, (-1, ex.DH)) for t in bf(x @ model.qkv[layer].double()).split([ex.HQ * ex.DH, ex.HKV * ex.DH, ex.HKV * ex.DH], -1))
        q, k = (bf(ref.rope(t, pos, model.inv_freq, False, model.scale)) for t in (q, k))
        o = torch.empty_like(q)
        for h in range(ex.HQ):
            s = (q[:, h] @ k[:, h * ex.HKV // ex.HQ].T / ex.DH ** 0.5).masked_fill(~seen, -float("inf"))
            o[:, h] = torch.softmax(s, -1) @ v[:, h * ex.HKV // ex.HQ]
        x = bf(x + bf(bf(o).flatten(1) @ model.out[layer].double()))
    return x[-1]


@pytest.mark.parametrize("tokens,beams,steps,window,sinks,chunk", [(700, 4, 20, 100, 4, 128), (150, 3, 40, 33, 17, 64), (90, 2, 5, 1000, 0, 90)])
def test_beams_are_those_of_a_dense_decoder(ex, tokens, beams, steps, window, sinks, chunk):
    model = ex.Model(seed=tokens)
    prompt = torch.randint(0, ex.VOCAB, (tokens,), generator=torch.Generator().manual_seed(2)).cuda()
    kw = {} if window < tokens else {"pages": beams * (-(-(tokens + steps) // ex.PAGE)) + 4}
    said, score, x, cache = ex.run(model, prompt, beams=beams, steps=steps, chunk=chunk, window=window, sinks=sinks, **kw)
    assert len({tuple(t) for t in said.tolist()}) == beams
    for b in range(beams):
        # the rows that chose the last token: a handful of bf16 roundings apart (2^-9 of values of a few units, some ten of them)
        want = dense(ex, model, torch.cat((prompt, said[b, :-1])), window, sinks)
        err = (x[b].double() - want).abs().max().item()
        assert err <= 2.0 ** -9 * 10 * want.abs().max().item(), err
    # every page is held by as many table entries as its count says
    count = torch.bincount(cache.table[cache.table >= 0].long().flatten(), minlength=cache.refs.numel())
    assert torch.equal(count.int(), cache.refs)


def test_the_command_runs(ex, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["windowed_beams.py", "--tokens", "300", "--steps", "6", "--window", "64"])
    ex.main()
    assert "positions through" in capsys.readouterr().out
