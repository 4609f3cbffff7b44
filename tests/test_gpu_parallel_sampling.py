"""examples/parallel_sampling.py: the operators of a decode step behind a common
prompt, run together as they are used. Every step is held against the operators
that know of no sharing and no few tokens (TreeAttention, EwForward) on the same
tokens, and its draw against the definition on the step's own logits."""
import importlib.util
import os

import pytest
import torch

from tests.test_gpu_sample import row_of

pytestmark = pytest.mark.gpu
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


def load(name):
    s = importlib.util.spec_from_file_location(name, os.path.join(EXAMPLES, name + ".py"))
    m = importlib.util.module_from_spec(s)
    s.loader.exec_module(m)
    return m


# held: tokens that a sample has room for; from (n - 1) * held = 32768 on the shared
# pages are read once (heads 2 of 64).
@pytest.mark.parametrize("n,length,most,held", [(2, 150, 3, 3), (8, 260, 20, 20), (32, 17, 4, 4),
                                                (32, 260, 4, 1024), (24, 300, 12, 1600)])
def test_steps_against_the_other_operators(n, length, most, held):
    ex = load("parallel_sampling")
    base = ex.base
    w = base.weights("cuda")
    g = torch.Generator().manual_seed(n)
    prompt = torch.randint(0, base.VOCAB, (length,), generator=g).tolist()
    s = ex.Sampler(w, prompt, n, held)
    # The same samples as requests of their own, each with its copy of the prompt.
    plain = base.Worker(w, n, 8 * n, base.room([prompt], most, 1))
    plain.prefill([prompt] * n)
    last = [prompt[-1]] * n
    for step in range(most):
        u = torch.rand(n, generator=g).cuda()
        tokens = s.step(u).tolist()
        plain.rows([[t] for t in last], [[1]] * n, [[0]] * n)
        want = plain.forward()[:n]
        plain.lengths += 1
        # Activations of 16 bits that are rounded in other places: as far apart as
        # two orders of the example's own steps may lie.
        assert float((s.logits - want).abs().max()) <= base.TIE, step
        for t in range(n):
            wt, sure, maybe, slack = row_of(s.logits[t], 0.8, 50,
                                            float(torch.tensor(0.95)), float(torch.tensor(0.01)))
            i, kept = tokens[t], maybe
            assert kept[i], (step, t)
            mass = float(wt[kept].sum())
            upto = float(torch.cumsum(wt * kept, 0)[i])
            # (0.8 as a float32 is 2^-26 off: t / 0.8 up to 64 moves a weight by 2^-20)
            room = slack + 2.0 ** -18 * mass
            assert upto - float(wt[i]) <= float(u[t]) * mass + room and upto > float(u[t]) * mass - room
        last = tokens
    assert s.status.all()
    # What the samples hold of the prompt is held once.
    table = s.cache.page_table.cpu()
    whole = (length - 1) // base.PAGE
    assert (table[:, :whole] == table[0, :whole]).all()


def test_it_runs():
    ex = load("parallel_sampling")
    rows, prompt, s = ex.main(4, 5)
    assert len(rows) == 4 and all(len(r) == 5 for r in rows)
    assert all(0 <= t < ex.base.VOCAB for r in rows for t in r)
    assert s.lengths.tolist() == [len(prompt) - 1 + 5] * 4
