"""The example's decoder beyond the sizes of its first test: it has room for the
tokens that are asked for, and stops where it has none."""
import pytest
import torch

from tests.test_gpu_spec_example import ex  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def test_long_answers_have_their_pages(ex):  # noqa: F811
    print("[gpu] speculative decoding, 300 tokens of 3 requests", flush=True)
    prompts = [[1, 2, 3], [9] * 40, [5]]
    tokens, steps, worker = ex.speculative(ex.weights("cuda"), prompts, 300)
    assert [len(t) for t in tokens] == [300] * 3 and steps <= 300
    L = worker.lengths.tolist()
    for p, n in zip(prompts, L):  # the last step may pass the 300th token
        assert len(p) - 1 + 300 <= n < len(p) - 1 + 300 + len(ex.TREE)
    held = [-(-n // ex.PAGE) for n in L]
    assert worker.cache.held.tolist() == held and int(worker.cache.refcount.sum()) == sum(held)


def test_longer_answers_are_the_greedy_ones_up_to_ties(ex):  # noqa: F811
    print("[gpu] speculative decoding, 250 tokens of 4 requests", flush=True)
    tokens, one_by_one, steps = ex.main(250)  # raises where they part without a tie
    assert [len(t) for t in tokens] == [len(t) for t in one_by_one] == [250] * 4
    assert steps < 200


def test_prompts_in_chunks_of_any_size_give_the_same_cache(ex):  # noqa: F811
    print("[gpu] a prompt of 150 tokens in chunks of 1, 32 and 63 rows", flush=True)
    w, prompt = ex.weights("cuda"), [(7 * i * i) % ex.VOCAB for i in range(150)]
    logits = []
    for T in (1, 32, 100):
        worker = ex.Worker(w, 1, T)
        worker.prefill([prompt])
        assert worker.lengths.tolist() == [149]
        worker.rows([prompt[-1:]], [[1]], [[0]])
        logits.append(worker.forward()[0].clone())
    # bf16 activations through two layers, added in other orders: a few per cent
    # of the logits' spread.
    for x in logits[1:]:
        assert (x - logits[0]).abs().max() < 0.1 * logits[0].std()


def test_a_worker_without_pages_says_so(ex):  # noqa: F811
    print("[gpu] a worker that runs out of pages", flush=True)
    w = ex.weights("cuda")
    worker = ex.Worker(w, 1, 4, max_tokens=ex.PAGE)
    room = worker.cache.page_table.shape[1] * ex.PAGE
    worker.prefill([[1] * (room + 1)])  # the last token is not cached
    assert worker.lengths.tolist() == [room]
    worker.rows([[1]], [[1]], [[0]])
    with pytest.raises(RuntimeError, match="no pages"):
        worker.forward()
    with pytest.raises(ValueError, match="angles"):
        ex.Worker(w, 1, 1, max_tokens=1 << 20)
    torch.cuda.synchronize()
