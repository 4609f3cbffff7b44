"""The operators together: greedy decoding of drafted trees in the example's
decoder gives the tokens of greedy decoding one by one, in fewer forwards, and
the kept rows' KV segments reach the checkpoint store."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    path = os.path.join(ROOT, "examples", "spec_decode.py")
    s = importlib.util.spec_from_file_location("spec_decode_example", path)
    m = importlib.util.module_from_spec(s)
    s.loader.exec_module(m)
    return m


def test_drafted_trees_give_the_greedy_tokens(ex):
    print("[gpu] speculative decoding, 40 tokens of 4 requests", flush=True)
    tokens, one_by_one, steps = ex.main(40)
    assert tokens == one_by_one
    assert steps < 30  # some drafts are kept, or there is nothing to test


def test_pages_and_checkpoint_after_decoding(ex):
    print("[gpu] speculative decoding with checkpoints", flush=True)
    w = ex.weights("cuda")
    prompts = [[1, 2, 3], [9] * 20]
    store = ex.host_store(ex.LAYERS * 2 * 17 * ex.PAGE * ex.HKV * ex.D * 2)
    tokens, _, worker = ex.speculative(w, prompts, 25, store)
    torch.cuda.synchronize()
    c = worker.cache
    assert c.k.numel() * 2 == store["k"].numel()
    L = worker.lengths.tolist()
    assert [len(t) for t in tokens] == [25, 25]
    held = [-(-n // ex.PAGE) for n in L]
    assert c.held.tolist() == held and int(c.refcount.sum()) == sum(held)
    saved = store["k"].view(torch.bfloat16).view(c.k.shape)
    table = c.page_table.tolist()
    for b, p in enumerate(prompts):
        for pos in range(len(p) - 1, L[b]):  # every row since the prompt
            page, row = table[b][pos // ex.PAGE], pos % ex.PAGE
            assert torch.equal(saved[:, page, row], c.k[:, page, row].cpu()), (b, pos)
    assert int(store["commit"][0]) == 1 + ex.LAYERS * sum(L[b] - len(p) + 1
                                                          for b, p in enumerate(prompts))
    # A fork goes on with the same context.
    src, dst = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (0, 1))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.trim(torch.tensor([L[0], 0], dtype=torch.int32, device="cuda"))
    worker.lengths[1] = 0
    c.fork(worker.lengths, src, dst, status)
    assert status.tolist() == [1] and worker.lengths.tolist() == [L[0], L[0]]
