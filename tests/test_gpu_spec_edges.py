"""The paged-cache operators where they were once wrong, against the float64
oracle (tolerances as derived in ``test_gpu_spec_decode``, or where they are
used)."""
import math

import numpy as np
import pytest
import torch

from paper_2601_01310_amd import spec
from tests.test_gpu_spec_decode import (DEV, check_attention, f64, ints, make_pool, random_masks,
                                        say)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,Hq,Hkv,D,dtype,page", [
    (33, 4, 1, 128, torch.bfloat16, 16), (64, 2, 1, 64, torch.float16, 4),
    (64, 2, 2, 256, torch.bfloat16, 32), (40, 8, 2, 128, torch.float16, 64)])
def test_trees_that_fill_their_mask_words(n, Hq, Hkv, D, dtype, page):
    """Contexts after which a tile's second half lies past the mask's last
    word, the last request's row among them."""
    say(f"attention, {n} nodes in one word, Hq={Hq} D={D}")
    rng = np.random.default_rng(n + D)
    L = [64, 31, 28, 32]
    cache, table = make_pool([x + n for x in L], page, Hkv, D, dtype, rng)
    off = [n * b for b in range(len(L) + 1)]
    q = torch.randn((n * len(L), Hq, D), device=DEV).to(dtype)
    mask = random_masks([n] * len(L), rng)
    out = spec.TreeAttention(cache, q, ints(off), ints(L), mask, max_nodes=n)()
    check_attention(out, f64(q), cache, table, 0, off, L, mask, 1 / math.sqrt(D), dtype)
