"""tg_prefix_attention with chunks of prompts behind a shared prefix: requests of many
rows, causal among themselves, against the float64 oracle (tolerances: those of
test_gpu_prefix_attention)."""
import pytest
import torch

from tests.test_gpu_prefix_attention import BF, F16, make, run
from tests.test_gpu_spec_decode import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,groups,Hq,Hkv,D,dtype,page", [
    ([(260, 300), (300, 64), (256, 129)], [(0, 3, 256)], 4, 2, 128, BF, 16),
    ([(400, 1000), (390, 1), (385, 0), (384, 77)], [(0, 4, 384)], 6, 2, 64, F16, 32),
    ([(300, 150), (290, 33), (700, 70)], [(0, 2, 288), (2, 1, 700)], 3, 1, 256, BF, 64),
    # Single rows beside a chunk: kernels for few rows, groups of many.
    ([(520, 1)] * 40 + [(515, 400)], [(0, 41, 512)], 8, 1, 128, F16, 16),
])
def test_chunks_against_float64(requests, groups, Hq, Hkv, D, dtype, page):
    say(f"prefix chunks {requests[:4]} {groups} Hq={Hq} Hkv={Hkv} D={D} page={page}")
    x = make(requests, groups, Hq, Hkv, D, dtype, page, len(requests) + D, mask=False)
    run(x, groups, Hq, D, max_nodes=max(n for _, n in requests))
    run(x, groups, Hq, D, layer=0)  # without max_nodes: the kernels for the mean rows
