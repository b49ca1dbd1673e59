"""The final state in the place of the first, over clusters of every size and chains that several clusters share."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests.test_gpu_recurrence import tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,n,c,dtype", [(460, 140, 64, torch.bfloat16), (230, 300, 40, torch.float16), (60, 700, 96, torch.float32),
                                         (2, 1100, 33, torch.bfloat16), (3, 129, 64, torch.float32), (1, 8193, 64, torch.bfloat16), (300, 40, 66, torch.bfloat16)])
def test_the_final_state_in_the_place_of_the_first(b, n, c, dtype):
    gate, x, _, h0, _, lens = tensors(b, n, c, dtype, n)
    out, final, states = B.gs_recurrence_forward(gate, x, h0, lens)
    for _ in range(10):
        state = h0.clone()
        again, same, kept = B.gs_recurrence_forward(gate, x, state, lens, final=state)
        assert same is state and torch.equal(state, final) and torch.equal(again, out) and torch.equal(kept, states)
