"""The sequence path at the ends of what its calls allow: the most heads of keys over long histories, scratch asked for once and used for
smaller batches, scores without a finite one among them, kernels that run for seconds.  Inputs, oracle and error bounds are those of
test_gpu_sequence.py."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from paper_2510_18239_b200 import binding
from test_gpu_sequence import check_history, check_tree, lime

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,dh,keys", [("f32", 640, 72, 100), ("f32", 1024, 128, 300), ("bf16", 593, 72, 950), ("bf16", 1024, 128, 1000)])
def test_the_most_heads_over_histories_of_many_tiles(dtype, heads, dh, keys):
    """So many heads of keys occupy the card by themselves: no row tile is cut, however long, and there is nothing to join."""
    gen = torch.Generator().manual_seed(heads)
    m = lime(dtype, heads, heads, dh)
    check_history(m, gen, dtype, heads, heads, dh, [2], [keys], 1 / np.sqrt(dh))
    check_tree(m, gen, dtype, heads, heads, dh, [3], [keys], 64, "drafts")
    check_tree(m, gen, dtype, heads, heads, dh, [1], [keys], 64, "none")
