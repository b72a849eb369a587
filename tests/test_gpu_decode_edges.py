"""The operators over a paged cache at the ends of their ranges, against their definitions in 64 bits."""
import pytest
import torch

import decode as D                                        # (beside this file)
import paper_2505_12065_amd as ann
from test_gpu_decode import attend, close, dev            # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("window", [1, 1001, MOST - 1, MOST])
def test_attention_negative_lengths_with_any_window(dtype, page, window):
    """A negative length is none, whatever is taken off it."""
    def edit(q, k, v, table, lens):
        lens[1:5] = torch.tensor([LEAST, LEAST + 1000, -3, -1], dtype=torch.int32)
        return q, k, v, table, lens
    out = attend(dtype, [700, 10, 10, 10, 10, 0, 33], 4, 2, 64, page, window=window, mass=True, seed=31, edit=edit)
    assert (out[1:6] == 0).all()
