"""Arguments that the Python half of the binding checks before a device is touched."""
import pytest
import torch

import paper_2505_12065_amd as ann


@pytest.mark.parametrize("args", [(1, 8, 2, 64, torch.float16, 2 ** 32 + 100), (2 ** 32 + 1, 8, 2, 64, torch.float16, 100), (1, 2 ** 32 + 8, 2, 64, torch.float16, 100),
                                  (1, 8, 2, 64, torch.float16, -2 ** 32 + 100)])
def test_workspace_bytes_of_sizes_beyond_32_bits(args):
    with pytest.raises(ValueError):
        ann.ann_paged_attention_workspace_bytes(*args)
