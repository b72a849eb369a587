"""Outputs of the operators that take many tokens at once in the place of inputs that workgroups go on reading: refused through the C ABI, without a device."""
import pytest

from paper_2505_12065_amd import binding
from test_decode_abi import P, call                       # (beside this file)
from test_many_abi import APPEND, CHUNK, SHARED

ROW = 64 * 2                                              # bytes


@pytest.mark.parametrize("name,base,kw", [
    ("ann_rotate_append", APPEND, dict(qkv=99 * P, q=99 * P)), ("ann_rotate_append", APPEND, dict(qkv=99 * P, q=99 * P + (2 * 8 + 7) * ROW)),
    ("ann_rotate_append", APPEND, dict(qkv=99 * P, q=99 * P - (3 * 4 - 1) * ROW)), ("ann_rotate_append", APPEND, dict(qkv=99 * P, q=99 * P, T=1, head=72)),
    *[(name, base, dict(q=99 * P, out=99 * P, **kw)) for name, base in (("ann_chunk_attention", CHUNK), ("ann_shared_attention", SHARED)) for kw in (dict(row=512), dict(head=72), dict(row=0))],
    *[(name, base, dict(q=99 * P, out=99 * P + by * ROW)) for name, base in (("ann_chunk_attention", CHUNK), ("ann_shared_attention", SHARED)) for by in (1, 11, -1, -11)]])
def test_refused(name, base, kw):
    # (every pointer its own but for those in question)
    apart = {key: (7 + i) * P for i, (key, value) in enumerate(base.items()) if value == P}
    assert call(name, base, **dict(apart, **kw)) == binding.ANN_ERR_INVALID
    assert "in the place of" in binding.ann_last_error()
