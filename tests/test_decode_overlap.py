"""Outputs in the place of inputs that workgroups go on reading: refused through the C ABI, without a device."""
import pytest

from paper_2505_12065_amd import binding
from test_decode_abi import EVICT, P, RULES, call         # (beside this file)


@pytest.mark.parametrize("name,base,kw", [
    ("ann_cache_evict", EVICT, dict(lengths=2 * P, new_lengths=2 * P)), ("ann_cache_evict", EVICT, dict(mass=3 * P, new_mass=3 * P)),
    ("ann_logit_rules", RULES, dict(logits=4 * P, out=4 * P, row=100, out_row=104))])
def test_refused(name, base, kw):
    # (every pointer its own but for those in question)
    apart = {key: (7 + i) * P for i, (key, value) in enumerate(base.items()) if value == P}
    assert call(name, base, **dict(apart, **kw)) == binding.ANN_ERR_INVALID
    assert "may" in binding.ann_last_error()
