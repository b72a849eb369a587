"""Argument errors of the operators over a paged cache, through the C ABI without a device."""
import ctypes

import pytest

from paper_2505_12065_amd import binding

P = 0x10000                                               # aligned, never dereferenced by the checks under test
E, A = binding.ANN_ERR_INVALID, binding.ANN_ERR_ALIGNMENT


def cache(**kw):
    c = binding.PagedCache(P, P, 2048, 1024, 64, 2048, 1024, 64, 10, 2, 16, 64, 1)
    for name, value in kw.items():
        setattr(c, name, value)
    return ctypes.byref(c)


ROTATE = dict(qkv=P, token=512, head=64, T=3, q_heads=4, qw=P, kw=P, eps=1e-6, positions=P, cos_sin=P, most=100, rot=64, pairs=0, slots=P,
              cache=None, q=P, stream=None)
ATTEND = dict(q=P, row=256, head=64, B=3, q_heads=4, cache=None, table=P, width=5, lengths=P, most=80, scale=0.1, window=0, out=P, lse=P,
              mass=None, mass_slots=0, stream=None)
EVICT = dict(cache=None, table=P, width=5, lengths=P, B=3, mass=P, mass_slots=80, new_table=P, new_width=2, budget=20, first=2, recent=3,
             kept=P, new_lengths=P, new_mass=P, new_slots=32, stream=None)
RULES = dict(logits=P, row=100, B=3, V=100, dtype=0, tokens=P, T=5, lengths=P, prompts=P, r=P, p=P, f=P, bt=P, bv=P, K=2, masks=P, n_masks=2,
             rows=P, out=P, out_row=100, stream=None)
BAD_CACHE = [(dict(k=None), E), (dict(v=None), E), (dict(pages=0), E), (dict(heads=0), E), (dict(slots=24), E), (dict(slots=0), E), (dict(slots=2048), E),
             (dict(d=0), E), (dict(d=264), E), (dict(d=60), A), (dict(dtype=5), E), (dict(k=P + 8), A), (dict(v=P + 2), A), (dict(k_slot=60), A),
             (dict(v_page=-64), E), (dict(k_page=2 ** 62), E)]


def call(name, base, **kw):
    args = dict(base, **kw)
    if "cache" in args and args["cache"] is None:
        args["cache"] = cache()
    return getattr(binding.lib(), name)(*args.values())


@pytest.mark.parametrize("fields,code", BAD_CACHE)
def test_a_cache_that_is_none(fields, code):
    for name, base in (("ann_qk_norm_rotate", ROTATE), ("ann_paged_attention", ATTEND), ("ann_cache_evict", EVICT)):
        assert call(name, base, cache=cache(**fields)) == code, (name, fields)
        assert binding.ann_last_error()


@pytest.mark.parametrize("name,base,kw,code", [
    *[("ann_qk_norm_rotate", ROTATE, kw, code) for kw, code in (
        (dict(qkv=None), E), (dict(qw=None), E), (dict(kw=None), E), (dict(positions=None), E), (dict(cos_sin=None), E), (dict(slots=None), E),
        (dict(q=None), E), (dict(T=-1), E), (dict(q_heads=0), E), (dict(rot=24), E), (dict(rot=80), E), (dict(rot=-16), E), (dict(most=-1), E),
        (dict(eps=float("nan")), E), (dict(token=-512), E), (dict(token=2 ** 60), E), (dict(head=60), A), (dict(qkv=P + 4), A), (dict(q=P + 8), A),
        (dict(qw=P + 2), A), (dict(slots=P + 2), A), (dict(T=2 ** 23), E))],
    *[("ann_paged_attention", ATTEND, kw, code) for kw, code in (
        (dict(q=None), E), (dict(table=None), E), (dict(lengths=None), E), (dict(out=None), E), (dict(B=-1), E), (dict(q_heads=3), E), (dict(q_heads=0), E),
        (dict(width=0), E), (dict(width=2 ** 28), E), (dict(most=0), E), (dict(most=81), E), (dict(scale=float("inf")), E), (dict(window=-1), E),
        (dict(mass=P, mass_slots=79), E), (dict(row=260), A), (dict(q=P + 8), A), (dict(out=P + 2), A), (dict(lse=P + 2), A), (dict(B=2 ** 21), E))],
    *[("ann_cache_evict", EVICT, kw, code) for kw, code in (
        (dict(table=None), E), (dict(lengths=None), E), (dict(mass=None), E), (dict(new_table=None), E), (dict(kept=None), E), (dict(new_mass=None), E),
        (dict(new_lengths=None), E), (dict(B=-1), E), (dict(width=0), E), (dict(new_width=0), E), (dict(mass_slots=0), E), (dict(budget=0), E),
        (dict(budget=33, new_slots=99), E), (dict(new_slots=19), E), (dict(first=-1), E), (dict(recent=-1), E), (dict(first=18), E),
        (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), E), (dict(mass=P + 2), A), (dict(kept=P + 1), A))],
    *[("ann_logit_rules", RULES, kw, code) for kw, code in (
        (dict(logits=None), E), (dict(tokens=None), E), (dict(lengths=None), E), (dict(prompts=None), E), (dict(r=None), E), (dict(p=None), E),
        (dict(f=None), E), (dict(bt=None), E), (dict(bv=None), E), (dict(masks=None), E), (dict(rows=None), E), (dict(out=None), E), (dict(dtype=3), E),
        (dict(B=-1), E), (dict(V=0), E), (dict(T=-1), E), (dict(T=2 ** 24), E), (dict(K=4097), E), (dict(K=-1), E), (dict(n_masks=-1), E), (dict(row=99), E),
        (dict(out_row=99), E), (dict(logits=P + 1), A), (dict(out=P + 2, dtype=2), A), (dict(masks=P + 2), A), (dict(B=2 ** 22, V=5000, row=5000, out_row=5000), E))],
])
def test_refused(name, base, kw, code):
    assert call(name, base, **kw) == code, binding.ann_last_error()
    assert binding.ann_last_error()


def test_nothing_to_do_is_no_error():
    assert call("ann_qk_norm_rotate", ROTATE, T=0) == 0
    for name, base in (("ann_paged_attention", ATTEND), ("ann_cache_evict", EVICT), ("ann_logit_rules", RULES)):
        assert call(name, base, B=0) == 0


def test_workspace_bytes():
    f = binding.lib().ann_paged_attention_workspace_bytes
    for bad in ((0, 8, 2, 64, 0, 100, 0), (1, 7, 2, 64, 0, 100, 0), (1, 8, 0, 64, 0, 100, 0), (1, 8, 2, 300, 0, 100, 0), (1, 8, 2, 64, 9, 100, 0), (1, 8, 2, 64, 0, 0, 0)):
        assert f(*bad) == E
    assert 0 < f(1, 8, 2, 64, 0, 100_000, 0) <= f(2, 8, 2, 64, 0, 100_000, 0) <= f(2, 8, 2, 64, 0, 100_000, 1)


def test_constants_and_structure():
    import os
    import re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ann.h")).read()
    for name in ("ANN_PAGE_MAX", "ANN_HEAD_MAX", "ANN_HISTORY_MAX", "ANN_BIAS_MAX"):
        assert int(re.search(r"#define\s+%s\s+(\d+)" % name, header).group(1)) == getattr(binding, name)
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct ann_paged_cache \{(.*?)\}", header, re.S).group(1), flags=re.S)
    fields = [(kind, n.strip(" *")) for kind, names in re.findall(r"(void|int64_t|int32_t)\s+([^;]+);", body) for n in names.split(",")]
    kinds = {"void": ctypes.c_void_p, "int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32}
    assert [(n, kinds[k]) for k, n in fields] == binding.PagedCache._fields_
