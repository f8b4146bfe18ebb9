"""The verification operators' host side: what the library and the binding refuse before anything is launched (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2605_02218_b200 import api

FAR = 1 << 20          # an address that no call reaches


def _cache(**kw):
    c = dict(store=api.COVSPEC_BF16, pages=4, heads=2, page_size=16, head_dim=128, k=FAR, v=FAR, k_scale=None, v_scale=None,
             k_page_stride=2 * 16 * 128, v_page_stride=2 * 16 * 128)
    return api.Cache(*{**c, **kw}.values())


def _tokens(**kw):
    t = dict(batch=2, offsets=FAR, lengths=FAR, table=FAR, table_width=3, table_stride=3)
    return api.Tokens(*{**t, **kw}.values())


BAD_CACHES = [
    (dict(k=None), -1), (dict(v=None), -1), (dict(store=5), -1), (dict(store=-1), -1), (dict(store=api.COVSPEC_E4M3), -1),
    (dict(store=api.COVSPEC_INT8, k_scale=FAR), -1), (dict(head_dim=96), -3), (dict(head_dim=0), -3), (dict(page_size=24), -3),
    (dict(page_size=0), -3), (dict(page_size=4), -3), (dict(page_size=8192), -3), (dict(pages=0), -2), (dict(heads=0), -2),
    (dict(k_page_stride=2 * 16 * 128 - 8), -2), (dict(v_page_stride=0), -2), (dict(k_page_stride=2 * 16 * 128 + 4), -1),
    (dict(k=FAR + 8), -1), (dict(heads=2 ** 20, page_size=4096), -2),
]
BAD_TOKENS = [(dict(offsets=None), -1), (dict(lengths=None), -1), (dict(table=None), -1), (dict(batch=0), -2),
              (dict(table_width=0), -2), (dict(table_stride=2), -2)]


def _write(cache, tokens, **kw):
    a = dict(dtype=api.COVSPEC_BF16, n=5, k=FAR, v=FAR, ks=256, vs=256, rows=None, row_offsets=None, source=5)
    return api.load_library().covspec_cache_write(cache and C.byref(cache), tokens and C.byref(tokens), *{**a, **kw}.values(), None)


def _read(cache, tokens, **kw):
    a = dict(dtype=api.COVSPEC_BF16, n=5, k=FAR, v=FAR)
    return api.load_library().covspec_cache_read(cache and C.byref(cache), tokens and C.byref(tokens), *{**a, **kw}.values(), None)


def _attend(cache, tokens, **kw):
    a = dict(dtype=api.COVSPEC_BF16, n=5, q=FAR, q_stride=512, q_heads=4, scale=0.1, window=0, max_new=0, out=FAR, out_stride=512,
             lse=None, work=FAR, size=1 << 40)
    return api.load_library().covspec_cache_attend(cache and C.byref(cache), tokens and C.byref(tokens), *{**a, **kw}.values(), None)


@pytest.mark.parametrize("call", [_write, _read, _attend])
def test_bad_caches_and_tokens_are_refused(call):
    for kw, status in BAD_CACHES:
        assert call(_cache(**kw), _tokens()) == status, kw
    for kw, status in BAD_TOKENS:
        assert call(_cache(), _tokens(**kw)) == status, kw
    assert call(None, _tokens()) == -1 and call(_cache(), None) == -1
    assert call(_cache(), _tokens(), n=-1) == -2
    assert call(_cache(), _tokens(), n=0) == 0                  # nothing to do, nothing launched


def test_bad_arguments_of_the_cache_calls_are_refused():
    for kw, status in [(dict(dtype=3), -1), (dict(k=None), -1), (dict(v=FAR + 4), -1), (dict(ks=255), -2), (dict(vs=128), -2),
                       (dict(ks=260), -1), (dict(rows=FAR), -1), (dict(source=4), -2), (dict(source=-1), -2)]:
        assert _write(_cache(), _tokens(), **kw) == status, kw
    for kw, status in [(dict(dtype=4), -1), (dict(k=None), -1), (dict(v=FAR + 8), -1)]:
        assert _read(_cache(), _tokens(), **kw) == status, kw
    for kw, status in [(dict(dtype=api.COVSPEC_F32), -3), (dict(dtype=api.COVSPEC_F16), -3), (dict(q=None), -1), (dict(out=None), -1),
                       (dict(q=FAR + 2), -1), (dict(q_heads=3), -2), (dict(q_heads=0), -2), (dict(q_stride=511), -2),
                       (dict(out_stride=516), -1), (dict(window=-1), -1), (dict(max_new=-1), -1), (dict(scale=float("nan")), -1),
                       (dict(work=None), -1), (dict(n=2 ** 30), -2)]:
        assert _attend(_cache(), _tokens(), **kw) == status, kw
    assert _attend(_cache(store=api.COVSPEC_F32), _tokens()) == -3
    lib = api.load_library()
    assert lib.covspec_cache_attend_workspace(None, 4) == -1
    assert lib.covspec_cache_attend_workspace(C.byref(_cache()), 3) == -2


def test_bad_arguments_of_the_logit_edits_are_refused():
    lib = api.load_library()

    def edit(e=None, **kw):
        given = dict(batch=1, row_offsets=FAR)
        given.update(e or {})
        a = {**dict(dtype=api.COVSPEC_F16, rows=3, vocab=100, ld=104, z=FAR, out=FAR), **kw}
        return lib.covspec_edit_logits(*a.values(), C.byref(api.Edits(**given)), None)
    for e, kw, status in [
            ({}, dict(z=None), -1), ({}, dict(out=None), -1), ({}, dict(dtype=3), -1), ({}, dict(rows=-1), -2), ({}, dict(vocab=0), -2),
            ({}, dict(ld=96), -2), ({}, dict(ld=101), -2), ({}, dict(z=FAR + 2), -1), (dict(row_offsets=None), {}, -1),
            (dict(batch=0), {}, -2), (dict(history=FAR), {}, -1), (dict(bias_ids=FAR), {}, -1),
            (dict(bias_ids=FAR, bias_values=FAR), {}, -1), (dict(history_len=-1), {}, -2), (dict(bias_len=-1), {}, -2),
            (dict(mask=FAR, mask_stride=12), {}, -2)]:
        assert edit(e, **kw) == status, (e, kw)
    assert lib.covspec_edit_logits(api.COVSPEC_F16, 3, 100, 104, FAR, FAR, None, None) == -1
    assert edit(rows=0) == 0


def test_the_binding_wants_tensors_on_a_device():
    z = torch.zeros(2, 64, dtype=torch.float16)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        api.edit_logits(z, off)
    with pytest.raises(TypeError):
        api.edit_logits(z.double(), off)
    k = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.PagedCache(k, k)
    with pytest.raises(TypeError):
        api.PagedCache(k, k.half())
    with pytest.raises(TypeError):
        api.PagedCache(k.double(), k.double())
