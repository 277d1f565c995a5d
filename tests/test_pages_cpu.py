"""What the operators on ragged batches and 8-bit pages refuse, on the host and before anything is enqueued (no device needed), and the plain
form of the pages that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
from tests import pages_reference as ref

OK = 4096                                       # an aligned address that is never dereferenced
FAR = [OK + (i << 40) for i in range(12)]       # such addresses, far apart
BAD, SPACE = kf.KF_EINVAL, kf.KF_ENOSPC


def _filled(struct, base, kw):
    a = struct()
    for name, value in {**base, **kw}.items():
        setattr(a, name, value)
    return a


def _ragged(**kw):
    return _filled(kf.kf_ragged_args, dict(tokens=10, sequences=2, n_heads=4, n_kv_heads=2, head_dim=64, type=0, bias_mode=0, logit_scale=0.0, d_alibi_slopes=None,
                                           q_token_stride=256, q_head_stride=64, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64,
                                           out_token_stride=256, out_head_stride=64), kw)


def _call_ragged(a, p=None):
    return kf.LIB.kf_prefill_attend_ragged(C.byref(a) if a is not None else None, *(p or FAR[:5]), None)


@pytest.mark.parametrize("bad", [dict(tokens=0), dict(tokens=(1 << 28) + 1), dict(sequences=0), dict(sequences=(1 << 20) + 1), dict(n_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=3),
                                 dict(n_heads=65536 * 2), dict(head_dim=96), dict(type=2), dict(type=-1), dict(bias_mode=1), dict(bias_mode=2), dict(bias_mode=1, d_alibi_slopes=OK + 2),
                                 dict(logit_scale=-1.0), dict(logit_scale=float("nan")), dict(logit_scale=float("inf")), dict(q_token_stride=0), dict(q_head_stride=0), dict(k_token_stride=132),
                                 dict(k_head_stride=32), dict(v_token_stride=-128), dict(v_head_stride=1 << 38), dict(out_token_stride=128), dict(out_head_stride=256),
                                 dict(debug_fail_first_wait=2), dict(debug_fail_first_wait=-1),
                                 dict(sequences=1 << 20, n_heads=4096), dict(tokens=1 << 28, n_heads=2048)])
def test_ragged_arguments_are_checked(bad):
    assert _call_ragged(_ragged(**bad)) == BAD


def test_ragged_pointers_are_checked():
    a = _ragged()
    assert _call_ragged(None) == BAD
    for i in range(5):                                   # q, k, v, begin, out
        for value in (None, FAR[i] + 2):
            p = FAR[:5]
            p[i] = value
            assert _call_ragged(a, p) == BAD, (i, value)
    for i in range(4):                                   # out shares memory with what is read
        p = FAR[:5]
        p[4] = p[i]
        assert _call_ragged(a, p) == BAD, i
    p = FAR[:5]
    p[4] = p[0] + 2 * 10 * 256 - 16                      # its last rows only
    assert _call_ragged(a, p) == BAD
    a = _ragged(bias_mode=1, d_alibi_slopes=FAR[4] + 64)
    assert _call_ragged(a) == BAD


def _cache(**kw):
    return _filled(kf.kf_page_cache, dict(n_pages=20, page_tokens=16, n_kv_heads=2, head_dim=64, sequences=3, table_width=4), kw)


BAD_CACHES = [dict(n_pages=0), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256), dict(n_kv_heads=0), dict(n_kv_heads=70000), dict(head_dim=80), dict(sequences=0),
              dict(sequences=(1 << 20) + 1), dict(table_width=0), dict(table_width=1 << 26), dict(n_pages=1 << 26), dict(n_pages=-1)]


def _rows(**kw):
    return _filled(kf.kf_page_rows, dict(tokens=7, type=1, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64), kw)


def _call_write(c, r, p=None):
    return kf.LIB.kf_pages_write(C.byref(c) if c is not None else None, C.byref(r) if r is not None else None, *(p or FAR[:7]), None)


def _call_read(c, r, p=None):
    return kf.LIB.kf_pages_read(C.byref(c), C.byref(r), *(p or FAR[:7]), None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_page_caches_are_checked(bad):
    c = _cache(**bad)
    assert _call_write(c, _rows()) == BAD and _call_read(c, _rows()) == BAD
    assert kf.LIB.kf_pages_attend_scratch_bytes(C.byref(_attend(c))) == 0
    u = kf.kf_pages_update_args(cache=c, n_layers=1)
    assert kf.LIB.kf_pages_update_scratch_bytes(C.byref(u)) == 0
    assert kf.LIB.kf_pages_compact(C.byref(c), 8, 4, *FAR[:7], None) == BAD


@pytest.mark.parametrize("bad", [dict(tokens=0), dict(tokens=(1 << 28) + 1), dict(type=2), dict(k_token_stride=60), dict(k_head_stride=68), dict(v_token_stride=0), dict(v_head_stride=-64)])
def test_page_rows_are_checked(bad):
    assert _call_write(_cache(), _rows(**bad)) == BAD and _call_read(_cache(), _rows(**bad)) == BAD


def test_page_row_pointers_are_checked():
    c, r = _cache(), _rows()
    assert _call_write(None, r) == BAD and _call_write(c, None) == BAD
    for i, offset in enumerate((8, 8, 2, 2, 2, 8, 4)):   # k, v, begin, length, table, cache, scale
        p = FAR[:7]
        p[i] += offset
        assert _call_write(c, r, p) == BAD, i
        p[i] = None
        assert _call_write(c, r, p) == BAD, i            # without begin there has to be one row per sequence
    for i in range(5):
        for to in (5, 6):                                # cache and scale share memory with nothing
            p = FAR[:7]
            p[to] = p[i]
            assert _call_write(c, r, p) == BAD, (i, to)
    for i, offset in enumerate((8, 4, 2, 2, 2, 8, 8)):   # cache, scale, table, begin, first, k, v
        p = FAR[:7]
        p[i] += offset
        assert _call_read(c, r, p) == BAD, i
        if i != 4:
            p[i] = None
            assert _call_read(c, r, p) == BAD, i
    for i in range(5):
        for to in (5, 6):
            p = FAR[:7]
            p[to] = p[i]
            assert _call_read(c, r, p) == BAD, (i, to)
    p = FAR[:7]
    p[6] = p[5] + 64
    assert _call_read(c, r, p) == BAD                    # k in v
    assert _call_read(c, _rows(k_token_stride=64)) == BAD                                  # rows that overlap


def _attend(c=None, **kw):
    return _filled(kf.kf_pages_attend_args, dict(cache=c or _cache(), n_heads=4, type=0, bias_mode=0, logit_scale=0.0, d_alibi_slopes=None, q_sequence_stride=256, q_head_stride=64,
                                                 out_sequence_stride=256, out_head_stride=64), kw)


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=3), dict(n_heads=65536 * 2), dict(type=2), dict(bias_mode=1), dict(bias_mode=-1), dict(logit_scale=-1.0),
                                 dict(logit_scale=float("nan")), dict(q_sequence_stride=60), dict(q_head_stride=0), dict(out_sequence_stride=100), dict(out_head_stride=32),
                                 dict(out_sequence_stride=64), dict(debug_fail_first_wait=2),
                                 dict(cache=_cache(sequences=1 << 20, table_width=1 << 16))])
def test_attend_arguments_are_checked(bad):
    a = _attend(**bad)
    assert kf.LIB.kf_pages_attend_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_pages_attend(C.byref(a), *FAR[:7], 1 << 40, None) == BAD


def test_attend_pointers_are_checked():
    a = _attend()
    need = kf.LIB.kf_pages_attend_scratch_bytes(C.byref(a))
    assert need > 0 and need % 256 == 0
    assert need == kf.kf_pages_attend_scratch_bytes(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_heads=4, n_kv_heads=2, head_dim=64)

    def rc(p, nbytes=need):
        return kf.LIB.kf_pages_attend(C.byref(a), *p, nbytes, None)
    assert rc(FAR[:7], need - 1) == SPACE
    for i, offset in enumerate((8, 8, 4, 2, 2, 8, 128)):     # q, cache, scale, table, length, out, scratch
        p = FAR[:7]
        p[i] += offset
        assert rc(p) == BAD, i
        p[i] = None
        assert rc(p) == BAD, i
    for to in (5, 6):
        for i in range(5):
            p = FAR[:7]
            p[to] = p[i]
            assert rc(p) == BAD, (i, to)
    p = FAR[:7]
    p[6] = p[5]
    assert rc(p) == BAD


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(n_layers=70000), dict(cache=_cache(sequences=8193)), dict(cache=_cache(sequences=8192, table_width=1 << 16))])
def test_update_arguments_are_checked(bad):
    a = _filled(kf.kf_pages_update_args, dict(cache=_cache(), n_layers=2, grow=1), bad)
    assert kf.LIB.kf_pages_update_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_pages_update(C.byref(a), *FAR[:9], 1 << 40, None) == BAD


def test_update_pointers_are_checked():
    a = _filled(kf.kf_pages_update_args, dict(cache=_cache(), n_layers=2, grow=1), {})
    need = kf.LIB.kf_pages_update_scratch_bytes(C.byref(a))
    assert need > 0 and need == kf.kf_pages_update_scratch_bytes(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_kv_heads=2, head_dim=64, n_layers=2)

    def rc(p, nbytes=need):
        return kf.LIB.kf_pages_update(C.byref(a), *p, nbytes, None)
    assert rc(FAR[:9], need - 1) == SPACE
    for i, offset in enumerate((2, 2, 2, 2, 2, 8, 4, 2, 16)):   # table, length, refs, parent, grow, cache, scale, missing, scratch
        p = FAR[:9]
        p[i] += offset
        assert rc(p) == BAD, i
        if i not in (3, 4):
            p[i] = None
            assert rc(p) == BAD, i
    for i in range(9):
        for j in range(i):
            if (i, j) != (4, 3):                             # parents and growth are only read
                p = FAR[:9]
                p[i] = p[j]
                assert rc(p) == BAD, (i, j)


def test_compact_arguments_are_checked():
    c = _cache()

    def rc(keep=8, width=4, p=None):
        return kf.LIB.kf_pages_compact(C.byref(c), keep, width, *(p or FAR[:7]), None)
    for keep, width in ((0, 4), (-1, 4), (8, 0), (65, 4), (8, 1 << 26)):
        assert rc(keep, width) == BAD
    for i, offset in enumerate((2, 2, 2, 2, 2, 8, 4)):       # table, length, keep, n_keep, new_table, cache, scale
        p = FAR[:7]
        p[i] += offset
        assert rc(p=p) == BAD, i
        p[i] = None
        assert rc(p=p) == BAD, i
    for i in range(5):
        for to in (5, 6):
            p = FAR[:7]
            p[to] = p[i]
            assert rc(p=p) == BAD


def test_binding_refuses_what_is_no_tensor_of_the_kind():
    x = torch.zeros(4, 2, 64)
    for call in (lambda: kf.kf_prefill_attend_ragged(q=x, k=x, v=x, begin=x, out=x), lambda: kf.kf_prefill_attend_ragged(q=None, k=x, v=x, begin=x, out=x),
                 lambda: kf.kf_pages_write(k=x, v=x, length=x, table=x, cache=x, scale=x), lambda: kf.kf_pages_attend(q=x, table=x, length=x, cache=x, scale=x, out=x),
                 lambda: kf.kf_pages_update(table=x, length=x, refs=x, cache=x, scale=x, missing=x),
                 lambda: kf.kf_pages_compact(cache=x, scale=x, table=x, length=x, keep=x, n_keep=x, new_table=x)):
        with pytest.raises(ValueError):
            call()


# ---- the plain form itself: what the header promises about scales

def test_plain_pages_hold_values_within_a_step_however_often_they_grow():
    rng = np.random.default_rng(0)
    cache, scale = np.zeros((1, 1, 2, 64, 64), np.int8), np.zeros((1, 1, 2), np.float32)
    rows = rng.standard_normal((2, 64, 1, 64)) * np.exp2(np.arange(64) / 8)[None, :, None, None]     # a scale that doubles every eighth row
    for t in range(64):
        ref.write(cache, scale, np.zeros((1, 1), np.int32), [t], rows[:, t:t + 1], [0, 1])
    error = np.abs(ref.held(cache, scale, np.zeros((1, 1), np.int32), 0, 64) - rows)
    step = scale[0, 0].astype(np.float64)[:, None, None, None]
    assert (error < step).all() and (error[:, 32:].max() > 0)
    assert (scale[0, 0] == 2.0 ** np.array([ref.power_of_two(np.abs(r).max()) for r in rows])).all()


@pytest.mark.parametrize("top,e", [(0.0, -120), (127.0, 0), (127.00001, 1), (1.0, -6), (63.5, -1), (65504.0, 10), (3.3895313892515355e38, 122), (2.0 ** -24, -30), (1e-40, -120)])
def test_plain_scales(top, e):
    assert ref.power_of_two(top) == e
