"""The operators on 8-bit pages where logits, scales and ranges lie at the ends of what they may be."""
import math

import numpy as np
import pytest
import torch

from tests import pages_reference as ref
from tests.test_gpu_pages import DEV, TYPES, _attend, _check, _ints, _kf, _pool, _table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e4, 1e8, 1e20, 1e32, 1e38])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("d,page,wide", [(64, 16, 0), (64, 64, 60), (128, 16, 60), (128, 32, 0), (256, 64, 60)])
def test_rows_whose_logits_are_all_huge(size, sign, d, page, wide):
    """All logits of a row are equal, finite and far from zero: their softmax is the mean.  Only feature 0 of keys and queries counts, so that a logit is one
    product, and equal in every tile whatever the binary32 roundings are."""
    n, Hkv = 200, 2
    pages = -(-n // page)
    cache, scale = _pool(pages, Hkv, page, d, seed=1)
    cache[:, :, 0], cache[:, :, 0, :, 0] = 0, 64
    scale[:, :, 0] = 2.0 ** -6                                       # keys: 1 in feature 0
    table = _table([n], page, pages, width=pages + wide)
    q = torch.zeros(1, 4, d, device=DEV, dtype=torch.bfloat16)
    q[..., 0] = sign * size
    out = _attend(q, table, [n], cache, scale, logit=1.0)
    v = torch.from_numpy(ref.held(cache.cpu().numpy(), scale.cpu().numpy(), table, 0, n)[1]).to(DEV).repeat_interleave(2, 1)
    want, weighted = v.mean(0), v.abs().mean(0)
    # all weights are equal: the output's rounding, and the binary32 arithmetic (2^-18)
    assert ((out[0].double() - want).abs() <= want.abs() * 2.0 ** -8 + weighted * 2.0 ** -18).all()
    # one key stands above the others by a fifth of the logits' size, far more than a softmax can tell from all
    cache[table[0, 3 // page], :, 0, 3 % page, 0] += sign * 13
    out = _attend(q, table, [n], cache, scale, logit=1.0)
    assert torch.equal(out[0], v[3].bfloat16())


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (256, 64)])
@pytest.mark.parametrize("after", [0, 1, 2, 3, 1000])
@pytest.mark.parametrize("S,longest,wide", [(400, 700, 0), (1, 100000, 0), (20, 500, 0), (20, 500, 1000)])
def test_a_wait_that_runs_out_in_the_middle(d, page, after, S, longest, wide):
    """Sequences and heads that a warp is done with before are right, bit for bit, those that it comes to later NaN; shares of many short sequences, parts of a long one, and
    a CTA for each."""
    Hkv = 16
    lengths = [longest * ((37 * i + 63) % 64) // 63 for i in range(S)]
    pages = sum(-(-n // page) for n in lengths) + 1
    cache, scale = _pool(pages, Hkv, page, d)
    table = _table(lengths, page, pages)
    table = np.concatenate([table, np.full((S, wide), -1, np.int32)], 1)
    q = torch.randn(S, 32, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)).half()
    want = _attend(q, table, lengths, cache, scale)
    got = _attend(q, table, lengths, cache, scale, debug_fail_first_wait=1, debug_fail_after=after)
    nan, tokens = torch.isnan(got).all(-1), torch.tensor(lengths, device=DEV)
    assert (nan | (got == want).all(-1)).all() and not nan[tokens == 0].any()
    assert not torch.isnan(want).any()
    if after == 0:
        assert nan[tokens > 0].all()
    if after == 1000:
        assert not nan.any()
    if after in (1, 2) and S == 400:        # shares: 73000 tiles or more of 16 heads over at most 1776 warps, at least 41 each
        assert nan.any() and not nan[tokens > 0].all()


@pytest.mark.parametrize("wide", [0, 60])
def test_values_near_the_smallest_scale(wide):
    """V scales of 2^-120: their outputs are far below one, but bfloat16 holds them."""
    d, page, n = 128, 32, 300
    pages = -(-n // page)
    cache, scale = _pool(pages, 2, page, d)
    table = _table([n], page, pages, width=pages + wide)
    q = torch.randn(1, 4, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)).bfloat16()
    scale[:, :, 1] = 2.0 ** -120
    out = _attend(q, table, [n], cache, scale)
    assert (out != 0).any()
    _check(out, q, table, [n], cache, scale)


@pytest.mark.parametrize("begin", [[0, 30, 30, 40], [0, 30, 20, 40], [-3, 10, 20, 40], [0, 10, 20, 400], [40, 30, 20, 10], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 7]])
def test_rows_of_ranges_that_are_not_valid_reach_no_page(begin):
    page, d, Hkv = 16, 64, 2
    cache, scale = _pool(12, Hkv, page, d)
    table = np.arange(12, dtype=np.int32).reshape(3, 4)[::-1].copy()
    want_c, want_s = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
    x = torch.randn(2, 40, Hkv, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)).half()
    b = torch.tensor(begin, device=DEV, dtype=torch.int64).to(torch.int32)
    _kf().kf_pages_write(k=x[0], v=x[1], begin=b, length=_ints([0, 3, 5]), table=_ints(table), cache=cache, scale=scale)
    got_c, got_s = cache.cpu().numpy(), scale.cpu().numpy()
    in_order = all(lo <= hi for lo, hi in zip(begin, begin[1:]))
    for s, (lo, hi) in enumerate(zip(begin, begin[1:])):
        if 0 <= lo < hi <= 40:
            ref.write(want_c, want_s, table[s:s + 1], [[0, 3, 5][s]], x.double().cpu().numpy(), [lo, hi])
            if not in_order:                    # what belongs to such a range is not said: only its own pages
                continue
        np.testing.assert_array_equal(got_c[table[s]], want_c[table[s]])
        np.testing.assert_array_equal(got_s[table[s]], want_s[table[s]])


@pytest.mark.parametrize("order", ["side by side", "head by head"])
def test_keys_and_values_that_alternate_in_one_buffer(order):
    """Both written into one tensor, as they are taken from one; and prompt attention with its output in the rows that hold q, k and v."""
    d, page, Hkv, T = 64, 16, 2, 70
    pages = -(-T // page)
    cache, scale = _pool(pages, Hkv, page, d)
    table, begin = _ints([list(range(pages))]), _ints([0, T])
    rows = torch.full((T, 2, Hkv, d) if order == "side by side" else (T, Hkv, 2, d), 5.0, device=DEV).half()
    k, v = (rows[:, 0], rows[:, 1]) if order == "side by side" else (rows[:, :, 0], rows[:, :, 1])
    apart = torch.empty(2, T, Hkv, d, device=DEV).half()
    _kf().kf_pages_read(table=table, cache=cache, scale=scale, k=k, v=v, begin=begin)
    _kf().kf_pages_read(table=table, cache=cache, scale=scale, k=apart[0], v=apart[1], begin=begin)
    assert torch.equal(k, apart[0]) and torch.equal(v, apart[1])
    with pytest.raises(_kf().KeyformerError):
        _kf().kf_pages_read(table=table, cache=cache, scale=scale, k=k, v=k, begin=begin)
    wide = torch.randn(T, 4 + 2 * Hkv + 4, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)).half()
    q, k, v, out = wide[:, :4], wide[:, 4:4 + Hkv], wide[:, 4 + Hkv:4 + 2 * Hkv], wide[:, 4 + 2 * Hkv:]
    want, before = torch.empty(T, 4, d, device=DEV).half(), wide.clone()
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=want)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    assert torch.equal(out, want) and torch.equal(wide[:, :4 + 2 * Hkv], before[:, :4 + 2 * Hkv])
    with pytest.raises(_kf().KeyformerError):
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=wide[:, 4 + 2 * Hkv - 1:-1])
