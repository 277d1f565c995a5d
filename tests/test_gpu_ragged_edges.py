"""kf_prefill_attend_ragged: places without rows, waits that run out in the middle, weights and logits at the ends of their types."""
import math

import pytest
import torch

from tests import pages_reference as ref
from tests.test_gpu_ragged import DEV, TYPES, _check, _inputs, _kf

pytestmark = pytest.mark.gpu


def test_a_million_sequences_of_which_a_few_have_rows():
    """The places of a million empty sequences lie before those of the few at the front: 900000 of them for every CTA, longer than one bounded wait lasts."""
    S, H, d = 1 << 20, 128, 64
    lengths = [40, 0, 129, 3]
    q, k, v, begin, out = _inputs(lengths, H, H, d, torch.bfloat16, before=2, behind=6)
    whole = torch.full((S + 1,), int(begin[-1]), device=DEV, dtype=torch.int32)
    whole[:len(begin)] = begin
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=whole, out=out)
    _check(q, k, v, begin, out)


@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 1), (128, 6, 6), (256, 4, 2)])
@pytest.mark.parametrize("lengths", [[300, 5], [0] * 40 + [77] + [0] * 300 + [130, 0, 1] + [0] * 50])
def test_a_buffer_much_longer_than_its_sequences(d, H, Hkv, lengths):
    q, k, v, begin, out = _inputs(lengths, H, Hkv, d, torch.float16, before=1, behind=20000)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    _check(q, k, v, begin, out)


@pytest.mark.parametrize("d,H,Hkv", [(64, 8, 2), (128, 8, 8), (256, 4, 2)])
@pytest.mark.parametrize("after", [0, 1, 3, -1, -2, -4])
def test_a_wait_that_runs_out_in_the_middle(d, H, Hkv, after):
    """The pieces of work before it are right, bit for bit, all others NaN, however many have been claimed, and rows of nobody as they were.  A negative number: a role that waits
    for its next piece gives up and leaves, so that pieces that have been handed out are taken by some roles only, or by none."""
    lengths = [(53 * i) % 500 for i in range(150)]
    q, k, v, begin, out = _inputs(lengths, H, Hkv, d, torch.bfloat16, before=1, behind=400)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    _check(q, k, v, begin, out)
    got = torch.full_like(out, 7.0)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=got, debug_fail_first_wait=1, debug_fail_after=after)
    own = slice(int(begin[0]), int(begin[-1]))
    nan = torch.isnan(got[own]).all(-1)
    assert (nan | (got[own] == out[own]).all(-1)).all() and nan.any()
    assert nan.all() if after in (0, -1) else not nan.all()
    assert (got[:1] == 7.0).all() and (got[own.stop:] == 7.0).all()
    got.fill_(7.0)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=got)
    assert torch.equal(got, out)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("alibi", [False, True])
def test_rows_whose_logits_are_all_large(d, dtype, sign, alibi):
    """Logits of a million, all equal: a row is the mean of the values up to it.  Then one key that stands above all others."""
    q, k, v, begin, out = _inputs([300, 40], 4, 2, d, TYPES[dtype])
    q[:], k[:] = 0, 0
    q[..., 0], k[..., 0] = sign * 1000.0, 1000.0
    kw = dict(bias_mode=1, alibi_slopes_dev=torch.zeros(4, device=DEV)) if alibi else {}
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=1.0, **kw)
    # rounded weights are all the same, so they and the output are off by half a step each; binary32 arithmetic below 2^-18
    half = torch.finfo(TYPES[dtype]).eps / 2
    floor = 2.0 ** -25 if dtype == "fp16" else 0.0
    for lo, hi in ((0, 300), (300, 340)):
        rows = v[lo:hi].double().repeat_interleave(2, 1)
        count = torch.arange(1, hi - lo + 1, device=DEV)[:, None, None]
        want, weighted = rows.cumsum(0) / count, rows.abs().cumsum(0) / count
        assert ((out[lo:hi].double() - want).abs() <= half * want.abs() + (half + 2.0 ** -18) * weighted + floor).all()
    k[3, :, 0] += sign * 8.0
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=1.0, **kw)
    want = v[3].double().repeat_interleave(2, 0)
    assert ((out[3:300].double() - want).abs() <= (2 * half + 2.0 ** -18) * want.abs() + floor).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("exponent", [21.3, 24.7, 27.4, 30.2, 31.6])
@pytest.mark.parametrize("d", [64, 256])
def test_weights_below_the_normal_numbers(dtype, exponent, d):
    """One key with weight 1 and no value, thousands with weights between 2^-21 and 2^-32 that are no powers of two: each is off by at most 2^-32 in
    binary16 (a half step of the subnormal numbers, 2^-25, at 2^7 times the weight), beside its relative rounding."""
    n, H = 4001, 2
    q, k, v, begin, out = _inputs([n], H, 1, d, TYPES[dtype])
    q[:], k[:] = 0, 0
    q[..., 0], k[1:, :, 0] = 1.0, -exponent
    v[:], v[1:] = 0, 1000.0
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=math.log(2.0))
    want, weighted, size = ref.attend_rows(q[-1:].double(), k.double(), v.double(), math.log(2.0), causal=False)
    limit = ref.bound(want, weighted, size, out.dtype, d, True) + (2.0 ** -32 * 1000.0 * (n - 1) if dtype == "fp16" else 0)
    assert ((out[-1:].double() - want).abs() <= limit).all()
    assert (out[-1] > 0).all()
