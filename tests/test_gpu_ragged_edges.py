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
