"""The context-free operators where a call goes wrong or its inputs are at the edge of what is allowed."""
import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
from tests.test_gpu_operators import DEV, Packed

pytestmark = pytest.mark.gpu


def _state(s):
    return [torch.nan_to_num(t.clone()) for t in (s.cache, s.pos, s.acc, s.length)]


@pytest.mark.parametrize("batch,heads,kv,d,k", [(40, 4, 4, 64, 300), (1, 3, 3, 128, 2500), (2, 8, 2, 128, 700), (1, 16, 2, 256, 300)])
def test_packed_step_whose_rows_do_not_arrive(batch, heads, kv, d, k):
    """debug_fail_first_wait: every warp gives up its first wait, as if the bounded wait had run out (the copies in flight are waited for all the same).
    The units say so and keep their state; one without entries has nothing to wait for.  The next call finds nothing of it."""
    make = lambda: Packed(batch, heads, kv, d, k, 20, lengths=[k, 0, k // 2], seed=61)     # noqa: E731
    s, plain = make(), make()
    inputs = s.inputs(1)
    scratch = torch.zeros(kf.kf_packed_scratch_bytes(batch=batch, n_heads=heads, n_kv_heads=kv, head_dim=d, budget_k=k), dtype=torch.uint8, device=DEV)
    before = _state(s)
    out, score, slot, _ = s.call(1, *inputs, scratch=scratch, debug_fail_first_wait=1)
    torch.cuda.synchronize()
    length = before[3].tolist()
    out, after = out.view(s.U, -1), _state(s)
    for u, n in enumerate(length):
        if n:
            assert torch.isnan(out[u]).all() and torch.isnan(score[u, :n + 1]).all() and (score[u, n + 1:] == -5.0).all() and slot[u] == kf.KF_ETIMEOUT
            assert all(torch.equal(now[u], old[u]) for now, old in zip(after, before))
        else:
            assert torch.isfinite(out[u]).all() and slot[u] == 0 and after[3][u] == 1 and score[u, 0] == 1.0
    for t, old in zip((s.cache, s.pos, s.acc, s.length), (plain.cache, plain.pos, plain.acc, plain.length)):
        t.copy_(old)
    again, want = s.call(1, *inputs, scratch=scratch), plain.call(1, *inputs)
    assert all(torch.equal(a, b) for a, b in zip(again, want)) and torch.isfinite(again[0]).all()
    assert all(torch.equal(a, b) for a, b in zip(_state(s), _state(plain)))


def test_packed_step_checks_the_self_test_argument():
    s = Packed(1, 2, 2, 64, 8, 2)
    with pytest.raises(kf.KeyformerError):
        s.call(1, *s.inputs(1), debug_fail_first_wait=2)


@pytest.mark.parametrize("batch,heads,kv,d,k", [(40, 4, 4, 64, 60), (1, 2, 2, 128, 2300), (2, 8, 2, 128, 90)])
def test_packed_step_without_an_entry_to_evict(batch, heads, kv, d, k):
    """A position passed twice with w = k: every entry of the full cache lies inside the window.  The step says so in slot_out; outputs and scores are those
    of a step that stores its row."""
    s = Packed(batch, heads, kv, d, k, k, noise=kf.KF_NOISE_NONE, seed=71)        # noise would depend on the position
    s.step(1)
    state = [t.clone() for t in (s.cache, s.pos, s.acc, s.length)]
    inputs = s.inputs(2)
    want, want_score, slot, _ = s.call(2, *inputs)                        # the next position: the oldest leaves
    assert (slot >= 0).all()
    for t, old in zip((s.cache, s.pos, s.acc, s.length), state):
        t.copy_(old)
    s.n -= 1                                                              # step 2 at the position of step 1
    out, score, slot, _ = s.call(2, *inputs)
    assert (slot == kf.KF_EBOUNDS).all()
    assert torch.equal(out, want) and torch.equal(score, want_score)
    assert torch.equal(s.cache, state[0]) and torch.equal(s.pos, state[1]) and torch.equal(s.length, state[3])
    assert torch.equal(s.acc, state[2] + score[:, :k])
