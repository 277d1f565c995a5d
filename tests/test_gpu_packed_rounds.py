"""The step over a 4-bit cache where a warp of the streaming kernel takes several rounds: buffers filled again, barriers that change parity,
positions and noise of later rounds, output references that move while the sums are not zero.  Compared with the oracle entry by entry."""
import math

import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
from tests import operators_reference as ref
from tests.test_gpu_operators import DEV, Packed, _randn

pytestmark = pytest.mark.gpu

WARPS, SPAN, TILE = 4, 64, 32          # of the streaming kernel: warps per CTA, slots per warp and round, slots per tile
ROUND = WARPS * SPAN                   # slots of one round of a CTA


def slots_per_split(batch, heads, kv, d, k):
    """Slots a CTA works off, from the number of partial results the scratch has room for."""
    align = lambda n: (n + 255) // 256 * 256                                               # noqa: E731
    total = kf.kf_packed_scratch_bytes(batch=batch, n_heads=heads, n_kv_heads=kv, head_dim=d, budget_k=k)
    partials = total - align(batch * heads * (k + 1) * 4)
    splits = partials // (batch * heads * (4 + d) * 4)
    tiles = -(-k // TILE)
    per = -(-tiles // splits)
    return -(-per * TILE // ROUND) * ROUND


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_several_rounds_per_warp(d, group):
    """Three rounds; one cache full, the other ending inside a later round of a CTA."""
    k = 33001
    assert slots_per_split(1, 2 * group, 2, d, k) == 3 * ROUND
    s = Packed(1, 2 * group, 2, d, k, 7000, lengths=[k, 26500], alibi=group == 2, seed=50 + d + group)
    assert 26500 % (3 * ROUND) > ROUND and 26500 % ROUND % SPAN != 0
    s.step(1)
    if group in (1, 4):
        s.step(2)


def test_several_rounds_in_many_caches():
    """As many caches as give every CTA half a cache, of all lengths."""
    assert slots_per_split(125, 8, 8, 64, 1500) == 3 * ROUND
    s = Packed(125, 8, 8, 64, 1500, 300, lengths=[1500, 0, 1, 255, 257, 511, 767, 768, 769, 1031, 1279, 1499], seed=90)
    s.step(1)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_output_references_move_in_later_rounds(d, group):
    """In the second round of odd warps and the third of even ones, one entry lies e^5.5 and more above what the warp has met: its sums are scaled
    down, and what they hold still counts for a percent or more of the output (the other entries' values lie 3 away from zero, the tall ones' around
    it).  The heads' logits of the tall entries differ, so that every head has a factor of its own."""
    k, w = 33001, 7000
    per = slots_per_split(1, 2 * group, 2, d, k)
    assert per == 3 * ROUND
    s = Packed(1, 2 * group, 2, d, k, w, seed=70 + d + group, loud=0.0, noise=kf.KF_NOISE_NONE)
    q = s.inputs(1)[0].double().cpu().view(2, group, d)
    slot = torch.arange(k)
    inside = slot % per
    rnd, warp, split = inside // ROUND, inside % ROUND // SPAN, slot // per
    tall = (rnd == torch.where(warp % 2 == 1, 1, 2)) & (inside % SPAN == (13 * warp + 29) % SPAN)
    logit = 9.0 * (1.0 + 0.12 * torch.arange(group, dtype=torch.float64) / max(1, group - 1))
    along = torch.linalg.pinv(q) @ (logit * math.sqrt(d))                                  # the row with these logits
    K = torch.where(tall[:, None].to(DEV), along[:, None].float().to(DEV), _randn(s.seed, 2, k, d)).half()
    away = 3.0 * (1 - 2 * (torch.arange(d, device=DEV) % 2))
    V = torch.where(tall[:, None].to(DEV), _randn(s.seed + 1, 2, k, d), _randn(s.seed + 1, 2, k, d) + away).half()
    kf.kf_pack_cache(K=K, V=V, cache=s.cache)
    # the kernel's rule on the logits of the stored rows: where references move, and the share of what was summed before the last move
    Kr = torch.from_numpy(ref.rows_of(s.cache.cpu().numpy(), d)[0]).to(DEV).double()
    x = np.moveaxis((q.to(DEV) @ Kr.transpose(1, 2) / math.sqrt(d)).cpu().numpy(), 2, 0)   # [k, 2, group]
    at = (rnd.numpy(), split.numpy(), warp.numpy())
    peak = np.full((3, int(split.max()) + 1, WARPS, 2, group), -np.inf)
    total = np.zeros_like(peak)
    np.maximum.at(peak, at, x)
    np.add.at(total, at, np.exp(x))
    held, before, moved = peak[0].copy(), np.zeros_like(peak[0]), np.zeros((2, group), int)
    for r in (1, 2):
        up = peak[r] > held + 5.5
        moved += up.sum((0, 1))
        before = np.where(up, total[:r].sum(0), before)
        held = np.where(up, peak[r], held)
    assert (moved > 40).all(), moved
    assert (before.sum((0, 1)) > 3e-3 * total.sum((0, 1, 2))).all()
    s.step(1)


def test_many_small_weights_count_together():
    """33 million entries, one in each warp 2^25.5 times as heavy as the others: those are 0.3 % of the output's weight, and all of its value."""
    d, k = 64, 1 << 25
    per = slots_per_split(1, 1, 1, d, k)
    warps = k // per * WARPS
    assert k % per == 0 and per // WARPS == 1 << 17
    row = lambda kv: torch.full((1, 1, d), kv, dtype=torch.float16, device=DEV)            # noqa: E731
    slots = [torch.zeros(1, 1, 80, dtype=torch.uint8, device=DEV) for _ in range(2)]
    kf.kf_pack_cache(K=row(0.0), V=row(8.0), cache=slots[0])               # constant groups are exact
    kf.kf_pack_cache(K=row(2.21), V=row(0.0), cache=slots[1])
    cache = slots[0].repeat(1, k, 1)
    cache.view(k // per, per // SPAN, SPAN, 80)[:, :WARPS, 5] = slots[1][0, 0]
    logit = float(row(2.21)[0, 0, 0]) * d / 8.0
    pos = torch.arange(k, dtype=torch.int32, device=DEV).view(1, k)
    acc, length = torch.zeros(1, k, device=DEV), torch.full((1,), k, dtype=torch.int32, device=DEV)
    out, q = torch.zeros(1, 1, d, dtype=torch.float16, device=DEV), torch.ones(1, 1, d, dtype=torch.float16, device=DEV)
    kf.kf_decode_step_packed(batch=1, n_heads=1, head_dim=d, budget_k=k, recent_w=10, layer=0, position=k, tau=1.0, cache=cache, pos=pos, acc=acc, length=length,
                             q=q, knew=row(0.0), vnew=row(8.0), out=out, noise_mode=kf.KF_NOISE_NONE)
    light = (k - warps + 1) * math.exp(-logit)
    want = 8.0 * light / (warps + light)
    # a weight is off by 2^-32 of its warp's largest (half a step of the smallest binary16 numbers, times 2^-7), by 2^-22 of the exponent's 26 and in its
    # logit by 72 2^-23 of 18; the sums by less, the output by a rounding
    off = 8.0 * per / WARPS * 2.0 ** -32 + want * (26 * 2.0 ** -22 + 72 * 2.0 ** -23 * 18 + 2.0 ** -20 + 2.0 ** -11)
    assert want > 0.02 and (out.double() - want).abs().max() <= off, (out.double() - want).abs().max()
