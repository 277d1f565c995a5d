"""What the context-free operators refuse, on the host and before anything is enqueued (no device needed), and the plain
4-bit form that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
from tests import operators_reference as ref

OK = 4096      # an aligned address that is never dereferenced
FAR = [OK + (i << 32) for i in range(16)]      # such addresses, far apart


def test_slot_sizes():
    assert [kf.kf_packed_slot_bytes(d) for d in (64, 128, 256, 96, 0, -64)] == [80, 160, 320, 0, 0, 0]


@pytest.mark.parametrize("call", ["pack", "unpack"])
def test_row_conversion_refusals(call):
    def rc(units=2, n=3, k=4, d=64, a=FAR[0], b=FAR[1], length=None, c=FAR[2]):
        if call == "pack":
            return kf.LIB.kf_pack_cache(units, n, k, d, a, b, length, c, None)
        return kf.LIB.kf_unpack_cache(units, n, k, d, c, length, a, b, None)
    for bad in (dict(units=0), dict(n=0), dict(n=5), dict(d=96), dict(a=None), dict(b=None), dict(c=None), dict(a=OK + 2), dict(b=OK + 8), dict(c=OK + 4),
                dict(length=OK + 2), dict(units=1 << 40), dict(units=-1), dict(c=FAR[0]), dict(c=FAR[1] + 128)):
        assert rc(**bad) == kf.KF_EINVAL, bad
    if call == "unpack":
        assert rc(a=FAR[1] + 128) == kf.KF_EINVAL


def _step(**kw):
    a = kf.kf_packed_step()
    base = dict(batch=2, n_heads=4, n_kv_heads=0, head_dim=64, budget_k=32, recent_w=8, layer=0, position=5, noise_mode=0, bias_mode=0, tau=1.0)
    base.update(kw)
    for name, value in base.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("bad", [dict(batch=0), dict(n_heads=0), dict(head_dim=32), dict(n_kv_heads=3), dict(n_kv_heads=8), dict(n_kv_heads=-1), dict(budget_k=0),
                                 dict(recent_w=33), dict(recent_w=-1), dict(layer=-1), dict(position=-1), dict(tau=0.0), dict(tau=float("nan")),
                                 dict(tau=float("inf")), dict(noise_mode=4), dict(noise_mode=-1), dict(noise_mode=3, noise_sigma=-1.0), dict(bias_mode=1),
                                 dict(bias_mode=2), dict(logit_scale=-1.0), dict(batch=70000), dict(n_heads=32, n_kv_heads=1), dict(budget_k=(1 << 26) + 1)])
def test_packed_step_arguments_are_checked(bad):
    a = _step(**bad)
    assert kf.LIB.kf_packed_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_decode_step_packed(C.byref(a), *[OK] * 8, None, None, None, OK, 1 << 30, None) == kf.KF_EINVAL


def test_packed_step_pointers_are_checked():
    a = _step()
    need = kf.LIB.kf_packed_scratch_bytes(C.byref(a))
    assert need == kf.kf_packed_scratch_bytes(batch=2, n_heads=4, head_dim=64, budget_k=32) and need % 256 == 0

    def rc(index=None, value=None, nbytes=need):
        p = FAR[:12]
        if index is not None:
            p[index] = value
        return kf.LIB.kf_decode_step_packed(C.byref(a), *p, nbytes, None)
    for i in range(8):                                   # everything up to d_out is required
        assert rc(i, None) == kf.KF_EINVAL
    assert rc(11, None) == kf.KF_EINVAL
    for i in (0, 4, 5, 6, 7):                            # cache, q, k_new, v_new, out
        assert rc(i, OK + 8) == kf.KF_EINVAL
    for i in (1, 2, 3, 8, 9):                            # positions, scores, counts, score_opt, slot_opt
        assert rc(i, OK + 2) == kf.KF_EINVAL
    assert rc(10, OK + 1) == kf.KF_EINVAL and rc(11, OK + 128) == kf.KF_EINVAL
    for i in (4, 5, 6):                                  # the output in place of q, k_new, v_new
        assert rc(7, FAR[i] + 16) == kf.KF_EINVAL
    assert rc(nbytes=need - 1) == kf.KF_ENOSPC
    assert kf.LIB.kf_decode_step_packed(None, *[OK] * 12, need, None) == kf.KF_EINVAL


def _norm(**kw):
    a = kf.kf_qk_norm_args()
    base = dict(batch=2, n_tokens=3, n_heads=4, n_kv_heads=2, head_dim=64, input_type=0, batch_stride=3 * 512, token_stride=512, norm_mode=1, eps=1e-6,
                rotary_dims=32, rotary_style=0, rotary_base=10000.0, position0=0)
    base.update(kw)
    for name, value in base.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("bad", [dict(batch=0), dict(n_tokens=0), dict(n_heads=0), dict(n_kv_heads=0), dict(head_dim=80), dict(input_type=2), dict(token_stride=504),
                                 dict(token_stride=516), dict(batch_stride=1540), dict(batch_stride=-8), dict(norm_mode=2), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(rotary_dims=4), dict(rotary_dims=48), dict(rotary_dims=128), dict(rotary_dims=-8), dict(rotary_base=1.0),
                                 dict(rotary_base=float("inf")), dict(rotary_style=2), dict(norm_mode=0), dict(batch=1 << 20, n_tokens=1 << 12)])
def test_norm_rotate_arguments_are_checked(bad):
    a = _norm(**bad)
    assert kf.LIB.kf_qk_norm_rotate(C.byref(a), *[OK] * 7, None) == kf.KF_EINVAL      # norm_mode 0: weights were passed


def test_norm_rotate_pointers_are_checked():
    a = _norm()
    for i in (0, 4, 5):
        p = [OK] * 7
        p[i] = None
        assert kf.LIB.kf_qk_norm_rotate(C.byref(a), *p, None) == kf.KF_EINVAL
    for i, off in ((0, 8), (1, 8), (2, 2), (3, 2), (4, 8), (5, 4), (6, 8)):
        p = FAR[:7]
        p[i] += off
        assert kf.LIB.kf_qk_norm_rotate(C.byref(a), *p, None) == kf.KF_EINVAL
    for i, j in ((4, 0), (5, 0), (6, 0), (5, 4), (6, 4), (6, 5)):      # outputs that overlap
        p = FAR[:7]
        p[i] = p[j] + 512
        assert kf.LIB.kf_qk_norm_rotate(C.byref(a), *p, None) == kf.KF_EINVAL
    a = _norm(position0=2 ** 31 - 2)                      # positions would pass 2^31 - 1
    assert kf.LIB.kf_qk_norm_rotate(C.byref(a), OK, OK, OK, None, OK, OK, OK, None) == kf.KF_EINVAL


def _beam(**kw):
    a = kf.kf_beam_args()
    base = dict(batch=2, beams=3, vocab=100, take=6, logits_type=0, pad_token=0, row_stride=100)
    base.update(kw)
    for name, value in base.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("bad", [dict(batch=0), dict(beams=0), dict(beams=33), dict(vocab=0), dict(take=0), dict(take=65), dict(vocab=1, row_stride=1, take=4),
                                 dict(logits_type=3), dict(logits_type=-1), dict(row_stride=99), dict(pad_token=-1), dict(pad_token=100), dict(batch=30000)])
def test_beam_select_arguments_are_checked(bad):
    a = _beam(**bad)
    assert kf.LIB.kf_beam_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_beam_select(C.byref(a), *[OK] * 7, 1 << 30, None) == kf.KF_EINVAL


def test_beam_select_pointers_are_checked():
    a = _beam()
    need = kf.LIB.kf_beam_scratch_bytes(C.byref(a))
    for i in (0, 1, 3, 4, 5, 6):
        p = [OK] * 7
        p[i] = None
        assert kf.LIB.kf_beam_select(C.byref(a), *p, need, None) == kf.KF_EINVAL
    for i, off in ((0, 1), (1, 2), (3, 2), (4, 2), (5, 2), (6, 64)):
        p = FAR[:7]
        p[i] += off
        assert kf.LIB.kf_beam_select(C.byref(a), *p, need, None) == kf.KF_EINVAL
    for i, j in ((3, 1), (4, 3), (5, 3), (5, 4)):                      # new scores over the old ones, outputs over one another
        p = FAR[:7]
        p[i] = p[j] + 8
        assert kf.LIB.kf_beam_select(C.byref(a), *p, need, None) == kf.KF_EINVAL
    assert kf.LIB.kf_beam_select(C.byref(a), *FAR[:7], need - 1, None) == kf.KF_ENOSPC


def test_reorder_arguments_are_checked():
    def rc(n=1, batch=2, beams=4, parent=OK, **kw):
        b = kf.kf_row_buffer(FAR[1], 64, 0, 1)
        for name, value in kw.items():
            setattr(b, name, value)
        return kf.LIB.kf_reorder_rows(C.byref(b), n, batch, beams, parent, None)
    for bad in (dict(n=0), dict(n=9), dict(batch=0), dict(batch=65536), dict(beams=0), dict(beams=33), dict(parent=None), dict(parent=OK + 2), dict(d_base=None),
                dict(row_bytes=0), dict(row_bytes=-16), dict(outer=0), dict(outer=2, outer_stride=64 * 8 - 1)):
        assert rc(**bad) == kf.KF_EINVAL, bad
    two = (kf.kf_row_buffer * 2)(kf.kf_row_buffer(FAR[0], 64, 0, 1), kf.kf_row_buffer(FAR[0] + 256, 64, 0, 1))      # 512 bytes each
    assert kf.LIB.kf_reorder_rows(two, 2, 2, 4, FAR[3], None) == kf.KF_EINVAL
    assert kf.LIB.kf_reorder_rows(two, 1, 2, 4, FAR[0] + 64, None) == kf.KF_EINVAL                             # the parents inside a buffer
    assert kf.LIB.kf_reorder_rows(None, 1, 1, 1, OK, None) == kf.KF_EINVAL
    assert kf.LIB.kf_reorder_beams(None, 0, 1, OK, None) == kf.KF_EINVAL


def test_binding_refuses_host_tensors():
    t = torch.zeros(2, 3, 64, dtype=torch.float16)
    cache = torch.zeros(2, 3, 80, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        kf.kf_pack_cache(K=t, V=t, cache=cache)
    with pytest.raises(ValueError, match="CUDA"):
        kf.kf_reorder_rows(buffers=[t], parent=torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        kf.kf_qk_norm_rotate(qkv=t, n_heads=1, n_kv_heads=1, head_dim=64, q=t, k=t)


def test_plain_four_bit_rows():
    """Every value of a finite group comes back within half a step and a rounding, the smallest exactly, none above the largest."""
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((50, 128)) * np.exp(rng.standard_normal((50, 1)) * 3)).astype(np.float16)
    x[0] = 1.5                                            # constant: exact
    x[1, :32] = np.linspace(-65504, 65504, 32).astype(np.float16)
    slots = ref.slots_of(x, x[::-1].copy())
    k, v = ref.rows_of(slots, 128)
    assert slots.shape == (50, 160) and np.array_equal(k, v[::-1])
    g, back = x.astype(np.float64).reshape(50, 4, 32), k.astype(np.float64).reshape(50, 4, 32)
    low, high = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
    scale = ref.half_down((high - low) / 15).astype(np.float64)
    # half a step (the last code also stands for what the scale's rounding left out: 15 steps of relative 2^-10 or absolute 2^-24), one rounding
    bound = scale / 2 + 15 * np.maximum(scale * 2.0 ** -10, 2.0 ** -24) + np.abs(g).max(-1, keepdims=True) * 2.0 ** -11
    assert (np.abs(back - g) <= bound).all() and (back <= high).all()
    assert (np.where(g == low, back, low) == low).all() and (back[0] == 1.5).all()
