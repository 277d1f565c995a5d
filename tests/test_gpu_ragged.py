"""kf_prefill_attend_ragged against a plain form in 64 bits (tests/pages_reference.py, which also derives the bounds)."""
import math

import pytest
import torch

from tests import pages_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _kf():
    import paper_2403_09054_b200 as kf
    return kf


def _inputs(lengths, H, Hkv, d, dtype, layout="fused", seed=0, before=0, behind=0, spread=1.0):
    """Rows of sequences of these lengths, `before` rows of nobody in front and `behind` at the end."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T = max(1, before + sum(lengths) + behind)
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=gen)   # noqa: E731
    q, k, v = normal(T, H, d) * spread, normal(T, Hkv, d), normal(T, Hkv, d)
    if layout == "fused":
        rows = torch.cat([q, k, v], 1).to(dtype)
        q, k, v = rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
        out = torch.full((T, H, d), 7.0, device=DEV, dtype=dtype)
    elif layout == "heads":
        q, k, v = (x.transpose(0, 1).contiguous().to(dtype).transpose(0, 1) for x in (q, k, v))
        out = torch.full((H, T, d), 7.0, device=DEV, dtype=dtype).transpose(0, 1)
    else:       # odd strides: every second row of rows with room behind the heads
        def odd(x):
            wide = torch.full((2 * x.shape[0], x.shape[1] + 1, d + 8), 9.0, device=DEV, dtype=dtype)
            wide[::2, :-1, :d] = x.to(dtype)
            return wide[::2, :-1, :d]
        q, k, v, out = odd(q), odd(k), odd(v), odd(torch.full((T, H, d), 7.0, device=DEV))
    begin = [before + sum(lengths[:i]) for i in range(len(lengths) + 1)]
    return q, k, v, torch.tensor(begin, device=DEV, dtype=torch.int32), out


def _check(q, k, v, begin, out, slopes=None, scale=None, skip=()):
    H, d = q.shape[1:]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    owned = torch.zeros(q.shape[0], dtype=torch.bool, device=DEV)
    b = begin.tolist()
    for i, (lo, hi) in enumerate(zip(b, b[1:])):
        if i in skip or hi <= lo:
            continue
        owned[lo:hi] = True
        want, weighted, size = ref.attend_rows(q[lo:hi].double(), k[lo:hi].double(), v[lo:hi].double(), scale, slopes)
        error = (out[lo:hi].double() - want).abs()
        limit = ref.bound(want, weighted, size, out.dtype, d, True)
        assert torch.isfinite(out[lo:hi]).all() and (error <= limit).all(), (i, hi - lo, float((error / limit).max()))
    assert (out[~owned] == 7.0).all()       # rows of no sequence are left as they were


LENGTHS = [0, 1, 2, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 0]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv,layout,alibi", [(2, 2, "fused", False), (4, 2, "heads", True), (4, 1, "odd", False), (8, 1, "fused", True), (6, 2, "heads", False), (16, 1, "odd", True),
                                                (1, 1, "odd", True)])
def test_every_length_and_layout(d, dtype, H, Hkv, layout, alibi):
    q, k, v, begin, out = _inputs(LENGTHS, H, Hkv, d, TYPES[dtype], layout, before=3, behind=5)
    slopes = torch.exp2(-8.0 * torch.arange(1, H + 1, device=DEV) / H) if alibi else None
    kf = _kf()
    kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, bias_mode=1 if alibi else 0, alibi_slopes_dev=slopes)
    _check(q, k, v, begin, out, slopes)


@pytest.mark.parametrize("d,H,Hkv,lengths", [(64, 2, 1, [2500]), (128, 4, 4, [1, 3001]), (128, 8, 1, [1999, 700]), (256, 2, 2, [1111, 1])])
def test_long_sequences(d, H, Hkv, lengths):
    q, k, v, begin, out = _inputs(lengths, H, Hkv, d, torch.bfloat16)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=0.3)
    _check(q, k, v, begin, out, scale=0.3)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_row(d):
    q, k, v, begin, out = _inputs([1], 4, 2, d, torch.float16)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    assert torch.equal(out, v.repeat_interleave(2, 1))


@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 1), (128, 2, 2), (256, 2, 1)])
def test_what_belongs_to_others_reaches_no_output(d, H, Hkv):
    """Rows of the neighbours, and of nobody, that are NaN or infinite."""
    lengths = [40, 100, 129, 1, 200]
    q, k, v, begin, out = _inputs(lengths, H, Hkv, d, torch.bfloat16, before=2, behind=300)
    b = begin.tolist()
    for bad in ([0, 2, 4], [1, 3]):
        spoilt = torch.zeros(q.shape[0], dtype=torch.bool, device=DEV)
        spoilt[:2] = True
        spoilt[b[-1]:] = True
        for i in bad:
            spoilt[b[i]:b[i + 1]] = True
        for x in (q, k, v):
            x[spoilt] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device=DEV, dtype=x.dtype).repeat(d // 4)
        out.fill_(7.0)
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
        for i in bad:
            assert torch.isnan(out[b[i]:b[i + 1]]).any()
            out[b[i]:b[i + 1]] = 7.0
        q, k, v, _, _ = _inputs(lengths, H, Hkv, d, torch.bfloat16, before=2, behind=300)
        _check(q, k, v, begin, out, skip=bad)


def test_later_keys_that_are_not_finite_reach_no_earlier_row():
    q, k, v, begin, out = _inputs([300], 2, 2, 128, torch.float16)
    k[150:] = float("nan")
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    first = torch.tensor([0, 150], device=DEV)
    out[150:] = 7.0
    _check(q, k, v, first, out)


@pytest.mark.parametrize("begin", [[0, 50, 40, 90], [-5, 20, 60, 90], [0, 30, 60, 1000], [90, 60, 30, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0], [95, 96, 97, 98]])
def test_ranges_that_are_not_valid_touch_nothing(begin):
    q, k, v, _, out = _inputs([97], 2, 1, 64, torch.float16)
    b = torch.tensor(begin, device=DEV, dtype=torch.int64).to(torch.int32)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=b, out=out)
    inside = torch.zeros(97, dtype=torch.bool, device=DEV)
    for lo, hi in zip(begin, begin[1:]):
        if 0 <= lo < hi <= 97:
            inside[lo:hi] = True
    assert (out[~inside] == 7.0).all()
    if all(x <= y for x, y in zip(begin, begin[1:])):
        _check(q, k, v, b, out, skip=[i for i, (lo, hi) in enumerate(zip(begin, begin[1:])) if lo < 0 or hi > 97])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1)])
def test_references_that_move(d, H, Hkv):
    """Logits that grow from tile to tile (each row's reference moves again and again), fall, and jump once."""
    n = 700
    q, k, v, begin, out = _inputs([n, n, n], H, Hkv, d, torch.float16)
    q[:] = 0
    q[..., 0] = 4.0
    k[:, :, 0] = torch.cat([torch.arange(n) / 4.0, -torch.arange(n) / 4.0, torch.where(torch.arange(n) == 333, 100.0, 0.0)]).to(DEV)[:, None].half()
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=0.5)
    _check(q, k, v, begin, out, scale=0.5)


def test_slopes_of_any_sign():
    """Biases that grow with the distance make the references move with every tile."""
    H = 4
    slopes = torch.tensor([-0.5, -2.0, 0.0, 3.0], device=DEV)
    for d in (64, 128, 256):
        q, k, v, begin, out = _inputs([700, 130], H, 2, d, torch.bfloat16)
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, bias_mode=1, alibi_slopes_dev=slopes)
        _check(q, k, v, begin, out, slopes)


def test_a_very_long_sequence():
    """150000 tokens: no wait runs out, and rows of every part are right."""
    n, H, d = 150000, 2, 64
    q, k, v, begin, out = _inputs([n], H, 1, d, torch.bfloat16)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    for i in (0, 127, 128, 40000, 65535, 65536, 99999, n - 2, n - 1):
        want, weighted, size = ref.attend_rows(q[i:i + 1].double(), k[:i + 1].double(), v[:i + 1].double(), 1 / math.sqrt(d), causal=False)
        assert ((out[i:i + 1].double() - want).abs() <= ref.bound(want, weighted, size, out.dtype, d, True)).all(), i
    assert torch.isfinite(out).all()


def test_nothing_to_do():
    q, k, v, _, out = _inputs([50], 4, 2, 128, torch.float16)
    for begin in ([0, 0], [50, 50, 50], [7] * 300):
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=torch.tensor(begin, device=DEV, dtype=torch.int32), out=out)
    torch.cuda.synchronize()
    assert (out == 7.0).all()


@pytest.mark.parametrize("dtype,exponent", [("fp16", 20), ("bf16", 30)])
def test_many_small_weights_count(dtype, exponent):
    """One key with weight 1 and 4000 with 2^-20 or 2^-30: a weight that stands far below the largest is not dropped."""
    n, d = 4001, 64
    q, k, v, begin, out = _inputs([n], 1, 1, d, TYPES[dtype])
    q[:], k[:] = 0, 0
    q[..., 0], k[1:, :, 0] = 1.0, -exponent
    v[:], v[1:] = 0, 1000.0
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, logit_scale=math.log(2.0))
    small = 1000.0 * 4000 * 2.0 ** -exponent
    assert float((out[-1].float() - small).abs().max()) <= small * (4000 * 2.0 ** -exponent + 2 * torch.finfo(out.dtype).eps)


def test_a_wait_that_runs_out_makes_the_rows_nan():
    for d in (64, 256):
        q, k, v, begin, out = _inputs([40, 300], 2, 1, d, torch.float16, behind=4)
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, debug_fail_first_wait=1)
        assert torch.isnan(out[:340]).all() and (out[340:] == 7.0).all()
        _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
        _check(q, k, v, begin, out)


def test_a_wait_that_runs_out_with_many_places():
    """More places than CTAs run at once: those that are claimed after the failure are NaN too."""
    lengths = [(13 * i) % 300 for i in range(200)]
    q, k, v, begin, out = _inputs(lengths, 8, 2, 128, torch.bfloat16)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, debug_fail_first_wait=1)
    assert torch.isnan(out).all()
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    _check(q, k, v, begin, out)


@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 4), (128, 12, 4), (256, 8, 4)])
def test_calls_of_many_items(d, H, Hkv):
    """Several items for every CTA, of every length: what one leaves behind does not reach the next."""
    lengths = [(37 * i) % 400 for i in range(150)]
    q, k, v, begin, out = _inputs(lengths, H, Hkv, d, torch.float16, "heads")
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    first = out.clone()
    _check(q, k, v, begin, out)
    out.fill_(7.0)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    assert torch.equal(first, out)              # whoever claims what, the same bits


def test_many_sequences():
    lengths = [(7 * i) % 5 for i in range(3000)]
    q, k, v, begin, out = _inputs(lengths, 2, 1, 64, torch.float16)
    _kf().kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    b = begin.tolist()
    sample = [i for i in range(3000) if i % 97 < 3]
    for i in sample:
        if lengths[i]:
            _check(q[b[i]:b[i + 1]], k[b[i]:b[i + 1]], v[b[i]:b[i + 1]], torch.tensor([0, lengths[i]]), out[b[i]:b[i + 1]])


def test_other_streams_and_captured():
    q, k, v, begin, out = _inputs([100, 57, 300], 4, 2, 128, torch.bfloat16)
    kf, side, other = _kf(), torch.cuda.Stream(), torch.cuda.Stream()
    out2 = torch.full_like(out, 7.0)
    torch.cuda.synchronize()
    kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out, stream=side)      # two calls at once
    kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out2, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    # other values and other ranges, replayed
    q2, k2, v2, _, _ = _inputs([100, 57, 300], 4, 2, 128, torch.bfloat16, seed=5)
    for a, b in ((q, q2), (k, k2), (v, v2)):
        a.copy_(b)
    begin.copy_(torch.tensor([0, 11, 11, 400]))
    out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    _check(q, k, v, begin, out)


def test_as_the_prompt_attention_of_one_length():
    """Prompts of one length: what kf_prefill_attend computes from the same rows, within both calls' roundings."""
    B, H, n, d = 2, 4, 384, 128
    q, k, v, begin, out = _inputs([n] * B, H, H, d, torch.float16, "fused")
    kf = _kf()
    ctx = kf.Keyformer(n_layers=1, batch=B, n_heads=H, head_dim=d, budget_k=64, recent_w=16, max_prompt_len=n, gen_len_T=4)
    major = [x.reshape(B, n, H, d).transpose(1, 2).contiguous() for x in (q, k, v)]
    there = torch.empty(B, H, n, d, device=DEV, dtype=torch.float16)
    ctx.kf_prefill_attend(*major, there)
    kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=begin, out=out)
    want, weighted, size = ref.attend_rows(q[:n].double(), k[:n].double(), v[:n].double(), 1 / math.sqrt(d))
    error = (out[:n].float() - there[0].transpose(0, 1).float()).abs()
    assert (error <= 2 * ref.bound(want, weighted, size, torch.float16, d, True)).all()


def test_refusals_on_a_device():
    kf = _kf()
    q, k, v, begin, out = _inputs([10], 2, 1, 64, torch.float16)
    call = lambda **kw: kf.kf_prefill_attend_ragged(**{**dict(q=q, k=k, v=v, begin=begin, out=out), **kw})   # noqa: E731
    for bad in (dict(k=k.bfloat16()), dict(q=q.float()), dict(begin=begin.long()), dict(begin=begin[:1]), dict(begin=begin.cpu()), dict(out=out[:5]), dict(v=v[..., ::2]),
                dict(k=k[..., :32]), dict(out=out.float())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(k=torch.cat([k, k[:, :0]], 1).expand(10, 3, 64), v=v.expand(10, 3, 64)), dict(out=q), dict(k=k[:1].expand(10, 1, 64)), dict(logit_scale=-1.0), dict(bias_mode=1)):
        with pytest.raises(kf.KeyformerError) as e:
            call(**bad)
        assert e.value.code == kf.KF_EINVAL
    assert (out == 7.0).all()
