"""The operators on 8-bit pages against plain forms in 64 bits (tests/pages_reference.py)."""
import math

import numpy as np
import pytest
import torch

from tests import pages_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _kf():
    import paper_2403_09054_b200 as kf
    return kf


def _ints(v):
    return torch.tensor(v, device=DEV, dtype=torch.int32)


def _pool(pages, Hkv, page, d, seed=0, layers=None, powers=True):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    lead = (pages, Hkv, 2) if layers is None else (layers, pages, Hkv, 2)
    cache = torch.randint(-127, 128, (*lead, page, d), device=DEV, generator=gen, dtype=torch.int8)
    scale = torch.randint(-6, -3, lead, device=DEV, generator=gen).float() if powers else None
    scale = torch.pow(torch.tensor(2.0, device=DEV, dtype=torch.float64), scale.double()).float() if powers else 0.001 + torch.rand(lead, device=DEV, generator=gen) * 0.1
    return cache, scale


def _table(lengths, page, pages, seed=0, width=None):
    """Distinct pages in no order, -1 behind a sequence's last."""
    rng = np.random.default_rng(seed)
    order, at = rng.permutation(pages), 0
    width = width or max(1, max(-(-n // page) for n in lengths))
    t = np.full((len(lengths), width), -1, np.int32)
    for s, n in enumerate(lengths):
        m = -(-n // page)
        t[s, :m] = order[at:at + m]
        at += m
    assert at <= pages
    return t


# ------------------------------------------------------------------------------------------------ write and read

@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_rows_written_bit_by_bit(page, d, dtype):
    """Four sequences that grow by parts of any size, scales that grow now and then: codes and scales bit for bit, and everything else as it was."""
    Hkv, S, rng = 3, 4, np.random.default_rng(page + d)
    cache, scale = _pool(30, Hkv, page, d)
    table = _table([7 * page] * S, page, 30)
    want_c, want_s = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
    length = np.array([0, 1, page - 1, page + 3], np.int32)
    t_dev = _ints(table)
    for step in range(6):
        counts = rng.choice([0, 1, 2, page // 2, page, page + 1, 2 * page - 1], S)
        begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        T = max(1, begin[-1])
        x = torch.from_numpy(rng.standard_normal((2, T, Hkv, d)) * 2.0 ** rng.integers(-3, 4, (2, T, Hkv, 1))).to(DEV).to(TYPES[dtype])
        rows = torch.cat([x[0], x[1]], 1)                            # side by side
        _kf().kf_pages_write(k=rows[:, :Hkv], v=rows[:, Hkv:], begin=_ints(begin.tolist()), length=_ints(length.tolist()), table=t_dev, cache=cache, scale=scale)
        ref.write(want_c, want_s, table, length, x.double().cpu().numpy(), begin)
        np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
        np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
        length = np.minimum(length + counts, 7 * page).astype(np.int32)
    # and back, from any token on
    first = np.array([0, 1, 5, 0], np.int32)
    counts = np.maximum(0, length - first)
    begin = np.concatenate([[2], 2 + np.cumsum(counts)]).astype(np.int32)
    k = torch.full((Hkv, begin[-1] + 3, d), 5.0, device=DEV, dtype=TYPES[dtype]).transpose(0, 1)
    v = torch.full((begin[-1] + 3, Hkv, d), 5.0, device=DEV, dtype=TYPES[dtype])
    _kf().kf_pages_read(table=t_dev, cache=cache, scale=scale, k=k, v=v, begin=_ints(begin.tolist()), first=_ints(first.tolist()))
    for s in range(S):
        for side, got in enumerate((k, v)):
            want = torch.from_numpy(ref.held(want_c, want_s, table, s, int(length[s]))[side][first[s]:]).to(DEV).to(TYPES[dtype])
            assert torch.equal(got[begin[s]:begin[s + 1]], want)
    for got in (k, v):
        assert (got[:2] == 5.0).all() and (got[begin[-1]:] == 5.0).all()


@pytest.mark.parametrize("page,d", [(16, 64), (16, 128), (16, 256), (32, 128), (64, 64), (128, 128), (128, 256)])
@pytest.mark.parametrize("shift", [0, 8])
def test_many_pages_there_and_back_at_any_alignment(page, d, shift):
    """As many pages as fill the machine several times, in one call; rows that begin on 32 bytes or only on 16."""
    Hkv, lengths = 16, [2 * page * i + (i * 7) % page for i in range(1, 22)]
    T, pages = sum(lengths), sum(-(-n // page) for n in lengths)
    cache, scale = _pool(pages, Hkv, page, d)
    table = _ints(_table(lengths, page, pages))
    begin = _ints(np.cumsum([0] + lengths).tolist())
    x = torch.randn(2, T, Hkv, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(page + d)).half()

    def rows():
        return torch.full((2, T, Hkv, d + 16), 5.0, device=DEV, dtype=torch.float16)
    src, dst = rows(), rows()
    src[..., shift:shift + d] = x
    _kf().kf_pages_write(k=src[0, ..., shift:shift + d], v=src[1, ..., shift:shift + d], begin=begin, length=torch.zeros_like(begin[1:]), table=table, cache=cache, scale=scale)
    _kf().kf_pages_read(k=dst[0, ..., shift:shift + d], v=dst[1, ..., shift:shift + d], begin=begin, table=table, cache=cache, scale=scale)
    for s in range(0, len(lengths), 5):
        n, b = lengths[s], int(begin[s])
        for side in range(2):
            ids = table[s, :-(-n // page)].long()
            held = (cache[ids, :, side].double() * scale[ids, :, side].double()[..., None, None]).transpose(1, 2).flatten(0, 1)[:n]
            assert torch.equal(dst[side, b:b + n, :, shift:shift + d], held.half())
            per = torch.nn.functional.pad(x[side, b:b + n].double().abs().amax(-1).t(), (0, len(ids) * page - n)).view(Hkv, len(ids), page).amax(-1)
            step = torch.where(per > 0, scale[ids, :, side].double().t(), torch.zeros_like(per))
            assert (per <= 127 * step).all() and (per > 63.5 * step).all()                        # the smallest power of two that holds the page's rows
            off = (held - x[side, b:b + n].double()).abs().amax(-1).t()
            assert (torch.nn.functional.pad(off, (0, len(ids) * page - n)).view(Hkv, len(ids), page).amax(-1) <= step / 2).all()
    assert (dst[..., :shift] == 5.0).all() and (dst[..., shift + d:] == 5.0).all()


def test_one_row_per_sequence():
    page, d, Hkv, S = 16, 128, 8, 50
    cache, scale = _pool(200, Hkv, page, d)
    length = [(11 * i) % 49 for i in range(S)]
    table = _table([n + 1 for n in length], page, 200)
    x = torch.randn(2, S, Hkv, d, device=DEV).bfloat16()
    want_c, want_s = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
    _kf().kf_pages_write(k=x[0], v=x[1], length=_ints(length), table=_ints(table), cache=cache, scale=scale)
    ref.write(want_c, want_s, table, length, x.double().cpu().numpy(), list(range(S + 1)))
    np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)


@pytest.mark.parametrize("dtype,values", [("fp16", [65504.0, 2.0 ** -24, 0.0, -65504.0, 1.0, 6.1e-5]), ("bf16", [3.0e38, 1e-40, 0.0, -3.0e38, 127.0, 1e-30])])
def test_rows_of_extreme_values(dtype, values):
    """The largest and smallest numbers, zeros, and ties, one value per sequence."""
    S, page, d = len(values) + 1, 16, 64
    x = torch.tensor(values, device=DEV).to(TYPES[dtype])[:, None, None].expand(-1, 1, d).clone()
    ties = ((torch.arange(d, device=DEV) % 32 + 0.5) * (1 - 2 * (torch.arange(d, device=DEV) % 2))).to(TYPES[dtype])
    ties[0] = 127.0
    x = torch.cat([x, ties[None, None]])
    cache, scale = torch.zeros(S, 1, 2, page, d, device=DEV, dtype=torch.int8), torch.zeros(S, 1, 2, device=DEV)
    want_c, want_s = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
    table = np.arange(S, dtype=np.int32)[:, None]
    _kf().kf_pages_write(k=x, v=-x, length=_ints([0] * S), table=_ints(table), cache=cache, scale=scale)
    ref.write(want_c, want_s, table, [0] * S, torch.stack([x, -x]).double().cpu().numpy(), list(range(S + 1)))
    np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)


def test_rows_that_are_not_finite_spoil_their_page_head_and_side_alone():
    page, d, Hkv = 16, 64, 2
    cache, scale = _pool(4, Hkv, page, d)
    table, length = _ints([[0, 1], [2, 3]]), _ints([0, 0])
    x = torch.randn(2, 40, Hkv, d, device=DEV).half()
    x[0, 17, 1, 5] = float("nan")       # keys of head 1, second page of sequence 0
    x[1, 20, 0, 63] = -float("inf")     # values of head 0, first page of sequence 1
    _kf().kf_pages_write(k=x[0], v=x[1], begin=_ints([0, 20, 40]), length=length, table=table, cache=cache, scale=scale)
    bad = torch.zeros_like(scale, dtype=torch.bool)
    bad[1, 1, 0] = bad[2, 0, 1] = True
    assert torch.equal(torch.isnan(scale), bad)
    # a page that is spoilt stays so while it fills
    _kf().kf_pages_write(k=x[0, :2], v=x[1, :2], length=_ints([20, 20]), table=table, cache=cache, scale=scale)
    assert torch.equal(torch.isnan(scale), bad)
    # and is whole again when it is written from its start
    _kf().kf_pages_write(k=x[0, :2], v=x[1, :2], length=_ints([16, 0]), table=table, cache=cache, scale=scale)
    assert torch.isfinite(scale).all()


def test_rows_without_a_page_are_not_written():
    page, d, Hkv = 16, 64, 1
    cache, scale = _pool(6, Hkv, page, d)
    before = cache.clone(), scale.clone()
    table = _ints([[6, 0], [-1, 1], [2, -7], [3, 4], [5, 5]])
    x = torch.randn(2, 100, Hkv, d, device=DEV).half()
    # sequence 3 would run behind the table, sequence 4 has a negative length
    _kf().kf_pages_write(k=x[0], v=x[1], begin=_ints([0, 20, 40, 60, 80, 100]), length=_ints([0, 0, 0, 30, -1]), table=table, cache=cache, scale=scale)
    wanted = torch.zeros(6, page, dtype=torch.bool, device=DEV)
    wanted[0, :4] = wanted[1, :4] = True
    wanted[2, :] = True
    wanted[4, 14:] = True
    moved = (cache != before[0]).any(-1).any(1).any(1)              # [pages, page]
    assert not moved[3].any() and not moved[5].any() and not moved[0, 4:].any() and not moved[1, 4:].any() and moved[4, 14:].all() and moved[2].all()
    assert torch.equal(scale[[3, 5]], before[1][[3, 5]])
    out = torch.full((2, 64, Hkv, d), 5.0, device=DEV).half()
    _kf().kf_pages_read(table=table, cache=cache, scale=scale, k=out[0], v=out[1], begin=_ints([0, 20, 36, 44, 64, 64]), first=_ints([0, 0, -4, 30, 0]))
    nan = torch.isnan(out).all(-1).all(-1).all(0)
    assert nan.tolist() == [True] * 16 + [False] * 4 + [True] * 16 + [True] * 4 + [False] * 4 + [False] * 2 + [True] * 18


@pytest.mark.parametrize("begin", [[0, 30, 20, 40], [-3, 10, 20, 40], [0, 10, 20, 400], [40, 30, 20, 10], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 7]])
def test_row_ranges_that_are_not_valid(begin):
    page, d, Hkv = 16, 64, 1
    cache, scale = _pool(12, Hkv, page, d)
    table = _ints(np.arange(12).reshape(3, 4).tolist())
    x = torch.randn(2, 40, Hkv, d, device=DEV).half()
    b = torch.tensor(begin, device=DEV, dtype=torch.int64).to(torch.int32)
    out = torch.full((2, 40, Hkv, d), 5.0, device=DEV).half()
    _kf().kf_pages_read(table=table, cache=cache, scale=scale, k=out[0], v=out[1], begin=b)
    inside = torch.zeros(40, dtype=torch.bool, device=DEV)
    for lo, hi in zip(begin, begin[1:]):
        if 0 <= lo < hi <= 40:
            inside[lo:hi] = True
    assert (out[:, ~inside] == 5.0).all()
    _kf().kf_pages_write(k=x[0], v=x[1], begin=b, length=_ints([0, 0, 0]), table=table, cache=cache, scale=scale)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ attention

def _attend(q, table, lengths, cache, scale, slopes=None, logit=0.0, out=None, **kw):
    out = torch.full_like(q, 7.0) if out is None else out
    _kf().kf_pages_attend(q=q, table=_ints(table), length=_ints(lengths), cache=cache, scale=scale, out=out, bias_mode=0 if slopes is None else 1, alibi_slopes_dev=slopes,
                          logit_scale=logit, **kw)
    return out


def _check(out, q, table, lengths, cache, scale, slopes=None, logit=None, only=None):
    d, c, s = q.shape[2], cache.cpu().numpy(), scale.cpu().numpy()
    for i, n in enumerate(lengths):
        if only is not None and i not in only:
            continue
        if n == 0:
            assert (out[i] == 0).all()
            continue
        k, v = torch.from_numpy(ref.held(c, s, table, i, n)).to(DEV)
        want, weighted, size = ref.attend_rows(q[i:i + 1].double(), k, v, 1 / math.sqrt(d) if logit is None else logit, slopes, causal=False)
        unit = torch.from_numpy(s[table[i]][np.arange(n) // c.shape[3], :, 1].astype(np.float64)).to(DEV)                # [n, Hkv]
        floor = ref.weight_floor(q[i:i + 1].double(), k, 1 / math.sqrt(d) if logit is None else logit, slopes, unit)
        error, limit = (out[i:i + 1].double() - want).abs(), ref.bound(want, weighted, size, out.dtype, d, False) + floor
        assert (error <= limit).all(), (i, n, float((error / limit).max()))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("H,Hkv,dtype,alibi", [(3, 3, "fp16", False), (8, 4, "bf16", True), (5, 1, "fp16", True), (16, 2, "bf16", False), (16, 1, "fp16", False), (20, 1, "bf16", True)])
def test_attention_over_pages(d, page, H, Hkv, dtype, alibi):
    lengths = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 0, 127, 128, 129, 500, 1025]
    pages = sum(-(-n // page) for n in lengths) + 3
    cache, scale = _pool(pages, Hkv, page, d, powers=not alibi)
    table = _table(lengths, page, pages)
    q = torch.randn(len(lengths), H, d, device=DEV).to(TYPES[dtype])
    slopes = torch.exp2(-8.0 * torch.arange(1, H + 1, device=DEV) / H) if alibi else None
    out = _attend(q, table, lengths, cache, scale, slopes)
    _check(out, q, table, lengths, cache, scale, slopes)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("H,Hkv,dtype,alibi", [(4, 4, "bf16", True), (16, 2, "fp16", False), (12, 1, "bf16", False)])
def test_short_sequences_of_few_caches(d, page, H, Hkv, dtype, alibi):
    """Tables with room for a few tiles only: a CTA takes all of a sequence and cache."""
    lengths = [0, 1, 15, 16, 17, 33, 64, 100, 127, 128, 255, 256]
    if d > 64 and page < 128:
        lengths += [200, 3]
    pages = sum(-(-n // page) for n in lengths) + 3
    cache, scale = _pool(pages, Hkv, page, d)
    table = _table(lengths, page, pages)
    q = torch.randn(len(lengths), H, d, device=DEV).to(TYPES[dtype])
    slopes = torch.exp2(-8.0 * torch.arange(1, H + 1, device=DEV) / H) if alibi else None
    out = _attend(q, table, lengths, cache, scale, slopes)
    _check(out, q, table, lengths, cache, scale, slopes)
    # a wider table takes the other form, which splits sequences: the same within both roundings
    wide = np.concatenate([table, np.full((len(lengths), 40), -1, np.int32)], 1)
    _check(_attend(q, wide, lengths, cache, scale, slopes), q, wide, lengths, cache, scale, slopes)


def test_one_token_is_its_value_row():
    cache, scale = _pool(3, 2, 16, 128)
    q = torch.randn(1, 4, 128, device=DEV).half()
    out = _attend(q, [[2]], [1], cache, scale)
    assert torch.equal(out[0], (cache[2, :, 1, 0].float() * scale[2, :, 1, None]).half().repeat_interleave(2, 0))


@pytest.mark.parametrize("S,H,Hkv,page,d,longest", [(1, 32, 4, 16, 128, 40000), (2, 8, 8, 64, 64, 9999), (1, 2, 2, 128, 256, 20001), (300, 4, 2, 16, 64, 300), (700, 1, 1, 32, 128, 40)])
def test_long_and_many(S, H, Hkv, page, d, longest):
    """One long sequence cut over the whole GPU; more sequences than a CTA has threads."""
    lengths = [longest * ((37 * i + 63) % 64) // 63 for i in range(S)]
    pages = sum(-(-n // page) for n in lengths) + 1
    cache, scale = _pool(pages, Hkv, page, d)
    table = _table(lengths, page, pages)
    q = torch.randn(S, H, d, device=DEV).bfloat16()
    out = _attend(q, table, lengths, cache, scale)
    _check(out, q, table, lengths, cache, scale, only=None if S < 10 else set(range(0, S, 37)))
    for i, n in enumerate(lengths):
        assert n > 0 or (out[i] == 0).all()


def test_a_cache_beyond_32_bits():
    """4.5 GB of pages, the sequence in the last ones."""
    page, d, Hkv = 128, 128, 16
    pages = 8700
    cache = torch.zeros(pages, Hkv, 2, page, d, device=DEV, dtype=torch.int8)
    assert cache.numel() > 2 ** 32
    scale = torch.full((pages, Hkv, 2), 0.03125, device=DEV)
    cache[-3:] = _pool(3, Hkv, page, d)[0]
    n = 300
    table = [[pages - 1, pages - 3, pages - 2]]
    q = torch.randn(1, Hkv, d, device=DEV).half()
    out = _attend(q, table, [n], cache, scale)
    local = [[2, 0, 1]]
    _check(out, q, np.array(local), [n], cache[-3:], scale[-3:])
    x = torch.randn(2, 1, Hkv, d, device=DEV).half()
    _kf().kf_pages_write(k=x[0], v=x[1], length=_ints([n]), table=_ints(table), cache=cache, scale=scale)
    back = torch.zeros(2, 1, Hkv, d, device=DEV).half()
    _kf().kf_pages_read(table=_ints(table), cache=cache, scale=scale, k=back[0], v=back[1], begin=_ints([0, 1]), first=_ints([n]))
    assert float((back - x).abs().max()) <= float(scale[-2:].max()) / 2


@pytest.mark.parametrize("page", [16, 64])
def test_scales_that_differ_from_page_to_page(page):
    """V scales from 2^-20 to 2^8 and zero, and K scales that make a page's logits tower over the others: small pages with large weights and large
    pages with small weights both count."""
    d, Hkv, n = 64, 2, 900
    pages = -(-n // page)
    for order in (1, -1):
        cache, scale = _pool(pages, Hkv, page, d)
        steps = torch.arange(pages, device=DEV)
        towers = torch.exp2(((steps * 5) % 29 - 20).float())
        scale[:, :, 1] = (towers if order > 0 else towers.flip(0))[:, None]
        scale[3, :, 1] = 0.0
        scale[:, 0, 0] = torch.exp2((steps % 7 - 9).float())
        table = _table([n], page, pages)
        q = torch.randn(1, 8, d, device=DEV).half()
        out = _attend(q, table, [n], cache, scale)
        _check(out, q, table, [n], cache, scale)
    scale[:, :, 1] = 2.0 ** -120                                # pages that hold zeros: nothing overflows
    cache[:, :, 1] = 0
    assert (_attend(q, table, [n], cache, scale) == 0).all()


def test_queries_of_every_size():
    """bfloat16 queries far outside binary16, and zeros."""
    d, page = 128, 32
    cache, scale = _pool(8, 1, page, d)
    table = _table([200], page, 8)
    q = torch.randn(1, 4, d, device=DEV)
    q[0, 0] *= 1e30
    q[0, 1] *= 1e-30
    q[0, 2] = 0
    q = q.bfloat16()
    for logit in (1e-30, 1.0):
        heads = [0, 2, 3] if logit < 1 else [1, 2]
        out = _attend(q, table, [200], cache, scale, logit=logit)
        _check(out[:, heads], q[:, heads], table, [200], cache, scale, logit=logit)


def test_what_is_not_the_sequences_reaches_no_output():
    """Scales of pages that belong to others are NaN, unused rows hold anything."""
    page, d = 32, 128
    cache, scale = _pool(12, 2, page, d)
    lengths = [33, 0, 64, 5]
    table = _table(lengths, page, 12, width=4)
    want = _attend(torch.ones(4, 2, d, device=DEV).half(), table, lengths, cache, scale)
    used = set(table[table >= 0].tolist())
    for p in range(12):
        if p not in used:
            scale[p] = float("nan")
    table[table < 0] = [p for p in range(12) if p not in used][0]
    for s, n in enumerate(lengths):
        if n % page:
            cache[table[s, n // page], :, :, n % page:] = -128
    assert torch.equal(want, _attend(torch.ones(4, 2, d, device=DEV).half(), table, lengths, cache, scale))


@pytest.mark.parametrize("page", [16, 64])
def test_missing_pages_and_lengths_that_are_not_valid_give_nan(page):
    d, n = 64, 200
    width = -(-n // page)
    cache, scale = _pool(8 * width, 2, page, d)
    lengths = [n] * 8
    table = _table(lengths, page, 8 * width)
    q = torch.randn(8, 4, d, device=DEV).half()
    lengths[1], lengths[2], lengths[3] = -1, width * page + 1, 2 ** 31 - 1
    table[4, 0], table[5, width - 1], table[6, 1] = -1, 8 * width, 2 ** 31 - 1
    out = _attend(q, table, lengths, cache, scale)
    assert torch.isnan(out[1:7]).all()
    _check(out, q, table, lengths, cache, scale, only={0, 7})
    scale[table[7, 1], 1, 1] = float("nan")                     # values of one head
    out = _attend(q, table, lengths, cache, scale)
    assert torch.isnan(out[7, 2:]).all() and torch.isfinite(out[7, :2]).all()


def test_strides():
    d, page = 128, 16
    lengths = [70, 5, 300]
    cache, scale = _pool(30, 2, page, d)
    table = _table(lengths, page, 30)
    wide = torch.randn(6, 9, d + 8, device=DEV).half()
    q = wide[::2, 1:9:2, :d]
    out = torch.full((4, 3, d), 7.0, device=DEV).half().transpose(0, 1)
    _attend(q, table, lengths, cache, scale, out=out)
    _check(out, q, table, lengths, cache, scale)


def test_a_wait_that_runs_out_makes_the_output_nan():
    cache, scale = _pool(100, 2, 16, 64)
    lengths = [700, 0, 3]
    table = _table(lengths, 16, 100)
    q = torch.randn(3, 4, 64, device=DEV).half()
    for width in (table.shape[1], 10):                          # both forms
        lengths[0] = min(lengths[0], 16 * width)
        part = np.ascontiguousarray(table[:, :width])
        out = _attend(q, part, lengths, cache, scale, debug_fail_first_wait=1)
        assert torch.isnan(out[[0, 2]]).all() and (out[1] == 0).all()
        _check(_attend(q, part, lengths, cache, scale), q, part, lengths, cache, scale)


def test_attention_on_streams_with_scratch_of_any_content_and_captured():
    lengths = [2000, 17, 900, 1]
    cache, scale = _pool(200, 2, 16, 128)
    table = _table(lengths, 16, 200)
    q = torch.randn(4, 8, 128, device=DEV).bfloat16()
    t, n, kf = _ints(table), _ints(lengths), _kf()
    outs = [torch.full_like(q, 7.0) for _ in range(3)]
    need = kf.kf_pages_attend_scratch_bytes(sequences=4, table_width=table.shape[1], n_pages=200, page_tokens=16, n_heads=8, n_kv_heads=2, head_dim=128)
    scratch = torch.full((need,), 255, device=DEV, dtype=torch.uint8)
    torch.cuda.synchronize()
    kf.kf_pages_attend(q=q, table=t, length=n, cache=cache, scale=scale, out=outs[0], stream=torch.cuda.Stream())
    kf.kf_pages_attend(q=q, table=t, length=n, cache=cache, scale=scale, out=outs[1], scratch=scratch, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kf.kf_pages_attend(q=q, table=t, length=n, cache=cache, scale=scale, out=outs[2], scratch=scratch)
    lengths = [1999, 2, 0, 1]                                    # replayed with other lengths: nothing of them is kept from the capture
    n.copy_(_ints(lengths))
    scratch.fill_(255)
    graph.replay()
    torch.cuda.synchronize()
    _check(outs[2], q, table, lengths, cache, scale)
    with pytest.raises(kf.KeyformerError) as e:
        kf.kf_pages_attend(q=q, table=t, length=n, cache=cache, scale=scale, out=outs[2], scratch=scratch[:need - 256])
    assert e.value.code == kf.KF_ENOSPC


# ------------------------------------------------------------------------------------------------ tables

def _update_case(S, W, page, pages, layers, Hkv, d, parent, length, grow, seed=0, pins=(), table=None):
    cache, scale = _pool(pages, Hkv, page, d, layers=layers, seed=seed)
    if table is None:
        table = _table([min(max(n, 0), W * page) for n in length], page, pages, width=W)
    refs = np.zeros(pages, np.int32)
    for p in table[table >= 0]:
        refs[p] += 1
    for p in pins:
        refs[p % pages] += 1
    dev = [_ints(table), _ints(length), torch.from_numpy(refs).to(DEV)]
    missing = _ints([-5])
    want = [table.copy(), np.array(length, np.int32), refs.copy()]
    want_c, want_s = cache.cpu().numpy(), scale.cpu().numpy()
    parents = list(range(S)) if parent is None else parent
    grows = [grow] * S if isinstance(grow, int) else grow
    want_missing = ref.update(*want, parents, grows, page, want_c, want_s)
    kw = dict(grow=grow if isinstance(grow, int) else _ints(grow))
    _kf().kf_pages_update(table=dev[0], length=dev[1], refs=dev[2], cache=cache, scale=scale, missing=missing, parent=None if parent is None else _ints(parent), **kw)
    for got, name, w in zip(dev, ("table", "length", "refs"), want):
        np.testing.assert_array_equal(got.cpu().numpy(), w, err_msg=name)
    assert int(missing) == want_missing
    np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
    return dev, cache, scale


@pytest.mark.parametrize("seed", range(12))
def test_updates_of_any_kind(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([16, 32, 64, 128]))
    S, W = int(rng.choice([1, 2, 7, 40])), int(rng.choice([2, 5, 9]))
    length = rng.integers(0, W * page + 1, S).tolist()
    pages = S * W + int(rng.choice([1, 30, 5000]))
    parent = rng.integers(-1, S, S).tolist() if seed % 4 else rng.integers(-3, S + 2, S).tolist()
    grow = rng.integers(-2, page * 2, S).tolist()
    _update_case(S, W, page, pages, int(rng.choice([1, 3])), int(rng.choice([1, 3])), 64, parent, length, grow, seed, pins=[0, 3, pages - 1])


def test_repeated_updates_keep_the_counts():
    """Twenty steps of a beam search with sequences that end and begin again: no page is lost or used twice."""
    S, W, page, pages = 12, 8, 16, 80
    rng = np.random.default_rng(5)
    length = rng.integers(0, 60, S).tolist()
    dev, cache, scale = _update_case(S, W, page, pages, 2, 2, 64, None, length, 1)
    table, n, refs = (x.cpu().numpy().copy() for x in dev)
    for step in range(20):
        parent = np.where(rng.random(S) < 0.15, -1, rng.integers(0, S, S)).tolist()
        grow = rng.integers(0, 20, S).tolist()
        want_c, want_s = cache.cpu().numpy(), scale.cpu().numpy()
        missing = _ints([0])
        want = ref.update(table, n, refs, parent, grow, page, want_c, want_s)
        _kf().kf_pages_update(table=dev[0], length=dev[1], refs=dev[2], cache=cache, scale=scale, missing=missing, parent=_ints(parent), grow=_ints(grow))
        for got, w in zip(dev, (table, n, refs)):
            np.testing.assert_array_equal(got.cpu().numpy(), w)
        assert int(missing) == want
        np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
        count = np.bincount(table[table >= 0], minlength=pages)
        np.testing.assert_array_equal(count, refs)
        # tokens arrive where there is room for them
        room = np.array([sum(1 for _ in __import__("itertools").takewhile(lambda p: p >= 0, row)) * page for row in table])
        n = np.minimum(np.minimum(n + np.array(grow), room), 100).astype(np.int32)
        dev[1].copy_(_ints(n))


def test_no_free_page_is_reported():
    dev, _, _ = _update_case(3, 4, 16, 6, 1, 1, 64, [0, 0, 0], [40, 16, 30], 30)     # ten pages wanted, four of six free
    assert (dev[0] == -1).any()


def test_a_table_that_is_too_narrow_is_reported():
    _update_case(2, 2, 16, 10, 1, 1, 64, None, [32, 20], [2 ** 31 - 1, 33])


def test_pages_that_are_pinned_are_never_handed_out():
    _update_case(2, 4, 16, 9, 1, 1, 64, [-1, -1], [20, 40], 60, pins=[0, 1, 2, 5])


def test_lengths_and_entries_that_are_not_valid():
    table = np.array([[0, 1, 99], [2, -1, -1], [-7, 3, 4], [5, 2 ** 31 - 1, 6]], np.int32)
    table[table > 9] = -1
    _update_case(4, 3, 16, 10, 2, 1, 64, [3, 0, 0, 2], [47, -9, 40, 100], 5, table=table)


def test_a_copy_of_a_page_that_is_missing_reads_as_nan():
    table = np.array([[0, -1], [2, -1]], np.int32)
    _, _, scale = _update_case(2, 2, 16, 8, 1, 2, 64, [0, 0], [20, 3], 0, table=table)
    assert torch.isnan(scale).sum() == 4


@pytest.mark.parametrize("S,W,pages", [(3000, 3, 20003), (8192, 1, 8195), (5, 4000, 70001)])
def test_large_tables(S, W, pages):
    rng = np.random.default_rng(S)
    length = rng.integers(0, W * 16 + 1, S).tolist() if S > 10 else [10, 60000, 17, 0, 30]
    _update_case(S, W, 16, pages, 1, 1, 64, rng.integers(-1, S, S).tolist(), length, 1)


def test_more_pages_at_once_than_one_cta_lists():
    _update_case(1, 12000, 16, 14000, 1, 1, 64, None, [100], 11000 * 16)


def test_a_row_of_calls_without_a_pause():
    """Launches begin behind the ones before: what a call wrote is there for the next, and nothing is overwritten that one before still reads."""
    kf, S, Hkv, d, page, W = _kf(), 6, 2, 64, 16, 20
    cache, scale = torch.zeros(S * W, Hkv, 2, page, d, device=DEV, dtype=torch.int8), torch.zeros(S * W, Hkv, 2, device=DEV)
    table, length = torch.full((S, W), -1, device=DEV, dtype=torch.int32), torch.zeros(S, device=DEV, dtype=torch.int32)
    refs, missing = torch.zeros(S * W, device=DEV, dtype=torch.int32), _ints([0])
    x = torch.randn(40, 2, S, Hkv, d, device=DEV).half()
    q, out = torch.randn(40, S, 4, d, device=DEV).half(), torch.zeros(40, S, 4, d, device=DEV).half()
    for step in range(40):
        kf.kf_pages_update(table=table, length=length, refs=refs, cache=cache, scale=scale, missing=missing, grow=1)
        kf.kf_pages_write(k=x[step, 0], v=x[step, 1], length=length, table=table, cache=cache, scale=scale)
        length.add_(1)
        kf.kf_pages_attend(q=q[step], table=table, length=length, cache=cache, scale=scale, out=out[step])
    want_c, want_s = np.zeros(cache.shape, np.int8), np.zeros(scale.shape, np.float32)
    t = table.cpu().numpy()
    for step in range(40):
        ref.write(want_c, want_s, t, [step] * S, x[step].double().cpu().numpy(), list(range(S + 1)))
        if step % 13 == 0 or step == 39:
            _check(out[step], q[step], t, [step + 1] * S, torch.from_numpy(want_c), torch.from_numpy(want_s))
    np.testing.assert_array_equal(cache.cpu().numpy(), want_c)


def test_updates_replayed():
    """One captured update steps a beam search on."""
    S, W, page, pages = 4, 6, 16, 64
    dev, cache, scale = _update_case(S, W, page, pages, 1, 1, 64, None, [5, 20, 31, 32], 1)
    table, n, refs = (x.cpu().numpy().copy() for x in dev)
    parent, missing = _ints([0, 0, 2, 2]), _ints([0])
    kf, graph = _kf(), torch.cuda.CUDAGraph()
    scratch = torch.full((kf.kf_pages_update_scratch_bytes(sequences=S, table_width=W, n_pages=pages, page_tokens=page, n_kv_heads=1, head_dim=64),), 255, device=DEV, dtype=torch.uint8)
    with torch.cuda.graph(graph):
        kf.kf_pages_update(table=dev[0], length=dev[1], refs=dev[2], cache=cache, scale=scale, missing=missing, parent=parent, grow=1, scratch=scratch)
        dev[1].add_(1)
    for step in range(5):
        want_c, want_s = cache.cpu().numpy(), scale.cpu().numpy()
        ref.update(table, n, refs, [0, 0, 2, 2] if step < 3 else [1, 1, 3, -1], [1] * S, page, want_c, want_s)
        if step == 3:
            parent.copy_(_ints([1, 1, 3, -1]))
        graph.replay()
        n = n + 1
        for got, w in zip(dev, (table, n, refs)):
            np.testing.assert_array_equal(got.cpu().numpy(), w)
        np.testing.assert_array_equal(cache.cpu().numpy(), want_c)


# ------------------------------------------------------------------------------------------------ compact

@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_compact(page, d):
    rng, Hkv = np.random.default_rng(page + d), 3
    lengths = [0, 1, 5, page, 3 * page + 1, 400]
    kept = [0, 1, 3, page, page + 1, 333]
    pages = sum(-(-n // page) for n in lengths + kept) + 2
    cache, scale = _pool(pages, Hkv, page, d)
    both = _table(lengths + kept, page, pages)
    table, new = both[:6], both[6:]
    keep = np.full((6, Hkv, 340), 2 ** 30, np.int32)
    for s in range(6):
        for h in range(Hkv):
            keep[s, h, :kept[s]] = np.sort(rng.permutation(lengths[s])[:kept[s]]) if h else rng.permutation(lengths[s])[:kept[s]]     # any order
    want_c, want_s = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
    old_c, old_s = want_c.copy(), want_s.copy()
    for s in range(6):
        for j0 in range(0, kept[s], page):
            p = new[s, j0 // page]
            for h in range(Hkv):
                at = keep[s, h, j0:min(j0 + page, kept[s])]
                source = table[s, at // page]
                top = old_s[source, h].max(0)                                   # [2]
                want_s[p, h] = top
                want_c[p, h, :, :len(at)] = np.rint(old_c[source, h, :, at % page] * (old_s[source, h] / top)[..., None]).transpose(1, 0, 2)
    _kf().kf_pages_compact(cache=cache, scale=scale, table=_ints(table), length=_ints(lengths), keep=_ints(keep), n_keep=_ints(kept), new_table=_ints(new))
    np.testing.assert_array_equal(cache.cpu().numpy(), want_c)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)


def test_compact_of_what_is_not_there():
    page, d, Hkv = 16, 64, 1
    cache, scale = _pool(12, Hkv, page, d)
    before = cache.clone()
    table, new = _ints([[0, 1], [2, -1], [3, 4]]), _ints([[5, 6], [7, -1], [12, 8]])
    keep = torch.arange(20, device=DEV, dtype=torch.int32).expand(3, 1, 20).contiguous()
    keep[0, 0, 3] = 32            # behind the sequence
    keep[0, 0, 17] = -1
    _kf().kf_pages_compact(cache=cache, scale=scale, table=table, length=_ints([32, 32, 32]), keep=keep, n_keep=_ints([18, 20, 99]), new_table=new)
    assert torch.isnan(scale[5]).all() and torch.isnan(scale[6]).all() and torch.isfinite(scale[[7, 8]]).all()       # tokens 16 .. of sequence 1 have no new page
    assert torch.equal(cache[:5], before[:5]) and torch.equal(cache[9:], before[9:]) and torch.equal(cache[8, :, :, 4:], before[8, :, :, 4:])
    assert torch.isfinite(scale[:5]).all() and torch.isfinite(scale[9:]).all()


# ------------------------------------------------------------------------------------------------ all of them together

def test_a_server_with_prompts_beams_and_a_reduced_cache():
    """Prompts of different lengths: norm and rotation, attention, pages; the positions that the prompt phase kept, compacted to half; beams forked;
    three generated tokens over the pages.  Every output against 64 bits on the values that the pages hold."""
    kf, H, Hkv, d, page = _kf(), 8, 4, 128, 16
    lengths, S, W, pages = [61, 130, 97, 128], 4, 12, 120
    T, gen = sum(lengths), torch.Generator(device=DEV).manual_seed(3)
    begin = [sum(lengths[:i]) for i in range(S + 1)]
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=gen)   # noqa: E731
    cache, scale = torch.zeros(pages, Hkv, 2, page, d, device=DEV, dtype=torch.int8), torch.zeros(pages, Hkv, 2, device=DEV)
    table, length, refs, missing = torch.full((S, W), -1, device=DEV, dtype=torch.int32), _ints([0] * S), torch.zeros(pages, device=DEV, dtype=torch.int32), _ints([0])
    state = dict(table=table, length=length, refs=refs, cache=cache, scale=scale, missing=missing)

    # prompts
    kf.kf_pages_update(**state, grow=_ints(lengths))
    q, k, v = (torch.empty(1, h, T, d, device=DEV, dtype=torch.float16) for h in (H, Hkv, Hkv))
    positions = torch.cat([torch.arange(n) for n in lengths]).int().to(DEV)[None]
    kf.kf_qk_norm_rotate(qkv=normal(1, T, (H + 2 * Hkv) * d).half(), n_heads=H, n_kv_heads=Hkv, head_dim=d, q=q, k=k, v=v, positions=positions, norm_mode=kf.KF_NORM_RMS, rotary_dims=64)
    q, k, v = (x[0].transpose(0, 1) for x in (q, k, v))
    out = torch.empty(T, H, d, device=DEV, dtype=torch.float16)
    kf.kf_prefill_attend_ragged(q=q, k=k, v=v, begin=_ints(begin), out=out)
    kf.kf_pages_write(k=k, v=v, begin=_ints(begin), length=length, table=table, cache=cache, scale=scale)
    length.add_(_ints(lengths))
    for i in range(S):
        rows = slice(begin[i], begin[i + 1])
        want, weighted, size = ref.attend_rows(q[rows].double(), k[rows].double(), v[rows].double(), 1 / math.sqrt(d))
        assert ((out[rows].double() - want).abs() <= ref.bound(want, weighted, size, torch.float16, d, True)).all()
    held = ref.held(cache.cpu().numpy(), scale.cpu().numpy(), table.cpu().numpy(), 1, 130)
    assert np.abs(held - torch.stack([k[begin[1]:begin[2]], v[begin[1]:begin[2]]]).double().cpu().numpy()).max() <= float(scale.max()) / 2

    # the prompt of sequence 3 reduced to what the method keeps, and put in its place
    ctx = kf.Keyformer(n_layers=1, batch=1, n_heads=H, n_kv_heads=Hkv, head_dim=d, budget_k=64, recent_w=16, max_prompt_len=128, gen_len_T=8)
    ctx.kf_prefill_score_prune(0, *(x[begin[3]:begin[4]].transpose(0, 1).contiguous() for x in (q, k, v)))
    pos = ctx.kf_view_state(0)[2][0].contiguous()                             # [Hkv, 64], ascending
    assert ctx.kf_poll_error() == 0
    new_table = _ints([[i for i in range(pages) if int(refs[i]) == 0][:4]])
    refs[new_table[0].long()] = 1                                              # the caller's own
    kf.kf_pages_compact(cache=cache, scale=scale, table=table[3:], length=length[3:], keep=pos[None].contiguous(), n_keep=_ints([64]), new_table=new_table)
    refs[table[3][table[3] >= 0].long()] -= 1
    table[3] = -1
    table[3, :4] = new_table[0]
    length[3] = 64
    kept = ref.held(cache.cpu().numpy(), scale.cpu().numpy(), table.cpu().numpy(), 3, 64)
    rows = torch.stack([torch.stack([x[begin[3]:begin[4]][pos[h].long(), h] for h in range(Hkv)], 1) for x in (k, v)]).double().cpu().numpy()
    assert np.abs(kept - rows).max() <= float(scale.max())                    # half a step when written, half a step when moved

    # three tokens; in the second step sequence 1 ends and goes on from sequence 0, in the third sequence 2 does
    for step, parent in enumerate(([0, 1, 2, 3], [0, 0, 2, 3], [1, 0, 0, 3])):
        kf.kf_pages_update(**state, parent=_ints(parent), grow=1)
        assert int(missing) == 0
        q, k, v = (torch.empty(S, h, 1, d, device=DEV, dtype=torch.float16) for h in (H, Hkv, Hkv))
        kf.kf_qk_norm_rotate(qkv=normal(S, 1, (H + 2 * Hkv) * d).half(), n_heads=H, n_kv_heads=Hkv, head_dim=d, q=q, k=k, v=v, positions=length[:, None].contiguous(),
                             norm_mode=kf.KF_NORM_RMS, rotary_dims=64)
        kf.kf_pages_write(k=k[:, :, 0], v=v[:, :, 0], length=length, table=table, cache=cache, scale=scale)
        length.add_(1)
        out = torch.empty(S, H, d, device=DEV, dtype=torch.float16)
        kf.kf_pages_attend(q=q[:, :, 0], table=table, length=length, cache=cache, scale=scale, out=out)
        _check(out, q[:, :, 0], table.cpu().numpy(), length.tolist(), cache, scale)
        count = np.bincount(table.cpu().numpy()[table.cpu().numpy() >= 0], minlength=pages)
        np.testing.assert_array_equal(count, refs.cpu().numpy())
    assert length.tolist() == [64, 64, 64, 67]
