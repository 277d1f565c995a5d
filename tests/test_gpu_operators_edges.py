"""The context-free operators where a call goes wrong or its inputs are at the edge of what is allowed."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
import workloads as W
from tests import lockstep
from tests import operators_reference as ref
from tests.test_gpu_operators import DEV, U16, Packed

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
    out, score = torch.full_like(inputs[0], 9.0), torch.full((s.U, k + 1), -5.0, device=DEV)
    slot, row = torch.full((s.U,), -7, dtype=torch.int32, device=DEV), torch.zeros(s.U, 2, d, dtype=torch.float16, device=DEV)
    args = kf.kf_packed_step(batch=batch, n_heads=heads, n_kv_heads=kv, head_dim=d, budget_k=k, recent_w=20, layer=0, position=s.n, noise_mode=s.noise, tau=1.0,
                             noise_seed=s.seed, debug_fail_first_wait=1)
    tensors = (s.cache, s.pos, s.acc, s.length, *inputs, out, score, slot, row, scratch)
    assert kf.LIB.kf_decode_step_packed(C.byref(args), *(t.data_ptr() for t in tensors), scratch.numel(), torch.cuda.current_stream().cuda_stream) == kf.KF_OK
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


@pytest.mark.parametrize("d,group", [(64, 1), (128, 4), (256, 8), (128, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_packed_step_with_cached_rows_that_are_not_finite(d, group, bad):
    """A K row makes its unit's outputs NaN, a V row its own 32 features of them; nothing else changes by a bit."""
    k, at = 700, 389
    make = lambda: Packed(1, 3 * group, 3, d, k, 100, seed=33)             # noqa: E731
    s, clean = make(), make()
    K, V = (torch.zeros(3, 1, d, dtype=torch.float16, device=DEV) for _ in range(2))
    kf.kf_unpack_cache(cache=s.cache[:, at:at + 1].contiguous(), K=K, V=V)
    K[0, 0, 5], V[1, 0, 40] = bad, bad
    one = torch.zeros(3, 1, 5 * d // 4, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=one)
    clean.cache[2, at] = one[2, 0]                                         # unit 2: the same row, packed once more
    s.cache[:, at] = one[:, 0]
    clean.cache[1, at, :d // 2], clean.cache[1, at, d:9 * d // 8] = one[1, 0, :d // 2], one[1, 0, d:9 * d // 8]      # unit 1: its K row too
    keep = [f for f in range(d // 32) if f != 1]
    v_codes, v_groups = clean.cache[1, at, d // 2:d].view(-1, 16), clean.cache[1, at, 9 * d // 8:].view(-1, 4)
    v_codes[keep], v_groups[keep] = one[1, 0, d // 2:d].view(-1, 16)[keep], one[1, 0, 9 * d // 8:].view(-1, 4)[keep]
    inputs = s.inputs(1)
    got, want = s.call(1, *inputs), clean.call(1, *inputs)
    out, ref_out = (t[0].view(3, group, d) for t in (got, want))
    assert torch.isnan(out[0]).all()
    assert torch.isnan(out[1, :, 32:64]).all()
    rest = torch.ones(d, dtype=torch.bool, device=DEV)
    rest[32:64] = False
    assert torch.equal(out[1][:, rest], ref_out[1][:, rest]) and torch.equal(out[2], ref_out[2]) and torch.isfinite(ref_out).all()
    for u in (1, 2):
        assert torch.equal(got[1][u], want[1][u]) and got[2][u] == want[2][u]
        assert torch.equal(s.acc[u], clean.acc[u]) and torch.equal(s.pos[u], clean.pos[u])


# ------------------------------------------------------------------------------------------------ norm and rotation

@pytest.mark.parametrize("d,halves", [(64, True), (128, False), (256, True)])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30, 1e30])
def test_norm_of_rows_whose_squares_leave_binary32(d, halves, eps):
    """bfloat16 rows from 2^-132 to 2^125, ordinary ones among them; tolerances as for ordinary rows (test_gpu_operators._check_norm)."""
    H, kv = 3, 2
    power = torch.tensor([0, 125, 100, 65, 63, 48, 30, -30, -48, -62, -64, -100, -126, -130, -132], device=DEV)
    n = len(power) * 2
    x = torch.randn(1, n, H + 2 * kv, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(d))
    x = x.clamp(-3.9, 3.9) * torch.exp2(power.double()).repeat(2)[:, None, None].float()
    x[:, n // 2:, ::2] = torch.randn(1, n // 2, (H + 2 * kv + 1) // 2, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(d + 1))
    x = x.bfloat16()                                     # in the second half extreme and ordinary heads alternate within a token
    x[0, 3, 1, 0] = 0.0
    qw, kw = ((1 + 0.3 * torch.randn(d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(i))).bfloat16() for i in (1, 2))
    q, k, v = (torch.empty(1, h, n, d, dtype=torch.float16, device=DEV) for h in (H, kv, kv))
    rows = x.view(1, n, -1)
    kf.kf_qk_norm_rotate(qkv=rows, n_heads=H, n_kv_heads=kv, head_dim=d, q=q, k=k, v=v, norm_mode=kf.KF_NORM_RMS, q_weight=qw, k_weight=kw, eps=eps,
                         rotary_dims=d, rotary_style=kf.KF_ROTARY_HALVES if halves else kf.KF_ROTARY_PAIRS)
    wide = lambda t: t.double().cpu().numpy()                                              # noqa: E731
    want = ref.norm_rotate(wide(rows), H, kv, d, np.arange(n)[None], wide(qw), wide(kw), True, np.float64(np.float32(eps)), d, 10000.0, halves)
    for got, w in zip((q, k), want):
        big = np.abs(w).max(-1, keepdims=True)
        assert big.max() > 1.0
        err = np.abs(wide(got) - w)
        assert (err <= U16 * np.abs(w) + 2.0 ** -25 + 2.0 ** -20 * big).all(), (err / big).max()
    assert torch.equal(v, x.view(1, n, H + 2 * kv, d)[:, :, H + kv:].transpose(1, 2).half())


def test_norm_of_rows_that_are_not_finite():
    """A NaN makes its row NaN; an infinity makes its own feature NaN and the others 0, as the formula has it; neighbouring rows do not notice."""
    d = 128
    for dtype in (torch.float16, torch.bfloat16):
        x = torch.randn(1, 2, 4, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(dtype)
        clean = x.clone()
        x[0, 0, 0, 5], x[0, 1, 2, 7] = float("nan"), float("inf")
        outs = []
        for rows in (clean, x):
            q, k = torch.empty(1, 2, 2, d, dtype=torch.float16, device=DEV), torch.empty(1, 1, 2, d, dtype=torch.float16, device=DEV)
            kf.kf_qk_norm_rotate(qkv=rows.view(1, 2, -1), n_heads=2, n_kv_heads=1, head_dim=d, q=q, k=k, norm_mode=kf.KF_NORM_RMS, eps=0.0)
            outs.append((q, k))
        (q0, k0), (q, k) = outs
        assert torch.isnan(q[0, 0, 0]).all() and torch.equal(q[0, 1], q0[0, 1]) and torch.equal(q[0, 0, 1], q0[0, 0, 1]) and torch.equal(k[0, 0, 0], k0[0, 0, 0])
        assert torch.isnan(k[0, 0, 1, 7]) and (torch.cat([k[0, 0, 1, :7], k[0, 0, 1, 8:]]) == 0).all()


# ------------------------------------------------------------------------------------------------ shared memory between a call's tensors

def test_inputs_may_share_memory_and_outputs_may_lie_between_rows():
    """What the refusals leave open: one row as query, key and value, and outputs in the unused columns of strided logits."""
    a, b = (Packed(1, 2, 2, 64, 30, 5, seed=15) for _ in range(2))
    row = a.inputs(1)[0]
    got = a.call(1, row, row, row)
    assert all(torch.equal(x, y) for x, y in zip(got, b.call(1, row, row.clone(), row.clone())))
    wide = torch.randn(2, 3, 600, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4))
    scores = torch.zeros(2, 3, device=DEV)
    make = lambda: [torch.zeros(2, 5, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]        # noqa: E731
    want = make()
    kf.kf_beam_select(logits=wide[..., :500], scores=scores, out_scores=want[0], out_parent=want[1], out_token=want[2])
    spare = wide[0, 1, 500:]                                              # 100 words behind a row
    inside = [spare[:10].view(2, 5), spare[20:30].view(torch.int32).view(2, 5), spare[90:].view(torch.int32).view(2, 5)]
    kf.kf_beam_select(logits=wide[..., :500], scores=scores, out_scores=inside[0], out_parent=inside[1], out_token=inside[2])
    assert all(torch.equal(x, y) for x, y in zip(inside, want))


def test_calls_refuse_tensors_that_share_memory():
    s = Packed(1, 1, 1, 64, 8, 2)
    q, _, _ = s.inputs(1)
    row = torch.zeros(1, 2, 64, dtype=torch.float16, device=DEV)
    with pytest.raises(kf.KeyformerError):                                # the quantised row in place of the row
        kf.kf_decode_step_packed(batch=1, n_heads=1, head_dim=64, budget_k=8, recent_w=2, layer=0, position=s.n, tau=1.0, cache=s.cache, pos=s.pos, acc=s.acc,
                                 length=s.length, q=q, knew=row[:, 0], vnew=row[:, 1], out=torch.empty_like(q), row_out=row)
    logits, scores = torch.zeros(2, 3, 50, device=DEV), torch.zeros(2, 3, device=DEV)
    with pytest.raises(kf.KeyformerError):
        kf.kf_beam_select(logits=logits, scores=scores, out_scores=torch.empty_like(scores), out_parent=scores.view(torch.int32),
                          out_token=torch.empty_like(scores, dtype=torch.int32))
    with pytest.raises(kf.KeyformerError):
        x = torch.zeros(1, 4, 192, dtype=torch.float16, device=DEV)
        k = torch.zeros(1, 1, 4, 64, dtype=torch.float16, device=DEV)
        kf.kf_qk_norm_rotate(qkv=x, n_heads=1, n_kv_heads=1, head_dim=64, q=torch.empty_like(k), k=k, positions=k.view(-1)[:8].view(torch.int32).view(1, 4))
    wl = W.Workload("beams", 1, 4, 2, 64, 70, 40, 8, 8, data_seed=2, noise_seed=5)
    ctx = lockstep.make_gpu(wl)
    ctx.kf_prefill_score_prune(0, *W.make_prompt(wl, 0, DEV))
    with pytest.raises(kf.KeyformerError):                                # the parents inside the context's own state
        ctx.kf_reorder_beams(0, ctx.kf_view_state(0)[4].view(-1)[:4].view(2, 2))
    ctx.kf_destroy()


# ------------------------------------------------------------------------------------------------ streams, graphs, the largest sizes

def _simple_calls():
    """(call(stream), outputs) of every operator that needs no scratch, on inputs of its own."""
    g = torch.Generator(device=DEV).manual_seed(8)
    K, V = (torch.randn(3, 50, 64, device=DEV, generator=g).half() for _ in range(2))
    cache = torch.zeros(3, 50, 80, dtype=torch.uint8, device=DEV)
    packed = torch.zeros_like(cache)
    kf.kf_pack_cache(K=K, V=V, cache=packed)
    Kb, Vb = torch.zeros_like(K), torch.zeros_like(V)
    x = torch.randn(2, 9, 4 * 64, device=DEV, generator=g).bfloat16()
    q, k = torch.zeros(2, 2, 9, 64, dtype=torch.float16, device=DEV), torch.zeros(2, 1, 9, 64, dtype=torch.float16, device=DEV)
    rows, parent = torch.randn(6, 4001, device=DEV, generator=g), torch.tensor([[1, 1, 0], [2, 0, 0]], dtype=torch.int32, device=DEV)
    return [(lambda st: kf.kf_pack_cache(K=K, V=V, cache=cache, stream=st), [cache]),
            (lambda st: kf.kf_unpack_cache(cache=packed, K=Kb, V=Vb, stream=st), [Kb, Vb]),
            (lambda st: kf.kf_qk_norm_rotate(qkv=x, n_heads=2, n_kv_heads=1, head_dim=64, q=q, k=k, norm_mode=kf.KF_NORM_RMS, rotary_dims=32, stream=st), [q, k]),
            (lambda st: kf.kf_reorder_rows(buffers=[rows], parent=parent, stream=st), [rows])]


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_calls_without_scratch_on_another_stream_and_replayed(which):
    call, outs = _simple_calls()[which]
    start = [t.clone() for t in outs]

    def reset():
        for t, old in zip(outs, start):
            t.copy_(old)
    call(None)
    want = [t.clone() for t in outs]
    assert any(not torch.equal(a, b) for a, b in zip(want, start))
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(None)
    for _ in range(2):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    del graph


@pytest.mark.parametrize("batch,heads", [(65535, 1), (1, 65535), (255, 257)])
def test_packed_step_of_the_most_units(batch, heads):
    """Units are independent: the largest grid gives what slices of it give.  Without noise, whose coordinates hold the batch row and the head."""
    units, k, d = batch * heads, 3, 64
    g = torch.Generator(device=DEV).manual_seed(6)
    K, V = (torch.randn(units, k, d, device=DEV, generator=g).half() for _ in range(2))
    cache = torch.zeros(units, k, 80, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=cache)
    pos = torch.tensor([4, 9, 7], dtype=torch.int32, device=DEV).repeat(units, 1)
    acc = torch.rand(units, k, device=DEV, generator=g)
    length = (torch.arange(units, device=DEV, dtype=torch.int32) % 4)
    q, kn, vn = (torch.randn(units, d, device=DEV, generator=g).half() for _ in range(3))

    def step(at, n, b, h):
        state = [t[at:at + n].clone() for t in (cache, pos, acc, length)]
        out, slot = torch.zeros(n, d, dtype=torch.float16, device=DEV), torch.full((n,), -9, dtype=torch.int32, device=DEV)
        kf.kf_decode_step_packed(batch=b, n_heads=h, head_dim=d, budget_k=k, recent_w=1, layer=0, position=10, tau=1.5, cache=state[0], pos=state[1], acc=state[2],
                                 length=state[3], q=q[at:at + n], knew=kn[at:at + n], vnew=vn[at:at + n], out=out, slot_out=slot, noise_mode=kf.KF_NOISE_NONE)
        return state + [out, slot]
    whole = step(0, units, batch, heads)
    for at, n in ((0, 1), (units // 2, 300), (units - 200, 200)):
        assert all(torch.equal(a[at:at + n], b) for a, b in zip(whole, step(at, n, n, 1)))
    assert (whole[5] >= 0).all() and torch.isfinite(whole[4]).all()


def test_beam_select_of_the_most_rows():
    """65535 rows, and rows of 33 million tokens (thousands of lists per beam), against torch's own sort."""
    logits = torch.randn(21845, 3, 5, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    out = [torch.zeros(21845, 15, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    kf.kf_beam_select(logits=logits, scores=torch.zeros(21845, 3, device=DEV), out_scores=out[0], out_parent=out[1], out_token=out[2])
    value = torch.log_softmax(logits.double(), -1).view(21845, 15)
    mine = torch.gather(value, 1, (out[1] * 5 + out[2]).long())
    assert (out[1] * 5 + out[2]).sort(1).values.equal(torch.arange(15, device=DEV, dtype=torch.int32).expand(21845, 15))
    assert (mine - value.sort(1, descending=True).values).abs().max() <= 1e-6 and (mine - out[0]).abs().max() <= 2e-6
    V, take = (1 << 25) + 3, 8
    logits = torch.randn(1, 4, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4)).mul_(3).half()
    scores = torch.tensor([[-1.0, 0.0, -0.5, -9.0]], device=DEV)
    out = [torch.zeros(1, take, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    kf.kf_beam_select(logits=logits, scores=scores, out_scores=out[0], out_parent=out[1], out_token=out[2])
    best = []
    for w in range(4):
        x = logits[0, w]
        top, at = torch.sort(x, descending=True, stable=True)              # equal values: the lower token first
        norm = torch.logsumexp(x.double(), 0)
        best += [(float(scores[0, w]) + float(top[i].double() - norm), -w, -int(at[i])) for i in range(take)]
    best = sorted(best, reverse=True)[:take]
    got = [(float(a), -int(b), -int(c)) for a, b, c in zip(*(t[0] for t in out))]
    for (value, w, t), (mine, gw, gt) in zip(best, got):
        # a sum of 33 million exponentials: 8192 partial sums of 8192, each within 2^-20 of its value
        assert abs(value - mine) <= 2e-6 + 2.0 ** -23 * abs(value) and (w, t) == (gw, gt)
