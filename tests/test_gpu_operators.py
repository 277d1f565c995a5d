"""The context-free operators on a GPU against plain 64-bit forms (tests/operators_reference.py) and, for the generation step
over a 4-bit cache, against the oracle on the rows that the codes stand for."""
import math

import numpy as np
import pytest
import torch

import paper_2403_09054_b200 as kf
import workloads as W
from oracle import keyformer_oracle as ko
from tests import lockstep
from tests import operators_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16 = 2.0 ** -11            # half a step of binary16, relative


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(*shape, device=DEV, generator=_gen(seed))


# ------------------------------------------------------------------------------------------------ 4-bit rows

def _special_rows(units, n, d, seed):
    loud = torch.exp(_randn(seed + 1, units, 1, d))
    x = (_randn(seed, units, n, d) * loud).half()
    flat = x.view(units * n, d)
    flat[0] = 2.5                                         # constant groups
    if flat.shape[0] > 5:
        flat[1, :32] = torch.linspace(-65504, 65504, 32, device=DEV).half()
        flat[2] = (_randn(seed + 2, d) * 2.0 ** -20).half()            # subnormal numbers
        flat[3, 5] = float("nan")
        flat[4, d - 1] = float("inf")
        flat[5, 33] = -float("inf")
    return x


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("units,n,k", [(1, 1, 1), (3, 7, 9), (2, 129, 129), (5, 31, 40)])
def test_pack_and_unpack(units, n, k, d):
    K, V = _special_rows(units, n, d, 10 * n + d), _special_rows(units, n, d, 10 * n + d + 5).flip(1).contiguous()
    cache = torch.full((units, k, 5 * d // 4), 0xA5, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=cache)
    want = ref.slots_of(K.cpu().numpy(), V.cpu().numpy())
    got = cache.cpu().numpy()
    assert (got[:, n:] == 0xA5).all()                     # slots behind the rows stay as they were
    # codes bit for bit; group parameters as numbers (a zero minimum may carry either sign, a NaN any payload)
    assert np.array_equal(got[:, :n, :d], want[..., :d])
    params = lambda a: np.ascontiguousarray(a[..., d:]).view(np.float16)                   # noqa: E731
    assert np.array_equal(params(got[:, :n]), params(want), equal_nan=True)
    Kb, Vb = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    kf.kf_unpack_cache(cache=cache, K=Kb, V=Vb)
    for back, expect in zip((Kb, Vb), ref.rows_of(want, d)):
        assert np.array_equal(back.cpu().numpy(), expect, equal_nan=True)


def test_pack_with_every_scale():
    """Groups whose span is just below, at and just above fifteen times each binary16 number: every scale there is, with its reciprocal, bit for bit."""
    scale = torch.arange(1, 0x7c00, dtype=torch.int16).view(torch.float16).double()
    top = (15 * scale).half()
    top = top[top.isfinite()]
    bits = top.view(torch.int16)
    top = torch.cat([(bits - 1).clamp(min=0).view(torch.float16), top, (bits + 1).clamp(max=0x7bff).view(torch.float16)])
    n = top.numel() // 8
    g = torch.rand(n * 8, 32, generator=torch.Generator().manual_seed(1)) * top[:n * 8, None].float()
    g[:, 3], g[:, 17] = 0.0, top[:n * 8].float()
    x = g.half().view(2, 1, n, 128)
    sign = torch.tensor([1.0, -1.0], dtype=torch.float16).repeat(n // 2 + 1)[:n, None]
    K, V = (x[0] * sign).contiguous().to(DEV), x[1].contiguous().to(DEV)
    cache = torch.zeros(1, n, 160, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=cache)
    want = ref.slots_of(K.cpu().numpy(), V.cpu().numpy())
    got = cache.cpu().numpy()
    assert np.array_equal(got[..., :128], want[..., :128])
    assert np.array_equal(got[..., 128:].view(np.float16), want[..., 128:].view(np.float16))


def test_pack_many_units_of_one_row():
    """More units than a grid dimension holds."""
    K, V = _randn(1, 70001, 1, 64).half(), _randn(2, 70001, 1, 64).half()
    cache = torch.zeros(70001, 1, 80, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=cache)
    assert np.array_equal(cache.cpu().numpy()[..., :64], ref.slots_of(K.cpu().numpy(), V.cpu().numpy())[..., :64])
    Kb, Vb = torch.zeros_like(K), torch.zeros_like(V)
    kf.kf_unpack_cache(cache=cache, K=Kb, V=Vb)
    assert np.array_equal(Kb.cpu().numpy(), ref.rows_of(cache.cpu().numpy(), 64)[0])


def test_pack_leaves_rows_behind_the_entry_count():
    K, V = _randn(1, 2, 3, 9, 64).half(), _randn(2, 2, 3, 9, 64).half()
    length = torch.tensor([[0, 1, 9], [5, 12, -3]], dtype=torch.int32, device=DEV)      # counts outside 0..n: all rows, none
    cache = torch.full((2, 3, 9, 80), 0x5A, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=cache, length=length)
    want = ref.slots_of(K.cpu().numpy(), V.cpu().numpy())
    got = cache.cpu().numpy()
    Kb = torch.full_like(K, 3.0)
    kf.kf_unpack_cache(cache=cache, K=Kb, V=torch.empty_like(V), length=length)
    Kb = Kb.cpu().numpy()
    for u, n in enumerate(length.flatten().clamp(0, 9).tolist()):
        b, h = divmod(u, 3)
        assert np.array_equal(got[b, h, :n], want[b, h, :n]) and (got[b, h, n:] == 0x5A).all()
        assert np.array_equal(Kb[b, h, :n], ref.rows_of(want, 64)[0][b, h, :n]) and (Kb[b, h, n:] == 3.0).all()


# ------------------------------------------------------------------------------------------------ the step over a 4-bit cache

class Packed:
    """A caller's state of one layer, and the oracle walking along on the rows the codes stand for."""

    def __init__(self, batch, heads, kv, d, k, w, lengths=None, noise=kf.KF_NOISE_GUMBEL, alibi=False, seed=0, layer=0, loud=0.4, late=0.0, logit_scale=0.0):
        self.shape = (batch, heads, kv, d, k, w)
        self.noise, self.alibi, self.layer, self.seed, self.logit_scale = noise, alibi, layer, 1000 + seed, logit_scale
        U = self.U = batch * kv
        rng = np.random.default_rng(seed)
        self.n = 3 * k + 5                                # the prompt's length; step s stands at n + s - 1
        self.length = torch.tensor([k] * U if lengths is None else [lengths[u % len(lengths)] for u in range(U)], dtype=torch.int32, device=DEV)
        K = (_randn(seed, U, k, d) * torch.exp(loud * _randn(seed + 1, U, 1, d)))
        K[:, k - k // 3:] *= 1.0 + late                   # entries met last with logits far above the others
        V = _randn(seed + 2, U, k, d)
        self.cache = torch.zeros(U, k, 5 * d // 4, dtype=torch.uint8, device=DEV)
        kf.kf_pack_cache(K=K.half(), V=V.half(), cache=self.cache)
        pos = np.stack([np.sort(rng.choice(self.n, k, replace=False)) for _ in range(U)])
        for u in range(U):                                # the window is there; slots in no order
            pos[u, k - min(w, k):] = np.arange(self.n - min(w, k), self.n)
            older = np.sort(rng.choice(self.n - min(w, k), k - min(w, k), replace=False))
            pos[u, :k - min(w, k)] = older
            pos[u] = rng.permutation(pos[u])
        self.pos = torch.from_numpy(pos.astype(np.int32)).to(DEV)
        self.acc = torch.exp(_randn(seed + 3, U, k))
        for u, n in enumerate(self.length.tolist()):      # whatever lies behind the last entry is never read
            self.cache[u, n:], self.pos[u, n:], self.acc[u, n:] = 0xFF, -1, float("nan")
        self.slopes = torch.tensor(W.alibi_slopes(heads), dtype=torch.float32, device=DEV) if alibi else None
        self.P = ko.Params(head_dim=d, n_heads=heads, budget_k=k, recent_w=w, gen_len_T=16, tau_init=1.0, tau_end=2.0, noise_seed=self.seed, noise_mode=noise,
                           bias_mode=int(alibi), alibi_slopes=W.alibi_slopes(heads).astype(np.float32) if alibi else None, n_kv_heads=kv, logit_scale=logit_scale)
        self.st = ko.State(self.P, [(layer, u // kv, u % kv) for u in range(U)])
        self.st.n_prompt = self.n
        self.reload()

    def reload(self):
        """The oracle's entries are what the caller's tensors hold, in slot order."""
        d, k = self.shape[3], self.shape[4]
        Kr, Vr = ref.rows_of(self.cache.cpu().numpy(), d)
        self.st.len[:] = self.length.cpu().numpy()
        for u, n in enumerate(self.st.len):
            self.st.pos[u, :n], self.st.acc[u, :n] = self.pos[u, :n].cpu().numpy(), self.acc[u, :n].double().cpu().numpy()
            self.st.K[u, :n], self.st.V[u, :n] = Kr[u, :n].view(np.uint16), Vr[u, :n].view(np.uint16)
        return Kr, Vr

    def inputs(self, step):
        B, H, kv, d, _, _ = self.shape
        return (_randn(self.seed + 7 * step, B, H, d).half(), _randn(self.seed + 7 * step + 1, B, kv, d).half(), _randn(self.seed + 7 * step + 2, B, kv, d).half())

    def call(self, step, q, kn, vn, **kw):
        B, H, kv, d, k, w = self.shape
        out = torch.full_like(q, 9.0)
        score = torch.full((self.U, k + 1), -5.0, device=DEV)
        slot = torch.full((self.U,), -7, dtype=torch.int32, device=DEV)
        row = torch.full((self.U, 2, d), 9.0, dtype=torch.float16, device=DEV)
        kf.kf_decode_step_packed(batch=B, n_heads=H, n_kv_heads=kv, head_dim=d, budget_k=k, recent_w=w, layer=self.layer, position=self.n + step - 1,
                                 tau=ko.tau(self.P, step), cache=self.cache, pos=self.pos, acc=self.acc, length=self.length, q=q, knew=kn, vnew=vn, out=out,
                                 score_out=score, slot_out=slot, row_out=row, noise_seed=self.seed, noise_mode=self.noise,
                                 bias_mode=kf.KF_BIAS_ALIBI if self.alibi else kf.KF_BIAS_NONE, alibi_slopes_dev=self.slopes, logit_scale=self.logit_scale, **kw)
        return out, score, slot, row

    def step(self, step, **kw):
        """One step, compared with the oracle entry by entry.

        Tolerances.  A logit is d products of binary16 numbers summed in binary32 in some order: at most (d + 8) 2^-23 of the sum of their
        magnitudes; the noise a relative 5e-6 of -ln u at worst (Gaussian form; 1e-6 for the others) and binary32 roundings of values below 20;
        an exponential 2^-22 of its argument (below 60) and of itself; a softmax twice that.  The output rounds each weight and itself to binary16."""
        B, H, kv, d, k, w = self.shape
        g = H // kv
        q, kn, vn = self.inputs(step)
        before = [t.clone() for t in (self.cache, self.pos, self.acc, self.length)]
        Kr, Vr = self.reload()
        len0 = self.st.len.copy()
        out, score, slot, row = (t.cpu().numpy() for t in self.call(step, q, kn, vn, **kw))
        torch.cuda.synchronize()
        flat = lambda t, *s: t.cpu().numpy().reshape(*s)                                   # noqa: E731
        out_ref, z_ref = self.st.decode_score(step, flat(q, self.U, g, d) if g > 1 else flat(q, self.U, d), flat(kn, self.U, d), flat(vn, self.U, d))
        out_ref = out_ref.reshape(self.U, g, d)
        scale = self.logit_scale or 1.0 / math.sqrt(d)
        qa, kna, vna = (np.abs(flat(t, self.U, -1, d).astype(np.float64)) for t in (q, kn, vn))
        fresh = ref.slots_of(flat(kn, self.U, d), flat(vn, self.U, d))
        kfresh, vfresh = ref.rows_of(fresh, d)
        assert np.array_equal(row, np.stack([kfresh, vfresh], 1))
        acc, pos, length, cache = (t.cpu().numpy() for t in (self.acc, self.pos, self.length, self.cache))
        for u in range(self.U):
            n = int(len0[u])
            mag = max(float((qa[u] @ np.abs(Kr[u, :n].astype(np.float64)).T).max()) if n else 0.0, float((qa[u] @ kna[u].T).max()))
            err_x = (d + 8) * 2.0 ** -23 * mag * scale + (2.0 ** -22 * 3 * self.n if self.alibi else 0.0)
            err_y = err_x + 5e-6 * 6 * 2 + 2.0 ** -22 * 20
            tol_z = 2 * (err_y + 2.0 ** -22 * 60)
            vmax = max(float(np.abs(Vr[u, :n].astype(np.float64)).max()) if n else 0.0, float(vna[u].max()))
            tol_o = vmax * (2 * (err_x + 2.0 ** -22 * 60) + U16) + U16 * np.abs(out_ref[u]) + 2.0 ** -25
            assert (np.abs(out.reshape(self.U, g, d)[u] - out_ref[u]) <= tol_o).all(), (u, np.abs(out.reshape(self.U, g, d)[u] - out_ref[u]).max(), vmax)
            z = z_ref[u, :n + 1]
            assert (np.abs(score[u, :n + 1] - z) <= tol_z * z + 1e-12).all(), (u, (np.abs(score[u, :n + 1] - z) / z).max(), tol_z)
            assert (score[u, n + 1:] == -5.0).all()
            total = self.st.acc[u, :n + 1].copy()
            tol_a = 2.0 ** -23 * np.abs(total) + tol_z * z
            if n < k:
                assert slot[u] == n and length[u] == n + 1
            else:                                          # the smallest outside the window, up to what the scores' errors leave open
                p = self.n + step - 1
                at = np.append(before[1][u].cpu().numpy(), p)
                may = np.where(at <= p - w)[0]
                gone = n if slot[u] < 0 else int(slot[u])
                assert length[u] == k and gone in may and total[gone] <= (total[may] + tol_a[may]).min() + tol_a[gone]
            s = int(slot[u])
            keep = np.arange(n) != s
            assert np.array_equal(pos[u, :n][keep], before[1][u, :n].cpu().numpy()[keep])
            assert (np.abs(acc[u, :n] - total[:n]) <= tol_a[:n])[keep].all()
            if s >= 0:
                assert pos[u, s] == self.n + step - 1 and abs(acc[u, s] - z[n]) <= tol_z * z[n]
                assert np.array_equal(ref.rows_of(cache[u, s], d)[0], kfresh[u]) and np.array_equal(cache[u, s][:d], fresh[u][:d])
            rest = np.ones(k, bool)
            rest[max(s, 0):max(s, 0) + (s >= 0)] = False
            assert np.array_equal(cache[u][rest], before[0][u].cpu().numpy()[rest])      # every other slot, used or not, byte for byte
        return slot


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_packed_step_walks_with_the_oracle(d, group):
    lengths = [77, 0, 1, 31, 32, 33, 76, 64]              # filling caches, an empty one, one that becomes full on the way
    s = Packed(2, 4 * group, 4, d, 77, 19, lengths=lengths, alibi=group in (1, 4), seed=d + group, layer=3)
    for step in range(1, 5):
        s.step(step)


@pytest.mark.parametrize("k,w", [(1, 0), (1, 1), (2, 1), (32, 0), (33, 33), (500, 100), (129, 0), (1300, 300), (4200, 1000)])
@pytest.mark.parametrize("d,group", [(128, 1), (64, 2)])
def test_packed_step_budgets_and_windows(k, w, d, group):
    s = Packed(1, 3 * group, 3, d, k, w, seed=k + w)
    for step in range(1, 4):
        s.step(step)


@pytest.mark.parametrize("noise", [kf.KF_NOISE_NONE, kf.KF_NOISE_CONST, kf.KF_NOISE_GAUSS])
def test_packed_step_other_adjustments(noise):
    s = Packed(2, 8, 4, 128, 150, 40, noise=noise, alibi=True, seed=5 + noise)
    for step in range(1, 4):
        s.step(step)


@pytest.mark.parametrize("d,group", [(64, 1), (128, 4), (256, 1)])
def test_packed_step_when_late_entries_dwarf_the_early_ones(d, group):
    """The reference of the output weights has to move in the middle of a warp's walk."""
    s = Packed(1, 2 * group, 2, d, 900, 100, seed=77, late=9.0, logit_scale=0.5 / math.sqrt(d))
    for step in range(1, 3):
        s.step(step)


def test_packed_step_many_units():
    """More caches than SMs: the other closing kernel and a plan with several tiles per warp."""
    s = Packed(40, 8, 8, 64, 300, 75, seed=9)
    s.step(1)
    s.step(2)


def test_packed_step_new_token_may_stay_outside():
    """w = 0 and a cache of high scores: the new token is the one that leaves; nothing but the scores changes."""
    s = Packed(1, 4, 4, 64, 40, 0, seed=31)
    s.acc += 50.0
    cache, pos = s.cache.clone(), s.pos.clone()
    assert (s.step(1) == -1).all()
    assert torch.equal(cache, s.cache) and torch.equal(pos, s.pos) and (s.length == 40).all()


def test_packed_step_skips_units_with_damaged_counts():
    s = Packed(1, 3, 3, 128, 50, 10, seed=12)
    s.length[0], s.length[2] = -1, 51
    before = [t.clone() for t in (s.cache, s.pos, s.acc, s.length)]
    out, score, slot, row = s.call(1, *s.inputs(1))
    for u in (0, 2):
        assert (out[0, u] == 9.0).all() and (score[u] == -5.0).all() and slot[u] == -7 and (row[u] == 9.0).all()
        for now, old in zip((s.cache, s.pos, s.acc, s.length), before):
            assert torch.equal(now[u], old[u]) or (torch.isnan(old[u].float()).any())
    assert (out[0, 1] != 9.0).any() and slot[1] >= 0


def test_packed_step_without_the_optional_outputs():
    """What is returned beside it does not change the state: bit for bit the same with and without."""
    a, b = (Packed(2, 4, 2, 128, 90, 20, lengths=[90, 40], seed=8) for _ in range(2))
    q, kn, vn = a.inputs(1)
    out = a.call(1, q, kn, vn)[0]
    mine = torch.empty_like(q)
    kf.kf_decode_step_packed(batch=2, n_heads=4, n_kv_heads=2, head_dim=128, budget_k=90, recent_w=20, layer=0, position=b.n, tau=ko.tau(b.P, 1), cache=b.cache,
                             pos=b.pos, acc=b.acc, length=b.length, q=q, knew=kn, vnew=vn, out=mine, noise_seed=b.seed)
    assert torch.equal(out, mine) and torch.equal(a.cache, b.cache) and torch.equal(a.pos, b.pos) and torch.equal(a.length, b.length)
    assert torch.equal(torch.nan_to_num(a.acc), torch.nan_to_num(b.acc))


def test_packed_steps_of_two_streams_at_once():
    """Two layers' steps in flight on two streams, each with scratch of its own from torch's allocator."""
    states = [Packed(4, 8, 8, 128, 700, 100, seed=40 + i) for i in range(2)]
    want = [Packed(4, 8, 8, 128, 700, 100, seed=40 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    inputs = [[s.inputs(step) for step in range(1, 9)] for s in states]
    torch.cuda.synchronize()
    outs = [[], []]
    for step in range(8):
        for i in range(2):
            outs[i].append(states[i].call(step + 1, *inputs[i][step], stream=streams[i])[0])
    torch.cuda.synchronize()
    for i in range(2):
        for step in range(8):
            assert torch.equal(outs[i][step], want[i].call(step + 1, *inputs[i][step])[0])
        assert torch.equal(states[i].cache, want[i].cache) and torch.equal(states[i].acc, want[i].acc)


def test_packed_step_is_reproducible_and_holds_nothing_between_calls():
    """The same state and inputs give the same bits: after another shape's call on the same scratch, on another stream, and replayed from a graph."""
    a = Packed(2, 8, 2, 128, 333, 80, seed=3)
    nbytes = kf.kf_packed_scratch_bytes(batch=2, n_heads=8, n_kv_heads=2, head_dim=128, budget_k=333)
    other = Packed(3, 4, 4, 64, 90, 10, seed=4)
    scratch = torch.full((max(nbytes, kf.kf_packed_scratch_bytes(batch=3, n_heads=4, n_kv_heads=4, head_dim=64, budget_k=90)),), 0xFF, dtype=torch.uint8, device=DEV)
    state = [t.clone() for t in (a.cache, a.pos, a.acc, a.length)]

    def reset():
        for t, old in zip((a.cache, a.pos, a.acc, a.length), state):
            t.copy_(old)
    inputs = a.inputs(1)
    first = [t.clone() for t in a.call(1, *inputs, scratch=scratch)] + [a.cache.clone(), a.acc.clone()]
    other.call(1, *other.inputs(1), scratch=scratch)
    reset()
    again = [t.clone() for t in a.call(1, *inputs, scratch=scratch)] + [a.cache.clone(), a.acc.clone()]
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    third = a.call(1, *inputs, stream=side)
    side.synchronize()
    third = list(third) + [a.cache.clone(), a.acc.clone()]
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = a.call(1, *inputs)
    reset()                                                # captured, not run
    for _ in range(2):
        reset()
        graph.replay()
    fourth = list(captured) + [a.cache.clone(), a.acc.clone()]
    for run in (again, third, fourth):
        for x, y in zip(first, run):
            assert torch.equal(x, y)
    del graph


def test_packed_step_after_the_prompt_phase():
    """The documented way into a 4-bit cache: a context scores and prunes the prompt, its layer is packed, generation goes on in 4 bits --
    close to the context's own steps (the rows differ by their quantisation), and exactly what the oracle makes of the quantised rows."""
    wl = W.Workload("packed", 1, 2, 4, 128, 300, 150, 40, 8, data_seed=3, noise_seed=11)
    gpu = lockstep.make_gpu(wl)
    gpu.kf_prefill_score_prune(0, *W.make_prompt(wl, 0, DEV))
    K, V, pos, acc, length = gpu.kf_view_state(0)
    s = Packed(2, 4, 4, 128, 150, 40, seed=1)
    s.n, s.seed, s.st.n_prompt = wl.prompt_len, wl.noise_seed, wl.prompt_len
    s.P.noise_seed = wl.noise_seed
    kf.kf_pack_cache(K=K, V=V, cache=s.cache.view(2, 4, 150, 160), length=length)
    s.pos.copy_(pos.view(8, 150))
    s.acc.copy_(acc.view(8, 150))
    s.length.copy_(length.view(8))
    for step in range(1, 4):
        s.step(step)
    gpu.kf_destroy()


def test_a_cache_whose_offsets_pass_32_bits():
    """4.3 GB of slots in one unit: one entry near the end outweighs 54 million indifferent ones; among those, all with the same score, the
    one with the highest position outside the window leaves."""
    d, k, w = 64, 54_000_000, 10
    cache = torch.zeros(1, k, 80, dtype=torch.uint8, device=DEV)           # scale and minimum 0: rows of zeros
    kn, vn, q = _randn(1, 1, 1, d).half(), _randn(2, 1, 1, d).half(), torch.ones(1, 1, d, dtype=torch.float16, device=DEV)
    K, V = torch.full((1, 1, d), 4.0, dtype=torch.float16, device=DEV), _randn(3, 1, 1, d).half()
    one = torch.zeros(1, 1, 80, dtype=torch.uint8, device=DEV)
    kf.kf_pack_cache(K=K, V=V, cache=one)
    at = k - 5
    cache[0, at] = one[0, 0]
    pos = torch.arange(k, dtype=torch.int32, device=DEV).view(1, k)
    acc, length = torch.zeros(1, k, device=DEV), torch.full((1,), k, dtype=torch.int32, device=DEV)
    out, slot, score = torch.zeros_like(q), torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, k + 1, device=DEV)
    kf.kf_decode_step_packed(batch=1, n_heads=1, head_dim=d, budget_k=k, recent_w=w, layer=0, position=k, tau=1.0, cache=cache, pos=pos, acc=acc, length=length,
                             q=q, knew=kn, vnew=vn, out=out, slot_out=slot, score_out=score, noise_mode=kf.KF_NOISE_NONE)
    x_new = float(kn.double().sum()) / 8                                   # q is all ones; the heavy entry's logit is 64 * 4 / 8 = 32
    total = math.exp(32.0) + (k - 1) + math.exp(x_new)
    rows = ref.rows_of(one.cpu().numpy(), d)[1][0, 0].astype(np.float64)
    want = (math.exp(32.0) * rows + math.exp(x_new) * vn.double().cpu().numpy()[0, 0]) / total
    assert (np.abs(out.double().cpu().numpy()[0, 0] - want) <= U16 * np.abs(want) + 2.0 ** -25 + 1e-5).all()
    assert abs(float(score[0, at]) - math.exp(32.0) / total) < 1e-5 and int(slot) == k - w and int(pos[0, k - w]) == k
    Kb = torch.zeros(1, k, d, dtype=torch.float16, device=DEV)
    Vb = torch.zeros_like(Kb)
    kf.kf_unpack_cache(cache=cache, K=Kb, V=Vb)
    assert np.array_equal(Vb[0, at].cpu().numpy(), rows.astype(np.float16)) and (Kb[0, at] == 4).all() and (Kb[0, at - 1] == 0).all()
    again = torch.zeros_like(cache)
    kf.kf_pack_cache(K=Kb, V=Vb, cache=again)
    back = torch.zeros(1, 1, d, dtype=torch.float16, device=DEV)
    kf.kf_unpack_cache(cache=again[:, at:at + 1].contiguous(), K=torch.zeros_like(back), V=back)
    again_rows = ref.rows_of(ref.slots_of(rows.astype(np.float16)[None], rows.astype(np.float16)[None]), d)[1][0]
    assert np.array_equal(back[0, 0].cpu().numpy(), again_rows)


# ------------------------------------------------------------------------------------------------ norm and rotation

def _check_norm(B, n, H, kv, d, dtype, R, halves, norm, base=10000.0, positions=None, position0=0, pad=0, weights=True, with_v=True, eps=1e-6, seed=0):
    width = (H + 2 * kv) * d
    store = (2 * _randn(seed, B, n, width + pad)).to(dtype)
    x = store[..., :width]
    qw, kw = ((1 + 0.3 * _randn(seed + i, d)).to(dtype) if weights and norm else None for i in (1, 2))
    q, k = torch.empty(B, H, n, d, dtype=torch.float16, device=DEV), torch.empty(B, kv, n, d, dtype=torch.float16, device=DEV)
    v = torch.empty_like(k) if with_v else None
    kf.kf_qk_norm_rotate(qkv=x, n_heads=H, n_kv_heads=kv, head_dim=d, q=q, k=k, v=v, positions=positions, position0=position0,
                         norm_mode=kf.KF_NORM_RMS if norm else kf.KF_NORM_NONE, q_weight=qw, k_weight=kw, eps=eps, rotary_dims=R, rotary_base=base,
                         rotary_style=kf.KF_ROTARY_HALVES if halves else kf.KF_ROTARY_PAIRS)
    at = positions.cpu().numpy() if positions is not None else np.broadcast_to(position0 + np.arange(n), (B, n))
    wide = lambda t: None if t is None else t.double().cpu().numpy()                       # noqa: E731
    want = ref.norm_rotate(wide(x), H, kv, d, at, wide(qw), wide(kw), norm, np.float64(np.float32(eps)), R, base, halves)
    for name, got, w in zip("qkv", (q, k, v), want):
        if got is None:
            continue
        # one rounding to binary16; before it a handful of binary32 roundings (norm: 2^-21 of the value; angle: half a turn in binary32, 2 pi 2^-25, and
        # sine and cosine to 2^-22), which a rotation spreads over the pair: bounded by the row's largest value
        big = np.abs(w).max(-1, keepdims=True)
        err = np.abs(got.double().cpu().numpy() - w)
        assert (err <= U16 * np.abs(w) + 2.0 ** -25 + 2.0 ** -20 * big).all(), (name, (err / big).max())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_norm_rotate_all_rotations(d, halves, dtype):
    for R in (0, 8, 16, 32, 64, 128, 256):
        if R <= d:
            _check_norm(2, 5, 4, 2, d, dtype, R, halves, True, seed=R + d)
            _check_norm(1, 3, 1, 1, d, dtype, R, halves, False, seed=R + d)


@pytest.mark.parametrize("B,n,H,kv", [(1, 1, 1, 1), (33, 1, 32, 8), (3, 129, 5, 5), (1, 2000, 16, 1), (7, 3, 64, 8)])
def test_norm_rotate_shapes_and_strides(B, n, H, kv):
    _check_norm(B, n, H, kv, 64, torch.bfloat16, 32, True, True, pad=24, seed=n)            # rows with something between them
    _check_norm(B, n, H, kv, 128, torch.float16, 128, False, True, with_v=False, weights=False, position0=777, seed=n)


def test_norm_rotate_far_positions():
    """Positions up to the largest int32 (and below zero): whole turns come off in binary64."""
    at = torch.tensor([[0, 1, 2 ** 31 - 1, 1_000_003, -5, -(2 ** 31)]], dtype=torch.int32, device=DEV)
    for halves in (False, True):
        _check_norm(1, 6, 2, 1, 128, torch.float16, 128, halves, True, positions=at, seed=8)
        _check_norm(1, 6, 2, 1, 64, torch.bfloat16, 16, halves, False, positions=at, base=500000.0, seed=9)
    _check_norm(1, 4, 2, 1, 64, torch.float16, 64, False, False, position0=2 ** 31 - 4, seed=10)


def test_norm_rotate_of_more_than_two_to_the_31_values():
    B, n, H, d = 3, 5600, 1022, 128
    x = torch.randint(-3000, 3000, (B, n, (H + 2) * d), dtype=torch.int16, device=DEV, generator=_gen(4)).half().div_(1000)
    q, k, v = (torch.empty(B, h, n, d, dtype=torch.float16, device=DEV) for h in (H, 1, 1))
    kf.kf_qk_norm_rotate(qkv=x, n_heads=H, n_kv_heads=1, head_dim=d, q=q, k=k, v=v, norm_mode=kf.KF_NORM_RMS, rotary_dims=128, rotary_style=kf.KF_ROTARY_HALVES)
    for b, t in ((0, 0), (2, n - 1), (1, 4000)):
        row = x[b, t].double().cpu().numpy()[None, None]
        want = ref.norm_rotate(row, H, 1, d, np.array([[t]]), None, None, True, np.float64(np.float32(1e-6)), 128, 10000.0, True)
        for got, w in zip((q[b, :, t], k[b, :, t], v[b, :, t]), want):
            w = w[0, :, 0]
            assert (np.abs(got.double().cpu().numpy() - w) <= U16 * np.abs(w) + 2.0 ** -20 * np.abs(w).max(-1, keepdims=True)).all()


def test_norm_rotate_small_and_zero_rows():
    x = torch.zeros(1, 3, 4 * 64, dtype=torch.float16, device=DEV)
    x[0, 1] = 2.0 ** -24                                    # squares vanish beside eps
    x[0, 2] = 60000.0
    q, k, v = (torch.empty(1, h, 3, 64, dtype=torch.float16, device=DEV) for h in (2, 1, 1))
    kf.kf_qk_norm_rotate(qkv=x, n_heads=2, n_kv_heads=1, head_dim=64, q=q, k=k, v=v, norm_mode=kf.KF_NORM_RMS, rotary_dims=64)
    assert (q[:, :, 0] == 0).all() and (k[:, :, 0] == 0).all() and torch.isfinite(q).all() and (v[0, 0, 2] == 60000.0).all()
    assert (q[0, 0, 2].double().square().mean() - 1).abs() < 2e-3


def test_norm_rotate_agrees_with_the_library_rotation():
    """KF_ROTARY_PAIRS is the embedding of rotary_dims: rotated here or by the context, the prompt scores are the same up to the rotated
    copies' rounding (both round the same values to binary16)."""
    wl = W.Workload("rot", 1, 1, 4, 64, 90, 90, 10, 0, data_seed=6, positional="rotary", rotary_dims=32, rotary_in_library=True)
    q, k, v = W.make_prompt(wl, 0, DEV)
    scores = []
    for R in (32, 0):
        g = kf.Keyformer(n_layers=1, batch=1, n_heads=4, head_dim=64, budget_k=90, recent_w=10, max_prompt_len=90, gen_len_T=0, rotary_dims=R)
        if R == 0:
            rows = torch.cat([t.transpose(1, 2).reshape(1, 90, -1) for t in (q, k, v)], -1).contiguous()
            q, k, v = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
            kf.kf_qk_norm_rotate(qkv=rows, n_heads=4, n_kv_heads=4, head_dim=64, q=q, k=k, v=v, rotary_dims=32)
        out = torch.empty(1, 4, 90, device=DEV)
        g.kf_prefill_score_prune(0, q, k, v, score_out=out)
        assert g.kf_poll_error() == 0
        scores.append(out.double().cpu().numpy())
        g.kf_destroy()
    # a rotated feature that the two round to neighbouring binary16 numbers changes a logit by 2^-10 |q||k| / sqrt(d) at most
    assert (np.abs(scores[0] - scores[1]) <= 2e-2 * np.abs(scores[0])).all()


# ------------------------------------------------------------------------------------------------ beams

def _check_beams(logits, scores, take, finished=None, pad=0, **kw):
    B, Wb, V = logits.shape
    out = [torch.full((B, take), -9, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    kf.kf_beam_select(logits=logits, scores=scores, out_scores=out[0], out_parent=out[1], out_token=out[2], finished=finished, pad_token=pad, **kw)
    got, parent, token = (t.cpu().numpy() for t in out)
    lg, sc = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    fin = None if finished is None else finished.cpu().numpy()
    for b in range(B):
        value = ref.beam_values(lg[b], sc[b], None if fin is None else fin[b], pad)
        order = np.argsort(-value, kind="stable")[:take]
        place = parent[b].astype(np.int64) * V + token[b]
        assert len(set(place.tolist())) == take and (token[b] < V).all() and (parent[b] < Wb).all()
        # a row's sum of exponentials is summed in binary32: two beams' continuations closer than 1e-6 may change places
        want, mine = value[order], value[place]
        same = (place == order) | (np.abs(mine - want) <= 1e-6)
        assert same.all(), (b, place, order, mine, want)
        finite = np.isfinite(want)
        assert np.array_equal(finite, np.isfinite(got[b])) and (got[b][~finite] == -np.inf).all()
        assert np.array_equal(place[~finite], order[~finite])
        assert (np.abs(got[b][finite] - want[finite]) <= 2.0 ** -24 * np.abs(want[finite]) + 1e-6).all()
    return got, parent, token


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,beams,V,take", [(1, 1, 1, 1), (2, 3, 5, 15), (1, 4, 50257, 8), (3, 5, 2049, 10), (40, 8, 8193, 16), (2, 32, 777, 64), (1, 1, 300, 64), (5, 2, 65536, 1)])
def test_beam_select(B, beams, V, take, dtype):
    logits = (4 * _randn(V + take, B, beams, V)).to(dtype)
    _check_beams(logits, -10 * torch.rand(B, beams, device=DEV, generator=_gen(3)), take)


def test_beam_select_ties_go_to_the_lower_beam_and_token():
    logits = torch.randint(0, 4, (2, 4, 3001), device=DEV, generator=_gen(1)).half()        # four values only: thousands of equal ones
    logits[:, 1] = logits[:, 0]
    logits[:, 3] = logits[:, 0]
    scores = torch.tensor([[-1.0, -1.0, -2.0, -1.0], [0.0, 0.0, 0.0, 0.0]], device=DEV)
    for take in (1, 7, 64):
        _check_beams(logits, scores, take)
    constant = torch.full((1, 3, 9000), 2.0, device=DEV)
    got, parent, token = _check_beams(constant, torch.zeros(1, 3, device=DEV), 64)
    assert (parent == 0).all() and (token[0] == np.arange(64)).all()
    _check_beams(torch.zeros(60, 3, 9000, device=DEV, dtype=torch.float16), torch.zeros(60, 3, device=DEV), 5)


def test_beam_select_forbidden_tokens_and_dead_beams():
    inf = float("inf")
    logits = _randn(5, 4, 4, 501).half()
    logits[0, 0] = -inf                                     # nothing left of a beam
    logits[0, 1, 10:] = -inf
    logits[1] = -inf                                        # nothing left of a request
    logits[2, 2, 7], logits[2, 2, 8] = float("nan"), inf
    logits[3, :, 3:] = -inf                                 # fewer live continuations than are asked for
    scores = torch.tensor([[0.0, -1, -2, -3], [0.0, -1, -2, -3], [0.0, -inf, float("nan"), inf], [0.0, -1, -inf, -1]], device=DEV)
    for take in (2, 8, 40):
        _check_beams(logits, scores, take)
    first = torch.full((4, 4), -inf, device=DEV)            # the first token of a search: one live beam
    first[:, 0] = 0
    _check_beams(_randn(6, 4, 4, 20000), first, 8)
    _check_beams(torch.full((1, 2, 30), float("nan"), device=DEV), torch.zeros(1, 2, device=DEV), 60)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_beam_select_masks_of_the_lowest_value(dtype):
    """Tokens masked with the type's lowest finite value are tokens all the same: a row of nothing else is uniform."""
    low = torch.finfo(dtype).min
    logits = (2 * _randn(11, 3, 4, 9001)).to(dtype)
    logits[0, :, 100:] = low
    logits[1, 2] = low
    logits[2] = low
    scores = torch.tensor([-1.0, -2.0, -0.5, -3.0], device=DEV).expand(3, 4).contiguous()
    for take in (4, 20):
        got, parent, token = _check_beams(logits, scores, take)
        assert (parent[2] == 2).all() and (token[2] == np.arange(take)).all() and abs(got[2, 0] - (-0.5 - math.log(9001))) < 1e-5


def test_beam_select_more_lists_than_are_held():
    _check_beams((3 * _randn(13, 1, 32, 600011)).half(), -torch.rand(1, 32, device=DEV, generator=_gen(5)), 4)
    _check_beams(torch.zeros(1, 32, 600011, device=DEV, dtype=torch.float16), torch.zeros(1, 32, device=DEV), 64)


@pytest.mark.parametrize("as_bool", [True, False])
def test_beam_select_finished_beams(as_bool):
    logits = _randn(9, 3, 4, 7001).bfloat16()
    scores = -3 * torch.rand(3, 4, device=DEV, generator=_gen(2))
    finished = torch.tensor([[1, 0, 0, 1], [1, 1, 1, 1], [0, 0, 1, 0]], device=DEV, dtype=torch.uint8)
    logits[0, 0] = float("nan")                             # never read
    scores[2, 2] = -float("inf")
    for take, pad in ((8, 0), (8, 7000), (20, 3)):
        _check_beams(logits, scores, take, finished=finished.bool() if as_bool else finished, pad=pad)
    # most beams at their end, a few continuations left: nothing but them and the padding counts
    many = torch.ones(6, 16, device=DEV, dtype=torch.uint8)
    many[:, 3], many[0, 11] = 0, 0
    for V, take in ((6213, 32), (6213, 9), (90, 64), (20000, 17)):
        _check_beams(_randn(V, 6, 16, V).half(), -3 * torch.rand(6, 16, device=DEV, generator=_gen(V)), take, finished=many, pad=V - 1)
    short = _randn(10, 1, 2, 3)
    for pad in range(3):
        _check_beams(short, torch.zeros(1, 2, device=DEV), 6, finished=torch.tensor([[1, 0]], dtype=torch.uint8, device=DEV), pad=pad)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_beam_select_rows_at_any_alignment(dtype):
    store = _randn(4, 2, 3, 1037).to(dtype)
    for off, V in ((0, 1037), (1, 1036), (3, 1001), (5, 1030), (7, 9)):
        _check_beams(store[:, :, off:off + V], torch.zeros(2, 3, device=DEV), 6)


def test_beam_select_on_another_stream_and_replayed():
    logits, scores = _randn(12, 2, 4, 50257), -torch.rand(2, 4, device=DEV, generator=_gen(4))
    want = [torch.from_numpy(t) for t in _check_beams(logits, scores, 8)]
    out = [torch.zeros(2, 8, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kf.kf_beam_select(logits=logits, scores=scores, out_scores=out[0], out_parent=out[1], out_token=out[2], stream=side)
    side.synchronize()
    assert all(torch.equal(a.cpu(), b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kf.kf_beam_select(logits=logits, scores=scores, out_scores=out[0], out_parent=out[1], out_token=out[2])
    logits.copy_(logits.flip(-1).clone())
    graph.replay()
    torch.cuda.synchronize()
    flipped = _check_beams(logits, scores, 8)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, flipped))
    del graph


@pytest.mark.parametrize("batch,beams", [(1, 1), (3, 2), (2, 4), (2, 5), (1, 16), (2, 32)])
def test_reorder_rows(batch, beams):
    g = _gen(batch + beams)
    parent = torch.randint(0, beams, (batch, beams), device=DEV, generator=g, dtype=torch.int32)
    parent[0] = torch.arange(beams - 1, -1, -1, device=DEV)                                  # all rows swap places
    n = batch * beams
    store = torch.randint(0, 255, (n * 1003 + 1,), device=DEV, dtype=torch.uint8, generator=g)
    bufs = [torch.randint(0, 255, (n, 7, 160), device=DEV, dtype=torch.uint8, generator=g), torch.randn(n, 5, device=DEV, generator=g),
            torch.randint(0, 99, (n,), device=DEV, dtype=torch.int32, generator=g), store[1:].view(n, 1003),        # odd rows at an odd address
            torch.randn(n, 30000, device=DEV, generator=g).half(), torch.randint(0, 255, (n, 1), device=DEV, dtype=torch.uint8, generator=g)]
    index = (parent.long() + torch.arange(batch, device=DEV)[:, None] * beams).flatten()
    want = [t[index] for t in bufs]
    kf.kf_reorder_rows(buffers=bufs, parent=parent)
    for i, (a, b) in enumerate(zip(bufs, want)):
        assert torch.equal(a, b), i


def test_reorder_rows_of_several_layers_and_stray_parents():
    a, b = _randn(1, 3, 8, 2, 33), torch.arange(24, device=DEV, dtype=torch.int32).view(3, 8)
    parent = torch.tensor([[1, -1, 4, 0], [7, 3, 2, 1]], dtype=torch.int32, device=DEV)      # -1, 4, 7: outside, left as they are
    index = torch.tensor([1, 1, 2, 0, 4, 7, 6, 5], device=DEV)
    want = [t[:, index].clone() for t in (a, b)]
    kf.kf_reorder_rows(buffers=[a, b], parent=parent, n_layers=3)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.parametrize("new_pos", [False, True])
def test_reorder_beams_of_a_context(new_pos):
    """Two requests of two beams: after the reordering every beam generates what its parent would have."""
    wl = W.Workload("beams", 2, 4, 2, 64, 70, 40, 8, 8, data_seed=2, noise_seed=5, positional="alibi")
    kw = dict(noise_mode=kf.KF_NOISE_NONE, pos_mode=kf.KF_POS_NEW if new_pos else kf.KF_POS_ORIGINAL)     # no noise: a beam's index does not matter
    gpu, plain = lockstep.make_gpu(wl, **kw), lockstep.make_gpu(wl, **kw)
    parent = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device=DEV)
    index = torch.tensor([1, 0, 3, 3], device=DEV)
    with pytest.raises(kf.KeyformerError):
        gpu.kf_reorder_beams(0, parent)                     # before the prompt phase
    for layer in range(2):
        prompt = W.make_prompt(wl, layer, DEV)
        gpu.kf_prefill_score_prune(layer, *prompt)
        plain.kf_prefill_score_prune(layer, *prompt)
    for step in range(1, 3):
        for layer in range(2):
            q, kn, vn = W.make_step(wl, layer, step, DEV)
            gpu.kf_decode_step(layer, step, q, kn, vn, torch.empty_like(q))
            plain.kf_decode_step(layer, step, q, kn, vn, torch.empty_like(q))
    launches = gpu.kf_launch_count()
    gpu.kf_reorder_beams(-1, parent)
    assert gpu.kf_launch_count() == launches + 1
    for layer in range(2):
        for mine, other in zip(gpu.kf_view_state(layer), plain.kf_view_state(layer)):
            assert torch.equal(mine, other[index])
        if new_pos:
            assert torch.equal(gpu.kf_view_place(layer), plain.kf_view_place(layer)[index])
    gpu.kf_reorder_beams(1, parent)                         # one layer alone: the swapped pair swaps back
    assert torch.equal(gpu.kf_view_state(1)[2], plain.kf_view_state(1)[2][index][index])
    assert torch.equal(gpu.kf_view_state(0)[2], plain.kf_view_state(0)[2][index])
    q, kn, vn = W.make_step(wl, 0, 3, DEV)
    a, b = torch.empty_like(q), torch.empty_like(q)
    gpu.kf_decode_step(0, 3, q[index].contiguous(), kn[index].contiguous(), vn[index].contiguous(), a)
    plain.kf_decode_step(0, 3, q, kn, vn, b)
    assert torch.equal(a, b[index])
    for bad in (torch.zeros(1, 3, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError):
            gpu.kf_reorder_beams(0, bad)
    lockstep.check_guards(gpu)
    lockstep.check_guards(plain)


# ------------------------------------------------------------------------------------------------ as they are used together

def test_beam_search_over_four_bit_caches():
    """A model of one attention layer generates with four beams for two requests: projection -> norm and rotation -> step over the 4-bit cache ->
    logits -> selection -> reordering.  Every stage is compared with its plain form on the inputs it was given."""
    B, beams, H, kv, d, V, k, w = 2, 4, 8, 2, 64, 999, 60, 16
    rows = B * beams
    s = Packed(rows, H, kv, d, k, w, lengths=[60, 44, 60, 59], seed=21)
    embed = _randn(1, V, (H + 2 * kv) * d).bfloat16()
    head = (_randn(2, H * d, V) * 0.1).half()
    qw, kw = (1 + 0.2 * _randn(3, d)).bfloat16(), (1 + 0.2 * _randn(4, d)).bfloat16()
    scores = torch.zeros(B, beams, device=DEV)
    scores[:, 1:] = -float("inf")
    tokens = torch.zeros(B, beams, dtype=torch.int32, device=DEV)
    finished = torch.zeros(B, beams, dtype=torch.uint8, device=DEV)
    eos = 5
    for step in range(1, 7):
        qkv = embed[tokens.flatten().long()].unsqueeze(1)
        q, kn, vn = (torch.empty(rows, h, d, dtype=torch.float16, device=DEV) for h in (H, kv, kv))
        kf.kf_qk_norm_rotate(qkv=qkv, n_heads=H, n_kv_heads=kv, head_dim=d, q=q, k=kn, v=vn, position0=s.n + step - 1, norm_mode=kf.KF_NORM_RMS,
                             q_weight=qw, k_weight=kw, rotary_dims=32)
        want = ref.norm_rotate(qkv.double().cpu().numpy(), H, kv, d, np.full((rows, 1), s.n + step - 1), qw.double().cpu().numpy(), kw.double().cpu().numpy(), True,
                               np.float64(np.float32(1e-6)), 32, 10000.0, False)
        for got, expect in zip((q, kn, vn), want):
            expect = expect[:, :, 0]
            assert (np.abs(got.double().cpu().numpy() - expect) <= U16 * np.abs(expect) + 2.0 ** -20 * np.abs(expect).max(-1, keepdims=True)).all()
        s.inputs = lambda _, now=(q, kn, vn): now
        outs = []
        call = s.call
        s.call = lambda *a, **kw_: outs.append(call(*a, **kw_)) or outs[-1]
        s.step(step)                                        # with the oracle
        s.call = call
        logits = (outs[0][0].view(rows, H * d) @ head).view(B, beams, V)
        new_scores, parent, token = _check_beams(logits, scores, beams, finished=finished, pad=eos)
        parent, tokens = torch.from_numpy(parent).to(DEV), torch.from_numpy(token).to(DEV)
        scores = torch.from_numpy(new_scores).to(DEV)
        finished = torch.gather(finished, 1, parent.long()) | (tokens == eos).to(torch.uint8)
        index = (parent.long() + torch.arange(B, device=DEV)[:, None] * beams).flatten()
        state = [t.view(rows, kv, *t.shape[1:]) for t in (s.cache, s.pos, s.acc, s.length)]
        expect = [t[index].clone() for t in state]
        kf.kf_reorder_rows(buffers=state, parent=parent)
        assert all(torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float())) for a, b in zip(state, expect))


def test_operators_refuse_what_does_not_fit():
    t = lambda *s, dt=torch.float16: torch.zeros(*s, dtype=dt, device=DEV)                  # noqa: E731
    u8, i32 = torch.uint8, torch.int32
    for bad in (dict(V=t(2, 3, 128)), dict(cache=t(2, 3, 160, dt=u8)), dict(cache=t(2, 2, 80, dt=u8)), dict(K=t(2, 3, 64, dt=torch.float32)), dict(length=t(3, dt=i32)),
                dict(K=t(2, 64, 3).transpose(1, 2)), dict(V=torch.zeros(2, 3, 64, dtype=torch.float16))):
        with pytest.raises((ValueError, kf.KeyformerError)):
            kf.kf_pack_cache(**{**dict(K=t(2, 3, 64), V=t(2, 3, 64), cache=t(2, 3, 80, dt=u8)), **bad})
    for bad in (dict(qkv=t(2, 4 * 64)), dict(qkv=t(1, 2, 4 * 64, dt=torch.float32)), dict(q=t(1, 2, 2, 32)), dict(positions=t(3, dt=i32)), dict(q_weight=t(64, dt=torch.bfloat16)),
                dict(rotary_dims=24), dict(qkv=t(1, 2, 4 * 64 + 4)[..., :256])):
        with pytest.raises((ValueError, kf.KeyformerError)):
            kf.kf_qk_norm_rotate(**{**dict(qkv=t(1, 2, 4 * 64), n_heads=2, n_kv_heads=1, head_dim=64, q=t(1, 2, 2, 64), k=t(1, 1, 2, 64), norm_mode=kf.KF_NORM_RMS), **bad})
    good = dict(logits=t(2, 3, 50), scores=t(2, 3, dt=torch.float32), out_scores=t(2, 4, dt=torch.float32), out_parent=t(2, 4, dt=i32), out_token=t(2, 4, dt=i32))
    for bad in (dict(logits=t(2, 3, 50, dt=torch.float64)), dict(logits=t(2, 50, 3).transpose(1, 2)), dict(scores=t(2, 2, dt=torch.float32)), dict(out_token=t(2, 4)),
                dict(pad_token=50), dict(scratch=t(16, dt=u8)), dict(logits=t(2, 6, 50)[:, :3])):
        with pytest.raises((ValueError, kf.KeyformerError)):
            kf.kf_beam_select(**{**good, **bad})
    for bad in (dict(buffers=[t(5, 3)]), dict(buffers=[t(6, 4)[:, :3]]), dict(parent=t(6, dt=i32)), dict(buffers=[]), dict(buffers=[t(6, 3)] * 9), dict(parent=t(2, 3)),
                dict(buffers=[t(6, 3)], n_layers=2)):
        with pytest.raises((ValueError, kf.KeyformerError)):
            kf.kf_reorder_rows(**{**dict(buffers=[t(6, 3)], parent=t(2, 3, dt=i32)), **bad})
    s = Packed(1, 2, 2, 64, 8, 2)
    for bad in (dict(scratch=t(256, dt=u8)),):
        with pytest.raises(kf.KeyformerError) as e:
            s.call(1, *s.inputs(1), **bad)
        assert e.value.code == kf.KF_ENOSPC
