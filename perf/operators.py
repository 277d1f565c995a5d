"""The operators around the generation step, as they are timed and checked: their inputs, their plain forms and their exact values.

Five operators in the order in which a beam-searching model meets them for every generated token:

  norm_rotate   projection rows -> normed and rotated queries and keys and the values, head-major (kf_qk_norm_rotate)
  pack          rows of a reduced fp16 cache -> slots held in 4 bits, and back (kf_pack_cache, kf_unpack_cache)
  step          one generation step over a 4-bit cache: attend, score, accumulate, evict, replace (kf_decode_step_packed)
  select        the best continuations over beams and vocabulary (kf_beam_select)
  reorder       cache state of a beam replaced by its parent's, in place (kf_reorder_rows)

A case is a dict of plain values; ``run`` makes one pass, in elementary torch operations (``own`` false) or through the
library's calls (``own`` true).
"""
from __future__ import annotations

import functools
import math

import torch

own = False

GROUP = 32          # features that share a scale and a minimum in a 4-bit row
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # projection of one token of 32 running sequences, queries and keys normed and half of the features rotated in interleaved pairs
        dict(name="norm_rotate_token", op="norm_rotate", batch=32, tokens=1, heads=32, kv_heads=8, dim=128, dtype="bf16", rotary=64, halves=False, norm=True),
        # a batch of 4k prompts on the way to the prompt phase, rotation of whole heads in halves
        dict(name="norm_rotate_prompt", op="norm_rotate", batch=8, tokens=4096, heads=32, kv_heads=32, dim=128, dtype="fp16", rotary=128, halves=True, norm=True),
        # the reduced cache of one GPT-J-like layer after its prompt, an odd budget
        dict(name="pack_gptj_odd", op="pack", units=16, slots=1021, dim=256),
        # one Cerebras-GPT-like layer: 32 sequences x 32 heads x 2048 kept entries
        dict(name="pack_cerebras", op="pack", units=1024, slots=2048, dim=128),
        # the smallest workload: four heads, latency only
        dict(name="step_tiny", op="step", batch=1, heads=4, kv_heads=4, dim=64, budget=256, window=64, noise="gumbel", alibi=False, ragged=False),
        # one MPT-like long-context layer for one sequence, ALiBi in the logits
        dict(name="step_mpt", op="step", batch=1, heads=32, kv_heads=32, dim=128, budget=4096, window=1024, noise="gumbel", alibi=True, ragged=False),
        # 32 query heads on 8 caches, an odd budget, caches filled to different lengths (empty ones and full ones among them)
        dict(name="step_gqa8_ragged", op="step", batch=32, heads=32, kv_heads=8, dim=128, budget=1999, window=499, noise="gumbel", alibi=False, ragged=True),
        # batched decoding with one cache per head: one layer of the throughput workload
        dict(name="step_cerebras", op="step", batch=32, heads=32, kv_heads=32, dim=128, budget=2048, window=512, noise="gumbel", alibi=False, ragged=False),
        # one request with four beams
        dict(name="select_4beams", op="select", batch=1, beams=4, vocab=50257, take=8, dtype="fp32", finished=False),
        # a full batch of eight-beam requests in half precision, some beams at their end
        dict(name="select_batch", op="select", batch=32, beams=8, vocab=50400, take=16, dtype="fp16", finished=True),
        # four beams of one request, a GPT-J-like layer in 4 bits, two of them continued from the others
        dict(name="reorder_gptj", op="reorder", batch=1, beams=4, kv_heads=16, dim=256, budget=1024, survivors=2),
        # eight requests of four beams, one Cerebras-GPT-like layer in 4 bits
        dict(name="reorder_cerebras", op="reorder", batch=8, beams=4, kv_heads=32, dim=128, budget=2048, survivors=2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["norm_rotate", "pack", "step", "step", "select", "reorder"])
    dim = rng.choice([64, 128, 256])
    if op == "norm_rotate":
        group = rng.choice([1, 2, 4, 8])
        kv = rng.choice([1, 2, 4, 8])
        tokens = _log_int(rng, 1, 4096)
        return dict(op=op, batch=_log_int(rng, 1, 32) if tokens < 512 else rng.randint(1, 4), tokens=tokens, heads=kv * group, kv_heads=kv, dim=dim,
                    dtype=rng.choice(["fp16", "bf16"]), rotary=rng.choice([0, 8, 32, 64, dim]), halves=rng.random() < 0.5, norm=rng.random() < 0.8)
    if op == "pack":
        return dict(op=op, units=_log_int(rng, 1, 256), slots=_log_int(rng, 1, 4096), dim=dim)
    if op == "step":
        group, kv = rng.choice([1, 1, 2, 4, 8]), rng.choice([1, 2, 4, 8, 16])
        batch = _log_int(rng, 1, 16)
        budget = _log_int(rng, 1, min(6000, 2 ** 28 // (batch * kv * dim * max(1, group // 2))))
        return dict(op=op, batch=batch, heads=kv * group, kv_heads=kv, dim=dim, budget=budget, window=rng.choice([0, budget // 4, budget // 2, budget]),
                    noise=rng.choice(["gumbel", "gumbel", "none", "const"]), alibi=rng.random() < 0.5, ragged=rng.random() < 0.5)
    if op == "select":
        batch, beams = _log_int(rng, 1, 32), rng.choice([1, 2, 3, 4, 5, 8, 16])
        vocab = _log_int(rng, 64, min(131072, 12_000_000 // (batch * beams)))
        return dict(op=op, batch=batch, beams=beams, vocab=vocab, take=rng.choice([1, beams, 2 * beams]),
                    dtype=rng.choice(["fp16", "bf16", "fp32"]), finished=rng.random() < 0.5)
    batch, beams, kv = _log_int(rng, 1, 8), rng.choice([2, 3, 4, 5, 8]), rng.choice([1, 2, 8, 16])
    return dict(op=op, batch=batch, beams=beams, kv_heads=kv, dim=dim, budget=_log_int(rng, 1, min(4000, 2 ** 28 // (batch * beams * kv * dim))),
                survivors=rng.randint(1, beams - 1))


# ------------------------------------------------------------------------------------------------ inputs

def _pack_plain(x):
    """Rows [..., d] of binary16 values -> (codes uint8 [..., d/2], (scale, minimum) binary16 [..., d/32, 2])."""
    g = x.float().unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = _half_down((high - low) / 15.0)
    inverse = torch.where(scale > 0, 1.0 / scale.float(), torch.zeros_like(low))
    code = ((g - low) * inverse).round().clamp(0, 15).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.cat([scale, low.half()], -1)


def _half_down(x):
    """Non-negative binary32 -> the largest binary16 number that is not above it."""
    h = x.half()
    return torch.where(h.float() > x, (h.view(torch.int16) - 1).view(torch.float16), h)


def _slot_bytes(k, v):
    """Slots of a packed cache: K codes, V codes, K groups, V groups."""
    (kc, kg), (vc, vg) = _pack_plain(k), _pack_plain(v)
    return torch.cat([kc, vc, kg.flatten(-2).view(torch.uint8), vg.flatten(-2).view(torch.uint8)], -1)


def _unpack_plain(slots, d):
    """Slots [..., 5d/4] -> the K and V rows they stand for, [..., 2, d], values of binary16 held in binary32."""
    codes = slots[..., :d].unflatten(-1, (2, d // 2))
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP))
    groups = slots[..., d:].contiguous().view(torch.float16).float().unflatten(-1, (2, -1, 2))
    return (code * groups[..., :1] + groups[..., 1:]).half().float().flatten(-2)


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=dev, generator=gen)     # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, device=dev, generator=gen)     # noqa: E731
    c = dict(case)
    return {"case": c, **globals()["_prepare_" + c["op"]](c, seed, dev, normal, uniform)}


def _prepare_norm_rotate(c, seed, dev, normal, uniform):
    dt = DTYPES[c["dtype"]]
    B, n, H, Hkv, d = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
    qkv = (2.0 * normal(B, n, (H + 2 * Hkv) * d)).to(dt)
    first = (uniform(B, 1) * 100000).int()                                     # where each sequence stands in its text
    return {"qkv": qkv, "positions": (first + torch.arange(n, device=dev, dtype=torch.int32)).contiguous(),
            "q_weight": (1 + 0.2 * normal(d)).to(dt) if c["norm"] else None, "k_weight": (1 + 0.2 * normal(d)).to(dt) if c["norm"] else None,
            "q": torch.zeros(B, H, n, d, device=dev, dtype=torch.float16), "k": torch.zeros(B, Hkv, n, d, device=dev, dtype=torch.float16),
            "v": torch.zeros(B, Hkv, n, d, device=dev, dtype=torch.float16)}


def _prepare_pack(c, seed, dev, normal, uniform):
    U, k, d = c["units"], c["slots"], c["dim"]
    loud = torch.exp(0.8 * normal(U, 1, d))                                    # keys have features that are larger everywhere
    return {"K": (normal(U, k, d) * loud).half(), "V": normal(U, k, d).half(),
            "cache": torch.zeros(U, k, 5 * d // 4, device=dev, dtype=torch.uint8),
            "K_out": torch.zeros(U, k, d, device=dev, dtype=torch.float16), "V_out": torch.zeros(U, k, d, device=dev, dtype=torch.float16)}


def _lengths(units, budget, ragged):
    """Entries in use per unit: all of them, or spread from none to all."""
    return [budget * ((37 * u) % 64) // 63 if ragged else budget for u in range(units)]


def _prepare_step(c, seed, dev, normal, uniform):
    B, H, Hkv, d, k, w = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["budget"], c["window"]
    U, p = B * Hkv, 3 * k + 8
    q = normal(B, H, d)
    loud = torch.exp(0.4 * normal(U, 1, d))
    cache = _slot_bytes((normal(U, k, d) * loud).half(), normal(U, k, d).half())
    # positions: the most recent entries without gaps, the older ones with gaps, in no order of slots
    gap = 1 + (uniform(U, k) * 2.999).int()
    gap[:, max(0, k - w):] = 1
    ahead = gap.flip(1).cumsum(1).flip(1) - gap
    pos = torch.gather(p - 1 - ahead, 1, uniform(U, k).argsort(1)).int().contiguous()
    length = torch.tensor(_lengths(U, k, c["ragged"]), device=dev, dtype=torch.int32)
    used = torch.arange(k, device=dev) < length[:, None]
    slopes = torch.exp2(-8.0 * torch.arange(1, H + 1, device=dev, dtype=torch.float32) / H) if c["alibi"] else None
    return {"cache": cache, "pos": torch.where(used, pos, -1).int(), "acc": torch.where(used, torch.exp(normal(U, k)), 0.0), "length": length,
            "q": q.half(), "knew": normal(B, Hkv, d).half(), "vnew": normal(B, Hkv, d).half(), "slopes": slopes,
            "out": torch.zeros(B, H, d, device=dev, dtype=torch.float16), "score": torch.zeros(U, k + 1, device=dev),
            "slot": torch.zeros(U, device=dev, dtype=torch.int32), "row": torch.zeros(U, 2, d, device=dev, dtype=torch.float16),
            "position": p, "step": 0, "seed": seed & 0xFFFFFFFF}


def _prepare_select(c, seed, dev, normal, uniform):
    B, W, V = c["batch"], c["beams"], c["vocab"]
    logits = (3.0 * normal(B, W, V)).to(DTYPES[c["dtype"]])
    logits[uniform(B, W, V) < 0.05] = -math.inf                                # tokens that a rule has forbidden
    done = (uniform(B, W) < 0.3).to(torch.uint8) if c["finished"] else None
    return {"logits": logits, "scores": -20 * uniform(B, W), "finished": done, "pad": min(V - 1, 2),
            "out_scores": torch.zeros(B, c["take"], device=dev), "out_parent": torch.zeros(B, c["take"], device=dev, dtype=torch.int32),
            "out_token": torch.zeros(B, c["take"], device=dev, dtype=torch.int32)}


def _prepare_reorder(c, seed, dev, normal, uniform):
    B, W, Hkv, d, k, s = c["batch"], c["beams"], c["kv_heads"], c["dim"], c["budget"], c["survivors"]
    order = uniform(B, W).argsort(1)                                           # the first `survivors` of it go on, the rest adopt their state
    source = torch.gather(order, 1, (torch.arange(W, device=dev) % s).expand(B, W))
    parent = torch.empty(B, W, device=dev, dtype=torch.int64).scatter_(1, order, source).int()
    rows = (B * W, Hkv, k)
    return {"buffers": [(uniform(*rows, 5 * d // 4) * 256).to(torch.uint8), torch.exp(normal(*rows)), (uniform(*rows) * 10000).int(),
                        torch.full((B * W, Hkv), k, device=dev, dtype=torch.int32)],
            "parent": parent}


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if own:
        import paper_2403_09054_b200 as kf
        return globals()["_own_" + state["case"]["op"]](kf, state)
    return globals()["_plain_" + state["case"]["op"]](state)


def _own_norm_rotate(kf, s):
    c = s["case"]
    kf.kf_qk_norm_rotate(qkv=s["qkv"], n_heads=c["heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"], q=s["q"], k=s["k"], v=s["v"], positions=s["positions"],
                         norm_mode=kf.KF_NORM_RMS if c["norm"] else kf.KF_NORM_NONE, q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                         rotary_dims=c["rotary"], rotary_base=10000.0, rotary_style=kf.KF_ROTARY_HALVES if c["halves"] else kf.KF_ROTARY_PAIRS)
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _own_pack(kf, s):
    kf.kf_pack_cache(K=s["K"], V=s["V"], cache=s["cache"])
    kf.kf_unpack_cache(cache=s["cache"], K=s["K_out"], V=s["V_out"])
    return {"K": s["K_out"], "V": s["V_out"]}


def _advance(s):
    """The position and the temperature of the token that this pass generates."""
    s["position"], s["step"] = s["position"] + 1, s["step"] + 1
    return s["position"] - 1, 1.0 + min(s["step"], 256) / 256.0


def _own_step(kf, s):
    c = s["case"]
    position, tau = _advance(s)
    kf.kf_decode_step_packed(batch=c["batch"], n_heads=c["heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"], budget_k=c["budget"], recent_w=c["window"],
                             layer=0, position=position, tau=tau, cache=s["cache"], pos=s["pos"], acc=s["acc"], length=s["length"],
                             q=s["q"], knew=s["knew"], vnew=s["vnew"], out=s["out"], score_out=s["score"], slot_out=s["slot"], row_out=s["row"],
                             noise_seed=s["seed"], noise_mode={"gumbel": kf.KF_NOISE_GUMBEL, "none": kf.KF_NOISE_NONE, "const": kf.KF_NOISE_CONST}[c["noise"]],
                             noise_const=0.5772, bias_mode=kf.KF_BIAS_ALIBI if c["alibi"] else kf.KF_BIAS_NONE, alibi_slopes_dev=s["slopes"])
    return _step_outputs(s)


def _step_outputs(s):
    return {"out": s["out"], "score": s["score"], "slot": s["slot"], "row": s["row"], "pos": s["pos"], "acc": s["acc"], "length": s["length"]}


def _own_select(kf, s):
    kf.kf_beam_select(logits=s["logits"], scores=s["scores"], out_scores=s["out_scores"], out_parent=s["out_parent"], out_token=s["out_token"],
                      finished=s["finished"], pad_token=s["pad"])
    return {"scores": s["out_scores"], "parent": s["out_parent"], "token": s["out_token"]}


def _own_reorder(kf, s):
    kf.kf_reorder_rows(buffers=s["buffers"], parent=s["parent"])
    return _reorder_outputs(s)


def _reorder_outputs(s):
    """The cache as the values its slots stand for is what a step reads; here its bytes have only moved, and equal bytes are equal values."""
    return {"cache": s["buffers"][0], "acc": s["buffers"][1], "pos": s["buffers"][2], "length": s["buffers"][3]}


def _plain_norm_rotate(s):
    c = s["case"]
    B, n, H, Hkv, d, R = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rotary"]
    x = s["qkv"].float().view(B, n, H + 2 * Hkv, d)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s["q_weight"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s["k_weight"].float()
    if R:
        angle = s["positions"].double()[:, :, None, None] * torch.exp2(torch.arange(0, R, 2, device=x.device, dtype=torch.float64) * (-math.log2(10000.0) / R))
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = _turn(q, cos, sin, R, c["halves"]), _turn(k, cos, sin, R, c["halves"])
    for name, value in (("q", q), ("k", k), ("v", v)):
        s[name].copy_(value.transpose(1, 2))
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _turn(x, cos, sin, R, halves):
    a, b = (x[..., :R // 2], x[..., R // 2:R]) if halves else (x[..., 0:R:2], x[..., 1:R:2])
    a, b = a * cos - b * sin, a * sin + b * cos
    return torch.cat([torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2), x[..., R:]], -1)


def _plain_pack(s):
    d = s["case"]["dim"]
    s["cache"].copy_(_slot_bytes(s["K"], s["V"]))
    rows = _unpack_plain(s["cache"], d)
    s["K_out"].copy_(rows[..., 0, :])
    s["V_out"].copy_(rows[..., 1, :])
    return {"K": s["K_out"], "V": s["V_out"]}


def _mul_wide(a, m):
    """High and low 32 bits of a * m for 32-bit words held in int64."""
    low, high = (a & 0xFFFF) * m, (a >> 16) * m
    mid = (low >> 16) + (high & 0xFFFFFFFF)
    return (high >> 32 << 16) + (mid >> 16), (((mid & 0xFFFF) << 16) | (low & 0xFFFF))


def _philox_round(x, key):
    hi0, lo0 = _mul_wide(x[0], 0xD2511F53)
    hi2, lo2 = _mul_wide(x[2], 0xCD9E8D57)
    return hi2 ^ x[1] ^ key[0], lo2, hi0 ^ x[3] ^ key[1], lo0


def _gumbel_plain(seed, row, head, i, j):
    """Standard Gumbel noise of the logits (query position i, key positions j) from ten Philox rounds; counters (j / 4, i, head, row)."""
    keys = [((seed + r * 0x9E3779B9) & 0xFFFFFFFF, (r * 0xBB67AE85) & 0xFFFFFFFF) for r in range(10)]
    x = functools.reduce(_philox_round, keys, torch.broadcast_tensors(j >> 2, torch.full_like(j, i), head, row))
    word = torch.stack(torch.broadcast_tensors(*x), -1).gather(-1, (j & 3).expand_as(x[0])[..., None])[..., 0]
    u = ((word >> 9).float() + 0.5) / 8388608.0
    return -torch.log(-torch.log(u))


def _plain_step(s):
    c = s["case"]
    B, H, Hkv, d, k, w = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["budget"], c["window"]
    U, G, dev = B * Hkv, H // Hkv, s["q"].device
    p, tau = _advance(s)
    used = torch.arange(k, device=dev) < s["length"][:, None]                              # [U, k]
    rows = torch.where(used[:, None, :, None], _unpack_plain(s["cache"], d).transpose(1, 2), 0.0)   # [U, 2, k, d]
    # the new token joins as the last entry, with the row that was passed
    keys = torch.cat([rows[:, 0], s["knew"].float().view(U, 1, d)], 1)
    values = torch.cat([rows[:, 1], s["vnew"].float().view(U, 1, d)], 1)
    joined = torch.cat([used, torch.ones(U, 1, device=dev, dtype=torch.bool)], 1)[:, None]  # [U, 1, k + 1]
    pos = torch.cat([s["pos"].long(), torch.full((U, 1), p, device=dev)], 1)
    x = s["q"].float().view(U, G, d) @ keys.transpose(1, 2) * (1.0 / math.sqrt(d))
    if c["alibi"]:
        x = x - s["slopes"].view(Hkv, G).repeat(B, 1)[:, :, None] * (p - pos)[:, None].float()
    if c["noise"] == "gumbel":
        head = torch.arange(H, device=dev).view(1, Hkv, G).expand(B, Hkv, G).reshape(U, G, 1)
        row = torch.arange(B, device=dev).repeat_interleave(Hkv).view(U, 1, 1)
        y = x + _gumbel_plain(s["seed"], row, head, p, pos.clamp(min=0)[:, None])
    else:
        y = x + (0.5772 if c["noise"] == "const" else 0.0)
    x, y = (torch.where(joined, t, -math.inf) for t in (x, y / tau))
    weight = torch.exp(x - x.amax(-1, keepdim=True))
    s["out"].copy_((weight @ values / weight.sum(-1, keepdim=True)).view(B, H, d))
    z = torch.exp(y - y.amax(-1, keepdim=True))
    z = (z / z.sum(-1, keepdim=True)).mean(1)                                              # [U, k + 1], nothing behind the last entry
    # accumulate; the new token starts from nothing
    total = torch.cat([s["acc"], torch.zeros(U, 1, device=dev)], 1) + z
    s["acc"].copy_(torch.where(used, total[:, :k], s["acc"]))
    # the smallest score among the entries outside the window leaves, of equal ones the one with the higher position
    may_go = joined[:, 0] & (pos <= p - w)
    least = torch.where(may_go, total, math.inf).amin(1, keepdim=True)
    leaves = torch.where(may_go & (total == least), pos, -1).argmax(1)
    full = s["length"] >= k
    slot = torch.where(full, torch.where(leaves == k, -1, leaves), s["length"].long())
    fresh = _slot_bytes(s["knew"].view(U, d), s["vnew"].view(U, d))
    s["row"].copy_(_unpack_plain(fresh, d))
    # the score of an entry stands at its slot, that of the new token behind them
    index = torch.arange(k + 1, device=dev)
    score = torch.where(index == s["length"][:, None], z[:, k:], torch.where(index < s["length"][:, None], z, s["score"]))
    s["score"].copy_(score)
    here = torch.arange(k, device=dev) == slot[:, None]
    s["pos"].copy_(torch.where(here, p, s["pos"]))
    s["acc"].copy_(torch.where(here, z[:, k:], s["acc"]))
    s["cache"][torch.arange(U, device=dev), slot.clamp(min=0)] = torch.where(slot[:, None] >= 0, fresh, s["cache"][torch.arange(U, device=dev), slot.clamp(min=0)])
    s["slot"].copy_(slot)
    s["length"].copy_(torch.where(full, s["length"], s["length"] + 1))
    return _step_outputs(s)


def _plain_select(s):
    c = s["case"]
    V, n = c["vocab"], c["take"]
    x = s["logits"].double()                                # in 64 bits: two continuations may differ by less than 32 can tell
    x = torch.where(x.isfinite(), x, -math.inf)
    if s["finished"] is not None:                           # a beam at its end goes on with the padding token alone, at no cost
        pad = torch.where(torch.arange(V, device=x.device) == s["pad"], 0.0, -math.inf).double()
        x = torch.where(s["finished"].bool()[..., None], pad, x)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0.0)
    value = s["scores"].double()[..., None] + (x - top - torch.exp(x - top).sum(-1, keepdim=True).log())
    value = torch.where(value.isfinite(), value, -math.inf).flatten(1)
    best, at = value.sort(dim=-1, descending=True, stable=True)
    s["out_scores"].copy_(best[:, :n])
    s["out_parent"].copy_(at[:, :n] // V)
    s["out_token"].copy_(at[:, :n] % V)
    return {"scores": s["out_scores"], "parent": s["out_parent"], "token": s["out_token"]}


def _plain_reorder(s):
    B, W = s["parent"].shape
    index = (s["parent"].long() + torch.arange(B, device=s["parent"].device)[:, None] * W).flatten()
    cache, acc, pos, length = s["buffers"]
    cache.copy_(cache[index])
    acc.copy_(acc[index])
    pos.copy_(pos[index])
    length.copy_(length[index])
    return _reorder_outputs(s)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "norm_rotate":
        values = c["batch"] * c["tokens"] * (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": 4 * values + 4 * c["batch"] * c["tokens"], "flops": 6 * values}
    if c["op"] == "pack":      # rows in, slots out, slots in, rows out
        values = 2 * c["units"] * c["slots"] * c["dim"]
        return {"bytes": values * (2 + 0.625 + 0.625 + 2), "flops": 8 * values}
    if c["op"] == "step":
        units, d = c["batch"] * c["kv_heads"], c["dim"]
        entries = sum(_lengths(units, c["budget"], c["ragged"]))
        # slots, positions, scores in and out, the score of this step; the token's q, k, v and the output
        return {"bytes": entries * (1.25 * d + 4 + 8 + 4) + c["batch"] * c["heads"] * d * 4 + units * d * 8, "flops": 4 * entries * d * c["heads"] // c["kv_heads"]}
    if c["op"] == "select":
        values = c["batch"] * c["beams"] * c["vocab"]
        return {"bytes": values * (4 if c["dtype"] == "fp32" else 2) + c["batch"] * c["take"] * 12, "flops": 4 * values}
    moved = c["batch"] * (c["beams"] - c["survivors"])
    read = c["batch"] * min(c["survivors"], c["beams"] - c["survivors"])
    row = c["kv_heads"] * c["budget"] * (1.25 * c["dim"] + 8) + 4 * c["kv_heads"]
    return {"bytes": (moved + read) * row + 4 * c["batch"] * c["beams"], "flops": 0}


# ------------------------------------------------------------------------------------------------ exact values

def exact(case, seed):
    """What run() returns the first time for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    return globals()["_exact_" + case["op"]](case, s)


def _exact_norm_rotate(c, s):
    B, n, H, Hkv, d, R = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rotary"]
    x = s["qkv"].double().reshape(B, n, H + 2 * Hkv, d).permute(0, 2, 1, 3).contiguous()
    for rows, weight in ((slice(0, H), s["q_weight"]), (slice(H, H + Hkv), s["k_weight"])):
        if c["norm"]:
            x[:, rows] *= weight.double() / ((x[:, rows] ** 2).sum(-1, keepdim=True) / d + 1e-6).sqrt()
    for i in range(R // 2):                                # one pair of features after the other, as a complex number
        one, two = (i, i + R // 2) if c["halves"] else (2 * i, 2 * i + 1)
        angle = s["positions"].double() * 10000.0 ** (-2.0 * i / R)
        turned = torch.complex(x[:, :H + Hkv, :, one], x[:, :H + Hkv, :, two]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        x[:, :H + Hkv, :, one], x[:, :H + Hkv, :, two] = turned.real, turned.imag
    return {"q": x[:, :H], "k": x[:, H:H + Hkv], "v": x[:, H + Hkv:]}


def _grid(x):
    """Rows [..., d] -> the values that their 4-bit form stands for, in 64 bits."""
    g = x.double().reshape(*x.shape[:-1], -1, GROUP)
    low = g.min(-1, keepdim=True).values
    wide = (g.max(-1, keepdim=True).values - low) / 15
    # binary16 numbers below 2^-14 are multiples of 2^-24, the others have eleven significant bits
    unit = torch.exp2(torch.clamp(torch.frexp(wide)[1].double() - 11, min=-24.0))
    step = torch.floor(wide.float().double() / unit) * unit
    # the code is decided in binary32: both sides of a border have to agree on it
    code = torch.round((g.float() - low.float()) * torch.where(step > 0, 1 / step.float(), torch.zeros_like(low).float())).clamp(0, 15)
    return (code.double() * step + low).to(torch.float16).double().reshape(x.shape)


def _exact_pack(c, s):
    out = {}
    for name in ("K", "V"):
        out[name] = torch.cat([_grid(part) for part in s[name].split(64)])
    return out


def _exact_noise(c, seed, b, h, i, j):
    """Standard Gumbel variates from the counter-based generator, for one (row, head), on 64-bit words of the host."""
    import numpy as np
    j = np.asarray(j, dtype=np.uint64)
    x = [j >> np.uint64(2), np.full_like(j, i), np.full_like(j, h), np.full_like(j, b)]
    k0, k1, low = seed, 0, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(q >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), q & low, (p >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    word = np.choose((j & np.uint64(3)).astype(np.int64), x)
    return -np.log(-np.log(((word >> np.uint64(9)).astype(np.float64) + 0.5) / 2.0 ** 23))


def _exact_step(c, s):
    B, H, Hkv, d, k, w = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["budget"], c["window"]
    G, dev, p, tau = H // Hkv, s["q"].device, s["position"], 1.0 + 1.0 / 256.0
    lens, pos_all, acc_all = s["length"].tolist(), s["pos"].cpu(), s["acc"].double()
    out, score, acc = torch.zeros(B, H, d, device=dev, dtype=torch.float64), s["score"].double(), acc_all.clone()
    pos, slots, rows = pos_all.clone(), [], torch.zeros(B * Hkv, 2, d, device=dev, dtype=torch.float64)
    for u, n in enumerate(lens):
        b, hk = divmod(u, Hkv)
        kn, vn = s["knew"][b, hk], s["vnew"][b, hk]
        raw = s["cache"][u, :n]
        code = torch.stack([raw[:, :d] % 16, raw[:, :d] // 16], -1).reshape(n, 2, d // GROUP, GROUP).double()
        params = raw[:, d:].contiguous().view(torch.float16).double().reshape(n, 2, d // GROUP, 2)
        held = (code * params[..., :1] + params[..., 1:]).to(torch.float16).double().reshape(n, 2, d)
        keys, values = torch.cat([held[:, 0], kn.double()[None]]), torch.cat([held[:, 1], vn.double()[None]])
        at = pos_all[u, :n].tolist() + [p]
        x = s["q"][b, hk * G:(hk + 1) * G].double() @ keys.T / math.sqrt(d)
        if c["alibi"]:
            x = x - s["slopes"][hk * G:(hk + 1) * G].double()[:, None] * (p - torch.tensor(at, device=dev, dtype=torch.float64))
        noise = 0.5772 if c["noise"] == "const" else 0.0
        if c["noise"] == "gumbel":
            noise = torch.stack([torch.from_numpy(_exact_noise(c, s["seed"], b, hk * G + g, p, at)) for g in range(G)]).to(dev)
        out[b, hk * G:(hk + 1) * G] = torch.softmax(x, -1) @ values
        z = torch.softmax((x + noise) / tau, -1).mean(0)
        score[u, :n + 1] = z
        acc[u, :n] += z[:n]
        slot = n
        if n == k:
            total = torch.cat([acc[u], z[n:]]).tolist()
            slot = min((total[j], -at[j], j) for j in range(n + 1) if at[j] <= p - w)[2]
            slot = -1 if slot == n else slot
        if slot >= 0:
            pos[u, slot], acc[u, slot] = p, z[n]
        slots.append(slot)
        rows[u] = _grid(torch.stack([kn, vn]))
    return {"out": out, "score": score, "slot": torch.tensor(slots, dtype=torch.int32), "row": rows, "pos": pos, "acc": acc,
            "length": torch.tensor([min(k, n + 1) for n in lens], dtype=torch.int32)}


def _exact_select(c, s):
    V, n, out = c["vocab"], c["take"], {"scores": [], "parent": [], "token": []}
    for b in range(c["batch"]):
        value = s["logits"][b].double()
        value[~torch.isfinite(value)] = -math.inf
        for w in range(c["beams"]):
            if s["finished"] is not None and s["finished"][b, w]:
                value[w] = -math.inf
                value[w, s["pad"]] = 0.0
        value = (torch.nan_to_num(torch.log_softmax(value, -1), nan=-math.inf) + s["scores"][b].double()[:, None]).flatten().cpu()
        # the largest n by value, of equal ones the first
        border = torch.topk(value, n).values[-1]
        chosen = sorted((-float(value[i]), int(i)) for i in torch.cat([(value > border).nonzero(), (value == border).nonzero()[:n]]).flatten())[:n]
        out["scores"].append([-v for v, _ in chosen])
        out["parent"].append([i // V for _, i in chosen])
        out["token"].append([i % V for _, i in chosen])
    return {"scores": torch.tensor(out["scores"], dtype=torch.float64), "parent": torch.tensor(out["parent"], dtype=torch.int32),
            "token": torch.tensor(out["token"], dtype=torch.int32)}


def _exact_reorder(c, s):
    W, new = c["beams"], [t.clone() for t in s["buffers"]]
    for b, parents in enumerate(s["parent"].tolist()):
        for w, source in enumerate(parents):
            for to, old in zip(new, s["buffers"]):
                to[b * W + w] = old[b * W + source]
    return {"cache": new[0], "acc": new[1].double(), "pos": new[2], "length": new[3]}
