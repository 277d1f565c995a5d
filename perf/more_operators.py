"""The operators of ragged batches over paged 8-bit caches, as they are timed and checked: their inputs, their plain forms and their exact values.

Five operators in the order in which a program that serves sequences of different lengths meets them:

  ragged    causal attention over prompts of different lengths, one after the other without padding (kf_prefill_attend_ragged)
  write     rows of new tokens into pages held in 8 bits, and back (kf_pages_write, kf_pages_read)
  attend    one token of every sequence over its pages (kf_pages_attend)
  update    sequences forked, ended and grown: tables, reference counts, copies of pages that are filled in part (kf_pages_update)
  compact   the rows that a selection kept, per head, into new pages (kf_pages_compact)

A cache is int8 [pages][key/value heads][2: K, V][page][dim] with one binary32 scale per (page, head, K or V); a value is code times scale.
A case is a dict of plain values; ``run`` makes one pass, in elementary torch operations (``own`` false) or through the library's
calls (``own`` true).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
LOWEST = -120       # exponent of the scale of a page that holds zeros only


def _two_to(e):
    """2^e for whole numbers e from -160 to 160 (binary64), without a rounding of an exponential."""
    return torch.tensor([2.0 ** i for i in range(-160, 161)], device=e.device, dtype=torch.float64)[e.long() + 160]


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # short requests that arrived together, grouped heads, queries, keys and values still side by side in their projection's rows
        dict(name="ragged_short", op="ragged", sequences=48, longest=97, spread=True, heads=32, kv_heads=8, dim=128, dtype="bf16", fused=True, alibi=False),
        # an MPT-like layer over prompts of every length, ALiBi in the logits, head-major rows as the norm and rotation leave them
        dict(name="ragged_mpt", op="ragged", sequences=6, longest=4096, spread=True, heads=32, kv_heads=32, dim=128, dtype="fp16", fused=False, alibi=True),
        # two long documents
        dict(name="ragged_long", op="ragged", sequences=2, longest=8192, spread=False, heads=32, kv_heads=8, dim=128, dtype="bf16", fused=True, alibi=False),
        # one generated token of 64 running sequences, at any place of a page
        dict(name="write_token", op="write", sequences=64, longest=1, spread=False, before=700, heads=8, dim=128, page=16, dtype="bf16"),
        # a batch of prompts behind prefixes that are there already, one cache per head
        dict(name="write_prompts", op="write", sequences=8, longest=4096, spread=True, before=333, heads=32, dim=128, page=64, dtype="fp16"),
        # three conversations of a small model with eight query heads per cache: latency only
        dict(name="attend_few", op="attend", sequences=3, longest=301, spread=True, heads=32, kv_heads=4, dim=64, page=16, dtype="bf16", alibi=False),
        # 48 sequences from one token to 8192, 32 query heads on 8 caches
        dict(name="attend_gqa", op="attend", sequences=48, longest=8192, spread=True, heads=32, kv_heads=8, dim=128, page=32, dtype="bf16", alibi=False),
        # batched decoding with one cache per head and nothing dropped, ALiBi: the workload that a reduced cache is compared with
        dict(name="attend_mha", op="attend", sequences=32, longest=4096, spread=False, heads=32, kv_heads=32, dim=128, page=64, dtype="fp16", alibi=True),
        # four requests of four beams over four GPT-J-like layers, two of the beams continued from the others
        dict(name="update_beams", op="update", sequences=16, beams=4, survivors=2, ended=0, longest=1021, spread=True, heads=16, dim=256, page=16, layers=4),
        # a server's step: 256 sequences, every eighth one has ended and gives its place to a prompt
        dict(name="update_server", op="update", sequences=256, beams=1, survivors=1, ended=8, longest=2048, spread=True, heads=8, dim=128, page=16, layers=2),
        # the prompt of one GPT-J-like layer reduced to half of it
        dict(name="compact_gptj", op="compact", sequences=1, longest=2047, spread=False, heads=16, dim=256, page=16),
        # a batch of Cerebras-GPT-like prompts reduced to half
        dict(name="compact_cerebras", op="compact", sequences=16, longest=4096, spread=True, heads=32, dim=128, page=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["ragged", "ragged", "write", "attend", "attend", "update", "compact"])
    dim, page = rng.choice([64, 128, 256]), rng.choice([16, 32, 64, 128])
    sequences, kv = _log_int(rng, 1, 64), rng.choice([1, 2, 4, 8, 16])
    if op == "ragged":
        heads = kv * rng.choice([1, 2, 3, 4, 8])
        longest = _log_int(rng, 1, min(6000, int(math.sqrt(2 ** 31 / (sequences * heads)))))
        return dict(op=op, sequences=sequences, longest=longest, spread=rng.random() < 0.7, heads=heads, kv_heads=kv, dim=dim, dtype=rng.choice(["fp16", "bf16"]),
                    fused=rng.random() < 0.5, alibi=rng.random() < 0.4)
    most = 2 ** 27 // (sequences * kv * dim)
    if op == "write":
        return dict(op=op, sequences=sequences, longest=_log_int(rng, 1, min(4000, most)), spread=rng.random() < 0.7, before=rng.choice([0, 1, 15, 64, 333, 1000]),
                    heads=kv, dim=dim, page=page, dtype=rng.choice(["fp16", "bf16"]))
    if op == "attend":
        return dict(op=op, sequences=sequences, longest=_log_int(rng, 1, min(20000, 2 * most)), spread=rng.random() < 0.6, heads=kv * rng.choice([1, 2, 3, 4, 5, 8, 16]),
                    kv_heads=kv, dim=dim, page=page, dtype=rng.choice(["fp16", "bf16"]), alibi=rng.random() < 0.4)
    if op == "update":
        beams = rng.choice([1, 2, 3, 4, 8])
        sequences = beams * _log_int(rng, 1, 32)
        return dict(op=op, sequences=sequences, beams=beams, survivors=rng.randint(1, beams), ended=rng.choice([0, 0, 3, 8]),
                    longest=_log_int(rng, 1, min(4000, 2 ** 27 // (sequences * kv * dim))), spread=rng.random() < 0.7, heads=kv, dim=dim, page=page, layers=rng.choice([1, 2, 5]))
    return dict(op=op, sequences=sequences, longest=_log_int(rng, 1, min(6000, most)), spread=rng.random() < 0.7, heads=kv, dim=dim, page=page)


def _lengths(c):
    """Tokens of every sequence: all the longest, or spread from none to the longest."""
    n, longest = c["sequences"], c["longest"]
    return [longest * ((37 * i + 63) % 64) // 63 if c["spread"] else longest for i in range(n)]


def _starts(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=dev, generator=gen)     # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, device=dev, generator=gen)     # noqa: E731
    whole = lambda values: torch.tensor(values, device=dev, dtype=torch.int32)  # noqa: E731
    c = dict(case)
    return {"case": c, **globals()["_prepare_" + c["op"]](c, dev, normal, uniform, whole)}


def _slopes(c, dev):
    return torch.exp2(-8.0 * torch.arange(1, c["heads"] + 1, device=dev, dtype=torch.float32) / c["heads"]) if c["alibi"] else None


def _prepare_ragged(c, dev, normal, uniform, whole):
    H, Hkv, d, dt = c["heads"], c["kv_heads"], c["dim"], DTYPES[c["dtype"]]
    begin = _starts(_lengths(c))
    T = max(1, begin[-1])
    loud = torch.exp(0.4 * normal(Hkv, d))
    q, k, v = normal(T, H, d), normal(T, Hkv, d) * loud, normal(T, Hkv, d)
    if c["fused"]:
        rows = torch.cat([q, k, v], 1).to(dt)
        q, k, v = rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
    else:
        q, k, v = (x.transpose(0, 1).contiguous().to(dt).transpose(0, 1) for x in (q, k, v))
    return {"q": q, "k": k, "v": v, "begin": whole(begin), "slopes": _slopes(c, dev), "out": torch.zeros(T, H, d, device=dev, dtype=dt)}


def _pool(c, tokens, spare, normal, uniform, whole, dev, layers=None):
    """Pages for sequences that may hold `tokens` each, in no order: cache, scales, and the table (-1 behind a sequence's last page)."""
    page, Hkv, d = c["page"], c["heads"] if "kv_heads" not in c else c["kv_heads"], c["dim"]
    held = [-(-n // page) for n in tokens]
    pages = sum(held) + spare
    width = max(1, max(held))
    order = uniform(pages).argsort().int()
    column = torch.arange(width, device=dev)
    used = column < whole(held)[:, None]
    at = whole(_starts(held)[:-1]).long()[:, None] + column
    table = torch.where(used, order[at.clamp(max=pages - 1)], -1).int().contiguous()
    shape = (pages, Hkv, 2) if layers is None else (layers, pages, Hkv, 2)
    cache = torch.empty(*shape, page, d, device=dev, dtype=torch.int8)
    for part in cache.flatten(0, -5).split(4096) if layers is None else cache.flatten(0, 1).split(4096):
        part.copy_((35 * normal(*part.shape)).round().clamp(-127, 127))
    return cache, _two_to((uniform(*shape) * 3 - 6).floor()).float(), table


def _prepare_write(c, dev, normal, uniform, whole):
    lengths, dt, Hkv, d, page = _lengths(c), DTYPES[c["dtype"]], c["heads"], c["dim"], c["page"]
    before = [(c["before"] * (29 * i % 64 + 1)) // 64 for i in range(c["sequences"])]
    cache, scale, table = _pool(c, [a + b for a, b in zip(before, lengths)], 7, normal, uniform, whole, dev)
    begin, T = _starts(lengths), max(1, sum(lengths))
    loud = torch.exp(0.8 * normal(Hkv, d))
    from_page = [b // page * page for b in before]                             # read back from the first page that changes
    back = _starts([b + n - f for b, n, f in zip(before, lengths, from_page)])
    return {"k": (normal(T, Hkv, d) * loud).to(dt), "v": normal(T, Hkv, d).to(dt), "begin": whole(begin), "before": whole(before), "table": table,
            "cache": cache, "scale": scale, "first": whole(from_page), "back": whole(back),
            "k_out": torch.zeros(max(1, back[-1]), Hkv, d, device=dev, dtype=dt), "v_out": torch.zeros(max(1, back[-1]), Hkv, d, device=dev, dtype=dt)}


def _prepare_attend(c, dev, normal, uniform, whole):
    lengths, dt = _lengths(c), DTYPES[c["dtype"]]
    cache, scale, table = _pool(c, lengths, 7, normal, uniform, whole, dev)
    return {"q": normal(c["sequences"], c["heads"], c["dim"]).to(dt), "cache": cache, "scale": scale, "table": table, "length": whole(lengths),
            "slopes": _slopes(c, dev), "out": torch.zeros(c["sequences"], c["heads"], c["dim"], device=dev, dtype=dt)}


def _parents(c):
    """Whom every sequence continues (-1: it has ended), and how many tokens it is about to get."""
    parent, grow = [], []
    for s, n in enumerate(_lengths(c)):
        request, beam = divmod(s, c["beams"])
        ends = c["ended"] and s % c["ended"] == 1
        parent.append(-1 if ends else request * c["beams"] + (beam if beam < c["survivors"] else (beam * 7 + request) % c["survivors"]))
        grow.append(max(1, n // 3) if ends else 1)
    return parent, grow


def _prepare_update(c, dev, normal, uniform, whole):
    lengths, page = _lengths(c), c["page"]
    parent, grow = _parents(c)
    cache, scale, table = _pool(c, lengths, sum(-(-g // page) + 1 for g in grow) + 5, normal, uniform, whole, dev, layers=c["layers"])
    table = torch.cat([table, torch.full((c["sequences"], 2), -1, device=dev, dtype=torch.int32)], 1).contiguous()   # room to grow
    refs = torch.zeros(cache.shape[1], device=dev, dtype=torch.int32)
    refs[table[table >= 0].long()] = 1
    return {"cache": cache, "scale": scale, "table": table, "length": whole(lengths), "refs": refs, "parent": whole(parent), "grow": whole(grow),
            "missing": torch.zeros(1, device=dev, dtype=torch.int32)}


def _prepare_compact(c, dev, normal, uniform, whole):
    lengths, page, Hkv, S = _lengths(c), c["page"], c["heads"], c["sequences"]
    kept = [(n + 1) // 2 for n in lengths]
    cache, scale, table = _pool(c, lengths + kept, 7, normal, uniform, whole, dev)
    width = max(1, max(kept))
    order = torch.where(torch.arange(c["longest"], device=dev) < whole(lengths)[:, None, None], uniform(S, Hkv, c["longest"]), 2.0).argsort(-1)[..., :width]
    keep = torch.where(torch.arange(width, device=dev) < whole(kept)[:, None, None], order, 2 ** 30).sort(-1)[0].int().contiguous()
    back = _starts(kept)
    return {"cache": cache, "scale": scale, "table": table[:S].contiguous(), "length": whole(lengths), "keep": keep, "n_keep": whole(kept),
            "new_table": table[S:].contiguous(), "back": whole(back),
            "k_out": torch.zeros(max(1, back[-1]), Hkv, c["dim"], device=dev, dtype=torch.float16),
            "v_out": torch.zeros(max(1, back[-1]), Hkv, c["dim"], device=dev, dtype=torch.float16)}


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if own:
        import paper_2403_09054_b200 as kf
        return globals()["_own_" + state["case"]["op"]](kf, state)
    return globals()["_plain_" + state["case"]["op"]](state)


def _own_ragged(kf, s):
    kf.kf_prefill_attend_ragged(q=s["q"], k=s["k"], v=s["v"], begin=s["begin"], out=s["out"],
                                bias_mode=kf.KF_BIAS_ALIBI if s["case"]["alibi"] else kf.KF_BIAS_NONE, alibi_slopes_dev=s["slopes"])
    return {"out": s["out"]}


def _own_write(kf, s):
    kf.kf_pages_write(k=s["k"], v=s["v"], begin=s["begin"], length=s["before"], table=s["table"], cache=s["cache"], scale=s["scale"])
    kf.kf_pages_read(table=s["table"], cache=s["cache"], scale=s["scale"], begin=s["back"], first=s["first"], k=s["k_out"], v=s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"], "scale": s["scale"]}


def _own_attend(kf, s):
    kf.kf_pages_attend(q=s["q"], table=s["table"], length=s["length"], cache=s["cache"], scale=s["scale"], out=s["out"],
                       bias_mode=kf.KF_BIAS_ALIBI if s["case"]["alibi"] else kf.KF_BIAS_NONE, alibi_slopes_dev=s["slopes"])
    return {"out": s["out"]}


def _own_update(kf, s):
    kf.kf_pages_update(table=s["table"], length=s["length"], refs=s["refs"], cache=s["cache"], scale=s["scale"], parent=s["parent"], grow=s["grow"],
                       missing=s["missing"])
    return _update_outputs(s)


def _update_outputs(s):
    """The cache's bytes have only moved here: equal bytes are equal values."""
    return {n: s[n] for n in ("table", "length", "refs", "missing", "cache", "scale")}


def _own_compact(kf, s):
    kf.kf_pages_compact(cache=s["cache"], scale=s["scale"], table=s["table"], length=s["length"], keep=s["keep"], n_keep=s["n_keep"], new_table=s["new_table"])
    kf.kf_pages_read(table=s["new_table"], cache=s["cache"], scale=s["scale"], begin=s["back"], k=s["k_out"], v=s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _owner(begin, rows):
    """Of packed rows: the sequence and the place in it. Rows behind the last sequence count to the last one."""
    at = torch.arange(rows, device=begin.device)
    sequence = (torch.searchsorted(begin.long(), at, right=True) - 1).clamp(max=begin.numel() - 2)
    return sequence, at - begin.long()[sequence]


def _plain_ragged(s):
    c = s["case"]
    S, H, Hkv, d = c["sequences"], c["heads"], c["kv_heads"], c["dim"]
    begin, dev = s["begin"].long(), s["q"].device
    n = (begin[1:] - begin[:-1])
    T, longest = int(begin[-1]), max(1, int(n.max()))
    sequence, place = _owner(s["begin"], T)
    padded = lambda x, heads: torch.zeros(S, longest, heads, d, device=dev).index_put_((sequence, place), x[:T].float())   # noqa: E731
    q = padded(s["q"], H).view(S, longest, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4)                # [S, Hkv, G, n, d]
    k, v = (padded(s[x], Hkv).permute(0, 2, 1, 3)[:, :, None] for x in ("k", "v"))                  # [S, Hkv, 1, n, d]
    x = q @ k.transpose(-1, -2)
    x *= 1.0 / math.sqrt(d)
    i = torch.arange(longest, device=dev)
    if c["alibi"]:
        x -= s["slopes"].view(Hkv, -1, 1, 1) * (i[:, None] - i).float()
    x.masked_fill_(i > i[:, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    out = (x @ v / x.sum(-1, keepdim=True)).permute(0, 3, 1, 2, 4).reshape(S, longest, H, d)
    s["out"][:T] = out[sequence, place].to(s["out"].dtype)
    return {"out": s["out"]}


def _power(top):
    """The smallest power of two e with top <= 127 e, as a number; 2^LOWEST where there are zeros only."""
    m, x = torch.frexp(top)
    e = torch.where(m <= 127 / 128, x - 7, x - 6)
    return _two_to(torch.where(top > 0, e, LOWEST).clamp(min=LOWEST)).float()


def _plain_write(s):
    c = s["case"]
    page, S, cache, scale = c["page"], c["sequences"], s["cache"], s["scale"]
    dev, T = cache.device, int(s["begin"][-1])
    sequence, place = _owner(s["begin"], T)
    at = s["before"].long()[sequence] + place
    phys, row = s["table"][sequence, at // page].long(), at % page
    x = torch.stack([s["k"][:T], s["v"][:T]], 2).float()                          # [T, Hkv, 2, d]
    top = torch.zeros_like(scale).scatter_reduce_(0, phys[:, None, None].expand(-1, *scale.shape[1:]), x.abs().amax(-1), "amax")
    new = _power(top)
    # pages that hold rows already keep their scale at least, and their rows move to the new one
    grows = s["begin"][1:] > s["begin"][:-1]
    filled = s["before"].long()[grows] % page
    tail = s["table"][torch.arange(S, device=dev)[grows], (s["before"].long() // page)[grows].clamp(max=s["table"].shape[1] - 1)].long()
    tail, filled = tail[filled > 0], filled[filled > 0]
    new[tail] = torch.maximum(new[tail], scale[tail])
    moved = (cache[tail].float() * (scale[tail] / new[tail])[..., None, None]).round().to(torch.int8)
    cache[tail] = torch.where((torch.arange(page, device=dev) < filled[:, None])[:, None, None, :, None], moved, cache[tail])
    touched = torch.zeros(scale.shape[0], device=dev, dtype=torch.bool)
    touched[phys] = True
    scale.copy_(torch.where(touched[:, None, None], new, scale))
    cache[phys, :, :, row] = (x / scale[phys][..., None]).round().to(torch.int8)
    _read_plain(s, s["table"], s["back"], s["first"])
    return {"k": s["k_out"], "v": s["v_out"], "scale": scale}


def _read_plain(s, table, begin, first):
    page, T = s["case"]["page"], int(begin[-1])
    sequence, place = _owner(begin, T)
    at = place if first is None else place + first.long()[sequence]
    phys = table[sequence, at // page].long()
    values = s["cache"][phys, :, :, at % page].float() * s["scale"][phys][..., None]
    s["k_out"][:T], s["v_out"][:T] = values[:, :, 0].to(s["k_out"].dtype), values[:, :, 1].to(s["v_out"].dtype)


def _plain_attend(s):
    c = s["case"]
    S, H, Hkv, d, page = c["sequences"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    rows = s["cache"][s["table"].long().clamp(min=0)].float() * s["scale"][s["table"].long().clamp(min=0)][..., None, None]   # [S, W, Hkv, 2, page, d]
    k, v = rows.permute(3, 0, 2, 1, 4, 5).reshape(2, S, Hkv, -1, d)
    x = s["q"].float().view(S, Hkv, H // Hkv, d) @ k.transpose(-1, -2) * (1.0 / math.sqrt(d))
    at, n = torch.arange(k.shape[2], device=k.device), s["length"].long()[:, None, None, None]
    if c["alibi"]:
        x = x - s["slopes"].view(Hkv, -1, 1) * (n - 1 - at).float()
    here = at < n
    x = torch.where(here, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    weight = torch.where(here, torch.exp(x - torch.where(top.isfinite(), top, 0.0)), 0.0)
    total = weight.sum(-1, keepdim=True)
    s["out"].copy_((weight @ v / torch.where(total > 0, total, 1.0)).view(S, H, d))     # no row: zeros
    return {"out": s["out"]}


def _plain_update(s):
    c = s["case"]
    table, page, dev = s["table"].long(), c["page"], s["table"].device
    S, W = table.shape
    mine, j = torch.arange(S, device=dev), torch.arange(W, device=dev)
    alive, parent = s["parent"] >= 0, s["parent"].long().clamp(min=0)
    length = torch.where(alive, s["length"].long()[parent], 0)
    full, part = length // page, length % page
    # the first sequence that goes on from a parent keeps the page that is filled in part, the others get a copy
    first = torch.full((S,), S, device=dev).scatter_reduce_(0, parent[alive], mine[alive], "amin")
    keeps = alive & (first[parent] == mine)
    tail = (j == full[:, None]) & (part > 0)[:, None]
    stays = alive[:, None] & ((j < full[:, None]) | tail & keeps[:, None])
    old = table[parent]
    fresh = (j < ((length + s["grow"] + page - 1) // page)[:, None]) & ~stays
    refs = s["refs"] - torch.bincount(table[table >= 0], minlength=s["refs"].numel()) + torch.bincount(old[stays], minlength=s["refs"].numel())
    new = torch.where(stays, old, -1)
    free, wanted = (refs == 0).nonzero()[:, 0], fresh.nonzero()
    n = min(free.numel(), wanted.shape[0])
    new[wanted[:n, 0], wanted[:n, 1]] = free[:n]
    refs[free[:n]] = 1
    copied = tail & fresh & (new >= 0)
    source, to, rows = old[copied], new[copied], part[:, None].expand(S, W)[copied]
    here = (torch.arange(page, device=dev) < rows[:, None])[:, None, None, :, None]
    s["cache"][:, to] = torch.where(here, s["cache"][:, source], s["cache"][:, to])
    s["scale"][:, to] = s["scale"][:, source]
    s["table"].copy_(new)
    s["length"].copy_(length)
    s["refs"].copy_(refs)
    s["missing"].fill_(wanted.shape[0] - n)
    return _update_outputs(s)


def _plain_compact(s):
    c = s["case"]
    S, Hkv, page, dev = c["sequences"], c["heads"], c["page"], s["cache"].device
    W = s["new_table"].shape[1]
    j = torch.arange(W * page, device=dev)
    taken = (j < s["n_keep"][:, None])[:, None].expand(S, Hkv, -1)                # [S, Hkv, W page]
    keep = torch.zeros(S, Hkv, W * page, device=dev, dtype=torch.int64)
    keep[..., :s["keep"].shape[2]] = s["keep"]
    sequence, head, to = taken.nonzero().unbind(1)
    at = keep[taken]
    source = s["table"][sequence, at // page].long()
    codes, scale = s["cache"][source, head, :, at % page], s["scale"][source, head]        # [n, 2, d], [n, 2]
    every = torch.zeros(S, Hkv, W * page, 2, device=dev)
    every[taken] = scale
    top = every.unflatten(2, (W, page)).amax(3)                                   # [S, Hkv, W, 2]
    new = s["new_table"].long()[sequence, to // page]
    target = top[sequence, head, to // page]
    s["cache"][new, head, :, to % page] = (codes.float() * (scale / target)[..., None]).round().to(torch.int8)
    s["scale"][new, head] = target
    _read_plain(s, s["new_table"], s["back"], None)
    return {"k": s["k_out"], "v": s["v_out"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    lengths, d = _lengths(c), c["dim"]
    T = sum(lengths)
    if c["op"] == "ragged":
        return {"bytes": T * (2 * c["heads"] + 2 * c["kv_heads"]) * d * 2, "flops": 4 * d * c["heads"] * sum(n * (n + 1) // 2 for n in lengths)}
    if c["op"] == "write":     # rows in, codes out; then the pages that have changed in, their rows out
        s = [c["before"] * (29 * i % 64 + 1) // 64 % c["page"] for i in range(c["sequences"])]
        return {"bytes": 2 * c["heads"] * d * (T * 3 + (T + sum(s)) * 3), "flops": 8 * T * c["heads"] * d}
    if c["op"] == "attend":
        return {"bytes": 2 * T * c["kv_heads"] * d + 4 * c["sequences"] * c["heads"] * d, "flops": 4 * T * c["heads"] * d}
    if c["op"] == "update":    # tables and counts in and out, the rows of part-filled pages that a second sequence goes on from
        parent, _ = _parents(c)
        seen, rows = set(), 0
        for p in parent:
            rows += lengths[p] % c["page"] if p in seen else 0
            seen |= {p} - {-1}
        pages = sum(-(-n // c["page"]) for n in lengths)
        return {"bytes": 16 * pages + 4 * c["layers"] * rows * c["heads"] * d, "flops": 0}
    kept = sum((n + 1) // 2 for n in lengths)      # kept rows in and out; in again and out as 16-bit values
    return {"bytes": 2 * kept * c["heads"] * d * (1 + 1 + 1 + 2) + 4 * kept * c["heads"], "flops": 0}


# ------------------------------------------------------------------------------------------------ exact values

def exact(case, seed):
    """What run() returns the first time for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    return globals()["_exact_" + case["op"]](case, s)


def _exact_ragged(c, s):
    G, d, begin = c["heads"] // c["kv_heads"], c["dim"], s["begin"].tolist()
    out = s["out"].double()
    for a, b in zip(begin, begin[1:]):
        seen = torch.ones(b - a, b - a, device=out.device, dtype=torch.bool).tril()
        back = torch.arange(b - a, device=out.device, dtype=torch.float64)
        for h in range(c["heads"]):
            x = s["q"][a:b, h].double() @ s["k"][a:b, h // G].double().T / math.sqrt(d)
            if c["alibi"]:
                x = x + s["slopes"][h].double() * (back - back[:, None])
            out[a:b, h] = torch.softmax(torch.where(seen, x, -math.inf), -1) @ s["v"][a:b, h // G].double()
    return {"out": out}


def _exponent(top):
    """The smallest whole number e with top <= 127 * 2^e, at least LOWEST, by trial."""
    e = torch.full_like(top, LOWEST, dtype=torch.int64)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):
        e = torch.where(top > 127 * _two_to(e + step - 1), e + step, e)
    return e


def _exact_write(c, s):
    page, out = c["page"], {"k": [], "v": []}
    scale, table, before, begin = s["scale"].double(), s["table"].tolist(), s["before"].tolist(), s["begin"].tolist()
    for i in range(c["sequences"]):
        for name, side in (("k", 0), ("v", 1)):
            rows, filled = s[name][begin[i]:begin[i + 1]].double(), before[i] % page
            if not len(rows):
                held = table[i][before[i] // page] if filled else 0       # nothing new: the page is read back as it was
                out[name].append(s["cache"][held, :, side, :filled].double().transpose(0, 1) * scale[held, :, side].double()[:, None])
                continue
            pages = table[i][before[i] // page:-(-(before[i] + len(rows)) // page)]
            place = (torch.arange(len(rows), device=scale.device) + filled) // page
            e = torch.stack([_exponent(rows[place == p].abs().amax((0, 2))) for p in range(len(pages))])      # [pages, heads]
            old = s["cache"][pages[0], :, side, :filled].double().transpose(0, 1)
            was = torch.frexp(scale[pages[0], :, side]).exponent - 1
            e[0] = torch.maximum(e[0], was) if filled else e[0]
            unit = _two_to(e[place])[..., None]
            out[name] += [torch.round(old * _two_to(was - e[0])[:, None]) * _two_to(e[0])[:, None], torch.round(rows / unit) * unit]
            scale[pages, :, side] = _two_to(e)
    empty = s["k_out"][:1].double() if not s["back"][-1] else s["k_out"][:0].double()
    return {"k": torch.cat(out["k"] + [empty]), "v": torch.cat(out["v"] + [empty]), "scale": scale}


def _exact_attend(c, s):
    Hkv, d, page = c["kv_heads"], c["dim"], c["page"]
    G, out = c["heads"] // Hkv, torch.zeros(s["out"].shape, device=s["out"].device, dtype=torch.float64)
    for i, n in enumerate(_lengths(c)):
        if not n:
            continue
        pages = s["table"][i, :-(-n // page)].long()
        for h in range(Hkv):
            held = s["cache"][pages, h].double() * s["scale"][pages, h].double()[..., None, None]
            k, v = held.transpose(0, 1).reshape(2, -1, d)[:, :n]
            x = s["q"][i, h * G:(h + 1) * G].double() @ k.T / math.sqrt(d)
            if c["alibi"]:
                x = x - s["slopes"][h * G:(h + 1) * G].double()[:, None] * torch.arange(n - 1, -1, -1, device=x.device)
            out[i, h * G:(h + 1) * G] = torch.softmax(x, -1) @ v
    return {"out": out}


def _exact_update(c, s):
    page, table, refs = c["page"], s["table"].tolist(), s["refs"].tolist()
    length, parent, grow = s["length"].tolist(), s["parent"].tolist(), s["grow"].tolist()
    cache, scale, W = s["cache"].clone(), s["scale"].double(), s["table"].shape[1]
    for row in table:
        for p in row:
            refs[p] -= p >= 0
    new, lengths, kept = [], [], set()
    for s_, p in enumerate(parent):
        n = length[p] if p >= 0 else 0
        keeps = n % page > 0 and p not in kept
        row = table[p][:n // page + keeps] if p >= 0 else []
        kept |= {p} if keeps else set()
        for q in row:
            refs[q] += 1
        new.append(row)
        lengths.append(n)
    free = (p for p, r in enumerate(list(refs)) if r == 0)
    for row, n, g, p in zip(new, lengths, grow, parent):
        while len(row) < -(-(n + g) // page):
            q = next(free)
            refs[q] = 1
            if len(row) < -(-n // page):
                old = table[p][len(row)]
                cache[:, q, :, :, :n % page] = s["cache"][:, old, :, :, :n % page]
                scale[:, q] = s["scale"][:, old].double()
            row.append(q)
    whole = lambda v: torch.tensor(v, dtype=torch.int32)     # noqa: E731
    return {"table": whole([row + [-1] * (W - len(row)) for row in new]), "length": whole(lengths), "refs": whole(refs), "missing": whole([0]), "cache": cache,
            "scale": scale}


def _exact_compact(c, s):
    page, out = c["page"], {"k": [], "v": []}
    for i, n in enumerate(s["n_keep"].tolist()):
        if not n:
            continue
        at = s["keep"][i, :, :n].long()                                                    # [heads, n]
        pages, head = s["table"][i].long()[at // page], torch.arange(c["heads"], device=at.device)[:, None]
        for name, side in (("k", 0), ("v", 1)):
            unit = s["scale"][pages, head, side].double()
            value = s["cache"][pages, head, side, at % page].double() * unit[..., None]
            wide = [part.amax(1, keepdim=True).expand_as(part) for part in unit.split(page, 1)]
            wide = torch.cat(wide, 1)[..., None]
            out[name].append((torch.round(value / wide) * wide).transpose(0, 1))
    empty = s["k_out"][:1].double() if not s["back"][-1] else s["k_out"][:0].double()
    return {"k": torch.cat(out["k"] + [empty]), "v": torch.cat(out["v"] + [empty])}
