"""Measured calls of the paged key-value cache: the append of new tokens, the attention of one new token over it, and the eviction
of tokens by the attention weight that they gathered, each with its plain form.

Kinds of cases:
  attend   one new token per sequence attends to its cached tokens; with `wh` the attention weights are added up per token and
           KV head (wh = H_kv) or per token (wh = 1)
  append   new tokens enter the cache: keys rotated at their positions, values as they are
  evict    every sequence keeps `keep` tokens (per KV head where wh = H_kv): the first ones, the recent ones and those of the
           largest weights; what is kept behind slot `keep` moves into the slots that became free

The cache: pages of P tokens, rows [H_kv, d]; the pages of a sequence lie anywhere in the pool.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(name=None, **kw):
    c = dict(kind="attend", dtype="bf16", B=1, H=32, H_kv=8, d=128, P=16, len=4096, ragged=False, wh=0, joined=False, style=0, theta=10000.0)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def _append(name=None, **kw):
    c = dict(kind="append", dtype="bf16", B=1, H_kv=8, d=128, P=16, len=1000, n_tok=1, ragged=False, wh=0, joined=False, style=0, theta=10000.0)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def _evict(name=None, **kw):
    c = dict(kind="evict", dtype="bf16", B=1, H_kv=8, d=128, P=16, len=4096, keep=2048, sink=4, recent=64, ragged=False, wh=8, joined=False)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # a short conversation in full precision: launches and latency are all there is
        _attend("attend_f32_b1_333", dtype="f32", H_kv=32, len=333),
        # interactive use of a grouped-query model
        _attend("attend_b1_4k_gqa", len=4100),
        # batch serving of a 7B-class multi-head model
        _attend("attend_b16_4k_mha", B=16, H_kv=32),
        # batch serving of a grouped-query model: sequences of all lengths, keys and values in one pool
        _attend("attend_b32_gqa_ragged", B=32, P=64, len=6002, ragged=True, joined=True),
        # one very long context
        _attend("attend_b1_128k_gqa", P=128, len=131072, theta=500000.0),
        # a layer whose cache is bounded by eviction: weights per KV head
        _attend("attend_weights_b8_8k", B=8, len=8191, wh=8),
        # the same with one weight per token, small heads, pages that are no power of two
        _attend("attend_weights_joint_b3_d64", B=3, H=16, H_kv=4, d=64, P=24, len=10007, ragged=True, wh=1, style=1),
        # the new token of a large batch
        _append("append_b64", B=64, P=16, len=1000, ragged=True, wh=8),
        # a batch of prompts of different lengths
        _append("append_prompts_b6_4k", B=6, P=64, len=0, n_tok=4001, ragged=True),
        # a cache held at its bound: one token leaves at every step
        _evict("evict_step_b16", B=16, len=2049, keep=2048),
        # prompts cut down to their share, one list of tokens for all heads
        _evict("evict_prompts_b4_32k", B=4, len=32768, keep=4096, wh=1, ragged=True),
        # full precision, odd sizes, a list for each head
        _evict("evict_f32_b2_9k", dtype="f32", B=2, P=24, len=9001, keep=1003),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "evict"])
    H_kv = rng.choice([1, 4, 8, 8, 32])
    c = dict(dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), H_kv=H_kv, d=rng.choice([64, 128, 128]), P=rng.choice([1, 7, 8, 16, 16, 24, 64, 128, 256]),
             B=_log_int(rng, 1, 64), ragged=rng.random() < 0.6, wh=rng.choice([0, 1, H_kv]), joined=rng.random() < 0.4)
    room = 400_000_000 // (c["B"] * H_kv * c["d"] * (2 if c["dtype"] == "bf16" else 4))   # cached tokens of a sequence
    if kind == "attend":
        return _attend(**c, H=H_kv * rng.choice([1, 4, 4, 8] if H_kv < 32 else [1]), len=_log_int(rng, 1, min(131072, room)), style=rng.randint(0, 1),
                       theta=rng.choice([10000.0, 500000.0]))
    if kind == "append":
        n_tok = rng.choice([1, _log_int(rng, 1, max(1, min(4001, room // 16, 24000 // c["B"])))])
        return _append(**c, len=_log_int(rng, 1, max(1, min(4000, room // 8))) - 1, n_tok=n_tok, style=rng.randint(0, 1), theta=rng.choice([10000.0, 500000.0]))
    c["wh"] = rng.choice([1, H_kv])
    n = _log_int(rng, 64, max(64, min(32768, room // 4, 2_000_000 // (c["B"] * c["wh"]))))
    keep = rng.choice([n - 1, n - rng.randint(1, 32), _log_int(rng, 32, n)])
    return _evict(**c, len=n, keep=keep, sink=rng.choice([0, 4, 16]), recent=rng.choice([0, 16, min(64, keep // 2)]))


def _lengths(c):
    """Cached tokens of each sequence; in a ragged batch from len / B to len, in no order."""
    return [c["len"] * ((37 * b + c["B"] - 1) % c["B"] + 1) // c["B"] if c["ragged"] else c["len"] for b in range(c["B"])]


def _new_tokens(c):
    return [c["n_tok"] - (b * c["n_tok"] // (2 * c["B"]) if c["ragged"] else 0) for b in range(c["B"])]


class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=dtype)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV, dtype=torch.int32)


def prepare(case, seed):
    c, R = case, _Rand(seed)
    dt, B, H_kv, d, P = DTYPES[c["dtype"]], c["B"], c["H_kv"], c["d"], c["P"]
    mp = -(-(c["len"] + c.get("n_tok", 1)) // P)
    n_pages = B * mp + 3
    if c["joined"]:
        pool = R.normal(n_pages, 2, P, H_kv, d, dtype=dt)
        Kp, Vp = pool[:, 0], pool[:, 1]
    else:
        Kp, Vp = R.normal(n_pages, P, H_kv, d, dtype=dt), R.normal(n_pages, P, H_kv, d, dtype=dt)
    table = torch.randperm(n_pages, generator=R.g, device=DEV)[: B * mp].to(torch.int32).view(B, mp).contiguous()
    lens = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    cap, wh = mp * P, c["wh"]
    s = {"case": c, "Kp": Kp, "Vp": Vp, "table": table, "lens": lens, "seq_len": lens.clone(), "n_new": None, "pos": None, "weights": None}
    # tokens were evicted before: positions have gaps except among the first and the recent ones, and stand in any order
    gap = R.ints(1, 4, B, max(1, wh), cap)
    slot = torch.arange(cap, device=DEV)
    near = lens[:, None, None] - slot <= c.get("recent", 16)
    gap = torch.where((slot < 16) | near, torch.ones_like(gap), gap)
    pos = (torch.cumsum(gap, dim=-1) - 1).to(torch.int32)
    # (the newest token of every list stands at one position, the sequence's)
    newest = pos.gather(2, (lens.long() - 1).clamp(min=0)[:, None, None].expand(B, max(1, wh), 1))
    last = newest.amax(dim=1, keepdim=True)
    pos = torch.where(near, pos + (last - newest), pos)
    s["q_pos"] = last.view(B).contiguous()
    weights = torch.exp(2.0 * R.normal(B, max(1, wh), cap)) * (R.uniform(B, max(1, wh), cap) > 0.02)
    if c["kind"] == "evict":
        order = R.uniform(B, wh, cap) + torch.where(slot < 16, slot - 100.0, 0.0)
        order = torch.argsort(torch.where(slot < lens[:, None, None], order, slot.to(torch.float32) + 2), dim=-1)
        # one buffer, so that one copy takes an eviction back (data pointers are aligned to 16 bytes)
        n = B * wh * cap
        pad = torch.zeros(-n % 4, dtype=torch.int32, device=DEV)
        s["small0"] = torch.cat([weights.view(-1).view(torch.int32), pad, pos.gather(2, order).view(-1), pad, lens])
        s["small"] = s["small0"].clone()
        at = n + len(pad)
        s["weights"] = s["small"][:n].view(torch.float32).view(B, wh, cap)
        s["pos"], s["seq_len"] = s["small"][at:at + n].view(B, wh, cap), s["small"][2 * at:]
        s["src"] = torch.zeros((B, wh, c["keep"]), dtype=torch.int32, device=DEV)
    else:
        if wh:
            s["pos"], s["weights"] = pos, weights
        n_new = _new_tokens(c) if c["kind"] == "append" else [0]
        if c["kind"] == "append":
            s["k_new"], s["v_new"] = R.normal(B, c["n_tok"], H_kv, d, dtype=dt), R.normal(B, c["n_tok"], H_kv, d, dtype=dt)
            s["q_pos"] = s["q_pos"] + 1
            if c["ragged"] and c["n_tok"] > 1:
                s["n_new"] = torch.tensor(n_new, dtype=torch.int32, device=DEV)
        else:
            # (twice the keys' spread: the logits' deviation is 2)
            s["q"] = (2.0 * R.normal(B, c["H"], d)).to(dt)
            s["out"] = torch.empty((B, c["H"], d), dtype=dt, device=DEV)
    if own:   # the handle that a serving program keeps: descriptor and workspace
        from paper_2510_24273_amd import binding
        desc = binding.make_paged_desc(B, c.get("H", H_kv), H_kv, d, P, mp, n_pages, c["dtype"], weight_heads=wh, page_stride=Kp.stride(0),
                                       rope_theta=c.get("theta", 10000.0), rope_style=c.get("style", 0))
        s["cache"] = binding.Paged(desc, DEV)
    return s


def _plain_rotate(x, pos, theta, style):
    """x [..., heads, d] turned by RoPE at pos [...]; pairs (i, i + d/2), or (2i, 2i + 1)."""
    d = x.shape[-1]
    angle = pos.double()[..., None, None] * theta ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    c, s = angle.cos().float(), angle.sin().float()
    x = x.float()
    if style:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    a, b = x[..., : d // 2], x[..., d // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _plain_attend(s):
    c = s["case"]
    B, H, H_kv, d = c["B"], c["H"], c["H_kv"], c["d"]
    q = _plain_rotate(s["q"], s["q_pos"], c["theta"], c["style"]).view(B, H_kv, H // H_kv, d) * d ** -0.5
    K = s["Kp"][s["table"].long()].float().view(B, -1, H_kv, d).permute(0, 2, 3, 1).contiguous()
    logits = q @ K                                                               # [B, H_kv, group, slots]
    del K
    slot = torch.arange(logits.shape[-1], device=logits.device)
    logits = torch.where(slot < s["seq_len"][:, None, None, None], logits, -math.inf)
    m = logits.amax(dim=-1, keepdim=True)
    e = torch.exp(logits - torch.where(torch.isinf(m), 0.0, m))
    total = e.sum(dim=-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    V = s["Vp"][s["table"].long()].float().view(B, -1, H_kv, d).permute(0, 2, 1, 3).contiguous()
    out = (p @ V).view(B, H, d).to(s["out"].dtype)
    if c["wh"]:
        s["weights"] += p.sum(dim=2) if c["wh"] == H_kv else p.sum(dim=(1, 2))[:, None]
        return {"out": out, "weights": s["weights"]}
    return {"out": out}


def _run_attend(s):
    if not own:
        return _plain_attend(s)
    s["cache"].attend(s["q"], s["q_pos"], s["table"], s["Kp"], s["Vp"], s["seq_len"], s["out"], weights=s["weights"])
    return {"out": s["out"], "weights": s["weights"]} if s["case"]["wh"] else {"out": s["out"]}


def _plain_append(s):
    c = s["case"]
    B, P, n_tok = c["B"], c["P"], c["n_tok"]
    t = torch.arange(n_tok, device=DEV)
    n_new = s["n_new"].long() if s["n_new"] is not None else torch.full((B,), n_tok, device=DEV)
    pos = s["q_pos"].long()[:, None] + t
    slot = s["seq_len"].long()[:, None] + t
    k = _plain_rotate(s["k_new"], pos, c["theta"], c["style"]).to(s["Kp"].dtype)
    b, at = torch.nonzero(t < n_new[:, None], as_tuple=True)
    slot, pos = slot[b, at], pos[b, at]
    page, row = s["table"].long()[b, slot // P], slot % P
    s["Kp"][page, row] = k[b, at]
    s["Vp"][page, row] = s["v_new"][b, at]
    if c["wh"]:
        s["pos"][b, :, slot] = pos[:, None].to(torch.int32)
        s["weights"][b, :, slot] = 0.0
    s["seq_len"] += n_new.to(torch.int32)


def _run_append(s):
    # (the previous pass's tokens are taken back, as after a rejected draft of speculative decoding)
    s["seq_len"].copy_(s["lens"])
    if own:
        s["cache"].append(s["k_new"], s["v_new"], s["q_pos"], s["table"], s["Kp"], s["Vp"], s["seq_len"], n_tok=s["case"]["n_tok"], n_new=s["n_new"],
                          pos=s["pos"], weights=s["weights"])
    else:
        _plain_append(s)
    r = {"Kp": s["Kp"], "Vp": s["Vp"], "seq_len": s["seq_len"]}
    return dict(r, pos=s["pos"], weights=s["weights"]) if s["case"]["wh"] else r


def _plain_evict(s):
    c = s["case"]
    B, H_kv, P, wh, keep = c["B"], c["H_kv"], c["P"], c["wh"], c["keep"]
    cap = s["pos"].shape[-1]
    slot = torch.arange(cap, device=DEV)
    here = slot < s["seq_len"][:, None, None]
    bits = s["weights"].view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7fffffff))                     # in the order of the floats, -0 = +0
    key = torch.where(torch.isnan(s["weights"]), -(1 << 33), key)
    kept_always = (s["pos"] < c["sink"]) | (s["pos"].long() > s["q_pos"].long()[:, None, None] - c["recent"])
    key = torch.where(kept_always, 1 << 33, key)
    key = torch.where(here, key, -(1 << 34))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = torch.zeros_like(here.expand(B, wh, cap)).scatter_(2, order, True) & here
    # the i-th free slot below `keep` takes the i-th kept row behind it
    moves = kept[..., keep:]
    sources = torch.sort(torch.where(moves, slot[keep:], cap), dim=-1).values
    free = ~kept[..., :keep] & here[..., :keep]
    rank = (torch.cumsum(free, dim=-1) - 1).clamp(min=0, max=max(0, cap - keep - 1))
    src = torch.where(free, sources.gather(2, rank), slot[:keep]) if cap > keep else slot[:keep].expand(B, wh, keep).clone()
    live = here[..., :keep].expand(B, wh, keep)
    table = s["table"].long()
    src = torch.where(live, src, 0)
    b = torch.arange(B, device=DEV)[:, None, None]
    at, to = (table[b, src // P], src % P), (table[:, slot[:keep] // P][:, None].expand(B, wh, keep), (slot[:keep] % P).expand(B, wh, keep))
    put = torch.nonzero(live & (src != slot[:keep]), as_tuple=True)
    for pool in (s["Kp"], s["Vp"]):
        if wh == 1:
            pool[to[0][put], to[1][put]] = pool[at[0][put], at[1][put]]
        else:
            pool[to[0][put], to[1][put], put[1]] = pool[at[0][put], at[1][put], put[1]]
    s["weights"][..., :keep] = torch.where(live, s["weights"].gather(2, src), s["weights"][..., :keep])
    s["pos"][..., :keep] = torch.where(live, s["pos"].gather(2, src), s["pos"][..., :keep])
    s["src"].copy_(torch.where(live, src, -1))
    s["seq_len"].clamp_(max=keep)


def _run_evict(s):
    c = s["case"]
    # (the previous pass's eviction is taken back; the rows that it moved still stand where they came from)
    s["small"].copy_(s["small0"])
    if own:
        s["cache"].evict(s["q_pos"], s["table"], s["Kp"], s["Vp"], s["seq_len"], s["pos"], s["weights"], c["keep"], n_sink=c["sink"],
                         n_recent=c["recent"], src=s["src"])
    else:
        _plain_evict(s)
    return {"Kp": s["Kp"], "Vp": s["Vp"], "seq_len": s["seq_len"], "pos": s["pos"], "weights": s["weights"], "src": s["src"]}


_RUN = {"attend": _run_attend, "append": _run_append, "evict": _run_evict}


def run(state):
    return _RUN[state["case"]["kind"]](state)


def work(case):
    c = case
    e, row = (2 if c["dtype"] == "bf16" else 4), c["H_kv"] * c["d"]
    lens = _lengths(c)
    if c["kind"] == "attend":
        io = 2 * c["B"] * c["H"] * c["d"] * e
        return {"bytes": 2 * sum(lens) * row * e + io + 8 * c["wh"] * sum(lens), "flops": 4 * sum(lens) * c["H"] * c["d"]}
    if c["kind"] == "append":
        n = sum(_new_tokens(c))
        return {"bytes": 4 * n * row * e + 8 * c["wh"] * n, "flops": 3 * n * row}
    # weights, positions; of the tokens behind `keep` about as many are kept as of all that compete
    gone = [max(0, n - c["keep"]) for n in lens]
    moved = [g * max(0, c["keep"] - c["sink"] - c["recent"]) / max(1, n - c["sink"] - c["recent"]) for g, n in zip(gone, lens)]
    each = row if c["wh"] == 1 else c["d"]
    byts = c["wh"] * (8 * sum(n for n, g in zip(lens, gone) if g) + 4 * c["B"] * c["keep"] + sum(moved) * (4 * each * e + 16))
    return {"bytes": int(byts), "flops": c["wh"] * sum(lens)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------


def _turn(x, position, theta, style):
    """One row [heads, d] of doubles, as complex numbers turned by position * theta^(-2i/d)."""
    d = x.shape[-1]
    i = torch.arange(d // 2, dtype=torch.float64, device=x.device)
    w = torch.polar(torch.ones_like(i), position.double() * torch.pow(torch.tensor(theta, dtype=torch.float64, device=x.device), -2.0 * i / d))
    if style:
        return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2).contiguous()) * w).reshape(x.shape)
    z = torch.complex(x[..., : d // 2].contiguous(), x[..., d // 2:].contiguous()) * w
    return torch.cat([z.real, z.imag], dim=-1)


def _rows(pool, table, P, n):
    """The first n rows of a sequence, as doubles [n, H_kv, d]."""
    j = torch.arange(n, device=pool.device)
    return pool[table.long()[j // P], j % P].double()


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros((c["B"], c["H"], c["d"]), dtype=torch.float64, device=DEV)
    weights = s["weights"].double() if c["wh"] else None
    group = c["H"] // c["H_kv"]
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        q = _turn(s["q"][b].double(), s["q_pos"][b], c["theta"], c["style"])
        K, V = _rows(s["Kp"], s["table"][b], c["P"], n), _rows(s["Vp"], s["table"][b], c["P"], n)
        for g in range(c["H_kv"]):
            p = torch.softmax(K[:, g] @ q[g * group:(g + 1) * group].T / math.sqrt(c["d"]), dim=0)       # [n, group]
            out[b, g * group:(g + 1) * group] = p.T @ V[:, g]
            if c["wh"]:
                weights[b, g if c["wh"] == c["H_kv"] else 0, :n] += p.sum(dim=1)
    return {"out": out, "weights": weights} if c["wh"] else {"out": out}


def _exact_append(s):
    c = s["case"]
    Kp, Vp = s["Kp"].double(), s["Vp"].double()
    lens, news = _lengths(c), _new_tokens(c)
    if s["n_new"] is None:
        news = [c["n_tok"]] * c["B"]
    pos, weights = (s["pos"].clone(), s["weights"].double()) if c["wh"] else (None, None)
    for b, (n, new) in enumerate(zip(lens, news)):
        t = torch.arange(new, device=DEV)
        at = s["table"][b].long()[(n + t) // c["P"]], (n + t) % c["P"]
        Kp[at] = _turn(s["k_new"][b, :new].double(), (s["q_pos"][b] + t)[:, None, None], c["theta"], c["style"])
        Vp[at] = s["v_new"][b, :new].double()
        if c["wh"]:
            pos[b, :, n:n + new] = (s["q_pos"][b] + t).to(torch.int32)
            weights[b, :, n:n + new] = 0.0
    r = {"Kp": Kp, "Vp": Vp, "seq_len": torch.tensor([n + m for n, m in zip(lens, news)], dtype=torch.int32)}
    return dict(r, pos=pos, weights=weights) if c["wh"] else r


def _exact_evict(s):
    c = s["case"]
    Kp, Vp, pos, weights = s["Kp"].double(), s["Vp"].double(), s["pos"].clone(), s["weights"].double()
    src = torch.full((c["B"], c["wh"], c["keep"]), -1, dtype=torch.int32)
    lens = _lengths(c)
    for b, n in enumerate(lens):
        first = int(s["q_pos"][b]) - c["recent"] + 1
        for a in range(c["wh"]):
            w, p = s["weights"][b, a, :n].tolist(), s["pos"][b, a, :n].tolist()
            rank = sorted(range(n), key=lambda j: (not (p[j] < c["sink"] or p[j] >= first), -w[j], j))  # noqa: B023
            kept = set(rank[: c["keep"]])
            line = list(range(min(n, c["keep"])))
            late = iter(sorted(j for j in kept if j >= c["keep"]))
            line = [j if j in kept else next(late) for j in line]
            src[b, a, : len(line)] = torch.tensor(line, dtype=torch.int32)
            to = torch.arange(len(line), device=DEV)
            frm = torch.tensor(line, device=DEV)
            t = s["table"][b].long()
            heads = slice(None) if c["wh"] == 1 else a
            for new, old in ((Kp, s["Kp"]), (Vp, s["Vp"])):
                new[t[to // c["P"]], to % c["P"], heads] = old[t[frm // c["P"]], frm % c["P"], heads].double()
            pos[b, a, : len(line)] = s["pos"][b, a, frm]
            weights[b, a, : len(line)] = s["weights"][b, a, frm].double()
    return {"Kp": Kp, "Vp": Vp, "seq_len": torch.tensor([min(n, c["keep"]) for n in lens], dtype=torch.int32), "pos": pos, "weights": weights, "src": src}


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"attend": _exact_attend, "append": _exact_append, "evict": _exact_evict}[case["kind"]](s)
