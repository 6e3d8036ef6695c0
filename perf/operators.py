"""Attention over a structured set of (query, key) pairs, as a list of cases that can be timed.

Two operators, each as a prompt, a training pass and a single-token step:

  window   softmax attention over a causal band of `window` keys and the first `sinks` keys
  decay    linear attention with one decay per head: a causal sum of outer products that fades

Tokens of all sequences lie behind one another, [tokens, heads, d]; `offsets` says where each begins.
``own`` false: plain torch operations in 32 bits; true: the calls of ``paper_2211_10482_b200``.
"""
import math
import random

import torch

own = False

# ---------------------------------------------------------------------------------------- cases


def listed():
    return [
        # one short chat turn on a small model: latency counts
        dict(name="window_turn", op="window", seqs=1, longest=197, extra=0, H=8, Hk=8, d=64, window=64, sinks=4),
        # a batch of prompts of uneven length, some of one token, behind caches of 40 tokens
        dict(name="window_prompts", op="window", seqs=12, longest=2111, extra=40, H=16, Hk=4, d=128, window=512, sinks=4),
        # one long document, long window
        dict(name="window_document", op="window", seqs=1, longest=32768, extra=0, H=16, Hk=4, d=128, window=4096, sinks=16),
        # training on packed sequences of uneven length
        dict(name="window_train", op="window_train", seqs=4, longest=4096, extra=0, H=16, Hk=4, d=128, window=1024, sinks=4),
        # training of a small model whose heads are no power of two
        dict(name="window_train_odd", op="window_train", seqs=5, longest=601, extra=0, H=6, Hk=3, d=80, window=100, sinks=1),
        # one user decoding behind a long context
        dict(name="window_step_one", op="window_step", seqs=1, longest=40000, H=16, Hk=8, d=128, window=8192, sinks=16, page=16),
        # a serving batch, caches of uneven length in pages
        dict(name="window_step_batch", op="window_step", seqs=64, longest=6000, H=32, Hk=8, d=128, window=2048, sinks=4, page=64),
        # prompts of uneven length, states carried in and out
        dict(name="decay_prompts", op="decay", seqs=9, longest=1333, H=8, dk=64, dv=64, state=True),
        # one long document: few heads, so the length has to be split
        dict(name="decay_document", op="decay", seqs=1, longest=65536, H=16, dk=128, dv=128, state=False),
        # training on packed sequences, truncated back-propagation: the state's gradient too
        dict(name="decay_train", op="decay_train", seqs=6, longest=4096, H=16, dk=128, dv=128, state=True),
        # one user decoding
        dict(name="decay_step_one", op="decay_step", seqs=1, H=16, dk=128, dv=128),
        # a serving batch
        dict(name="decay_step_batch", op="decay_step", seqs=200, H=16, dk=128, dv=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "window_train", "window_step", "decay", "decay_train", "decay_step"])
    c = dict(op=op)
    if op.startswith("window"):
        c["Hk"] = rng.choice([1, 2, 3, 4, 8])
        c["H"] = c["Hk"] * rng.choice([1, 2, 4])
        c["d"] = rng.choice([32, 64, 64, 80, 96, 128, 128])
        c["sinks"] = rng.choice([0, 1, 4, 16, 130])
        if op == "window_step":
            c["seqs"] = _log(rng, 1, 96)
            c["page"] = rng.choice([1, 16, 64, 100, 256])
            c["longest"] = _log(rng, 1, max(2, 120000 // c["seqs"]))
            c["window"] = _log(rng, 1, 8192)
        else:
            c["longest"] = _log(rng, 1, 16384 if op == "window" else 4096)
            c["seqs"] = _log(rng, 1, max(1, min(24, (16384 if op == "window" else 12288) // c["longest"])))
            c["extra"] = rng.choice([0, 0, 40, 777])
            c["window"] = _log(rng, 1, 4096 if op == "window" else 1500)
    else:
        c["H"] = rng.choice([1, 2, 4, 5, 8, 16])
        c["dk"] = rng.choice([32, 64, 80, 128, 128])
        c["dv"] = rng.choice([32, 64, 96, 128, 128])
        if op == "decay_step":
            c["seqs"] = _log(rng, 1, 200)
        else:
            c["longest"] = _log(rng, 1, 32768 if op == "decay" else 4096)
            c["seqs"] = _log(rng, 1, max(1, min(24, 32768 // c["longest"])))
            c["state"] = rng.choice([True, False])
    return c


def _lengths(case):
    """Token counts of the sequences; the first is the longest."""
    rng = random.Random(case["seqs"] * 1000003 + case.get("longest", 1))
    n = case.get("longest", 1)
    return [n] + [rng.choice([1, rng.randint(1, n), rng.randint(1, n), n]) for _ in range(case["seqs"] - 1)]


def _key_lengths(case):
    """Keys of each sequence: `extra` tokens were in its cache before."""
    return [n + case.get("extra", 0) for n in _lengths(case)]


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _pairs(lq, lk, window, sinks):
    """Visible (query, key) pairs of one sequence."""
    n = 0
    first = lk - lq
    for t in (range(first, lk) if lq < 300 else range(first, min(lk, first + window + sinks))):
        low = max(0, t - window + 1)
        n += t + 1 - low + min(low, sinks)
    rest = lk - (first + window + sinks)
    if lq >= 300 and rest > 0:
        n += rest * (window + sinks)
    return n


def work(case):
    op, lengths = case["op"], _lengths(case)
    tokens = sum(lengths)
    if op.startswith("window"):
        H, Hk, d = case["H"], case["Hk"], case["d"]
        if op == "window_step":
            rows = sum(min(n, case["window"] + case["sinks"]) for n in lengths)
            return {"bytes": 4 * rows * Hk * d + 4 * len(lengths) * (H + 2 * Hk) * d, "flops": 4 * rows * H * d}
        keys = sum(_key_lengths(case))
        pairs = sum(_pairs(q, k, case["window"], case["sinks"]) for q, k in zip(lengths, _key_lengths(case)))
        b = 4 * tokens * H * d + 4 * keys * Hk * d + 4 * tokens * H
        if op == "window":
            return {"bytes": b, "flops": 4 * pairs * H * d}
        return {"bytes": b + 4 * tokens * H * d + 4 * keys * Hk * d, "flops": 14 * pairs * H * d}
    H, dk, dv = case["H"], case["dk"], case["dv"]
    state = case["seqs"] * H * dk * dv
    if op == "decay_step":
        return {"bytes": 8 * state + 4 * case["seqs"] * H * (dk + dv), "flops": 6 * state}
    b = 4 * tokens * H * (dk + dv) + 4 * state * (2 if case["state"] else 1)
    if op == "decay":
        return {"bytes": b, "flops": 4 * tokens * H * dk * dv}
    b += 2 * tokens * H * (2 * dk + 2 * dv) + (8 * state if case["state"] else 0)
    return {"bytes": b, "flops": 14 * tokens * H * dk * dv}


# ------------------------------------------------------------------------------------- inputs


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s, op, lengths = dict(case), case["op"], _lengths(case)
    tokens, H = sum(lengths), case["H"]
    s["longest_q"] = max(lengths)
    if op == "window_step":
        Hk, d, page = case["Hk"], case["d"], case["page"]
        per = -(-max(lengths) // page)
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        first = _ints(_offsets(used)[:-1])
        slot = torch.arange(per, device="cuda", dtype=torch.int32)
        at = (first[:, None] + slot).clamp(max=pages - 1).long()
        s["table"] = torch.where(slot < _ints(used)[:, None], order[at], torch.zeros_like(order[at])).contiguous()
        s["lens"] = _ints(lengths)
        s["k_pages"], s["v_pages"] = (_normal(g, pages, page, Hk, d) for _ in range(2))
        s["q"], s["k"], s["v"] = _normal(g, case["seqs"], H, d), _normal(g, case["seqs"], Hk, d), _normal(g, case["seqs"], Hk, d)
    elif op.startswith("window"):
        Hk, d, keys = case["Hk"], case["d"], _key_lengths(case)
        s["longest_k"] = max(keys)
        s["q_offsets"], s["k_offsets"] = _ints(_offsets(lengths)), _ints(_offsets(keys))
        # one projection gives queries, keys and values where no cache lies before them: its slices have the rows' stride
        if case["extra"] == 0:
            s["q"], s["k"], s["v"] = _normal(g, tokens, H + 2 * Hk, d).split([H, Hk, Hk], 1)
        else:
            s["q"], s["k"], s["v"] = _normal(g, tokens, H, d), _normal(g, sum(keys), Hk, d), _normal(g, sum(keys), Hk, d)
        if op == "window_train":
            s["dout"] = _normal(g, tokens, H, d)
    else:
        dk, dv = case["dk"], case["dv"]
        # fixed slopes, from heads that forget within a few tokens to heads that hold hundreds
        s["log_decay"] = -torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H).float()
        n = case["seqs"] if op == "decay_step" else tokens
        s["q"], s["k"], s["v"] = _normal(g, n, H, dk), _normal(g, n, H, dk), _normal(g, n, H, dv)
        if op == "decay_step":
            s["state"] = torch.randn((n, H, dk, dv), generator=g, device="cuda")
        else:
            s["offsets"] = _ints(_offsets(lengths))
            shape = (case["seqs"], H, dk, dv)
            s["state"] = torch.randn(shape, generator=g, device="cuda") if case["state"] else None
            if op == "decay_train":
                s["dout"] = _normal(g, tokens, H, dv)
                s["dstate"] = torch.randn(shape, generator=g, device="cuda") if case["state"] else None
    return s


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ------------------------------------------------------------------------ the framework's calls


def _own_window(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_window(s["q"], s["k"], s["v"], s["window"], s["sinks"], s["q_offsets"], s["k_offsets"])


def _own_window_train(s):
    import paper_2211_10482_b200 as st
    q, k, v, mask = s["q"], s["k"], s["v"], (s["window"], s["sinks"], s["q_offsets"], s["k_offsets"])
    out, lse = st.st_attn_window(q, k, v, *mask)
    return (out, lse, *st.st_attn_window_grad(q, k, v, out, lse, s["dout"], *mask))


def _own_window_step(s):
    import paper_2211_10482_b200 as st
    out = st.st_attn_window_step(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["window"], s["sinks"])
    return out, s["k_pages"], s["v_pages"]


def _own_decay(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_decay(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], s["state"])


def _own_decay_train(s):
    import paper_2211_10482_b200 as st
    q, k, v, a, at = s["q"], s["k"], s["v"], s["log_decay"], s["offsets"]
    out, last = st.st_attn_decay(q, k, v, a, at, s["state"])
    grads = st.st_attn_decay_grad(q, k, v, a, s["dout"], at, s["state"], s["dstate"])
    return (out, last, *(grads if s["state"] is not None else grads[:3]))


def _own_decay_step(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_decay_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"]), s["state"]


_own = dict(window=_own_window, window_train=_own_window_train, window_step=_own_window_step, decay=_own_decay,
            decay_train=_own_decay_train, decay_step=_own_decay_step)

# --------------------------------------------------------------------- the plain form: window

_BLOCK = 256          # queries that share one gathered range of keys


def _blocks(s):
    """Blocks of queries with the keys that any of them sees: row of every query [B, n, i], row of every key [B, n, j],
    whether the query exists, and which pairs are visible [B, n, i, j]."""
    qo, ko = s["q_offsets"].long(), s["k_offsets"].long()
    lq, lk = (o[1:] - o[:-1] for o in (qo, ko))
    dev = qo.device
    n = -(-s["longest_q"] // _BLOCK)
    window, sinks = min(s["window"], s["longest_k"]), min(s["sinks"], s["longest_k"])
    i = torch.arange(n * _BLOCK, device=dev).view(1, n, _BLOCK)
    live = i < lq[:, None, None]
    q_row = (qo[:-1, None, None] + i).clamp(max=max(0, s["q"].shape[0] - 1))
    t = i + (lk - lq)[:, None, None]
    near = t[:, :, :1] - window + 1 + torch.arange(window + _BLOCK - 1, device=dev)
    first = torch.arange(sinks, device=dev).expand(near.shape[0], n, sinks)
    key = torch.cat([first, near], 2)
    T, K = t[..., None], key[:, :, None, :]
    is_sink = torch.arange(key.shape[2], device=dev) < sinks
    seen = torch.where(is_sink, K <= T - window, (K <= T) & (K > T - window)) & (K >= 0) & live[..., None]
    k_row = (ko[:-1, None, None] + key).clamp(0, max(0, s["k"].shape[0] - 1))
    return q_row, k_row, live, seen


def _plain_scores(s):
    q_row, k_row, live, seen = _blocks(s)
    H, Hk, d = s["H"], s["Hk"], s["d"]
    q = s["q"].float()[q_row].unflatten(3, (Hk, H // Hk))
    k, v = s["k"].float()[k_row], s["v"].float()[k_row]
    x = torch.einsum("bnihgd,bnjhd->bnhgij", q, k) / math.sqrt(d)
    x.masked_fill_(~seen[:, :, None, None], -math.inf)
    most = x.amax(-1, keepdim=True)
    p = x.sub_(most.masked_fill(most == -math.inf, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.clamp(min=1e-30))
    lse = (most + total.log()).squeeze(-1).permute(0, 1, 4, 2, 3).flatten(3)
    out = torch.einsum("bnhgij,bnjhd->bnihgd", p, v).flatten(3, 4)
    return q_row, k_row, live, q, k, v, p, out, lse


def _rows(blocks, row, live, tokens, dtype):
    """The padded blocks' rows where they lie in the packed tokens; what is padding goes to a row behind them."""
    out = torch.empty((tokens + 1, *blocks.shape[live.dim():]), dtype=dtype, device=blocks.device)
    out[torch.where(live, row, tokens)] = blocks.to(dtype)
    return out[:tokens]


def _plain_window(s):
    q_row, _, live, _, _, _, _, out, lse = _plain_scores(s)
    tokens = s["q"].shape[0]
    return _rows(out, q_row, live, tokens, torch.bfloat16), _rows(lse, q_row, live, tokens, torch.float32)


def _plain_window_train(s):
    q_row, k_row, live, q, k, v, p, out, lse = _plain_scores(s)
    scale, tokens = 1.0 / math.sqrt(s["d"]), s["q"].shape[0]
    do = (s["dout"].float()[q_row] * live[..., None, None]).unflatten(3, q.shape[3:5])
    dv = torch.einsum("bnhgij,bnihgd->bnjhd", p, do)
    ds = torch.einsum("bnihgd,bnjhd->bnhgij", do, v)
    delta = (do * out.unflatten(3, q.shape[3:5])).sum(-1).permute(0, 1, 3, 4, 2)
    ds = ds.sub_(delta[..., None]).mul_(p).mul_(scale)
    dq = torch.einsum("bnhgij,bnjhd->bnihgd", ds, k).flatten(3, 4)
    dk = torch.einsum("bnhgij,bnihgd->bnjhd", ds, q)
    at = k_row.flatten()
    dk, dv = (torch.zeros(s["k"].shape, device=at.device).index_add_(0, at, x.flatten(0, 2)).to(torch.bfloat16) for x in (dk, dv))
    o, lse, dq = (_rows(x, q_row, live, tokens, t) for x, t in ((out, torch.bfloat16), (lse, torch.float32), (dq, torch.bfloat16)))
    return o, lse, dq, dk, dv


def _plain_window_step(s):
    H, Hk, d, page = s["H"], s["Hk"], s["d"], s["page"]
    lens, table = s["lens"].long(), s["table"].long()
    seq = torch.arange(lens.numel(), device=lens.device)
    last = (lens - 1).clamp(min=0)
    at = table[seq, last // page], last % page
    s["k_pages"][at], s["v_pages"][at] = s["k"], s["v"]
    window, sinks = min(s["window"], s["longest_q"]), min(s["sinks"], s["longest_q"])
    j = torch.arange(sinks + window, device=lens.device)
    near = lens[:, None] - window + j[sinks:] - sinks
    key = torch.cat([j[:sinks].expand(lens.numel(), sinks), near], 1)
    seen = torch.where(j < sinks, key < lens[:, None] - window, key >= 0) & (key < lens[:, None])
    key = key.clamp(min=0).minimum(last[:, None])
    at = table.gather(1, key // page), key % page
    k, v = s["k_pages"][at].float(), s["v_pages"][at].float()
    q = s["q"].float().unflatten(1, (Hk, H // Hk))
    x = torch.einsum("bhgd,bjhd->bhgj", q, k) / math.sqrt(d)
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    return torch.einsum("bhgj,bjhd->bhgd", p, v).flatten(1, 2).to(torch.bfloat16), s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------------- the plain form: decay

_CHUNK = 128


def _chunks(x, row, live):
    return (x.float()[row] * live[..., None, None]).unflatten(1, (-1, _CHUNK))


def _powers(a, n):
    """exp(a n) for every head and exponent; the exponent's product in 64 bits, as positions reach far."""
    return torch.exp(a.double().view(-1, *[1] * n.dim()) * n.double()).float()


def _fade(q, k, v, a, state, scale):
    """sum_{s<=t} e^{a(t-s)} (q_t.k_s) v_s + e^{a(t+1)} q_t.state, times scale, on chunks [B, n, i, H, d]."""
    n, C = q.shape[1:3]
    i = torch.arange(C, device=q.device)
    gap = i[:, None] - i
    near = torch.where(gap >= 0, _powers(a, gap.clamp(min=0)), 0.0)
    x = torch.einsum("bnihd,bnjhd->bnhij", q, k) * near
    out = torch.einsum("bnhij,bnjhe->bnihe", x, v)
    u = torch.einsum("bnjhd,hj,bnjhe->bnhde", k, _powers(a, C - 1 - i), v)
    m = torch.arange(n, device=q.device)
    gap = m[:, None] - 1 - m
    far = torch.where(gap >= 0, _powers(a, C * gap.clamp(min=0)), 0.0)
    held = torch.einsum("hmn,bnhde->bmhde", far, u)
    if state is not None:
        held = held + torch.einsum("hm,bhde->bmhde", _powers(a, C * m), state)
    out = out + torch.einsum("bnihd,hi,bnhde->bnihe", q, _powers(a, i + 1), held)
    return (out * scale).flatten(1, 2)


def _decay_rows(s, offsets, back=False):
    """Row of every token of every sequence, padded to whole chunks; back: in reversed order."""
    length = offsets[1:] - offsets[:-1]
    i = torch.arange(-(-s["longest_q"] // _CHUNK) * _CHUNK, device=offsets.device)[None]
    live = i < length[:, None]
    at = length[:, None] - 1 - i if back else i
    return (offsets[:-1, None] + at).clamp(0, s["q"].shape[0] - 1), live, i.expand(live.shape), length


def _sum_outer(x, y, w, live):
    return torch.einsum("bthd,hbt,bthe->bhde", x, w * live, y)


def _plain_decay(s):
    a, state, tokens = s["log_decay"], s["state"], s["q"].shape[0]
    row, live, i, length = _decay_rows(s, s["offsets"].long())
    q, k, v = (_chunks(s[n], row, live) for n in "qkv")
    out = _rows(_fade(q, k, v, a, state, 1.0 / math.sqrt(s["dk"])), row, live, tokens, torch.bfloat16)
    last = _sum_outer(k.flatten(1, 2), v.flatten(1, 2), _powers(a, (length[:, None] - 1 - i).clamp(min=0)), live)
    if state is not None:
        last = last + _powers(a, length).T[..., None, None] * state
    return out, last


def _plain_decay_train(s):
    a, state, dlast, tokens, scale = s["log_decay"], s["state"], s["dstate"], s["q"].shape[0], 1.0 / math.sqrt(s["dk"])
    offsets = s["offsets"].long()
    out, last = _plain_decay(s)
    row, live, i, length = _decay_rows(s, offsets)
    q, k, v, do = (_chunks(s[n], row, live) for n in ("q", "k", "v", "dout"))
    dq = _rows(_fade(do, v, k, a, None if state is None else state.transpose(2, 3), scale), row, live, tokens, torch.bfloat16)
    first = _sum_outer(q.flatten(1, 2), do.flatten(1, 2), _powers(a, i + 1), live) * scale
    row, live, _, _ = _decay_rows(s, offsets, back=True)
    q, k, v, do = (_chunks(s[n], row, live) for n in ("q", "k", "v", "dout"))
    # what the last state's gradient brings to token s has one factor e^a less than _fade gives it, and no scale
    held = None if dlast is None else dlast * (torch.exp(-a.double()).float() / scale).view(-1, 1, 1)
    dk = _rows(_fade(v, do, q, a, None if held is None else held.transpose(2, 3), scale), row, live, tokens, torch.bfloat16)
    dv = _rows(_fade(k, q, do, a, held, scale), row, live, tokens, torch.bfloat16)
    if dlast is None:
        return out, last, dq, dk, dv
    return out, last, dq, dk, dv, first + _powers(a, length).T[..., None, None] * dlast


def _plain_decay_step(s):
    q, k, v = (s[n].float() for n in "qkv")
    state = s["state"].mul_(s["log_decay"].exp().view(-1, 1, 1)).add_(k[..., None] * v[:, :, None])
    out = torch.einsum("bhd,bhde->bhe", q, state) / math.sqrt(s["dk"])
    return out.to(torch.bfloat16), state


_plain = dict(window=_plain_window, window_train=_plain_window_train, window_step=_plain_window_step, decay=_plain_decay,
              decay_train=_plain_decay_train, decay_step=_plain_decay_step)

# ------------------------------------------------------------------- the definitions in 64 bits


def _visible(t, s, window, sinks):
    return (s <= t) & ((s > t - window) | (s < sinks))


def _softmax_rows(q, k, v, t0, window, sinks):
    """Output and log-sum-exp of queries at positions t0.. against all keys; q [i, H, d], k and v [j, Hk, d], in 64 bits."""
    g = q.shape[1] // k.shape[1]
    k, v = (x.repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))
    x = q.transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(q.shape[2])
    t = torch.arange(t0, t0 + q.shape[0], device=q.device)[:, None]
    x = x.masked_fill(~_visible(t, torch.arange(k.shape[1], device=q.device), window, sinks), -math.inf)
    lse = torch.logsumexp(x, -1)
    return (torch.exp(x - lse[..., None]) @ v).transpose(0, 1), lse.transpose(0, 1)


def _fading_rows(q, k, v, a, state, t0):
    """Queries at positions t0.. of one sequence; q [i, H, dk], k [j, H, dk], v [j, H, dv], in 64 bits."""
    t = torch.arange(t0, t0 + q.shape[0], device=q.device, dtype=torch.float64)
    gap = t[:, None] - torch.arange(k.shape[0], device=q.device)
    w = torch.where(gap >= 0, torch.exp(a.view(-1, 1, 1) * gap.clamp(min=0)), 0.0)
    out = ((q.transpose(0, 1) @ k.permute(1, 2, 0)) * w) @ v.transpose(0, 1)
    if state is not None:
        out = out + torch.exp(a[:, None] * (t + 1))[..., None] * (q.transpose(0, 1) @ state)
    return out.transpose(0, 1) / math.sqrt(q.shape[2])


def _last_state(k, v, a, state):
    n = k.shape[0]
    w = torch.exp(a * torch.arange(n - 1, -1, -1, device=k.device, dtype=torch.float64)[:, None])
    last = torch.einsum("thd,th,the->hde", k, w, v)
    return last if state is None else last + torch.exp(a * n).view(-1, 1, 1) * state


def exact(case, seed):
    s, op, lengths = prepare(case, seed), case["op"], _lengths(case)
    wide = {n: x.double() for n, x in s.items() if isinstance(x, torch.Tensor) and x.is_floating_point() and "pages" not in n}
    if op == "window_step":
        outs = []
        for b, n in enumerate(lengths):
            rows = s["table"][b].long().repeat_interleave(case["page"])[:n], torch.arange(n, device="cuda") % case["page"]
            s["k_pages"][rows[0][-1], rows[1][-1]], s["v_pages"][rows[0][-1], rows[1][-1]] = s["k"][b], s["v"][b]
            k, v = s["k_pages"][rows].double(), s["v_pages"][rows].double()
            outs.append(_softmax_rows(wide["q"][b : b + 1], k, v, n - 1, case["window"], case["sinks"])[0])
        return torch.cat(outs), s["k_pages"], s["v_pages"]
    if op == "decay_step":
        state = wide["state"] * torch.exp(wide["log_decay"]).view(-1, 1, 1) + wide["k"][..., None] * wide["v"][:, :, None]
        return torch.einsum("bhd,bhde->bhe", wide["q"], state) / math.sqrt(case["dk"]), state
    train, q_at = op.endswith("train"), _offsets(lengths)
    if train and sum(n * n for n in lengths) * case["H"] > 3e9:
        return None
    k_at = _offsets(_key_lengths(case)) if op.startswith("window") else q_at
    parts = []
    for b, n in enumerate(lengths):
        q, k, v = wide["q"][q_at[b] : q_at[b + 1]], wide["k"][k_at[b] : k_at[b + 1]], wide["v"][k_at[b] : k_at[b + 1]]
        leaves = [q, k, v]
        state = wide["state"][b] if wide.get("state") is not None else None
        if state is not None:
            leaves.append(state)
        if train:
            leaves = [x.clone().requires_grad_() for x in leaves]
            q, k, v, state = (*leaves, None)[:4]
        t0, step = k.shape[0] - n, n if train else max(64, int(2e8) // (case["H"] * k.shape[0]))
        got = []
        for i in range(0, n, step):
            rows = q[i : i + step]
            end = t0 + i + rows.shape[0]
            if op.startswith("window"):
                got.append(_softmax_rows(rows, k[:end], v[:end], t0 + i, case["window"], case["sinks"]))
            else:
                got.append((_fading_rows(rows, k[:end], v[:end], wide["log_decay"], state, i),))
        outs = [torch.cat(x) for x in zip(*got)]
        if op.startswith("decay"):
            outs.append(_last_state(k, v, wide["log_decay"], state)[None])
        grads = []
        if train:
            loss = (outs[0] * wide["dout"][q_at[b] : q_at[b + 1]]).sum()
            if state is not None:
                loss = loss + (outs[1][0] * wide["dstate"][b]).sum()
            loss.backward()
            grads = [x.grad for x in leaves]
            if state is not None:
                grads[3] = grads[3][None]
        parts.append([x.detach() for x in outs] + grads)
    return tuple(torch.cat(x) for x in zip(*parts))
