"""Operators around attention over a cache in pages, as a list of cases that can be timed.

  rotate   RMS norms of queries and keys for each head with the position rotation in the same pass; ``rotate_train``: with its gradient
  store    new tokens of every sequence written to a cache in pages (bfloat16, or quantised to 8 or 4 bits), then all of it read back
           as rows: a piece of a prompt, before the attention that takes it
  step     attention of one token of every sequence over such a cache
  shared   the same for a batch in which groups of sequences share a long prefix

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
        # one decoding step of 48 users far into their contexts: latency counts
        dict(name="rotate_turn", op="rotate", tokens=48, H=32, Hk=8, d=128, rot=128, pairs="half", norm=True, far=200000, joined=False),
        # prompts of a model that rotates half of each head, interleaved, without norms; queries and keys are slices of one projection
        dict(name="rotate_prompts", op="rotate", tokens=12289, H=16, Hk=8, d=128, rot=64, pairs="interleaved", norm=False, far=30000, joined=True),
        # training on packed sequences, norms with weights
        dict(name="rotate_train", op="rotate_train", tokens=32768, H=16, Hk=4, d=128, rot=128, pairs="half", norm=True, far=8192, joined=False),
        # training of a small model whose heads are no power of two, rotated in part
        dict(name="rotate_train_odd", op="rotate_train", tokens=3005, H=6, Hk=3, d=80, rot=32, pairs="interleaved", norm=True, far=4096, joined=False),
        # short turns of a few chats behind what is cached, 8 bits
        dict(name="store_turns", op="store", cells=8, seqs=3, longest=57, cached=300, Hk=8, d=128, page=16),
        # a batch of prompts of uneven length, 8 bits
        dict(name="store_prompts", op="store", cells=8, seqs=12, longest=4096, cached=40, Hk=8, d=128, page=64),
        # a piece of one long prompt, everything before it read back, 4 bits
        dict(name="store_piece", op="store", cells=4, seqs=1, longest=2048, cached=60000, Hk=8, d=128, page=16),
        # one user decoding behind a long context, a window over it, 8 bits
        dict(name="step_one", op="step", cells=8, seqs=1, longest=40000, H=32, Hk=8, d=128, page=16, window=8192, sinks=16),
        # a serving batch, contexts of uneven length, 8 bits
        dict(name="step_batch", op="step", cells=8, seqs=64, longest=6000, H=32, Hk=8, d=128, page=64, window=1 << 30, sinks=0),
        # the same at 4 bits
        dict(name="step_batch_4", op="step", cells=4, seqs=64, longest=6000, H=32, Hk=8, d=128, page=64, window=1 << 30, sinks=0),
        # eight samples of one prompt
        dict(name="shared_samples", op="shared", groups=1, seqs=8, prefix=4001, own=120, H=32, Hk=8, d=128, page=16),
        # a serving batch behind two long instructions
        dict(name="shared_batch", op="shared", groups=2, seqs=128, prefix=16384, own=700, H=32, Hk=8, d=128, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    c = dict(op=rng.choice(["rotate", "rotate_train", "store", "store", "step", "step", "shared"]))
    c["Hk"] = rng.choice([1, 2, 3, 4, 8])
    c["d"] = rng.choice([32, 64, 64, 80, 96, 128, 128])
    if c["op"] in ("rotate", "rotate_train"):
        c["H"] = c["Hk"] * rng.choice([1, 2, 4, 5])
        c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2, 16, 20, 2])
        c["pairs"] = rng.choice(["half", "interleaved"])
        c["norm"] = rng.choice([True, True, False])
        c["joined"] = rng.choice([True, False])
        c["far"] = _log(rng, 16, 1000000)
        c["tokens"] = _log(rng, 1, min(32768, 80000000 // ((c["H"] + c["Hk"]) * c["d"])))
    elif c["op"] == "store":
        c["cells"] = rng.choice([4, 8, 16])
        c["page"] = rng.choice([1, 16, 64, 100, 256])
        c["longest"] = _log(rng, 1, 8192)
        c["seqs"] = _log(rng, 1, max(1, min(200, 40000 // c["longest"])))
        c["cached"] = rng.choice([0, _log(rng, 1, max(1, 40000 // c["seqs"]))])
    elif c["op"] == "step":
        c["H"] = c["Hk"] * rng.choice([1, 2, 4, 8, 17])
        c["cells"] = rng.choice([4, 8, 8, 16])
        c["page"] = rng.choice([1, 16, 64, 100, 256])
        c["seqs"] = _log(rng, 1, 96)
        c["longest"] = _log(rng, 1, max(2, 200000 // c["seqs"]))
        c["window"] = rng.choice([1 << 30, _log(rng, 1, 8192)])
        c["sinks"] = rng.choice([0, 1, 4, 130])
    else:
        c["H"] = c["Hk"] * rng.choice([1, 2, 4, 8])
        c["page"] = rng.choice([1, 16, 64, 100, 256])
        c["seqs"] = _log(rng, 1, 128)
        c["groups"] = min(c["seqs"], rng.choice([1, 1, 2, 5]))
        c["prefix"] = _log(rng, 1, 16384)
        c["own"] = _log(rng, 1, 800)
    return c


def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(n, longest, rng):
    """Token counts of n sequences; the first is the longest."""
    return [longest] + [rng.choice([0, 1, rng.randint(1, longest), rng.randint(1, longest), rng.randint(1, longest), longest]) for _ in range(n - 1)]


def _shape(case):
    """What the case leaves to chance: lengths of the sequences, and of groups and their prefixes."""
    rng, op = _rng(case), case["op"]
    if op == "store":
        new = _lengths(case["seqs"], case["longest"], rng)
        return dict(new=new, lens=[n + rng.randint(0, case["cached"]) if i else n + case["cached"] for i, n in enumerate(new)])
    if op == "step":
        return dict(lens=_lengths(case["seqs"], case["longest"], rng))
    lens = [max(1, n) for n in _lengths(case["seqs"], case["own"], rng)]
    cuts = sorted(rng.sample(range(1, case["seqs"]), case["groups"] - 1))
    prefix = [case["prefix"]] + [rng.randint(case["prefix"] // 2, case["prefix"]) for _ in range(case["groups"] - 1)]
    return dict(lens=lens, groups=[0, *cuts, case["seqs"]], prefix=prefix)


def _row_bytes(case):
    """Bytes of a token's key or value of one head."""
    d = case["d"]
    return {16: 2 * d, 8: d + 4, 4: d // 2 + 4 * -(-d // 32)}[case.get("cells", 16)]


def work(case):
    op, d, Hk = case["op"], case["d"], case["Hk"]
    if op in ("rotate", "rotate_train"):
        n = case["tokens"] * (case["H"] + Hk) * d
        return {"bytes": (4 if op == "rotate" else 8) * n + 4 * case["tokens"], "flops": (8 if op == "rotate" else 24) * n}
    s = _shape(case)
    if op == "store":
        new, old = sum(s["new"]), sum(s["lens"]) - sum(s["new"])
        cells = 2 * Hk * _row_bytes(case)
        rows = 4 * Hk * d
        return {"bytes": new * (rows + cells) + old * cells + (new + old) * rows, "flops": 4 * (2 * new + old) * Hk * d}
    H = case["H"]
    if op == "step":
        keys = [min(n, case["window"] + case["sinks"]) for n in s["lens"]]
        return {"bytes": 2 * sum(keys) * Hk * _row_bytes(case) + 4 * case["seqs"] * H * d, "flops": 4 * sum(keys) * H * d}
    sizes = [b - a for a, b in zip(s["groups"], s["groups"][1:])]
    pairs = sum(n * p for n, p in zip(sizes, s["prefix"])) + sum(s["lens"])
    return {"bytes": 4 * (sum(s["prefix"]) + sum(s["lens"])) * Hk * d + 4 * case["seqs"] * H * d, "flops": 4 * pairs * H * d}


# ------------------------------------------------------------------------------------- inputs


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _keys(g, *shape):
    """Keys: some columns are much larger than the others, the same ones at every token."""
    f = 1 + 7 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.06)
    return (torch.randn(shape, generator=g, device="cuda") * f).to(torch.bfloat16)


def _frequencies(rot):
    """Base 500000, wavelengths of more than 8192 positions stretched eightfold, those below 2048 not at all."""
    f = 500000.0 ** -(torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    ramp = ((8192 / (2 * math.pi / f) - 1) / 3).clamp(0, 1)
    return (f / 8 * (1 - ramp) + f * ramp).float().cuda()


def _table(g, lens, page, pages):
    """Pages of every sequence in any order, no page in two sequences."""
    used = [-(-n // page) for n in lens]
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    slot = torch.arange(max(1, max(used)), device="cuda", dtype=torch.int32)
    at = (_ints(_offsets(used)[:-1])[:, None] + slot).clamp(max=pages - 1).long()
    return torch.where(slot < _ints(used)[:, None], order[at], torch.zeros_like(order[at])).contiguous(), sum(used), order


def _pages_for(lens, page):
    return sum(-(-n // page) for n in lens) + 3


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s, op, d, Hk = dict(case), case["op"], case["d"], case["Hk"]
    if op in ("rotate", "rotate_train"):
        n, H = case["tokens"], case["H"]
        if case["joined"]:
            s["q"], s["k"], _ = _normal(g, n, H + 2 * Hk, d).split([H, Hk, Hk], 1)
        else:
            s["q"], s["k"] = _normal(g, n, H, d), _normal(g, n, Hk, d)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device="cuda", dtype=torch.int32)
        s["freq"] = _frequencies(case["rot"])
        s["qw"], s["kw"] = ((1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16) if case["norm"] else None for _ in range(2))
        s["eps"] = 1e-6 if case["norm"] else None
        if op == "rotate_train":
            s["dq"], s["dk"] = _normal(g, n, H, d), _normal(g, n, Hk, d)
        return s
    s.update(_shape(case))
    page = case["page"]
    if op == "shared":
        everything = s["prefix"] + s["lens"]
        pages = _pages_for(everything, page)
        table, _, _ = _table(g, everything, page, pages)
        s["prefix_table"], s["table"] = table[: case["groups"]].contiguous(), table[case["groups"] :].contiguous()
        s["prefix_lens"], s["group_offsets"] = _ints(s["prefix"]), _ints(s["groups"])
    else:
        pages = _pages_for(s["lens"], page)
        s["table"], _, _ = _table(g, s["lens"], page, pages)
    s["lens_host"], s["lens"] = s["lens"], _ints(s["lens"])
    k, v = _keys(g, pages, page, Hk, d), _normal(g, pages, page, Hk, d)
    if case.get("cells", 16) == 16:
        s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"] = k, v, None, None
    else:
        s["k_pages"], s["k_scales"] = _quantise(k, case["cells"])
        s["v_pages"], s["v_scales"] = _quantise(v, case["cells"])
    if op == "store":
        new = sum(s["new"])
        s["k"], s["v"] = _keys(g, new, Hk, d), _normal(g, new, Hk, d)
        s["new_offsets"], s["all_offsets"], s["rows"] = _ints(_offsets(s["new"])), _ints(_offsets(s["lens_host"])), sum(s["lens_host"])
    else:
        s["q"] = _normal(g, case["seqs"], case["H"], d)
    return s


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ------------------------------------------------------------------------ the framework's calls


def _own_rotate(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_rotate(s["q"], s["k"], s["positions"], s["freq"], s["pairs"] == "interleaved", s["qw"], s["kw"], s["eps"])


def _own_rotate_train(s):
    import paper_2211_10482_b200 as st
    how = (s["positions"], s["freq"], s["pairs"] == "interleaved", s["qw"], s["kw"], s["eps"])
    q, k = st.st_attn_rotate(s["q"], s["k"], *how)
    grads = st.st_attn_rotate_grad(s["q"], s["k"], s["dq"], s["dk"], *how)
    return (q, k, *grads) if s["norm"] else (q, k, *grads[:2])


def _own_store(s):
    import paper_2211_10482_b200 as st
    pages = s["k_pages"], s["v_pages"], s["table"], s["lens"]
    scales = dict(k_scales=s["k_scales"], v_scales=s["v_scales"])
    st.st_attn_cache_write(s["k"], s["v"], *pages, s["new_offsets"], **scales)
    return st.st_attn_cache_read(*pages, s["all_offsets"], s["rows"], **scales)


def _own_step(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_cache_step(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["window"], s["sinks"],
                                 k_scales=s["k_scales"], v_scales=s["v_scales"])


def _own_shared(s):
    import paper_2211_10482_b200 as st
    return st.st_attn_shared_step(s["q"], s["k_pages"], s["v_pages"], s["prefix_table"], s["prefix_lens"], s["table"], s["lens"], s["group_offsets"])


_own = dict(rotate=_own_rotate, rotate_train=_own_rotate_train, store=_own_store, step=_own_step, shared=_own_shared)

# ---------------------------------------------------------------------- the plain form: rotation


def _turn(x, angle, rot, pairs, back=False):
    """Pairs of the first `rot` columns turned by their token's angles; x float32 [n, heads, d]."""
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if back:
        s = -s
    a, b = (x[..., : rot // 2], x[..., rot // 2 : rot]) if pairs == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.cat([a, b], -1) if pairs == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _angles(s):
    return s["positions"].double()[:, None] * s["freq"].double()          # positions reach far: in 64 bits


def _normed(x, w, eps):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w.float()


def _plain_rotate(s):
    angle = _angles(s)
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x = _normed(x, w, s["eps"]) if s["norm"] else x.float()
        out.append(_turn(x, angle, s["rot"], s["pairs"]).to(torch.bfloat16))
    return tuple(out)


def _plain_rotate_train(s):
    angle = _angles(s)
    grads, sums = [], []
    for x, w, dy in ((s["q"], s["qw"], s["dq"]), (s["k"], s["kw"], s["dk"])):
        g = _turn(dy.float(), angle, s["rot"], s["pairs"], back=True)
        if s["norm"]:
            x = x.float()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
            n = x * r
            sums.append((g * n).sum((0, 1)))
            g = g * w.float()
            g = r * (g - n * (g * n).mean(-1, keepdim=True))
        grads.append(g.to(torch.bfloat16))
    return (*_plain_rotate(s), *grads, *sums)


# ------------------------------------------------------------------------- the plain form: cells

_TINY = 2.0 ** -100


def _divided(a, b):
    """a / b, rounded once: torch may take a quotient of a tensor and a number as a product with a reciprocal."""
    return torch.div(torch.as_tensor(a, dtype=torch.float32, device="cuda").expand(b.shape), b)


def _quantise(x, cells):
    """8 bits: int8 [.., d] with one float32 scale a row.  4 bits: uint8 [.., d/2] (even column low), bfloat16 [.., groups, 2]: step and lowest
    value of 32 columns."""
    x = x.float()
    if cells == 8:
        most = x.abs().amax(-1, keepdim=True)
        some = most >= _TINY
        inv = torch.where(some, _divided(127.0, most.clamp(min=_TINY)), 0.0)
        return torch.round(x * inv).to(torch.int8), torch.where(some, torch.div(most, torch.full_like(most, 127.0)), 0.0).squeeze(-1)
    d = x.shape[-1]
    groups = -(-d // 32)
    padded = torch.cat([x, x[..., -1:].expand(*x.shape[:-1], groups * 32 - d)], -1).unflatten(-1, (groups, 32))
    lo, hi = padded.amin(-1, keepdim=True), padded.amax(-1, keepdim=True)
    spread = hi - lo
    step = torch.div(spread, torch.full_like(spread, 15.0)).to(torch.bfloat16).float()
    some = step >= _TINY
    step = torch.where(some, step, 0.0)
    inv = torch.where(some, _divided(1.0, step.clamp(min=_TINY)), 0.0)
    q = torch.round((padded - lo) * inv).clamp(0, 15).flatten(-2)[..., :d].to(torch.uint8)
    return (q[..., 0::2] | (q[..., 1::2] << 4)).contiguous(), torch.cat([step, lo], -1).to(torch.bfloat16)


def _values(cells, scales, bits):
    """What cells stand for, float32."""
    if bits == 16:
        return cells.float()
    if bits == 8:
        return cells.float() * scales[..., None]
    q = torch.stack([cells & 15, cells >> 4], -1).flatten(-2).float()
    step, lo = (scales[..., i].float().repeat_interleave(32, -1)[..., : q.shape[-1]] for i in (0, 1))
    return lo + step * q


def _gathered(s, at, name):
    """Rows of the pages as float32; at: (pages, places)."""
    scales = s[name + "_scales"]
    return _values(s[name + "_pages"][at], None if scales is None else scales[at], s.get("cells", 16))


def _row_places(s, offsets, rows):
    """Page and place of every packed row: the rows of a sequence are its last tokens."""
    offsets, table, lens = offsets.long(), s["table"].long(), s["lens"].long()
    count = offsets[1:] - offsets[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count, output_size=rows)
    position = torch.arange(rows, device="cuda") - offsets[seq] + (lens - count)[seq]
    return table[seq, position // s["page"]], position % s["page"]


def _plain_store(s):
    at = _row_places(s, s["new_offsets"], s["k"].shape[0])
    for name in ("k", "v"):
        if s["cells"] == 16:
            s[name + "_pages"][at] = s[name]
        else:
            s[name + "_pages"][at], s[name + "_scales"][at] = _quantise(s[name], s["cells"])
    at = _row_places(s, s["all_offsets"], s["rows"])
    return tuple(_gathered(s, at, name).to(torch.bfloat16) for name in ("k", "v"))


# -------------------------------------------------------------------------- the plain form: steps


def _own_keys(s, window, sinks):
    """Page, place and visibility of every key that a sequence's last token may see, [seqs, keys]."""
    lens, table, page = s["lens"].long(), s["table"].long(), s["page"]
    longest = max(s["lens_host"])
    window, sinks = min(window, longest), min(sinks, longest)
    j = torch.arange(sinks + window, device="cuda")
    near = lens[:, None] - window + j[sinks:] - sinks
    key = torch.cat([j[:sinks].expand(lens.numel(), sinks), near], 1)
    seen = torch.where(j < sinks, key < lens[:, None] - window, key >= 0) & (key < lens[:, None])
    key = torch.where(seen, key, 0)
    return (table.gather(1, key // page), key % page), seen


def _softmaxed(x, seen, v):
    x = x.masked_fill(~seen, -math.inf)
    most = x.amax(-1, keepdim=True)
    p = (x - most.masked_fill(most == -math.inf, 0.0)).exp()
    return torch.einsum("bhgj,bjhd->bhgd", p / p.sum(-1, keepdim=True).clamp(min=1e-30), v)


def _plain_step(s):
    at, seen = _own_keys(s, s["window"], s["sinks"])
    k, v = _gathered(s, at, "k"), _gathered(s, at, "v")
    q = s["q"].float().unflatten(1, (s["Hk"], s["H"] // s["Hk"]))
    x = torch.einsum("bhgd,bjhd->bhgj", q, k) / math.sqrt(s["d"])
    return _softmaxed(x, seen[:, None, None], v).flatten(1, 2).to(torch.bfloat16)


def _plain_shared(s):
    d, page, q = s["d"], s["page"], s["q"].float().unflatten(1, (s["Hk"], s["H"] // s["Hk"])) / math.sqrt(s["d"])
    at, seen = _own_keys(s, 1 << 30, 0)
    own_k, own_v = s["k_pages"][at].float(), s["v_pages"][at].float()
    outs = []
    for a, b, n, table in zip(s["groups"], s["groups"][1:], s["prefix"], s["prefix_table"].long()):
        t = torch.arange(n, device="cuda")
        k, v = (s[name][table[t // page], t % page].float() for name in ("k_pages", "v_pages"))
        near = torch.einsum("bhgd,bjhd->bhgj", q[a:b], own_k[a:b]).masked_fill(~seen[a:b, None, None], -math.inf)
        x = torch.cat([torch.einsum("bhgd,jhd->bhgj", q[a:b], k), near], -1)
        p = (x - x.amax(-1, keepdim=True)).exp()
        p = p / p.sum(-1, keepdim=True)
        outs.append(torch.einsum("bhgj,jhd->bhgd", p[..., :n], v) + torch.einsum("bhgj,bjhd->bhgd", p[..., n:], own_v[a:b]))
    return torch.cat(outs).flatten(1, 2).to(torch.bfloat16)


_plain = dict(rotate=_plain_rotate, rotate_train=_plain_rotate_train, store=_plain_store, step=_plain_step, shared=_plain_shared)

# ------------------------------------------------------------------- the definitions in 64 bits


def _matrix_turned(x, s):
    """Each pair as a complex number times e^(i angle); x [n, heads, d] in 64 bits."""
    rot, half = s["rot"], s["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (i, i + half) if s["pairs"] == "half" else (2 * i, 2 * i + 1)
    angle = torch.outer(s["positions"].double(), s["freq"].double())
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return x.index_copy(2, first, z.real).index_copy(2, second, z.imag)


def _exact_rotation(s):
    outs, leaves, loss = [], [], 0.0
    for x, w, dy in ((s["q"], s["qw"], s.get("dq")), (s["k"], s["kw"], s.get("dk"))):
        x = x.double().requires_grad_()
        w = w.double().requires_grad_() if w is not None else None
        n = x if w is None else x / (x.pow(2).sum(-1, keepdim=True) / s["d"] + s["eps"]).sqrt() * w
        y = _matrix_turned(n, s)
        outs.append(y.detach())
        leaves.append((x, w))
        if dy is not None:
            loss = loss + (y * dy.double()).sum()
    if s["op"] == "rotate":
        return tuple(outs)
    loss.backward()
    grads = [x.grad for x, _ in leaves] + [w.grad for _, w in leaves if w is not None]
    return (*outs, *grads)


def _exact_cell_values(x, bits):
    """What a row of cells would stand for, from the formulas; x [.., d] in 64 bits."""
    if bits == 16:
        return x
    if bits == 8:
        scale = x.abs().amax(-1, keepdim=True) / 127
        return torch.where(scale > 0, torch.round(x / scale.clamp(min=1e-300)) * scale, 0.0)
    out = []
    for part in x.split(32, -1):
        lo, hi = part.amin(-1, keepdim=True), part.amax(-1, keepdim=True)
        step = ((hi - lo) / 15).float().to(torch.bfloat16).double()
        out.append(torch.where(step > 0, lo + step * torch.round((part - lo) / step.clamp(min=1e-300)).clamp(max=15), lo))
    return torch.cat(out, -1)


def _held(s, name, table, n):
    """Tokens 0..n-1 behind one row of a table, as stored, in 64 bits: [n, Hk, d]."""
    where = table.long().repeat_interleave(s["page"])[:n], torch.arange(n, device="cuda") % s["page"]
    cells, bits = s[name + "_pages"][where], s.get("cells", 16)
    if bits == 16:
        return cells.double()
    scales = s[name + "_scales"][where].double()
    if bits == 8:
        return cells.double() * scales.unsqueeze(-1)
    out = torch.empty((*cells.shape[:-1], s["d"]), dtype=torch.float64, device="cuda")
    for c in range(s["d"]):
        nibble = (cells[..., c // 2].int() >> (4 * (c % 2))) & 15
        out[..., c] = scales[..., c // 32, 1] + scales[..., c // 32, 0] * nibble.double()
    return out


def _attended(q, k, v):
    """One token's heads q [H, d] over all keys, in 64 bits."""
    g = q.shape[0] // k.shape[1]
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    x = torch.stack([k[:, h // g] @ q[h] for h in range(q.shape[0])]) / math.sqrt(q.shape[1])
    p = torch.softmax(x, -1)
    return torch.stack([p[h] @ v[:, h // g] for h in range(q.shape[0])])


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("rotate", "rotate_train"):
        return _exact_rotation(s)
    if op == "store":
        outs = []
        for name in ("k", "v"):
            new = _exact_cell_values(s[name].double(), case["cells"]).split(s["new"])
            parts = []
            for b, (n, fresh) in enumerate(zip(s["lens_host"], new)):
                parts += [_held(s, name, s["table"][b], n - fresh.shape[0]), fresh]
            outs.append(torch.cat(parts))
        return tuple(outs)
    outs = []
    if op == "step":
        for b, n in enumerate(s["lens_host"]):
            k, v = (_held(s, name, s["table"][b], n) for name in ("k", "v"))
            low = max(0, n - case["window"])
            first = min(case["sinks"], low)
            k, v = (torch.cat([x[:first], x[low:]]) for x in (k, v))
            outs.append(_attended(s["q"][b].double(), k, v))
        return torch.stack(outs)
    for i, (a, b) in enumerate(zip(s["groups"], s["groups"][1:])):
        shared = [_held(s, name, s["prefix_table"][i], s["prefix"][i]) for name in ("k", "v")]
        for n in range(a, b):
            mine = [_held(s, name, s["table"][n], s["lens_host"][n]) for name in ("k", "v")]
            outs.append(_attended(s["q"][n].double(), *(torch.cat(x) for x in zip(shared, mine))))
    return torch.stack(outs)
