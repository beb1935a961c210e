"""Operators around a paged KV cache, as a serving or training program calls them: rotary positions with several axes, new
tokens written to their pages, attention of a chunk of new tokens over the pages, the attention weight that every cached token
received, and the eviction of the tokens that received least.

Five kinds of case:

* ``rope``    Q and K of a prompt or a training batch rotated (forward, or backward = the inverse rotation of the gradients);
* ``append``  the packed new tokens of several sequences: Q and K rotated, K and V written to the pages;
* ``chunk``   attention of each sequence's new tokens over its pages, causal, with the log-sum-exp of every row;
* ``mass``    per cached token and KV head, the weights that the new rows gave it, added to what it had;
* ``evict``   the tokens with the most weight kept, with the first and the last ones, and moved to other pages.

`run` computes them in elementary torch operations, or, where `own` is true, by the framework's calls.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- the cases

def _rope(name=None, *, batch, n, h_q, h_kv, d, pairs, axes, interleaved, inverse, dtype, far=0):
    c = dict(kind="rope", batch=batch, n=n, h_q=h_q, h_kv=h_kv, d=d, pairs=pairs, axes=axes, interleaved=interleaved,
             inverse=inverse, dtype=dtype, far=far)
    return dict(c, name=name) if name else c


def _paged(kind, name=None, *, batch, new, kv, h_q, h_kv, d, page, dtype, **more):
    c = dict(kind=kind, batch=batch, new=new, kv=kv, h_q=h_q, h_kv=h_kv, d=d, page=page, dtype=dtype, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a training step on image and text tokens: the queries and keys of one 8K sequence, positions in time, height and width
        _rope("rope_8k", batch=1, n=8192, h_q=32, h_kv=8, d=128, pairs=64, axes=3, interleaved=False, inverse=False, dtype="bf16"),
        # its backward pass in a small fp32 model: adjacent pairs, part of the head rotated, odd lengths, far positions
        _rope("rope_grad_f32", batch=2, n=1500, h_q=8, h_kv=4, d=64, pairs=24, axes=2, interleaved=True, inverse=True, dtype="f32",
              far=1000000),
        # one token of each of sixteen conversations enters its cache: the smallest call, where latency counts
        _paged("append", "append_16x1", batch=16, new=1, kv=500, h_q=32, h_kv=8, d=128, page=64, dtype="bf16", pairs=64, axes=1,
               interleaved=False),
        # prompts of several users, up to 4096 tokens each, enter the cache in one call
        _paged("append", "append_prompts", batch=4, new=4096, kv=5000, h_q=32, h_kv=8, d=128, page=128, dtype="bf16", pairs=64,
               axes=3, interleaved=False),
        # one token of each of sixteen long conversations, of lengths up to 65536
        _paged("chunk", "chunk_16x1_64k", batch=16, new=1, kv=65536, h_q=32, h_kv=8, d=128, page=64, dtype="bf16"),
        # a long prompt's last piece: 4096 new tokens over 12288 cached ones
        _paged("chunk", "chunk_4k_over_12k", batch=1, new=4096, kv=16384, h_q=32, h_kv=8, d=128, page=128, dtype="bf16"),
        # short chunks of different lengths beside each other, three query heads a KV head, small pages
        _paged("chunk", "chunk_ragged", batch=5, new=300, kv=2000, h_q=12, h_kv=4, d=64, page=16, dtype="bf16"),
        # a small model in fp32, pages that end inside a tile
        _paged("chunk", "chunk_f32", batch=2, new=200, kv=1500, h_q=8, h_kv=2, d=64, page=48, dtype="f32"),
        # a decode step's weights over sixteen caches of up to 32768 tokens
        _paged("mass", "mass_16x1_32k", batch=16, new=1, kv=32768, h_q=32, h_kv=8, d=128, page=64, dtype="bf16", decay=0.95),
        # the weights that a prompt's last 2048 tokens gave to its 8192
        _paged("mass", "mass_2k_of_8k", batch=1, new=2048, kv=8192, h_q=32, h_kv=8, d=128, page=128, dtype="bf16", decay=1.0),
        # sixteen caches of up to 32768 tokens brought down to 4096
        _paged("evict", "evict_16x32k", batch=16, new=1, kv=32768, h_q=32, h_kv=8, d=128, page=64, dtype="bf16", keep=4096, sinks=4,
               recent=512),
        # short caches, one of them below the limit already
        _paged("evict", "evict_small", batch=3, new=1, kv=700, h_q=4, h_kv=2, d=64, page=48, dtype="f32", keep=256, sinks=4,
               recent=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "chunk", "chunk", "mass", "evict"])
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rope":
        h_kv = rng.choice([1, 2, 4, 8])
        h_q = h_kv * rng.choice([1, 2, 4])
        batch, n = rng.randint(1, 4), _log(rng, 1, 8192)
        while batch * n * (h_q + h_kv) * d > 8192 * 40 * 128:
            n = max(1, n // 2)
        return _rope(batch=batch, n=n, h_q=h_q, h_kv=h_kv, d=d, pairs=rng.choice([d // 2, d // 2, d // 4, d // 2 - 4]),
                     axes=rng.randint(1, 4), interleaved=rng.random() < 0.4, inverse=rng.random() < 0.5, dtype=dtype,
                     far=rng.choice([0, 0, 1000000]))
    h_kv = rng.choice([1, 2, 4, 8])
    h_q = h_kv * rng.choice([1, 2, 3, 4, 8])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    batch, kv = _log(rng, 1, 16), _log(rng, 16, 65536)
    new = min(kv, _log(rng, 1, 4096)) if rng.random() < 0.7 else 1
    common = dict(h_q=h_q, h_kv=h_kv, d=d, page=page, dtype=dtype)
    if kind == "append":
        while batch * max(new * (h_q + h_kv), kv * h_kv) * d > 4 * 5000 * 40 * 64:
            new, kv = max(1, new // 2), max(1, kv // 2)
        return _paged("append", batch=batch, new=min(new, kv), kv=kv, pairs=rng.choice([d // 2, d // 4]), axes=rng.randint(1, 4),
                      interleaved=rng.random() < 0.4, **common)
    if kind == "evict":
        while batch * kv * h_kv * d > 16 * 32768 * 8 * 64:
            kv = max(16, kv // 2)
        keep = max(8, int(kv * rng.uniform(0.05, 0.9)))
        return _paged("evict", batch=batch, new=1, kv=kv, keep=keep, sinks=rng.choice([0, 1, 4]), recent=max(1, keep // rng.randint(2, 8)),
                      **common)
    # fp32 runs on other units: a sixteenth of the products and half of the tokens
    most_pairs = (1 << 31) // (2 if kind == "mass" else 1) // (16 if dtype == "f32" else 1)
    while batch * new * kv * h_q > most_pairs or batch * kv * h_kv * d > 16 * 32768 * 8 * 64 // (2 if dtype == "f32" else 1):
        if new > 64 and batch * new * kv * h_q > most_pairs:
            new //= 2
        else:
            kv = max(16, kv // 2)
            new = min(new, kv)
    more = {"decay": rng.choice([1.0, 0.9])} if kind == "mass" else {}
    return _paged(kind, batch=batch, new=new, kv=kv, **common, **more)


# ---------------------------------------------------------------- inputs

def _lengths(case):
    """New and cached tokens of every sequence: the first has the most, the others are spread below."""
    rng = random.Random("%d %d %d" % (case["batch"], case["new"], case["kv"]))
    kv, new = [case["kv"]], [min(case["new"], case["kv"])]
    for _ in range(case["batch"] - 1):
        kv.append(rng.randint(max(1, case["kv"] // 4), case["kv"]))
        new.append(min(kv[-1], rng.randint(1, case["new"])))
    return new, kv


def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)
    return out.mul_(scale) if scale != 1.0 else out


def _table(gen, kv, page):
    """Pages of every sequence in a random order over the pool; -1 behind a sequence's last page."""
    need = [-(-n // page) for n in kv]
    width, total = max(need), sum(need)
    order = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(kv), width), -1, dtype=torch.int32, device=DEV)
    have = torch.arange(width, device=DEV)[None] < torch.tensor(need, device=DEV)[:, None]
    table[have] = order
    return table, total


def _axes_of(case):
    """Axis and frequency of every rotated pair: sections of the pairs, one after the other, of one falling series."""
    pairs, axes = case["pairs"], case["axes"]
    return [i * axes // pairs for i in range(pairs)], [10000.0 ** (-i / pairs) for i in range(pairs)]


def _positions(gen, case, tokens):
    top = case.get("far") or 40000
    low = 0 if not case.get("far") else top // 2
    return torch.randint(low, top, (case["axes"], tokens), generator=gen, device=DEV, dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[case["dtype"]]
    s = {"case": case}
    d, h_q, h_kv = case["d"], case["h_q"], case["h_kv"]
    if case["kind"] == "rope":
        b, n = case["batch"], case["n"]
        s["Q"], s["K"] = _randn(gen, b, n, h_q, d, dtype=t), _randn(gen, b, n, h_kv, d, dtype=t)
        s["pos"] = _positions(gen, case, b * n).view(case["axes"], b, n)
        s["Qout"], s["Kout"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
        return s
    new, kv = _lengths(case)
    rows, page = sum(new), case["page"]
    s["table"], pages = _table(gen, kv, page)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s["q_start"] = torch.tensor([0] + new, device=DEV).cumsum(0).to(torch.int32)
    s["Kpool"] = _randn(gen, pages, page, h_kv, d, dtype=t)
    if case["kind"] != "mass":
        s["Vpool"] = _randn(gen, pages, page, h_kv, d, dtype=t)
    slots = s["table"].shape[1] * page
    if case["kind"] == "append":
        s["Q"], s["K"], s["V"] = (_randn(gen, rows, h, d, dtype=t) for h in (h_q, h_kv, h_kv))
        s["pos"] = _positions(gen, case, rows)
        s["Qout"] = torch.empty_like(s["Q"])
    elif case["kind"] in ("chunk", "mass"):
        # scores with a deviation of two: some keys hold most of a row's weight, as trained attention has it
        s["Q"] = _randn(gen, rows, h_q, d, dtype=t, scale=2.0)
        s["O"], s["lse"] = torch.empty_like(s["Q"]), torch.empty(rows, h_q, device=DEV)
        if case["kind"] == "mass":
            s["lse"] = _log_sums(s)
            s["mass"] = torch.rand(case["batch"], h_kv, slots, generator=gen, device=DEV)
            s["mass_out"] = torch.zeros_like(s["mass"])
    else:
        # accumulated weights have a heavy tail, and ties where nothing was attended
        m = _randn(gen, case["batch"], h_kv, slots, scale=2.0).exp_()
        s["mass"] = torch.where(m < 0.1, torch.zeros_like(m), m)
        keep = case["keep"]
        width = -(-keep // page)
        pages_to = case["batch"] * width
        s["to_table"] = torch.randperm(pages_to, generator=gen, device=DEV).to(torch.int32).view(case["batch"], width)
        s["Kto"], s["Vto"] = (torch.zeros(pages_to, page, h_kv, d, dtype=t, device=DEV) for _ in range(2))
        s["mass_to"] = torch.zeros(case["batch"], h_kv, width * page, device=DEV)
        s["kept"] = torch.empty(case["batch"], h_kv, keep, dtype=torch.int32, device=DEV)
        s["new_len"] = torch.empty(case["batch"], dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _rotate(case, x, pos, inverse):
    """x [tokens, heads, d] in fp32; angles in 64 bits, because fp32 has no fraction left at a far position."""
    pairs = case["pairs"]
    axis, freq = _axes_of(case)
    at = pos.reshape(case["axes"], -1)[torch.tensor(axis, device=DEV)].double()          # [pairs, tokens]
    theta = (at * torch.tensor(freq, dtype=torch.float64, device=DEV)[:, None]).t()
    cos, sin = theta.cos().float()[:, None, :], theta.sin().float()[:, None, :]
    if inverse:
        sin = -sin
    part, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    if case["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = part[..., :pairs], part[..., pairs:]
        part = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([part, rest], -1)


def _rows_of(s):
    """Sequence and place in its chunk of every packed row, and its slot in the cache."""
    rows = torch.arange(s["Q"].shape[0], device=DEV)
    start, kv = s["q_start"].long(), s["kv_len"].long()
    seq = torch.searchsorted(start, rows, right=True) - 1
    i = rows - start[seq]
    return seq, i, kv[seq] - (start[seq + 1] - start[seq]) + i


def _pages(s, pool):
    """A pool's rows by sequence and slot, fp32: [batch, h_kv, slots, d]."""
    page = pool.shape[1]
    slot = torch.arange(s["table"].shape[1] * page, device=DEV)
    phys = s["table"].long().clamp(min=0)[:, slot // page]
    return pool[phys, slot % page].float().transpose(1, 2)


def _scores(s):
    """Scores [batch, h_kv, g * new, slots] of every padded row, -inf where the slot is not before or at the row's own."""
    case = s["case"]
    b, h_kv, g, d = case["batch"], case["h_kv"], case["h_q"] // case["h_kv"], case["d"]
    seq, i, slot = _rows_of(s)
    most = min(case["new"], case["kv"])
    q = torch.zeros(b, most, h_kv, g, d, device=DEV)
    q[seq, i] = s["Q"].float().view(-1, h_kv, g, d)
    last = torch.full((b, most), -1, device=DEV)
    last[seq, i] = slot
    k = _pages(s, s["Kpool"])
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(b, h_kv, g * most, d) * (1 / math.sqrt(d)), k.transpose(2, 3))
    seen = torch.arange(k.shape[2], device=DEV) <= last[:, :, None]                 # [b, most, slots]
    x.view(b, h_kv, g, most, -1).masked_fill_(~seen[:, None, None], -math.inf)
    return x, seq, i, seen


def _packed(s, x, seq, i):
    """[batch, h_kv, g * new, ...] back to packed rows [rows, h_q, ...]."""
    case = s["case"]
    b, h_kv, g = case["batch"], case["h_kv"], case["h_q"] // case["h_kv"]
    x = x.view(b, h_kv, g, x.shape[2] // g, *x.shape[3:])
    return x.movedim(3, 1)[seq, i].flatten(1, 2)


def _log_sums(s):
    x, seq, i, _ = _scores(s)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    return _packed(s, (top + x.sub_(top).exp_().sum(-1, keepdim=True).log())[..., 0], seq, i).contiguous()


def _plain_rope(s):
    case = s["case"]
    for x, y in (("Q", "Qout"), ("K", "Kout")):
        flat = s[x].float().view(-1, s[x].shape[2], case["d"])
        s[y].copy_(_rotate(case, flat, s["pos"], case["inverse"]).view_as(s[x]))
    return {"Q": s["Qout"], "K": s["Kout"]}


def _plain_append(s):
    case = s["case"]
    seq, _, slot = _rows_of(s)
    phys = s["table"].long()[seq, slot // case["page"]]
    s["Qout"].copy_(_rotate(case, s["Q"].float(), s["pos"], False))
    s["Kpool"][phys, slot % case["page"]] = _rotate(case, s["K"].float(), s["pos"], False).to(s["Kpool"].dtype)
    s["Vpool"][phys, slot % case["page"]] = s["V"]
    return {"Q": s["Qout"], "Kpool": s["Kpool"], "Vpool": s["Vpool"]}


def _plain_chunk(s):
    x, seq, i, _ = _scores(s)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _pages(s, s["Vpool"])).div_(total.clamp(min=1e-30))
    s["O"].copy_(_packed(s, o, seq, i))
    s["lse"].copy_(_packed(s, (top + total.log())[..., 0], seq, i))
    return {"O": s["O"], "lse": s["lse"]}


def _plain_mass(s):
    case = s["case"]
    b, h_kv, g = case["batch"], case["h_kv"], case["h_q"] // case["h_kv"]
    x, seq, i, _ = _scores(s)
    most = x.shape[2] // g
    lse = torch.zeros(b, most, h_kv, g, device=DEV)
    lse[seq, i] = s["lse"].view(-1, h_kv, g)
    w = x.sub_(lse.permute(0, 2, 3, 1).reshape(b, h_kv, g * most, 1)).exp_().sum(2)
    kv, start = s["kv_len"].long(), s["q_start"].long()
    slot = torch.arange(w.shape[2], device=DEV)
    old = slot < (kv - (start[1:] - start[:-1]))[:, None]
    w += torch.where(old[:, None], s["mass"] * case["decay"], torch.zeros_like(w))
    s["mass_out"].copy_(torch.where((slot < kv[:, None])[:, None], w, s["mass_out"]))
    return {"mass": s["mass_out"]}


def _plain_evict(s):
    case = s["case"]
    keep, sinks, recent, page = case["keep"], case["sinks"], case["recent"], case["page"]
    kv = s["kv_len"].long()[:, None, None]
    slot = torch.arange(s["mass"].shape[2], device=DEV)
    always = (slot < sinks) | (slot >= kv - recent)
    order = torch.where(slot < kv, torch.where(always, math.inf, s["mass"]), -math.inf)
    best = order.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    new_len = kv[:, 0, 0].clamp(max=keep)
    j = torch.arange(keep, device=DEV)
    have = j < new_len[:, None, None]
    pad = torch.nn.functional.pad(best, (0, keep - best.shape[-1]), value=1 << 30)
    kept = torch.where(have, pad, 1 << 30).sort(dim=-1).values
    s["kept"].copy_(torch.where(have, kept, -1))
    s["new_len"].copy_(new_len)
    b, r, to = torch.nonzero(have.expand_as(kept), as_tuple=True)
    src = kept[b, r, to]
    s["mass_to"][b, r, to] = s["mass"][b, r, src]
    for x, y in (("Kpool", "Kto"), ("Vpool", "Vto")):
        s[y][s["to_table"].long()[b, to // page], to % page, r] = s[x][s["table"].long()[b, src // page], src % page, r]
    return {"kept": s["kept"], "len": s["new_len"], "K": s["Kto"], "V": s["Vto"], "mass": s["mass_to"]}


# ---------------------------------------------------------------- the framework's calls

def _rope_of(B, s):
    if "rope" not in s:
        axis, freq = _axes_of(s["case"])
        s["rope"] = B.make_rope(freq, axis=axis, interleaved=s["case"]["interleaved"])
    return s["rope"]


def _call(s):
    from paper_2605_18753_b200 import binding as B

    case = s["case"]
    kind = case["kind"]
    if kind == "rope":
        if "p" not in s:
            s["p"] = B.make_params(batch=case["batch"], seq_q=case["n"], seq_kv=case["n"], h_q=case["h_q"], h_kv=case["h_kv"],
                                   head_dim=case["d"], block=64, dtype=TYPES[case["dtype"]], alpha=1.5)
        B.dash_attn_rope(s["p"], _rope_of(B, s), s["pos"], s["Q"], s["K"], s["Qout"], s["Kout"], inverse=case["inverse"])
        return {"Q": s["Qout"], "K": s["Kout"]}
    if "p" not in s:
        s["p"] = B.params_for_paged(s["Kpool"], s.get("Vpool"), s["table"], h_q=case["h_q"], Q=s.get("Q"), K=s.get("K"),
                                    V=s.get("V"), O=s.get("O", s.get("Qout")))
    p = s["p"]
    if kind == "append":
        B.dash_attn_append_paged(p, _rope_of(B, s), s["pos"], s["q_start"], s["kv_len"], s["table"], s["Q"], s["Qout"], s["K"],
                                 s["V"], s["Kpool"], s["Vpool"])
        return {"Q": s["Qout"], "Kpool": s["Kpool"], "Vpool": s["Vpool"]}
    if kind == "evict":
        B.dash_attn_evict_paged(p, s["mass"], s["kv_len"], s["table"], s["Kpool"], s["Vpool"], s["kept"], s["new_len"],
                                s["to_table"], s["Kto"], s["Vto"], s["mass_to"], keep=case["keep"], sinks=case["sinks"],
                                recent=case["recent"])
        return {"kept": s["kept"], "len": s["new_len"], "K": s["Kto"], "V": s["Vto"], "mass": s["mass_to"]}
    if "ws" not in s:
        s["ws"] = B.alloc_paged_workspace(p)
    if kind == "chunk":
        B.dash_attn_attend_chunk_paged(p, s["Q"], s["Kpool"], s["Vpool"], s["table"], s["q_start"], s["kv_len"], s["O"], s["lse"],
                                       s["ws"])
        return {"O": s["O"], "lse": s["lse"]}
    B.dash_attn_key_mass_paged(p, s["Q"], s["Kpool"], s["table"], s["q_start"], s["kv_len"], s["lse"], s["mass"], s["mass_out"],
                               s["ws"], decay=case["decay"])
    return {"mass": s["mass_out"]}


def run(state):
    if own:
        return _call(state)
    return {"rope": _plain_rope, "append": _plain_append, "chunk": _plain_chunk, "mass": _plain_mass,
            "evict": _plain_evict}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    d, h_q, h_kv = case["d"], case["h_q"], case["h_kv"]
    if case["kind"] == "rope":
        values = case["batch"] * case["n"] * (h_q + h_kv) * d
        return {"bytes": 2 * values * e + 4 * case["axes"] * case["batch"] * case["n"], "flops": 3 * values}
    new, kv = _lengths(case)
    if case["kind"] == "append":
        return {"bytes": sum(new) * (2 * (h_q + 2 * h_kv) * d * e + 4 * case["axes"]), "flops": 3 * sum(new) * (h_q + h_kv) * d}
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in kv) * h_kv
        return {"bytes": 4 * sum(kv) * h_kv + kept * (4 * d * e + 12), "flops": 0}
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, kv)) * h_q
    rows, cached = sum(new) * h_q, sum(kv) * h_kv
    if case["kind"] == "chunk":
        return {"bytes": 2 * cached * d * e + 2 * rows * d * e + 4 * rows, "flops": 4 * d * pairs}
    return {"bytes": cached * (d * e + 8) + rows * (d * e + 4), "flops": 2 * d * pairs}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _turned(case, x, pos, sign):
    """Rotation of x [tokens, heads, d], pair by pair as a complex product."""
    x = x.double()
    out = x.clone()
    axis, freq = _axes_of(case)
    flat = pos.reshape(case["axes"], -1).double()
    for i in range(case["pairs"]):
        lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + case["pairs"])
        unit = torch.polar(torch.ones_like(flat[0]), sign * flat[axis[i]] * freq[i])
        z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * unit[:, None]
        out[..., lo], out[..., hi] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        turn = lambda x: _turned(case, x.flatten(0, 1), s["pos"], -1.0 if case["inverse"] else 1.0).view(x.shape)  # noqa: E731
        return {"Q": turn(s["Q"]), "K": turn(s["K"])}
    new, kv = _lengths(case)
    table, page = s["table"].cpu(), case["page"]
    first = [sum(new[:b]) for b in range(len(new))]
    if case["kind"] == "append":
        k = _turned(case, s["K"], s["pos"], 1.0)
        pools = {"Kpool": s["Kpool"].double(), "Vpool": s["Vpool"].double()}
        for b, (n, length) in enumerate(zip(new, kv)):
            for i in range(n):
                p, t = divmod(length - n + i, page)
                pools["Kpool"][table[b, p], t] = k[first[b] + i]
                pools["Vpool"][table[b, p], t] = s["V"][first[b] + i].double()
        return {"Q": _turned(case, s["Q"], s["pos"], 1.0), **pools}
    if case["kind"] == "evict":
        mass = s["mass"].cpu().double()
        kept, out = torch.full(s["kept"].shape, -1, dtype=torch.int32), torch.zeros(s["mass_to"].shape, dtype=torch.float64)
        for b, length in enumerate(kv):
            for r in range(case["h_kv"]):
                chosen = torch.arange(length)
                if length > case["keep"]:
                    lo, hi = case["sinks"], length - case["recent"]
                    middle = lo + torch.from_numpy((-mass[b, r, lo:hi].numpy()).argsort(kind="stable"))
                    middle = middle[: case["keep"] - case["sinks"] - case["recent"]].sort().values
                    chosen = torch.cat([chosen[:lo], middle, chosen[hi:]])
                kept[b, r, : len(chosen)] = chosen.to(torch.int32)
                out[b, r, : len(chosen)] = mass[b, r, chosen]
        return {"kept": kept, "len": torch.tensor([min(n, case["keep"]) for n in kv], dtype=torch.int32), "K": None, "V": None,
                "mass": out}
    g, d = case["h_q"] // case["h_kv"], case["d"]
    rows = s["Q"].shape[0]
    o = torch.zeros(rows, case["h_q"], d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(rows, case["h_q"], dtype=torch.float64, device=DEV)
    mass = s["mass_out"].double() if case["kind"] == "mass" else None
    for b, (n, length) in enumerate(zip(new, kv)):
        seen = torch.arange(length, device=DEV)[None] <= torch.arange(length - n, length, device=DEV)[:, None]
        ids = s["table"][b, : -(-length // page)].long()
        at = slice(first[b], first[b] + n)
        for r in range(case["h_kv"]):
            k = s["Kpool"][ids, :, r].double().flatten(0, 1)[:length]
            v = s["Vpool"][ids, :, r].double().flatten(0, 1)[:length] if mass is None else None
            total = torch.zeros(length, dtype=torch.float64, device=DEV)
            for h in range(r * g, (r + 1) * g):
                x = (s["Q"][at, h].double() @ k.t() / math.sqrt(d)).masked_fill_(~seen, -math.inf)
                if mass is not None:
                    total += x.sub_(s["lse"][at, h, None].double()).exp_().sum(0)
                    continue
                lse[at, h] = torch.logsumexp(x, -1)
                o[at, h] = x.sub_(lse[at, h, None]).exp_() @ v
            if mass is not None:
                mass[b, r, :length] = total
                mass[b, r, : length - n] += case["decay"] * s["mass"][b, r, : length - n].double()
    return {"O": o, "lse": lse} if mass is None else {"mass": mass}
