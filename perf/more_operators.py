"""Cases of the paged cache: rows appended to it with the position rotation applied on the way, attention over the pages
that a cheap score selects, and attention of a batch whose sequences share a long prefix.

A paged cache is a pool of pages of 16, 32, 64 or 128 positions, k and v each bf16 [pages, KV heads, positions, 128].
Position p of sequence b lies in page table[b][p // page].  With every page go the bounds of its keys, the least and the
largest value of each channel over the positions it holds: k_min and k_max, bf16 [pages, KV heads, 128].
"""
import math

import torch

own = False

DIM = 128
THETA, TRAINED, LOW, HIGH, FAST, SLOW = 500000.0, 8192, 1.0, 4.0, 32.0, 1.0
_contexts = {}   # a program keeps one context per shape of its batch


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of the decode loop, its projection in 32 bits, frequencies scaled by wavelength bands: latency
        dict(name="append token", op="append", batch=1, q_heads=32, kv_heads=8, page=64, start=32801, tokens=1, ragged=False,
             dtype="float32", rot=128, layout="half", scaling="bands", factor=8.0),
        # one token of every sequence of a serving batch
        dict(name="append batch", op="append", batch=64, q_heads=32, kv_heads=8, page=128, start=2500, tokens=1, ragged=False,
             dtype="float32", rot=128, layout="half", scaling="none", factor=1.0),
        # a prompt
        dict(name="append prompt", op="append", batch=1, q_heads=32, kv_heads=8, page=64, start=0, tokens=32768, ragged=False,
             dtype="bfloat16", rot=128, layout="half", scaling="none", factor=1.0),
        # chunked prompts of a ragged batch: pages partly filled, sequences without new rows, half of a head rotated
        dict(name="append ragged chunk", op="append", batch=16, q_heads=28, kv_heads=4, page=16, start=10007, tokens=1000,
             ragged=True, dtype="bfloat16", rot=64, layout="interleaved", scaling="ramp", factor=4.0),
        # a short context: latency
        dict(name="sparse 1000", op="sparse", batch=1, q_heads=32, kv_heads=8, page=16, length=1000, top=16, ragged=False),
        # the ordinary decode step, 2048 positions attended
        dict(name="sparse 32768", op="sparse", batch=1, q_heads=32, kv_heads=8, page=64, length=32768, top=32, ragged=False),
        # a long context
        dict(name="sparse 131072", op="sparse", batch=1, q_heads=32, kv_heads=8, page=64, length=131072, top=64, ragged=False),
        # a ragged batch with seven query heads to a KV head, sequences that are masked or empty
        dict(name="sparse ragged batch", op="sparse", batch=16, q_heads=28, kv_heads=4, page=32, length=65535, top=128,
             ragged=True),
        # a few answers to one short prompt: latency
        dict(name="shared 4 x 1024", op="shared", batch=4, q_heads=32, kv_heads=8, page=16, prefix=1024, rest=200, ragged=False),
        # a serving batch behind one system prompt, lengths apart, sequences that are masked or shorter than the prefix
        dict(name="shared ragged 16 x 8192", op="shared", batch=16, q_heads=28, kv_heads=4, page=64, prefix=8192, rest=2000,
             ragged=True),
        # many samples of one long document
        dict(name="shared 64 x 32768", op="shared", batch=64, q_heads=32, kv_heads=8, page=64, prefix=32768, rest=500,
             ragged=False),
        # more rows than one pass over the prefix can take
        dict(name="shared 128 x 16384", op="shared", batch=128, q_heads=28, kv_heads=4, page=128, prefix=16384, rest=777,
             ragged=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "sparse", "shared"])
    page = rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.randint(1, 8)
    if op == "append":
        dtype = rng.choice(["float32", "bfloat16"])
        batch = _log(rng, 1, 64)
        most = 32768 * 48 * (1 if dtype == "bfloat16" else 0.6) / (q_heads + 2 * kv_heads) / batch
        tokens = 1 if rng.random() < 0.3 else _log(rng, 1, min(32768, max(1, int(most))))
        return dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, page=page,
                    start=rng.randrange(0, 1 + min(40000, 600000 // (batch * kv_heads))), tokens=tokens,
                    ragged=batch > 1 and rng.random() < 0.7, dtype=dtype, rot=16 * rng.randint(1, 8),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "bands", "ramp"]),
                    factor=rng.choice([2.0, 4.0, 8.0, 10.0]))
    if op == "sparse":
        batch = _log(rng, 1, 16)
        length = _log(rng, 1, min(131072, 16 * 4 * 65535 // (batch * kv_heads)))
        top = _log(rng, 1, max(1, min(-(-length // page), 16 * 4 * 4096 // (batch * kv_heads * page), 512)))
        return dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, page=page, length=length, top=top,
                    ragged=batch > 1 and rng.random() < 0.7)
    batch = _log(rng, 1, 128)
    most = 32768 * 64 * 32 // (batch * q_heads)
    prefix = 0 if rng.random() < 0.15 else page * _log(rng, 1, max(1, min(32768, most, 32768 * 8 // kv_heads) // page))
    rest = _log(rng, 1, min(32768, 64 * 8 * 600 // (batch * kv_heads)))
    return dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, page=page, prefix=prefix, rest=rest,
                ragged=batch > 1 and rng.random() < 0.6)


def _spread(batch, most, ragged):
    """A size per sequence: all alike, or spread below the largest, the second none and the fourth a single one."""
    if not ragged:
        return [most] * batch
    sizes = [most] + [most * (5 * b % 16 + 1) // 17 for b in range(1, batch)]
    sizes[1] = 0
    if batch > 3:
        sizes[3] = min(most, 1)
    return sizes


def _lengths(case):
    """Positions that every sequence holds when the pass is over."""
    batch, ragged = case["batch"], case["ragged"]
    if case["op"] == "append":
        return [a + n for a, n in zip(_spread(batch, case["start"], ragged), _counts(case))]
    if case["op"] == "sparse":
        return _spread(batch, case["length"], ragged)
    lens = [case["prefix"] + n for n in _spread(batch, case["rest"], ragged)]
    if ragged and batch > 5:
        lens[5] = case["prefix"] // 3                          # ended before its prefix did
    return lens


def _counts(case):
    return _spread(case["batch"], case["tokens"], case["ragged"])[::-1]


# ------------------------------------------------------------------------------------------------------ the inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    batch, nq, nkv, page = case["batch"], case["q_heads"], case["kv_heads"], case["page"]
    lens = _lengths(case)
    s = dict(case=case, op=case["op"])
    shared = case.get("prefix", 0) // page                     # pages that all sequences have in common
    each = -(-max(max(lens), 1) // page) + 1
    taken = [max(-(-n // page) - shared, 0) + 1 for n in lens]
    pages = shared + sum(taken) + 3
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    at = torch.full((batch, each), -1, dtype=torch.int64)      # no page where a sequence does not reach
    first = shared
    for b in range(batch):
        own_pages = min(taken[b], each - shared)
        at[b, :shared] = torch.arange(shared)
        at[b, shared: shared + own_pages] = torch.arange(first, first + own_pages)
        first += taken[b]
    at = at.to(dev)
    s["table"] = torch.where(at >= 0, order[at.clamp(min=0)], -1).contiguous()
    if shared:
        s["shared"] = order[:shared].clone()
    channel = torch.exp(0.5 * normal(DIM))                     # keys have channels of larger magnitude
    s["k"] = (normal(pages, nkv, page, DIM) * channel).to(torch.bfloat16)
    s["v"] = (normal(pages, nkv, page, DIM) + normal(DIM)).to(torch.bfloat16)      # values have a mean
    if case["op"] == "append":
        start, count, nt = _spread(batch, case["start"], case["ragged"]), _counts(case), case["tokens"]
        s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
        s["count"] = torch.tensor(count, dtype=torch.int32, device=dev)
        s["len"] = s["start"].clone()
        s["k_min"], s["k_max"] = s["k"].amin(2), s["k"].amax(2)
        s["qkv"] = normal(batch, nt, (nq + 2 * nkv) * DIM).to(getattr(torch, case["dtype"]))
        s["q"] = torch.zeros((batch, nt, nq, DIM), dtype=torch.bfloat16, device=dev)
        return s
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    q = normal(batch, nq, DIM)
    s["q"] = q.to(torch.bfloat16)
    # a few positions have keys near the mean query of a sequence's group: more of them in some pages than in others
    mean = q.view(batch, nkv, -1, DIM).mean(2)
    near = 6.0 * mean / mean.norm(dim=-1, keepdim=True)
    whose = torch.randint(0, batch, (pages,), generator=gen, device=dev)
    if not shared:
        whose[s["table"].clamp(min=0).long()] = torch.arange(batch, device=dev)[:, None].expand(batch, each)
    rate = 0.2 * torch.rand((pages,), generator=gen, device=dev) ** 8
    heavy = torch.rand((pages, page), generator=gen, device=dev) < rate[:, None]
    hp, hr = heavy.nonzero(as_tuple=True)
    s["k"][hp, :, hr] = (s["k"][hp, :, hr].float() + near[whose[hp]]).to(torch.bfloat16)
    s["active"] = None
    if case["ragged"]:
        s["active"] = (torch.arange(batch, device=dev) % 5 != 4).to(torch.int32)
    s["out"] = torch.zeros((batch, nq, DIM), dtype=torch.bfloat16, device=dev)
    if case["op"] == "sparse":
        held = s["k"].float()
        # a sequence's last page: its bounds are those of the positions that it holds
        live = torch.ones((pages, page), dtype=torch.bool, device=dev)
        ends = [(b, n) for b, n in enumerate(lens) if n % page]
        for b, n in ends:
            live[s["table"][b, n // page].long()] = torch.arange(page, device=dev) < n % page
        live = live[:, None, :, None]
        s["k_min"] = held.masked_fill(~live, math.inf).amin(2).to(torch.bfloat16)
        s["k_max"] = held.masked_fill(~live, -math.inf).amax(2).to(torch.bfloat16)
        s["page_idx"] = torch.full((batch, nkv, case["top"]), -1, dtype=torch.int32, device=dev)
    return s


# -------------------------------------------------------------------------------------------------- the plain forms
def _frequencies(case, dev):
    """Radians per position of every rotated pair, and what sine and cosine are multiplied by; in 64 bits."""
    rot, factor = case["rot"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    f = THETA ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "bands":       # long wavelengths are stretched, short ones kept, those between blended
        keep = ((TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 1.0
    if case["scaling"] == "ramp":        # by the pair's number, between those that turn FAST and SLOW times in all
        lo, hi = (rot * math.log(TRAINED / (n * 2 * math.pi)) / (2 * math.log(THETA)) for n in (FAST, SLOW))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _plain_append(s):
    case = s["case"]
    nq, nkv, rot, page, nt = case["q_heads"], case["kv_heads"], case["rot"], case["page"], case["tokens"]
    dev = s["k"].device
    t = torch.arange(nt, device=dev)
    pos = s["start"].long()[:, None] + t                                   # [B, T]
    f, amp = _frequencies(case, dev)
    a = pos.double()[..., None] * f
    cos, sin = ((g(a) * amp).float()[:, :, None] for g in (torch.cos, torch.sin))
    x = s["qkv"].view(*pos.shape, nq + 2 * nkv, DIM).float()
    head, kept = x[:, :, : nq + nkv, :rot], x[:, :, : nq + nkv, rot:]
    if case["layout"] == "half":
        u, w = head[..., : rot // 2], head[..., rot // 2:]
        turned = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
    else:
        u, w = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)
    y = torch.cat([turned, kept], -1).to(torch.bfloat16)
    live = t < s["count"][:, None]
    bi, ti = live.nonzero(as_tuple=True)
    s["q"][bi, ti] = y[bi, ti, :nq]
    new = y[bi, ti, nq:]                                                   # [n, Hkv, 128]
    p = pos[bi, ti]
    at, row = s["table"][bi, p // page].long(), p % page
    s["k"][at, :, row] = new
    s["v"][at, :, row] = s["qkv"].view(*pos.shape, nq + 2 * nkv, DIM)[bi, ti, nq + nkv:].to(torch.bfloat16)
    # a page whose first position is written begins anew; the bounds of another take the new keys in
    fresh = at[row == 0]
    s["k_min"][fresh], s["k_max"][fresh] = math.inf, -math.inf
    where = at[:, None, None].expand(-1, nkv, DIM)
    for name, how in (("k_min", "amin"), ("k_max", "amax")):
        s[name].copy_(s[name].float().scatter_reduce(0, where, new.float(), how))
    s["len"].copy_(s["start"] + s["count"])


def _softmax(x, live):
    """Of the last axis, over the places where live; rows without any are zeros."""
    x = x.masked_fill(~live, -math.inf)
    some = live.any(-1, keepdim=True)
    x = torch.exp(x - torch.where(some, x.amax(-1, keepdim=True), 0.0))
    return x / torch.where(some, x.sum(-1, keepdim=True), 1.0)


def _answer(s, o):
    on = (s["len"] >= 0) if s["active"] is None else s["active"] != 0
    s["out"].copy_(torch.where(on[:, None, None], o.reshape(s["out"].shape), s["out"].float()))


def _plain_sparse(s):
    case = s["case"]
    batch, nkv, page, top = case["batch"], case["kv_heads"], case["page"], case["top"]
    dev = s["q"].device
    n = -(-s["len"].long() // page)                                        # pages of every sequence
    most = int(-(-max(_lengths(case)) // page))
    where = s["table"][:, :most].clamp(min=0).long()
    p = torch.arange(most, device=dev)
    # the largest product that a key within the page's bounds can have with a query of the group; in 64 bits, because
    # pages next to the border of the selection lie close together
    q = s["q"].double().view(batch, nkv, -1, DIM)
    lo, hi = (s[m][where].double().permute(0, 2, 3, 1) for m in ("k_min", "k_max"))     # [B, Hkv, 128, P]
    score = (q.clamp(min=0) @ hi + q.clamp(max=0) @ lo).amax(2)            # [B, Hkv, P]
    keep = (p < 1) | (p >= n[:, None] - 1)                                 # the first page and the last one always
    score = torch.where(keep[:, None], math.inf, score).masked_fill((p >= n[:, None])[:, None], -math.inf)
    took = min(top, most)
    idx = score.sort(dim=-1, descending=True, stable=True).indices[..., :took]
    past = torch.arange(took, device=dev) >= n[:, None]
    idx = idx.masked_fill(past[:, None], 1 << 30).sort(-1).values
    idx = idx.masked_fill(idx == 1 << 30, -1)
    on = torch.ones_like(s["len"]) if s["active"] is None else s["active"]
    whole = torch.full_like(s["page_idx"], -1)
    whole[..., :took] = idx
    s["page_idx"].copy_(torch.where(on[:, None, None] != 0, whole, s["page_idx"]))
    at = s["table"].long()[torch.arange(batch, device=dev)[:, None, None], idx.clamp(min=0)].clamp(min=0)
    head = torch.arange(nkv, device=dev)[:, None]
    k = s["k"][at, head].float().flatten(2, 3)                             # [B, Hkv, took * page, 128]
    v = s["v"][at, head].float().flatten(2, 3)
    pos = idx[..., None] * page + torch.arange(page, device=dev)
    live = ((idx >= 0)[..., None] & (pos < s["len"][:, None, None, None])).flatten(2)
    x = s["q"].float().view(batch, nkv, -1, DIM) @ k.transpose(-1, -2) / math.sqrt(DIM)
    _answer(s, _softmax(x, live[:, :, None]) @ v.masked_fill(~live[..., None], 0.0))


def _plain_shared(s):
    case = s["case"]
    batch, nkv, page, prefix = case["batch"], case["kv_heads"], case["page"], case["prefix"]
    dev = s["q"].device
    q = s["q"].float().view(batch, nkv, -1, DIM)
    most = s["table"].shape[1] * page - prefix
    where = s["table"][:, prefix // page:].clamp(min=0).long()
    k, v = (s[m][where].float().permute(0, 2, 1, 3, 4).flatten(2, 3) for m in ("k", "v"))   # [B, Hkv, most, 128]
    live = (torch.arange(prefix + most, device=dev) < s["len"][:, None])[:, None, None]     # [B, 1, 1, N]
    v = v.masked_fill(~live[:, :, 0, prefix:, None], 0.0)
    x = q @ k.transpose(-1, -2)
    if prefix:
        pk, pv = (s[m][s["shared"].long()].float().transpose(0, 1).flatten(1, 2) for m in ("k", "v"))  # [Hkv, prefix, 128]
        rows = q.transpose(0, 1).flatten(1, 2)                             # [Hkv, B * G, 128]
        px = (rows @ pk.transpose(-1, -2)).view(nkv, batch, -1, prefix).transpose(0, 1)
        x = torch.cat([px, x], -1)
    p = _softmax(x / math.sqrt(DIM), live)
    o = p[..., prefix:] @ v
    if prefix:
        first = p[..., :prefix].transpose(0, 1).flatten(1, 2) @ pv
        o = o + first.view(nkv, batch, -1, DIM).transpose(0, 1)
    _answer(s, o)


# ------------------------------------------------------------------------------------------------------ the own calls
def _context(case, longest):
    from paper_2411_05787_b200 import rkv
    key = (case["batch"], case["q_heads"], case["kv_heads"], longest, 64)
    if key not in _contexts:
        _contexts[key] = rkv.Context(*key)
    return _contexts[key]


def _own(s):
    case, op = s["case"], s["op"]
    from paper_2411_05787_b200 import rkv
    if "cache" not in s:
        longest = -(-max(max(_lengths(case)), 1) // 1024) * 1024
        s["longest"] = longest
        s["ctx"] = _context(case, longest)
        s["cache"] = rkv.paged_cache_struct(s["k"], s["v"], s["table"], s["len"], s.get("k_min"), s.get("k_max"))
        if op == "append":
            s["rope"] = rkv.RopeTable(case["rot"], THETA, case["layout"], case["scaling"], case["factor"],
                                      trained_len=TRAINED, low=LOW, high=HIGH, fast=FAST, slow=SLOW, device=s["k"].device)
    if op == "append":
        s["ctx"].paged_append(s["qkv"], s["cache"], s["rope"], s["q"], start=s["start"], count=s["count"])
    elif op == "sparse":
        s["ctx"].paged_sparse_attention(s["q"], s["cache"], case["top"], s["page_idx"], s["out"], active=s["active"])
    else:
        s["ctx"].paged_attention(s["q"], s["cache"], s["out"], active=s["active"], shared=s.get("shared"))


def run(state):
    s = state
    if own:
        _own(s)
    elif s["op"] == "append":
        _plain_append(s)
    elif s["op"] == "sparse":
        _plain_sparse(s)
    else:
        _plain_shared(s)
    if s["op"] == "append":
        return {m: s[m] for m in ("q", "k", "v", "k_min", "k_max", "len")}
    if s["op"] == "sparse":
        return {"page_idx": s["page_idx"], "out": s["out"]}
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------------------- the work
def work(case):
    nq, nkv, page = case["q_heads"], case["kv_heads"], case["page"]
    row = 2 * DIM                                              # bytes of one bf16 row
    if case["op"] == "append":
        n = sum(_counts(case))
        size = 4 if case["dtype"] == "float32" else 2
        heads = n * (nq + 2 * nkv)
        return {"bytes": heads * DIM * size + heads * row, "flops": 3 * n * (nq + nkv) * case["rot"]}
    lens = [n for b, n in enumerate(_lengths(case)) if not case["ragged"] or b % 5 != 4]
    ends = 2 * len(lens) * nq * row                            # queries and outputs
    if case["op"] == "sparse":
        pages = [-(-n // page) for n in lens]
        took = [min(n, case["top"] * page) for n in lens]
        rows = sum(took) * nkv * 2 + sum(pages) * nkv * 2
        return {"bytes": rows * row + ends + len(lens) * nkv * case["top"] * 4,
                "flops": 4 * DIM * nq * sum(took) + 4 * DIM * nq * sum(pages)}
    alone = sum(n - case["prefix"] if n >= case["prefix"] else n for n in lens)
    return {"bytes": (case["prefix"] + alone) * nkv * 2 * row + ends, "flops": 4 * DIM * nq * sum(lens)}


# ------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    """Sequence by sequence and head by head, from the inputs alone."""
    s = prepare(case, seed)
    nq, nkv, page = case["q_heads"], case["kv_heads"], case["page"]
    group, dev = nq // nkv, s["k"].device
    lens = _lengths(case)
    if case["op"] == "append":
        return _exact_append(s, case, lens, dev)
    live = [True] * case["batch"] if s["active"] is None else [bool(a) for a in s["active"].tolist()]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=dev)
    idx = None
    if case["op"] == "sparse":
        idx = torch.full(s["page_idx"].shape, -1, dtype=torch.int64)
    for b, n in enumerate(lens):
        if not live[b] or n == 0:
            continue
        pages = s["table"][b, : -(-n // page)].long()
        k, v = s["k"][pages].double(), s["v"][pages].double()              # [P, Hkv, page, 128]
        for g in range(nkv):
            q = s["q"][b, g * group: (g + 1) * group].double()
            chosen = torch.arange(len(pages), device=dev)
            if idx is not None:
                rows = torch.arange(len(pages) * page, device=dev).view(-1, page, 1)
                lo = k[:, g].masked_fill(rows >= n, math.inf).amin(1)      # the bounds, from the keys themselves
                hi = k[:, g].masked_fill(rows >= n, -math.inf).amax(1)
                best = torch.stack([torch.maximum(lo * h, hi * h).sum(-1) for h in q]).amax(0).tolist()
                best[0] = best[-1] = math.inf
                chosen = sorted(sorted(range(len(pages)), key=lambda i: (-best[i], i))[: case["top"]])
                idx[b, g, : len(chosen)] = torch.tensor(chosen)
                chosen = torch.tensor(chosen, device=dev)
            pos = (chosen[:, None] * page + torch.arange(page, device=dev)).flatten()
            kk, vv = (m[chosen, g].flatten(0, 1)[pos < n] for m in (k, v))
            w = q @ kk.t() / math.sqrt(DIM)
            out[b, g * group: (g + 1) * group] = torch.softmax(w, -1) @ vv
    return {"out": out} if idx is None else {"out": out, "page_idx": idx.to(torch.int32)}


def _exact_append(s, case, lens, dev):
    nq, nkv, page, rot = case["q_heads"], case["kv_heads"], case["page"], case["rot"]
    f, amp = _frequencies(case, dev)
    held = {m: s[m].double() for m in ("q", "k", "v", "k_min", "k_max")}
    for b, (first, count) in enumerate(zip(s["start"].tolist(), s["count"].tolist())):
        if count == 0:
            continue
        x = s["qkv"][b, :count].double().view(count, nq + 2 * nkv, DIM)
        angle = torch.arange(first, first + count, dtype=torch.float64, device=dev)[:, None] * f
        turn = torch.polar(torch.full_like(angle, amp), angle)[:, None]    # a rotation is a product with e^ia
        part = x[:, : nq + nkv, :rot].clone()
        i = torch.arange(rot // 2, device=dev)
        re, im = (i, i + rot // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(part[..., re], part[..., im]) * turn
        part[..., re], part[..., im] = z.real, z.imag
        x[:, : nq + nkv, :rot] = part
        held["q"][b, :count] = x[:, :nq]
        pos = torch.arange(first, first + count, device=dev)
        at = s["table"][b].long()[pos // page]
        held["k"][at, :, pos % page] = x[:, nq: nq + nkv]
        held["v"][at, :, pos % page] = x[:, nq + nkv:]
        for i in range(first // page, (first + count - 1) // page + 1):
            here = x[max(i * page - first, 0): (i + 1) * page - first, nq: nq + nkv]
            lo, hi = here.amin(0), here.amax(0)
            to = int(s["table"][b, i])
            if i * page < first:
                lo, hi = torch.minimum(lo, held["k_min"][to]), torch.maximum(hi, held["k_max"][to])
            held["k_min"][to], held["k_max"][to] = lo, hi
    held["len"] = torch.tensor(lens, dtype=torch.int32)
    return held
