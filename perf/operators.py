"""Cases of the 8-bit full cache and of the rotary positions in front of it: storing rows, attention over them, the
rebuild of the bf16 small cache from them, and the rotation of queries and keys.

The 8-bit cache holds e4m3 rows of 128 channels and one scale, a power of two, per block of 64 positions and KV head
(K and V apart).  Sequence b, KV head g, position p is row row_offset[b] + g * cap[b] + p; row_offset and cap are
multiples of 64, so that a row's block is row // 64.  A block's scale is the smallest power of two (not below 2^-126)
with which its largest magnitude is at most 448; rows that join a block of larger magnitude than it had raise the
scale, and the rows it held are encoded again.
"""
import math

import torch

own = False

DIM, BLOCK = 128, 64
_contexts = {}   # a program keeps one context per shape of its batch


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one decoded token of one sequence joins a long cache: latency
        dict(name="store token", op="store", batch=1, kv_heads=8, start=32801, tokens=1, ragged=False, strided=False),
        # a prompt's rows, in one call
        dict(name="store prompt", op="store", batch=1, kv_heads=8, start=0, tokens=32768, ragged=False, strided=False),
        # chunked prompts of a ragged batch: partly filled blocks, sequences without new rows, V read out of a projection
        dict(name="store ragged chunk", op="store", batch=4, kv_heads=4, start=10007, tokens=2000, ragged=True, strided=True),
        # a short context: latency
        dict(name="attend 1000", op="attend", batch=1, q_heads=32, kv_heads=8, length=1000, ragged=False, scores=True),
        # the ordinary full step
        dict(name="attend 32768", op="attend", batch=1, q_heads=32, kv_heads=8, length=32768, ragged=False, scores=True),
        # a long context, attention alone
        dict(name="attend 131072", op="attend", batch=1, q_heads=32, kv_heads=8, length=131072, ragged=False, scores=False),
        # a ragged batch with seven query heads to a KV head, sequences that are masked or empty
        dict(name="attend ragged batch", op="attend", batch=16, q_heads=28, kv_heads=4, length=65535, ragged=True, scores=True),
        # the rebuild of one sequence's small cache, and of a ragged batch's
        dict(name="rebuild 2048", op="rebuild", batch=1, kv_heads=8, length=32768, keep=2048, ragged=False),
        dict(name="rebuild ragged batch", op="rebuild", batch=4, kv_heads=4, length=65536, keep=4096, ragged=True),
        # one token of the decode loop, frequencies scaled by wavelength bands
        dict(name="rope token", op="rope", tokens=1, q_heads=32, kv_heads=8, first=32801, rot=128, layout="half",
             dtype="float32", scaling="bands", factor=8.0),
        # a prompt
        dict(name="rope prompt", op="rope", tokens=32768, q_heads=32, kv_heads=8, first=0, rot=128, layout="half",
             dtype="bfloat16", scaling="none", factor=1.0),
        # a chunk far into a long context: half of the head rotated, adjacent pairs, frequencies ramped
        dict(name="rope interleaved part", op="rope", tokens=4097, q_heads=28, kv_heads=4, first=120011, rot=64,
             layout="interleaved", dtype="bfloat16", scaling="ramp", factor=4.0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "attend", "attend", "rebuild", "rope"])
    if op == "rope":
        dtype = rng.choice(["float32", "bfloat16", "bfloat16"])
        return dict(op=op, tokens=_log(rng, 1, 21000 if dtype == "float32" else 32768), q_heads=rng.choice([8, 28, 32]),
                    kv_heads=rng.choice([1, 4, 8]), first=rng.randrange(0, 131072), rot=16 * rng.randint(1, 8),
                    layout=rng.choice(["half", "interleaved"]), dtype=dtype,
                    scaling=rng.choice(["none", "linear", "bands", "ramp"]), factor=rng.choice([2.0, 4.0, 8.0, 10.0]))
    kv_heads = rng.choice([1, 2, 4, 8])
    batch = _log(rng, 1, 16)
    ragged = batch > 1 and rng.random() < 0.7
    room = 16 * 4 * 40000 // (batch * kv_heads)     # positions per (sequence, KV head), the largest listed batch's
    if op == "store":
        tokens = _log(rng, 1, max(1, min(32768, 32768 * 8 // (batch * kv_heads))))
        return dict(op=op, batch=batch, kv_heads=kv_heads, start=rng.randrange(0, max(1, min(16384, room // 4))),
                    tokens=tokens, ragged=ragged, strided=rng.random() < 0.5)
    length = _log(rng, 1, min(131072, room))
    if op == "attend":
        return dict(op=op, batch=batch, q_heads=kv_heads * rng.randint(1, 8), kv_heads=kv_heads, length=length,
                    ragged=ragged, scores=rng.random() < 0.6)
    length = max(1, min(length, 65536 * 16 // (batch * kv_heads)))
    return dict(op=op, batch=batch, kv_heads=kv_heads, length=length,
                keep=_log(rng, 1, max(1, min(length, 8192, 65536 // (batch * kv_heads)))), ragged=ragged)


def _spread(batch, most, ragged, least=0):
    """A size per sequence: all alike, or spread below the largest, the second least and the fourth a single one."""
    if not ragged:
        return [most] * batch
    sizes = [most] + [least + (most - least) * (5 * b % 16 + 1) // 17 for b in range(1, batch)]
    sizes[1] = least
    if batch > 3:
        sizes[3] = min(most, 1)
    return sizes


def _round64(n):
    return max(BLOCK, -(-n // BLOCK) * BLOCK)


# ------------------------------------------------------------------------------------------------------ the inputs
def _layout(caps, kv_heads, dev):
    """(row_offset, cap, rows in all) of a packed cache."""
    cap = torch.tensor(caps, dtype=torch.int32, device=dev)
    size = cap.long() * kv_heads
    return torch.cumsum(size, 0) - size, cap, int(sum(caps)) * kv_heads


def _scale_of(most):
    """The scale of blocks whose largest magnitudes are `most`."""
    m, e = torch.frexp(most)                                   # most = m 2^e, 0.5 <= m < 1;  448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return torch.ldexp(torch.ones_like(most), torch.where(most > 0, e, -126))


def _filled(rows, spread, mean, gen, dev):
    """An 8-bit cache of random rows: codes and scales."""
    x = torch.randn((rows, DIM), generator=gen, device=dev, dtype=torch.float32) * spread + mean
    scale = _scale_of(x.view(-1, BLOCK * DIM).abs().amax(1))
    return (x / scale.repeat_interleave(BLOCK)[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    s = dict(case=case, op=case["op"])
    if case["op"] == "rope":
        nt, nq, nkv = case["tokens"], case["q_heads"], case["kv_heads"]
        s["qkv"] = normal(nt, (nq + 2 * nkv) * DIM).to(getattr(torch, case["dtype"]))
        s["pos"] = torch.arange(case["first"], case["first"] + nt, dtype=torch.int32, device=dev)
        for name, heads in (("q", nq), ("k", nkv), ("v", nkv)):
            s[name] = torch.zeros((nt, heads, DIM), dtype=torch.bfloat16, device=dev)
        return s
    batch, kv_heads = case["batch"], case["kv_heads"]
    channel = torch.exp(0.5 * normal(DIM))                     # keys have channels of larger magnitude
    if case["op"] == "store":
        start = _spread(batch, case["start"], case["ragged"])
        count = _spread(batch, case["tokens"], case["ragged"])[::-1]
        caps = [_round64(case["start"] + case["tokens"])] * batch
    else:
        lens = _spread(batch, case["length"], case["ragged"])
        caps = [_round64(n + 1) for n in lens]
    s["row_offset"], s["cap"], rows = _layout(caps, kv_heads, dev)
    s["k8"], s["k_scale"] = _filled(rows, channel, 0.0, gen, dev)
    s["v8"], s["v_scale"] = _filled(rows, 1.0, normal(DIM), gen, dev)   # values have a mean
    if case["op"] == "store":
        nt = case["tokens"]
        s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
        s["count"] = torch.tensor(count, dtype=torch.int32, device=dev)
        s["len"] = s["start"].clone()
        loud = torch.exp2(torch.arange(kv_heads, device=dev) % 3)[:, None]      # some heads' new rows raise the scale
        s["k_new"] = (normal(batch, nt, kv_heads, DIM) * channel * loud).to(torch.bfloat16)
        if case["strided"]:                                    # V as it lies in the projection's rows
            s["v_new"] = normal(batch, nt, 3 * kv_heads, DIM).to(torch.bfloat16)[:, :, 2 * kv_heads:]
        else:
            s["v_new"] = normal(batch, nt, kv_heads, DIM).to(torch.bfloat16)
        return s
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    if case["op"] == "attend":
        nq = case["q_heads"]
        q = normal(batch, nq, DIM)
        s["q"] = q.to(torch.bfloat16)
        # one position in a hundred has a key near the group's mean query
        heavy = torch.rand((rows,), generator=gen, device=dev) < 0.01
        mean = q.view(batch, kv_heads, -1, DIM).mean(2)
        near = (6.0 * mean / mean.norm(dim=-1, keepdim=True)).view(-1, DIM)
        of_row = torch.repeat_interleave(torch.arange(batch * kv_heads, device=dev),
                                         s["cap"].long().repeat_interleave(kv_heads))
        at = heavy.nonzero()[:, 0]
        lift = near[of_row[at]] / s["k_scale"][at // BLOCK][:, None]
        s["k8"][at] = (s["k8"][at].float() + lift).clamp(-448, 448).to(torch.float8_e4m3fn)
        s["active"] = None
        if case["ragged"]:
            s["active"] = (torch.arange(batch, device=dev) % 5 != 4).to(torch.int32)
        s["out"] = torch.zeros((batch, nq, DIM), dtype=torch.bfloat16, device=dev)
        if case["scores"]:
            s["scores"] = torch.zeros((batch, kv_heads, max(lens)), dtype=torch.float32, device=dev)
            s["k_small"] = torch.ones((batch,), dtype=torch.int32, device=dev)
        return s
    keep = [min(n, k) for n, k in zip(lens, _spread(batch, case["keep"], case["ragged"]))]
    k_max = max(keep)
    s["k_small"] = torch.tensor(keep, dtype=torch.int32, device=dev)
    order = torch.rand((batch, kv_heads, max(lens)), generator=gen, device=dev)
    order.masked_fill_(torch.arange(max(lens), device=dev) >= s["len"][:, None, None], 2.0)
    idx = order.argsort(-1)[..., :k_max].to(torch.int32)
    past = torch.arange(k_max, device=dev) >= s["k_small"][:, None, None]
    idx = idx.masked_fill(past, 1 << 30).sort(-1).values
    s["topk_idx"] = idx.masked_fill(past, -1).contiguous()
    s["small_offset"], s["small_cap"], small_rows = _layout([_round64(k) for k in keep], kv_heads, dev)
    s["small_k"] = torch.zeros((small_rows, DIM), dtype=torch.bfloat16, device=dev)
    s["small_v"] = torch.zeros((small_rows, DIM), dtype=torch.bfloat16, device=dev)
    s["small_len"] = torch.zeros((batch,), dtype=torch.int32, device=dev)
    return s


# -------------------------------------------------------------------------------------------------- the plain forms
def _head_rows(row_offset, cap, kv_heads):
    """First row of every (sequence, KV head): [B, Hkv]."""
    return row_offset[:, None] + torch.arange(kv_heads, device=cap.device) * cap.long()[:, None]


def _plain_store(s, x, codes, scale):
    batch, nt, kv_heads, _ = x.shape
    dev = x.device
    head = _head_rows(s["row_offset"], s["cap"], kv_heads)
    start, count, cap = s["start"].long(), s["count"].long(), s["cap"].long()
    t = torch.arange(nt, device=dev)
    live = (t < count[:, None]) & (start[:, None] + t < cap[:, None])
    b_at, t_at = live.nonzero(as_tuple=True)
    rows = head[b_at] + (start[b_at] + t_at)[:, None]                      # [n, Hkv]
    new = x[b_at, t_at].float()                                            # [n, Hkv, 128]
    most = torch.full_like(scale, -1.0)
    most.scatter_reduce_(0, (rows // BLOCK).flatten(), new.abs().amax(-1).flatten(), "amax")
    fresh = torch.where(most >= 0, _scale_of(most.clamp(min=0)), scale)
    # the block that new rows join: its scale does not fall, and its older rows are encoded again
    joins = (start % BLOCK > 0) & (live.any(1))
    first = (head + (start // BLOCK * BLOCK)[:, None])[joins]              # [j, Hkv] first rows of such blocks
    old = scale[first // BLOCK]
    fresh[first // BLOCK] = torch.maximum(old, fresh[first // BLOCK])
    older = torch.arange(BLOCK, device=dev) < (start % BLOCK)[joins][:, None, None]
    at = first[..., None] + torch.arange(BLOCK, device=dev)
    held = codes[at]
    again = (held.float() * (old / fresh[first // BLOCK])[..., None, None]).to(torch.float8_e4m3fn)
    codes[at] = torch.where(older[..., None], again.float(), held.float()).to(torch.float8_e4m3fn)
    codes[rows] = (new / fresh[rows // BLOCK][..., None]).to(torch.float8_e4m3fn)
    scale.copy_(fresh)
    return live.sum(1)


def _positions(s, codes, scale, kv_heads, longest):
    """Every sequence's rows as values, side by side: [B, Hkv, longest, 128]."""
    head = _head_rows(s["row_offset"], s["cap"], kv_heads)
    rows = head[..., None] + torch.minimum(torch.arange(longest, device=head.device), s["cap"].long()[:, None] - 1)[:, None]
    return codes[rows].float() * scale[rows // BLOCK][..., None]


def _plain_attend(s):
    case = s["case"]
    batch, kv_heads, longest = case["batch"], case["kv_heads"], case["length"]
    live = torch.arange(longest, device=s["q"].device) < s["len"][:, None]                    # [B, N]
    some = (s["len"] > 0)[:, None, None, None]
    on = torch.ones_like(s["len"]) if s["active"] is None else s["active"]
    on = (on != 0)[:, None, None]
    q = s["q"].float().view(batch, kv_heads, -1, DIM)
    x = q @ _positions(s, s["k8"], s["k_scale"], kv_heads, longest).transpose(-1, -2) / math.sqrt(DIM)
    x = x.masked_fill(~live[:, None, None], -math.inf)
    x = torch.exp(x - torch.where(some, x.amax(-1, keepdim=True), 0.0))
    p = x / torch.where(some, x.sum(-1, keepdim=True), 1.0)
    v = _positions(s, s["v8"], s["v_scale"], kv_heads, longest).masked_fill(~live[:, None, :, None], 0.0)
    s["out"].copy_(torch.where(on, (p @ v).view(batch, -1, DIM), s["out"].float()))
    if case["scores"]:
        s["scores"].copy_(torch.where(on & live[:, None], p.amax(2), s["scores"]))


def _plain_rebuild(s):
    kv_heads, k_max = s["topk_idx"].shape[1:]
    head = _head_rows(s["row_offset"], s["cap"], kv_heads)
    to = _head_rows(s["small_offset"], s["small_cap"], kv_heads)
    m = torch.minimum(s["k_small"], s["len"])
    r = torch.arange(k_max, device=m.device)
    live = ((r < m[:, None])[:, None] & (s["topk_idx"] >= 0)).nonzero(as_tuple=True)
    rows = head[live[0], live[1]] + s["topk_idx"][live].long()
    at = to[live[0], live[1]] + live[2]
    s["small_k"][at] = (s["k8"][rows].float() * s["k_scale"][rows // BLOCK][:, None]).to(torch.bfloat16)
    s["small_v"][at] = (s["v8"][rows].float() * s["v_scale"][rows // BLOCK][:, None]).to(torch.bfloat16)
    s["small_len"].copy_(m)


THETA, TRAINED, LOW, HIGH, FAST, SLOW = 500000.0, 8192, 1.0, 4.0, 32.0, 1.0


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


def _plain_rope(s):
    case = s["case"]
    nt, nq, nkv, rot = case["tokens"], case["q_heads"], case["kv_heads"], case["rot"]
    f, amp = _frequencies(case, s["pos"].device)
    a = s["pos"].double()[:, None] * f
    cos, sin = ((t(a) * amp).float()[:, None] for t in (torch.cos, torch.sin))
    x = s["qkv"].view(nt, nq + 2 * nkv, DIM).float()
    head, rest = x[:, : nq + nkv, :rot], x[:, : nq + nkv, rot:]
    if case["layout"] == "half":
        u, w = head[..., : rot // 2], head[..., rot // 2:]
        turned = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
    else:
        u, w = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)
    y = torch.cat([turned, rest], -1)
    s["q"].copy_(y[:, :nq])
    s["k"].copy_(y[:, nq:])
    s["v"].copy_(x[:, nq + nkv:])


# ------------------------------------------------------------------------------------------------------ the own calls
def _context(case, longest):
    from paper_2411_05787_b200 import rkv
    key = (case.get("batch", 1), case.get("q_heads", case["kv_heads"]), case["kv_heads"], longest, case.get("keep", 1))
    if key not in _contexts:
        _contexts[key] = rkv.Context(*key)
    return _contexts[key]


def _own(s):
    case, op = s["case"], s["op"]
    from paper_2411_05787_b200 import rkv
    if op == "rope":
        if "table" not in s:
            s["table"] = rkv.RopeTable(case["rot"], THETA, case["layout"], case["scaling"], case["factor"],
                                       trained_len=TRAINED, low=LOW, high=HIGH, fast=FAST, slow=SLOW,
                                       device=s["qkv"].device)
            s["ctx"] = _context(dict(kv_heads=1), 1)      # (the rotation takes its heads from its tensors)
        s["ctx"].rope(s["qkv"], s["pos"], s["table"], s["q"], s["k"], s["v"])
        return
    if "cache" not in s:
        s["cache"] = rkv.quant_cache_struct(s["k8"], s["v8"], s["k_scale"], s["v_scale"], s["row_offset"], s["cap"],
                                            s["len"])
        s["ctx"] = _context(case, int(s["cap"].max()))
        if op == "rebuild":
            s["small"] = rkv.cache_struct(s["small_k"], s["small_v"], s["small_offset"], s["small_cap"], s["small_len"])
    ctx, cache = s["ctx"], s["cache"]
    if op == "store":
        ctx.quant_store(s["k_new"], s["v_new"], cache, start=s["start"], count=s["count"])
    elif op == "attend":
        ctx.quant_full_attention(s["q"], cache, s["out"], active=s["active"], max_len_hint=case["length"],
                                 keep_logits=case["scores"])
        if case["scores"]:
            ctx.score_keys(s["q"], cache, s["k_small"], 1, active=s["active"], scores=s["scores"])
    else:
        ctx.quant_gather_small(s["topk_idx"], s["k_small"], s["topk_idx"].shape[-1], cache, s["small"])


def run(s):
    if own:
        _own(s)
    elif s["op"] == "store":
        count = _plain_store(s, s["k_new"], s["k8"], s["k_scale"])
        _plain_store(s, s["v_new"], s["v8"], s["v_scale"])
        s["len"].copy_(s["start"] + count)
    elif s["op"] == "attend":
        _plain_attend(s)
    elif s["op"] == "rebuild":
        _plain_rebuild(s)
    else:
        _plain_rope(s)
    return {name: s[name] for name in _outputs(s["case"])}


def _outputs(case):
    if case["op"] == "store":
        return ["k8", "v8", "k_scale", "v_scale", "len"]
    if case["op"] == "attend":
        return ["out", "scores"] if case["scores"] else ["out"]
    return ["small_k", "small_v", "small_len"] if case["op"] == "rebuild" else ["q", "k", "v"]


def work(case):
    if case["op"] == "rope":
        n = case["tokens"] * DIM
        heads = case["q_heads"] + 2 * case["kv_heads"]
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": n * heads * (size + 2) + 4 * case["tokens"],
                "flops": 3 * case["tokens"] * case["rot"] * (case["q_heads"] + case["kv_heads"])}
    batch, kv_heads = case["batch"], case["kv_heads"]
    if case["op"] == "store":
        rows = sum(_spread(batch, case["tokens"], case["ragged"])) * kv_heads
        return {"bytes": rows * 2 * (2 * DIM + DIM) + rows * 2 * 4 // BLOCK + 16 * batch, "flops": rows * 2 * DIM * 2}
    lens = _spread(batch, case["length"], case["ragged"])
    if case["op"] == "rebuild":
        rows = sum(min(n, k) for n, k in zip(lens, _spread(batch, case["keep"], case["ragged"]))) * kv_heads
        return {"bytes": rows * (2 * (DIM + 2 * DIM) + 4 + 8), "flops": rows * 2 * DIM}
    on = [n for b, n in enumerate(lens) if not (case["ragged"] and b % 5 == 4)]
    rows = sum(on) * kv_heads
    per = 2 * DIM + (4 if case["scores"] else 0)
    return {"bytes": rows * per + rows * 8 // BLOCK + len(on) * case["q_heads"] * DIM * 4,
            "flops": 4 * sum(on) * case["q_heads"] * DIM}


# ------------------------------------------------------------------------------------- the definition, in 64 bits
def _nearest_code(y):
    """The value on the e4m3 grid nearest to y, ties to even."""
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exact_frequencies(case):
    """Radians per position of every rotated pair, from its wavelength in positions; and the amplitude."""
    rot, factor, how = case["rot"], case["factor"], case["scaling"]
    turns = lambda n: rot * math.log(TRAINED / (2 * math.pi * n), THETA) / 2      # the pair that turns n times in all
    low, high = max(0, math.floor(turns(FAST))), min(rot - 1, math.ceil(turns(SLOW)))
    got = []
    for i in range(rot // 2):
        wave = 2 * math.pi * math.exp(2 * i / rot * math.log(THETA))
        slow = 2 * math.pi / (wave * factor)
        fast = 2 * math.pi / wave
        if how == "none":
            got.append(fast)
        elif how == "linear":
            got.append(slow)
        elif how == "bands":
            if wave < TRAINED / HIGH:
                got.append(fast)
            elif wave > TRAINED / LOW:
                got.append(slow)
            else:
                part = (TRAINED / wave - LOW) / (HIGH - LOW)
                got.append((1 - part) * slow + part * fast)
        else:
            part = 0.0 if i <= low else min(1.0, (i - low) / max(high - low, 0.001))
            got.append(part * slow + (1 - part) * fast)
    return got, 1.0 + 0.1 * math.log(factor) if how == "ramp" else 1.0


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        nq, nkv, rot = case["q_heads"], case["kv_heads"], case["rot"]
        f, amp = (torch.tensor(v, dtype=torch.float64, device=s["pos"].device) for v in _exact_frequencies(case))
        x = s["qkv"].double().view(-1, nq + 2 * nkv, DIM)
        one = torch.arange(rot // 2, device=x.device)
        u, w = (one, one + rot // 2) if case["layout"] == "half" else (2 * one, 2 * one + 1)
        z = torch.complex(x[:, : nq + nkv, u], x[:, : nq + nkv, w])
        z = z * torch.polar(amp.expand(len(x), rot // 2).contiguous(), torch.outer(s["pos"].double(), f))[:, None]
        x[:, : nq + nkv, u], x[:, : nq + nkv, w] = z.real, z.imag
        return {"q": x[:, :nq], "k": x[:, nq: nq + nkv], "v": x[:, nq + nkv:]}
    offset, cap = s["row_offset"].tolist(), s["cap"].tolist()
    kv_heads = case["kv_heads"]
    spans = [(b, g, offset[b] + g * cap[b]) for b in range(case["batch"]) for g in range(kv_heads)]
    if case["op"] == "store":
        start, count = s["start"].tolist(), s["count"].tolist()
        got = {"len": torch.tensor([p + min(n, c - p) for p, n, c in zip(start, count, cap)])}
        for name in ("k", "v"):
            codes, scale, new = s[name + "8"].double(), s[name + "_scale"].double(), s[name + "_new"]
            for b, g, row in spans:
                lo, hi = start[b], min(start[b] + count[b], cap[b])
                if hi <= lo:
                    continue
                first, last = lo // BLOCK * BLOCK, _round64(hi)
                held, was = codes[row + first: row + last], scale[(row + first) // BLOCK: (row + last) // BLOCK]
                value = torch.zeros_like(held)
                value[: lo - first] = held[: lo - first] * was[0]
                value[lo - first: hi - first] = new[b, : hi - lo, g].double()
                fresh = value.clone()
                fresh[: lo - first] = 0
                most = fresh.view(-1, BLOCK * DIM).abs().amax(1)
                part, up = torch.frexp(most / 448.0)                   # 2^(up - 1) is enough where it is just that
                up = torch.where(part == 0.5, up - 1, up).clamp(min=-126)
                now = torch.ldexp(torch.ones_like(most), torch.where(most > 0, up, -126))
                if lo > first:
                    now[0] = torch.maximum(now[0], was[0])
                code = _nearest_code(value / now.repeat_interleave(BLOCK)[:, None])
                code[hi - first:] = held[hi - first:]
                codes[row + first: row + last] = code
                scale[(row + first) // BLOCK: (row + last) // BLOCK] = now
            got[name + "8"], got[name + "_scale"] = codes, scale
        return got
    lens = s["len"].tolist()

    def values(name, rows):
        return s[name + "8"][rows].double() * s[name + "_scale"][rows // BLOCK].double()[:, None]

    if case["op"] == "rebuild":
        keep, to, room = s["k_small"].tolist(), s["small_offset"].tolist(), s["small_cap"].tolist()
        got = {"small_" + name: torch.zeros_like(s["small_" + name], dtype=torch.float64) for name in "kv"}
        for b, g, row in spans:
            n = min(keep[b], lens[b])
            for name in "kv":
                got["small_" + name][to[b] + g * room[b]:][:n] = values(name, row + s["topk_idx"][b, g, :n].long())
        return got
    group = case["q_heads"] // kv_heads
    out = torch.zeros_like(s["out"], dtype=torch.float64)
    scores = torch.zeros((case["batch"], kv_heads, max(lens)), dtype=torch.float64, device=out.device)
    for b, g, row in spans:
        if lens[b] == 0 or (s["active"] is not None and b % 5 == 4):
            continue
        rows = torch.arange(row, row + lens[b], device=out.device)
        heads = slice(g * group, (g + 1) * group)
        p = torch.softmax(s["q"][b, heads].double() @ values("k", rows).T / math.sqrt(DIM), -1)
        out[b, heads] = p @ values("v", rows)
        scores[b, g, : lens[b]] = p.amax(0)
    return {"out": out, "scores": scores} if case["scores"] else {"out": out}
