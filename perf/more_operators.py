"""The operators between a projection and its attention whose speed is followed:
finishing the rows of a projection (norms of queries and keys for each head and
the position rotation) and appending them to a cache in bf16 or in 4 bits, packing
a cache into 4 bits and reading it back, attention of a tree of drafted tokens
over a cache in 4 bits, and causal attention of whole prompts over a cache.

Each has its plain form in torch beside the call of this library.  Projected rows
are N(0, 1) with a size of their own for each head; queries N(0, 1.5) (a head
attends to some entries more than to others); one key dim in sixteen is four times
as large as the others, as keys before quantisation often have them.

A cache in 4 bits holds for each 16 consecutive dims of an entry a scale s of one
byte and 16 whole numbers c in -7 .. 7, and stands for s c.  The scale byte has five
bits of exponent (bias 15, the lowest for subnormals) and three of fraction, and is
that of the number nearest to a seventh of the largest magnitude of the 16, at most
896, ties to the even one; c is the whole number nearest to x / s, ties to the even
one, and 0 where s is.  Codes are c + 8: of 8 dims in a 32-bit word, dim 2e is in
bits 4e .. 4e + 3 and dim 2e + 1 in bits 4e + 16 .. 4e + 19.
"""
import math

import numpy as np
import torch

own = False
EPS, THETA = 1e-6, 1e6
ROOM = 37  # positions of a cache past what it holds and the call's own rows
MOST_SCORES = 2_000_000_000  # of a plain form at once

RAGGED_LENS = "6130 6416 2466 5349 5631 376 2509 7495 1702 5900 3266 3948 5116 817 1839 2625"
RAGGED_ROWS = "5 14 17 12 3 14 6 17 14 10 12 4 6 6 16 0"
ONE_EACH = "1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1"


def listed():
    return [
        # the smallest call: a block of five of the tiny decoder, no norms of its heads
        {"name": "append-tiny-5", "op": "append", "nq": 4, "nkv": 2, "d": 64, "lens": "200", "rows": "5",
         "type": "f32", "norm": False, "rotary": 64},
        # the prompt of five minutes of audio and an instruction
        {"name": "append-7b-7564", "op": "append", "nq": 28, "nkv": 4, "d": 128, "lens": "0", "rows": "7564",
         "type": "bf16", "norm": True, "rotary": 128},
        # a server's round of drafted blocks into caches of 4 bits, read back as they are checked
        {"name": "append4-7b-ragged16", "op": "append4", "nq": 28, "nkv": 4, "d": 128, "lens": RAGGED_LENS,
         "rows": RAGGED_ROWS, "type": "bf16", "norm": True, "rotary": 128},
        # the tiny decoder's prefix packed after its prefill
        {"name": "pack-tiny", "op": "pack", "layers": 2, "nkv": 2, "d": 64, "lens": "200"},
        # ten minutes of retained audio, every layer of the target, packed and read back
        {"name": "pack-7b-15128", "op": "pack", "layers": 28, "nkv": 4, "d": 128, "lens": "15128"},
        # the smallest call of attention: the tiny decoder's heads, a block of five as a chain
        {"name": "attend4-tiny-5", "op": "attend4", "nq": 4, "nkv": 2, "d": 64, "lens": "200", "rows": "5",
         "tree": "chain", "q": "bf16"},
        # one token of the target over ten minutes of audio
        {"name": "attend4-7b-decode-15128", "op": "attend4", "nq": 28, "nkv": 4, "d": 128, "lens": "15128",
         "rows": "1", "tree": "chain", "q": "bf16"},
        # a server's step: one token each of 16 requests
        {"name": "attend4-7b-decode-16", "op": "attend4", "nq": 28, "nkv": 4, "d": 128, "lens": RAGGED_LENS,
         "rows": ONE_EACH, "tree": "chain", "q": "bf16"},
        # a server's round of drafted trees, 32-bit queries, one request without rows
        {"name": "attend4-7b-ragged16", "op": "attend4", "nq": 28, "nkv": 4, "d": 128, "lens": RAGGED_LENS,
         "rows": RAGGED_ROWS, "tree": "random", "q": "f32"},
        # a short prompt of the tiny decoder
        {"name": "prompt-tiny-201", "op": "prompt", "nq": 4, "nkv": 2, "d": 64, "lens": "0", "rows": "201"},
        # a server's prompts side by side, two of them after what their caches hold already
        {"name": "prompt-7b-packed", "op": "prompt", "nq": 28, "nkv": 4, "d": 128, "lens": "0 0 814 0 1564 0 0 0",
         "rows": "1564 375 64 2029 301 1 814 967"},
        # the prompt of five minutes of audio and an instruction
        {"name": "prompt-7b-7564", "op": "prompt", "nq": 28, "nkv": 4, "d": 128, "lens": "0", "rows": "7564"},
    ]


def _ints(text):
    return [int(t) for t in text.split()]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


HEADS = ((4, 2, 64), (12, 2, 128), (28, 4, 128), (8, 8, 64), (16, 1, 128))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("append", "append4", "pack", "attend4", "attend4", "prompt", "prompt"))
        case = {"op": op}
        text = lambda values: " ".join(map(str, values))  # noqa: E731
        if op == "pack":
            case["layers"] = rng.choice((1, 2, 28))
            case["nkv"], case["d"] = rng.choice(((2, 64), (2, 128), (4, 128), (8, 64)))
            batch = 1 if rng.random() < 0.5 else _log_uniform(rng, 2, 16)
            case["lens"] = text(_log_uniform(rng, 1, 15128) for _ in range(batch))
            if _cost(case) <= most:
                return case
            continue
        case["nq"], case["nkv"], case["d"] = rng.choice(HEADS)
        batch = 1 if rng.random() < 0.5 else _log_uniform(rng, 2, 64 if op != "prompt" else 16)
        if op == "attend4":
            lens = [_log_uniform(rng, 1, 15128) for _ in range(batch)]
            top = rng.choice((1, 1, 17, 64))
            rows = [1 if top == 1 and batch == 1 else rng.randint(0, top) for _ in range(batch)]
            case["tree"], case["q"] = rng.choice(("chain", "random")), rng.choice(("bf16", "f32"))
        else:
            # new prompts, and rows after what is there already; or a step of a block each
            lens = [0 if rng.random() < 0.5 else _log_uniform(rng, 1, 7564) for _ in range(batch)]
            top = 7564 if op == "prompt" or rng.random() < 0.5 else 17
            rows = [_log_uniform(rng, 1, top) for _ in range(batch)]
            if op != "prompt":
                case["type"], case["norm"] = rng.choice(("bf16", "f32")), rng.random() < 0.6
                case["rotary"] = rng.choice((case["d"], case["d"], case["d"] // 2))
        case["lens"], case["rows"] = text(lens), text(rows)
        scores = batch * case["nq"] * max(rows) * max(n + r for n, r in zip(lens, rows))
        if sum(rows) and _cost(case) <= most and (op in ("append", "append4") or scores <= MOST_SCORES):
            return case


# ---- inputs -----------------------------------------------------------------------

def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(seed, stream, *shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=_generator(seed, stream))


def _parents(case, seed):
    """Each request's rows' parents within it (-1: the prefix itself)."""
    rng = np.random.default_rng(seed)
    return [[i - 1 if case["tree"] == "chain" or i == 0 else int(rng.integers(0, i)) for i in range(r)]
            for r in _ints(case["rows"])]


def _visible(case, seed):
    """Bit j of row i: row i sees row j of its request (itself and its ancestors)."""
    bits = []
    for parents in _parents(case, seed):
        of = []
        for i, p in enumerate(parents):
            of.append((1 << i) | (of[p] if p >= 0 else 0))
        bits += of
    return torch.from_numpy(np.array(bits, dtype=np.uint64).view(np.int64)).cuda()


def _keys(seed, stream, *shape):
    x = _normal(seed, stream, *shape, dtype=torch.bfloat16)
    x[..., 3::16] *= 4
    return x


def _shape(case, layers=1):
    lens = _ints(case["lens"])
    rows = _ints(case["rows"]) if "rows" in case else [0] * len(lens)
    return (layers, len(lens), case["nkv"], max(n + r for n, r in zip(lens, rows)) + ROOM, case["d"])


def _projected(case, seed):
    """The rows of a fused projection, queries, keys and values of a row side by side."""
    heads = case["nq"] + 2 * case["nkv"]
    x = _normal(seed, 1, sum(_ints(case["rows"])), heads, case["d"])
    x *= _normal(seed, 2, heads, 1).mul_(0.5).exp_()
    gains = [1 + 0.2 * _normal(seed, 3 + i, case["d"]) for i in range(2)] if case["norm"] else [None, None]
    return x.bfloat16() if case["type"] == "bf16" else x, gains


def _attention_inputs(case, seed):
    q = _normal(seed, 3, sum(_ints(case["rows"])), case["nq"], case["d"]) * 1.5
    shape = _shape(case)
    return (q if case.get("q") == "f32" else q.bfloat16(), _keys(seed, 1, *shape),
            _normal(seed, 2, *shape, dtype=torch.bfloat16))


def prepare(case, seed):
    op = case["op"]
    lens = _ints(case["lens"])
    st = {"op": op, "case": case, "lens": lens}
    st["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if op != "pack":
        rows = st["rows"] = _ints(case["rows"])
        total, r_max, starts = sum(rows), max(rows), np.cumsum([0] + rows)
        st["n_rows"] = torch.tensor(rows, device="cuda")
        # where each request's rows lie, padded to the longest request's; of each row its request and place
        pad = np.minimum(starts[:-1, None] + np.arange(r_max)[None], total - 1)
        st["pad"] = torch.from_numpy(pad).cuda()
        st["of"] = torch.tensor([b for b, r in enumerate(rows) for _ in range(r)], device="cuda")
        st["place"] = torch.tensor([i for r in rows for i in range(r)], device="cuda")
        st["at"] = st["of"] * r_max + st["place"]
    layers = case.get("layers", 1)
    shape = _shape(case, layers)
    codes = [(*shape[:-1], case["d"] // 2), (*shape[:-1], case["d"] // 16)]
    if op in ("append", "append4"):
        x, (st["q_norm"], st["k_norm"]) = _projected(case, seed)
        st["q"], st["k_new"], st["v_new"] = x.split([case["nq"], case["nkv"], case["nkv"]], dim=1)
        st["q_out"] = torch.empty(st["q"].shape, dtype=x.dtype, device="cuda")
        st["end"] = st["kv_len"] + torch.tensor(rows, dtype=torch.int32, device="cuda")
    if op == "append":
        st["k"], st["v"] = _keys(seed, 6, *shape), _normal(seed, 7, *shape, dtype=torch.bfloat16)
    elif op == "append4":
        st["packed"] = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in codes * 2]
        st["k"], st["v"] = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    elif op == "pack":
        st["k_in"], st["v_in"] = _keys(seed, 1, *shape), _normal(seed, 2, *shape, dtype=torch.bfloat16)
        st["packed"] = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in codes * 2]
        st["k"], st["v"] = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        st["q"], k, v = _attention_inputs(case, seed)
        st["scale"] = 1.0 / math.sqrt(case["d"])
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((total, case["nq"]), dtype=torch.float32, device="cuda")
        if op == "attend4":
            st["visible"] = _visible(case, seed)
            st["packed"] = [t for x in (k, v) for t in _pack(x)]
        else:
            st["k"], st["v"] = k, v
    if own:
        import paper_2609_37617_gb300 as lib
        if "packed" in st:
            st["cache4"] = lib.Cache4(*st["packed"])
        if "k" in st:
            st["cache"] = lib.Cache(st["k"], st["v"])
        if op == "pack":
            st["cache_in"] = lib.Cache(st["k_in"], st["v_in"])
    return st


# ---- one pass -----------------------------------------------------------------------

def run(st):
    op = st["op"]
    if own:
        c = st["case"]
        if op in ("append", "append4"):
            st["cache" if op == "append" else "cache4"].append(
                st["q"], st["k_new"], st["v_new"], st["kv_len"], st["rows"], q_norm=st["q_norm"],
                k_norm=st["k_norm"], eps=EPS, theta=THETA, rotary=c["rotary"], out=st["q_out"])
            if op == "append4":
                st["cache4"].read(st["cache"], st["end"], start=st["kv_len"], layer=0, max_entries=max(st["rows"]))
        elif op == "pack":
            st["cache4"].write(st["cache_in"], st["kv_len"], max_entries=max(st["lens"]))
            st["cache4"].read(st["cache"], st["kv_len"], max_entries=max(st["lens"]))
        elif op == "attend4":
            st["cache4"].tree_attention(st["q"], st["kv_len"], st["rows"], st["visible"], scale=st["scale"],
                                        max_len=max(st["lens"]), out=st["out"], lse=st["lse"])
        else:
            st["cache"].prompt_attention(st["q"], st["kv_len"], st["rows"], scale=st["scale"],
                                         max_len=max(st["lens"]), out=st["out"], lse=st["lse"])
    elif op in ("append", "append4"):
        _append_plain(st)
    elif op == "pack":
        _pack_plain(st)
    else:
        _attend_plain(st)
    if op in ("append", "append4"):
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    if op == "pack":
        return {"k": st["k"], "v": st["v"]}
    return {"out": st["out"], "lse": st["lse"]}


# ---- the plain forms ------------------------------------------------------------------

def _pack(x):
    """The codes and scale bytes of values, in 64 bits: which of two neighbours is
    nearer is decided without a rounding."""
    blocks = x.double().reshape(*x.shape[:-1], -1, 16)
    t = blocks.abs().amax(-1) / torch.full((), 7.0, dtype=torch.float64, device=x.device)
    low = torch.full_like(t, -14)
    e = torch.where(t > 0, torch.maximum((torch.frexp(t).exponent - 1).double(), low), low)
    s = torch.minimum(torch.round(t * torch.exp2(3 - e)) * torch.exp2(e - 3), torch.full_like(t, 896.0))
    c = torch.round(blocks / torch.where(s > 0, s, torch.ones_like(s))[..., None]).clamp_(-7, 7)
    c = torch.where((s > 0)[..., None], c, torch.zeros_like(c)).long().reshape(*x.shape[:-1], -1, 4, 2) + 8
    # four dims of a word's lower half, its even ones, then the odd ones
    c = c.transpose(-1, -2).reshape(*x.shape[:-1], -1, 2)
    codes = (c[..., 0] | (c[..., 1] << 4)).to(torch.uint8)
    return codes, (s.half().view(torch.int16) >> 7).to(torch.uint8)


def _unpack(codes, scales):
    """The values that codes and scale bytes stand for, in 32 bits."""
    c = torch.stack((codes & 15, codes >> 4), -1).int().reshape(*codes.shape[:-1], -1, 2, 4) - 8
    c = c.transpose(-1, -2).reshape(*codes.shape[:-1], -1, 16)
    s = (scales.to(torch.int16) << 7).view(torch.float16).float().clamp(max=896.0)
    return (c.float() * s[..., None]).flatten(-2)


def _pack_plain(st):
    for x, (codes, scales), to in zip((st["k_in"], st["v_in"]), (st["packed"][:2], st["packed"][2:]),
                                      (st["k"], st["v"])):
        there = (torch.arange(x.shape[3], device="cuda") < st["kv_len"][:, None])[None, :, None, :, None]
        new_codes, new_scales = _pack(x)
        codes.copy_(torch.where(there, new_codes, codes))
        scales.copy_(torch.where(there, new_scales, scales))
        to.copy_(torch.where(there, _unpack(codes, scales).bfloat16(), to))


def _finish_plain(x, gain, position, rotary):
    """Rows of heads normed and rotated.  In 64 bits: angles of far positions, and
    values next to the border of two codes."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.double()
    half = rotary // 2
    freq = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = position.double()[:, None, None] * freq
    a, b, rest = x.split([half, half, x.shape[-1] - rotary], dim=-1)
    cos, sin = angle.cos(), angle.sin()
    return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1)


def _append_plain(st):
    c, at = st["case"], st["kv_len"].long()[st["of"]] + st["place"]
    st["q_out"].copy_(_finish_plain(st["q"], st["q_norm"], at, c["rotary"]))
    k = _finish_plain(st["k_new"], st["k_norm"], at, c["rotary"])
    for i, (x, to) in enumerate(((k, st["k"]), (st["v_new"], st["v"]))):
        if st["op"] == "append4":
            for held, new in zip(st["packed"][2 * i:2 * i + 2], _pack(x)):
                held[0, st["of"], :, at] = new
            x = _unpack(*(t[0, st["of"], :, at] for t in st["packed"][2 * i:2 * i + 2]))
        to[0, st["of"], :, at] = x.bfloat16()


def _attend_plain(st):
    c, q = st["case"], st["q"]
    batch, nkv, d, group = len(st["lens"]), c["nkv"], c["d"], c["nq"] // c["nkv"]
    longest = max(n + r for n, r in zip(st["lens"], st["rows"]))
    if st["op"] == "attend4":
        k, v = (_unpack(*(t[0, :, :, :longest] for t in st["packed"][i:i + 2])) for i in (0, 2))
    else:
        k, v = (st[x][0, :, :, :longest].float() for x in "kv")
    qp = q.float()[st["pad"]].view(batch, -1, nkv, group, d).permute(0, 2, 1, 3, 4)
    r_max = qp.shape[2]
    s = (qp.reshape(batch, nkv, r_max * group, d) @ k.transpose(2, 3)).mul_(st["scale"])
    rel = torch.arange(longest, device="cuda")[None] - st["kv_len"].long()[:, None]
    if st["op"] == "attend4":
        bit = (st["visible"][st["pad"]][:, :, None] >> rel.clamp(0, 63)[:, None]) & 1
        tail = (rel >= 0) & (rel < st["n_rows"][:, None])
        seen = (rel < 0)[:, None] | (tail[:, None] & (bit == 1))
    else:
        seen = rel[:, None] <= torch.arange(r_max, device="cuda")[None, :, None]
    s = s.view(batch, nkv, r_max, group, longest).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    o = e.view(batch, nkv, r_max * group, longest) @ v
    o = o.view(batch, nkv, r_max, group, d) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(batch * r_max, c["nq"], d)[st["at"]]
    st["out"] = o.to(q.dtype)
    st["lse"] = lse.permute(0, 2, 1, 3).reshape(batch * r_max, c["nq"])[st["at"]].contiguous()


# ---- what a call cannot do without -------------------------------------------------

def work(case):
    op, lens, d, nkv = case["op"], _ints(case["lens"]), case["d"], case["nkv"]
    packed = d // 2 + d // 16  # bytes of a key or value of one head
    if op == "pack":
        entries = 2 * case["layers"] * nkv * sum(lens)
        return {"bytes": entries * 2 * (2 * d + packed), "flops": 4 * entries * d}
    rows, nq = _ints(case["rows"]), case["nq"]
    total = sum(rows)
    if op in ("append", "append4"):
        size = 2 if case["type"] == "bf16" else 4
        entry = 2 * d if op == "append" else 2 * packed + 2 * d
        return {"bytes": total * ((2 * nq + 2 * nkv) * d * size + 2 * nkv * entry),
                "flops": total * (nq + nkv) * d * 7}
    seen = sum(r * n + r * (r + 1) // 2 for n, r in zip(lens, rows))
    entries = 2 * nkv * sum(n + r for n, r in zip(lens, rows) if r)
    size = 4 if case.get("q") == "f32" else 2
    nbytes = entries * (packed if op == "attend4" else 2 * d) + total * nq * (2 * d * size + 4)
    return {"bytes": nbytes + (8 * total if op == "attend4" else 0), "flops": 4 * nq * d * seen}


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 150


# ---- the same in 64 bits ------------------------------------------------------------

def _scale_table():
    """The value of each scale byte that is written, by the byte."""
    byte = torch.arange(0xC7, device="cuda")
    e, f = (byte >> 3).double(), (byte & 7).double()
    return torch.where(e > 0, torch.exp2(e - 15) * (1 + f / 8), torch.exp2(torch.full_like(f, -14)) * f / 8)


def _exact_values(x):
    """What values become in 4 bits, from the table of scales: its neighbours of a
    seventh of the largest magnitude are compared, then each value's neighbours."""
    table = _scale_table()
    b = x.double().unflatten(-1, (-1, 16))
    a = b.abs().max(-1).values
    above = torch.searchsorted(7 * table, a.contiguous()).clamp(1, len(table) - 1)
    over, under = 7 * table[above] - a, a - 7 * table[above - 1]
    take = torch.where((over < under) | ((over == under) & (above % 2 == 0)), above, above - 1)
    s = table[take][..., None]
    low = torch.floor(torch.where(s > 0, b / s, torch.zeros_like(b)))
    over, under = (low + 1) * s - b, b - low * s
    up = (over < under) | ((over == under) & (low.remainder(2) == 1))
    return ((low + up).clamp(-7, 7) * s).flatten(-2)


def exact(case, seed):
    op = case["op"]
    if op in ("attend4", "prompt"):
        return _exact_attention(case, seed)
    if op == "pack":
        shape = _shape(case, case["layers"])
        found = {}
        for name, x in (("k", _keys(seed, 1, *shape)), ("v", _normal(seed, 2, *shape, dtype=torch.bfloat16))):
            found[name] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
            for layer in range(shape[0]):
                for b, n in enumerate(_ints(case["lens"])):
                    found[name][layer, b, :, :n] = _exact_values(x[layer, b, :, :n]).bfloat16()
        return found
    x, gains = _projected(case, seed)
    lens, rows, shape, rotary = _ints(case["lens"]), _ints(case["rows"]), _shape(case), case["rotary"]
    if op == "append":
        k, v = _keys(seed, 6, *shape).double(), _normal(seed, 7, *shape, dtype=torch.bfloat16).double()
    else:
        k, v = (torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(2))
    nq, nkv, d, r0, queries = case["nq"], case["nkv"], case["d"], 0, []
    turn = torch.exp(-math.log(THETA) * 2 / rotary * torch.arange(rotary // 2, dtype=torch.float64, device="cuda"))
    for b, (n, r) in enumerate(zip(lens, rows)):
        y = x[r0:r0 + r].double()
        for part, gain in ((slice(0, nq), gains[0]), (slice(nq, nq + nkv), gains[1])):
            z = y[:, part]
            if gain is not None:
                z *= gain.double() * (z.pow(2).sum(-1, keepdim=True) / d + EPS).rsqrt()
            # pairs of dims as complex numbers, turned by their angle
            angle = torch.arange(n, n + r, dtype=torch.float64, device="cuda")[:, None] * turn
            pair = torch.complex(z[..., :rotary // 2].contiguous(), z[..., rotary // 2:rotary].contiguous())
            pair = pair * torch.polar(torch.ones_like(angle), angle)[:, None]
            z[..., :rotary] = torch.cat((pair.real, pair.imag), -1)
        queries.append(y[:, :nq])
        for to, new in ((k, y[:, nq:nq + nkv]), (v, y[:, nq + nkv:])):
            to[0, b, :, n:n + r] = (new if op == "append" else _exact_values(new)).transpose(0, 1)
        r0 += r
    return {"q": torch.cat(queries), "k": k, "v": v}


def _exact_attention(case, seed):
    q_all, k_all, v_all = _attention_inputs(case, seed)
    group, d = case["nq"] // case["nkv"], case["d"]
    outs, lses, r0 = [], [], 0
    parents = _parents(case, seed) if case["op"] == "attend4" else None
    for b, (n, r) in enumerate(zip(_ints(case["lens"]), _ints(case["rows"]))):
        if not r:
            continue
        if parents is not None:
            seen = torch.zeros(r, n + r, dtype=torch.bool)
            seen[:, :n] = True
            for i in range(r):
                j = i
                while j >= 0:
                    seen[i, n + j] = True
                    j = parents[b][j]
            seen = seen.cuda()
        else:
            seen = torch.ones(r, n + r, dtype=torch.bool, device="cuda").tril(n)
        q = q_all[r0:r0 + r].double().view(r, case["nkv"], group, d).permute(1, 2, 0, 3)
        out, lse = [], []
        for g in range(case["nkv"]):
            k, v = k_all[0, b, g, :n + r], v_all[0, b, g, :n + r]
            if parents is not None:
                k, v = _exact_values(k), _exact_values(v)
            s = torch.einsum("hid,td->hit", q[g], k.double()) / math.sqrt(d)
            s.masked_fill_(~seen, -math.inf)
            lse.append(torch.logsumexp(s, -1))
            out.append(torch.einsum("hit,td->ihd", s.sub_(lse[-1][..., None]).exp_(), v.double()))
        outs.append(torch.cat(out, 1))
        lses.append(torch.cat(lse, 0).t())
        r0 += r
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
