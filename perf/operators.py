"""The operators on caller's caches and logits whose speed is followed: attention
of a tree of drafted tokens over a cache, the attention weight that each cache
entry gathers, eviction by that weight, probabilities at a temperature, and the
acceptance of drafted tokens from given random numbers.

Each has its plain form in torch beside the call of this library.  Queries, keys
and values are N(0, 1) (queries N(0, 1.5): a head attends to some entries more
than to others), gathered weights are heavy-tailed, probabilities have a few
likely tokens over a long tail, as a language model's have.
"""
import math

import numpy as np
import torch

own = False
ROOM = 64  # positions of a cache past the prefix and the call's own rows

RAGGED_LENS = "6130 6416 2466 5349 5631 376 2509 7495 1702 5900 3266 3948 5116 817 1839 2625"
RAGGED_ROWS = "5 14 17 12 3 14 6 17 14 10 12 4 6 6 16 0"


def listed():
    return [
        # the smallest call: the tiny decoder's heads, a block of five as a chain
        {"name": "tree-tiny-chain5", "op": "tree", "nq": 4, "nkv": 2, "d": 64, "lens": "200", "rows": "5",
         "tree": "chain", "q": "bf16"},
        # one token of the target over a minute of audio: the single-token form
        {"name": "tree-7b-decode", "op": "tree", "nq": 28, "nkv": 4, "d": 128, "lens": "1564", "rows": "1",
         "tree": "chain", "q": "bf16"},
        # ten minutes of audio retained and the widest tree
        {"name": "tree-7b-long-64", "op": "tree", "nq": 28, "nkv": 4, "d": 128, "lens": "15128", "rows": "64",
         "tree": "random", "q": "bf16"},
        # a server's round: ragged prefixes and trees, one request without rows, fp32 queries
        {"name": "tree-7b-ragged16", "op": "tree", "nq": 28, "nkv": 4, "d": 128, "lens": RAGGED_LENS,
         "rows": RAGGED_ROWS, "tree": "random", "q": "f32"},
        # 30 s of audio, a block of nine of the drafter-sized decoder
        {"name": "weights-1.5b-9", "op": "weights", "nq": 12, "nkv": 2, "d": 128, "lens": "814", "rows": "9",
         "tree": "chain", "q": "bf16"},
        {"name": "weights-7b-ragged16", "op": "weights", "nq": 28, "nkv": 4, "d": 128, "lens": RAGGED_LENS,
         "rows": RAGGED_ROWS, "tree": "random", "q": "f32"},
        # the tiny decoder's cache cut to three quarters
        {"name": "evict-tiny", "op": "evict", "layers": 2, "nkv": 2, "d": 64, "lens": "200", "keep": "150",
         "recent": 50},
        # ten minutes of retained audio cut to three quarters, every layer of the target
        {"name": "evict-7b-long", "op": "evict", "layers": 28, "nkv": 4, "d": 128, "lens": "15128",
         "keep": "11346", "recent": 128},
        # one block of the target: nine rows of logits
        {"name": "probs-7b-9", "op": "probs", "rows": 9, "vocab": 152064, "temperature": 0.7},
        # a server's round of 145 rows
        {"name": "probs-7b-145", "op": "probs", "rows": 145, "vocab": 152064, "temperature": 1.0},
        # one block of eight candidates from a drafter that gives no probabilities
        {"name": "accept-7b-k8", "op": "accept", "vocab": 152064, "ks": "8", "draft": False},
        # a server's round with the drafter's probabilities, every block width
        {"name": "accept-7b-ragged16", "op": "accept", "vocab": 152064,
         "ks": "4 13 16 11 2 13 5 16 13 9 11 3 5 5 15 0", "draft": True},
    ]


def _ints(text):
    return [int(t) for t in text.split()]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("tree", "tree", "weights", "evict", "probs", "accept"))
        case = {"op": op}
        if op in ("tree", "weights"):
            case["nq"], case["nkv"], case["d"] = rng.choice(((4, 2, 64), (12, 2, 128), (28, 4, 128), (8, 8, 64), (16, 1, 128)))
            batch = 1 if rng.random() < 0.5 else _log_uniform(rng, 2, 64)
            case["lens"] = " ".join(str(_log_uniform(rng, 1, 15128)) for _ in range(batch))
            case["rows"] = " ".join(str(rng.randint(0 if batch > 1 else 1, rng.choice((1, 17, 64)))) for _ in range(batch))
            if not sum(_ints(case["rows"])):
                continue
            case["tree"] = rng.choice(("chain", "random"))
            case["q"] = rng.choice(("bf16", "f32"))
        elif op == "evict":
            case["layers"] = rng.choice((1, 2, 28))
            case["nkv"], case["d"] = rng.choice(((2, 64), (2, 128), (4, 128), (8, 64)))
            batch = 1 if rng.random() < 0.5 else _log_uniform(rng, 2, 16)
            lens = [_log_uniform(rng, 16, 15128) for _ in range(batch)]
            case["lens"] = " ".join(map(str, lens))
            case["recent"] = rng.randint(0, 16)
            case["keep"] = " ".join(str(max(case["recent"], round(n * rng.uniform(0.1, 1.1)))) for n in lens)
        elif op == "probs":
            case["rows"] = _log_uniform(rng, 1, 300)
            case["vocab"] = rng.choice((4096, 151936, 152064, _log_uniform(rng, 100, 200000)))
            case["temperature"] = round(rng.uniform(0.3, 1.5), 2)
        else:
            batch = 1 if rng.random() < 0.4 else _log_uniform(rng, 2, 64)
            case["vocab"] = rng.choice((4096, 151936, 152064, _log_uniform(rng, 100, 200000)))
            case["ks"] = " ".join(str(rng.randint(0, 16)) for _ in range(batch))
            case["draft"] = rng.random() < 0.6
        if _cost(case) <= most:
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


def _attention_inputs(case, seed):
    lens, rows = _ints(case["lens"]), _ints(case["rows"])
    cap = max(n + r for n, r in zip(lens, rows)) + ROOM
    shape = (1, len(lens), case["nkv"], cap, case["d"])
    q = _normal(seed, 3, sum(rows), case["nq"], case["d"]) * 1.5
    return {"lens": lens, "rows": rows, "cap": cap, "k": _normal(seed, 1, *shape, dtype=torch.bfloat16),
            "v": _normal(seed, 2, *shape, dtype=torch.bfloat16),
            "q": q.bfloat16() if case["q"] == "bf16" else q, "visible": _visible(case, seed)}


def _logits(seed, stream, rows, vocab):
    x = _normal(seed, stream, rows, vocab) * 2.5
    at = torch.randint(0, vocab, (rows, 3), generator=_generator(seed, stream + 1), device="cuda")
    return x.scatter_add_(1, at, torch.tensor([[16.0, 15.0, 14.0]], device="cuda").expand(rows, 3))


def _accept_inputs(case, seed):
    ks = _ints(case["ks"])
    total, rows = sum(ks), sum(ks) + len(ks)
    logits = _logits(seed, 1, rows, case["vocab"])
    probs = logits.softmax(1)
    row_of = torch.tensor([r for b, k in enumerate(ks) for r in range(sum(ks[:b]) + b, sum(ks[:b]) + b + k)],
                          dtype=torch.int64, device="cuda")
    draft, cand = None, torch.zeros(0, dtype=torch.int32, device="cuda")
    if total:
        draft = (logits[row_of] + 0.7 * _normal(seed, 4, total, case["vocab"])).softmax(1)
        cand = torch.multinomial(draft, 1, generator=_generator(seed, 5))[:, 0].int()
    u = torch.rand(rows, generator=_generator(seed, 6), device="cuda")
    return {"ks": ks, "probs": probs, "cand": cand, "u": u, "draft": draft if case["draft"] else None}


def prepare(case, seed):
    op = case["op"]
    st = {"op": op, "case": case}
    if op in ("tree", "weights"):
        st.update(_attention_inputs(case, seed))
        st["scale"] = 1.0 / math.sqrt(case["d"])
        st["kv_len"] = torch.tensor(st["lens"], dtype=torch.int32, device="cuda")
        st["n_rows"] = torch.tensor(st["rows"], device="cuda")
        total = sum(st["rows"])
        # where each request's rows lie, padded to the longest request's
        r_max, starts = max(st["rows"]), np.cumsum([0] + st["rows"])
        pad = np.minimum(starts[:-1, None] + np.arange(r_max)[None], total - 1)
        st["pad"] = torch.from_numpy(pad).cuda()
        st["at"] = torch.tensor([b * r_max + i for b, r in enumerate(st["rows"]) for i in range(r)], device="cuda")
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((total, case["nq"]), dtype=torch.float32, device="cuda")
        if op == "weights":
            st["lse"] = _tree_plain(st)[1]
            st["w"] = _normal(seed, 7, 1, len(st["lens"]), case["nkv"], st["cap"]).square()
    elif op == "evict":
        lens, keep = _ints(case["lens"]), _ints(case["keep"])
        shape = (case["layers"], len(lens), case["nkv"], max(lens) + ROOM, case["d"])
        st["k"], st["v"] = (_normal(seed, i, *shape, dtype=torch.bfloat16) for i in (1, 2))
        st["w"] = _normal(seed, 3, *shape[:-1]).square().square()
        st["len0"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        st["kv_len"] = st["len0"].clone()
        st["keep"], st["keep_d"] = keep, torch.tensor(keep, dtype=torch.int32, device="cuda")
    elif op == "probs":
        st["x"] = _logits(seed, 1, case["rows"], case["vocab"])
        st["out"] = torch.empty_like(st["x"])
    else:
        st.update(_accept_inputs(case, seed))
        ks = st["ks"]
        k_max = max(max(ks), 1)
        row0 = torch.tensor([sum(ks[:b]) + b for b in range(len(ks))], device="cuda")
        cand0 = torch.tensor([sum(ks[:b]) for b in range(len(ks))], device="cuda")
        st["row0"], st["cand0"], st["k_d"] = row0, cand0, torch.tensor(ks, device="cuda")
        i = torch.arange(k_max, device="cuda")[None]
        st["live"] = i < st["k_d"][:, None]
        st["cand_at"] = (cand0[:, None] + i).clamp(max=max(sum(ks) - 1, 0))
        st["row_at"] = torch.where(st["live"], row0[:, None] + i, row0[:, None])
        st["n"], st["token"] = (torch.empty(len(ks), dtype=torch.int32, device="cuda") for _ in range(2))
    if own:
        import paper_2609_37617_gb300 as lib
        st["lib"] = lib
        if op in ("tree", "weights", "evict"):
            st["cache"] = lib.Cache(st["k"], st["v"])
    return st


# ---- one pass -----------------------------------------------------------------------

def run(st):
    op = st["op"]
    if op == "evict":
        st["kv_len"].copy_(st["len0"])
    if own:
        lib = st["lib"]
        if op == "tree":
            st["cache"].tree_attention(st["q"], st["kv_len"], st["rows"], st["visible"], scale=st["scale"],
                                       max_len=max(st["lens"]), out=st["out"], lse=st["lse"])
        elif op == "weights":
            st["cache"].attention_weights(st["q"], st["lse"], st["w"], st["kv_len"], st["rows"], st["visible"],
                                          scale=st["scale"], max_len=max(st["lens"]))
        elif op == "evict":
            st["cache"].evict(st["w"], st["kv_len"], st["keep"], recent=st["case"]["recent"])
        elif op == "probs":
            lib.token_probs(st["x"], st["case"]["temperature"], out=st["out"])
        else:
            lib.accept_sampled(st["probs"], st["cand"], st["ks"], st["u"], st["n"], st["token"],
                               draft_probs=st["draft"])
    elif op == "tree":
        st["out"], st["lse"] = _tree_plain(st)
    elif op == "weights":
        _weights_plain(st)
    elif op == "evict":
        _evict_plain(st)
    elif op == "probs":
        x = st["x"] / st["case"]["temperature"]
        e = (x - x.amax(1, keepdim=True)).exp()
        st["out"] = e / e.sum(1, keepdim=True)
    else:
        _accept_plain(st)
    if op == "tree":
        return {"out": st["out"], "lse": st["lse"]}
    if op == "weights":
        return {"w": st["w"]}
    if op == "evict":
        return {"k": st["k"], "v": st["v"], "w": st["w"], "len": st["kv_len"]}
    if op == "probs":
        return {"probs": st["out"]}
    return {"n_accepted": st["n"], "token": st["token"]}


# ---- the plain forms ------------------------------------------------------------------

def _scores(st):
    """Scaled scores [batch][n_kv][rows][group][positions], -inf where a row does not see."""
    c, q = st["case"], st["q"]
    batch, nkv, d, group = len(st["lens"]), c["nkv"], c["d"], c["nq"] // c["nkv"]
    longest = max(n + r for n, r in zip(st["lens"], st["rows"]))
    qp = q.float()[st["pad"]].view(batch, -1, nkv, group, d).permute(0, 2, 1, 3, 4)
    r_max = qp.shape[2]
    keys = st["k"][0, :, :, :longest].float()
    s = (qp.reshape(batch, nkv, r_max * group, d) @ keys.transpose(2, 3)) * st["scale"]
    rel = torch.arange(longest, device="cuda")[None] - st["kv_len"].long()[:, None]
    bit = (st["visible"][st["pad"]][:, :, None] >> rel.clamp(0, 63)[:, None]) & 1
    tail = (rel >= 0) & (rel < st["n_rows"][:, None])
    seen = (rel < 0)[:, None] | (tail[:, None] & (bit == 1))
    return s.view(batch, nkv, r_max, group, longest).masked_fill(~seen[:, None, :, None], -math.inf), longest


def _tree_plain(st):
    c = st["case"]
    s, longest = _scores(st)
    batch, nkv, r_max, group, _ = s.shape
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = (s - m).exp()
    total = e.sum(-1, keepdim=True)
    o = e.view(batch, nkv, r_max * group, longest) @ st["v"][0, :, :, :longest].float()
    o = o.view(batch, nkv, r_max, group, c["d"]) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(batch * r_max, c["nq"], c["d"])[st["at"]]
    return o.to(st["q"].dtype), lse.permute(0, 2, 1, 3).reshape(batch * r_max, c["nq"])[st["at"]].contiguous()


def _weights_plain(st):
    s, longest = _scores(st)
    batch, nkv, r_max, group, _ = s.shape
    lse = st["lse"][st["pad"]].view(batch, r_max, nkv, group).permute(0, 2, 1, 3)[..., None]
    live = (torch.arange(r_max, device="cuda")[None] < st["n_rows"][:, None])[:, None, :, None, None]
    p = torch.where(live & (s > -math.inf), (s - lse).exp(), torch.zeros_like(s)).sum((2, 3))
    rel = (torch.arange(longest, device="cuda")[None] - st["kv_len"].long()[:, None])[:, None]
    rows = st["n_rows"][:, None, None]
    w = st["w"][0, :, :, :longest]
    w.copy_(torch.where(rows == 0, w, torch.where(rel < 0, w + p, torch.where(rel < rows, p, w))))


def _evict_plain(st):
    length = st["kv_len"].long()[None, :, None, None]
    keep = torch.minimum(st["keep_d"].long()[None, :, None, None], length)
    cap = st["w"].shape[-1]
    pos = torch.arange(cap, device="cuda")[None, None, None]
    key = torch.where(pos >= length, -math.inf, torch.where(pos >= length - st["case"]["recent"], math.inf, st["w"]))
    most = max(st["keep"]) if max(st["keep"]) < cap else cap
    chosen = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :most]
    j = pos[..., :most]
    # the places that a request keeps, in order; past them every entry stays where it is
    chosen = torch.where(j < keep, chosen, cap).sort(-1).values
    chosen = torch.where(j < keep, chosen, j)
    st["w"][..., :most] = st["w"].gather(-1, chosen)
    at = chosen[..., None].expand(*chosen.shape, st["k"].shape[-1])
    st["k"][..., :most, :] = st["k"].gather(-2, at)
    st["v"][..., :most, :] = st["v"].gather(-2, at)
    st["kv_len"].copy_(keep.view(-1))


def _accept_plain(st):
    probs, live = st["probs"], st["live"]
    if st["cand"].numel():
        cand = st["cand"].long()[st["cand_at"]]
        p = probs[st["row_at"], cand].double()
        q = st["draft"][st["cand_at"], cand].double() if st["draft"] is not None else torch.ones_like(p)
        ok = live & (st["u"][st["row_at"]].double() * q < p)
        n = ok.long().cumprod(1).sum(1)
    else:
        n = torch.zeros_like(st["k_d"])
    rest = probs[st["row0"] + n].double()
    if st["cand"].numel():
        at = (st["cand0"] + n).clamp(max=st["cand"].numel() - 1)
        if st["draft"] is not None:
            taken = st["draft"][at].double()
        else:
            taken = torch.zeros_like(rest).scatter_(1, st["cand"].long()[at][:, None], 1.0)
        rest = torch.where((n < st["k_d"])[:, None], (rest - taken).clamp(min=0.0), rest)
    cdf = rest.cumsum(1)
    border = st["u"][st["row0"] + st["k_d"]].double() * cdf[:, -1]
    token = (cdf <= border[:, None]).sum(1)
    st["n"], st["token"] = n.int(), token.int()


# ---- what a call cannot do without -------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("tree", "weights"):
        lens, rows = _ints(case["lens"]), _ints(case["rows"])
        q = sum(rows) * case["nq"] * case["d"]
        size = 2 if case["q"] == "bf16" else 4
        entries = case["nkv"] * sum(n + r for n, r in zip(lens, rows) if r)
        seen = sum(r * n + r * (r + 1) // 2 for n, r in zip(lens, rows))
        if op == "tree":
            nbytes = entries * case["d"] * 4 + 2 * q * size + sum(rows) * (4 * case["nq"] + 8)
            return {"bytes": nbytes, "flops": 4 * case["nq"] * case["d"] * seen}
        nbytes = entries * (case["d"] * 2 + 8) + q * size + sum(rows) * (4 * case["nq"] + 8)
        return {"bytes": nbytes, "flops": 2 * case["nq"] * case["d"] * seen}
    if op == "evict":
        heads = case["layers"] * case["nkv"]
        pairs = list(zip(_ints(case["lens"]), _ints(case["keep"])))
        cut = sum(k for n, k in pairs if k < n)
        nbytes = heads * (cut * (case["d"] * 8 + 4) + 4 * sum(n for n, k in pairs if k < n)) + 8 * len(pairs)
        return {"bytes": nbytes, "flops": heads * sum(n for n, k in pairs if k < n)}
    if op == "probs":
        n = case["rows"] * case["vocab"]
        return {"bytes": 8 * n, "flops": 5 * n}
    ks = _ints(case["ks"])
    n = case["vocab"] * sum(2 if case["draft"] and k else 1 for k in ks)
    return {"bytes": 4 * n + 16 * sum(ks) + 12 * len(ks), "flops": 3 * n}


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 150


# ---- the same in 64 bits ------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op in ("tree", "weights"):
        return _exact_attention(case, seed)
    if op == "probs":
        x = _logits(seed, 1, case["rows"], case["vocab"]).double() / case["temperature"]
        return {"probs": torch.exp(x - torch.logsumexp(x, 1, keepdim=True))}
    if op == "evict":
        # copies and comparisons: nothing to compute but which entries stay
        lens, keep = _ints(case["lens"]), _ints(case["keep"])
        shape = (case["layers"], len(lens), case["nkv"], max(lens) + ROOM, case["d"])
        k, v = (_normal(seed, i, *shape, dtype=torch.bfloat16) for i in (1, 2))
        w = _normal(seed, 3, *shape[:-1]).square().square()
        for b, (n, most) in enumerate(zip(lens, keep)):
            if most >= n:
                continue
            old = n - min(case["recent"], most)
            order = torch.argsort(-w[:, b, :, :old].double(), dim=-1, stable=True)[..., :most - (n - old)]
            stay = torch.zeros(w[:, b, :, :n].shape, dtype=torch.bool, device="cuda")
            stay.scatter_(-1, order, True)
            stay[..., old:] = True
            for t in (k, v, w):
                t[:, b, :, :most] = t[:, b, :, :n][stay].view(*t[:, b, :, :most].shape)
        return {"k": k, "v": v, "w": w, "len": None}
    x, n_out, tokens, r, c = _accept_inputs(case, seed), [], [], 0, 0
    u = x["u"].double().cpu().numpy()
    for k in x["ks"]:
        n = 0
        while n < k:
            t = int(x["cand"][c + n])
            q = float(x["draft"][c + n, t]) if x["draft"] is not None else 1.0
            if not u[r + n] * q < float(x["probs"][r + n, t]):
                break
            n += 1
        left = x["probs"][r + n].double().cpu().numpy()
        if n < k:
            if x["draft"] is not None:
                left = left - x["draft"][c + n].double().cpu().numpy()
            else:
                left[int(x["cand"][c + n])] -= 1.0
            left = np.maximum(left, 0.0)
        cdf = np.cumsum(left)
        n_out.append(n)
        tokens.append(int(np.searchsorted(cdf, u[r + k] * cdf[-1], side="right")))
        r, c = r + k + 1, c + k
    return {"n_accepted": np.array(n_out, dtype=np.int32), "token": np.array(tokens, dtype=np.int32)}


def _exact_attention(case, seed):
    x = _attention_inputs(case, seed)
    group, d = case["nq"] // case["nkv"], case["d"]
    outs, lses, r0 = [], [], 0
    w = _normal(seed, 7, 1, len(x["lens"]), case["nkv"], x["cap"]).square().double() if case["op"] == "weights" else None
    for b, (n, parents) in enumerate(zip(x["lens"], _parents(case, seed))):
        r = len(parents)
        if not r:
            continue
        seen = torch.zeros(r, n + r, dtype=torch.bool)
        seen[:, :n] = True
        for i in range(r):
            j = i
            while j >= 0:
                seen[i, n + j] = True
                j = parents[j]
        q = x["q"][r0:r0 + r].double().view(r, case["nkv"], group, d).permute(1, 2, 0, 3)
        s = torch.einsum("ghid,gtd->ghit", q, x["k"][0, b, :, :n + r].double()) / math.sqrt(d)
        s = s.masked_fill(~seen.cuda(), -math.inf)
        lse = torch.logsumexp(s, -1)
        if w is not None:
            # the call reads 32-bit sums: the weights follow from those it is given
            p = torch.exp(s - lse.float().double()[..., None]).sum((1, 2))
            w[0, b, :, :n] += p[:, :n]
            w[0, b, :, n:n + r] = p[:, n:]
        else:
            o = torch.einsum("ghit,gtd->ighd", s.softmax(-1), x["v"][0, b, :, :n + r].double())
            outs.append(o.reshape(r, case["nq"], d))
            lses.append(lse.permute(2, 0, 1).reshape(r, case["nq"]))
        r0 += r
    return {"w": w} if w is not None else {"out": torch.cat(outs), "lse": torch.cat(lses)}
