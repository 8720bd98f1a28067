"""The operators on caches and logits against their 64-bit forms: sizes and
masks where they can go wrong, what they must leave alone, streams, captured
graphs and a run of them together."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (28, 4, 128), (8, 8, 64), (16, 1, 128), (12, 2, 128)]


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_37617_gb300 as p
    return p


class Inputs:
    """A cache whose places past each request's entries hold NaN, and rows over
    it (q spread by `spread`)."""

    def __init__(self, heads, lens, rows, masks, q_type=torch.bfloat16, seed=0, room=37, layers=1, spread=1.5,
                 pad=0):
        nq, nkv, d = heads
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.lens, self.rows, self.masks = heads, lens, rows, masks
        cap = max(n + r for n, r in zip(lens, rows)) + room
        shape = (layers, len(lens), nkv, cap, d)
        self.k, self.v = (torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
        for b, (n, r) in enumerate(zip(lens, rows)):
            self.k[:, b, :, n + r:] = math.nan
            self.v[:, b, :, n + r:] = math.nan
        total = sum(rows)
        # rows of q may lie apart, as in a fused projection's output
        wide = torch.randn((total, nq + pad, d), generator=g, device="cuda") * spread
        self.q = wide.to(q_type)[:, :nq]
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.visible = ref.mask_tensor(masks) if total else None
        self.scale = d ** -0.5
        self.starts = np.cumsum([0] + list(rows))

    def request(self, b, layer=0):
        n, r = self.lens[b], self.rows[b]
        q = self.q[self.starts[b]:self.starts[b + 1]].double()
        return (q, self.k[layer, b, :, :n + r].double(), self.v[layer, b, :, :n + r].double(),
                ref.seen_matrix(n, self.masks[b]))


def check_attention(x, out, lse, layer=0):
    half_step = torch.finfo(x.q.dtype).eps / 2
    for b in range(len(x.lens)):
        if not x.rows[b]:
            continue
        sl = slice(x.starts[b], x.starts[b + 1])
        want, tol, want_lse, tol_lse = ref.attention(*x.request(b, layer), x.scale)
        got = out[sl].double()
        assert torch.isfinite(got).all()
        over = (got - want).abs() - (want.abs() * half_step * (1 + 2.0 ** -6) + tol)
        assert over.max() <= 0, (b, float(over.max()), float((got - want).abs().max()))
        empty = want_lse == -math.inf
        got_lse = lse[sl].double()
        assert (got_lse[empty] == -math.inf).all() and (got[empty] == 0).all()
        assert ((got_lse - want_lse)[~empty].abs() <= tol_lse[~empty]).all()


def run_attention(lib, x, layer=0, **kw):
    cache = lib.Cache(x.k, x.v)
    lse = torch.full((sum(x.rows), x.heads[0]), 7.0, device="cuda")
    out = cache.tree_attention(x.q, x.kv_len, x.rows, x.visible, layer=layer, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("length", [0, 1, 63, 127, 128, 129, 1000])
@pytest.mark.parametrize("rows", [1, 5, 64])
def test_attention_sizes(lib, heads, length, rows, q_type):
    masks = ref.tree_masks([rows], np.random.default_rng(length + rows))
    x = Inputs(heads, [length], [rows], masks, q_type, seed=length)
    check_attention(x, *run_attention(lib, x))


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128)])
def test_attention_ragged(lib, heads, q_type):
    lens = [0, 1, 700, 2055, 128, 64, 3333, 17]
    rows = [3, 0, 17, 1, 0, 64, 9, 33]
    masks = ref.tree_masks(rows, np.random.default_rng(5))
    x = Inputs(heads, lens, rows, masks, q_type, layers=2, pad=3)
    check_attention(x, *run_attention(lib, x, layer=1), layer=1)
    # the bound of the lengths sizes the launch and nothing else
    check_attention(x, *run_attention(lib, x, layer=1, max_len=3333), layer=1)
    check_attention(x, *run_attention(lib, x, layer=1, max_len=1), layer=1)  # (too low a bound)


@pytest.mark.parametrize("requests", [1, 3, 4, 12])
def test_attention_whole_items_and_clusters(lib, requests):
    """Lengths on both sides of what one CTA, a cluster of them and even shares do."""
    rng = np.random.default_rng(requests)
    for longest in (255, 257, 2000, 5000, 7000):
        lens = [int(t) for t in rng.integers(0, longest, requests)]
        lens[0] = longest
        rows = [int(t) for t in rng.integers(0, 6, requests)]
        rows[0] = 2
        for heads in ((28, 4, 128), (4, 2, 64)):
            for q_type in (torch.bfloat16, torch.float32):
                x = Inputs(heads, lens, rows, ref.tree_masks(rows, rng), q_type, seed=longest)
                check_attention(x, *run_attention(lib, x, max_len=longest))


@pytest.mark.parametrize("length", [6000, 15128])
def test_attention_long(lib, length):
    for heads, rows, q_type in (((28, 4, 128), 1, torch.bfloat16), ((28, 4, 128), 17, torch.float32),
                                ((4, 2, 64), 64, torch.bfloat16)):
        x = Inputs(heads, [length], [rows], ref.chain_masks([rows]), q_type, seed=length)
        x.visible = None  # a chain
        check_attention(x, *run_attention(lib, x))


def test_attention_most_requests(lib):
    rng = np.random.default_rng(2)
    lens = [int(t) for t in rng.integers(0, 700, 64)]
    rows = [int(t) for t in rng.integers(0, 18, 64)]
    x = Inputs((12, 2, 128), lens, rows, ref.tree_masks(rows, rng), torch.float32)
    check_attention(x, *run_attention(lib, x))


def test_attention_far_offset(lib):
    """Entries whose offset in the cache passes 2^31 elements."""
    layers, cap = 66, 65536
    k = torch.zeros((layers, 1, 4, cap, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert (layers - 1) * 4 * cap * 128 > 2 ** 31
    x = Inputs((28, 4, 128), [300], [5], ref.tree_masks([5], np.random.default_rng(0)))
    n = 305
    k[-1, :, :, :n] = x.k[0, :, :, :n]
    v[-1, :, :, :n] = x.v[0, :, :, :n]
    cache = lib.Cache(k, v)
    lse = torch.empty((5, 28), device="cuda")
    out = cache.tree_attention(x.q, x.kv_len, x.rows, x.visible, layer=layers - 1, lse=lse)
    check_attention(x, out, lse)
    w = torch.zeros(k.shape[:4], device="cuda")
    cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible, layer=layers - 1)
    want, tol = ref.weights(*[t for i, t in enumerate(x.request(0)) if i != 2], x.scale, lse.double())
    assert ((w[-1, 0, :, :n].double() - want).abs() <= tol).all()
    assert (w[:-1] == 0).all() and (w[-1, 0, :, n:] == 0).all()


def test_full_cache(lib):
    """The rows' entries end with the cache; a length one further is skipped."""
    x = Inputs((4, 2, 64), [251], [5], ref.chain_masks([5]), room=0)
    check_attention(x, *run_attention(lib, x))
    cache = lib.Cache(x.k, x.v)
    for bad in (252, -1, 2 ** 31 - 1, -2 ** 31):
        x.kv_len.fill_(bad)
        out = torch.full_like(x.q, 3.0).contiguous()
        lse = torch.full((5, 4), 3.0, device="cuda")
        w = torch.full(x.k.shape[:4], 3.0, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache.tree_attention(x.q, x.kv_len, x.rows, out=out, lse=lse, error_bits=err)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY
        err.zero_()
        cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, error_bits=err)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY
        assert (out == 3).all() and (lse == 3).all() and (w == 3).all()
        cache.tree_attention(x.q, x.kv_len, x.rows, out=out, lse=lse)  # no flag to set
        torch.cuda.synchronize()


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("length", [0, 130])
def test_masks(lib, length, q_type):
    """Rows that see no row of their own request (nothing at all with no
    prefix), rows that see later rows, all rows, bits past the rows."""
    masks = [[0, 0b1, 0b11110, 0b11111, (2 ** 64 - 1) ^ 0b11111, 2 ** 64 - 1]]
    x = Inputs((28, 4, 128), [length], [6], masks, q_type)
    check_attention(x, *run_attention(lib, x))
    check_weights(lib, x)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("length", [0, 127, 300])
def test_masked_places_do_not_matter(lib, length, value):
    """NaN and infinities in entries that a row does not see change nothing for
    it; a row that sees such a value gets what the formula gives."""
    masks = [[0b1, 0b11, 0b101, 0b1001, 0b10101]]
    x = Inputs((28, 4, 128), [length], [5], masks)
    base, base_lse = run_attention(lib, x)
    for which in (x.k, x.v):
        kept = which[0, 0, :, length + 1].clone()
        which[0, 0, :, length + 1] = value  # seen by row 1 alone
        out, lse = run_attention(lib, x)
        for i in (0, 2, 3, 4):
            assert torch.equal(out[i], base[i]) and torch.equal(lse[i], base_lse[i])
        which[0, 0, :, length + 1] = kept
    # one element of a value: its dim alone
    x.v[0, 0, :, length + 1, 3] = value
    out, lse = run_attention(lib, x)
    got = out[1, :, 3]
    assert torch.isnan(got).all() if math.isnan(value) else (got == value).all()
    rest = [e for e in range(128) if e != 3]
    assert torch.equal(out[1][:, rest], base[1][:, rest]) and torch.equal(lse, base_lse)


def test_extreme_scores(lib):
    """Scores far apart and of one sign; a key of the type's lowest value."""
    x = Inputs((4, 2, 64), [400], [5], ref.chain_masks([5]), torch.bfloat16, spread=60.0)
    check_attention(x, *run_attention(lib, x))
    x.q.copy_(x.q.abs() * 0.02)
    x.k[0, 0, :, 7] = torch.finfo(torch.bfloat16).min / 4096  # a weight of 0, a finite score
    out, lse = run_attention(lib, x)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def check_weights(lib, x, **kw):
    cache = lib.Cache(x.k, x.v)
    total = sum(x.rows)
    lse = torch.empty((total, x.heads[0]), dtype=torch.float64, device="cuda")
    for b in range(len(x.lens)):
        if x.rows[b]:
            lse[x.starts[b]:x.starts[b + 1]] = ref.attention(*x.request(b), x.scale)[2]
    lse = lse.float()
    g = torch.Generator(device="cuda").manual_seed(9)
    w0 = torch.rand(x.k.shape[:4], generator=g, device="cuda")
    w = w0.clone()
    cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible, **kw)
    torch.cuda.synchronize()
    for b, (n, r) in enumerate(zip(x.lens, x.rows)):
        if not r:
            assert torch.equal(w[0, b], w0[0, b])
            continue
        q, k, _, seen = x.request(b)
        want, tol = ref.weights(q, k, seen, x.scale, lse[x.starts[b]:x.starts[b + 1]].double())
        want = want.clone()
        want[:, :n] += w0[0, b, :, :n].double()
        got = w[0, b, :, :n + r].double()
        assert ((got - want).abs() <= tol + want.abs() * 2.0 ** -23).all(), (b, float((got - want).abs().max()))
        assert torch.equal(w[0, b, :, n + r:], w0[0, b, :, n + r:])


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("length,rows", [(0, 1), (0, 64), (1, 5), (127, 1), (128, 17), (129, 64), (1000, 9)])
def test_weights_sizes(lib, heads, length, rows, q_type):
    masks = ref.tree_masks([rows], np.random.default_rng(length + rows))
    check_weights(lib, Inputs(heads, [length], [rows], masks, q_type, seed=length, pad=1))


def test_weights_ragged(lib):
    lens = [0, 1, 700, 2055, 128, 64, 5333, 17]
    rows = [3, 0, 17, 1, 0, 64, 9, 33]
    for q_type in (torch.bfloat16, torch.float32):
        x = Inputs((28, 4, 128), lens, rows, ref.tree_masks(rows, np.random.default_rng(5)), q_type)
        check_weights(lib, x)
        check_weights(lib, x, max_len=5333)


def test_weights_masked_keys(lib):
    x = Inputs((28, 4, 128), [130], [5], [[0b1, 0b10, 0b101, 0b1001, 0b10001]])
    out, lse = run_attention(lib, x)
    cache = lib.Cache(x.k, x.v)
    w = torch.zeros(x.k.shape[:4], device="cuda")
    cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible)
    total = w[0, 0].sum(1)
    # every row's weights sum to 1: five rows of seven heads to a kv head
    assert ((total - 35).abs() <= 35 * 2.0 ** -12).all()


# ---- eviction -------------------------------------------------------------------

def evict_case(lib, shape, lens, keep, recent, weights=None, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(shape[:4], generator=g, device="cuda") if weights is None else weights.clone()
    bits = lambda t: t.view(torch.int16).cpu().numpy().copy()  # noqa: E731
    hk, hv, hw = bits(k), bits(v), w.cpu().numpy().copy()
    new = ref.evict(hk, hv, hw, lens, keep, recent)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lib.Cache(k, v).evict(w, kv_len, keep, recent)
    torch.cuda.synchronize()
    assert kv_len.tolist() == new
    assert np.array_equal(bits(k), hk) and np.array_equal(bits(v), hv)
    assert np.array_equal(w.cpu().numpy().view(np.int32), hw.view(np.int32))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length,keep,recent", [
    (0, 0, 0), (1, 0, 0), (1, 1, 1), (2, 1, 0), (2, 1, 5), (31, 30, 0), (33, 32, 1), (200, 150, 50),
    (200, 0, 3), (200, 200, 3), (200, 300, 3), (200, 1, 1), (1025, 1024, 0), (1025, 77, 77), (3000, 2250, 16)])
def test_evict_sizes(lib, d, length, keep, recent):
    evict_case(lib, (2, 1, 2, length + 5, d), [length], [keep], recent, seed=length)


def test_evict_ragged(lib):
    lens = [0, 5, 900, 2500, 2505, -3, 2506, 64]
    keep = [3, 5, 450, 10, 2504, 1, 1, 63]
    evict_case(lib, (3, 8, 4, 2505, 128), lens, keep, 7)


def test_evict_whole_capacity(lib):
    evict_case(lib, (1, 1, 1, 65536, 64), [65536], [49152], 128)


def test_evict_ties_and_special_weights(lib):
    shape = (1, 1, 2, 600, 64)
    w = torch.zeros(shape[:4], device="cuda")
    evict_case(lib, shape, [590], [300], 10, w)                  # all equal
    w[0, 0, 0, ::2] = -0.0                                       # -0 equals 0
    evict_case(lib, shape, [590], [300], 10, w)
    pick = torch.tensor([math.nan, math.inf, -math.inf, 1.0, -1.0, 0.0, 1e-40, 3.4e38], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    w = pick[torch.randint(0, len(pick), shape[:4], generator=g, device="cuda")]
    for keep in (1, 50, 150, 300, 500, 589):
        evict_case(lib, shape, [590], [keep], 0, w)
    evict_case(lib, shape, [590], [300], 0, torch.full(shape[:4], math.nan, device="cuda"))


def test_evict_equal_high_bits(lib):
    """Weights that differ in their last bits only."""
    shape = (1, 2, 2, 3000, 64)
    base = torch.full(shape[:4], 1.0, device="cuda").view(torch.int32)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (base + torch.randint(0, 200, shape[:4], generator=g, device="cuda", dtype=torch.int32)).view(torch.float32)
    evict_case(lib, shape, [2999, 1500], [1000, 1499], 4, w)


# ---- probabilities ---------------------------------------------------------------

@pytest.mark.parametrize("rows,vocab,temperature", [
    (1, 1, 1.0), (3, 2, 0.5), (2, 31, 2.0), (5, 4096, 0.7), (2, 4097, 1.0), (1, 50001, 0.3), (9, 152064, 0.7),
    (3, 151936, 1.3), (1, 400003, 1.0), (300, 129, 1.0),
    (75, 152064, 0.7), (103, 90004, 1.0), (2, 500000, 1.0), (70000, 5, 1.0)])
def test_probs(lib, rows, vocab, temperature):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((rows, vocab), generator=g, device="cuda") * 5
    want = torch.softmax(x.double() / temperature, 1)
    # the exponent's argument y = (x - max) log2(e) / T, up to |y|, is off by 2^-22 |y|
    # in all (its factor, the difference, the product), the exponential by 2^-21, the
    # sum of positive terms and the quotient by the sum's depth of at most 2^8 additions
    y = (x.double() - x.double().amax(1, keepdim=True)).abs() * (math.log2(math.e) / temperature)
    tol = want * (y * 2.0 ** -22 + 2.0 ** -21 + 2.0 ** -15) + 2.0 ** -126
    got = lib.token_probs(x, temperature)
    assert ((got.double() - want).abs() <= tol).all()
    again = lib.token_probs(x, temperature, out=x)  # in place
    assert again is x and torch.equal(again, got)


def test_probs_special_rows(lib):
    x = torch.randn((6, 5000), device="cuda")
    x[0, 1:] = -math.inf
    x[1] = -math.inf
    x[2, 4999] = math.nan
    x[3, 7] = math.inf
    x[4, ::2] = -math.inf
    x[5] = torch.finfo(torch.float32).min
    p = lib.token_probs(x, 0.8)
    assert p[0, 0] == 1 and (p[0, 1:] == 0).all()
    assert (p[1] == 0).all() and torch.isnan(p[2]).all() and torch.isnan(p[3]).all()
    assert (p[4, ::2] == 0).all() and abs(float(p[4].double().sum()) - 1) < 2.0 ** -15
    assert ((p[5].double() * 5000 - 1).abs() <= 2.0 ** -15).all()


# ---- acceptance -------------------------------------------------------------------

def dyadic_rows(rng, rows, vocab, live):
    """Probabilities that are multiples of 2^-20 and sum to 1: every sum of them is
    exact in 32 bits' 24."""
    out = np.zeros((rows, vocab), dtype=np.float32)
    for r in range(rows):
        at = rng.choice(vocab, size=min(live, vocab), replace=False)
        cuts = np.sort(rng.integers(0, 2 ** 20 + 1, len(at) - 1)) if len(at) > 1 else np.array([], dtype=int)
        parts = np.diff(np.concatenate([[0], cuts, [2 ** 20]]))
        out[r, at] = (parts / 2.0 ** 20).astype(np.float32)
    return out


def run_accept(lib, probs, draft, cand, ks, u):
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device="cuda")  # noqa: E731
    n = torch.full((len(ks),), -7, dtype=torch.int32, device="cuda")
    tok = torch.full((len(ks),), -7, dtype=torch.int32, device="cuda")
    lib.accept_sampled(dev(probs, torch.float32), dev(cand, torch.int32) if sum(ks) else None, ks,
                       dev(u, torch.float32), n, tok,
                       draft_probs=None if draft is None else dev(draft, torch.float32))
    torch.cuda.synchronize()
    return n.tolist(), tok.tolist()


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab,live", [(1, 1), (2, 2), (33, 20), (1000, 40), (4096, 4096), (152064, 3000), (151937, 500),
                                        (1000004, 5000), (1000003, 5000)])
def test_accept(lib, vocab, live, with_draft):
    rng = np.random.default_rng(vocab + with_draft)
    for ks in ([0], [1], [16], [0, 3, 16, 1, 8, 0, 5]):
        rows, total = sum(ks) + len(ks), sum(ks)
        probs = dyadic_rows(rng, rows, vocab, live)
        draft = dyadic_rows(rng, max(total, 1), vocab, live)[:total] if with_draft else None
        cand = []
        r = 0
        for k in ks:
            for i in range(k):
                likely = np.flatnonzero(probs[r + i] > 0) if rng.random() < 0.8 else np.arange(vocab)
                cand.append(int(rng.choice(likely)))
            r += k + 1
        # random numbers that are dyadic too, among them the borders of the sums
        u = (rng.integers(0, 2 ** 20, rows) / 2.0 ** 20).astype(np.float32)
        u[rng.random(rows) < 0.3] = 0.0
        want = ref.accept(probs.astype(np.float64), None if draft is None else draft.astype(np.float64), cand, ks,
                          u.astype(np.float64))
        assert run_accept(lib, probs, draft, cand, ks, u) == want


def test_accept_borders(lib):
    """u on the border of two tokens takes the upper one; zero weights are passed over."""
    p = np.zeros((1, 4000), dtype=np.float32)
    p[0, [5, 1030, 3999]] = [0.25, 0.5, 0.25]
    below = np.nextafter(np.float32(0.25), np.float32(0))
    for u, want in ((0.0, 5), (below, 5), (0.25, 1030), (0.74, 1030), (0.75, 3999), (1 - 2.0 ** -24, 3999)):
        assert run_accept(lib, p, None, [], [0], [u]) == ([0], [want])


def test_accept_special_rows(lib):
    V = 3000
    p = np.zeros((2, V), dtype=np.float32)
    p[:, 7] = 1.0
    q = np.zeros((1, V), dtype=np.float32)
    # the candidate cannot stand (p = 0); nothing is left over q: the token comes from p
    q[0, 7], q[0, 9] = 1.0, 0.5
    assert run_accept(lib, p, q, [9], [1], [0.5, 0.3]) == ([0], [7])
    # a candidate of certainty with u = 1 - 2^-24 and p = 1 stands, with p = 0 never does
    assert run_accept(lib, p, None, [7], [1], [1 - 2.0 ** -24, 0.3]) == ([1], [7])
    assert run_accept(lib, p, None, [8], [1], [0.0, 0.3]) == ([0], [7])
    # out of the vocabulary
    for c in (-1, V, 2 ** 31 - 1):
        assert run_accept(lib, p, None, [c], [1], [0.0, 0.3]) == ([0], [7])
    # rows that hold nothing, NaN and negative weights
    z = np.zeros((1, V), dtype=np.float32)
    assert run_accept(lib, z, None, [], [0], [0.5]) == ([0], [-1])
    z[0, :10] = [math.nan, -1.0, 0.25, math.nan, 0.0, 0.25, -math.inf, 0.0, 0.0, math.nan]
    assert run_accept(lib, z, None, [], [0], [0.5]) == ([0], [5])
    p[0, 7] = math.nan  # a NaN probability accepts nothing
    assert run_accept(lib, p, None, [7], [1], [0.0, 0.5]) == ([0], [-1])


def test_accept_follows_the_target(lib):
    """Over a grid of random numbers the accepted-or-drawn first token has the
    target's distribution, whatever the drafter's is: every pair (u_0, u_1) of a
    64 x 64 grid, for each candidate weighted by its draft probability."""
    V, N = 5, 64
    p = np.array([8, 16, 4, 32, 4], dtype=np.float32) / 64
    q = np.array([32, 8, 16, 8, 0], dtype=np.float32) / 64
    mass = np.zeros(V)
    grid = (np.arange(N) / N).astype(np.float32)
    for c in range(V):
        if q[c] == 0:
            continue
        for u0 in grid:  # a call of 64 requests: one for each u_1
            probs = np.tile(p, (2 * N, 1))
            u = np.empty(2 * N, dtype=np.float32)
            u[0::2], u[1::2] = u0, grid
            n, tok = run_accept(lib, probs, np.tile(q, (N, 1)), [c] * N, [1] * N, u)
            for a, t in zip(n, tok):
                mass[c if a else t] += q[c]
    mass /= N * N
    # each test is decided exactly on the grid up to one cell of u_0 and of u_1
    assert np.abs(mass - p).max() <= 2.0 / N


# ---- streams, graphs, runs ----------------------------------------------------------

def run_together(lib, x, w, probs_in, cand, ks, u, keep, stream=0):
    """A step as a decoder would run it: attention with its sums, the weights it
    gives, eviction, probabilities, acceptance."""
    cache = lib.Cache(x.k, x.v)
    out, lse = torch.empty(x.q.shape, dtype=x.q.dtype, device="cuda"), torch.empty(x.q.shape[:2], device="cuda")
    p = torch.empty_like(probs_in)
    n, tok = (torch.zeros(len(ks), dtype=torch.int32, device="cuda") for _ in range(2))

    def step(s):
        cache.tree_attention(x.q, x.kv_len, x.rows, x.visible, out=out, lse=lse, stream=s)
        cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible, stream=s)
        cache.evict(w, x.kv_len, keep, recent=4, stream=s)
        lib.token_probs(probs_in, 0.9, out=p, stream=s)
        lib.accept_sampled(p, cand, ks, u, n, tok, stream=s)
    return step, (out, lse, w, x.k, x.v, x.kv_len, p, n, tok)


def together_inputs(seed=0):
    rows = [5, 9]
    x = Inputs((28, 4, 128), [700, 1300], rows, ref.tree_masks(rows, np.random.default_rng(seed)), seed=seed)
    for t in (x.k, x.v):
        t[torch.isnan(t)] = 0
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.rand(x.k.shape[:4], generator=g, device="cuda")
    logits = torch.randn((14, 4096), generator=g, device="cuda") * 4
    cand = logits[[0, 1, 2, 3] + list(range(5, 13))].argmax(1).int()
    u = torch.rand(14, generator=g, device="cuda")
    return x, w, logits, cand, [4, 8], u, [600, 1301]


def test_run_together(lib):
    args = together_inputs()
    x, w, logits, cand, ks, u, keep = args
    k0, v0, w0 = x.k.clone(), x.v.clone(), w.clone()
    step, (out, lse, w, k, v, kv_len, p, n, tok) = run_together(lib, *args)
    step(0)
    torch.cuda.synchronize()
    y, *_ = together_inputs()
    check_attention(y, out, lse)
    # the eviction by the weights of this very call
    hw = w0.cpu().numpy().copy()
    cache = lib.Cache(k0, v0)
    w1 = w0.clone()
    cache.attention_weights(y.q, lse, w1, y.kv_len, y.rows, y.visible)
    hw = w1.cpu().numpy().copy()
    hk, hv = (t.view(torch.int16).cpu().numpy().copy() for t in (k0, v0))
    assert kv_len.tolist() == ref.evict(hk, hv, hw, [700, 1300], keep, 4)
    assert np.array_equal(k.view(torch.int16).cpu().numpy(), hk) and np.array_equal(v.view(torch.int16).cpu().numpy(), hv)
    assert np.array_equal(w.cpu().numpy(), hw)
    assert (n.tolist(), tok.tolist()) == ref.accept(p.double().cpu().numpy(), None, cand.tolist(), ks,
                                                    u.double().cpu().numpy())


def test_graph_and_stream(lib):
    """The same step on another stream, and captured and replayed: bit for bit the
    same, replay after replay from the same inputs."""
    step, outs = run_together(lib, *together_inputs(3))
    first = [t.clone() for t in outs]  # inputs among them
    step(0)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]

    def restore():
        for t, f in zip(outs, first):
            t.copy_(f)
    s = torch.cuda.Stream()
    restore()
    torch.cuda.synchronize()
    step(s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    g = torch.cuda.CUDAGraph()
    restore()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        step(s.cuda_stream)
    for _ in range(3):
        restore()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_back_to_back(lib):
    """Calls that follow one another without a wait on one workspace."""
    xs = [Inputs((28, 4, 128), [n], [r], ref.tree_masks([r], np.random.default_rng(n)), seed=n)
          for n, r in ((3000, 17), (15, 3), (2999, 1), (700, 64))]
    outs = []
    k, v = xs[0].k, xs[0].v
    caches = [lib.Cache(x.k, x.v) for x in xs]
    for c in caches:
        c._workspace = caches[0]._workspace if caches[0]._workspace.numel() >= c._workspace.numel() else c._workspace
    for _ in range(3):
        for x, c in zip(xs, caches):
            lse = torch.empty((sum(x.rows), 28), device="cuda")
            outs.append((x, c.tree_attention(x.q, x.kv_len, x.rows, x.visible, lse=lse), lse))
    torch.cuda.synchronize()
    for x, out, lse in outs:
        check_attention(x, out, lse)
    for i in range(len(xs)):  # bit for bit the same each time
        assert torch.equal(outs[i][1], outs[i + len(xs)][1]) and torch.equal(outs[i][1], outs[i + 2 * len(xs)][1])


# ---- calls at the edges of what is allowed ------------------------------------------

def test_smallest_and_largest_temperatures(lib):
    """At the smallest temperature a row is its maxima, at the largest it is even."""
    x = torch.zeros((3, 1000), device="cuda")
    x[0, 17], x[1, 3], x[1, 900] = 1.0, 2.0, 2.0
    x[2, ::2] = -math.inf
    p = lib.token_probs(x, 1e-45)
    assert p[0, 17] == 1 and p[0].sum() == 1
    assert p[1, 3] == 0.5 and p[1, 900] == 0.5 and p[1].sum() == 1
    assert (p[2, ::2] == 0).all() and ((p[2, 1::2].double() * 500 - 1).abs() <= 2.0 ** -15).all()
    p = lib.token_probs(x, 3e38)
    assert ((p[:2].double() * 1000 - 1).abs() <= 2.0 ** -15).all() and (p[2, ::2] == 0).all()


@pytest.mark.parametrize("heads", [(1024, 1, 64), (640, 5, 128)])
def test_many_heads_to_a_kv_head(lib, heads):
    """Hundreds of query tiles of one kv head, one after another in a CTA."""
    rows, lens = [64, 1, 20], [130, 0, 515]
    masks = ref.tree_masks(rows, np.random.default_rng(7))
    x = Inputs(heads, lens, rows, masks, torch.float32)
    out, lse = run_attention(lib, x)
    check_attention(x, out, lse)
    check_weights(lib, x)


def test_two_streams_at_once(lib):
    """Calls that overlap, each on a stream, cache and workspace of its own, give
    what they give alone."""
    xs = [Inputs((28, 4, 128), [n, 40], [r, 3], ref.tree_masks([r, 3], np.random.default_rng(n)), t, seed=n)
          for n, r, t in ((9000, 30, torch.float32), (8000, 64, torch.bfloat16))]
    caches = [lib.Cache(x.k, x.v) for x in xs]
    logits = [torch.randn((40, 60000), device="cuda") for _ in xs]

    def step(i, stream):
        x = xs[i]
        lse = torch.empty((sum(x.rows), 28), device="cuda")
        w = torch.zeros(x.k.shape[:4], device="cuda")
        outs = [torch.empty_like(x.q, memory_format=torch.contiguous_format), lse, w, torch.empty_like(logits[i])]
        torch.cuda.synchronize()

        def run():
            caches[i].tree_attention(x.q, x.kv_len, x.rows, x.visible, lse=lse, out=outs[0], stream=stream)
            caches[i].attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible, stream=stream)
            lib.token_probs(logits[i], 0.9, out=outs[3], stream=stream)
        return run, outs
    streams = [torch.cuda.Stream() for _ in xs]
    alone = []
    for i in range(2):
        run, outs = step(i, streams[i].cuda_stream)
        for _ in range(4):
            run()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in outs])
    pairs = [step(i, streams[i].cuda_stream) for i in range(2)]
    for _ in range(4):
        for run, _ in pairs:
            run()
    torch.cuda.synchronize()
    for (_, outs), want in zip(pairs, alone):
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_accept_the_same_candidate_twice(lib):
    """One token at several places, each place with its own row; random numbers that
    are no numbers, or outside [0, 1), take the nearest that is one (NaN: 0)."""
    V = 2000
    p = np.zeros((3, V), dtype=np.float32)
    p[0, [4, 9]], p[1, [4, 9]], p[2, [4, 9]] = [0.75, 0.25], [0.25, 0.75], [0.5, 0.5]
    assert run_accept(lib, p, None, [4, 4], [2], [0.5, 0.2, 0.1]) == ([2], [4])
    assert run_accept(lib, p, None, [4, 4], [2], [0.5, 0.5, 0.1]) == ([1], [9])
    for u, want in ((math.nan, 4), (-1.0, 4), (1.0, 9), (7.0, 9), (math.inf, 9), (-math.inf, 4)):
        assert run_accept(lib, p[:1], None, [], [0], [u]) == ([0], [want])


def test_probs_and_acceptance_off_16_bytes(lib):
    """Rows whose first value lies 4 bytes behind a 16-byte boundary."""
    rng = np.random.default_rng(5)
    x = torch.randn((5, 4096), device="cuda")
    off = torch.empty(5 * 4096 + 1, device="cuda")[1:].view(5, 4096)
    off.copy_(x)
    p = lib.token_probs(off, 0.7, out=torch.empty(5 * 4096 + 1, device="cuda")[1:].view(5, 4096))
    want = lib.token_probs(x, 0.7)
    assert ((p - want).abs() <= want * 2.0 ** -14).all()
    rows = dyadic_rows(rng, 5, 4096, 300)
    dev = torch.empty(5 * 4096 + 1, device="cuda")[1:].view(5, 4096)
    dev.copy_(torch.from_numpy(rows))
    cand = [int(np.flatnonzero(rows[i])[3]) for i in (0, 1, 3)]
    u = (rng.integers(0, 2 ** 20, 5) / 2.0 ** 20).astype(np.float32)
    n, tok = (torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(2))
    lib.accept_sampled(dev, torch.tensor(cand, dtype=torch.int32, device="cuda"), [2, 1],
                       torch.from_numpy(u).cuda(), n, tok)
    assert (n.tolist(), tok.tolist()) == ref.accept(rows.astype(np.float64), None, cand, [2, 1], u.astype(np.float64))


def test_cache_of_another_device(lib, monkeypatch):
    """A cache made on one device is refused while another is current."""
    x = Inputs((4, 2, 64), [40], [3], ref.tree_masks([3], np.random.default_rng(1)))
    cache = lib.Cache(x.k, x.v)
    monkeypatch.setattr(cache, "_current", lambda: x.k.get_device() + 1)
    w = torch.zeros(x.k.shape[:4], device="cuda")
    for call in (lambda: cache.tree_attention(x.q, x.kv_len, x.rows, x.visible),
                 lambda: cache.attention_weights(x.q, w, w, x.kv_len, x.rows, x.visible),
                 lambda: cache.evict(w, x.kv_len, [20])):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()


FIRST_USE = """
import torch
import paper_2609_37617_gb300 as lib
g = torch.Generator(device="cuda").manual_seed(3)
k, v = (torch.randn((1, 2, 4, 2000, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
cache, rows = lib.Cache(k, v), [9, 4]
q = torch.randn((13, 28, 128), generator=g, device="cuda")
kv_len = torch.tensor([1900, 333], dtype=torch.int32, device="cuda")
lse, out = torch.empty((13, 28), device="cuda"), torch.empty_like(q)
w = torch.rand((1, 2, 4, 2000), generator=g, device="cuda")
logits = torch.randn((90, 152064), generator=g, device="cuda")
probs = torch.empty_like(logits)
cand = torch.zeros(8, dtype=torch.int32, device="cuda")
u = torch.full((9,), 0.5, device="cuda")
n, tok = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(2))
state = [t.clone() for t in (k, v, w, kv_len)]

def step(s):
    cache.tree_attention(q, kv_len, rows, out=out, lse=lse, stream=s)
    cache.attention_weights(q, lse, w, kv_len, rows, stream=s)
    cache.evict(w, kv_len, [1000, 300], recent=16, stream=s)
    lib.token_probs(logits, 0.8, out=probs, stream=s)
    lib.accept_sampled(probs[:9], cand, [8], u, n, tok, stream=s)

def results():
    torch.cuda.synchronize()
    return [t.clone() for t in (out, lse, w, k, v, kv_len, probs, n, tok)]
torch.cuda.synchronize()
s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=s):
    step(s.cuda_stream)
graph.replay()
first = results()
for t, old in zip((k, v, w, kv_len), state):
    t.copy_(old)
torch.cuda.synchronize()
step(0)
assert all(torch.equal(a, b) for a, b in zip(results(), first))
"""


def test_first_use_under_capture(lib):
    """A process whose first call of each operator is captured."""
    subprocess.run([sys.executable, "-c", FIRST_USE], check=True, timeout=120,
                   cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


# ---- rows and entries that are not finite --------------------------------------------

# (requests' lengths, rows): an item in one CTA, in a cluster, in even shares; the last also two
# requests, so that CTAs end one item and begin another
CUTS = [([200], [3]), ([1564], [3]), ([15128], [3]), ([9000, 8000], [3, 64])]


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cut", range(len(CUTS)))
def test_nan_reaches_the_row_however_the_work_is_cut(lib, cut, q_type):
    """A query that holds NaN, keys of NaN over some tiles, a part or all of the prefix:
    the rows that they enter get NaN in out and lse, all others the same bits as before."""
    lens, rows = CUTS[cut]
    masks = ref.tree_masks(rows, np.random.default_rng(cut))
    x = Inputs((28, 4, 128), lens, rows, masks, q_type, seed=cut)
    base, base_lse = run_attention(lib, x)

    def check(out, lse, rows_of, heads):
        hit = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
        for r in rows_of:
            hit[r, heads] = True
        assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
        assert torch.equal(out[~hit], base[~hit]) and torch.equal(lse[~hit], base_lse[~hit])

    kept = x.q[1, 9, 100].clone()
    x.q[1, 9, 100] = math.nan
    check(*run_attention(lib, x), [1], [9])
    x.q[1, 9, 100] = kept
    n = lens[0]
    for a, b in ((0, 1), (0, 128), (n // 2, n), (0, 7 * n // 8), (n // 3, n // 3 + 700), (0, n)):
        kept = x.k[0, 0, 2, a:min(b, n)].clone()
        x.k[0, 0, 2, a:min(b, n)] = math.nan
        check(*run_attention(lib, x), range(rows[0]), list(range(14, 21)))
        x.k[0, 0, 2, a:min(b, n)] = kept


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cut", range(len(CUTS)))
def test_infinite_values_of_the_prefix(lib, cut, q_type):
    """out = sum p_t v_t with an infinite v_t of the prefix is that infinity (two of both signs:
    NaN) in its dim and its kv head's rows, the same bits as before elsewhere; however
    small p_t is beside the others."""
    lens, rows = CUTS[cut]
    masks = ref.tree_masks(rows, np.random.default_rng(cut))
    x = Inputs((28, 4, 128), lens, rows, masks, q_type, seed=cut)
    n = lens[0]
    # scores far apart: weights that are 0 in 32 bits beside others
    x.k[0, 0, 1, 5] *= 40
    x.k[0, 0, 1, n - 1] *= 40
    x.k[0, 0, 1, n // 2] *= 40
    base, base_lse = run_attention(lib, x)
    assert torch.isfinite(base).all()
    mine, heads = list(range(rows[0])), list(range(7, 14))
    for at, value in ((0, math.inf), (5, -math.inf), (n // 2, math.inf), (n // 2 + 1, math.nan), (n - 1, -math.inf),
                      (n - 2, math.inf), (n // 3, -math.inf)):
        kept = x.v[0, 0, 1, at, 70].clone()
        x.v[0, 0, 1, at, 70] = value
        out, lse = run_attention(lib, x)
        got = out[mine][:, heads, 70]
        assert (torch.isnan(got) if math.isnan(value) else got == value).all(), (at, value)
        out[mine[0]:mine[-1] + 1, heads[0]:heads[-1] + 1, 70] = base[mine[0]:mine[-1] + 1, heads[0]:heads[-1] + 1, 70]
        assert torch.equal(out, base) and torch.equal(lse, base_lse), (at, value)
        x.v[0, 0, 1, at, 70] = kept
    x.v[0, 0, 1, 3, 70], x.v[0, 0, 1, n - 3, 70] = math.inf, -math.inf
    x.v[0, 0, 1, 2, 33], x.v[0, 0, 1, 4, 33] = math.inf, math.inf
    x.v[0, 0, 1, 2] = math.inf  # a whole entry, beside the last two
    out, _ = run_attention(lib, x)
    got = out[mine][:, heads]
    assert torch.isnan(got[..., 70]).all()
    assert (got[..., [e for e in range(128) if e != 70]] == math.inf).all()


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(28, 4, 128), (4, 2, 64)])
@pytest.mark.parametrize("cut", range(len(CUTS)))
def test_infinite_keys(lib, cut, heads, q_type):
    """A score of -inf is a weight of 0, in the prefix and in the rows' own entries;
    one of +inf makes its row NaN."""
    lens, rows = CUTS[cut]
    nq, nkv, d = heads
    masks = ref.chain_masks(rows)
    x = Inputs(heads, lens, rows, masks, q_type, seed=cut)
    x.q[:, :, 5] = -x.q[:, :, 5].abs() - 2.0 ** -6
    x.q[:, :, 6] = x.q[:, :, 6].abs() + 2.0 ** -6
    n, r = lens[0], rows[0]
    gone = sorted({0, 77, 127, n // 2, n - 1, n})  # (n: the first row's own entry)
    for t in gone:
        x.k[0, 0, 0, t, 5] = math.inf
        x.k[0, 0, 0, t, 6] = -math.inf if t % 2 else x.k[0, 0, 0, t, 6]
    out, lse = run_attention(lib, x)
    # the formula without those entries, for kv head 0; the other heads as they are
    q, k, v, seen = x.request(0)
    less = seen.clone()
    less[:, gone] = False
    G, half_step = nq // nkv, torch.finfo(q_type).eps / 2
    for g in range(nkv):
        qg, kg, vg = q[:, g * G:(g + 1) * G], k[g:g + 1], v[g:g + 1]
        want, tol, want_lse, tol_lse = ref.attention(qg, kg, vg, less if g == 0 else seen, x.scale)
        got = out[:r, g * G:(g + 1) * G].double()
        assert ((got - want).abs() <= want.abs() * half_step * (1 + 2.0 ** -6) + tol).all()
        assert ((lse[:r, g * G:(g + 1) * G].double() - want_lse).abs() <= tol_lse).all()
    w = torch.zeros(x.k.shape[:4], device="cuda")
    lib.Cache(x.k, x.v).attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible)
    want, tol = ref.weights(q[:, :G], k[:1], less, x.scale, lse[:r, :G].double())
    got = w[0, 0, :1, :n + r].double()
    assert ((got - want).abs() <= tol + want.abs() * 2.0 ** -23).all() and (got[0, gone] == 0).all()
    # +inf: the rows that see it, NaN
    x.k[0, 0, 0, 9, 6] = math.inf
    x.k[0, 0, 0, 9, 5] = 0.0
    out, lse = run_attention(lib, x)
    assert torch.isnan(out[:r, :G]).all() and torch.isnan(lse[:r, :G]).all()
    assert torch.isfinite(out[:r, G:]).all() and torch.isfinite(out[r:]).all()


def test_clusters_beside_other_work(lib):
    """Rows and requests whose clusters hold CTAs with nothing to do, call after call while another
    stream fills the SMs: the same results each time."""
    rng = np.random.default_rng(11)
    ks, V = [1, 0, 3, 2], 40
    probs = dyadic_rows(rng, sum(ks) + len(ks), V, 20)
    draft = dyadic_rows(rng, sum(ks), V, 20)
    cand = [int(t) for t in rng.integers(0, V, sum(ks))]
    u = (rng.integers(0, 2 ** 20, len(probs)) / 2.0 ** 20).astype(np.float32)
    want = ref.accept(probs.astype(np.float64), draft.astype(np.float64), cand, ks, u.astype(np.float64))
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device="cuda")  # noqa: E731
    p, q, c, r = dev(probs, torch.float32), dev(draft, torch.float32), dev(cand, torch.int32), dev(u, torch.float32)
    n, tok = (torch.empty((300, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((90, 90004), generator=g, device="cuda") * 4  # (clusters that go from row to row)
    y = torch.randn((3, 20490), generator=g, device="cuda") * 4
    first = [lib.token_probs(t, 0.9) for t in (x, y)]
    other = torch.cuda.Stream()
    big = torch.randn((2048, 2048), device="cuda")
    torch.cuda.synchronize()
    for i in range(300):
        if i % 3 == 0:
            with torch.cuda.stream(other):
                big @ big
        lib.accept_sampled(p, c, ks, r, n[i], tok[i], draft_probs=q)
        if i % 5 == 0:
            for t, f in zip((x, y), first):
                assert torch.equal(lib.token_probs(t, 0.9), f)
    torch.cuda.synchronize()
    assert all(a == want[0] for a in n.tolist()) and all(t == want[1] for t in tok.tolist())


def test_one_workspace_for_several_caches(lib, monkeypatch):
    """Calls in even shares, which leave parts in the workspace, an eviction and small calls one
    after another without a wait, all on one workspace: bit for bit what each gives alone."""
    sizes = [(15128, 17), (9000, 64), (200, 3), (12000, 1), (8100, 9)]
    xs = [Inputs((28, 4, 128), [n], [r], ref.tree_masks([r], np.random.default_rng(n)), seed=n) for n, r in sizes]
    alone = [run_attention(lib, x) for x in xs]
    caches = [lib.Cache(x.k, x.v) for x in xs]
    shared = max((c._workspace for c in caches), key=lambda t: t.numel())
    for c in caches:
        c._workspace = shared
    # (a cache of the same shape as the first, to be cut)
    cut = [torch.randn_like(x, dtype=torch.float32).bfloat16() for x in (xs[2].k, xs[2].v)]
    evict = lib.Cache(*cut)
    assert evict._workspace.numel() <= shared.numel()
    evict._workspace = shared
    given = []
    for name, at in (("as2d_tree_attention", 5), ("as2d_cache_evict", 5)):
        f = getattr(lib._lib, name)
        monkeypatch.setattr(lib._lib, name, lambda *a, f=f, at=at: (given.append(a[at]), f(*a))[1])
    outs, w = [], torch.rand(cut[0].shape[:4], device="cuda")
    for _ in range(4):
        for i, (x, c) in enumerate(zip(xs, caches)):
            lse = torch.empty((sum(x.rows), 28), device="cuda")
            outs.append((i, c.tree_attention(x.q, x.kv_len, x.rows, x.visible, lse=lse), lse))
            if i % 2:
                evict.evict(w, torch.tensor([200], dtype=torch.int32, device="cuda"), [150], recent=5)
    torch.cuda.synchronize()
    assert len(given) == 28 and set(given) == {shared.data_ptr()}
    for i, out, lse in outs:
        assert torch.equal(out, alone[i][0]) and torch.equal(lse, alone[i][1])


def test_torchs_current_stream(lib):
    """Without a stream given, a call follows what torch's current stream does before it and
    precedes what it does next, and its result belongs there."""
    args = together_inputs(5)
    step, outs = run_together(lib, *args)
    first = [t.clone() for t in outs]
    step(0)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    x, w, logits, cand, ks, u, keep = args
    q, lg = x.q.clone(), logits.clone()
    for t, f in zip(outs, first):
        t.copy_(f)
    x.q.zero_()
    logits.zero_()
    big = torch.randn((8192, 8192), device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(3):
            big @ big
        x.q.copy_(q)  # long after the calls are enqueued
        logits.copy_(lg)
        cache = lib.Cache(x.k, x.v)
        lse = torch.empty(x.q.shape[:2], device="cuda")
        out = cache.tree_attention(x.q, x.kv_len, x.rows, x.visible, lse=lse)
        cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible)
        cache.evict(w, x.kv_len, keep, recent=4)
        p = lib.token_probs(logits, 0.9)
        n, tok = (torch.zeros(len(ks), dtype=torch.int32, device="cuda") for _ in range(2))
        lib.accept_sampled(p, cand, ks, u, n, tok)
        got = [t.clone() for t in (out, lse, w, x.k, x.v, x.kv_len, p, n, tok)]
        del out, p, cache  # may be given away while the calls run
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_results_made_for_a_given_stream(lib):
    """A result made for a call on another stream than torch's current one is not memory that
    the current one may still be using, nor given back to it while the call runs."""
    x = torch.randn((64, 50000), device="cuda")
    want = lib.token_probs(x, 0.7)
    at = Inputs((4, 2, 64), [300], [5], ref.tree_masks([5], np.random.default_rng(2)))
    base, _ = run_attention(lib, at)
    s = torch.cuda.Stream()
    cache = lib.Cache(at.k, at.v)
    torch.cuda.synchronize()
    for other in (s.cuda_stream, 0):
        with torch.cuda.stream(s if other == 0 else torch.cuda.default_stream()):
            p = lib.token_probs(x, 0.7, stream=other)
            out = cache.tree_attention(at.q, at.kv_len, at.rows, at.visible, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(p, want) and torch.equal(out, base)
    # (memory freed on the current stream is not taken for another one's result)
    free = torch.empty_like(x)
    address = free.data_ptr()
    del free
    p = lib.token_probs(x, 0.7, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert p.data_ptr() != address and torch.equal(p, want)


def test_integers_beyond_32_bits(lib):
    """Counts and indices that 32 bits do not hold are refused, not taken modulo 2^32."""
    x = Inputs((4, 2, 64), [40], [3], ref.tree_masks([3], np.random.default_rng(1)))
    cache, w = lib.Cache(x.k, x.v), torch.zeros(x.k.shape[:4], device="cuda")
    lse = torch.zeros((3, 4), device="cuda")
    n, tok = (torch.full((2,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    p, u = torch.ones((2, 8), device="cuda"), torch.zeros(2, device="cuda")
    far = 2 ** 32
    for call in (lambda: cache.evict(w, x.kv_len, [far + 20]), lambda: cache.evict(w, x.kv_len, [far]),
                 lambda: cache.evict(w, x.kv_len, [2 ** 63 - 1]), lambda: cache.evict(w, x.kv_len, [20], recent=far),
                 lambda: cache.tree_attention(x.q, x.kv_len, x.rows, layer=far),
                 lambda: cache.tree_attention(x.q, x.kv_len, x.rows, max_len=far),
                 lambda: cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, layer=-far),
                 lambda: lib.accept_sampled(p, None, [far, -far], u, n, tok)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    torch.cuda.synchronize()
    assert x.kv_len.tolist() == [40] and (w == 0).all() and n.tolist() == [-7, -7]
    with pytest.raises(lib.AS2DError):  # (what 32 bits hold goes on to the library's own checks)
        cache.tree_attention(x.q, x.kv_len, x.rows, layer=1)


def test_captured_on_torchs_current_stream(lib):
    """The step captured as torch captures its own work, results made in the graph's memory among
    it; replayed, and everything given back afterwards."""
    args = together_inputs(8)
    x, w, logits, cand, ks, u, keep = args
    inputs = (x.k, x.v, x.kv_len, w)
    first = [t.clone() for t in inputs]
    cache = lib.Cache(x.k, x.v)

    def step():
        lse = torch.empty(x.q.shape[:2], device="cuda")
        out = cache.tree_attention(x.q, x.kv_len, x.rows, x.visible, lse=lse)
        cache.attention_weights(x.q, lse, w, x.kv_len, x.rows, x.visible)
        cache.evict(w, x.kv_len, keep, recent=4)
        p = lib.token_probs(logits, 0.9)
        n, tok = (torch.empty(len(ks), dtype=torch.int32, device="cuda") for _ in range(2))
        lib.accept_sampled(p, cand, ks, u, n, tok)
        return out, lse, p, n, tok
    want = [t.clone() for t in step() + inputs]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        made = step()
    for _ in range(3):
        for t, f in zip(inputs, first):
            t.copy_(f)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(made + inputs, want))
    torch.cuda.synchronize()
    del made, graph, cache
    torch.cuda.empty_cache()
    again = lib.Cache(x.k, x.v)
    for t, f in zip(inputs, first):
        t.copy_(f)
    assert torch.equal(again.tree_attention(x.q, x.kv_len, x.rows, x.visible), want[0])


def test_accept_largest_and_smallest_weights(lib):
    """Weights whose total 32 bits do not hold give no token; the smallest ones do."""
    p = np.zeros((1, 4000), dtype=np.float32)
    p[0, [5, 9, 3990]] = 3e38
    assert run_accept(lib, p, None, [], [0], [0.5]) == ([0], [-1])
    p[0, [9, 3990]] = 0.0
    assert run_accept(lib, p, None, [], [0], [0.5]) == ([0], [5])
    p[0, 5] = 0.0
    p[0, [3, 3990]] = 1e-44
    for u, want in ((0.0, 3), (0.25, 3), (0.75, 3990), (1 - 2.0 ** -24, 3990)):
        assert run_accept(lib, p, None, [], [0], [u]) == ([0], [want])
