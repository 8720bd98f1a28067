"""The operators between a projection and its attention against their 64-bit forms:
rows appended to caches in bf16 and in 4 bits, caches packed and read back, attention over
caches in 4 bits and of whole prompts, and a run of them together."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from tests import cache4_reference as ref
from tests import operator_reference as trees

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (28, 4, 128), (8, 8, 64), (16, 1, 128), (12, 2, 128)]


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_37617_gb300 as p
    return p


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- rows appended ---------------------------------------------------------------

class Rows:
    """Rows of a fused projection and where they go."""

    def __init__(self, heads, lens, rows, dtype, norm=True, rotary=None, seed=0, room=37, layers=2, spread=1.0):
        nq, nkv, d = heads
        g = generator(seed)
        self.heads, self.lens, self.rows = heads, lens, rows
        self.rotary = d if rotary is None else rotary
        x = torch.randn(sum(rows), nq + 2 * nkv, d, generator=g, device="cuda") * spread
        x *= torch.randn(nq + 2 * nkv, 1, generator=g, device="cuda").exp()
        self.q, self.k, self.v = x.to(dtype).split([nq, nkv, nkv], dim=1)
        self.gains = [1 + 0.3 * torch.randn(d, generator=g, device="cuda") if norm else None for _ in range(2)]
        self.kv_len = ints(lens)
        self.shape = (layers, len(lens), nkv, max(n + r for n, r in zip(lens, rows)) + room, d)
        self.place = ints([n + i for n, r in zip(lens, rows) for i in range(r)])
        self.of = [b for b, r in enumerate(rows) for _ in range(r)]
        self.call = dict(q_norm=self.gains[0], k_norm=self.gains[1], rotary=self.rotary, eps=1e-5, theta=10000.0)

    def want(self, positions=None):
        at = self.place if positions is None else positions
        eps = float(np.float32(1e-5))
        return [ref.finish(x, g, at, self.rotary, eps, 10000.0) for x, g in zip((self.q, self.k), self.gains)]

    def packed(self, fill=0x5A):
        d = self.shape[4]
        return [torch.full((*self.shape[:4], w), fill, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 16) * 2]


SETS = [([0], [1]), ([200], [5]), ([0, 7, 300, 12], [33, 0, 1, 300]), ([4000] * 3, [64, 2, 700])]


def check_queries(x, out, want):
    y, mag = want
    half_step = torch.finfo(out.dtype).eps / 2
    over = (out.double() - y).abs() - (y.abs() * half_step * (1 + 2.0 ** -6) + mag * ref.FINISH)
    assert over.max() <= 0, float(over.max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens,rows", SETS)
@pytest.mark.parametrize("norm,part", [(True, 1.0), (False, 0.5), (True, 0)])
def test_append(lib, heads, lens, rows, dtype, norm, part):
    x = Rows(heads, lens, rows, dtype, norm, int(part * heads[2]) // 32 * 32)
    k, v = (torch.full(x.shape, 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = lib.Cache(k, v).append(x.q, x.k, x.v, x.kv_len, rows, layer=1, **x.call)
    torch.cuda.synchronize()
    want_q, want_k = x.want()
    check_queries(x, out, want_q)
    at = x.place.long()
    check_queries(x, k[1, x.of, :, at], want_k)
    assert torch.equal(v[1, x.of, :, at], x.v.bfloat16())
    for c in (k, v):  # nothing else is written
        c[1, x.of, :, at] = 3.0
        assert (c == 3.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens,rows", SETS)
@pytest.mark.parametrize("norm,part", [(True, 1.0), (False, 0.5), (False, 0)])
def test_append4(lib, heads, lens, rows, dtype, norm, part):
    """Codes and scales are those of the exact values, every one of them."""
    x = Rows(heads, lens, rows, dtype, norm, int(part * heads[2]) // 32 * 32, seed=len(rows))
    c4 = x.packed()
    err = ints([0])
    out = lib.Cache4(*c4).append(x.q, x.k, x.v, x.kv_len, rows, layer=1, error_bits=err, **x.call)
    torch.cuda.synchronize()
    want_q, want_k = x.want()
    check_queries(x, out, want_q)
    assert err.item() == 0
    at = x.place.long()
    for y, codes, scales in ((want_k[0], *c4[:2]), (x.v.double(), *c4[2:])):
        want = ref.pack(y)
        assert torch.equal(scales[1, x.of, :, at], want[1])
        assert torch.equal(codes[1, x.of, :, at], want[0])
    for c in c4:
        c[1, x.of, :, at] = 0x5A
        assert (c == 0x5A).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append4_many(lib, dtype):
    """Enough rows that values next to a border are among them (some 10 of a million)."""
    x = Rows((4, 2, 128), [0], [20000], dtype, layers=1, seed=3)
    c4 = x.packed()
    lib.Cache4(*c4).append(x.q, x.k, x.v, x.kv_len, x.rows, **x.call)
    at = x.place.long()
    for y, codes, scales in ((x.want()[1][0], *c4[:2]), (x.v.double(), *c4[2:])):
        want = ref.pack(y)
        assert torch.equal(scales[0, x.of, :, at], want[1])
        assert torch.equal(codes[0, x.of, :, at], want[0])


def test_positions(lib):
    """Positions of the caller's: far ones, negative ones, the same twice."""
    for d in (64, 128):
        x = Rows((4, 2, d), [5], [6], torch.float32, False)
        pos = ints([0, 1, 2 ** 31 - 1, -1, -2 ** 31, 1])
        k, v = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        out = lib.Cache(k, v).append(x.q, x.k, x.v, x.kv_len, x.rows, positions=pos, **x.call)
        # (angles of 2^31 in 64 bits: the frequency's rounding turns them by 2^31 2^-52)
        y, mag = x.want(pos)[0]
        assert ((out.double() - y).abs() <= mag * (ref.FINISH + 2.0 ** -19)).all()
        assert torch.equal(out[0], x.q[0]) and not torch.equal(out[1], out[5])


def test_append_skips(lib):
    """A length that leaves no room: flagged, nothing written; the other request goes on."""
    x = Rows((4, 2, 64), [3, 9], [5, 4], torch.bfloat16, room=0, layers=1)
    for bad in (-1, x.shape[3] - 4, 2 ** 31 - 1, -2 ** 31):
        x.kv_len[0] = bad
        k, v = (torch.full(x.shape, 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        c4, err = x.packed(), ints([0])
        out = torch.full(x.q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
        lib.Cache(k, v).append(x.q, x.k, x.v, x.kv_len, x.rows, out=out, error_bits=err, **x.call)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY
        assert (k[:, 0] == 3).all() and (v[:, 0] == 3).all() and (out[:5] == 3).all()
        assert torch.equal(v[0, 1, :, 9:13].transpose(0, 1), x.v[5:]) and not (out[5:] == 3).all()
        err.zero_()
        lib.Cache4(*c4).append(x.q, x.k, x.v, x.kv_len, x.rows, error_bits=err, **x.call)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY and all((c[:, 0] == 0x5A).all() for c in c4)


def test_append4_not_finite(lib):
    for value in (math.nan, math.inf, -math.inf):
        x = Rows((4, 2, 64), [3], [4], torch.float32, False, 0)
        x.v[2, 1, 20] = value
        c4, err = x.packed(), ints([0])
        lib.Cache4(*c4).append(x.q, x.k, x.v, x.kv_len, x.rows, error_bits=err, **x.call)
        assert err.item() == lib.AS2D_DEVERR_NOT_FINITE
        want = ref.pack(x.v.double())
        for c, w in zip(c4[2:], want):
            assert torch.equal(c[0, x.of, :, x.place.long()], w)
        got = ref.unpack(*want)[2, 1, 20].item()
        assert got == (0 if math.isnan(value) else math.copysign(7 * 896, value))


# ---- a cache packed and read back ----------------------------------------------------

def caches(lib, shape, seed=0, cap4=None):
    k, v = (torch.randn(shape, generator=generator(seed + i), device="cuda").bfloat16() for i in range(2))
    c4 = [torch.full((*shape[:3], cap4 or shape[3], w), 0x5A, dtype=torch.uint8, device="cuda")
          for w in (shape[4] // 2, shape[4] // 16) * 2]
    return k, v, c4


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,start", [([1], None), ([300], [299]), ([0, 17, 1000, 64], None),
                                        ([5, 17, 1000, 64], [5, 0, 333, 70])])
def test_write_and_read(lib, d, lens, start):
    shape = (3, len(lens), 2, max(lens) + 3, d)
    k, v, c4 = caches(lib, shape, cap4=max(lens) + 8)
    back = [torch.full(shape, 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache4, end = lib.Cache4(*c4), ints(lens)
    first = None if start is None else ints(start)
    err = ints([0])
    for layer, most in ((1, 0), (None, max(lens))):
        for c in c4:
            c.fill_(0x5A)
        cache4.write(lib.Cache(k, v), end, first, layer, most, err)
        cache4.read(lib.Cache(*back), end, first, layer, 1, err)
        assert err.item() == 0
        for x, y, codes, scales in ((k, back[0], *c4[:2]), (v, back[1], *c4[2:])):
            want = ref.pack(x)
            for i in range(shape[0]):
                for b, n in enumerate(lens):
                    s = 0 if start is None else min(start[b], n)
                    if layer is None or i == layer:
                        assert torch.equal(codes[i, b, :, s:n], want[0][i, b, :, s:n])
                        assert torch.equal(scales[i, b, :, s:n], want[1][i, b, :, s:n])
                        assert torch.equal(y[i, b, :, s:n].double(), ref.unpack(*(w[i, b, :, s:n] for w in want)))
                    else:
                        s = n
                        assert (codes[i, b] == 0x5A).all()
                    assert (codes[i, b, :, n:] == 0x5A).all() and (scales[i, b, :, :s] == 0x5A).all()
                    assert (y[i, b, :, n:] == 3).all() and (y[i, b, :, :s] == 3).all()


def test_every_byte_reads(lib):
    """All scales and codes, those that nothing writes among them."""
    scales = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 1, 1, 32, 8).contiguous()
    codes = torch.randint(0, 256, (1, 1, 1, 32, 64), generator=generator(1), device="cuda").to(torch.uint8)
    k, v = (torch.zeros((1, 1, 1, 32, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.Cache4(codes, scales, codes, scales).read(lib.Cache(k, v), ints([32]))
    want = ref.unpack(codes, scales)
    assert torch.equal(k.double(), want) and torch.equal(v.double(), want) and torch.isfinite(want).all()


def test_values_at_the_edges(lib):
    """Zeros, the smallest and largest numbers, scales between two of them, values between
    two codes, NaN and infinities."""
    rows = [torch.zeros(16, dtype=torch.float64)]
    for most in (2.0 ** -133, 2.0 ** -20, 7 * 2.0 ** -18, 7 * 2.0 ** -17, 2.0 ** -13, 1.0, 7.0, 6272.0, 7000.0, 70000.0, 3e38):
        rows.append(torch.linspace(-most, most, 16, dtype=torch.float64))
    for s in (1.0, 1.0625, 1.1875, 2.0 ** -15 * 1.25, 864.0):  # sevenths on a border
        rows.append(torch.linspace(-7 * s, 7 * s, 16, dtype=torch.float64))
    rows.append(torch.arange(-7.5, 8.5, dtype=torch.float64).clamp(-7, 7))  # codes on a border
    for bad in (math.nan, math.inf, -math.inf):
        row = torch.linspace(-1, 1, 16, dtype=torch.float64)
        row[5] = bad
        rows.append(row)
    x = torch.stack(rows).bfloat16().cuda()
    x = torch.cat([x, x.new_zeros((-len(x)) % 4, 16)]).view(1, 1, 1, -1, 64)
    c4 = [torch.zeros((*x.shape[:4], w), dtype=torch.uint8, device="cuda") for w in (32, 4, 32, 4)]
    err = ints([0])
    lib.Cache4(*c4).write(lib.Cache(x.contiguous(), x.clone()), ints([x.shape[3]]), error_bits=err)
    want = ref.pack(x)
    assert err.item() == lib.AS2D_DEVERR_NOT_FINITE
    for i in (0, 2):
        assert torch.equal(c4[i + 1], want[1]) and torch.equal(c4[i], want[0])


def test_write_skips(lib):
    k, v, c4 = caches(lib, (1, 2, 2, 20, 64))
    for start, end in (([-1, 0], [5, 3]), ([0, 0], [21, 3]), ([3, 0], [2 ** 31 - 1, 3])):
        for c in c4:
            c.fill_(0x5A)
        err = ints([0])
        lib.Cache4(*c4).write(lib.Cache(k, v), ints(end), ints(start), error_bits=err)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY
        assert all((c[:, 0] == 0x5A).all() for c in c4) and torch.equal(c4[0][0, 1, :, :3], ref.pack(k)[0][0, 1, :, :3])


# ---- attention over a cache in 4 bits ------------------------------------------------

class Inputs:
    """A cache in 4 bits whose places past each request's entries hold any bytes, and
    rows over it."""

    def __init__(self, heads, lens, rows, masks, q_type=torch.bfloat16, seed=0, room=37, layers=1, spread=1.5, pad=0):
        nq, nkv, d = heads
        g = generator(seed)
        self.heads, self.lens, self.rows, self.masks = heads, lens, rows, masks
        cap = max(n + r for n, r in zip(lens, rows)) + room
        shape = (layers, len(lens), nkv, cap)
        self.c4 = []
        for _ in range(2):
            x = torch.randn((*shape, d), generator=g, device="cuda")
            x[..., 3::16] *= 4
            self.c4 += list(ref.pack(x))
        for b, (n, r) in enumerate(zip(lens, rows)):
            for c in self.c4:
                c[:, b, :, n + r:] = 0xFF
        total = sum(rows)
        wide = torch.randn((total, nq + pad, d), generator=g, device="cuda") * spread
        self.q = wide.to(q_type)[:, :nq]
        self.kv_len = ints(lens)
        self.visible = trees.mask_tensor(masks) if total else None
        self.scale = d ** -0.5
        self.starts = np.cumsum([0] + list(rows))

    def request(self, b, layer=0):
        n = self.lens[b] + self.rows[b]
        k, v = (ref.unpack(*(c[layer, b, :, :n] for c in self.c4[i:i + 2])) for i in (0, 2))
        return self.q[self.starts[b]:self.starts[b + 1]].double(), k, v, trees.seen_matrix(self.lens[b], self.masks[b])


def check(x, out, lse, layer=0, p_rel=None):
    """p_rel: bf16 queries' weights are one 16-bit float, 32-bit ones' two, as the queries."""
    f32 = x.q.dtype == torch.float32
    half_step = torch.finfo(x.q.dtype).eps / 2
    for b in range(len(x.lens)):
        if not x.rows[b]:
            continue
        sl = slice(x.starts[b], x.starts[b + 1])
        want, tol, want_lse, tol_lse = ref.attention(*x.request(b, layer), x.scale, 2.0 ** -21 if f32 else 0.0,
                                                     p_rel or (2.0 ** -21 if f32 else 2.0 ** -11))
        got = out[sl].double()
        assert torch.isfinite(got).all()
        over = (got - want).abs() - (want.abs() * half_step * (1 + 2.0 ** -6) + tol)
        assert over.max() <= 0, (b, float(over.max()), float((got - want).abs().max()))
        empty = want_lse == -math.inf
        got_lse = lse[sl].double()
        assert (got_lse[empty] == -math.inf).all() and (got[empty] == 0).all()
        assert ((got_lse - want_lse)[~empty].abs() <= tol_lse[~empty]).all()


def attend4(lib, x, layer=0, **kw):
    lse = torch.full((sum(x.rows), x.heads[0]), 7.0, device="cuda")
    out = lib.Cache4(*x.c4).tree_attention(x.q, x.kv_len, x.rows, x.visible, layer=layer, scale=x.scale, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("length", [0, 1, 15, 63, 127, 128, 129, 1000])
@pytest.mark.parametrize("rows", [1, 2, 5, 64])
def test_attention4_sizes(lib, heads, length, rows, q_type):
    masks = trees.tree_masks([rows], np.random.default_rng(length + rows))
    x = Inputs(heads, [length], [rows], masks, q_type, seed=length, room=length % 5)
    check(x, *attend4(lib, x))


class Roomy(Inputs):
    """The same in a cache of 65536 entries: with no bound of the lengths, many queries are
    taken together whatever the lengths are."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        for i, c in enumerate(self.c4):
            self.c4[i] = torch.full((*c.shape[:3], 65536, c.shape[4]), 0xFF, dtype=torch.uint8, device="cuda")
            self.c4[i][:, :, :, :c.shape[3]] = c


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 8, 64), (48, 2, 128)])
@pytest.mark.parametrize("length", [0, 1, 63, 127, 128, 129, 1000])
@pytest.mark.parametrize("rows", [5, 19, 64])
def test_attention4_sizes_in_a_large_cache(lib, heads, length, rows, q_type):
    rows = max(rows, 17 * heads[1] // heads[0] + 1)
    masks = trees.tree_masks([rows], np.random.default_rng(length + rows))
    x = Roomy(heads, [length], [rows], masks, q_type, seed=length)
    many = attend4(lib, x)
    check(x, *many)
    check(x, *attend4(lib, x, max_len=max(length, 1)))


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
def test_attention4_in_a_large_cache(lib, q_type):
    """Masks, skips and what is not finite where many queries are taken together."""
    masks = [[0, 0b1, 0b11110, 0b11111, (2 ** 64 - 1) ^ 0b11111, 2 ** 64 - 1]]
    for length in (0, 130):
        x = Roomy((28, 4, 128), [length], [6], masks, q_type)
        base, base_lse = attend4(lib, x)
        check(x, base, base_lse)
        for c in x.c4:
            c[0, 0, :, length + 1] = 0xFE
        out, lse = attend4(lib, x)
        for i in (0, 1, 4):
            assert torch.equal(out[i], base[i]) and torch.equal(lse[i], base_lse[i])
    x = Roomy((28, 4, 128), [400], [5], trees.chain_masks([5]), q_type, spread=60.0)
    base, base_lse = attend4(lib, x)
    check(x, base, base_lse)
    for value in (math.nan, math.inf):
        x.q[2, 3, 7] = value
        out, lse = attend4(lib, x)
        assert torch.isnan(out[2, 3]).all() and torch.isnan(lse[2, 3])
        out[2, 3], lse[2, 3] = base[2, 3], base_lse[2, 3]
        assert torch.equal(out, base) and torch.equal(lse, base_lse)
    for bad in (65532, -1, 2 ** 31 - 1, -2 ** 31):
        x.kv_len.fill_(bad)
        out, lse, err = torch.full_like(x.q, 3.0).contiguous(), torch.full((5, 28), 3.0, device="cuda"), ints([0])
        lib.Cache4(*x.c4).tree_attention(x.q, x.kv_len, x.rows, out=out, lse=lse, error_bits=err)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY and (out == 3).all() and (lse == 3).all()


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("most", [1, 2, 64])
def test_attention4_ragged(lib, heads, q_type, most):
    lens = [0, 1, 700, 2055, 128, 64, 3333, 17]
    rows = [min(r, most) for r in (3, 0, 17, 1, 0, 64, 9, 33)]
    masks = trees.tree_masks(rows, np.random.default_rng(5))
    x = Inputs(heads, lens, rows, masks, q_type, layers=2, pad=3)
    for most in (0, 3333, 1):  # the bound of the lengths sizes the launch and nothing else
        check(x, *attend4(lib, x, layer=1, max_len=most), layer=1)


@pytest.mark.parametrize("length", [6000, 15128])
def test_attention4_long(lib, length):
    for heads, rows, q_type in (((28, 4, 128), 1, torch.bfloat16), ((28, 4, 128), 17, torch.float32),
                                ((4, 2, 64), 64, torch.bfloat16), ((4, 2, 64), 1, torch.float32)):
        x = Inputs(heads, [length], [rows], trees.chain_masks([rows]), q_type, seed=length)
        x.visible = None  # a chain
        check(x, *attend4(lib, x))


def test_attention4_most_requests(lib):
    rng = np.random.default_rng(2)
    lens = [int(t) for t in rng.integers(0, 700, 64)]
    for most in (2, 18):
        rows = [int(t) for t in rng.integers(0, most, 64)]
        x = Inputs((12, 2, 128), lens, rows, trees.tree_masks(rows, rng), torch.float32)
        check(x, *attend4(lib, x))


def test_attention4_many_heads(lib):
    """1024 query heads to a kv head."""
    x = Inputs((1024, 1, 64), [300], [3], trees.chain_masks([3]))
    check(x, *attend4(lib, x))


def test_attention4_far_offset(lib):
    """Entries whose offset in the cache passes 2^31 bytes of codes."""
    layers, cap = 140, 65536
    c4 = [torch.zeros((layers, 1, 4, cap, w), dtype=torch.uint8, device="cuda") for w in (64, 8, 64, 8)]
    assert (layers - 1) * 4 * cap * 64 > 2 ** 31
    x = Inputs((28, 4, 128), [300], [5], trees.tree_masks([5], np.random.default_rng(0)))
    for far, c in zip(c4, x.c4):
        far[-1, :, :, :305] = c[0, :, :, :305]
    lse = torch.empty((5, 28), device="cuda")
    out = lib.Cache4(*c4).tree_attention(x.q, x.kv_len, x.rows, x.visible, layer=layers - 1, lse=lse)
    check(x, out, lse)


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("length", [0, 130, 700])
def test_attention4_masks(lib, length, q_type):
    """Rows that see no row of their own request (nothing at all with no prefix), rows that
    see later rows, all rows, bits past the rows."""
    masks = [[0, 0b1, 0b11110, 0b11111, (2 ** 64 - 1) ^ 0b11111, 2 ** 64 - 1]]
    for heads in ((28, 4, 128), (4, 4, 64)):
        x = Inputs(heads, [length], [6], masks, q_type)
        check(x, *attend4(lib, x))
        # what a row does not see changes nothing for it
        base, base_lse = attend4(lib, x)
        for c in x.c4:
            c[0, 0, :, length + 1] = 0xFF  # seen by rows 2, 3 and 5
        out, lse = attend4(lib, x)
        for i in (0, 1, 4):
            assert torch.equal(out[i], base[i]) and torch.equal(lse[i], base_lse[i])


def test_attention4_skips(lib):
    """A length with no room is skipped and flagged; one that fills the cache is not."""
    x = Inputs((4, 2, 64), [251], [5], trees.chain_masks([5]), room=0)
    check(x, *attend4(lib, x))
    for most in (0, 2):
        for bad in (252, -1, 2 ** 31 - 1, -2 ** 31):
            x.kv_len.fill_(bad)
            out, lse, err = torch.full_like(x.q, 3.0).contiguous(), torch.full((5, 4), 3.0, device="cuda"), ints([0])
            lib.Cache4(*x.c4).tree_attention(x.q, x.kv_len, x.rows, out=out, lse=lse, error_bits=err, max_len=most)
            assert err.item() == lib.AS2D_DEVERR_CAPACITY and (out == 3).all() and (lse == 3).all()


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
def test_attention4_queries_of_any_size(lib, q_type):
    """Queries far from 1, with the scale that brings their scores back; scores far apart;
    zeros; queries that are not finite."""
    for heads, lens in (((4, 2, 64), [400]), ((28, 4, 128), [400]), ((28, 4, 128), [5000, 4000])):  # few, many queries
        rows = [5] * len(lens)
        for size in (2.0 ** -100, 2.0 ** -20, 2.0 ** 20, 2.0 ** 100):
            x = Inputs(heads, lens, rows, trees.chain_masks(rows), q_type, spread=size)
            x.scale = 0.125 / size
            check(x, *attend4(lib, x))
        x = Inputs(heads, lens, rows, trees.chain_masks(rows), q_type, spread=60.0)
        check(x, *attend4(lib, x))
        x.q[1] = 0
        check(x, *attend4(lib, x))
        base, base_lse = attend4(lib, x)
        for value in (math.nan, math.inf):
            x.q[2, 3, 7] = value
            out, lse = attend4(lib, x)
            assert torch.isnan(out[2, 3]).all() and torch.isnan(lse[2, 3])
            out[2, 3], lse[2, 3] = base[2, 3], base_lse[2, 3]
            assert torch.equal(out, base) and torch.equal(lse, base_lse)


# ---- prompts ---------------------------------------------------------------------

class Prompt(Inputs):
    """A cache in bf16 whose places past each request's entries hold NaN."""

    def __init__(self, heads, lens, rows, seed=0, room=37, layers=1, spread=1.5, pad=0):
        nq, nkv, d = heads
        g = generator(seed)
        self.heads, self.lens, self.rows = heads, lens, rows
        shape = (layers, len(lens), nkv, max(n + r for n, r in zip(lens, rows)) + room, d)
        self.k, self.v = (torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
        for b, (n, r) in enumerate(zip(lens, rows)):
            self.k[:, b, :, n + r:] = math.nan
            self.v[:, b, :, n + r:] = math.nan
        self.q = (torch.randn((sum(rows), nq + pad, d), generator=g, device="cuda") * spread).bfloat16()[:, :nq]
        self.kv_len, self.scale = ints(lens), d ** -0.5
        self.starts = np.cumsum([0] + list(rows))

    def request(self, b, layer=0):
        n = self.lens[b] + self.rows[b]
        return (self.q[self.starts[b]:self.starts[b + 1]].double(), self.k[layer, b, :, :n].double(),
                self.v[layer, b, :, :n].double(), ref.causal(self.lens[b], self.rows[b]))


def prompt(lib, x, layer=0, **kw):
    lse = torch.full((sum(x.rows), x.heads[0]), 7.0, device="cuda")
    out = lib.Cache(x.k, x.v).prompt_attention(x.q, x.kv_len, x.rows, layer=layer, scale=x.scale, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


P_REL = 2.0 ** -8  # the weights are one bf16 number


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("length", [0, 1, 127, 128, 700])
@pytest.mark.parametrize("rows", [1, 2, 17, 37, 128, 129, 300, 1000])
def test_prompt_sizes(lib, heads, length, rows):
    x = Prompt(heads, [length], [rows], seed=rows)
    check(x, *prompt(lib, x), p_rel=P_REL)


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (8, 8, 64)])
def test_prompt_packed(lib, heads):
    lens = [0, 5, 700, 0, 0, 1300, 128, 0]
    rows = [1, 0, 300, 517, 64, 1, 128, 33]
    x = Prompt(heads, lens, rows, layers=2, pad=2)
    for most in (0, 1300, 1):
        check(x, *prompt(lib, x, layer=1, max_len=most), layer=1, p_rel=P_REL)


@pytest.mark.parametrize("behind", [0.0, 1.0, math.nan])
@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 8, 64)])
def test_prompt_many_short(lib, heads, behind):
    """64 requests of a tile or two each, several to a CTA, with anything behind their entries."""
    rng = np.random.default_rng(9)
    lens = [int(t) for t in rng.integers(0, 200, 64) * rng.integers(0, 2, 64)]
    rows = [int(t) for t in rng.integers(0, 90, 64)]
    x = Prompt(heads, lens, rows)
    for b, (n, r) in enumerate(zip(lens, rows)):
        x.k[:, b, :, n + r:] = x.v[:, b, :, n + r:] = behind
    out, lse = prompt(lib, x)
    check(x, out, lse, p_rel=P_REL)
    for most in (0, 1, 199):
        again = prompt(lib, x, max_len=most)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_prompt_long(lib):
    x = Prompt((28, 4, 128), [0], [5000])
    check(x, *prompt(lib, x), p_rel=P_REL)
    x = Prompt((28, 4, 128), [15000], [200])
    check(x, *prompt(lib, x), p_rel=P_REL)


@pytest.mark.parametrize("heads", [(28, 4, 128), (4, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("lens,rows", [([5000], [1]), ([5000], [30]), ([15128], [70]), ([3000, 10, 0], [40, 3, 1]),
                                       ([2000], [200]), ([9000, 64], [5, 127])])
def test_prompt_few_rows_after_many(lib, heads, lens, rows):
    """Items cut along their keys and joined; short requests beside long ones."""
    x = Prompt(heads, lens, rows, seed=sum(rows))
    base, base_lse = prompt(lib, x)
    check(x, base, base_lse, p_rel=P_REL)
    check(x, *prompt(lib, x, max_len=max(lens)), p_rel=P_REL)
    check(x, *prompt(lib, x, max_len=1), p_rel=P_REL)
    # a value that is not finite among the rows' own: of the first row's entry, and of the last's
    for at in (lens[0], lens[0] + rows[0] - 1):
        kept = x.v[0, 0, 0, at, 7].clone()
        x.v[0, 0, 0, at, 7] = math.nan
        out, lse = prompt(lib, x)
        first, G = at - lens[0], heads[0] // heads[1]
        assert torch.equal(lse, base_lse) and torch.equal(out[:first], base[:first])
        assert torch.isnan(out[first:rows[0], :G, 7]).all() and torch.equal(out[rows[0]:], base[rows[0]:])
        rest = [e for e in range(heads[2]) if e != 7]
        assert torch.equal(out[..., rest], base[..., rest])
        x.v[0, 0, 0, at, 7] = kept


def test_prompt_many_heads(lib):
    x = Prompt((1024, 1, 64), [100], [90])  # more than 2^16 queries
    check(x, *prompt(lib, x), p_rel=P_REL)


def test_prompt_far_offset(lib):
    layers, cap = 66, 65536
    k = torch.zeros((layers, 1, 4, cap, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    x = Prompt((28, 4, 128), [100], [205])
    for far, c in ((k, x.k), (v, x.v)):
        far[-1, :, :, :305] = c[0, :, :, :305]
    lse = torch.empty((205, 28), device="cuda")
    out = lib.Cache(k, v).prompt_attention(x.q, x.kv_len, x.rows, layer=layers - 1, lse=lse)
    check(x, out, lse, p_rel=P_REL)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads", [(4, 4, 64), (28, 4, 128)])
def test_prompt_masked_places_do_not_matter(lib, heads, value):
    """What is not finite in entries that a row does not see changes nothing for it; rows that
    see it are not finite there."""
    for length, rows, at in ((0, 300, 150), (130, 40, 135), (300, 600, 899), (0, 130, 0), (200, 300, 100)):
        x = Prompt(heads, [length], [rows])
        base, base_lse = prompt(lib, x)
        first = max(at - length, 0)  # the first row that sees it
        kept = x.v[0, 0, :, at].clone()
        x.v[0, 0, 1, at, 5] = value
        out, lse = prompt(lib, x)
        G = heads[0] // heads[1]
        assert torch.equal(out[:first], base[:first]) and torch.equal(lse, base_lse)
        assert not torch.isfinite(out[first:, G:2 * G, 5]).any()
        rest = [e for e in range(heads[2]) if e != 5]
        assert torch.equal(out[first:, G:2 * G][..., rest], base[first:, G:2 * G][..., rest])
        assert torch.equal(out[:, 2 * G:], base[:, 2 * G:])
        x.v[0, 0, :, at] = kept
        x.k[0, 0, :, at] = math.nan
        out, lse = prompt(lib, x)
        assert torch.equal(out[:first], base[:first]) and torch.equal(lse[:first], base_lse[:first])
        assert torch.isnan(out[first:]).all() and torch.isnan(lse[first:]).all()


def test_prompt_skips(lib):
    x = Prompt((4, 2, 64), [100, 20], [60, 30], room=0)
    base, base_lse = prompt(lib, x)
    check(x, base, base_lse, p_rel=P_REL)
    for bad in (101, -1, 2 ** 31 - 1, -2 ** 31):
        x.kv_len[0] = bad
        out, lse, err = torch.full_like(base, 3.0), torch.full_like(base_lse, 3.0), ints([0])
        lib.Cache(x.k, x.v).prompt_attention(x.q, x.kv_len, x.rows, out=out, lse=lse, error_bits=err)
        assert err.item() == lib.AS2D_DEVERR_CAPACITY
        assert (out[:60] == 3).all() and (lse[:60] == 3).all() and torch.equal(out[60:], base[60:])


@pytest.mark.parametrize("lens,rows", [([50], [200]), ([0], [1500]), ([6000], [40])])
def test_prompt_queries_and_keys_not_finite(lib, lens, rows):
    """A query that is not finite makes its row NaN and no other; a key that holds infinities gives
    a score of either sign: a weight of 0, or NaN."""
    x = Prompt((28, 4, 128), lens, rows)
    base, base_lse = prompt(lib, x)
    at, kept = (rows[0] // 3, 9), x.q[rows[0] // 3, 9, 100].clone()
    for value in (math.nan, math.inf):
        x.q[at[0], at[1], 100] = value
        out, lse = prompt(lib, x)
        assert torch.isnan(out[at]).all() and torch.isnan(lse[at])
        out[at], lse[at] = base[at], base_lse[at]
        assert torch.equal(out, base) and torch.equal(lse, base_lse)
    x.q[at[0], at[1], 100] = kept
    x.k[0, 0, 1, 3, 64] = math.inf
    out, lse = prompt(lib, x)
    sees = torch.arange(rows[0], device="cuda") + lens[0] >= 3
    gone = (x.q[:, 7:14, 64] < 0) & sees[:, None]  # a score of -inf: as if the entry were not there
    # (entry 3 is the only one that is -inf: what is left is the softmax of the others)
    bad = (x.q[:, 7:14, 64] > 0) & sees[:, None]
    assert torch.isnan(out[:, 7:14][bad]).all() and torch.isnan(lse[:, 7:14][bad]).all()
    assert torch.isfinite(out[:, 7:14][gone]).all() and (lse[:, 7:14][gone] <= base_lse[:, 7:14][gone] + 1e-4).all()
    rest = [h for h in range(28) if not 7 <= h < 14]
    assert torch.equal(out[:, rest], base[:, rest])


def test_prompt_references_that_jump(lib):
    """Scores that grow along the keys, by little and by much, so that a row's reference has to follow;
    that fall; and whose first tiles are far below the others."""
    for steps in ((0.02,), (1.0,), (-0.5,), (0.0, 300.0, 0.0)):
        x = Prompt((28, 4, 128), [0], [1300])
        n, at = 1300 // len(steps), 0.0
        level = torch.empty(1300, device="cuda")
        for i, s in enumerate(steps):
            if len(steps) > 1:
                level[i * n:] = at = at + s
            else:
                level = torch.arange(1300, device="cuda") * s
        # one dim of the queries is 1, that of the keys the level: the scores move with it
        x.q[..., 5] = 1.0
        x.k[0, 0, :, :1300, 5] = level.bfloat16()
        x.scale = 1.0
        x.q[..., :5] *= 0.1
        x.q[..., 6:] *= 0.1
        check(x, *prompt(lib, x), p_rel=P_REL)


def test_prompt_extreme_scores(lib):
    x = Prompt((4, 2, 64), [50], [200], spread=60.0)
    check(x, *prompt(lib, x), p_rel=P_REL)


# ---- together --------------------------------------------------------------------

def test_a_run_of_them(lib):
    """A prompt appended and attended to, its cache packed, tokens appended and attended to in
    4 bits: each step against its 64-bit form on what the steps before left."""
    heads, rows = (28, 4, 128), [300, 64]
    cap = 331
    x = Rows(heads, [0, 0], rows, torch.bfloat16, layers=1, room=cap - 300)
    k, v = (torch.full(x.shape, math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = lib.Cache(k, v)
    q = cache.append(x.q, x.k, x.v, x.kv_len, rows, **x.call)
    p = Prompt(heads, [0, 0], rows)
    p.q, p.k, p.v = q, k, v
    check(p, *prompt(lib, p), p_rel=P_REL)
    c4 = x.packed(0xFF)
    cache4, lens = lib.Cache4(*c4), ints(rows)
    cache4.write(cache, lens)
    steps = [[1, 1], [5, 3]]
    for n in steps:
        before = lens.tolist()
        y = Rows(heads, before, n, torch.bfloat16, layers=1, seed=sum(n), room=cap - max(a + b for a, b in zip(before, n)))
        q = cache4.append(y.q, y.k, y.v, lens, n, **y.call)
        t = Inputs(heads, before, n, trees.chain_masks(n))
        t.q, t.c4, t.kv_len = q, c4, lens
        t.visible = None
        check(t, *attend4(lib, t))
        lens += ints(n)
    back = lib.Cache(torch.zeros_like(k), torch.zeros_like(v))
    cache4.read(back, lens)
    want = ref.pack(k[0, :, :, :64].double())
    assert torch.equal(back.k[0, :, :, :64].double(), ref.unpack(*want))


def test_captured_and_on_other_streams(lib):
    """Each call captured into a graph as a first call, replayed on new inputs; the same on a
    stream that is not torch's."""
    heads, n = (28, 4, 128), [3, 2]
    x = Rows(heads, [700, 90], n, torch.bfloat16, layers=1)
    p = Prompt(heads, [300, 0], [140, 200])
    t = Inputs(heads, [700, 90], n, trees.chain_masks(n))
    k, v = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c4 = x.packed(0)
    q, k_new, v_new = (u.clone() for u in (x.q, x.k, x.v))

    def calls(stream=None):
        kw = dict(x.call, stream=stream)
        cache, cache4 = lib.Cache(k, v), lib.Cache4(*c4)
        held.extend((cache, cache4))
        got = [cache.append(q, k_new, v_new, x.kv_len, n, **kw), cache4.append(q, k_new, v_new, x.kv_len, n, **kw)]
        t4, pc = lib.Cache4(*t.c4), lib.Cache(p.k, p.v)
        held.extend((t4, pc))
        got.append(t4.tree_attention(t.q, t.kv_len, n, t.visible, stream=stream))
        got.append(pc.prompt_attention(p.q, p.kv_len, p.rows, stream=stream))
        cache4.read(cache, x.kv_len + 3 if stream is None else ends, start=x.kv_len, stream=stream)
        return got + [k, v] + c4

    ends, held = x.kv_len + 3, []
    want = [y.clone() for y in calls()]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = calls()
    for u in (q, k_new, v_new):
        u.mul_(2)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    again = [y.clone() for y in got]
    now = calls()
    torch.cuda.synchronize()
    for a, b in zip(again, now):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert not torch.equal(again[0], want[0]) and torch.equal(again[2], want[2])
    other = torch.cuda.Stream()
    own = calls(other.cuda_stream)
    other.synchronize()
    for a, b in zip(again, own):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


FIRST_USE = """
import torch
import paper_2609_37617_gb300 as lib
g = torch.Generator(device="cuda").manual_seed(0)
k, v = (torch.randn((1, 2, 4, 900, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
c4 = [torch.zeros((1, 2, 4, 900, w), dtype=torch.uint8, device="cuda") for w in (64, 8, 64, 8)]
x = torch.randn((7, 36, 128), generator=g, device="cuda").bfloat16()
q, kn, vn = x.split([28, 4, 4], 1)
n = torch.tensor([600, 300], dtype=torch.int32, device="cuda")
cache, cache4 = lib.Cache(k, v), lib.Cache4(*c4)
def calls():
    cache4.write(cache, n)
    a = cache.append(q, kn, vn, n, [4, 3])
    b = cache4.append(q, kn, vn, n, [4, 3])
    return [a, b, cache.prompt_attention(a, n, [4, 3]), cache4.tree_attention(b, n, [4, 3]),
            cache4.tree_attention(b[:2].contiguous(), n, [1, 1])]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
torch.cuda.synchronize()
for a, b in zip([t.clone() for t in got], calls()):
    torch.cuda.synchronize()
    assert torch.equal(a, b) and a.abs().sum() > 0
"""


def test_first_use_under_capture(lib):
    """Kernels' attributes and the device's properties are found out on first use, also where
    that is captured."""
    subprocess.run([sys.executable, "-c", FIRST_USE], check=True, timeout=120,
                   cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_binding_refusals(lib):
    x = Rows((4, 2, 64), [3, 9], [5, 4], torch.bfloat16, layers=1)
    k, v = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache, c4 = lib.Cache(k, v), x.packed()
    cache4 = lib.Cache4(*c4)
    good = dict(q=x.q, k=x.k, v=x.v, kv_len=x.kv_len, rows=x.rows)
    for c in (cache, cache4):
        c.append(**good)
        for change, error in ((dict(q=x.q.cpu()), ValueError), (dict(k=x.k.float()), TypeError), (dict(q=x.q.half()), TypeError),
                              (dict(v=x.v[:8]), ValueError), (dict(k=x.k[:, :1]), ValueError), (dict(q=None), TypeError),
                              (dict(q=x.q[..., :32]), ValueError), (dict(v=x.v.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
                              (dict(rows=[5, 5]), ValueError), (dict(rows=[9]), ValueError), (dict(rows=[2 ** 32 + 5, 4 - 2 ** 32]), ValueError),
                              (dict(kv_len=x.kv_len.long()), TypeError), (dict(kv_len=x.kv_len[:1]), ValueError),
                              (dict(layer=2 ** 32), ValueError), (dict(layer=1), lib.AS2DError), (dict(rotary=2 ** 32), ValueError),
                              (dict(rotary=16), lib.AS2DError), (dict(q_norm=x.gains[0][:32]), ValueError),
                              (dict(k_norm=x.gains[1].double()), TypeError), (dict(positions=x.place[:3]), ValueError),
                              (dict(out=torch.empty_like(x.q, dtype=torch.float32)), TypeError),
                              (dict(theta=-1.0), lib.AS2DError), (dict(eps=math.nan, q_norm=x.gains[0]), lib.AS2DError)):
            with pytest.raises(error):
                c.append(**dict(good, **change))
    for change, error in ((dict(cache=c4), TypeError), (dict(end=x.kv_len.long()), TypeError), (dict(start=x.kv_len[:1]), ValueError),
                          (dict(layer=1), lib.AS2DError), (dict(max_entries=2 ** 31), ValueError), (dict(max_entries=-1), lib.AS2DError)):
        for f in (cache4.write, cache4.read):
            with pytest.raises(error):
                f(**dict(dict(cache=cache, end=x.kv_len), **change))
    for bad in ((c4[0], c4[1], c4[2], c4[1][..., :1]), (c4[0].int(), *c4[1:]), (c4[0][0], *c4[1:]), (c4[0].cpu(), *c4[1:])):
        with pytest.raises((TypeError, ValueError)):
            lib.Cache4(*bad)
    with pytest.raises(lib.AS2DError):
        cache.prompt_attention(x.q.float().contiguous(), x.kv_len, x.rows)
    out = torch.empty(9 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")[8:].view(9, 4, 64)  # 16 bytes off
    with pytest.raises(lib.AS2DError):
        cache.prompt_attention(x.q.contiguous(), x.kv_len, x.rows, out=out)
    torch.cuda.synchronize()


def test_results_repeat(lib):
    """The same call twice gives the same bits."""
    t = Inputs((28, 4, 128), [5000, 300, 40], [7, 1, 64], trees.chain_masks([7, 1, 64]))
    a, b = attend4(lib, t), attend4(lib, t)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    p = Prompt((28, 4, 128), [500, 0], [700, 1200])
    a, b = prompt(lib, p), prompt(lib, p)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
