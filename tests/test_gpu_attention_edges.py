"""Attention of prompts, of trees and over caches in 4 bits where a row's maximum is none, far above its
first one, or beyond 32 bits, beside other rows that this must not change."""
import math

import pytest
import torch

from tests import cache4_reference as ref
from tests import operator_reference as trees
from tests import test_gpu_new_rows as rows_of
from tests import test_gpu_operators as operators

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_37617_gb300 as p
    return p


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# ---- prompts: rows without a reference beside rows whose reference moves ------------

def jumping(lens, rows):
    """A prompt's scores that rise by 300 and by 20 along the keys: dim 5 of the queries is 1, that of the
    keys the level."""
    x = rows_of.Prompt((28, 4, 128), [lens], [rows])
    n = lens + rows
    x.q *= 0.1
    x.q[..., 5] = 1.0
    x.k[0, 0, :, :n // 3, 5] = 0.0
    x.k[0, 0, :, n // 3:2 * n // 3, 5] = 300.0
    x.k[0, 0, :, 2 * n // 3:n, 5] = 320.0
    x.scale = 1.0
    return x


@pytest.mark.parametrize("lens,rows", [(0, 1300), (6000, 40)])
def test_prompt_references_jump_beside_nan(lib, lens, rows):
    """NaN queries, which never get a reference, change no other row, of their warp (32 queries of
    neighbouring rows) or not."""
    x = jumping(lens, rows)
    base, base_lse = rows_of.prompt(lib, x)
    rows_of.check(x, base, base_lse, p_rel=rows_of.P_REL)
    at = [(0, 3), (rows // 2, 9), (rows - 2, 0), (rows - 1, 27)]
    for value in (math.nan, math.inf):
        for i, h in at:
            x.q[i, h, 100] = value
        out, lse = rows_of.prompt(lib, x)
        for i, h in at:
            assert torch.isnan(out[i, h]).all() and torch.isnan(lse[i, h])
            out[i, h], lse[i, h] = base[i, h], base_lse[i, h]
        assert same(out, base) and same(lse, base_lse)


@pytest.mark.parametrize("lens,rows", [(0, 1300), (6000, 40)])
def test_prompt_references_jump_after_nothing(lib, lens, rows):
    """Rows whose first 200 scores are -inf get their first reference late, beside a row that is NaN from
    the first on; the rows' result is that of the entries after those."""
    x = jumping(lens, rows)
    x.k[0, 0, :, :200, 64] = math.inf
    x.q[..., 64] = -1.0
    base, base_lse = rows_of.prompt(lib, x)

    def request(b, layer=0):
        q, k, v, seen = rows_of.Prompt.request(x, b, layer)
        k, seen = k.clone(), seen.clone()
        k[:, :200, 64] = 0.0
        seen[:, :200] = False
        return q, k, v, seen
    x.request = request
    rows_of.check(x, base, base_lse, p_rel=rows_of.P_REL)
    i, h = rows - 2, 9
    x.q[i, h, 100] = math.nan
    out, lse = rows_of.prompt(lib, x)
    assert torch.isnan(out[i, h]).all() and torch.isnan(lse[i, h])
    out[i, h], lse[i, h] = base[i, h], base_lse[i, h]
    assert same(out, base) and same(lse, base_lse)


# ---- scores far from 1, and beyond 32 bits -----------------------------------------

SIZES = (2.0 ** 18, 2.0 ** 24, 2.0 ** 28, 2.0 ** 34, 2.0 ** 60, 2.0 ** 120)


def check_far(x, out, lse, p_rel):
    """Where one score of a row is so far above the others that no rounding of sums (d products, each
    addition off by 2^-23 of their magnitudes) can change that, the row is that entry's value, to its weight's
    rounding p_rel."""
    r0 = clear = 0
    for b, r in enumerate(x.rows):
        if not r:
            continue
        q, k, v, seen = x.request(b)
        G = q.shape[1] // k.shape[0]
        half_step = torch.finfo(out.dtype).eps / 2
        for h in range(q.shape[1]):
            s = (q[:, h] @ k[h // G].T * x.scale).masked_fill(~seen.to(q.device), -math.inf)
            off = (q[:, h].abs() @ k[h // G].abs().T * x.scale).amax(-1) * q.shape[2] * 2.0 ** -22
            top, at = s.topk(2, -1)
            got, got_lse = out[r0:r0 + r, h].double(), lse[r0:r0 + r, h].double()
            assert torch.isfinite(got).all() and torch.isfinite(got_lse).all()
            assert ((got_lse - top[:, 0]).abs() <= off + math.log(s.shape[1])).all()
            # (the others' weights together below 2^-30)
            won = top[:, 0] - top[:, 1] > 2 * off + 21 + math.log(s.shape[1])
            want = v[h // G][at[:, 0]]
            over = (got - want).abs() - want.abs() * (half_step * (1 + 2.0 ** -6) + p_rel) - v.abs().max() * 2.0 ** -20
            assert not won.any() or over[won].max() <= 0, float(over[won].max())
            clear += int(won.sum())
        r0 += r
    assert clear * 2 > sum(x.rows) * q.shape[1]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("lens,rows", [(0, 700), (6000, 40)])
def test_prompt_scores_far(lib, lens, rows, size):
    x = rows_of.Prompt((28, 4, 128), [lens], [rows])
    x.scale = size
    check_far(x, *rows_of.prompt(lib, x), rows_of.P_REL)


@pytest.mark.parametrize("lens,rows", [(0, 1300), (300, 200), (6000, 40)])
def test_prompt_scores_beyond_32_bits(lib, lens, rows):
    """Finite queries and keys whose product is finite and whose score is not: +inf makes the row NaN, -inf
    is a weight of 0; in the first key tile and in a later one."""
    for at in (3, lens + rows // 2 - 20):
        x = rows_of.Prompt((28, 4, 128), [lens], [rows])
        x.scale = 2.0
        x.k[0, 0, :, at, 7] = 2.0 ** 64
        base, base_lse = rows_of.prompt(lib, x)
        assert torch.isfinite(base).all() and torch.isfinite(base_lse).all()
        i, h = rows - 1, 9
        x.q[i, h] = 0
        x.q[i, h, 7] = 2.0 ** 63
        out, lse = rows_of.prompt(lib, x)
        assert torch.isnan(out[i, h]).all() and torch.isnan(lse[i, h])
        out[i, h], lse[i, h] = base[i, h], base_lse[i, h]
        assert same(out, base) and same(lse, base_lse)
        x.q[i, h, 7] = -2.0 ** 63
        out, lse = rows_of.prompt(lib, x)
        assert torch.isfinite(out[i, h]).all() and torch.isfinite(lse[i, h])


def next_to_each_other(x, n):
    """Scores 3 2^60 + j 2^38, and from the second key tile on the next one in 32 bits, with a j at which the
    scale (1, in base 2) rounds both to the same number.  (Sums of products no larger than half of
    them, so that none of their bits are cut off.)"""
    c = torch.tensor(1.0) * 1.4426950408889634
    j = next(j for j in range(128) if len({float(torch.tensor(3 * 2.0 ** 60 + i * 2.0 ** 38) * c) for i in (j, j + 1)}) == 1)
    x.q.zero_()
    x.q[..., :4], x.q[..., 4:6] = 1.5 * 2.0 ** 29, 2.0 ** 18
    k = x.k[0, 0, :, :n]
    k.zero_()
    k[..., :4], k[..., 4], k[:, 128:, 5] = 2.0 ** 30, j * 2.0 ** 20, 2.0 ** 20


def check_next_to_each_other(x, out, lse):
    """Results are means of what the rows see, whichever of the two scores' entries they are of."""
    _, _, v, seen = x.request(0)
    G = out.shape[1] // v.shape[0]
    for g in range(v.shape[0]):
        for i in range(len(out)):
            values = v[g][seen[i].to(v.device)]
            low, high = values.amin(0), values.amax(0)
            got, room = out[i, g * G:(g + 1) * G].double(), 2.0 ** -7 * values.abs().amax(0)
            assert ((got >= low - room) & (got <= high + room)).all()
    assert ((lse.double() / (3 * 2.0 ** 60) - 1).abs() < 2.0 ** -15).all()


@pytest.mark.parametrize("lens,rows", [(0, 300), (6000, 40)])
def test_prompt_scores_next_to_each_other(lib, lens, rows):
    x = rows_of.Prompt((28, 4, 128), [lens], [rows])
    next_to_each_other(x, lens + rows)
    x.scale = 1.0
    check_next_to_each_other(x, *rows_of.prompt(lib, x))


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
def test_attention4_scores_far(lib, q_type, size):
    """Few queries together, many (in a large cache), and many cut between CTAs."""
    for kind, lens, rows in ((rows_of.Inputs, [400], [5]), (rows_of.Roomy, [400], [19]),
                             (rows_of.Inputs, [5000, 40], [64, 3])):
        x = kind((28, 4, 128), lens, rows, trees.chain_masks(rows), q_type)
        x.scale = size
        check_far(x, *rows_of.attend4(lib, x), 2.0 ** -11)


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,length,large", [((4, 2, 64), 400, False), ((28, 4, 128), 400, False),
                                                ((28, 4, 128), 400, True), ((8, 8, 64), 400, True)])
def test_attention4_scores_beyond_32_bits(lib, heads, length, large, q_type):
    """Over a cache in 4 bits a finite query with scores of +inf gives NaN, whether few queries are taken
    together or (in a large cache) many."""
    rows = 19 if large else 5
    x = (rows_of.Roomy if large else rows_of.Inputs)(heads, [length], [rows], trees.chain_masks([rows]), q_type)
    x.scale = 1.0
    base, base_lse = rows_of.attend4(lib, x)
    i, h = rows - 2, 3
    for at in (0, 3):  # (3: four times as large as other dims)
        x.q[i, h] = 0
        x.q[i, h, at] = 1.5 * 2.0 ** 127
        out, lse = rows_of.attend4(lib, x)
        assert torch.isnan(out[i, h]).all() and torch.isnan(lse[i, h])
        out[i, h], lse[i, h] = base[i, h], base_lse[i, h]
        assert same(out, base) and same(lse, base_lse)


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,lens,rows,jump", [((4, 2, 64), [200], [1], 128), ((4, 2, 64), [200], [5], 128),
                                                  ((28, 4, 128), [900] * 16, [19] * 16, 512)])
@pytest.mark.parametrize("level,more", [(0, 64), (2 ** 10, 64), (2 ** 24, 64), (-2 ** 24, 4)])
def test_attention4_weights_at_their_limit(lib, heads, lens, rows, jump, q_type, level, more):
    """Scores (base 2, exact) that rise by just 8 from one of a warp's key tiles to a later one, which a
    weight's range has room for: beside references that are rounded too.  Few queries together, and many."""
    x = rows_of.Inputs(heads, lens, rows, trees.chain_masks(rows), q_type)
    n = lens[0] + rows[0]
    k = torch.zeros((n, heads[2]), dtype=torch.float64, device="cuda")
    k[:, 0] = k[:, 16] = k[jump:, 32] = 4.0
    k[:, 1] = k[:, 17] = k[:, 33] = 7.0  # (the scales: 1)
    for c, packed in zip(x.c4[:2], ref.pack(k)):
        c[0, :, :, :n] = packed
    x.q.zero_()
    x.q[..., 0], x.q[..., 16], x.q[..., 32] = level / 4, more / 4, 2.0
    x.scale = math.log(2.0)
    out, lse = rows_of.attend4(lib, x)
    half_step = torch.finfo(q_type).eps / 2
    for b in range(len(lens)):
        sl = slice(x.starts[b], x.starts[b + 1])
        _, _, v, seen = x.request(b)
        w = torch.where(torch.arange(n, device="cuda") < jump, 1.0, 256.0).double() * seen.to("cuda")
        want = torch.einsum("it,gtd->igd", w / w.sum(-1, keepdim=True), v).repeat_interleave(heads[0] // heads[1], 1)
        # (a weight's rounding; the scale's base 2 is 1 to 2^-23, of scores that differ by 8)
        room = want.abs() * half_step * (1 + 2.0 ** -6) + v.abs().max() * 2.0 ** -10
        assert ((out[sl].double() - want).abs() <= room).all()
        want_lse = (level + more + w.sum(-1).log2()) * math.log(2.0)
        assert ((lse[sl].double() - want_lse[:, None]).abs() <= want_lse[:, None].abs() * 2.0 ** -21 + 2.0 ** -12).all()


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", SIZES)
def test_tree_attention_scores_far(lib, size, q_type):
    """The same over a cache in bf16: items done whole, by clusters and by even shares.  (32-bit queries
    enter the products to 2^-17 of themselves.)"""
    for lens, rows in (([200], [5]), ([3000], [5]), ([5000, 40], [64, 3])):
        x = operators.Inputs((28, 4, 128), lens, rows, trees.chain_masks(rows), q_type)
        x.scale = size
        check_far(x, *operators.run_attention(lib, x, scale=size), 2.0 ** -16)


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("length", [300, 3000])
def test_tree_attention_scores_next_to_each_other(lib, length, q_type):
    x = operators.Inputs((28, 4, 128), [length], [5], trees.chain_masks([5]), q_type)
    next_to_each_other(x, length + 5)
    check_next_to_each_other(x, *operators.run_attention(lib, x, scale=1.0))


@pytest.mark.parametrize("q_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("length", [200, 3000, 15128])
def test_tree_attention_scores_beyond_32_bits(lib, length, q_type):
    """The same over a cache in bf16: items done whole, by clusters and by even shares."""
    lens, rows = ([length], [5]) if length < 15128 else ([length, 40], [64, 3])
    x = operators.Inputs((28, 4, 128), lens, rows, trees.chain_masks(rows), q_type)
    for at in (3, length + 1):
        kept = x.k[0, 0, :, at, 7].clone()
        x.k[0, 0, :, at, 7] = 2.0 ** 64
        x.q[3, 9] = 1.0
        base, base_lse = operators.run_attention(lib, x, scale=2.0)
        assert torch.isfinite(base).all() and torch.isfinite(base_lse).all()
        x.q[3, 9] = 0
        x.q[3, 9, 7] = 2.0 ** 63
        out, lse = operators.run_attention(lib, x, scale=2.0)
        assert torch.isnan(out[3, 9]).all() and torch.isnan(lse[3, 9])
        out[3, 9], lse[3, 9] = base[3, 9], base_lse[3, 9]
        assert same(out, base) and same(lse, base_lse)
        x.k[0, 0, :, at, 7] = kept


# ---- requests without rows --------------------------------------------------------

@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31])
def test_lengths_of_requests_without_rows(lib, bad):
    """The length of a request that has no rows in a call is not looked at: nothing is flagged."""
    x = rows_of.Prompt((4, 2, 64), [100, 20, 7], [60, 0, 5])
    base, base_lse = rows_of.prompt(lib, x)
    t = rows_of.Inputs((4, 2, 64), [100, 20, 7], [6, 0, 5], trees.chain_masks([6, 0, 5]))
    base4, base4_lse = rows_of.attend4(lib, t)
    x.kv_len[1] = t.kv_len[1] = bad
    err = rows_of.ints([0])
    out, lse = rows_of.prompt(lib, x, error_bits=err)
    assert err.item() == 0 and same(out, base) and same(lse, base_lse)
    out, lse = rows_of.attend4(lib, t, error_bits=err)
    assert err.item() == 0 and same(out, base4) and same(lse, base4_lse)
    cache = lib.Cache(x.k, x.v)
    cache.tree_attention(x.q[:11].contiguous(), x.kv_len, [6, 0, 5], error_bits=err)
    new = torch.randn((11, 8, 64), device="cuda").bfloat16()
    cache.append(new[:, :4], new[:, 4:6], new[:, 6:], x.kv_len, [6, 0, 5], error_bits=err)
    lib.Cache4(*t.c4).append(new[:, :4], new[:, 4:6], new[:, 6:], t.kv_len, [6, 0, 5], error_bits=err)
    assert err.item() == 0
