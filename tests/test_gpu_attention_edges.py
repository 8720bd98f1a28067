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
