"""The operators on a verification state: trees of candidates, sampled acceptance,
tracked weights and eviction, against the oracle and a 64-bit forward pass."""
import math

import numpy as np
import pytest
import torch

import oracle
from synth import device as D
from synth import workloads as W
from tests import operator_reference as ref
from tests.helpers import LOGIT_TOL, MARGIN_SURE, Pair, run_gpu_block, sharp_root

pytestmark = pytest.mark.gpu

L0, CAP = 200, 256


@pytest.fixture(scope="module")
def pair():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return Pair(W.TINY, seed=0)


@pytest.fixture(scope="module")
def sharp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return Pair(W.TINY, seed=0, gains="sharp")


@pytest.fixture(scope="module")
def sharp_text(sharp):
    root, cont, _ = sharp_root(sharp.oracle, lambda: sharp.oracle_cache(L0, CAP), L0, 9)
    return root, [int(t) for t in cont]


def ints(values):
    return torch.tensor(list(values) or [0], dtype=torch.int32, device="cuda")


def run_tree(st, cfg, cands, parents, want_logits=True):
    ks = [len(c) for c in cands]
    rows, batch = sum(ks) + len(ks), len(ks)
    n, corr = (torch.full((batch,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    greedy = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    path = torch.full((batch, 16), -7, dtype=torch.int32, device="cuda")
    logits = torch.empty((rows, cfg.vocab), dtype=torch.float32, device="cuda") if want_logits else None
    st.verify_tree(ints(t for c in cands for t in c), ints(t for p in parents for t in p), ks, n, corr, greedy,
                   logits, path)
    torch.cuda.synchronize()
    return (n.tolist(), corr.tolist(), greedy.cpu().numpy(), logits.cpu().numpy() if want_logits else None,
            path.tolist())


def ancestors(parents, i):
    """Rows from below the root down to row i."""
    out = []
    while i > 0:
        out.append(i)
        i = parents[i - 1]
    return out[::-1]


def check_tree_logits(p, req, length, root, cand, parents, logits, greedy):
    for i in range(len(cand) + 1):
        chain = [cand[j - 1] for j in ancestors(parents, i)]
        want = p.oracle.verify_block(p.oracle_cache(length, CAP, req=req), length, root, chain)
        assert np.abs(want["logits"][-1] - logits[i]).max() <= LOGIT_TOL
        if want["margin"][-1] > MARGIN_SURE:
            assert greedy[i] == want["greedy"][-1]


@pytest.mark.parametrize("k", [1, 3, 8, 16])
def test_tree_logits(pair, k):
    """Each row's logits are those of its path decoded one token after another."""
    rng = np.random.default_rng(k)
    cfg = pair.cfg
    cand = [int(t) for t in rng.integers(0, cfg.vocab, k)]
    parents = [int(rng.integers(0, i + 1)) for i in range(k)]
    root = int(W.root_tokens(cfg, 1, 0)[0])
    st = pair.state([L0], CAP, [root])
    n, corr, greedy, logits, path = run_tree(st, cfg, [cand], [parents])
    st.check()
    check_tree_logits(pair, 0, L0, root, cand, parents, logits, greedy)
    ln, rt = st.read_state()
    assert ln == [L0 + n[0] + 1] and rt == corr and corr[0] == greedy[path[0][n[0] - 1] if n[0] else 0]
    st.close()


def test_tree_ragged_batch(pair):
    """Requests of several prefixes, widths and shapes in one call; one with no
    candidates; and a second call on what the first left."""
    rng = np.random.default_rng(7)
    cfg, lens = pair.cfg, [1, 200, 130, 0]
    roots = [int(t) for t in W.root_tokens(cfg, 4, 3)]
    st = pair.state(lens, CAP, roots)
    cands = [[int(t) for t in rng.integers(0, cfg.vocab, k)] for k in (5, 16, 0, 9)]
    parents = [[int(rng.integers(0, i + 1)) for i in range(len(c))] for c in cands]
    n, corr, greedy, logits, path = run_tree(st, cfg, cands, parents)
    st.check()
    r = 0
    for b, (cand, par) in enumerate(zip(cands, parents)):
        check_tree_logits(pair, b, lens[b], roots[b], cand, par, logits[r:r + len(cand) + 1], greedy[r:])
        r += len(cand) + 1
    ln, rt = st.read_state()
    assert ln == [a + m + 1 for a, m in zip(lens, n)] and rt == corr
    n2, corr2, _, logits2, _ = run_tree(st, cfg, [[], [3], [], [5]], [[], [0], [], [0]])
    for b, row in ((0, 0), (1, 1), (2, 3), (3, 4)):
        oc = pair.oracle_cache(lens[b], CAP, req=b)
        done = pair.oracle.verify_block(oc, lens[b], roots[b], [cands[b][j - 1] for j in path[b] if j > 0])
        want = pair.oracle.verify_block(oc, lens[b] + len([j for j in path[b] if j > 0]) + 1, corr[b], [])
        assert done["n_accepted"] >= 0
        assert np.abs(want["logits"][0] - logits2[row]).max() <= LOGIT_TOL
    st.close()


TREES = [
    # (candidates: c1.. of the greedy text by number, 0 a wrong token), parents, accepted path
    ([0, 1, 0, 2, 0, 3], [0, 0, 1, 2, 2, 4], [2, 4, 6]),
    ([1, 2, 3, 4], [0, 1, 2, 3], [1, 2, 3, 4]),                 # a chain, all right
    ([0, 0, 0], [0, 0, 0], []),                                   # nothing right
    ([2, 1, 0], [0, 0, 2], [2]),                                  # right token, wrong place
    ([1, 1, 2, 2], [0, 0, 1, 2], [1, 3]),                         # twice the same: the first
    ([0] * 11 + [1, 2, 3, 4, 5], [0] * 11 + [0, 12, 13, 14, 15], [12, 13, 14, 15, 16]),
    ([], [], []),
]


@pytest.mark.parametrize("tree", range(len(TREES)))
def test_tree_acceptance(sharp, sharp_text, tree):
    """The path that the greedy text takes is accepted, exactly, and its entries
    lie where a chain of them would have put them."""
    numbers, parents, want = TREES[tree]
    cfg, (root, cont) = sharp.cfg, sharp_text
    wrong = next(t for t in range(cfg.vocab) if t not in cont)
    cand = [cont[j - 1] if j else wrong for j in numbers]
    st = sharp.state([L0], CAP, [root])
    n, corr, _, _, path = run_tree(st, cfg, [cand], [parents], want_logits=False)
    st.check()
    assert n == [len(want)] and corr == [cont[len(want)]]
    assert path == [want + [-1] * (16 - len(want))]
    ln, rt = st.read_state()
    assert ln == [L0 + len(want) + 1] and rt == corr
    # the cache against a chain's: entries off by the order of 32-bit sums, which
    # may turn a rounding to bf16 by one step of 2^-7
    chain = sharp.state([L0], CAP, [root])
    run_gpu_block(chain, cfg, [[cont[j] for j in range(len(want))]])
    for a, b in ((st.kc, chain.kc), (st.vc, chain.vc)):
        a, b = (t[..., L0:L0 + len(want) + 1, :].double() for t in (a, b))
        assert ((a - b).abs() <= b.abs() * 2.0 ** -7 + 2.0 ** -12).all()
        assert torch.isnan(st.kc[..., L0 + len(cand) + 1:, :].float()).all()
    # and the next call goes on with the text
    n2, corr2, _, _ = run_gpu_block(st, cfg, [[cont[len(want) + 1]]], want_logits=False)
    assert list(n2) == [1] and list(corr2) == [cont[len(want) + 2]]
    st.close()
    chain.close()


def test_tree_bad_parents(sharp, sharp_text):
    """A parent that is no earlier row drops its request and no other."""
    cfg, (root, cont) = sharp.cfg, sharp_text
    import paper_2609_37617_gb300 as lib
    for bad in ([0, 2, 1], [0, 1, 3], [-1, 0, 0], [0, 2 ** 31 - 1, 0], [1, 0, 0]):
        st = sharp.state([L0, L0], CAP, [root, root])
        kc, vc = D.device_kv(cfg, [L0], CAP, 0)
        st.kc[:, 1], st.vc[:, 1] = kc[:, 0], vc[:, 0]  # twice request 0's prefix
        n, corr, _, _, path = run_tree(st, cfg, [cont[:3], cont[:3]], [bad, [0, 1, 2]], want_logits=False)
        assert n == [-1, 3] and corr == [-1, cont[3]]
        assert path[0] == [-1] * 16 and path[1][:4] == [1, 2, 3, -1]
        with pytest.raises(lib.AS2DError, match="parent"):
            st.check()
        assert st.read_state() == ([L0, L0 + 4], [root, cont[3]])
        st.close()


def test_tree_refusals(pair):
    import paper_2609_37617_gb300 as lib
    st = pair.state([L0], L0 + 3, [1])
    n = ints([0])
    c = ints([1, 2, 3])
    out = lib.make_verify_out(n.data_ptr(), n.data_ptr())
    import ctypes
    call = lambda cand, par, k: lib._lib.as2d_verify_tree(  # noqa: E731
        st.handle, cand, par, lib._i32_array(k), ctypes.byref(out), None, None)
    assert call(c.data_ptr(), None, [1]) == lib.AS2D_ERR_INVALID_ARG
    assert call(None, c.data_ptr(), [1]) == lib.AS2D_ERR_INVALID_ARG
    assert call(c.data_ptr(), c.data_ptr(), [3]) == lib.AS2D_ERR_CAPACITY
    assert call(c.data_ptr(), c.data_ptr(), [17]) == lib.AS2D_ERR_INVALID_ARG
    assert call(c.data_ptr(), c.data_ptr(), [-1]) == lib.AS2D_ERR_INVALID_ARG
    assert st.read_state() == ([L0], [1])
    w = torch.zeros(st.kc.shape[:4], device="cuda")
    with pytest.raises(lib.AS2DError):
        st.evict([5])  # nothing tracked
    st.track_weights(w)
    with pytest.raises(lib.AS2DError):
        st.evict([-1])
    with pytest.raises(lib.AS2DError):
        st.evict([5], recent=-1)
    with pytest.raises(ValueError):
        st.evict([5, 5])
    with pytest.raises(lib.AS2DError):
        st.prefill(ints([1]))
    st.track_weights(None)
    st.prefill(ints([1]))
    st.check()
    probs, u = torch.empty((2, pair.cfg.vocab), device="cuda"), torch.zeros(2, device="cuda")
    for t in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(lib.AS2DError):
            st.verify_sampled(c, [1], u, t, probs, n, n)
    st.close()


# ---- sampled acceptance ------------------------------------------------------------

@pytest.mark.parametrize("with_draft", [False, True])
def test_sampled(pair, with_draft):
    """The rows' probabilities, n and the token that the rule gives on them in 64
    bits; the state moves on accordingly."""
    cfg, T = pair.cfg, 0.25
    lens, ks = [200, 31, 130], [4, 0, 7]
    rng = np.random.default_rng(1 + with_draft)
    roots = [int(t) for t in W.root_tokens(cfg, 3, 3)]
    total = sum(ks)
    for _ in range(6):
        cands = [[int(t) for t in rng.integers(0, cfg.vocab, k)] for k in ks]
        twin = pair.state(lens, CAP, roots)
        _, _, greedy, logits = run_gpu_block(twin, cfg, cands)
        p = np.exp(logits.astype(np.float64) / T)
        p /= p.sum(1, keepdims=True)
        flat = [t for c in cands for t in c]
        draft = None
        if with_draft:  # flat but for some mass at the candidate
            draft = rng.random((total, cfg.vocab)) + 0.1
            draft /= draft.sum(1, keepdims=True)
            draft = draft.astype(np.float32)
        u = rng.random(total + 3).astype(np.float32)
        r = 0
        for k in ks:  # most tests pass, so that paths of every length occur
            u[r:r + k] *= 2e-3 if not with_draft else 1.0
            r += k + 1
        probs = torch.empty((total + 3, cfg.vocab), device="cuda")
        n, corr = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
        g = torch.zeros(total + 3, dtype=torch.int32, device="cuda")
        st = pair.state(lens, CAP, roots)
        st.verify_sampled(ints(flat), ks, torch.from_numpy(u).cuda(), T, probs, n, corr,
                          draft_probs=None if draft is None else torch.from_numpy(draft).cuda(), greedy=g)
        st.check()
        assert np.abs(probs.cpu().numpy() - p).max() <= p.max() * 2.0 ** -15
        assert np.array_equal(g.cpu().numpy(), greedy)
        # exactly the rule on the probabilities that the call returns
        want = ref.accept(probs.double().cpu().numpy(), None if draft is None else draft.astype(np.float64), flat, ks,
                          u.astype(np.float64))
        assert (n.tolist(), corr.tolist()) == want
        assert st.read_state() == ([a + m + 1 for a, m in zip(lens, n.tolist())], corr.tolist())
        # the next call starts from the drawn tokens
        n2, _, _, l2 = run_gpu_block(st, cfg, [[], [], []])
        for b in range(3):
            oc = pair.oracle_cache(lens[b], CAP, req=b)
            m = n.tolist()[b]
            for i, t in enumerate([roots[b]] + cands[b][:m] + [corr.tolist()[b]]):
                w = pair.oracle.decode_step(oc, lens[b] + i, t)
            assert np.abs(w - l2[b]).max() <= LOGIT_TOL
        st.close()
        twin.close()


def test_sampled_without_a_token(pair):
    """NaN in a request's cache makes its rows' logits NaN: it is dropped with a
    device error, the other request goes on."""
    import paper_2609_37617_gb300 as lib
    st = pair.state([L0, 50], CAP, [1, 2])
    st.vc[:, 0, :, 3] = math.nan
    probs, u = torch.empty((3, pair.cfg.vocab), device="cuda"), torch.full((3,), 0.5, device="cuda")
    n, corr = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
    st.verify_sampled(ints([5]), [1, 0], u, 1.0, probs, n, corr)
    with pytest.raises(lib.AS2DError, match="no token"):
        st.check()
    assert n.tolist() == [-1, 0] and corr.tolist()[0] == -1 and corr.tolist()[1] >= 0
    ln, rt = st.read_state()
    assert ln == [L0, 51] and rt == [1, corr.tolist()[1]]
    st.close()


# ---- tracked weights and eviction ----------------------------------------------------

def forward(p, k, v, entries, pos, token):
    """Logits of one token at position pos over the first `entries` cache places of
    one request (k, v [layers][n_kv][cap][d] in double), in 64 bits; also each
    layer's attention weight of those places and its own, [layers][n_kv][entries + 1]."""
    cfg = p.cfg
    w = {n: t.double() for n, t in D.device_weights(cfg, p.seed, p.gains).items()}
    d, half, G = cfg.head_dim, cfg.head_dim // 2, cfg.n_q // cfg.n_kv
    ang = pos * cfg.rope_theta ** (-2.0 * torch.arange(half, device="cuda").double() / d)

    def norm(x, g):
        return x * torch.rsqrt(x.square().mean() + cfg.rms_eps) * g

    def rot(x):
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)
    x, gathered = w["embed"][token], []
    for layer in range(cfg.n_layers):
        y = norm(x, w[f"attn_norm.{layer}"])
        q = rot((w[f"w_q.{layer}"] @ y).view(cfg.n_q, d)).view(cfg.n_kv, G, d)
        kn = rot((w[f"w_k.{layer}"] @ y).view(cfg.n_kv, 1, d)).bfloat16().double()
        vn = (w[f"w_v.{layer}"] @ y).view(cfg.n_kv, 1, d).bfloat16().double()
        ks, vs = torch.cat([k[layer, :, :entries], kn], 1), torch.cat([v[layer, :, :entries], vn], 1)
        pr = (q @ ks.transpose(1, 2) / math.sqrt(d)).softmax(-1)
        gathered.append(pr.sum(1))
        x = x + w[f"w_o.{layer}"] @ (pr @ vs).reshape(-1)
        y = norm(x, w[f"mlp_norm.{layer}"])
        x = x + w[f"w_down.{layer}"] @ (torch.nn.functional.silu(w[f"w_gate.{layer}"] @ y) * (w[f"w_up.{layer}"] @ y))
    return w["lm_head"] @ norm(x, w["final_norm"]), torch.stack(gathered)


def test_tracked_weights(pair):
    """A decode step's weights in every layer, added to what was there; a block's
    weights sum to its rows; entries that fall away leave theirs behind."""
    cfg = pair.cfg
    lens, roots = [130, 0], [5, 6]
    st = pair.state(lens, CAP, roots)
    w0 = torch.rand(st.kc.shape[:4], device="cuda")
    w = w0.clone()
    st.track_weights(w)
    _, _, _, logits = run_gpu_block(st, cfg, [[], []])
    st.check()
    for b in range(2):
        n = lens[b]
        kd, vd = st.kc[:, b].double(), st.vc[:, b].double()
        want_logits, want = forward(pair, kd, vd, n, n, roots[b])
        assert (want_logits - torch.from_numpy(logits[b]).cuda()).abs().max() <= LOGIT_TOL
        # queries and keys of layers behind the first carry the pass's 2^-16-ish
        # errors, and keys round to bf16 (2^-8 of a score's own part): entries of
        # the prefix are off by some 2^-10 of their weight at most
        got = w[:, b].double()
        assert ((got[..., :n] - w0[:, b, :, :n] - want[..., :n]).abs() <= want[..., :n] * 2.0 ** -10 + 2.0 ** -22).all()
        assert ((got[..., n] - want[..., n]).abs() <= want[..., n] * 2.0 ** -5 + 2.0 ** -22).all()
        assert torch.equal(w[:, b, :, n + 1:], w0[:, b, :, n + 1:])
    before = w.clone()
    run_tree(st, cfg, [[1, 2, 3], [4]], [[0, 0, 1], [0]], want_logits=False)
    for b, rows in ((0, 4), (1, 2)):
        n = lens[b] + 1
        gained = (w[:, b, :, :n] - before[:, b, :, :n]).sum(-1) + w[:, b, :, n:n + rows].sum(-1)
        # (accepted entries may have moved up over rejected ones)
        if st.read_state()[0][b] == n + 1:
            assert ((gained - 2 * rows).abs() <= 2 * rows * 2.0 ** -12).all()
    st.close()


def test_tree_weights_move(sharp, sharp_text):
    """The accepted entries' weights move with them."""
    cfg, (root, cont) = sharp.cfg, sharp_text
    wrong = next(t for t in range(cfg.vocab) if t not in cont)
    tree = [wrong, cont[0], wrong, cont[1]]
    st, chain = sharp.state([L0], CAP, [root]), sharp.state([L0], CAP, [root])
    w, wc = (torch.zeros(st.kc.shape[:4], device="cuda") for _ in range(2))
    st.track_weights(w)
    chain.track_weights(wc)
    run_tree(st, cfg, [tree], [[0, 0, 2, 2]], want_logits=False)
    run_gpu_block(chain, cfg, [[cont[0], cont[1]]], want_logits=False)
    assert st.read_state() == chain.read_state()
    a, b = w[..., L0:L0 + 3], wc[..., L0:L0 + 3]
    # the chain's rows' weights of these entries, less what the tree's wrong rows add
    # to the root's and the first's: the last accepted one is seen by itself alone
    assert ((a[..., 2] - b[..., 2]).abs() <= b[..., 2] * 2.0 ** -6 + 2.0 ** -20).all()
    assert (a[..., :2] >= b[..., :2] * (1 - 2.0 ** -6)).all()
    st.close()
    chain.close()


def test_evict_and_go_on(pair):
    """Eviction by tracked weights leaves what the rule says in every layer, and
    the next tokens stand at their true positions over the entries that are left."""
    cfg = pair.cfg
    lens, roots = [200, 77, 10], [5, 6, 7]
    st = pair.state(lens, CAP, roots)
    w = torch.rand(st.kc.shape[:4], device="cuda")
    st.track_weights(w)
    run_gpu_block(st, cfg, [[1, 2], [], [3]], want_logits=False)
    held, _ = st.read_state()
    bits = lambda t: t.view(torch.int16).cpu().numpy().copy()  # noqa: E731
    hk, hv, hw = bits(st.kc), bits(st.vc), w.cpu().numpy().copy()
    keep = [120, 40, 50]
    new = ref.evict(hk, hv, hw, held, keep, 8)
    assert new[2] == held[2] and new[0] == 120
    st.evict(keep, recent=8)
    st.check()
    ln, rt = st.read_state()
    assert ln == new
    assert np.array_equal(bits(st.kc), hk) and np.array_equal(bits(st.vc), hv) and np.array_equal(w.cpu().numpy(), hw)
    for step in range(2):  # a decode step, then one on top of it
        _, corr, _, logits = run_gpu_block(st, cfg, [[], [], []])
        for b in range(3):
            want, _ = forward(pair, st.kc[:, b].double(), st.vc[:, b].double(), ln[b], held[b] + step, rt[b])
            assert (want - torch.from_numpy(logits[b]).cuda()).abs().max() <= LOGIT_TOL
        ln2, rt = st.read_state()
        assert ln2 == [n + 1 for n in ln] and rt == list(corr)
        ln = ln2
    # back to what the eviction left, and no further
    import paper_2609_37617_gb300 as lib
    st.rollback([120, 40, ln[2]], rt)
    st.check()
    st.rollback([119, 40, 0], rt)
    with pytest.raises(lib.AS2DError, match="eviction"):
        st.check()
    assert st.read_state()[0] == [120, 40, 0]
    _, _, _, logits = run_gpu_block(st, cfg, [[], [], []])
    want, _ = forward(pair, st.kc[:, 0].double(), st.vc[:, 0].double(), 120, held[0], rt[0])
    assert (want - torch.from_numpy(logits[0]).cuda()).abs().max() <= LOGIT_TOL
    st.close()


def test_evict_again_and_past_the_table(pair):
    """Evictions add up: positions go beyond the capacity."""
    cfg = pair.cfg
    cap = 64
    st = pair.state([40], cap, [5])
    w = torch.rand(st.kc.shape[:4], device="cuda")
    st.track_weights(w)
    pos, root = 40, 5
    for _ in range(6):
        run_gpu_block(st, cfg, [[1] * 16], want_logits=False)
        ln, _ = st.read_state()
        pos += ln[0] - 40
        st.evict([40], recent=4)
        ln, rt = st.read_state()
        assert ln == [40]
    for _ in range(20):
        (n, c, _, logits) = run_gpu_block(st, cfg, [[]])
        want, _ = forward(pair, st.kc[:, 0].double(), st.vc[:, 0].double(), 40, pos, rt[0])
        assert (want - torch.from_numpy(logits[0]).cuda()).abs().max() <= LOGIT_TOL
        pos += 1
        st.evict([40], recent=4)
        ln, rt = st.read_state()
    assert pos > cap
    st.check()
    st.close()


def test_state_graph(sharp, sharp_text):
    """A tree call and an eviction captured on first use and replayed."""
    cfg, (root, cont) = sharp.cfg, sharp_text
    wrong = next(t for t in range(cfg.vocab) if t not in cont)
    st = sharp.state([L0], CAP, [root])
    k0, v0 = st.kc.clone(), st.vc.clone()
    w = torch.zeros(st.kc.shape[:4], device="cuda")
    st.track_weights(w)
    cand, par = ints([wrong, cont[0], cont[1]]), ints([0, 0, 2])
    n, corr = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.zeros((1, 16), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        st.verify_tree(cand, par, [3], n, corr, path=path, stream=s.cuda_stream)
    for _ in range(2):
        st.kc.copy_(k0)
        st.vc.copy_(v0)
        st.rollback([L0], [root], stream=s.cuda_stream)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        st.check()
        assert n.tolist() == [2] and corr.tolist() == [cont[2]] and path.tolist()[0][:3] == [2, 3, -1]
        assert st.read_state() == ([L0 + 3], [cont[2]])
    st.close()


def test_an_eviction_that_is_captured_has_not_run(pair):
    """Calls between the capture of an eviction and its first replay see every entry."""
    cfg = pair.cfg
    st = pair.state([L0], CAP, [5])
    w = torch.rand(st.kc.shape[:4], device="cuda")
    st.track_weights(w)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        st.evict([20], recent=4, stream=s.cuda_stream)
    st.track_weights(None)
    _, corr, _, logits = run_gpu_block(st, cfg, [[]])
    want, _ = forward(pair, st.kc[:, 0].double(), st.vc[:, 0].double(), L0, L0, 5)
    assert (want - torch.from_numpy(logits[0]).cuda()).abs().max() <= LOGIT_TOL
    g.replay()
    torch.cuda.synchronize()
    assert st.read_state() == ([20], list(corr))
    _, _, _, logits = run_gpu_block(st, cfg, [[]])
    want, _ = forward(pair, st.kc[:, 0].double(), st.vc[:, 0].double(), 20, L0 + 1, corr[0])
    assert (want - torch.from_numpy(logits[0]).cuda()).abs().max() <= LOGIT_TOL
    st.check()
    st.close()


def test_prefill_after_an_eviction(pair):
    """Tokens prefilled over what an eviction left stand at their true positions: what
    decode steps over them give."""
    cfg = pair.cfg
    tokens = [5, 9, 2, 11, 7, 3, 8]
    caches = []
    for whole in (True, False):
        st = pair.state([L0], CAP, [5])
        w = torch.linspace(0, 1, CAP, device="cuda").expand(st.kc.shape[:4]).contiguous()
        st.track_weights(w)
        st.evict([90], recent=4)
        st.track_weights(None)
        first = ints([0])
        if whole:
            with pytest.raises(Exception, match="tracked|track|refused|weights"):
                st.track_weights(w)
                st.prefill(ints(tokens), first)
            st.track_weights(None)
            st.prefill(ints(tokens), first)
        else:
            for i, t in enumerate(tokens):
                st.rollback([90 + i], [t])
                _, corr, _, logits = run_gpu_block(st, cfg, [[]])
                want, _ = forward(pair, st.kc[:, 0].double(), st.vc[:, 0].double(), 90 + i, L0 + i, t)
                assert (want - torch.from_numpy(logits[0]).cuda()).abs().max() <= LOGIT_TOL
            margin = np.sort(logits[0].ravel())[-1] - np.sort(logits[0].ravel())[-2]
        st.check()
        ln, rt = st.read_state()
        assert ln == [90 + len(tokens)]
        caches.append((st, st.kc[:, 0, :, 90:ln[0]].float(), st.vc[:, 0, :, 90:ln[0]].float(), rt))
    (a, ka, va, ra), (b, kb, vb, rb) = caches
    # (the bar of prefilled entries against the decode steps' elsewhere)
    assert (ka - kb).abs().max() <= 3e-2 and (va - vb).abs().max() <= 3e-2
    if margin > MARGIN_SURE:
        assert ra == rb
    a.close()
    b.close()


@pytest.mark.parametrize("length,cap", [(L0, CAP), (3000, 3100), (8000, 8100)])
def test_waits_that_run_out(pair, length, cap):
    """A wait limit of 0 in the attention of trees and the gathered weights: the call
    comes to an end and is flagged, and with the limit restored the next one gives
    what it gives on a fresh state.  (One CTA to an item, a cluster, even shares.)"""
    import paper_2609_37617_gb300 as lib
    cfg, cand, parents = pair.cfg, [1, 2, 3, 4], [0, 0, 1, 2]
    fresh, st = (pair.state([length], cap, [5]) for _ in range(2))
    w0, w1 = (torch.zeros(st.kc.shape[:4], device="cuda") for _ in range(2))
    fresh.track_weights(w0)
    want = run_tree(fresh, cfg, [cand], [parents])
    k0, v0 = st.kc.clone(), st.vc.clone()
    st.track_weights(w1)
    st.set_wait_limit(0)
    for _ in range(3):
        run_tree(st, cfg, [cand], [parents], want_logits=False)
        st.rollback([length], [5])
    torch.cuda.synchronize()
    with pytest.raises(lib.AS2DError, match="timed out"):
        st.check()
    st.check()
    st.set_wait_limit(2_000_000_000)
    st.rollback([length], [5])
    for t, old in ((st.kc, k0), (st.vc, v0)):
        t.copy_(old)
    w1.zero_()
    torch.cuda.synchronize()
    got = run_tree(st, cfg, [cand], [parents])
    st.check()
    assert got[0] == want[0] and got[1] == want[1] and np.array_equal(got[3], want[3]) and torch.equal(w0, w1)
    st.close()
    fresh.close()


def test_a_state_without_the_operators_is_as_before(pair):
    """Calls before, between and after calls along trees give the same bits."""
    cfg = pair.cfg
    a, b = (pair.state([L0], CAP, [9]) for _ in range(2))
    one = run_gpu_block(a, cfg, [[1, 2, 3]])
    run_tree(b, cfg, [[1, 2]], [[0, 0]], want_logits=False)
    b.rollback([L0], [9])
    two = run_gpu_block(b, cfg, [[1, 2, 3]])
    assert all(np.array_equal(x, y) for x, y in zip(one, two))
    a.close()
    b.close()


@pytest.mark.parametrize("captured", [False, True])
def test_a_rollback_refused_below_an_eviction_changes_nothing(pair, captured):
    """The calls right after it see every entry that is there (several chunks of the
    chain's attention), whether the eviction was enqueued or captured and replayed."""
    import paper_2609_37617_gb300 as lib
    cfg, length, cap, keep = pair.cfg, 4000, 4200, 2600
    results = []
    for refused in (False, True):
        st = pair.state([length, 30], cap, [5, 6])
        w = torch.linspace(0, 1, cap, device="cuda").expand(st.kc.shape[:4]).contiguous()
        st.track_weights(w)
        if captured:
            s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=s):
                st.evict([keep, 100], recent=4, stream=s.cuda_stream)
            g.replay()
            torch.cuda.synchronize()
        else:
            st.evict([keep, 100], recent=4)
        st.track_weights(None)
        if refused:
            st.rollback([100, 30], [7, 6])
        calls = [run_gpu_block(st, cfg, [[1, 2], [3]]), run_gpu_block(st, cfg, [[], [4]])]
        if refused:
            with pytest.raises(lib.AS2DError, match="eviction"):
                st.check()
        st.check()
        ln, rt = st.read_state()
        # what is left can be rolled back to, and gone on from
        st.rollback([keep, 30], [8, 9])
        calls.append(run_gpu_block(st, cfg, [[1], []]))
        st.check()
        assert st.read_state()[0] == [keep + 1 + int(calls[-1][0][0]), 31]
        results.append((ln, rt, calls))
        st.close()
    (ln, rt, calls), (ln2, rt2, calls2) = results
    assert ln == ln2 and rt == rt2 and ln[0] > keep
    for a, b in zip(calls, calls2):
        assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_a_dropped_request_leaves_its_tracked_weights(pair):
    """A bad parent, or a token outside the vocabulary, drops a request before its rows'
    weights are gathered; the other requests' are those of a call without it."""
    import paper_2609_37617_gb300 as lib
    cfg, lens = pair.cfg, [150, 200, 30]
    w0 = torch.rand((cfg.n_layers, 3, cfg.n_kv, CAP), device="cuda")
    results = []
    for cand, parents, match in (([1, 2], [0, 1], None), ([1, 2], [2, 1], "parent"), ([1, cfg.vocab], [0, 1], "vocab"),
                                 ([-1, 2], [0, 1], "vocab")):
        st = pair.state(lens, CAP, [5, 6, 7])
        w = w0.clone()
        st.track_weights(w)
        n, _, _, _, _ = run_tree(st, cfg, [cand, [3, 4, 5], []], [parents, [0, 0, 1], []], want_logits=False)
        if match:
            with pytest.raises(lib.AS2DError, match=match):
                st.check()
            assert n[0] == -1 and torch.equal(w[:, 0], w0[:, 0])
        else:
            st.check()
            assert not torch.equal(w[:, 0, :, :lens[0]], w0[:, 0, :, :lens[0]])
        results.append(w[:, 1:])
        st.close()
    # (the others' sums may come in another order where the work is cut elsewhere)
    for w in results[1:]:
        assert ((w - results[0]).abs() <= results[0].abs() * 2.0 ** -9 + 2.0 ** -20).all()


def test_launches_are_counted(pair):
    """A pass along a tree counts one kernel more a layer where the attention's parts are
    joined by a second one (long prefixes), none where it is not."""
    import paper_2609_37617_gb300 as lib
    cfg, counts = pair.cfg, []
    for length, cap in ((L0, CAP), (3000, 3100), (8000, 8100)):
        st = pair.state([length], cap, [5])
        lib.as2d_kv_profile_read(st.handle)
        run_tree(st, cfg, [[1, 2, 3]], [[0, 0, 1]], want_logits=False)
        counts.append(lib.as2d_kv_profile_read(st.handle)[3])
        st.check()
        st.close()
    assert counts[0] == counts[1] == counts[2] - cfg.n_layers


def test_addresses_off_their_types(pair):
    """Refused on the host, with nothing enqueued or changed."""
    import ctypes
    import paper_2609_37617_gb300 as lib
    st = pair.state([L0], CAP, [1])
    n, c = ints([0]), ints([1, 2, 3])
    f = torch.zeros((4, pair.cfg.vocab), device="cuda")
    out, k = lib.make_verify_out(n.data_ptr(), n.data_ptr()), lib._i32_array([2])
    tree = lambda par, path: lib._lib.as2d_verify_tree(  # noqa: E731
        st.handle, c.data_ptr(), par, k, ctypes.byref(out), path, None)
    sampled = lambda q, u, p: lib._lib.as2d_verify_sampled(  # noqa: E731
        st.handle, c.data_ptr(), k, q, u, 1.0, ctypes.byref(out), p, None)
    at = f.data_ptr()
    for off in (1, 2, 3):
        for status in (tree(c.data_ptr() + off, None), tree(c.data_ptr(), n.data_ptr() + off), sampled(at + off, at, at),
                       sampled(None, at + off, at), sampled(None, at, at + off),
                       lib._lib.as2d_kv_track_weights(st.handle, at + off)):
            assert status == lib.AS2D_ERR_INVALID_ARG and "aligned" in lib.as2d_last_error()
    st.check()
    assert st.read_state() == ([L0], [1])
    st.close()


def test_counts_of_a_state(pair):
    """One count to each request, of 32 bits."""
    st = pair.state([L0, 30], CAP, [1, 2])
    st.track_weights(torch.zeros(st.kc.shape[:4], device="cuda"))
    n, c = ints([0, 0]), ints([1, 2, 3])
    probs, u = torch.empty((4, pair.cfg.vocab), device="cuda"), torch.zeros(4, device="cuda")
    for k in ([1], [1, 1, 1], [2 ** 32 + 1, 1], [1, 2 ** 32]):
        for call in (lambda: st.verify_tree(c, ints([0, 0, 0]), k, n, n), lambda: st.evict(k),
                     lambda: st.verify_sampled(c, k, u, 1.0, probs, n, n)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        st.evict([20, 20], recent=2 ** 32)
    st.check()
    assert st.read_state() == ([L0, 30], [1, 2])
    st.close()


def test_tensors_of_a_state(pair):
    """Tensors of another type, device or layout, or too few elements, are refused before the call."""
    st, V = pair.state([L0, 30], CAP, [1, 2]), pair.cfg.vocab
    z = lambda *s, t=torch.int32, d="cuda": torch.zeros(s, dtype=t, device=d)  # noqa: E731
    f = torch.float32

    def tree(**kw):
        a = dict(candidates=z(3), parents=z(3), k=[2, 1], n_accepted=z(2), correction=z(2), greedy=z(5),
                 logits=z(5, V, t=f), path=z(2, 16))
        a.update(kw)
        st.verify_tree(**a)

    def sampled(**kw):
        a = dict(candidates=z(3), k=[2, 1], u=z(5, t=f), temperature=1.0, probs=z(5, V, t=f), n_accepted=z(2),
                 correction=z(2), draft_probs=z(3, V, t=f), greedy=z(5))
        a.update(kw)
        st.verify_sampled(**a)
    both = [("candidates", 3), ("n_accepted", 2), ("correction", 2), ("greedy", 5)]
    for call, names in ((tree, both + [("parents", 3), ("path", 32)]), (sampled, both)):
        for name, n in names:
            for bad in (z(n - 1), z(n, d="cpu"), z(n, t=torch.int64), z(2 * n)[::2]):
                with pytest.raises((ValueError, TypeError), match=name):
                    call(**{name: bad})
    for call, names in ((tree, [("logits", 5 * V)]), (sampled, [("u", 5), ("probs", 5 * V), ("draft_probs", 3 * V)]),
                        (lambda weights: st.track_weights(weights), [("weights", st.kc[..., 0].numel())])):
        for name, n in names:
            for bad in (z(n - 1, t=f), z(n, t=f, d="cpu"), z(n, t=torch.float64), z(n, t=torch.bfloat16), z(2 * n, t=f)[::2]):
                with pytest.raises((ValueError, TypeError), match=name):
                    call(**{name: bad})
    st.check()
    assert st.read_state() == ([L0, 30], [1, 2])
    tree()
    sampled()
    st.check()
    st.close()


def test_sampled_drops_a_bad_token(pair):
    """A candidate outside the vocabulary drops its request, its tracked weights as they were;
    the other goes on by the rule."""
    import paper_2609_37617_gb300 as lib
    cfg = pair.cfg
    for bad in (cfg.vocab, -1, 2 ** 31 - 1):
        st = pair.state([L0, 50], CAP, [1, 2])
        w0 = torch.rand(st.kc.shape[:4], device="cuda")
        w = w0.clone()
        st.track_weights(w)
        probs, u = torch.empty((5, cfg.vocab), device="cuda"), torch.full((5,), 0.5, device="cuda")
        n, corr = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
        st.verify_sampled(ints([5, bad, 9]), [2, 1], u, 0.5, probs, n, corr)
        with pytest.raises(lib.AS2DError, match="vocab"):
            st.check()
        want = ref.accept(probs[3:].double().cpu().numpy(), None, [9], [1], [0.5, 0.5])
        assert n.tolist() == [-1] + want[0] and corr.tolist() == [-1] + want[1]
        assert st.read_state() == ([L0, 51 + want[0][0]], [1, want[1][0]])
        assert torch.equal(w[:, 0], w0[:, 0]) and not torch.equal(w[:, 1, :, :50], w0[:, 1, :, :50])
        st.close()


def test_a_rollback_after_an_eviction_of_nothing(pair):
    """An eviction that is to keep more than there is sets no floor: the host's bound follows a
    rollback below it, so that the capacity is there to be used again."""
    cfg = pair.cfg
    st = pair.state([L0], CAP, [5])
    st.track_weights(torch.zeros(st.kc.shape[:4], device="cuda"))
    st.evict([240], recent=4)
    st.track_weights(None)
    st.rollback([10], [7])
    for _ in range(14):  # 14 calls of 17 rows at most: 248 places, where 56 are left behind L0
        run_gpu_block(st, cfg, [[1] * 16], want_logits=False)
    st.check()
    assert 24 <= st.read_state()[0][0] <= 248
    st.close()
