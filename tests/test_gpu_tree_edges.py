"""Edges of the operators for drafted tokens, against plain 64-bit references."""
import pytest
import torch

from paper_2308_13137_amd import oq
from tests import tree_ref
from tests.test_gpu_serve import i32, rand
from tests.test_gpu_tree import chain, star
from tests.test_gpu_tree_verify import check_verify

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------ verification
@pytest.mark.parametrize("V", [300, 32000])
@pytest.mark.parametrize("gap", [17.0, 36.0, 40.0, 45.0, 60.0, 80.0])
@pytest.mark.parametrize("place", [1, 2, 4])
def test_verify_siblings_of_a_peak(V, gap, place):
    """Without replacement: all of q but 2^-24 to 2^-115 lies on one sibling's token.  Once that is rejected, what
    q has left is the sum of the others, not what a sum of all of them leaves."""
    n, g = 9, torch.Generator().manual_seed(int(gap) + V + place)
    kept = 0
    for seed in range(4):
        x = torch.randn(n, V, generator=g)
        y = x + 0.3 * torch.randn(n, V, generator=g)
        y[:, 7] += gap + 8.0
        P, Q = torch.softmax(x, 1), torch.softmax(y, 1)
        rest = Q[0].clone()
        rest[7] = 0.0
        others = torch.multinomial(rest / rest.max(), n - 2, generator=g).tolist()
        P[:, others[:place - 1]] = 0.0                       # siblings before the peak are rejected
        token = torch.tensor([0] + others[:place - 1] + [7] + others[place - 1:], dtype=torch.int32)
        u = torch.rand(n, generator=g) * (1.0, 0.5, 1.0, 0.1)[seed]
        u[place] = 0.9                                       # the peak is rejected: the target's share is a 300th
        kept += check_verify([star(n)], [0, n], token, P, Q, u, torch.rand(1, generator=g), replace=False) - 1
    assert kept > 0


@pytest.mark.parametrize("V,n", [(5, 5), (64, 40), (1003, 40), (130, 120), (20011, 128)])
def test_verify_rejected_tokens_side_by_side(V, n):
    """Long chains of rejections whose tokens are neighbours, and one of them twice."""
    g = torch.Generator().manual_seed(V)
    for first in (0, max(0, V - n)):
        Q = torch.softmax(3 * torch.randn(n, V, generator=g), 1)
        P = torch.softmax(3 * torch.randn(n, V, generator=g), 1)
        token = torch.arange(first - 1, first - 1 + n, dtype=torch.int32)
        P[:, first:first + 3 * n // 4] = 0.0                 # rejected whatever u
        for seed in range(4):
            u, un = 1.0 - torch.rand(n, generator=g) * (0.5, 1e-2, 1e-4, 1.0)[seed], torch.rand(1, generator=g)
            u = u.clamp(max=1 - 2.0 ** -24)
            check_verify([star(n)], [0, n], token, P, Q, u, un, replace=False)
            twice = token.clone()
            twice[n // 2:] = token[1:1 + n - n // 2]
            check_verify([star(n)], [0, n], twice, P, Q, u, un, replace=False)


@pytest.mark.parametrize("V", [40, 5000])
def test_verify_siblings_of_a_token_that_is_not_finite(V):
    """A rejected token's probability that is NaN, or infinite in the draft: nothing is drawn, and no sibling is
    kept."""
    n, g = 4, torch.Generator().manual_seed(V)
    P, Q = (torch.softmax(torch.randn(n, V, generator=g), 1) for _ in range(2))
    un, parent, start = torch.full((1,), 0.5, device="cuda"), i32(star(n)), i32([0, n])
    for token in ([0, 9, 3, 4], [0, V - 1, 9, 7]):
        bad = token[1]
        for p, q in ((float("nan"), None), (None, float("nan")), (None, float("inf"))):
            a, b = P.clone(), Q.clone()
            if p is not None:
                a[0, bad] = p
            if q is not None:
                b[0, bad] = q
            for replace in (False, True):
                path, count, nxt = oq.tree_verify(i32(token), parent, start, n, a.cuda(),
                                                  torch.tensor([0, 0.9, 0.0, 0.0], device="cuda"), un, Q=b.cuda(),
                                                  replace=replace)
                assert count.item() == 1 and nxt.item() == -1, (token, p, q, replace)


# ------------------------------------------------------------------ probabilities
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [4, 1003, 70001])
def test_probs_of_differences_that_pass_fp32(V, dt):
    """The type's ends at temperatures that bring them near each other again: (x - max) / t is finite though
    x - max is not."""
    big = torch.finfo(dt).max
    x = rand(V, 7, V, dtype=dt) * 1e30
    x[:, 1], x[:, 2], x[:, V - 1] = big, -big, -big / 2
    x[6, 0] = -float("inf")
    t = torch.tensor([1.0, 1.0000001, 1e30, 3e37, 1e38, torch.finfo(F32).max, 1e38], device="cuda")
    want, tol = tree_ref.probs64(x, t)
    got = oq.token_probs(x, t).cpu().double()
    assert ((got - want).abs() <= tol).all() and got[6, 0] == 0
    assert (got[4:6, 2] > 0).all()


def test_probs_at_huge_temperatures():
    """Largest logits of any size below values near the type's lowest: the scale log2(e) / t is below fp32's normal
    numbers."""
    big = torch.finfo(F32).max
    x = torch.tensor([[1.0, -big, -big / 3, 0.0, -big / 7]], device="cuda").repeat(8, 1)
    x[4:6, 0], x[6:, 0] = 1e28, 1e35
    t = torch.tensor([big, 3.1e38, 2.0 ** 127, 2.0 ** 101, big, 2.0 ** 126, big, 2.0 ** 100], device="cuda")
    want, tol = tree_ref.probs64(x, t)
    assert ((oq.token_probs(x, t).cpu().double() - want).abs() <= tol).all()


def test_probs_of_differences_below_fp32s_normal_numbers():
    """Logits and temperatures that are tiny alike."""
    step = 2.0 ** -149
    x = torch.tensor([[0.0, -1.0, 3.0, 2.0, -700.0], [5.0, 5.0, -5.0, 4.0, 0.0], [8e6, 8e6 - 3, 8e6 - 1, 0.0, 8e6 - 2]],
                     dtype=torch.float64)
    x = torch.cat([(x * step).float(), x[:2].float() * 2.0 ** -100, x[:1].float() * 2.0 ** 100]).cuda()
    assert (x[0] != 0).sum() == 4
    t = torch.tensor([2 * step, 7 * step, step, 2.0 ** -100, 2.0 ** -101, step], device="cuda")
    want, tol = tree_ref.probs64(x, t)
    assert ((oq.token_probs(x, t).cpu().double() - want).abs() <= tol).all()


# ------------------------------------------------------------------ what is kept
def split(r, H, Hkv, d):
    return r[:, :H * d], r[:, H * d:(H + Hkv) * d], r[:, (H + Hkv) * d:]


def test_commit_of_rows_behind_the_step():
    """A sequence whose rows leave the step's tensors was not appended, and nothing of it is kept or moved, whatever
    its count; the others' paths are."""
    H, Hkv, d, P, n = 2, 1, 64, 32, 6
    cache = oq.KVCache(6, P, Hkv, d, 3)
    for w, v in ((cache.k_window, 3.0), (cache.v_window, 4.0)):
        w.copy_(v + torch.randn(w.shape, generator=torch.Generator().manual_seed(1)))
    x = rand(1, 2 * n + 3, (H + 2 * Hkv) * d, dtype=BF)      # three rows less than the third tree has
    T = len(x)
    table, length = i32([[0, 1], [2, 3], [4, 5]]), i32([29, 3, 29])
    args = (table, length, i32([0, n, 2 * n, 3 * n]), n)
    q = cache.append_tree(*split(x, H, Hkv, d), *args, i32(chain(n) + star(n) + [-1] * 3))
    assert torch.isnan(q[2 * n:].float()).all() and torch.isfinite(q[:2 * n].float()).all()
    before = [t.clone() for t in (cache.k_window, cache.v_window, cache.k_codes, cache.v_codes, cache.k_scale)]
    path = i32([[0, 1, 2, 3, 4, 5], [0, 4, 9, 9, 9, 9], [0, 2, 3, 4, 5, 9]])
    cache.commit(path, i32([6, 2, 5]), *args, tokens=T)
    now = (cache.k_window, cache.v_window, cache.k_codes, cache.v_codes, cache.k_scale)
    for a, b, of_pages in zip(now, before, (False, False, True, True, True)):
        rest = slice(4, 6) if of_pages else slice(2, 3)
        assert torch.equal(a[rest], b[rest])
    assert cache.k_scale[0, 0] > 0 and not torch.equal(now[0][1], before[0][1])
    k, v = cache.read(table, i32([29, 3, 0]), i32([35, 5, 0]), i32([0, 0, 0, 0]), i32([0, 6, 8, 8]), 8, 6)
    kept = torch.cat([torch.arange(3, 6), torch.tensor([n, n + 4])])
    want_k, want_v = (t[kept.cuda()] for t in split(x, H, Hkv, d)[1:])
    assert torch.equal(k[3:], want_k) and torch.equal(v[3:], want_v)      # (the first three are in a page's codes)


def test_commit_with_a_bound_of_nodes_above_the_page():
    """max_q is a bound: like the step's other calls, commit takes one that passes the page, where the step's rows do
    not."""
    H, Hkv, d, P, n = 2, 1, 64, 32, 5
    x = rand(2, n, (H + 2 * Hkv) * d, dtype=BF)
    got = []
    for max_q in (n, 64):
        c = oq.KVCache(2, P, Hkv, d, 1)
        tree = [-1, 0, 0, 1, 1]
        args, parent = (i32([[0, 1]]), i32([30]), i32([0, n]), max_q), i32(tree)
        q = c.append_tree(*split(x, H, Hkv, d), *args, parent)
        c.attend_tree(q, *args, parent)
        P1 = torch.eye(8, device="cuda")[[2, 3, 1, 1, 5]].contiguous()
        path, count, nxt = oq.tree_verify(i32([0, 2, 4, 6, 3]), parent, i32([0, n]), max_q, P1, torch.zeros(n, device="cuda"),
                                          torch.zeros(1, device="cuda"))
        assert path.shape == (1, max_q) and count.item() == 3 and nxt.item() == 5
        c.commit(path, count, *args, tokens=n)
        got.append((c.k_codes, c.v_codes, c.k_scale, c.k_window[0, 1, :, :d], c.v_window[0, 1]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    with pytest.raises(oq.OQError):
        c.commit(path, count, *args, tokens=33)
    with pytest.raises(oq.OQError):
        c.commit(path, count, *args, tokens=-1)


def test_commits_in_the_profile():
    """A commit counts its rows' bytes, not those of every row that a batch may have."""
    c = oq.KVCache(4, 32, 2, 64, 2)
    oq.profile_enable()
    try:
        for kw in ({}, dict(tokens=7)):
            oq.profile_reset()
            c.commit(i32([[0], [0]]), i32([0, 0]), i32([[0, 1], [2, 3]]), i32([0, 0]), i32([0, 5, 7]), 5, **kw)
            work = sum(w for _, _, w in oq.profile_read().values())
            assert 0 < work <= 8 * 2 * 5 * 2 * 64, kw
    finally:
        oq.profile_enable(False)
        oq.profile_reset()


# ------------------------------------------------------------------ very many rows
def test_probs_of_more_rows_than_a_launch_has_workgroups():
    """2^22 workgroups of 1,024 threads are more than a launch can have."""
    T, V = 2 ** 22 + 5, 3
    x = rand(1, T, V, dtype=BF)
    t = torch.ones(T, device="cuda")
    t[-2:] = torch.tensor([0.0, 2.0])
    got = oq.token_probs(x, t)
    for rows in (slice(0, 70), slice(2 ** 21 - 40, 2 ** 21 + 40), slice(2 ** 22 - 40, T)):
        assert torch.equal(got[rows], oq.token_probs(x[rows].clone(), t[rows].clone()))
    assert ((got.sum(1) - 1).abs() < 1e-6).all()


def test_verify_more_trees_than_a_launch_has_workgroups():
    n, V = 2 ** 22 + 3, 2
    P = torch.eye(V, device="cuda")[torch.arange(n, device="cuda") % V].contiguous()
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    zero = torch.zeros(n, device="cuda")
    path, count, nxt = oq.tree_verify(torch.zeros_like(start[:n]), torch.full_like(start[:n], -1), start, 1, P, zero, zero)
    assert (path == 0).all() and (count == 1).all() and torch.equal(nxt, start[:n] % V)


# ------------------------------------------------------------------ rows side by side
def test_probs_beside_their_logits():
    """Probabilities in the columns behind (or before) the logits: they share rows, but no value."""
    T, V = 70, 129
    wide = torch.full((T, 2 * V + 3), 7.0, device="cuda")
    x = rand(1, T, V)
    want = oq.token_probs(x)
    for a, b in ((0, V), (V + 3, 0), (0, V + 3), (V, 0)):
        wide.fill_(7.0)
        wide[:, a:a + V] = x
        oq.token_probs(wide[:, a:a + V], out=wide[:, b:b + V])
        assert torch.equal(wide[:, b:b + V], want) and torch.equal(wide[:, a:a + V], x) and (wide == 7).sum() == 3 * T
    for b in (V - 1, 1, 0):
        with pytest.raises(oq.OQError, match="overlap"):
            oq.token_probs(wide[:, :V], out=wide[:, b:b + V])


def test_verify_outputs_beside_the_rows():
    """An output in the columns behind P's."""
    n, V, m = 3, 50, 2
    parent, start = i32([-1, 0] * n), i32([0, 2, 4, 6])
    wide = torch.full((2 * n, V + 4), 7.0, device="cuda")
    wide[:, :V] = torch.softmax(rand(1, 2 * n, V), 1)
    token, u, un = i32([0, 3] * n), torch.full((2 * n,), 0.1, device="cuda"), torch.full((n,), 0.5, device="cuda")
    path, count, nxt = oq.tree_verify(token, parent, start, m, wide[:, :V], u, un)
    rest = torch.zeros(3 * n, dtype=torch.int32, device="cuda")
    keep = wide.clone()

    def call(at):                                            # count: three values from column `at` of the first row
        wide.copy_(keep)
        torch.cuda.synchronize()
        r = oq.lib().oq_tree_verify(n, m, 2 * n, start.data_ptr(), parent.data_ptr(), token.data_ptr(), wide.data_ptr(),
                                    V + 4, None, 0, V, 1, u.data_ptr(), un.data_ptr(), rest.data_ptr(), m,
                                    wide.data_ptr() + 4 * at, rest[2 * n:].data_ptr(), None)
        torch.cuda.synchronize()
        return r

    for at in (V, V + 1, V + 4 + V):
        assert call(at) == 0
        assert torch.equal(rest[:2 * n].view(n, m), path) and torch.equal(rest[2 * n:], nxt)
        assert torch.equal(wide.view(-1)[at:at + n].view(torch.int32), count) and torch.equal(wide[:, :V], keep[:, :V])
    for at in (V - 1, V - n, V + 2, 0):
        assert call(at) != 0
